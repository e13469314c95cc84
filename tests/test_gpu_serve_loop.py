"""The example of a serving loop: prefill, compression, decoding behind the compressed prompt, end to end."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_serve_loop():
    spec = importlib.util.spec_from_file_location("serve_loop", os.path.join(ROOT, "examples", "serve_loop.py"))
    loop = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(loop)
    for prompt, budget, samples, tokens in ((1500, 256, 6, 20), (700, 64, 1, 33), (530, 100, 20, 3)):
        r = loop.main(prompt, budget, samples, tokens)
        assert r["kept"] == min(budget, prompt) and r["decoded"] == tokens and r["finite"]
        # Of a row's largest value: half a step of the output, and of the weights, the rotated queries and the rotated keys of a shared prefix behind many rows each one
        # rounding (2^-8) times a score's size (below 8 here: normalised states through projections of unit rows)
        assert r["error"] < (1 + 1 + 8 + 8) * 2.0 ** -8, r
