"""The tolerances of tests/serve_exact.py, held against kernels that are right and kernels that are wrong, in 64 bits on the host: what makes the roundings that are stated passes, and what leaves something out or rounds
more does not."""
import numpy as np
import pytest
import torch

import serve_exact as X
import serve_plain as P


@pytest.mark.parametrize("spec", X.specs(), ids=lambda s: s["name"])
def test_right_and_wrong_kernels(spec):
    call = X.make(spec, "cpu")
    ref, var = call.value()
    to_type = X.to_bf16 if call.c.dtype == torch.bfloat16 else lambda x: x.astype(np.float32).astype(np.float64)
    assert X.wrong(call, to_type(call.value(held=True)[0]), ref, var) == []
    for m in spec["mutants"]:
        assert not X.applies(call, m) or X.wrong(call, to_type(call.value(mutant=m)[0]), ref, var), "nothing says that %r is wrong" % m


def test_every_mutant_is_told_somewhere():
    assert {m for s in X.specs() for m in s["mutants"]} == set(X.MUTANTS)


def test_the_value_is_the_other_reference_s():
    """Two ways to the same value: serve_plain's loop and this one."""
    c = P.Case(1, (40, 7), (3, 20), device="cpu", stored_rotated=False, prefix=(30,), groups=(0, 2))
    ref, _ = c.want(scale=0.2)
    mine, _ = X.Call(c, scale=0.2, shared=True).value()
    assert np.abs(ref - mine).max() < 1e-12
