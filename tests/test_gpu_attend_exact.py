"""tri_attend and tri_attend_shared against 64 bits, no further off than the roundings that include/tri.h states (tests/serve_exact.py; tests/test_attend_tolerances.py says what these tolerances tell apart)."""
import pytest
import torch

import serve_exact as X
from test_gpu_attend import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("spec", X.specs(), ids=lambda s: s["name"])
def test_no_more_roundings_than_stated(spec):
    from paper_2604_04921_amd import binding as B
    call = X.make(spec, "cuda")
    c = call.c
    tokens = None
    if call.head_len is not None:
        whole = torch.zeros((c.layers, c.S, c.H), dtype=torch.int32, device="cuda")
        whole[c.layer] = torch.from_numpy(call.head_len).cuda()
        tokens = c.step(B, head_len=whole)
    out = run(B, c, causal=call.causal, scale=call.scale, shared=call.shared, tokens=tokens)
    torch.cuda.synchronize()
    assert X.wrong(call, out.double().cpu().numpy(), *call.value()) == []
