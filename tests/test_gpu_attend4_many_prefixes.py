"""tri_attend4_shared with a prefix in 4 bits to nearly every sequence, more than 64 rows in the step, against 64 bits (tests/serve_exact.py's tolerances)."""
import numpy as np
import pytest
import torch

import pack4_plain as K
import serve_exact as X

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def case(name, dtype, block, given):
    g = np.random.Generator(np.random.Philox(key=[3, 33]))
    few = lambda n, top: tuple(int(x) for x in g.integers(0, top, n))   # noqa: E731
    kw = dict(dtype=dtype, block=block, given_rotated=given, pairs=int(given))
    if name == "one token each":
        S = 40
        return K.Case(101, few(S, 130), (1,) * S, G=4, H=2, prefix=few(S, 400), groups=tuple(range(S + 1)), **kw)
    if name == "groups of eight heads":
        S = 70
        return K.Case(102, few(S, 20), (1,) * S, G=8, H=1, prefix=few(S - 1, 200) + (1500,), groups=tuple(range(S + 1)), **kw)
    if name == "some tokens each":
        S = 12
        return K.Case(103, few(S, 90), (3, 1, 0, 5, 2, 2, 1, 0, 4, 1, 1, 9), G=4, H=2, prefix=few(S, 300), groups=tuple(range(S + 1)), **kw)
    # a large group beside small ones, groups without a sequence, prefixes without a key
    return K.Case(104, few(30, 60), (1,) * 28 + (2, 3), G=5, H=2, prefix=(700, 0, 40, 5, 300, 0, 64), groups=(0, 1, 2, 2, 25, 26, 28, 30), **kw)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("block, given", [(0, False), (4, True), (16, False), (64, True)])
@pytest.mark.parametrize("name", ["one token each", "groups of eight heads", "some tokens each", "uneven"])
def test_many_prefixes(name, dtype, block, given):
    from paper_2604_04921_amd import binding as B
    c = case(name, dtype, block, given)
    assert c.T * c.G > 64
    call = X.Call(c, shared=True)
    ref, var = call.value()
    got = K.attend(B, c)
    torch.cuda.synchronize()
    assert X.wrong(call, got.double().cpu().numpy(), ref, var) == []
    for m in ("prefix", "own"):   # (what leaves one of the two out is told from it)
        assert X.wrong(call, call.value(mutant=m)[0], ref, var)
    assert torch.equal(K.attend(B, c), got)
