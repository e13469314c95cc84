"""tri_append4 and tri_pack4 at the end of fp32's range: rows whose largest rotated element is 2^128 but for what fp32 does not tell.  From 2^128 on the 32 are no numbers, below it they are (include/tri.h)."""
import numpy as np
import pytest
import torch

import pack4_plain as K
import serve_plain as P
import test_gpu_pack4 as G

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
THETA, TOKENS = 1e6, 400


def rows_at_the_border(dtype, pairs):
    """x [TOKENS][128] float64 of the type's numbers, pos [TOKENS]: one part of one band of each rotated row is 2^128 (1 + d), |d| < 2^-21; what lies around it is large, too."""
    g = np.random.Generator(np.random.Philox(key=[17 + pairs, 5]))
    store = lambda x: torch.from_numpy(x.astype(np.float32)).to(dtype).double().numpy()   # noqa: E731
    found, where = [], []
    for _ in range(40):
        n = 1 << 19
        pos, band, flip = g.integers(1, 1 << 20, n), g.integers(0, 24, n), g.random(n) < 0.5   # (bands that have come far, any angle)
        turn = np.exp(1j * np.remainder(pos * THETA ** (-2.0 * band / 128), 2 * np.pi))
        other = g.uniform(-0.4, 0.4, n)   # (were the other part zero, squares of bf16 numbers would add up to 2^256: none are that near it)
        z = 2.0 ** 128 * (1 + g.uniform(-2.0 ** -21, 2.0 ** -21, n) + 1j * other) * np.where(flip, 1j, 1) / turn
        with np.errstate(over="ignore"):
            re, im = store(z.real), store(z.imag)
        with np.errstate(invalid="ignore"):
            y = (re + 1j * im) * turn
        for i in np.flatnonzero(np.abs(np.where(flip, y.imag, y.real) / 2.0 ** 128 - 1) < 2.0 ** -21)[:TOKENS - len(found)]:
            at = [2 * band[i], 2 * band[i] + 1] if pairs == 0 else [band[i], band[i] + 64]
            rest = store(g.standard_normal(128) * np.exp2(g.integers(100, 124, 128)))
            rest[at] = re[i], im[i]
            found.append(rest)
            where.append(pos[i])
        if len(found) == TOKENS:
            break
    return np.array(found), np.array(where, dtype=np.int32)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
def test_the_largest_is_next_to_what_is_no_number(dtype, pairs):
    from paper_2604_04921_amd import binding as B
    x, pos = rows_at_the_border(dtype, pairs)
    largest = np.abs(P.turn(x, pos.astype(np.int64), THETA, pairs)).max(-1)
    near = np.abs(largest / 2.0 ** 128 - 1)
    assert (near < 2.0 ** -20).all() and min(int((largest >= 2.0 ** 128).sum()), int((largest < 2.0 ** 128).sum())) > TOKENS // 8
    c = K.Case(18, (3,), (TOKENS,), H=2, G=1, dtype=dtype, pairs=pairs, theta=THETA)
    c.pos = pos
    rows = c.put(np.stack([x, -x], axis=1))
    G.check_append(B, c, [3], k_new=rows, v_new=c.put(c.g.standard_normal((c.T, c.H, 128))))
    # the same rows packed from a cache
    i32 = dict(dtype=torch.int32, device="cuda")
    n = torch.tensor([TOKENS], **i32)
    k = rows.transpose(0, 1).contiguous()[None, None]
    places = torch.from_numpy(np.broadcast_to(pos, (1, 1, 2, TOKENS)).copy()).cuda()
    dst = G.empty4(1, 1, 2, TOKENS, 0, c.g)
    want = G.host(dst)
    turned = P.turn(k.double().cpu().numpy(), places.cpu().numpy(), THETA, pairs)
    for h in range(2):
        for j in range(TOKENS):
            G.put(want, (0, 0, h, j), turned[0, 0, h, j], k[0, 0, h, j].double().cpu().numpy(), int(pos[j]))
    four = B.Cache4(dst["k4"], dst["v4"], dst["ks4"], dst["vs4"], dst["pos_gpu"], n, n, TOKENS, rows=dtype)
    B.tri_pack4(B.Model(1, 2, 2, 128, THETA, [1], pairs=pairs), B.Cache(k, k, places, n, n, TOKENS), four, TOKENS)
    torch.cuda.synchronize()
    G.check_fields(dst, want)
