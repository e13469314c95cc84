"""tri_append against 64 bits and bit for bit where it copies: what is written, where, and that nothing else is."""
import numpy as np
import pytest
import torch

import serve_plain as P

pytestmark = pytest.mark.gpu


def bits(t):
    return t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32).cpu().numpy()


def append(B, c, lens, tokens, k_new, v_new, head_len=None, step=None, new_len=True, n=None, stream=None):
    own = dict(c.own, lens_gpu=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cache = c.descriptor(B, own)
    if n is not None:
        cache.c.max_seq_len = n
    got = torch.full((c.S,), -1, dtype=torch.int32, device="cuda") if new_len else None
    B.tri_append(c.model(B), cache, c.layer, step or c.step(B, head_len=head_len), k_new, v_new, got, stream=stream)
    torch.cuda.synchronize()
    return None if got is None else got.tolist()


def expected(c, lens, k_new, v_new, k, v, pos, tol, cap=None, table=None, head_len=None):
    """The cache in place: k (float64), v, pos as arrays of the GPU's layout; tol is where a rotated element may be off."""
    turned = c.stored_rotated and not c.given_rotated
    kn = k_new.double().cpu().numpy()
    if turned:
        size = np.abs(P.bands(kn, c.pairs))
        size = P.rows(size + 1j * size, c.pairs)   # of the band, for the products' own error
        kn = P.turn(kn, np.broadcast_to(c.pos[:, None], kn.shape[:2]), c.theta, c.pairs)
    for s in range(c.S):
        for i in range(c.tokens[s]):
            t = c.start[s] + i
            for h in range(c.H):
                n = (lens[s] if head_len is None else int(head_len[s][h])) + i
                if n >= (c.own["cap"] if cap is None else cap):
                    continue
                where = (c.layer, s, h, n)
                if c.block:
                    b = int((c.own["table"] if table is None else table)[s, n // c.block])
                    if b < 0 or b >= k.shape[1]:
                        continue
                    where = (c.layer, b, h, n % c.block)
                k[where] = kn[t, h]
                if turned:
                    u = P.HALF[c.dtype]
                    angle = 2.0 ** -18 if c.dtype == torch.bfloat16 else 4 * 2.0 ** -24
                    tol[where] = u * np.abs(kn[t, h]) * 1.01 + size[t, h] * angle + 1e-30
                v[where] = v_new[t, h].double().cpu().numpy()
                pos[where] = c.pos[t]


def check(B, c, lens, cap=None, table=None, head_len=None, k_new=None, v_new=None, **kw):
    own = c.own
    for f in ("k_gpu", "v_gpu"):
        own[f].nan_to_num_(nan=3.0, posinf=4.0)
    k, v, pos = (own[f].double().cpu().numpy() if f != "pos_gpu" else own[f].cpu().numpy() for f in ("k_gpu", "v_gpu", "pos_gpu"))
    tol = np.zeros_like(k)
    if k_new is None:
        k_new = c.put(c.g.standard_normal((c.T, c.H, 128)))
        v_new = c.put(c.g.standard_normal((c.T, c.H, 128)))
    expected(c, lens, k_new, v_new, k, v, pos, tol, cap, table, head_len)
    heads = None
    if head_len is not None:
        heads = torch.zeros((c.layers, c.S, c.H), dtype=torch.int32, device="cuda")
        heads[c.layer] = torch.from_numpy(head_len).cuda()
    got = append(B, c, lens, None, k_new, v_new, head_len=heads, n=cap, **kw)
    assert np.array_equal(own["pos_gpu"].cpu().numpy(), pos)
    assert np.array_equal(own["v_gpu"].double().cpu().numpy(), v)
    off = np.abs(own["k_gpu"].double().cpu().numpy() - k)
    worst = np.unravel_index(np.argmax(off - tol), off.shape)
    assert np.all(off <= tol), (worst, off[worst], tol[worst])
    top = c.own["cap"] if cap is None else cap
    if got is not None:
        before = lens if head_len is None else [int(x) for x in head_len[:, 0]]
        assert got == [min(n + t, top) for n, t in zip(before, c.tokens)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
@pytest.mark.parametrize("stored,given", [(True, False), (True, True), (False, False)], ids=["turned", "both_post", "both_pre"])
@pytest.mark.parametrize("block", [0, 1, 4, 16, 64])
def test_layouts(dtype, pairs, stored, given, block):
    from paper_2604_04921_amd import binding as B
    for seed, (lens, tokens, H) in enumerate([((5,), (1,), 1), ((0, 31, 100), (3, 1, 70), 3), ((9, 0, 0, 16), (0, 0, 200, 0), 8), ((1,) * 70, (1,) * 70, 2)]):
        c = P.Case(seed, lens, tokens, H=H, G=1, dtype=dtype, pairs=pairs, stored_rotated=stored, given_rotated=given, block=block)
        check(B, c, list(lens))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pos0", [2 ** 31 - 600, -2 ** 31, -3, 2 ** 24 + 1])
def test_far_positions(dtype, pos0):
    from paper_2604_04921_amd import binding as B
    c = P.Case(5, (100, 7), (300, 1), dtype=dtype, pos0=pos0, theta=1e4)
    check(B, c, [100, 7])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_full_caches_and_blocks_that_are_not_there(dtype):
    """Tokens beyond max_seq_len, or in a block whose id is out of the pool, are not written; lengths are read into their range."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(6, (40, 10, 0), (30, 20, 9), dtype=dtype, block=16)
    check(B, c, [40, 10, 0], cap=57)
    c = P.Case(7, (40, 10, 0), (30, 20, 9), dtype=dtype, block=16)
    pool = c.own["k_gpu"].shape[1]
    table = c.own["table"].copy()
    table[0, 3], table[1, 1], table[2, 0] = -1, pool, 2 ** 31 - 1
    c.own["table_gpu"].copy_(torch.from_numpy(table))
    check(B, c, [40, 10, 0], table=table)
    c = P.Case(8, (40, 10), (3, 2), dtype=dtype)
    k_new = c.put(c.g.standard_normal((c.T, c.H, 128)))
    before = c.own["k_gpu"].clone()
    assert append(B, c, [10 ** 9, 2 ** 31 - 1], None, k_new, k_new) == [c.own["cap"]] * 2   # read as max_seq_len: full
    assert np.array_equal(bits(before), bits(c.own["k_gpu"]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_lengths_per_head(dtype):
    from paper_2604_04921_amd import binding as B
    c = P.Case(9, (60, 30), (5, 1), H=3, dtype=dtype, block=4)
    check(B, c, [60, 30], head_len=np.array([[60, 0, 17], [2, 30, 1]], dtype=np.int32))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_rows_of_a_fused_projection_on_another_stream(dtype):
    """k and v as views of one output, heads before tokens; one token per sequence without start, at cur_pos."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(10, (60, 30, 2), (1, 1, 1), H=2, dtype=dtype)
    wide = c.put(c.g.standard_normal((9, c.T, 128)))
    k_new, v_new = wide[4:6].transpose(0, 1), wide[6:8].transpose(0, 1)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    step = c.step(B, plain=True)
    check(B, c, [60, 30, 2], k_new=k_new, v_new=v_new, step=step, stream=side)


@pytest.mark.parametrize("block", [0, 64])
def test_offsets_beyond_32_bits(block):
    """Heads (contiguous) and blocks (paged) that lie more than 2^32 bytes behind the first."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(12, (70,), (30,), H=2, layers=1, layer=0, block=block)
    own = c.own
    if block:
        far, farv = (torch.zeros((1, 140000, 2, block, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))   # 4.6 GB each
        farp = torch.zeros((1, 140000, 2, block), dtype=torch.int32, device="cuda")
        n = own["k_gpu"].shape[1]
        own["table_gpu"] += 140000 - n
    else:
        n, rows = own["cap"], (1 << 31) // 128 + 500
        far, farv = (torch.zeros((1, 1, 2, rows, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        farp = torch.zeros((1, 1, 2, rows), dtype=torch.int32, device="cuda")
    k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    near = {f: own[f].nan_to_num_(nan=3.0, posinf=4.0).clone() if f != "pos_gpu" else own[f].clone() for f in ("k_gpu", "v_gpu", "pos_gpu")}
    part = (slice(None), slice(-n, None)) if block else (slice(None), slice(None), slice(None), slice(0, n))
    far[part], farv[part], farp[part] = near["k_gpu"], near["v_gpu"], near["pos_gpu"]
    own.update(k_gpu=far, v_gpu=farv, pos_gpu=farp)
    append(B, c, [70], None, k_new, v_new)
    # the same call on the near cache
    if block:
        own["table_gpu"] -= 140000 - n
    own.update(near)
    append(B, c, [70], None, k_new, v_new)
    for got, want in ((far, near["k_gpu"]), (farv, near["v_gpu"]), (farp, near["pos_gpu"])):
        assert torch.equal(got[part], want)
    assert int(torch.count_nonzero(farp)) == int(torch.count_nonzero(near["pos_gpu"]))   # and nowhere else


def test_graph_of_a_step():
    """An append and the attention over what it wrote, behind a shared prefix, captured once and replayed with other rows, eager work in between."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(13, (40, 7, 0), (1, 1, 1), block=16, prefix=(300,), layers=1, layer=0)
    own = c.own
    lens = torch.tensor([40, 7, 0], dtype=torch.int32, device="cuda")
    after = torch.zeros_like(lens)
    model, tokens = c.model(B), c.step(B)
    before, behind, prefix = c.descriptor(B, own, lens), c.descriptor(B, own, after), c.descriptor(B, c.prefix)
    k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    out = torch.zeros_like(c.q_gpu)
    ws = torch.empty(B.tri_attend_workspace_size(model, behind, tokens, prefix), dtype=torch.uint8, device="cuda")

    def step(to):
        B.tri_append(model, before, 0, tokens, k_new, v_new, after)
        B.tri_attend_shared(model, prefix, None, behind, 0, tokens, c.q_gpu, to, workspace=ws)
    step(out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for i in range(4):
        k_new.mul_(-1.0 if i % 2 else 0.5)
        v_new.add_(1.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = torch.zeros_like(out)
        after.fill_(-1)
        step(want)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and after.tolist() == [41, 8, 1]
        ws.fill_(0xff)


def test_then_attended():
    """A prompt and single tokens appended call by call give the attention of the cache they make."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(11, (0, 0), (60, 33), block=16, layers=1, layer=0, stored_rotated=False)
    rows_k = torch.cat([c.put(c.own["k"][s, :, :n].swapaxes(0, 1)) for s, n in enumerate(c.tokens)])
    rows_v = torch.cat([c.put(c.own["v"][s, :, :n].swapaxes(0, 1)) for s, n in enumerate(c.tokens)])
    c.own["k_gpu"].fill_(float("nan"))
    c.own["v_gpu"].fill_(float("nan"))
    c.own["pos_gpu"].fill_(-1)
    model = c.model(B)
    length = [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2)]
    at = [0, 0]
    pos = torch.from_numpy(c.pos).cuda()
    for many in ((40, 30), (1, 1), (19, 2)):
        ids = torch.cat([torch.arange(c.start[s] + at[s], c.start[s] + at[s] + many[s]) for s in range(2)]).cuda()
        start = torch.tensor([0, many[0], sum(many)], dtype=torch.int32, device="cuda")
        tokens = B.Tokens(pos[ids].contiguous(), start=start, max_tokens=max(many))
        B.tri_append(model, c.descriptor(B, c.own, length[0]), 0, tokens, rows_k[ids], rows_v[ids], length[1])
        length.reverse()
        at = [a + m for a, m in zip(at, many)]
    out = torch.empty_like(c.q_gpu)
    tokens, cache = c.step(B), c.descriptor(B, c.own, length[0])
    ws = torch.empty(max(256, B.tri_attend_workspace_size(model, cache, tokens)), dtype=torch.uint8, device="cuda")
    B.tri_attend(model, cache, 0, tokens, c.q_gpu, out, workspace=ws)
    torch.cuda.synchronize()
    assert length[0].tolist() == [60, 33]
    ref, tol = c.want(roundings=2)
    assert np.all(np.abs(out.double().cpu().numpy() - ref) <= tol)
