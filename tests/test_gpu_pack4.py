"""tri_append4, tri_pack4 and tri_unpack4, bit for bit: the 4-bit numbers are those of the exactly rotated elements, what is written where, and that nothing else is."""
import numpy as np
import pytest
import torch

import pack4_plain as K
import serve_plain as P

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FIELDS = ("k4", "v4", "ks4", "vs4", "pos_gpu")


def host(cache):
    return {f: cache[f].cpu().numpy().copy() for f in FIELDS}


def check_fields(got, want):
    for f in FIELDS:
        a = got[f].cpu().numpy()
        assert K.same_codes(a, want[f]) if f in ("k4", "v4") else np.array_equal(a, want[f]), f


def put(want, where, k, v, pos):
    for f, x in (("k", k), ("v", v)):
        want[f + "4"][where], want[f + "s4"][where] = K.encode(x)
    want["pos_gpu"][where] = pos


def turned(c, x, pos):
    return P.turn(x, pos, c.theta, c.pairs) if not c.given_rotated else x


def check_append(B, c, lens, cap=None, table=None, head_len=None, k_new=None, v_new=None, step=None, stream=None, cur=None):
    own = c.own
    if k_new is None:
        k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    want = host(own)
    kn = turned(c, k_new.double().cpu().numpy(), np.broadcast_to(c.pos[:, None], (c.T, c.H)))
    vn = v_new.double().cpu().numpy()
    for s in range(c.S):
        for i in range(c.tokens[s]):
            t = c.start[s] + i
            for h in range(c.H):
                n = (lens[s] if head_len is None else int(head_len[s][h])) + i
                if n >= (own["cap"] if cap is None else cap):
                    continue
                where = (c.layer, s, h, n)
                if c.block:
                    b = int((own["table"] if table is None else table)[s, n // c.block])
                    if b < 0 or b >= own["pos_gpu"].shape[1]:
                        continue
                    where = (c.layer, b, h, n % c.block)
                put(want, where, kn[t, h], vn[t, h], c.pos[t])
    heads = None
    if head_len is not None:
        heads = torch.zeros((c.layers, c.S, c.H), dtype=torch.int32, device="cuda")
        heads[c.layer] = torch.from_numpy(head_len).cuda()
    cache = K.descriptor(B, c, own, torch.tensor(lens, dtype=torch.int32, device="cuda"), cur)
    if cap is not None:
        cache.c.c.max_seq_len = cap
    got = torch.full((c.S,), -1, dtype=torch.int32, device="cuda")
    B.tri_append4(c.model(B), cache, c.layer, step or c.step(B, head_len=heads), k_new, v_new, got, stream=stream)
    torch.cuda.synchronize()
    check_fields(own, want)
    top = own["cap"] if cap is None else cap
    before = lens if head_len is None else [int(x) for x in head_len[:, 0]]
    assert got.tolist() == [min(max(n, 0) + t, top) for n, t in zip(before, c.tokens)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
@pytest.mark.parametrize("given", [False, True], ids=["turned", "as_they_are"])
@pytest.mark.parametrize("block", [0, 1, 4, 16, 64])
def test_append_layouts(dtype, pairs, given, block):
    from paper_2604_04921_amd import binding as B
    for seed, (lens, tokens, H) in enumerate([((5,), (1,), 1), ((0, 31, 100), (3, 1, 70), 3), ((9, 0, 0, 16), (0, 0, 200, 0), 8), ((1,) * 70, (1,) * 70, 2)]):
        c = K.Case(seed, lens, tokens, H=H, G=1, dtype=dtype, pairs=pairs, given_rotated=given, block=block)
        check_append(B, c, list(lens))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pos0", [2 ** 31 - 600, -2 ** 31, -3, 2 ** 24 + 1])
def test_append_far_positions(dtype, pos0):
    from paper_2604_04921_amd import binding as B
    c = K.Case(5, (100, 7), (300, 1), dtype=dtype, pos0=pos0, theta=1e4)
    check_append(B, c, [100, 7])


@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
def test_elements_and_scales_next_to_a_border(pairs):
    """Rows made so that after the rotation elements lie on a border between two numbers, and a group's largest on the border between two scales, but for what fp32 does not tell: 64 bits say which side."""
    from paper_2604_04921_amd import binding as B
    for dtype in (F32, BF16):
        c = K.Case(15, (0,), (400,), H=2, G=1, dtype=dtype, pairs=pairs, theta=1e6)
        g = c.g
        at = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])[g.integers(0, 7, (c.T, c.H, 128))] * np.where(g.random((c.T, c.H, 128)) < 0.5, -1, 1)
        at[..., ::32] = 7.0 * np.where(g.random(at[..., ::32].shape) < 0.5, -1, 1)   # the scales' border
        back = P.turn(at, -np.broadcast_to(c.pos[:, None].astype(np.int64), (c.T, c.H)), c.theta, c.pairs)
        k_new = c.put(back)
        # (rounded to the rows' type the rotated elements lie around the borders within some 2^-24 or 2^-8 of them; most in fp32 are among those that fp32 products leave open)
        if dtype == F32:
            far = np.abs(P.turn(k_new.double().cpu().numpy(), np.broadcast_to(c.pos[:, None], (c.T, c.H)), c.theta, c.pairs) - at)
            assert np.median(far) < 2.0 ** -22
        check_append(B, c, [0], k_new=k_new, v_new=c.put(at))


@pytest.mark.parametrize("given", [False, True], ids=["turned", "as_they_are"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_magnitudes_and_not_numbers(dtype, given):
    """From below the least scale to the largest numbers there are, zeros, NaN and infinities."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(16, (3,), (300,), H=2, G=1, dtype=dtype, given_rotated=given, pairs=1)
    x = c.g.standard_normal((2, c.T, c.H, 128))
    x *= np.exp2(c.g.integers(-120, 124, (2, c.T, c.H, 1)).astype(np.float64))
    x[:, 0:20] = np.sign(x[:, 0:20]) * 2.0 ** -133 * np.arange(1, 129)                      # subnormal in both types
    x[:, 20:30] = np.sign(x[:, 20:30]) * 2.0 ** -126 * (1 + np.arange(128) % 7)
    x[:, 30:40] = np.sign(x[:, 30:40]) * (2.0 ** 127 * np.linspace(0.1, 0.7, 128))   # (rotated: below 2^128)
    x[:, 40:45] = 0
    x[1, 45:50] = 2.0 ** 127 * np.linspace(0.5, 1.99, 128)                                   # values are not rotated: the cap's errors
    x[0, 50, 0, 5], x[0, 51, 1, 70], x[0, 52, 0, 127], x[1, 53, 0, 1], x[1, 54, 1, 99] = np.nan, np.inf, -np.inf, np.nan, -np.inf
    with np.errstate(invalid="ignore"):
        check_append(B, c, [3], k_new=c.put(x[0]), v_new=c.put(x[1]))
    assert int((c.own["ks4"] == 255).sum()) >= 3 and int((c.own["vs4"][c.layer, 0, :, 53:60] == 255).sum()) == 2


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_full_caches_and_blocks_that_are_not_there(dtype):
    from paper_2604_04921_amd import binding as B
    c = K.Case(6, (40, 10, 0), (30, 20, 9), dtype=dtype, block=16)
    check_append(B, c, [40, 10, 0], cap=57)
    c = K.Case(7, (40, 10, 0), (30, 20, 9), dtype=dtype, block=16)
    table = c.own["table"].copy()
    table[0, 3], table[1, 1], table[2, 0] = -1, c.own["pos_gpu"].shape[1], 2 ** 31 - 1
    c.own["table_gpu"].copy_(torch.from_numpy(table))
    check_append(B, c, [40, 10, 0], table=table)
    c = K.Case(8, (40, 10), (3, 2), dtype=dtype)
    check_append(B, c, [10 ** 9, 2 ** 31 - 1])   # read as max_seq_len: full


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_lengths_per_head(dtype):
    from paper_2604_04921_amd import binding as B
    c = K.Case(9, (60, 30), (5, 1), H=3, dtype=dtype, block=4)
    check_append(B, c, [60, 30], head_len=np.array([[60, 0, 17], [2, 30, 1]], dtype=np.int32))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_append_rows_of_a_fused_projection_on_another_stream(dtype):
    """k and v as views of one output, heads before tokens; one token per sequence without start, at cur_pos."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(10, (60, 30, 2), (1, 1, 1), H=2, dtype=dtype)
    wide = c.put(c.g.standard_normal((9, c.T, 128)))
    step = c.step(B, plain=True)
    step.c.pos = None
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    check_append(B, c, [60, 30, 2], k_new=wide[4:6].transpose(0, 1), v_new=wide[6:8].transpose(0, 1), step=step, stream=side, cur=torch.from_numpy(c.pos).cuda())


def empty4(L, S, H, cap, block, g, spare=3):
    """An empty cache of 4 bits as a dict, filled with a pattern."""
    table, blocks = None, S
    if block:
        cap = -(-cap // block) * block
        mb = cap // block
        blocks = S * mb + spare
        table = g.permutation(blocks)[:S * mb].reshape(S, mb).astype(np.int32)
    lead = (L, blocks, H, block) if block else (L, S, H, cap)
    new = lambda *w: torch.full(lead + w, 0x5a, dtype=torch.uint8, device="cuda")   # noqa: E731
    return dict(k4=new(64), v4=new(64), ks4=new(4), vs4=new(4), pos_gpu=torch.full(lead, -5, dtype=torch.int32, device="cuda"), cap=cap, table=table,
                table_gpu=None if table is None else torch.from_numpy(table).cuda(), lens_gpu=torch.zeros(S, dtype=torch.int32, device="cuda"))


def at(table, block, l, s, h, n):
    return (l, s, h, n) if not block else (l, int(table[s, n // block]), h, n % block)


def full_cache(g, dtype, L, S, H, cap, block):
    e = empty4(L, S, H, cap, block, g)
    lead = tuple(e["pos_gpu"].shape)
    x = dict(k=torch.from_numpy(g.standard_normal(lead + (128,))).to(dtype).cuda(), v=torch.from_numpy(g.standard_normal(lead + (128,))).to(dtype).cuda(),
             pos=torch.from_numpy(g.integers(0, 200000, lead).astype(np.int32)).cuda())
    return dict(e, **x)


def kept(g, L, S, H, lens, budget):
    idx, cnt = np.full((L, S, H, budget), -1, dtype=np.int32), np.zeros((L, S, H), dtype=np.int32)
    for l in range(L):
        for s in range(S):
            for h in range(H):
                cnt[l, s, h] = n = min(lens[s], budget) if h % 2 == 0 else g.integers(0, min(lens[s], budget) + 1)
                idx[l, s, h, :n] = np.sort(g.choice(lens[s], size=n, replace=False))
    return idx, cnt


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairs,rotated", [(0, False), (1, False), (0, True)], ids=["interleaved", "half", "as_they_are"])
@pytest.mark.parametrize("block,block4", [(0, 0), (16, 4), (0, 64), (1, 0)])
def test_pack_and_read_back(dtype, pairs, rotated, block, block4):
    from paper_2604_04921_amd import binding as B
    for seed, (L, lens, H, budget, pick) in enumerate([(1, (1,), 1, 1, True), (2, (37, 100, 0), 3, 40, True), (3, (70, 5), 2, 64, False), (1, (200, 31), 2, 500, False), (2, (33, 64), 2, 33, "counts")]):
        g = np.random.Generator(np.random.Philox(key=[seed, 90]))
        S, cap = len(lens), max(lens) + 2
        src, dst = full_cache(g, dtype, L, S, H, cap, block), empty4(L, S, H, min(budget, cap), block4, g)
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        model = B.Model(L, H, H, 128, 1e6, [1], pairs=pairs)
        full = B.Cache(src["k"], src["v"], src["pos_gpu"], n, n, cap, block_table=src["table_gpu"], k_rotated=rotated)
        src["pos_gpu"].copy_(src["pos"])
        idx, cnt = kept(g, L, S, H, lens, budget)
        use_idx, use_cnt = pick is True, bool(pick)
        if not use_idx:
            cnt = cnt if use_cnt else np.broadcast_to(np.minimum(lens, budget)[None, :, None], (L, S, H)).astype(np.int32, order="C")
            idx = np.broadcast_to(np.arange(budget, dtype=np.int32), (L, S, H, budget))
        want = host(dst)
        k, v, pos = src["k"].double().cpu().numpy(), src["v"].double().cpu().numpy(), src["pos"].cpu().numpy()
        for l in range(L):
            for s in range(S):
                for h in range(H):
                    for j in range(cnt[l, s, h]):
                        f = at(src["table"], block, l, s, h, idx[l, s, h, j])
                        kk = k[f] if rotated else P.turn(k[f], pos[f], 1e6, pairs)
                        put(want, at(dst["table"], block4, l, s, h, j), kk, v[f], pos[f])
        new_len = torch.full((S,), -1, dtype=torch.int32, device="cuda")
        four = B.Cache4(dst["k4"], dst["v4"], dst["ks4"], dst["vs4"], dst["pos_gpu"], new_len, new_len, dst["cap"], block_table=dst["table_gpu"], rows=dtype)
        B.tri_pack4(model, full, four, budget, torch.from_numpy(np.ascontiguousarray(idx)).cuda() if use_idx else None, torch.from_numpy(cnt).cuda() if use_cnt else None, new_len)
        torch.cuda.synchronize()
        check_fields(dst, want)
        assert new_len.tolist() == cnt[0, :, 0].tolist()
        # read back: what it stands for, in either type, nothing beyond it; and packed again it is what it was
        counts = torch.from_numpy(cnt).cuda()
        for other, oblock in ((BF16, block), (F32, 8)):
            back = full_cache(g, other, L, S, H, cap, oblock)
            bw = {f: back[f].double().cpu().numpy() for f in ("k", "v")}
            bp = back["pos"].cpu().numpy().copy()
            for l in range(L):
                for s in range(S):
                    for h in range(H):
                        for j in range(cnt[l, s, h]):
                            f, t = at(dst["table"], block4, l, s, h, j), at(back["table"], oblock, l, s, h, j)
                            bw["k"][t], bw["v"][t] = K.decode(want["k4"][f], want["ks4"][f]), K.decode(want["v4"][f], want["vs4"][f])
                            bp[t] = want["pos_gpu"][f]
            target = B.Cache(back["k"], back["v"], back["pos"], n, n, cap, block_table=back["table_gpu"], k_rotated=True)
            again_len = torch.full((S,), -1, dtype=torch.int32, device="cuda")
            B.tri_unpack4(model, four, target, min(budget, cap), None, counts, again_len)
            torch.cuda.synchronize()
            for f in ("k", "v"):
                assert np.array_equal(back[f].double().cpu().numpy(), bw[f])
            assert np.array_equal(back["pos"].cpu().numpy(), bp) and again_len.tolist() == cnt[0, :, 0].tolist()
            third = {f: torch.full_like(dst[f], 0x5a if f != "pos_gpu" else -5) for f in FIELDS}
            four2 = B.Cache4(third["k4"], third["v4"], third["ks4"], third["vs4"], third["pos_gpu"], new_len, new_len, dst["cap"], block_table=dst["table_gpu"], rows=dtype)
            B.tri_pack4(model, target, four2, dst["cap"], None, counts)
            torch.cuda.synchronize()
            check_fields(third, want)


def test_read_back_chosen_slots_lengths_and_blocks_that_are_not_there():
    """Slots in any order and twice, indices and counts out of range, blocks that there are not on either side."""
    from paper_2604_04921_amd import binding as B
    g = np.random.Generator(np.random.Philox(key=[7, 91]))
    L, S, H, lens, budget, block = 2, 2, 2, (90, 60), 50, 16
    src = full_cache(g, BF16, L, S, H, 96, 0)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    model = B.Model(L, H, H, 128, 1e6, [1])
    src["pos_gpu"].copy_(src["pos"])
    full = B.Cache(src["k"], src["v"], src["pos_gpu"], n, n, 96, k_rotated=True)
    dst = empty4(L, S, H, 96, block, g)
    pool = dst["pos_gpu"].shape[1]
    table = dst["table"].copy()
    table[0, 1], table[1, 2] = -1, pool
    dst["table_gpu"].copy_(torch.from_numpy(table))
    want = host(dst)
    for l in range(L):
        for s in range(S):
            for h in range(H):
                for j in range(lens[s]):
                    if 0 <= table[s, j // block] < pool:
                        put(want, at(table, block, l, s, h, j), src["k"][l, s, h, j].double().cpu().numpy(), src["v"][l, s, h, j].double().cpu().numpy(), int(src["pos"][l, s, h, j]))
    four = B.Cache4(dst["k4"], dst["v4"], dst["ks4"], dst["vs4"], dst["pos_gpu"], n, n, 96, block_table=dst["table_gpu"])
    B.tri_pack4(model, full, four, 96)
    torch.cuda.synchronize()
    check_fields(dst, want)
    idx = g.integers(-5, 120, (L, S, H, budget)).astype(np.int32)
    idx[0, 0, 0, :4] = [2, 2, -2 ** 31, 2 ** 31 - 1]
    cnt = np.array([[[50, 3], [0, 70]], [[-4, 20], [2 ** 31 - 1, 1]]], dtype=np.int32)
    back = full_cache(g, BF16, L, S, H, 64, 0)
    bk, bv, bp = (back[f].double().cpu().numpy() for f in ("k", "v", "pos"))
    for l in range(L):
        for s in range(S):
            for h in range(H):
                for j in range(min(max(cnt[l, s, h], 0), budget)):
                    i = min(max(int(idx[l, s, h, j]), 0), 95)
                    if 0 <= table[s, i // block] < pool:
                        f = at(table, block, l, s, h, i)
                        bk[l, s, h, j], bv[l, s, h, j], bp[l, s, h, j] = K.decode(want["k4"][f], want["ks4"][f]), K.decode(want["v4"][f], want["vs4"][f]), want["pos_gpu"][f]
    target = B.Cache(back["k"], back["v"], back["pos"], n, n, 64, k_rotated=True)
    B.tri_unpack4(model, four, target, budget, torch.from_numpy(idx).cuda(), torch.from_numpy(cnt).cuda())
    torch.cuda.synchronize()
    for f, w in (("k", bk), ("v", bv), ("pos", bp)):
        assert np.array_equal(back[f].double().cpu().numpy(), w, equal_nan=True), f


@pytest.mark.parametrize("block", [0, 64])
def test_offsets_beyond_32_bits(block):
    """Heads (contiguous) and blocks (paged) that lie more than 2^32 bytes behind the first."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(12, (70,), (30,), H=2, layers=1, layer=0, block=block)
    own = c.own
    if block:
        blocks, part, n = 540000, None, own["k4"].shape[1]
        lead, part = (1, blocks, 2, block), (slice(None), slice(-n, None))
    else:
        n = own["cap"]
        lead, part = (1, 1, 2, (1 << 32) // 64 + 500), (slice(None), slice(None), slice(None), slice(0, n))
    far = {f: torch.zeros(lead + w, dtype=own[f].dtype, device="cuda") for f, w in (("k4", (64,)), ("v4", (64,)), ("ks4", (4,)), ("vs4", (4,)), ("pos_gpu", ()))}
    k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    lens = torch.tensor([70], dtype=torch.int32, device="cuda")
    near = {f: own[f].clone() for f in FIELDS}
    for f in FIELDS:
        far[f][part] = near[f]
    shift = blocks - n if block else 0
    if block:
        own["table_gpu"] += shift
    B.tri_append4(c.model(B), K.descriptor(B, c, dict(own, **far), lens), 0, c.step(B), k_new, v_new)
    if block:
        own["table_gpu"] -= shift
    B.tri_append4(c.model(B), K.descriptor(B, c, dict(own, **near), lens), 0, c.step(B), k_new, v_new)
    torch.cuda.synchronize()
    for f in FIELDS:
        assert torch.equal(far[f][part], near[f]), f
    assert int(torch.count_nonzero(far["pos_gpu"])) == int(torch.count_nonzero(near["pos_gpu"]))   # and nowhere else
    # read from there
    backs = []
    for x, by in ((far, shift), (near, 0)):
        if block:
            own["table_gpu"] += by
        back = [torch.zeros((1, 1, 2, 112, 128), dtype=BF16, device="cuda") for _ in range(2)] + [torch.zeros((1, 1, 2, 112), dtype=torch.int32, device="cuda")]
        full = torch.tensor([100], dtype=torch.int32, device="cuda")
        B.tri_unpack4(c.model(B), K.descriptor(B, c, dict(own, **x), full), B.Cache(*back, full, full, 112, k_rotated=True), 112)
        torch.cuda.synchronize()
        if block:
            own["table_gpu"] -= by
        backs.append(back)
    assert all(torch.equal(a, b) for a, b in zip(*backs)) and int(torch.count_nonzero(backs[0][0])) > 10000
