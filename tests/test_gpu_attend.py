"""tri_attend and tri_attend_shared against 64 bits: types, layouts, lengths, masks, pages, strides, what must not be read."""
import numpy as np
import pytest
import torch

import serve_plain as P

pytestmark = pytest.mark.gpu


def run(B, c, causal=True, scale=None, shared=False, tokens=None, own=None, out=None, q=None, stream=None):
    model, own, tokens = c.model(B), own or c.descriptor(B, c.own), tokens or c.step(B)
    prefix = c.descriptor(B, c.prefix) if shared else None
    ws = torch.full((max(B.tri_attend_workspace_size(model, own, tokens, prefix), 256),), 0xff, dtype=torch.uint8, device="cuda")   # (NaN)
    out = torch.full_like(c.q_gpu, float("nan")) if out is None else out
    q = c.q_gpu if q is None else q
    if shared:
        group = torch.from_numpy(c.groups).cuda()
        B.tri_attend_shared(model, prefix, group, own, c.layer, tokens, q, out, scale=scale, causal=causal, workspace=ws, stream=stream)
    else:
        B.tri_attend(model, own, c.layer, tokens, q, out, scale=scale, causal=causal, workspace=ws, stream=stream)
    return out


def check(out, want):
    torch.cuda.synchronize()
    ref, tol = want
    got = out.double().cpu().numpy()
    off = np.abs(got - ref)
    worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off) / tol), off.shape)
    assert np.all(off <= tol), "at %s: %r, not %r +- %r" % (worst, got[worst], ref[worst], tol[worst])


# the roundings to bf16 that a case's kernel makes on the way to a product: of q, of the rotated key and of the weight where rows are many
def roundings(c):
    return 2 if c.dtype == torch.bfloat16 else 0


ROWS = [(1,), (1, 1, 1), (2, 1, 3), (5, 9, 1, 40), (130, 3, 77)]
OLD = {1: [(0,), (1,), (15,), (16,), (17,), (31,), (32,), (33,), (63,), (64,), (65,), (127,), (128,), (129,), (255,), (700,), (2500,)], 3: [(0, 1, 600), (64, 5, 130), (1000, 37, 256)],
       4: [(0, 300, 17, 64), (33, 1, 0, 500)]}


def sweep():
    n = 0
    for tokens in ROWS:
        for lens in OLD[len(tokens)]:
            n += 1
            yield pytest.param(n, lens, tokens, id="%s+%s" % ("_".join(map(str, lens)), "_".join(map(str, tokens))))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("seed,lens,tokens", list(sweep()))
def test_lengths(seed, lens, tokens, dtype):
    from paper_2604_04921_amd import binding as B
    c = P.Case(seed, lens, tokens, G=[4, 8, 1, 7, 3, 2, 5, 6][seed % 8], H=1 + seed % 2, dtype=dtype, pairs=seed % 2, stored_rotated=seed % 3 != 0,
               given_rotated=seed % 5 < 2, block=[0, 16, 64, 1, 32, 8, 256][seed % 7], order=["dense", "scattered"][seed // 2 % 2], appended=seed % 4 != 1)
    causal = seed % 6 != 5
    check(run(B, c, causal), c.want(causal=causal, roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("stored", [False, True], ids=["pre", "post"])
@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
@pytest.mark.parametrize("block", [0, 1, 2, 4, 8, 16, 32, 64, 128])
def test_layouts(dtype, stored, pairs, block):
    from paper_2604_04921_amd import binding as B
    for tokens in ((1, 1), (3, 20), (70, 1)):
        c = P.Case(block + 1000, (333, 90), tokens, dtype=dtype, pairs=pairs, stored_rotated=stored, block=block, order="scattered")
        check(run(B, c), c.want(roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1, 1), (4, 2, 3), (33, 64, 7), (150, 1, 129)])
@pytest.mark.parametrize("G", range(1, 9))
def test_every_key_counts_once(dtype, tokens, G):
    """Queries of zero weigh all keys alike, and value n is one in dimension n mod 128: the output says how many of the keys of each residue
    were attended to, up to its own rounding."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(G, (1500, 0, 777), tokens, H=1, G=G, dtype=dtype, zero_q=True, block=16 * (G % 2), order="dense", layers=1, layer=0)
    N = c.own["cap"]
    v = np.eye(128)[np.arange(N) % 128]
    c.own["v"][:] = v
    pages = c.own["table"]
    one = c.put(v)
    if pages is None:
        c.own["v_gpu"][0] = one[None, None]
    else:
        for s in range(c.S):
            c.own["v_gpu"][0, c.own["table_gpu"][s].long()] = one.view(-1, 1, c.block, 128)
    ref, _ = c.want()
    check(run(B, c), (ref, (P.HALF[dtype] + 2.0 ** -20) * np.abs(ref) + 1e-30))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("block", [0, 1, 16])
@pytest.mark.parametrize("backwards", [False, True])
def test_prompts_over_themselves(dtype, block, backwards):
    """A prompt's tokens over their own keys, whose later ones most rows leave out: in order, and with the slots of the one sequence turned round (every row then attends to the last slots)."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(81, (0, 0, 3), (700, 1300, 90), H=1, G=2, dtype=dtype, block=block, layers=1, layer=0, stored_rotated=block != 16)
    if backwards:
        n = c.own["total"][1]
        for f in ("k", "v", "pos"):
            c.own[f][1, :, :n] = c.own[f][1][:, :n][:, ::-1].copy()
        if block:
            pages = c.own["table"]
            for f in ("k", "v", "pos"):
                x = c.own[f][1]
                x = np.moveaxis(x.reshape((1, -1, block) + x.shape[2:]), 0, 1)
                x = torch.from_numpy(np.ascontiguousarray(x)).to(c.own[f + "_gpu"].dtype).cuda()
                keep = c.own[f + "_gpu"][0, pages[1]]
                live = (torch.arange(x.shape[0] * block, device="cuda") < n).view(x.shape[0], 1, block, *([1] * (x.dim() - 3)))
                c.own[f + "_gpu"][0, pages[1]] = torch.where(live, x, keep)
        else:
            for f in ("k", "v", "pos"):
                c.own[f + "_gpu"][0, 1, :, :n] = torch.from_numpy(np.ascontiguousarray(c.own[f][1, :, :n])).to(c.own[f + "_gpu"].dtype).cuda()
    check(run(B, c), c.want(roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1, 1, 1, 1, 1), (2, 1, 5, 1, 3, 2), (40, 20, 1, 9, 3, 2)])
@pytest.mark.parametrize("prefix,groups", [((500,), (0, 6)), ((70, 1, 300), (0, 2, 3, 6)), ((40, 0), (0, 6, 6)), ((1000, 33), (0, 1, 6))])
def test_shared(dtype, tokens, prefix, groups):
    from paper_2604_04921_amd import binding as B
    for i, (block, stored, order) in enumerate([(0, True, "dense"), (16, False, "scattered"), (64, True, "dense"), (4, False, "dense")]):
        c = P.Case(50 + i, (0, 40, 1, 0, 130, 17), tokens, dtype=dtype, G=[4, 8, 3, 6][i], block=block, stored_rotated=stored, order=order, prefix=prefix, groups=groups,
                   pairs=i % 2, appended=i != 2)
        check(run(B, c, causal=i != 3, shared=True), c.want(causal=i != 3, roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (3, 2), (50, 64), (150, 2)])
def test_rows_without_a_key(dtype, tokens):
    """Sequences without keys, and tokens ahead of every key: zeros."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(3, (0, 200), tokens, dtype=dtype, appended=False)
    out = run(B, c)
    check(out, c.want(roundings=roundings(c)))
    assert not out[:tokens[0]].any()
    c = P.Case(5, (0, 0), tokens, dtype=dtype, appended=False, block=16)   # (no sequence has a key; the first page of the table is not read for one)
    assert not run(B, c).any()
    c = P.Case(4, (40, 200), tokens, dtype=dtype, appended=False, pos0=1000)
    c.pos[:] = np.where(np.arange(c.T) % 2, c.pos, 5)
    out = run(B, c)
    check(out, c.want(roundings=roundings(c)))
    assert not out[::2].any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("tokens", [(1,), (3,), (8,), (40,), (200,)])
def test_not_numbers_stay_with_their_key(dtype, bad, tokens):
    """A key or value that is not a number, behind the position of some of the tokens: those are untouched by it, and the others get what it gives."""
    from paper_2604_04921_amd import binding as B
    for which in ("v", "k"):
        c = P.Case(9, (77,), tokens, dtype=dtype, layers=1, layer=0, H=1)
        T = tokens[0]
        at = 77 + T // 2 if T > 1 else 30
        if T == 1:
            c.own["pos"][0, 0, at] = 10 ** 6
            c.own["pos_gpu"][0, 0, 0, at] = 10 ** 6
        ref, tol = c.want(roundings=roundings(c))
        c.own[which + "_gpu"][0, 0, 0, at, 5] = bad
        got = run(B, c)
        torch.cuda.synchronize()
        got = got.double().cpu().numpy()
        free = c.pos < c.own["pos"][0, 0, at]
        assert np.all(np.abs(got - ref)[free] <= tol[free])
        if (~free).any() and which == "v":
            hit = got[~free][:, :, 5]
            assert np.all(np.isnan(hit)) if np.isnan(bad) else np.all(hit == bad)
            rest = np.arange(128) != 5
            assert np.all((np.abs(got - ref) <= tol)[~free][:, :, rest])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (5, 2), (40, 90)])
def test_lengths_per_head(dtype, tokens):
    from paper_2604_04921_amd import binding as B
    c = P.Case(21, (300, 150), tokens, H=3, dtype=dtype, block=16)
    lens = np.array([[300, 1, 17], [0, 150, 149]], dtype=np.int32)
    whole = torch.zeros((c.layers, 2, 3), dtype=torch.int32, device="cuda")
    whole[c.layer] = torch.from_numpy(lens).cuda()
    check(run(B, c, tokens=c.step(B, head_len=whole)), c.want(head_len=lens, roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (20, 9), (100, 40)])
@pytest.mark.parametrize("block", [2, 16, 64])
def test_blocks_that_are_not_there(dtype, tokens, block):
    """Occupied slots whose block id is negative or beyond the pool hold no key."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(22, (300, 140), tokens, dtype=dtype, block=block, layers=1, layer=0)
    pool = c.own["k_gpu"].shape[1]
    gone = np.zeros((c.S, c.own["cap"]), dtype=bool)
    for s, b, to in ((0, 0, -1), (0, 1, pool), (1, 1, 2 ** 31 - 1), (1, 0, -2 ** 31)):
        c.own["table_gpu"][s, b] = to
        gone[s, b * block:(b + 1) * block] = True
    # the same cache without those keys
    for s in range(c.S):
        n = c.own["total"][s]
        left = np.flatnonzero(~gone[s, :n])
        for f in ("k", "v", "pos"):
            c.own[f][s, :, :len(left)] = c.own[f][s][:, left]
        c.own["total"][s] = len(left)
    check(run(B, c), c.want(roundings=roundings(c)))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_strided_rows_streams_and_defaults(dtype):
    """q out of a fused projection's output, out into a wider buffer, heads before tokens, on a stream of its own; one token per sequence without start, at cur_pos."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(31, (500, 64, 3), (1, 1, 1), dtype=dtype, G=4, H=2)
    wide = torch.randn((c.T, 16, 128), device="cuda").to(dtype)
    wide[:, 3:11] = c.q_gpu
    out = torch.full((10, c.T, 128), 7.0, device="cuda", dtype=dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    own = c.own
    cache = B.Cache(own["k_gpu"], own["v_gpu"], own["pos_gpu"], own["lens_gpu"], torch.from_numpy(c.pos).cuda(), own["cap"], k_rotated=True)
    tokens = c.step(B, plain=True)
    tokens.c.pos = None
    torch.cuda.synchronize()
    run(B, c, own=cache, tokens=tokens, q=wide[:, 3:11], out=out[1:9].transpose(0, 1), stream=side)
    torch.cuda.synchronize()
    check(out[1:9].transpose(0, 1), c.want(roundings=roundings(c)))
    assert (out[0] == 7).all() and (out[9] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1,), (12,), (100,)])
def test_far_positions_and_scale(dtype, tokens):
    from paper_2604_04921_amd import binding as B
    for pos0 in (2 ** 31 - 2000, -2 ** 31, -500):
        c = P.Case(41, (900,), tokens, dtype=dtype, pos0=pos0, stored_rotated=False, pairs=1, theta=5e5)
        check(run(B, c, scale=0.02), c.want(scale=0.02, roundings=roundings(c)))


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("block", [0, 64])
def test_offsets_beyond_32_bits(tokens, block):
    """Heads (contiguous) and blocks (paged) that lie more than 2^32 bytes behind the first."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(51, (300,), (tokens,), H=2, layers=1, layer=0, block=block)
    k, v, pos = c.own["k_gpu"], c.own["v_gpu"], c.own["pos_gpu"]
    if block:
        far = torch.empty((1, 140000, 2, block, 128), dtype=k.dtype, device="cuda")   # 4.6 GB
        farv, farp = torch.empty_like(far), torch.empty((1, 140000, 2, block), dtype=torch.int32, device="cuda")
        n = k.shape[1]
        far[:, -n:], farv[:, -n:], farp[:, -n:] = k, v, pos
        c.own["table_gpu"] += 140000 - n
    else:
        rows = (1 << 31) // 128 + 500
        far, farv = (torch.empty((1, 1, 2, rows, 128), dtype=k.dtype, device="cuda") for _ in range(2))
        farp = torch.empty((1, 1, 2, rows), dtype=torch.int32, device="cuda")
        n = k.shape[3]
        far[:, :, :, :n], farv[:, :, :, :n], farp[:, :, :, :n] = k, v, pos
    c.own.update(k_gpu=far, v_gpu=farv, pos_gpu=farp)
    check(run(B, c), c.want(roundings=roundings(c)))


@pytest.mark.parametrize("tokens", [1, 20, 70])
@pytest.mark.parametrize("stored", [False, True], ids=["pre", "post"])
def test_slots_far_apart(tokens, stored):
    """Slots 2^24 elements apart and more: rows whose addresses 32 bits do not hold (the general kernel, in bf16)."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(52, (30,), (tokens,), H=2, layers=1, layer=0, stored_rotated=stored, pairs=int(stored))
    n, apart = c.own["cap"], 1 << 24
    k, v = (torch.empty((n, apart), dtype=torch.bfloat16, device="cuda") for _ in range(2))   # (only the slots' rows of it are touched)
    for to, f in ((k, "k_gpu"), (v, "v_gpu")):
        to[:, :256] = c.own[f][0, 0].transpose(0, 1).reshape(n, 256)
    strided = [t.as_strided((1, 1, 2, n, 128), (0, 0, 128, apart, 1)) for t in (k, v)]
    c.own.update(k_gpu=strided[0], v_gpu=strided[1])
    check(run(B, c), c.want(roundings=roundings(c)))


def test_graph_replays():
    """A step's append and attention captured once and replayed, with eager work between the replays."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(61, (400, 90), (1, 1), order="scattered", room=8)
    model, own, tokens = c.model(B), c.descriptor(B, c.own), c.step(B)
    ws = torch.empty(max(B.tri_attend_workspace_size(model, own, tokens), 256), dtype=torch.uint8, device="cuda")
    eager = run(B, c).clone()
    out = torch.zeros_like(eager)
    q = torch.zeros_like(c.q_gpu)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.tri_attend(model, own, c.layer, tokens, q, out, workspace=ws)
    for i in range(4):
        q.copy_(c.q_gpu if i % 2 == 0 else -c.q_gpu)
        graph.replay()
        torch.cuda.synchronize()
        want = run(B, c, q=q.clone())
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(out, eager) == (i % 2 == 0)
        ws.fill_(0xff)


def test_same_bits_every_time():
    from paper_2604_04921_amd import binding as B
    for tokens in ((1, 1), (30, 90)):
        c = P.Case(71, (5000, 777), tokens)
        first = run(B, c)
        for _ in range(3):
            assert torch.equal(run(B, c), first)


def exact_and_expected(c, scale):
    """The output in 64 bits, and the mean square that a row's error may have: output and weights rounded to bf16 (each off by at most 2^-8 of the value, evenly: a third of its square), q and turned keys to fp16 (2^-11), each
    rounding by itself; a score's error moves the output by weight x (value - output)."""
    out, square = np.zeros((c.T, c.H * c.G, 128)), np.zeros((c.T, c.H * c.G))
    q = P.turn(c.q, np.broadcast_to(c.pos[:, None], c.q.shape[:2]), c.theta, c.pairs)
    n = c.own["total"][0]
    for hq in range(c.H * c.G):
        k, v, pos = (c.own[f][0, hq // c.G, :n] for f in ("k", "v", "pos"))
        if not c.stored_rotated:
            k = P.turn(k, pos, c.theta, c.pairs)
        s = np.where(pos[None] <= c.pos[:, None], scale * q[:, hq] @ k.T, -np.inf)
        w = np.exp(s - s.max(1, keepdims=True))
        w /= w.sum(1, keepdims=True)
        o = out[:, hq] = w @ v
        score = scale ** 2 * ((q[:, hq] ** 2) @ (k ** 2).T) * (1 if c.stored_rotated else 2) * 2.0 ** -22 / 3
        apart = (v ** 2).sum(1)[None] - 2 * o @ v.T + (o ** 2).sum(1, keepdims=True)
        square[:, hq] = (w ** 2 * (score + 2.0 ** -16 / 3) * apart).sum(1) + 2.0 ** -16 / 3 * (o ** 2).sum(1)
    return out, square


@pytest.mark.parametrize("stored", [False, True], ids=["pre", "post"])
@pytest.mark.parametrize("tokens,block,pairs", [(3, 0, 0), (8, 16, 1), (60, 0, 0), (60, 64, 1), (60, 4, 0)])
def test_large_scores_keep_their_digits(tokens, block, pairs, stored):
    """Scores whose terms are several times 1: what q and turned keys are rounded to shows in the error of all outputs together."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(91, (1500,), (tokens,), G=4, layers=1, layer=0, stored_rotated=stored, block=block, pairs=pairs)
    ref, square = exact_and_expected(c, 0.3)
    got = run(B, c, scale=0.3)
    torch.cuda.synchronize()
    off = ((got.double().cpu().numpy() - ref) ** 2).sum()
    print("%.5f of %.5f" % (np.sqrt(off / (ref ** 2).sum()), np.sqrt(square.sum() / (ref ** 2).sum())))
    assert off <= square.sum()


@pytest.mark.parametrize("stored", [False, True], ids=["pre", "post"])
@pytest.mark.parametrize("power", [-60, -20, 13, 20, 100])
@pytest.mark.parametrize("tokens", [(3,), (60,)])
def test_magnitudes(tokens, power, stored):
    """Keys that fp16 does not hold, large and small, beside a third that is 2^-40 times the others and some zeros; queries the other way round."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(92, (700,), tokens, layers=1, layer=0, stored_rotated=stored)
    by = np.ldexp(1.0, power - 40 * (np.arange(c.own["cap"]) % 3 == 1))
    by[::50] = 0
    c.own["k"] *= by[:, None]
    c.own["k_gpu"] *= torch.from_numpy(by).float().cuda()[:, None]
    c.q, c.q_gpu = np.ldexp(c.q, -power), torch.ldexp(c.q_gpu.float(), torch.tensor(-power, device="cuda")).to(c.dtype)
    c.own["k_gpu"] = c.own["k_gpu"].to(c.dtype)
    check(run(B, c), c.want(roundings=roundings(c)))
