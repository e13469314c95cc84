"""tri_attend4 and tri_attend4_shared against 64 bits, no further off than the roundings that include/tri.h states (tests/attend4_cases.py, tests/serve_exact.py)."""
import numpy as np
import pytest
import torch

import attend4_cases as A
import pack4_plain as K
import serve_exact as X

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def wrong(call, got):
    torch.cuda.synchronize()
    return X.wrong(call, got.double().cpu().numpy(), *call.value())


@pytest.mark.parametrize("spec", A.specs(), ids=lambda s: s["name"])
def test_no_more_roundings_than_stated(spec):
    from paper_2604_04921_amd import binding as B
    call = A.make(spec, "cuda")
    c = call.c
    tokens = None
    if call.head_len is not None:
        whole = torch.zeros((c.layers, c.S, c.H), dtype=torch.int32, device="cuda")
        whole[c.layer] = torch.from_numpy(call.head_len).cuda()
        tokens = c.step(B, head_len=whole)
    assert wrong(call, K.attend(B, c, scale=call.scale, causal=call.causal, tokens=tokens)) == []


class Added(X.Call):
    """With the error of the matrix instruction's sums.  It adds the products of eight neighbouring dimensions as multiples of 2^-13 of the largest one's power of two (measured: 256 + 1.875 2^-5 + 1.875 2^-6 ... in one eight loses
    what is below 2^-5, in two it loses nothing), so that each of the other seven is off by less than that, its square by a third of that squared on average; these sums are added in fp32.  The later parts of a query, of 2^-4, 2^-8
    and 2^-12 of it, add less than a 255th to the squares."""

    def scores(self, q, k, kind, mutant, held):
        sc, var = super().scores(q, k, kind, mutant, held)
        largest = np.abs(q[:, None].reshape(len(q), 1, 16, 8) * k[None].reshape(1, len(k), 16, 8)).max(-1) if len(k) else np.zeros((len(q), 0, 16))
        return sc, var + (self.scale * 2.0 ** -13) ** 2 * 7 / 3 * 256 / 255 * (largest ** 2).sum(-1)


@pytest.mark.parametrize("tokens, G", [((9, 1), 4), ((16, 3), 4), ((12,), 5), ((8, 8, 8), 8), ((33,), 1)])
@pytest.mark.parametrize("block, rotated", [(0, False), (4, True), (16, False), (64, True)])
def test_up_to_64_rows_are_held_as_few_are(monkeypatch, tokens, G, block, rotated):
    """33 to 64 rows per KV head, against the tolerance of 16 bits for queries and weights."""
    from paper_2604_04921_amd import binding as B
    monkeypatch.setattr(X, "kernel_of", lambda c, rows: "few")
    c = K.Case(31 + len(tokens) + block, (700, 64, 300)[:len(tokens)], tokens, G=G, block=block, given_rotated=rotated, H=3)
    call = Added(c, scale=0.3)
    assert wrong(call, K.attend(B, c, scale=call.scale)) == []


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (9, 30), (70, 200)])
@pytest.mark.parametrize("block", [0, 4, 16])
def test_rows_without_a_key_get_zeros(dtype, tokens, block):
    """An empty sequence; tokens before all keys."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(3, (0, 200), tokens, dtype=dtype, block=block, appended=False)
    pos = torch.from_numpy(c.pos).cuda()
    pos[c.start[1]] = -1   # before all keys
    out = K.attend(B, c, tokens=B.Tokens(pos, start=torch.from_numpy(c.start).cuda(), max_tokens=max(tokens)))
    torch.cuda.synchronize()
    assert (out[:c.start[1] + 1] == 0).all()
    if tokens[1] > 1:
        assert (out[c.start[1] + 1:].abs().amax(dim=(1, 2)) > 0).all()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1,), (3,), (8,), (40,), (200,)])
@pytest.mark.parametrize("block", [0, 4, 16])
def test_not_numbers_stay_with_their_key(dtype, tokens, block):
    """32 elements of a key or value that are no numbers, behind the position of some of the tokens: those are untouched by them, and the others get NaN -- everywhere, or in these dimensions."""
    from paper_2604_04921_amd import binding as B
    for which in ("v", "k"):
        c = K.Case(9, (77,), tokens, dtype=dtype, layers=1, layer=0, H=1, block=block)
        T = tokens[0]
        at = 77 + T // 2 if T > 1 else 30
        slot = (0, 0, 0, at) if not block else (0, int(c.own["table"][0, at // block]), 0, at % block)
        if T == 1:
            c.own["pos"][0, 0, at] = 10 ** 6
            c.own["pos_gpu"][slot] = 10 ** 6
        call = X.Call(c)
        ref, var = call.value()
        c.own[which + "s4"][slot][2] = 255
        got = K.attend(B, c)
        torch.cuda.synchronize()
        got = got.double().cpu().numpy()
        limit = X.P.HALF[dtype] * np.abs(ref) + 6 * np.sqrt(var) + 1e-30
        free = c.pos < c.own["pos"][0, 0, at]
        assert np.all(np.abs(got - ref)[free] <= limit[free])
        if (~free).any():
            if which == "k":
                assert np.isnan(got[~free]).all()
                continue
            hit = np.zeros(128, dtype=bool)
            hit[64:96] = True
            assert np.isnan(got[~free][:, :, hit]).all()
            assert np.all((np.abs(got - ref) <= limit)[~free][:, :, ~hit])


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("block", [0, 2, 16, 64])
def test_what_is_not_occupied_is_not_used(dtype, block):
    """Whatever lies beyond the lengths (here it is no number, then large numbers), the outputs have the same bits."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(13, (77, 300, 5), (1, 3, 2), dtype=dtype, block=block, room=100, layers=1, layer=0)
    first = K.attend(B, c)
    dead = np.arange(c.own["cap"])[None] >= np.asarray(c.own["total"])[:, None]
    for f, fill in (("k4", 0x77), ("v4", 0xff), ("ks4", 200), ("vs4", 200)):
        for s in range(c.S):
            for n in np.flatnonzero(dead[s]):
                where = (0, s, slice(None), n) if not block else (0, int(c.own["table"][s, n // block]), slice(None), n % block)
                c.own[f][where] = fill
    assert torch.equal(K.attend(B, c), first)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_strided_rows_streams_and_defaults(dtype):
    """q out of a fused projection's output, out into a wider buffer, heads before tokens, on a stream of its own; one token per sequence without start, at cur_pos; k and v side by side in one array."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(31, (500, 64, 3), (1, 1, 1), dtype=dtype, G=4, H=2)
    wide = torch.randn((c.T, 16, 128), device="cuda").to(dtype)
    wide[:, 3:11] = c.q_gpu
    out = torch.full((10, c.T, 128), 7.0, device="cuda", dtype=dtype)
    own = c.own
    both = torch.full(own["k4"].shape[:4] + (3, 64), 0xaa, dtype=torch.uint8, device="cuda")
    both[..., 0, :], both[..., 2, :] = own["k4"], own["v4"]
    n = own["lens_gpu"]
    cache = B.Cache4(both[..., 0, :], both[..., 2, :], own["ks4"], own["vs4"], own["pos_gpu"], n, torch.from_numpy(c.pos).cuda(), own["cap"], rows=dtype)
    tokens = c.step(B, plain=True)
    tokens.c.pos = None
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    K.attend(B, c, q=wide[:, 3:11], out=out[1:9].transpose(0, 1), tokens=tokens, stream=side, desc=cache)
    torch.cuda.synchronize()
    assert wrong(X.Call(c), out[1:9].transpose(0, 1)) == []
    assert (out[0] == 7).all() and (out[9] == 7).all()


@pytest.mark.parametrize("tokens", [1, 40])
@pytest.mark.parametrize("block", [0, 64])
def test_offsets_beyond_32_bits(tokens, block):
    """Heads (contiguous) and blocks (paged) that lie more than 2^32 bytes behind the first."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(51, (300,), (tokens,), H=2, layers=1, layer=0, block=block)
    own = c.own
    n = own["k4"].shape[1] if block else own["cap"]
    lead = (1, 540000, 2, block) if block else (1, 1, 2, (1 << 32) // 64 + 500)
    part = (slice(None), slice(-n, None)) if block else (slice(None), slice(None), slice(None), slice(0, n))
    for f, w in (("k4", (64,)), ("v4", (64,)), ("ks4", (4,)), ("vs4", (4,)), ("pos_gpu", ())):
        far = torch.empty(lead + w, dtype=own[f].dtype, device="cuda")
        far[part] = own[f]
        own[f] = far
    if block:
        own["table_gpu"] += 540000 - n
    assert wrong(X.Call(c), K.attend(B, c)) == []


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (60, 9)])
def test_capacities_far_above_the_lengths(dtype, tokens):
    """max_seq_len is a capacity: the lengths decide."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(52, (300, 2000), tokens, H=2, layers=1, layer=0, block=16, dtype=dtype)
    table = torch.full((2, 8192), -1, dtype=torch.int32, device="cuda")
    table[:, :c.own["table_gpu"].shape[1]] = c.own["table_gpu"]
    c.own["table_gpu"], c.own["cap"] = table, 131072
    assert wrong(X.Call(c), K.attend(B, c)) == []


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (30, 90), (200, 300)])
def test_same_bits_every_time(dtype, tokens):
    from paper_2604_04921_amd import binding as B
    c = K.Case(71, (5000, 777), tokens, dtype=dtype)
    first = K.attend(B, c)
    for _ in range(3):
        assert torch.equal(K.attend(B, c), first)


def test_two_streams_with_a_workspace_each():
    from paper_2604_04921_amd import binding as B
    cases = [K.Case(81 + i, (3000, 50), (2, 1), block=16) for i in range(2)]
    want = [K.attend(B, c).clone() for c in cases]
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in cases], [torch.zeros_like(w) for w in want]
    spaces = [torch.empty(max(256, B.tri_attend4_workspace_size(c.model(B), K.descriptor(B, c, c.own), c.step(B))), dtype=torch.uint8, device="cuda") for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s, o, w in zip(cases, streams, outs, spaces):
            K.attend(B, c, out=o, stream=s, ws=w)
    torch.cuda.synchronize()
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_two_graphs_with_one_workspace():
    """Replayed in turn on one stream, the workspace being anything in between."""
    from paper_2604_04921_amd import binding as B
    cases = [K.Case(91, (3000, 50), (2, 1), block=16), K.Case(92, (900,), (70,), block=4)]
    want = [K.attend(B, c).clone() for c in cases]
    calls = [(c.model(B), K.descriptor(B, c, c.packed()), c.layer, c.step(B), c.q_gpu, torch.zeros_like(c.q_gpu)) for c in cases]
    ws = torch.full((max([256] + [B.tri_attend4_workspace_size(a[0], a[1], a[3]) for a in calls]),), 255, dtype=torch.uint8, device="cuda")
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    torch.cuda.synchronize()
    for g, a in zip(graphs, calls):
        with torch.cuda.graph(g):
            B.tri_attend4(*a, workspace=ws)
    for i in range(6):
        calls[i % 2][5].fill_(3.0)
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(calls[i % 2][5], want[i % 2])
        if i % 3 == 0:
            ws.fill_(i)


@pytest.mark.parametrize("shared", [False, True])
def test_graph_of_a_step(shared):
    """An append in 4 bits and the attention over what it wrote (or an append to the sequences' own caches behind a prefix in 4 bits), captured once and replayed with other rows, eager work in between."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(13, (40, 7, 0), (1, 1, 1), block=16, prefix=(300,) if shared else None, layers=1, layer=0)
    own = c.own
    lens = torch.tensor([40, 7, 0], dtype=torch.int32, device="cuda")
    after = torch.zeros_like(lens)
    model, tokens = c.model(B), c.step(B)
    describe = c.descriptor if shared else lambda B, own, lens: K.descriptor(B, c, own, lens)   # noqa: E731
    before, behind = describe(B, own, lens), describe(B, own, after)
    prefix = K.descriptor(B, c, c.prefix) if shared else None
    k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    out = torch.zeros_like(c.q_gpu)
    size = B.tri_attend4_workspace_size(model, prefix, tokens, behind) if shared else B.tri_attend4_workspace_size(model, behind, tokens)
    ws = torch.empty(max(256, size), dtype=torch.uint8, device="cuda")

    def step(to):
        if shared:
            B.tri_append(model, before, 0, tokens, k_new, v_new, after)
            B.tri_attend4_shared(model, prefix, None, behind, 0, tokens, c.q_gpu, to, workspace=ws)
        else:
            B.tri_append4(model, before, 0, tokens, k_new, v_new, after)
            B.tri_attend4(model, behind, 0, tokens, c.q_gpu, to, workspace=ws)
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


@pytest.mark.parametrize("pairs", [0, 1], ids=["interleaved", "half"])
def test_compressed_packed_appended_attended_and_scored_again(pairs):
    """The operators in their order: a cache is compressed, what is kept goes into 4 bits, tokens are appended and attended to, and the cache is read back, scored and packed again."""
    from paper_2604_04921_amd import binding as B
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    L, S, H, G, N, budget, window = 2, 2, 2, 4, 700, 256, 20
    Hq, cap = H * G, budget + window
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF16)   # noqa: E731
    i32 = dict(dtype=torch.int32, device="cuda")
    model = B.Model(L, Hq, H, 128, 1e6, [1, 2, 4, 8], pairs=pairs)
    k, v, pos = rand(L, S, H, N, 128), rand(L, S, H, N, 128), torch.arange(N, **i32).expand(L, S, H, N).contiguous()
    centers = torch.empty((L, Hq, 64, 3), device="cuda")
    B.tri_build_centers(model, rand(300, L, Hq, 128), centers)
    n, cur = torch.tensor([N, 500], **i32), torch.tensor([N, 500], **i32)
    full = B.Cache(k, v, pos, n, cur, N)
    idx, cnt = torch.empty((L, S, H, budget), **i32), torch.empty((L, S, H), **i32)
    final = torch.empty((L, S, H, N), device="cuda")
    ws = torch.empty(B.tri_workspace_size(model, full, budget), dtype=torch.uint8, device="cuda")
    B.tri_score(model, centers, full, final, None, ws)
    B.tri_select_topk(model, final, full, budget, idx, cnt, ws)
    new = lambda *w: torch.full((L, S, H, cap) + w, 0xff, dtype=torch.uint8, device="cuda")   # noqa: E731
    four = (new(64), new(64), new(4), new(4), torch.full((L, S, H, cap), -1, **i32))
    lens = [torch.zeros(S, **i32) for _ in range(2)]
    packed = [B.Cache4(*four, x, x, cap) for x in lens]
    B.tri_pack4(model, full, packed[0], budget, idx, cnt, lens[0])
    rows = []
    for t in range(window):
        at = (cur + t).contiguous()
        tokens = B.Tokens(at)
        for l in range(L):
            kn, vn, q = rand(S, H, 128), rand(S, H, 128), rand(S, Hq, 128)
            B.tri_append4(model, packed[0], l, tokens, kn, vn, lens[1])
            out = torch.empty_like(q)
            aws = torch.empty(max(256, B.tri_attend4_workspace_size(model, packed[1], tokens)), dtype=torch.uint8, device="cuda")
            B.tri_attend4(model, packed[1], l, tokens, q, out, workspace=aws)
        rows.append((q, out, at))
        lens.reverse()
        packed.reverse()
    torch.cuda.synchronize()
    assert lens[0].tolist() == [cap, cap]
    back = [torch.zeros((L, S, H, cap, 128), dtype=BF16, device="cuda") for _ in range(2)] + [torch.zeros((L, S, H, cap), **i32)]
    again = B.Cache(*back, lens[0], at, cap, k_rotated=True)
    B.tri_unpack4(model, packed[0], again, cap)
    # the last step's attention from what was read back, in 64 bits
    q, out, at = rows[-1]
    turned = K.P.turn(q.double().cpu().numpy(), np.broadcast_to(at.cpu().numpy()[:, None], (S, Hq)), 1e6, pairs)
    for s in range(S):
        for h in range(Hq):
            kk, vv = (back[i][L - 1, s, h // G].double().cpu().numpy() for i in range(2))
            o, w, off = K.P.attend(turned[s, h:h + 1], kk, vv, np.ones((1, cap), dtype=bool), 128 ** -0.5)
            assert np.all(np.abs(out[s, h].double().cpu().numpy() - o[0]) <= K.P.bound(o, w, off, BF16, 0, turned=True)[0])
    # and the next compression keeps the same keys of it as of the numbers that it reads back
    final2 = torch.empty((L, S, H, cap), device="cuda")
    ws2 = torch.empty(B.tri_workspace_size(model, again, budget), dtype=torch.uint8, device="cuda")
    B.tri_score(model, centers, again, final2, None, ws2)
    B.tri_select_topk(model, final2, again, budget, idx, cnt, ws2)
    kept = four[0].clone()
    B.tri_pack4(model, again, packed[0], budget, idx, cnt, lens[1])
    torch.cuda.synchronize()
    assert lens[1].tolist() == [budget, budget] and (cnt == budget).all()
    want = torch.gather(kept, 3, idx.long()[..., None].expand(-1, -1, -1, -1, 64))
    assert K.same_codes(four[0][:, :, :, :budget].cpu().numpy(), want.cpu().numpy())   # (the rows themselves: packing them again changes nothing)
