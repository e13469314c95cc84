"""tri_append4 where a workgroup takes four heads of its tokens (from 32768 rows of K on), bit for bit, and what one head at a time writes of the same rows."""
import numpy as np
import pytest
import torch

import pack4_plain as K
import test_gpu_pack4 as G

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
ROWS = 32768


def check_append(B, c, lens, cap=None, table=None, head_len=None, k_new=None, v_new=None, stream=None):
    """test_gpu_pack4's check_append, all rows at once."""
    own, lens = c.own, np.asarray(lens)
    if k_new is None:
        k_new, v_new = (c.put(c.g.standard_normal((c.T, c.H, 128))) for _ in range(2))
    want = G.host(own)
    top = own["cap"] if cap is None else cap
    s = np.repeat(np.arange(c.S), c.tokens)
    n = (np.broadcast_to(lens[:, None], (c.S, c.H)) if head_len is None else head_len)[s] + (np.arange(c.T) - c.start[s])[:, None]   # [T][H]
    s, h = np.broadcast_to(s[:, None], n.shape), np.broadcast_to(np.arange(c.H), n.shape)
    there, block, slot = n < top, s, n
    if c.block:
        block, slot = (own["table"] if table is None else table)[s, np.minimum(n, top - 1) // c.block], n % c.block
        there = there & (block >= 0) & (block < own["pos_gpu"].shape[1])
    where = (c.layer, block[there], h[there], slot[there])
    pos = np.broadcast_to(c.pos[:, None], n.shape)
    k = k_new.double().cpu().numpy()
    for f, x in (("k", k if c.given_rotated else K.P.turn(k, pos, c.theta, c.pairs)), ("v", v_new.double().cpu().numpy())):
        code, scale = K.encode(x)
        want[f + "4"][where], want[f + "s4"][where] = code[there], scale[there]
    want["pos_gpu"][where] = pos[there]
    heads = None
    if head_len is not None:
        heads = torch.zeros((c.layers, c.S, c.H), dtype=torch.int32, device="cuda")
        heads[c.layer] = torch.from_numpy(head_len).cuda()
    cache = K.descriptor(B, c, own, torch.tensor(lens.tolist(), dtype=torch.int32, device="cuda"))
    if cap is not None:
        cache.c.c.max_seq_len = cap
    got = torch.full((c.S,), -1, dtype=torch.int32, device="cuda")
    B.tri_append4(c.model(B), cache, c.layer, c.step(B, head_len=heads), k_new, v_new, got, stream=stream)
    torch.cuda.synchronize()
    G.check_fields(own, want)
    assert got.tolist() == np.minimum((lens if head_len is None else head_len[:, 0]) + np.asarray(c.tokens), top).tolist()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pairs, given", [(0, False), (1, False), (0, True)], ids=["interleaved", "half", "as_they_are"])
@pytest.mark.parametrize("H, tokens, block", [(8, (2048, 0, 1, 2047), 16), (5, (6554,), 0), (3, (10900, 23), 4), (1, (ROWS,), 64)], ids=lambda x: str(x).replace(" ", ""))
def test_four_heads(dtype, pairs, given, H, tokens, block):
    """Numbers of heads that are no multiple of four, empty sequences, tokens that end inside a workgroup's 32."""
    from paper_2604_04921_amd import binding as B
    assert sum(tokens) * H >= ROWS
    lens = [5, 0, 31, 2][:len(tokens)]
    c = K.Case(40 + H, lens, tokens, H=H, G=1, dtype=dtype, pairs=pairs, given_rotated=given, block=block, layers=1, layer=0, theta=1e6)
    check_append(B, c, lens)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_lengths_per_head_and_blocks_that_are_not_there(dtype):
    """Every head's place is found anew; a missing block of one sequence, full caches."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(50, (60, 30), (5000, 1600), H=5, G=1, dtype=dtype, pairs=1, block=16, layers=1, layer=0, theta=1e6)
    assert c.T * 5 >= ROWS
    table = c.own["table"].copy()
    table[0, 7], table[1, 20] = -1, c.own["pos_gpu"].shape[1]
    c.own["table_gpu"].copy_(torch.from_numpy(table))
    check_append(B, c, [60, 30], cap=4900, table=table, head_len=np.array([[60, 0, 17, 5, 44], [2, 30, 1, 29, 0]], dtype=np.int32))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_elements_next_to_a_border(dtype):
    """Among elements that lie on borders between numbers and scales but for what fp32 does not tell, too: the angles that four heads share are those that one works out."""
    from paper_2604_04921_amd import binding as B
    for pairs in (0, 1):
        c = K.Case(60, (0,), (4100,), H=8, G=1, dtype=dtype, pairs=pairs, layers=1, layer=0, theta=1e6)
        at = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])[c.g.integers(0, 7, (c.T, c.H, 128))] * np.where(c.g.random((c.T, c.H, 128)) < 0.5, -1, 1)
        at[..., ::32] = 7.0
        back = K.P.turn(at, -np.broadcast_to(c.pos[:, None].astype(np.int64), (c.T, c.H)), c.theta, c.pairs)
        assert c.T * c.H >= ROWS
        check_append(B, c, [0], k_new=c.put(back), v_new=c.put(at))


def test_strided_rows_on_another_stream():
    """Heads before tokens in a fused projection's output, 32768 rows and one token fewer: the same bits, head for head."""
    from paper_2604_04921_amd import binding as B
    c = K.Case(70, (3,), (4096,), H=8, G=1, block=64, layers=1, layer=0, theta=1e6)
    wide = c.put(c.g.standard_normal((17, c.T, 128)))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    first = {f: c.own[f].clone() for f in G.FIELDS}
    check_append(B, c, [3], k_new=wide[0:8].transpose(0, 1), v_new=wide[8:16].transpose(0, 1), stream=side)
    four = {f: c.own[f].clone() for f in G.FIELDS}
    for f in G.FIELDS:
        c.own[f].copy_(first[f])
    one = dict(k_new=wide[0:8, :4095].transpose(0, 1), v_new=wide[8:16, :4095].transpose(0, 1))
    lens = torch.tensor([3], dtype=torch.int32, device="cuda")
    step = B.Tokens(torch.from_numpy(c.pos[:4095]).cuda(), start=torch.tensor([0, 4095], dtype=torch.int32, device="cuda"))
    B.tri_append4(c.model(B), K.descriptor(B, c, c.own, lens), 0, step, **one)
    torch.cuda.synchronize()
    last = (3 + 4095) // 64, (3 + 4095) % 64
    block = int(c.own["table"][0, last[0]])
    for f in G.FIELDS:
        four[f][0, block, :, last[1]] = first[f][0, block, :, last[1]]
        assert torch.equal(four[f], c.own[f]), f
