"""Caches whose capacity (max_seq_len) is far above the lengths that occur: the same keys, each once."""
import numpy as np
import pytest
import torch

import serve_plain as P
from test_gpu_attend import check, roundings, run

pytestmark = pytest.mark.gpu


def roomy(B, c, cache, bound):
    """The cache's descriptor with another bound: contiguous ones' memory ends with the longest sequence, paged ones' tables name no block beyond it."""
    if cache["table"] is None:
        d = c.descriptor(B, cache)
        d.c.max_seq_len = bound
        return d
    wide = torch.full((len(cache["total"]), -(-bound // c.block)), -1, dtype=torch.int32, device="cuda")
    wide[:, :cache["table_gpu"].shape[1]] = cache["table_gpu"]
    return B.Cache(cache["k_gpu"], cache["v_gpu"], cache["pos_gpu"], cache["lens_gpu"], cache["lens_gpu"], bound, block_table=wide, k_rotated=c.stored_rotated)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bound", [5000, 131072, 1 << 20])
@pytest.mark.parametrize("block", [0, 4, 16])
@pytest.mark.parametrize("tokens", [(1, 1, 1), (8, 2, 3), (300, 64, 7), (1500, 1, 1)])
def test_every_key_counts_once(dtype, tokens, block, bound):
    """Queries of zero weigh all keys alike, and value n is one in dimension n mod 128: the output counts the keys of each residue."""
    from paper_2604_04921_amd import binding as B
    c = P.Case(7, (1500, 0, 777), tokens, H=1, G=4, dtype=dtype, zero_q=True, block=block, layers=1, layer=0)
    v = np.eye(128)[np.arange(c.own["cap"]) % 128]
    c.own["v"][:] = v
    one = c.put(v)
    if block:
        for s in range(c.S):
            c.own["v_gpu"][0, c.own["table_gpu"][s].long()] = one.view(-1, 1, block, 128)
    else:
        c.own["v_gpu"][0] = one[None, None]
    ref, _ = c.want()
    check(run(B, c, own=roomy(B, c, c.own, bound)), (ref, (P.HALF[dtype] + 2.0 ** -20) * np.abs(ref) + 1e-30))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("tokens", [(1, 1), (5, 2), (200, 90)])
def test_behind_prefixes(dtype, tokens):
    from paper_2604_04921_amd import binding as B
    for block in (0, 16):
        c = P.Case(8, (300, 20), tokens, dtype=dtype, block=block, prefix=(700,), groups=(0, 2))
        own, prefix = (roomy(B, c, x, 131072) for x in (c.own, c.prefix))
        model, step = c.model(B), c.step(B)
        ws = torch.full((max(B.tri_attend_workspace_size(model, own, step, prefix), 256),), 0xff, dtype=torch.uint8, device="cuda")
        out = torch.full_like(c.q_gpu, float("nan"))
        B.tri_attend_shared(model, prefix, torch.from_numpy(c.groups).cuda(), own, c.layer, step, c.q_gpu, out, workspace=ws)
        check(out, c.want(roundings=roundings(c)))
