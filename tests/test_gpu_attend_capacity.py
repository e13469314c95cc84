"""A cache's capacity (max_seq_len) says how many workgroups there are, not where the work lies: the same lengths in far larger caches take no several times as long.  Parts without a key once left all work to one of
the GPU's eight XCDs, twenty times as long; what is allowed here is four times."""
import statistics

import pytest
import torch

import serve_plain as P

pytestmark = pytest.mark.gpu


def microseconds(f):
    times = []
    for _ in range(7):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        f()
        a.record()
        for _ in range(5):
            f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 200)
    return statistics.median(times)


@pytest.mark.parametrize("seqs,keys,tokens,dtype", [(64, 2000, 1, torch.bfloat16), (16, 2000, 1, torch.bfloat16), (8, 3000, 8, torch.bfloat16), (2, 4000, 500, torch.bfloat16), (2, 2000, 256, torch.float32),
                                                    (16, 2000, 1, torch.float32)])
def test_time_by_lengths(seqs, keys, tokens, dtype):
    from paper_2604_04921_amd import binding as B
    H, G = 8, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    k, v = (torch.randn((1, seqs, H, keys, 128), generator=g, device="cuda").to(dtype) for _ in range(2))
    pos = torch.arange(keys, device="cuda", dtype=torch.int32).expand(1, seqs, H, keys).contiguous()
    lens = torch.full((seqs,), keys, dtype=torch.int32, device="cuda")
    q = torch.randn((seqs * tokens, H * G, 128), generator=g, device="cuda").to(dtype)
    model = B.Model(1, H * G, H, 128, 1e6, [1])
    step = B.Tokens(torch.arange(keys - tokens, keys, device="cuda", dtype=torch.int32).repeat(seqs), start=torch.arange(seqs + 1, device="cuda", dtype=torch.int32) * tokens, max_tokens=tokens)
    took, outs = {}, {}
    for bound in (keys, 22400, 45000, 90000, 131072, 180000):
        cache = B.Cache(k, v, pos, lens, lens, bound, k_rotated=True)   # (memory ends with the longest sequence: no length passes it)
        ws = torch.empty(max(B.tri_attend_workspace_size(model, cache, step), 256), dtype=torch.uint8, device="cuda")
        out = outs[bound] = torch.empty_like(q)
        took[bound] = microseconds(lambda: B.tri_attend(model, cache, 0, step, q, out, workspace=ws))   # noqa: B023
    print({n: "%.0f us" % t for n, t in took.items()})
    assert max(took.values()) < 4 * took[keys] + 50
    for out in outs.values():
        assert (out.double() - outs[keys].double()).norm() <= 8 * P.HALF[dtype] * outs[keys].double().norm()
