"""Calls too large for a launch are refused before anything is enqueued, and no call asks for more threads than HIP takes (fewer than 2^32 on an axis).  No GPU: see test_serve_refusals."""
import pytest

from test_serve_refusals import UNSUPPORTED, answers

WIDE = dict(layers=1, layer=0, heads=32, kv=8, s_seq=1 << 20, st=4096, ost=4096, qst=4096, dtype=0, pdtype=0)


def launches(log):
    got = []
    for line in log.splitlines():
        if line.startswith("launch"):
            x, y, z, block = (int(w) for w in line.split()[2:6])
            got.append((x * block, y, z))
    return got


# ragged batches whose bound on a sequence's tokens is far above their mean; long prompts over long caches; many rows to join; many rows to append
LARGE = [dict(entry="attend", seqs=256, most=8192, tokens=20000, n=32768), dict(entry="attend", seqs=2000, most=8192, tokens=20000, n=32768), dict(entry="attend", seqs=1, most=400000, tokens=400000, n=400000),
         dict(entry="attend", seqs=8000, most=1, tokens=8000, n=131072), dict(entry="attend", seqs=1, most=1 << 20, tokens=1 << 20, n=1 << 20, dtype=1), dict(entry="attend", seqs=4000, most=4000, tokens=8000, n=4096, dtype=1),
         dict(entry="shared", seqs=3, most=1, tokens=3, pseqs=3, n=64, pn=1 << 20), dict(entry="shared", seqs=1000, most=1, tokens=700000, pseqs=4, n=64, pn=1 << 20),
         dict(entry="shared", seqs=64, most=8192, tokens=20000, pseqs=64, n=32768, pn=1 << 20), dict(entry="append", seqs=3, tokens=1 << 25, most=1 << 25), dict(entry="append", seqs=3, tokens=(1 << 25) - 1, most=1 << 24),
         dict(entry="append", seqs=3, tokens=1 << 26, most=1 << 25, dtype=1), dict(entry="append", seqs=3, tokens=(1 << 26) - 1, most=1 << 25, dtype=1)]


def test_no_launch_is_larger_than_hip_takes():
    for c, (status, log) in zip(LARGE, answers([dict(WIDE, **c) for c in LARGE])):
        assert status in (0, UNSUPPORTED), c
        assert (status == 0) == bool(launches(log)), c
        assert all(x < 1 << 32 and y < 65536 and z < 65536 for x, y, z in launches(log)), (c, log)


@pytest.mark.parametrize("c", [dict(entry="attend", seqs=256, most=100000, tokens=200000, n=32768), dict(entry="shared", seqs=256, most=1, tokens=200000, pseqs=1000, n=64, pn=4096),
                               dict(entry="append", seqs=3, tokens=(1 << 25) - 1, most=1 << 24)], ids=["row tiles", "row tiles of prefixes", "rows"])
def test_refused(c):
    """More than 2^24 workgroups of 256 threads."""
    status, log = answers([dict(WIDE, **c)])[0]
    assert status == UNSUPPORTED and not log
    if c["entry"] != "append":
        size = answers([dict(WIDE, **dict(c, entry="size", prefix=c["entry"] == "shared"))])[0][0]
        assert size == (1 << 64) - 1


@pytest.mark.parametrize("c", [dict(entry="attend", seqs=1, most=131072, tokens=131072, n=1024), dict(entry="attend", seqs=64, most=8192, tokens=65536, n=8192, dtype=1),
                               dict(entry="attend", seqs=8000, most=1, tokens=8000, n=4096), dict(entry="append", seqs=3, tokens=(1 << 25) - 2, most=1 << 24)])
def test_taken(c):
    status, log = answers([dict(WIDE, **c)])[0]
    assert status == 0 and launches(log)
