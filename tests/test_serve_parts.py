"""How much workspace attention wants: partial results are bounded by the work there is, not by the length that a cache could have.  No GPU: see test_serve_refusals."""
import pytest

from test_serve_refusals import answers

WIDE = dict(entry="size", layers=1, layer=0, heads=32, kv=8, s_seq=1 << 24, st=4096, ost=4096, qst=4096, seqs=1, pseqs=1, prefix=False)
MOST = 64 << 20   # of sums, of one cache's parts


def sizes(cases):
    return [a[0] for a in answers([dict(WIDE, **c) for c in cases])]


def rows(c):
    return c["tokens"] * 32


@pytest.mark.parametrize("dtype", [0, 1], ids=["f32", "bf16"])
@pytest.mark.parametrize("tokens", [256, 2048, 8192, 32768])
def test_a_long_bound(dtype, tokens):
    """A prompt in caches of growing capacity: what one part takes (row sums, a maximum and a total each), or parts of MOST bytes together."""
    for c, size in zip(*(lambda cs: (cs, sizes(cs)))([dict(tokens=tokens, most=tokens, n=n, dtype=dtype) for n in (8192, 131072, 1 << 20)])):
        assert size <= max(MOST, 2 * rows(c) * 512) * 1.02 + 512, (c, size)


def test_many_sequences():
    for seqs, tokens, most in ((64, 4096, 64), (256, 2048, 8), (256, 20000, 8192)):
        for dtype in (0, 1):
            c = dict(seqs=seqs, tokens=tokens, most=most, n=131072, dtype=dtype)
            assert sizes([c])[0] <= max(MOST, 2 * rows(c) * 512) * 1.02 + 512


def test_prefixes():
    c = dict(seqs=256, tokens=20000, most=8192, n=4096, dtype=1, prefix=True, pn=1 << 20)
    assert sizes([c])[0] <= 2 * max(MOST, 2 * rows(c) * 512) * 1.02 + 512


def test_small_steps_keep_their_parts():
    """A long context is cut for one token as before: its rows are few."""
    few = sizes([dict(tokens=1, most=1, n=n, dtype=1) for n in (2176, 131072)])
    assert few[0] < few[1] <= 32 * 256 * 520 + 1024


@pytest.mark.parametrize("c", [dict(dtype=2), dict(dtype=-1), dict(pdtype=7, prefix=True), dict(dtype=1, pdtype=0, prefix=True)])
def test_types_that_there_are_not(c):
    """The size goes by the type: one that the calls refuse has none."""
    assert sizes([dict(tokens=1, most=1, n=131072, **c)]) == [(1 << 64) - 1]
