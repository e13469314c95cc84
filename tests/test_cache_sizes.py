"""Caches whose arrays are smaller than a call would read or write are refused by the binding, before the library sees a pointer.  No GPU: the library is a stand-in that writes down its arguments."""
import pytest
import torch

import test_pack4_binding as P
import test_serve_binding as F
from paper_2604_04921_amd import binding as B
from test_pack4_binding import lib   # noqa: F401  (the stand-in)

L, S, H, G, N = P.L, P.S, P.H, P.G, P.N
i32, u8 = P.i32, P.u8


def four(layers=L, seqs=S, heads=H, slots=N, n=None, most=None, table=None):
    lead = (layers, seqs, heads, slots)
    n = seqs if n is None else n
    return B.Cache4(u8(*lead, 64), u8(*lead, 64), u8(*lead, 4), u8(*lead, 4), i32(*lead), i32(n), i32(n), slots if most is None else most, block_table=table)


def full(layers=L, seqs=S, heads=H, slots=N, n=None, most=None, table=None, pos=None, v=None):
    lead = (layers, seqs, heads, slots)
    n = seqs if n is None else n
    k = torch.zeros(lead + (128,), dtype=torch.bfloat16)
    if v is not None:   # the same strides, fewer entries
        v = k[tuple(slice(0, x) for x in v)]
    return B.Cache(k, k if v is None else v, i32(*(lead if pos is None else pos)), i32(n), i32(n), slots if most is None else most, block_table=table, k_rotated=True)


MOVES = [(P.pack, full, four), (P.unpack, four, full)]
IDS = ["pack", "unpack"]


@pytest.mark.parametrize("move, src, dst", MOVES, ids=IDS)
def test_destinations(lib, move, src, dst):   # noqa: F811
    budget = 7
    fine = [dst(), dst(slots=budget), dst(seqs=S, n=1, slots=budget, most=2), dst(layers=L + 1, seqs=S + 1, heads=H + 1), dst(seqs=9, slots=4, n=S, most=8, table=i32(S, 2)),
            dst(seqs=9, slots=4, n=1, most=1, table=i32(S, 2))]
    for d in fine:   # (a destination's own lengths and capacity are not read)
        move(src=src(), dst=d)
    move(src=src(most=5), dst=dst(slots=5))
    assert len(lib.calls) == len(fine) + 1
    bad = [dst(slots=budget - 1), dst(seqs=S - 1), dst(layers=L - 1), dst(heads=H - 1), dst(seqs=9, slots=4, n=1, most=8, table=i32(S - 1, 2)), dst(layers=L - 1, seqs=9, slots=4, n=S, most=8, table=i32(S, 2))]
    for d in bad:
        with pytest.raises(ValueError):
            move(src=src(), dst=d)
    for b, d in ((N, dst(slots=N - 1)), (2 * N, dst(slots=N - 1))):   # (no more than the source's slots are written)
        with pytest.raises(ValueError):
            move(src=src(), dst=d, budget=b, idx=None)
    move(src=src(), dst=dst(), budget=2 * N, idx=None)
    assert len(lib.calls) == len(fine) + 2


@pytest.mark.parametrize("move, src, dst", MOVES, ids=IDS)
def test_sources(lib, move, src, dst):   # noqa: F811
    move(src=src(layers=L + 1, seqs=S + 1, heads=H + 2, n=S), dst=dst())
    assert len(lib.calls) == 1
    for s in (src(layers=L - 1), src(heads=H - 1)):
        with pytest.raises(ValueError):
            move(src=s, dst=dst())
    assert len(lib.calls) == 1


def test_arrays_of_a_full_cache(lib):   # noqa: F811
    """Its keys, values and positions are arrays of their own: the smallest counts, on either side."""
    for kw in (dict(pos=(L, S, H, N - 1)), dict(pos=(L, S - 1, H, N)), dict(pos=(L - 1, S, H, N)), dict(pos=(L, S, H - 1, N)), dict(v=(L, S, H, N - 1)), dict(v=(L, S - 1, H, N)), dict(n=S, seqs=S - 1), dict(most=N + 1)):
        with pytest.raises(ValueError):
            P.pack(src=full(**kw))
        if "most" not in kw:
            with pytest.raises(ValueError):
                P.unpack(dst=full(**kw), budget=N, idx=None)
    for kw in (dict(pos=(L, 8, H, 4)), dict(pos=(L, 9, H, 3)), dict(v=(L, 8, H, 4))):   # blocks, and slots of a block
        with pytest.raises(ValueError):
            P.pack(src=full(seqs=9, slots=4, n=S, most=8, table=i32(S, 2), **kw))
    assert not lib.calls


@pytest.mark.parametrize("entry", [P.append, P.attend, F.append, F.attend])
def test_layers_and_heads_of_a_step(lib, entry):   # noqa: F811
    """A layer's call needs that layer, and the model's heads."""
    make = four if entry in (P.append, P.attend) else full
    entry(cache=make(layers=1))   # (of layer 0)
    entry(cache=make(heads=H + 1))
    assert len(lib.calls) == 2
    for c in (make(heads=H - 1), make(layers=0)):
        with pytest.raises(ValueError):
            entry(cache=c)
    assert len(lib.calls) == 2


@pytest.mark.parametrize("entry, prefix", [(P.shared, four), (F.shared, full)], ids=["four", "full"])
def test_layers_and_heads_behind_prefixes(lib, entry, prefix):   # noqa: F811
    entry(prefix=prefix(seqs=2, layers=1), cache=full(layers=1))
    assert len(lib.calls) == 1
    for bad in (dict(prefix=prefix(seqs=2, heads=H - 1)), dict(cache=full(heads=H - 1)), dict(prefix=prefix(seqs=2, layers=0)), dict(cache=full(layers=0))):
        with pytest.raises(ValueError):
            entry(**bad)
    assert len(lib.calls) == 1


def test_the_layer_that_is_asked_for(lib):   # noqa: F811
    model = B.Model(4, H * G, H, 128, 1e6, [1])
    for layer, c in ((1, four()), (0, four(layers=1))):
        B.tri_append4(model, c, layer, P.step(), P.rows(H), P.rows(H), stream=P.STREAM)
    for layer, c in ((2, four()), (1, four(layers=1)), (3, four())):
        with pytest.raises(ValueError):
            B.tri_append4(model, c, layer, P.step(), P.rows(H), P.rows(H), stream=P.STREAM)
        with pytest.raises(ValueError):
            B.tri_attend4(model, c, layer, P.step(), P.rows(H * G), P.rows(H * G), stream=P.STREAM)
    assert len(lib.calls) == 2
