"""What the binding of tri_append, tri_attend and tri_attend_shared refuses before the library sees a pointer (arrays that the kernels would read or write beyond), and what it lets through.  No GPU: the
library is a stand-in that writes down its arguments."""
import types

import pytest
import torch

from paper_2604_04921_amd import binding as B

L, S, H, G, N, T = 2, 3, 2, 4, 32, 5
STREAM = types.SimpleNamespace(cuda_stream=0)


class Recorder:
    """Stands in for libtri.so."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def entry(*args):
            self.calls.append((name, args))
            return 0
        return entry


@pytest.fixture
def lib(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(B, "_lib", r)
    return r


def i32(*shape, **kw):
    return torch.zeros(shape, dtype=torch.int32, **kw)


def cache(seqs=S, device="cpu"):
    k, v = (torch.zeros((L, seqs, H, N, 128), dtype=torch.bfloat16, device=device) for _ in range(2))
    return B.Cache(k, v, i32(L, seqs, H, N, device=device), i32(seqs, device=device), i32(seqs, device=device), N)


def step(start=S + 1, head_len=None, pos=T, device="cpu"):
    return B.Tokens(i32(pos, device=device), start=None if start is None else i32(start, device=device), max_tokens=2,
                    head_len=None if head_len is None else i32(*head_len, device=device))


def rows(heads, tokens=T, device="cpu"):
    return torch.zeros((tokens, heads, 128), dtype=torch.bfloat16, device=device)


MODEL = B.Model(L, H * G, H, 128, 1e6, [1])


def append(**kw):
    a = dict(cache=cache(), tokens=step(), k=rows(H), v=rows(H), new=i32(S))
    a.update(kw)
    B.tri_append(MODEL, a["cache"], 0, a["tokens"], a["k"], a["v"], a["new"], stream=STREAM)


def attend(**kw):
    a = dict(cache=cache(), tokens=step(), q=rows(H * G), out=rows(H * G), ws=torch.zeros(256, dtype=torch.uint8))
    a.update(kw)
    B.tri_attend(MODEL, a["cache"], 0, a["tokens"], a["q"], a["out"], workspace=a["ws"], stream=STREAM)


def shared(**kw):
    a = dict(prefix=cache(2), group=i32(3), cache=cache(), tokens=step(), q=rows(H * G), out=rows(H * G), ws=torch.zeros(256, dtype=torch.uint8))
    a.update(kw)
    B.tri_attend_shared(MODEL, a["prefix"], a["group"], a["cache"], 0, a["tokens"], a["q"], a["out"], workspace=a["ws"], stream=STREAM)


@pytest.mark.parametrize("entry", [append, attend, shared])
def test_arrays_of_the_step(lib, entry):
    """start has an entry per sequence and one more, head_len one per head-instance."""
    entry(tokens=step(head_len=(L, S, H)))
    entry(tokens=step(head_len=(L * S * H,)))
    entry(tokens=step(start=S + 4))   # (the first S + 1 are read)
    entry(cache=cache(T), tokens=step(start=None), **({"new": i32(T)} if entry is append else {}))
    assert len(lib.calls) == 4
    for bad in (step(start=S), step(start=1), step(head_len=(S, H)), step(head_len=(L, S, H - 1)), step(head_len=(L, S + 1, H))):
        with pytest.raises(ValueError):
            entry(tokens=bad)
    assert len(lib.calls) == 4


def test_new_lengths(lib):
    append(new=None)
    append(new=i32(S + 2))
    assert len(lib.calls) == 2
    for bad in (i32(S - 1), torch.zeros(S, dtype=torch.int64), torch.zeros(S), i32(2 * S)[::2]):
        with pytest.raises((ValueError, TypeError)):
            append(new=bad)
    assert len(lib.calls) == 2


def test_workspace_and_group(lib):
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(512, dtype=torch.uint8)[::2]):   # (fewer bytes, or other ones, than elements)
        for entry in (attend, shared):
            with pytest.raises(ValueError):
                entry(ws=bad)
    assert not lib.calls


def test_other_devices(lib):
    """Everything lies where the cache does.  ("meta" stands for another device.)"""
    for entry, heads, fields in ((append, H, ("k", "v")), (attend, H * G, ("q", "out")), (shared, H * G, ("q", "out"))):
        for f in fields:
            with pytest.raises(ValueError):
                entry(**{f: rows(heads, device="meta")})
        with pytest.raises(ValueError):
            entry(tokens=step(device="meta"))
    with pytest.raises(ValueError):
        append(new=i32(S, device="meta"))
    with pytest.raises(ValueError):
        attend(ws=torch.zeros(256, dtype=torch.uint8, device="meta"))
    with pytest.raises(ValueError):
        shared(group=i32(3, device="meta"))
    with pytest.raises(ValueError):
        shared(prefix=cache(2, device="meta"))
    assert not lib.calls


def test_strides_that_nothing_depends_on(lib):
    """One token, or one head: whatever stride it has, no row lies there."""
    one = B.Tokens(i32(1), start=i32(S + 1))
    k = torch.zeros((4, H, 128), dtype=torch.bfloat16)
    append(tokens=one, k=k[1:2], v=k.as_strided((1, H, 128), (7, 128, 1)))
    assert lib.calls[-1][1][6:8] == (0, 128)
    model = B.Model(L, 1, 1, 128, 1e6, [1])
    c = B.Cache(*(torch.zeros((L, S, 1, N, 128), dtype=torch.bfloat16) for _ in range(2)), i32(L, S, 1, N), i32(S), i32(S), N)
    q = torch.zeros((T, 1, 128), dtype=torch.bfloat16)
    B.tri_append(model, c, 0, step(), q, q.as_strided((T, 1, 128), (128, 3, 1)), stream=STREAM)
    assert lib.calls[-1][1][6:8] == (128, 0)
    with pytest.raises(ValueError):
        append(k=rows(H), v=torch.zeros((T, 2 * H, 128), dtype=torch.bfloat16)[:, :H])
