"""What the binding of the 4-bit caches' entry points refuses before the library sees a pointer, and what it lets through.  No GPU: the library is a stand-in that writes down its arguments."""
import types

import pytest
import torch

from paper_2604_04921_amd import binding as B

L, S, H, G, N, T = 2, 3, 2, 4, 32, 5
STREAM = types.SimpleNamespace(cuda_stream=0)
MODEL = B.Model(L, H * G, H, 128, 1e6, [1])


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


def u8(*shape, **kw):
    return torch.zeros(shape, dtype=torch.uint8, **kw)


def cache(seqs=S, device="cpu", dtype=torch.bfloat16):
    k, v = (torch.zeros((L, seqs, H, N, 128), dtype=dtype, device=device) for _ in range(2))
    return B.Cache(k, v, i32(L, seqs, H, N, device=device), i32(seqs, device=device), i32(seqs, device=device), N, k_rotated=True)


def parts(seqs=S, device="cpu", **kw):
    lead = (L, seqs, H, N)
    p = dict(k=u8(*lead, 64, device=device), v=u8(*lead, 64, device=device), ks=u8(*lead, 4, device=device), vs=u8(*lead, 4, device=device), pos=i32(*lead, device=device), n=i32(seqs, device=device))
    p.update(kw)
    return p


def cache4(seqs=S, device="cpu", rows=torch.bfloat16, table=None, **kw):
    p = parts(seqs, device, **kw)
    return B.Cache4(p["k"], p["v"], p["ks"], p["vs"], p["pos"], p["n"], p["n"], N, block_table=table, rows=rows)


def step(start=S + 1, head_len=None, pos=T, device="cpu"):
    return B.Tokens(i32(pos, device=device), start=None if start is None else i32(start, device=device), max_tokens=2,
                    head_len=None if head_len is None else i32(*head_len, device=device))


def rows(heads, tokens=T, device="cpu", dtype=torch.bfloat16):
    return torch.zeros((tokens, heads, 128), dtype=dtype, device=device)


def append(**kw):
    a = dict(cache=cache4(), tokens=step(), k=rows(H), v=rows(H), new=i32(S))
    a.update(kw)
    B.tri_append4(MODEL, a["cache"], 0, a["tokens"], a["k"], a["v"], a["new"], stream=STREAM)


def attend(**kw):
    a = dict(cache=cache4(), tokens=step(), q=rows(H * G), out=rows(H * G), ws=u8(256))
    a.update(kw)
    B.tri_attend4(MODEL, a["cache"], 0, a["tokens"], a["q"], a["out"], workspace=a["ws"], stream=STREAM)


def shared(**kw):
    a = dict(prefix=cache4(2), group=i32(3), cache=cache(), tokens=step(), q=rows(H * G), out=rows(H * G), ws=u8(256))
    a.update(kw)
    B.tri_attend4_shared(MODEL, a["prefix"], a["group"], a["cache"], 0, a["tokens"], a["q"], a["out"], workspace=a["ws"], stream=STREAM)


def pack(**kw):
    a = dict(src=cache(), dst=cache4(), budget=7, idx=i32(L, S, H, 7), cnt=i32(L, S, H), new=i32(S))
    a.update(kw)
    B.tri_pack4(MODEL, a["src"], a["dst"], a["budget"], a["idx"], a["cnt"], a["new"], stream=STREAM)


def unpack(**kw):
    a = dict(src=cache4(), dst=cache(), budget=7, idx=i32(L, S, H, 7), cnt=i32(L, S, H), new=i32(S))
    a.update(kw)
    B.tri_unpack4(MODEL, a["src"], a["dst"], a["budget"], a["idx"], a["cnt"], a["new"], stream=STREAM)


def test_caches():
    c = cache4()
    assert c.c.c.dtype == B.TRI_FP4 and c.c.c.stride_slot == 128 and c.c.c.stride_head == N * 128 and c.c.c.k_rotated == 1 and c.c.rows == B.TRI_BF16
    assert cache4(rows=torch.float32).c.rows == B.TRI_F32
    wide = u8(L, S, H, N, 2, 64)   # keys and values side by side
    assert cache4(k=wide[..., 0, :], v=wide[..., 1, :]).c.c.stride_slot == 256
    table = i32(S, 3)
    assert (lambda x: (x.block_size, x.max_blocks_per_seq, x.n_blocks))(cache4(table=table).c.c) == (N, 3, S)
    lead = (L, S, H, N)
    for bad in (dict(k=u8(*lead, 128)), dict(v=u8(L, S, H, N + 1, 64)), dict(k=torch.zeros((*lead, 64), dtype=torch.int8)), dict(ks=u8(*lead, 8)), dict(vs=u8(L, S, H, N, 8)[..., :4]),
                dict(ks=u8(*lead, 4).transpose(2, 3)), dict(pos=i32(L, S, H, N + 1)), dict(pos=torch.zeros(lead)), dict(k=u8(*lead, 64, device="meta")), dict(n=torch.zeros(S)), dict(n=i32(2 * S)[::2]),
                dict(n=i32(S, device="meta")), dict(pos=i32(*lead, device="meta"))):
        with pytest.raises(ValueError):
            cache4(**bad)
    with pytest.raises(ValueError):
        cache4(table=i32(S, 6)[:, ::2])
    with pytest.raises(TypeError):
        cache4(rows=torch.float16)


def test_caches_that_are_smaller_than_said():
    p = parts()
    arrays = [p[n] for n in ("k", "v", "ks", "vs", "pos")]
    assert B.Cache4(*arrays, i32(S - 1), i32(S - 1), N - 1).n_seqs == S - 1
    for n, cur, most, table in ((S, S - 1, N, None), (S + 1, S + 1, N, None), (S, S, N + 1, None), (S, S, N, i32(S - 1, 3)), (S, S, N, i32(3 * S))):
        with pytest.raises(ValueError):
            B.Cache4(*arrays, i32(n), i32(cur), most, block_table=table)
    assert B.Cache4(*arrays, i32(S), i32(S), 3 * N, block_table=i32(S, 3)).c.c.max_seq_len == 3 * N


@pytest.mark.parametrize("entry", [append, attend, shared])
def test_arrays_of_the_step(lib, entry):
    entry(tokens=step(head_len=(L, S, H)))
    entry(tokens=step(start=S + 4))   # (the first S + 1 are read)
    assert len(lib.calls) == 2
    for bad in (step(start=S), step(start=1), step(head_len=(S, H)), step(head_len=(L, S + 1, H)), step(device="meta")):
        with pytest.raises(ValueError):
            entry(tokens=bad)
    assert len(lib.calls) == 2


def test_rows_are_of_the_cache_s_type(lib):
    for entry, heads, fields in ((append, H, ("k", "v")), (attend, H * G, ("q", "out"))):
        entry(cache=cache4(rows=torch.float32), **{f: rows(heads, dtype=torch.float32) for f in fields})
        for f in fields:
            for bad in (rows(heads, dtype=torch.float32), rows(heads, T + 1), rows(heads + 1), rows(heads, device="meta")):
                with pytest.raises((TypeError, ValueError)):
                    entry(**{f: bad})
    assert len(lib.calls) == 2
    with pytest.raises(ValueError):
        append(k=rows(H), v=rows(2 * H)[:, :H])   # other strides
    for bad in (i32(S - 1), torch.zeros(S, dtype=torch.int64), i32(2 * S)[::2], i32(S, device="meta")):
        with pytest.raises((TypeError, ValueError)):
            append(new=bad)
    assert len(lib.calls) == 2


@pytest.mark.parametrize("entry", [pack, unpack])
def test_slots(lib, entry):
    entry()
    entry(idx=None, cnt=None, new=None)
    entry(idx=i32(L * S * H * 7))
    assert len(lib.calls) == 3
    for bad in (dict(idx=i32(L, S, H, 6)), dict(idx=torch.zeros((L, S, H, 7), dtype=torch.int64)), dict(idx=i32(L, S, H, 14)[..., ::2]), dict(cnt=i32(S, H)), dict(cnt=i32(L, S, H, device="meta")),
                dict(new=i32(S - 1)), dict(new=torch.zeros(S)), dict(dst=(cache if entry is unpack else cache4)(device="meta"))):
        with pytest.raises((TypeError, ValueError)):
            entry(**bad)
    assert len(lib.calls) == 3


def test_workspaces_groups_and_devices(lib):
    for bad in (u8(1).expand(1 << 20), u8(512)[::2], u8(256, device="meta")):
        for entry in (attend, shared):
            with pytest.raises(ValueError):
                entry(ws=bad)
    for bad in (dict(group=i32(2)), dict(group=i32(6)[::2]), dict(group=torch.zeros(3)), dict(group=i32(3, device="meta")), dict(prefix=cache4(2, device="meta"))):
        with pytest.raises(ValueError):
            shared(**bad)
    assert not lib.calls
