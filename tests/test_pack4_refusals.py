"""What the entry points of 4-bit caches refuse, on the host before anything is enqueued (no GPU), and what they launch for good arguments: the library runs on a runtime that launches nothing
(fake_hip.cpp)."""
import ctypes
import json
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
ANY = 1 << 20   # an address: nothing is dereferenced
INVALID, UNSUPPORTED, WORKSPACE = -1, -2, -3

GOOD = dict(layers=2, heads=8, kv=2, theta=1e6, pairs=1, k=ANY, v=ANY, cpos=ANY, dtype=2, seqs=3, seq_len=ANY, cur_pos=ANY, n=1000, block=0, table=0, blocks=0,
            s_layer=1 << 20, s_seq=1 << 18, s_head=1 << 17, s_slot=128, rotated=1, n_blocks=0, ks=ANY, vs=ANY, rows=1, layer=1, tokens=5, most=3, start=ANY, pos=ANY, head_len=0, given=0,
            k_new=ANY, v_new=ANY, st=1024, sh=128, new_len=2 * ANY, q=ANY, out=2 * ANY, qst=1024, qsh=128, ost=1024, osh=128, scale=0.1, causal=1, ws=ANY, ws_bytes=1 << 40,
            group=ANY, budget=100, idx=ANY, cnt=3 * ANY, own=True,
            # the cache in full precision: source, destination or the sequences' own
            fk=5 * ANY, fv=6 * ANY, fpos=7 * ANY, fdtype=1, fseqs=3, fn=500, fblock=0, fblocks=0, ftable=0, frot=1, fslot=128, fn_blocks=0)


def call(T, lib, c):
    import numpy as np
    c = dict(GOOD, **c)
    offsets = np.arange(1, 3, dtype=np.int64)
    model = ctypes.byref(T.TriModel(c["layers"], c["heads"], c["kv"], c.get("head_dim", 128), c["theta"], c["pairs"], 2, offsets.ctypes.data_as(ctypes.c_void_p), 0, None))
    base = T.TriCache(c["k"], c["v"], c["cpos"], c["dtype"], c["seqs"], c["seq_len"], c["cur_pos"], c["n"], c["block"], c["table"], c["blocks"], c["s_layer"], c["s_seq"],
                      c["s_head"], c["s_slot"], 0, 0, 0, c["rotated"], c["n_blocks"])
    four = T.TriCache4(base, c["ks"], c["vs"], c["rows"])
    full = T.TriCache(c["fk"], c["fv"], c["fpos"], c["fdtype"], c["fseqs"], ANY, ANY, c["fn"], c["fblock"], c["ftable"], c["fblocks"], 1 << 20, 1 << 18, 1 << 17, c["fslot"], 0, 0, 0,
                      c["frot"], c["fn_blocks"])
    tok = T.TriTokens(c["tokens"], c["most"], c["start"], c["pos"], c["head_len"], c["given"])
    at = T.TriAttention(c["q"], c["out"], c["qst"], c["qsh"], c["ost"], c["osh"], c["scale"], c["causal"])
    four, full, tok, at = [None if c.get("no_" + n) else ctypes.byref(x) for n, x in (("cache", four), ("full", full), ("tokens", tok), ("attention", at))]
    e = c["entry"]
    if e == "append":
        return lib.tri_append4(model, four, c["layer"], tok, c["k_new"], c["v_new"], c["st"], c["sh"], c["new_len"], None)
    if e == "pack":
        return lib.tri_pack4(model, full, four, c["budget"], c["idx"], c["cnt"], c["new_len"], None)
    if e == "unpack":
        return lib.tri_unpack4(model, four, full, c["budget"], c["idx"], c["cnt"], c["new_len"], None)
    if e == "attend":
        return lib.tri_attend4(model, four, c["layer"], tok, at, c["ws"], c["ws_bytes"], None)
    if e == "size":
        return lib.tri_attend4_workspace_size(model, four, full if c["own"] else None, tok)
    return lib.tri_attend4_shared(model, four, c["group"], full, c["layer"], tok, at, c["ws"], c["ws_bytes"], None)


def answers(calls):
    import tempfile
    with tempfile.TemporaryDirectory(prefix="fake_hip_") as tmp:
        so = os.path.join(tmp, "libfake_hip.so")
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.cpp"), "-o", so], check=True)
        out = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
        assert out.returncode == 0, out.stderr
    return json.loads(out.stdout)


BAD_MODEL = [(dict(head_dim=64), UNSUPPORTED), (dict(heads=18), UNSUPPORTED), (dict(heads=7), INVALID), (dict(theta=1.0), INVALID), (dict(pairs=2), INVALID)]
BAD_FOUR = [(dict(no_cache=1), INVALID), (dict(k=0), INVALID), (dict(v=0), INVALID), (dict(cpos=0), INVALID), (dict(k=ANY + 8), INVALID), (dict(dtype=1), INVALID), (dict(dtype=0), INVALID),
            (dict(block=3, table=ANY, blocks=999), INVALID), (dict(block=16, table=0, blocks=999), INVALID), (dict(block=16, table=ANY, blocks=2), INVALID), (dict(s_slot=64), INVALID),
            (dict(s_slot=144), INVALID), (dict(s_head=-32), INVALID), (dict(s_head=(1 << 17) + 16), INVALID), (dict(s_slot=1 << 24), UNSUPPORTED), (dict(n_blocks=-1), INVALID), (dict(rotated=0), UNSUPPORTED),
            (dict(ks=0), INVALID), (dict(vs=0), INVALID), (dict(ks=ANY + 2), INVALID)]
BAD_LENGTHS = [(dict(seqs=0), INVALID), (dict(n=-1), INVALID), (dict(seq_len=0), INVALID), (dict(cur_pos=0), INVALID)]
BAD_FULL = [(dict(no_full=1), INVALID), (dict(fk=0), INVALID), (dict(fv=0), INVALID), (dict(fpos=0), INVALID), (dict(fdtype=2), INVALID), (dict(fdtype=7), INVALID), (dict(fblock=24), INVALID), (dict(fslot=100), INVALID),
            (dict(fn_blocks=-3), INVALID)]
BAD_TOKENS = [(dict(no_tokens=1), INVALID), (dict(tokens=-1), INVALID), (dict(start=0), INVALID), (dict(most=0), INVALID), (dict(most=6), INVALID), (dict(pos=0), INVALID), (dict(given=2), INVALID),
              (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(rows=2), INVALID), (dict(rows=-1), INVALID)]
BAD_ROWS = [(dict(q=0), INVALID), (dict(q=ANY + 4), INVALID), (dict(out=0), INVALID), (dict(out=ANY), INVALID), (dict(out=ANY + 2), INVALID), (dict(qst=1020), INVALID),
            (dict(qsh=-128), INVALID), (dict(ost=-1024), INVALID), (dict(osh=129), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(causal=2), INVALID), (dict(no_attention=1), INVALID)]
BAD_MOVE = [(dict(budget=0), INVALID), (dict(budget=-5), INVALID), (dict(fk=ANY), INVALID), (dict(fpos=ANY), INVALID), (dict(new_len=3 * ANY), INVALID), (dict(new_len=ANY), INVALID)]
CASES = {
    "append": BAD_MODEL + BAD_FOUR + BAD_LENGTHS + BAD_TOKENS + [(dict(k_new=0), INVALID), (dict(v_new=0), INVALID), (dict(k_new=ANY + 8), INVALID), (dict(st=1020), INVALID), (dict(sh=-128), INVALID),
                                                                 (dict(new_len=ANY), INVALID), (dict(head_len=2 * ANY), INVALID), (dict(seqs=40000), UNSUPPORTED),
                                                                 (dict(tokens=2 ** 31 - 1, kv=8), UNSUPPORTED)],
    "pack": BAD_MODEL + BAD_FOUR + BAD_FULL + BAD_MOVE + [(dict(fseqs=0), INVALID), (dict(fn=-1), INVALID), (dict(block=16, table=ANY, blocks=6, budget=97), INVALID),
                                                          (dict(fn=1 << 30, budget=1 << 30, block=1 << 20, table=ANY, blocks=1 << 11), UNSUPPORTED)],
    "unpack": BAD_MODEL + BAD_FOUR + BAD_LENGTHS + BAD_FULL + BAD_MOVE + [(dict(frot=0), UNSUPPORTED), (dict(fblock=16, ftable=ANY, fblocks=6, budget=97), INVALID),
                                                                          (dict(layers=60000, seqs=300, budget=1000), UNSUPPORTED)],
    "attend": BAD_MODEL + BAD_FOUR + BAD_LENGTHS + BAD_TOKENS + BAD_ROWS + [(dict(n=1 << 20, ws=0), WORKSPACE), (dict(n=1 << 20, ws=ANY + 64), WORKSPACE), (dict(n=1 << 20, ws_bytes=100), WORKSPACE),
                                                                            (dict(seqs=40000, tokens=40000), UNSUPPORTED), (dict(tokens=2 ** 31 - 1, most=1), UNSUPPORTED), (dict(n=2 ** 31 - 4096), UNSUPPORTED)],
    "shared": BAD_MODEL + BAD_FOUR + BAD_LENGTHS + BAD_TOKENS + BAD_ROWS + BAD_FULL + [(dict(group=0), INVALID), (dict(fdtype=0), INVALID), (dict(fseqs=0), INVALID), (dict(fn=-1), INVALID), (dict(ws=0), WORKSPACE),
                                                                                       (dict(rows=0), INVALID), (dict(fseqs=40000), UNSUPPORTED), (dict(n=2 ** 31 - 1), UNSUPPORTED)],
}


@pytest.fixture(scope="module")
def refused():
    calls = [dict(c, entry=e) for e, cases in CASES.items() for c, _ in cases]
    return dict(zip((json.dumps(c, sort_keys=True) for c in calls), answers(calls)))


@pytest.mark.parametrize("entry", list(CASES))
def test_refusals(refused, entry):
    for c, want in CASES[entry]:
        status, log = refused[json.dumps(dict(c, entry=entry), sort_keys=True)]
        assert status == want, (entry, c, status)
        assert "launch" not in log, (entry, c, log)   # nothing is enqueued


def launches(c):
    status, log = answers([c])[0]
    assert status == 0, (c, status)
    return [line.split() for line in log.splitlines() if line.startswith("launch")]


def test_what_good_calls_launch():
    assert len(launches(dict(entry="append"))) == 1
    assert len(launches(dict(entry="append", rows=0, st=1024))) == 1
    assert len(launches(dict(entry="append", k_new=0, v_new=0, tokens=0))) == 1   # the lengths alone
    assert len(launches(dict(entry="append", tokens=0, new_len=0))) == 0
    assert len(launches(dict(entry="append", start=0, tokens=3, pos=0))) == 1
    for entry in ("pack", "unpack"):
        assert len(launches(dict(entry=entry))) == 1
        assert len(launches(dict(entry=entry, idx=0, cnt=0, new_len=0))) == 1
        assert len(launches(dict(entry=entry, n=0, fn=0, idx=0, cnt=0, new_len=0))) == 0
        assert len(launches(dict(entry=entry, n=0, fn=0))) == 1   # the lengths alone
    assert len(launches(dict(entry="pack", fseqs=2, seqs=0, seq_len=0, cur_pos=0, n=-1, rows=9))) == 1   # (a destination's are not read)
    assert len(launches(dict(entry="attend", tokens=0))) == 0
    assert len(launches(dict(entry="attend", n=100, ws=0, ws_bytes=0))) == 1       # short rows: straight to the output
    assert len(launches(dict(entry="attend", n=100000))) == 2
    assert len(launches(dict(entry="shared"))) == 3
    assert len(launches(dict(entry="shared", seqs=1, group=0))) == 3


def test_launches_fit():
    """No launch asks for more threads than HIP takes (fewer than 2^32 on an axis)."""
    wide = dict(layers=1, layer=0, heads=32, kv=8, s_seq=1 << 20, st=4096, ost=4096, qst=4096)
    large = [dict(entry="append", seqs=3, tokens=(1 << 26) - 1, most=1 << 25), dict(entry="attend", seqs=256, most=8192, tokens=20000, n=32768), dict(entry="attend", seqs=2000, most=8192, tokens=20000, n=32768),
             dict(entry="attend", seqs=1, most=400000, tokens=400000, n=400000, rows=0), dict(entry="attend", seqs=8000, most=1, tokens=8000, n=131072), dict(entry="attend", seqs=256, most=100000, tokens=200000, n=32768),
             dict(entry="shared", fseqs=1000, most=1, tokens=700000, seqs=4, fn=64, n=1 << 20, rows=0, fdtype=0), dict(entry="pack", layers=60, fseqs=500, fn=32768, budget=32768), dict(entry="unpack", layers=60, seqs=1000, n=32768, budget=32768)]
    for c, (status, log) in zip(large, answers([dict(wide, **c) for c in large])):
        assert status in (0, UNSUPPORTED), (c, status)
        lines = [[int(w) for w in line.split()[2:6]] for line in log.splitlines() if line.startswith("launch")]
        assert (status == 0) == bool(lines), c
        assert all(x * block < 1 << 32 and y < 65536 and z < 65536 for x, y, z, block in lines), (c, log)


def test_workspace_size():
    # geometry alone: no cache's pointers are read, and what is invalid is said
    sizes = [a[0] for a in answers([dict(entry="size", k=0, v=0, cpos=0, ks=0, fk=0), dict(entry="size", n=100, own=False), dict(entry="size", most=0), dict(entry="size", no_cache=1),
                                    dict(entry="size", dtype=1), dict(entry="size", rows=2), dict(entry="size", fdtype=0)])]
    assert 0 < sizes[0] < 1 << 40 and sizes[1] == 0
    assert all(n == ctypes.c_size_t(-1).value for n in sizes[2:])


if __name__ == "__main__":
    import types
    fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
    fake.fake_log.restype = ctypes.c_char_p
    sys.modules["torch"] = types.ModuleType("torch")
    sys.path.insert(0, ROOT)
    from paper_2604_04921_amd import binding
    lib = binding.lib()
    results = []
    for one in json.load(sys.stdin):
        status = call(binding, lib, one)
        results.append((status, fake.fake_log().decode()))
    json.dump(results, sys.stdout)
