"""What tri_append, tri_attend and tri_attend_shared refuse, on the host before anything is enqueued (no GPU), and what they launch for good arguments: the library runs on a
runtime that launches nothing (fake_hip.cpp)."""
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

GOOD = dict(layers=2, heads=8, kv=2, theta=1e6, pairs=1, k=ANY, v=ANY, cpos=ANY, dtype=1, seqs=3, seq_len=ANY, cur_pos=ANY, n=1000, block=0, table=0, blocks=0,
            s_layer=1 << 20, s_seq=1 << 18, s_head=1 << 17, s_slot=128, rotated=1, n_blocks=0, layer=1, tokens=5, most=3, start=ANY, pos=ANY, head_len=0, given=0,
            k_new=ANY, v_new=ANY, st=1024, sh=128, new_len=2 * ANY, q=ANY, out=2 * ANY, qst=1024, qsh=128, ost=1024, osh=128, scale=0.1, causal=1, ws=ANY, ws_bytes=1 << 40,
            prefix=True, group=ANY, pn=5000, pseqs=2, pdtype=1, pblock=0, pk=ANY, pn_blocks=0)


def call(T, lib, c):
    import numpy as np
    c = dict(GOOD, **c)
    offsets = np.arange(1, 3, dtype=np.int64)
    head_dim = c.get("head_dim", 128)
    model = ctypes.byref(T.TriModel(c["layers"], c["heads"], c["kv"], head_dim, c["theta"], c["pairs"], 2, offsets.ctypes.data_as(ctypes.c_void_p), 0, None))
    cache = T.TriCache(c["k"], c["v"], c["cpos"], c["dtype"], c["seqs"], c["seq_len"], c["cur_pos"], c["n"], c["block"], c["table"], c["blocks"], c["s_layer"], c["s_seq"],
                       c["s_head"], c["s_slot"], 0, 0, 0, c["rotated"], c["n_blocks"])
    pre = T.TriCache(c["pk"], ANY, ANY, c["pdtype"], c["pseqs"], ANY, ANY, c["pn"], c["pblock"], ANY, 1 << 20, 1 << 20, 1 << 18, 1 << 17, 128, 0, 0, 0, 1, c["pn_blocks"])
    tok = T.TriTokens(c["tokens"], c["most"], c["start"], c["pos"], c["head_len"], c["given"])
    at = T.TriAttention(c["q"], c["out"], c["qst"], c["qsh"], c["ost"], c["osh"], c["scale"], c["causal"])
    cache, pre, tok, at = [None if c.get("no_" + n) else ctypes.byref(x) for n, x in (("cache", cache), ("prefix", pre), ("tokens", tok), ("attention", at))]
    if c["entry"] == "append":
        return lib.tri_append(model, cache, c["layer"], tok, c["k_new"], c["v_new"], c["st"], c["sh"], c["new_len"], None)
    if c["entry"] == "attend":
        return lib.tri_attend(model, cache, c["layer"], tok, at, c["ws"], c["ws_bytes"], None)
    if c["entry"] == "size":
        return lib.tri_attend_workspace_size(model, pre if c["prefix"] else None, cache, tok)
    return lib.tri_attend_shared(model, pre, c["group"], cache, c["layer"], tok, at, c["ws"], c["ws_bytes"], None)


def answers(calls):
    import tempfile
    with tempfile.TemporaryDirectory(prefix="fake_hip_") as tmp:
        so = os.path.join(tmp, "libfake_hip.so")
        subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.cpp"), "-o", so], check=True)
        out = subprocess.run([sys.executable, os.path.abspath(__file__), so], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
        assert out.returncode == 0, out.stderr
    return json.loads(out.stdout)


BAD_CACHE = [(dict(k=0), INVALID), (dict(v=0), INVALID), (dict(cpos=0), INVALID), (dict(k=ANY + 8), INVALID), (dict(dtype=2), INVALID), (dict(seqs=0), INVALID),
             (dict(n=-1), INVALID), (dict(seq_len=0), INVALID), (dict(cur_pos=0), INVALID), (dict(block=3, table=ANY, blocks=999), INVALID),
             (dict(block=16, table=0, blocks=999), INVALID), (dict(block=16, table=ANY, blocks=2), INVALID), (dict(s_slot=64), INVALID), (dict(s_slot=132), INVALID),
             (dict(s_head=-8), INVALID), (dict(n_blocks=-1), INVALID), (dict(layer=-1), INVALID), (dict(layer=2), INVALID), (dict(head_dim=64), UNSUPPORTED),
             (dict(heads=18), UNSUPPORTED), (dict(heads=7), INVALID), (dict(theta=1.0), INVALID), (dict(pairs=2), INVALID), (dict(no_cache=1), INVALID)]
BAD_TOKENS = [(dict(no_tokens=1), INVALID), (dict(tokens=-1), INVALID), (dict(start=0), INVALID), (dict(most=0), INVALID), (dict(most=6), INVALID), (dict(pos=0), INVALID),
              (dict(given=2), INVALID), (dict(seqs=40000), UNSUPPORTED)]
BAD_ROWS = [(dict(q=0), INVALID), (dict(q=ANY + 4), INVALID), (dict(out=0), INVALID), (dict(out=ANY), INVALID), (dict(out=ANY + 2), INVALID), (dict(qst=1020), INVALID),
            (dict(qsh=-128), INVALID), (dict(ost=-1024), INVALID), (dict(osh=129), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
            (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(causal=2), INVALID), (dict(no_attention=1), INVALID)]
CASES = {
    "append": BAD_CACHE + BAD_TOKENS + [(dict(k_new=0), INVALID), (dict(v_new=0), INVALID), (dict(k_new=ANY + 8), INVALID), (dict(st=1020), INVALID), (dict(sh=-128), INVALID),
                                        (dict(new_len=ANY), INVALID), (dict(head_len=2 * ANY), INVALID), (dict(given=1, rotated=0), UNSUPPORTED),
                                        (dict(tokens=2 ** 31 - 1), UNSUPPORTED)],
    "attend": BAD_CACHE + BAD_TOKENS + BAD_ROWS + [(dict(n=1 << 20, ws=0), WORKSPACE), (dict(n=1 << 20, ws=ANY + 64), WORKSPACE), (dict(n=1 << 20, ws_bytes=100), WORKSPACE),
                                                   (dict(tokens=2 ** 31 - 1, most=1), UNSUPPORTED)],
    "shared": BAD_CACHE + BAD_TOKENS + BAD_ROWS + [(dict(no_prefix=1), INVALID), (dict(group=0), INVALID), (dict(pdtype=0), INVALID), (dict(pseqs=0), INVALID),
                                                   (dict(pk=0), INVALID), (dict(pn=-1), INVALID), (dict(pblock=24), INVALID), (dict(pn_blocks=-3), INVALID), (dict(ws=0), WORKSPACE)],
}


def test_refusals():
    calls = [(dict(c, entry=e), want) for e, cases in CASES.items() for c, want in cases]
    for (c, want), (status, log) in zip(calls, answers([c for c, _ in calls])):
        assert status == want, (c, status)
        assert "launch" not in log, (c, log)   # nothing is enqueued


def launches(c):
    status, log = answers([c])[0]
    assert status == 0, (c, status)
    return [line.split() for line in log.splitlines() if line.startswith("launch")]


def test_what_good_calls_launch():
    assert len(launches(dict(entry="append"))) == 1
    assert len(launches(dict(entry="append", k_new=0, v_new=0, tokens=0))) == 1   # the lengths alone
    assert len(launches(dict(entry="append", tokens=0, new_len=0))) == 0
    assert len(launches(dict(entry="append", start=0, tokens=3, pos=0))) == 1
    assert len(launches(dict(entry="attend", tokens=0))) == 0
    assert len(launches(dict(entry="attend", n=100, ws=0, ws_bytes=0))) == 1       # short rows: straight to the output
    assert len(launches(dict(entry="attend", n=100000))) == 2
    assert len(launches(dict(entry="shared"))) == 2                # few workgroups: both caches at once, and the joining
    assert len(launches(dict(entry="shared", rotated=0))) == 3     # (of two layouts)
    assert len(launches(dict(entry="shared", tokens=50, most=30))) == 3


def test_workspace_size():
    # geometry alone: no cache's pointers are read, and what is invalid is said
    sizes = [a[0] for a in answers([dict(entry="size", k=0, v=0, cpos=0, pk=0), dict(entry="size", n=100, prefix=False), dict(entry="size", most=0),
                                    dict(entry="size", no_cache=1)])]
    assert 0 < sizes[0] < 1 << 40 and sizes[1] == 0
    assert sizes[2] == sizes[3] == ctypes.c_size_t(-1).value


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
