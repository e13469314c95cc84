"""Cases of attention over caches of 4 bits for serve_exact's tolerances (keys and values are what the 4-bit numbers stand for; queries and weights are held as include/tri.h says).  Test infrastructure."""
import numpy as np
import torch

import pack4_plain as K
import serve_exact as X
import serve_plain as P


def make(spec, device):
    c = K.Case(spec["seed"], spec["lens"], spec["tokens"], device=device, **spec["case"])
    kw = dict(spec["call"])
    cache = c.packed()
    if spec["absent"]:
        kw["gone"] = np.zeros((c.S, c.own["cap"]), dtype=bool)
        pool = cache["pos_gpu"].shape[1]
        for s, b, to in ((0, 0, -1), (0, 1, pool), (1, 1, 2 ** 31 - 1), (1, 0, -2 ** 31)):
            cache["table_gpu"][s, b] = to
            kw["gone"][s, b * c.block:(b + 1) * c.block] = True
    if spec["power"] is not None:   # keys of that power of two beside a third 2^-40 times as large and some zeros; queries the other way round
        by = np.ldexp(1.0, spec["power"] - 40 * (np.arange(cache["cap"]) % 3 == 1))
        by[::50] = 0
        cache["k"] *= by[:, None]
        K.pack(cache, c.layers, c.layer, device)
        c.q, c.q_gpu = np.ldexp(c.q, -spec["power"]), torch.ldexp(c.q_gpu.float(), torch.tensor(-spec["power"], device=device)).to(c.dtype)
    return X.Call(c, shared=c.prefix is not None, **kw)


def specs():
    """All cases; mutants: which wrong kernels (serve_exact.MUTANTS) a case has to tell from a right one."""
    seed = 900

    def spec(name, lens, tokens, mutants, call=None, absent=False, power=None, **case):
        nonlocal seed
        seed += 1
        return dict(name="%s %s" % ("f32" if case.get("dtype") == torch.float32 else "bf16", name), seed=seed, lens=lens, tokens=tokens, mutants=mutants, call=call or {}, absent=absent, power=power, case=case)
    for dtype in (torch.bfloat16, torch.float32):
        # lengths and numbers of rows: few (up to 8, 16, 32), many
        for tokens, old in (((1,), (0,)), ((1,), (700,)), ((1,), (2500,)), ((1,), (9000,)), ((1, 1, 1), (0, 1, 600)), ((2, 1, 4), (1000, 37, 256)), ((8, 1), (300, 5)), ((9,), (400,)), ((40, 1), (130, 600)),
                            ((130, 3, 77), (64, 5, 1300))):
            for i, (given, block) in enumerate(((False, 0), (False, 16), (True, 4), (True, 64))):
                mutants = ("zeros",) + (("q", "last") if max(old) else ()) + (("mask",) if max(tokens) > 1 else ()) + (("weights",) if max(tokens) <= 8 and max(old) > 100 else ())
                yield spec("%s+%s %s, pages of %d" % (old, tokens, ("widened", "as they are")[i // 2], block), old, tokens, mutants, dtype=dtype, given_rotated=given, block=block, pairs=i % 2,
                           order="scattered" if i == 1 else "dense", H=1 + i % 2)
        # group sizes
        for G in (1, 2, 3, 5, 6, 7, 8):
            for tokens in ((1, 1), (3, 1), (50, 9)):
                yield spec("G %d %s" % (G, tokens), (300, 65), tokens, ("zeros", "q", "last"), dtype=dtype, G=G, block=16, H=3)
        # far positions: turned rows decide the output
        for pos0 in (2 ** 31 - 2000, -2 ** 31, -500):
            for tokens in ((1,), (8,), (12,), (100,)):
                yield spec("from %d %s" % (pos0, tokens), (900,), tokens, ("zeros", "q"), dict(scale=0.3), dtype=dtype, pos0=pos0, pairs=1, theta=5e5, H=1)
        # large scores: what turned rows are held in decides the error
        for tokens, block, pairs in (((3,), 0, 0), ((8,), 16, 1), ((60,), 0, 0), ((60,), 64, 1), ((60,), 4, 0)):
            yield spec("large scores %s, pages of %d" % (tokens, block), (1500,), tokens, ("zeros", "q", "products"), dict(scale=0.3), dtype=dtype, block=block, pairs=pairs, H=1)
        # behind prefixes
        for tokens, prefix, groups, kw in (((1,) * 8, (300,), (0, 8), {}), ((1,) * 6, (500,), (0, 6), dict(block=16)), ((1,) * 4, (700, 90), (0, 2, 4), dict(G=8, block=64)), ((2, 1, 5, 1, 3, 2), (1000,), (0, 6), {}),
                                           ((40, 20, 1, 9), (70, 300), (0, 2, 4), dict(block=16)), ((1, 1, 1), (400, 0, 90), (0, 1, 2, 3), dict(block=16)), ((1, 2), (260, 30), (0, 0, 2), dict(block=4))):
            few = sum(tokens) * kw.get("G", 4) <= 32
            yield spec("%s behind %s, pages of %d" % (tokens, prefix, kw.get("block", 0)), (0, 40, 130, 17, 90, 64, 200, 33)[:len(tokens)], tokens,
                       ("zeros", "q", "prefix", "own") + (("weights",) if few else ()), dtype=dtype, prefix=prefix, groups=groups, **kw)
        # blocks that are not there, lengths per head, no mask
        for tokens in ((1, 1), (20, 9), (100, 40)):
            for block in (2, 16, 64):
                yield spec("%s without blocks of %d" % (tokens, block), (300, 140), tokens, ("zeros", "absent"), absent=True, dtype=dtype, block=block, layers=1, layer=0)
            yield spec("%s lengths per head" % (tokens,), (300, 150), tokens, ("zeros", "last"), dict(head_len=np.array([[300, 1, 17], [0, 150, 149]], dtype=np.int32)), dtype=dtype, H=3, block=16)
            yield spec("%s no mask" % (tokens,), (300, 150), tokens, ("zeros", "q"), dict(causal=False), dtype=dtype)
    # scales far apart
    for power in (-60, -20, 13, 20, 100):
        for tokens in ((3,), (60,)):
            for dtype in (torch.bfloat16, torch.float32):
                yield spec("2^%d %s" % (power, tokens), (700,), tokens, ("zeros", "q"), dict(scale=0.3), power=power, dtype=dtype, layers=1, layer=0)
