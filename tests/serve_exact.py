"""How far an attention kernel may be off its 64-bit value when it rounds what it says it rounds, and nothing else.  Test infrastructure.

Every rounding on the way to an output is taken as evenly distributed over what its type allows (half a step at most: variance a third of its square) and independent of the others, so that an output's error has a variance
that follows from the case's own scores and values:
  a score's error e moves the output by w (v - o) e, w being the key's weight, v its value and o the output; a weight's relative error r by w v r (the sum of weights is taken before they are rounded).
An element is allowed six standard deviations and the output's own rounding; all elements together (bf16) the root mean square of that rounding, which the 64-bit value says, and one standard deviation.
The second is what tells weights held in 16 bits from weights held in 8.

What is held (include/tri.h): bf16, up to 32 rows (tokens x query heads of the group) per KV head: 16 bits of turned queries and keys and of weights; more rows: 11 bits of turned queries and keys, at most 2^-25 of the row's
power of two, 8 bits of weights.  fp32: fp32.
"""
import numpy as np
import torch

import serve_plain as P

D = P.D
ANGLE = 2.0 ** -19   # of a turned element, relative to its pair: the hardware's sine and cosine


def kernel_of(c, rows):
    return "f32" if c.dtype == torch.float32 else "few" if rows <= 32 else "many"


HELD = {"f32": (2.0 ** -21, 2.0 ** -21), "few": (2.0 ** -16, 2.0 ** -16), "many": (2.0 ** -11, 2.0 ** -8)}   # turned queries and keys, weights
ANGLES = {"f32": 2.0 ** -22, "few": ANGLE, "many": ANGLE}


def unit(x):
    """The power of two that brings a row's largest element to [1, 2)."""
    most = np.abs(x).max(-1, keepdims=True)
    return np.exp2(np.floor(np.log2(np.where(most > 0, most, 1.0))))


def to_bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def to_f16(x, by):
    return (x / by).astype(np.float16).astype(np.float64) * by


class Call:
    """A Case and how it is called.  mutant: what a wrong kernel would do (see MUTANTS), for the checks of the checks."""

    def __init__(self, case, scale=None, causal=True, shared=False, head_len=None, gone=None):
        self.c, self.scale, self.causal, self.shared, self.head_len, self.gone = case, D ** -0.5 if scale is None else scale, causal, shared, head_len, gone

    def parts(self, s, h, mutant):
        c = self.c
        n = c.own["total"][s] if self.head_len is None else int(self.head_len[s][h])
        there = np.ones(n, dtype=bool)
        if self.gone is not None and mutant != "absent":
            there = ~self.gone[s, :n]
        own = (*(c.own[f][s, h, :n][there] for f in ("k", "v", "pos")), max(c.tokens) * c.G)
        if not self.shared:
            return [own]
        p = int(np.searchsorted(c.groups, s, side="right")) - 1
        m = c.prefix["total"][p]
        prefix = (*(c.prefix[f][p, h, :m] for f in ("k", "v", "pos")), c.T * c.G)
        return [own] if mutant == "prefix" else [prefix] if mutant == "own" else [own, prefix]

    def value(self, mutant=None, held=False):
        """(outputs in 64 bits, variance of an exact kernel's error).  held: with the roundings that a right kernel makes, before the output's own."""
        c = self.c
        out, var = np.zeros((c.T, c.H * c.G, D)), np.zeros((c.T, c.H * c.G, D))
        for s in range(c.S):
            a, b = c.start[s], c.start[s + 1]
            if a == b:
                continue
            rows_pos = np.repeat(c.pos[a:b], c.G)
            for h in range(c.H):
                q = c.q[a:b, h * c.G:(h + 1) * c.G].reshape(-1, D)
                if not c.given_rotated and mutant != "q":
                    q = P.turn(q, rows_pos, c.theta, c.pairs)
                score, score_var, held_p, vs = [], [], [], []
                for k, v, pos, rows in self.parts(s, h, mutant):
                    kind = kernel_of(c, rows)
                    if not c.stored_rotated and mutant != "k" and len(k):
                        k = P.turn(k, pos, c.theta, c.pairs)
                    sc, sv = self.scores(q, k, kind, mutant, held)
                    keep = pos[None] <= rows_pos[:, None] if self.causal and mutant != "mask" else np.ones(sc.shape, dtype=bool)
                    score.append(np.where(keep, sc, -np.inf))
                    score_var.append(sv)
                    held_p.append(np.full(len(k), HELD[kind][1]))
                    vs.append(v)
                sc, sv, hp, v = np.concatenate(score, 1), np.concatenate(score_var, 1), np.concatenate(held_p), np.concatenate(vs)
                if mutant == "last" and sc.shape[1]:
                    sc[:, -1] = -np.inf
                any_key = np.isfinite(sc).any(1) if sc.shape[1] else np.zeros(len(q), dtype=bool)
                if not any_key.any():
                    continue
                top = np.where(any_key, np.max(np.where(np.isfinite(sc), sc, -np.inf), 1), 0.0)[:, None]
                p = np.where(any_key[:, None], np.exp(sc - top), 0.0)
                total = np.where(any_key, p.sum(1), 1.0)[:, None]
                w = p / total
                rounded = mutant == "weights" or held
                if rounded:
                    p = np.where((hp == 2.0 ** -8)[None] | (mutant == "weights"), to_bf16(p), p)
                o = (p / total) @ v
                v2 = v ** 2
                ww = w ** 2
                a_v = (ww * sv)
                spread = a_v @ v2 - 2 * o * (a_v @ v) + o ** 2 * a_v.sum(1, keepdims=True)
                vv = np.maximum(spread, 0) + (ww * (hp ** 2 / 3 + 2.0 ** -40)) @ v2
                out[a:b, h * c.G:(h + 1) * c.G] = o.reshape(b - a, c.G, D)
                var[a:b, h * c.G:(h + 1) * c.G] = vv.reshape(b - a, c.G, D)
        return np.zeros_like(out) if mutant == "zeros" else out, var

    def scores(self, q, k, kind, mutant, held):
        c, rel = self.c, HELD[kind][0]
        turned_q, turned_k = not c.given_rotated, not c.stored_rotated
        f16 = kind == "many" and turned_q   # (keys are pre-RoPE only where queries are turned or given turned; either way the products run in fp16)
        f16 |= kind == "many" and turned_k
        if mutant == "products":            # turned rows as bf16 numbers
            q, k = to_bf16(q), to_bf16(k)
        elif held and f16 and len(k):
            uk = unit(k)
            q, k = to_f16(q, unit(q)), to_f16(k, np.where(np.abs(k).max(-1, keepdims=True) < 2.0 ** -6, uk, np.maximum(uk * 2.0 ** -15, 1.0)))
        e_q, e_k = (np.abs(q) * (rel if t else 0) for q, t in ((q, turned_q), (k, turned_k)))
        if f16 and len(k):
            e_q = np.maximum(np.abs(q) * 2.0 ** -11, 2.0 ** -25 * unit(q))
            most = np.abs(k).max(-1, keepdims=True)
            floor = 2.0 ** -25 * np.where(most == 0, 0, np.where(most < 2.0 ** -6, unit(k), np.maximum(unit(k), 1.0)))
            e_k = np.maximum(e_k, floor)
        sc = self.scale * (q @ k.T)
        var = (e_q ** 2 / 3) @ (k ** 2).T + (q ** 2) @ (e_k ** 2 / 3).T
        m2 = lambda x: P.bands(x, c.pairs).real ** 2 + P.bands(x, c.pairs).imag ** 2   # noqa: E731
        angle = (turned_q + turned_k) * ANGLES[kind] ** 2 / 3
        var = self.scale ** 2 * (var + (angle + 2.0 ** -40) * (m2(q) @ m2(k).T))
        return sc, var


MUTANTS = ("zeros", "q", "k", "mask", "prefix", "own", "last", "absent", "products", "weights")


def applies(call, mutant):
    """Whether a mutant computes something else in this call."""
    c = call.c
    if mutant == "q":
        return not c.given_rotated
    if mutant == "k":
        return not c.stored_rotated
    if mutant in ("prefix", "own"):
        return call.shared
    if mutant == "absent":
        return call.gone is not None
    if mutant == "mask":
        return call.causal
    if mutant in ("products", "weights"):
        return c.dtype == torch.bfloat16
    return True


def wrong(call, got, ref, var):
    """What is wrong with an output: a list of words, empty where nothing is."""
    u = P.HALF[call.c.dtype]
    off = got - ref
    bad = []
    if not np.all(np.abs(off) <= u * np.abs(ref) + 6 * np.sqrt(var) + 1e-30):
        worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, np.abs(off)) / (u * np.abs(ref) + 6 * np.sqrt(var) + 1e-30)), off.shape)
        bad.append("at %s %r, not %r: %.1f standard deviations of %.2g" % (worst, got[worst], ref[worst], np.abs(off[worst]) / np.sqrt(var[worst] + 1e-60), np.sqrt(var[worst])))
    if call.c.dtype == torch.bfloat16:
        own = np.sqrt(((to_bf16(ref) - ref) ** 2).mean())
        limit = own * (1 + 2 / np.sqrt(ref.size)) + np.sqrt(var.mean())
        rms = np.sqrt((off ** 2).mean())
        if not rms <= limit:
            bad.append("root mean square %.3g, not %.3g (%.3g of it the outputs' rounding)" % (rms, limit, own))
    return bad


def make(spec, device):
    """The Call that a spec describes, its caches on `device`."""
    c = P.Case(spec["seed"], spec["lens"], spec["tokens"], device=device, **spec["case"])
    kw = dict(spec["call"])
    if spec["absent"]:
        kw["gone"] = np.zeros((c.S, c.own["cap"]), dtype=bool)
        pool = c.own["k_gpu"].shape[1]
        for s, b, to in ((0, 0, -1), (0, 1, pool), (1, 1, 2 ** 31 - 1), (1, 0, -2 ** 31)):
            c.own["table_gpu"][s, b] = to
            kw["gone"][s, b * c.block:(b + 1) * c.block] = True
    if spec["power"] is not None:   # keys of that power of two beside a third 2^-40 times as large and some zeros; queries the other way round
        by = np.ldexp(1.0, spec["power"] - 40 * (np.arange(c.own["cap"]) % 3 == 1))
        by[::50] = 0
        c.own["k"] *= by[:, None]
        c.own["k_gpu"] = (c.own["k_gpu"].double() * torch.from_numpy(by).to(device)[:, None]).to(c.dtype)
        c.q, c.q_gpu = np.ldexp(c.q, -spec["power"]), torch.ldexp(c.q_gpu.float(), torch.tensor(-spec["power"], device=device)).to(c.dtype)
    return Call(c, **kw)


def specs():
    """All cases; mutants: which wrong kernels a case has to tell from a right one."""
    seed = 500

    def spec(name, lens, tokens, mutants, call=None, absent=False, power=None, **case):
        nonlocal seed
        seed += 1
        return dict(name="%s %s" % ("f32" if case.get("dtype") == torch.float32 else "bf16", name), seed=seed, lens=lens, tokens=tokens, mutants=mutants, call=call or {}, absent=absent, power=power, case=case)
    for dtype in (torch.bfloat16, torch.float32):
        # lengths and numbers of rows: few (up to 8, 16, 32), many
        for tokens, old in (((1,), (700,)), ((1,), (2500,)), ((1, 1, 1), (0, 1, 600)), ((2, 1, 4), (1000, 37, 256)), ((8, 1), (300, 5)), ((9,), (400,)), ((40, 1), (130, 600)), ((130, 3, 77), (64, 5, 1300))):
            for i, (stored, given, block) in enumerate(((False, False, 0), (True, False, 16), (True, True, 4))):
                mutants = ("zeros", "q", "k", "last") + (("mask",) if max(tokens) > 1 and i != 1 else ()) + (("weights",) if max(tokens) <= 8 and max(old) > 100 else ())
                yield spec("%s+%s %s" % (old, tokens, ("pre", "widened", "as they are")[i]), old, tokens, mutants, dtype=dtype, stored_rotated=stored, given_rotated=given, block=block, pairs=i % 2,
                           order="scattered" if i == 1 else "dense", H=1 + i % 2)
        # far positions: turned rows decide the output
        for pos0 in (2 ** 31 - 2000, -2 ** 31, -500):
            for tokens in ((1,), (8,), (12,), (100,)):
                yield spec("from %d %s" % (pos0, tokens), (900,), tokens, ("zeros", "q", "k", "products"), dict(scale=0.3), dtype=dtype, pos0=pos0, stored_rotated=False, pairs=1, theta=5e5, H=1)
        # large scores: what turned rows are held in decides the error
        for tokens, block, pairs in (((3,), 0, 0), ((8,), 16, 1), ((60,), 0, 0), ((60,), 64, 1), ((60,), 4, 0)):
            yield spec("large scores %s, pages of %d" % (tokens, block), (1500,), tokens, ("zeros", "q", "k", "products"), dict(scale=0.3), dtype=dtype, stored_rotated=False, block=block, pairs=pairs, H=1)
        # behind prefixes: both caches in one launch (few rows in either), in two
        for tokens, prefix, groups, kw in (((1,) * 8, (300,), (0, 8), {}), ((1,) * 6, (500,), (0, 6), dict(block=16)), ((1,) * 4, (700, 90), (0, 2, 4), dict(G=8, block=64)), ((2, 1, 5, 1, 3, 2), (1000,), (0, 6), {}),
                                           ((40, 20, 1, 9), (70, 300), (0, 2, 4), dict(block=16))):
            few = sum(tokens) * kw.get("G", 4) <= 32
            for stored in (False, True):
                yield spec("%s behind %s %s, pages of %d" % (tokens, prefix, "post" if stored else "pre", kw.get("block", 0)), (0, 40, 130, 17, 90, 64, 200, 33)[:len(tokens)], tokens,
                           ("zeros", "q", "prefix", "own") + (("weights",) if few else ()), dict(shared=True), dtype=dtype, prefix=prefix, groups=groups, stored_rotated=stored, **kw)
        # blocks that are not there, lengths per head, no mask
        for tokens in ((1, 1), (20, 9), (100, 40)):
            for block in (2, 16, 64):
                yield spec("%s without blocks of %d" % (tokens, block), (300, 140), tokens, ("zeros", "absent"), absent=True, dtype=dtype, block=block, layers=1, layer=0)
            yield spec("%s lengths per head" % (tokens,), (300, 150), tokens, ("zeros", "last"), dict(head_len=np.array([[300, 1, 17], [0, 150, 149]], dtype=np.int32)), dtype=dtype, H=3, block=16)
            yield spec("%s no mask" % (tokens,), (300, 150), tokens, ("zeros", "q", "k"), dict(causal=False), dtype=dtype, stored_rotated=False)
    # keys that fp16 does not hold
    for power in (-60, -20, 13, 20, 100):
        for tokens in ((3,), (60,)):
            for stored in (False, True):
                yield spec("2^%d %s %s" % (power, tokens, "post" if stored else "pre"), (700,), tokens, ("zeros", "q", "k"), dict(scale=0.3), power=power, layers=1, layer=0, stored_rotated=stored)
