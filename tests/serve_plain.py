"""tri_append, tri_attend and tri_attend_shared in 64 bits from their definitions, and how far the kernels may be off.  Test infrastructure."""
import math

import numpy as np
import torch

D, F = 128, 64
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}   # half a step of a rounding, relative to the value


def bands(x, pairs):
    """[..., D] -> complex [..., F]; pairs 0: interleaved, 1: half-split."""
    return x[..., 0::2] + 1j * x[..., 1::2] if pairs == 0 else x[..., :F] + 1j * x[..., F:]


def rows(z, pairs):
    if pairs == 1:
        return np.concatenate([z.real, z.imag], axis=-1)
    return np.stack([z.real, z.imag], axis=-1).reshape(*z.shape[:-1], D)


def turn(x, pos, theta, pairs):
    """x [..., D] float64 rotated by pos [...] (angles reduced in extended precision)."""
    w = np.power(np.longdouble(theta), -2 * np.arange(F, dtype=np.longdouble) / D)
    a = np.asarray(pos, dtype=np.longdouble)[..., None] * w
    a = np.remainder(a, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64)
    return rows(bands(x, pairs) * np.exp(1j * a), pairs)


def attend(q, k, v, keep, scale):
    """q [R][D], k, v [N][D], keep [R][N] -> out [R][D], the most |scale q.k| could be off per unit of relative error, sum p |v|."""
    s = scale * (q @ k.T)
    reach = scale * (np.abs(bands(q, 1)) @ np.abs(bands(k, 1)).T) * 2.0   # |q_i k_i + q_j k_j| of a pair is at most this
    out, weight, off = np.zeros((len(q), D)), np.zeros((len(q), D)), np.zeros(len(q))
    for r in range(len(q)):
        n = keep[r]
        if not n.any():
            continue
        e = np.exp(s[r, n] - s[r, n].max())
        p = e / e.sum()
        out[r], weight[r], off[r] = p @ v[n], p @ np.abs(v[n]), reach[r, n].max()
    return out, weight, off


def bound(out, weight, off, dtype, roundings=0, turned=False):
    """roundings: how often q, k and p are rounded to bf16 on the way to a product (0: held in more bits, 2^-16 at least).
    A score is then off by off * (roundings of q and k, the rotation, fp32 sums), weights by twice that and by their own rounding."""
    u = HALF[dtype]
    held = 2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -22
    angle = (2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -21) if turned else 0.0
    d = off * (2 * held + roundings * 2.0 ** -8 + angle + 2.0 ** -19)
    return u * np.abs(out) + weight * (2 * d + 2 * held + (2.0 ** -7 if roundings else 0.0))[:, None] * (1 + u) + 1e-30


class Case:
    """A cache (contiguous or paged) with a step's tokens, on the host in float64 and on the GPU."""

    def __init__(self, seed, lens, tokens, H=2, G=4, dtype=torch.bfloat16, pairs=0, stored_rotated=True, given_rotated=False, block=0, order="dense",
                 theta=1e6, prefix=None, groups=None, layers=2, layer=1, room=0, pos0=0, appended=True, zero_q=False, device="cuda"):
        g = np.random.Generator(np.random.Philox(key=[seed, 77]))
        self.g, self.H, self.G, self.dtype, self.pairs, self.theta, self.block = g, H, G, dtype, pairs, theta, block
        self.stored_rotated, self.given_rotated, self.layers, self.layer, self.device = stored_rotated, given_rotated, layers, layer, device
        self.lens, self.tokens = list(lens), list(tokens)
        self.S, self.T = len(lens), int(sum(tokens))
        self.start = np.concatenate([[0], np.cumsum(tokens)]).astype(np.int32)
        span = 3 if order == "scattered" else 1
        self.prefix = None
        top = pos0
        if prefix is not None:
            top = pos0 + span * max(prefix) if prefix else pos0
            self.prefix = self._cache([int(n) for n in prefix], [0] * len(prefix), [pos0] * len(prefix), order, span, 0)
            self.groups = np.asarray([0, self.S] if groups is None else groups, dtype=np.int32)
        self.pos = np.concatenate([top + span * n + np.arange(t) for n, t in zip(lens, tokens)] + [np.zeros(0)]).astype(np.int32)
        self.own = self._cache(self.lens, self.tokens if appended else [0] * self.S, [top] * self.S, order, span, room)
        q = g.standard_normal((self.T, H * G, D)) * (0.0 if zero_q else 1.0)
        self.q = self.store(q)
        self.q_gpu = self.put(self.q)

    def store(self, x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(self.dtype).double().numpy()

    def put(self, x):
        return torch.from_numpy(np.ascontiguousarray(x)).to(self.dtype).to(self.device)

    def _cache(self, lens, new, base, order, span, room):
        g, H, S = self.g, self.H, len(lens)
        total = [a + b for a, b in zip(lens, new)]
        cap = max(max(total) + room, 1)
        if self.block:
            cap = -(-cap // self.block) * self.block
        k, v = self.store(g.standard_normal((S, H, cap, D))), self.store(g.standard_normal((S, H, cap, D)))
        pos = np.full((S, H, cap), -7, dtype=np.int32)
        for s in range(S):
            for h in range(H):
                old = np.sort(g.choice(span * lens[s], size=lens[s], replace=False)) if span > 1 else np.arange(lens[s])
                if order == "scattered":
                    g.shuffle(old)
                pos[s, h, :lens[s]] = base[s] + old
                pos[s, h, lens[s]:total[s]] = base[s] + span * lens[s] + np.arange(new[s])
        c = dict(k=k, v=v, pos=pos, total=total, cap=cap)
        dead = np.arange(cap)[None, :] >= np.asarray(total)[:, None]
        kg, vg = k.copy(), v.copy()
        kg[np.broadcast_to(dead[:, None], kg.shape[:3])] = np.nan
        vg[np.broadcast_to(dead[:, None], vg.shape[:3])] = np.inf
        c["table"] = None
        if self.block:
            mb = cap // self.block
            order_of = g.permutation(S * mb + 3)[:S * mb]   # (three blocks of the pool are nobody's)
            c["table"] = order_of.reshape(S, mb).astype(np.int32)

            def paged(x, fill):
                y = np.full((S * mb + 3, H, self.block) + x.shape[3:], fill, dtype=x.dtype)
                y[order_of] = np.moveaxis(x.reshape((S, H, mb, self.block) + x.shape[3:]), 1, 2).reshape((S * mb, H, self.block) + x.shape[3:])
                return y
            kg, vg, pg = paged(kg, np.nan), paged(vg, np.nan), paged(pos, 0)
        else:
            pg = pos
        def layered(x):
            t = torch.zeros((self.layers,) + tuple(x.shape), dtype=x.dtype, device=self.device)
            t[self.layer] = x
            return t
        c["k_gpu"], c["v_gpu"] = layered(self.put(kg)), layered(self.put(vg))
        c["pos_gpu"] = layered(torch.from_numpy(pg).to(self.device))
        c["table_gpu"] = None if c["table"] is None else torch.from_numpy(c["table"]).to(self.device)
        c["lens_gpu"] = torch.tensor(total, dtype=torch.int32, device=self.device)
        return c

    def descriptor(self, B, c, lens=None):
        n = c["lens_gpu"] if lens is None else lens
        return B.Cache(c["k_gpu"], c["v_gpu"], c["pos_gpu"], n, n, c["cap"], block_table=c["table_gpu"], k_rotated=self.stored_rotated)

    def model(self, B):
        return B.Model(self.layers, self.H * self.G, self.H, D, self.theta, [1], pairs=self.pairs)

    def step(self, B, **kw):
        one = all(t == 1 for t in self.tokens) and kw.pop("plain", False)
        return B.Tokens(torch.from_numpy(self.pos).to(self.device), start=None if one else torch.from_numpy(self.start).to(self.device),
                        max_tokens=max(self.tokens), rotated=self.given_rotated, **kw)

    def want(self, scale=None, causal=True, roundings=0, head_len=None):
        """(out [T][Hq][D], tolerance) in 64 bits."""
        scale = D ** -0.5 if scale is None else scale
        out, tol = np.zeros((self.T, self.H * self.G, D)), np.zeros((self.T, self.H * self.G, D))
        qt = self.q if self.given_rotated else turn(self.q, np.broadcast_to(self.pos[:, None], self.q.shape[:2]), self.theta, self.pairs)
        for s in range(self.S):
            a, b = self.start[s], self.start[s + 1]
            for h in range(self.H):
                parts = [(self.own, s, self.own["total"][s] if head_len is None else int(head_len[s][h]))]
                if self.prefix is not None:
                    p = int(np.searchsorted(self.groups, s, side="right")) - 1
                    parts.append((self.prefix, p, self.prefix["total"][p]))
                k = np.concatenate([c["k"][i, h, :n] for c, i, n in parts])
                v = np.concatenate([c["v"][i, h, :n] for c, i, n in parts])
                pos = np.concatenate([c["pos"][i, h, :n] for c, i, n in parts])
                if not self.stored_rotated:
                    k = turn(k, pos, self.theta, self.pairs)
                keep = np.repeat(pos[None, :] <= self.pos[a:b, None] if causal else np.ones((b - a, len(pos)), dtype=bool), self.G, axis=0)
                rows_q = qt[a:b, h * self.G:(h + 1) * self.G].reshape(-1, D)
                o, w, off = attend(rows_q, k, v, keep, scale)
                t = bound(o, w, off, self.dtype, roundings, turned=not (self.stored_rotated and self.given_rotated))
                out[a:b, h * self.G:(h + 1) * self.G] = o.reshape(b - a, self.G, D)
                tol[a:b, h * self.G:(h + 1) * self.G] = t.reshape(b - a, self.G, D)
        return out, tol
