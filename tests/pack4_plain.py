"""Caches of 4 bits in 64 bits from their definition (include/tri.h), and serve_plain's cases with such caches.  Test infrastructure."""
import numpy as np
import torch

import serve_plain as P

D = P.D
NUMBERS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LEAST, MOST = -124, 125   # powers of two of scales


def encode(x):
    """x [..., D] float64 -> (4-bit numbers uint8 [..., 64], scale bytes uint8 [..., 4]): the nearest number is looked for among all."""
    g = np.asarray(x, dtype=np.float64).reshape(*x.shape[:-1], 4, 32)
    a = np.abs(g).max(-1)
    odd = ~np.isfinite(a) | (a >= 2.0 ** 128)
    a = np.where(odd, 0.0, a)
    e = np.full(a.shape, MOST)
    for p in range(MOST, LEAST - 1, -1):   # the least power with a <= 7 scales
        fits = a <= 7.0 * 2.0 ** p
        if not fits.any():
            break
        e[fits] = p
    with np.errstate(invalid="ignore"):
        t = np.abs(g) / np.ldexp(1.0, e)[..., None]
    code = np.zeros(g.shape, dtype=np.uint8)
    best = np.abs(t - NUMBERS[0])
    for i in range(1, 8):
        d = np.abs(t - NUMBERS[i])
        nearer = (d < best) | ((d == best) & (i % 2 == 0))   # of two as near the even code
        code[nearer], best = i, np.where(nearer, d, best)
    code[np.signbit(g)] |= 8
    code[odd] = 0
    code = code.reshape(*x.shape)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(odd, 255, e + 127).astype(np.uint8)


def decode(code, scale):
    n = np.stack([code & 15, code >> 4], axis=-1).reshape(*code.shape[:-1], 4, 32)
    unit = np.where(scale == 255, np.nan, np.ldexp(1.0, np.clip(scale.astype(np.int64), 0, 254) - 127))
    return (np.where(n & 8, -1.0, 1.0) * NUMBERS[n & 7] * unit[..., None]).reshape(*code.shape[:-1], D)


def same_codes(got, want):
    """Whether two arrays of 4-bit numbers are equal, a zero's sign aside (an element within rounding of zero has either)."""
    z = lambda c: np.where((c & 15) == 8, c & 0xf0, c)   # noqa: E731
    y = lambda c: np.where((c >> 4) == 8, c & 0x0f, c)   # noqa: E731
    return np.array_equal(y(z(got)), y(z(want)))


def pack(cache, layers, layer, device, decoded=True):
    """A serve_plain.Case's cache dict with its keys and values in 4 bits: k4, v4, ks4, vs4 on the device (what lies beyond the lengths is no number); k and v become what these stand for."""
    fields = {}
    for f in ("k", "v"):
        code, scale = encode(cache[f])
        if decoded:
            cache[f] = decode(code, scale)
        fields[f + "4"], fields[f + "s4"] = code, scale
    dead = np.arange(cache["cap"])[None, :] >= np.asarray(cache["total"])[:, None]
    for name, x in fields.items():
        x[np.broadcast_to(dead[:, None], x.shape[:3])] = 255
        if cache["table"] is not None:
            block = cache["pos_gpu"].shape[3]
            S, H, mb = x.shape[0], x.shape[1], cache["cap"] // block
            y = np.full((cache["pos_gpu"].shape[1], H, block) + x.shape[3:], 255, dtype=np.uint8)
            y[cache["table"].reshape(-1)] = np.moveaxis(x.reshape((S, H, mb, block) + x.shape[3:]), 1, 2).reshape((S * mb, H, block) + x.shape[3:])
            x = y
        t = torch.zeros((layers,) + x.shape, dtype=torch.uint8, device=device)
        t[layer] = torch.from_numpy(np.ascontiguousarray(x)).to(device)
        cache[name] = t
    return cache


def descriptor(B, case, cache, lens=None, cur=None):
    n = cache["lens_gpu"] if lens is None else lens
    return B.Cache4(cache["k4"], cache["v4"], cache["ks4"], cache["vs4"], cache["pos_gpu"], n, n if cur is None else cur, cache["cap"], block_table=cache["table_gpu"], rows=case.dtype)


class Case(P.Case):
    """serve_plain.Case whose own cache (or, with a prefix, whose prefix) is held in 4 bits."""

    def __init__(self, *args, **kw):
        super().__init__(*args, stored_rotated=True, **kw)
        pack(self.packed(), self.layers, self.layer, self.device)

    def packed(self):
        return self.own if self.prefix is None else self.prefix


def attend(B, c, q=None, out=None, scale=None, causal=True, tokens=None, stream=None, desc=None, ws=None):
    """tri_attend4, or tri_attend4_shared where the case has a prefix."""
    q = c.q_gpu if q is None else q
    out = torch.full_like(c.q_gpu, 9.0) if out is None else out
    tokens = tokens or c.step(B)
    model, packed = c.model(B), desc or descriptor(B, c, c.packed())
    own = None if c.prefix is None else c.descriptor(B, c.own)
    if ws is None:
        ws = torch.full((max(256, B.tri_attend4_workspace_size(model, packed, tokens, own)),), 255, dtype=torch.uint8, device=c.device)
    kw = dict(scale=scale, causal=causal, workspace=ws, stream=stream)
    if own is None:
        B.tri_attend4(model, packed, c.layer, tokens, q, out, **kw)
    else:
        group = torch.from_numpy(c.groups).to(c.device)
        B.tri_attend4_shared(model, packed, group, own, c.layer, tokens, q, out, **kw)
    return out
