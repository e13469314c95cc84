"""The operators on a KV cache held in 4 bits whose speed is measured: what a program calls for every layer of every step.

  append   tri_append4: the step's new keys and values to the end of every sequence's cache, rotated by position on the way and rounded to 4 bits;
           then tri_unpack4 of that cache, so that what was written is seen
  pack     tri_pack4: the keys that a compression keeps (or all) of a cache in full precision, into one of 4 bits; then tri_unpack4 of that
  read     tri_unpack4: a cache of 4 bits back into one in full precision, as the next compression's scores want it
  attend   tri_attend4: the step's queries over the cache of 4 bits -- one token per sequence (decoding), a few, or a chunk of a prompt
  shared   tri_attend4_shared: the same for sequences with caches of their own in full precision behind prefixes held in 4 bits, read once for all

The format: a row of 128 elements is 64 bytes of 4-bit numbers (bit 3 the sign, bits 0 to 2 one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; even
dimensions in the low halves of the bytes) and a scale byte b for every 32 of them, which stands for 2^(b - 127), 255 for "not a number".  Of 32 elements of
largest magnitude a, the scale is the least power of two, 2^-124 to 2^125, with a <= 7 scales; an element is the nearest number that there is, the one of even code
where two are as near.  Keys are rotated before they are rounded, exactly: the 4-bit number is that of the rotated element, not of a rounding of it.

A case is one layer but where it says otherwise.  Geometries, lengths and the base of the rotation are those of this repository's configurations (8 KV
heads x 4 or 8 query heads of 128; caches of 2176 to 131072 keys; theta 1e6) or lie between them.  Keys and queries are complex centres per
head and band (magnitude lognormal, phase uniform) with noise of 0.3 of the magnitude, queries at half that scale, values unit Gaussians.
"scattered" caches are what evictions in place leave: slots in random order, at random positions, other ones for every head.

Fields: n, n_min are the most and the least cached keys of a sequence before the step, tokens, tok_min its new tokens; given says whether the step's q and k rows (or
a packed cache's source) are pre- or post-RoPE, appended whether the cache holds the new tokens' own keys already, block is the page size (0: contiguous), keep the
slots kept per head (0: all), prefix the shared keys of each of `groups` groups of sequences.
"""
import math

import torch

D, F = 128, 64
THETA = 1e6


def _case(name, op, **kw):
    c = dict(name=name, op=op, layers=1, seqs=1, kv_heads=8, group=4, n=2176, n_min=2176, tokens=1, tok_min=1, dtype="bf16", pairs="half",
             given="pre", appended=True, order="dense", block=0, causal=True, keep=0, prefix=0, groups=1)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one sequence, in the middle of a window of 128 since the last compression: the smallest there is, latency only
        _case("append_one", "append", n=63, n_min=63),
        # the prompts of four requests at once, ragged, in pages of 16
        _case("append_prompts", "append", seqs=4, n=0, n_min=0, tokens=8192, tok_min=700, block=16, pairs="interleaved"),
        # after a compression: the 2048 kept keys of 2176, pre-RoPE, in four layers of eight sequences, into pages of 16
        _case("pack_kept", "pack", layers=4, seqs=8, keep=2048, block=16, pairs="interleaved"),
        # fp32, post-RoPE: whole caches of three sequences, odd lengths and heads
        _case("pack_f32", "pack", seqs=3, kv_heads=5, n=4099, n_min=1, dtype="f32", given="post"),
        # one layer of one sequence at the steady state, read back to be scored
        _case("read_one", "read", order="scattered"),
        # sixteen ragged sequences in pages of 64, two layers
        _case("read_paged", "read", layers=2, seqs=16, n=8192, n_min=100, block=64),
        # decoding at the steady state of a compressed cache: budget + window, scattered
        _case("attend_one", "attend", order="scattered", pairs="interleaved"),
        # decoding for a serving engine's ragged batch in pages of 16
        _case("attend_paged", "attend", seqs=32, n=32768, n_min=1000, block=16),
        # chunks of two prompts over what is cached of them already
        _case("attend_chunk", "attend", seqs=2, n=7168, n_min=5000, tokens=1024, tok_min=900, given="post", block=64),
        # fp32, a few tokens per sequence (drafted ones being verified), odd sizes
        _case("attend_f32", "attend", seqs=3, kv_heads=2, group=3, n=4099, n_min=1, tokens=3, tok_min=1, dtype="f32", pairs="interleaved"),
        # eight samples of one prompt whose cache was compressed; the samples' own caches are short
        _case("shared_small", "shared", seqs=8, n=130, n_min=0, order="scattered", prefix=2048, pairs="interleaved"),
        # a batch of 64 behind one long system prompt, in pages of 16
        _case("shared_batch", "shared", seqs=64, n=1024, n_min=5, block=16, prefix=32768, given="post"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "pack", "read", "attend", "attend", "shared"])
    c = _case("", op, kv_heads=rng.choice([1, 2, 4, 5, 8, 8, 8]), group=rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
              pairs=rng.choice(["half", "interleaved"]), given=rng.choice(["pre", "post"]),
              block=rng.choice([0, 0, 16, 16, 1, 8, 32, 64, 256]), order=rng.choice(["dense", "dense", "scattered"]), causal=rng.random() < 0.8)
    del c["name"]
    c["seqs"] = _log(rng, 1, 256)
    most = 131072 * 8
    if op == "append":
        c["n"] = _log(rng, 1, 512) - 1
        c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 1, 8192)
        most = 18000 * 8
    elif op in ("pack", "read"):
        c["layers"], c["tokens"] = rng.choice([1, 1, 2, 4]), 0
        c["n"] = _log(rng, 1, 32768)
        most = 4 * 8 * 2176 * 8 if op == "pack" else most
        if op == "pack":
            c["keep"] = rng.choice([0, _log(rng, 1, c["n"] + 1)])
    elif op == "attend":
        c["n"] = _log(rng, 1, 131072)
        c["tokens"] = 1 if rng.random() < 0.5 else _log(rng, 1, 1024)
        c["appended"] = rng.random() < 0.85
    else:
        c["seqs"] = _log(rng, 2, 256)
        c["n"] = _log(rng, 1, 1025) - 1
        c["tokens"] = 1 if rng.random() < 0.8 else rng.randint(1, 8)
        c["prefix"] = _log(rng, 100, 65536)
        c["groups"] = min(rng.choice([1, 1, 1, 2, 3]), c["seqs"])
    c["n_min"] = c["n"] if rng.random() < 0.4 else rng.randint(0, c["n"])
    c["tok_min"] = c["tokens"] if rng.random() < 0.5 else rng.randint(min(1, c["tokens"]), c["tokens"])
    # no dearer than the largest listed ones: cached keys, and products of query rows with keys
    heads = c["kv_heads"] * c["layers"] * (4 if c["dtype"] == "f32" else 1)
    while c["seqs"] > c["groups"] and c["seqs"] * (c["n"] + c["tokens"]) * heads > most:
        c["seqs"] //= 2
    c["seqs"] = max(c["seqs"], c["groups"])
    while c["seqs"] * (c["n"] + c["tokens"]) * heads > most:
        c["n"], c["tokens"] = c["n"] // 2, max(min(1, c["tokens"]), c["tokens"] // 2)
    rows = c["seqs"] * c["tokens"] * c["group"] * heads
    while op in ("attend", "shared") and rows * (c["n"] + c["tokens"] + c["prefix"]) > 200e6:
        if c["tokens"] > 8:
            c["tokens"] //= 2
        else:
            c["n"], c["prefix"] = c["n"] // 2, c["prefix"] // 2
        rows = c["seqs"] * c["tokens"] * c["group"] * heads
    c["n_min"], c["tok_min"] = min(c["n_min"], c["n"]), min(c["tok_min"], c["tokens"])
    return c


# ---------------------------------------------------------------------------------------------------------------- inputs


def _spread(lo, hi, count):
    """`count` whole numbers over [lo, hi], the first of them hi: the golden ratio's multiples."""
    return [hi - int((hi - lo + 0.999) * ((s * 0.6180339887498949) % 1.0)) for s in range(count)]


def _lengths(c):
    """Cached keys before the step, and new tokens, of every sequence."""
    new = _spread(c["tok_min"], c["tokens"], c["seqs"]) if c["op"] in ("append", "attend", "shared") else [0] * c["seqs"]
    return _spread(c["n_min"], c["n"], c["seqs"]), new


def _groups(c):
    """The first sequence of every group of sequences with a prefix of its own."""
    return [g * c["seqs"] // c["groups"] for g in range(c["groups"] + 1)]


def _gen(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((int(seed) * 1000003 + tag) & 0x7FFFFFFFFFFF)
    return g


def _join(re, im, pairs):
    """Bands (re, im) [..., F] -> head vectors [..., D]."""
    return torch.cat([re, im], dim=-1) if pairs == "half" else torch.stack([re, im], dim=-1).flatten(-2)


def _split(x, pairs):
    return (x[..., :F], x[..., F:]) if pairs == "half" else (x[..., 0::2], x[..., 1::2])


def _rows(c, seed, tag, shape, heads, scale):
    """Pre-RoPE rows [*shape, heads, D] around the heads' centres."""
    g = _gen(seed, tag)
    mag = torch.exp(torch.randn(heads, F, generator=g, device="cuda"))
    ph = torch.rand(heads, F, generator=g, device="cuda") * (2 * math.pi)
    sd = mag * (0.3 / math.sqrt(2.0))
    re, im = (mag * f(ph) + sd * torch.randn(*shape, heads, F, generator=g, device="cuda") for f in (torch.cos, torch.sin))
    return _join(re, im, c["pairs"]) * scale


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _rotate(x, pos, pairs):
    """x [..., D] turned by pos [...], in the type of x; angles in 64 bits."""
    w = THETA ** (torch.arange(F, device=x.device, dtype=torch.float64) * (-2.0 / D))
    a = pos.double()[..., None] * w
    cos, sin = torch.cos(a).to(x.dtype), torch.sin(a).to(x.dtype)
    re, im = _split(x, pairs)
    return _join(re * cos - im * sin, re * sin + im * cos, pairs)


def _encode(x):
    """x [..., D] -> its 4-bit numbers, two to a byte [..., 64], and scale bytes [..., 4].  All steps are exact in the type of x."""
    g = x.unflatten(-1, (4, 32))
    a = g.abs().amax(dim=-1)
    m, k = torch.frexp(a)
    e = torch.where(m <= 0.875, k - 3, k - 2).clamp(-124, 125)
    t = torch.ldexp(g, -e[..., None]).abs()
    code = ((t > 0.25).byte() + (t >= 0.75).byte() + (t > 1.25).byte() + (t >= 1.75).byte() + (t > 2.5).byte() + (t >= 3.5).byte() + (t > 5.0).byte())
    code = (code + 8 * torch.signbit(g).byte()).flatten(-2)
    odd = ~torch.isfinite(a)
    return code[..., 0::2] + 16 * code[..., 1::2], torch.where(odd, 255, e + 127).byte()


def _pages(c, seed, tag, S, cap, block):
    """A block table in random order, and how slots [L][S][H][cap](...) become pages [L][blocks][H][block](...)."""
    if not block:
        return None, lambda x: x.contiguous()
    mb = cap // block
    order = torch.randperm(S * mb, generator=_gen(seed, tag), device="cuda")

    def paged(x):
        y = x.unflatten(3, (mb, block)).transpose(2, 3).flatten(1, 2)
        out = torch.empty(y.shape, dtype=y.dtype, device=y.device)
        out[:, order] = y
        return out
    return order.view(S, mb).to(torch.int32).contiguous(), paged


def _cache(c, seed, tag, lens, new, base, order, block, rotated, packed):
    """A cache of all layers with lens[s] + new[s] keys, what lies beyond them not a number; `packed`: in 4 bits.
    Positions begin at base[s]; the last new[s] keys are the step's own, behind all others."""
    S, H, L = len(lens), c["kv_heads"], c["layers"]
    total = [a + b for a, b in zip(lens, new)]
    cap = max(1, max(total))
    span = 4 if order == "scattered" else 1
    if block:
        cap = -(-cap // block) * block
    slot = torch.arange(cap, device="cuda", dtype=torch.int64)
    n_old, n_all, first = (torch.tensor(x, device="cuda")[:, None, None] for x in (lens, total, base))
    g = _gen(seed, tag + 5)
    if order == "scattered":
        r = torch.rand(L, S, H, cap, generator=g, device="cuda").masked_fill(slot >= n_old, 2.0)
        pos = torch.argsort(torch.argsort(r, dim=3), dim=3) * span + torch.randint(0, span, (L, S, H, cap), generator=g, device="cuda")
    else:
        pos = slot.expand(L, S, H, cap)
    pos = (torch.where(slot < n_old, pos, n_old * span + (slot - n_old)) + first).to(torch.int32)
    k = _rows(c, seed, tag, (L, S, cap), H, 1.0).transpose(2, 3)
    if rotated:
        k = _rotate(k, pos, c["pairs"])
    v = torch.randn(L, S, H, cap, D, generator=g, device="cuda")
    gone = (slot >= n_all)[..., None]
    k, v = k.masked_fill(gone, float("nan")), v.masked_fill(gone, float("nan"))
    table, paged = _pages(c, seed, tag + 6, S, cap, block)
    x = dict(pos=paged(pos), table=table, cap=cap, block=block, lens=torch.tensor(total, device="cuda", dtype=torch.int32))
    if packed:
        for f, y in (("k", k), ("v", v)):
            code, scale = _encode(y)
            x[f], x[f + "s"] = paged(code), paged(scale)
    else:
        x["k"], x["v"] = paged(k.to(_dtype(c))), paged(v.to(_dtype(c)))
    return x


def _inputs(c, seed):
    dt, S, H, G, L, op = _dtype(c), c["seqs"], c["kv_heads"], c["group"], c["layers"], c["op"]
    lens, new = _lengths(c)
    first = _groups(c)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    T = start[-1]
    i32 = dict(device="cuda", dtype=torch.int32)
    span = 4 if c["order"] == "scattered" else 1
    base = [c["prefix"] * span] * S
    pos = torch.tensor([base[s] + lens[s] * span + i for s in range(S) for i in range(new[s])], **i32)
    st = dict(c=c, start=torch.tensor(start, **i32), pos=pos, most=max(new), T=T)
    if op in ("append", "pack", "read"):
        if op == "pack":
            src = st["source"] = _cache(c, seed, 700, lens, new, base, c["order"], c["block"], c["given"] == "post", False)
            keep = c["keep"] or src["cap"]
            cap = keep if not c["block"] else -(-keep // c["block"]) * c["block"]
            st["keep"] = keep
            if c["keep"]:
                count = src["lens"].clamp(max=keep)[None, :, None].expand(L, S, H)
                r = torch.rand(L, S, H, src["cap"], generator=_gen(seed, 710), device="cuda")
                r = r.masked_fill(torch.arange(src["cap"], device="cuda") >= src["lens"][:, None, None], 2.0)
                pick = torch.argsort(r, dim=3)[..., :keep]
                if pick.shape[3] < keep:
                    pick = torch.nn.functional.pad(pick, (0, keep - pick.shape[3]))
                live = torch.arange(keep, device="cuda") < count[..., None]
                idx = torch.where(live, pick, src["cap"]).sort(dim=3).values
                st["idx"], st["count"] = torch.where(live, idx, 0).to(torch.int32).contiguous(), count.to(torch.int32).contiguous()
            table, paged = _pages(c, seed, 720, S, cap, c["block"])
            empty = lambda w, t: paged(torch.zeros((L, S, H, cap) + w, dtype=t, device="cuda"))  # noqa: E731
            st["cache"] = dict(k=empty((64,), torch.uint8), v=empty((64,), torch.uint8), ks=empty((4,), torch.uint8), vs=empty((4,), torch.uint8), pos=empty((), torch.int32),
                               table=table, cap=cap, block=c["block"], lens=src["lens"].clamp(max=keep))
            st["after"] = st["cache"]["lens"]
        else:
            st["cache"] = _cache(c, seed, 100, lens, new, base, c["order"], c["block"], True, True)
            st["after"] = st["cache"]["lens"]
        if op == "append":
            st["before"] = torch.tensor(lens, **i32)
            # rows of the fused projection's output: q, then k, then v of every token
            qkv = torch.zeros(T, (G + 2) * H, D, device="cuda", dtype=dt)
            k = _rows(c, seed, 200, (T,), H, 1.0)
            qkv[:, G * H:(G + 1) * H] = (_rotate(k, pos[:, None].expand(T, H), c["pairs"]) if c["given"] == "post" else k).to(dt)
            qkv[:, (G + 1) * H:] = torch.randn(T, H, D, generator=_gen(seed, 210), device="cuda").to(dt)
            st["k_new"], st["v_new"] = qkv[:, G * H:(G + 1) * H], qkv[:, (G + 1) * H:]
        cap = st["cache"]["cap"]
        back = dict(cap=cap, block=0, table=None, lens=st["after"], pos=torch.full((L, S, H, cap), -1, **i32))
        back["k"], back["v"] = (torch.zeros((L, S, H, cap, D), dtype=dt, device="cuda") for _ in range(2))
        st["back"] = back
        return st
    q = _rows(c, seed, 300, (T,), G * H, 0.5)
    if c["given"] == "post":
        q = _rotate(q, pos[:, None].expand(T, G * H), c["pairs"])
    st["q"] = q.to(dt)
    own = new if c["appended"] else [0] * S
    if op == "attend":
        st["cache"] = _cache(c, seed, 100, lens, own, base, c["order"], c["block"], True, True)
    else:
        P = c["groups"]
        st["first"] = torch.tensor(first, **i32)
        st["cache"] = _cache(c, seed, 400, [c["prefix"]] * P, [0] * P, [0] * P, c["order"], c["block"], True, True)
        st["own"] = _cache(c, seed, 100, lens, own, base, c["order"], c["block"], True, False)
        st["most_group"] = max(start[first[g + 1]] - start[first[g]] for g in range(P))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:   # the descriptors, workspace and output that a program keeps from step to step
        from paper_2604_04921_amd import binding as B
        c, op = case, case["op"]
        st["B"] = B
        st["model"] = B.Model(c["layers"], c["kv_heads"] * c["group"], c["kv_heads"], D, THETA, [1],
                              pairs=B.TRI_PAIR_HALF if c["pairs"] == "half" else B.TRI_PAIR_INTERLEAVED)

        def packed(x, lens):
            return B.Cache4(x["k"], x["v"], x["ks"], x["vs"], x["pos"], lens, lens, x["cap"], block_table=x["table"], rows=_dtype(c))

        def full(x, rotated):
            return B.Cache(x["k"], x["v"], x["pos"], x["lens"], x["lens"], x["cap"], block_table=x["table"], k_rotated=rotated)
        st["desc"] = packed(st["cache"], st["cache"]["lens"])
        if op in ("append", "pack", "read"):
            st["back_desc"] = full(st["back"], True)
            if op == "append":
                st["desc_before"] = packed(st["cache"], st["before"])
            if op == "pack":
                st["source_desc"] = full(st["source"], c["given"] == "post")
            st["new_len"] = torch.empty_like(st["after"])
        if op in ("append", "attend", "shared"):
            st["tokens"] = B.Tokens(st["pos"], start=st["start"], max_tokens=st["most"], rotated=c["given"] == "post")
        if op in ("attend", "shared"):
            st["out"] = torch.empty_like(st["q"])
            st["own_desc"] = full(st["own"], True) if op == "shared" else None
            size = B.tri_attend4_workspace_size(st["model"], st["desc"], st["tokens"], st["own_desc"])
            st["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------------------- plain form


def _decode(code, scale, dtype):
    """4-bit numbers [..., 64] and scale bytes [..., 4] -> rows [..., D]."""
    n = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
    n = torch.cat([n, -n])
    pair = torch.stack([n.repeat(16), n.repeat_interleave(16)], dim=1)             # a byte's two numbers
    unit = torch.ldexp(torch.ones(256, device=code.device), torch.arange(256, device=code.device) - 127)
    unit[255] = float("nan")
    x = pair[code.int()].flatten(-2).unflatten(-1, (4, 32)) * unit[scale.int()][..., None]
    return x.flatten(-2).to(dtype)


def _slots_of(x, t):
    """What lies in a cache's slots in their order: [L][S][H][N](...)."""
    return t[:, x["table"].long()].transpose(2, 3).flatten(3, 4) if x["block"] else t


def _values(x, dtype):
    """Keys, values and positions of a cache of 4 bits, in slot order."""
    return [_decode(_slots_of(x, x[f]), _slots_of(x, x[f + "s"]), dtype) for f in ("k", "v")] + [_slots_of(x, x["pos"])]


def _plain_read(st):
    x, back = st["cache"], st["back"]
    k, v, pos = _values(x, back["k"].dtype)
    there = (torch.arange(x["cap"], device="cuda") < st["after"][:, None])[None, :, None, :]
    back["k"].copy_(torch.where(there[..., None], k, back["k"]))
    back["v"].copy_(torch.where(there[..., None], v, back["v"]))
    back["pos"].copy_(torch.where(there, pos, back["pos"]))
    return [back["k"], back["v"], back["pos"], st["after"]]


def _plain_append(st):
    c, x = st["c"], st["cache"]
    t = torch.arange(st["T"], device="cuda")
    s = torch.searchsorted(st["start"][1:].long().contiguous(), t, right=True)
    slot = (st["before"][s] + (t - st["start"][s])).long()
    k = st["k_new"].double()
    if c["given"] == "pre":
        k = _rotate(k, st["pos"][:, None].expand(k.shape[:2]), c["pairs"])
    where = s
    if c["block"]:
        where, slot = x["table"][s, slot // c["block"]].long(), slot % c["block"]
    for f, rows in (("k", k), ("v", st["v_new"].float())):
        code, scale = _encode(rows)
        x[f][0][where, :, slot], x[f + "s"][0][where, :, slot] = code, scale
    x["pos"][0][where, :, slot] = st["pos"][:, None].expand(st["T"], c["kv_heads"])
    st["after"] = st["before"] + (st["start"][1:] - st["start"][:-1])
    return _plain_read(st)


def _plain_pack(st):
    c, x, src = st["c"], st["cache"], st["source"]
    k, v, pos = (_slots_of(src, src[f]) for f in ("k", "v", "pos"))
    count = src["lens"].clamp(max=st["keep"])[None, :, None].expand(pos.shape[:3])
    if "idx" in st:
        idx, count = st["idx"].long(), st["count"]
        pos = pos.gather(3, idx)
        k, v = (y.gather(3, idx[..., None].expand(*idx.shape, D)) for y in (k, v))
    if c["given"] == "pre":
        k = _rotate(k.double(), pos, c["pairs"])
    n = pos.shape[3]
    there = torch.arange(n, device="cuda") < count[..., None]
    (kc, ks), (vc, vs) = _encode(k), _encode(v.float())
    for f, new in (("k", kc), ("ks", ks), ("v", vc), ("vs", vs), ("pos", pos)):
        old = _slots_of(x, x[f])[:, :, :, :n]
        new = torch.where(there.view(there.shape + (1,) * (new.dim() - 4)), new, old)
        if c["block"]:
            slot = torch.arange(n, device="cuda")
            page = x["table"].long()[:, slot // c["block"]]
            x[f][:, page, :, (slot % c["block"])] = new.permute(1, 3, 0, 2, *range(4, new.dim()))
        else:
            x[f][:, :, :, :n] = new
    st["after"] = count[0, :, 0].to(torch.int32)
    return _plain_read(st)


def _scores(c, q, qpos, there, x, k, v, pos):
    """Unnormalised attention of padded queries q [S][T][Hq][D] at qpos [S][T] (there: which exist) over a cache: the rows' highest score,
    sum of exponentials and weighted sum of values, [S][T][Hq](, D)."""
    T, H, G, N = q.shape[1], c["kv_heads"], c["group"], k.shape[2]
    valid = torch.arange(N, device=k.device) < x["lens"][:, None]
    k = torch.where(valid[:, None, :, None], k, 0.0)
    v = torch.where(valid[:, None, :, None], v, 0.0)
    rows = q.unflatten(2, (H, G)).permute(0, 2, 1, 3, 4).flatten(2, 3)             # [S][H][T * G][D]
    s = torch.matmul(rows, k.transpose(2, 3).contiguous()).unflatten(2, (T, G)) * (1.0 / math.sqrt(D))
    keep = valid[:, None, None, None, :] & there[:, None, :, None, None]
    if c["causal"]:
        keep = keep & (pos[:, :, None, None, :] <= qpos[:, None, :, None, None])
    s = torch.where(keep, s, -math.inf)
    m = s.amax(dim=-1, keepdim=True)
    p = torch.where(keep, torch.exp(s - torch.where(m == -math.inf, 0.0, m)), 0.0)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (T, G))
    back = [t.permute(0, 2, 1, 3, 4).flatten(2, 3) for t in (m, p.sum(dim=-1, keepdim=True), o)]
    return back[0][..., 0], back[1][..., 0], back[2]


def _parts(st, x, kvp, start, most):
    """_scores of the step's tokens over one cache, token by token: [T][Hq](, D).  start: the first token of every sequence of the cache."""
    c, T = st["c"], st["T"]
    idx = start[:-1, None].long() + torch.arange(most, device="cuda")
    there = idx < start[1:, None]
    idx = idx.clamp(max=T - 1)
    q = st["q"].float()
    if c["given"] == "pre":
        q = _rotate(q, st["pos"][:, None].expand(T, q.shape[1]), c["pairs"])
    parts = _scores(c, q[idx], st["pos"][idx], there, x, *(t[0] for t in kvp))
    t = torch.arange(T, device="cuda")
    s = torch.searchsorted(start[1:].long().contiguous(), t, right=True)
    return [p[s, t - start[s]] for p in parts]


def _plain_attend(st):
    x = st["cache"]
    if st["c"]["op"] == "attend":
        m, l, o = _parts(st, x, _values(x, torch.float32), st["start"], st["most"])
    else:
        y = st["own"]
        m, l, o = _parts(st, y, [_slots_of(y, y["k"]).float(), _slots_of(y, y["v"]).float(), _slots_of(y, y["pos"])], st["start"], st["most"])
        m2, l2, o2 = _parts(st, x, _values(x, torch.float32), st["start"][st["first"].long()], st["most_group"])
        both = torch.maximum(m, m2)
        both = torch.where(both == -math.inf, 0.0, both)
        a, b = torch.exp(m - both), torch.exp(m2 - both)
        l, o = a * l + b * l2, a[..., None] * o + b[..., None] * o2
    return [torch.where(l[..., None] > 0, o / l[..., None], 0.0).to(st["q"].dtype)]


def run(st):
    op = st["c"]["op"]
    if not own:
        return {"append": _plain_append, "pack": _plain_pack, "read": _plain_read}.get(op, _plain_attend)(st)
    B, c = st["B"], st["c"]
    if op == "attend":
        B.tri_attend4(st["model"], st["desc"], 0, st["tokens"], st["q"], st["out"], causal=c["causal"], workspace=st["ws"])
        return [st["out"]]
    if op == "shared":
        B.tri_attend4_shared(st["model"], st["desc"], st["first"], st["own_desc"], 0, st["tokens"], st["q"], st["out"], causal=c["causal"], workspace=st["ws"])
        return [st["out"]]
    x, back = st["cache"], st["back"]
    if op == "append":
        B.tri_append4(st["model"], st["desc_before"], 0, st["tokens"], st["k_new"], st["v_new"], st["new_len"])
    if op == "pack":
        B.tri_pack4(st["model"], st["source_desc"], st["desc"], st["keep"], st.get("idx"), st.get("count"), st["new_len"])
    B.tri_unpack4(st["model"], st["desc"], st["back_desc"], x["cap"])
    return [back["k"], back["v"], back["pos"], st["after"] if op == "read" else st["new_len"]]


def work(c):
    lens, new = _lengths(c)
    eb, H, L, G, T, op = 2 if c["dtype"] == "bf16" else 4, c["kv_heads"], c["layers"], c["group"], sum(new), c["op"]
    full, packed = 2 * D * eb + 4, 2 * (D // 2 + 4) + 4                            # bytes of a slot: key, value, position
    if op in ("append", "pack", "read"):
        slots = [n + t for n, t in zip(lens, new)]
        written = T * H
        if op == "pack":
            slots = [min(n, c["keep"] or n) for n in slots]
            written = sum(slots) * H * L
        elif op == "read":
            written = 0
        turned = written if c["given"] == "pre" else 0
        every = sum(slots) * H * L
        return dict(bytes=written * (full + packed) + (4 * written if c["keep"] else 0) + every * (packed + full), flops=turned * 6 * F + (written + every) * 2 * D)
    extra = new if c["appended"] else [0] * c["seqs"]
    own_keys, shared_keys = sum(lens) + sum(extra), c["prefix"] * c["groups"] * (op == "shared")
    pairs = 0
    for n, t, e in zip(lens, new, extra):
        pairs += t * (n + c["prefix"]) + ((t * (t + 1) // 2 if c["causal"] else t * t) if e else 0)
    pos = 0 if c["causal"] else 4
    keys = own_keys * (packed - pos) if op == "attend" else own_keys * (full - pos) + shared_keys * (packed - pos)
    return dict(bytes=keys * H + T * H * G * 2 * D * eb + 4 * T, flops=pairs * H * G * 4 * D + (T * H * G * 6 * F if c["given"] == "pre" else 0))


# ---------------------------------------------------------------------------------------------------------------- 64 bits


def _bands(x, pos, pairs):
    """Complex bands [..., F] of rows x [..., D], times e^(i omega pos) where pos is given."""
    x = x.double()
    z = torch.complex(x[..., :F].contiguous(), x[..., F:].contiguous()) if pairs == "half" else torch.view_as_complex(x.unflatten(-1, (F, 2)).contiguous())
    if pos is None:
        return z
    omega = torch.exp(torch.arange(F, device=x.device, dtype=torch.float64) * (-2.0 / D * math.log(THETA)))
    return z * torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos.double()[..., None] * omega)


def _turned(x, pos, pairs):
    z = _bands(x, pos, pairs)
    return torch.cat([z.real, z.imag], dim=-1) if pairs == "half" else torch.view_as_real(z).flatten(-2)


def _near(x):
    """What rows [..., D] in 64 bits read back as: in steps of 1/2, 1 or 2 scales, by magnitude."""
    g = x.unflatten(-1, (4, 32))
    a = g.abs().amax(dim=-1, keepdim=True)
    e = torch.where(a > 0, torch.ceil(torch.log2(a / 7.0)), -124.0)
    e = torch.where(a > 7.0 * torch.exp2(e), e + 1, e)                             # (where the logarithm's rounding crossed a whole number)
    e = torch.where((a <= 7.0 * torch.exp2(e - 1)) & (a > 0), e - 1, e).clamp(-124, 125)
    unit = torch.exp2(e)
    t = g / unit
    step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0))
    return (torch.round(t / step) * step).clamp(-6, 6).mul(unit).flatten(-2)       # (halves go to the even multiple)


def _held(x, s, n, layer=0, packed=True):
    """The first n keys, values and positions of sequence s, [H][n](...), in 64 bits, page by page."""
    def take(t):
        if not x["block"]:
            return t[layer, s, :, :n]
        return torch.cat(list(t[layer].index_select(0, x["table"][s, :max(1, -(-n // x["block"]))].long())), dim=1)[:, :n]
    k, v, pos = (take(x[f]) for f in ("k", "v", "pos"))
    if not packed:
        return k.double(), v.double(), pos
    got = []
    for code, scale in ((k, take(x["ks"])), (v, take(x["vs"]))):
        n4 = torch.stack([code & 15, code >> 4], dim=-1).flatten(-2).long()
        m = n4 & 7
        mag = torch.where(m < 2, m.double() * 0.5, (2 + (m & 1)).double() * torch.exp2((m >> 1).double() - 2))
        got.append((torch.where(n4 > 7, -mag, mag).unflatten(-1, (4, 32)) * torch.exp2(scale.double() - 127)[..., None]).flatten(-2))
    return got[0], got[1], pos


def exact(case, seed):
    c = case
    st = _inputs(c, seed)
    lens, new = _lengths(c)
    H, G, op, x, start = c["kv_heads"], c["group"], c["op"], st["cache"], st["start"].tolist()
    if op in ("append", "pack", "read"):
        back = st["back"]
        k, v, pos, after = back["k"].double(), back["v"].double(), back["pos"].clone(), []
        for s in range(c["seqs"]):
            for l in range(c["layers"]):
                if op == "pack":
                    n = min(lens[s], st["keep"])
                    sk, sv, sp = _held(st["source"], s, lens[s], l, packed=False)
                    if "idx" in st:
                        pick = st["idx"][l, s, :, :n].long()
                        sk, sv, sp = (torch.stack([t[h, pick[h]] for h in range(H)]) for t in (sk, sv, sp))
                    sk = _turned(sk, sp, c["pairs"]) if c["given"] == "pre" else sk
                    k[l, s, :, :n], v[l, s, :, :n], pos[l, s, :, :n] = _near(sk[:, :n]), _near(sv[:, :n]), sp[:, :n]
                else:
                    n = lens[s]
                    k[l, s, :, :n], v[l, s, :, :n], pos[l, s, :, :n] = _held(x, s, n, l)
                if op == "append":
                    a, b = start[s], start[s + 1]
                    rows = st["k_new"][a:b].double()
                    rows = _turned(rows, st["pos"][a:b, None].expand(b - a, H), c["pairs"]) if c["given"] == "pre" else rows
                    k[l, s, :, n:n + b - a] = _near(rows).transpose(0, 1)
                    v[l, s, :, n:n + b - a] = _near(st["v_new"][a:b].double()).transpose(0, 1)
                    pos[l, s, :, n:n + b - a] = st["pos"][a:b]
                    n += b - a
            after.append(n)
        return [k, v, pos, torch.tensor(after, device="cuda", dtype=torch.int32)]
    first = _groups(c)
    out = torch.zeros(st["T"], H * G, D, device="cuda", dtype=torch.float64)
    zq = _bands(st["q"], st["pos"][:, None].expand(st["q"].shape[:2]) if c["given"] == "pre" else None, c["pairs"])
    y = st["own"] if op == "shared" else x
    total = y["lens"].tolist()
    for g in range(c["groups"]):
        head = _held(x, g, c["prefix"]) if op == "shared" else None
        for s in range(first[g], first[g + 1]):
            a, b = start[s], start[s + 1]
            k, v, pos = _held(y, s, total[s], packed=op == "attend")
            if head:
                k, v, pos = (torch.cat([p, t], dim=1) for p, t in zip(head, (k, v, pos)))
            if k.shape[1] == 0:
                continue
            zs = zq[a:b].unflatten(1, (H, G))                                     # [t][H][G][F]
            for h in range(H):
                u, zk = zs[:, h].flatten(0, 1), _bands(k[h], None, c["pairs"])
                w = (u.real @ zk.real.T.contiguous() + u.imag @ zk.imag.T.contiguous()) / math.sqrt(D)
                if c["causal"]:
                    w = w.masked_fill((pos[h][None, :] > st["pos"][a:b, None]).repeat_interleave(G, 0), -math.inf)
                w = torch.nan_to_num(torch.exp(w - torch.logsumexp(w, dim=1, keepdim=True)), nan=0.0)
                out[a:b, h * G:(h + 1) * G] = (w @ v[h]).unflatten(0, (b - a, G))
    return [out]


own = False
