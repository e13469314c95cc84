"""The serving operators on a KV cache whose speed is measured: what a program calls for every layer of every step.

  append   tri_append: the step's new keys and values (and their positions) to the end of every sequence's cache,
           contiguous or paged, the rotation by position applied on the way where the cache holds post-RoPE keys
  attend   tri_attend: the step's queries over the cache -- one token per sequence (decoding), a few, or a chunk of a
           prompt; keys stored before or after the rotation, slots in any order, masked by position
  shared   tri_attend_shared: the same for sequences that share long prefixes, held and read once

A case is one layer.  Geometries, lengths and the base of the rotation are those of this repository's configurations (8 KV
heads x 4 or 8 query heads of 128; caches of 2176 to 131072 keys; theta 1e6) or lie between them.  Keys and queries follow the
recipe of its synthetic workload -- a complex centre per head and band (magnitude lognormal, phase uniform), noise of 0.3 of
its magnitude --, queries at half that scale, so that scores spread by about two, and values are unit Gaussians.
"scattered" caches are what evictions in place leave: slots in random order, at random positions, other ones for every head.

Fields: n, n_min are the most and the least cached keys of a sequence before the step, tokens, tok_min its new tokens, stored and given
say whether cached keys / the step's q and k rows are pre- or post-RoPE, appended whether the cache holds the new tokens' own keys
already, block is the page size (0: contiguous), prefix the shared keys of each of `groups` groups of sequences.
"""
import math

import torch

D, F = 128, 64
THETA = 1e6


def _case(name, op, **kw):
    c = dict(name=name, op=op, seqs=1, kv_heads=8, group=4, n=2176, n_min=2176, tokens=1, tok_min=1, dtype="bf16", pairs="half", stored="post",
             given="pre", appended=True, order="dense", block=0, causal=True, prefix=0, groups=1)
    c.update(kw)
    return c


def listed():
    return [
        # one token of one sequence: the smallest append there is, latency only
        _case("append_one", "append"),
        # a decoding step of a large batch in pages of 16
        _case("append_batch", "append", seqs=256, n=300, n_min=17, block=16),
        # the prompts of four requests at once, ragged
        _case("append_prompts", "append", seqs=4, n=0, n_min=0, tokens=8192, tok_min=700, block=16, pairs="interleaved"),
        # fp32, pre-RoPE caches (a copy): three sequences, odd numbers of tokens and heads
        _case("append_f32", "append", seqs=3, kv_heads=5, n=77, n_min=1, tokens=1023, tok_min=1, dtype="f32", pairs="interleaved"),
        # decoding at the steady state of a compressed cache: budget + window, pre-RoPE, scattered
        _case("attend_one", "attend", stored="pre", order="scattered", pairs="interleaved"),
        # decoding for a serving engine's ragged batch in pages of 16
        _case("attend_paged", "attend", seqs=32, n=32768, n_min=1000, block=16),
        # one long context, eight query heads per KV head, keys stored before the rotation
        _case("attend_long", "attend", group=8, n=131072, n_min=131072, stored="pre"),
        # chunks of two prompts over what is cached of them already
        _case("attend_chunk", "attend", seqs=2, n=7168, n_min=5000, tokens=1024, tok_min=900, given="post", block=64),
        # fp32, a few tokens per sequence (drafted ones being verified), odd sizes
        _case("attend_f32", "attend", seqs=3, kv_heads=2, group=3, n=4099, n_min=1, tokens=3, tok_min=1, dtype="f32", stored="pre", pairs="interleaved"),
        # eight samples of one prompt whose cache was compressed; the samples' own caches are short
        _case("shared_small", "shared", seqs=8, n=130, n_min=0, stored="pre", order="scattered", prefix=2048, pairs="interleaved"),
        # a batch of 64 behind one long system prompt, in pages of 16
        _case("shared_batch", "shared", seqs=64, n=1024, n_min=5, block=16, prefix=32768, given="post"),
        # two prompts, 256 sequences, eight query heads per KV head: as many query rows as a prompt's chunk has
        _case("shared_many", "shared", seqs=256, group=8, n=511, n_min=0, prefix=16384, groups=2, given="post"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "shared"])
    c = _case("", op, kv_heads=rng.choice([1, 2, 4, 5, 8, 8, 8]), group=rng.choice([1, 2, 3, 4, 4, 5, 6, 7, 8, 8]), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]),
              pairs=rng.choice(["half", "interleaved"]), stored=rng.choice(["post", "post", "pre"]), given=rng.choice(["pre", "post"]),
              block=rng.choice([0, 0, 16, 16, 1, 8, 32, 64, 256]), order=rng.choice(["dense", "dense", "scattered"]), causal=rng.random() < 0.8)
    del c["name"]
    c["seqs"] = _log(rng, 1, 256)
    if op == "append":
        c["n"] = _log(rng, 1, 512) - 1
        c["tokens"] = 1 if rng.random() < 0.4 else _log(rng, 1, 8192)
        if c["stored"] == "pre":
            c["given"] = "pre"
        most = dict(elements=18000)
    elif op == "attend":
        c["n"] = _log(rng, 1, 131072)
        c["tokens"] = 1 if rng.random() < 0.5 else _log(rng, 1, 1024)
        c["appended"] = rng.random() < 0.85
        most = dict(elements=131072)
    else:
        c["seqs"] = _log(rng, 2, 256)
        c["n"] = _log(rng, 1, 1025) - 1
        c["tokens"] = 1 if rng.random() < 0.8 else rng.randint(1, 8)
        c["prefix"] = _log(rng, 100, 65536)
        c["groups"] = rng.choice([1, 1, 1, 2, 3])
        c["groups"] = min(c["groups"], c["seqs"])
        most = dict(elements=131072)
    c["n_min"] = c["n"] if rng.random() < 0.4 else rng.randint(0, c["n"])
    c["tok_min"] = c["tokens"] if rng.random() < 0.5 else rng.randint(1, c["tokens"])
    # no dearer than the largest listed ones: cached keys, and products of query rows with keys
    heads = c["kv_heads"] * (4 if c["dtype"] == "f32" else 1)
    while c["seqs"] > c["groups"] and c["seqs"] * (c["n"] + c["tokens"]) * heads > most["elements"] * 8:
        c["seqs"] //= 2
    c["seqs"] = max(c["seqs"], c["groups"])
    while c["seqs"] * (c["n"] + c["tokens"]) * heads > most["elements"] * 8:
        c["n"], c["tokens"] = c["n"] // 2, max(1, c["tokens"] // 2)
    rows = c["seqs"] * c["tokens"] * c["group"] * heads
    while op != "append" and rows * (c["n"] + c["tokens"] + c["prefix"]) > 200e6:
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
    return _spread(c["n_min"], c["n"], c["seqs"]), _spread(c["tok_min"], c["tokens"], c["seqs"])


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


def _centres(c, seed, tag, heads):
    g = _gen(seed, tag)
    mag = torch.exp(torch.randn(heads, F, generator=g, device="cuda"))
    ph = torch.rand(heads, F, generator=g, device="cuda") * (2 * math.pi)
    return mag * torch.cos(ph), mag * torch.sin(ph), mag


def _rows(c, seed, tag, shape, heads, scale, dt):
    """Pre-RoPE rows [*shape, heads, D] around the heads' centres."""
    re, im, mag = _centres(c, seed, tag, heads)
    g = _gen(seed, tag + 1)
    sd = mag * (0.3 / math.sqrt(2.0))
    x = re + sd * torch.randn(*shape, heads, F, generator=g, device="cuda")
    y = im + sd * torch.randn(*shape, heads, F, generator=g, device="cuda")
    return (_join(x, y, c["pairs"]) * scale).to(dt)


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _rotate(x, pos, pairs):
    """x [..., D] turned by pos [...]: angles in 64 bits, products in 32."""
    w = THETA ** (torch.arange(F, device=x.device, dtype=torch.float64) * (-2.0 / D))
    a = pos.double()[..., None] * w
    cos, sin = torch.cos(a).float(), torch.sin(a).float()
    re, im = _split(x.float(), pairs)
    return _join(re * cos - im * sin, re * sin + im * cos, pairs)


def _cache(c, seed, tag, lens, new, base, order, block):
    """A cache [1][S or blocks][H][N or block][D] of one layer with lens[s] + new[s] keys, what lies beyond them left as NaN.
    Positions begin at base[s]; the last new[s] keys are the step's own, behind all others."""
    dt, S, H = _dtype(c), len(lens), c["kv_heads"]
    total = [a + b for a, b in zip(lens, new)]
    cap = max(1, max(total))
    span = 4 if order == "scattered" else 1
    g = _gen(seed, tag + 5)
    if block:
        cap = -(-cap // block) * block
    slot = torch.arange(cap, device="cuda", dtype=torch.int64)
    n_old = torch.tensor(lens, device="cuda")[:, None]
    n_all = torch.tensor(total, device="cuda")[:, None]
    first = torch.tensor(base, device="cuda")[:, None]
    pos = slot[None, :].expand(S, cap)
    if order == "scattered":
        # a stride that is prime to the length puts every head's slots into an order of its own
        r = torch.rand(S, H, cap, generator=g, device="cuda").masked_fill(slot[None, None, :] >= n_old[:, :, None], 2.0)
        pos = torch.argsort(torch.argsort(r, dim=2), dim=2) * span + torch.randint(0, span, (S, H, cap), generator=g, device="cuda")
    else:
        pos = pos[:, None, :].expand(S, H, cap)
    pos = torch.where(slot[None, None, :] < n_old[:, :, None], pos, n_old[:, :, None] * span + (slot[None, None, :] - n_old[:, :, None]))
    pos = (pos + first[:, :, None]).to(torch.int32)
    k = _rows(c, seed, tag, (S, cap), H, 1.0, torch.float32).transpose(1, 2)
    if c["stored"] == "post":
        k = _rotate(k, pos, c["pairs"])
    k = k.to(dt)
    v = torch.randn(S, H, cap, D, generator=g, device="cuda").to(dt)
    gone = (slot[None, :] >= n_all)[:, None, :, None]
    k, v = k.masked_fill(gone, float("nan")), v.masked_fill(gone, float("nan"))
    table = None
    if block:
        mb = cap // block
        order_of = torch.randperm(S * mb, generator=g, device="cuda")
        table = order_of.view(S, mb).to(torch.int32).contiguous()

        def paged(x):
            y = x.unflatten(2, (mb, block)).transpose(1, 2).flatten(0, 1)   # [S * mb][H][block](...)
            out = torch.empty_like(y)
            out[order_of] = y
            return out.contiguous()[None]
        k, v, pos = paged(k), paged(v), paged(pos)
    else:
        k, v, pos = k.contiguous()[None], v.contiguous()[None], pos.contiguous()[None]
    return dict(k=k, v=v, pos=pos, table=table, cap=cap, block=block, lens=torch.tensor(total, device="cuda", dtype=torch.int32))


def _inputs(c, seed):
    dt, S, H, G = _dtype(c), c["seqs"], c["kv_heads"], c["group"]
    lens, new = _lengths(c)
    first = _groups(c)
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    T = start[-1]
    base = [c["prefix"] * (4 if c["order"] == "scattered" else 1)] * S
    span = 4 if c["order"] == "scattered" else 1
    i32 = dict(device="cuda", dtype=torch.int32)
    pos = torch.tensor([base[s] + lens[s] * span + i for s in range(S) for i in range(new[s])], **i32)
    st = dict(c=c, start=torch.tensor(start, **i32), pos=pos, most=max(new), T=T)
    if c["op"] == "append":
        room = _cache(c, seed, 100, lens, new, base, "dense", c["block"])   # what lies in the new slots is overwritten
        st["cache"] = dict(room, k=torch.nan_to_num(room["k"]), v=torch.nan_to_num(room["v"]), lens=torch.tensor(lens, **i32))
        # rows of the fused projection's output: q, then k, then v of every token
        qkv = torch.zeros(T, (G + 2) * H, D, device="cuda", dtype=dt)
        qkv[:, G * H:(G + 1) * H] = _rows(c, seed, 200, (T,), H, 1.0, torch.float32).to(dt)
        qkv[:, (G + 1) * H:] = torch.randn(T, H, D, generator=_gen(seed, 210), device="cuda").to(dt)
        if c["given"] == "post":
            qkv[:, G * H:(G + 1) * H] = _rotate(qkv[:, G * H:(G + 1) * H], pos[:, None].expand(T, H), c["pairs"]).to(dt)
        st["k_new"], st["v_new"] = qkv[:, G * H:(G + 1) * H], qkv[:, (G + 1) * H:]
        return st
    st["cache"] = _cache(c, seed, 100, lens, new if c["appended"] else [0] * S, base, c["order"], c["block"])
    q = _rows(c, seed, 300, (T,), G * H, 0.5, torch.float32)
    if c["given"] == "post":
        q = _rotate(q, pos[:, None].expand(T, G * H), c["pairs"])
    st["q"] = q.to(dt)
    if c["op"] == "shared":
        P = c["groups"]
        st["first"] = torch.tensor(first, **i32)
        st["prefix"] = _cache(c, seed, 400, [c["prefix"]] * P, [0] * P, [0] * P, c["order"], c["block"])
        st["most_group"] = max(start[first[g + 1]] - start[first[g]] for g in range(P))
    return st


def prepare(case, seed):
    st = _inputs(case, seed)
    if own:   # the descriptors, workspace and output that a program keeps from step to step
        from paper_2604_04921_amd import binding as B
        c, T = case, st["T"]
        st["B"] = B
        st["model"] = B.Model(1, c["kv_heads"] * c["group"], c["kv_heads"], D, THETA, [1],
                              pairs=B.TRI_PAIR_HALF if c["pairs"] == "half" else B.TRI_PAIR_INTERLEAVED)

        def descriptor(x):
            return B.Cache(x["k"], x["v"], x["pos"], x["lens"], x["lens"], x["cap"], block_table=x["table"], k_rotated=c["stored"] == "post")
        st["desc"] = descriptor(st["cache"])
        st["tokens"] = B.Tokens(st["pos"], start=st["start"], max_tokens=st["most"], rotated=c["given"] == "post")
        st["prefix_desc"] = descriptor(st["prefix"]) if c["op"] == "shared" else None
        if c["op"] == "append":
            st["new_len"] = torch.empty_like(st["cache"]["lens"])
        else:
            st["out"] = torch.empty_like(st["q"])
            size = B.tri_attend_workspace_size(st["model"], st["desc"], st["tokens"], st["prefix_desc"])
            st["ws"] = torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------------------- plain form


def _whole(x):
    """A cache's keys, values and positions in slot order: [S][H][N](...)."""
    k, v, pos = x["k"][0], x["v"][0], x["pos"][0]
    if x["block"]:
        table = x["table"].long()
        k, v, pos = (t[table].transpose(1, 2).flatten(2, 3) for t in (k, v, pos))
    return k, v, pos


def _scores(c, q, qpos, there, x):
    """Unnormalised attention of padded queries q [S][T][Hq][D] at qpos [S][T] (there: which exist) over a cache: the rows' highest score,
    sum of exponentials and weighted sum of values, [S][T][Hq](, D)."""
    k, v, pos = _whole(x)
    S, T, H, G, N = q.shape[0], q.shape[1], c["kv_heads"], c["group"], k.shape[2]
    valid = torch.arange(N, device=k.device) < x["lens"][:, None]
    k = torch.where(valid[:, None, :, None], k.float(), 0.0)
    v = torch.where(valid[:, None, :, None], v.float(), 0.0)
    if c["stored"] == "pre":
        k = _rotate(k, pos, c["pairs"])
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


def _parts(st, x, start, most):
    """_scores of the step's tokens over one cache, token by token: [T][Hq](, D).  start: the first token of every sequence of the cache."""
    c, T = st["c"], st["T"]
    idx = start[:-1, None].long() + torch.arange(most, device="cuda")
    there = idx < start[1:, None]
    idx = idx.clamp(max=T - 1)
    q = st["q"].float()
    if c["given"] == "pre":
        q = _rotate(q, st["pos"][:, None].expand(T, q.shape[1]), c["pairs"])
    parts = _scores(c, q[idx], st["pos"][idx], there, x)
    t = torch.arange(T, device="cuda")
    s = torch.searchsorted(start[1:].long().contiguous(), t, right=True)
    return [p[s, t - start[s]] for p in parts]


def _plain_append(st):
    c, x = st["c"], st["cache"]
    t = torch.arange(st["T"], device="cuda")
    s = torch.searchsorted(st["start"][1:].long().contiguous(), t, right=True)
    slot = (x["lens"][s] + (t - st["start"][s])).long()
    k = st["k_new"]
    if c["stored"] == "post" and c["given"] == "pre":
        k = _rotate(k, st["pos"][:, None].expand(k.shape[:2]), c["pairs"]).to(k.dtype)
    where = s
    if c["block"]:
        where, slot = x["table"][s, slot // c["block"]].long(), slot % c["block"]
    x["k"][0][where, :, slot] = k
    x["v"][0][where, :, slot] = st["v_new"]
    x["pos"][0][where, :, slot] = st["pos"][:, None].expand(st["T"], c["kv_heads"])
    return [x["k"], x["v"], x["pos"], x["lens"] + (st["start"][1:] - st["start"][:-1])]


def _plain_attend(st):
    m, l, o = _parts(st, st["cache"], st["start"], st["most"])
    if st["c"]["op"] == "shared":
        m2, l2, o2 = _parts(st, st["prefix"], st["start"][st["first"].long()], st["most_group"])
        both = torch.maximum(m, m2)
        both = torch.where(both == -math.inf, 0.0, both)
        a, b = torch.exp(m - both), torch.exp(m2 - both)
        l, o = a * l + b * l2, a[..., None] * o + b[..., None] * o2
    return [torch.where(l[..., None] > 0, o / l[..., None], 0.0).to(st["q"].dtype)]


def run(st):
    op = st["c"]["op"]
    if not own:
        return _plain_append(st) if op == "append" else _plain_attend(st)
    B = st["B"]
    if op == "append":
        x = st["cache"]
        B.tri_append(st["model"], st["desc"], 0, st["tokens"], st["k_new"], st["v_new"], st["new_len"])
        return [x["k"], x["v"], x["pos"], st["new_len"]]
    if op == "attend":
        B.tri_attend(st["model"], st["desc"], 0, st["tokens"], st["q"], st["out"], causal=st["c"]["causal"], workspace=st["ws"])
    else:
        B.tri_attend_shared(st["model"], st["prefix_desc"], st["first"], st["desc"], 0, st["tokens"], st["q"], st["out"], causal=st["c"]["causal"],
                            workspace=st["ws"])
    return [st["out"]]


def work(c):
    lens, new = _lengths(c)
    eb, H, T = 2 if c["dtype"] == "bf16" else 4, c["kv_heads"], sum(new)
    if c["op"] == "append":
        turned = c["stored"] == "post" and c["given"] == "pre"
        return dict(bytes=T * H * (4 * D * eb + 4) + 4 * T + 12 * c["seqs"], flops=T * H * 6 * F if turned else 0)
    extra = new if c["appended"] else [0] * c["seqs"]
    keys = sum(lens) + sum(extra) + c["prefix"] * c["groups"] * (c["op"] == "shared")
    pairs = 0
    for n, t, e in zip(lens, new, extra):
        pairs += t * (n + c["prefix"]) + ((t * (t + 1) // 2 if c["causal"] else t * t) if e else 0)
    turns = (T * H * c["group"] if c["given"] == "pre" else 0) + (keys * H if c["stored"] == "pre" else 0)
    return dict(bytes=keys * H * (2 * D * eb + (4 if c["causal"] or c["stored"] == "pre" else 0)) + T * H * c["group"] * 2 * D * eb + 4 * T,
                flops=pairs * H * c["group"] * 4 * D + turns * 6 * F)


# ---------------------------------------------------------------------------------------------------------------- 64 bits


def _bands(x, pos, pairs):
    """Complex bands [..., F] of rows x [..., D], times e^(i omega pos) where pos is given."""
    x = x.double()
    z = torch.complex(x[..., :F].contiguous(), x[..., F:].contiguous()) if pairs == "half" else torch.view_as_complex(x.unflatten(-1, (F, 2)).contiguous())
    if pos is None:
        return z
    omega = torch.exp(torch.arange(F, device=x.device, dtype=torch.float64) * (-2.0 / D * math.log(THETA)))
    return z * torch.polar(torch.ones((), dtype=torch.float64, device=x.device), pos.double()[..., None] * omega)


def _slots(x, s, n):
    """The first n keys, values and positions of sequence s, [H][n](...), page by page."""
    if not x["block"]:
        return [x[f][0, s, :, :n] for f in ("k", "v", "pos")]
    pages = x["table"][s, :-(-n // x["block"])].long()
    return [torch.cat([t for t in x[f][0].index_select(0, pages)], dim=1)[:, :n] if n else x[f][0, 0, :, :0] for f in ("k", "v", "pos")]


def exact(case, seed):
    c = case
    st = _inputs(c, seed)
    lens, new = _lengths(c)
    H, G, x = c["kv_heads"], c["group"], st["cache"]
    start = st["start"].tolist()
    if c["op"] == "append":
        k, v, pos = x["k"].double(), x["v"].double(), x["pos"].clone()
        rows = st["k_new"].double()
        if c["stored"] == "post" and c["given"] == "pre":
            z = _bands(rows, st["pos"][:, None].expand(rows.shape[:2]), c["pairs"])
            rows = torch.cat([z.real, z.imag], dim=-1) if c["pairs"] == "half" else torch.view_as_real(z).flatten(-2)
        for s in range(c["seqs"]):
            n, a, b = lens[s], start[s], start[s + 1]
            at = torch.arange(n, n + b - a, device="cuda")
            row = x["table"][s].long()[at // c["block"]] if c["block"] else torch.full_like(at, s)
            at = at % c["block"] if c["block"] else at
            for h in range(H):
                k[0, row, h, at], v[0, row, h, at], pos[0, row, h, at] = rows[a:b, h], st["v_new"][a:b, h].double(), st["pos"][a:b]
        return [k, v, pos, torch.tensor([n + t for n, t in zip(lens, new)], device="cuda", dtype=torch.int32)]
    first = _groups(c)
    out = torch.zeros(st["T"], H * G, D, device="cuda", dtype=torch.float64)
    zq = _bands(st["q"], st["pos"][:, None].expand(st["q"].shape[:2]) if c["given"] == "pre" else None, c["pairs"])
    total = x["lens"].tolist()
    for g in range(c["groups"]):
        head = _slots(st["prefix"], g, c["prefix"]) if c["op"] == "shared" else None
        zhead = _bands(head[0], head[2] if c["stored"] == "pre" else None, c["pairs"]) if head else None
        for s in range(first[g], first[g + 1]):
            a, b = start[s], start[s + 1]
            k, v, pos = _slots(x, s, total[s])
            zk = _bands(k, pos if c["stored"] == "pre" else None, c["pairs"])
            v = v.double()
            if head:
                zk, v, pos = torch.cat([zhead, zk], dim=1), torch.cat([head[1].double(), v], dim=1), torch.cat([head[2], pos], dim=1)
            if zk.shape[1] == 0:
                continue
            zs = zq[a:b].unflatten(1, (H, G))                                     # [t][H][G][F]
            for h in range(H):
                u = zs[:, h].flatten(0, 1)
                w = (u.real @ zk[h].real.T.contiguous() + u.imag @ zk[h].imag.T.contiguous()) / math.sqrt(D)
                if c["causal"]:
                    w = w.masked_fill((pos[h][None, :] > st["pos"][a:b, None]).repeat_interleave(G, 0), -math.inf)
                w = torch.nan_to_num(torch.exp(w - torch.logsumexp(w, dim=1, keepdim=True)), nan=0.0)
                out[a:b, h * G:(h + 1) * G] = (w @ v[h]).unflatten(0, (b - a, G))
    return [out]


own = False
