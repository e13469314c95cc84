"""A serving loop on the library: one prompt, several samples of its answer.

The prompt is prefilled in chunks (tri_append, tri_attend), its cache is compressed once to a budget of keys per head
(tri_build_centers, tri_compress_step) and shared by all samples; every sample's own tokens go to a paged cache of its own
(tri_append) and attend to both (tri_attend_shared).  The model is a toy (random projections, no vocabulary): what it shows is which call
goes where, and which lengths each one reads.

    python examples/serve_loop.py [--prompt 1500] [--budget 256] [--samples 6] [--tokens 20]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_04921_amd import binding as T

LAYERS, HQ, HKV, D, THETA, HIDDEN, BLOCK = 2, 8, 2, 128, 1e6, 256, 16
DEV, BF16 = "cuda", torch.bfloat16


class Toy:
    """Per layer: a fused projection to q, k and v, and one back."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        w = lambda *s: (torch.randn(*s, generator=g, device=DEV) / math.sqrt(s[0])).to(BF16)   # noqa: E731
        self.qkv = [w(HIDDEN, (HQ + 2 * HKV) * D) for _ in range(LAYERS)]
        self.back = [w(HQ * D, HIDDEN) for _ in range(LAYERS)]

    def step(self, x, attention):
        """x [T][HIDDEN]; attention(layer, q, k, v) -> [T][HQ][D]; rows are views of the projection's output."""
        for layer in range(LAYERS):
            qkv = (x @ self.qkv[layer]).view(-1, HQ + 2 * HKV, D)
            out = attention(layer, qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:])
            x = x + out.reshape(-1, HQ * D) @ self.back[layer]
            x = x / x.float().norm(dim=1, keepdim=True).to(BF16) * math.sqrt(HIDDEN)
        return x


class Prompt:
    """A contiguous cache of pre-RoPE keys (what the compression's scores are defined on) for one sequence."""

    def __init__(self, model, room):
        self.model, self.room = model, room
        self.k = torch.empty((LAYERS, 1, HKV, room, D), dtype=BF16, device=DEV)
        self.v, self.pos = torch.empty_like(self.k), torch.empty((LAYERS, 1, HKV, room), dtype=torch.int32, device=DEV)
        self.length = torch.zeros(1, dtype=torch.int32, device=DEV)

    def cache(self, length, cur):
        return T.Cache(self.k, self.v, self.pos, length, cur, self.room)

    def prefill(self, toy, x, chunk=512):
        queries = []
        for t0 in range(0, len(x), chunk):
            n = min(chunk, len(x) - t0)
            pos = torch.arange(t0, t0 + n, dtype=torch.int32, device=DEV)
            tokens = T.Tokens(pos, start=torch.tensor([0, n], dtype=torch.int32, device=DEV))
            after = torch.empty_like(self.length)
            before_cache, after_cache = self.cache(self.length, pos[-1:]), self.cache(after, pos[-1:])
            ws = torch.empty(max(1, T.tri_attend_workspace_size(self.model, after_cache, tokens)), dtype=torch.uint8, device=DEV)
            seen = []

            def attention(layer, q, k, v):
                T.tri_append(self.model, before_cache, layer, tokens, k, v, after)   # reads the lengths before the step, writes those behind it
                out = torch.empty((n, HQ, D), dtype=BF16, device=DEV)
                T.tri_attend(self.model, after_cache, layer, tokens, q, out, workspace=ws)
                seen.append(q)
                return out
            last = toy.step(x[t0:t0 + n], attention)
            queries.append(torch.stack(seen, dim=1))
            self.length = after
        return last, torch.cat(queries)   # [tokens][layers][HQ][D]: what the calibration takes

    def compress(self, queries, budget):
        centers = torch.empty((LAYERS, HQ, D // 2, 3), dtype=torch.float32, device=DEV)
        T.tri_build_centers(self.model, queries.contiguous(), centers)
        cur = self.length.clone()
        kept = torch.empty((LAYERS, 1, HKV, budget), dtype=torch.int32, device=DEV)
        count, after = torch.empty((LAYERS, 1, HKV), dtype=torch.int32, device=DEV), torch.empty_like(self.length)
        cache = self.cache(self.length, cur)
        ws = torch.empty(T.tri_workspace_size(self.model, cache, budget), dtype=torch.uint8, device=DEV)
        T.tri_compress_step(self.model, centers, cache, None, budget, kept, count, after, ws)   # in place, fewest moves
        self.length, self.next_pos = after, cur


class Samples:
    """Paged caches of post-RoPE keys: pages are handed out as sequences grow."""

    def __init__(self, model, count, tokens):
        self.model, self.count, self.room = model, count, tokens
        per = -(-tokens // BLOCK)
        blocks = count * per
        self.k = torch.empty((LAYERS, blocks, HKV, BLOCK, D), dtype=BF16, device=DEV)
        self.v, self.pos = torch.empty_like(self.k), torch.empty((LAYERS, blocks, HKV, BLOCK), dtype=torch.int32, device=DEV)
        self.free = list(torch.randperm(blocks, generator=torch.Generator().manual_seed(1)).tolist())
        self.table = torch.full((count, per), -1, dtype=torch.int32, device=DEV)   # -1: no page yet
        self.lengths = [torch.zeros(count, dtype=torch.int32, device=DEV) for _ in range(2)]
        self.out = torch.empty((count, HQ, D), dtype=BF16, device=DEV)
        self.ws, self.done = None, 0

    def decode(self, toy, x, prompt):
        if self.done % BLOCK == 0:   # every sample begins a page
            self.table[:, self.done // BLOCK] = torch.tensor([self.free.pop() for _ in range(self.count)], dtype=torch.int32, device=DEV)
        pos = (prompt.next_pos + self.done).expand(self.count).contiguous()
        tokens = T.Tokens(pos)   # one token per sequence
        before, after = (T.Cache(self.k, self.v, self.pos, n, pos, self.room, block_table=self.table, k_rotated=True) for n in self.lengths)
        shared = prompt.cache(prompt.length, pos[:1])
        if self.ws is None:
            self.ws = torch.empty(max(1, T.tri_attend_workspace_size(self.model, after, tokens, shared)), dtype=torch.uint8, device=DEV)
        self.last = []

        def attention(layer, q, k, v):
            T.tri_append(self.model, before, layer, tokens, k, v, self.lengths[1])   # rotated on the way
            T.tri_attend_shared(self.model, shared, None, after, layer, tokens, q, self.out, workspace=self.ws)
            self.last.append((q, self.out.clone(), pos))
            return self.out
        x = toy.step(x, attention)
        self.lengths.reverse()
        self.done += 1
        return x


def _turn(x, pos, sign=1.0):
    w = THETA ** (torch.arange(D // 2, device=x.device, dtype=torch.float64) * (-2.0 / D))
    a = pos.double()[..., None] * w * sign
    re, im = x.double()[..., 0::2], x.double()[..., 1::2]
    return torch.stack([re * a.cos() - im * a.sin(), re * a.sin() + im * a.cos()], dim=-1).flatten(-2)


def plain(samples, prompt, layer):
    """The last step's attention of one layer in 64 bits, from what the caches hold."""
    q, got, pos = samples.last[layer]
    n, own = int(prompt.length[0]), int(samples.lengths[0][0])
    pages = samples.table[:, :-(-own // BLOCK)].long()
    worst = 0.0
    for s in range(samples.count):
        for h in range(HKV):
            k1 = _turn(prompt.k[layer, 0, h, :n], prompt.pos[layer, 0, h, :n])
            k2 = samples.k[layer, pages[s], h].flatten(0, 1)[:own].double()
            v = torch.cat([prompt.v[layer, 0, h, :n].double(), samples.v[layer, pages[s], h].flatten(0, 1)[:own].double()])
            rows = _turn(q[s, h * (HQ // HKV):(h + 1) * (HQ // HKV)], pos[s].expand(HQ // HKV))
            p = torch.softmax(rows @ torch.cat([k1, k2]).T / math.sqrt(D), dim=1)
            want = p @ v
            worst = max(worst, float((got[s, h * (HQ // HKV):(h + 1) * (HQ // HKV)].double() - want).abs().max() / want.abs().max()))
    return worst


def main(prompt=1500, budget=256, samples=6, tokens=20, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    toy = Toy(seed)
    model = T.Model(LAYERS, HQ, HKV, D, THETA, [1 << j for j in range(8)])
    p = Prompt(model, prompt)
    last, queries = p.prefill(toy, torch.randn(prompt, HIDDEN, generator=g, device=DEV).to(BF16))
    p.compress(queries, budget)
    s = Samples(model, samples, tokens)
    x = last[-1:].expand(samples, HIDDEN) + 0.1 * torch.randn(samples, HIDDEN, generator=g, device=DEV).to(BF16)   # (the samples' draws)
    for _ in range(tokens):
        x = s.decode(toy, x, p)
    off = max(plain(s, p, layer) for layer in range(LAYERS))
    return dict(kept=int(p.length[0]), decoded=int(s.lengths[0][0]), error=off, finite=bool(torch.isfinite(x).all()))


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    for name, default in (("prompt", 1500), ("budget", 256), ("samples", 6), ("tokens", 20)):
        a.add_argument("--" + name, type=int, default=default)
    r = main(**vars(a.parse_args()))
    print("prompt kept at %(kept)d keys per head, %(decoded)d tokens per sample; last step against 64 bits: %(error).1e of the largest value" % r)
