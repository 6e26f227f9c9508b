"""An attention layer that serves many requests: a shared quantised product with each request's adapter, and a cache held in 4 bits whose pages
requests share.

    python examples/serving_layer.py [--hidden 4096 --heads 32 --kv-heads 8 --prompts 700 1500 90 --beams 4 --rank 16 --tokens 16 --dtype bf16]

Per layer: the QKV product (fq.gemm) and the requests' adapters (fq.adapters), head norms and rotary positions (fq.qk_norm_rope), the cache's writes
(fq.kv4_write), attention (fq.attention_prompt for prompts, fq.attention_tree_kv4 for tokens), the output product (fq.gemm).  Tables, lengths and
references of the pages live on the device (fq.pages_take, fq.pages_fork, fq.pages_free, fq.pages_compact).  Run as a program it takes a batch of prompts, forks each
into beams, and goes on token by token, beams becoming continuations of one another; times are printed per call.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from examples.attention_layer import AttentionLayer  # noqa: E402
from paper_2308_09723_amd import fq  # noqa: E402


def room(prompts, beams, tokens, page=64):
    """Tokens of a table's rows, and pages of a pool, for beams of prompts that go on for so many tokens: the prompts' pages, and of each beam those of its own."""
    pages = sum((n + page - 1) // page for n in prompts) + len(prompts) * beams * ((tokens + page - 1) // page + 1)
    return max(prompts) + tokens, pages


class SharedCache:
    """A pool of pages held in 4 bits, and the rows of a table that hold them.  Rows that there is no room for are an error (grow, fork: the host waits for the lengths; a
    captured step would look at them behind its replays)."""

    def __init__(self, pages, rows, tokens, kv_heads, head_dim, page=64):
        self.page, self.kv_heads = page, kv_heads
        self.pages = fq.kv4_cache(pages, page, kv_heads, head_dim)
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.table = torch.full((rows, (tokens + page - 1) // page), -1, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")

    def grow(self, tokens):
        """Room for so many more tokens in every row (int32 [rows], on the device); the lengths from before."""
        before = self.lens.clone()
        wanted = before + tokens
        fq.pages_take(self.refs, self.page, self.table, self.lens, wanted)
        short = (self.lens != wanted).nonzero()[:, 0].tolist()
        if short:       # (their next keys have no place, and attention would read another row's in it)
            raise RuntimeError(f"no room for the next tokens of rows {short}: too few pages, or too few entries in the table")
        return before

    def slots(self, rows, positions):
        """Slots of places in rows (on the device)."""
        positions = positions.long()
        return self.table[rows, positions // self.page].long() * self.page + positions % self.page

    def fork(self, parents, release=True):
        self.table, self.lens = fq.pages_fork(self.refs, self.page, self.table, self.lens, parents, [self.pages], release=release)
        short = (self.lens < 0).nonzero()[:, 0].tolist()
        if short:
            raise RuntimeError(f"no pages for children {short}")

    def free(self, rows=None):
        fq.pages_free(self.refs, self.page, self.table, self.lens, rows)

    def compact(self):
        fq.pages_compact(self.refs, self.page, self.table, self.lens, [self.pages])


class ServingLayer(AttentionLayer):
    def __init__(self, hidden, heads, kv_heads, adapters=4, rank=16, **kw):
        super().__init__(hidden, heads, kv_heads, **kw)
        dtype = self.q_norm.dtype
        gen = torch.Generator(device="cuda").manual_seed(kw.get("seed", 0) + 1)
        N = (heads + 2 * kv_heads) * self.D
        self.a = (torch.randn((adapters, rank, hidden), generator=gen, device="cuda") * hidden ** -0.5).to(dtype)
        self.b = (torch.randn((adapters, N, rank), generator=gen, device="cuda") * 0.2).to(dtype)
        self.scales = torch.ones(adapters, device="cuda")

    def _ready(self, x, positions, ids):
        """Queries and keys, normalised and rotated, and values, of rows x with adapters ids."""
        product = fq.adapters(x, self.a, self.b, ids, fq.gemm(x, *self.qkv, self.bits, self.group), scales=self.scales)
        q, k = fq.qk_norm_rope(product, self.heads, self.kv_heads, self.table, positions, self.q_norm, self.k_norm)
        return q, k, product.view(x.shape[0], -1, self.D)[:, self.heads + self.kv_heads:]

    def prompts(self, x, lengths, cache, ids):
        """x: the prompts' rows one after the other, one for each of the first rows of an empty cache; ids: each prompt's adapter."""
        offsets = [0]
        for n in lengths:
            offsets.append(offsets[-1] + n)
        rows = torch.cat([torch.full((n,), b) for b, n in enumerate(lengths)]).cuda()
        positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
        cache.grow(torch.tensor(list(lengths) + [0] * (cache.lens.numel() - len(lengths)), dtype=torch.int32, device="cuda"))
        q, k, v = self._ready(x, positions, ids[rows].contiguous())
        fq.kv4_write(k, v, cache.pages, cache.page, cache.slots(rows, positions))
        return self._output(fq.attention_prompt(q, k, v, offsets))

    def tokens(self, x, cache, ids):
        """x [rows, hidden]: one more token of every row."""
        before = cache.grow(1)
        rows = torch.arange(x.shape[0], device="cuda")
        q, k, v = self._ready(x, before, ids)
        fq.kv4_write(k, v, cache.pages, cache.page, cache.slots(rows, before))
        return self._output(fq.attention_tree_kv4(q.unsqueeze(1), cache.pages, cache.page, self.kv_heads, cache.table, before))


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--hidden", type=int, default=4096)
    parser.add_argument("--heads", type=int, default=32)
    parser.add_argument("--kv-heads", type=int, default=8)
    parser.add_argument("--prompts", type=int, nargs="+", default=[700, 1500, 90])
    parser.add_argument("--beams", type=int, default=4)
    parser.add_argument("--rank", type=int, default=16)
    parser.add_argument("--tokens", type=int, default=16)
    parser.add_argument("--dtype", choices=["f16", "bf16"], default="bf16")
    a = parser.parse_args()
    dtype = torch.float16 if a.dtype == "f16" else torch.bfloat16
    layer = ServingLayer(a.hidden, a.heads, a.kv_heads, rank=a.rank, dtype=dtype)
    n = len(a.prompts)
    longest, pages = room(a.prompts, a.beams, a.tokens + 1)        # (the loop's tokens, and one that is timed)
    cache = SharedCache(pages, n, longest, a.kv_heads, layer.D)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def rows(n):
        return torch.randn((n, a.hidden), generator=gen, device="cuda").to(dtype)

    def timed(what, call):
        torch.cuda.synchronize()
        began = time.perf_counter()
        out = call()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - began) * 1e3:.2f} ms, {int((cache.refs > 0).sum())} pages held")
        return out

    ids = torch.arange(n, dtype=torch.int32, device="cuda") % layer.a.shape[0]
    timed("prompts", lambda: layer.prompts(rows(sum(a.prompts)), a.prompts, cache, ids))
    beams = torch.arange(n * a.beams, dtype=torch.int32, device="cuda") // a.beams
    timed("beams", lambda: cache.fork(beams))
    ids = ids[beams.long()].contiguous()
    for step in range(a.tokens):
        y = layer.tokens(rows(n * a.beams), cache, ids)
        # (in place of a choice among logits: beams go on as random ones of their group)
        chosen = beams * a.beams + torch.randint(0, a.beams, beams.shape, generator=gen, device="cuda", dtype=torch.int32)
        cache.fork(chosen)
    timed("one token each", lambda: layer.tokens(rows(n * a.beams), cache, ids))
    timed("gathered", cache.compact)
    timed("freed", cache.free)
    assert bool(torch.isfinite(y).all()) and not bool((cache.refs > 0).any())


if __name__ == "__main__":
    main()
