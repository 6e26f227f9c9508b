"""An attention layer on quantised weights: prompts through fq_attention_prompt, drafted tokens through fq_attention_tree.

    python examples/attention_layer.py [--hidden 4096 --heads 32 --kv-heads 8 --prompts 700 1500 90 --drafted 12 --dtype bf16]

The layer is the four calls that a program makes per layer: the QKV product (fq.gemm), head norms, rotary positions and the cache's
writes (fq.qk_norm_rope), attention, and the output product (fq.gemm).  Run as a program it takes a batch of prompts, then one tree of
drafted tokens for each of them, keeps the longest branch, and goes on token by token; times are printed per call.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2308_09723_amd import fq  # noqa: E402


class Cache:
    """Keys and values of several sequences in pages that are handed out as sequences grow."""

    def __init__(self, sequences, tokens, kv_heads, head_dim, page=64, dtype=torch.bfloat16):
        self.page, self.width = page, (tokens + page - 1) // page
        pages = sequences * self.width
        self.k, self.v = (torch.zeros((pages, page, kv_heads, head_dim), dtype=dtype, device="cuda") for _ in range(2))
        # (as the pages of a long-running program: in no order)
        self.host_table = torch.randperm(pages, generator=torch.Generator().manual_seed(0)).view(sequences, self.width)
        self.table = self.host_table.to(torch.int32).cuda()
        self.lens = [0] * sequences

    def places(self, sequence, positions):
        """Slots of places in a sequence."""
        at = torch.as_tensor(positions)
        return self.host_table[sequence, at // self.page] * self.page + at % self.page


class AttentionLayer:
    def __init__(self, hidden, heads, kv_heads, bits=4, group=128, most_positions=8192, dtype=torch.bfloat16, seed=0):
        self.heads, self.kv_heads, self.D = heads, kv_heads, hidden // heads
        self.bits, self.group = bits, group
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def weights(K, N):
            return fq.quantize((torch.randn((K, N), generator=gen, device="cuda") * K ** -0.5).to(torch.float16), bits, group)

        self.qkv = weights(hidden, (heads + 2 * kv_heads) * self.D)
        self.out = weights(heads * self.D, hidden)
        self.q_norm, self.k_norm = (1 + 0.1 * torch.randn(self.D, generator=gen, device="cuda").to(dtype) for _ in range(2))
        self.table = fq.rope_table(most_positions, self.D)

    def _rows(self, x, positions, slots, cache):
        """The QKV product of x; queries ready, keys and values in the cache (and as tensors)."""
        rows = fq.gemm(x, *self.qkv, self.bits, self.group)
        k = torch.empty((x.shape[0], self.kv_heads, self.D), dtype=x.dtype, device=x.device)
        q, k = fq.qk_norm_rope(rows, self.heads, self.kv_heads, self.table, positions, self.q_norm, self.k_norm, k_out=k, k_cache=cache.k,
                               v_cache=cache.v, slots=slots)
        return q, k, rows.view(x.shape[0], -1, self.D)[:, self.heads + self.kv_heads:]

    def _output(self, attended):
        return fq.gemm(attended.reshape(-1, self.heads * self.D), *self.out, self.bits, self.group)

    def prompts(self, x, lengths, cache):
        """x: the prompts' rows one after the other, one prompt per sequence of an empty cache."""
        offsets = [0]
        for n in lengths:
            offsets.append(offsets[-1] + n)
        positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
        slots = torch.cat([cache.places(b, torch.arange(n)) for b, n in enumerate(lengths)]).cuda()
        q, k, v = self._rows(x, positions, slots, cache)
        cache.lens = list(lengths)
        return self._output(fq.attention_prompt(q, k, v, offsets))

    def drafted(self, x, parents, cache):
        """x [sequences * nodes, hidden]: a tree of drafted tokens (parents: fq.tree_mask) for every sequence.  Their keys and values lie
        behind the sequence's; keep() makes some of them part of it."""
        nodes, sequences = len(parents), len(cache.lens)
        depth = []
        for p in parents:
            depth.append(0 if p < 0 else depth[p] + 1)
        positions = torch.tensor([c + d for c in cache.lens for d in depth], dtype=torch.int32, device="cuda")
        slots = torch.cat([cache.places(b, torch.arange(c, c + nodes)) for b, c in enumerate(cache.lens)]).cuda()
        q, _, _ = self._rows(x, positions, slots, cache)
        lens = torch.tensor(cache.lens, dtype=torch.int32, device="cuda")
        mask = None if parents == list(range(-1, nodes - 1)) else fq.tree_mask(parents)
        attended = fq.attention_tree(q.view(sequences, nodes, self.heads, self.D), cache.k, cache.v, cache.table, lens, mask=mask)
        return self._output(attended)

    @staticmethod
    def keep(branch, cache):
        """Makes the drafted tokens `branch` (node numbers, from the context on) part of every sequence."""
        for b, c in enumerate(cache.lens):
            old, new = (cache.places(b, torch.tensor(at)).cuda() for at in ([c + i for i in branch], list(range(c, c + len(branch)))))
            for t in (cache.k, cache.v):
                rows = t.view(-1, t.shape[2] * t.shape[3])
                rows[new] = rows[old]
        cache.lens = [c + len(branch) for c in cache.lens]


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--hidden", type=int, default=4096)
    parser.add_argument("--heads", type=int, default=32)
    parser.add_argument("--kv-heads", type=int, default=8)
    parser.add_argument("--prompts", type=int, nargs="+", default=[700, 1500, 90])
    parser.add_argument("--drafted", type=int, default=12)
    parser.add_argument("--tokens", type=int, default=8)
    parser.add_argument("--dtype", choices=["f16", "bf16"], default="bf16")
    a = parser.parse_args()
    dtype = torch.float16 if a.dtype == "f16" else torch.bfloat16
    layer = AttentionLayer(a.hidden, a.heads, a.kv_heads, dtype=dtype)
    cache = Cache(len(a.prompts), max(a.prompts) + 2 * a.drafted + a.tokens, a.kv_heads, layer.D, dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def rows(n):
        return torch.randn((n, a.hidden), generator=gen, device="cuda").to(dtype)

    def timed(what, call):
        torch.cuda.synchronize()
        began = time.perf_counter()
        out = call()
        torch.cuda.synchronize()
        print(f"{what}: {(time.perf_counter() - began) * 1e3:.2f} ms, {tuple(out.shape)}, mean square {float(out.float().square().mean()):.4f}")
        return out

    for _ in range(2):      # (the first time round kernels are loaded)
        x = rows(sum(a.prompts))
        timed("prompts", lambda: layer.prompts(x, a.prompts, cache))
        # a tree: every node hangs from the one before it or from the one before that
        parents = [-1] + [i - 1 - (i % 3 == 2) for i in range(1, a.drafted)]
        x = rows(len(a.prompts) * a.drafted)
        timed("drafted tree", lambda: layer.drafted(x, parents, cache))
        branch, node = [], a.drafted - 1
        while node >= 0:
            branch.insert(0, node)
            node = parents[node]
        layer.keep(branch, cache)
        for _ in range(a.tokens):
            x = rows(len(a.prompts))
            y = layer.drafted(x, [-1], cache)
            layer.keep([0], cache)
        timed("one token each", lambda: layer.drafted(x, [-1], cache))
        assert bool(torch.isfinite(y).all())


if __name__ == "__main__":
    main()
