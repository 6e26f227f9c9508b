"""Plain attention and rotary positions in 64 bits on the host, and how far a correct implementation may be from them.

A result of the library has at most these errors against the 64-bit one of the same 16-bit inputs, u being half a unit in the last
place of the 16-bit type (2^-11 binary16, 2^-8 bfloat16), A = sum_j softmax_j |v_j|:
  u |out|            the rounding of the result
  u A                the rounding of the softmax's numerators for their product with the values
  2 d A              scores that are off by d, binary32 sums of head_dim products: d = (head_dim + 8) 2^-24 max_j sum |q k_j| scale
                     (the numerators change by a factor of at most e^d, their sum by the same)
  2^-22 A            exponentials, sums and the division in binary32 (a few units each; sums of thousands of positive terms in blocks)
  2^-25 (1 + sum |v|) numerators and results below the smallest normal binary16
"""
import math

import numpy as np
import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def attend(q, k, v, seen, scale):
    """q [R, D], k and v [L, D], seen [R, L] bool -> (result, tolerance) [R, D]; rows that see nothing are zeros."""
    unit = UNIT[q.dtype]
    D = q.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, tol = torch.zeros((q.shape[0], D), dtype=torch.float64), torch.zeros((q.shape[0], D), dtype=torch.float64)
    for i in range(q.shape[0]):
        j = torch.nonzero(seen[i])[:, 0]
        if len(j) == 0:
            continue
        terms = q[i] * k[j]
        s = terms.sum(1) * scale
        p = torch.exp(s - s.max())
        p = p / p.sum()
        out[i] = (p[:, None] * v[j]).sum(0)
        A = (p[:, None] * v[j].abs()).sum(0)
        d = (D + 8) * 2.0 ** -24 * float(terms.abs().sum(1).max()) * scale
        tol[i] = unit * out[i].abs() + (unit + 2 * d + 2.0 ** -22) * A + 2.0 ** -25 * (1 + v[j].abs().sum(0))
    return out, tol


def prompt(q, k, v, q_offsets, k_offsets, scale=None):
    """Host tensors [rows, heads, D], [keys, kv_heads, D] -> (result, tolerance)."""
    scale = scale or 1 / math.sqrt(q.shape[2])
    group = q.shape[1] // k.shape[1]
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for a, b, e, f in zip(q_offsets, q_offsets[1:], k_offsets, k_offsets[1:]):
        seen = torch.arange(f - e)[None] <= torch.arange(b - a)[:, None] + (f - e) - (b - a)
        for h in range(q.shape[1]):
            out[a:b, h], tol[a:b, h] = attend(q[a:b, h], k[e:f, h // group], v[e:f, h // group], seen, scale)
    return out, tol


def tree(q, k_cache, v_cache, table, lens, sees, scale=None):
    """Host tensors; sees [sequences, nodes, nodes] bool (which drafted tokens a node sees)."""
    scale = scale or 1 / math.sqrt(q.shape[3])
    B, n, heads, D = q.shape
    page, kv_heads = k_cache.shape[1:3]
    group = heads // kv_heads
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for b in range(B):
        context = int(lens[b])
        if context < 0:
            continue
        seen = torch.cat([torch.ones((n, context), dtype=torch.bool), sees[b]], 1)[:, :table.shape[1] * page]
        at = torch.arange(seen.shape[1])
        pages, places = table[b].long()[at // page], at % page
        for h in range(heads):
            out[b, :, h], tol[b, :, h] = attend(q[b, :, h], k_cache[pages, places, h // group], v_cache[pages, places, h // group], seen, scale)
    return out, tol


def chain(B, n):
    return torch.ones((n, n), dtype=torch.bool).tril()[None].expand(B, n, n)


def from_parents(parents):
    """[nodes, nodes] bool: each node sees itself and its ancestors."""
    n = len(parents)
    sees = torch.zeros((n, n), dtype=torch.bool)
    for i, p in enumerate(parents):
        if p >= 0:
            sees[i] = sees[p]
        sees[i, i] = True
    return sees


def words(sees):
    """[..., nodes, nodes] bool -> int64 [..., nodes, words]."""
    n = sees.shape[-1]
    count = (n + 63) // 64
    bits = torch.zeros(sees.shape[:-1] + (count * 64,), dtype=torch.bool)
    bits[..., :n] = sees
    packed = np.packbits(bits.numpy(), axis=-1, bitorder="little").view(np.int64)
    return torch.from_numpy(np.ascontiguousarray(packed))


def norm_rope(heads, weight, eps, table, positions, interleaved):
    """heads [tokens, H, D] -> (result, tolerance): binary32 arithmetic on up to 128 squares, then four operations, then one rounding."""
    unit = UNIT[heads.dtype]
    D = heads.shape[2]
    x = heads.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    out, size = x.clone(), x.abs()
    rot = 0 if table is None else table.shape[1]
    if rot:
        p = positions.long().clamp(0, table.shape[0] - 1)
        c, s = table[p, :rot // 2].double()[:, None], table[p, rot // 2:].double()[:, None]
        a = slice(0, rot, 2) if interleaved else slice(0, rot // 2)
        b = slice(1, rot, 2) if interleaved else slice(rot // 2, rot)
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        both = x[..., a].abs() + x[..., b].abs()
        size = size.clone()
        size[..., a] = size[..., b] = both
    return out, unit * out.abs() + (D + 16) * 2.0 ** -24 * size + 2.0 ** -25


def compare(got, want, tol, what):
    got = got.cpu().double()
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    off = (got - want).abs() - tol
    assert float(off.max()) <= 0, f"{what}: {float((got - want).abs().max())} off, {float(((got - want).abs() / tol.clamp_min(1e-30)).max())} times what is allowed"
