"""Performance cases of the attention operators: what stands between the QKV product and the output projection of a layer.

`own` says which side runs: the plain form (elementary torch operations in 32 bits, rounded once at the end) or the library.
`listed()` names the cases, `draw()` makes more of the same ranges, `prepare()` builds what a program holds before the call,
`run()` is one pass, `work()` the bytes and operations the pass cannot do without and `exact()` the result in 64 bits.

Kinds of cases (key "kind"):
  rope    head norms and rotary positions of a QKV product's rows, keys and values into a paged cache   (fq.qk_norm_rope)
  prompt  causal attention over packed prompts, keys possibly longer than queries (a prefix)           (fq.attention_prompt)
  tree    drafted tokens (a tree, a chain or one token per sequence) over a paged cache                 (fq.attention_tree)
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# (query heads, key heads, values per head)
HEADS = [(32, 8, 128), (32, 32, 128), (96, 96, 128), (40, 8, 128), (16, 2, 64), (12, 12, 64), (32, 32, 80), (24, 4, 96), (28, 4, 128)]


# ------------------------------------------------------------------------------------------------ the cases
def _rope(name, tokens, heads, act, rot, interleaved=False, norm=True, page=64, cache=True):
    return {"name": name, "kind": "rope", "tokens": tokens, "hq": heads[0], "hk": heads[1], "d": heads[2], "act": act, "rot": rot,
            "interleaved": interleaved, "norm": norm, "page": page, "cache": cache}


def _prompt(name, sequences, shortest, longest, heads, act, prefix=0):
    return {"name": name, "kind": "prompt", "sequences": sequences, "shortest": shortest, "longest": longest, "prefix": prefix,
            "hq": heads[0], "hk": heads[1], "d": heads[2], "act": act}


def _tree(name, sequences, nodes, shortest, longest, heads, act, page, masked):
    return {"name": name, "kind": "tree", "sequences": sequences, "nodes": nodes, "shortest": shortest, "longest": longest,
            "page": page, "masked": masked, "hq": heads[0], "hk": heads[1], "d": heads[2], "act": act}


def listed():
    return [
        # one step of generation for eight sequences: a call of microseconds
        _rope("rope_step_t8_bf16", 8, (32, 8, 128), "bf16", 128, page=16),
        # a prompt of a layer of 4096 channels, rotation alone, no cache yet
        _rope("rope_prompt_t2048_f16", 2048, (32, 32, 128), "f16", 128, norm=False, cache=False),
        # many packed prompts of a layer of 12288 channels, half of each head rotated, pairs side by side
        _rope("rope_packed_t16383_bf16", 16383, (96, 96, 128), "bf16", 64, interleaved=True),
        # one short prompt: fewer blocks than compute units
        _prompt("prompt_short_77_bf16", 1, 77, 77, (32, 8, 128), "bf16"),
        # a batch of prompts as they come
        _prompt("prompt_ragged_24_bf16", 24, 17, 1500, (32, 8, 128), "bf16"),
        # one long prompt, grouped heads: the compute-bound end
        _prompt("prompt_long_8192_bf16", 1, 8192, 8192, (32, 8, 128), "bf16"),
        # a layer of 12288 channels, a key head for each query head
        _prompt("prompt_wide_2_f16", 2, 1531, 2048, (96, 96, 128), "f16"),
        # the next pieces of prompts whose beginnings are known: few rows, many keys, heads of 80
        _prompt("prompt_prefix_3_f16_d80", 3, 100, 300, (32, 32, 80), "f16", prefix=4001),
        # one token of one sequence: latency
        _tree("tree_one_token_777_f16", 1, 1, 777, 777, (32, 8, 128), "f16", 16, False),
        # one token each of 64 sequences of very different lengths: the cache's bytes
        _tree("tree_tokens_64_bf16", 64, 1, 100, 8191, (32, 8, 128), "bf16", 64, False),
        # trees of 48 drafted tokens for eight sequences
        _tree("tree_draft_48_f16", 8, 48, 500, 4095, (32, 8, 128), "f16", 32, True),
        # sixteen drafted tokens at the end of one very long context
        _tree("tree_long_130999_bf16", 1, 16, 130999, 130999, (32, 8, 128), "bf16", 128, True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: a rope pass (a quarter of the draws), a prompt or a tree; none above the listed ones of its kind."""
    kind = rng.choices(["rope", "prompt", "tree"], [0.25, 0.375, 0.375])[0]
    most = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        case = _drawn(kind, rng)
        if all(work(case)[of] <= max(w[of] for w in most) for of in ("bytes", "flops")):
            return case


def _drawn(kind, rng):
    heads, act = rng.choice(HEADS), rng.choice(["f16", "bf16"])
    if kind == "rope":
        case = _rope("", _log_int(rng, 1, 16383), heads, act, rng.choice([heads[2], heads[2], heads[2] // 2]),
                     rng.random() < 0.4, rng.random() < 0.7, rng.choice([16, 32, 64, 128]), rng.random() < 0.7)
    elif kind == "prompt":
        longest = _log_int(rng, 33, 8192)
        prefix = _log_int(rng, 1, 8192) if rng.random() < 0.3 else 0
        # (the plain form pads sequences to the longest: their scores are kept to those of the long prompt)
        padded = max(1, 32 * 8192 * 8192 // (heads[0] * longest * (longest + prefix)))
        case = _prompt("", _log_int(rng, 1, max(1, min(32, padded, 16384 // longest))), _log_int(rng, max(1, longest // 50), longest),
                       longest, heads, act, prefix)
    else:
        nodes, longest = rng.choice([1, 1, _log_int(rng, 2, 100)]), _log_int(rng, 16, 131071)
        padded = max(1, 131071 * 8 * 128 // (longest * heads[1] * heads[2]))
        case = _tree("", _log_int(rng, 1, min(128, padded)), nodes, _log_int(rng, max(1, longest // 80), longest), longest, heads, act,
                     rng.choice([16, 32, 64, 128]), nodes > 1 and rng.random() < 0.7)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ what a program holds
def _lengths(case):
    """The sequences' lengths: spread over the range, the longest among them.  The same for every seed, as work() needs them."""
    rng = random.Random(f"{case['sequences']} {case['shortest']} {case['longest']}")
    lengths = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(case["sequences"])]
    lengths[rng.randrange(len(lengths))] = case["longest"]
    return lengths


def _prefixes(case):
    """What each prompt has before its queries: up to case["prefix"] keys."""
    rng = random.Random(f"{case['sequences']} {case['prefix']}")
    return [rng.randint(case["prefix"] // 2, case["prefix"]) for _ in range(case["sequences"])]


def _offsets(lengths):
    offsets = [0]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    return offsets


def _parents(nodes, rng):
    """A drafted tree: every node hangs from one of the few before it, several from the context itself (-1)."""
    return [max(-1, i - 1 - _skip(rng)) for i in range(nodes)]


def _skip(rng):
    return min(12, int(rng.expovariate(0.4)))


def _mask_words(parents):
    """For every node 64-bit words with the bits of itself and of its ancestors."""
    words = (len(parents) + 63) // 64
    seen = []
    for i, p in enumerate(parents):
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    signed = [[(s >> 64 * w) & (1 << 64) - 1 for w in range(words)] for s in seen]
    return [[v - (1 << 64) if v >> 63 else v for v in row] for row in signed]


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 1000003 + 17)
    rng = random.Random(seed)
    dtype, hq, hk, d = DTYPES[case["act"]], case["hq"], case["hk"], case["d"]

    def normal(*size, sigma=1.0):
        return torch.empty(size, dtype=dtype, device=DEV).normal_(0.0, sigma, generator=gen)

    state = dict(case)
    if case["kind"] == "rope":
        tokens, rot, page = case["tokens"], case["rot"], case["page"]
        state["qkv"] = normal(tokens, (hq + 2 * hk) * d, sigma=1.7)
        state["q_weight"] = normal(d, sigma=0.2) + 1 if case["norm"] else None
        state["k_weight"] = normal(d, sigma=0.2) + 1 if case["norm"] else None
        # cosines, then sines, of position x frequency
        angle = torch.arange(20000, dtype=torch.float64)[:, None] / 10000.0 ** (torch.arange(0, rot, 2, dtype=torch.float64) / rot)
        state["table"] = torch.cat([angle.cos(), angle.sin()], 1).float().to(DEV)
        first = rng.randrange(3000)
        state["positions"] = (torch.arange(tokens, dtype=torch.int32, device=DEV) + first).contiguous()
        if case["cache"]:
            pages = (tokens + page - 1) // page + 3
            state["k_cache"] = normal(pages, page, hk, d)
            state["v_cache"] = normal(pages, page, hk, d)
            order = torch.randperm(pages, generator=gen, device=DEV)
            at = torch.arange(tokens, device=DEV) + rng.randrange(page)
            state["slots"] = (order[at // page] * page + at % page).contiguous()
        return state
    if case["kind"] == "prompt":
        lengths = _lengths(case)
        state["q_offsets"] = _offsets(lengths)
        state["k_offsets"] = _offsets([n + p for n, p in zip(lengths, _prefixes(case))])
        state["q_starts"] = torch.tensor(state["q_offsets"], device=DEV)
        state["k_starts"] = torch.tensor(state["k_offsets"], device=DEV)
        rows, keys = state["q_offsets"][-1], state["k_offsets"][-1]
        state["q"] = normal(rows, hq, d, sigma=1.5)
        state["k"] = normal(keys, hk, d)
        if case["prefix"]:
            state["v"] = normal(keys, hk, d)
        else:       # values lie where the QKV product has left them
            state["v"] = normal(keys, (hq + 2 * hk) * d)[:, (hq + hk) * d:].view(keys, hk, d)
        return state
    lengths, page, nodes, n = _lengths(case), case["page"], case["nodes"], case["sequences"]
    width = (case["longest"] + nodes + page - 1) // page
    used = [(c + nodes + page - 1) // page for c in lengths]
    pages = sum(used) + 5
    state["k_cache"] = normal(pages, page, hk, d)
    state["v_cache"] = normal(pages, page, hk, d)
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    starts = torch.tensor(_offsets(used)[:-1], device=DEV)
    column = torch.arange(width, device=DEV)[None]
    column = torch.minimum(column, torch.tensor(used, device=DEV)[:, None] - 1)
    state["page_table"] = order[starts[:, None] + column].contiguous()
    state["context_lens"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    state["q"] = normal(n, nodes, hq, d, sigma=1.5)
    state["mask"] = None
    if case["masked"]:
        state["mask"] = torch.tensor([_mask_words(_parents(nodes, rng)) for _ in range(n)], dtype=torch.int64, device=DEV)
    return state


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _RUN_OWN[state["kind"]](state)
    return _RUN_PLAIN[state["kind"]](state)


def _own_rope(s):
    from paper_2308_09723_amd import fq
    q, k = fq.qk_norm_rope(s["qkv"], s["hq"], s["hk"], s["table"], s["positions"], q_weight=s["q_weight"], k_weight=s["k_weight"],
                           eps=1e-6, interleaved=s["interleaved"], k_cache=s.get("k_cache"), v_cache=s.get("v_cache"),
                           slots=s.get("slots"))
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]} if s["cache"] else {"q": q, "k": k}


def _own_prompt(s):
    from paper_2308_09723_amd import fq
    return fq.attention_prompt(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"] if s["prefix"] else None)


def _own_tree(s):
    from paper_2308_09723_amd import fq
    return fq.attention_tree(s["q"], s["k_cache"], s["v_cache"], s["page_table"], s["context_lens"], mask=s["mask"])


def _turned(x, cos, sin, interleaved):
    """The rotated part of heads x [tokens, heads, rot]."""
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _plain_rope(s):
    hq, hk, d, rot = s["hq"], s["hk"], s["d"], s["rot"]
    x = s["qkv"].view(-1, hq + 2 * hk, d)
    cos, sin = s["table"][s["positions"].long()].chunk(2, -1)

    def head(part, weight):
        y = part.float()
        if weight is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
        return torch.cat([_turned(y[..., :rot], cos, sin, s["interleaved"]), y[..., rot:]], -1).to(part.dtype)

    q, k = head(x[:, :hq], s["q_weight"]), head(x[:, hq:hq + hk], s["k_weight"])
    if not s["cache"]:
        return {"q": q, "k": k}
    s["k_cache"].view(-1, hk, d).index_copy_(0, s["slots"], k)
    s["v_cache"].view(-1, hk, d).index_copy_(0, s["slots"], x[:, hq + hk:])
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _attend(q, k, v, seen):
    """softmax(q k^T / sqrt(d)) v in 32 bits; q [B, R, Hq, D], k and v [B, L, Hk, D], seen [B, R, L] -> [B, R, Hq, D]."""
    B, R, hq, d = q.shape
    hk = k.shape[2]
    g = hq // hk
    q = q.float().view(B, R, hk, g, d).permute(0, 2, 3, 1, 4).reshape(B, hk, g * R, d)
    k = k.float().permute(0, 2, 3, 1).contiguous()
    v = v.float().permute(0, 2, 1, 3).contiguous()
    p = torch.matmul(q, k).view(B, hk, g, R, -1)
    p.mul_(1.0 / math.sqrt(d)).masked_fill_(~seen[:, None, None], float("-inf"))
    p.sub_(p.amax(-1, keepdim=True).clamp_min_(-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, hk, g * R, -1), v).view(B, hk, g, R, d) / total.clamp_min_(1e-30)
    return out.permute(0, 3, 1, 2, 4).reshape(B, R, hq, d)


def _plain_prompt(s):
    q0, k0 = s["q_starts"], s["k_starts"]
    rows, keys = s["q"].shape[0], s["k"].shape[0]
    nq, nk = q0[1:] - q0[:-1], k0[1:] - k0[:-1]
    # sequences padded to the longest
    longest_q = s["longest"]
    longest_k = s["longest"] + s["prefix"]
    i, j = torch.arange(longest_q, device=DEV), torch.arange(longest_k, device=DEV)
    row = (q0[:-1, None] + i).clamp_max_(rows - 1)
    key = (k0[:-1, None] + j).clamp_max_(keys - 1)
    seen = (j[None, None] <= i[None, :, None] + (nk - nq)[:, None, None]) & (j[None, None] < nk[:, None, None])
    out = _attend(s["q"][row], s["k"][key], s["v"][key], seen)
    of = torch.arange(rows, device=DEV)
    sequence = torch.searchsorted(q0, of, right=True) - 1
    return out[sequence, of - q0[sequence]].to(s["q"].dtype)


def _plain_tree(s):
    B, R = s["q"].shape[:2]
    hk, d = s["k_cache"].shape[2:]
    table = s["page_table"].long()
    k, v = s["k_cache"][table].view(B, -1, hk, d), s["v_cache"][table].view(B, -1, hk, d)
    drafted = torch.arange(k.shape[1], device=DEV)[None] - s["context_lens"].long()[:, None]       # [B, L]: which drafted token
    i = torch.arange(R, device=DEV)
    if s["mask"] is None:
        sees = (i[None, :] <= i[:, None]).expand(B, R, R)
    else:
        sees = (s["mask"][..., None] >> torch.arange(64, device=DEV) & 1).flatten(-2)[..., :R].bool()
    at = drafted.clamp(0, R - 1)[:, None].expand(B, R, -1)
    seen = (drafted < 0)[:, None] | ((drafted >= 0) & (drafted < R))[:, None] & sees.gather(2, at)
    return _attend(s["q"], k, v, seen).to(s["q"].dtype)


_RUN_OWN = {"rope": _own_rope, "prompt": _own_prompt, "tree": _own_tree}
_RUN_PLAIN = {"rope": _plain_rope, "prompt": _plain_prompt, "tree": _plain_tree}


# ------------------------------------------------------------------------------------------------ what it cannot do without
def work(case):
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["kind"] == "rope":
        read = case["tokens"] * ((hq + (2 if case["cache"] else 1) * hk) * d * 2 + case["rot"] * 4 + (12 if case["cache"] else 4))
        wrote = case["tokens"] * (hq + (2 if case["cache"] else 1) * hk) * d * 2
        return {"bytes": read + wrote, "flops": case["tokens"] * (hq + hk) * (3 * case["rot"] + (4 * d if case["norm"] else 0))}
    if case["kind"] == "prompt":
        lengths = _lengths(case)
        keys = [n + p for n, p in zip(lengths, _prefixes(case))]
        pairs = sum(n * (m - n) + n * (n + 1) // 2 for n, m in zip(lengths, keys))
        return {"bytes": 2 * d * (2 * sum(lengths) * hq + 2 * sum(keys) * hk), "flops": 4 * d * hq * pairs}
    lengths, nodes = _lengths(case), case["nodes"]
    keys = sum(c + nodes for c in lengths)
    pages = sum((c + nodes + case["page"] - 1) // case["page"] for c in lengths)
    return {"bytes": 2 * d * (2 * keys * hk + 2 * nodes * hq * len(lengths)) + 4 * pages + (8 * nodes * len(lengths) if case["masked"] else 0),
            "flops": 4 * d * hq * nodes * keys}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _exact_heads(q, k, v, seen):
    """q [R, Hq, D], k and v [L, Hk, D], seen [R, L] -> [R, Hq, D], from the definition, one key head at a time."""
    R, hq, d = q.shape
    hk = k.shape[1]
    out = torch.empty((R, hq, d), dtype=torch.float64, device=DEV)
    for h in range(hk):
        kt, vh = k[:, h].double().t().contiguous(), v[:, h].double()
        for x in range(h * (hq // hk), (h + 1) * (hq // hk)):
            score = (q[:, x].double() @ kt) / math.sqrt(d)
            weight = torch.where(seen, torch.exp(score - torch.where(seen, score, -math.inf).amax(1, keepdim=True)), 0.0)
            out[:, x] = (weight @ vh) / weight.sum(1, keepdim=True)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    hq, hk, d = case["hq"], case["hk"], case["d"]
    if case["kind"] == "rope":
        heads = s["qkv"].view(-1, hq + 2 * hk, d).double()
        half = case["rot"] // 2
        turn = torch.complex(s["table"][:, :half].double(), s["table"][:, half:].double())[s["positions"].long()][:, None]

        def one(x, weight):
            if weight is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6) * weight.double()
            out = x.clone()
            first = slice(0, 2 * half, 2) if case["interleaved"] else slice(0, half)
            second = slice(1, 2 * half, 2) if case["interleaved"] else slice(half, 2 * half)
            z = torch.complex(x[..., first].contiguous(), x[..., second].contiguous()) * turn
            out[..., first], out[..., second] = z.real, z.imag
            return out

        q, k = one(heads[:, :hq], s["q_weight"]), one(heads[:, hq:hq + hk], s["k_weight"])
        if not case["cache"]:
            return {"q": q, "k": k}
        caches = []
        for cache, rows in ((s["k_cache"], k), (s["v_cache"], heads[:, hq + hk:])):
            full = cache.double()
            full.view(-1, hk, d)[s["slots"]] = rows
            caches.append(full)
        return {"q": q, "k_cache": caches[0], "v_cache": caches[1]}
    if case["kind"] == "prompt":
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        bounds = zip(s["q_offsets"], s["q_offsets"][1:], s["k_offsets"], s["k_offsets"][1:])
        for a, b, e, f in bounds:
            last = torch.arange(b - a, device=DEV)[:, None] + (f - e) - (b - a)
            seen = torch.arange(f - e, device=DEV)[None] <= last
            out[a:b] = _exact_heads(s["q"][a:b], s["k"][e:f], s["v"][e:f], seen)
        return out
    nodes = case["nodes"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    words = None if s["mask"] is None else s["mask"].tolist()
    for b, context in enumerate(_lengths(case)):
        at = torch.arange(context + nodes, device=DEV)
        slots = s["page_table"][b].long()[at // case["page"]] * case["page"] + at % case["page"]
        sees = [[(words[b][i][j // 64] >> j % 64 & 1) == 1 if words else j <= i for j in range(nodes)] for i in range(nodes)]
        seen = torch.cat([torch.ones((nodes, context), dtype=torch.bool), torch.tensor(sees)], 1).to(DEV)
        out[b] = _exact_heads(s["q"][b], s["k_cache"].view(-1, hk, d)[slots], s["v_cache"].view(-1, hk, d)[slots], seen)
    return out
