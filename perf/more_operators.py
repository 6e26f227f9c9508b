"""Performance cases of what serving many requests adds to a layer: a cache held in 4 bits, the pages that requests share, their adapters.

`own` says which side runs: the plain form (elementary torch operations in 32 bits, rounded once at the end) or the library.
`listed()` names the cases, `draw()` makes more of the same ranges, `prepare()` builds what a program holds before the call,
`run()` is one pass, `work()` the bytes and operations the pass cannot do without and `exact()` the result in 64 bits.

Kinds of cases (key "kind"):
  store    keys and values into a cache held in 4 bits, and a sequence's read back as 16-bit values  (fq.kv4_write, fq.kv4_read)
  attend   drafted tokens (a tree, a chain or one token per sequence) over such a cache              (fq.attention_tree_kv4)
  fork     sequences replaced by others' continuations, pages shared, the last one copied            (fq.pages_fork)
  compact  a cache's pages moved to its beginning                                                    (fq.pages_compact)
  adapt    low-rank adapters of many requests added to a shared product                              (fq.adapters)

The cache held in 4 bits: pages of [kv_heads][page_size / 16] records of 16 tokens of one head; with S = ceil(head_dim / 32) a record
is 576 S bytes: keys' codes [4 a][16 token][S t][4 b], values' codes [4 a][16 n][S j][4 b], keys' scales [4 a][S group][4 b] and values'
scales, both 16 bits wide.  A byte holds two codes, sign and magnitude: bits 7 and 2 .. 0, and bits 6 and 5 .. 3.  Keys: values
32 t + 8 a + b and four further of the token; values: token 4 a + b's values 32 j + n and sixteen further; scales: of token 4 a + b.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
# significant bits of a scale, and the exponent of the type's smallest value: a code times a scale is a value of the type
SCALES = {"f16": (8, -24), "bf16": (5, -133)}
# (query heads, key heads, values per head)
HEADS = [(32, 8, 128), (32, 32, 128), (40, 8, 128), (16, 2, 64), (12, 12, 64), (32, 32, 80), (24, 4, 96), (28, 4, 128)]


# ------------------------------------------------------------------------------------------------ the cases
def _store(name, tokens, prefix, heads, act, page):
    return {"name": name, "kind": "store", "tokens": tokens, "prefix": prefix, "hk": heads[1], "d": heads[2], "act": act, "page": page}


def _attend(name, sequences, nodes, shortest, longest, heads, act, page, masked):
    return {"name": name, "kind": "attend", "sequences": sequences, "nodes": nodes, "shortest": shortest, "longest": longest,
            "page": page, "masked": masked, "hq": heads[0], "hk": heads[1], "d": heads[2], "act": act}


def _fork(name, groups, beams, shortest, longest, page, page_bytes, layers):
    return {"name": name, "kind": "fork", "groups": groups, "beams": beams, "shortest": shortest, "longest": longest, "page": page,
            "page_bytes": page_bytes, "layers": layers}


def _compact(name, sequences, shortest, longest, page, page_bytes, layers, spread):
    return {"name": name, "kind": "compact", "sequences": sequences, "shortest": shortest, "longest": longest, "page": page,
            "page_bytes": page_bytes, "layers": layers, "spread": spread}


def _adapt(name, requests, rows, adapters, rank, K, N, act):
    return {"name": name, "kind": "adapt", "requests": requests, "rows": rows, "adapters": adapters, "rank": rank, "K": K, "N": N,
            "act": act}


def listed():
    return [
        # the next piece of a prompt, of a few tokens: a call of microseconds
        _store("store_piece_33_bf16", 33, 700, (32, 8, 128), "bf16", 16),
        # a batch of prompts' tokens, and their keys and values for the prompt's attention
        _store("store_prompt_16383_f16", 16383, 0, (32, 8, 128), "f16", 64),
        # one token of one sequence, a key head for each query head, of 80 values: latency
        _attend("kv4_one_token_777_f16", 1, 1, 777, 777, (32, 32, 80), "f16", 16, False),
        # one token each of 64 sequences of very different lengths: the cache's bytes
        _attend("kv4_tokens_64_bf16", 64, 1, 100, 8191, (32, 8, 128), "bf16", 64, False),
        # trees of 48 drafted tokens for eight sequences
        _attend("kv4_draft_48_f16", 8, 48, 500, 4095, (32, 8, 128), "f16", 32, True),
        # the next pieces of two prompts over what the cache has of them
        _attend("kv4_pieces_700_bf16", 2, 700, 2500, 3900, (32, 8, 128), "bf16", 64, False),
        # a step of four beams of one sequence, in one layer: latency
        _fork("fork_beams_4", 1, 4, 777, 777, 16, 18432, 1),
        # a step of eight beams each of 32 sequences: copies of 8 layers' pages
        _fork("fork_beams_256", 32, 8, 100, 2000, 64, 73728, 8),
        # 64 sequences' cache of 16 layers gathered where a third of the pages are free
        _compact("compact_64", 64, 200, 4095, 64, 73728, 16, 1.5),
        # one token of one request: latency
        _adapt("adapt_one_bf16", 1, 1, 4, 8, 1024, 1024, "bf16"),
        # one token each of 64 requests, each with its adapter, beside a QKV product
        _adapt("adapt_tokens_64_bf16", 64, 64, 64, 16, 4096, 6144, "bf16"),
        # prompts of five requests, beside a QKV product of 12288 channels
        _adapt("adapt_prompts_2900_f16", 5, 2900, 8, 64, 12288, 36864, "f16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case, none above the listed ones of its kind."""
    kind = rng.choices(["store", "attend", "fork", "compact", "adapt"], [0.15, 0.4, 0.1, 0.1, 0.25])[0]
    most = [work(c) for c in listed() if c["kind"] == kind]
    while True:
        case = _drawn(kind, rng)
        if all(work(case)[of] <= max(w[of] for w in most) for of in ("bytes", "flops")):
            return case


def _drawn(kind, rng):
    heads, act, page = rng.choice(HEADS), rng.choice(["f16", "bf16"]), rng.choice([16, 32, 48, 64, 128])
    if kind == "store":
        tokens = _log_int(rng, 1, 16383)
        case = _store("", tokens, _log_int(rng, 1, 8000) if rng.random() < 0.5 else 0, heads, act, page)
    elif kind == "attend":
        nodes, longest = rng.choice([1, 1, _log_int(rng, 2, 40), _log_int(rng, 20, 700)]), _log_int(rng, 16, 32767)
        # (the plain form pads sequences to the longest: their keys and scores are kept to those of the listed cases)
        padded = max(1, min(8191 * 64 * 8 * 128 // (longest * heads[1] * heads[2]), 3900 * 700 * 2 * 32 // (longest * nodes * heads[0])))
        case = _attend("", _log_int(rng, 1, min(128, padded)), nodes, _log_int(rng, max(1, longest // 80), longest), longest, heads, act,
                       page, 1 < nodes <= 100 and rng.random() < 0.7)
    elif kind == "fork":
        longest = _log_int(rng, 16, 4095)
        case = _fork("", _log_int(rng, 1, 32), rng.randint(1, 8), _log_int(rng, max(1, longest // 20), longest), longest, page,
                     1152 * (page // 16) * rng.choice([2, 8, 16, 33]), _log_int(rng, 1, 16))
    elif kind == "compact":
        longest = _log_int(rng, 16, 4095)
        case = _compact("", _log_int(rng, 1, 64), _log_int(rng, max(1, longest // 20), longest), longest, page,
                        1152 * (page // 16) * rng.choice([2, 8, 16]), _log_int(rng, 1, 16), rng.choice([1.1, 1.5, 3.0]))
    else:
        rows = _log_int(rng, 1, 2900)
        case = _adapt("", rng.choice([rows, _log_int(rng, 1, min(rows, 24))]) if rows <= 256 else _log_int(rng, 1, 24), rows,
                      _log_int(rng, 1, 64), rng.choice([8, 16, 16, 24, 32, 64]), rng.choice([768, 1024, 2048, 4096, 5120, 8192, 12288]),
                      rng.choice([776, 1024, 1536, 2048, 4096, 6144, 11008, 12288, 36864]), act)
    del case["name"]
    return case


# ------------------------------------------------------------------------------------------------ what a program holds
def _lengths(case, count):
    """The sequences' lengths: spread over the range, the longest among them.  The same for every seed, as work() needs them."""
    rng = random.Random(f"{count} {case['shortest']} {case['longest']}")
    lengths = [_log_int(rng, case["shortest"], case["longest"]) for _ in range(count)]
    lengths[rng.randrange(len(lengths))] = case["longest"]
    return lengths


def _parents(case):
    """Whose continuation each beam becomes: within its group, better ones more often."""
    rng = random.Random(f"{case['groups']} {case['beams']}")
    return [g * case["beams"] + min(case["beams"] - 1, int(rng.expovariate(0.7))) for g in range(case["groups"]) for _ in range(case["beams"])]


def _segments(case):
    """The adapter of each row, the same for every seed: requests' rows side by side, one request in eight without an adapter."""
    rng = random.Random(f"{case['requests']} {case['rows']} {case['adapters']}")
    cuts = sorted(rng.sample(range(1, case["rows"]), case["requests"] - 1)) if case["requests"] > 1 else []
    ids = []
    for i, (a, b) in enumerate(zip([0] + cuts, cuts + [case["rows"]])):
        ids += [(-1 if i % 8 == 7 else i % case["adapters"])] * (b - a)
    return ids


def _mask_words(nodes, rng):
    """A drafted tree: for every node 64-bit words with the bits of itself and of its ancestors."""
    words = (nodes + 63) // 64
    seen = []
    for i in range(nodes):
        p = max(-1, i - 1 - min(12, int(rng.expovariate(0.4))))
        seen.append((seen[p] if p >= 0 else 0) | 1 << i)
    rows = [[(s >> 64 * w) & (1 << 64) - 1 for w in range(words)] for s in seen]
    return [[v - (1 << 64) if v >> 63 else v for v in row] for row in rows]


def _page_table(used, pages, gen):
    """Pages of sequences that use so many each, in no order; behind them entries of the last one."""
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    starts = torch.tensor([sum(used[:i]) for i in range(len(used))], device=DEV)
    column = torch.minimum(torch.arange(max(used), device=DEV)[None], torch.tensor(used, device=DEV)[:, None] - 1)
    return order[starts[:, None] + column].contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 1000003 + 29)
    rng = random.Random(seed)
    kind, state = case["kind"], dict(case)

    def normal(*size, sigma=1.0):
        return torch.empty(size, dtype=DTYPES[case["act"]], device=DEV).normal_(0.0, sigma, generator=gen)

    if kind in ("store", "attend"):
        page, hk, d = case["page"], case["hk"], case["d"]
        record = 576 * ((d + 31) // 32)
    if kind == "store":
        tokens, prefix = case["tokens"], case["prefix"]
        used = (tokens + prefix + page - 1) // page
        pages = used + 3
        at = torch.arange(tokens + prefix, device=DEV)
        slots = torch.randperm(pages, generator=gen, device=DEV)[at // page] * page + at % page
        state["slots"], state["written"] = slots, slots[prefix:].contiguous()
        state["cache"] = torch.zeros((pages, hk * (page // 16) * record), dtype=torch.uint8, device=DEV)
        if prefix:
            _put(state["cache"], normal(prefix, hk, d, sigma=2.0), normal(prefix, hk, d), slots[:prefix], page, case["act"])
        state["k"] = normal(tokens, hk, d, sigma=2.0)
        state["v"] = normal(tokens, 3 * hk * d)[:, 2 * hk * d:].view(tokens, hk, d)      # values lie where the QKV product has left them
    elif kind == "attend":
        lengths, nodes, n, hq = _lengths(case, case["sequences"]), case["nodes"], case["sequences"], case["hq"]
        used = [(c + nodes + page - 1) // page for c in lengths]
        pages = sum(used) + 5
        table = _page_table(used, pages, gen)
        state["cache"] = torch.zeros((pages, hk * (page // 16) * record), dtype=torch.uint8, device=DEV)
        step = max(1, (1 << 17) // page)
        for first in range(0, pages, step):      # every slot of every page holds keys and values
            slots = torch.arange(first * page, min(pages, first + step) * page, device=DEV)
            _put(state["cache"], normal(slots.numel(), hk, d), normal(slots.numel(), hk, d), slots, page, case["act"])
        state["page_table"] = table
        state["context_lens"] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        state["q"] = normal(n, nodes, hq, d, sigma=1.5)
        state["mask"] = None
        if case["masked"]:
            state["mask"] = torch.tensor([_mask_words(nodes, rng) for _ in range(n)], dtype=torch.int64, device=DEV)
    elif kind in ("fork", "compact"):
        count = case["groups"] * case["beams"] if kind == "fork" else case["sequences"]
        lengths = _lengths(case, count)
        if kind == "fork":      # beams of a sequence are of its length
            lengths = [lengths[i // case["beams"] * case["beams"]] for i in range(count)]
            state["parents"] = torch.tensor(_parents(case), dtype=torch.int32, device=DEV)
        used = [(c + case["page"] - 1) // case["page"] for c in lengths]
        pages = sum(used) + count + 3 if kind == "fork" else int(sum(used) * case["spread"]) + 1
        table = _page_table(used, pages, gen)
        table[torch.arange(table.shape[1], device=DEV)[None] >= torch.tensor(used, device=DEV)[:, None]] = -1
        state["page_table"], state["context_lens"] = table, torch.tensor(lengths, dtype=torch.int32, device=DEV)
        state["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
        state["refs"][table[table >= 0].long()] = 1
        state["buffers"] = torch.empty((case["layers"], pages, case["page_bytes"] // 8), dtype=torch.int64, device=DEV)
        state["buffers"].random_(generator=gen)
    else:
        state["ids"] = torch.tensor(_segments(case), dtype=torch.int32, device=DEV)
        state["x"] = normal(case["rows"], case["K"])
        state["a"] = normal(case["adapters"], case["rank"], case["K"], sigma=case["K"] ** -0.5)
        state["b"] = normal(case["adapters"], case["N"], case["rank"], sigma=0.05)
        state["scales"] = torch.empty(case["adapters"], device=DEV).uniform_(0.5, 2.0, generator=gen)
        state["product"] = normal(case["rows"], case["N"])
    return state


# ------------------------------------------------------------------------------------------------ the cache, plainly
def _quantised(x, act):
    """x [rows, heads, d] -> codes [rows, heads, 32 S] (whole numbers) and scales [rows, heads, S], both float64.
    Scales in 64 bits: which of two is taken is decided by a quotient."""
    bits, least = SCALES[act]
    rows, heads, d = x.shape
    groups = (d + 31) // 32
    w = torch.zeros((rows, heads, groups * 32), dtype=torch.float64, device=x.device)
    w[..., :d] = x.double()
    w = w.view(rows, heads, groups, 32)
    least_scale = w.abs().amax(-1) / 7.5
    exponent = torch.frexp(least_scale)[1]
    step = ((exponent - bits).clamp_min(least).long() + 1023 << 52).view(torch.float64)       # a power of two
    scale = torch.where(least_scale > 0, torch.ceil(least_scale / step) * step, 0.0)
    codes = torch.where(scale[..., None] > 0, torch.round(w / scale[..., None]), 0.0).clamp(-7, 7)
    return codes.view(rows, heads, groups * 32), scale


def _records(cache, page, d):
    """The parts of all records [pages, heads, page / 16, ...]: codes of keys and of values, scales of both (bytes)."""
    S = (d + 31) // 32
    r = cache.view(cache.shape[0], -1, page // 16, 576 * S)
    return (r[..., :256 * S].unflatten(-1, (4, 16, S, 4)), r[..., 256 * S:512 * S].unflatten(-1, (4, 16, S, 4)),
            r[..., 512 * S:544 * S].unflatten(-1, (4, S, 4, 2)), r[..., 544 * S:].unflatten(-1, (4, S, 4, 2)))


def _two(first, second):
    """Two codes in a byte."""
    return ((first < 0) * 128 + first.abs() + (second < 0) * 64 + second.abs() * 8).to(torch.uint8)


def _put(cache, k, v, slots, page, act):
    """Keys and values [rows, heads, d] into the cache's slots."""
    d, S, heads = k.shape[-1], (k.shape[-1] + 31) // 32, k.shape[1]
    at, tile, token = slots // page, slots % page // 16, slots % 16
    key_codes, value_codes, key_scales, value_scales = _records(cache, page, d)
    for x, codes, scales, keys in ((k, key_codes, key_scales, True), (v, value_codes, value_scales, False)):
        q, s = _quantised(x, act)
        s = s.to(DTYPES[act]).contiguous().view(torch.uint8).view(-1, heads, S, 2)
        scales.permute(0, 2, 3, 5, 1, 4, 6)[at, tile, token // 4, token % 4] = s
        if keys:
            q = q.view(-1, heads, S, 4, 2, 4)       # t, a, half, b
            codes.permute(0, 2, 4, 1, 5, 3, 6)[at, tile, token] = _two(q[:, :, :, :, 0], q[:, :, :, :, 1])
        else:
            q = q.view(-1, heads, S, 2, 16)         # j, half, n
            codes.permute(0, 2, 3, 6, 1, 5, 4)[at, tile, token // 4, token % 4] = _two(q[:, :, :, 0], q[:, :, :, 1])


def _taken(cache, pages, page, d, act):
    """Keys and values of whole pages, in 32 bits: pages [...] -> two [..., page, heads, d]."""
    S = (d + 31) // 32
    kc, vc, ks, vs = _records(cache[pages.reshape(-1)], page, d)
    n, heads, tiles = kc.shape[:3]

    def values(codes, scales, order, size):
        first = (codes & 7).float() * (1 - 2 * (codes >> 7).float())
        second = (codes >> 3 & 7).float() * (1 - 2 * (codes >> 6 & 1).float())
        q = torch.stack([first, second], -1).permute(order).reshape(n, tiles * 16, heads, S, 32)
        s = scales.contiguous().view(DTYPES[act])[..., 0].float().permute(0, 2, 3, 5, 1, 4).reshape(n, tiles * 16, heads, S, 1)
        return (q * s).reshape(*size, tiles * 16, heads, S * 32)[..., :d]

    # codes [n, heads, tiles, 4 a, 16, S, 4 b, 2]: keys (token, heads, t, a, half, b); values (a, b, heads, j, half, n)
    return values(kc, ks, (0, 2, 4, 1, 5, 3, 7, 6), pages.shape), values(vc, vs, (0, 2, 3, 6, 1, 5, 7, 4), pages.shape)


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _RUN_OWN[state["kind"]](state)
    return _RUN_PLAIN[state["kind"]](state)


def _own_store(s):
    from paper_2308_09723_amd import fq
    fq.kv4_write(s["k"], s["v"], s["cache"], s["page"], s["written"])
    k, v = fq.kv4_read(s["cache"], s["page"], s["hk"], s["d"], s["slots"], s["k"].dtype)
    return {"k": k, "v": v}


def _own_attend(s):
    from paper_2308_09723_amd import fq
    return fq.attention_tree_kv4(s["q"], s["cache"], s["page"], s["hk"], s["page_table"], s["context_lens"], mask=s["mask"])


def _own_fork(s):
    from paper_2308_09723_amd import fq
    s["page_table"], s["context_lens"] = fq.pages_fork(s["refs"], s["page"], s["page_table"], s["context_lens"], s["parents"], s["buffers"],
                                                       release=True)
    return {"page_table": s["page_table"], "context_lens": s["context_lens"], "refs": s["refs"], "buffers": s["buffers"]}


def _own_compact(s):
    from paper_2308_09723_amd import fq
    refs, table = s["refs"].clone(), s["page_table"].clone()       # (the pass can be made again: its sources stay where they are)
    fq.pages_compact(refs, s["page"], table, s["context_lens"], s["buffers"])
    return {"page_table": table, "refs": refs, "buffers": s["buffers"]}


def _own_adapt(s):
    from paper_2308_09723_amd import fq
    out = s["product"].clone()
    fq.adapters(s["x"], s["a"], s["b"], s["ids"], out, scales=s["scales"])
    return out


def _plain_store(s):
    _put(s["cache"], s["k"], s["v"], s["written"], s["page"], s["act"])
    pages = s["slots"][::s["page"]] // s["page"]
    k, v = _taken(s["cache"], pages, s["page"], s["d"], s["act"])
    n = s["slots"].numel()
    return {"k": k.flatten(0, 1)[:n].to(DTYPES[s["act"]]), "v": v.flatten(0, 1)[:n].to(DTYPES[s["act"]])}


def _softmax_product(q, k, v, seen):
    """softmax(q k^T / sqrt(d)) v in 32 bits; q [B, R, Hq, D], k and v [B, L, Hk, D], seen [B, R, L] -> [B, R, Hq, D]."""
    B, R, hq, d = q.shape
    hk = k.shape[2]
    g = hq // hk
    q = q.float().view(B, R, hk, g, d).permute(0, 2, 3, 1, 4).reshape(B, hk, g * R, d)
    p = torch.matmul(q, k.permute(0, 2, 3, 1).contiguous()).view(B, hk, g, R, -1)
    p.mul_(1.0 / math.sqrt(d)).masked_fill_(~seen[:, None, None], float("-inf"))
    p.sub_(p.amax(-1, keepdim=True).clamp_min_(-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, hk, g * R, -1), v.permute(0, 2, 1, 3).contiguous()).view(B, hk, g, R, d) / total.clamp_min_(1e-30)
    return out.permute(0, 3, 1, 2, 4).reshape(B, R, hq, d)


def _plain_attend(s):
    B, R = s["q"].shape[:2]
    k, v = _taken(s["cache"], s["page_table"].long(), s["page"], s["d"], s["act"])
    k, v = k.flatten(1, 2), v.flatten(1, 2)
    drafted = torch.arange(k.shape[1], device=DEV)[None] - s["context_lens"].long()[:, None]       # [B, L]: which drafted token
    i = torch.arange(R, device=DEV)
    if s["mask"] is None:
        sees = (i[None, :] <= i[:, None]).expand(B, R, R)
    else:
        sees = (s["mask"][..., None] >> torch.arange(64, device=DEV) & 1).flatten(-2)[..., :R].bool()
    at = drafted.clamp(0, R - 1)[:, None].expand(B, R, -1)
    seen = (drafted < 0)[:, None] | ((drafted >= 0) & (drafted < R))[:, None] & sees.gather(2, at)
    return _softmax_product(s["q"], k, v, seen).to(s["q"].dtype)


def _plain_fork(s):
    refs, page, table, lens, parents = s["refs"], s["page"], s["page_table"], s["context_lens"], s["parents"].long()
    n, width = table.shape
    column = torch.arange(width, device=DEV)[None]
    full, part = lens // page, lens % page > 0
    i = torch.arange(parents.numel(), device=DEV)
    first = ((parents[None] == parents[:, None]) & (i[None] < i[:, None])).any(1).logical_not()
    # the children's references to whole pages, less all of the old rows' but those to last pages that a child takes over
    rows, child_full = table[parents], full[parents]
    held = column < child_full[:, None]
    refs.index_add_(0, rows[held].long(), torch.ones_like(rows[held]))
    taken_over = torch.zeros(n, dtype=torch.bool, device=DEV).index_fill_(0, parents, True)
    gone = (column < full[:, None]) | (column == full[:, None]) & (part & ~taken_over)[:, None]
    refs.index_add_(0, table[gone].long(), -torch.ones_like(table[gone]))
    # last pages: the parent's own for its first child, copies for the others, in the lowest free pages
    wanted = part[parents] & ~first
    free = torch.nonzero(refs <= 0)[:, 0]
    rank = torch.cumsum(wanted, 0) - 1
    fresh = free[rank.clamp(0, free.numel() - 1)]
    last = rows.gather(1, child_full.long().clamp_max(width - 1)[:, None])[:, 0]
    own_page = torch.where(wanted, fresh.to(torch.int32), last)
    new = torch.where(held, rows, torch.where((column == child_full[:, None]) & part[parents][:, None], own_page[:, None], -1))
    refs[fresh[wanted]] = 1
    s["buffers"][:, fresh[wanted]] = s["buffers"][:, last[wanted].long()]
    s["page_table"], s["context_lens"] = new, lens[parents]
    return {"page_table": new, "context_lens": s["context_lens"], "refs": refs, "buffers": s["buffers"]}


def _plain_compact(s):
    refs, table = s["refs"].clone(), s["page_table"].clone()
    used = refs > 0
    count = used.sum()
    at = torch.arange(refs.numel(), device=DEV)
    source, target = torch.nonzero(used & (at >= count))[:, 0], torch.nonzero(~used & (at < count))[:, 0]
    place = at.to(torch.int32)
    place[source] = target.to(torch.int32)
    table = torch.where(table >= 0, place[table.long().clamp_min(0)], table)
    refs[target] = refs[source]
    refs[source] = 0
    s["buffers"][:, target] = s["buffers"][:, source]
    return {"page_table": table, "refs": refs, "buffers": s["buffers"]}


def _plain_adapt(s):
    out = s["product"].clone()
    n, r, K = s["a"].shape
    has = (s["ids"][:, None] == torch.arange(n, device=DEV)[None]).float()         # [rows, adapters]
    # all adapters' products, of which a row keeps its own
    t = torch.matmul(s["x"].float(), s["a"].float().view(n * r, K).t()).view(-1, n, r) * (has * s["scales"])[..., None]
    b = s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    return (out.float() + torch.matmul(t.view(-1, n * r), b)).to(out.dtype)


_RUN_OWN = {"store": _own_store, "attend": _own_attend, "fork": _own_fork, "compact": _own_compact, "adapt": _own_adapt}
_RUN_PLAIN = {"store": _plain_store, "attend": _plain_attend, "fork": _plain_fork, "compact": _plain_compact, "adapt": _plain_adapt}


# ------------------------------------------------------------------------------------------------ what it cannot do without
def work(case):
    kind = case["kind"]
    if kind in ("store", "attend"):
        hk, d = case["hk"], case["d"]
        token = 2 * hk * (d / 2 + 2 * ((d + 31) // 32))       # bytes of a token's keys and values in the cache
    if kind == "store":
        tokens, read = case["tokens"], case["tokens"] + case["prefix"]
        return {"bytes": (tokens + read) * (4 * hk * d + token + 8), "flops": 6 * hk * d * (tokens + read)}
    if kind == "attend":
        lengths, nodes, hq = _lengths(case, case["sequences"]), case["nodes"], case["hq"]
        keys = sum(c + nodes for c in lengths)
        pages = sum((c + nodes + case["page"] - 1) // case["page"] for c in lengths)
        pairs = sum(nodes * c + (nodes * nodes if case["masked"] else nodes * (nodes + 1) // 2) for c in lengths)
        words = nodes * ((nodes + 63) // 64) * len(lengths) if case["masked"] else 0
        return {"bytes": keys * token + 4 * d * nodes * hq * len(lengths) + 4 * pages + 8 * words, "flops": 4 * d * hq * pairs}
    if kind == "fork":
        lengths = _lengths(case, case["groups"] * case["beams"])
        parents = _parents(case)
        lengths = [lengths[i // case["beams"] * case["beams"]] for i in range(len(parents))]
        copies = sum(1 for i, p in enumerate(parents) if lengths[p] % case["page"] and p in parents[:i])
        entries = sum((c + case["page"] - 1) // case["page"] for c in lengths)
        return {"bytes": 2 * copies * case["page_bytes"] * case["layers"] + 16 * entries, "flops": 0}
    if kind == "compact":
        used = sum((c + case["page"] - 1) // case["page"] for c in _lengths(case, case["sequences"]))
        pages = int(used * case["spread"]) + 1
        moves = round(used * (pages - used) / pages)           # about: pages in no order
        return {"bytes": 2 * moves * case["page_bytes"] * case["layers"] + 8 * used + 8 * pages, "flops": 0}
    ids = _segments(case)
    rows, each = sum(1 for x in ids if x >= 0), len(set(x for x in ids if x >= 0))
    r, K, N = case["rank"], case["K"], case["N"]
    return {"bytes": 2 * rows * K + 4 * case["rows"] * N + 2 * each * r * (K + N) + 4 * case["rows"], "flops": 2 * rows * r * (K + N)}


# ------------------------------------------------------------------------------------------------ 64-bit results
def _scale_of(m, act):
    """The scale of a group from its largest magnitude, by counting up from what is too small."""
    bits, least = SCALES[act]
    top = torch.floor(torch.log2(m.clamp_min(1e-300) / 7.5)) - 1
    step = ((top - bits + 1).clamp_min(least).long() + 1023 << 52).view(torch.float64)
    n = torch.floor(m / (7.5 * step)).clamp_min(0)
    for _ in range(2):                      # a step for each binade that the guess may lie below
        n = torch.where(n * step * 7.5 < m, n + 1, n)
        wide = n > 2.0 ** bits              # too many bits: twice the step
        step = torch.where(wide, 2 * step, step)
        n = torch.where(wide, torch.floor(m / (7.5 * step)), n)
        n = torch.where(n * step * 7.5 < m, n + 1, n)
    return n * step


def _kept(x, act):
    """What the cache keeps of x [..., d], in 64 bits: group by group."""
    x = x.double()
    parts = []
    for g in range(0, x.shape[-1], 32):
        part = x[..., g:g + 32]
        s = _scale_of(part.abs().amax(-1, keepdim=True), act)
        q = torch.where(s > 0, part / torch.where(s > 0, s, 1.0), 0.0)
        low = torch.floor(q)
        up = (q - low > 0.5) | (q - low == 0.5) & (low % 2 == 1)
        parts.append((low + up.double()).clamp(-7, 7) * s)
    return torch.cat(parts, -1)


def _found(cache, slots, page, heads, d, act):
    """Keys and values in slots [n], from the addresses of their bytes: two [n, heads, d] in 64 bits."""
    S = (d + 31) // 32
    flat = cache.reshape(-1)
    at = (slots // page)[:, None, None] * cache.shape[1] + (torch.arange(heads, device=DEV)[None, :, None] * (page // 16)
                                                          + (slots % page // 16)[:, None, None]) * 576 * S
    token, x = (slots % 16)[:, None, None], torch.arange(d, device=DEV)[None, None]
    at_k = (x % 32 // 8 * 16 + token) * 4 * S + x // 32 * 4 + x % 4
    at_v = 256 * S + (token // 4 * 16 + x % 16) * 4 * S + x // 32 * 4 + token % 4
    at_s = 512 * S + token // 4 * 8 * S + x // 32 * 8 + token % 4 * 2

    def one(codes, scales, second):
        b = flat[at + codes].long()
        q = torch.where(second, (b >> 3 & 7) * (1 - 2 * (b >> 6 & 1)), (b & 7) * (1 - 2 * (b >> 7)))
        bits = flat[at + scales].long() + 256 * flat[at + scales + 1].long()
        return q.double() * (bits - (bits >> 15 << 16)).to(torch.int16).view(DTYPES[act]).double()

    return one(at_k, at_s, x % 8 >= 4), one(at_v, at_s + 32 * S, x % 32 >= 16)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "store":
        k, v = _kept(s["k"], case["act"]), _kept(s["v"], case["act"])
        if case["prefix"]:
            before = _found(s["cache"], s["slots"][:case["prefix"]], case["page"], case["hk"], case["d"], case["act"])
            k, v = torch.cat([before[0], k]), torch.cat([before[1], v])
        return {"k": k, "v": v}
    if kind == "attend":
        nodes, hq, hk, d = case["nodes"], case["hq"], case["hk"], case["d"]
        out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
        words = None if s["mask"] is None else s["mask"].tolist()
        for b, context in enumerate(_lengths(case, case["sequences"])):
            at = torch.arange(context + nodes, device=DEV)
            slots = s["page_table"][b].long()[at // case["page"]] * case["page"] + at % case["page"]
            k, v = _found(s["cache"], slots, case["page"], hk, d, case["act"])
            if words:
                sees = torch.tensor([[(words[b][i][j // 64] >> j % 64 & 1) == 1 for j in range(nodes)] for i in range(nodes)])
            else:
                sees = torch.ones((nodes, nodes), dtype=torch.bool).tril()
            seen = torch.cat([torch.ones((nodes, context), dtype=torch.bool), sees], 1).to(DEV)
            for h in range(hq):
                key, value = k[:, h // (hq // hk)].t().contiguous(), v[:, h // (hq // hk)].contiguous()
                score = (s["q"][b, :, h].double() @ key) / math.sqrt(d)
                score = torch.where(seen, score, -math.inf)
                weight = torch.exp(score - score.amax(1, keepdim=True))
                out[b, :, h] = (weight @ value) / weight.sum(1, keepdim=True)
        return out
    if kind in ("fork", "compact"):
        return None                          # whole numbers
    out = s["product"].double()
    for x in sorted(set(_segments(case))):
        rows = torch.nonzero(s["ids"] == x)[:, 0]
        if x >= 0:
            out[rows] += s["scales"][x].double() * (s["x"][rows].double() @ s["a"][x].double().t().contiguous() @ s["b"][x].double().t().contiguous())
    return out
