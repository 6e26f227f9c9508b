"""Head norms with rotary positions, attention over prompts and over a paged cache, against 64-bit host implementations."""
import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _normal(size, dtype, seed, sigma=1.0):
    return (torch.randn(size, generator=torch.Generator().manual_seed(seed)) * sigma).to(dtype)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def _banded(shape, dtype):
    """An output with sentinels around it, and a function that checks them."""
    n = 1
    for s in shape:
        n *= s
    whole = torch.full((n + 512,), 123.0, dtype=dtype, device="cuda")

    def check():
        assert bool((whole[:256] == 123.0).all()) and bool((whole[256 + n:] == 123.0).all()), "written outside the output"

    return whole[256:256 + n].view(shape), check


# ------------------------------------------------------------------------------------------------ norms and rotary positions
def _rope_case(tokens, hq, hk, D, rot, dtype, interleaved, norm, seed, cache_page=0, stride=0, k_out=False):
    width = (hq + 2 * hk) * D
    qkv = _normal((tokens, width + stride), dtype, seed, 1.7).cuda()[:, :width]
    host = qkv.cpu().view(tokens, hq + 2 * hk, D)
    wq = (_normal((D,), dtype, seed + 1, 0.2) + 1) if norm else None
    wk = (_normal((D,), dtype, seed + 2, 0.2) + 1) if norm else None
    table = fq.rope_table(50, rot, device="cpu") if rot else None
    positions = torch.randint(-3, 55, (tokens,), generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
    kw, slots = {}, None
    if cache_page:
        pages = tokens // cache_page + 3
        slots = torch.randperm(pages * cache_page, generator=torch.Generator().manual_seed(seed))[:tokens]
        if tokens > 2:
            slots[1], slots[tokens // 2] = -1, pages * cache_page       # padding; outside the cache
        kc, vc = _normal((pages, cache_page, hk, D), dtype, seed + 3), _normal((pages, cache_page, hk, D), dtype, seed + 4)
        kw = {"k_cache": kc.cuda(), "v_cache": vc.cuda(), "slots": slots.cuda()}
    q_out, check_q = _banded((tokens, hq, D), dtype)
    if k_out or not cache_page:
        kw["k_out"], check_k = _banded((tokens, hk, D), dtype)
    q, k = fq.qk_norm_rope(qkv, hq, hk, None if table is None else table.cuda(), positions.cuda(), None if wq is None else wq.cuda(),
                           None if wk is None else wk.cuda(), 1e-5, interleaved, q_out=q_out, **kw)
    torch.cuda.synchronize()
    assert q is q_out
    check_q()
    want, tol = ref.norm_rope(host[:, :hq], wq, 1e-5, table, positions, interleaved)
    ref.compare(q, want, tol, "q")
    want, tol = ref.norm_rope(host[:, hq:hq + hk], wk, 1e-5, table, positions, interleaved)
    if k is not None:
        check_k()
        ref.compare(k, want, tol, "k")
    else:
        assert cache_page
    if cache_page:
        at = torch.tensor([t for t in range(tokens) if 0 <= slots[t] < kc.shape[0] * cache_page], dtype=torch.long)
        k_want, k_tol = kc.double().view(-1, hk, D), torch.zeros((kc.shape[0] * cache_page, hk, D), dtype=torch.float64)
        k_want[slots[at]], k_tol[slots[at]] = want[at], tol[at]
        ref.compare(kw["k_cache"].view(-1, hk, D), k_want, k_tol, "keys in the cache")
        vc.view(-1, hk, D)[slots[at]] = host[at, hq + hk:]
        assert torch.equal(kw["v_cache"].cpu().view(torch.int16), vc.view(torch.int16)), "values in the cache"


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D,rot", [(128, 128), (128, 64), (80, 80), (80, 40), (96, 96), (64, 64), (64, 0), (8, 8), (24, 16), (72, 72), (120, 8)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope(dtype, D, rot, interleaved):
    _rope_case(5, 6, 2, D, rot, dtype, interleaved, True, D + rot)


@pytest.mark.parametrize("tokens,hq,hk,D,norm,page,stride,k_out", [
    (1, 1, 1, 128, True, 1, 0, False), (1, 32, 8, 128, True, 16, 0, False), (9, 32, 8, 128, True, 16, 24, True), (37, 12, 12, 64, False, 7, 8, True),
    (131, 5, 5, 96, True, 64, 0, False), (3, 96, 96, 128, True, 128, 0, False), (300, 3, 1, 80, False, 32, 0, False), (77, 33, 11, 40, True, 5, 8, True),
    (64, 32, 4, 128, True, 0, 1024, True),
])
def test_norm_rope_cache(tokens, hq, hk, D, norm, page, stride, k_out):
    _rope_case(tokens, hq, hk, D, D, BF16, False, norm, tokens + hq, page, stride, k_out)
    _rope_case(tokens, hq, hk, D, D - D // 2 // 8 * 8, F16, True, norm, tokens + hq, page, stride, k_out)


def test_norm_rope_one_weight_alone_and_nothing_to_do():
    D, hq, hk = 64, 4, 2
    qkv = _normal((11, (hq + 2 * hk) * D), F16, 3).cuda()
    w = _normal((D,), F16, 4).cuda()
    q, k = fq.qk_norm_rope(qkv, hq, hk, None, None, q_weight=w)
    heads = qkv.cpu().view(11, hq + 2 * hk, D)
    ref.compare(q, *ref.norm_rope(heads[:, :hq], w.cpu(), 1e-6, None, None, False), "q")
    assert torch.equal(k.cpu(), heads[:, hq:hq + hk])
    q, k = fq.qk_norm_rope(qkv[:0], hq, hk, None, None, q_weight=w)
    assert q.shape == (0, hq, D) and k.shape == (0, hk, D)


def test_norm_rope_into_a_cache_of_heads_first_and_far_pages():
    """Pages [kv_heads, page_size, D], and a page more than 2^32 bytes behind the first."""
    D, hq, hk, page = 128, 2, 2, 8
    qkv = _normal((3, (hq + 2 * hk) * D), BF16, 5).cuda()
    far = 2 ** 31 + 4096
    flat = [torch.zeros(far + hk * page * D, dtype=BF16, device="cuda") for _ in range(2)]
    kc, vc = (f.as_strided((2, page, hk, D), (far, D, page * D, 1)) for f in flat)
    fq.qk_norm_rope(qkv, hq, hk, None, None, k_cache=kc, v_cache=vc, slots=torch.tensor([15, 2, 8], device="cuda"))
    heads = qkv.view(3, hq + 2 * hk, D)
    for cache, first in ((kc, hq), (vc, hq + hk)):
        for t, (n, at) in enumerate(((1, 7), (0, 2), (1, 0))):
            assert torch.equal(cache[n, at], heads[t, first:first + hk])
        assert int((cache != 0).sum()) == int((heads[:, first:first + hk] != 0).sum())


# ------------------------------------------------------------------------------------------------ prompts
def _prompt_case(q_lens, k_lens, hq, hk, D, dtype, seed, sigma=1.5, scale=None, k_pad=0):
    q = _normal((sum(q_lens), hq, D), dtype, seed, sigma)
    k, v = _normal((sum(k_lens), hk, D + k_pad), dtype, seed + 1)[..., :D], _normal((sum(k_lens), hk, D), dtype, seed + 2)
    qo, ko = _offsets(q_lens), _offsets(k_lens)
    out, check = _banded(q.shape, dtype)
    kd = torch.empty((sum(k_lens), hk, D + k_pad), dtype=dtype, device="cuda")[..., :D]
    kd.copy_(k)
    got = fq.attention_prompt(q.cuda(), kd, v.cuda(), qo, None if q_lens == k_lens else ko, scale=scale, out=out)
    torch.cuda.synchronize()
    check()
    want, tol = ref.prompt(q, k, v, qo, ko, scale)
    ref.compare(got, want, tol, f"prompt {q_lens} {k_lens}")
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("lens", [[1], [2], [17, 0, 33], [63, 64, 65], [127, 130]])
def test_prompt(dtype, D, lens):
    _prompt_case(lens, lens, 4, 2, D, dtype, D + len(lens))


@pytest.mark.parametrize("q_lens,k_lens,hq,hk,D", [
    ([1, 1, 1], [1, 200, 64], 8, 1, 128),           # one query: its prefix and itself
    ([5, 70], [300, 71], 3, 3, 64),
    ([129, 3], [513, 1000], 4, 4, 80),
    ([40], [10], 4, 2, 128),                        # fewer keys than queries: rows that see nothing
    ([130, 9, 4], [5, 0, 4], 2, 1, 96),             # no keys at all
    ([0, 0, 3], [7, 0, 3], 2, 2, 64),               # keys without queries
    ([260], [260], 16, 2, 64), ([400], [400], 5, 1, 128), ([300, 200, 100], [300, 200, 100], 6, 6, 96),
    ([2], [3000], 2, 1, 128),                       # few rows, many keys
])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_prompt_prefixes_and_groups(dtype, q_lens, k_lens, hq, hk, D):
    _prompt_case(q_lens, k_lens, hq, hk, D, dtype, sum(k_lens))


def test_prompt_many_sequences():
    lens = [(i * 7) % 11 for i in range(300)]
    _prompt_case(lens, lens, 2, 1, 64, F16, 9)
    keys = [(i * 5) % 13 for i in range(300)]
    _prompt_case(lens, keys, 2, 1, 64, BF16, 10)


@pytest.mark.parametrize("sigma,scale", [(1e-3, None), (30.0, None), (2.0, 1.0), (8.0, 0.01)])
def test_prompt_flat_and_peaked_scores(sigma, scale):
    """Scores all alike, and scores hundreds apart (every numerator but one vanishes)."""
    _prompt_case([150], [150], 2, 2, 64, F16, 21, sigma, scale)
    _prompt_case([150], [150], 2, 2, 128, BF16, 22, sigma, scale)


def test_prompt_growing_scores():
    """The largest score moves with every key: the running maximum is renewed again and again."""
    n, D = 300, 64
    q = torch.ones((n, 2, D), dtype=F16)
    k = (torch.arange(n)[:, None, None] / 20.0).expand(n, 1, D).to(F16).contiguous()
    v = _normal((n, 1, D), F16, 31)
    for keys in (k, -k, k.flip(0).contiguous()):
        got = fq.attention_prompt(q.cuda(), keys.cuda(), v.cuda(), [0, n], scale=1.0)
        ref.compare(got, *ref.prompt(q, keys, v, [0, n], [0, n], 1.0), "growing scores")


def test_prompt_strided_views_of_one_buffer():
    """q, k and v where the QKV product leaves them."""
    rows, hq, hk, D = 190, 6, 3, 64
    qkv = _normal((rows, (hq + 2 * hk) * D), BF16, 41).cuda().view(rows, hq + 2 * hk, D)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:]
    got = fq.attention_prompt(q, k, v, [0, 100, 190])
    ref.compare(got, *ref.prompt(q.cpu(), k.cpu(), v.cpu(), [0, 100, 190], [0, 100, 190]), "views")
    # heads first
    t = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    assert t[0].stride(0) == D
    assert torch.equal(fq.attention_prompt(*t, [0, 100, 190]), got)
    # one row of keys and values for all (stride 0)
    one_k, one_v = k[:1].expand(rows, hk, D), v[:1].expand(rows, hk, D)
    same = fq.attention_prompt(q, one_k, one_v, [0, rows])
    ref.compare(same, *ref.prompt(q.cpu(), one_k.cpu(), one_v.cpu(), [0, rows], [0, rows]), "one row for all")


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_prompt_what_is_not_seen_has_no_part(bad, D):
    """A key and a value that are not finite change the rows that see them and no other."""
    n, at, hq, hk = 140, 77, 4, 2
    q, k, v = (_normal((n, h, D), BF16, 50 + i) for i, h in enumerate((hq, hk, hk)))
    want, tol = ref.prompt(q, k, v, [0, n], [0, n])
    for broken in ("k", "v", "both", "next sequence"):
        k2, v2 = k.clone(), v.clone()
        offsets = [0, n] if broken != "next sequence" else [0, at, n]
        if broken in ("k", "both", "next sequence"):
            k2[at] = bad
        if broken in ("v", "both", "next sequence"):
            v2[at] = bad
        got = fq.attention_prompt(q.cuda(), k2.cuda(), v2.cuda(), offsets).cpu()
        ref.compare(got[:at], want[:at], tol[:at], f"rows before the {bad} in {broken}")
        if broken == "v":
            assert not bool(torch.isfinite(got[at:]).any()), "the rows that see it show it"
            if bad != bad:
                assert bool(torch.isnan(got[at:].float()).all())
        if broken == "both":
            assert bool(torch.isnan(got[at].float()).all())


def test_prompt_lowest_values_and_nothing_written_without_rows():
    n, D = 70, 64
    low = torch.finfo(BF16).min
    q, k, v = (torch.full((n, 1, D), x, dtype=BF16) for x in (1.0, low / 1e4, 1.0))
    v[3] = 2.0
    got = fq.attention_prompt(q.cuda(), k.cuda(), v.cuda(), [0, n])
    ref.compare(got, *ref.prompt(q, k, v, [0, n], [0, n]), "lowest scores")
    out, check = _banded((0, 1, D), BF16)
    fq.attention_prompt(q[:0].cuda(), k[:0].cuda(), v[:0].cuda(), [0, 0], out=out)
    torch.cuda.synchronize()
    check()


def test_prompt_offsets_beyond_32_bits():
    """Keys whose rows are 2^26 values apart: the last lie 2^33 bytes behind the first."""
    n, D = 70, 64
    stride = 2 ** 26
    flat = torch.zeros((n - 1) * stride + D, dtype=F16, device="cuda")
    k = flat.as_strided((n, 1, D), (stride, D, 1))
    host = [_normal((n, 1, D), F16, 60 + i) for i in range(3)]
    k.copy_(host[1])
    got = fq.attention_prompt(host[0].cuda(), k, host[2].cuda(), [0, n])
    ref.compare(got, *ref.prompt(*host, [0, n], [0, n]), "far rows")
    k.copy_(host[2])
    got = fq.attention_prompt(host[0].cuda(), host[1].cuda(), k, [0, n])
    ref.compare(got, *ref.prompt(*host, [0, n], [0, n]), "far values")


def test_prompt_is_deterministic_and_runs_on_the_current_stream():
    lens = [700, 90, 333]
    q, k, v = (_normal((sum(lens), h, 128), BF16, 70 + i).cuda() for i, h in enumerate((8, 2, 2)))
    first = fq.attention_prompt(q, k, v, _offsets(lens))
    for _ in range(3):
        assert torch.equal(fq.attention_prompt(q, k, v, _offsets(lens)), first)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        k2 = k * 1.0
        for _ in range(20):
            k2 = k2 * 1.0
        got = fq.attention_prompt(q, k2, v, _offsets(lens))
    side.synchronize()
    assert torch.equal(got, first)


# ------------------------------------------------------------------------------------------------ trees over a cache
def _cache(lens, nodes, page, hk, D, dtype, seed, spare=3):
    """Caches, a table of shuffled pages (unused entries are out of the cache) and the lengths."""
    used = [max(0, c + nodes + page - 1) // page if c >= 0 else 0 for c in lens]
    pages = sum(used) + spare
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    width = max(used + [1])
    table = torch.full((len(lens), width), 2 ** 31 - 1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    return (_normal((pages, page, hk, D), dtype, seed + 1), _normal((pages, page, hk, D), dtype, seed + 2), table,
            torch.tensor(lens, dtype=torch.int32))


def _random_tree(n, seed):
    gen = torch.Generator().manual_seed(seed)
    return [int(torch.randint(-1, i, (1,), generator=gen)) if i else -1 for i in range(n)]


def _tree_case(lens, nodes, hq, hk, D, page, dtype, masked, seed, scale=None):
    kc, vc, table, context = _cache(lens, nodes, page, hk, D, dtype, seed)
    q = _normal((len(lens), nodes, hq, D), dtype, seed + 3, 1.5)
    sees, mask = ref.chain(len(lens), nodes), None
    if masked == "shared":
        one = ref.from_parents(_random_tree(nodes, seed))
        sees, mask = one[None].expand(len(lens), nodes, nodes), ref.words(one).cuda()
    elif masked:
        sees = torch.stack([ref.from_parents(_random_tree(nodes, seed + b)) for b in range(len(lens))])
        mask = ref.words(sees).cuda()
    out, check = _banded(q.shape, dtype)
    got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), context.cuda(), mask=mask, scale=scale, out=out)
    torch.cuda.synchronize()
    check()
    ref.compare(got, *ref.tree(q, kc, vc, table, context, sees, scale), f"tree {lens} {nodes}")
    return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [8, 40, 64, 72, 80, 96, 104, 128])
@pytest.mark.parametrize("nodes,masked", [(1, False), (9, True)])
def test_tree_head_sizes(dtype, D, nodes, masked):
    _tree_case([0, 1, 31, 150], nodes, 4, 2, D, 16, dtype, masked, D + nodes)


@pytest.mark.parametrize("lens,nodes,hq,hk,D,page,masked", [
    ([0], 1, 1, 1, 128, 16, False),                    # a first token alone
    ([700], 1, 32, 8, 128, 16, False), ([5, 64, 63, 65, 127, 128, 129], 1, 8, 8, 64, 64, False),
    ([-1, 40, 0], 3, 4, 2, 64, 16, True),              # a sequence that is not there
    ([100, 37], 5, 6, 2, 96, 1, True),                 # pages of one token
    ([100, 37], 4, 6, 2, 128, 7, "shared"),            # pages of seven
    ([33, 300], 2, 16, 1, 128, 1000, False),           # pages longer than the context
    ([90, 17], 64, 4, 2, 64, 32, True), ([90, 17], 65, 4, 2, 128, 32, True), ([31], 130, 2, 1, 128, 16, "shared"),
    ([20, 200], 100, 3, 3, 80, 16, False),             # a long chain: the next piece of a prompt
    ([1000, 2], 16, 8, 2, 128, 128, True), ([513], 12, 40, 8, 128, 16, True), ([260], 48, 12, 4, 128, 64, "shared"),
    ([3000, 10, 900], 1, 4, 4, 128, 32, False), ([2500], 1, 28, 4, 128, 16, False), ([40] * 70, 1, 4, 1, 64, 16, False),
    ([129], 1, 33, 1, 64, 16, False), ([150], 1, 65, 1, 128, 16, False), ([150], 1, 200, 1, 64, 16, False),
])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_tree(dtype, lens, nodes, hq, hk, D, page, masked):
    _tree_case(lens, nodes, hq, hk, D, page, dtype, masked, nodes + sum(lens))


@pytest.mark.parametrize("nodes,hq", [(3, 2), (20, 4), (50, 4)])
def test_tree_rows_that_see_nothing(nodes, hq):
    """Masks of zeros over no context: zeros; over a context: the context alone."""
    kc, vc, table, _ = _cache([0, 40], nodes, 16, 2, 64, BF16, 5)
    q = _normal((2, nodes, hq, 64), BF16, 6)
    sees = torch.zeros((2, nodes, nodes), dtype=torch.bool)
    sees[0, 1, 0] = True
    lens = torch.tensor([0, 40], dtype=torch.int32)
    got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), lens.cuda(), mask=ref.words(sees).cuda())
    ref.compare(got, *ref.tree(q, kc, vc, table, lens, sees), "empty masks")
    assert int((got[0, 0] != 0).sum()) == 0 and int((got[0, 2:] != 0).sum()) == 0


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("nodes,hq,hk,D", [(1, 4, 1, 128), (7, 4, 2, 64), (40, 4, 1, 128), (70, 6, 2, 80)])
def test_tree_what_is_not_seen_has_no_part(bad, nodes, hq, hk, D):
    """Not finite: slots behind a sequence's tokens, unused pages, drafted tokens that others do not see."""
    lens = [70, 13, 200]
    kc, vc, table, context = _cache(lens, nodes, 16, hk, D, F16, 8)
    used = torch.zeros(kc.shape[:2], dtype=torch.bool)
    for b, c in enumerate(lens):
        at = torch.arange(c + nodes)
        used[table[b].long()[at // 16], at % 16] = True
    q = _normal((3, nodes, hq, D), F16, 9, 1.5)
    sees = torch.stack([ref.from_parents(_random_tree(nodes, b)) for b in range(3)])
    want, tol = ref.tree(q, kc, vc, table, context, sees)
    kc[~used], vc[~used] = bad, bad
    args = (table.cuda(), context.cuda(), ref.words(sees).cuda())
    ref.compare(fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), *args), want, tol, "behind the tokens")
    if nodes > 1:
        d = nodes - 1
        for b, c in enumerate(lens):
            kc[table[b, (c + d) // 16].long(), (c + d) % 16] = bad
            vc[table[b, (c + d) // 16].long(), (c + d) % 16] = bad
        got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), *args).cpu()
        ref.compare(got[:, :d], want[:, :d], tol[:, :d], "a drafted token")
        assert bool(torch.isnan(got[:, d].float()).all())


def test_tree_context_beyond_the_table_is_not_seen():
    kc, vc, table, _ = _cache([60], 4, 16, 1, 64, F16, 11)
    q = _normal((1, 4, 2, 64), F16, 12)
    for c in (62, 64, 100, 2 ** 31 - 1):
        lens = torch.tensor([c], dtype=torch.int32)
        seen = min(c, 64)
        sees = torch.zeros((1, 4, 64), dtype=torch.bool)
        sees[0, :, :seen] = True
        for i in range(4):
            sees[0, i, seen:min(64, seen + i + 1)] = True
        got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), lens.cuda())
        for h in range(2):
            want, tol = ref.attend(q[0, :, h], kc[table[0].long()].view(-1, 64), vc[table[0].long()].view(-1, 64), sees[0], 0.125)
            ref.compare(got[0, :, h], want, tol, f"context {c}")


@pytest.mark.parametrize("nodes", [1, 40])
def test_tree_pages_of_heads_first_strided_queries_and_far_pages(nodes):
    hk, hq, D, page = 2, 6, 128, 16
    kc, vc, table, context = _cache([50, 20], nodes, page, hk, D, BF16, 14)
    q = _normal((2, nodes, hq, D), BF16, 15)
    want, tol = ref.tree(q, kc, vc, table, context, ref.chain(2, nodes))
    wide = torch.zeros((2, nodes, hq + 4, D), dtype=BF16, device="cuda")
    wide[:, :, :hq] = q.cuda()
    stride = 2 ** 31 // (kc.shape[0] - 1) // 8 * 8 + 4096       # the last page more than 2^32 bytes behind the first
    caches = []
    for c in (kc, vc):
        flat = torch.zeros((c.shape[0] - 1) * stride + hk * page * D, dtype=BF16, device="cuda")
        caches.append(flat.as_strided(c.shape, (stride, D, page * D, 1)))
        caches[-1].copy_(c)
    got = fq.attention_tree(wide[:, :, :hq], *caches, table.cuda(), context.cuda())
    ref.compare(got, want, tol, "far pages")


@pytest.mark.parametrize("nodes,hq", [(1, 8), (6, 8), (40, 8)])
def test_tree_captured_and_replayed_with_other_lengths(nodes, hq):
    lens = [900, 33, 0, 411]
    kc, vc, table, context = _cache(lens, nodes, 16, 2, 128, BF16, 17)
    q = _normal((4, nodes, hq, 128), BF16, 18).cuda()
    kd, vd, td, cd = kc.cuda(), vc.cuda(), table.cuda(), context.cuda()
    eager = fq.attention_tree(q, kd, vd, td, cd)
    need = fq.attention_tree_workspace_bytes(4, nodes, hq, 2, 128, table.shape[1], 16)
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(eager)
    fq.attention_tree(q, kd, vd, td, cd, out=out, workspace=ws)
    assert torch.equal(out, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.attention_tree(q, kd, vd, td, cd, out=out, workspace=ws)
    for now in (lens, [12, 33, 7, 400], lens, [-1, 0, 899, 1]):
        now = [min(x, table.shape[1] * 16 - nodes) for x in now]
        cd.copy_(torch.tensor(now, dtype=torch.int32))
        td.copy_(torch.where(table == 2 ** 31 - 1, torch.zeros_like(table), table))
        want = fq.attention_tree(q, kd, vd, td, cd)
        out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_tree_is_deterministic():
    kc, vc, table, context = (t.cuda() for t in _cache([4000, 17, 2300], 5, 32, 4, 128, F16, 19))
    q = _normal((3, 5, 16, 128), F16, 20).cuda()
    first = fq.attention_tree(q, kc, vc, table, context)
    for _ in range(5):
        assert torch.equal(fq.attention_tree(q, kc, vc, table, context), first)


def test_one_token_is_the_prompts_last_row():
    """The two attentions agree where they compute the same thing."""
    n, hq, hk, D, page = 333, 8, 2, 128, 16
    q, k, v = _normal((n, hq, D), F16, 23), _normal((n, hk, D), F16, 24), _normal((n, hk, D), F16, 25)
    pages = (n + page - 1) // page
    kc, vc = torch.zeros((pages * page, hk, D), dtype=F16), torch.zeros((pages * page, hk, D), dtype=F16)
    kc[:n], vc[:n] = k, v
    table = torch.arange(pages, dtype=torch.int32)[None]
    whole = fq.attention_prompt(q.cuda(), k.cuda(), v.cuda(), [0, n])
    caches = (kc.view(pages, page, hk, D).cuda(), vc.view(pages, page, hk, D).cuda(), table.cuda())
    want, tol = ref.prompt(q, k, v, [0, n], [0, n])
    for nodes in (1, 30):
        got = fq.attention_tree(q[None, n - nodes:].cuda(), *caches, torch.tensor([n - nodes], dtype=torch.int32, device="cuda"))
        ref.compare(got[0], want[n - nodes:], tol[n - nodes:], "tree")
        ref.compare(whole[n - nodes:], want[n - nodes:], tol[n - nodes:], "prompt")


# ------------------------------------------------------------------------------------------------ the native calls and the Python they stand in for
def test_native_calls_and_python_give_the_same(monkeypatch):
    tokens, hq, hk, D = 40, 8, 2, 64
    qkv = _normal((tokens, (hq + 2 * hk) * D), F16, 80).cuda()
    w = _normal((D,), F16, 81).cuda()
    table, positions = fq.rope_table(64, D), torch.arange(tokens, dtype=torch.int32, device="cuda")
    slots = torch.arange(tokens, device="cuda")
    pages = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    lens = torch.tensor([tokens - 4], dtype=torch.int32, device="cuda")
    mask = fq.tree_mask([-1, 0, 0, 1])
    small = torch.empty(16, dtype=torch.uint8, device="cuda")

    def everything():
        kc, vc = (torch.zeros((3, 16, hk, D), dtype=F16, device="cuda") for _ in range(2))
        q, k = fq.qk_norm_rope(qkv, hq, hk, table, positions, w, w)
        q2, none = fq.qk_norm_rope(qkv, hq, hk, table, positions, q_weight=w, k_cache=kc, v_cache=vc, slots=slots)
        assert none is None
        given = torch.empty_like(k)
        assert fq.qk_norm_rope(qkv, hq, hk, None, None, k_weight=w, interleaved=True, k_out=given, k_cache=kc, v_cache=vc, slots=slots)[1] is given
        v = qkv.view(tokens, -1, D)[:, hq + hk:]
        out = torch.empty_like(q)
        assert fq.attention_prompt(q, k, v, [0, 10, tokens], out=out) is out
        p2 = fq.attention_prompt(q[:30], k, v, (0, 10, 30), (0, 10, tokens), scale=0.3, workspace=small)
        drafted = q[tokens - 4:][None]
        t = fq.attention_tree(drafted, kc, vc, pages, lens, mask=mask)
        t2 = fq.attention_tree(drafted, kc, vc, pages, lens, mask=mask[None], scale=1, workspace=small)
        return [q, k, q2, given, kc, vc, out, p2, t, t2, fq.attention_tree(drafted, kc, vc, pages, lens)]

    first = everything()
    with monkeypatch.context() as m:
        m.setattr(fq, "_native", fq._NoNative())
        second = everything()
    for a, b in zip(first, second):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("native", [True, False])
def test_torch_calls_refuse_what_does_not_fit(monkeypatch, native):
    if not native:
        monkeypatch.setattr(fq, "_native", fq._NoNative())
    x = torch.zeros((8, 768), dtype=F16, device="cuda")
    q, k = x.view(8, 6, 128), x.view(8, 6, 128)[:, :2]
    cache = torch.zeros((2, 16, 2, 128), dtype=F16, device="cuda")
    q4, table, lens = x.view(1, 8, 6, 128), torch.zeros((1, 2), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    positions, rope = torch.zeros(8, dtype=torch.int32, device="cuda"), fq.rope_table(4, 128)
    slots = torch.arange(8, device="cuda")
    for call in (
        lambda: fq.attention_prompt(q, k, k, [0, 7]), lambda: fq.attention_prompt(q, k, k, [0, 9]), lambda: fq.attention_prompt(q, k, k, [0, 5, 3, 8]),
        lambda: fq.attention_prompt(q, k, k, [0, 8], [0, 4, 8]), lambda: fq.attention_prompt(q, k[:7], k, [0, 8], [0, 8]),
        lambda: fq.attention_prompt(q, k.bfloat16(), k, [0, 8]), lambda: fq.attention_prompt(q, k, k, [0, 8], scale=-1.0),
        lambda: fq.attention_prompt(q, k, k, [0, 8], scale=0.0), lambda: fq.attention_prompt(q, k, k, [0, 8], out=q[:, :5]),
        lambda: fq.attention_prompt(q, k, k, [0, 8], out=q), lambda: fq.attention_prompt(q[:, :5], k, k, [0, 8]),
        lambda: fq.attention_prompt(q[..., 1:], k[..., 1:], k[..., 1:], [0, 8]),
        lambda: fq.attention_tree(q4, cache, cache[:1], table, lens), lambda: fq.attention_tree(q4, cache, cache.bfloat16(), table, lens),
        lambda: fq.attention_tree(q4, cache, cache, table.long(), lens), lambda: fq.attention_tree(q4, cache, cache, table[0], lens),
        lambda: fq.attention_tree(q4, cache, cache, table, lens.cpu()), lambda: fq.attention_tree(q4, cache, cache, table, lens, mask=slots[:4, None]),
        lambda: fq.attention_tree(q4, cache, cache, table, lens, mask=slots.int()[:, None]), lambda: fq.attention_tree(q4, cache, cache, table, lens, scale=-1.0),
        lambda: fq.attention_tree(q4, cache, cache, table, lens, out=q4), lambda: fq.attention_tree(x.view(1, 8, 12, 64), cache, cache, table, lens),
        lambda: fq.qk_norm_rope(x, 2, 2, rope, None), lambda: fq.qk_norm_rope(x, 2, 2, rope, positions.long()), lambda: fq.qk_norm_rope(x, 2, 3, None, None),
        lambda: fq.qk_norm_rope(x, 2, 2, rope, positions, k_cache=cache, v_cache=cache), lambda: fq.qk_norm_rope(x, 2, 2, rope, positions, q_weight=x[0, :64]),
        lambda: fq.qk_norm_rope(x, 2, 2, rope, positions, k_cache=cache[:, :, :1], v_cache=cache[:, :, :1], slots=slots),
        lambda: fq.qk_norm_rope(x, 2, 2, rope, positions, eps=-1.0), lambda: fq.qk_norm_rope(x, 2, 2, fq.rope_table(4, 136), positions),
        lambda: fq.qk_norm_rope(x, 2, 2, rope, positions, k_cache=cache, v_cache=cache, slots=slots[:4]),
    ):
        with pytest.raises(fq.FqError):
            call()
    with pytest.raises(TypeError):
        fq.attention_tree(q4.float(), cache, cache, table, lens)
    torch.cuda.synchronize()


@pytest.mark.parametrize("count", [2, 15, 16, 17, 33, 63, 64, 65, 127, 128, 200])
def test_tree_many_sequences_find_their_places(count):
    """The line of tiles over few and many sequences, lengths that make units of one tile and of several."""
    lens = [(i * 37) % 230 if i % 5 else -1 if i % 2 else 0 for i in range(count)]
    _tree_case(lens, 1, 2, 1, 64, 16, F16, False, count)
    _tree_case(lens, 3, 8, 2, 64, 16, BF16, True, count)
    if count < 70:
        _tree_case(lens, 40, 2, 1, 64, 16, F16, "shared", count)
        _tree_case(lens, 70, 2, 1, 64, 16, F16, "shared", count)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("lens,nodes,hq,hk,D", [
    ([150, 0, 700], 35, 4, 1, 128), ([90, 333], 48, 8, 2, 128), ([200], 43, 3, 1, 104),        # 129 - 192 rows: three tiles of 64
    ([2100], 40, 4, 1, 128),                                                                   # a unit of many pieces, of few values
    ([544] * 7, 32, 32, 8, 128),                                                               # nine pieces each, of many values
])
def test_tree_rows_in_tiles(dtype, lens, nodes, hq, hk, D):
    _tree_case(lens, nodes, hq, hk, D, 16, dtype, True, nodes + len(lens))


@pytest.mark.parametrize("nodes,hq", [(1, 2), (12, 8), (30, 8), (48, 8)])
def test_tree_of_a_table_for_long_contexts(nodes, hq):
    """Tables for more keys than the caches hold, whose sequences are short."""
    lens, hk, D = [700, 70], 2, 128
    kc, vc, table, context = _cache(lens, nodes, 16, hk, D, BF16, 21)
    wide = torch.cat([table, torch.full((2, 9000), 2 ** 31 - 1, dtype=torch.int32)], 1)
    q = _normal((2, nodes, hq, D), BF16, 22, 1.5)
    sees = torch.stack([ref.from_parents(_random_tree(nodes, b)) for b in range(2)])
    got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), wide.cuda(), context.cuda(), mask=ref.words(sees).cuda())
    ref.compare(got, *ref.tree(q, kc, vc, table, context, sees), "a wide table")
