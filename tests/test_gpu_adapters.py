"""Low-rank adapters of many requests against 64 bits.

A result has at most these errors, u being half a unit in the last place of the 16-bit type (2^-11 binary16, 2^-8 bfloat16), t the inner sums times the
scale, T = sum_k |x a| scale:
  u |out|                           the rounding of the result
  sum_r |b| (K + 8) 2^-24 T         binary32 sums of K products
  sum_r |b| e                       t as two 16-bit numbers: e = 2^-16 |t| (bfloat16: 2^-8 twice, with half a unit's slack), 2^-21 max_r |t| (binary16: 2^-22 of the row's
                                    largest, which the division brings to 1/2 .. 1)
  (2 rank + 8) 2^-24 (sum_r |t b| + |out before|)      the outer sum and the addition, in binary32
  2^-25                             results below the smallest normal binary16
"""
import math

import pytest
import torch

from paper_2308_09723_amd import fq

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16
UNIT = {F16: 2.0 ** -11, BF16: 2.0 ** -8}


def _normal(size, dtype, seed, sigma=1.0):
    return (torch.randn(size, generator=torch.Generator().manual_seed(seed)) * sigma).to(dtype)


def _reference(x, a, b, ids, out, scales):
    want, tol = out.double().clone(), torch.zeros(out.shape, dtype=torch.float64)
    K, rank = x.shape[1], a.shape[1]
    for m, i in enumerate(ids.tolist()):
        if not 0 <= i < a.shape[0]:
            continue
        scale = 1.0 if scales is None else float(scales[i])
        terms = x[m].double()[None] * a[i].double() * scale
        t, big = terms.sum(1), terms.abs().sum(1)
        B = b[i].double()
        want[m] += B @ t
        e = 2.0 ** -16 * t.abs() if x.dtype == BF16 else 2.0 ** -21 * t.abs().max().expand(rank)
        tol[m] = UNIT[x.dtype] * want[m].abs() + B.abs() @ ((K + 8) * 2.0 ** -24 * big + e) \
            + (2 * rank + 8) * 2.0 ** -24 * (B.abs() @ t.abs() + out[m].double().abs()) + 2.0 ** -25
    return want, tol


def _check(rows, N, K, adapters, rank, ids, dtype, seed, scales=True, sigma=1.0, x=None, a=None, b=None, workspace=None):
    x = _normal((rows, K), dtype, seed, sigma) if x is None else x
    a = _normal((adapters, rank, K), dtype, seed + 1, K ** -0.5) if a is None else a
    b = _normal((adapters, N, rank), dtype, seed + 2, 0.3) if b is None else b
    ids = torch.tensor(ids, dtype=torch.int32)
    s = torch.rand(adapters, generator=torch.Generator().manual_seed(seed + 3)) * 2 - 0.5 if scales else None
    whole = torch.full((rows + 2, N + 16), 77.0, dtype=dtype, device="cuda")       # rows in wider ones, sentinels around
    out = whole[1:rows + 1, 8:N + 8]
    before = _normal((rows, N), dtype, seed + 4)
    out.copy_(before)
    wide = torch.empty((rows, K + 24), dtype=dtype, device="cuda")
    wide[:, :K] = x.cuda()
    got = fq.adapters(wide[:, :K], a.cuda(), b.cuda(), ids.cuda(), out, scales=None if s is None else s.cuda(), workspace=workspace)
    assert got is out
    edge = whole.clone()
    edge[1:rows + 1, 8:N + 8] = 77.0
    assert bool((edge == 77.0).all()), "written outside the output"
    want, tol = _reference(x, a, b, ids, before, s)
    got = out.cpu().double()
    none = (ids < 0) | (ids >= adapters)
    assert torch.equal(got[none], before.double()[none])
    fine = want.isfinite()
    off = ((got - want).abs() - tol)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{float(off.max()):.3g} too far"
    return got


CASES = [  # rows, N, K, adapters, rank, ids
    (1, 8, 8, 1, 8, "first"), (1, 1024, 1024, 4, 8, "first"), (3, 776, 520, 2, 24, "turns"), (16, 64, 4096, 16, 16, "turns"), (17, 200, 64, 3, 32, "some"),
    (64, 1536, 2048, 64, 16, "turns"), (64, 96, 40, 5, 128, "any"), (65, 136, 72, 4, 8, "runs"), (63, 256, 264, 3, 72, "some"), (100, 328, 1032, 7, 64, "runs"), (256, 128, 256, 2, 40, "runs"), (257, 264, 512, 5, 16, "runs"),
    (300, 136, 328, 40, 72, "any"), (700, 72, 96, 3, 64, "runs"), (1000, 520, 64, 9, 128, "runs"), (600, 24, 4104, 1, 32, "first"),
    (256, 72, 264, 20, 48, "any"), (512, 64, 128, 3, 8, "runs"), (130, 200, 72, 9, 128, "turns"), (100, 328, 1032, 9, 64, "any"), (255, 1032, 16, 300, 16, "turns"),
]


def _ids(rows, adapters, how, seed):
    gen = torch.Generator().manual_seed(seed)
    if how == "first":
        return [0] * rows
    if how == "turns":
        return [i % adapters for i in range(rows)]
    if how == "some":
        return [i % adapters if i % 3 else -1 for i in range(rows)]
    if how == "any":
        return torch.randint(-1, adapters + 1, (rows,), generator=gen).tolist()
    return [(i * 7 // rows) % (adapters + 1) - 1 for i in range(rows)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,N,K,adapters,rank,how", CASES)
def test_adapters(rows, N, K, adapters, rank, how, dtype):
    _check(rows, N, K, adapters, rank, _ids(rows, adapters, how, rows), dtype, rows + K, scales=rows % 2 == 0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [40, 300])
def test_large_and_small_inner_sums(rows, dtype):
    """Inner sums beyond binary16's range, or far below: the type of t is no limit."""
    ids = [i % 3 for i in range(rows)]
    a = _normal((3, 16, 256), dtype, 5, 1.0) * torch.tensor([200.0, 1.0, 2.0 ** -9]).to(dtype)[:, None, None]
    b = _normal((3, 64, 16), dtype, 6, 1.0) * torch.tensor([2.0 ** -14, 1.0, 200.0]).to(dtype)[:, None, None]
    _check(rows, 64, 256, 3, 16, ids, dtype, 7, sigma=30.0, a=a, b=b)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [20, 320])
def test_others_infinities_and_nans_stay_theirs(rows, dtype):
    ids = [i % 4 for i in range(rows)]
    x, a, b = _normal((rows, 64), dtype, 1), _normal((4, 8, 64), dtype, 2, 0.1), _normal((4, 40, 8), dtype, 3)
    a[1, 3, 7], a[2, 0, 0], b[2, 5, 1], b[1, 39, 0] = math.inf, math.nan, math.nan, -math.inf
    x[3], x[4, 5] = math.nan, math.inf
    got = _check(rows, 40, 64, 4, 8, ids, dtype, 4, x=x, a=a, b=b)
    clean = torch.tensor([i % 4 in (0, 3) and i not in (3, 4) for i in range(rows)])
    assert bool(got[clean].isfinite().all())
    assert bool(got[3].isnan().all()) and not bool(got[4].isfinite().any())


def test_captured_with_other_adapters():
    """A captured call is replayed with other rows, adapters and scales; eager calls in between share its workspace."""
    rows, N, K, rank = 48, 512, 1024, 16
    x, out, ids, scales = torch.empty((rows, K), dtype=BF16, device="cuda"), torch.empty((rows, N), dtype=BF16, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), \
        torch.ones(6, device="cuda")
    a, b = _normal((6, rank, K), BF16, 1, K ** -0.5).cuda(), _normal((6, N, rank), BF16, 2).cuda()
    ws = torch.empty(fq.adapters_workspace_bytes(rows, 6, rank, N, K), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        fq.adapters(x.zero_(), a, b, ids, out.zero_(), scales, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        fq.adapters(x, a, b, ids, out, scales, ws)
    for i in range(5):
        x.copy_(_normal((rows, K), BF16, 10 + i))
        ids.copy_(torch.randint(-1, 6, (rows,), generator=torch.Generator().manual_seed(i)))
        scales.copy_(torch.rand(6, generator=torch.Generator().manual_seed(i)))
        before = _normal((rows, N), BF16, 20 + i).cuda()
        out.copy_(before)
        graph.replay()
        torch.cuda.synchronize()
        eager = fq.adapters(x, a, b, ids, before.clone(), scales, ws)
        assert torch.equal(out, eager)
        want, tol = _reference(x.cpu(), a.cpu(), b.cpu(), ids.cpu(), before.cpu(), scales.cpu())
        assert bool(((eager.cpu().double() - want).abs() <= tol).all())


@pytest.mark.parametrize("rows", [3, 300])
def test_adapters_beyond_four_gigabytes(rows):
    N, rank, count = 1 << 18, 128, 70
    b = torch.empty((count, N, rank), dtype=F16, device="cuda")
    for i in range(count):
        b[i].fill_(0.0)
    x, a = _normal((rows, 16), F16, 1), _normal((count, rank, 16), F16, 2)
    at = torch.randint(0, N, (40,), generator=torch.Generator().manual_seed(3))
    at[0], at[1] = 0, N - 1
    used = [0, 66, 69]       # (66 * 2^18 * 128 values of two bytes)
    part = _normal((3, 40, rank), F16, 4)
    for i, id in enumerate(used):
        b[id, at.cuda()] = part[i].cuda()
        part[i] = b[id, at.cuda()].cpu()
    ids = torch.tensor([used[i % 3] for i in range(rows)], dtype=torch.int32)
    out = torch.zeros((rows, N), dtype=F16, device="cuda")
    fq.adapters(x.cuda(), a.cuda(), b, ids.cuda(), out)
    small = torch.zeros((count, 40, rank), dtype=F16)
    small[used] = part
    want, tol = _reference(x, a, small, ids, torch.zeros((rows, 40), dtype=F16), None)
    assert bool(((out[:, at.cuda()].cpu().double() - want).abs() <= tol).all())
    other = torch.ones(N, dtype=torch.bool, device="cuda")
    other[at.cuda()] = False
    assert not bool((out * other).any())


@pytest.mark.parametrize("rows", [20, 600])
def test_inner_sums_that_bfloat16_would_round_to_infinity(rows):
    """t between bfloat16's largest number and binary32's, exactly the scale here."""
    x, a = torch.zeros((rows, 64), dtype=BF16), torch.zeros((1, 8, 64), dtype=BF16)
    x[:, 0], a[0, :, 0] = 1.0, torch.tensor([1.0, -1.0] * 4)
    b = (torch.arange(16 * 8).view(1, 16, 8) % 11 * 2.0 ** -128).to(BF16)
    before = _normal((rows, 16), BF16, 1)
    scales = torch.tensor([3.4e38])
    assert float(scales[0]) > torch.finfo(BF16).max
    got = fq.adapters(x.cuda(), a.cuda(), b.cuda(), torch.zeros(rows, dtype=torch.int32).cuda(), before.cuda(), scales.cuda()).cpu().double()
    want, tol = _reference(x, a, b, torch.zeros(rows, dtype=torch.int32), before, scales)
    assert bool(((got - want).abs() <= tol).all())
