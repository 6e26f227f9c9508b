"""Adapters whose inner sums or weights are infinite: infinities where the formula has them, NaNs only where it has them."""
import math

import pytest
import torch

from paper_2308_09723_amd import fq

from test_gpu_adapters import BF16, F16, _normal, _reference

pytestmark = pytest.mark.gpu


def _check(x, a, b, ids, before, scales=None):
    got = fq.adapters(x.cuda(), a.cuda(), b.cuda(), ids.cuda(), before.cuda(), None if scales is None else scales.cuda()).cpu().double()
    want, tol = _reference(x, a, b, ids, before, scales)
    want = torch.where(want.abs() > torch.finfo(x.dtype).max, want.sign() * math.inf, want)
    assert torch.equal(got.isnan(), want.isnan())
    assert torch.equal(got[want.isinf()], want[want.isinf()])
    fine = want.isfinite()
    assert bool(((got - want).abs() <= tol)[fine].all())
    return want


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows", [20, 600])
def test_an_infinite_inner_sum_beside_large_ones(rows, dtype):
    """t = (infinity, 90000, -600, 0 ...): sums that binary16 does not hold stay finite beside an infinite one."""
    x, a = torch.zeros((rows, 64), dtype=dtype), torch.zeros((2, 8, 64), dtype=dtype)
    x[:, 0], x[:, 1] = 1.0, 300.0
    a[0, 0, 0], a[0, 1, 1], a[0, 2, 1] = math.inf, 300.0, -2.0
    a[1, 0, 1], a[1, 1, 1] = 2.0 ** -10, 200.0
    b = torch.ones((2, 40, 8), dtype=dtype)
    b[:, ::2, 0] = -1.0
    b[:, :, 1] = (torch.arange(40) % 3 - 1).to(dtype) * 0.5
    b[0, 7, 0] = 0.0        # (an infinity times zero)
    ids = torch.arange(rows, dtype=torch.int32) % 3 - 1
    want = _check(x, a, b, ids, _normal((rows, 40), dtype, 1))
    assert int(want.isinf().sum()) == 39 * int((ids == 0).sum()) and int(want.isnan().sum()) == int((ids == 0).sum())


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rows,rank", [(20, 8), (600, 8), (300, 72), (2000, 40)])
def test_infinite_weights(rows, rank, dtype):
    """Weights of B: inner sums that 16 bits hold exactly, and such that they do not; infinities of both signs, one times an inner sum of zero, one beside a NaN."""
    x, a = _normal((rows, 64), dtype, 1), _normal((3, rank, 64), dtype, 2, 0.2)
    a[0] = 0.0
    a[0, :, 0] = torch.tensor([1.0, 2.0, 0.0, -3.0] * (rank // 4)).to(dtype)
    x[:, 0] = torch.where(torch.arange(rows) % 2 == 0, 1.0, -1.0).to(dtype)
    b = _normal((3, 264, rank), dtype, 3)
    for i in (0, 1):
        b[i, 5, 1], b[i, 130, 0], b[i, 263, 7] = math.inf, -math.inf, math.inf
        b[i, 9, 2], b[i, 12, rank - 1] = math.inf, math.inf          # (adapter 0: zero times the first)
        b[i, 77, 0], b[i, 77, 3] = math.inf, math.inf                # (adapter 0: an infinity less another)
        b[i, 200, 1], b[i, 200, 5] = math.inf, math.nan
    ids = torch.arange(rows, dtype=torch.int32) * 4 // rows - 1
    want = _check(x, a, b, ids, _normal((rows, 264), dtype, 4))
    assert int(want.isinf().sum()) >= 4 * int((ids == 0).sum()) and bool(want[ids == 2].isfinite().all())


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_infinite_inner_sums_and_weights(dtype):
    """Both at once, and outputs that were infinite before."""
    rows = 600
    x, a, b = _normal((rows, 64), dtype, 1), _normal((2, 8, 64), dtype, 2), _normal((2, 136, 8), dtype, 3)
    x[:, 0] = 1.0
    a[0, 3, 0], b[0, 4, 3], b[0, 135, 3] = math.inf, math.inf, -math.inf
    before = _normal((rows, 136), dtype, 4)
    before[::7, 4], before[::7, 20], before[1::7, 6] = -math.inf, math.inf, math.nan
    _check(x, a, b, torch.arange(rows, dtype=torch.int32) % 2, before)
