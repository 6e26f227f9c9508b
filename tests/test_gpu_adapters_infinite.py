"""Adapters whose inner sums are infinite: infinities where the formula has them, NaNs only where it has them."""
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
