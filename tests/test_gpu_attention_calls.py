"""The attention calls on torch tensors: layouts that are taken, arguments that are not."""
import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(params=["native", "python"])
def way(request, monkeypatch):
    """Both ways that a call may go."""
    fq._stream()
    if request.param == "python":
        monkeypatch.setattr(fq, "_native", fq._NoNative())
    return request.param


def _normal(size, dtype, seed):
    return torch.randn(size, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _paged(sequences, tokens, hk, D, page=16):
    pages = (tokens + page - 1) // page
    kc, vc = (_normal((sequences * pages, page, hk, D), F16, i) for i in (1, 2))
    return kc, vc, torch.arange(sequences * pages, dtype=torch.int32).view(sequences, pages)


def test_one_token_of_each_sequence_where_the_qkv_product_leaves_them(way):
    """Queries [sequences, 1, heads, head_dim] as views of wider rows: the stride of the one token says nothing."""
    B, hq, hk, D = 6, 4, 2, 64
    kc, vc, table = _paged(B, 40, hk, D)
    rows = _normal((B, (hq + 2 * hk) * D), F16, 3)
    lens = torch.tensor([39, 5, 0, 17, 22, 30], dtype=torch.int32)
    q = rows[:, :hq * D].reshape(B, 1, hq, D)
    want, tol = ref.tree(q, kc, vc, table, lens, ref.chain(B, 1))
    wide = rows.cuda()
    args = (kc.cuda(), vc.cuda(), table.cuda(), lens.cuda())
    for view in (wide[:, :hq * D].view(B, 1, hq, D), wide.view(B, -1, D)[:, :hq].unsqueeze(1), wide.view(B, -1, D)[:, None, :hq]):
        ref.compare(fq.attention_tree(view, *args), want, tol, str(view.stride()))
    # one sequence, one token, in a tensor of any strides of these two
    one = wide[:1, :hq * D].as_strided((1, 1, hq, D), (3, 5, D, 1))
    ref.compare(fq.attention_tree(one, args[0], args[1], args[2][:1], args[3][:1]), want[:1], tol[:1], "one row")


def test_a_scale_that_binary32_does_not_hold_is_refused(way):
    """(1e-50 is zero there, which stands for 1 / sqrt(head_dim))"""
    kc, vc, table = _paged(1, 40, 2, 64)
    q = _normal((1, 1, 4, 64), F16, 3).cuda()
    lens = torch.tensor([20], dtype=torch.int32).cuda()
    x = _normal((20, 4, 64), F16, 4).cuda()
    for scale in (1e-50, 1e39, 0.0, -1e-50, float("nan"), float("inf")):
        with pytest.raises(fq.FqError):
            fq.attention_tree(q, kc.cuda(), vc.cuda(), table.cuda(), lens, scale=scale)
        with pytest.raises(fq.FqError):
            fq.attention_prompt(x, x, x, [0, 20], scale=scale)
    small = fq.attention_prompt(x, x, x, [0, 20], scale=1e-40)      # (subnormal: all keys weigh the same)
    v = x.double().cpu()
    want = v.cumsum(0) / torch.arange(1, 21)[:, None, None]
    ref.compare(small, want, 2 * ref.UNIT[F16] * v.abs().cumsum(0) / torch.arange(1, 21)[:, None, None] + 2.0 ** -24, "tiny scale")


def test_a_workspace_that_is_not_beside_the_queries_is_refused(way):
    """(its address would be written to)"""
    kc, vc, table = _paged(1, 4000, 2, 64)
    q = _normal((1, 1, 4, 64), F16, 3).cuda()
    args = (q, kc.cuda(), vc.cuda(), table.cuda(), torch.tensor([3900], dtype=torch.int32).cuda())
    need = fq.attention_tree_workspace_bytes(1, 1, 4, 2, 64, table.shape[1], 16)
    rows, keys = _normal((2, 4, 64), F16, 5).cuda(), _normal((3000, 2, 64), F16, 6).cuda()
    need_prompt = fq.attention_prompt_workspace_bytes(4, 2, 64, [0, 2], [0, 3000])
    assert need and need_prompt
    size = max(need, need_prompt)
    for wrong in (torch.empty(size, dtype=torch.uint8), torch.empty(1, dtype=torch.uint8, device="cuda").expand(size),
                  torch.empty(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(fq.FqError):
            fq.attention_tree(*args, workspace=wrong)
        with pytest.raises(fq.FqError):
            fq.attention_prompt(rows, keys, keys, [0, 2], [0, 3000], workspace=wrong)
    good = torch.empty((size + 3) // 4, dtype=torch.float32, device="cuda")
    assert torch.equal(fq.attention_tree(*args, workspace=good), fq.attention_tree(*args))
    assert torch.equal(fq.attention_tree(*args, workspace=good[:1]), fq.attention_tree(*args))       # (too small: as if none were given)
    assert torch.equal(fq.attention_prompt(rows, keys, keys, [0, 2], [0, 3000], workspace=good), fq.attention_prompt(rows, keys, keys, [0, 2], [0, 3000]))


def test_offsets_that_32_bits_do_not_hold_are_refused(way):
    """(2^32 + 3 is no row, and its lower half is one)"""
    x = _normal((9, 4, 64), F16, 4).cuda()
    for wrong in ([0, 2 ** 32 + 3, 9], [0, 2 ** 31, 9], [0, -2 ** 32 + 3, 9]):
        with pytest.raises(fq.FqError):
            fq.attention_prompt(x, x, x, wrong)
        with pytest.raises(fq.FqError):
            fq.attention_prompt(x, x, x, [0, 3, 9], wrong)
    want = fq.attention_prompt(x, x, x, [0, 3, 9])
    for offsets in ((0, 3, 9), torch.tensor([0, 3, 9]), torch.tensor([0, 3, 9], dtype=torch.int32).numpy()):
        assert torch.equal(fq.attention_prompt(x, x, x, offsets), want)
        assert torch.equal(fq.attention_prompt(x, x, x, [0, 3, 9], offsets), want)
