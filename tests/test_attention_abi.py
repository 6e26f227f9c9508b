"""What the attention calls refuse, before anything is launched (no GPU), and their host helpers."""
import ctypes

import pytest

from paper_2308_09723_amd import fq

BAD, NOT_HERE, SCRATCH = fq.FQ_ERR_INVALID_ARG, fq.FQ_ERR_UNSUPPORTED, fq.FQ_ERR_WORKSPACE
P = 1 << 20      # an address that no check follows


def _pages(**kw):
    a = dict(k=P << 8, v=P << 9, pages=10, page_size=16, page_stride=16 * 256, token_stride=256, head_stride=128)
    a.update(kw)
    return fq.KvPages(*a.values())


def _rope(**kw):
    a = dict(qkv=P, act=0, tokens=4, stride=768, hq=2, hk=2, D=128, qw=P << 1, kw=P << 1, eps=1e-6, table=P << 2, rows=10, rot=128,
             inter=0, pos=P << 3, q=P << 4, k=P << 5, cache=_pages(), slots=P << 6)
    a.update(kw)
    return fq.qk_norm_rope_raw(*a.values())


@pytest.mark.parametrize("change,status", [
    (dict(qkv=None), BAD), (dict(q=None), BAD), (dict(act=2), BAD), (dict(tokens=-1), BAD), (dict(stride=760), BAD), (dict(hq=0), BAD),
    (dict(hk=0), BAD), (dict(hq=3), BAD), (dict(D=0), BAD), (dict(eps=-1.0), BAD), (dict(eps=float("nan")), BAD), (dict(eps=float("inf")), BAD),
    (dict(table=None), BAD), (dict(rows=0), BAD), (dict(pos=None), BAD), (dict(rot=-8), BAD), (dict(rot=136), BAD),
    (dict(k=None, cache=None, slots=None), BAD), (dict(slots=None), BAD), (dict(cache=None), BAD), (dict(q=P + 16), BAD), (dict(k=P + 16), BAD),
    (dict(k=P << 4), BAD), (dict(cache=_pages(k=0)), BAD), (dict(cache=_pages(pages=0)), BAD), (dict(cache=_pages(page_size=0)), BAD),
    (dict(cache=_pages(token_stride=64)), BAD), (dict(cache=_pages(head_stride=-128)), BAD),
    (dict(rot=4), NOT_HERE), (dict(D=136, stride=816), NOT_HERE), (dict(D=100, rot=96, stride=600), NOT_HERE), (dict(tokens=1 << 25), NOT_HERE),
    (dict(stride=772), NOT_HERE), (dict(qkv=P + 8), NOT_HERE), (dict(q=(P << 4) + 2), NOT_HERE), (dict(qw=P + 2), NOT_HERE),
    (dict(cache=_pages(k=P + 2)), NOT_HERE), (dict(cache=_pages(head_stride=132)), NOT_HERE), (dict(cache=_pages(pages=1 << 30)), NOT_HERE),
    (dict(hq=5000, hk=2500, stride=10000 * 128), NOT_HERE),
])
def test_norm_rope_refuses(change, status):
    assert _rope(**change) == status


def test_no_tokens_is_no_work():
    assert _rope(tokens=0, qkv=None, q=None) == fq.FQ_OK
    assert _rope(tokens=0, act=7) == BAD


def _prompt(**kw):
    a = dict(q=fq.Heads(P, 512, 128), k=fq.Heads(P << 1, 256, 128), v=fq.Heads(P << 2, 256, 128), act=0, hq=4, hk=2, D=128, qo=[0, 3, 9], ko=None,
             scale=0.0, out=P << 4)
    a.update(kw)
    need = fq.attention_prompt_workspace_bytes(a["hq"], a["hk"], a["D"], a["qo"], a["ko"])
    return fq.attention_prompt_raw(*a.values(), P << 10, need)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(k=None), BAD), (dict(v=None), BAD), (dict(out=None), BAD), (dict(q=fq.Heads(0, 512, 128)), BAD),
    (dict(act=-1), BAD), (dict(hq=0), BAD), (dict(hk=3), BAD), (dict(D=0), BAD), (dict(qo=[1, 3, 9]), BAD), (dict(qo=[0, 5, 3]), BAD),
    (dict(qo=[0, -1, 3]), BAD), (dict(ko=[0, 5, 4]), BAD), (dict(ko=[2, 5, 7]), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD),
    (dict(scale=float("inf")), BAD), (dict(out=P), BAD), (dict(out=P << 1), BAD), (dict(out=P << 2), BAD), (dict(q=fq.Heads(P, -512, 128)), BAD),
    (dict(D=136), NOT_HERE), (dict(D=12), NOT_HERE), (dict(hq=8192), NOT_HERE), (dict(q=fq.Heads(P + 4, 512, 128)), NOT_HERE),
    (dict(k=fq.Heads(P << 1, 260, 128)), NOT_HERE), (dict(v=fq.Heads(P << 2, 256, 132)), NOT_HERE), (dict(out=(P << 4) + 8), NOT_HERE),
    (dict(qo=[0] * 65538), NOT_HERE), (dict(q=fq.Heads(P, 1 << 60, 128)), NOT_HERE),
])
def test_prompt_refuses(change, status):
    assert _prompt(**change) == status


def test_prompt_without_rows_is_no_work():
    assert _prompt(qo=[0], q=None, k=None, v=None, out=None) == fq.FQ_OK
    assert _prompt(qo=[0, 0, 0], ko=[0, 4, 9], q=None, out=None) == fq.FQ_OK
    assert fq.attention_prompt_workspace_bytes(4, 3, 128, [0, 4]) == 0 and fq.attention_prompt_workspace_bytes(4, 2, 128, [1, 4]) == 0


def _tree(**kw):
    a = dict(q=fq.Heads(P, 512, 128), act=1, B=3, n=5, hq=4, hk=2, D=128, cache=_pages(), table=P << 3, width=4, lens=P << 4, mask=None, mask_stride=0,
             scale=0.0, out=P << 5)
    a.update(kw)
    need = fq.attention_tree_workspace_bytes(a["B"], a["n"], a["hq"], a["hk"], a["D"], a["width"], a["cache"].page_size if a["cache"] else 16)
    return fq.attention_tree_raw(*a.values(), P << 10, need)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(cache=None), BAD), (dict(table=None), BAD), (dict(lens=None), BAD), (dict(out=None), BAD), (dict(act=3), BAD),
    (dict(B=-1), BAD), (dict(n=-1), BAD), (dict(hq=5), BAD), (dict(width=-1), BAD), (dict(mask=P << 6, mask_stride=4), BAD), (dict(mask_stride=-1), BAD),
    (dict(scale=-0.5), BAD), (dict(scale=float("nan")), BAD), (dict(out=P), BAD), (dict(cache=_pages(v=0)), BAD), (dict(cache=_pages(page_size=-1)), BAD),
    (dict(cache=_pages(page_stride=64)), BAD),
    (dict(D=256), NOT_HERE), (dict(D=20), NOT_HERE), (dict(B=1 << 17), NOT_HERE), (dict(n=1 << 21), NOT_HERE), (dict(B=65536, n=1024), NOT_HERE),
    (dict(width=1 << 28), NOT_HERE), (dict(q=fq.Heads(P + 8, 512, 128)), NOT_HERE), (dict(cache=_pages(token_stride=260)), NOT_HERE),
    (dict(cache=_pages(v=P + 2)), NOT_HERE), (dict(out=P + 2), NOT_HERE),
])
def test_tree_refuses(change, status):
    assert _tree(**change) == status


def test_tree_without_rows_is_no_work():
    assert _tree(B=0, q=None) == fq.FQ_OK and _tree(n=0, q=None) == fq.FQ_OK
    assert fq.attention_tree_workspace_bytes(3, 5, 4, 3, 128, 4, 16) == 0


def test_a_workspace_too_small_is_refused():
    """(where one is needed at all)"""
    qo, ko = [0, 2], [0, 20000]
    need = fq.attention_prompt_workspace_bytes(4, 2, 128, qo, ko)
    if need:
        rows = fq.Heads(P, 512, 128), fq.Heads(P << 3, 256, 128), fq.Heads(P << 6, 256, 128)
        assert fq.attention_prompt_raw(*rows, 0, 4, 2, 128, qo, ko, 0.0, P << 10, P << 11, need - 1) == SCRATCH
        assert fq.attention_prompt_raw(*rows, 0, 4, 2, 128, qo, ko, 0.0, P << 10, None, need) == SCRATCH
    need = fq.attention_tree_workspace_bytes(2, 1, 8, 2, 128, 512, 16)
    if need:
        args = (fq.Heads(P, 1024, 128), 0, 2, 1, 8, 2, 128, _pages(), P << 3, 512, P << 4, None, 0, 0.0, P << 5)
        assert fq.attention_tree_raw(*args, P << 10, need - 1) == SCRATCH
        assert fq.attention_tree_raw(*args, None, need) == SCRATCH


def test_structs_are_the_headers():
    assert ctypes.sizeof(fq.Heads) == 24 and ctypes.sizeof(fq.KvPages) == 56
    assert fq.KvPages.page_stride.offset == 32


def test_tree_mask():
    m = fq.tree_mask([-1, 0, 0, 1, -1], device="cpu")
    assert m.tolist() == [[1], [3], [5], [11], [16]]
    wide = fq.tree_mask([-1] + list(range(69)), device="cpu")
    assert wide.shape == (70, 2) and wide[69].tolist() == [-1, 63] and wide[63].tolist() == [-1, 0] and wide[62].tolist() == [2 ** 63 - 1, 0]
    assert fq.tree_mask([[-1, 0], [-1, -1]], device="cpu").tolist() == [[[1], [3]], [[1], [2]]]
    for wrong in ([0], [-1, 1], [-2]):
        with pytest.raises(ValueError):
            fq.tree_mask(wrong, device="cpu")


def test_rope_table():
    import math
    t = fq.rope_table(7, 8, base=100.0, device="cpu")
    assert t.shape == (7, 8)
    for p in range(7):
        for i in range(4):
            angle = p * 100.0 ** (-2 * i / 8)
            assert abs(float(t[p, i]) - math.cos(angle)) <= 2 ** -24 and abs(float(t[p, 4 + i]) - math.sin(angle)) <= 2 ** -24


def test_torch_calls_refuse_host_tensors_and_shapes_that_do_not_fit():
    import torch
    x = torch.zeros((4, 768), dtype=torch.float16)
    for call in (lambda: fq.qk_norm_rope(x, 2, 2, None, None), lambda: fq.attention_prompt(*[x.view(4, 6, 128)] * 3, [0, 4]),
                 lambda: fq.attention_tree(x.view(1, 4, 6, 128), *[x.view(1, 4, 6, 128)] * 2, None, None)):
        with pytest.raises(fq.FqError):
            call()
    with pytest.raises(TypeError):
        fq.attention_prompt(*[x.view(4, 6, 128).float()] * 3, [0, 4])
