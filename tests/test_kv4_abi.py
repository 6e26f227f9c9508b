"""What the calls of a cache held in 4 bits refuse, before anything is launched (no GPU), and the quantiser's definition."""
import ctypes
import math

import pytest
import torch

from paper_2308_09723_amd import fq

import kv4_util as ref

BAD, NOT_HERE, SCRATCH = fq.FQ_ERR_INVALID_ARG, fq.FQ_ERR_UNSUPPORTED, fq.FQ_ERR_WORKSPACE
P = 1 << 20      # an address that no check follows


def _pages(**kw):
    a = dict(data=P << 8, pages=10, page_size=16, page_stride=2 * 2304)
    a.update(kw)
    return fq.Kv4Pages(*a.values())


def test_page_bytes():
    assert fq.kv4_page_bytes(16, 2, 128) == 2 * 16 * 2 * (64 + 8)
    assert fq.kv4_page_bytes(64, 3, 80) == fq.kv4_page_bytes(64, 3, 96) == 3 * 64 * 2 * (48 + 6)
    assert fq.kv4_page_bytes(48, 1, 8) == 48 * 2 * (16 + 2)
    for bad in ((0, 2, 128), (8, 2, 128), (24, 2, 128), (16, 0, 128), (16, 2, 0), (16, 2, 136), (16, 2, 12), (-16, 2, 128)):
        assert fq.kv4_page_bytes(*bad) == 0


def _write(**kw):
    a = dict(k=fq.Heads(P, 256, 128), v=fq.Heads(P << 1, 256, 128), act=0, tokens=5, hk=2, D=128, cache=_pages(), slots=P << 2)
    a.update(kw)
    return fq.kv4_write_raw(*a.values())


SHAPES = [
    (dict(act=2), BAD), (dict(tokens=-1), BAD), (dict(hk=0), BAD), (dict(D=0), BAD), (dict(cache=None), BAD), (dict(cache=_pages(data=0)), BAD),
    (dict(cache=_pages(pages=0)), BAD), (dict(cache=_pages(page_size=0)), BAD), (dict(cache=_pages(page_stride=2 * 2304 - 16)), BAD),
    (dict(cache=_pages(page_stride=-4608)), BAD), (dict(D=12), NOT_HERE), (dict(D=136), NOT_HERE), (dict(tokens=1 << 24), NOT_HERE),
    (dict(cache=_pages(page_size=24)), NOT_HERE), (dict(cache=_pages(page_size=8)), NOT_HERE), (dict(cache=_pages(data=(P << 8) + 8)), NOT_HERE),
    (dict(cache=_pages(page_stride=4616)), NOT_HERE), (dict(cache=_pages(pages=1 << 28)), NOT_HERE), (dict(cache=_pages(page_stride=1 << 60)), NOT_HERE),
    (dict(hk=4097), NOT_HERE),
]


@pytest.mark.parametrize("change,status", SHAPES + [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(slots=None), BAD), (dict(k=fq.Heads(0, 256, 128)), BAD), (dict(v=fq.Heads(P, -256, 128)), BAD),
    (dict(k=fq.Heads(P << 8, 256, 128)), BAD), (dict(v=fq.Heads((P << 8) + 10 * 4608 - 16, 256, 128)), BAD), (dict(slots=P << 8), BAD),
    (dict(k=fq.Heads(P + 2, 256, 128)), NOT_HERE), (dict(v=fq.Heads(P, 256, 132)), NOT_HERE), (dict(k=fq.Heads(P, 1 << 60, 128)), NOT_HERE),
])
def test_write_refuses(change, status):
    assert _write(**change) == status


def _read(**kw):
    a = dict(cache=_pages(), act=1, tokens=5, hk=2, D=128, slots=P << 2, k=P, v=P << 1)
    a.update(kw)
    return fq.kv4_read_raw(*a.values())


@pytest.mark.parametrize("change,status", SHAPES + [
    (dict(k=None), BAD), (dict(v=None), BAD), (dict(slots=None), BAD), (dict(k=P << 1), BAD), (dict(v=P + 16), BAD), (dict(k=P << 8), BAD),
    (dict(v=P << 2), BAD), (dict(k=P + 2), NOT_HERE), (dict(v=P + 8), NOT_HERE),
])
def test_read_refuses(change, status):
    assert _read(**change) == status


def test_no_tokens_is_no_work():
    assert _write(tokens=0, k=None, v=None, slots=None) == fq.FQ_OK
    assert _read(tokens=0, k=None, v=None, slots=None) == fq.FQ_OK


def _tree(**kw):
    a = dict(q=fq.Heads(P, 512, 128), act=1, B=3, n=5, hq=4, hk=2, D=128, cache=_pages(), table=P << 3, width=4, lens=P << 4, mask=None, mask_stride=0,
             scale=0.0, out=P << 5)
    ws = kw.pop("ws", P << 10)
    a.update(kw)
    page = a["cache"].page_size if a["cache"] else 16
    need = fq.attention_tree_kv4_workspace_bytes(a["B"], a["n"], a["hq"], a["hk"], a["D"], a["width"], page)
    return fq.attention_tree_kv4_raw(*a.values(), ws, need)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), BAD), (dict(cache=None), BAD), (dict(table=None), BAD), (dict(lens=None), BAD), (dict(out=None), BAD), (dict(act=3), BAD),
    (dict(B=-1), BAD), (dict(n=-1), BAD), (dict(width=-1), BAD), (dict(hk=3), BAD), (dict(hq=0), BAD), (dict(scale=-1.0), BAD), (dict(scale=float("nan")), BAD),
    (dict(mask=P << 6, mask_stride=4), BAD), (dict(mask_stride=-1), BAD), (dict(out=P), BAD), (dict(out=P << 8), BAD), (dict(out=P << 3), BAD), (dict(out=P << 4), BAD),
    (dict(cache=_pages(data=0)), BAD), (dict(cache=_pages(pages=0)), BAD), (dict(cache=_pages(page_stride=100)), BAD), (dict(cache=_pages(page_size=24)), NOT_HERE),
    (dict(cache=_pages(data=P + 4)), NOT_HERE), (dict(D=100), NOT_HERE), (dict(out=(P << 5) + 4), NOT_HERE), (dict(q=fq.Heads(P + 2, 512, 128)), NOT_HERE),
    (dict(B=65537), NOT_HERE), (dict(n=(1 << 20) + 1), NOT_HERE), (dict(width=1 << 28), NOT_HERE), (dict(width=4000, ws=None), SCRATCH),
])
def test_attention_refuses(change, status):
    assert _tree(**change) == status


def test_nothing_to_attend_to_is_no_work():
    assert _tree(B=0, q=None, table=None, lens=None, out=None) == fq.FQ_OK
    assert _tree(n=0, q=None, out=None) == fq.FQ_OK
    assert fq.attention_tree_kv4_workspace_bytes(3, 5, 4, 2, 128, 400, 24) == 0
    assert fq.attention_tree_kv4_workspace_bytes(3, 5, 4, 2, 128, 400, 32) > 0


def test_torch_calls_refuse():
    k = torch.zeros((4, 2, 64), dtype=torch.float16)
    with pytest.raises(fq.FqError):
        fq.kv4_write(k, k, torch.zeros((2, fq.kv4_page_bytes(16, 2, 64)), dtype=torch.uint8), 16, torch.arange(4))       # host memory
    with pytest.raises(TypeError):
        fq.kv4_write(k.float(), k.float(), torch.zeros((2, 8), dtype=torch.uint8), 16, torch.arange(4))
    with pytest.raises(fq.FqError):
        fq.kv4_cache(4, 24, 2, 64, device="cpu")
    assert tuple(fq.kv4_cache(4, 32, 2, 64, device="cpu").shape) == (4, fq.kv4_page_bytes(32, 2, 64))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_what_a_cache_stands_for_is_a_value_of_its_type(dtype):
    """Code times scale is exact, no value is further off than half a scale but the one that 7.5 scales are for, and no smaller scale does."""
    bits, least = ref.SCALES[dtype]
    gen = torch.Generator().manual_seed(3)
    x = torch.cat([torch.randn((60, 96), generator=gen) * 10.0 ** torch.randint(-9, 5, (60, 1), generator=gen).float(), torch.zeros((1, 96))]).to(dtype)
    q, s, value = ref.quantise(x)
    assert torch.equal(value.to(dtype).double(), value)
    each = s.repeat_interleave(32, 1)[:, :96]
    assert bool(((value - x.double()).abs() <= each / 2).all()) and bool((s[-1] == 0).all()) and bool((q.abs() <= 7).all())
    m = x.double().abs().view(61, 3, 32).amax(2)
    assert bool((7.5 * s >= m).all())
    for top, scale in zip(m.flatten().tolist(), s.flatten().tolist()):
        if scale > 0:
            e = max(math.frexp(scale)[1] - bits - (math.frexp(scale)[0] == 0.5), least)      # the next smaller scale
            assert 7.5 * (scale - 2.0 ** e) < top


@pytest.mark.parametrize("D", [8, 32, 40, 80, 96, 128])
def test_every_token_has_bytes_of_its_own(D):
    slots = torch.arange(64)
    keys, _, values, _, key_scales, value_scales = ref.places(slots, 32, 3, D)
    owner = {}
    for x in (keys, values, key_scales, value_scales, key_scales + 1, value_scales + 1):
        for n in range(64):
            for at in x[n].flatten().tolist():
                assert owner.setdefault(at, n) == n and 0 <= at < 2 * fq.kv4_page_bytes(32, 3, D)
