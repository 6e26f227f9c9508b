"""What the calls of pages that sequences share refuse, before anything is launched (no GPU)."""
import pytest
import torch

from paper_2308_09723_amd import fq

BAD, NOT_HERE, SCRATCH = fq.FQ_ERR_INVALID_ARG, fq.FQ_ERR_UNSUPPORTED, fq.FQ_ERR_WORKSPACE
P = 1 << 20      # an address that no check follows


def _buffers(*changes):
    out = (fq.PageBuffer * len(changes))()
    for i, kw in enumerate(changes):
        a = dict(data=P << 10, count=2, stride=1 << 20, page_stride=4096, page_bytes=4096)
        a.update(kw)
        out[i] = fq.PageBuffer(*a.values())
    return out


BUFFERS = [(_buffers(dict(data=0)), BAD), (_buffers({}, dict(page_bytes=0)), BAD), (_buffers(dict(page_stride=4080)), BAD), (_buffers(dict(count=-1)), BAD),
           (_buffers(dict(stride=-16)), BAD), (_buffers(dict(page_stride=-4096)), BAD), (_buffers(dict(data=(P << 10) + 8)), NOT_HERE),
           (_buffers(dict(page_bytes=4088)), NOT_HERE), (_buffers(dict(page_stride=4104)), NOT_HERE), (_buffers(dict(stride=24)), NOT_HERE),
           (_buffers(dict(stride=1 << 60)), NOT_HERE), (_buffers(dict(page_stride=1 << 60)), NOT_HERE), (_buffers(dict(count=1 << 21)), NOT_HERE)]


def _copy(**kw):
    a = dict(buffers=_buffers({}), pages=10, src=P, dst=P << 1, moves=3)
    a.update(kw)
    return fq.pages_copy_raw(*a.values())


@pytest.mark.parametrize("change,status", [(dict(buffers=b), s) for b, s in BUFFERS] + [
    (dict(pages=-1), BAD), (dict(moves=-1), BAD), (dict(src=None), BAD), (dict(dst=None), BAD), (dict(src=P << 10), BAD), (dict(dst=(P << 10) + (1 << 20)), BAD),
    (dict(src=P + 2), NOT_HERE), (dict(pages=1 << 31), NOT_HERE), (dict(moves=1 << 31), NOT_HERE),
])
def test_copy_refuses(change, status):
    assert _copy(**change) == status


POOL = [(dict(refs=None), BAD), (dict(pages=-1), BAD), (dict(page=0), BAD), (dict(table=None), BAD), (dict(rows=-1), BAD), (dict(width=-1), BAD),
        (dict(lens=None), BAD), (dict(refs=P << 1), BAD), (dict(lens=P << 1), BAD), (dict(lens=P), BAD), (dict(rows=8193), NOT_HERE),
        (dict(width=(1 << 17) + 1), NOT_HERE), (dict(pages=1 << 31), NOT_HERE), (dict(refs=P + 2), NOT_HERE), (dict(table=(P << 1) + 1), NOT_HERE)]


def _take(**kw):
    a = dict(refs=P, pages=10, page=16, table=P << 1, rows=3, width=4, lens=P << 2, wanted=P << 3)
    a.update(kw)
    return fq.pages_take_raw(*a.values())


@pytest.mark.parametrize("change,status", POOL + [(dict(wanted=None), BAD), (dict(wanted=P), BAD), (dict(wanted=P << 2), BAD), (dict(wanted=(P << 3) + 2), NOT_HERE)])
def test_take_refuses(change, status):
    assert _take(**change) == status


def _fork(**kw):
    a = dict(refs=P, pages=10, page=16, table=P << 1, rows=3, width=4, lens=P << 2, parents=P << 3, children=5, release=1, table_out=P << 4, lens_out=P << 5,
             buffers=_buffers({}), ws=P << 6)
    a.update(kw)
    less = a.pop("less", 0)
    return fq.pages_fork_raw(*a.values(), fq.pages_fork_workspace_bytes(a["rows"], a["children"]) - less)


@pytest.mark.parametrize("change,status", POOL + [(dict(buffers=b), s) for b, s in BUFFERS] + [
    (dict(parents=None), BAD), (dict(children=-1), BAD), (dict(table_out=None), BAD), (dict(lens_out=None), BAD), (dict(table_out=P << 1), BAD), (dict(lens_out=P << 2), BAD),
    (dict(lens_out=P << 3), BAD), (dict(table_out=P), BAD), (dict(lens_out=P << 4), BAD), (dict(ws=P), BAD), (dict(ws=P << 4), BAD), (dict(ws=(P << 6) + 2), NOT_HERE),
    (dict(children=8193), NOT_HERE), (dict(ws=None), SCRATCH), (dict(less=1), SCRATCH), (dict(table=P << 10), BAD),
    (dict(refs=P << 10), BAD), (dict(table_out=P << 10), BAD), (dict(lens_out=(P << 10) + 40), BAD), (dict(ws=P << 10), BAD), (dict(parents=P << 10), BAD),
])
def test_fork_refuses(change, status):
    assert _fork(**change) == status


def _free(**kw):
    a = dict(refs=P, pages=10, page=16, table=P << 1, rows=3, width=4, lens=P << 2, which=P << 3, count=2)
    a.update(kw)
    return fq.pages_free_raw(*a.values())


@pytest.mark.parametrize("change,status", POOL + [(dict(count=-1), BAD), (dict(which=P), BAD), (dict(count=8193), NOT_HERE), (dict(which=(P << 3) + 1), NOT_HERE)])
def test_free_refuses(change, status):
    assert _free(**change) == status


def _compact(**kw):
    a = dict(refs=P, pages=10, page=16, table=P << 1, rows=3, width=4, lens=P << 2, buffers=_buffers({}), ws=P << 6)
    a.update(kw)
    less = a.pop("less", 0)
    return fq.pages_compact_raw(*a.values(), max(0, fq.pages_compact_workspace_bytes(a["pages"]) - less))


@pytest.mark.parametrize("change,status", POOL + [(dict(buffers=b), s) for b, s in BUFFERS] + [
    (dict(ws=None), SCRATCH), (dict(less=1), SCRATCH), (dict(ws=P), BAD), (dict(ws=P << 10), BAD), (dict(refs=P << 10), BAD), (dict(table=P << 10), BAD),
    (dict(lens=P << 10), BAD), (dict(ws=(P << 6) + 2), NOT_HERE),
])
def test_compact_refuses(change, status):
    assert _compact(**change) == status


def test_nothing_to_do():
    assert _copy(moves=0, src=None, dst=None) == fq.FQ_OK and _copy(buffers=_buffers()) == fq.FQ_OK
    assert _take(rows=0, table=None, lens=None, wanted=None) == fq.FQ_OK
    assert _fork(children=0, release=0, ws=None, table_out=None, lens_out=None, parents=None) == fq.FQ_OK
    assert _free(count=0) == fq.FQ_OK
    assert _compact(pages=0, refs=None, ws=None) == fq.FQ_OK


def test_torch_calls_refuse():
    refs, table, lens = torch.zeros(4, dtype=torch.int32), torch.zeros((2, 3), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: fq.pages_take(refs, 16, table, lens, lens), lambda: fq.pages_fork(refs, 16, table, lens, lens), lambda: fq.pages_free(refs, 16, table, lens),
                 lambda: fq.pages_compact(refs, 16, table, lens)):        # host memory
        with pytest.raises(fq.FqError):
            call()
