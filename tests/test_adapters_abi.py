"""What the adapters' call refuses, before anything is launched (no GPU)."""
import pytest
import torch

from paper_2308_09723_amd import fq

BAD, NOT_HERE, SCRATCH = fq.FQ_ERR_INVALID_ARG, fq.FQ_ERR_UNSUPPORTED, fq.FQ_ERR_WORKSPACE
P = 1 << 22      # an address that no check follows


def _call(**kw):
    a = dict(x=P, x_stride=128, act=0, rows=5, N=192, K=128, a=P << 1, b=P << 2, adapters=3, rank=16, ids=P << 3, scales=P << 4, out=P << 5, out_stride=192, ws=P << 6)
    a.update(kw)
    less = a.pop("less", 0)
    need = fq.adapters_workspace_bytes(a["rows"], a["adapters"], a["rank"], a["N"], a["K"])
    return fq.adapters_raw(*a.values(), max(0, need - less))


@pytest.mark.parametrize("change,status", [
    (dict(x=None), BAD), (dict(a=None), BAD), (dict(b=None), BAD), (dict(ids=None), BAD), (dict(out=None), BAD), (dict(act=2), BAD), (dict(rows=-1), BAD),
    (dict(N=0), BAD), (dict(K=0), BAD), (dict(adapters=-1), BAD), (dict(rank=0), BAD), (dict(x_stride=120), BAD), (dict(out_stride=184), BAD), (dict(x_stride=-128), BAD),
    (dict(out=P), BAD), (dict(out=P + 4 * 128 * 2), BAD), (dict(out=P << 1), BAD), (dict(out=P << 2), BAD), (dict(out=P << 3), BAD), (dict(out=P << 4), BAD), (dict(ws=P), BAD),
    (dict(ws=P << 5), BAD), (dict(rank=12), NOT_HERE), (dict(rank=136), NOT_HERE), (dict(N=196, out_stride=200), NOT_HERE), (dict(K=124), NOT_HERE),
    (dict(x_stride=132), NOT_HERE), (dict(out_stride=196), NOT_HERE), (dict(x=P + 2), NOT_HERE), (dict(a=P + 8), NOT_HERE), (dict(b=P + 8), NOT_HERE), (dict(out=(P << 5) + 8), NOT_HERE),
    (dict(ids=(P << 3) + 2), NOT_HERE), (dict(scales=(P << 4) + 2), NOT_HERE), (dict(ws=(P << 6) + 4), NOT_HERE), (dict(rows=(1 << 20) + 1), NOT_HERE),
    (dict(adapters=(1 << 20) + 1), NOT_HERE), (dict(x_stride=1 << 60), NOT_HERE), (dict(N=1 << 25, out_stride=1 << 25), NOT_HERE), (dict(ws=None), SCRATCH), (dict(less=1), SCRATCH),
])
def test_refuses(change, status):
    assert _call(**change) == status


def test_nothing_to_add():
    assert _call(rows=0, x=None, ids=None, out=None, ws=None) == fq.FQ_OK and _call(adapters=0, a=None, b=None, ws=None) == fq.FQ_OK
    assert fq.adapters_workspace_bytes(0, 3, 16, 192, 128) == 0 and fq.adapters_workspace_bytes(5, 3, 12, 192, 128) == 0
    for rows in (1, 15, 16, 257, 100000):
        assert fq.adapters_workspace_bytes(rows, 3, 24, 192, 4096) >= rows * 32 * 4


def test_torch_call_refuses():
    x, out, ids = torch.zeros((2, 64), dtype=torch.float16), torch.zeros((2, 32), dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(fq.FqError):
        fq.adapters(x, torch.zeros((1, 8, 64), dtype=torch.float16), torch.zeros((1, 32, 8), dtype=torch.float16), ids, out)       # host memory
    with pytest.raises(TypeError):
        fq.adapters(x.float(), None, None, ids, out)
