"""The calls of a cache in 4 bits, of shared pages and of adapters on torch tensors: natively and from Python, the same results and the same refusals."""
import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


class _Python:
    """Stands in for the native module: every call goes the Python way."""

    def __getattr__(self, name):
        return lambda *args: None


def _normal(size, dtype, seed):
    return torch.randn(size, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def _ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _both(monkeypatch, call):
    """What a call gives natively and from Python."""
    fq._stream()
    mine = call()
    monkeypatch.setattr(fq, "_native", _Python())
    python = call()
    monkeypatch.undo()
    return mine, python


def _refused(call):
    with pytest.raises(Exception) as e:
        call()
    return type(e.value), str(e.value)


def _same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_cache(monkeypatch, dtype):
    hk, D, page = 2, 128, 32
    rows = _normal((40, (4 + 2 * hk) * D), dtype, 1).view(40, -1, D)
    q, k, v = rows[:, :4], rows[:, 4:4 + hk], rows[:, 4 + hk:]
    slots = (torch.arange(40) * 7 % 96).cuda()
    table, lens = torch.tensor([[1, 2, 0], [0, 1, 2]], dtype=torch.int32).cuda(), _ints(33, 50)
    mask = fq.tree_mask([-1, 0, 0, 1])

    def run():
        cache = fq.kv4_cache(3, page, hk, D)
        fq.kv4_write(k, v, cache, page, slots)
        out = [cache.clone(), *fq.kv4_read(cache, page, hk, D, slots, dtype)]
        given = torch.empty_like(out[1]), torch.empty_like(out[1])
        back = fq.kv4_read(cache, page, hk, D, slots[:40], dtype, *given)
        assert back[0] is given[0] and back[1] is given[1]
        tree = q[:8].view(2, 4, 4, D) if q[:8].is_contiguous() else q[:8].unflatten(0, (2, 4))
        out += [*given, fq.attention_tree_kv4(tree, cache, page, hk, table, lens), fq.attention_tree_kv4(tree, cache, page, hk, table, lens, mask=mask, scale=0.2)]
        for ws in (torch.empty(4, dtype=torch.int64, device="cuda"), torch.empty(1 << 20, dtype=torch.float32, device="cuda")):
            o = torch.empty((2, 4, 4, D), dtype=dtype, device="cuda")
            assert fq.attention_tree_kv4(tree, cache, page, hk, table, lens, out=o, workspace=ws) is o
            out.append(o)
        out += [fq.attention_tree_kv4(q[:2, None], cache, page, hk, table, lens), fq.attention_tree_kv4(q[:0, None], cache, page, hk, table[:0], lens[:0])]
        fq.kv4_write(k[:0], v[:0], cache, page, slots[:0])
        out.append(cache)
        return out

    _same(*_both(monkeypatch, run))


def test_cache_refusals(monkeypatch):
    k = _normal((4, 2, 64), F16, 1)
    cache, slots = fq.kv4_cache(3, 16, 2, 64), torch.arange(4).cuda()
    q, table, lens = _normal((1, 1, 4, 64), F16, 2), torch.zeros((1, 3), dtype=torch.int32, device="cuda"), _ints(0)
    attend = fq.attention_tree_kv4
    calls = [
        lambda: fq.kv4_write(k, k[:3], cache, 16, slots), lambda: fq.kv4_write(k, k, cache, 32, slots), lambda: fq.kv4_write(k, k, cache[:, :-16], 16, slots),
        lambda: fq.kv4_write(k, k, cache, 16, slots.int()), lambda: fq.kv4_write(k, k, cache, 16, slots[:3]), lambda: fq.kv4_write(k, k.to(BF16), cache, 16, slots),
        lambda: fq.kv4_write(k, k, cache.view(torch.int8), 16, slots), lambda: fq.kv4_write(k, k, cache, 16, slots.cpu()), lambda: fq.kv4_write(k.cpu(), k.cpu(), cache, 16, slots),
        lambda: fq.kv4_write(k, k, cache.cpu(), 16, slots), lambda: fq.kv4_write(k, k, cache, 15, slots), lambda: fq.kv4_write(k, k, cache, 0, slots), lambda: fq.kv4_write(k, k, cache, -16, slots),
        lambda: fq.kv4_write(k[..., ::2], k[..., ::2], cache, 16, slots), lambda: fq.kv4_write(k[..., 1:9], k[..., 1:9], fq.kv4_cache(1, 16, 2, 8), 16, slots),
        lambda: fq.kv4_write(k.view(4, 128), k.view(4, 128), cache, 16, slots), lambda: fq.kv4_write(k.float(), k.float(), cache, 16, slots),
        lambda: fq.kv4_write(k, k, cache.as_strided((3, cache.shape[1]), (cache.shape[1] - 16, 1)), 16, slots),
        lambda: fq.kv4_read(cache, 16, 4, 64, slots, F16), lambda: fq.kv4_read(cache, 16, 2, 64, slots.int(), F16), lambda: fq.kv4_read(cache, 16, 2, 64, slots, torch.float32),
        lambda: fq.kv4_read(cache, 16, 2, 64, slots, F16, k_out=k[:2]), lambda: fq.kv4_read(cache, 16, 2, 64, slots, BF16, k_out=torch.empty_like(k)),
        lambda: fq.kv4_read(cache, 16, 2, 64, slots, F16, v_out=k.float()), lambda: fq.kv4_read(cache, 16, 2, 64, slots.cpu(), F16), lambda: fq.kv4_read(cache.cpu(), 16, 2, 64, slots, F16),
        lambda: attend(q, cache, 16, 3, table, lens), lambda: attend(q, cache, 16, 2, table.long(), lens), lambda: attend(q, cache, 16, 2, table, lens.long()),
        lambda: attend(q, cache, 16, 2, table, lens, scale=1e-50), lambda: attend(q, cache, 16, 2, table, lens, scale=float("nan")),
        lambda: attend(q, cache, 16, 2, table, lens, mask=torch.zeros((2, 1), dtype=torch.int64, device="cuda")),
        lambda: attend(q, cache, 16, 2, table, lens, mask=torch.zeros((1, 1), dtype=torch.int32, device="cuda")),
        lambda: attend(q, cache, 16, 2, table, lens, workspace=torch.zeros(1 << 20, dtype=torch.uint8)), lambda: attend(q, cache, 16, 2, table, lens, out=q),
        lambda: attend(q, cache, 16, 2, table, lens, out=q.float()), lambda: attend(q, cache, 16, 2, table[:, ::2], lens), lambda: attend(q, cache, 16, 2, table.cpu(), lens),
        lambda: attend(q, cache, 16, 2, table.expand(2, 3), lens), lambda: attend(q.cpu(), cache, 16, 2, table, lens), lambda: attend(q.float(), cache, 16, 2, table, lens),
        lambda: attend(q[0], cache, 16, 2, table, lens), lambda: attend(q, cache, 16, 8, table, lens), lambda: attend(q[..., :63], cache, 16, 2, table, lens),
    ]
    mine, python = _both(monkeypatch, lambda: [_refused(c) for c in calls])
    assert mine == python
    assert all(kind in (fq.FqError, TypeError, AssertionError, ValueError) for kind, _ in mine), mine


def _pool(pages=12, rows=3, width=4, page=16):
    refs, table, lens = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.full((rows, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda")
    return refs, table, lens, torch.arange(2 * pages * 64, device="cuda").view(2, pages, 64), torch.arange(pages * 24, device="cuda").view(pages, 24).half()


def test_pages(monkeypatch):
    def run():
        refs, table, lens, stack, other = _pool()
        fq.pages_take(refs, 16, table, lens, _ints(33, 16, 60))
        out = [refs.clone(), table.clone(), lens.clone()]
        for buffers, release in ((stack, False), ([other], False), ([], False), ((), True), ([stack[0], other], True)):
            table, lens = fq.pages_fork(refs, 16, table, lens, _ints(0, 2, 1), buffers, release)
            out += [refs.clone(), table, lens, stack.clone(), other.clone()]
            table, lens = table.clone(), lens.clone()
        ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
        t, n = torch.empty((2, 4), dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
        got = fq.pages_fork(refs, 16, table, lens, _ints(1, 7), stack, False, t, n, ws)
        assert got[0] is t and got[1] is n
        fq.pages_free(refs, 16, t, n)
        out += [t.clone(), n.clone(), refs.clone()]
        fq.pages_free(refs, 16, table, lens, _ints(0, 0, 9))
        fq.pages_free(refs, 16, table, lens, _ints())
        fq.pages_compact(refs, 16, table, lens, stack)
        fq.pages_compact(refs, 16, table, lens, [other], ws)
        fq.pages_compact(refs, 16, table, lens)
        fq.pages_take(refs, 16, table[:0], lens[:0], lens[:0])
        out += [refs, table, lens, stack, other, *fq.pages_fork(refs, 16, table, lens, _ints(), stack)]
        return out

    _same(*_both(monkeypatch, run))


def test_pages_refusals(monkeypatch):
    refs, table, lens, stack, other = _pool()
    want = _ints(1, 1, 1)
    fork, compact = fq.pages_fork, fq.pages_compact
    calls = [
        lambda: fq.pages_take(refs.long(), 16, table, lens, want), lambda: fq.pages_take(refs, 0, table, lens, want), lambda: fq.pages_take(refs, 16, table[:2], lens, want),
        lambda: fq.pages_take(refs, 16, table, lens, want[:2]), lambda: fq.pages_take(refs, 16, table[:, ::2], lens, want), lambda: fq.pages_take(refs.cpu(), 16, table, lens, want),
        lambda: fq.pages_take(refs, 16, table, lens, lens), lambda: fq.pages_take(refs, 16, table, lens, want.cpu()), lambda: fq.pages_take(refs.view(2, 6), 16, table, lens, want),
        lambda: fork(refs, 16, table, lens, want.long(), stack), lambda: fork(refs, 16, table, lens, want, stack[:, :5]), lambda: fork(refs, 16, table, lens, want, [other[:3]]),
        lambda: fork(refs, 16, table, lens, want, [other.t()]), lambda: fork(refs, 16, table, lens, want, other.cpu()), lambda: fork(refs, 16, table, lens, want, stack, table_out=table),
        lambda: fork(refs, 16, table, lens, want, stack, lens_out=lens), lambda: fork(refs, 16, table, lens, want, stack, table_out=table[:2].clone()),
        lambda: fork(refs, 16, table, lens, want, [other[:, ::2]]), lambda: fork(refs, 16, table, lens, want, [other[:, :3]]), lambda: fork(refs, -1, table, lens, want, stack),
        lambda: fork(refs, 16, table, lens, want, stack, workspace=torch.empty(1 << 16, dtype=torch.uint8)),
        lambda: fq.pages_free(refs, 16, table, lens, want.long()), lambda: fq.pages_free(refs, 0, table, lens), lambda: fq.pages_free(refs, 16, table, lens[:2]),
        lambda: fq.pages_free(refs, 16, table, lens, want.cpu()), lambda: compact(refs, 16, table, lens, [stack]), lambda: compact(refs, 0, table, lens, stack),
        lambda: compact(refs, 16, table, lens, stack, workspace=torch.empty(1 << 16, dtype=torch.uint8)), lambda: compact(refs, 16, table, lens.long(), stack),
        lambda: compact(refs, 16, table, lens, [other, other.cpu()]),
    ]
    mine, python = _both(monkeypatch, lambda: [_refused(c) for c in calls])
    assert mine == python
    assert all(kind is fq.FqError for kind, _ in mine), mine
    assert int(refs.max()) == 0 and int(table.max()) == -1       # nothing was done


@pytest.mark.parametrize("rows", [1, 50, 200])
def test_adapters(monkeypatch, rows):
    wide = _normal((rows, 128 + 512), BF16, 1)
    a, b, ids, scales = _normal((3, 8, 512), BF16, 2), _normal((3, 96, 8), BF16, 3), torch.arange(rows, dtype=torch.int32, device="cuda") % 4 - 1, torch.tensor([1.0, 0.5, -2.0], device="cuda")

    def run():
        out = []
        for s in (None, scales):
            for ws in (None, torch.empty(4, device="cuda"), torch.empty(1 << 22, dtype=torch.uint8, device="cuda")):
                o = wide.clone()
                assert fq.adapters(wide[:, 128:], a, b, ids, o[:, :96], s, ws).data_ptr() == o.data_ptr()
                out.append(o)
        o = wide.clone()
        out += [fq.adapters(wide[:0, 128:], a, b, ids[:0], o[:0, :96]), fq.adapters(wide[:, 128:], a[:0], b[:0], ids, o[:, :96]), o]
        return out

    _same(*_both(monkeypatch, run))


def test_adapters_refusals(monkeypatch):
    x, a, b, ids, out = _normal((5, 64), F16, 1), _normal((2, 8, 64), F16, 2), _normal((2, 40, 8), F16, 3), _ints(0, 1, 0, -1, 1), _normal((5, 40), F16, 4)
    before = out.clone()
    call = fq.adapters
    calls = [
        lambda: call(x.float(), a, b, ids, out), lambda: call(x, a.to(BF16), b, ids, out), lambda: call(x, a, b.to(BF16), ids, out), lambda: call(x, a, b, ids.long(), out),
        lambda: call(x, a, b, ids[:4], out), lambda: call(x[:4], a, b, ids, out), lambda: call(x, a[:1], b, ids, out), lambda: call(x, a[:, :4], b, ids, out), lambda: call(x, a, b, ids, out[:, :32]),
        lambda: call(x, a, b, ids, out.to(BF16)), lambda: call(x.cpu(), a, b, ids, out), lambda: call(x, a.cpu(), b, ids, out), lambda: call(x, a, b, ids.cpu(), out), lambda: call(x, a, b, ids, out.cpu()),
        lambda: call(x, a, b, ids, out, scales=torch.ones(3, device="cuda")), lambda: call(x, a, b, ids, out, scales=torch.ones(2, dtype=torch.float64, device="cuda")),
        lambda: call(x, a, b, ids, out, scales=torch.ones(2)), lambda: call(x, a, b, ids, out, workspace=torch.empty(1 << 20, dtype=torch.uint8)),
        lambda: call(x, a, b, ids, x[:, :40]), lambda: call(x, a[:, :, ::2], b, ids, out), lambda: call(x[:, :60], a[:, :, :60].contiguous(), b, ids, out),
        lambda: call(x, a[:, :5].contiguous(), b[:, :, :5].contiguous(), ids, out), lambda: call(x, a, b[:, :39].contiguous(), ids, out[:, :39]),
        lambda: call(x[:1].expand(5, 64), a, b, ids, out[:1].expand(5, 40)), lambda: call(x[0], a, b, ids, out),
    ]
    mine, python = _both(monkeypatch, lambda: [_refused(c) for c in calls])
    assert mine == python
    assert all(kind in (fq.FqError, TypeError, AssertionError, IndexError) for kind, _ in mine), mine
    assert torch.equal(out, before)


def test_tensors_of_another_device_are_refused(monkeypatch):
    """A call goes to the current device's stream: with another current device it is not made."""
    fq._stream()
    monkeypatch.setattr(fq, "_native", _Python())
    monkeypatch.setattr(fq, "_device", lambda: 1)
    k, slots, cache = _normal((4, 2, 64), F16, 1), torch.arange(4).cuda(), fq.kv4_cache(3, 16, 2, 64)
    refs, table, lens, stack, _ = _pool()
    for call in (lambda: fq.kv4_write(k, k, cache, 16, slots), lambda: fq.kv4_read(cache, 16, 2, 64, slots, F16),
                 lambda: fq.attention_tree_kv4(k[:1, None], cache, 16, 2, table[:1], lens[:1]), lambda: fq.pages_copy(stack, lens, lens), lambda: fq.pages_take(refs, 16, table, lens, lens.clone()),
                 lambda: fq.pages_fork(refs, 16, table, lens, lens, stack), lambda: fq.pages_free(refs, 16, table, lens), lambda: fq.pages_compact(refs, 16, table, lens, stack),
                 lambda: fq.adapters(k[:, 0], k[:1, :, :].repeat(1, 4, 1), k[:1, :, :8].repeat(1, 4, 1).contiguous(), slots.int(), k[:, 1, :8])):
        with pytest.raises(fq.FqError):
            call()
    assert not bool(cache.any()) and int(refs.max()) == 0


def test_on_another_stream(monkeypatch):
    """Work waits for the current stream's, and for nothing else's."""
    x, a, b = _normal((2000, 1024), BF16, 1), _normal((1, 16, 1024), BF16, 2), _normal((1, 512, 16), BF16, 3)
    ids = torch.zeros(2000, dtype=torch.int32, device="cuda")
    refs, table, lens, stack, _ = _pool()
    cache = fq.kv4_cache(2000 * 4 // 16 + 1, 16, 4, 128)
    torch.cuda.synchronize()

    def run():
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            y = x.float().mul(2).to(BF16)
            out = torch.zeros((2000, 512), dtype=BF16, device="cuda")
            fq.adapters(y, a, b, ids, out)
            fq.kv4_write(out.view(-1, 4, 128), out.view(-1, 4, 128), cache, 16, torch.arange(2000, device="cuda"))
            k, v = fq.kv4_read(cache, 16, 4, 128, torch.arange(2000, device="cuda"), BF16)
            z = k.float().mul(1).to(BF16)
        s.synchronize()
        return [out, k, v, z, cache.clone()]

    mine, python = _both(monkeypatch, run)
    _same(mine, python)
    out = torch.zeros((2000, 512), dtype=BF16, device="cuda")
    assert torch.equal(mine[0], fq.adapters(x * 2, a, b, ids, out))


def test_two_captured_calls_share_a_workspace():
    """Two graphs with one workspace, replayed one after the other on a stream."""
    B, hq, hk, D, page, width = 4, 8, 2, 128, 16, 400
    cache = fq.kv4_cache(B * width, page, hk, D)
    n = B * width * page
    fq.kv4_write(_normal((n, hk, D), BF16, 1), _normal((n, hk, D), BF16, 2), cache, page, torch.arange(n, device="cuda"))
    table = torch.randperm(B * width, generator=torch.Generator().manual_seed(3)).to(torch.int32).view(B, width).cuda()
    ws = torch.empty(max(fq.attention_tree_kv4_workspace_bytes(B, nodes, hq, hk, D, width, page) for nodes in (1, 6)), dtype=torch.uint8, device="cuda")
    calls = []
    for nodes in (1, 6):
        q, lens, out = _normal((B, nodes, hq, D), BF16, nodes), _ints(6300, 5, 2000, 4444), torch.empty((B, nodes, hq, D), dtype=BF16, device="cuda")
        want = fq.attention_tree_kv4(q, cache, page, hk, table, lens)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            fq.attention_tree_kv4(q, cache, page, hk, table, lens, out=out, workspace=ws)
        calls.append((graph, out, want, q, lens))
    for i in range(6):
        for _, out, *_ in calls:
            out.fill_(7.0)
        for graph, *_ in calls[::-1 if i % 2 else 1]:
            graph.replay()
        torch.cuda.synchronize()
        for _, out, want, q, lens in calls:
            assert torch.equal(out, want)
            assert torch.equal(fq.attention_tree_kv4(q, cache, page, hk, table, lens, workspace=ws), want)
