"""The example of a serving layer (examples/serving_layer.py): prompts, forks and tokens against 64-bit attention over what each sequence's tokens were."""
import importlib.util
import os

import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref
import kv4_util

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_layer.py")
_spec = importlib.util.spec_from_file_location("serving_layer", _PATH)
example = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(example)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (4, 4)])
def test_beams_of_prompts(dtype, heads, kv_heads):
    hidden, lengths, page = 512, [70, 5, 131], 16
    D = hidden // heads
    layer = example.ServingLayer(hidden, heads, kv_heads, adapters=3, rank=8, dtype=dtype)
    cache = example.SharedCache(80, 3, 200, kv_heads, D, page=page)
    gen = torch.Generator(device="cuda").manual_seed(3)

    def rows(n):
        return torch.randn((n, hidden), generator=gen, device="cuda").to(dtype)

    def ready(x, positions, ids):
        """The layer's product with adapters in 64 bits beside it, and queries, keys and values of it."""
        plain = fq.gemm(x, *layer.qkv, layer.bits, layer.group)
        product = fq.adapters(x, layer.a, layer.b, ids, plain.clone(), scales=layer.scales)
        want = plain.double()
        for m, i in enumerate(ids.tolist()):
            if i >= 0:
                want[m] += layer.b[i].double() @ (layer.a[i].double() @ x[m].double())
        # (half a unit of the result, and inner sums in 16 + 8 or 21 bits of terms that add up to at most some ten times as much)
        assert bool(((product.double() - want).abs() <= ref.UNIT[dtype] * want.abs() + 2.0 ** -10).all())
        q, k = fq.qk_norm_rope(product, heads, kv_heads, layer.table, positions, layer.q_norm, layer.k_norm)
        return q, k, product.view(x.shape[0], -1, D)[:, heads + kv_heads:]

    def stored(t):
        return kv4_util.quantise(t.cpu())[2].to(dtype)

    # every sequence's keys and values, as its cache ought to have them
    ids = torch.tensor([2, -1, 0], dtype=torch.int32, device="cuda")
    x = rows(206)
    got = layer.prompts(x, lengths, cache, ids)
    each = torch.repeat_interleave(ids, torch.tensor(lengths, device="cuda")).contiguous()
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
    q, k, v = ready(x, positions, each)
    offsets = [0, 70, 75, 206]
    attended = fq.attention_prompt(q, k, v, offsets)
    ref.compare(attended, *ref.prompt(q.cpu(), k.cpu(), v.cpu(), offsets, offsets), "prompts")
    assert torch.equal(got, layer._output(attended))
    keys, values = ([stored(t[a:b]) for a, b in zip(offsets, offsets[1:])] for t in (k, v))

    def check(what):
        assert cache.lens.tolist() == [len(t) for t in keys], what
        for b, (kk, vv) in enumerate(zip(keys, values)):
            at = torch.arange(len(kk), device="cuda")
            for got, want in zip(fq.kv4_read(cache.pages, page, kv_heads, D, cache.slots(b, at), dtype), (kk, vv)):
                assert torch.equal(got.cpu(), want), f"{what}: sequence {b}"
        # the pages' references are those of the rows
        held = torch.zeros(80, dtype=torch.int32)
        for b, kk in enumerate(keys):
            for p in cache.table[b, :-(-len(kk) // page)].tolist():
                held[p] += 1
        assert torch.equal(cache.refs.cpu(), held), what

    check("prompts")
    beams = [0, 0, 0, 1, 1, 2, 2]
    for step, parents in enumerate((beams, [1, 0, 1, 3, 4, 5, 5], [0, 1, 2, 4, 4, 5, 6], [2, 2, 2, 3, 3, 6, 6], [6, 0, 3])):
        cache.fork(torch.tensor(parents, dtype=torch.int32, device="cuda"))
        keys, values, ids = [keys[p] for p in parents], [values[p] for p in parents], ids[torch.tensor(parents, device="cuda")].contiguous()
        check(f"fork {step}")
        if step == 2:
            cache.compact()
            assert int((cache.refs > 0).nonzero().max()) + 1 == int((cache.refs > 0).sum())
            check("gathered")
        for token in range(1 + 7 * (step % 2)):
            x = rows(len(parents))
            before = torch.tensor([len(t) for t in keys], dtype=torch.int32)
            q, k, v = ready(x, before.cuda(), ids)
            keys, values = ([torch.cat([old, stored(new[None])]) for old, new in zip(olds, t)] for olds, t in ((keys, k), (values, v)))
            got = layer.tokens(x, cache, ids)
            check(f"step {step} token {token}")
            attended = fq.attention_tree_kv4(q.unsqueeze(1), cache.pages, page, kv_heads, cache.table, before.cuda())
            for b, (kk, vv) in enumerate(zip(keys, values)):
                for h in range(heads):
                    g = h * kv_heads // heads
                    want, tol = ref.attend(q[b, h:h + 1].cpu(), kk[:, g], vv[:, g], torch.ones((1, len(kk)), dtype=torch.bool), D ** -0.5)
                    ref.compare(attended[b, :, h], want, tol, f"step {step} sequence {b}")
            assert torch.equal(got, layer._output(attended))
    cache.free(torch.tensor([1], dtype=torch.int32, device="cuda"))
    keys[1], values[1] = keys[1][:0], values[1][:0]
    check("freed one")
    cache.free()
    assert int(cache.refs.sum()) == 0 and not bool(cache.lens.any())
