"""The example layer (examples/attention_layer.py): its calls against the single operators and 64-bit attention, on quantised products."""
import importlib.util
import os

import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
_spec = importlib.util.spec_from_file_location("attention_layer", _PATH)
example = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(example)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (4, 4)])
def test_prompts_then_a_tree_then_its_branch(dtype, heads, kv_heads):
    hidden, lengths = 512, [70, 5, 131]
    D = hidden // heads
    layer = example.AttentionLayer(hidden, heads, kv_heads, dtype=dtype)
    cache = example.Cache(3, 200, kv_heads, D, page=16, dtype=dtype)
    gen = torch.Generator(device="cuda").manual_seed(3)
    offsets = [0, 70, 75, 206]

    def rows(n):
        return torch.randn((n, hidden), generator=gen, device="cuda").to(dtype)

    def cached(b, n):
        at = cache.places(b, torch.arange(n))
        return tuple(t.view(-1, kv_heads, D).cpu()[at] for t in (cache.k, cache.v))

    x = rows(206)
    got = layer.prompts(x, lengths, cache)
    assert got.shape == (206, hidden)
    # the same products once more, and attention in 64 bits over what lies in the cache
    product = fq.gemm(x, *layer.qkv, layer.bits, layer.group)
    positions = torch.cat([torch.arange(n, dtype=torch.int32) for n in lengths]).cuda()
    q, k = fq.qk_norm_rope(product, heads, kv_heads, layer.table, positions, layer.q_norm, layer.k_norm)
    for b, n in enumerate(lengths):
        kc, vc = cached(b, n)
        assert torch.equal(kc, k[offsets[b]:offsets[b + 1]].cpu())
        assert torch.equal(vc, product.view(206, -1, D)[offsets[b]:offsets[b + 1], heads + kv_heads:].cpu())
    v = product.view(206, -1, D)[:, heads + kv_heads:]
    attended = fq.attention_prompt(q, k, v, offsets)
    ref.compare(attended, *ref.prompt(q.cpu(), k.cpu(), v.cpu(), offsets, offsets), "prompts")
    assert torch.equal(got, fq.gemm(attended.reshape(206, -1), *layer.out, layer.bits, layer.group))

    parents = [-1, 0, 0, 1, 3, 2]
    x = rows(3 * 6)
    got = layer.drafted(x, parents, cache)
    product = fq.gemm(x, *layer.qkv, layer.bits, layer.group)
    depth = [0, 1, 1, 2, 3, 2]
    positions = torch.tensor([n + d for n in lengths for d in depth], dtype=torch.int32, device="cuda")
    q, k = fq.qk_norm_rope(product, heads, kv_heads, layer.table, positions, layer.q_norm, layer.k_norm)
    sees = ref.from_parents(parents)[None].expand(3, 6, 6)
    want, tol = ref.tree(q.view(3, 6, heads, D).cpu(), cache.k.cpu(), cache.v.cpu(), cache.table.cpu(), torch.tensor(lengths), sees)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    attended = fq.attention_tree(q.view(3, 6, heads, D), cache.k, cache.v, cache.table, lens, mask=fq.tree_mask(parents))
    ref.compare(attended, want, tol, "tree")
    assert torch.equal(got, fq.gemm(attended.reshape(18, -1), *layer.out, layer.bits, layer.group))

    # the branch 0, 1, 3, 4 becomes part of the sequences: the next token sees what a chain of these tokens would have left
    before = [cached(b, n + 6) for b, n in enumerate(lengths)]
    layer.keep([0, 1, 3, 4], cache)
    assert cache.lens == [n + 4 for n in lengths]
    for b, n in enumerate(lengths):
        for now, was in zip(cached(b, n + 4), before[b]):
            assert torch.equal(now, torch.cat([was[:n], was[n:][[0, 1, 3, 4]]]))
    x = rows(3)
    got = layer.drafted(x, [-1], cache)
    product = fq.gemm(x, *layer.qkv, layer.bits, layer.group)
    q, _ = fq.qk_norm_rope(product, heads, kv_heads, layer.table, torch.tensor(cache.lens, dtype=torch.int32, device="cuda"), layer.q_norm,
                           layer.k_norm)
    want, tol = ref.tree(q.view(3, 1, heads, D).cpu(), cache.k.cpu(), cache.v.cpu(), cache.table.cpu(), torch.tensor(cache.lens), ref.chain(3, 1))
    attended = fq.attention_tree(q.view(3, 1, heads, D), cache.k, cache.v, cache.table, torch.tensor(cache.lens, dtype=torch.int32, device="cuda"))
    ref.compare(attended, want, tol, "one token")
    assert torch.equal(got, fq.gemm(attended.reshape(3, -1), *layer.out, layer.bits, layer.group))
