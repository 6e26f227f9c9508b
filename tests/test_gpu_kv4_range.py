"""Attention over a cache held in 4 bits where queries times codes leave binary32 though queries times keys do not."""
import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as attention
import kv4_util as ref

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.mark.parametrize("nodes,hq,hk", [(1, 2, 2), (1, 8, 2), (2, 8, 2), (6, 8, 2), (10, 8, 2)])
@pytest.mark.parametrize("D,lens", [(64, [100, 37]), (128, [300, 2]), (40, [3000])])
def test_large_queries_and_small_keys(nodes, hq, hk, D, lens):
    """Queries of 2^121 and keys of 2^-121: a group's codes (up to 7, of the queries' signs or the opposite ones) times the queries pass 2^128 either way.  1, 4, 8, 24 and 40 rows of a key head."""
    for signs in (-1.0, 1.0):
        gen = torch.Generator().manual_seed(nodes + D)
        page, B = 16, len(lens)
        total = [n + nodes for n in lens]
        width = max((n + page - 1) // page for n in total)
        table = torch.randperm(B * width, generator=gen).view(B, width).to(torch.int32)
        toward = torch.where(torch.rand((hk, D), generator=gen) < 0.5, -1.0, 1.0)
        q = (1 + 0.5 * torch.rand((B, nodes, hq, D), generator=gen)) * toward.repeat_interleave(hq // hk, 0) * 2.0 ** 121
        q = q.to(BF16)
        k, v = torch.zeros((B * width, page, hk, D), dtype=BF16), torch.zeros((B * width, page, hk, D), dtype=BF16)
        cache = torch.zeros((B * width, fq.kv4_page_bytes(page, hk, D)), dtype=torch.uint8, device="cuda")
        for b, n in enumerate(total):
            j = torch.arange(n)
            slots = table[b].long()[j // page] * page + j % page
            # every other key against the queries (or along them), the others zeros
            keys = (signs * toward[None] * (1 + 0.1 * torch.rand((n, hk, D), generator=gen)) * 2.0 ** -121 * (j % 2 == 0)[:, None, None]).to(BF16)
            values = torch.randn((n, hk, D), generator=gen).to(BF16) + (j % 2)[:, None, None].to(BF16) * 4
            fq.kv4_write(keys.cuda(), values.cuda(), cache, page, slots.cuda())
            k.view(-1, hk, D)[slots], v.view(-1, hk, D)[slots] = ref.quantise(keys)[2].to(BF16), ref.quantise(values)[2].to(BF16)
        scale = 1.0 / (1.25 * D)       # (scores of about -1, or 1, and zeros)
        got = fq.attention_tree_kv4(q.cuda(), cache, page, hk, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), scale=scale)
        want, tol = attention.tree(q, k, v, table, lens, attention.chain(B, nodes), scale)
        attention.compare(got, want, tol, f"{nodes} {hq}/{hk}/{D} {signs}")
