"""The example of a serving layer where tables end with a whole page, and where pages or entries run out."""
import sys

import pytest
import torch

from test_serving_example import example

pytestmark = pytest.mark.gpu


def test_tables_that_end_with_a_page(monkeypatch):
    """1500 tokens and 36: 24 pages of 64, and one token more."""
    monkeypatch.setattr(sys, "argv", ["serving_layer.py", "--hidden", "512", "--heads", "8", "--kv-heads", "2", "--prompts", "70", "1500", "9", "--beams", "2", "--tokens", "36"])
    example.main()


@pytest.mark.parametrize("what", ["pages", "entries", "children"])
def test_no_room(what):
    hidden, page = 512, 16
    layer = example.ServingLayer(hidden, 8, 2, adapters=2, rank=8)
    pages = {"pages": 5, "entries": 20, "children": 6}[what]
    cache = example.SharedCache(pages, 2, 48 if what == "entries" else 200, 2, layer.D, page=page)
    x = torch.randn((48 + 30, hidden), device="cuda").to(torch.bfloat16)
    ids = torch.zeros(2, dtype=torch.int32, device="cuda")
    layer.prompts(x, [48, 30], cache, ids)       # three pages and two
    if what == "children":
        with pytest.raises(RuntimeError, match=r"\[2, 3\]"):
            cache.fork(torch.tensor([0, 1, 1, 1], dtype=torch.int32, device="cuda"), release=False)
        return
    held = cache.table.clone()
    with pytest.raises(RuntimeError, match=r"\[0\]"):
        layer.tokens(x[:2], cache, ids)
    assert torch.equal(cache.table, held) and cache.lens.tolist() == [48, 31]
    cache.free(torch.tensor([1], dtype=torch.int32, device="cuda"))
    if what == "pages":                          # (another row's pages)
        cache.grow(torch.tensor([1, 0], dtype=torch.int32, device="cuda"))
        assert cache.lens.tolist() == [49, 0]
