"""The example of a serving layer: what it makes room for, and what it says where there is none (no GPU)."""
import importlib.util
import os
import random

import pytest
import torch

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "serving_layer.py")
_spec = importlib.util.spec_from_file_location("serving_layer", _PATH)
example = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(example)


@pytest.mark.parametrize("seed", range(40))
def test_room(seed):
    """Rows of a table hold the longest prompt and every token after it; the pool what beams hold that share their prompt's full pages and nothing else, whatever their steps."""
    rng = random.Random(seed)
    page = rng.choice([16, 48, 64])
    prompts, beams, tokens = [rng.randrange(1, 2000) for _ in range(rng.randrange(1, 5))], rng.randrange(1, 9), rng.randrange(0, 1200)
    if seed % 4 == 0:
        tokens = -max(prompts) % page + page        # (the prompt and the tokens are whole pages)
    longest, pages = example.room(prompts, beams, tokens, page)
    assert -(-longest // page) * page >= max(prompts) + tokens
    held = sum(n // page + beams * (-(-(n + tokens) // page) - n // page) for n in prompts)
    assert pages >= held


def _cache(monkeypatch, lens, take=None, fork=None):
    cache = object.__new__(example.SharedCache)
    cache.page, cache.kv_heads, cache.pages = 16, 2, None
    cache.refs, cache.table = torch.zeros(4, dtype=torch.int32), torch.full((len(lens), 3), -1, dtype=torch.int32)
    cache.lens = torch.tensor(lens, dtype=torch.int32)
    monkeypatch.setattr(example.fq, "pages_take", take)
    monkeypatch.setattr(example.fq, "pages_fork", fork)
    return cache


def test_rows_that_cannot_grow_are_an_error(monkeypatch):
    def take(refs, page, table, lens, wanted):      # (all but row 1 get what they want)
        kept = int(lens[1])
        lens.copy_(wanted)
        lens[1] = kept

    cache = _cache(monkeypatch, [3, 16, 40], take)
    with pytest.raises(RuntimeError, match=r"\[1\]"):
        cache.grow(1)
    cache = _cache(monkeypatch, [3, 16, 40], lambda refs, page, table, lens, wanted: lens.copy_(wanted))
    assert cache.grow(torch.tensor([1, 0, 2])).tolist() == [3, 16, 40] and cache.lens.tolist() == [4, 16, 42]


def test_children_that_there_is_no_page_for_are_an_error(monkeypatch):
    def fork(refs, page, table, lens, parents, buffers, release):
        out = lens[parents.long()].clone()
        out[2] = -1
        return table[parents.long()], out

    cache = _cache(monkeypatch, [3, 16], fork=fork)
    with pytest.raises(RuntimeError, match=r"\[2\]"):
        cache.fork(torch.tensor([0, 0, 0, 1], dtype=torch.int32))
