"""Sizes at the attention calls' limits: what is counted there, on the host (no GPU)."""
import os
import shutil
import subprocess

import pytest

from paper_2308_09723_amd import fq

HERE = os.path.dirname(os.path.abspath(__file__))
P = 1 << 20      # an address that no check follows


def _tree(sequences, nodes, hq, hk, D, width, page):
    """(workspace, status) of a call whose tensors lie far apart; its workspace is refused, so that nothing can be launched."""
    need = fq.attention_tree_workspace_bytes(sequences, nodes, hq, hk, D, width, page)
    cache = fq.KvPages(P << 22, P << 23, 1 << 10, page, page * hk * D, hk * D, D)
    status = fq.attention_tree_raw(fq.Heads(P << 24, hq * D, D), 0, sequences, nodes, hq, hk, D, cache, P, width, P << 1, None, 0, 0.0, P << 26, None, 0)
    return need, status


@pytest.mark.parametrize("nodes,hq,hk", [(1 << 20, 4096, 1), (1 << 19, 4096, 1), (3 << 18, 4096, 1), (1 << 20, 2048, 1), (1 << 20, 4096, 2),
                                         ((1 << 18) + 1, 4096, 1)])
@pytest.mark.parametrize("width", [1, 512])
def test_tree_rows_that_32_bits_do_not_count_are_refused(nodes, hq, hk, width):
    assert _tree(1, nodes, hq, hk, 8, width, 16) == (0, fq.FQ_ERR_UNSUPPORTED)


def test_tree_tiles_beyond_a_launch_are_refused_by_both():
    """65536 sequences of 256 key heads are 2^24 tiles; one head fewer is not.  (Four heads of 2^30 rows each are 2^25.)"""
    assert _tree(65536, 1, 256, 256, 8, 512, 16) == (0, fq.FQ_ERR_UNSUPPORTED)
    assert _tree(1, 1 << 20, 4096, 4, 8, 512, 16) == (0, fq.FQ_ERR_UNSUPPORTED)
    need, status = _tree(65536, 1, 255, 255, 8, 512, 16)
    assert 0 < need < 1 << 34 and status == fq.FQ_ERR_WORKSPACE


def test_tree_rows_just_within():
    for nodes, hq, hk in ((1 << 18, 4096, 1), (1 << 20, 1024, 1)):
        need, status = _tree(1, nodes, hq, hk, 8, 512, 16)
        assert 0 < need < 1 << 34 and status == fq.FQ_ERR_WORKSPACE


def _overlap(q=P << 24, out=P << 26, table=P, lens=P << 1, mask=None):
    """fq_attention_tree with a cache of 10 pages of 16 x 2 x 128 values at P << 8 and P << 9, 3 sequences of 5 nodes, 4 heads."""
    cache = fq.KvPages(P << 8, P << 9, 10, 16, 4096, 256, 128)
    need = fq.attention_tree_workspace_bytes(3, 5, 4, 2, 128, 64, 16)
    assert need      # (and is not given: a call that nothing else stops ends there)
    return fq.attention_tree_raw(fq.Heads(q, 512, 128), 1, 3, 5, 4, 2, 128, cache, table, 64, lens, mask, 0, 0.0, out, None, 0)


def test_tree_output_over_an_input():
    cache_bytes, out_bytes = 10 * 4096 * 2, 3 * 5 * 4 * 128 * 2
    for first, size in ((P << 8, cache_bytes), (P << 9, cache_bytes), (P, 3 * 64 * 4), (P << 1, 16)):
        for at in (first, first + size - 16, first - out_bytes + 16):
            assert _overlap(out=at // 16 * 16) == fq.FQ_ERR_INVALID_ARG, (first, at)
        for at in (first + (size + 15) // 16 * 16, first - out_bytes):
            assert _overlap(out=at) == fq.FQ_ERR_WORKSPACE, (first, at)
    assert _overlap(out=P << 26, mask=(P << 26) + 64) == fq.FQ_ERR_INVALID_ARG
    assert _overlap(out=P << 26, mask=(P << 26) + out_bytes) == fq.FQ_ERR_WORKSPACE


@pytest.mark.parametrize("change", [dict(qkv=P << 8), dict(q=P << 8), dict(q=(P << 9) + 10 * 4096 * 2 - 16), dict(k=P << 9), dict(k=(P << 8) + 4096)])
def test_norm_rope_within_the_cache(change):
    a = dict(qkv=P << 12, act=0, tokens=4, stride=768, hq=2, hk=2, D=128, qw=None, kw=None, eps=1e-6, table=None, rows=0, rot=0, inter=0, pos=None,
             q=P << 13, k=P << 14, cache=fq.KvPages(P << 8, P << 9, 10, 16, 4096, 256, 128), slots=P)
    a.update(change)
    assert fq.qk_norm_rope_raw(*a.values()) == fq.FQ_ERR_INVALID_ARG


def test_norm_rope_of_2_to_24_tokens_is_more_than_a_launch():
    """(2^32 threads; of one token fewer something else is wrong)"""
    def call(tokens, q_out=P << 40):
        return fq.qk_norm_rope_raw(P, 0, tokens, 32, 1, 1, 8, None, None, 0.0, None, 0, 0, 0, None, q_out, P << 41, None, None)
    assert call(1 << 24) == fq.FQ_ERR_UNSUPPORTED
    assert call((1 << 24) - 1, q_out=P) == fq.FQ_ERR_INVALID_ARG      # (over qkv)


def test_prompts_of_which_a_later_launch_is_too_large_start_none():
    """128 sequences a launch: the 129th alone is too much."""
    def call(last, hq=4096):
        offsets = list(range(129)) + [128 + last]
        heads = [fq.Heads(P << 20 + i, hq * 8, 8) for i in range(3)]
        need = fq.attention_prompt_workspace_bytes(hq, hq, 8, offsets)
        return need, fq.attention_prompt_raw(*heads, 0, hq, hq, 8, offsets, None, 0.0, P << 24, None, 0)
    assert call(4096 * 128 - 127) == (0, fq.FQ_ERR_UNSUPPORTED)
    assert call(4096 * 128) == (0, fq.FQ_ERR_UNSUPPORTED)
    # one tile fewer is not, nor is it when pieces would make it so: few heads, many keys
    offsets, keys = [0, 2], [0, 2 ** 31 - 1025]
    assert fq.attention_prompt_workspace_bytes(4, 4, 8, offsets, keys) > 0


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_parts_of_the_longest_contexts(tmp_path):
    """Keys up to 2^31 - 1025 in parts of up to 2^30, as the kernels go through them (attention_parts_check.cpp)."""
    exe = str(tmp_path / "parts")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-o", exe, os.path.join(HERE, "attention_parts_check.cpp")], check=True)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert out.returncode == 0, out.stdout[-2000:]
    walks, wrong = (int(out.stdout.split()[i]) for i in (-4, -2))
    assert walks > 1000 and wrong == 0


def _prompt_bytes(rows, behind, hq, hk, D):
    def offsets(lengths):
        out = [0]
        for n in lengths:
            out.append(out[-1] + n)
        return out
    return fq.attention_prompt_workspace_bytes(hq, hk, D, offsets(rows), offsets([r + b for r, b in zip(rows, behind)]))


@pytest.mark.parametrize("rows,behind,most", [
    ([512] * 16 + [256], [0] * 16 + [8000], 0), ([128] * 64 + [256], [0] * 64 + [8000], 0), ([512] * 64 + [256], [0] * 64 + [32000], 0),
    ([128] * 128, [0] * 127 + [131000], 5),
])
def test_one_long_prompt_among_many_short_ones(rows, behind, most):
    """Every tile's sums are written and read for the long prompt's pieces: fewer of them, or none (times in plan_splits)."""
    tiles = sum((r + 127) // 128 for r in rows)
    assert _prompt_bytes(rows, behind, 32, 8, 128) <= most * tiles * 32 * 128 * 130 * 4


@pytest.mark.parametrize("rows,hq,hk,D", [(1024, 32, 8, 128), (1000, 32, 32, 128), (1024, 28, 4, 128), (1024, 24, 4, 96), (2324, 32, 8, 128)])
def test_one_prompt_that_is_through_sooner_whole(rows, hq, hk, D):
    assert _prompt_bytes([rows], [0], hq, hk, D) == 0


def test_long_prompts_are_cut():
    piece = 128 * 66 * 4
    assert _prompt_bytes([3397], [0], 12, 12, 64) == 27 * 12 * 3 * piece
    assert _prompt_bytes([3] * 20 + [5], [0] * 20 + [3995], 16, 4, 64) == 21 * 16 * 3 * piece
    assert _prompt_bytes([100], [7900], 32, 8, 64) == 32 * 15 * piece
