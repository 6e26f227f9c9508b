"""Attention whose keys are cut into pieces that other blocks add up: pieces of different numbers of tiles, empty ones, many sequences, and
rows that are computed once more, one by one."""
import pytest
import torch

from paper_2308_09723_amd import fq

import attention_util as ref

pytestmark = pytest.mark.gpu

F16, BF16 = torch.float16, torch.bfloat16


def _normal(size, dtype, seed, sigma=1.0):
    return (torch.randn(size, generator=torch.Generator().manual_seed(seed)) * sigma).to(dtype)


def _offsets(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


# ------------------------------------------------------------------------------------------------ prompts
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("q_lens,k_lens,hq,hk,D", [
    ([3] * 20 + [5], [3] * 20 + [4000], 16, 4, 64),                    # pieces for one sequence's sake: of the others' all but one are empty
    ([2, 130, 1, 7] * 5, [2, 130, 2500, 300] * 5, 16, 16, 40),
    ([1] * 100 + [3, 0, 2], [40] * 100 + [6000, 10, 0], 4, 1, 128),    # and rows that see nothing among them
    ([1, 200, 9], [5000, 200, 777], 8, 2, 96),                         # few blocks
    ([1300], [1300], 12, 3, 80),                                       # a prompt's own early rows have fewer tiles than there are pieces
    ([2100], [2100], 16, 2, 64),
    ([140, 20], [3000, 15], 2, 1, 72),
])
def test_prompts_in_pieces(dtype, q_lens, k_lens, hq, hk, D):
    qo, ko = _offsets(q_lens), _offsets(k_lens)
    assert fq.attention_prompt_workspace_bytes(hq, hk, D, qo, ko) > 0, "not cut"
    q, k, v = _normal((qo[-1], hq, D), dtype, 1, 1.5), _normal((ko[-1], hk, D), dtype, 2), _normal((ko[-1], hk, D), dtype, 3)
    ws = torch.full((fq.attention_prompt_workspace_bytes(hq, hk, D, qo, ko),), 255, dtype=torch.uint8, device="cuda")      # (NaN, if it were read)
    got = fq.attention_prompt(q.cuda(), k.cuda(), v.cuda(), qo, ko, workspace=ws).cpu()
    assert torch.equal(fq.attention_prompt(q.cuda(), k.cuda(), v.cuda(), qo, ko, workspace=ws).cpu(), got)
    for b, (rows, keys) in enumerate(zip(q_lens, k_lens)):
        if rows == 0:
            continue
        pick = torch.unique(torch.cat([torch.arange(min(rows, 3)), torch.randint(0, rows, (40,), generator=torch.Generator().manual_seed(b)),
                                       torch.arange(max(0, rows - 3), rows)]))
        seen = torch.arange(keys)[None] <= pick[:, None] + keys - rows
        for h in {0, hq - 1, hq // 2}:
            part = slice(ko[b], ko[b + 1])
            want, tol = ref.attend(q[qo[b] + pick, h], k[part, h // (hq // hk)], v[part, h // (hq // hk)], seen, D ** -0.5)
            ref.compare(got[qo[b] + pick, h], want, tol, f"sequence {b}, head {h}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_in_pieces_with_what_rows_do_not_see(bad, D):
    """The last key and the last value are not finite: the rows before the last are computed once more, and left as sums."""
    rows, keys = 40, 3000
    q, k, v = _normal((rows, 2, D), BF16, 4, 1.5), _normal((keys, 1, D), BF16, 5), _normal((keys, 1, D), BF16, 6)
    assert fq.attention_prompt_workspace_bytes(2, 1, D, [0, rows], [0, keys]) > 0
    want, tol = ref.prompt(q, k, v, [0, rows], [0, keys])
    k[-1], v[-1] = bad, bad
    got = fq.attention_prompt(q.cuda(), k.cuda(), v.cuda(), [0, rows], [0, keys]).cpu()
    ref.compare(got[:-1], want[:-1], tol[:-1], "rows before the last")
    assert bool(torch.isnan(got[-1].float()).all())


# ------------------------------------------------------------------------------------------------ trees
def _tree_case(lens, nodes, hq, hk, D, page, dtype, seed, hide=None):
    """A tree case over a cache of shuffled pages, whose units are cut.  hide: what the last node's key and value are, which only it sees."""
    used = [max(0, c + nodes + page - 1) // page if c >= 0 else 0 for c in lens]
    pages, width = sum(used) + 2, max(used)
    assert fq.attention_tree_workspace_bytes(len(lens), nodes, hq, hk, D, width, page) > 0, "not cut"
    order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.full((len(lens), width), -1, dtype=torch.int32), 0
    for b, n in enumerate(used):
        table[b, :n] = order[at:at + n]
        at += n
    kc, vc = _normal((pages, page, hk, D), dtype, seed + 1), _normal((pages, page, hk, D), dtype, seed + 2)
    q, context = _normal((len(lens), nodes, hq, D), dtype, seed + 3, 1.5), torch.tensor(lens, dtype=torch.int32)
    sees = ref.chain(len(lens), nodes)
    want, tol = ref.tree(q, kc, vc, table, context, sees)
    last = nodes
    if hide is not None:
        last = nodes - 1
        for b, c in enumerate(lens):
            place = table[b, (c + last) // page].long(), (c + last) % page
            kc[place], vc[place] = hide, hide
    got = fq.attention_tree(q.cuda(), kc.cuda(), vc.cuda(), table.cuda(), context.cuda()).cpu()
    ref.compare(got[:, :last], want[:, :last], tol[:, :last], f"{len(lens)} sequences, {nodes} nodes")
    if hide is not None:
        assert bool(torch.isnan(got[:, last].float()).all())


# (nodes, query heads, key heads), and keys of a tile: up to 32 rows a key head, one, two and four heads a block; tiles of 64 and of 128 rows
ROWS = [(3, 3, 1, 128), (3, 4, 2, 64), (2, 16, 4, 32), (20, 2, 1, 64), (70, 1, 1, 64)]


@pytest.mark.parametrize("count", [1, 2, 63, 64, 65, 128, 200])
@pytest.mark.parametrize("nodes,hq,hk,tile", ROWS)
def test_trees_of_many_sequences_in_pieces(count, nodes, hq, hk, tile):
    """Sequences of one tile, of several, of none and one of many more than may be left whole, wherever it stands."""
    for longest in {0, count // 2, count - 1}:
        lens = [(i * 37) % (2 * tile) if i % 5 else -1 if i % 2 else 0 for i in range(count)]
        lens[longest] = 13 * tile + 5
        _tree_case(lens, nodes, hq, hk, 64, 16, BF16 if count % 2 else F16, count + longest)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("nodes,hq,hk,tile", ROWS)
def test_trees_in_pieces_with_what_rows_do_not_see(bad, nodes, hq, hk, tile, D):
    """The last drafted token is not finite: the other rows are computed once more, and left as sums."""
    _tree_case([20 * tile, 3, 9 * tile + 1], nodes, hq, hk, D, 16, F16, 7, hide=bad)
