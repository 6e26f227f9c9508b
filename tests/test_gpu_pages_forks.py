"""Forks of rows that share pages: whole tables, all buffers, and what a fork costs whose old rows stay."""
import random

import pytest
import torch

from paper_2308_09723_amd import fq

from test_gpu_pages import Model, Pool

pytestmark = pytest.mark.gpu


class ListedPool(Pool):
    """Whose buffers are a list of four."""

    def buffers(self):
        return [self.stack[0], self.stack[1], self.stack[2], self.other]

    def fork(self, parents, release):
        parents = torch.tensor(parents, dtype=torch.int32).cuda()
        self.table, self.lens = fq.pages_fork(self.refs, self.m.page, self.table, self.lens, parents, self.buffers(), release=release)

    def check_all(self, what):
        """Tables as they stand, entries behind a row's pages as well."""
        assert self.refs.tolist() == self.m.refs, what
        assert self.lens.tolist() == self.m.lens, what
        assert self.table.tolist() == self.m.rows, what
        self.check_holds(what)
        want = torch.tensor(self.m.holds).cuda().half()
        assert bool((self.other == want[:, None, None]).all()), what


@pytest.mark.parametrize("release", [False, True])
@pytest.mark.parametrize("rows,children,width,pages", [
    (5, 9, 8, 60), (6, 14, 5, 23), (40, 3, 30, 900), (1, 1, 4, 3), (30, 60, 6, 100),
    # (more than one block does alone: rows, children, entries)
    (1100, 7, 2, 1000), (3, 1030, 2, 1000), (2, 30, 2300, 1000),
])
def test_whole_tables_and_listed_buffers(rows, children, width, pages, release):
    """Entries behind a row's pages are -1, of a child that there is no page for all of them; every buffer of a list has the copies."""
    for seed in range(3):
        rng = random.Random(rows * 10 + seed)
        page = 4
        m = Model(pages, page, width)
        m.rows, m.lens = [[-1] * width for _ in range(rows)], [0] * rows
        p = ListedPool(m)
        wanted = [rng.randrange(0, min(width, 6) * page + 1) for _ in range(rows)]
        p.take(wanted)
        m.take(wanted)
        p.check_all(f"take {seed}")
        parents = [rng.randrange(-1, rows + 1) for _ in range(children)]
        p.fork(parents, release)
        m.fork(parents, release)
        p.check_all(f"fork {seed}")
        if release:        # (the pool's rows are all in the table)
            fq.pages_compact(p.refs, page, p.table, p.lens, p.buffers())
            m.compact()
            p.check_all(f"compact {seed}")


@pytest.mark.parametrize("rows,children,width", [(1024, 4, 700), (1000, 1, 3000), (300, 299, 200)])
def test_few_children_of_many_rows(rows, children, width):
    """The old rows stay: references are counted by the children's entries."""
    rng = random.Random(children)
    m = Model(900, 4, width)
    m.rows, m.lens = [[-1] * width for _ in range(rows)], [0] * rows
    p = ListedPool(m, words=2)
    at = [rng.randrange(rows) for _ in range(12)] + [0, rows - 1]
    wanted = [rng.randrange(1, 4 * min(width, 40)) if r in at else 0 for r in range(rows)]
    p.take(wanted)
    m.take(wanted)
    parents = [rng.choice(at) for _ in range(children)]
    parents[-1] = parents[0]
    p.fork(parents, False)
    m.fork(parents, False)
    p.check_all("fork")


def test_forks_whose_old_rows_stay_cost_what_their_children_have():
    """Four children of a table of 1024 rows of 16384 entries as of one of four rows: a fork looks at its parents' entries alone (all the table's, by one block, would be some
    hundred times as long)."""
    times = {}
    for rows in (4, 1024):
        refs = torch.zeros(64, dtype=torch.int32, device="cuda")
        table = torch.full((rows, 16384), -1, dtype=torch.int32, device="cuda")
        lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        wanted = torch.zeros(rows, dtype=torch.int32, device="cuda")
        wanted[:4] = 100
        fq.pages_take(refs, 16, table, lens, wanted)
        parents = torch.arange(4, dtype=torch.int32, device="cuda")
        out, lens_out = torch.empty((4, 16384), dtype=torch.int32, device="cuda"), torch.empty(4, dtype=torch.int32, device="cuda")
        ws = torch.empty(fq.pages_fork_workspace_bytes(rows, 4), dtype=torch.uint8, device="cuda")
        least = float("inf")
        for i in range(12):
            refs[40:] = 0
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            fq.pages_fork(refs, 16, table, lens, parents, table_out=out, lens_out=lens_out, workspace=ws)
            end.record()
            end.synchronize()
            least = min(least, begin.elapsed_time(end))
        times[rows] = least
    assert times[1024] < 8 * times[4], times
