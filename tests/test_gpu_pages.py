"""Pages that sequences share, against a model of them in Python: tables, references, lengths and contents, exactly."""
import random

import pytest
import torch

from paper_2308_09723_amd import fq

pytestmark = pytest.mark.gpu


class Model:
    """The definition: a pool, rows of pages, and what the pages hold."""

    def __init__(self, pages, page, width):
        self.page, self.width, self.refs = page, width, [0] * pages
        self.rows, self.lens, self.holds = [], [], list(range(1000, 1000 + pages))

    def used(self, length):
        return min(self.width, -(-max(0, length) // self.page))

    def free_pages(self):
        return [p for p, r in enumerate(self.refs) if r <= 0]

    def refer(self, p, by):
        if 0 <= p < len(self.refs):
            self.refs[p] += by

    def take(self, wanted):
        short, free, at = False, self.free_pages(), 0
        for r, want in enumerate(wanted):
            if self.lens[r] < 0 or want <= self.lens[r] or -(-want // self.page) > self.width:
                continue
            have, need = self.used(self.lens[r]), self.used(want) - self.used(self.lens[r])
            if need and (short or len(free) - at < need):
                short = True
                continue
            for j in range(have, have + need):
                p = free[at]
                at += 1
                self.refs[p], self.rows[r][j] = 1, p
            self.lens[r] = want

    def fork(self, parents, release):
        old, lens, first = [list(r) for r in self.rows], list(self.lens), {}
        rows, out, wants = [], [], []
        for i, p in enumerate(parents):
            row, length = [-1] * self.width, lens[p] if 0 <= p < len(old) else 0
            fits = -(-max(0, length) // self.page) <= self.width
            whole = max(0, length) // self.page if fits else self.width
            part = fits and length > 0 and length % self.page != 0
            for j in range(whole):
                row[j] = old[p][j]
                self.refer(row[j], 1)
            if part and release and p not in first:
                row[whole] = old[p][whole]
            elif part:
                wants.append((i, p, whole))
            if 0 <= p < len(old):
                first.setdefault(p, i)
            rows.append(row)
            out.append(length)
        if release:
            for r, row in enumerate(old):
                for j in range(self.used(lens[r])):
                    if not (j == lens[r] // self.page and r in first):
                        self.refer(row[j], -1)
        short, copies, free = [], [], self.free_pages()
        for n, (i, p, whole) in enumerate(wants):
            if n >= len(free):
                short.append((i, whole))
                continue
            page = free[n]
            rows[i][whole], self.refs[page] = page, 1
            copies.append((old[p][whole], page))
        for i, whole in short:
            for j in range(whole):
                self.refer(rows[i][j], -1)
            rows[i], out[i] = rows[i][:0] + [-1] * whole + rows[i][whole:], -1
        for a, b in copies:
            if 0 <= a < len(self.refs):
                self.holds[b] = self.holds[a]
        self.rows, self.lens = rows, out

    def free(self, which):
        for r in which:
            if 0 <= r < len(self.rows):
                for j in range(self.used(self.lens[r])):
                    self.refer(self.rows[r][j], -1)
                    self.rows[r][j] = -1
                self.lens[r] = 0

    def compact(self):
        used = sum(r > 0 for r in self.refs)
        holes = [p for p in range(used) if self.refs[p] <= 0]
        moved = dict(zip([p for p in range(used, len(self.refs)) if self.refs[p] > 0], holes))
        for a, b in moved.items():
            self.refs[b], self.refs[a], self.holds[b] = self.refs[a], 0, self.holds[a]
        for r, row in enumerate(self.rows):
            for j in range(self.used(self.lens[r])):
                row[j] = moved.get(row[j], row[j])


class Pool:
    """The same on the device; every page of two buffers (one of three tensors, one a list's) is filled with a number."""

    def __init__(self, model, words=40):
        self.m = model
        n = len(model.refs)
        self.refs = torch.tensor(model.refs, dtype=torch.int32).cuda()
        self.stack = torch.zeros((3, n, words), dtype=torch.int64, device="cuda")
        self.other = torch.zeros((n, 5, 8 * words), dtype=torch.float16, device="cuda")
        self.stack += torch.tensor(model.holds).cuda()[None, :, None]
        self.other += torch.tensor(model.holds).cuda()[:, None, None].half()
        self.set_rows()

    def set_rows(self):
        self.table = torch.tensor(self.m.rows, dtype=torch.int32).view(len(self.m.rows), self.m.width).cuda()
        self.lens = torch.tensor(self.m.lens, dtype=torch.int32).cuda()

    def take(self, wanted):
        fq.pages_take(self.refs, self.m.page, self.table, self.lens, torch.tensor(wanted, dtype=torch.int32).cuda())

    def fork(self, parents, release):
        parents = torch.tensor(parents, dtype=torch.int32).cuda()
        self.table, self.lens = fq.pages_fork(self.refs, self.m.page, self.table, self.lens, parents, self.stack, release=release)

    def check(self, what):
        assert self.refs.tolist() == self.m.refs, what
        assert self.lens.tolist() == self.m.lens, what
        for r, row in enumerate(self.table.tolist()):
            n = self.m.used(self.m.lens[r])
            assert row[:n] == self.m.rows[r][:n], f"{what}: row {r}"

    def check_holds(self, what):
        want = torch.tensor(self.m.holds).cuda()
        assert bool((self.stack == want[None, :, None]).all()), what


@pytest.mark.parametrize("seed,pages,page,width,rows", [(0, 40, 16, 8, 5), (1, 300, 16, 20, 30), (2, 9, 4, 3, 6), (3, 5000, 64, 60, 100), (4, 700, 1, 25, 40), (5, 3, 16, 2, 4)])
def test_steps_of_a_pool(seed, pages, page, width, rows):
    """Rows grow, fork, are given up and gathered, in any order, with too few pages now and then."""
    rng = random.Random(seed)
    m = Model(pages, page, width)
    m.rows, m.lens = [[-1] * width for _ in range(rows)], [0] * rows
    m.lens[rng.randrange(rows)] = -1
    p = Pool(m)
    for step in range(14):
        kind = rng.choice(["take", "take", "fork", "release", "free", "compact"])
        what = f"step {step}: {kind}"
        if kind == "take":
            wanted = [min(width * page + rng.choice([0, 0, 1]), max(0, n) + rng.randrange(0, 3 * page)) for n in m.lens]
            p.take(wanted)
            m.take(wanted)
        elif kind in ("fork", "release"):
            parents = [rng.randrange(-1, len(m.rows) + 1) for _ in range(rows)]
            release = kind == "release"
            if not release:       # the old rows go on as well
                old = (p.table.clone(), p.lens.clone(), [list(r) for r in m.rows], list(m.lens))
            p.fork(parents, release)
            m.fork(parents, release)
            if not release:
                p.check(what)
                p.check_holds(what)
                m.rows, m.lens = m.rows[:rows // 2] + old[2][rows // 2:], m.lens[:rows // 2] + old[3][rows // 2:]
                lost = Model(pages, page, width)      # (what is dropped is freed)
                lost.refs, lost.rows, lost.lens = m.refs, [list(r) for r in p.table.tolist()[rows // 2:]] + old[2][:rows // 2], p.lens.tolist()[rows // 2:] + old[3][:rows // 2]
                table, lens = torch.cat([p.table[rows // 2:], old[0][:rows // 2]]).contiguous(), torch.cat([p.lens[rows // 2:], old[1][:rows // 2]])
                lost.free(range(len(lost.rows)))
                fq.pages_free(p.refs, page, table, lens)
                assert int(table.max()) == -1 if table.numel() and bool((lens >= 0).any()) else True
                p.table, p.lens = torch.cat([p.table[:rows // 2], old[0][rows // 2:]]).contiguous(), torch.cat([p.lens[:rows // 2], old[1][rows // 2:]])
        elif kind == "free":
            which = [rng.randrange(-1, len(m.rows) + 1) for _ in range(rng.randrange(1, 4))]
            which.append(which[0])       # twice
            fq.pages_free(p.refs, page, p.table, p.lens, torch.tensor(which, dtype=torch.int32).cuda())
            m.free(which)
        else:
            fq.pages_compact(p.refs, page, p.table, p.lens, p.stack)
            m.compact()
        p.check(what)
        p.check_holds(what)
    assert all(r >= 0 for r in m.refs)


def test_large_tables():
    """Above what one block does alone: 300 rows of 400 entries, 90 000 pages."""
    rng = random.Random(9)
    m = Model(90000, 16, 400)
    m.refs[0], m.refs[1], m.refs[5000] = 1, 1, 1       # kept for something else
    m.rows, m.lens = [[-1] * 400 for _ in range(300)], [0] * 300
    p = Pool(m, words=2)
    wanted = [rng.randrange(0, 6400) for _ in range(300)]
    p.take(wanted)
    m.take(wanted)
    p.check("take")
    for release in (False, True):
        parents = [rng.randrange(300) for _ in range(300)]
        p.fork(parents, release)
        m.fork(parents, release)
        p.check(f"fork {release}")
        p.check_holds(f"fork {release}")
    fq.pages_free(p.refs, 16, p.table, p.lens, torch.arange(0, 300, 3, dtype=torch.int32).cuda())
    m.free(range(0, 300, 3))
    p.check("free")
    # (the rows of the first fork's parents were dropped: their pages stay used)
    fq.pages_compact(p.refs, 16, p.table, p.lens, p.stack)
    m.compact()
    p.check("compact")
    p.check_holds("compact")


def test_copies():
    """Pairs outside the pool and pages onto themselves are left out; buffers of odd sizes, strided ones, more than a launch's."""
    gen = torch.Generator().manual_seed(2)
    for shapes in ([(7, 3, 8)], [(7, 16), (7, 4000), (7, 5, 24)], [(7, 8 + 8 * (i % 5)) for i in range(45)]):
        host = [torch.randint(-9, 9, s, generator=gen).half() for s in shapes]
        device = [torch.zeros((7, 2) + tuple(s[1:]), dtype=torch.float16, device="cuda") for s in shapes]       # every other page's room is not the buffer's
        views = [d[:, 0] for d in device]
        for v, h in zip(views, host):
            v.copy_(h)
        fq.pages_copy(views, torch.tensor([0, 3, -1, 7, 5, 6], dtype=torch.int32).cuda(), torch.tensor([1, 4, 2, 2, 5, -1], dtype=torch.int32).cuda())
        for v, h, d in zip(views, host, device):
            h[1], h[4] = h[0], h[3]
            assert torch.equal(v.cpu(), h) and not bool(d[:, 1].any())


def test_copies_refuse():
    x = torch.zeros((4, 8, 16), dtype=torch.float16, device="cuda")
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    for bad in ([x.transpose(1, 2)], [x[:, :, :8]], x.cpu(), [x[:, 0, :4]]):
        with pytest.raises((fq.FqError, IndexError)):
            fq.pages_copy(bad, at, at + 1)
    with pytest.raises(fq.FqError):
        fq.pages_copy([x], at.long(), at)
    with pytest.raises(fq.FqError):
        fq.pages_copy([x, x[:3]], at, at + 1)


def test_captured_steps():
    """A step of beams that is captured and replayed goes on as eager ones do."""
    rng = random.Random(4)
    m = Model(60, 16, 10)
    m.rows, m.lens = [[-1] * 10 for _ in range(6)], [0] * 6
    p = Pool(m)
    p.take([70, 3, 70, 71, 16, 0])
    m.take([70, 3, 70, 71, 16, 0])
    parents, out, lens_out = torch.zeros(6, dtype=torch.int32, device="cuda"), p.table.clone(), p.lens.clone()
    one = torch.ones(6, dtype=torch.int32, device="cuda")
    ws = torch.empty(fq.pages_fork_workspace_bytes(6, 6), dtype=torch.uint8, device="cuda")
    grown = p.lens.clone()

    def step():
        torch.add(p.lens, one, out=grown)
        fq.pages_take(p.refs, 16, p.table, p.lens, grown)
        fq.pages_fork(p.refs, 16, p.table, p.lens, parents, p.stack, release=True, table_out=out, lens_out=lens_out, workspace=ws)
        p.table.copy_(out)
        p.lens.copy_(lens_out)

    def model(new):
        m.take([n + 1 for n in m.lens])
        m.fork(new, True)

    def choose():
        new = [rng.randrange(6) for _ in range(6)]
        parents.copy_(torch.tensor(new, dtype=torch.int32))
        return new

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        new = choose()
        step()
        model(new)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(30):
        new = choose()
        graph.replay()
        model(new)
        if i % 4 == 0:       # eager steps in between
            torch.cuda.synchronize()
            new = choose()
            step()
            model(new)
        p.check(f"replay {i}")
        p.check_holds(f"replay {i}")


def test_pages_beyond_four_gigabytes():
    pages, words = 5000, 1 << 18       # 1 MiB a page
    cache = torch.zeros((pages, words), dtype=torch.int32, device="cuda")
    cache[4999] = torch.arange(words, device="cuda").int()
    cache[4500] = 7
    fq.pages_copy([cache], torch.tensor([4999, 4500], dtype=torch.int32).cuda(), torch.tensor([4300, 2], dtype=torch.int32).cuda())
    assert torch.equal(cache[4300], cache[4999]) and bool((cache[2] == 7).all())
    assert int(cache[4299].any()) + int(cache[4301].any()) + int(cache[3].any()) == 0


@pytest.mark.parametrize("rows,children,width", [(0, 3, 4), (3, 0, 4), (5, 7, 0), (1, 1, 1), (1024, 1024, 60), (1025, 3, 2), (1, 1025, 3), (1024, 1024, 70)])
def test_forks_of_any_size(rows, children, width):
    """No rows, no children, tables without entries; where one block ends to do it all."""
    rng = random.Random(rows + children)
    page = 4
    m = Model(3 * rows + children + 5000, page, width)
    m.rows, m.lens = [[-1] * width for _ in range(rows)], [0] * rows
    p = Pool(m, words=2)
    if rows:
        wanted = [rng.randrange(0, 3 * page) for _ in range(rows)]
        p.take(wanted)
        m.take(wanted)
        p.check("take")
    for release in (False, True):
        parents = [rng.randrange(-1, rows + 1) for _ in range(children)]
        if not release:
            kept = (p.table, p.lens, m.rows, m.lens)
        p.fork(parents, release)
        m.fork(parents, release)
        p.check(f"fork {release}")
        p.check_holds(f"fork {release}")
        if not release:
            p.table, p.lens = kept[:2]
            m.rows, m.lens = [list(r) for r in kept[2]], list(kept[3])
