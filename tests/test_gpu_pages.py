"""as_pages_fork / grow / compact against a plain page-by-page model: exact equality."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2210_15458_b200 import binding
    return binding


class Model:
    """Lanes as lists of page ids, contents as python lists."""

    def __init__(self, n_pages, page_size, max_pages):
        self.P, self.M = page_size, max_pages
        self.ref = [0] * n_pages
        self.rows, self.lens = [], []

    def take(self):
        for g, r in enumerate(self.ref):
            if r == 0:
                self.ref[g] = 1
                return g
        return None

    def grow(self, add):
        status, out = [], False
        free = self.ref.count(0)
        wanted = 0
        for i, a in enumerate(add):
            n, m = self.lens[i], self.lens[i] + a
            if a < 0 or n < 0 or m > self.M * self.P:
                status.append(-1)
                continue
            need = -(-m // self.P) - -(-n // self.P)
            wanted += need
            if need and wanted > free:
                status.append(-6)
                continue
            self.rows[i] += [self.take() for _ in range(need)]
            self.lens[i] = m
            status.append(0)
        return status

    def fork(self, parent):
        kids = [[i for i, p in enumerate(parent) if p == j] for j in range(len(self.rows))]
        for j, row in enumerate(self.rows):
            for m, g in enumerate(row):
                part = (m + 1) * self.P > self.lens[j]
                self.ref[g] += (min(len(kids[j]), 1) if part else len(kids[j])) - 1
        rows, lens, status, moves = [], [], [], []
        for i, p in enumerate(parent):
            if p < 0 or p >= len(self.rows):
                rows.append([]), lens.append(0), status.append(0 if p == -1 else -1)
                continue
            row, n, st = list(self.rows[p]), self.lens[p], 0
            if n % self.P and kids[p][0] != i:
                g = self.take()
                if g is None:
                    row.pop()
                    n, st = n // self.P * self.P, -6
                else:
                    moves.append((row[-1], g))
                    row[-1] = g
            rows.append(row), lens.append(n), status.append(st)
        self.rows, self.lens = rows, lens
        return status, moves

    def compact(self):
        used = sum(r > 0 for r in self.ref)
        holes = [g for g in range(used) if self.ref[g] == 0]
        late = [g for g in range(used, len(self.ref)) if self.ref[g] > 0]
        to = dict(zip(late, holes))
        for s, d in to.items():
            self.ref[d], self.ref[s] = self.ref[s], 0
        self.rows = [[to.get(g, g) for g in row] for row in self.rows]
        return used, list(to.items())

    def table(self):
        return torch.tensor([r + [-1] * (self.M - len(r)) for r in self.rows], dtype=torch.int32).view(len(self.rows), self.M)


def same(m, table, length, ref):
    assert torch.equal(table.cpu(), m.table())
    assert length.tolist() == m.lens and ref.tolist() == m.ref


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("n_pages,P,M,lanes", [(7, 4, 3, 2), (40, 16, 6, 5), (300, 3, 20, 37), (5000, 64, 30, 200), (20000, 16, 90, 1500)])
def test_a_life_of_the_pool(B, seed, n_pages, P, M, lanes):
    rnd = random.Random(seed * 1000 + n_pages)
    m = Model(n_pages, P, M)
    m.rows, m.lens = [[] for _ in range(lanes)], [0] * lanes
    table = torch.full((lanes, M), -1, dtype=torch.int32, device="cuda")
    length = torch.zeros(lanes, dtype=torch.int32, device="cuda")
    ref = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    pool = torch.randint(0, 1 << 30, (3, n_pages, 8), dtype=torch.int32, device="cuda")
    held = pool.cpu().clone()
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for step in range(6):
        add = [rnd.choice((0, 1, 1, P, rnd.randint(0, M * P // 2))) for _ in range(len(m.rows))]
        if step == 2:
            add[0] = -1
        status = torch.empty(len(add), dtype=torch.int32, device="cuda")
        B.as_pages_grow(i32(add), table, length, ref, P, lane_status=status)
        assert status.tolist() == m.grow(add)
        same(m, table, length, ref)
        n = len(m.rows)
        parent = [rnd.choice((-1, rnd.randrange(n), rnd.randrange(min(n, 3)))) for _ in range(rnd.choice((n, max(1, n // 2), lanes)))]
        if step == 3:
            parent[0] = n + 5
        status = torch.empty(len(parent), dtype=torch.int32, device="cuda")
        table, length, ref = B.as_pages_fork(i32(parent), table, length, ref, P, pool, ref_out=ref if step % 2 else None, lane_status=status)
        want, moves = m.fork(parent)
        assert status.tolist() == want
        same(m, table, length, ref)
        for s, d in moves:
            held[:, d] = held[:, s]
        assert torch.equal(pool.cpu(), held)
        if step % 2:
            used = B.as_pages_compact(table, ref, pool)
            want, moves = m.compact()
            assert int(used) == want
            same(m, table, length, ref)
            for s, d in moves:
                held[:, d] = held[:, s]
            assert torch.equal(pool.cpu(), held)


def test_the_pool_runs_out(B):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, length, ref = torch.full((4, 3), -1, dtype=torch.int32, device="cuda"), i32([0, 0, 0, 0]), i32([1, 0, 1, 0, 0])
    status = i32([9, 9, 9, 9])
    B.as_pages_grow(i32([4, 9, 1, 0]), table, length, ref, 4, lane_status=status)
    # lane 0 gets page 1; lane 1 wants three of the two left; lane 2 stands behind it; lane 3 wants none
    assert status.tolist() == [0, B.ERR_NO_PAGES, B.ERR_NO_PAGES, 0]
    assert table.tolist() == [[1, -1, -1]] + [[-1] * 3] * 3 and length.tolist() == [4, 0, 0, 0] and ref.tolist() == [1, 1, 1, 0, 0]
    # a part page, three children, one page for a copy
    table, length, ref = i32([[2, 0, -1]]), i32([6]), i32([1, 1, 1])
    status = i32([9, 9, 9])
    t, n, r = B.as_pages_fork(i32([0, 0, 0]), table, length, torch.cat([ref, i32([0])]), 4, lane_status=status)
    assert status.tolist() == [0, 0, B.ERR_NO_PAGES] and n.tolist() == [6, 6, 4]
    assert t.tolist() == [[2, 0, -1], [2, 3, -1], [2, -1, -1]] and r.tolist() == [1, 1, 3, 1]


def test_bad_rows_are_read_as_empty(B):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, length, ref = i32([[0, 9], [1, -1], [2, 3]]), i32([8, 3, 99]), i32([1, 1, 1, 1])
    status = i32([9] * 4)
    t, n, r = B.as_pages_fork(i32([0, 1, 2, -1]), table, length, ref, 4, lane_status=status)
    assert status.tolist() == [B.ERR_INVALID_ARG, 0, B.ERR_INVALID_ARG, 0]
    assert n.tolist() == [0, 3, 0, 0] and t.tolist() == [[-1, -1], [1, -1], [-1, -1], [-1, -1]] and r.tolist() == [1, 1, 1, 1]


def test_copies_of_odd_sizes_and_no_lanes(B):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for words in (4, 12, 4096, 4100, 20004):
        pool = torch.randint(0, 1 << 30, (2, 5, words), dtype=torch.int32, device="cuda")
        want = pool.clone()
        t, n, r = B.as_pages_fork(i32([0, 0, 0]), i32([[4]]), i32([1]), i32([0, 0, 0, 0, 1]), 2, pool)
        want[:, 0], want[:, 1] = want[:, 4], want[:, 4]
        assert t.tolist() == [[4], [0], [1]] and torch.equal(pool, want)
    ref = i32([1, 0, 2])
    t, n, r = B.as_pages_fork(i32([]), torch.empty(0, 2, dtype=torch.int32, device="cuda"), i32([]), ref, 4)
    assert t.shape == (0, 2) and r.tolist() == [1, 0, 2]
    t, n, r = B.as_pages_fork(i32([]), i32([[0, 2]]), i32([8]), i32([1, 0, 1]), 4)      # every lane dropped
    assert r.tolist() == [0, 0, 0]
    used = B.as_pages_compact(torch.empty(0, 2, dtype=torch.int32, device="cuda"), ref)
    assert int(used) == 2 and ref.tolist() == [1, 2, 0]


def test_other_stream(B):
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, length, ref = i32([[0, 1], [2, -1]]), i32([5, 2]), i32([1, 1, 1, 0, 0, 0])
    pool = torch.arange(2 * 6 * 4, dtype=torch.int32, device="cuda").view(2, 6, 4)
    parent = i32([0, 1, 0, 1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        t, n, r = B.as_pages_fork(parent, table, length, ref, 4, pool)
        B.as_pages_grow(i32([1, 1, 1, 4]), t, n, r, 4)
    s.synchronize()
    assert t.tolist() == [[0, 1], [2, -1], [0, 3], [4, 5]] and n.tolist() == [6, 3, 6, 6] and r.tolist() == [2, 1, 1, 1, 1, 1]
    assert torch.equal(pool[:, 3], pool[:, 1]) and torch.equal(pool[:, 4], pool[:, 2])


def test_compact_leaves_entries_of_pages_that_nobody_holds(B):
    """Rows that a finished lane left behind name free pages: below the pages in use, or behind them.  They stay."""
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table, ref = i32([[7, 2, -1], [5, 9, 3], [8, 1, 100]]), i32([0, 1, 1, 0, 0, 0, 0, 1, 0, 0])      # 5, 9, 3 and 8 are free
    work = torch.full((B.as_pages_work_bytes(3, 3, 10) // 4,), 0x77777777, dtype=torch.int32, device="cuda")
    used = B.as_pages_compact(table, ref, work=work)
    assert int(used) == 3 and ref.tolist() == [1, 1, 1] + [0] * 7
    assert table.tolist() == [[0, 2, -1], [5, 9, 3], [8, 1, 100]]
