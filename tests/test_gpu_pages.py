"""The page calls against a model of them in plain Python: counts, tables, lengths and data are equal, call after call."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

PAGE = 64


@pytest.fixture(scope="module")
def rd():
    from paper_2508_09072_b200 import binding
    r = binding.Reader(0)
    yield r
    r.close()


def binding():
    from paper_2508_09072_b200 import binding as b
    return b


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32).reshape(-1).cuda() if np.ndim(x) < 2 else torch.tensor(np.asarray(x), dtype=torch.int32).cuda()


def pages(n):
    return (n + PAGE - 1) // PAGE


class Model:
    """refs, table, lens as lists; data[pool][page]: the page's content as bytes."""

    def __init__(self, rng, num_pages, rows, width, n_pools, page_bytes):
        self.refs, self.table, self.lens = [0] * num_pages, [[-1] * width for _ in range(rows)], [0] * rows
        self.pools = [rng.integers(0, 256, (num_pages, page_bytes), dtype=np.uint8) for _ in range(n_pools)]
        self.width = width

    def device(self):
        b = binding()
        return b.Pages(i32(self.refs), i32(self.table), i32(self.lens), [torch.from_numpy(p.copy()).cuda() for p in self.pools])

    def same(self, p):
        assert p.refs.tolist() == self.refs
        assert p.page_table.tolist() == self.table
        assert p.seq_lens.tolist() == self.lens
        for want, got in zip(self.pools, p.pools):
            assert np.array_equal(want, got.cpu().numpy().reshape(want.shape))

    def consistent(self):
        count = [0] * len(self.refs)
        for row in self.table:
            for e in row:
                if e >= 0:
                    count[e] += 1
        assert count == self.refs

    def fork(self, src, dst):
        b, st, new, seen = binding(), [], [], set()
        for s, d in zip(src, dst):
            ok_row = 0 <= s < len(self.lens) and 0 <= d < len(self.lens) and d not in seen
            if 0 <= d < len(self.lens):
                seen.add(d)
            if not ok_row:
                st.append(b.ERR_INVALID_ARG)
            elif not 0 <= self.lens[s] <= self.width * PAGE:
                st.append(b.ERR_CAPACITY)
            elif any(not 0 <= e < len(self.refs) for e in self.table[s][:pages(self.lens[s])]):
                st.append(b.ERR_BAD_PAGE)
            else:
                st.append(0)
                new.append((d, self.lens[s], self.table[s][:pages(self.lens[s])]))
        for _, _, row in new:
            for e in row:
                self.refs[e] += 1
        for d, n, row in new:
            for e in self.table[d]:
                if 0 <= e < len(self.refs):
                    self.refs[e] -= 1
            self.table[d] = row + [-1] * (self.width - len(row))
            self.lens[d] = n
        return st

    def reserve(self, rows, tokens):
        b, st, wants, seen = binding(), [], [], set()
        refs = list(self.refs)
        for r, t in zip(rows, tokens):
            want = []
            if not 0 <= r < len(self.lens) or t < 0 or r in seen:
                st.append(b.ERR_INVALID_ARG)
            elif self.lens[r] < 0 or self.lens[r] + t > self.width * PAGE:
                st.append(b.ERR_CAPACITY)
            else:
                n = self.lens[r]
                span = range(n // PAGE, pages(n + t)) if t else range(0)
                row = self.table[r]
                if any(row[e] >= len(refs) for e in span) or (t and n % PAGE and row[n // PAGE] < 0):
                    st.append(b.ERR_BAD_PAGE)
                else:
                    st.append(0)
                    want = [e for e in span if row[e] < 0 or refs[row[e]] > 1]
            if 0 <= r < len(self.lens):
                seen.add(r)
            wants.append(want)
        free = [p for p, c in enumerate(refs) if c == 0]
        at, full = 0, False
        for i, (r, want) in enumerate(zip(rows, wants)):
            if not want:
                continue
            if full or at + len(want) > len(free):
                full = True
                st[i] = b.ERR_CAPACITY
                continue
            for e in want:
                old, page = self.table[r][e], free[at]
                at += 1
                self.table[r][e] = page
                self.refs[page] = 1
                if old >= 0:
                    self.refs[old] -= 1
                if self.lens[r] % PAGE and e == self.lens[r] // PAGE:
                    for pool in self.pools:
                        pool[page] = pool[old]
        return st

    def free(self, rows, keep=None):
        b, st = binding(), []
        bad = {}
        for i, r in enumerate(rows):
            k = keep[i] if keep is not None else 0
            if not 0 <= r < len(self.lens) or k < 0:
                st.append(b.ERR_INVALID_ARG)
                continue
            st.append(0)
            for e in range(pages(k), self.width):
                old = self.table[r][e]
                self.table[r][e] = -1
                if old >= len(self.refs):
                    st[-1] = b.ERR_BAD_PAGE
                elif old >= 0:
                    self.refs[old] -= 1
            self.lens[r] = min(self.lens[r], k)
        return st

    def compact(self):
        used = sum(c != 0 for c in self.refs)
        holes = [p for p in range(used) if self.refs[p] == 0]
        movers = [p for p in range(used, len(self.refs)) if self.refs[p] != 0]
        to = dict(zip(movers, holes))
        for a, z in to.items():
            for pool in self.pools:
                pool[z] = pool[a]
            self.refs[z], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(e, e) for e in row] for row in self.table]
        return used


@pytest.mark.parametrize("seed,num_pages,rows,width,pools,page_bytes", [
    (0, 20, 6, 5, 2, 2304), (1, 100, 12, 12, 3, 16), (2, 300, 40, 9, 2, 36864), (3, 5000, 200, 40, 1, 48), (4, 37, 8, 70, 2, 16400), (5, 9000, 1100, 10, 1, 16)])
def test_random_sequences_of_calls(rd, seed, num_pages, rows, width, pools, page_bytes):
    rng = np.random.default_rng(seed)
    m = Model(rng, num_pages, rows, width, pools, page_bytes)
    p = m.device()
    for step in range(40):
        what = rng.integers(0, 10)
        n = int(rng.integers(1, rows + 1))
        if what < 4:
            r = rng.permutation(rows)[:n].tolist()
            t = rng.integers(0, max(2, 2 * PAGE * num_pages // (rows * 2)), n).tolist()
            assert rd.pages_reserve(p, i32(r), i32(t)).tolist() == m.reserve(r, t)
            # what was reserved is written: lengths grow where pages are there
            for row in range(rows):
                room = next((e for e in range(width) if m.table[row][e] < 0), width) * PAGE
                m.lens[row] = int(rng.integers(min(m.lens[row], room), room + 1))
            p.seq_lens.copy_(i32(m.lens))
        elif what < 7:
            src, dst = rng.integers(0, rows, n).tolist(), rng.permutation(rows)[:n].tolist()
            assert rd.pages_fork(p, i32(src), i32(dst)).tolist() == m.fork(src, dst)
        elif what < 9:
            r = rng.integers(0, rows, n).tolist()
            keep = None if rng.random() < 0.3 else rng.integers(0, width * PAGE + 5, n).tolist()
            st = rd.pages_free(p, i32(r), None if keep is None else i32(keep)).tolist()
            assert st == m.free(r, keep)
        else:
            assert rd.pages_compact(p).tolist() == [m.compact()]
            assert all(c == 0 for c in m.refs[sum(c != 0 for c in m.refs):])
        m.consistent()
        m.same(p)


def filled(rng, num_pages=60, rows=6, width=8, lens=(100, 64, 0, 200, 1, 0), pools=2, page_bytes=4608):
    m = Model(rng, num_pages, rows, width, pools, page_bytes)
    order = rng.permutation(num_pages).tolist()
    for r, n in enumerate(lens):
        for e in range(pages(n)):
            m.table[r][e] = order.pop()
            m.refs[m.table[r][e]] = 1
        m.lens[r] = n
    return m


def test_rows_are_permuted_at_once(rd):
    m = filled(np.random.default_rng(30))
    p = m.device()
    before = [list(x) for x in m.table]
    src, dst = [1, 0, 3, 3, 2], [0, 1, 3, 2, 4]
    assert rd.pages_fork(p, i32(src), i32(dst)).tolist() == m.fork(src, dst) == [0] * 5
    m.same(p)
    assert m.table[0] == before[1] and m.table[1] == before[0] and m.table[2] == before[3] and m.table[4] == before[2]


def test_requests_that_cannot_be(rd):
    b = binding()
    m = filled(np.random.default_rng(31))
    m.table[3][1] = 60            # outside the pool
    m.lens[4] = -1
    p = m.device()
    src, dst = [0, 9, 0, -1, 3, 4, 1, 0], [2, 2, 6, 1, 1, 5, 5, 4]
    want = m.fork(src, dst)
    assert rd.pages_fork(p, i32(src), i32(dst)).tolist() == want == [0, b.ERR_INVALID_ARG, b.ERR_INVALID_ARG, b.ERR_INVALID_ARG, b.ERR_INVALID_ARG,
                                                                     b.ERR_CAPACITY, b.ERR_INVALID_ARG, 0]
    m.same(p)
    m.lens[5] = 513               # longer than its row
    m.lens[2] = 70
    m.table[2][1] = -1            # committed positions without a page
    p = m.device()
    rows, tokens = [0, 0, 3, 5, 2, 7, 1, 4], [500, 1, 10, 0, 1, 1, -1, 1]
    want = m.reserve(rows, tokens)
    assert rd.pages_reserve(p, i32(rows), i32(tokens)).tolist() == want
    assert want[1] == b.ERR_INVALID_ARG and want[0] == want[3] == b.ERR_CAPACITY and want[4] == b.ERR_BAD_PAGE and want[5] == want[6] == b.ERR_INVALID_ARG
    m.same(p)
    rows, keep = [3, -1, 6, 0, 1], [0, 0, 0, 64, -2]
    want = m.free(rows, keep)
    assert rd.pages_free(p, i32(rows), i32(keep)).tolist() == want == [b.ERR_BAD_PAGE, b.ERR_INVALID_ARG, b.ERR_INVALID_ARG, 0, b.ERR_INVALID_ARG]
    m.same(p)


def test_a_pool_that_runs_out(rd):
    b = binding()
    m = filled(np.random.default_rng(32), num_pages=12)    # 7 in use
    p = m.device()
    rows, tokens = [1, 2, 0, 3, 4, 5], [64, 128, 28, 129, 5, 64]   # 1, 2, 0 (room in its page), 3 (two in the way), 0, 1
    want = m.reserve(rows, tokens)
    assert rd.pages_reserve(p, i32(rows), i32(tokens)).tolist() == want == [0, 0, 0, b.ERR_CAPACITY, 0, b.ERR_CAPACITY]
    m.same(p)


def test_shared_pages_are_copied_before_they_are_written(rd):
    m = filled(np.random.default_rng(33))
    p = m.device()
    assert rd.pages_fork(p, i32([0, 0]), i32([2, 5])).tolist() == m.fork([0, 0], [2, 5])
    rows = [2, 5, 0]              # all holders at once: a page each, the shared one is released
    shared = m.table[0][1]
    assert rd.pages_reserve(p, i32(rows), i32([1, 1, 1])).tolist() == m.reserve(rows, [1, 1, 1]) == [0, 0, 0]
    m.same(p)
    assert m.refs[shared] == 0 and m.refs[m.table[0][0]] == 3


@pytest.mark.parametrize("held", [0, 1, 499, 500])
def test_compaction_of_empty_and_full_pools(rd, held):
    rng = np.random.default_rng(34)
    m = Model(rng, 500, 10, 50, 2, 64)
    for i, page in enumerate(rng.permutation(500)[:held].tolist()):
        m.table[i // 50][i % 50] = page
        m.refs[page] = 1
    p = m.device()
    assert rd.pages_compact(p).tolist() == [m.compact()] == [held]
    m.same(p)
    assert rd.pages_compact(p).tolist() == [held]
    m.same(p)


def test_pages_held_outside_the_table_move_too_and_others_stay(rd):
    """A count of the caller's own keeps a page from being handed out; entries that name no page of the pool are left alone."""
    m = filled(np.random.default_rng(35))
    m.refs[59] = m.refs[59] + 1
    m.table[5][7] = 77
    p = m.device()
    assert rd.pages_compact(p).tolist() == [m.compact()]
    m.same(p)


def test_copies_between_pools(rd):
    b = binding()
    rng = np.random.default_rng(36)
    for page_bytes, n_pools in ((16, 1), (2304, 3), (16384 * 2 + 16, 2), (64, 140)):
        a = [torch.from_numpy(rng.integers(0, 256, (20, page_bytes), dtype=np.uint8)).cuda() for _ in range(n_pools)]
        z = [torch.zeros(9, page_bytes, dtype=torch.uint8, device="cuda") for _ in range(n_pools)]
        st = rd.pages_copy(a, z, i32([3, 19, 20, 0, -1, 7]), i32([8, 0, 1, 9, 2, 3]))
        assert st.tolist() == [0, 0, b.ERR_BAD_PAGE, b.ERR_BAD_PAGE, b.ERR_BAD_PAGE, 0]
        for x, y in zip(a, z):
            want = torch.zeros_like(y)
            want[8], want[0], want[3] = x[3], x[19], x[7]
            assert torch.equal(y, want)
    assert rd.pages_copy(a, z, i32([]), i32([])).tolist() == []


def test_bf16_pools_of_many_layers_and_captured_calls(rd):
    """150 pools; a captured step (free, fork, reserve) follows what the arrays hold at its replay."""
    b = binding()
    rng = np.random.default_rng(37)
    m = filled(rng, pools=150, page_bytes=2 * 64 * 16 * 2)
    p = m.device()
    p.pools = [x.view(torch.bfloat16).view(60, 2, 64, 16) for x in p.pools]
    src, dst, tokens = i32([0, 3]), i32([2, 5]), i32([3, 70])
    status = [torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(3)]
    ws = torch.empty_like(rd.pages_workspace(p, 2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rd.pages_free(p, dst, status=status[0])
        rd.pages_fork(p, src, dst, status=status[1], workspace=ws)
        rd.pages_reserve(p, dst, tokens, status=status[2], workspace=ws)
    as_model = lambda: b.Pages(p.refs, p.page_table, p.seq_lens, [x.view(torch.uint8) if x.dtype == torch.uint8 else x.view(60, -1).view(torch.uint8) for x in p.pools])  # noqa: E731
    for s, d, t in (([0, 3], [2, 5], [3, 70]), ([1, 3], [5, 0], [1, 1]), ([3, 3], [1, 4], [64, 0])):
        src.copy_(i32(s)), dst.copy_(i32(d)), tokens.copy_(i32(t))
        graph.replay()
        torch.cuda.synchronize()
        assert status[0].tolist() == m.free(d) and status[1].tolist() == m.fork(s, d) and status[2].tolist() == m.reserve(d, t)
        m.same(as_model())


def test_workspaces_of_earlier_calls_stay(rd):
    """The reader's own workspace is replaced by a larger one, never given back: a captured call may still use it."""
    m = filled(np.random.default_rng(38))
    p = m.device()
    a = rd.pages_workspace(p, 1)
    large = rd.pages_workspace(p, 100000)
    assert large.numel() > a.numel() and rd.pages_workspace(p, 1) is large and any(x is a for x in rd._pages_ws)


def test_more_rows_than_threads(rd):
    rng = np.random.default_rng(39)
    rows, width = 20000, 3
    m = Model(rng, 50000, rows, width, 1, 16)
    p = m.device()
    t = rng.integers(0, 130, rows).tolist()
    r = rng.permutation(rows).tolist()
    assert rd.pages_reserve(p, i32(r), i32(t)).tolist() == m.reserve(r, t)
    for i, x in zip(r, t):
        m.lens[i] = x
    p.seq_lens.copy_(i32(m.lens))
    src, dst = rng.integers(0, rows, 15000).tolist(), rng.permutation(rows)[:15000].tolist()
    assert rd.pages_fork(p, i32(src), i32(dst)).tolist() == m.fork(src, dst)
    t = rng.integers(0, 30, rows).tolist()
    assert rd.pages_reserve(p, i32(r), i32(t)).tolist() == m.reserve(r, t)
    m.same(p)
    assert rd.pages_free(p, i32(r[::2]), None).tolist() == m.free(r[::2])
    assert rd.pages_compact(p).tolist() == [m.compact()]
    m.same(p)


@pytest.mark.parametrize("num_pages", [300, 6000])
@pytest.mark.parametrize("n", [2, 31, 32, 33, 512, 513, 1500])
def test_rows_named_more_than_once(rd, n, num_pages):
    """The first request that names a row is the one that counts, however many there are."""
    rng = np.random.default_rng(n)
    rows, width = 700, 6
    m = Model(rng, num_pages, rows, width, 1, 16)
    p = m.device()
    r = rng.integers(-2, rows + 2, n).tolist()
    r[n - 1] = r[0] = 5
    t = rng.integers(0, 2 * PAGE, n).tolist()
    assert rd.pages_reserve(p, i32(r), i32(t)).tolist() == m.reserve(r, t)
    m.same(p)
    for row in range(rows):
        m.lens[row] = next((e for e in range(width) if m.table[row][e] < 0), width) * PAGE
    p.seq_lens.copy_(i32(m.lens))
    src = rng.integers(0, rows, n).tolist()
    assert rd.pages_fork(p, i32(src), i32(r)).tolist() == m.fork(src, r)
    m.same(p)


@pytest.mark.parametrize("held", [0, 1, 4999, 5000])
def test_compaction_of_large_pools(rd, held):
    rng = np.random.default_rng(36)
    m = Model(rng, 5000, 100, 50, 1, 32)
    for i, page in enumerate(rng.permutation(5000)[:held].tolist()):
        m.table[i // 50][i % 50] = page
        m.refs[page] = 1
    p = m.device()
    assert rd.pages_compact(p).tolist() == [m.compact()] == [held]
    m.same(p)
