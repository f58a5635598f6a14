"""Copying, forking, freeing and compacting the pages of a cache against the same done on the host, a page at a time."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09800_b200 import build
    build.build()
    return t


@pytest.fixture(scope="module")
def serving(torch):
    from paper_2609_09800_b200 import serving as mod
    return mod


@pytest.fixture(scope="module")
def hbf(torch):
    from paper_2609_09800_b200 import hbf as mod
    return mod


class Cache:
    """A cache on the device and the same state in lists; `expect_*` change the lists."""

    def __init__(self, torch, slabs, pages, words, page, rows, cols, seed=0, layout="slabs"):
        g = torch.Generator(device="cuda"); g.manual_seed(seed)
        self.torch, self.page, self.cols = torch, page, cols
        rnd = lambda *s: torch.randint(-2 ** 31, 2 ** 31 - 1, s, device="cuda", generator=g, dtype=torch.int32)
        if layout == "slabs":
            self.data = rnd(slabs, pages, words)
        elif layout == "pages":                              # all slabs of a page side by side
            self.data = rnd(pages, slabs, words).transpose(0, 1)
        else:                                                # gaps behind pages and slabs
            self.data = rnd(slabs, pages + 1, words + 4)[:, :pages, :words]
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        wide = torch.full((rows, cols + 3), -1, dtype=torch.int32, device="cuda")
        self.tables = wide[:, :cols]
        self.h_refs, self.h_lens, self.h_tables = [0] * pages, [0] * rows, [[-1] * cols for _ in range(rows)]
        self.h_data = self.data.clone()
        self.order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()

    def fill(self, row, length):
        """Gives an empty row its tokens, on pages in no order."""
        for j in range(-(-length // self.page)):
            p = next(p for p in self.order if self.h_refs[p] == 0)
            self.h_refs[p], self.h_tables[row][j] = 1, p
        self.h_lens[row] = length

    def upload(self):
        t = self.torch
        self.refs.copy_(t.tensor(self.h_refs)); self.lens.copy_(t.tensor(self.h_lens, dtype=t.int32).reshape(-1))
        if self.h_lens:
            self.tables.copy_(t.tensor(self.h_tables))

    def plan(self, serving, **kw):
        return serving.CachePages(self.data, self.refs, self.tables, self.lens, self.page, **kw)

    def ints(self, v):
        return self.torch.tensor(v, dtype=self.torch.int32, device="cuda")

    def held(self, row):
        return -(-self.h_lens[row] // self.page)

    def move(self, moves):
        for a, b in moves:
            self.h_data[:, b] = self.h_data[:, a]
        return len(moves)

    def expect_fork(self, parents, children):
        free, moves, lens, tables = [p for p, r in enumerate(self.h_refs) if r == 0], [], list(self.h_lens), [list(r) for r in self.h_tables]
        for a, c in zip(parents, children):
            self.h_lens[c], self.h_tables[c] = lens[a], [-1] * self.cols
            for j in range(-(-lens[a] // self.page)):
                p = tables[a][j]
                if (j + 1) * self.page > lens[a]:
                    q = free.pop(0); moves.append((p, q)); p = q
                self.h_refs[p] += 1; self.h_tables[c][j] = p
        return self.move(moves)

    def expect_free(self, rows):
        for r in rows:
            for j in range(self.held(r)):
                self.h_refs[self.h_tables[r][j]] -= 1
            self.h_lens[r], self.h_tables[r] = 0, [-1] * self.cols

    def expect_compact(self):
        n = sum(r > 0 for r in self.h_refs)
        moves = list(zip([p for p in range(n, len(self.h_refs)) if self.h_refs[p] > 0], [p for p in range(n) if self.h_refs[p] <= 0]))
        to = dict(moves)
        for r in range(len(self.h_lens)):
            for j in range(self.held(r)):
                self.h_tables[r][j] = to.get(self.h_tables[r][j], self.h_tables[r][j])
        for a, b in moves:
            self.h_refs[b], self.h_refs[a] = self.h_refs[a], 0
        return self.move(moves), n

    def check(self):
        t = self.torch
        assert self.refs.tolist() == self.h_refs and self.lens.tolist() == self.h_lens and self.tables.tolist() == self.h_tables
        assert t.equal(self.data, self.h_data)


SIZES = [
    # slabs, pages, words of 4 bytes, tokens a page, rows, columns
    (1, 8, 4, 1, 4, 3), (3, 40, 12, 4, 9, 10), (2, 200, 1028, 7, 30, 12), (5, 3000, 4, 16, 60, 80), (96, 64, 256, 16, 10, 9), (1, 70_000, 4, 2, 40, 900),
]


@pytest.mark.parametrize("layout", ["slabs", "pages", "gaps"])
@pytest.mark.parametrize("size", SIZES, ids=["x".join(map(str, s)) for s in SIZES])
def test_a_life_of_forks_frees_and_compactions(torch, serving, size, layout):
    slabs, pages, words, page, rows, cols = size
    c = Cache(torch, *size, seed=pages, layout=layout)
    rng = torch.Generator().manual_seed(pages + 1)
    rnd = lambda n: int(torch.randint(0, n, (1,), generator=rng))
    for r in range(rows // 3):
        most = min(cols, sum(x == 0 for x in c.h_refs) // 2) * page
        c.fill(r, rnd(most + 1))
    c.upload()
    plan = c.plan(serving)
    for turn in range(4):
        empty, full = [r for r in range(rows) if c.h_lens[r] == 0], [r for r in range(rows) if c.h_lens[r]]
        n = min(len(empty), 1 + rnd(max(1, rows // 3)), sum(x == 0 for x in c.h_refs)) if full else 0
        parents, children = [full[rnd(len(full))] for _ in range(n)], [empty[i] for i in torch.randperm(len(empty), generator=rng).tolist()[:n]]
        moved = c.expect_fork(parents, children)
        plan.fork(c.ints(parents), c.ints(children))
        assert plan.result()["moved"] == moved
        c.check()
        full = [r for r in range(rows) if c.h_lens[r]]
        gone = [full[i] for i in torch.randperm(len(full), generator=rng).tolist()[:1 + len(full) // 3]] if full else []
        c.expect_free(gone)
        plan.free(c.ints(gone))
        plan.result()
        c.check()
        if turn % 2:
            moved, n = c.expect_compact()
            plan.compact()
            assert plan.result() == {"moved": moved, "in_use": n}
            c.check()
            plan.compact()                                   # once more: nothing is left to move
            assert plan.result() == {"moved": 0, "in_use": n}
            c.check()


@pytest.mark.parametrize("layout", ["slabs", "pages", "gaps"])
@pytest.mark.parametrize("n", [0, 1, 7, 100])
def test_copy(torch, serving, n, layout):
    c = Cache(torch, 3, 210, 36, 4, 2, 5, layout=layout)
    plan = c.plan(serving)
    src, dst = [c.order[i // 2] for i in range(n)], c.order[100:100 + n]          # a source may be read twice
    moved = c.move(list(zip(src, dst)))
    plan.copy(c.ints(src), c.ints(dst))
    assert plan.result()["moved"] == moved == n
    c.check()


def test_a_fork_of_a_row_that_is_a_child_too_takes_it_as_it_was(torch, serving):
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    c.fill(0, 10); c.fill(1, 8)
    c.upload()
    plan = c.plan(serving)
    parents, children = [0, 3, 0, 1], [3, 4, 5, 2]            # row 3 was empty: row 4 stays so
    c.expect_fork(parents, children)
    plan.fork(c.ints(parents), c.ints(children))
    assert plan.result()["moved"] == 2
    c.check()
    assert c.h_lens[4] == 0


REFUSED = {
    "copy to a page named twice": lambda c, p: p.copy(c.ints([1, 2]), c.ints([3, 3])),
    "copy from a page that is a destination": lambda c, p: p.copy(c.ints([1, 3]), c.ints([3, 4])),
    "copy to a page that is none": lambda c, p: p.copy(c.ints([1]), c.ints([30])),
    "copy from a page that is none": lambda c, p: p.copy(c.ints([-1]), c.ints([3])),
    "fork of a row that is none": lambda c, p: p.fork(c.ints([6]), c.ints([3])),
    "fork into a row that is none": lambda c, p: p.fork(c.ints([0]), c.ints([-1])),
    "fork into a row in use": lambda c, p: p.fork(c.ints([0]), c.ints([1])),
    "fork into the same row twice": lambda c, p: p.fork(c.ints([0, 1]), c.ints([3, 3])),
    "fork of a table with a page that is none": lambda c, p: (c.tables[0, 1:2].fill_(77), p.fork(c.ints([0]), c.ints([3]))),
    "fork of a table with a free page": lambda c, p: (c.refs[c.h_tables[0][0]].fill_(0), p.fork(c.ints([0]), c.ints([3]))),
    "fork of a length past the table": lambda c, p: (c.lens[0].fill_(21), p.fork(c.ints([0]), c.ints([3]))),
    "free of a row that is none": lambda c, p: p.free(c.ints([1, 6])),
    "free of the same row twice": lambda c, p: p.free(c.ints([1, 1])),
    "free of a negative length": lambda c, p: (c.lens[1].fill_(-1), p.free(c.ints([1]))),
    "free of a table with a page that is none": lambda c, p: (c.tables[1, 0:1].fill_(-1), p.free(c.ints([1]))),
}


@pytest.mark.parametrize("what", list(REFUSED))
def test_a_refused_call_changes_nothing(torch, serving, hbf, what):
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    c.fill(0, 10); c.fill(1, 17)
    c.upload()
    plan = c.plan(serving)
    before = None

    class Watch:                                             # the state as the call itself finds it
        def __getattr__(self, name):
            def call(*a):
                nonlocal before
                before = [t.clone() for t in (c.data, c.refs, c.lens, c.tables)]
                getattr(plan, name)(*a)
            return call
    REFUSED[what](c, Watch())
    with pytest.raises(hbf.HbfError) as e:
        plan.result()
    assert e.value.code == hbf.E_INVAL
    assert all(torch.equal(a, b) for a, b in zip(before, (c.data, c.refs, c.lens, c.tables)))


def test_a_fork_without_room_changes_nothing(torch, serving, hbf):
    c = Cache(torch, 2, 8, 8, 4, 6, 5)
    c.fill(0, 18)                                            # five pages of eight
    c.upload()
    plan = c.plan(serving)
    plan.fork(c.ints([0] * 4), c.ints([1, 2, 3, 4]))
    with pytest.raises(hbf.HbfError) as e:
        plan.result()
    assert e.value.code == hbf.E_CAPACITY
    c.check()
    c.expect_fork([0] * 3, [1, 2, 3])
    plan.fork(c.ints([0] * 3), c.ints([1, 2, 3]))
    assert plan.result()["moved"] == 3
    c.check()


def test_captured_and_replayed(torch, serving):
    c = Cache(torch, 4, 60, 64, 4, 8, 6)
    c.fill(0, 22); c.fill(1, 9)
    c.upload()
    st = torch.cuda.Stream()
    plan = c.plan(serving, stream=st)
    parents, children, gone = c.ints([0, 1, 0]), c.ints([4, 5, 6]), c.ints([0, 4])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        plan.fork(parents, children)
        plan.free(gone)
        plan.compact()
    c.check()                                                # nothing has run yet
    for turn in range(2):
        with torch.cuda.stream(st):
            graph.replay()
        c.expect_fork([0, 1, 0], [4, 5, 6]); c.expect_free([0, 4]); moved, n = c.expect_compact()
        assert plan.result() == {"moved": moved, "in_use": n}
        c.check()
        for r in (5, 6):                                     # the rows that the next replay forks into, and from
            c.expect_free([r])
        c.fill(0, 22); c.upload(); c.h_data.copy_(c.data)
        torch.cuda.synchronize()


@pytest.mark.parametrize("pages", [392_100, 393_216, 1 << 20])
def test_caches_of_many_pages(torch, serving, pages):
    """Marks of all pages in shared memory, at its sizes' border and at the most pages that there may be."""
    data = torch.zeros(1, pages, 4, dtype=torch.int32, device="cuda")
    data[0, :, 0] = torch.arange(pages, device="cuda")
    refs, lens = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.tensor([2, 0], dtype=torch.int32, device="cuda")
    held = torch.tensor([pages - 1, 7], device="cuda", dtype=torch.int32)
    refs[held.long()] = 1
    tables = torch.stack([held, torch.full_like(held, -1)])
    plan = serving.CachePages(data, refs, tables, lens, 1)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    plan.copy(ints(5), ints(pages - 2))
    assert plan.result()["moved"] == 1 and int(data[0, pages - 2, 0]) == 5
    plan.fork(ints(0), ints(1))
    plan.result()
    plan.compact()
    assert plan.result() == {"moved": 2, "in_use": 2}
    assert tables.tolist() == [[1, 0], [1, 0]] and data[0, :2, 0].tolist() == [7, pages - 1] and refs[:3].tolist() == [2, 2, 0]


def test_records_before_any_call(torch, serving):
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    plan = c.plan(serving)
    assert plan.accesses().shape[0] == 0
    plan._ws.random_(0, 256)                                 # whatever lies in a workspace
    plan._ws[:4] = 0
    plan._moves = 40
    rec = plan.accesses()
    assert rec.shape[0] == 160


def test_offsets_past_32_bits(torch, serving):
    pages, words = 5000, 4096 * 64                           # 5.2 GB
    data = torch.zeros(1, pages, words, dtype=torch.int32, device="cuda")
    data[0, -1] = torch.arange(words, device="cuda"); data[0, 3] = 7
    refs, lens = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.tensor([1, 1], dtype=torch.int32, device="cuda")
    refs[-1] = 1; refs[3] = 1
    tables = torch.tensor([[pages - 1], [3]], dtype=torch.int32, device="cuda")
    plan = serving.CachePages(data, refs, tables, lens, 16)
    plan.compact()
    assert plan.result() == {"moved": 2, "in_use": 2}
    assert tables.tolist() == [[1], [0]] and (data[0, 0] == 7).all() and torch.equal(data[0, 1], torch.arange(words, device="cuda", dtype=torch.int32))


def test_records(torch, serving):
    c = Cache(torch, 3, 40, 16, 4, 9, 5)
    c.fill(0, 10); c.fill(1, 8); c.fill(2, 3)
    c.upload()
    plan = c.plan(serving)
    parents, children = [0, 1, 2], [5, 4, 3]
    src = [c.h_tables[0][2], c.h_tables[2][0]]
    c.expect_fork(parents, children)
    dst = [c.h_tables[5][2], c.h_tables[3][0]]
    plan.fork(c.ints(parents), c.ints(children))
    rec = plan.accesses(9, 2).cpu().tolist()
    addr = lambda s, p: c.data.data_ptr() + (s * 40 + p) * 64
    want = [r for a, b in zip(src, dst) for s in range(3) for r in ([addr(s, a), 64], [addr(s, b), 64 + (1 << 32)])]
    want += [[0, 1]] * (2 * 3 * 3 - len(want))
    assert [[a, b] for a, _, b in rec] == want and [i for _, i, _ in rec] == [9 + 2 * k for k in range(18)]


def test_binding_refuses(torch, serving, hbf):
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    plan = c.plan(serving)
    with pytest.raises(ValueError):
        plan.copy(c.ints([1, 2]), c.ints([3]))
    with pytest.raises(ValueError):
        plan.free(c.ints([1]).long())
    with pytest.raises(ValueError):
        serving.CachePages(c.data, c.refs[:-1], c.tables, c.lens, 4)
    with pytest.raises(ValueError):
        serving.CachePages(c.data[:, :, ::2], c.refs, c.tables, c.lens, 4)
    with pytest.raises(hbf.HbfError):
        serving.CachePages(c.data[:, :, :6].contiguous(), c.refs, c.tables, c.lens, 4)      # pages of 24 bytes
    with pytest.raises(hbf.HbfError):
        plan.free(c.ints([0] * 7))                           # more than there are rows


def test_a_call_refused_at_once_leaves_the_records_of_the_one_before(torch, serving, hbf):
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    c.fill(0, 10)
    c.upload()
    plan = c.plan(serving)
    plan.copy(c.ints([1, 2, 3]), c.ints([11, 12, 13]))
    n, want = plan.access_count(), plan.accesses(7, 2).tolist()
    assert n == 2 * 3 * 2
    with pytest.raises(hbf.HbfError):
        plan.free(c.ints([0] * 7))                           # more than there are rows
    assert plan.access_count() == n and plan.accesses(7, 2).tolist() == want and plan.result()["moved"] == 3
    with pytest.raises(hbf.HbfError):
        plan.copy(c.ints([1] * 31), c.ints([2] * 31))        # more than there are pages
    assert plan.access_count() == n and plan.accesses(7, 2).tolist() == want
