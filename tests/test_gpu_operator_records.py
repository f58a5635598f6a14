"""Room that a caller gives for an operator's records: exactly as many, dense, or refused."""
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


def attention(torch, serving):
    k, v = (torch.randn(9, 16, 2, 64, device="cuda").bfloat16() for _ in range(2))
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    op = serving.PrefixAttention(k, v, 2, 4, ints(1, 2, 3), 40, ints(4, 5, 6, 7).view(2, 2), ints(20, 3), 20)
    op(torch.randn(2, 4, 64, device="cuda").bfloat16())
    return op, 2 * (3 + 4)


def moe(torch, serving):
    op = serving.MoeLayer(torch.randn(8, 3 * 64 * 32, device="cuda").bfloat16(), 64, 32, 2, 5, tile_bytes=5000)
    op(torch.randn(3, 64, device="cuda").bfloat16(), torch.randn(3, 8, device="cuda"))
    return op, 6 * 3


def pages(torch, serving):
    zeros = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    op = serving.CachePages(zeros(3, 20, 8), zeros(20), zeros(2, 4), zeros(2), 4)
    op.copy(torch.arange(5, dtype=torch.int32, device="cuda"), torch.arange(10, 15, dtype=torch.int32, device="cuda"))
    return op, 2 * 5 * 3


@pytest.mark.parametrize("make", [attention, moe, pages], ids=["attention", "moe", "pages"])
def test_room_for_records(torch, serving, make):
    op, n = make(torch, serving)
    want = op.accesses(100, 3)
    assert want.shape == (n, 3) and op.access_count() == n
    new = lambda *s, **kw: torch.full(s, -5, **{"dtype": torch.int64, "device": "cuda", **kw})
    out = new(n, 3)
    assert op.accesses(100, 3, out) is out and torch.equal(out, want)
    for bad in (new(n - 1, 3), new(n + 1, 3), new(3 * n), new(n, 4)[:, :3], new(2 * n, 3)[::2], new(3, n).t(), new(n, 3, dtype=torch.int32), new(n, 3, dtype=torch.float64),
                new(n, 3, device="cpu"), new(0, 3)):
        kept = bad.clone()
        with pytest.raises(ValueError):
            op.accesses(100, 3, bad)
        torch.cuda.synchronize()
        assert torch.equal(bad, kept)


def test_no_records_want_no_room(torch, serving):
    op = serving.MoeLayer(torch.randn(8, 3 * 64 * 32, device="cuda").bfloat16(), 64, 32, 2, 5)
    assert op.accesses().shape == (0, 3)
    with pytest.raises(ValueError):
        op.accesses(0, 0, torch.zeros(1, 3, dtype=torch.int64, device="cuda"))


def test_records_of_the_pages_that_a_compaction_moved(torch, serving):
    from paper_2609_09800_b200 import hbf, workloads as wl
    slabs, pages = 4, 10_000
    data = torch.zeros(slabs, pages, 8, dtype=torch.int32, device="cuda")
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    refs, lens, tables = torch.zeros(pages, dtype=torch.int32, device="cuda"), ints(6, 4), ints([0, 9_000], [5_000, -1])
    refs[[0, 5_000, 9_000]] = 1
    op = serving.CachePages(data, refs, tables, lens, 4)
    op.compact()
    moved = op.result()["moved"]
    assert moved == 2 and op.access_count() == pages * slabs and op.access_count(moved) == 2 * 2 * slabs
    some, every = op.accesses(100, 3, moved=moved), op.accesses(100, 3)
    assert torch.equal(some, every[:16]) and (some[:, 0] != 0).all() and not every[16:, 0].any()
    for wrong in (-1, pages // 2 + 1):
        with pytest.raises(ValueError):
            op.accesses(moved=wrong)
    with pytest.raises(ValueError):
        op.accesses(0, 0, torch.empty_like(every), moved=moved)
    ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["tiny"]))
    ctx.register_range(data.data_ptr(), data.numel() * 4, 3)
    acc, comp, stall, stats = ctx.serve(op, 100, 3, moved=moved)
    res = ctx.last_result()
    assert torch.equal(acc, some) and res["code"] == 0 and res["n_modeled"] == 16 and res["n_native"] == 0
    op.compact()                                             # nothing is left to move: no records, and nothing to serve
    assert op.result()["moved"] == 0
    acc, comp, _, _ = ctx.serve(op, 100, 3, moved=0)
    assert acc.shape == (0, 3) and comp.numel() == 0
