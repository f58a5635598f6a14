"""Calls that the header allows at its limits and in combinations that the operators' own files leave out."""
import math

import pytest

from test_gpu_attention import Case as Attention, serving, torch  # noqa: F401  (fixtures)
from test_gpu_cache_pages import Cache
from test_gpu_moe import Case as Moe

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 64, 32, 129, 16), (8, 64, 32, 512, 16), (9, 64, 32, 300, 7), (40, 128, 64, 70, 4), (64, 72, 40, 512, 16), (128, 64, 24, 128, 16), (20, 64, 32, 5, 5)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("renorm", [True, False])
def test_experts(torch, serving, shape, renorm):  # noqa: F811
    c = Moe(torch, *shape, seed=sum(shape), renorm=renorm)
    c.check(c.run(serving))
    T, _, _, E, K = shape
    c.scores.copy_(torch.randint(0, 4, c.scores.shape, device="cuda").float())               # ties
    c.scores[0, :E // 2] = -math.inf
    c.scores[T // 2] = -math.inf
    c.scores[T // 2, E - 1] = -3.0
    got = c.run(serving)
    c.check(got)
    assert got[1][T // 2].tolist() == [E - 1] + [-1] * (K - 1)
    if T > 1:
        c.scores[T - 1, E // 3] = math.nan
        got = c.run(serving)
        c.check(got, rows=list(range(T - 1)))
        assert torch.isnan(got[0][T - 1]).all() and (got[1][T - 1] == -1).all()


@pytest.mark.parametrize("T, E, K", [(3, 300, 16), (64, 512, 16), (128, 100, 9)])
def test_experts_records(torch, serving, T, E, K):  # noqa: F811
    c = Moe(torch, T, 64, 32, E, K)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    plan = c.plan(serving, tile_bytes=7000, stream=st)
    with torch.cuda.stream(st):
        _, chosen, _ = c.run(serving, plan)
        rec = plan.accesses(5, 1).cpu().tolist()
    used, size, row = sorted(set(chosen.flatten().tolist())), 6 * 64 * 32, c.w.stride(0) * 2
    want = [[c.w.data_ptr() + e * row + o, min(7000, size - o)] for e in used for o in range(0, size, 7000)]
    want += [[0, 1]] * (min(E, T * K) * 2 - len(want))
    assert [[a, b] for a, _, b in rec] == want


@pytest.mark.parametrize("shape", [(300, 8, 2, 64, 16, 100, 40), (1, 128, 1, 128, 16, 300, 40), (700, 4, 4, 64, 7, 0, 30), (2, 24, 8, 64, 1000, 700, 1500), (500, 48, 16, 128, 8, 200, 20)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("layout", ["slots", "gaps"])
def test_attention(torch, serving, shape, layout):  # noqa: F811
    c = Attention(torch, *shape, seed=sum(shape), layout=layout)
    lse = torch.empty(c.B, c.Hq, device="cuda")
    c.check(c.plan(serving)(c.q, lse=lse), lse)


@pytest.mark.parametrize("page", [1, 16])
def test_more_rows_than_a_block_has_threads(torch, serving, page):  # noqa: F811
    rows, cols = 2600, 4
    c = Cache(torch, 2, 9000, 8, page, rows, cols)
    for r in range(0, 1300):
        n = (r * 7) % (cols * page + 1)
        for j in range(-(-n // page)):
            p = c.order[r * cols + j]
            c.h_refs[p], c.h_tables[r][j] = 1, p
        c.h_lens[r] = n
    c.upload()
    plan = c.plan(serving)
    parents, children = [(i * 3) % 1300 for i in range(1300)], list(range(2599, 1299, -1))
    moved = c.expect_fork(parents, children)
    plan.fork(c.ints(parents), c.ints(children))
    assert plan.result()["moved"] == moved
    c.check()
    gone = list(range(0, 2600, 2))
    c.expect_free(gone)
    plan.free(c.ints(gone))
    plan.result()
    c.check()
    moved, n = c.expect_compact()
    plan.compact()
    assert plan.result() == {"moved": moved, "in_use": n}
    c.check()
