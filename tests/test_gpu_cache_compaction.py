"""Compaction of a cache whose rows are not sound: refused like the other calls on its pages, with nothing changed."""
import pytest

from test_gpu_cache_pages import Cache, hbf, serving, torch  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

BAD = {
    "a negative length": lambda c: c.lens[1].fill_(-1),
    "a length past the table": lambda c: c.lens[1].fill_(21),
    "a page that is none": lambda c: c.tables[1, 0:1].fill_(-1),
    "a page past the last": lambda c: c.tables[1, 4:5].fill_(c.refs.numel()),
    "a free page": lambda c: c.refs[c.h_tables[1][2]].fill_(0),
    "a row past the first thousand": lambda c: c.lens[-1].fill_(-1),
}


@pytest.mark.parametrize("words", [8, 40_000], ids=["one block", "two kernels"])
@pytest.mark.parametrize("what", list(BAD))
def test_refused_and_nothing_changed(torch, serving, hbf, what, words):  # noqa: F811
    c = Cache(torch, 2, 30, words, 4, 1500, 5)
    c.fill(0, 10); c.fill(1, 17); c.fill(2, 20)
    c.upload()
    BAD[what](c)
    plan = c.plan(serving)
    before = [t.clone() for t in (c.data, c.refs, c.lens, c.tables)]
    plan.compact()
    with pytest.raises(hbf.HbfError) as e:
        plan.result()
    assert e.value.code == hbf.E_INVAL
    assert all(torch.equal(a, b) for a, b in zip(before, (c.data, c.refs, c.lens, c.tables)))


def test_what_does_not_count_may_be_anything(torch, serving):  # noqa: F811
    """Entries behind a row's length, and rows without tokens, are not looked at."""
    c = Cache(torch, 2, 30, 8, 4, 6, 5)
    c.fill(0, 10); c.fill(1, 17)
    c.upload()
    c.tables[0, 3:] = 77; c.h_tables[0][3:] = [77, 77]
    c.tables[4] = -9; c.h_tables[4] = [-9] * 5
    plan = c.plan(serving)
    moved, n = c.expect_compact()
    plan.compact()
    assert plan.result() == {"moved": moved, "in_use": n}
    c.check()
