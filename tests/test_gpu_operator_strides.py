"""Dimensions of size one have no stride to speak of: whatever it says, the call is that of a dense tensor."""
import pytest

from test_gpu_attention import Case as Attention, serving, torch  # noqa: F401  (fixtures)
from test_gpu_moe import Case as Moe

pytestmark = pytest.mark.gpu


def odd(t, *strides):
    """The same values under other strides for the dimensions of size one."""
    assert all(s is None or n == 1 for n, s in zip(t.shape, strides))
    out = t.as_strided(t.shape, [o if s is None else s for s, o in zip(strides, t.stride())])
    return out


@pytest.mark.parametrize("shape", [(1, 8, 2, 128, 16, 100, 30), (1, 1, 1, 64, 16, 100, 30), (5, 1, 1, 128, 1, 40, 20), (130, 32, 1, 64, 16, 6000, 0), (3, 4, 4, 64, 16, 0, 16)],
                         ids=lambda s: "x".join(map(str, s)))
def test_attention(torch, serving, shape):  # noqa: F811
    c = Attention(torch, *shape, seed=sum(shape), poison=False)
    want = c.plan(serving)(c.q)
    B, H, d = c.q.shape
    one = lambda n, s: s if n == 1 else None
    c.k, c.v = (odd(t, one(t.shape[0], 3), one(t.shape[1], 5 + i), one(t.shape[2], 7 * i + 1), None) for i, t in enumerate((c.k, c.v)))
    q, out = odd(c.q, one(B, 1027), one(H, 3), None), odd(torch.zeros_like(c.q), one(B, 11), one(H, 9), None)
    c.pp, c.op = odd(c.pp, one(c.pp.numel(), 4)), odd(c.op, None, one(c.op.shape[1], 6))
    c.lens = odd(c.lens, one(B, 2))
    plan = c.plan(serving)
    assert plan(q, out) is out and torch.equal(out, want)
    assert plan.accesses().shape[0] == plan.access_count()


def test_moe_of_one_expert(torch, serving):  # noqa: F811
    c = Moe(torch, 20, 64, 32, 1, 1)
    want = [t.clone() for t in c.run(serving)]
    c.scores = odd(c.scores, None, 20)
    assert all(torch.equal(a, b) for a, b in zip(c.run(serving), want))
    c = Moe(torch, 1, 64, 32, 4, 2)
    want = [t.clone() for t in c.run(serving)]
    c.x, c.scores = odd(c.x, 3, None), odd(c.scores, 1, None)
    assert all(torch.equal(a, b) for a, b in zip(c.run(serving), want))


def test_pages_of_one(torch, serving):  # noqa: F811
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    data = torch.randint(0, 100, (1, 6, 8), dtype=torch.int32, device="cuda")
    lens, refs, tables = ints(3), ints(0, 0, 0, 0, 1, 0), ints(4).view(1, 1)
    before = data.clone()
    plan = serving.CachePages(odd(data, 5, None, None), refs, odd(tables, 7, 9), odd(lens, 3), 4)
    plan.compact()
    assert plan.result() == {"moved": 1, "in_use": 1} and tables.tolist() == [[0]] and torch.equal(data[0, 0], before[0, 4])


def test_what_is_not_there(torch, serving):  # noqa: F811
    c = Attention(torch, 2, 8, 2, 64, 16, 40, 20, poison=False)
    for args in ((None, 40, c.op, c.lens, 20), (c.pp, 40, None, c.lens, 20), (c.pp, 40, c.op, None, 20)):
        with pytest.raises(ValueError):
            serving.PrefixAttention(c.k, c.v, 2, 8, *args)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")
    for shape in ((0, 4, 8), (2, 0, 8), (2, 4, 0)):
        with pytest.raises(ValueError):
            serving.CachePages(ints(*shape), ints(shape[1]), ints(2, 3), ints(2), 4)
