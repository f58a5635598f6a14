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
