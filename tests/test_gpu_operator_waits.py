"""Waits of the tensor-memory kernels that run out: what depends on them is NaN, the call ends, and the next one is right.  Nothing stalls: the limit of
polls is lowered, to none or to so few that a wait may be given up anywhere."""
import pytest

from test_gpu_attention import Case as Attention
from test_gpu_moe import Case as Moe

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


@pytest.fixture
def polls(torch):
    from paper_2609_09800_b200 import hbf
    yield hbf.lib().hbf_debug_operator_waits
    torch.cuda.synchronize()
    hbf.lib().hbf_debug_operator_waits(-1)


# pages that tensor copies fetch, with a tile that the prefix ends in and without; pages that they cannot; one tile of rows; a single piece
WIDE = [(128, 32, 4, 128, 16, 640, 12), (128, 32, 4, 64, 16, 1000, 0), (101, 32, 4, 128, 12, 640, 9), (67, 32, 1, 128, 16, 3000, 0), (1216, 64, 8, 64, 16, 300, 0)]
IDS = ["x".join(map(str, s)) for s in WIDE]


@pytest.mark.parametrize("shape", WIDE, ids=IDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_attention_gives_up_at_once(torch, serving, polls, shape, dtype):
    c = Attention(torch, *shape, dtype=dtype, seed=sum(shape), poison=False)
    plan = c.plan(serving)
    lse = torch.empty(c.B, c.Hq, device="cuda")
    good = plan(c.q).clone()
    polls(0)
    out = plan(c.q, lse=lse)
    torch.cuda.synchronize()
    assert torch.isnan(out).all() and torch.isnan(lse).all()
    polls(-1)
    assert torch.equal(plan(c.q), good)


@pytest.mark.parametrize("tokens", [9, 64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_experts_give_up_at_once(torch, serving, polls, tokens, dtype):
    c = Moe(torch, tokens, 1000, 520, 12, 3, dtype=dtype, seed=tokens)
    plan = c.plan(serving)
    good = [t.clone() for t in c.run(serving, plan)]
    polls(0)
    out, chosen, weights = c.run(serving, plan)
    torch.cuda.synchronize()
    assert torch.isnan(out).all() and torch.equal(chosen, good[1]) and torch.equal(weights, good[2])
    polls(-1)
    assert all(torch.equal(a, b) for a, b in zip(c.run(serving, plan), good))


@pytest.mark.parametrize("limit", [1, 2, 3])
@pytest.mark.parametrize("shape", WIDE[:4], ids=IDS[:4])
def test_attention_gives_up_anywhere(torch, serving, polls, shape, limit):
    """A row is right to the bit or NaN throughout."""
    c = Attention(torch, *shape, seed=sum(shape), poison=False)
    plan = c.plan(serving)
    good = plan(c.q).clone()
    for _ in range(10):
        polls(limit)
        out = plan(c.q)
        torch.cuda.synchronize()
        gone = torch.isnan(out).all(-1)
        assert torch.equal(out[~gone], good[~gone])
        polls(-1)
        assert torch.equal(plan(c.q), good)


@pytest.mark.parametrize("limit", [1, 2, 3])
@pytest.mark.parametrize("tokens", [9, 64])
def test_experts_give_up_anywhere(torch, serving, polls, tokens, limit):
    """A number is right to the bit or NaN."""
    c = Moe(torch, tokens, 2048, 768, 64, 4, seed=tokens)
    plan = c.plan(serving)
    good = plan(c.x, c.scores).clone()
    for _ in range(10):
        polls(limit)
        out = plan(c.x, c.scores)
        torch.cuda.synchronize()
        gone = torch.isnan(out)
        assert torch.equal(out[~gone], good[~gone])
        polls(-1)
        assert torch.equal(plan(c.x, c.scores), good)


def test_kernels_without_such_waits_know_no_limit(torch, serving, polls):
    c, m = Attention(torch, 3, 8, 2, 128, 16, 500, 40), Moe(torch, 8, 256, 64, 12, 3)
    polls(0)
    c.check(c.plan(serving)(c.q))
    m.check(m.run(serving))
