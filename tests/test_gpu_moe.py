"""A mixture-of-experts layer for a few tokens against a plain implementation in 64 bits.

Tolerance, from the arithmetic (eps the type's spacing at 1).  Gate and up sums of D products in 32 bits: off by at most g = (D + 16) 2^-23 of
the sums of the magnitudes, Ga and Ua.  h = w silu(gate) up: |silu'| <= 1.1, so off by w (1.1 g Ga |up| + |silu| g Ua), and 2^-19 |h| for exp, the
division and the weight, and, held as two numbers of the type, (eps / 2)^2 |h| plus the type's smallest step.  The down product adds (I + K + 16) 2^-23 of the
sum of its magnitudes; the output is rounded once, eps / 2."""
import math

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


class Case:
    def __init__(self, torch, T, D, I, E, K, dtype="bf16", seed=0, pad=0, renorm=True):
        g = torch.Generator(device="cuda"); g.manual_seed(seed)
        self.torch, self.dt = torch, {"bf16": torch.bfloat16, "fp16": torch.float16}[dtype]
        self.T, self.D, self.I, self.E, self.K, self.renorm = T, D, I, E, K, renorm
        w = torch.randn(E, 3 * I * D + pad, device="cuda", generator=g)
        w[:, :2 * I * D] *= D ** -0.5; w[:, 2 * I * D:] *= I ** -0.5
        self.w = w.to(self.dt)
        self.x = torch.randn(T, D, device="cuda", generator=g).to(self.dt)
        self.scores = torch.randn(T, E, device="cuda", generator=g)

    def plan(self, serving, **kw):
        return serving.MoeLayer(self.w, self.D, self.I, self.K, kw.pop("max_tokens", self.T), renormalise=self.renorm, **kw)

    def expect(self):
        torch, D, I = self.torch, self.D, self.I
        rows = self.scores.tolist()
        chosen = torch.full((self.T, self.K), -1, dtype=torch.int64)
        weights = torch.zeros(self.T, self.K, dtype=torch.float64)
        for t, row in enumerate(rows):
            if any(math.isnan(s) for s in row):
                continue
            order = [e for e in sorted(range(self.E), key=lambda e: (-row[e], e)) if row[e] != -math.inf]
            pick = order[:self.K]
            total = sum(math.exp(row[e] - row[order[0]]) for e in (pick if self.renorm else order)) if pick else 1.0
            for j, e in enumerate(pick):
                chosen[t, j], weights[t, j] = e, math.exp(row[e] - row[order[0]]) / total
        out = torch.zeros(self.T, D, dtype=torch.float64, device="cuda")
        err = torch.zeros_like(out)
        half, g = torch.finfo(self.dt).eps / 2, (D + 16) * 2.0 ** -23
        for e in sorted(set(chosen.flatten().tolist()) - {-1}):
            t, j = torch.nonzero(chosen == e, as_tuple=True)
            w = weights[t, j].cuda()[:, None]
            G, U, W = self.w[e, :I * D].double().view(I, D), self.w[e, I * D:2 * I * D].double().view(I, D), self.w[e, 2 * I * D:3 * I * D].double().view(D, I)
            x = self.x[t.cuda()].double()
            gate, up = x @ G.t(), x @ U.t()
            ga, ua = x.abs() @ G.abs().t(), x.abs() @ U.abs().t()
            silu = gate * torch.sigmoid(gate)
            h = w * silu * up
            dh = w * (1.1 * g * ga * up.abs() + silu.abs() * g * ua) + h.abs() * (2.0 ** -19 + half * half) + torch.finfo(self.dt).smallest_normal * torch.finfo(self.dt).eps
            out[t.cuda()] += h @ W.t()
            err[t.cuda()] += dh @ W.abs().t() + (I + self.K + 16) * 2.0 ** -23 * (h.abs() @ W.abs().t())
        return out, half * out.abs() + (1 + half) * err + torch.finfo(self.dt).tiny, chosen, weights

    def run(self, serving, plan=None):
        torch = self.torch
        plan = plan or self.plan(serving)
        chosen = torch.full((self.T, self.K), 99, dtype=torch.int32, device="cuda")
        weights = torch.full((self.T, self.K), 99.0, device="cuda")
        return plan(self.x, self.scores, None, chosen, weights), chosen, weights

    def check(self, got, rows=slice(None)):
        torch = self.torch
        out, chosen, weights = got
        want, tol, c, w = self.expect()
        assert torch.equal(chosen.cpu().long(), c)
        assert torch.allclose(weights.cpu().double(), w, rtol=2.0 ** -20, atol=1e-37)
        err = ((out.double() - want).abs() / tol)[rows]
        assert torch.isfinite(out[rows]).all() and (err <= 1).all(), "off by %g of the tolerance" % float(err.max())


SHAPES = [
    # T, D, I, E, K
    (1, 8, 8, 1, 1), (1, 2048, 768, 16, 8), (2, 64, 32, 2, 2), (3, 1000, 520, 12, 3), (5, 72, 200, 40, 16), (8, 512, 1024, 8, 2), (9, 256, 128, 3, 1),
    (17, 4096, 64, 9, 4), (33, 128, 40, 2, 2), (40, 136, 264, 4, 4), (64, 2048, 768, 16, 8), (65, 264, 72, 512, 16), (100, 512, 24, 5, 1), (128, 384, 96, 3, 3),
    (128, 2400, 64, 6, 2), (7, 8, 2048, 33, 5), (128, 64, 64, 1, 1), (8, 2048, 1024, 24, 8), (3, 4096, 2048, 6, 2), (16, 20000, 16, 3, 2),
]


@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_against_64_bits(torch, serving, shape, dtype):
    c = Case(torch, *shape, dtype=dtype, seed=sum(shape))
    c.check(c.run(serving))


def test_softmax_over_all(torch, serving):
    c = Case(torch, 6, 128, 64, 70, 4, renorm=False)
    c.check(c.run(serving))


def test_ties_go_to_the_lowest_expert(torch, serving):
    c = Case(torch, 12, 64, 32, 100, 8)
    c.scores.copy_(torch.randint(0, 3, c.scores.shape, device="cuda").float() - 1.0)
    c.scores[0] = 0.0; c.scores[1] = -0.0
    c.scores[2, ::2] = -0.0; c.scores[2, 1::2] = 0.0
    got = c.run(serving)
    for t in (0, 1):
        assert got[1][t].tolist() == list(range(8))
    c.check(got)


def test_masked_scores_and_rows_without_experts(torch, serving):
    c = Case(torch, 6, 64, 32, 40, 4)
    c.scores[0] = -math.inf                                  # nothing is left
    c.scores[1, :37] = -math.inf                             # fewer than top_k are
    c.scores[2] = torch.finfo(torch.float32).min             # the type's lowest value is a score like any other
    c.scores[3, 5] = torch.finfo(torch.float32).max
    c.scores[4] *= 1e30
    got = c.run(serving)
    c.check(got)
    assert not got[0][0].any() and (got[1][0] == -1).all() and got[1][1].tolist()[3] == -1


def test_nan_scores_have_no_choice_and_infinity_no_weights(torch, serving):
    c = Case(torch, 10, 64, 32, 40, 4)
    c.scores[3, 7] = math.nan
    c.scores[9, 39] = math.nan
    got = c.run(serving)
    c.check(got, rows=[0, 1, 2, 4, 5, 6, 7, 8])
    assert torch.isnan(got[0][[3, 9]]).all() and (got[1][[3, 9]] == -1).all()
    c.scores[5, 1] = math.inf
    out, chosen, weights = c.run(serving)
    assert chosen[5, 0] == 1 and torch.isnan(out[5]).all() and torch.isfinite(out[4]).all()


def test_one_token_s_values_stay_with_it(torch, serving):
    """Infinities in a token, or in an expert that others did not choose, reach no one else."""
    c = Case(torch, 20, 256, 64, 4, 1)
    c.scores.fill_(-1.0); c.scores[:, 0] = 1.0; c.scores[5, 1] = 2.0; c.scores[6, 2] = 2.0
    clean = c.run(serving)[0].clone()
    c.x[2, 100] = math.inf
    c.w[1] = math.inf
    c.w[2, 2 * 256 * 64 + 5] = math.nan
    c.w[3] = math.nan                                        # chosen by nobody
    out = c.run(serving)[0]
    keep = [t for t in range(20) if t not in (2, 5, 6)]
    assert torch.equal(out[keep], clean[keep])
    assert not torch.isfinite(out[2]).any() and not torch.isfinite(out[5]).any() and torch.isnan(out[6, 0])


def test_strides_of_rows_and_experts(torch, serving):
    from paper_2609_09800_b200 import hbf
    c = Case(torch, 11, 128, 64, 6, 2, pad=64)
    sc = torch.randn(11, 20, device="cuda")
    sc[:, :6] = c.scores
    plan = c.plan(serving, max_tokens=128)
    wide = torch.full((11, 300), 5.0, device="cuda", dtype=c.dt)
    with pytest.raises(hbf.HbfError):                        # rows of 300: not all on 16-byte boundaries
        plan(wide[:, 8:136], sc[:, :6], wide[:, 140:268])
    wide = torch.full((11, 304), 5.0, device="cuda", dtype=c.dt)
    x, out = wide[:, 8:136], wide[:, 140:268]
    x.copy_(c.x)
    plan(x, sc[:, :6], out)
    want, tol, _, _ = c.expect()
    assert ((out.double() - want).abs() <= tol).all() and (wide[:, :8] == 5.0).all() and (wide[:, 268:] == 5.0).all() and (wide[:, 136:140] == 5.0).all()


def test_in_place(torch, serving):
    """The output may lie on the tokens: they are read before the output is written."""
    c = Case(torch, 9, 512, 64, 6, 2)
    x = c.x.clone()
    c.plan(serving)(x, c.scores, x)
    want, tol, _, _ = c.expect()
    assert ((x.double() - want).abs() <= tol).all()


def test_any_number_of_tokens_up_to_the_most(torch, serving):
    big = Case(torch, 128, 128, 64, 10, 3)
    plan = big.plan(serving)
    for n in (0, 1, 2, 8, 9, 31, 64, 127, 128):
        c = Case(torch, 128, 128, 64, 10, 3)
        c.T, c.x, c.scores = n, big.x[:n], big.scores[:n]
        got = c.run(serving, plan)
        if n:
            c.check(got)


def test_a_large_image_of_experts(torch, serving):
    """Experts at offsets past 2^32 bytes; the last one is chosen."""
    D, I, E = 2048, 1024, 400
    w = torch.zeros(E, 3 * D * I, device="cuda", dtype=torch.bfloat16)
    c = Case(torch, 3, D, I, 2, 2)
    w[[E - 2, E - 1]] = c.w
    want = c.run(serving)[0]
    scores = torch.full((3, E), -50.0, device="cuda")
    scores[:, E - 2:] = c.scores
    got = serving.MoeLayer(w, D, I, 2, 3)(c.x, scores)
    assert torch.equal(got, want)


def test_captured_and_replayed(torch, serving):
    c = Case(torch, 20, 256, 64, 30, 4)
    st = torch.cuda.Stream()
    plan = c.plan(serving, stream=st)
    out = torch.empty_like(c.x); chosen = torch.empty(20, 4, dtype=torch.int32, device="cuda"); weights = torch.empty(20, 4, device="cuda")
    torch.cuda.synchronize()
    plan(c.x, c.scores, out, chosen, weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        plan(c.x, c.scores, out, chosen, weights)
    for turn in range(3):
        c.scores.copy_(torch.randn(20, 30, device="cuda")); c.x.mul_(-1.5); out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        c.check((out, chosen, weights))


def test_the_same_call_gives_the_same_bits_on_two_streams(torch, serving):
    cases = [Case(torch, 64, 1024, 256, 32, 4, seed=s) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    plans = [c.plan(serving, stream=s) for c, s in zip(cases, streams)]
    want = [c.plan(serving)(c.x, c.scores) for c in cases]
    outs = [torch.empty_like(c.x) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, p, o in zip(cases, plans, outs):
            p(c.x, c.scores, o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_binding_refuses(torch, serving):
    from paper_2609_09800_b200 import hbf
    c = Case(torch, 4, 64, 32, 8, 2)
    plan = c.plan(serving)
    with pytest.raises(ValueError):
        plan(torch.cat([c.x, c.x]), c.scores)                # more tokens than the plan was made for
    with pytest.raises(ValueError):
        plan(c.x.float(), c.scores)
    with pytest.raises(ValueError):
        plan(c.x, c.scores[:, :7])
    with pytest.raises(ValueError):
        plan(c.x, c.scores.double())
    with pytest.raises(ValueError):
        plan(c.x, c.scores, c.x.t())
    with pytest.raises(ValueError):
        plan(c.x, c.scores, None, torch.empty(4, 2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        serving.MoeLayer(c.w, 64, 40, 2, 4)
    with pytest.raises(hbf.HbfError):
        serving.MoeLayer(c.w, 64, 32, 9, 4)
    with pytest.raises(hbf.HbfError):
        serving.MoeLayer(c.w, 64, 32, 2, 129)
    with pytest.raises(hbf.HbfError):
        plan(torch.empty(4 * 64 + 8, dtype=c.dt, device="cuda")[4:][:256].view(4, 64), c.scores)


def test_records(torch, serving):
    c = Case(torch, 5, 64, 32, 40, 3)
    plan = c.plan(serving, tile_bytes=5000)
    _, chosen, _ = c.run(serving, plan)
    rec = plan.accesses(50, 3).cpu().tolist()
    used = sorted(set(chosen.flatten().tolist()))
    size, row = 6 * 64 * 32, c.w.stride(0) * 2
    want = [[c.w.data_ptr() + e * row + o, min(5000, size - o)] for e in used for o in range(0, size, 5000)]
    want += [[0, 1]] * (15 * 3 - len(want))
    assert [[a, b] for a, _, b in rec] == want and [i for _, i, _ in rec] == [50 + 3 * k for k in range(45)]


@pytest.mark.parametrize("T", [4, 20])
def test_a_refused_call_has_no_records(torch, serving, T):
    from paper_2609_09800_b200 import hbf
    c = Case(torch, T, 64, 32, 8, 2)
    plan = c.plan(serving, tile_bytes=4096)
    plan(c.x, c.scores)
    assert plan.accesses().shape[0] == plan.access_count() > 0
    with pytest.raises(hbf.HbfError):                        # not on a 16-byte boundary
        plan(torch.empty(T * 64 + 8, dtype=c.dt, device="cuda")[4:][:T * 64].view(T, 64), c.scores.clone())
    assert plan.access_count() == 0 and plan.accesses().shape[0] == 0
    plan(c.x[:1], c.scores[:1])
    assert plan.access_count() == 2 * 3
