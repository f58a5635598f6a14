"""Shared-prefix attention against a plain implementation in 64 bits.

Tolerance, from the arithmetic.  With eps the type's spacing at 1: the output is rounded once, eps / 2 of its magnitude.  A weight p is
exp2 of a score in 32 bits: the score's sum of d products is off by at most (d + 8) * 2^-23 of the sum S of their magnitudes (times the
scale), which is the weight's relative error up to second order, and exp2, the running rescales and the sums add some 2^-18.  Weights enter the
second product as two numbers of the type, leaving 2 (eps / 2)^2 (the first is rounded down, so up to eps is left for the second), or, where a tile of 128 rows goes through
tensor memory, as one, leaving eps / 2.
All of these multiply A = sum p |v|, for the numerator and once more for the denominator."""
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


DT = {"bf16": "bfloat16", "fp16": "float16"}


class Case:
    def __init__(self, torch, B, Hq, Hk, d, page, prefix, own, dtype="bf16", seed=0, lens=None, layout="slots", poison=True, k_scale=1.0):
        g = torch.Generator(device="cuda"); g.manual_seed(seed)
        self.torch, self.dt = torch, getattr(torch, DT[dtype])
        self.B, self.Hq, self.Hk, self.d, self.page, self.prefix, self.own = B, Hq, Hk, d, page, prefix, own
        n_p, n_o = -(-prefix // page), -(-own // page)
        n = n_p + B * n_o + 2
        mk = lambda *s: torch.randn(*s, device="cuda", generator=g).to(self.dt)
        if layout == "slots":
            self.k, self.v = mk(n, page, Hk, d) * k_scale, mk(n, page, Hk, d)
        elif layout == "heads":
            self.k, self.v = ((mk(n, Hk, page, d) * s).transpose(1, 2) for s in (k_scale, 1.0))
        else:                                                # keys and values of a page side by side, with a gap behind
            both = mk(n, 2, page, Hk, d + 8)
            self.k, self.v = both[:, 0, :, :, :d], both[:, 1, :, :, :d]
        self.q = mk(B, Hq, d)
        order = torch.randperm(n, device="cuda", generator=g).to(torch.int32)
        self.pp, self.op = order[:n_p].contiguous(), order[n_p:n_p + B * n_o].reshape(B, n_o).contiguous()
        if lens is None:
            lens = torch.randint(0, own + 1, (B,), device="cuda", generator=g)
        self.lens = torch.as_tensor(lens, device="cuda", dtype=torch.int32)
        if poison:                                           # what lies behind a sequence's end counts for nothing, whatever it is
            with torch.no_grad():
                if prefix % page:
                    for t, bad in ((self.k, math.nan), (self.v, math.inf)):
                        t[self.pp[-1].long(), prefix % page:] = bad
                for b in range(B):
                    L = int(self.lens[b])
                    for j in range(n_o):
                        if (j + 1) * page > L:
                            for t, bad in ((self.k, math.inf), (self.v, math.nan)):
                                t[self.op[b, j].long(), max(0, L - j * page):] = bad

    def plan(self, serving, **kw):
        return serving.PrefixAttention(self.k, self.v, self.B, self.Hq, self.pp if self.prefix else None, self.prefix,
                                       self.op if self.own else None, self.lens if self.own else None, self.own, **kw)

    def expect(self, scale=None, q=None):
        """out, log-sum-exp, A and S * scale in 64 bits."""
        torch = self.torch
        scale = self.d ** -0.5 if scale is None else scale
        G = self.Hq // self.Hk
        q = self.q if q is None else q
        out = torch.zeros(self.B, self.Hq, self.d, dtype=torch.float64, device="cuda")
        A, S = torch.zeros_like(out), torch.zeros(self.B, self.Hq, dtype=torch.float64, device="cuda")
        lse = torch.full((self.B, self.Hq), -math.inf, dtype=torch.float64, device="cuda")
        take = lambda t, pages, n: t[pages.long()].flatten(0, 1)[:n].double() if n else t.new_zeros(0, self.Hk, self.d).double()
        pk, pv = take(self.k, self.pp, self.prefix), take(self.v, self.pp, self.prefix)
        for b in range(self.B):
            n = int(self.lens[b]) if self.own else 0
            k, v = (torch.cat([x, take(t, self.op[b], n)]) for x, t in ((pk, self.k), (pv, self.v)))
            if k.shape[0] == 0:
                continue
            qb = q[b].double().view(self.Hk, G, self.d)
            s = torch.einsum("hgd,lhd->hgl", qb, k) * scale
            p = torch.softmax(s, -1)
            out[b] = torch.einsum("hgl,lhd->hgd", p, v).reshape(self.Hq, self.d)
            A[b] = torch.einsum("hgl,lhd->hgd", p, v.abs()).reshape(self.Hq, self.d)
            S[b] = (torch.einsum("hgd,lhd->hgl", qb.abs(), k.abs()).amax(-1) * abs(scale)).reshape(self.Hq)
            lse[b] = torch.logsumexp(s, -1).reshape(self.Hq)
        return out, lse, A, S

    def check(self, out, lse=None, scale=None, q=None):
        torch = self.torch
        want, want_lse, A, S = self.expect(scale, q)
        half = torch.finfo(self.dt).eps / 2
        weight = half if self.B * (self.Hq // self.Hk) > 16 else 2 * half * half
        rel = weight + 2 * (self.d + 8) * 2.0 ** -23 * S + 2.0 ** -18
        tol = half * want.abs() + (1 + half) * A * rel[..., None] + torch.finfo(self.dt).tiny
        err = (out.double() - want).abs()
        assert torch.isfinite(out).all()
        assert (err <= tol).all(), "off by %g of the tolerance" % float((err / tol).max())
        if lse is not None:
            none = torch.isinf(want_lse)
            assert torch.equal(torch.isinf(lse) & (lse < 0), none)
            assert ((lse.double() - want_lse)[~none].abs() <= ((self.d + 8) * 2.0 ** -23 * S + 2.0 ** -18 + 2.0 ** -22 * want_lse.abs())[~none]).all()


SHAPES = [
    # B, Hq, Hk, d, page, prefix, own
    (1, 1, 1, 64, 1, 1, 0), (1, 1, 1, 128, 16, 0, 1), (1, 8, 1, 128, 16, 17, 3), (2, 8, 4, 64, 8, 0, 70), (3, 32, 4, 128, 16, 129, 65),
    (4, 16, 1, 128, 12, 1000, 100), (5, 35, 5, 64, 7, 333, 41), (2, 40, 2, 128, 32, 300, 50), (1, 64, 2, 64, 100, 512, 300), (9, 8, 8, 128, 64, 2049, 130),
    (2, 32, 4, 128, 16, 5000, 0), (1, 32, 4, 128, 3, 4097, 1300),
    # more rows than one tile: the prefix for many requests
    (16, 32, 4, 128, 16, 200, 40), (33, 8, 1, 64, 16, 1111, 20), (64, 32, 4, 128, 16, 1025, 90), (17, 10, 2, 64, 12, 777, 33), (40, 7, 7, 128, 16, 130, 9),
    (5, 14, 2, 128, 1, 64, 5), (128, 16, 2, 128, 64, 4000, 0), (70, 16, 1, 64, 100, 127, 0), (24, 8, 4, 128, 16, 128, 64), (100, 4, 4, 64, 8, 3, 2),
]


@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_against_64_bits(torch, serving, shape, dtype):
    c = Case(torch, *shape, dtype=dtype, seed=sum(shape))
    lse = torch.empty(c.B, c.Hq, device="cuda")
    c.check(c.plan(serving)(c.q, lse=lse), lse)


# enough rows and keys for the prefix to go through tensor memory: pages that copies fetch whole, pages that they cannot, one tile of rows in the
# last pair, the prefix's end in a tile and on its border, a single piece
WIDE = [(128, 32, 4, 128, 16, 512, 20), (128, 32, 4, 128, 64, 700, 0), (101, 32, 4, 128, 12, 640, 9), (128, 32, 4, 64, 8, 1000, 30), (128, 64, 4, 64, 1, 513, 3),
        (120, 40, 8, 64, 100, 640, 11), (128, 16, 1, 128, 24, 1500, 5), (16, 128, 8, 128, 256, 999, 33), (128, 128, 8, 64, 16, 385, 2), (67, 32, 1, 128, 16, 3000, 0)]


@pytest.mark.parametrize("shape", WIDE, ids=["x".join(map(str, s)) for s in WIDE])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_wide_against_64_bits(torch, serving, shape, dtype):
    c = Case(torch, *shape, dtype=dtype, seed=sum(shape))
    lse = torch.empty(c.B, c.Hq, device="cuda")
    c.check(c.plan(serving)(c.q, lse=lse), lse)


@pytest.mark.parametrize("d,page", [(64, 16), (128, 12)])
def test_wide_in_one_piece(torch, serving, d, page):
    """So many rows that every block has all keys of its rows and writes the output itself."""
    c = Case(torch, 1216, 64, 8, d, page, 300, 0, seed=9)
    lse = torch.empty(c.B, c.Hq, device="cuda")
    c.check(c.plan(serving)(c.q, lse=lse), lse)


def test_nobody(torch, serving):
    """A batch of no requests: nothing is read or written, by any of the calls."""
    from paper_2609_09800_b200 import hbf
    import ctypes as C
    c = Case(torch, 2, 8, 2, 64, 16, 40, 20, poison=False)
    a = c.plan(serving)._a
    a.batch = 0
    lib = hbf.lib()
    assert lib.hbf_attention_workspace_bytes(C.byref(a)) == 256
    assert lib.hbf_prefix_attention(C.byref(a), None, 0, None) == hbf.OK
    n = lib.hbf_attention_access_count(C.byref(a))
    assert n == 6
    rec = torch.empty(n, 3, dtype=torch.int64, device="cuda")
    assert lib.hbf_attention_accesses(C.byref(a), 0, 0, rec.data_ptr(), n, None) == hbf.OK
    assert (rec[:, 0] > 0).all()


@pytest.mark.parametrize("layout", ["heads", "gaps"])
@pytest.mark.parametrize("d", [64, 128])
def test_wide_page_layouts(torch, serving, layout, d):
    c = Case(torch, 128, 32, 4, d, 16, 900, 12, seed=5, layout=layout)
    x = c.q.clone()
    c.plan(serving)(x, x)                                    # in place, too
    c.check(x)


@pytest.mark.parametrize("d", [64, 128])
def test_wide_scales_and_rising_scores(torch, serving, d):
    c = Case(torch, 128, 16, 2, d, 16, 1601, 30, k_scale=4.0)
    for scale in (0.5, -0.25, 0.0):
        c.check(c.plan(serving, scale=scale)(c.q), scale=scale)
    c = Case(torch, 128, 16, 2, d, 16, 1600, 10, lens=[10] * 128)
    ramp = torch.linspace(0.01, 6.0, 1600, device="cuda").view(100, 16, 1, 1)
    c.k[c.pp.long()] = (c.q[0, 0].sign() * ramp).to(c.dt)
    c.check(c.plan(serving)(c.q))


@pytest.mark.parametrize("page", [16, 12])
def test_wide_nan_infinity_and_pages_that_are_none(torch, serving, page):
    mk = lambda: Case(torch, 128, 32, 4, 128, page, 640, 12, lens=[12] * 128, poison=False)
    c = mk()
    clean = c.plan(serving)(c.q)
    c.v[c.pp[2].long(), 3, 1, 5] = math.inf
    out = c.plan(serving)(c.q)
    assert torch.isinf(out[:, 8:16, 5]).all() and torch.equal(out[:, :8], clean[:, :8]) and torch.equal(out[:, 16:], clean[:, 16:])
    c = mk()
    c.k[c.pp[30].long(), 0, 2] = math.nan
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[:, 16:24]).all() and torch.equal(out[:, :16], clean[:, :16])
    c = mk()
    c.q[7, 9, 3] = math.inf
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[7, 9]).all() and torch.equal(out[8:], clean[8:])
    for bad in (-1, 1 << 30):
        c = mk()
        c.pp[20] = bad
        assert torch.isnan(c.plan(serving)(c.q)).all()
    c = mk()
    c.lens[3] = 13
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[3]).all() and torch.equal(out[4:], clean[4:])


def test_wide_captured_and_on_two_streams(torch, serving):
    cases = [Case(torch, 128, 16, 2, 128, 16, 1700, 64, seed=s, poison=False) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    plans = [c.plan(serving, stream=s) for c, s in zip(cases, streams)]
    outs = [torch.empty_like(c.q) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, p, o in zip(cases, plans, outs):
            p(c.q, o)
    torch.cuda.synchronize()
    for c, o in zip(cases, outs):
        c.check(o)
    c, plan, out, st = cases[0], plans[0], outs[0], streams[0]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        plan(c.q, out)
    for turn in range(2):
        c.lens.copy_(torch.randint(0, 65, c.lens.shape, device="cuda")); c.q.mul_(-1.0); out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        c.check(out)
        first = out.clone()
        plan(c.q, out)
        torch.cuda.synchronize()
        assert torch.equal(first, out)


@pytest.mark.parametrize("layout", ["heads", "gaps"])
@pytest.mark.parametrize("shape", [(3, 16, 4, 128, 16, 100, 30), (20, 16, 2, 64, 16, 300, 30), (30, 24, 4, 128, 8, 515, 12)])
def test_page_layouts_and_strided_rows(torch, serving, layout, shape):
    c = Case(torch, *shape, seed=5, layout=layout)
    B, H, d = c.q.shape
    wide = torch.full((B, H + 3, 2 * d), 7.0, device="cuda", dtype=c.dt)
    q, out = wide[:, :H, :d], wide[:, :H, d:]
    q.copy_(c.q)
    c.plan(serving)(q, out)
    c.check(out)
    assert (wide[:, H:] == 7.0).all() and torch.equal(q, c.q)


def test_out_may_be_q(torch, serving):
    for shape in [(3, 8, 2, 128, 16, 50, 20), (2, 8, 2, 64, 16, 0, 9), (40, 8, 2, 128, 16, 500, 20)]:
        c = Case(torch, *shape)
        x = c.q.clone()
        c.plan(serving)(x, x)
        c.check(x)


def test_rows_without_keys_are_zeros(torch, serving):
    c = Case(torch, 4, 8, 2, 128, 16, 0, 40, lens=[0, 40, 0, 1])
    lse = torch.empty(4, 8, device="cuda")
    out = c.plan(serving)(c.q, lse=lse)
    c.check(out, lse)
    assert not out[0].any() and not out[2].any()
    c = Case(torch, 2, 8, 2, 64, 16, 0, 0)
    out = torch.full_like(c.q, 3.0)
    c.plan(serving)(c.q, out)
    assert not out.any()


def test_lengths_and_tables_are_read_at_every_call(torch, serving):
    c = Case(torch, 3, 8, 2, 128, 16, 40, 64, lens=[0, 0, 0], poison=False)
    plan = c.plan(serving)
    for lens in ([64, 1, 0], [16, 17, 63], [0, 0, 0]):
        c.lens.copy_(torch.tensor(lens, device="cuda"))
        c.op.copy_(c.op.flip(0).clone())
        c.check(plan(c.q))


@pytest.mark.parametrize("B", [2, 40])
def test_large_scores_and_a_given_scale(torch, serving, B):
    """Weights from 1 down to nothing, signs of the scale, a scale of zero."""
    c = Case(torch, B, 16, 2, 64, 16, 400, 30, k_scale=4.0)
    for scale in (0.5, -0.25, 0.0):
        c.check(c.plan(serving, scale=scale)(c.q), scale=scale)


def test_a_rising_sequence_of_scores(torch, serving):
    """Every stage raises the maximum: keys grow along the sequence, in the prefix and behind it."""
    for B in (2, 40):
        c = Case(torch, B, 8, 1, 64, 16, 700, 100, lens=[100] * B)
        ramp = torch.linspace(0.01, 6.0, 720, device="cuda")[:704].view(44, 16, 1, 1)
        c.k[c.pp.long()] = (c.q[0, 0].sign() * ramp).to(c.dt)
        c.check(c.plan(serving)(c.q))


@pytest.mark.parametrize("B", [3, 40])
def test_what_does_not_exist_makes_its_rows_nan(torch, serving, B):
    c = Case(torch, B, 8, 2, 128, 16, 100, 40, lens=[40] * B, poison=False)
    c.op[1, 0] = -1
    c.op[2, 2] = c.k.shape[0]
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[1]).all() and torch.isnan(out[2]).all()
    good = [b for b in range(B) if b not in (1, 2)]
    want = Case(torch, B, 8, 2, 128, 16, 100, 40, lens=[40] * B, poison=False)
    assert torch.equal(out[good], want.plan(serving)(want.q)[good])
    c = Case(torch, B, 8, 2, 128, 16, 100, 40, lens=[40] * B, poison=False)
    c.lens[0], c.lens[1] = 41, -1
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[:2]).all() and torch.isfinite(out[2:]).all()
    c = Case(torch, B, 8, 2, 128, 16, 100, 40, poison=False)
    c.pp[3] = 1 << 30
    assert torch.isnan(c.plan(serving)(c.q)).all()


@pytest.mark.parametrize("B", [2, 40])
def test_nan_and_infinity_in_keys_in_use_are_not_lost(torch, serving, B):
    c = Case(torch, B, 8, 2, 128, 16, 100, 40, lens=[40] * B, poison=False)
    c.v[c.pp[2].long(), 3, 1, 5] = math.inf
    out = c.plan(serving)(c.q)
    assert torch.isinf(out[:, 4:, 5]).all() and torch.isfinite(out[:, :4]).all()
    c = Case(torch, B, 8, 2, 128, 16, 100, 40, lens=[40] * B, poison=False)
    c.k[c.op[1, 0].long(), 0, 0] = math.nan
    out = c.plan(serving)(c.q)
    assert torch.isnan(out[1, :4]).all() and torch.isfinite(out[1, 4:]).all() and torch.isfinite(out[0]).all()


@pytest.mark.parametrize("what", ["pages", "heads"])
def test_a_stride_of_zero(torch, serving, what):
    """Pages, or key heads, that are all the same memory."""
    for B in (3, 128):
        c = Case(torch, B, 32, 4, 64, 16, 900, 20, poison=False)
        c.k, c.v = (t[:1].expand(t.shape) if what == "pages" else t[:, :, :1].expand(t.shape) for t in (c.k, c.v))
        c.check(c.plan(serving)(c.q))


def test_offsets_past_32_bits(torch, serving):
    """A cache of 6 GB, the pages in use at its end."""
    n, page, Hk, d = 12_000, 256, 4, 128
    k = torch.zeros(n, page, Hk, d, device="cuda", dtype=torch.bfloat16)
    small = Case(torch, 3, 8, 4, d, page, 700, 300, poison=False)
    last = small.k.shape[0]
    k[-last:] = small.k
    v = torch.zeros_like(k); v[-last:] = small.v
    want = small.plan(serving)(small.q)
    small.k, small.v = k, v
    small.pp += n - last; small.op += n - last
    assert torch.equal(small.plan(serving)(small.q), want)


@pytest.mark.parametrize("shape", [(2, 8, 2, 128, 16, 300, 64), (40, 8, 2, 128, 16, 300, 64)])
def test_captured_and_replayed_on_another_stream(torch, serving, shape):
    c = Case(torch, *shape, poison=False)
    st = torch.cuda.Stream()
    plan = c.plan(serving, stream=st)
    out = torch.empty_like(c.q)
    torch.cuda.synchronize()
    plan(c.q, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        plan(c.q, out)
    for turn in range(3):
        c.lens.copy_(torch.randint(0, 65, c.lens.shape, device="cuda")); c.q.mul_(-1.0); out.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            graph.replay()
        torch.cuda.synchronize()
        c.check(out)


def test_two_plans_on_two_streams(torch, serving):
    cases = [Case(torch, 40, 8, 2, 128, 16, 3000, 64, seed=s, poison=False) for s in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    plans = [c.plan(serving, stream=s) for c, s in zip(cases, streams)]
    outs = [torch.empty_like(c.q) for c in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, p, o in zip(cases, plans, outs):
            p(c.q, o)
    torch.cuda.synchronize()
    for c, o in zip(cases, outs):
        c.check(o)


def test_the_same_call_gives_the_same_bits(torch, serving):
    for shape in [(3, 32, 4, 128, 16, 5000, 300), (64, 32, 4, 128, 16, 3000, 200)]:
        c = Case(torch, *shape, poison=False)
        plan = c.plan(serving)
        first = plan(c.q).clone()
        for _ in range(5):
            assert torch.equal(plan(c.q), first)


def test_binding_refuses(torch, serving):
    from paper_2609_09800_b200 import hbf
    c = Case(torch, 2, 8, 2, 128, 16, 40, 20, poison=False)
    plan = c.plan(serving)
    for q in (c.q[:1], c.q.float(), c.q.cpu(), c.q.transpose(0, 1)):
        with pytest.raises(ValueError):
            plan(q)
    with pytest.raises(ValueError):
        serving.PrefixAttention(c.k, c.v[:-1], 2, 8)
    with pytest.raises(ValueError):
        serving.PrefixAttention(c.k, c.v, 2, 8, c.pp[:1], 40)
    with pytest.raises(ValueError):
        serving.PrefixAttention(c.k, c.v, 2, 8, None, 0, c.op, c.lens, 200)
    with pytest.raises(hbf.HbfError):
        serving.PrefixAttention(c.k, c.v, 2, 7, c.pp, 40)
    off = torch.empty(2 * 8 * 128 + 8, dtype=c.dt, device="cuda")[4:][:2 * 8 * 128].view(2, 8, 128)
    with pytest.raises(hbf.HbfError):                        # not on a 16-byte boundary
        plan(c.q, off)
    import ctypes as C
    plan(c.q)
    lib = hbf.lib()
    a = plan._a
    assert lib.hbf_prefix_attention(C.byref(a), plan._ws_ptr, plan._ws_bytes - 256, None) == hbf.E_WORKSPACE
    assert lib.hbf_prefix_attention(C.byref(a), plan._ws_ptr + 128, plan._ws_bytes, None) == hbf.E_WORKSPACE
    host = torch.zeros(64, dtype=c.dt).pin_memory()
    a.kv.k = host.data_ptr()                                 # host memory is not the device's
    assert lib.hbf_prefix_attention(C.byref(a), plan._ws_ptr, plan._ws_bytes, None) == hbf.E_INVAL


def test_records(torch, serving):
    c = Case(torch, 3, 8, 2, 128, 16, 40, 33, lens=[33, 0, 16])
    plan = c.plan(serving)
    rec = plan.accesses(1000, 7).cpu()
    words = c.page * c.Hk * c.d * 2
    pages = [(int(p), True) for p in c.pp] + [(int(c.op[b, j]), j * 16 < int(c.lens[b])) for b in range(3) for j in range(3)]
    assert rec.shape == (2 * len(pages), 3)
    for i, (p, there) in enumerate(pages):
        for which, t in enumerate((c.k, c.v)):
            addr, issue, rest = rec[2 * i + which].tolist()
            assert issue == 1000 + 7 * (2 * i + which)
            assert (addr, rest) == ((t.data_ptr() + p * words, words) if there else (0, 1))
