"""The cache of an executed layer through forks, frees and compactions: every row holds its own tokens, and every page is held by as many rows as say so."""
import pytest

pytestmark = pytest.mark.gpu

from paper_2609_09800_b200 import workloads as wl


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2609_09800_b200 import build
    build.build()
    return t


@pytest.fixture(scope="module")
def mods(torch):
    from paper_2609_09800_b200 import hbf, serving
    return hbf, serving


SMALL = dict(hidden=256, inter=64, n_experts=12, top_k=3, q_heads=16, kv_heads=4, head_dim=64)


class Rows:
    """A layer and, beside it on the host, the tokens that each of its rows should hold: lists of [2, kv_heads, head_dim]."""

    def __init__(self, torch, mods, batch, prefix, own, seed=0, page=16, stream=None):
        hbf, serving = mods
        self.torch, self.batch, self.prefix, self.page = torch, batch, prefix, page
        self.ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["serving"]), stream=stream)
        self.layer = serving.ServedLayer(self.ctx, batch=batch, prefix_tokens=prefix, own_tokens=own, page_tokens=page, seed=seed, **SMALL)
        self.room = prefix // page * page + -(-(prefix % page + own) // page) * page      # a row's most tokens
        self.g = torch.Generator(device="cuda"); self.g.manual_seed(seed + 1)
        first = list(self.gather(0))
        self.rows = [list(first) for _ in range(batch + 1)]

    def gather(self, row):
        L = self.layer
        n = int(L.lens[row])
        pages = L.tables[row, :-(-n // self.page)].long()
        return L.kv[:, pages].flatten(1, 2)[:, :n].transpose(0, 1).clone()

    def ints(self, v):
        return self.torch.tensor(v, dtype=self.torch.int32, device="cuda")

    def append(self):
        k, v = (self.torch.randn(self.batch, 4, 64, device="cuda", generator=self.g).bfloat16() for _ in range(2))
        took = self.layer.append(k, v).tolist()
        for b in range(self.batch):
            row = self.rows[b + 1]
            assert took[b] == (self.prefix <= len(row) < self.room), (b, len(row))
            if took[b]:
                row.append(self.torch.stack([k[b], v[b]]))

    def free(self, rows):
        self.layer.cache.free(self.ints(rows)); self.layer.cache.result()
        for r in rows:
            self.rows[r] = []

    def fork(self, parents, children):
        self.layer.cache.fork(self.ints(parents), self.ints(children)); self.layer.cache.result()
        for p, c in zip(parents, children):
            self.rows[c] = list(self.rows[p])

    def compact(self):
        self.layer.cache.compact()
        return self.layer.cache.result()

    def check(self):
        L, torch = self.layer, self.torch
        held = [0] * (L.refs.numel())
        for r, want in enumerate(self.rows):
            assert int(L.lens[r]) == len(want)
            got = self.gather(r)
            assert len(want) == 0 or torch.equal(got, torch.stack(want)), "row %d" % r
            for p in L.tables[r, :-(-len(want) // self.page)].tolist():
                held[p] += 1
        assert L.refs.tolist() == held


@pytest.mark.parametrize("prefix, own", [(40, 60), (48, 70), (7, 40), (0, 50)])
def test_rows_keep_their_tokens(torch, mods, prefix, own):
    r = Rows(torch, mods, 3, prefix, own)
    r.check()
    for _ in range(5):
        r.append()
    r.free([1])
    r.check()
    r.compact()
    r.check()
    for _ in range(9):                                       # into a page of their own behind the one that they were in
        r.append()
    r.check()
    if prefix:
        r.fork([0], [1])                                     # takes the lowest free page, which nobody may still write
        r.check()
    for _ in range(20):
        r.append()
        r.check()
    r.free([3]); r.compact(); r.fork([2], [3])
    for _ in range(r.room):
        r.append()
    r.check()


def test_pages_come_back_however_often_rows_begin_again(torch, mods):
    r = Rows(torch, mods, 6, 30, 50, seed=4)
    pick = torch.Generator().manual_seed(2)
    rnd = lambda n: int(torch.randint(0, n, (1,), generator=pick))
    for turn in range(12):
        for _ in range(rnd(30)):
            r.append()
        gone = sorted({1 + rnd(6) for _ in range(1 + rnd(4))})
        r.free(gone)
        if rnd(2):
            r.compact()
            assert r.compact()["moved"] == 0
        r.check()
        stay = [0] + [i for i in range(1, 7) if i not in gone]
        r.fork([stay[rnd(len(stay))] for _ in gone], gone)
        r.check()
    for _ in range(r.room):                                  # all the room that there ever was
        r.append()
    r.check()
    assert all(len(t) == r.room for t in r.rows[1:])


def test_a_layer_on_a_stream_of_its_own(torch, mods):
    """Everything that a layer is made of is made on its context's stream: work that the current stream still has to do delays none of it."""
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    wrong = [torch.full((20,), 7, dtype=torch.int32, device="cuda") for _ in range(64)]      # what memory of that size may hold
    torch.cuda.synchronize()
    del wrong
    torch.cuda._sleep(200_000_000)                           # some 0.1 s of the current stream
    r = Rows(torch, mods, 20, 40, 30, stream=stream)
    torch.cuda.synchronize()
    r.check()
    assert r.layer.lens.tolist() == [40] * 21


@pytest.mark.parametrize("prefix", [40, 7, 0])
def test_a_request_without_tokens_attends_to_nothing(torch, mods, prefix):
    r = Rows(torch, mods, 4, prefix, 30)
    for _ in range(3):
        r.append()
    r.free([2, 4])
    rnd = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    q, x, scores = rnd(4, 16, 64), rnd(4, 256), torch.randn(4, 12, device="cuda")
    out, y, served = r.layer.step(q, x, scores)
    assert not out[[1, 3]].any() and torch.isfinite(y).all()
    for b in (0, 2):
        k, v = torch.stack(r.rows[b + 1]).double().unbind(1)
        p = torch.softmax(torch.einsum("hgd,lhd->hgl", q[b].double().view(4, 4, 64), k) * 64 ** -0.5, -1)
        want = torch.einsum("hgl,lhd->hgd", p, v).reshape(16, 64)
        size = torch.einsum("hgl,lhd->hgd", p, v.abs()).reshape(16, 64)
        # the output rounded once, the weights at most once, the rest in 32 bits
        assert ((out[b].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -16) * size).all()
    # the pages of requests without tokens are not read
    pages = served[0][0][:, 0].view(-1, 2)[prefix // 16:].view(4, -1, 2)
    assert not pages[[1, 3]].any() and pages[[0, 2], 0].all()


def test_a_refused_token_takes_no_page(torch, mods):
    r = Rows(torch, mods, 3, 16, 40)
    good, L = torch.randn(3, 4, 64, device="cuda").bfloat16(), r.layer
    for bad in (good.float(), good[:2], good[:, :3], good.cpu(), good[:, :, :32], good[None], good[:1]):
        for k, v in ((good, bad), (bad, good)):
            with pytest.raises(ValueError):
                L.append(k, v)
    r.check()                                                # a page of its own would have begun
    r.append()
    r.check()
