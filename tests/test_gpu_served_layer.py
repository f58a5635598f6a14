"""The operators together, as a serving loop uses them: requests fork from a shared prefix, grow, attend, go through the experts, some end, the cache
closes up, and what is left attends as before; the accesses of every step are served by the model, bit for bit as the oracle serves them."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

from oracle import hbfo
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


SMALL = dict(batch=20, prefix_tokens=1003, own_tokens=24, hidden=256, inter=64, n_experts=12, top_k=3, q_heads=16, kv_heads=4, head_dim=64)


def reference(torch, layer, q):
    """Attention in 64 bits from the requests' whole tables."""
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    B, H, d = q.shape
    for b in range(B):
        n = int(layer.lens[b + 1])
        if n == 0:
            continue
        pages = layer.tables[b + 1, :-(-n // layer.page)].long()
        k, v = (layer.kv[i, pages].flatten(0, 1)[:n].double() for i in range(2))
        qb = q[b].double().view(k.shape[1], -1, d)
        p = torch.softmax(torch.einsum("hgd,lhd->hgl", qb, k) * d ** -0.5, -1)
        out[b] = torch.einsum("hgl,lhd->hgd", p, v).reshape(H, d)
    return out


def close(torch, got, want):
    """bf16: the output rounded once, a weight twice at most, sums of magnitudes below 8."""
    return ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -8 * 1.0).all()


def test_a_serving_loop(torch, mods):
    hbf, serving = mods
    prof = wl.load_profile("nominal", **wl.GEOMETRY["serving"])
    ctx, o = hbf.Context(prof), hbfo.Oracle(prof)
    layer = serving.ServedLayer(ctx, **SMALL, seed=3)
    mib = lambda t: -(-t.numel() * 2 // (1 << 20)) << 20
    o.register_range(layer.experts.data_ptr(), layer.experts.numel() * 2, 3, 0, 0, 0)
    o.register_range(layer.kv.data_ptr(), layer.kv.numel() * 2, 3, 0, 0, mib(layer.experts))
    B = SMALL["batch"]
    # the requests share the prefix's 62 full pages and have a copy of the one that it had begun
    assert int(layer.refs[0]) == B + 1 and (layer.lens == 1003).all()
    assert (layer.tables[1:, :62] == layer.tables[0, :62]).all() and len(set(layer.tables[1:, 62].tolist()) | {int(layer.tables[0, 62])}) == B + 1
    rnd = lambda *s: torch.randn(*s, device="cuda").bfloat16()

    def served(what):
        for acc, comp, stall, stats in what:
            rec = np.ascontiguousarray(acc.cpu().numpy()).view(hbfo.ACCESS_DTYPE).reshape(-1)
            _, c_o, s_o, _, ds_o = o.submit(rec)
            assert np.array_equal(comp.cpu().numpy(), c_o) and np.array_equal(stall.cpu().numpy(), s_o)
            got = stats.cpu().numpy().view(hbf.DIE_STATS_DTYPE).reshape(-1)
            assert all(np.array_equal(got[k], ds_o[k]) for k in hbf.DIE_STATS_DTYPE.names)
        assert np.array_equal(ctx.get_busy_until(), o.busy_until())

    issue = 0
    for step in range(5):
        layer.append(rnd(B, 4, 64), rnd(B, 4, 64))
        q, x, scores = rnd(B, 16, 64), rnd(B, 256), torch.randn(B, 12, device="cuda")
        att, y, what = layer.step(q, x, scores, issue, 15)
        assert close(torch, att, reference(torch, layer, q)) and torch.isfinite(y).all()
        served(what)
        issue += 15 * sum(int(w[0].shape[0]) for w in what)
    # seven requests end; the cache closes up, which programs pages; the others attend as before
    gone = torch.tensor([2, 3, 5, 8, 13, 19, 20], device="cuda", dtype=torch.int32)
    # (the pages that a request has not grown into yet are held outside its length: given back by hand, as they were taken)
    for r in gone.tolist():
        unused = layer.tables[r, -(-int(layer.lens[r]) // layer.page):]
        layer.refs[unused[unused >= 0].long()] -= 1
    layer.cache.free(gone)
    layer.cache.result()
    for r in range(1, B + 1):
        if r not in gone.tolist():
            unused = layer.tables[r, -(-int(layer.lens[r]) // layer.page):]
            layer.refs[unused[unused >= 0].long()] -= 1
            unused.fill_(-1)
    before = layer.attention(q).clone()
    layer.cache.compact()
    moved = layer.cache.result()
    served([ctx.serve(layer.cache, issue, 15)])
    held = {int(p) for r in range(B + 1) for p in layer.tables[r, :-(-int(layer.lens[r]) // layer.page)]}
    assert moved["in_use"] == len(held) and held == set(range(len(held))) and moved["moved"] > 0
    keep = [b for b in range(B) if b + 1 not in gone.tolist()]
    layer.attention._keep[2].copy_(layer.tables[0, :62])          # the prefix's list, which the plan reads at every call
    torch.sub(layer.lens[1:], layer.base_tokens, out=layer.own_len)
    layer.own_len.clamp_(min=0)
    after = layer.attention(q)
    assert torch.equal(after[keep], before[keep])
    want = reference(torch, layer, q)
    assert close(torch, after[keep], want[keep])


@pytest.mark.parametrize("prefix, own", [(40, 5), (48, 16), (7, 0), (0, 3), (0, 0)])
def test_requests_stop_growing_where_their_room_ends(torch, mods, prefix, own):
    hbf, serving = mods
    ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["serving"]))
    layer = serving.ServedLayer(ctx, **dict(SMALL, batch=3, prefix_tokens=prefix, own_tokens=own))
    room = -(-(prefix % 16 + own) // 16) * 16 - prefix % 16      # tokens that the pages hold
    rnd = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    for i in range(room + 40):
        full = layer.kv.clone() if i >= room else None
        assert layer.append(rnd(3, 4, 64), rnd(3, 4, 64)).tolist() == [i < room] * 3
        assert layer.lens.tolist() == [prefix] + [prefix + min(i + 1, room)] * 3
        assert full is None or torch.equal(full[:, :-1], layer.kv[:, :-1])
    q = rnd(3, 16, 64)
    out, _, _ = layer.step(q, rnd(3, 256), torch.randn(3, 12, device="cuda"))
    assert close(torch, out, reference(torch, layer, q))


def test_a_freed_request_takes_no_token(torch, mods):
    hbf, serving = mods
    ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["serving"]))
    layer = serving.ServedLayer(ctx, **dict(SMALL, batch=3, prefix_tokens=40, own_tokens=5))
    rnd = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    layer.cache.free(torch.tensor([2], device="cuda", dtype=torch.int32))
    layer.cache.result()
    assert layer.append(rnd(3, 4, 64), rnd(3, 4, 64)).tolist() == [True, False, True] and layer.lens.tolist() == [40, 41, 0, 41]
    layer.cache.fork(torch.tensor([0], device="cuda", dtype=torch.int32), torch.tensor([2], device="cuda", dtype=torch.int32))
    layer.cache.result()
    q = rnd(3, 16, 64)
    out, _, _ = layer.step(q, rnd(3, 256), torch.randn(3, 12, device="cuda"))
    assert layer.lens.tolist() == [40, 41, 40, 41] and close(torch, out, reference(torch, layer, q))


def test_serving_needs_the_same_stream(torch, mods):
    hbf, serving = mods
    ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["tiny"]))
    w = torch.randn(4, 3 * 64 * 32, device="cuda").bfloat16()
    op = serving.MoeLayer(w, 64, 32, 1, 4, stream=torch.cuda.Stream())
    with pytest.raises(ValueError):
        ctx.serve(op)


def test_native_places_cost_nothing(torch, mods):
    """Records of places that an operator did not use are native: no queue sees them."""
    hbf, serving = mods
    ctx = hbf.Context(wl.load_profile("nominal", **wl.GEOMETRY["tiny"]))
    w = torch.randn(8, 3 * 64 * 32, device="cuda").bfloat16()
    ctx.register_range(w.data_ptr(), w.numel() * 2, 1)
    op = serving.MoeLayer(w, 64, 32, 1, 4, tile_bytes=4096)
    scores = torch.full((4, 8), -1.0, device="cuda"); scores[:, 5] = 1.0
    op(torch.randn(4, 64, device="cuda").bfloat16(), scores)
    acc, comp, stall, stats = ctx.serve(op, 100, 3)
    res = ctx.last_result()
    assert acc.shape[0] == 4 * 3 and res["n_modeled"] == 3 and res["n_native"] == 9 and res["code"] == 0
    assert int((stall > 0).sum()) == 3 and int(stats[:, 4].sum()) == 3
