"""The operators of a served layer whose memory lies in registered ranges, as cases that can be timed: attention of a batch that
shares a long prefix, a mixture-of-experts layer for a few tokens, and the operations on the pages of a key/value cache.

A case is a dict of plain values.  Its "kind" says which operator it is:

  attention  one decode step of a batch: every request's query token against the prefix that all share (read once) and against
             the keys that only the request has; keys and values in pages, found through page tables
  moe        one layer's experts for a few tokens: the top-k choice from the router's scores, gate and up product, SiLU, down
             product, the weighted sum; the experts lie one behind the other as in the weight image (gate, up, down)
  pages      bookkeeping of a paged cache with the copies it takes; "action" is copy (listed pages), fork (rows that begin as
             another row's tokens, full pages shared, a started page copied) or retire (rows given back, then what is left
             moved to the lowest page numbers)

With `own` false the operators are computed from elementary torch operations in 32 bits; with `own` true by the library's kernels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # One user's next token behind an 8K system prompt: latency, eight query rows per key head.
        dict(name="attention_1x8k", kind="attention", batch=1, q_heads=32, kv_heads=4, dim=128, page=16, prefix=8192, own=100, dtype="bf16"),
        # The shared-prefix serving stream's step: 64 requests behind 8K tokens, each with up to 512 tokens of its own.
        dict(name="attention_64x8k", kind="attention", batch=64, q_heads=32, kv_heads=4, dim=128, page=16, prefix=8192, own=512, dtype="bf16"),
        # A large batch behind a 32K document, with long answers: the largest call.
        dict(name="attention_128x32k", kind="attention", batch=128, q_heads=32, kv_heads=4, dim=128, page=64, prefix=32768, own=2048, dtype="fp16"),
        # Odd sizes: pages of 12 tokens, five heads a group, heads of 64, a prefix that ends inside a page, rows without own tokens.
        dict(name="attention_13x5k_odd", kind="attention", batch=13, q_heads=10, kv_heads=2, dim=64, page=12, prefix=5001, own=333, dtype="bf16"),
        # Single-token decode of the weight-streaming model: eight experts are read.
        dict(name="moe_1", kind="moe", tokens=1, hidden=2048, inter=768, experts=128, top_k=8, dtype="bf16"),
        # A handful of requests: up to 64 of the experts.
        dict(name="moe_8", kind="moe", tokens=8, hidden=2048, inter=768, experts=128, top_k=8, dtype="bf16"),
        # The batch of the shared-prefix stream: nearly every expert, a few tokens each; the largest call.
        dict(name="moe_64", kind="moe", tokens=64, hidden=2048, inter=768, experts=128, top_k=8, dtype="bf16"),
        # Sizes that are no multiple of any tile, few experts with many tokens each.
        dict(name="moe_37_odd", kind="moe", tokens=37, hidden=1000, inter=520, experts=12, top_k=3, dtype="fp16"),
        # A beam of three in a small cache: latency.
        dict(name="pages_fork_3", kind="pages", action="fork", slabs=4, pages=256, page_bytes=4096, page=4, rows=8, forks=3, length=403),
        # 64 requests fork from the prefix of the serving stream, all 48 layers' keys and values.
        dict(name="pages_fork_64", kind="pages", action="fork", slabs=96, pages=640, page_bytes=16384, page=16, rows=72, forks=64, length=8185),
        # Half of the requests end, what the others hold closes up.
        dict(name="pages_retire_40", kind="pages", action="retire", slabs=96, pages=900, page_bytes=16384, page=16, rows=80, forks=40, length=150),
        # A swap of 300 pages into another part of the cache, odd page size.
        dict(name="pages_copy_300", kind="pages", action="copy", slabs=31, pages=1000, page_bytes=12304, page=7, rows=4, forks=300, length=70),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attention", "moe", "pages"])
    dtype = rng.choice(["bf16", "fp16"])
    if kind == "attention":
        kv_heads, group = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
        batch, heads = _log(rng, 1, 128), kv_heads * group
        prefix = _log(rng, 1, min(32768, (128 * 32 * 32768) // (batch * heads)))
        own_len = _log(rng, 1, min(2048, 128 * 2048 * 4 // (batch * kv_heads)))
        return dict(kind=kind, batch=batch, q_heads=heads, kv_heads=kv_heads, dim=rng.choice([64, 128]), page=rng.choice([1, 8, 12, 16, 32, 64, 100]),
                    prefix=prefix, own=own_len, dtype=dtype)
    if kind == "moe":
        experts = _log(rng, 2, 128)
        hidden, inter = 8 * _log(rng, 16, 512), 8 * _log(rng, 8, 256)
        experts = max(1, min(experts, 128 * 2048 * 768 // (hidden * inter)))
        return dict(kind=kind, tokens=_log(rng, 1, 128), hidden=hidden, inter=inter, experts=experts, top_k=rng.randint(1, min(8, experts)), dtype=dtype)
    action = rng.choice(["copy", "fork", "retire"])
    page, page_bytes, slabs = rng.choice([1, 4, 7, 16, 64]), 16 * _log(rng, 16, 2048), _log(rng, 1, 96)
    pages = max(24, min(_log(rng, 24, 4000), (900 * 96 * 16384) // (slabs * page_bytes)))
    forks = _log(rng, 1, max(1, min(64, pages // 12)))
    rows = max(2, 2 * forks)
    longest = page * (pages // 3) if action == "fork" else max(1, page * (pages // rows) - 1)
    return dict(kind=kind, action=action, slabs=slabs, pages=pages, page_bytes=page_bytes, page=page, rows=rows,
                forks=min(pages // 2, 6 * forks) if action == "copy" else forks, length=_log(rng, 1, longest))


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _prepare_attention(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    B, page = c["batch"], c["page"]
    n_prefix, n_own = -(-c["prefix"] // page), -(-c["own"] // page)
    n_pages = n_prefix + B * n_own + 3
    k, v = (torch.randn(n_pages, page, c["kv_heads"], c["dim"], device="cuda", generator=g, dtype=dt) for _ in range(2))
    q = torch.randn(B, c["q_heads"], c["dim"], device="cuda", generator=g, dtype=dt)
    order = torch.randperm(n_pages, device="cuda", generator=g).to(torch.int32)           # a cache in use: pages in no order
    own_len = torch.randint(0, c["own"] + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    own_len[0] = c["own"]
    s = dict(case=c, k=k, v=v, q=q, out=torch.empty_like(q), prefix_pages=order[:n_prefix].contiguous(),
             own_pages=order[n_prefix:n_prefix + B * n_own].reshape(B, n_own).contiguous(), own_len=own_len)
    if own:
        from paper_2609_09800_b200 import serving
        s["plan"] = serving.PrefixAttention(k, v, B, c["q_heads"], s["prefix_pages"], c["prefix"], s["own_pages"], own_len, c["own"])
    return s


def _prepare_moe(c, seed):
    g, dt = _gen(seed), DTYPES[c["dtype"]]
    T, D, I, E = c["tokens"], c["hidden"], c["inter"], c["experts"]
    w = torch.randn(E, 3 * I * D, device="cuda", generator=g, dtype=dt)
    w[:, :2 * I * D] *= D ** -0.5
    w[:, 2 * I * D:] *= I ** -0.5
    x = torch.randn(T, D, device="cuda", generator=g, dtype=dt)
    # experts are not equally popular: a score for each expert, and one for each token and expert
    scores = torch.randn(E, device="cuda", generator=g) * 0.7 + torch.randn(T, E, device="cuda", generator=g)
    s = dict(case=c, w=w, x=x, scores=scores, out=torch.empty_like(x), chosen=torch.empty(T, c["top_k"], device="cuda", dtype=torch.int32),
             weights=torch.empty(T, c["top_k"], device="cuda"))
    if own:
        from paper_2609_09800_b200 import serving
        s["plan"] = serving.MoeLayer(w, D, I, c["top_k"], T)
    return s


def _prepare_pages(c, seed):
    g = _gen(seed)
    P, page, R = c["pages"], c["page"], c["rows"]
    data = torch.randint(-30000, 30000, (c["slabs"], P, c["page_bytes"] // 2), device="cuda", generator=g, dtype=torch.int16)
    order = torch.randperm(P, device="cuda", generator=g).to(torch.int32)
    width = -(-c["length"] // page) + 1
    # one buffer for what the pages' owner keeps: references of each page, length of each row, each row's table
    meta = torch.zeros(P + R + R * width, device="cuda", dtype=torch.int32)
    refs, lens, tables = meta[:P], meta[P:P + R], meta[P + R:].view(R, width)
    tables.fill_(-1)
    s = dict(case=c, data=data, meta=meta, refs=refs, lens=lens, tables=tables, first=torch.empty_like(meta))
    n = c["forks"]
    if c["action"] == "copy":
        s["src"], s["dst"] = order[:n].contiguous(), order[n:2 * n].contiguous()
    elif c["action"] == "fork":                                                           # row 0 is the parent of all
        held = -(-c["length"] // page)
        tables[0, :held] = order[:held]
        refs[order[:held].long()] = 1
        lens[0] = c["length"]
        s["parents"] = torch.zeros(n, device="cuda", dtype=torch.int32)
        s["children"] = (torch.randperm(R - 1, device="cuda", generator=g)[:n] + 1).to(torch.int32)
    else:                                                                                 # rows of differing lengths; some are given back
        lens.copy_(torch.randint(max(1, c["length"] // 2), c["length"] + 1, (R,), device="cuda", generator=g, dtype=torch.int32))
        held = (lens + page - 1) // page
        at = torch.arange(width, device="cuda")[None, :]
        begin = (held.cumsum(0) - held)[:, None]
        tables.copy_(torch.where(at < held[:, None], order[(begin + at).clamp(max=P - 1).long()], tables))
        refs[order[:int(held.sum())].long()] = 1
        s["gone"] = torch.randperm(R, device="cuda", generator=g)[:n].to(torch.int32)
    s["first"].copy_(meta)
    if own:
        from paper_2609_09800_b200 import serving
        s["plan"] = serving.CachePages(data, refs, tables, lens, page)
    return s


def prepare(case, seed):
    return {"attention": _prepare_attention, "moe": _prepare_moe, "pages": _prepare_pages}[case["kind"]](case, seed)


# ---- one pass -------------------------------------------------------------------------------------------------------------------

def _run_attention(s):
    if own:
        s["plan"](s["q"], s["out"])
        return s["out"]
    c = s["case"]
    B, Hk, d, page = c["batch"], c["kv_heads"], c["dim"], c["page"]
    G, L = c["q_heads"] // Hk, c["prefix"]
    q = s["q"].float().view(B, Hk, G, d) * d ** -0.5
    pk, pv = (t[s["prefix_pages"].long()].flatten(0, 1)[:L].float() for t in (s["k"], s["v"]))         # [L, Hk, d]
    ok, ov = (t[s["own_pages"].long()].flatten(1, 2).float() for t in (s["k"], s["v"]))                # [B, own, Hk, d]
    sp = torch.einsum("bhgd,lhd->bhgl", q, pk)
    so = torch.einsum("bhgd,blhd->bhgl", q, ok)
    there = torch.arange(ok.shape[1], device="cuda")[None, :] < s["own_len"][:, None]                  # [B, own]
    so = so.masked_fill(~there[:, None, None, :], -math.inf)
    m = torch.maximum(sp.amax(-1, keepdim=True), so.amax(-1, keepdim=True))
    ep, eo = torch.exp(sp - m), torch.exp(so - m)
    total = ep.sum(-1, keepdim=True) + eo.sum(-1, keepdim=True)
    o = torch.einsum("bhgl,lhd->bhgd", ep, pv) + torch.einsum("bhgl,blhd->bhgd", eo, ov.masked_fill(~there[:, :, None, None], 0.0))
    s["out"].copy_((o / total).reshape(B, c["q_heads"], d))
    return s["out"]


def _run_moe(s):
    if own:
        s["plan"](s["x"], s["scores"], s["out"], s["chosen"], s["weights"])
        return s["out"], s["chosen"], s["weights"]
    c = s["case"]
    T, D, I, E, K = c["tokens"], c["hidden"], c["inter"], c["experts"], c["top_k"]
    top, chosen = torch.sort(s["scores"], dim=1, descending=True, stable=True)                         # ties: the lowest number first
    top, chosen = top[:, :K], chosen[:, :K]
    weights = torch.exp(top - top[:, :1])
    weights = weights / weights.sum(1, keepdim=True)
    # the experts in use first, at most T * K of them, each with room for all tokens
    used = torch.zeros(E, device="cuda").scatter_(0, chosen.reshape(-1), 1.0)
    A = min(E, T * K)
    active = torch.sort(used, descending=True, stable=True).indices[:A]
    gate = torch.zeros(T, E, device="cuda").scatter_(1, chosen, weights)[:, active]                    # [T, A]
    w = s["w"][active].float()
    gu = w[:, :2 * I * D].view(A, 2 * I, D)
    x = s["x"].float()
    h = torch.matmul(gu, x.t())                                                                        # [A, 2 I, T]
    h = h[:, :I] * torch.sigmoid(h[:, :I]) * h[:, I:]
    y = torch.bmm(w[:, 2 * I * D:].view(A, D, I), h)                                                   # [A, D, T]
    s["out"].copy_(torch.einsum("adt,ta->td", y, gate))
    s["chosen"].copy_(chosen)
    s["weights"].copy_(weights)
    return s["out"], s["chosen"], s["weights"]


def _run_pages(s):
    c = s["case"]
    data, refs, lens, tables, page = s["data"], s["refs"], s["lens"], s["tables"], c["page"]
    s["meta"].copy_(s["first"])                                                                        # the bookkeeping as prepared: a pass can be repeated
    if own:
        if c["action"] == "copy":
            s["plan"].copy(s["src"], s["dst"])
        elif c["action"] == "fork":
            s["plan"].fork(s["parents"], s["children"])
        else:
            s["plan"].free(s["gone"])
            s["plan"].compact()
        return data, refs, lens, tables
    at = torch.arange(tables.shape[1], device="cuda")[None, :]
    if c["action"] == "copy":
        data[:, s["dst"].long()] = data[:, s["src"].long()]
    elif c["action"] == "fork":
        p, ch = s["parents"].long(), s["children"].long()
        full, begun = lens[p] // page, (lens[p] % page > 0).int()
        new = torch.nonzero(refs == 0).flatten()[(begun.cumsum(0) - 1).clamp(min=0).long()]            # lowest free pages, in the order of the children
        shared = (at < full[:, None]) & (at >= 0)
        last = (at == full[:, None]) & (begun[:, None] > 0)
        old = tables[p]
        tables[ch] = torch.where(shared, old, torch.where(last, new[:, None].int(), -1))
        lens[ch] = lens[p]
        refs.scatter_add_(0, old[shared].long(), torch.ones_like(old[shared]))
        mine = begun > 0
        refs[new[mine]] = 1
        data[:, new[mine]] = data[:, old[last].long()]
    else:
        r = s["gone"].long()
        back = tables[r][at < ((lens[r] + page - 1) // page)[:, None]]
        refs.scatter_add_(0, back.long(), -torch.ones_like(back))
        tables[r] = -1
        lens[r] = 0
        live = refs > 0
        n = int(live.sum())
        holes, movers = torch.nonzero(~live[:n]).flatten(), torch.nonzero(live[n:]).flatten() + n
        data[:, holes] = data[:, movers]
        to = torch.arange(c["pages"], device="cuda", dtype=torch.int32)
        to[movers] = holes.int()
        refs[holes] = refs[movers]
        refs[movers] = 0
        tables.copy_(torch.where(tables >= 0, to[tables.clamp(min=0).long()], tables))
    return data, refs, lens, tables


def run(state):
    return {"attention": _run_attention, "moe": _run_moe, "pages": _run_pages}[state["case"]["kind"]](state)


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------------

def work(c):
    if c["kind"] == "attention":                        # every key and value in use once (own lengths: half of the most on average), queries and outputs
        tokens = c["prefix"] + c["batch"] * c["own"] / 2
        rows = c["batch"] * c["q_heads"]
        return {"bytes": 4 * tokens * c["kv_heads"] * c["dim"] + 4 * rows * c["dim"], "flops": 4.0 * rows * c["dim"] * (c["prefix"] + c["own"] / 2)}
    if c["kind"] == "moe":                              # the weights of the experts in use (an even choice is assumed), activations
        T, D, I, E, K = c["tokens"], c["hidden"], c["inter"], c["experts"], c["top_k"]
        used = E * (1.0 - (1.0 - K / E) ** T)
        return {"bytes": 6.0 * used * D * I + 4.0 * T * D + 4.0 * T * E + 8.0 * T * K, "flops": 6.0 * T * K * D * I}
    width = -(-c["length"] // c["page"]) + 1
    meta = 8.0 * (c["pages"] + c["rows"] * (1 + width))
    if c["action"] == "copy":
        moved = c["forks"]
    elif c["action"] == "fork":
        moved = c["forks"] if c["length"] % c["page"] else 0
    else:                                               # of the pages still held, those that lie behind as many as are held
        held = 0.75 * c["length"] / c["page"] * (c["rows"] - c["forks"])
        moved = held * max(0.0, 1.0 - held / c["pages"])
    return {"bytes": 2.0 * moved * c["slabs"] * c["page_bytes"] + meta, "flops": 0.0}


# ---- the same from the definitions, in 64 bits ---------------------------------------------------------------------------------------

def _exact_attention(s):
    """Request by request: the softmax over the concatenation of the prefix's and the request's own keys."""
    c = s["case"]
    Hk, d = c["kv_heads"], c["dim"]
    G, out = c["q_heads"] // Hk, torch.empty(s["q"].shape, device="cuda", dtype=torch.float64)
    gather = lambda t, pages, n: t.index_select(0, pages.long()).reshape(-1, Hk, d)[:n].double().transpose(0, 1)
    pk, pv = gather(s["k"], s["prefix_pages"], c["prefix"]), gather(s["v"], s["prefix_pages"], c["prefix"])
    for b, n in enumerate(s["own_len"].tolist()):
        k = torch.cat([pk, gather(s["k"], s["own_pages"][b], n)], 1)
        v = torch.cat([pv, gather(s["v"], s["own_pages"][b], n)], 1)
        p = torch.softmax(s["q"][b].double().view(Hk, G, d) @ k.transpose(1, 2) / math.sqrt(d), -1)
        out[b] = (p @ v).reshape(Hk * G, d)
    return out


def _exact_moe(s):
    """Expert by expert, over the tokens that chose it."""
    c = s["case"]
    D, I, K = c["hidden"], c["inter"], c["top_k"]
    order = [sorted(range(c["experts"]), key=lambda e: (-row[e], e))[:K] for row in s["scores"].tolist()]
    chosen = torch.tensor(order, device="cuda", dtype=torch.int64)
    weights = torch.softmax(s["scores"].double().gather(1, chosen), 1)
    out = torch.zeros(s["x"].shape, device="cuda", dtype=torch.float64)
    for e in sorted({e for row in order for e in row}):
        t, at = torch.nonzero(chosen == e, as_tuple=True)
        gate, up, down = (m.double() for m in s["w"][e].split([I * D, I * D, D * I]))
        x = s["x"][t].double()
        h = torch.nn.functional.silu(x @ gate.view(I, D).t()) * (x @ up.view(I, D).t())
        out[t] += weights[t, at][:, None] * (h @ down.view(D, I).t())
    return out, chosen.int(), weights


def _exact_pages(s):
    """The bookkeeping on the host, a page at a time."""
    c, page, data = s["case"], s["case"]["page"], s["data"]
    refs, lens, tables = s["refs"].tolist(), s["lens"].tolist(), s["tables"].tolist()
    moves = []
    if c["action"] == "copy":
        moves = list(zip(s["src"].tolist(), s["dst"].tolist()))
    elif c["action"] == "fork":
        free = iter([i for i, r in enumerate(refs) if r == 0])
        for p, ch in zip(s["parents"].tolist(), s["children"].tolist()):
            lens[ch] = lens[p]
            tables[ch] = [-1] * len(tables[p])
            for j in range(-(-lens[p] // page)):
                if (j + 1) * page <= lens[p]:
                    tables[ch][j] = tables[p][j]
                else:
                    tables[ch][j] = next(free)
                    refs[tables[ch][j]] = 0
                    moves.append((tables[p][j], tables[ch][j]))
                refs[tables[ch][j]] += 1
    else:
        for r in s["gone"].tolist():
            for j in range(-(-lens[r] // page)):
                refs[tables[r][j]] -= 1
            lens[r], tables[r] = 0, [-1] * len(tables[r])
        n = sum(r > 0 for r in refs)
        holes = [i for i in range(n) if refs[i] == 0]
        movers = [i for i in range(n, c["pages"]) if refs[i] > 0]
        moves = list(zip(movers, holes))
        new = dict(moves)
        for a, b in moves:
            refs[b], refs[a] = refs[a], 0
        tables = [[new.get(p, p) for p in row] for row in tables]
    for a, b in moves:
        data[:, b] = data[:, a]
    whole = lambda v: torch.tensor(v, device="cuda", dtype=torch.int32)
    return data, whole(refs), whole(lens), whole(tables)


def exact(case, seed):
    return {"attention": _exact_attention, "moe": _exact_moe, "pages": _exact_pages}[case["kind"]](prepare(case, seed))
