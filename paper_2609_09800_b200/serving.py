"""Operators of a served layer whose memory lies in registered ranges (``include/hbf.h``): thin classes over the C calls.

An object keeps what a serving loop keeps between calls (the argument struct, the workspace); its calls run on the stream it was
made for, like a ``Context``'s, allocate nothing when the outputs are given, and wait for nothing.  ``accesses`` gives the records of
what the last call read and programmed, for ``Context.serve`` or ``Context.submit_batch``.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes as C

from . import hbf

_RECORD_WORDS = 3                                             # a 24-byte access record as int64


def _check(ok, what):
    if not ok:
        raise ValueError(what)


class _Operator:
    def __init__(self, anchor, stream):
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("hbf needs a CUDA device; there is no CPU fallback")
        self._torch = torch
        self._lib = hbf.lib()
        self.device = anchor.device
        _check(anchor.is_cuda and self.device.index == torch.cuda.current_device(), "the operator's memory is not on the current CUDA device")
        self.stream = stream if stream is not None else torch.cuda.current_stream()
        _check(self.stream.device == self.device, "the stream belongs to another device")
        self._st = self.stream.cuda_stream
        self._dev, self._i32, self._f32 = self.device.index, torch.int32, torch.float32

    def _int32(self, t, what, dims):
        _check(t is not None and t.dtype == self._torch.int32 and t.dim() == dims and t.device == self.device and (t.shape[-1] < 2 or t.numel() == 0 or t.stride(-1) == 1),
               "%s has to be an int32 tensor of %d dimension(s) on %s" % (what, dims, self.device))
        return t

    def _room(self, nbytes):
        if nbytes == 0:
            raise hbf.HbfError(hbf.E_INVAL, type(self).__name__)
        with self._torch.cuda.stream(self.stream):
            return self._torch.empty(nbytes, dtype=self._torch.uint8, device=self.device)

    def _records(self, n, out):
        """Room for n records: the caller's, of exactly as many, or new."""
        if out is None:
            with self._torch.cuda.stream(self.stream):
                return self._torch.empty(n, _RECORD_WORDS, dtype=self._torch.int64, device=self.device)
        _check(out.dtype == self._torch.int64 and out.shape == (n, _RECORD_WORDS) and out.device == self.device and out.is_contiguous(),
               "out has to be a contiguous int64 tensor of [%d, %d] on %s" % (n, _RECORD_WORDS, self.device))
        return out

    def _raise(self, rc, what):
        if rc != 0:
            raise hbf.HbfError(rc, what)


def _strides(t):
    """Strides, those of dimensions of size one (which may be anything) as if the tensor were dense."""
    out, dense = [], 1
    for n, st in zip(reversed(t.shape), reversed(t.stride())):
        out.append(st if n > 1 else dense)
        dense *= n
    return tuple(reversed(out))


def _dtype_of(t, torch):
    _check(t.dtype in (torch.bfloat16, torch.float16), "values have to be bfloat16 or float16")
    return hbf.BF16 if t.dtype == torch.bfloat16 else hbf.FP16


class PrefixAttention(_Operator):
    """``hbf_prefix_attention``: one decode step's attention for a batch that shares a prefix.

    k, v: [pages, page_tokens, kv_heads, head_dim], alike in strides, the last dimension dense (a view with pages of [kv_heads, page_tokens,
    head_dim] transposed will do).  prefix_pages: int32 [>= ceil(prefix_len / page_tokens)].  own_pages: int32 [batch, columns], own_len: int32
    [batch], both read anew at every call; max_own_len bounds the lengths.  scale defaults to head_dim ** -0.5."""

    def __init__(self, k, v, batch, q_heads, prefix_pages=None, prefix_len=0, own_pages=None, own_len=None, max_own_len=0, scale=None, stream=None):
        super().__init__(k, stream)
        torch = self._torch
        _check(k.dim() == 4 and k.shape == v.shape and _strides(k) == _strides(v) and k.dtype == v.dtype and v.device == self.device and k.stride(3) == 1,
               "k and v have to be alike: [pages, page_tokens, kv_heads, head_dim], dense in the last dimension")
        a = self._a = hbf.hbf_attention_t()
        a.kv.n_pages, a.kv.page_tokens, a.kv.kv_heads, a.kv.head_dim = k.shape
        a.kv.dtype = _dtype_of(k, torch)
        a.kv.k, a.kv.v = k.data_ptr(), v.data_ptr()
        a.kv.page_stride, a.kv.slot_stride, a.kv.head_stride = _strides(k)[:3]
        a.batch, a.q_heads, a.prefix_len, a.max_own_len = batch, q_heads, prefix_len, max_own_len
        a.scale = scale if scale is not None else a.kv.head_dim ** -0.5
        pages_for = lambda n: -(-n // a.kv.page_tokens)
        if prefix_len:
            self._int32(prefix_pages, "prefix_pages", 1)
            _check(prefix_pages.numel() >= pages_for(prefix_len), "prefix_pages is shorter than the prefix")
            a.prefix_pages = prefix_pages.data_ptr()
        if max_own_len:
            self._int32(own_pages, "own_pages", 2), self._int32(own_len, "own_len", 1)
            _check(own_pages.shape[0] == batch and own_len.numel() == batch and own_pages.shape[1] >= pages_for(max_own_len) and
                   (batch < 2 or own_pages.stride(0) >= own_pages.shape[1]), "own_pages or own_len does not hold the batch's own keys")
            a.own_pages, a.own_len = own_pages.data_ptr(), own_len.data_ptr()
            a.own_pages_stride = own_pages.stride(0) if batch > 1 else own_pages.shape[1]
        self._keep = (k, v, prefix_pages, own_pages, own_len)
        self._ref = C.byref(a)
        self._ws = self._room(self._lib.hbf_attention_workspace_bytes(self._ref))
        self._ws_ptr, self._ws_bytes = self._ws.data_ptr(), self._ws.numel()
        self._shape, self._dtype, self._alone = torch.Size((batch, q_heads, k.shape[3])), k.dtype, batch == 1 or q_heads == 1

    def __call__(self, q, out=None, lse=None):
        """q: [batch, q_heads, head_dim]; returns out (made if not given).  lse: float32 [batch, q_heads], filled if given."""
        if out is None:
            with self._torch.cuda.stream(self.stream):
                out = self._torch.empty(self._shape, dtype=self._dtype, device=self.device)
        qs, os = q.stride(), out.stride()
        if q.shape != self._shape or out.shape != self._shape or q.dtype is not self._dtype or out.dtype is not self._dtype or qs[2] != 1 or os[2] != 1 or \
                q.get_device() != self._dev or out.get_device() != self._dev:
            raise ValueError("q and out have to be [batch, q_heads, head_dim] of the cache's type, dense in the last dimension")
        if lse is not None:
            _check(lse.shape == self._shape[:2] and lse.dtype == self._torch.float32 and lse.device == self.device and lse.is_contiguous(), "lse has to be float32 [batch, q_heads]")
        a = self._a
        a.q, a.out, a.lse = q.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr()
        if self._alone:                                      # (one row, or one head)
            qs, os = _strides(q), _strides(out)
        a.q_row_stride, a.q_head_stride, a.out_row_stride, a.out_head_stride = qs[0], qs[1], os[0], os[1]
        rc = self._lib.hbf_prefix_attention(self._ref, self._ws_ptr, self._ws_bytes, self._st)
        if rc:
            self._raise(rc, "hbf_prefix_attention")
        return out

    def access_count(self):
        return self._lib.hbf_attention_access_count(self._ref)

    def accesses(self, issue_ns=0, gap_ns=0, out=None):
        """Records of the pages that a call reads, the prefix's once: int64 [n, 3]."""
        n = self.access_count()
        out = self._records(n, out)
        self._raise(self._lib.hbf_attention_accesses(self._ref, issue_ns, gap_ns, out.data_ptr(), n, self._st), "hbf_attention_accesses")
        return out


class MoeLayer(_Operator):
    """``hbf_moe_layer``: a mixture-of-experts layer for up to max_tokens (128 at most) tokens.

    experts: [n_experts, >= 3 * inter * hidden], a row an expert's gate, up and down one behind the other.  tile_bytes: size of the
    records that ``accesses`` writes."""

    def __init__(self, experts, hidden, inter, top_k, max_tokens, renormalise=True, tile_bytes=65536, stream=None):
        super().__init__(experts, stream)
        _check(experts.dim() == 2 and experts.shape[1] >= 3 * hidden * inter and experts.stride(1) == 1, "experts has to be [n_experts, >= 3 * inter * hidden], rows dense")
        m = self._m = hbf.hbf_moe_t()
        m.tokens, m.hidden, m.inter, m.n_experts, m.top_k = max_tokens, hidden, inter, experts.shape[0], top_k
        m.dtype, m.renormalise = _dtype_of(experts, self._torch), 1 if renormalise else 0
        m.experts, m.expert_stride = experts.data_ptr(), experts.stride(0) if experts.shape[0] > 1 else max(experts.stride(0), 3 * hidden * inter)
        self._keep = experts
        self._ref = C.byref(m)
        _check(max_tokens >= 1, "max_tokens has to be at least 1")
        self._ws = self._room(self._lib.hbf_moe_workspace_bytes(self._ref))
        self._ws_ptr, self._ws_bytes = self._ws.data_ptr(), self._ws.numel()
        self._dtype, self.max_tokens, self.tile_bytes = experts.dtype, max_tokens, tile_bytes
        self._last = None

    def __call__(self, x, scores, out=None, chosen=None, weights=None):
        """x: [tokens, hidden]; scores: float32 [tokens, n_experts]; returns out (made if not given).  chosen (int32) and weights (float32), both
        [tokens, top_k] and contiguous, are filled if given."""
        torch, m = self._torch, self._m
        if out is None:
            with torch.cuda.stream(self.stream):
                out = torch.empty(x.shape, dtype=self._dtype, device=self.device)
        n, want, dev = x.shape[0], (x.shape[0], m.hidden), self._dev
        xs, os, ss = x.stride(), out.stride(), scores.stride()
        if n > self.max_tokens or x.shape != want or out.shape != want or x.dtype is not self._dtype or out.dtype is not self._dtype or xs[1] != 1 or os[1] != 1 or \
                x.get_device() != dev or out.get_device() != dev:
            raise ValueError("x and out have to be [tokens <= max_tokens, hidden] of the experts' type, rows dense")
        if scores.shape != (n, m.n_experts) or scores.dtype is not self._f32 or scores.get_device() != dev or (ss[1] != 1 and m.n_experts > 1):
            raise ValueError("scores has to be float32 [tokens, n_experts], rows dense")
        for t, dt in ((chosen, self._i32), (weights, self._f32)):
            if t is not None and (t.shape != (n, m.top_k) or t.dtype is not dt or t.get_device() != dev or not t.is_contiguous()):
                raise ValueError("chosen (int32) and weights (float32) have to be [tokens, top_k], contiguous")
        m.tokens = n
        m.x, m.x_stride = x.data_ptr(), xs[0] if n > 1 else m.hidden
        m.scores, m.scores_stride = scores.data_ptr(), ss[0] if n > 1 else m.n_experts
        m.out, m.out_stride = out.data_ptr(), os[0] if n > 1 else m.hidden
        m.chosen, m.weights = None if chosen is None else chosen.data_ptr(), None if weights is None else weights.data_ptr()
        self._last = None                                    # a call that is refused has no accesses
        rc = self._lib.hbf_moe_layer(self._ref, self._ws_ptr, self._ws_bytes, self._st)
        if rc:
            self._raise(rc, "hbf_moe_layer")
        self._last = scores                                  # `accesses` makes the choice again
        return out

    def access_count(self):
        return self._lib.hbf_moe_access_count(self._ref, self.tile_bytes) if self._last is not None else 0

    def accesses(self, issue_ns=0, gap_ns=0, out=None):
        """Records of the experts that the last call read, from its scores as they are now: int64 [n, 3]."""
        n = self.access_count()
        out = self._records(n, out)
        self._raise(self._lib.hbf_moe_accesses(self._ref, self.tile_bytes, issue_ns, gap_ns, out.data_ptr(), n, self._st) if n else 0, "hbf_moe_accesses")
        return out


class CachePages(_Operator):
    """``hbf_pages_*``: the pages of a key/value cache, with the bookkeeping of who holds them.

    data: [slabs, pages, ...], a page dense; refs: int32 [pages]; tables: int32 [rows, columns]; lens: int32 [rows]; all changed in place.  Calls
    are asynchronous; ``result`` waits for the last one and raises if it was refused."""

    def __init__(self, data, refs, tables, lens, page_tokens, stream=None):
        super().__init__(data, stream)
        torch = self._torch
        _check(data.dim() >= 3 and data.numel() > 0 and data[0, 0].is_contiguous(), "data has to be [slabs, pages, ...] with dense pages")
        self._int32(refs, "refs", 1), self._int32(tables, "tables", 2), self._int32(lens, "lens", 1)
        _check(refs.numel() == data.shape[1] and lens.numel() == tables.shape[0], "refs has to hold the pages, lens the rows")
        p = self._p = hbf.hbf_pages_t()
        size = data.element_size()
        p.base, p.page_bytes = data.data_ptr(), data[0, 0].numel() * size
        p.n_slabs, p.n_pages, p.page_tokens = data.shape[0], data.shape[1], page_tokens
        p.page_stride = data.stride(1) * size if p.n_pages > 1 else p.page_bytes
        p.slab_stride = data.stride(0) * size if p.n_slabs > 1 else p.page_bytes * p.n_pages
        p.rows, p.table_cols = tables.shape
        p.table_stride = tables.stride(0) if p.rows > 1 else p.table_cols
        p.refs, p.lens, p.tables = refs.data_ptr(), lens.data_ptr(), tables.data_ptr()
        self._keep = (data, refs, tables, lens)
        self._ref = C.byref(p)
        self._ws = self._room(self._lib.hbf_pages_workspace_bytes(self._ref))
        self._ws_ptr, self._ws_bytes = self._ws.data_ptr(), self._ws.numel()
        with torch.cuda.stream(self.stream):
            self._result = torch.zeros(3, dtype=torch.int32, device=self.device)
        self._res_ptr = self._result.data_ptr()
        self._what, self._moves = "", 0

    def _list(self, t, what):
        if t.dtype is not self._i32 or t.dim() != 1 or t.get_device() != self._dev or not t.is_contiguous():
            raise ValueError("%s has to be a contiguous int32 tensor of one dimension on %s" % (what, self.device))
        return t.data_ptr()

    def _done(self, rc, what, moves):
        if rc:                                               # refused here: `result` and `accesses` stay those of the call before
            self._raise(rc, what)
        self._what, self._moves = what, moves

    def copy(self, src, dst):
        """Page src[i]'s bytes to page dst[i], in every slab."""
        n = src.numel()
        _check(dst.numel() == n, "src and dst differ in length")
        self._done(self._lib.hbf_pages_copy(self._ref, self._list(src, "src"), self._list(dst, "dst"), n, self._res_ptr, self._ws_ptr, self._ws_bytes, self._st),
                   "hbf_pages_copy", n)

    def fork(self, parents, children):
        """Row children[i], empty, becomes row parents[i]: full pages shared, a begun one copied."""
        n = parents.numel()
        _check(children.numel() == n, "parents and children differ in length")
        self._done(self._lib.hbf_pages_fork(self._ref, self._list(parents, "parents"), self._list(children, "children"), n, self._res_ptr, self._ws_ptr,
                                            self._ws_bytes, self._st), "hbf_pages_fork", n)

    def free(self, rows):
        """Gives the rows' pages back."""
        self._done(self._lib.hbf_pages_free(self._ref, self._list(rows, "rows"), rows.numel(), self._res_ptr, self._ws_ptr, self._ws_bytes, self._st), "hbf_pages_free", 0)

    def compact(self):
        """Moves the pages in use to the lowest numbers."""
        self._done(self._lib.hbf_pages_compact(self._ref, self._res_ptr, self._ws_ptr, self._ws_bytes, self._st), "hbf_pages_compact", self._p.n_pages // 2)

    def result(self):
        """Waits for the last call: {"moved": pages moved, "in_use": pages in use (compact only)}; HbfError if it was refused."""
        with self._torch.cuda.stream(self.stream):
            code, moved, in_use = self._result.tolist()
        self._raise(code, self._what)
        return {"moved": moved, "in_use": in_use}

    def access_count(self, moved=None):
        _check(moved is None or 0 <= moved <= self._moves, "the last call moves from 0 to %d pages" % self._moves)
        return 2 * (self._moves if moved is None else moved) * self._p.n_slabs

    def accesses(self, issue_ns=0, gap_ns=0, out=None, moved=None):
        """Records of the last call's moves, a read and a program for each page and slab: int64 [n, 3]; n is the most that the call can have
        moved, places past its moves are native.  The most is half of all pages for a compaction, however few moved: with moved, which
        ``result`` tells, there are as many records as that many pages make."""
        n = self.access_count(moved)
        out = self._records(n, out)
        self._raise(self._lib.hbf_pages_accesses(self._ref, self._ws_ptr, issue_ns, gap_ns, out.data_ptr(), n, self._st) if n else 0, "hbf_pages_accesses")
        return out


class ServedLayer:
    """One layer of the model that the streams ``decode_weights`` and ``prefix_kv`` stand for (``workloads``), executed: its experts and its
    key/value cache lie in ranges registered with a context, and every step serves the accesses that its operators make.

    Row 0 of the cache holds the shared prefix; the requests, rows 1 to batch, are forked from it, so that they share its full pages and
    begin with a copy of a page that it had begun; each then has room for own_tokens more, on pages that ``append`` takes as it comes to them.
    A page in use is thus always one that some row's length counts, as ``cache`` (a ``CachePages``) has it: requests may be freed through it,
    begin again as a fork of row 0 or of another request, and the cache may be compacted, in any order.  Row 0 stays: attention reads the prefix by its
    table.  Values are random (seed).  All of it runs on the context's stream; tensors of another stream are the caller's to order before it."""

    def __init__(self, ctx, batch=64, prefix_tokens=8192, own_tokens=64, page_tokens=16, hidden=2048, inter=768, n_experts=128, top_k=8, q_heads=32,
                 kv_heads=4, head_dim=128, seed=0):
        import torch
        self.ctx, self.batch, self.page = ctx, batch, page_tokens
        with torch.cuda.stream(ctx.stream):
            dev = torch.device("cuda", torch.cuda.current_device())
            g = torch.Generator(device=dev)
            g.manual_seed(seed)
            rnd = lambda *s: torch.randn(*s, device=dev, dtype=torch.bfloat16, generator=g)
            self.experts = rnd(n_experts, 3 * inter * hidden) * hidden ** -0.5
            full, started = divmod(prefix_tokens, page_tokens)
            mine = -(-(started + own_tokens) // page_tokens)      # pages of a request behind the full ones that it shares
            held = full + (1 if started else 0)
            pages = max(held + batch * mine, 1) + 1           # (the last is nobody's: see `append`)
            self.kv = rnd(2, pages, page_tokens, kv_heads, head_dim)
            i32 = lambda *s: torch.full(s, -1, dtype=torch.int32, device=dev)
            self.refs, self.lens, self.tables = i32(pages).fill_(0), i32(batch + 1).fill_(0), i32(batch + 1, full + mine + 1)
            self.tables[0, :held] = torch.arange(held, device=dev, dtype=torch.int32)
            self.refs[:held] = 1
            self.lens[0] = prefix_tokens
            self.own_len = torch.zeros(batch, dtype=torch.int32, device=dev)
            self._rows = torch.arange(1, batch + 1, device=dev, dtype=torch.int32)
            self._pages = torch.arange(pages - 1, device=dev)
            parents = torch.zeros_like(self._rows)
        self.cache = CachePages(self.kv[:, :-1], self.refs[:-1], self.tables, self.lens, page_tokens, stream=ctx.stream)
        self.cache.fork(parents, self._rows)
        self.cache.result()
        self.prefix_tokens, self.base_tokens = prefix_tokens, full * page_tokens
        self.attention = PrefixAttention(self.kv[0], self.kv[1], batch, q_heads, self.tables[0, :full] if full else None, self.base_tokens,
                                         self.tables[1:, full:], self.own_len, mine * page_tokens, stream=ctx.stream)
        self.moe = MoeLayer(self.experts, hidden, inter, top_k, batch, stream=ctx.stream)
        offset = 0
        for t in (self.experts, self.kv):                         # one range each, side by side on the media
            ctx.register_range(t.data_ptr(), t.numel() * t.element_size(), 3, 0, 0, offset)
            offset += -(-t.numel() * t.element_size() // (1 << 20)) << 20

    def append(self, k, v):
        """Every request's next token: k, v [batch, kv_heads, head_dim] go into its cache; a request whose pages are full takes the lowest free one, in
        the order of the requests.  A request that has no place for it stays as it is: its room is used up, no page is free, or its row was freed
        (holds less than the prefix; without a prefix an empty row is a request without tokens).  Returns who took it, bool [batch], on the
        device."""
        import torch
        want, dev = (self.batch,) + tuple(self.kv.shape[3:]), self.kv.device
        _check(all(tuple(t.shape) == want and t.dtype == self.kv.dtype and t.device == dev for t in (k, v)), "k and v have to be %s %s on %s" % (self.kv.dtype, want, dev))
        with torch.cuda.stream(self.ctx.stream):
            rows, lens, nobody = self.tables[1:], self.lens[1:], self.kv.shape[1] - 1
            last = self.tables.shape[1] - 1                       # (an entry of -1, past the room)
            col, at = (lens // self.page).long(), (lens % self.page).long()
            fits = (lens >= self.prefix_tokens) & (col < last)
            col.clamp_(min=0, max=last)
            # the n-th request that begins a page takes the n-th free one
            begins = fits & (at == 0)
            free = self.refs[:-1] == 0
            nth = torch.where(free, free.cumsum(0) - 1, self.batch).clamp_(max=self.batch)
            lowest = torch.full((self.batch + 1,), -1, dtype=torch.int64, device=nth.device).scatter_(0, nth, self._pages)
            lowest[self.batch] = -1                               # (where all that are not asked for ended)
            taken = torch.where(begins, lowest[(begins.cumsum(0) - 1).clamp_(min=0)], -1)
            page = torch.where(begins, taken, rows.gather(1, col[:, None])[:, 0].long())
            took = fits & (page >= 0) & (page < nobody)
            place = torch.where(took, page, nobody)
            self.kv[0, place, at], self.kv[1, place, at] = k, v
            rows.scatter_(1, col[:, None], torch.where(took, page, rows.gather(1, col[:, None])[:, 0].long()).int()[:, None])
            self.refs.index_add_(0, place, (begins & took).int())
            lens += took
        return took

    def step(self, q, x, scores, issue_ns=0, gap_ns=0):
        """Attention of the requests' queries q [batch, q_heads, head_dim], then the experts on x [batch, hidden] by the router's scores [batch,
        n_experts].  Returns (attention's output, experts' output, [what ``Context.serve`` returns for each]).  A request whose row holds no token
        (it was freed, or has none yet) attends to nothing: zeros."""
        import torch
        with torch.cuda.stream(self.ctx.stream):
            torch.sub(self.lens[1:], self.base_tokens, out=self.own_len)
            o = self.attention(q)
            o.masked_fill_((self.lens[1:] == 0)[:, None, None], 0.0)      # (of a length below the prefix's shared pages `attention` makes NaN)
        a = self.ctx.serve(self.attention, issue_ns, gap_ns)
        y = self.moe(x, scores)
        b = self.ctx.serve(self.moe, issue_ns + gap_ns * a[0].shape[0], gap_ns)
        return o, y, [a, b]
