// The pages of a key/value cache: copying, forking, freeing and compacting them, as a serving loop does between its steps.
//
// State, all the caller's, in device memory: refs[page] (rows that hold the page; 0 = free), lens[row] (tokens) and tables[row][j] (page
// of the tokens from j * page_tokens on; the first ceil(len / page_tokens) entries count).  A call is two kernels: a plan by one
// block, which looks at everything that the call depends on and works out the pages that move, and one over the whole device that does it;
// where the plan finds a fault, the second does nothing; what a block does in no more time than another launch takes, the plan's block does.
// Which page goes where follows from the state alone (the lowest free
// page first), so that the same calls give the same cache.  Bytes bound the moves (each page read once and written once); small calls
// cost two launches.
#include "tensor_ops.cuh"

namespace hbf {

constexpr int kPlanThreads = 1024, kMoveThreads = 256;

enum { kDoCopy = 0, kDoFork = 1, kDoFree = 2, kDoCompact = 3 };

struct PagesCtrl { int32_t code, moves, n_live; };   // the first words of the workspace

struct PagesDev {
    unsigned char *base; uint64_t page_bytes, page_stride, slab_stride;
    uint32_t n_slabs, n_pages, page_tokens, rows, cols, most; int64_t table_stride;      // most: moves that the workspace has places for
    int32_t *refs, *lens, *tables, *result;
    PagesCtrl *ctrl; int32_t *src, *dst, *extra;             // moves; for a fork the rows' lengths and new pages, for a compaction the pages' new numbers
    Div32 div_slabs;
};

__device__ __forceinline__ uint32_t held_pages(const PagesDev &p, int32_t len) { return ((uint32_t)len + p.page_tokens - 1u) / p.page_tokens; }

__device__ __forceinline__ bool len_bad(const PagesDev &p, int32_t len) { return len < 0 || (uint64_t)len > (uint64_t)p.cols * p.page_tokens; }

// exclusive sum over the block of one number a thread; the total for all
__device__ uint32_t block_scan(uint32_t v, uint32_t *total, uint32_t *warps) {
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= (uint32_t)o) s += u; }
    __syncthreads();
    if (lane == 31u) warps[warp] = s;
    __syncthreads();
    if (warp == 0u) {
        uint32_t w = warps[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, w, o); if (lane >= (uint32_t)o) w += u; }
        warps[lane] = w;
    }
    __syncthreads();
    *total = warps[31];
    return s - v + (warp ? warps[warp - 1u] : 0u);
}

// Every thread of the plan's block ends with this; with `alone` the block goes on with what the other kernel would do.
template <int kDo, uint32_t kThreads> __device__ __forceinline__ void apply_plan(const PagesDev &p, const int32_t *a, const int32_t *b, uint32_t n);
template <int kDo>
__device__ __forceinline__ void finish_plan(const PagesDev &p, int code, uint32_t moves, uint32_t n_live, const int32_t *a, const int32_t *b, uint32_t n, int alone) {
    if (threadIdx.x == 0) {
        const int32_t m = code == HBF_OK ? (int32_t)moves : 0;
        p.ctrl->code = code; p.ctrl->moves = m; p.ctrl->n_live = (int32_t)n_live;
        if (p.result) { p.result[0] = code; p.result[1] = m; p.result[2] = (int32_t)n_live; }
    }
    if (!alone) return;
    __syncthreads();                                         // (the moves that other threads wrote are there, too)
    apply_plan<kDo, kPlanThreads>(p, a, b, n);
}


// What the plan found: the rows' tables and the references, then the pages' bytes.  (Bulk copies through shared memory were no faster, and much
// slower for small pages: 48 slabs, pages of 4 KB 185 us against 105, of 16 KB 141 against 135.)
template <int kDo, uint32_t kThreads>
__device__ __forceinline__ void apply_plan(const PagesDev &p, const int32_t *a, const int32_t *b, uint32_t n) {
    const PagesCtrl c = *p.ctrl;
    if (c.code != HBF_OK) return;
    const uint32_t moves = (uint32_t)c.moves;
    const uint64_t step = (uint64_t)gridDim.x * kThreads, first = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
    if (kDo == kDoFork || kDo == kDoFree) {
        for (uint64_t k = first; k < (uint64_t)n * p.cols; k += step) {
            const uint32_t i = (uint32_t)(k / p.cols), j = (uint32_t)(k - (uint64_t)i * p.cols);
            const int32_t len = p.extra[i];
            int32_t entry = -1;
            if (kDo == kDoFork) {
                const uint32_t full = (uint32_t)len / p.page_tokens;
                if (j < full) {
                    entry = p.tables[(int64_t)a[i] * p.table_stride + j];
                    atomicAdd(&p.refs[entry], 1);
                } else if (j == full && (uint32_t)len % p.page_tokens) {
                    entry = p.dst[p.extra[n + i]];
                    p.refs[entry] = 1;
                }
                p.tables[(int64_t)b[i] * p.table_stride + j] = entry;
                if (j == 0u) p.lens[b[i]] = len;
            } else {
                int32_t *t = p.tables + (int64_t)a[i] * p.table_stride + j;
                if (j < held_pages(p, len)) atomicAdd(&p.refs[*t], -1);
                *t = -1;
                if (j == 0u) p.lens[a[i]] = 0;
            }
        }
    }
    if (kDo == kDoCompact) {
        const uint32_t live = (uint32_t)c.n_live;
        for (uint64_t k = first; k < (uint64_t)p.rows * p.cols; k += step) {
            const uint32_t i = (uint32_t)(k / p.cols), j = (uint32_t)(k - (uint64_t)i * p.cols);
            if (j >= held_pages(p, p.lens[i])) continue;
            int32_t *t = p.tables + (int64_t)i * p.table_stride + j;
            const uint32_t id = (uint32_t)*t;
            if (id >= live) *t = p.extra[id];                // (the plan has seen that it is a page in use: one that moves)
        }
        for (uint64_t k = first; k < moves; k += step) { p.refs[p.dst[k]] = p.refs[p.src[k]]; p.refs[p.src[k]] = 0; }
    }
    if (kThreads == (uint32_t)kPlanThreads) {                // the plan's block by itself: 16 bytes a thread of all that moves
        const uint32_t n16 = (uint32_t)(p.page_bytes / 16u), all = moves * p.n_slabs * n16;
#pragma unroll 4
        for (uint32_t i = threadIdx.x; i < all; i += kThreads) {
            const uint32_t u = i / n16, k = div32(u, p.div_slabs);
            const uint64_t at = (uint64_t)(u - k * p.n_slabs) * p.slab_stride + (uint64_t)(i - u * n16) * 16u;
            const uint4 v = *reinterpret_cast<const uint4 *>(p.base + at + (uint64_t)p.src[k] * p.page_stride);
            *reinterpret_cast<uint4 *>(p.base + at + (uint64_t)p.dst[k] * p.page_stride) = v;
        }
        return;
    }
    // a warp a piece of up to 16 KB, 4 KB of it on its way at once, a page in equal pieces
    const uint32_t n16 = (uint32_t)(p.page_bytes / 16u), per = (n16 + 1023u) / 1024u, piece = (n16 + per - 1u) / per, lane = lane_id();
    const uint64_t units = (uint64_t)moves * p.n_slabs * per;
    for (uint64_t q = (uint64_t)blockIdx.x * (kThreads / 32u) + (threadIdx.x >> 5); q < units; q += (uint64_t)gridDim.x * (kThreads / 32u)) {
        const uint32_t u = (uint32_t)(q / per), first = (uint32_t)(q - (uint64_t)u * per) * piece, last = min(first + piece, n16);
        const uint32_t k = div32(u, p.div_slabs);
        const uint64_t slab = (uint64_t)(u - k * p.n_slabs) * p.slab_stride;
        const unsigned char *from = p.base + slab + (uint64_t)p.src[k] * p.page_stride;
        unsigned char *to = p.base + slab + (uint64_t)p.dst[k] * p.page_stride;
        for (uint32_t i0 = first + lane; i0 < last; i0 += 256u) {
            uint4 v[8];
#pragma unroll
            for (uint32_t e = 0; e < 8u; ++e) {
                const uint32_t i = i0 + e * 32u;
                if (i < last) asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v[e].x), "=r"(v[e].y), "=r"(v[e].z), "=r"(v[e].w) : "l"(from + (uint64_t)i * 16u));
            }
#pragma unroll
            for (uint32_t e = 0; e < 8u; ++e) {
                const uint32_t i = i0 + e * 32u;
                if (i < last) *reinterpret_cast<uint4 *>(to + (uint64_t)i * 16u) = v[e];
            }
        }
    }
}

template <int kDo>
__global__ void __launch_bounds__(kMoveThreads)
k_pages_apply(const __grid_constant__ PagesDev p, const int32_t *a, const int32_t *b, uint32_t n) {
    pdl_wait();
    apply_plan<kDo, kMoveThreads>(p, a, b, n);
}

// The listed pairs are sound if every page exists, no destination is named twice and none is a source too (their order would count).
__global__ void __launch_bounds__(kPlanThreads)
k_plan_copy(const __grid_constant__ PagesDev p, const int32_t *src, const int32_t *dst, uint32_t n, int alone) {
    extern __shared__ uint32_t bits[];
    pdl_trigger();
    const uint32_t words = (p.n_pages + 31u) / 32u;
    for (uint32_t i = threadIdx.x; i < words; i += kPlanThreads) bits[i] = 0u;
    int bad = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const uint32_t d = (uint32_t)dst[i];
        if (d >= p.n_pages || (atomicOr(&bits[d >> 5], 1u << (d & 31u)) >> (d & 31u)) & 1u) bad = 1;
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const uint32_t s = (uint32_t)src[i];
        if (s >= p.n_pages || (bits[s >> 5] >> (s & 31u)) & 1u) bad = 1;
        p.src[i] = (int32_t)s; p.dst[i] = dst[i];
    }
    bad = __syncthreads_or(bad);
    finish_plan<kDoCopy>(p, bad ? HBF_E_INVAL : HBF_OK, n, 0u, src, dst, n, alone);
}

// A row's entries that count name pages in use.
__device__ __forceinline__ int row_bad(const PagesDev &p, uint32_t row, int32_t len, uint32_t from, uint32_t step) {
    int bad = 0;
    const int32_t *t = p.tables + (int64_t)row * p.table_stride;
    const uint32_t held = held_pages(p, len);
#pragma unroll 4
    for (uint32_t j = from; j < held; j += step) {
        const uint32_t id = (uint32_t)t[j];
        if (id >= p.n_pages || p.refs[id] <= 0) bad = 1;
    }
    return bad;
}

// Rows that begin as other rows' tokens: full pages are shared, a begun page is copied into the lowest free one, in the order of the list.
__global__ void __launch_bounds__(kPlanThreads)
k_plan_fork(const __grid_constant__ PagesDev p, const int32_t *parents, const int32_t *children, uint32_t n, int alone) {
    extern __shared__ uint32_t bits[];                       // rows named as children
    __shared__ uint32_t warps[32];
    __shared__ int s_bad;
    pdl_trigger();
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = lane_id();
    const bool free0 = tid < p.n_pages && p.refs[tid] == 0;  // (asked for now: what the pages' search begins with)
    for (uint32_t i = tid; i < (p.rows + 31u) / 32u; i += kPlanThreads) bits[i] = 0u;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    // The rows of the list: their lengths; the begun pages, in the order of the list; where another parent than the one before it begins (in
    // p.dst for now).  One scan for both counts.
    int bad = 0;
    uint32_t need = 0u, runs = 0u;
    for (uint32_t i0 = 0; i0 < n; i0 += kPlanThreads) {
        const uint32_t i = i0 + tid;
        uint32_t begun = 0u, run = 0u;
        int32_t from = 0;
        if (i < n) {
            const uint32_t a = (uint32_t)parents[i], c = (uint32_t)children[i], before = i ? (uint32_t)parents[i - 1u] : ~a;
            const int32_t len = a < p.rows ? p.lens[a] : -1;
            if (a >= p.rows || c >= p.rows || len_bad(p, len) || p.lens[c] != 0) bad = 1;
            else if ((atomicOr(&bits[c >> 5], 1u << (c & 31u)) >> (c & 31u)) & 1u) bad = 1;
            else {
                p.extra[i] = len;
                run = a != before ? 1u : 0u;
                begun = (uint32_t)len % p.page_tokens ? 1u : 0u;
                if (begun) from = p.tables[(int64_t)a * p.table_stride + (uint32_t)len / p.page_tokens];
            }
        }
        uint32_t total;
        const uint32_t at = block_scan(run << 16 | begun, &total, warps);
        if (run) p.dst[runs + (at >> 16)] = (int32_t)i;
        if (begun) { p.src[need + (at & 0xffffu)] = from; p.extra[n + i] = (int32_t)(need + (at & 0xffffu)); }
        need += total & 0xffffu; runs += total >> 16;
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (s_bad) { finish_plan<kDoFork>(p, HBF_E_INVAL, 0u, 0u, parents, children, n, 0); return; }
    // the parents' pages, a parent named several times in a row once: few parents by the whole block, many by a warp each
    const bool wide = runs <= 4u;
    for (uint32_t k = wide ? 0u : warp; k < runs; k += wide ? 1u : kPlanThreads / 32) {
        const uint32_t i = (uint32_t)p.dst[k];
        bad |= row_bad(p, (uint32_t)parents[i], p.extra[i], wide ? tid : lane, wide ? kPlanThreads : 32u);
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (s_bad) { finish_plan<kDoFork>(p, HBF_E_INVAL, 0u, 0u, parents, children, n, 0); return; }
    // as many free pages, the lowest
    uint32_t found = 0u;
    for (uint32_t i0 = 0; i0 < p.n_pages && found < need; i0 += kPlanThreads) {
        const uint32_t i = i0 + tid;
        const bool free = i0 ? i < p.n_pages && p.refs[i] == 0 : free0;
        const unsigned b = __ballot_sync(0xffffffffu, free);
        if (lane == 0u) warps[warp] = __popc(b);
        __syncthreads();
        const uint32_t all = warps[lane];
        uint32_t s = all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, s, o); if (lane >= (uint32_t)o) s += u; }
        const uint32_t at = found + __shfl_sync(0xffffffffu, s - all, warp) + __popc(b & lanemask_lt());
        if (free && at < need) p.dst[at] = (int32_t)i;
        found += __shfl_sync(0xffffffffu, s, 31);
        __syncthreads();
    }
    finish_plan<kDoFork>(p, found < need ? HBF_E_CAPACITY : HBF_OK, need, 0u, parents, children, n, alone);
}

__global__ void __launch_bounds__(kPlanThreads)
k_plan_free(const __grid_constant__ PagesDev p, const int32_t *rows, uint32_t n, int alone) {
    extern __shared__ uint32_t bits[];
    __shared__ int s_bad;
    pdl_trigger();
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = lane_id();
    for (uint32_t i = tid; i < (p.rows + 31u) / 32u; i += kPlanThreads) bits[i] = 0u;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    int bad = 0;
    for (uint32_t i = tid; i < n; i += kPlanThreads) {
        const uint32_t r = (uint32_t)rows[i];
        if (r >= p.rows || len_bad(p, p.lens[r])) bad = 1;
        else if ((atomicOr(&bits[r >> 5], 1u << (r & 31u)) >> (r & 31u)) & 1u) bad = 1;
        else p.extra[i] = p.lens[r];
    }
    if (bad) s_bad = 1;
    __syncthreads();
    if (!s_bad)
        for (uint32_t i = warp; i < n; i += kPlanThreads / 32)
            if (row_bad(p, (uint32_t)rows[i], p.extra[i], lane, 32u)) s_bad = 1;
    __syncthreads();
    finish_plan<kDoFree>(p, s_bad ? HBF_E_INVAL : HBF_OK, 0u, 0u, rows, nullptr, n, alone);
}

// Whether any row of the cache has a length or a counting entry that cannot be.  A warp takes up to 32 rows, an even share of them, and their
// entries one behind the other (at most 2^29, table_cols being 2^24 at most), an entry a lane, so that the loads of short rows are on their way together.
__device__ __forceinline__ int rows_bad(const PagesDev &p) {
    const uint32_t lane = lane_id(), share = min(32u, (p.rows + kPlanThreads / 32u - 1u) / (kPlanThreads / 32u));
    int bad = 0;
    for (uint32_t r0 = (threadIdx.x >> 5) * share; r0 < p.rows; r0 += kPlanThreads / 32u * share) {
        const int32_t len = lane < share && r0 + lane < p.rows ? p.lens[r0 + lane] : 0;
        const bool sound = !len_bad(p, len);
        if (!sound) bad = 1;
        const uint32_t held = sound ? held_pages(p, len) : 0u;
        uint32_t end = held;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const uint32_t u = __shfl_up_sync(0xffffffffu, end, o); if (lane >= (uint32_t)o) end += u; }
        const uint32_t first = end - held, total = __shfl_sync(0xffffffffu, end, 31);
#pragma unroll 4
        for (uint32_t e0 = 0; e0 < total; e0 += 32u) {
            const uint32_t e = e0 + lane;
            uint32_t at = 0u;                                // the last row whose entries begin no later than e
#pragma unroll
            for (uint32_t o = 16; o > 0u; o >>= 1) if (__shfl_sync(0xffffffffu, first, at + o) <= e) at += o;
            const uint32_t j = e - __shfl_sync(0xffffffffu, first, at);
            if (e < total) {
                const uint32_t id = (uint32_t)p.tables[(int64_t)(r0 + at) * p.table_stride + j];
                if (id >= p.n_pages || p.refs[id] <= 0) bad = 1;
            }
        }
    }
    return bad;
}

// The k-th page in use behind the first n_live moves into the k-th free one among them.
__global__ void __launch_bounds__(kPlanThreads)
k_plan_compact(const __grid_constant__ PagesDev p, int alone) {
    extern __shared__ uint32_t bits[];                       // pages in use
    __shared__ uint32_t warps[32];
    pdl_trigger();
    const uint32_t tid = threadIdx.x, lane = lane_id(), words = (p.n_pages + 31u) / 32u;
    const int bad = rows_bad(p);
    uint32_t mine = 0u;
    for (uint32_t w = tid >> 5; w < words; w += kPlanThreads / 32) {
        const uint32_t i = w * 32u + lane;
        const unsigned b = __ballot_sync(0xffffffffu, i < p.n_pages && p.refs[i] > 0);
        if (lane == 0u) { bits[w] = b; mine += __popc(b); }
    }
    uint32_t live;
    block_scan(mine, &live, warps);                          // (its barriers also publish the bits)
    const uint32_t each = (words + kPlanThreads - 1u) / kPlanThreads, w0 = min(words, tid * each), w1 = min(words, w0 + each);
    uint32_t holes = 0u, movers = 0u;
    auto below = [&](uint32_t w) { return w * 32u >= live ? 0u : live - w * 32u >= 32u ? 0xffffffffu : (1u << (live - w * 32u)) - 1u; };
    for (uint32_t w = w0; w < w1; ++w) { holes += __popc(~bits[w] & below(w)); movers += __popc(bits[w] & ~below(w)); }
    uint32_t total, moves;
    uint32_t h = block_scan(holes, &total, warps), m = block_scan(movers, &moves, warps);
    for (uint32_t w = w0; w < w1; ++w) {
        for (uint32_t b = ~bits[w] & below(w); b; b &= b - 1u) p.dst[h++] = (int32_t)(w * 32u + __ffs(b) - 1u);
        for (uint32_t b = bits[w] & ~below(w); b; b &= b - 1u) p.src[m++] = (int32_t)(w * 32u + __ffs(b) - 1u);
    }
    __syncthreads();
    for (uint32_t i = live + tid; i < p.n_pages; i += kPlanThreads) p.extra[i] = -1;
    __syncthreads();
    for (uint32_t k = tid; k < moves; k += kPlanThreads) p.extra[p.src[k]] = p.dst[k];
    const int any = __syncthreads_or(bad);
    finish_plan<kDoCompact>(p, any ? HBF_E_INVAL : HBF_OK, moves, live, nullptr, nullptr, 0u, alone);
}

// The records of the moves of the call before: for each page and slab a read and a program; the places behind them hold records of one byte
// at address 0, outside every range.
__global__ void __launch_bounds__(kMoveThreads)
k_pages_accesses(const __grid_constant__ PagesDev p, int64_t issue_ns, int64_t gap_ns, hbf_access_t *acc, uint64_t n) {
    const uint64_t moves = p.ctrl->code == HBF_OK ? min((uint32_t)p.ctrl->moves, p.most) : 0u;          // (whatever lies there)
    for (uint64_t i = (uint64_t)blockIdx.x * kMoveThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kMoveThreads) {
        hbf_access_t v = {0, issue_ns + (int64_t)i * gap_ns, 1, 0};
        const uint64_t u = i >> 1;
        if (u < moves * p.n_slabs) {
            const uint64_t k = u / p.n_slabs, s = u - k * p.n_slabs;
            v.addr = (uint64_t)(uintptr_t)p.base + s * p.slab_stride + (uint64_t)(i & 1u ? p.dst[k] : p.src[k]) * p.page_stride;
            v.bytes = (uint32_t)p.page_bytes; v.flags = (uint32_t)(i & 1u);
        }
        acc[i] = v;
    }
}

static bool pages_ok(const hbf_pages_t *p) {
    if (!p || !p->base || (uintptr_t)p->base % 16 || p->page_bytes == 0 || p->page_bytes % 16 || p->page_bytes > 0xfffffff0ull) return false;
    if (p->page_stride % 16 || p->slab_stride % 16 || p->page_stride < p->page_bytes || p->n_slabs == 0 || p->n_slabs > 65536u) return false;
    if (p->n_pages == 0 || p->n_pages > HBF_MAX_CACHE_PAGES || p->rows > HBF_MAX_CACHE_PAGES || p->page_tokens == 0 || p->page_tokens > (1u << 20)) return false;
    if ((uint64_t)p->n_pages * p->n_slabs > (1ull << 30)) return false;
    // pages of one slab behind one another, or slabs inside a page's stretch: no two pages overlap
    const uint64_t slab = (uint64_t)(p->n_pages - 1) * p->page_stride + p->page_bytes, page = (uint64_t)(p->n_slabs - 1) * p->slab_stride + p->page_bytes;
    if (p->n_slabs > 1 && p->slab_stride < slab && !(p->slab_stride >= p->page_bytes && p->page_stride >= page)) return false;
    return true;
}
static bool pages_state_ok(const hbf_pages_t *p) {
    if (!p->refs || (uintptr_t)p->refs % 4) return false;
    if (p->rows == 0) return true;
    return p->lens && p->tables && (uintptr_t)p->lens % 4 == 0 && (uintptr_t)p->tables % 4 == 0 && p->table_cols && p->table_cols <= (1u << 24) && p->table_stride >= (int64_t)p->table_cols
        && (uint64_t)p->table_cols * p->page_tokens < (1ull << 31);
}
static size_t pages_bytes(const hbf_pages_t *p) {            // control words, moves, and per page or row (twice, for a fork's lengths and places)
    const size_t most = p->n_pages > p->rows ? p->n_pages : p->rows;
    return (256u + most * 4u * 4u + 255u) / 256u * 256u;
}
static PagesDev pages_dev(const hbf_pages_t *p, void *ws, int32_t *result) {
    PagesDev d = {};
    d.base = static_cast<unsigned char *>(p->base); d.page_bytes = p->page_bytes; d.page_stride = p->page_stride; d.slab_stride = p->slab_stride;
    d.n_slabs = p->n_slabs; d.n_pages = p->n_pages; d.page_tokens = p->page_tokens; d.rows = p->rows; d.cols = p->rows ? p->table_cols : 0u; d.table_stride = p->table_stride;
    d.refs = p->refs; d.lens = p->lens; d.tables = p->tables; d.result = result;
    const size_t most = p->n_pages > p->rows ? p->n_pages : p->rows;
    d.most = (uint32_t)most; d.ctrl = static_cast<PagesCtrl *>(ws);
    d.src = reinterpret_cast<int32_t *>(static_cast<unsigned char *>(ws) + 256); d.dst = d.src + most; d.extra = d.dst + most;
    d.div_slabs = make_div32(p->n_slabs);
    return d;
}

// the checks that all four calls share, the plan's launch and the apply kernel's
template <int kDo, class Plan, class... Args>
static int pages_call(const hbf_pages_t *p, const int32_t *a, const int32_t *b, uint32_t n, uint64_t work, uint64_t most_moves, uint64_t entries, uint32_t mark_bits, int32_t *result, void *ws, size_t ws_bytes,
                      void *stream, Plan plan, const Args &...args) {
    if ((uintptr_t)result % 4) return HBF_E_INVAL;
    if (!ws || (uintptr_t)ws % 256 || ws_bytes < pages_bytes(p)) return HBF_E_WORKSPACE;
    uint32_t n_sm = 0;
    const int rc = device_of(p->base, &n_sm);
    if (rc != HBF_OK) return rc;
    const PagesDev d = pages_dev(p, ws, result);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t smem = ((size_t)mark_bits + 31u) / 32u * 4u;
    if (ensure_dyn_smem((const void *)plan, smem + 1024u) != cudaSuccess) return HBF_E_CUDA;          // (with what the plans hold besides)
    // One block alone while it is done about when a second kernel would begin.  A copy alone and with one: 32 KB 3.3 and 4.5 us, 64 KB 4.1 and 4.6,
    // 80 KB 4.6 and 4.6, 128 KB 5.6 and 4.6; rows freed: 1,024 entries 3.3 and 3.8, 2,048 3.8 and 3.9, 4,096 4.8 and 3.9, 32,768 18.4 and 4.2 (in a
    // graph; launched one by one 64 KB take 6.2 and 10.1).
    const int alone = most_moves * p->n_slabs * p->page_bytes <= 64u * 1024u && entries <= 2u * kPlanThreads;
    plan<<<1, kPlanThreads, smem, st>>>(d, args..., alone);
    if (cudaGetLastError() != cudaSuccess) return HBF_E_CUDA;
    if (alone) { g_kernel_launches += 1; return HBF_OK; }
    const uint64_t blocks = work < 1 ? 1 : work < 8ull * n_sm ? work : 8ull * n_sm;
    g_kernel_launches += 2;
    return launch_pdl(k_pages_apply<kDo>, (unsigned)blocks, kMoveThreads, 0, st, d, a, b, n) == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}

}  // namespace hbf

using namespace hbf;

extern "C" size_t hbf_pages_workspace_bytes(const hbf_pages_t *p) { return pages_ok(p) ? pages_bytes(p) : 0; }

extern "C" int hbf_pages_copy(const hbf_pages_t *p, const int32_t *d_src, const int32_t *d_dst, uint32_t n, int32_t *d_result, void *d_workspace,
                              size_t workspace_bytes, void *cuda_stream) {
    if (!pages_ok(p) || n > p->n_pages || (n && (!d_src || !d_dst || (uintptr_t)d_src % 4 || (uintptr_t)d_dst % 4))) return HBF_E_INVAL;
    return pages_call<kDoCopy>(p, d_src, d_dst, n, (uint64_t)n * p->n_slabs, n, 0, p->n_pages, d_result, d_workspace, workspace_bytes, cuda_stream, k_plan_copy, d_src, d_dst, n);
}

extern "C" int hbf_pages_fork(const hbf_pages_t *p, const int32_t *d_parents, const int32_t *d_children, uint32_t n, int32_t *d_result, void *d_workspace,
                              size_t workspace_bytes, void *cuda_stream) {
    if (!pages_ok(p) || !pages_state_ok(p) || n > p->rows || (n && (!d_parents || !d_children || (uintptr_t)d_parents % 4 || (uintptr_t)d_children % 4))) return HBF_E_INVAL;
    const uint64_t work = (uint64_t)n * p->n_slabs + (uint64_t)n * (p->rows ? p->table_cols : 0u) / kMoveThreads;
    return pages_call<kDoFork>(p, d_parents, d_children, n, work, n, (uint64_t)n * (p->rows ? p->table_cols : 0u), p->rows, d_result, d_workspace, workspace_bytes, cuda_stream, k_plan_fork, d_parents, d_children, n);
}

extern "C" int hbf_pages_free(const hbf_pages_t *p, const int32_t *d_rows, uint32_t n, int32_t *d_result, void *d_workspace, size_t workspace_bytes,
                              void *cuda_stream) {
    if (!pages_ok(p) || !pages_state_ok(p) || n > p->rows || (n && (!d_rows || (uintptr_t)d_rows % 4))) return HBF_E_INVAL;
    const uint64_t work = ((uint64_t)n * (p->rows ? p->table_cols : 0u) + kMoveThreads - 1) / kMoveThreads;
    return pages_call<kDoFree>(p, d_rows, nullptr, n, work, 0, (uint64_t)n * (p->rows ? p->table_cols : 0u), p->rows, d_result, d_workspace, workspace_bytes, cuda_stream, k_plan_free, d_rows, n);
}

extern "C" int hbf_pages_compact(const hbf_pages_t *p, int32_t *d_result, void *d_workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!pages_ok(p) || !pages_state_ok(p)) return HBF_E_INVAL;
    return pages_call<kDoCompact>(p, nullptr, nullptr, 0, (uint64_t)p->n_pages * p->n_slabs, p->n_pages / 2, (uint64_t)p->rows * (p->rows ? p->table_cols : 0u), p->n_pages, d_result, d_workspace, workspace_bytes, cuda_stream, k_plan_compact);
}

extern "C" int hbf_pages_accesses(const hbf_pages_t *p, const void *d_workspace, int64_t issue_ns, int64_t gap_ns, hbf_access_t *d_acc, uint64_t n, void *cuda_stream) {
    if (!pages_ok(p) || !d_workspace || (uintptr_t)d_workspace % 256 || issue_ns < 0 || gap_ns < 0 || n > HBF_MAX_BATCH || (n && (!d_acc || (uintptr_t)d_acc % 8))) return HBF_E_INVAL;
    if (n == 0) return HBF_OK;
    uint32_t n_sm = 0;
    const int rc = device_of(p->base, &n_sm);
    if (rc != HBF_OK) return rc;
    const uint64_t blocks = (n + kMoveThreads - 1) / kMoveThreads;
    k_pages_accesses<<<(unsigned)(blocks < 8u * n_sm ? blocks : 8u * n_sm), kMoveThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        pages_dev(p, const_cast<void *>(d_workspace), nullptr), issue_ns, gap_ns, d_acc, n);
    g_kernel_launches += 1;
    return cudaGetLastError() == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}
