// A mixture-of-experts layer for a few tokens in two kernels.
//
//   choice      the top_k largest of a token's scores, ties to the lowest expert; weights w = softmax over the chosen (or over all)
//   k_moe_up    h[pair] = w * silu(gate x) * (up x)             for every (expert, token that chose it) pair
//   k_moe_down  out[token] = sum over its experts of down h
//
// Bytes bound it: an expert's 6 * inter * hidden bytes are read once, whatever the number of its tokens (a few).  So the weights go
// from HBM past L1 into rings of shared memory and from there, as they lie, into the A operand of m16n8k16 products whose
// columns are tokens; no tile is ever padded to more than 8 tokens.  The order in which a product sums its 16-wide steps is free, so
// every lane takes 16 consecutive bytes of its row (two steps' worth) from weights and activations alike, and reads back
// only what it copied itself: no transposition, no barrier in the stream.
#include "tensor_ops.cuh"

namespace hbf {

constexpr int kMoeWarps = 16, kMoeThreads = kMoeWarps * 32;
constexpr int kMoeChunk = 32;                                // tokens of one expert that an item of the up kernel takes
constexpr int kUpRing = 5;                                   // 32-wide steps on their way, a warp: 80 KB of weights an SM
constexpr int kDownRing = 8;                                 // 128 KB an SM
constexpr int kUpStep = 1536, kDownStep = 1024;              // bytes a step: 16 rows of weights; 8 rows of activations

struct MoeDev {
    uint32_t T, D, I, E, K, renorm;
    const uint16_t *x; int64_t x_stride;
    const float *scores; int64_t scores_stride;
    const uint16_t *experts; int64_t expert_stride;
    uint16_t *out; int64_t out_stride;
    int32_t *chosen; float *weights;
    uint16_t *h_hi, *h_lo;                                   // [pairs by expert, then token][I]
    uint32_t rows;                                           // of the down product that a block takes, at most 16
    Div32 div_slices, div_steps;                             // ceil(I / 8); ceil(I / 32)
};

// What the choice leaves in shared memory, the same in every block that makes it.
struct Route {
    uint32_t mask[HBF_MOE_MAX_EXPERTS][HBF_MOE_MAX_TOKENS / 32];     // tokens of each expert
    uint16_t base[HBF_MOE_MAX_EXPERTS];                              // pairs of the experts before it
    uint16_t active[HBF_MOE_MAX_EXPERTS];                            // experts in use, ascending
    uint16_t entry[HBF_MOE_MAX_EXPERTS + HBF_MOE_MAX_TOKENS * HBF_MOE_MAX_TOP_K / kMoeChunk];   // expert * 8 + chunk of its tokens
    uint8_t token[HBF_MOE_MAX_TOKENS * HBF_MOE_MAX_TOP_K];           // of each pair
    float weight[HBF_MOE_MAX_TOKENS * HBF_MOE_MAX_TOP_K];
    uint32_t bad[HBF_MOE_MAX_TOKENS / 32];                           // tokens with a NaN among their scores
    uint32_t n_active, n_entries, scan[kMoeWarps][3];
};

__device__ __forceinline__ uint32_t ordered(float f) {              // larger scores, larger keys; -inf (never chosen): 0
    const uint32_t u = __float_as_uint(f + 0.0f);           // (-0 and 0 tie)
    const uint32_t k = u & 0x80000000u ? ~u : u | 0x80000000u;
    return f == -INFINITY ? 0u : k;
}
__device__ __forceinline__ float from_ordered(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
__device__ __forceinline__ float warp_sum_f(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// One token's choice by one warp: lane j < K holds the j-th chosen expert (-1: none left) and its weight.  Sixteen keys a lane at most.
__device__ __forceinline__ bool choose(const MoeDev &m, uint32_t t, int &expert, float &weight) {
    constexpr int kMost = HBF_MOE_MAX_EXPERTS / 32;
    const uint32_t lane = lane_id();
    const float *s = m.scores + (int64_t)t * m.scores_stride;
    uint32_t key[kMost];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        key[i] = 0u;
        if (i * 32u < m.E) {
            const uint32_t e = i * 32u + lane;
            if (e < m.E) { const float f = s[e]; nan |= f != f; key[i] = ordered(f); }
        }
    }
    expert = -1; weight = 0.0f;
    if (__any_sync(0xffffffffu, nan)) return false;
    float all = 0.0f;
    uint32_t mine = 0u, first = 0u;
    for (uint32_t j = 0; j < m.K; ++j) {
        uint32_t best = 0u;
#pragma unroll
        for (int i = 0; i < kMost; ++i) best = max(best, key[i]);
        best = __reduce_max_sync(0xffffffffu, best);
        if (best == 0u) break;
        uint32_t at = 0xffffffffu;
#pragma unroll
        for (int i = kMost - 1; i >= 0; --i) if (key[i] == best) at = i * 32u + lane;
        at = __reduce_min_sync(0xffffffffu, at);
        if (j == 0) {
            first = best;
            if (!m.renorm) {
#pragma unroll
                for (int i = 0; i < kMost; ++i) if (key[i]) all += expf(from_ordered(key[i]) - from_ordered(first));
                all = warp_sum_f(all);
            }
        }
        if (lane == j) { expert = (int)at; mine = best; }
#pragma unroll
        for (int i = 0; i < kMost; ++i) if (i * 32u + lane == at) key[i] = 0u;
    }
    const float p = expert >= 0 ? expf(from_ordered(mine) - from_ordered(first)) : 0.0f;
    if (m.renorm) all = warp_sum_f(p);
    if (expert >= 0) weight = p / all;
    return true;
}

// The whole batch's choice: about 1 us for a token and 16 warps, hidden in the down kernel behind the kernel before it.
__device__ void route(const MoeDev &m, Route &r, bool write) {
    constexpr int kMine = HBF_MOE_MAX_TOKENS / kMoeWarps;
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    for (uint32_t i = tid; i < m.E * 4u; i += kMoeThreads) r.mask[i >> 2][i & 3u] = 0u;
    if (tid < HBF_MOE_MAX_TOKENS / 32) r.bad[tid] = 0u;
    __syncthreads();
    int expert[kMine]; float weight[kMine];
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const uint32_t t = i * kMoeWarps + warp;
        expert[i] = -1; weight[i] = 0.0f;
        if (t < m.T) {
            const bool ok = choose(m, t, expert[i], weight[i]);
            if (!ok && lane == 0) atomicOr(&r.bad[t >> 5], 1u << (t & 31u));
            if (expert[i] >= 0) atomicOr(&r.mask[expert[i]][t >> 5], 1u << (t & 31u));
            if (write && lane < m.K) {
                if (m.chosen) m.chosen[(size_t)t * m.K + lane] = expert[i];
                if (m.weights) m.weights[(size_t)t * m.K + lane] = weight[i];
            }
        }
    }
    __syncthreads();
    // places of the experts in the list of pairs, of those in use, and of the items' entries: one scan over the experts
    uint32_t count = 0u, chunks = 0u;
    if (tid < m.E) {
#pragma unroll
        for (int w = 0; w < HBF_MOE_MAX_TOKENS / 32; ++w) count += __popc(r.mask[tid][w]);
        chunks = (count + kMoeChunk - 1) / kMoeChunk;
    }
    const uint32_t used = count ? 1u : 0u;
    uint32_t a = count, b = used, c = chunks;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t pa = __shfl_up_sync(0xffffffffu, a, o), pb = __shfl_up_sync(0xffffffffu, b, o), pc = __shfl_up_sync(0xffffffffu, c, o);
        if (lane >= (uint32_t)o) { a += pa; b += pb; c += pc; }
    }
    if (lane == 31u) { r.scan[warp][0] = a; r.scan[warp][1] = b; r.scan[warp][2] = c; }
    __syncthreads();
    for (uint32_t w = 0; w < warp; ++w) { a += r.scan[w][0]; b += r.scan[w][1]; c += r.scan[w][2]; }
    if (tid == kMoeThreads - 1) { r.n_active = b; r.n_entries = c; }
    if (tid < m.E) {
        r.base[tid] = (uint16_t)(a - count);
        if (used) {
            r.active[b - 1u] = (uint16_t)tid;
            for (uint32_t k = 0; k < chunks; ++k) r.entry[c - chunks + k] = (uint16_t)(tid * 8u + k);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const uint32_t t = i * kMoeWarps + warp;
        if (expert[i] >= 0) {
            uint32_t at = r.base[expert[i]];
#pragma unroll
            for (int w = 0; w < HBF_MOE_MAX_TOKENS / 32; ++w) {
                const uint32_t below = (uint32_t)w < (t >> 5) ? 0xffffffffu : (uint32_t)w == (t >> 5) ? (1u << (t & 31u)) - 1u : 0u;
                at += __popc(r.mask[expert[i]][w] & below);
            }
            r.token[at] = (uint8_t)t; r.weight[at] = weight[i];
        }
    }
    __syncthreads();
}
static_assert(HBF_MOE_MAX_EXPERTS <= kMoeThreads, "an expert a thread in the scan");
static_assert(HBF_MOE_MAX_TOKENS / kMoeChunk <= 8 && HBF_MOE_MAX_EXPERTS * 8 <= 65536 && HBF_MOE_MAX_TOKENS <= 256, "packed fields");

// Sixteen warps' sums of a 16 x 8 n product, left as they lie in the accumulators: eight lanes for a column of the pile, two warps' parts
// each, always in the same order.  f(tile, lane of the accumulator, its four sums) is called once for every column.
template <class F>
__device__ __forceinline__ void sum_over_warps(const float4 *pile, int tiles, F f) {
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, part = lane >> 2;
    for (uint32_t c0 = warp * 4u; c0 < (uint32_t)tiles * 32u; c0 += kMoeWarps * 4u) {
        const uint32_t col = c0 + (lane & 3u);
        float4 s = pile[(size_t)(part * 2u) * tiles * 32u + col];
        const float4 v = pile[(size_t)(part * 2u + 1u) * tiles * 32u + col];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            s.x += __shfl_xor_sync(0xffffffffu, s.x, o); s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
            s.z += __shfl_xor_sync(0xffffffffu, s.z, o); s.w += __shfl_xor_sync(0xffffffffu, s.w, o);
        }
        if (part == 0u) f(col >> 5, col & 31u, s);
    }
}

// Items of eight gate rows and the same eight up rows (rows 0..7 and 8..15 of one product, so a thread's sums hold both), one item a
// block at a time, the sum over `hidden` split among its warps; the ring runs on into the next item while an item's sums are joined.
template <class Ty>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_up(const __grid_constant__ MoeDev m) {
    extern __shared__ __align__(128) unsigned char smem[];
    Route &r = *reinterpret_cast<Route *>(smem);
    constexpr uint32_t kPileAt = (sizeof(Route) + 127u) / 128u * 128u, kRingAt = kPileAt + 2u * kMoeWarps * (kMoeChunk / 8) * 512u;
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, quad = lane & 3u;
    pdl_trigger();
    route(m, r, blockIdx.x == 0);
    const uint32_t slices = (m.I + 7u) / 8u, n_items = r.n_entries * slices;
    const uint32_t steps = ((m.D + 31u) / 32u + kMoeWarps - 1u) / kMoeWarps;               // of a warp, an item
    const uint32_t ring = smem_addr(smem) + kRingAt + warp * (kUpRing * kUpStep) + lane * 16u;

    uint32_t in_item = blockIdx.x, in_step = 0u, in_slot = 0u;
    const uint16_t *gate = nullptr, *up = nullptr, *xrow = nullptr;
    bool has_row = false, has_x = false;
    auto enter = [&]() {                                     // where this lane's rows of the item begin
        if (in_item >= n_items) return;
        const uint32_t en = div32(in_item, m.div_slices), sl = in_item - en * slices;
        const uint32_t e = r.entry[en] >> 3, chunk = r.entry[en] & 7u, i = sl * 8u + row;
        const uint16_t *w = m.experts + (int64_t)e * m.expert_stride;
        has_row = i < m.I;
        gate = w + (size_t)i * m.D; up = gate + (size_t)m.I * m.D;
        uint32_t n = 0u;
#pragma unroll
        for (int k = 0; k < HBF_MOE_MAX_TOKENS / 32; ++k) n += __popc(r.mask[e][k]);
        has_x = chunk * kMoeChunk + row < n;
        if (has_x) xrow = m.x + (int64_t)r.token[r.base[e] + chunk * kMoeChunk + row] * m.x_stride;
    };
    auto issue = [&]() {
        if (in_item < n_items) {
            const uint32_t k = (in_step * kMoeWarps + warp) * 32u + quad * 8u;
            const bool in = k < m.D, ok = in && has_row, okx = in && has_x;
            const uint32_t at = ring + in_slot * kUpStep;
            copy_async16(at, ok ? gate + k : m.experts, ok);
            copy_async16(at + 512u, ok ? up + k : m.experts, ok);
            copy_async16_shared(at + 1024u, okx ? xrow + k : m.x, okx);
            in_slot = in_slot + 1u == kUpRing ? 0u : in_slot + 1u;
            if (++in_step == steps) { in_step = 0u; in_item += gridDim.x; enter(); }
        }
        copy_commit();
    };
    enter();
#pragma unroll
    for (int i = 0; i < kUpRing; ++i) issue();

    uint32_t slot = 0u, turn = 0u;
    for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x, turn ^= 1u) {
        const uint32_t en = div32(item, m.div_slices), sl = item - en * slices;
        const uint32_t e = r.entry[en] >> 3, pair0 = r.base[e] + (r.entry[en] & 7u) * kMoeChunk;
        uint32_t n = 0u;
#pragma unroll
        for (int k = 0; k < HBF_MOE_MAX_TOKENS / 32; ++k) n += __popc(r.mask[e][k]);
        n = min(n - (r.entry[en] & 7u) * kMoeChunk, (uint32_t)kMoeChunk);
        const int tiles = (int)((n + 7u) / 8u);
        const uint16_t *more[kMoeChunk / 8 - 1];             // activations of the tokens past the first eight come straight from L1 or L2
#pragma unroll
        for (int j = 1; j < kMoeChunk / 8; ++j) more[j - 1] = j * 8u + row < n ? m.x + (int64_t)r.token[pair0 + j * 8u + row] * m.x_stride : nullptr;
        float acc[kMoeChunk / 8][4];
#pragma unroll
        for (int j = 0; j < kMoeChunk / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        for (uint32_t s = 0; s < steps; ++s) {
            copy_wait<kUpRing - 1>();
            const uint32_t at = ring + slot * kUpStep;
            const uint4 g = ld_shared16(at), u = ld_shared16(at + 512u), x = ld_shared16(at + 1024u);
            slot = slot + 1u == kUpRing ? 0u : slot + 1u;
            Ty::mma(acc[0], g.x, u.x, g.y, u.y, x.x, x.y);
            Ty::mma(acc[0], g.z, u.z, g.w, u.w, x.z, x.w);
            const uint32_t k = (s * kMoeWarps + warp) * 32u + quad * 8u;
#pragma unroll
            for (int j = 1; j < kMoeChunk / 8; ++j)
                if (j < tiles) {
                    const uint4 v = more[j - 1] && k < m.D ? __ldg(reinterpret_cast<const uint4 *>(more[j - 1] + k)) : make_uint4(0u, 0u, 0u, 0u);
                    Ty::mma(acc[j], g.x, u.x, g.y, u.y, v.x, v.y);
                    Ty::mma(acc[j], g.z, u.z, g.w, u.w, v.z, v.w);
                }
            issue();
        }
        // two piles in turn: a warp that is ahead writes the other one, and passes the next barrier only with all
        float4 *pile = reinterpret_cast<float4 *>(smem + kPileAt) + (size_t)turn * kMoeWarps * (kMoeChunk / 8) * 32u;
#pragma unroll
        for (int j = 0; j < kMoeChunk / 8; ++j)
            if (j < tiles) pile[((size_t)warp * tiles + j) * 32u + lane] = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
        __syncthreads();
        sum_over_warps(pile, tiles, [&](uint32_t tile, uint32_t l, const float4 &v) {
            const uint32_t i = sl * 8u + (l >> 2);
            if (i >= m.I) return;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t rank = tile * 8u + (l & 3u) * 2u + k;
                if (rank >= n) continue;
                const float g = k ? v.y : v.x, u = k ? v.w : v.z;
                const float h = r.weight[pair0 + rank] * (g / (1.0f + expf(-g)) * u);
                // held as the sum of two numbers of the weights' type (16 bits of significand for bf16, 22 for fp16): rounding h once to
                // the weights' type would cost as much again as rounding the layer's output does
                const typename Ty::type hi = Ty::from(h), lo = Ty::from(isfinite(h) ? h - Ty::to(hi) : 0.0f);
                const size_t at = (size_t)(pair0 + rank) * m.I + i;
                reinterpret_cast<typename Ty::type *>(m.h_hi)[at] = hi;
                reinterpret_cast<typename Ty::type *>(m.h_lo)[at] = isfinite(Ty::to(hi)) ? lo : Ty::from(0.0f);
            }
        });
    }
    copy_wait<0>();
}

__device__ __forceinline__ uint4 ld_l2(const uint16_t *p) {
    uint4 v; asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p)); return v;
}

// A block keeps up to 16 rows of the output for all tokens (columns of the products) and walks the experts in use; the steps of all
// experts, 32 wide, go to its warps in turn.  A column's sums grow only by the experts its token chose: what another token's expert holds,
// an infinity among it, cannot reach it through a zero.  The first weights are on their way while the kernel before still runs.
template <class Ty, int kTiles>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_down(const __grid_constant__ MoeDev m) {
    extern __shared__ __align__(128) unsigned char smem[];
    Route &r = *reinterpret_cast<Route *>(smem);
    constexpr uint32_t kRingAt = (sizeof(Route) + 127u) / 128u * 128u;
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, quad = lane & 3u;
    route(m, r, false);
    const uint32_t steps = (m.I + 31u) / 32u, n_steps = r.n_active * steps;
    const uint32_t ring = smem_addr(smem) + kRingAt + warp * (kDownRing * kDownStep) + lane * 16u;
    bool waited = false;
    for (uint32_t d0 = blockIdx.x * m.rows; d0 < m.D; d0 += gridDim.x * m.rows) {
        const uint32_t rows = min(m.rows, m.D - d0);
        uint32_t in = warp, in_slot = 0u;
        auto issue = [&]() {
            if (in < n_steps) {
                const uint32_t a = div32(in, m.div_steps), k = (in - a * steps) * 32u + quad * 8u;
                const uint16_t *w = m.experts + (int64_t)r.active[a] * m.expert_stride + (size_t)2 * m.I * m.D + (size_t)(d0 + row) * m.I + k;
                const bool ok0 = k < m.I && row < rows, ok1 = k < m.I && row + 8u < rows;
                const uint32_t at = ring + in_slot * kDownStep;
                copy_async16(at, ok0 ? w : m.experts, ok0);
                copy_async16(at + 512u, ok1 ? w + (size_t)8 * m.I : m.experts, ok1);
                in_slot = in_slot + 1u == kDownRing ? 0u : in_slot + 1u;
                in += kMoeWarps;
            }
            copy_commit();
        };
#pragma unroll
        for (int i = 0; i < kDownRing; ++i) issue();
        if (!waited) { pdl_wait(); waited = true; }
        float acc[kTiles][4];
#pragma unroll
        for (int j = 0; j < kTiles; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.0f;
        uint32_t slot = 0u;
        for (uint32_t st = warp; st < n_steps; st += kMoeWarps) {
            const uint32_t a = div32(st, m.div_steps), k = (st - a * steps) * 32u + quad * 8u, e = r.active[a];
            copy_wait<kDownRing - 1>();
            const uint32_t at = ring + slot * kDownStep;
            const uint4 w0 = ld_shared16(at), w1 = ld_shared16(at + 512u);
            slot = slot + 1u == kDownRing ? 0u : slot + 1u;
            uint32_t below = r.base[e];
#pragma unroll
            for (int j = 0; j < kTiles; ++j) {
                const uint32_t mine = (r.mask[e][j >> 2] >> ((j & 3) * 8)) & 0xffu;
                if (mine == 0u) continue;
                const bool there = ((mine >> row) & 1u) != 0u && k < m.I;
                const size_t h = (size_t)(below + __popc(mine & ((1u << row) - 1u))) * m.I + k;
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                const uint4 hi = there ? ld_l2(m.h_hi + h) : zero, lo = there ? ld_l2(m.h_lo + h) : zero;
                below += __popc(mine);
                float p[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                Ty::mma(p, w0.x, w1.x, w0.y, w1.y, hi.x, hi.y);
                Ty::mma(p, w0.z, w1.z, w0.w, w1.w, hi.z, hi.w);
                Ty::mma(p, w0.x, w1.x, w0.y, w1.y, lo.x, lo.y);
                Ty::mma(p, w0.z, w1.z, w0.w, w1.w, lo.z, lo.w);
                const bool c0 = (mine >> (quad * 2u)) & 1u, c1 = (mine >> (quad * 2u + 1u)) & 1u;
                if (c0) { acc[j][0] += p[0]; acc[j][2] += p[2]; }
                if (c1) { acc[j][1] += p[1]; acc[j][3] += p[3]; }
            }
            issue();
        }
        copy_wait<0>();
        __syncthreads();                                     // the rings are empty: their memory is the pile's
        float4 *pile = reinterpret_cast<float4 *>(smem + kRingAt);
#pragma unroll
        for (int j = 0; j < kTiles; ++j) pile[((size_t)warp * kTiles + j) * 32u + lane] = make_float4(acc[j][0], acc[j][1], acc[j][2], acc[j][3]);
        __syncthreads();
        sum_over_warps(pile, kTiles, [&](uint32_t tile, uint32_t l, const float4 &v) {
            const float sums[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t t = tile * 8u + (l & 3u) * 2u + (c & 1), d = (l >> 2) + (c >> 1) * 8u;
                if (t < m.T && d < rows) {
                    const float v1 = (r.bad[t >> 5] >> (t & 31u)) & 1u ? __int_as_float(0x7fc00000) : sums[c];
                    reinterpret_cast<typename Ty::type *>(m.out)[(int64_t)t * m.out_stride + d0 + d] = Ty::from(v1);
                }
            }
        });
        __syncthreads();
    }
    if (!waited) pdl_wait();
}

// The records of what a layer reads: every expert in use once, in tiles, experts ascending; the places behind them hold records of one
// byte at address 0, outside every range.
__global__ void __launch_bounds__(kMoeThreads)
k_moe_accesses(const __grid_constant__ MoeDev m, uint64_t expert_bytes, uint32_t tile_bytes, uint32_t tiles, int64_t issue_ns, int64_t gap_ns,
               hbf_access_t *acc, uint64_t n) {
    extern __shared__ __align__(128) unsigned char smem[];
    Route &r = *reinterpret_cast<Route *>(smem);
    route(m, r, false);
    for (uint64_t i = (uint64_t)blockIdx.x * kMoeThreads + threadIdx.x; i < n; i += (uint64_t)gridDim.x * kMoeThreads) {
        const uint32_t a = (uint32_t)(i / tiles), t = (uint32_t)(i - (uint64_t)a * tiles);
        hbf_access_t v = {0, issue_ns + (int64_t)i * gap_ns, 1, 0};
        if (a < r.n_active) {
            const uint64_t off = (uint64_t)t * tile_bytes, left = expert_bytes - off;
            v.addr = (uint64_t)(uintptr_t)(m.experts + (int64_t)r.active[a] * m.expert_stride) + off;
            v.bytes = left < tile_bytes ? (uint32_t)left : tile_bytes;
        }
        acc[i] = v;
    }
}

static bool moe_ok(const hbf_moe_t *m) {
    if (!m || m->tokens > HBF_MOE_MAX_TOKENS || m->n_experts == 0 || m->n_experts > HBF_MOE_MAX_EXPERTS) return false;
    if (m->top_k == 0 || m->top_k > HBF_MOE_MAX_TOP_K || m->top_k > m->n_experts || m->dtype > HBF_FP16 || m->renormalise > 1u) return false;
    if (m->hidden == 0 || m->inter == 0 || m->hidden % 8 || m->inter % 8 || m->hidden > (1u << 20) || m->inter > (1u << 20)) return false;
    if (m->expert_stride < 3 * (int64_t)m->hidden * m->inter || m->expert_stride % 8) return false;
    return true;
}
static bool moe_pointers_ok(const hbf_moe_t *m) {
    if (!m->scores || !m->experts || (uintptr_t)m->experts % 16 || (uintptr_t)m->scores % 4 || m->scores_stride < (int64_t)m->n_experts) return false;
    return true;
}
static MoeDev moe_dev(const hbf_moe_t *m) {
    MoeDev d = {};
    d.T = m->tokens; d.D = m->hidden; d.I = m->inter; d.E = m->n_experts; d.K = m->top_k; d.renorm = m->renormalise;
    d.x = static_cast<const uint16_t *>(m->x); d.x_stride = m->x_stride;
    d.scores = m->scores; d.scores_stride = m->scores_stride;
    d.experts = static_cast<const uint16_t *>(m->experts); d.expert_stride = m->expert_stride;
    d.out = static_cast<uint16_t *>(m->out); d.out_stride = m->out_stride;
    d.chosen = m->chosen; d.weights = m->weights;
    return d;
}

template <class Ty>
static cudaError_t launch_moe(MoeDev d, uint32_t n_sm, cudaStream_t st) {
    constexpr size_t kRoute = (sizeof(Route) + 127u) / 128u * 128u;
    constexpr size_t up_smem = kRoute + 2u * kMoeWarps * (kMoeChunk / 8) * 512u + (size_t)kMoeWarps * kUpRing * kUpStep;
    static_assert(up_smem <= 227 * 1024, "shared memory of the up kernel");
    const uint32_t slices = (d.I + 7u) / 8u;
    d.div_slices = make_div32(slices); d.div_steps = make_div32((d.I + 31u) / 32u);
    // an even share of the output's rows to every SM, 16 at most: 2,048 rows are 14 a block on 147 blocks
    const uint32_t rounds = (d.D + 16u * n_sm - 1u) / (16u * n_sm);
    d.rows = (d.D + rounds * n_sm - 1u) / (rounds * n_sm);
    const uint32_t down_blocks = min(n_sm, (d.D + d.rows - 1u) / d.rows);
    const uint64_t most = (uint64_t)min(d.E + d.T * d.K / kMoeChunk, d.T * d.K) * slices;
    cudaError_t e = ensure_dyn_smem((const void *)k_moe_up<Ty>, up_smem);
    if (e != cudaSuccess) return e;
    k_moe_up<Ty><<<(unsigned)(most < n_sm ? most : n_sm), kMoeThreads, up_smem, st>>>(d);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    const uint32_t tiles = d.T <= 8u ? 1u : d.T <= 16u ? 2u : d.T <= 32u ? 4u : d.T <= 64u ? 8u : 16u;
    const size_t ring = (size_t)kMoeWarps * kDownRing * kDownStep, pile = (size_t)kMoeWarps * tiles * 512u;
    const size_t down_smem = kRoute + (ring > pile ? ring : pile);
    void (*down)(MoeDev) = tiles == 1u ? k_moe_down<Ty, 1> : tiles == 2u ? k_moe_down<Ty, 2> : tiles == 4u ? k_moe_down<Ty, 4> : tiles == 8u ? k_moe_down<Ty, 8> : k_moe_down<Ty, 16>;
    if ((e = ensure_dyn_smem((const void *)down, down_smem)) != cudaSuccess) return e;
    g_kernel_launches += 2;
    return launch_pdl(down, down_blocks, kMoeThreads, down_smem, st, d);
}

}  // namespace hbf

using namespace hbf;

extern "C" size_t hbf_moe_workspace_bytes(const hbf_moe_t *m) {
    if (!moe_ok(m)) return 0;
    return ((size_t)m->tokens * m->top_k * m->inter * 4u + 255u) / 256u * 256u;
}

extern "C" int hbf_moe_layer(const hbf_moe_t *m, void *d_workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!moe_ok(m)) return HBF_E_INVAL;
    if (m->tokens == 0) return HBF_OK;
    if (!moe_pointers_ok(m) || !m->x || !m->out || (uintptr_t)m->x % 16 || (uintptr_t)m->out % 2 || m->x_stride % 8) return HBF_E_INVAL;
    if (m->x_stride < (int64_t)m->hidden || m->out_stride < (int64_t)m->hidden) return HBF_E_INVAL;
    if (!d_workspace || (uintptr_t)d_workspace % 256 || workspace_bytes < hbf_moe_workspace_bytes(m)) return HBF_E_WORKSPACE;
    uint32_t n_sm = 0;
    const int rc = device_of(m->experts, &n_sm);
    if (rc != HBF_OK) return rc;
    MoeDev d = moe_dev(m);
    d.h_hi = static_cast<uint16_t *>(d_workspace); d.h_lo = d.h_hi + (size_t)m->tokens * m->top_k * m->inter;
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return (m->dtype == HBF_BF16 ? launch_moe<Bf16>(d, n_sm, st) : launch_moe<Fp16>(d, n_sm, st)) == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}

extern "C" uint64_t hbf_moe_access_count(const hbf_moe_t *m, uint32_t tile_bytes) {
    if (!moe_ok(m) || tile_bytes == 0) return 0;
    const uint64_t bytes = 6ull * m->hidden * m->inter, used = (uint64_t)m->tokens * m->top_k;
    return (used < m->n_experts ? used : m->n_experts) * ((bytes + tile_bytes - 1) / tile_bytes);
}

extern "C" int hbf_moe_accesses(const hbf_moe_t *m, uint32_t tile_bytes, int64_t issue_ns, int64_t gap_ns, hbf_access_t *d_acc, uint64_t n, void *cuda_stream) {
    if (!moe_ok(m) || tile_bytes == 0 || issue_ns < 0 || gap_ns < 0) return HBF_E_INVAL;
    const uint64_t want = hbf_moe_access_count(m, tile_bytes);
    if (n != want || n > HBF_MAX_BATCH) return HBF_E_INVAL;
    if (n == 0) return HBF_OK;
    if (!moe_pointers_ok(m) || !d_acc || (uintptr_t)d_acc % 8) return HBF_E_INVAL;
    uint32_t n_sm = 0;
    const int rc = device_of(m->experts, &n_sm);
    if (rc != HBF_OK) return rc;
    const uint64_t bytes = 6ull * m->hidden * m->inter;
    const uint64_t blocks = (n + kMoeThreads * 4 - 1) / (kMoeThreads * 4);
    if (ensure_dyn_smem((const void *)k_moe_accesses, sizeof(Route)) != cudaSuccess) return HBF_E_CUDA;
    k_moe_accesses<<<(unsigned)(blocks < n_sm ? blocks : n_sm), kMoeThreads, sizeof(Route), static_cast<cudaStream_t>(cuda_stream)>>>(
        moe_dev(m), bytes, tile_bytes, (uint32_t)((bytes + tile_bytes - 1) / tile_bytes), issue_ns, gap_ns, d_acc, n);
    g_kernel_launches += 1;
    return cudaGetLastError() == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}
