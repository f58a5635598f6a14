// A mixture-of-experts layer for up to eight tokens in two kernels (moe_tiles.cu has the form for more).
//
//   choice      the top_k largest of a token's scores, ties to the lowest expert; weights w = softmax over the chosen (or over all)
//   k_moe_up    h[pair] = w * silu(gate x) * (up x)             for every (expert, token that chose it) pair
//   k_moe_down  out[token] = sum over its experts of down h
//
// Bytes bound it: an expert's 6 * inter * hidden bytes are read once, whatever the number of its tokens (a few).  So the weights go
// from HBM past L1 into rings of shared memory, 16 bytes a lane at a time, and from there, as they lie, into the A operand of m16n8k16
// products whose columns are tokens; no tile is ever padded to more than 8 tokens.  The order in which a product sums its 16-wide steps
// is free, so every lane takes 16 consecutive bytes of its row (two steps' worth) from weights and activations alike, and reads back only
// what it copied itself: no transposition, no barrier in the stream.  (Bulk copies of a row's stretch by a warp of their own, which need fewer
// instructions, were slower throughout: 64 tokens 556 us against 272, the copies of 0.5 to 1 KB leave the SM one after the other.)
#include <type_traits>

#include "moe.cuh"

namespace hbf {

// Rings of five and three steps, 80 and 96 KB of weights an SM on their way; longer ones were no faster, and neither was room for both kernels on
// an SM (a token 26.8 us against 24.7: half of the registers each, and the weights of the second take their share of the bandwidth early).
constexpr int kFewTokens = 8, kUpRing = 5, kDownRing = 3, kDownWide = 2;
using FewRoute = Route<kFewTokens>;
using FewTemp = RouteTemp<kFewTokens>;
constexpr uint32_t kFewBytes = kRouteBytes<kFewTokens>;

// Sixteen warps' sums of a 16 x 8 product, left as they lie in the accumulators: eight lanes for a column of the pile, two warps' parts
// each, always in the same order.  f(lane of the accumulator, its four sums) is called once for every column.
template <class F>
__device__ __forceinline__ void sum_over_warps(const float4 *pile, F f) {
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, part = lane >> 2, col = warp * 4u + (lane & 3u);
    if (warp >= 8u) return;
    float4 s = pile[part * 64u + col];
    const float4 v = pile[part * 64u + 32u + col];
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) {
        s.x += __shfl_xor_sync(0xffffffffu, s.x, o); s.y += __shfl_xor_sync(0xffffffffu, s.y, o);
        s.z += __shfl_xor_sync(0xffffffffu, s.z, o); s.w += __shfl_xor_sync(0xffffffffu, s.w, o);
    }
    if (part == 0u) f(col, s);
}

__device__ __forceinline__ uint4 ld_input(const uint16_t *p) { return __ldg(reinterpret_cast<const uint4 *>(p)); }
__device__ __forceinline__ uint4 ld_after16(const uint16_t *p) {                            // (see ld_after)
    uint4 v; asm volatile("ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p)); return v;
}

// Shared memory of the up kernel: the choice, the pile of sums twice, the rings.
constexpr uint32_t kUpRingAt = kFewBytes + 2u * kMoeWarps * 512u, kUpSmem = kUpRingAt + kMoeWarps * kUpRing * 1024u;

// Items of eight gate rows and the same eight up rows (rows 0..7 and 8..15 of one product, so a thread's sums hold both), one item a
// block at a time, the sum over `hidden` split among its warps in steps of 32; the ring runs on into the next item while an item's sums
// are joined.  Activations, which L1 or L2 holds, are asked for a step ahead.
template <class Ty>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_up(const __grid_constant__ MoeDev m) {
    extern __shared__ __align__(128) unsigned char smem[];
    FewRoute &r = *reinterpret_cast<FewRoute *>(smem);
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, quad = lane & 3u;
    pdl_trigger();
    route<false>(m, r, *reinterpret_cast<FewTemp *>(smem + kFewBytes), kFewTokens, blockIdx.x == 0);
    const uint32_t slices = m.I / 8u, n_items = r.n_entries * slices;
    const uint32_t steps = ((m.D + 31u) / 32u + kMoeWarps - 1u) / kMoeWarps;               // of a warp, an item
    const uint32_t ring = smem_addr(smem) + kUpRingAt + warp * (kUpRing * 1024u) + lane * 16u, k0 = warp * 32u + quad * 8u;
    constexpr uint32_t kStride = kMoeWarps * 32u;

    uint32_t in_item = blockIdx.x, in_k = k0, in_left = steps, in_slot = 0u;
    const uint16_t *gate = m.experts;
    auto place = [&]() {                                     // where this lane's rows of the item begin
        if (in_item >= n_items) return;
        const uint32_t en = div32(in_item, m.div_slices), i = (in_item - en * slices) * 8u + row;
        gate = m.experts + (int64_t)r.expert[en] * m.expert_stride + (size_t)i * m.D;
    };
    auto issue = [&]() {
        if (in_item < n_items) {
            const bool in = in_k < m.D;
            const uint16_t *g = in ? gate + in_k : m.experts;
            copy_async16(ring + in_slot * 1024u, g, in);
            copy_async16(ring + in_slot * 1024u + 512u, in ? g + (size_t)m.I * m.D : g, in);
            in_slot = in_slot + 1u == kUpRing ? 0u : in_slot + 1u;
            in_k += kStride;
            if (--in_left == 0u) { in_left = steps; in_k = k0; in_item += gridDim.x; place(); }
        }
        copy_commit();
    };
    place();
#pragma unroll 1
    for (int i = 0; i < kUpRing; ++i) issue();

    uint32_t slot = 0u, turn = 0u;
    for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x, turn ^= 1u) {
        const uint32_t en = div32(item, m.div_slices), sl = item - en * slices, n = r.count[en], pair0 = r.pair0[en];
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        const uint16_t *x = row < n ? m.x + (int64_t)r.token[pair0 + row] * m.x_stride : nullptr;
        uint4 now = x && k0 < m.D ? ld_input(x + k0) : zero;
        float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (uint32_t s = 0, k = k0 + kStride; s < steps; ++s, k += kStride) {
            const uint4 next = x && k < m.D && s + 1u < steps ? ld_input(x + k) : zero;
            copy_wait<kUpRing - 1>();
            const uint4 g = ld_shared16(ring + slot * 1024u), u = ld_shared16(ring + slot * 1024u + 512u);
            slot = slot + 1u == kUpRing ? 0u : slot + 1u;
            Ty::mma(acc, g.x, u.x, g.y, u.y, now.x, now.y);
            Ty::mma(acc, g.z, u.z, g.w, u.w, now.z, now.w);
            issue();
            now = next;
        }
        // two piles in turn: a warp that is ahead writes the other one, and passes the next barrier only with all
        float4 *pile = reinterpret_cast<float4 *>(smem + kFewBytes) + turn * (kMoeWarps * 32u);
        pile[warp * 32u + lane] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        __syncthreads();
        sum_over_warps(pile, [&](uint32_t l, const float4 &v) {
            const uint32_t i = sl * 8u + (l >> 2);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const uint32_t rank = (l & 3u) * 2u + k;
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

// Shared memory of the down kernel: the choice, every warp's sums of 16 rows for all tokens, the rings.
__host__ __device__ constexpr uint32_t down_sums(uint32_t tokens) { return kMoeWarps * tokens * 64u; }
constexpr uint32_t down_smem(uint32_t tokens) { return kFewBytes + down_sums(tokens) + kMoeWarps * kDownRing * kDownWide * 1024u; }
static_assert(kUpSmem <= 227 * 1024 && down_smem(kFewTokens) <= 227 * 1024 && sizeof(FewTemp) <= kMoeWarps * 1024u, "shared memory");

// A block keeps up to 16 rows of the output for all tokens and walks the steps of the experts in use, 32 kDownWide each, a stretch of
// them a warp.  An expert's products have its tokens as columns; a warp adds them to its sums in shared memory when it comes to the next one:
// a token's sums grow only by what its own experts hold, and in the order of the experts.  The ring's first weights are on their way while the
// kernel before still runs; activations, which L2 holds, are asked for a step ahead.
template <class Ty>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_down(const __grid_constant__ MoeDev m) {
    extern __shared__ __align__(128) unsigned char smem[];
    FewRoute &r = *reinterpret_cast<FewRoute *>(smem);
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5, row = lane >> 2, quad = lane & 3u;
    route<false>(m, r, *reinterpret_cast<FewTemp *>(smem + kFewBytes), kFewTokens, false);
    float *sums = reinterpret_cast<float *>(smem + kFewBytes);                              // [warp][token][16]
    float *mine = sums + (size_t)warp * m.T * 16u;
    constexpr uint32_t kStep = kDownWide * 32u, kSlot = kDownWide * 1024u;
    const uint32_t steps = (m.I + kStep - 1u) / kStep, n_steps = r.n_entries * steps;
    const uint32_t first = (uint32_t)((uint64_t)n_steps * warp / kMoeWarps), last = (uint32_t)((uint64_t)n_steps * (warp + 1u) / kMoeWarps);
    const uint32_t en0 = first / steps, s0 = first - en0 * steps;
    const uint32_t ring = smem_addr(smem) + kFewBytes + down_sums(m.T) + warp * (kDownRing * kSlot) + lane * 16u;
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    const size_t h_lo = (size_t)(m.h_lo - m.h_hi);
    bool waited = false;
    for (uint32_t d0 = blockIdx.x * m.rows; d0 < m.D; d0 += gridDim.x * m.rows) {
        const uint32_t rows = min(m.rows, m.D - d0);
        const bool row0 = row < rows, row1 = row + 8u < rows;
        const uint16_t *down = m.experts + (size_t)2 * m.I * m.D + (size_t)(d0 + row) * m.I, *w = down;
        uint32_t in_left = last - first, in_en = en0, in_s = s0, in_slot = 0u;
        auto place = [&]() { if (in_left) w = down + (int64_t)r.expert[in_en] * m.expert_stride; };
        auto issue = [&]() {
            if (in_left) {
#pragma unroll
                for (int b = 0; b < kDownWide; ++b) {
                    const uint32_t k = in_s * kStep + b * 32u + quad * 8u, at = ring + in_slot * kSlot + b * 1024u;
                    const bool in = k < m.I;
                    copy_async16(at, in && row0 ? w + k : m.experts, in && row0);
                    copy_async16(at + 512u, in && row1 ? w + (size_t)8 * m.I + k : m.experts, in && row1);
                }
                in_slot = in_slot + 1u == kDownRing ? 0u : in_slot + 1u;
                --in_left;
                if (++in_s == steps) { in_s = 0u; ++in_en; place(); }
            }
            copy_commit();
        };
        place();
#pragma unroll 1
        for (int i = 0; i < kDownRing; ++i) issue();
        for (uint32_t i = lane; i < m.T * 16u; i += 32u) mine[i] = 0.0f;
        __syncwarp();
        if (!waited) { pdl_wait(); waited = true; }
        uint32_t en = en0, s = s0, slot = 0u, n = 0u, pair0 = 0u, left = last - first;
        const uint16_t *h = m.h_hi;                          // this lane's row of the expert's tokens
        auto enter = [&]() { n = r.count[en]; pair0 = r.pair0[en]; h = m.h_hi + (size_t)(pair0 + row) * m.I; };
        auto load = [&](uint4 (&v)[kDownWide][2], uint32_t step) {
#pragma unroll
            for (int b = 0; b < kDownWide; ++b) {
                const uint32_t k = step * kStep + b * 32u + quad * 8u;
                const bool in = row < n && k < m.I;
                v[b][0] = in ? ld_after16(h + k) : zero;
                v[b][1] = in ? ld_after16(h + h_lo + k) : zero;
            }
        };
        uint4 now[kDownWide][2], then[kDownWide][2];
        if (left) { enter(); load(now, s); }
        float acc[2][4];                                     // two chains of products: the first and the second numbers
        auto clear = [&]() {
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[0][c] = acc[1][c] = 0.0f;
        };
        clear();
        auto turn = [&](uint4 (&cur)[kDownWide][2], uint4 (&next)[kDownWide][2]) {
            const uint32_t n_now = n, pair_now = pair0;
            const bool done = ++s == steps || left == 1u;    // the expert is done, or this warp's part of it
            if (s == steps) { s = 0u; ++en; if (left > 1u) enter(); }
            if (left > 1u) load(next, s);
            copy_wait<kDownRing - 1>();
#pragma unroll
            for (int b = 0; b < kDownWide; ++b) {
                const uint4 w0 = ld_shared16(ring + slot * kSlot + b * 1024u), w1 = ld_shared16(ring + slot * kSlot + b * 1024u + 512u);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    Ty::mma(acc[c], w0.x, w1.x, w0.y, w1.y, cur[b][c].x, cur[b][c].y);
                    Ty::mma(acc[c], w0.z, w1.z, w0.w, w1.w, cur[b][c].z, cur[b][c].w);
                }
            }
            slot = slot + 1u == kDownRing ? 0u : slot + 1u;
            issue();
            if (done) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t rank = quad * 2u + c;
                    if (rank < n_now) {
                        float *to = mine + r.token[pair_now + rank] * 16u + row;
                        to[0] += acc[0][c] + acc[1][c];
                        to[8] += acc[0][c + 2] + acc[1][c + 2];
                    }
                }
                clear();
                __syncwarp();
            }
            --left;
        };
#pragma unroll 1
        while (left) {
            turn(now, then);
            if (left) turn(then, now);
        }
        __syncthreads();
        for (uint32_t i = tid; i < m.T * 16u; i += kMoeThreads) {
            const uint32_t t = i >> 4, d = i & 15u;
            if (d >= rows) continue;
            float v = 0.0f;
#pragma unroll
            for (int k = 0; k < kMoeWarps; ++k) v += sums[(size_t)k * m.T * 16u + i];
            if ((r.bad[t >> 5] >> (t & 31u)) & 1u) v = __int_as_float(0x7fc00000);
            reinterpret_cast<typename Ty::type *>(m.out)[(int64_t)t * m.out_stride + d0 + d] = Ty::from(v);
        }
        __syncthreads();
    }
    copy_wait<0>();
    if (!waited) pdl_wait();
}

// The records of what a layer reads: every expert in use once, in tiles, experts ascending; the places behind them hold records of one
// byte at address 0, outside every range.
__global__ void __launch_bounds__(kMoeThreads)
k_moe_accesses(const __grid_constant__ MoeDev m, uint64_t expert_bytes, uint32_t tile_bytes, uint32_t tiles, int64_t issue_ns, int64_t gap_ns,
               hbf_access_t *acc, uint64_t n) {
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr int kTokens = HBF_MOE_MAX_TOKENS;
    Route<kTokens> &r = *reinterpret_cast<Route<kTokens> *>(smem);
    route<false>(m, r, *reinterpret_cast<RouteTemp<kTokens> *>(smem + kRouteBytes<kTokens>), 8u, false);
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
// Whether the layer goes through k_moe_up and k_moe_down: two launches instead of four, and for these few tokens faster whatever the
// weights (2048 x 768, top 8 of 128, 8 tokens, 351 MB in use: 75.6 us against 93.8; 4096 x 2048, top 2 of 8: 64.6 against 78.8).
static bool moe_few(const hbf_moe_t *m) { return m->tokens <= (uint32_t)kFewTokens; }
// The activations between the products, and past a few tokens the parts' sums and the choice; 0: the device cannot be asked.
static size_t moe_bytes(const hbf_moe_t *m, uint32_t *groups) {
    const size_t pairs = (size_t)m->tokens * m->top_k, h = (pairs * m->inter * 4u + 255u) / 256u * 256u;
    if (groups) *groups = 1u;
    if (moe_few(m)) return h;
    uint32_t n_sm = 0;
    if (sm_count(&n_sm) != HBF_OK) return 0;
    const uint32_t g = moe_groups(m->tokens, m->hidden, m->n_experts, m->top_k, n_sm);
    if (groups) *groups = g;
    return h + ((size_t)g * m->tokens * m->hidden * 4u + 255u) / 256u * 256u + (pairs * 6u + 255u) / 256u * 256u;
}
static MoeDev moe_dev(const hbf_moe_t *m) {
    MoeDev d = {};
    d.T = m->tokens; d.D = m->hidden; d.I = m->inter; d.E = m->n_experts; d.K = m->top_k; d.renorm = m->renormalise;
    d.x = static_cast<const uint16_t *>(m->x); d.x_stride = m->x_stride;
    d.scores = m->scores; d.scores_stride = m->scores_stride;
    d.experts = static_cast<const uint16_t *>(m->experts); d.expert_stride = m->expert_stride;
    d.out = static_cast<uint16_t *>(m->out); d.out_stride = m->out_stride;
    d.chosen = m->chosen; d.weights = m->weights; d.div_k = make_div32(d.K);
    d.polls = g_operator_polls.load(std::memory_order_relaxed);
    return d;
}

template <class Ty>
static cudaError_t launch_moe(MoeDev d, bool few, uint32_t n_sm, cudaStream_t st) {
    d.div_slices = make_div32(d.I / 8u);
    // an even share of the output's rows to every SM, 16 at most: 2,048 rows are 14 a block on 147 blocks
    const uint32_t rounds = (d.D + 16u * n_sm - 1u) / (16u * n_sm);
    d.rows = (d.D + rounds * n_sm - 1u) / (rounds * n_sm);
    if (few) {
        cudaError_t e = ensure_dyn_smem((const void *)k_moe_up<Ty>, kUpSmem);
        if (e == cudaSuccess) e = ensure_dyn_smem((const void *)k_moe_down<Ty>, down_smem(kFewTokens));
        if (e != cudaSuccess) return e;
        const uint64_t pairs = (uint64_t)d.T * d.K, most = (pairs < d.E ? pairs : d.E) * (d.I / 8u);
        k_moe_up<Ty><<<(unsigned)(most < n_sm ? most : n_sm), kMoeThreads, kUpSmem, st>>>(d);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        const uint32_t blocks = (d.D + d.rows - 1u) / d.rows;
        g_kernel_launches += 2;
        return launch_pdl(k_moe_down<Ty>, blocks < n_sm ? blocks : n_sm, kMoeThreads, down_smem(d.T), st, d);
    }
    return launch_moe_tiles(d, std::is_same<Ty, Bf16>::value, n_sm, st);
}

}  // namespace hbf

using namespace hbf;

extern "C" size_t hbf_moe_workspace_bytes(const hbf_moe_t *m) {
    if (!moe_ok(m)) return 0;
    return m->tokens ? moe_bytes(m, nullptr) : 256u;
}

extern "C" int hbf_moe_layer(const hbf_moe_t *m, void *d_workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!moe_ok(m)) return HBF_E_INVAL;
    if (m->tokens == 0) return HBF_OK;
    if (!moe_pointers_ok(m) || !m->x || !m->out || (uintptr_t)m->x % 16 || (uintptr_t)m->out % 2 || m->x_stride % 8) return HBF_E_INVAL;
    if (m->x_stride < (int64_t)m->hidden || m->out_stride < (int64_t)m->hidden) return HBF_E_INVAL;
    if (!d_workspace || (uintptr_t)d_workspace % 256) return HBF_E_WORKSPACE;
    uint32_t n_sm = 0;
    MoeDev d = moe_dev(m);
    const size_t need = moe_bytes(m, &d.groups);
    if (need == 0) return HBF_E_CUDA;
    if (workspace_bytes < need) return HBF_E_WORKSPACE;
    const int rc = device_of(m->experts, &n_sm);
    if (rc != HBF_OK) return rc;
    const size_t pairs = (size_t)m->tokens * m->top_k;
    d.h_hi = static_cast<uint16_t *>(d_workspace); d.h_lo = d.h_hi + pairs * m->inter;
    unsigned char *more = static_cast<unsigned char *>(d_workspace) + (pairs * m->inter * 4u + 255u) / 256u * 256u;
    d.part = reinterpret_cast<float *>(more);
    d.route_w = reinterpret_cast<float *>(more + ((size_t)d.groups * m->tokens * m->hidden * 4u + 255u) / 256u * 256u);
    d.route_e = reinterpret_cast<uint16_t *>(d.route_w + pairs);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    return (m->dtype == HBF_BF16 ? launch_moe<Bf16>(d, moe_few(m), n_sm, st) : launch_moe<Fp16>(d, moe_few(m), n_sm, st)) == cudaSuccess ? HBF_OK : HBF_E_CUDA;
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
    constexpr size_t smem = kRouteBytes<HBF_MOE_MAX_TOKENS> + sizeof(RouteTemp<HBF_MOE_MAX_TOKENS>);
    if (ensure_dyn_smem((const void *)k_moe_accesses, smem) != cudaSuccess) return HBF_E_CUDA;
    k_moe_accesses<<<(unsigned)(blocks < n_sm ? blocks : n_sm), kMoeThreads, smem, static_cast<cudaStream_t>(cuda_stream)>>>(
        moe_dev(m), bytes, tile_bytes, (uint32_t)((bytes + tile_bytes - 1) / tile_bytes), issue_ns, gap_ns, d_acc, n);
    g_kernel_launches += 1;
    return cudaGetLastError() == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}
