// What the kernels of the mixture-of-experts layer share: the parameters, and the choice of the experts.
#pragma once
#include "tensor_ops.cuh"

namespace hbf {

constexpr int kMoeWarps = 16, kMoeThreads = kMoeWarps * 32;

struct MoeDev {
    uint32_t T, D, I, E, K, renorm;
    const uint16_t *x; int64_t x_stride;
    const float *scores; int64_t scores_stride;
    const uint16_t *experts; int64_t expert_stride;
    uint16_t *out; int64_t out_stride;
    int32_t *chosen; float *weights;
    uint16_t *h_hi, *h_lo;                                   // [pairs by expert, then token][I]
    uint32_t rows;                                           // of the down product that a block takes, at most 16
    float *part; uint32_t groups;                            // moe_tiles.cu: [groups][T][D], the sums of a group's experts
    uint16_t *route_e; float *route_w;                       // and [T][K]: the choice, made by a kernel of its own (0xfffe: the token has none)
    Div32 div_slices, div_k;                                 // I / 8; K
    uint32_t polls;                                          // of a wait in moe_tiles.cu
};

// What the choice leaves in shared memory, the same in every block that makes it.  An entry is an expert in use with up to `chunk` of its
// tokens; entries by expert, pairs (expert, token) by entry.
template <int kTokens>
struct Route {
    static constexpr int kWords = (kTokens + 31) / 32, kPairs = kTokens * HBF_MOE_MAX_TOP_K, kEntries = HBF_MOE_MAX_EXPERTS + kPairs / 8;
    uint32_t mask[HBF_MOE_MAX_EXPERTS][kWords];                      // tokens of each expert
    uint16_t base[HBF_MOE_MAX_EXPERTS];                              // pairs of the experts before it
    uint16_t active[HBF_MOE_MAX_EXPERTS];                            // experts in use, ascending
    uint16_t expert[kEntries], pair0[kEntries];
    uint8_t count[kEntries];
    uint8_t token[kPairs];                                           // of each pair
    float weight[kPairs];
    uint32_t bad[kWords];                                            // tokens with a NaN among their scores
    uint32_t n_active, n_entries, scan[kMoeWarps][3];
};
template <int kTokens>
struct RouteTemp {                                                   // of the choice itself; the memory is used again behind it
    uint16_t expert[kTokens * HBF_MOE_MAX_TOP_K];
    float weight[kTokens * HBF_MOE_MAX_TOP_K];
};
template <int kTokens> constexpr uint32_t kRouteBytes = (sizeof(Route<kTokens>) + 127u) / 128u * 128u;

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

// The choice of kTok tokens t0, t0 + step, ... by one warp, kKeys neighbouring scores a lane.  A lane puts its own scores in order, once; a turn
// takes the largest of the lanes' first ones (the lowest lane that has it wins a tie, and in a lane the lowest expert comes first), and lane j
// keeps what turn j took.  Instructions bound it where a warp has several tokens (searching every lane's scores in every turn: 64 tokens of
// 128 experts 6.5 us; turns of several tokens at once hide each other's latency).
template <int kKeys, int kTok, bool kOwn, int kTokens>
__device__ __forceinline__ void choose(const MoeDev &m, Route<kTokens> &r, RouteTemp<kTokens> &tmp, uint32_t t0, uint32_t step, bool write) {
    const uint32_t lane = lane_id();
    uint32_t key[kTok][kKeys], first[kTok];
    float all[kTok];
    bool live[kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const uint32_t tok = t0 + t * step;
        const float *s = m.scores + (int64_t)tok * m.scores_stride;
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
            const uint32_t e = lane * kKeys + i;
            key[t][i] = __float_as_uint(tok < m.T && e < m.E ? s[e] : -INFINITY);
        }
    }
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        bool nan = false;
#pragma unroll
        for (int i = 0; i < kKeys; ++i) { const float f = __uint_as_float(key[t][i]); nan |= f != f; key[t][i] = ordered(f); }
        nan = __any_sync(0xffffffffu, nan);
        const uint32_t tok = t0 + t * step;
        live[t] = tok < m.T && !nan;
        if (!kOwn && nan && lane == 0u) atomicOr(&r.bad[tok >> 5], 1u << (tok & 31u));
        first[t] = 0u; all[t] = 0.0f;
    }
    uint32_t at[kTok][kKeys], mine[kTok], took[kTok];        // the scores' experts; of turn `lane`: expert and score
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
#pragma unroll
        for (int i = 0; i < kKeys; ++i) at[t][i] = lane * kKeys + i;
#pragma unroll
        for (int k = 0; k < kKeys; ++k)
#pragma unroll
            for (int i = k & 1; i + 1 < kKeys; i += 2) {
                const bool swap = key[t][i] < key[t][i + 1];
                const uint32_t u = key[t][i], v = key[t][i + 1], x = at[t][i], y = at[t][i + 1];
                key[t][i] = swap ? v : u; key[t][i + 1] = swap ? u : v; at[t][i] = swap ? y : x; at[t][i + 1] = swap ? x : y;
            }
        if (!m.renorm) {
            first[t] = __reduce_max_sync(0xffffffffu, key[t][0]);
#pragma unroll
            for (int i = 0; i < kKeys; ++i) all[t] += key[t][i] ? expf(from_ordered(key[t][i]) - from_ordered(first[t])) : 0.0f;
        }
        mine[t] = 0xffffu; took[t] = 0u;
        if (!live[t])
#pragma unroll
            for (int i = 0; i < kKeys; ++i) key[t][i] = 0u;
    }
#pragma unroll 1
    for (uint32_t j = 0; j < m.K; ++j) {
        uint32_t best[kTok];
#pragma unroll
        for (int t = 0; t < kTok; ++t) best[t] = __reduce_max_sync(0xffffffffu, key[t][0]);
#pragma unroll
        for (int t = 0; t < kTok; ++t) {
            const unsigned has = __ballot_sync(0xffffffffu, key[t][0] == best[t]);
            const uint32_t e = __shfl_sync(0xffffffffu, at[t][0], __ffs(has) - 1);
            if (j == 0u) first[t] = best[t];
            if (lane == j && best[t]) { mine[t] = e; took[t] = best[t]; }
            const bool won = e == at[t][0];                  // (of a lane whose scores are used up nothing is left to lose)
#pragma unroll
            for (int i = 0; i + 1 < kKeys; ++i) { key[t][i] = won ? key[t][i + 1] : key[t][i]; at[t][i] = won ? at[t][i + 1] : at[t][i]; }
            key[t][kKeys - 1] = won ? 0u : key[t][kKeys - 1];
        }
    }
    float p[kTok];
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const uint32_t tok = t0 + t * step;
        p[t] = mine[t] != 0xffffu ? expf(from_ordered(took[t]) - from_ordered(first[t])) : 0.0f;
        if (!kOwn && mine[t] != 0xffffu) atomicOr(&r.mask[mine[t]][tok >> 5], 1u << (tok & 31u));
        if (m.renorm) all[t] = p[t];
    }
#pragma unroll
    for (int t = 0; t < kTok; ++t) all[t] = warp_sum_f(all[t]);
#pragma unroll
    for (int t = 0; t < kTok; ++t) {
        const uint32_t tok = t0 + t * step, place = tok * m.K + lane;
        if (tok < m.T && lane < m.K) {
            const float w = mine[t] != 0xffffu ? p[t] / all[t] : 0.0f;
            if (kOwn) { m.route_e[place] = (uint16_t)(live[t] ? mine[t] : 0xfffeu); m.route_w[place] = w; }
            else { tmp.expert[place] = (uint16_t)mine[t]; tmp.weight[place] = w; }
            if (write) {
                if (m.chosen) m.chosen[place] = mine[t] != 0xffffu ? (int32_t)mine[t] : -1;
                if (m.weights) m.weights[place] = w;
            }
        }
    }
}

// The whole batch's choice by a block.  For a few tokens (one a warp) every block of both kernels makes it for itself, which costs less than a
// kernel of its own in front would; else that has made it (kLoad), a token a warp on as many SMs (64 tokens by every block's sixteen warps
// took 6.5 us in each of the two kernels), and the block only takes it over.
template <int kKeys, int kTok, int kTokens>
__device__ __forceinline__ void route_tokens(const MoeDev &m, Route<kTokens> &r, RouteTemp<kTokens> &tmp, bool write) {
    constexpr uint32_t kWarps = kMoeWarps;
#pragma unroll 1
    for (uint32_t t = threadIdx.x >> 5; t < m.T; t += kWarps * kTok) choose<kKeys, kTok, false>(m, r, tmp, t, kWarps, write);
}
template <bool kLoad, int kTokens>
__device__ __forceinline__ void route(const MoeDev &m, Route<kTokens> &r, RouteTemp<kTokens> &tmp, uint32_t chunk, bool write) {
    constexpr int kEach = HBF_MOE_MAX_EXPERTS / kMoeThreads, kWords = Route<kTokens>::kWords;  // experts a thread in the scan, side by side
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    for (uint32_t i = tid; i < m.E * kWords; i += kMoeThreads) r.mask[0][i] = 0u;
    if (tid < kWords) r.bad[tid] = 0u;
    __syncthreads();
    if (kLoad) {
#pragma unroll 1
        for (uint32_t i = tid; i < m.T * m.K; i += kMoeThreads) {
            uint32_t e = m.route_e[i];
            const float w = m.route_w[i];
            const uint32_t t = div32(i, m.div_k);
            if (e == 0xfffeu) { atomicOr(&r.bad[t >> 5], 1u << (t & 31u)); e = 0xffffu; }
            if (e != 0xffffu) atomicOr(&r.mask[e][t >> 5], 1u << (t & 31u));
            tmp.expert[i] = (uint16_t)e; tmp.weight[i] = w;
        }
    } else if (m.E > 128u) route_tokens<HBF_MOE_MAX_EXPERTS / 32, 1>(m, r, tmp, write);
    else if (kTokens > kMoeWarps && m.T > kMoeWarps) route_tokens<4, kTokens < 4 * kMoeWarps ? 1 : 4>(m, r, tmp, write);
    else route_tokens<4, 1>(m, r, tmp, write);
    __syncthreads();
    // places of the experts in the list of pairs, of those in use, and of the entries: one scan over the experts
    uint32_t count[kEach], a0 = 0u, b0 = 0u, c0 = 0u;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t e = tid * kEach + i;
        count[i] = 0u;
        if (e < m.E) {
#pragma unroll
            for (int w = 0; w < kWords; ++w) count[i] += __popc(r.mask[e][w]);
        }
        a0 += count[i]; b0 += count[i] ? 1u : 0u; c0 += (count[i] + chunk - 1u) / chunk;
    }
    uint32_t a = a0, b = b0, c = c0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t pa = __shfl_up_sync(0xffffffffu, a, o), pb = __shfl_up_sync(0xffffffffu, b, o), pc = __shfl_up_sync(0xffffffffu, c, o);
        if (lane >= (uint32_t)o) { a += pa; b += pb; c += pc; }
    }
    if (lane == 31u) { r.scan[warp][0] = a; r.scan[warp][1] = b; r.scan[warp][2] = c; }
    __syncthreads();
#pragma unroll 1
    for (uint32_t w = 0; w < warp; ++w) { a += r.scan[w][0]; b += r.scan[w][1]; c += r.scan[w][2]; }
    if (tid == kMoeThreads - 1) { r.n_active = b; r.n_entries = c; }
    a -= a0; b -= b0; c -= c0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t e = tid * kEach + i;
        if (e >= m.E) break;
        r.base[e] = (uint16_t)a;
        if (count[i]) r.active[b++] = (uint16_t)e;
#pragma unroll 1
        for (uint32_t k = 0; k < count[i]; k += chunk, ++c) {
            r.expert[c] = (uint16_t)e; r.pair0[c] = (uint16_t)(a + k); r.count[c] = (uint8_t)min(chunk, count[i] - k);
        }
        a += count[i];
    }
    __syncthreads();
#pragma unroll 1
    for (uint32_t i = tid; i < m.T * m.K; i += kMoeThreads) {
        const uint32_t e = tmp.expert[i], t = div32(i, m.div_k);
        if (e == 0xffffu) continue;
        uint32_t at = r.base[e];
#pragma unroll
        for (int w = 0; w < kWords; ++w)
            at += __popc(r.mask[e][w] & ((uint32_t)w < (t >> 5) ? 0xffffffffu : (uint32_t)w == (t >> 5) ? (1u << (t & 31u)) - 1u : 0u));
        r.token[at] = (uint8_t)t; r.weight[at] = tmp.weight[i];
    }
    __syncthreads();
}
static_assert(HBF_MOE_MAX_EXPERTS % kMoeThreads == 0 && HBF_MOE_MAX_TOKENS == 128, "the scan and the masks");

// The layer for more than a few tokens, on tensor memory (moe_tiles.cu).
cudaError_t launch_moe_tiles(const MoeDev &m, bool bf16, uint32_t n_sm, cudaStream_t st);
// Blocks that share a tile of 128 rows of the output, each with a part of the experts.
inline uint32_t moe_groups(uint32_t tokens, uint32_t hidden, uint32_t experts, uint32_t top_k, uint32_t n_sm) {
    const uint32_t tiles = (hidden + 127u) / 128u, pairs = tokens * top_k, most = pairs < experts + pairs / 32u ? pairs : experts + pairs / 32u;
    const uint32_t there = tiles < n_sm ? n_sm / tiles : 1u;
    return there < most ? there : most ? most : 1u;
}

}  // namespace hbf
