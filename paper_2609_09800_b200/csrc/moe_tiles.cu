// The mixture-of-experts layer for more than a few tokens.  With many experts in use the layer is bound by their bytes, and what counts is that
// nothing but the copies stands between HBM and the products: weights go by tensor copies into the swizzled layout that the 5th-generation
// tensor cores read, and 128 rows of them against 16 or 32 tokens are products into tensor memory that one thread issues.  (With m16n8k16
// products fed from registers, as moe_kernels.cu does for a few tokens, instructions bound it: 64 tokens, 837 MB of weights, 257 us.)
//
//   k_moe_choose      the tokens' experts, a token a warp
//   k_moe_up_tiles    up to 64 gate rows and the same up rows of an expert in use, times its tokens: h = w silu(gate) up
//   k_moe_down_tiles  128 rows of the output for all tokens, from a part of the experts: their sums, in the experts' order
//   k_moe_sum         the parts' sums, in their order
#include "moe.cuh"
#include "tensor_memory.cuh"

namespace hbf {

constexpr int kMtTokens = HBF_MOE_MAX_TOKENS, kMtChunk = 32;             // tokens of an expert that an entry takes
constexpr uint32_t kMtA = 128u * 128u, kMtB = kMtChunk * 128u;           // bytes of a stage, 64 of the sum's places: weights; activations (the down product: twice)
struct UpMaps { CUtensorMap rows[3]; };                                  // boxes of 64, 48 and 32 rows: a copy takes its thread 85 cycles, whatever its size
constexpr int kUpStages = 8, kDownStages = 5, kMtLag = 3;
constexpr uint32_t kUpStageBytes = kMtA + kMtB, kDownStageBytes = kMtA + 2u * kMtB;

struct MtShared {
    Route<kMtTokens> route;
    uint64_t full[kUpStages], empty[kUpStages], acc_full[2], acc_empty[2], products_done;
    uint32_t tmem, gave_up, copied;                          // copied: stages whose weights were asked for
};
constexpr uint32_t kUpTilesSmem = 1024u + kUpStages * kUpStageBytes + 2u * kMtChunk * 64u * 4u + sizeof(MtShared);
constexpr uint32_t down_tiles_smem(uint32_t tokens) { return 1024u + kDownStages * kDownStageBytes + tokens * 512u + sizeof(MtShared); }
static_assert(kUpTilesSmem <= 227 * 1024 && down_tiles_smem(kMtTokens) <= 227 * 1024 && sizeof(RouteTemp<kMtTokens>) <= kDownStages * kDownStageBytes, "shared memory");

__device__ __forceinline__ void tensor_copy3(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t y, int32_t z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Both kernels' blocks begin alike: barriers, tensor memory (two times 64 columns), the choice.  Warps 0 to 3: a lane of tensor memory a thread;
// 4 to 7: the activations' 16-byte copies; 8: tensor copies; 9: products; all 16 take the choice over.
template <int kStages>
__device__ __forceinline__ void begin_tiles(const MoeDev &m, MtShared &sh, unsigned char *tmp) {
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) { bar_init(smem_addr(&sh.full[i]), 129u); bar_init(smem_addr(&sh.empty[i]), 1u); }
        for (int i = 0; i < 2; ++i) { bar_init(smem_addr(&sh.acc_full[i]), 1u); bar_init(smem_addr(&sh.acc_empty[i]), 128u); }
        bar_init(smem_addr(&sh.products_done), 1u);
        sh.gave_up = sh.copied = 0u;
        bar_init_done();
    }
    if ((threadIdx.x >> 5) == 9u) { tensor_alloc(smem_addr(&sh.tmem), 128u); tensor_fence_before(); }
    route<true>(m, sh.route, *reinterpret_cast<RouteTemp<kMtTokens> *>(tmp), kMtChunk, false);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");         // the choice's memory is the ring's now
    __syncthreads();
    tensor_fence_after();
}
// Where a wait was given up, weights may be on their way: the stages that were asked for get the arrivals of the activations' threads that did not come
// to them (a stage is asked for only when the one a round before it was used), so that their barriers end when the copies have.  told: stages
// that this thread, of warps 4 to 7, said were there.
template <int kStages>
__device__ __forceinline__ void end_tiles(MtShared &sh, bool live, uint32_t told) {
    const uint32_t warp = threadIdx.x >> 5;
    tensor_fence_before();
    if (__syncthreads_or(live ? 0 : 1)) {
        const uint32_t copied = *(volatile uint32_t *)&sh.copied;
        if (warp >= 4u && warp < 8u) for (uint32_t n = told; n < copied; ++n) bar_arrive(smem_addr(&sh.full[n % kStages]));
        if (warp == 8u) for (uint32_t n = copied > (uint32_t)kStages ? copied - kStages : 0u; n < copied; ++n) wait_for_own(smem_addr(&sh.full[n % kStages]), (n / kStages) & 1u);
    }
    if (warp == 9u) { __syncwarp(); tensor_fence_after(); tensor_free(sh.tmem, 128u); }
}
// Nothing of the block is on its way when it gives its tensor memory back.
__device__ __forceinline__ void end_products(MtShared &sh) {
    products_arrive(smem_addr(&sh.products_done));
    wait_for_own(smem_addr(&sh.products_done), 0u);
}

// The activations' side of a ring: stage g's copies are issued by `copy(stage address)`; they are said to be there kMtLag stages later, and before
// a wait for a free stage.  stage: false when a wait was given up.
template <int kStages, uint32_t kBytes>
struct Gather {
    uint32_t ring, full, empty, polls;
    uint32_t gave_up;
    bool live;
    uint32_t g = 0u, told = 0u;
    __device__ __forceinline__ void tell() {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        bar_arrive(full + (told % kStages) * 8u);
        ++told;
    }
    template <class F> __device__ __forceinline__ bool stage(F copy) {
        if (g >= (uint32_t)kMtLag) { copy_wait<kMtLag - 1>(); tell(); }
        live = bar_wait(empty + (g % kStages) * 8u, ((g / kStages) & 1u) ^ 1u, live, polls, gave_up);
        if (!live) return false;
        copy(ring + (g % kStages) * kBytes + kMtA);
        copy_commit();
        ++g;
        return true;
    }
    __device__ __forceinline__ void finish() {
        copy_wait<0>();
        while (live && told < g) tell();
    }
};

__global__ void __launch_bounds__(32)
k_moe_choose(const __grid_constant__ MoeDev m) {
    pdl_trigger();
    Route<32> *none = nullptr;
    RouteTemp<32> *none_too = nullptr;
    if (m.E <= 128u) choose<4, 1, true>(m, *none, *none_too, blockIdx.x, 1u, true);
    else choose<HBF_MOE_MAX_EXPERTS / 32, 1, true>(m, *none, *none_too, blockIdx.x, 1u, true);
}

template <class Ty, bool kBf16>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_up_tiles(const __grid_constant__ MoeDev m, const __grid_constant__ UpMaps maps) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t ring = smem_addr(smem);
    float *ex = reinterpret_cast<float *>(smem + kUpStages * kUpStageBytes);                // [2][token][64]: the up rows' sums
    MtShared &sh = *reinterpret_cast<MtShared *>(smem + kUpStages * kUpStageBytes + 2u * kMtChunk * 64u * 4u);
    const Route<kMtTokens> &r = sh.route;
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    pdl_wait();                                              // the choice is made; it is for the kernel behind this one, too
    pdl_trigger();
    begin_tiles<kUpStages>(m, sh, smem);
    // rows of gate and up that an item takes: of 64, 48 and 32 those with which the blocks are done first
    uint32_t rows = 64u, best = 0xffffffffu;
#pragma unroll
    for (uint32_t c = 64u; c >= 32u; c -= 16u) {
        const uint32_t items = r.n_entries * ((m.I + c - 1u) / c), cost = (items + gridDim.x - 1u) / gridDim.x * c;
        if (cost < best) { best = cost; rows = c; }
    }
    const uint32_t tiles = (m.I + rows - 1u) / rows, n_items = r.n_entries * tiles, chunks = (m.D + 63u) / 64u;
    const uint32_t full = smem_addr(sh.full), empty = smem_addr(sh.empty), acc_full = smem_addr(sh.acc_full), acc_empty = smem_addr(sh.acc_empty);
    bool live = m.polls != 0u;
    uint32_t told = 0u;
    auto wait = [&](uint32_t bar, uint32_t parity) { live = bar_wait(bar, parity, live, m.polls, smem_addr(&sh.gave_up)); };
    if (warp == 8u) {
        if (lane == 0u) {
            uint32_t g = 0u;
            const CUtensorMap *map = &maps.rows[(64u - rows) / 16u];
            for (uint32_t item = blockIdx.x; item < n_items && live; item += gridDim.x) {
                const uint32_t en = item / tiles, i0 = (item - en * tiles) * rows, e = r.expert[en];
                for (uint32_t c = 0; c < chunks; ++c, ++g) {
                    const uint32_t s = g % kUpStages, at = ring + s * kUpStageBytes, bar = full + s * 8u;
                    wait(empty + s * 8u, ((g / kUpStages) & 1u) ^ 1u);
                    if (!live) break;
                    bar_arrive_bytes(bar, rows * 256u);
                    tensor_copy3(at, map, (int32_t)(c * 64u), (int32_t)i0, (int32_t)e, bar);
                    tensor_copy3(at + 8192u, map, (int32_t)(c * 64u), (int32_t)(m.I + i0), (int32_t)e, bar);
                }
            }
            sh.copied = g;
        }
    } else if (warp >= 4u && warp < 8u) {
        const uint32_t t = tid - 128u, col = t & 7u, row = t >> 3, to = row * 128u + ((col ^ (row & 7u)) * 16u);
        Gather<kUpStages, kUpStageBytes> in{ring, full, empty, m.polls, smem_addr(&sh.gave_up), live};
        for (uint32_t item = blockIdx.x; item < n_items && in.live; item += gridDim.x) {
            const uint32_t en = item / tiles, n = r.count[en], pair0 = r.pair0[en];
            const uint16_t *x0 = row < n ? m.x + (int64_t)r.token[pair0 + row] * m.x_stride : nullptr;
            const uint16_t *x1 = row + 16u < n ? m.x + (int64_t)r.token[pair0 + row + 16u] * m.x_stride : nullptr;
            for (uint32_t c = 0; c < chunks; ++c)
                if (!in.stage([&](uint32_t at) {
                    const uint32_t k = c * 64u + col * 8u;
                    const bool is = k < m.D;
                    if (x0) copy_async16_shared(at + to, is ? x0 + k : m.x, is);
                    if (x1) copy_async16_shared(at + 2048u + to, is ? x1 + k : m.x, is);
                })) break;
        }
        in.finish();
        live = in.live; told = in.told;
    } else if (warp == 9u) {
        if (lane == 0u) {
            uint32_t g = 0u, it = 0u;
            const TileDesc a0(ring, 16u, 1024u), b0(ring + kMtA, 16u, 1024u);
            for (uint32_t item = blockIdx.x; item < n_items && live; item += gridDim.x, ++it) {
                const uint32_t n = r.count[item / tiles], buf = it & 1u, id = product_desc(kBf16, false, 128u, n <= 16u ? 16u : 32u);
                wait(acc_empty + buf * 8u, ((it >> 1) & 1u) ^ 1u);
                tensor_fence_after();
                for (uint32_t c = 0; c < chunks; ++c, ++g) {
                    const uint32_t s = g % kUpStages;
                    wait(full + s * 8u, (g / kUpStages) & 1u);
                    if (!live) break;
                    tensor_fence_after();
                    TileDesc a = a0, b = b0;
                    a.lo += s * (kUpStageBytes >> 4); b.lo += s * (kUpStageBytes >> 4);
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k) product_ss(sh.tmem + buf * 32u, a.at(k * 32u), b.at(k * 32u), id, c || k ? 1u : 0u);
                    products_arrive(empty + s * 8u);
                }
                if (live) products_arrive(acc_full + buf * 8u);
            }
            end_products(sh);
        }
        __syncwarp();
    } else if (warp < 4u) {
        uint32_t it = 0u;
        for (uint32_t item = blockIdx.x; item < n_items; item += gridDim.x, ++it) {
            const uint32_t en = item / tiles, i0 = (item - en * tiles) * rows, n = r.count[en], pair0 = r.pair0[en], buf = it & 1u;
            wait(acc_full + buf * 8u, (it >> 1) & 1u);
            __syncwarp();
            tensor_fence_after();
            uint32_t v[32];
            tensor_load(sh.tmem + buf * 32u + ((warp * 32u) << 16), v);   // (columns past the tokens hold anything)
            tensor_loaded(v);
            tensor_fence_before();
            bar_arrive(acc_empty + buf * 8u);
            float *up = ex + buf * (kMtChunk * 64u);
            const uint32_t row = (warp & 1u) * 32u + lane;
            if (warp >= 2u) {
#pragma unroll
                for (int c = 0; c < kMtChunk; ++c) if ((uint32_t)c < n) up[c * 64 + row] = __uint_as_float(v[c]);
            }
            barrier_of(1, 128);                              // (the buffer after next is written behind the next one's barrier)
            const bool sound = live && !ld_flag(smem_addr(&sh.gave_up));          // (here: the other rows' threads may have given up)
            if (warp < 2u && row < rows && i0 + row < m.I) {
#pragma unroll
                for (int c = 0; c < kMtChunk; ++c)
                    if ((uint32_t)c < n) {
                        const float g = __uint_as_float(v[c]), u = up[c * 64 + row];
                        const float h = sound ? r.weight[pair0 + c] * (g / (1.0f + expf(-g)) * u) : __int_as_float(0x7fc00000);
                        // (held as the sum of two numbers: see k_moe_up)
                        const typename Ty::type hi = Ty::from(h), lo = Ty::from(isfinite(h) ? h - Ty::to(hi) : 0.0f);
                        const size_t at = (size_t)(pair0 + c) * m.I + i0 + row;
                        reinterpret_cast<typename Ty::type *>(m.h_hi)[at] = hi;
                        reinterpret_cast<typename Ty::type *>(m.h_lo)[at] = isfinite(Ty::to(hi)) ? lo : Ty::from(0.0f);
                    }
            }
        }
    }
    end_tiles<kUpStages>(sh, live, told);
}

template <class Ty, bool kBf16>
__global__ void __launch_bounds__(kMoeThreads, 1)
k_moe_down_tiles(const __grid_constant__ MoeDev m, const __grid_constant__ CUtensorMap w_map) {
    extern __shared__ unsigned char smem_raw[];
    unsigned char *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t ring = smem_addr(smem);
    float *sums = reinterpret_cast<float *>(smem + kDownStages * kDownStageBytes);          // [token][128]
    MtShared &sh = *reinterpret_cast<MtShared *>(smem + kDownStages * kDownStageBytes + m.T * 512u);
    const Route<kMtTokens> &r = sh.route;
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    pdl_trigger();
    begin_tiles<kDownStages>(m, sh, smem);
    const uint32_t d_tiles = (m.D + 127u) / 128u, group = blockIdx.x / d_tiles, d0 = (blockIdx.x - group * d_tiles) * 128u, chunks = (m.I + 63u) / 64u;
    const uint32_t en0 = r.n_entries * group / m.groups, en1 = r.n_entries * (group + 1u) / m.groups;
    const uint32_t full = smem_addr(sh.full), empty = smem_addr(sh.empty), acc_full = smem_addr(sh.acc_full), acc_empty = smem_addr(sh.acc_empty);
    bool live = m.polls != 0u;
    uint32_t told = 0u;
    auto wait = [&](uint32_t bar, uint32_t parity) { live = bar_wait(bar, parity, live, m.polls, smem_addr(&sh.gave_up)); };
    if (warp == 8u) {                                        // weights: as far ahead as the ring goes while the kernel before still runs
        if (lane == 0u) {
            uint32_t g = 0u;
            for (uint32_t en = en0; en < en1 && live; ++en)
                for (uint32_t c = 0; c < chunks; ++c, ++g) {
                    const uint32_t s = g % kDownStages, bar = full + s * 8u;
                    wait(empty + s * 8u, ((g / kDownStages) & 1u) ^ 1u);
                    if (!live) break;
                    bar_arrive_bytes(bar, kMtA);
                    tensor_copy3(ring + s * kDownStageBytes, &w_map, (int32_t)(c * 64u), (int32_t)d0, (int32_t)r.expert[en], bar);
                }
            sh.copied = g;
        }
    } else if (warp >= 4u && warp < 8u) {
        const uint32_t t = tid - 128u, col = t & 7u, row = t >> 3, to = row * 128u + ((col ^ (row & 7u)) * 16u);
        Gather<kDownStages, kDownStageBytes> in{ring, full, empty, m.polls, smem_addr(&sh.gave_up), live};
        pdl_wait();
        for (uint32_t en = en0; en < en1 && in.live; ++en) {
            const uint32_t n = r.count[en], pair0 = r.pair0[en];
            const size_t h0 = (size_t)(pair0 + row) * m.I, h1 = (size_t)(pair0 + row + 16u) * m.I;
            const bool is0 = row < n, is1 = row + 16u < n;
            const uint32_t second = n <= 16u ? 2048u : kMtB; // rows 16 or 32 and on: the second numbers
            for (uint32_t c = 0; c < chunks; ++c)
                if (!in.stage([&](uint32_t at) {
                    const uint32_t k = c * 64u + col * 8u;
                    const bool is = k < m.I;
                    const size_t a = is ? h0 + k : 0u, b = is ? h1 + k : 0u;
                    if (is0) { copy_async16(at + to, m.h_hi + a, is); copy_async16(at + second + to, m.h_lo + a, is); }
                    if (is1) { copy_async16(at + 2048u + to, m.h_hi + b, is); copy_async16(at + second + 2048u + to, m.h_lo + b, is); }
                })) break;
        }
        in.finish();
        live = in.live; told = in.told;
    } else if (warp == 9u) {
        if (lane == 0u) {
            uint32_t g = 0u, it = 0u;
            const TileDesc a0(ring, 16u, 1024u), b0(ring + kMtA, 16u, 1024u);
            for (uint32_t en = en0; en < en1 && live; ++en, ++it) {
                // first and second numbers are columns of one product (a product of 128 rows takes 60 cycles up to 64 columns)
                const uint32_t buf = it & 1u, id = product_desc(kBf16, false, 128u, r.count[en] <= 16u ? 32u : 64u);
                wait(acc_empty + buf * 8u, ((it >> 1) & 1u) ^ 1u);
                tensor_fence_after();
                for (uint32_t c = 0; c < chunks; ++c, ++g) {
                    const uint32_t s = g % kDownStages;
                    wait(full + s * 8u, (g / kDownStages) & 1u);
                    if (!live) break;
                    tensor_fence_after();
                    TileDesc a = a0, b = b0;
                    a.lo += s * (kDownStageBytes >> 4); b.lo += s * (kDownStageBytes >> 4);
#pragma unroll
                    for (uint32_t k = 0; k < 4u; ++k) product_ss(sh.tmem + buf * 64u, a.at(k * 32u), b.at(k * 32u), id, c || k ? 1u : 0u);
                    products_arrive(empty + s * 8u);
                }
                if (live) products_arrive(acc_full + buf * 8u);
            }
            end_products(sh);
        }
        __syncwarp();
    } else if (warp < 4u) {
        const uint32_t row = tid;                            // a row of the output a thread: its sums are nobody else's
        for (uint32_t t = 0; t < m.T; ++t) sums[t * 128u + row] = 0.0f;
        uint32_t it = 0u;
        for (uint32_t en = en0; en < en1; ++en, ++it) {
            const uint32_t n = r.count[en], pair0 = r.pair0[en], buf = it & 1u;
            wait(acc_full + buf * 8u, (it >> 1) & 1u);
            __syncwarp();
            tensor_fence_after();
            const uint32_t from = sh.tmem + buf * 64u + ((warp * 32u) << 16);
            for (uint32_t c0 = 0; c0 < n; c0 += 16u) {
                uint32_t v[16], w[16];
                tensor_load16(from + c0, v);
                tensor_load16(from + (n <= 16u ? 16u : 32u) + c0, w);
#pragma unroll
                for (int c = 0; c < 16; ++c) if (c0 + c < n) sums[r.token[pair0 + c0 + c] * 128u + row] += __uint_as_float(v[c]) + __uint_as_float(w[c]);
            }
            tensor_fence_before();
            bar_arrive(acc_empty + buf * 8u);
        }
        const bool sound = live && !ld_flag(smem_addr(&sh.gave_up));
        if (d0 + row < m.D)
            for (uint32_t t = 0; t < m.T; ++t) {
                const bool bad = !sound || (r.bad[t >> 5] >> (t & 31u)) & 1u;
                m.part[((size_t)group * m.T + t) * m.D + d0 + row] = bad ? __int_as_float(0x7fc00000) : sums[t * 128u + row];
            }
    }
    end_tiles<kDownStages>(sh, live, told);
}

template <class Ty>
__global__ void __launch_bounds__(256)
k_moe_sum(const __grid_constant__ MoeDev m) {
    const uint64_t pairs = (uint64_t)m.T * (m.D / 2u), i = (uint64_t)blockIdx.x * 256u + threadIdx.x;
    pdl_wait();
    if (i >= pairs) return;
    const uint32_t t = (uint32_t)(i / (m.D / 2u)), d = (uint32_t)(i - (uint64_t)t * (m.D / 2u)) * 2u;
    float a = 0.0f, b = 0.0f;
    const float *from = m.part + (size_t)t * m.D + d;
#pragma unroll 8
    for (uint32_t g = 0; g < m.groups; ++g) {
        const float2 v = __ldcg(reinterpret_cast<const float2 *>(from + (size_t)g * m.T * m.D));
        a += v.x; b += v.y;
    }
    typename Ty::type *to = reinterpret_cast<typename Ty::type *>(m.out) + (int64_t)t * m.out_stride + d;
    to[0] = Ty::from(a); to[1] = Ty::from(b);
}

static bool weights_map(CUtensorMap *map, const void *base, uint64_t k, uint64_t rows, const MoeDev &m, bool bf16, uint32_t box) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {k, rows, m.E}, strides[2] = {k * 2u, (cuuint64_t)m.expert_stride * 2u};
    const cuuint32_t boxes[3] = {64u, box, 1u}, steps[3] = {1u, 1u, 1u};
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Ty, bool kBf16>
static cudaError_t launch_tiles(const MoeDev &m, uint32_t n_sm, cudaStream_t st) {
    UpMaps up_maps;
    CUtensorMap down_map;
    for (uint32_t i = 0; i < 3u; ++i) if (!weights_map(&up_maps.rows[i], m.experts, m.D, 2ull * m.I, m, kBf16, 64u - 16u * i)) return cudaErrorInvalidValue;
    if (!weights_map(&down_map, m.experts + 2ull * m.I * m.D, m.I, m.D, m, kBf16, 128u)) return cudaErrorInvalidValue;
    const auto up = k_moe_up_tiles<Ty, kBf16>;
    const auto down = k_moe_down_tiles<Ty, kBf16>;
    cudaError_t e = ensure_dyn_smem((const void *)up, kUpTilesSmem);
    if (e == cudaSuccess) e = ensure_dyn_smem((const void *)down, down_tiles_smem(kMtTokens));
    if (e != cudaSuccess) return e;
    k_moe_choose<<<m.T, 32, 0, st>>>(m);
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    g_kernel_launches += 4;
    // k_moe_down_tiles may begin when every block of the up kernel has let it, which each does behind its own pdl_wait: the choice, written one kernel
    // before that, is there, and is read in front of the wait.  What the up kernel writes is read behind it (warps 4 to 7 of every block).
    if ((e = launch_pdl(up, n_sm, kMoeThreads, kUpTilesSmem, st, m, up_maps)) != cudaSuccess) return e;
    if ((e = launch_pdl(down, (m.D + 127u) / 128u * m.groups, kMoeThreads, down_tiles_smem(m.T), st, m, down_map)) != cudaSuccess) return e;
    return launch_pdl(k_moe_sum<Ty>, (unsigned)(((uint64_t)m.T * (m.D / 2u) + 255u) / 256u), 256, 0, st, m);
}
cudaError_t launch_moe_tiles(const MoeDev &m, bool bf16, uint32_t n_sm, cudaStream_t st) {
    return bf16 ? launch_tiles<Bf16, true>(m, n_sm, st) : launch_tiles<Fp16, false>(m, n_sm, st);
}

}  // namespace hbf
