// The shared prefix for many rows: tiles of 128 query rows (of any requests) against 128 keys at a time on the 5th-generation tensor
// cores.  For a tile of rows and one of keys: S = Q K^T into tensor memory, weights P = exp2(S - z) from there back into it (over S, in
// the values' type), O += P V with P read from tensor memory.  A block has two tiles of rows, so that one tile's products run while the
// other's weights are worked out, and the keys are read once for 256 rows.
//
// Warps 0 to 7 and 8 to 15: the first and the second tile of rows, two threads a row (the time from a tile's scores to its weights is part of
// the chain that bounds the kernel: with one thread a row it was 2,700 cycles of 5,000 for a tile of keys).  16 to 19: keys and values from
// their pages into the swizzled layout that the tensor cores read: a tensor copy for every stretch of slots of a page where pages are
// multiples of eight slots, else, and in a tile that the prefix ends in (behind its end there must be zeros), 16 bytes a thread at a
// time, which take 1,150 cycles a tile.  20: one thread issues the products.
#include "attention.cuh"
#include "tensor_memory.cuh"

namespace hbf {

constexpr int kPfThreads = 24 * 32, kPfRowThreads = 16 * 32, kPfTile = 128, kPfSlots = 4;
constexpr float kPfGrow = 8.0f;                              // sums are scaled again only when a row's maximum has grown by more (in powers of two)

// What lies in shared memory behind the tiles.
struct PfShared {
    uint64_t kv_full[kPfSlots], kv_empty[kPfSlots], q_full, s_full[2], p_full[2], o_full[2], products_done;
    int64_t place[2][kPfTile];                               // offset of each key of a tile; -1: none
    float other[2][2][kPfTile];                              // what the two threads of a row tell each other
    uint32_t tmem, bad, gave_up, most_copied;
};
template <int D> constexpr uint32_t kPfTileBytes = kPfTile * D * 2;
template <int D> constexpr uint32_t pf_smem() { return (2u + kPfSlots) * kPfTileBytes<D> + sizeof(PfShared) + 1024u; }

// A box of 64 values by some slots of one page and head, to the swizzled layout.
__device__ __forceinline__ void tensor_copy(uint32_t dst, const CUtensorMap *map, int32_t x, int32_t slot, int32_t head, int32_t page, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(slot), "r"(head), "r"(page), "r"(bar) : "memory");
}

// Two numbers at a time.
__device__ __forceinline__ uint64_t two_of(float a, float b) { uint64_t v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); return v; }
__device__ __forceinline__ void of_two(uint64_t v, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) { uint64_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) { uint64_t d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ float max3_nan(float a, float b, float c) { float d; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float min3_nan(float a, float b, float c) { float d; asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }

template <class Ty, int D, bool kBf16>
__global__ void __launch_bounds__(kPfThreads, 1)
k_prefix_tiles(const __grid_constant__ AttnDev p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, uint32_t box) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
    PfShared &sh = *reinterpret_cast<PfShared *>(smem_raw + (base - smem_addr(smem_raw)) + (2u + kPfSlots) * kPfTileBytes<D>);
    constexpr uint32_t kBytes = kPfTileBytes<D>;
    const uint32_t q_at = base, kv_at = base + 2u * kBytes;
    const uint32_t tid = threadIdx.x, lane = lane_id(), warp = tid >> 5;
    pdl_trigger();
    if (tid == (uint32_t)kPfRowThreads && box) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    // the piece: `row_tiles` counts pairs of tiles here
    uint32_t item = blockIdx.x;
    const uint32_t piece = item % p.prefix_pieces; item /= p.prefix_pieces;
    const uint32_t pair = item % p.row_tiles, head = item / p.row_tiles;
    const uint32_t begin = piece * p.prefix_chunk, end = min(p.prefix_len, begin + p.prefix_chunk);
    const uint32_t n_tiles = (end - begin + kPfTile - 1u) / kPfTile, all_rows = p.B * p.G, row0 = pair * 2u * kPfTile;
    const bool two = row0 + kPfTile < all_rows;
    if (tid == 0) {
        for (int i = 0; i < kPfSlots; ++i) { bar_init(smem_addr(&sh.kv_full[i]), 128u); bar_init(smem_addr(&sh.kv_empty[i]), 1u); }
        bar_init(smem_addr(&sh.q_full), 128u);
        for (int t = 0; t < 2; ++t) { bar_init(smem_addr(&sh.s_full[t]), 1u); bar_init(smem_addr(&sh.p_full[t]), 256u); bar_init(smem_addr(&sh.o_full[t]), 1u); }
        bar_init(smem_addr(&sh.products_done), 1u);
        sh.bad = sh.most_copied = 0u;
        sh.gave_up = p.polls == 0u ? 1u : 0u;
        bar_init_done();
    }
    if (warp == 20u) {
        tensor_alloc(smem_addr(&sh.tmem), 512u);
        tensor_fence_before();
    }
    __syncthreads();
    tensor_fence_after();
    const uint32_t tmem = sh.tmem;                           // S (and P) of both tiles, then O of both
    bool live = true;                                        // (without polls: set below, where it costs nothing; the rows' threads see gave_up)
    auto wait = [&](uint32_t bar, uint32_t parity) { live = bar_wait(bar, parity, live, p.polls, smem_addr(&sh.gave_up)); };
    // boxes of `box` slots (0: none): whole tiles; the stages of keys or values that this thread's warp has asked for (copies' warps)
    const uint32_t whole = box ? (end - begin) / kPfTile : 0u;
    uint32_t copied = 0u;

    // the registers that the block was launched with, 80 a thread, as 96 for the weights, 56 for the copies, 40 for the products
    if (warp >= 16u && warp < 20u) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        live = p.polls != 0u;
        // ---- keys and values: eight lanes a row of 128 bytes
        const uint32_t t = tid - (uint32_t)kPfRowThreads, w4 = warp - 16u, col = t & 7u, row = t >> 3;
        auto swizzled = [&](uint32_t r) { return r * 128u + ((col ^ (r & 7u)) * 16u); };
        auto find = [&](uint32_t i) {                        // thread t: key t of tile i
            const uint32_t k = begin + i * kPfTile + t;
            int64_t at = -1;
            if (k < end) {
                const uint32_t n = div32(k, p.div_page);
                const int32_t page = p.prefix_pages[n];
                if (!key_place(p, page, k - n * p.page_tokens, at)) { at = -1; sh.bad = 1u; }
            }
            sh.place[i & 1u][t] = at;
        };
        auto arrive = [&](uint32_t bar) { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); bar_arrive(bar); };
        // warp w takes the boxes w, w + 4, ...
        const uint32_t boxes = box ? kPfTile / box : 0u, my_boxes = boxes > w4 ? (boxes - w4 + 3u) / 4u : 0u;
        int32_t page = 0;                                    // lane l: that of this warp's box l
        uint32_t slot0 = 0u;
        auto look = [&](uint32_t i) {
            if (lane >= my_boxes || i >= whole) return;
            const uint32_t k = begin + i * kPfTile + (w4 + lane * 4u) * box, n = div32(k, p.div_page);
            page = p.prefix_pages[n]; slot0 = k - n * p.page_tokens;
        };
        look(0);
        for (uint32_t h = 0; h < (two ? 2u : 1u); ++h)
#pragma unroll
            for (uint32_t r = row; r < kPfTile; r += 16u) {
                const uint32_t n = row0 + h * kPfTile + r;
                const bool ok = n < all_rows;
                const uint32_t b = div32(n, p.div_g), g = n - b * p.G;
                const uint16_t *src = ok ? p.q + (int64_t)b * p.q_row + (int64_t)(head * p.G + g) * p.q_head + col * 8u : p.q;
#pragma unroll
                for (int x = 0; x < D / 64; ++x) copy_async16(q_at + h * kBytes + x * 16384u + swizzled(r), ok ? src + x * 64 : src, ok);
            }
        copy_commit();
        if (whole) {
            for (uint32_t i = 0; i < whole && live; ++i) {
                if (lane < my_boxes && (uint32_t)page >= p.n_pages) { sh.bad = 1u; page = -1; }        // (such a box is zeros)
                const int32_t page_now = page;
                const uint32_t slot_now = slot0;
                look(i + 1u);
#pragma unroll 1
                for (uint32_t kv = 0; kv < 2u; ++kv) {
                    const uint32_t n = 2u * i + kv, slot = n % kPfSlots, full = smem_addr(&sh.kv_full[slot]);
                    wait(smem_addr(&sh.kv_empty[slot]), ((n / kPfSlots) & 1u) ^ 1u);
                    live = __all_sync(0xffffffffu, live);
                    if (!live) break;
                    if (lane == 0u) bar_arrive_bytes(full, my_boxes * box * D * 2u);
                    else bar_arrive(full);
                    copied = n + 1u;
                    for (uint32_t j = 0; j < my_boxes; ++j) {
                        const int32_t pg = __shfl_sync(0xffffffffu, page_now, j);
                        const int32_t sl = (int32_t)__shfl_sync(0xffffffffu, slot_now, j);
                        if (lane == 0u) {
                            const uint32_t dst = kv_at + slot * kBytes + (w4 + j * 4u) * box * 128u;
#pragma unroll
                            for (int x = 0; x < D / 64; ++x) tensor_copy(dst + x * 16384u, kv ? &v_map : &k_map, x * 64, sl, (int32_t)head, pg, full);
                        }
                    }
                    if (n == 0u) { copy_wait<0>(); arrive(smem_addr(&sh.q_full)); }
                }
            }
        }
        if (whole < n_tiles) {
            find(whole);
            barrier_of(1, 128);
            for (uint32_t i = whole; i < n_tiles; ++i) {
                if (i + 1u < n_tiles) find(i + 1u);
                for (uint32_t kv = 0; kv < 2u; ++kv) {
                    const uint32_t n = 2u * i + kv, slot = n % kPfSlots, first = 2u * whole;
                    // what has come is said to be there before the wait for a free slot, which needs it to be used
                    if (n == 1u && live) { copy_wait<1>(); arrive(smem_addr(&sh.q_full)); }
                    if (n >= first + 2u && live) { copy_wait<1>(); arrive(smem_addr(&sh.kv_full[(n - 2u) % kPfSlots])); }
                    wait(smem_addr(&sh.kv_empty[slot]), ((n / kPfSlots) & 1u) ^ 1u);
                    if (!live) continue;                     // (to the barriers that the four warps meet at)
                    copied = n + 1u;
                    const uint32_t dst = kv_at + slot * kBytes;
                    const uint16_t *src = (kv ? p.v : p.k) + (int64_t)head * p.head_stride + col * 8u;
#pragma unroll
                    for (uint32_t r0 = 0; r0 < kPfTile; r0 += 16u) {
                        const int64_t at = sh.place[i & 1u][r0 + row];
                        const uint16_t *from = at >= 0 ? src + at : p.k;
#pragma unroll
                        for (int x = 0; x < D / 64; ++x) copy_async16(dst + x * 16384u + swizzled(r0 + row), at >= 0 ? from + x * 64 : from, at >= 0);
                    }
                    copy_commit();
                }
                barrier_of(1, 128);                          // the next tile's places are there, this one's are done with
            }
            copy_wait<1>(); if (live) arrive(smem_addr(&sh.kv_full[(2u * n_tiles - 2u) % kPfSlots]));
            copy_wait<0>(); if (live) arrive(smem_addr(&sh.kv_full[(2u * n_tiles - 1u) % kPfSlots]));
        }
        copy_wait<0>();
    } else if (warp >= 20u) {
        // ---- the products
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        if (warp == 20u && lane == 0u) {
            live = p.polls != 0u;
            const uint32_t id_s = product_desc(kBf16, false, 128u, 128u), id_o = product_desc(kBf16, true, 128u, D);
            const uint32_t tiles = two ? 2u : 1u;
            const uint32_t s_full = smem_addr(sh.s_full), o_full = smem_addr(sh.o_full);
            const TileDesc q0(q_at, 16u, 1024u), kv0(kv_at, 16u, 1024u), v0(kv_at, 16384u, 1024u);
            // (one thread issues a product every 64 cycles: what can be is worked out before)
            auto scores = [&](uint32_t t, uint32_t slot) {
                TileDesc q = q0, k0 = kv0;
                q.lo += t * (kBytes >> 4); k0.lo += slot * (kBytes >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    product_ss(tmem + t * 128u, q.at((k >> 2) * 16384u + (k & 3) * 32u), k0.at((k >> 2) * 16384u + (k & 3) * 32u), id_s, k ? 1u : 0u);
                products_arrive(s_full + t * 8u);
            };
            auto values = [&](uint32_t t, uint32_t slot, uint32_t add) {
                TileDesc v = v0;
                v.lo += slot * (kBytes >> 4);
                const uint32_t d = tmem + 256u + t * 128u, a = tmem + t * 128u;
#pragma unroll
                for (int k = 0; k < kPfTile / 16; ++k) product_ts(d, a + k * 8u, v.at(k * 2048u), id_o, k ? 1u : add);
                products_arrive(o_full + t * 8u);
            };
            wait(smem_addr(&sh.q_full), 0u);
            wait(smem_addr(&sh.kv_full[0]), 0u);
            if (live) {
                tensor_fence_after();
                for (uint32_t t = 0; t < tiles; ++t) scores(t, 0u);
                products_arrive(smem_addr(&sh.kv_empty[0]));
            }
            for (uint32_t i = 0; i < n_tiles && live; ++i) {
                const uint32_t nv = 2u * i + 1u, sv = nv % kPfSlots, nk = 2u * i + 2u, sk = nk % kPfSlots;
                const bool more = i + 1u < n_tiles;
                wait(smem_addr(&sh.kv_full[sv]), (nv / kPfSlots) & 1u);
                if (more) wait(smem_addr(&sh.kv_full[sk]), (nk / kPfSlots) & 1u);
                for (uint32_t t = 0; t < tiles; ++t) {
                    wait(smem_addr(&sh.p_full[t]), i & 1u);
                    if (!live) break;
                    tensor_fence_after();
                    values(t, sv, i ? 1u : 0u);
                    if (more) scores(t, sk);
                }
                if (!live) break;
                products_arrive(smem_addr(&sh.kv_empty[sv]));
                if (more) products_arrive(smem_addr(&sh.kv_empty[sk]));
            }
            // nothing of this block is on its way when it gives its memory back
            products_arrive(smem_addr(&sh.products_done));
            wait_for_own(smem_addr(&sh.products_done), 0u);
        }
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 96;");
        const uint32_t t = warp >> 3, half = (warp >> 2) & 1u, r = (warp & 3u) * 32u + lane;
        if (t == 0u || two) {
            // ---- weights: half a row a thread
            constexpr int kHalf = kPfTile / 2;
            const uint32_t lanes = ((warp & 3u) * 32u) << 16, s_at = tmem + t * 128u + lanes, o_at = tmem + 256u + t * 128u + half * (D / 2) + lanes;
            const float scale = p.scale_log2, lift = kBf16 ? 0.0f : 7.0f;     // weights are at most 2^8, in fp16 2^15
            const uint64_t scales = two_of(scale, scale);
            float m = -INFINITY, l = 0.0f;
            for (uint32_t i = 0; i < n_tiles; ++i) {
                wait(smem_addr(&sh.s_full[t]), i & 1u);
                __syncwarp();
                tensor_fence_after();
                const uint32_t left = min((uint32_t)kPfTile, end - begin - i * kPfTile), valid = left > half * kHalf ? min(left - half * kHalf, (uint32_t)kHalf) : 0u;
                uint32_t v[2][32];
                tensor_load(s_at + half * kHalf, v[0]);
                tensor_load(s_at + half * kHalf + 32u, v[1]);
                tensor_loaded(v[0]);
                tensor_loaded(v[1]);
                if (valid < (uint32_t)kHalf) {               // behind the prefix's end: the score that weighs nothing
#pragma unroll
                    for (int k = 0; k < kHalf; ++k) if ((uint32_t)k >= valid) v[k / 32][k % 32] = __float_as_uint(scale < 0.0f ? INFINITY : -INFINITY);
                }
                float e[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) e[c] = __uint_as_float(v[c / 2][(c % 2) * 16]);
                if (scale >= 0.0f) {
#pragma unroll
                    for (int k = 1; k < 15; k += 2)
#pragma unroll
                        for (int c = 0; c < 4; ++c) e[c] = max3_nan(e[c], __uint_as_float(v[c / 2][(c % 2) * 16 + k]), __uint_as_float(v[c / 2][(c % 2) * 16 + k + 1]));
#pragma unroll
                    for (int c = 0; c < 4; ++c) e[c] = max3_nan(e[c], e[c], __uint_as_float(v[c / 2][(c % 2) * 16 + 15]));
                    e[0] = max3_nan(e[0], e[1], max3_nan(e[2], e[2], e[3]));
                } else {
#pragma unroll
                    for (int k = 1; k < 15; k += 2)
#pragma unroll
                        for (int c = 0; c < 4; ++c) e[c] = min3_nan(e[c], __uint_as_float(v[c / 2][(c % 2) * 16 + k]), __uint_as_float(v[c / 2][(c % 2) * 16 + k + 1]));
#pragma unroll
                    for (int c = 0; c < 4; ++c) e[c] = min3_nan(e[c], e[c], __uint_as_float(v[c / 2][(c % 2) * 16 + 15]));
                    e[0] = min3_nan(e[0], e[1], min3_nan(e[2], e[2], e[3]));
                }
                float best = valid ? e[0] * scale : -INFINITY;
                // (the barrier also says that both halves' scores were read: the weights go over them)
                sh.other[t][half][r] = best;
                barrier_of(2u + t, 256u);
                const float theirs = sh.other[t][half ^ 1u][r];
                best = max3_nan(best, best, theirs);
                if (!(best < INFINITY)) l = __int_as_float(0x7fc00000);       // a NaN or an infinity among the scores: the row has no weights
                const bool grow = m != -INFINITY && best > m + kPfGrow;
                if (__any_sync(0xffffffffu, grow)) {         // the sums so far, scaled to the new maximum: when the products before are done
                    const float f = grow ? exp2_fast(m - best) : 1.0f;
                    wait(smem_addr(&sh.o_full[t]), (i - 1u) & 1u);
                    __syncwarp();
                    tensor_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[16];
                        tensor_load16(o_at + c * 16u, o);
#pragma unroll
                        for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                        tensor_store16(o_at + c * 16u, o);
                    }
                    l *= f;
                }
                if (grow || m == -INFINITY) m = best;
                const float z = m == -INFINITY ? 0.0f : m - lift;
                const uint64_t minus_z = two_of(-z, -z);
                uint64_t sum[2] = {0ull, 0ull};
                const bool whole = valid == (uint32_t)kHalf;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        float a, b;
                        of_two(fma_two(two_of(__uint_as_float(v[c][k]), __uint_as_float(v[c][k + 1])), scales, minus_z), a, b);
                        a = exp2_fast(a); b = exp2_fast(b);
                        if (!whole) { if (c * 32u + k >= valid) a = 0.0f; if (c * 32u + k + 1u >= valid) b = 0.0f; }
                        sum[(k / 2) & 1] = add_two(sum[(k / 2) & 1], two_of(a, b));
                        w[k / 2] = Ty::pack(a, b);
                    }
                    tensor_store16(s_at + half * 32u + c * 16u, w);
                }
                // (The weights' sum is of what they were before they were rounded, which the logarithm of the sum needs.  A second sum, of the rounded ones,
                // to divide by, took 9 % of a call: 128 requests behind 32K 154 us against 141.)
                float s0, s1;
                of_two(add_two(sum[0], sum[1]), s0, s1);
                if (m != -INFINITY) l += s0 + s1;
                tensor_stored();
                tensor_fence_before();
                bar_arrive(smem_addr(&sh.p_full[t]));
            }
            wait(smem_addr(&sh.o_full[t]), (n_tiles - 1u) & 1u);
            __syncwarp();
            tensor_fence_after();
            if (!live || (*(volatile uint32_t *)&sh.bad | *(volatile uint32_t *)&sh.gave_up)) l = __int_as_float(0x7fc00000);
            barrier_of(2u + t, 256u);
            sh.other[t][half][r] = l;
            barrier_of(2u + t, 256u);
            l += sh.other[t][half ^ 1u][r];
            const uint32_t n = row0 + t * kPfTile + r;
            const bool mine = n < all_rows;
            const uint32_t b = div32(n, p.div_g), h = head * p.G + (n - b * p.G);
            const size_t rows = (size_t)p.B * p.Hq, at = (size_t)(p.own_pieces + piece) * rows + (size_t)b * p.Hq + h;
            const float z = m - lift, inv = l == 0.0f ? 0.0f : 1.0f / l;
            if (p.pieces == 1u) {
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t v[16];
                    __syncwarp();
                    tensor_load16(o_at + c * 16u, v);
                    if (mine) {
                        uint4 *to = reinterpret_cast<uint4 *>(p.out + (int64_t)b * p.out_row + (int64_t)h * p.out_head + half * (D / 2) + c * 16);
#pragma unroll
                        for (int k = 0; k < 16; k += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) w[e] = l == 0.0f ? 0u : Ty::pack(__uint_as_float(v[k + 2 * e]) * inv, __uint_as_float(v[k + 2 * e + 1]) * inv);
                            to[k / 8] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                }
            } else {
                // Through shared memory, the queries' now that the products are done: a warp's rows by itself, so that whole lines are written.
                constexpr uint32_t kCols = D / 4, kChunks = D / 16, kAtOnce = 32u / kChunks;      // columns a turn; 16 bytes each; rows a store
                const uint32_t own = q_at + t * kBytes + (warp & 7u) * (32u * D), chunk = lane % kChunks;
#pragma unroll
                for (uint32_t c = 0; c < (D / 2) / kCols; ++c) {
                    __syncwarp();
#pragma unroll
                    for (uint32_t k = 0; k < kCols; k += 16u) {
                        uint32_t v[16];
                        tensor_load16(o_at + c * kCols + k, v);
#pragma unroll
                        for (uint32_t e = 0; e < 4u; ++e)
                            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(own + lane * D + (((k / 4u + e) ^ (lane % kChunks)) * 16u)),
                                         "r"(v[4 * e]), "r"(v[4 * e + 1]), "r"(v[4 * e + 2]), "r"(v[4 * e + 3]) : "memory");
                    }
                    __syncwarp();
#pragma unroll
                    for (uint32_t k = 0; k < 32u; k += kAtOnce) {
                        const uint32_t from = k + lane / kChunks;
                        const bool there = __shfl_sync(0xffffffffu, mine ? 1 : 0, from) != 0;
                        const uint64_t row = __shfl_sync(0xffffffffu, (unsigned long long)at, from);
                        const uint4 v = ld_shared16(own + from * D + ((chunk ^ (from % kChunks)) * 16u));
                        if (there) *reinterpret_cast<uint4 *>(p.part_o + row * D + half * (D / 2) + c * kCols + chunk * 4u) = v;
                    }
                }
            }
            if (mine && half == 0u) {
                if (p.pieces > 1u) p.part_ml[at] = make_float2(z, l);
                else if (p.lse) p.lse[(size_t)b * p.Hq + h] = l == 0.0f ? -INFINITY : (z + log2f(l)) * 0.69314718055994531f;
            }
            tensor_fence_before();
        }
    }
    if (__syncthreads_or(live ? 0 : 1) && warp >= 16u && warp < 20u) {
        // A wait was given up: tensor copies may be on their way.  A stage that some warps of the four have asked for gets the others' arrivals (none is
        // two rounds of the ring ahead of another), so that its barrier ends when the copies have; stages that were used before need no wait.
        atomicMax(&sh.most_copied, copied);
        barrier_of(1, 128);
        const uint32_t most = *(volatile uint32_t *)&sh.most_copied, by_box = min(most, 2u * whole);
        for (uint32_t n = copied; n < by_box; ++n) bar_arrive(smem_addr(&sh.kv_full[n % kPfSlots]));
        for (uint32_t n = most > kPfSlots ? most - kPfSlots : 0u; n < by_box; ++n) wait_for_own(smem_addr(&sh.kv_full[n % kPfSlots]), (n / kPfSlots) & 1u);
    }
    __syncwarp();
    if (warp == 20u) {
        tensor_fence_after();
        tensor_free(tmem, 512u);
    }
}

// A map of one of the cache's two buffers: values, slots, heads, pages.  false: its strides are none that such a map can have.
static bool cache_map(CUtensorMap *map, const AttnDev &p, const uint16_t *base, uint32_t dim, bool bf16, uint32_t box) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[4] = {dim, p.page_tokens, p.Hk, p.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)p.slot_stride * 2u, (cuuint64_t)p.head_stride * 2u, (cuuint64_t)p.page_stride * 2u};
    const cuuint32_t boxes[4] = {64u, box, 1u, 1u}, steps[4] = {1u, 1u, 1u, 1u};
    for (const cuuint64_t st : strides) if (st == 0u || st >= (1ull << 40)) return false;
    return encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<uint16_t *>(base), dims, strides, boxes, steps,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class Ty, int D, bool kBf16>
static cudaError_t launch_tiles(const AttnDev &p, cudaStream_t st) {
    const auto k = k_prefix_tiles<Ty, D, kBf16>;
    cudaError_t e = ensure_dyn_smem((const void *)k, pf_smem<D>());
    if (e != cudaSuccess) return e;
    // the warps' shares of the registers add up to what a block is launched with only if that is 80 a thread
    static std::atomic<int> regs{0};
    if (regs.load(std::memory_order_relaxed) == 0) {
        cudaFuncAttributes at = {};
        if ((e = cudaFuncGetAttributes(&at, k)) != cudaSuccess) return e;
        regs.store(at.numRegs, std::memory_order_relaxed);
    }
    if (regs.load(std::memory_order_relaxed) != 80) return cudaErrorInvalidKernelImage;
    g_kernel_launches += 1;
    CUtensorMap k_map = {}, v_map = {};
    uint32_t box = p.page_tokens & (0u - p.page_tokens);     // the largest power of two that a page is a multiple of
    if (box > (uint32_t)kPfTile) box = kPfTile;
    if (box < 8u || !cache_map(&k_map, p, p.k, D, kBf16, box) || !cache_map(&v_map, p, p.v, D, kBf16, box)) box = 0u;
    k<<<p.n_prefix_items, kPfThreads, pf_smem<D>(), st>>>(p, k_map, v_map, box);
    return cudaGetLastError();
}
cudaError_t launch_prefix_tiles(const AttnDev &p, uint32_t dim, bool bf16, cudaStream_t st) {
    if (bf16) return dim == 128u ? launch_tiles<Bf16, 128, true>(p, st) : launch_tiles<Bf16, 64, true>(p, st);
    return dim == 128u ? launch_tiles<Fp16, 128, false>(p, st) : launch_tiles<Fp16, 64, false>(p, st);
}

}  // namespace hbf
