// Attention of one decode step for a batch that shares a long prefix: row (request b, query head h) against the prefix's keys, which
// all rows have in common, and the keys that only request b has, both of key head h / G, in pages:
//   o = sum_i softmax(scale * q k_i) v_i over the prefix and the request's own keys.
//
// The softmax over both is joined from pieces: a piece (some rows, a stretch of keys) leaves its largest score m, its sum of weights
// l = sum exp(s - m) and sum exp(s - m) v, which add up after scaling by exp(m - M).  So the prefix is read once for
// all requests (a tile of rows that belong to different requests against the same keys), and long sequences of few requests are cut
// into enough pieces for the device.
#include "attention.cuh"

namespace hbf {

constexpr int kAttWarps = 4, kAttThreads = kAttWarps * 32;
constexpr int kStageKeys = 16;
template <int D> constexpr int kAttRing = D == 128 ? 2 : 4;  // stages on their way, a warp: 16 KB, 192 KB an SM
template <int D> constexpr size_t kAttSmem = (size_t)kAttWarps * kAttRing<D> * kStageKeys * D * 4;

// One piece by four warps: 8 kN rows (a group's heads of one request, or rows of several requests before the prefix), stages of 16 keys
// that go to the warps in turn, each with sums of its own, joined at the end.  Keys and values stream through a ring of each
// warp's own.  The products are S^T = K Q^T and O^T = V^T P^T, so that eight rows are a whole product and the 16 of its other side are keys
// or dimensions (with rows on that side half of the work was for rows that a group of eight heads does not have).  The sum over a head's
// dimensions may take its 16-wide steps in any order, so a lane takes 16 consecutive bytes of a key, copied by itself; values need the
// transpose, and lie in rows whose 16-byte columns are permuted by the row's number.  Latencies bound it (2.8 warps a scheduler,
// 0.32 instructions a cycle; 128 requests' own keys, 280 MB, at 5.4 TB/s, 0.82 of the measured copy rate).
template <class Ty, int D, int kN>
__global__ void __launch_bounds__(kAttThreads, 3)
k_attend(const __grid_constant__ AttnDev p) {
    extern __shared__ __align__(128) unsigned char smem[];
    constexpr int kRing = kAttRing<D>, kBlocks = D / 32, kRows = 8 * kN, kHalf = kStageKeys * D * 2, kStage = 2 * kHalf;
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, row = lane >> 2, quad = lane & 3u;
    pdl_trigger();
    uint32_t item = blockIdx.x, head, tile, piece, b = 0u, begin, end, slot_out;
    const int32_t *table;
    uint32_t n_rows;                                         // rows of the tile in use
    bool bad = false;
    const bool shared = item < p.n_prefix_items;
    if (shared) {
        piece = item % p.prefix_pieces; item /= p.prefix_pieces;
        tile = item % p.row_tiles; head = item / p.row_tiles;
        begin = piece * p.prefix_chunk; end = min(p.prefix_len, begin + p.prefix_chunk);
        table = p.prefix_pages;
        n_rows = min((uint32_t)kRows, p.B * p.G - tile * kRows);
        slot_out = p.own_pieces + piece;
    } else {
        item -= p.n_prefix_items;
        piece = item % p.own_pieces; item /= p.own_pieces;
        tile = item % p.group_tiles; item /= p.group_tiles;
        head = item % p.Hk; b = item / p.Hk;
        const int32_t len = p.own_len ? p.own_len[b] : 0;
        bad = len < 0 || (uint32_t)len > p.max_own;
        begin = piece * p.own_chunk; end = bad ? 0u : min((uint32_t)len, begin + p.own_chunk);
        table = p.own_pages + (size_t)b * p.own_stride;
        n_rows = min((uint32_t)kRows, p.G - tile * kRows);
        slot_out = piece;
    }
    // row r of the tile: request and query head
    auto place = [&](uint32_t r, uint32_t &rb, uint32_t &rh) {
        if (shared) { const uint32_t n = tile * kRows + r; rb = div32(n, p.div_g); rh = head * p.G + n - rb * p.G; }
        else { rb = b; rh = head * p.G + tile * kRows + r; }
    };

    const uint32_t base = smem_addr(smem) + warp * (kRing * kStage);
    const uint32_t stages = begin < end ? (end - begin + kStageKeys - 1u) / kStageKeys : 0u;
    uint32_t in = warp, in_slot = 0u;
    int32_t page0 = 0, page1 = 0; uint32_t at0 = 0u, at1 = 0u;
    auto look_up = [&]() {                                   // the pages of the next stage's two keys of this lane
        if (in >= stages) return;
        const uint32_t k0 = begin + in * kStageKeys + row, k1 = k0 + 8u;
        const uint32_t n0 = div32(k0, p.div_page), n1 = div32(k1, p.div_page);
        at0 = k0 - n0 * p.page_tokens; at1 = k1 - n1 * p.page_tokens;
        if (k0 < end) page0 = table[n0];
        if (k1 < end) page1 = table[n1];
    };
    auto issue = [&]() {
        if (in < stages) {
            const uint32_t k0 = begin + in * kStageKeys + row, k1 = k0 + 8u;
            int64_t o0, o1;
            bool ok0 = key_place(p, page0, at0, o0), ok1 = key_place(p, page1, at1, o1);
            bad |= (k0 < end && !ok0) || (k1 < end && !ok1);
            ok0 &= k0 < end; ok1 &= k1 < end;
            if (!ok0) o0 = 0;
            if (!ok1) o1 = 0;
            const int64_t off = (int64_t)head * p.head_stride + quad * 8u;
            const uint32_t dst = base + in_slot * kStage;
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                copy_async16(dst + (i * 2) * 512u + lane * 16u, p.k + o0 + off + i * 32, ok0);
                copy_async16(dst + (i * 2 + 1) * 512u + lane * 16u, p.k + o1 + off + i * 32, ok1);
            }
#pragma unroll
            for (int i = 0; i < kBlocks; ++i) {
                const uint32_t c = ((quad + 4u * i) ^ row) * 16u;
                copy_async16(dst + kHalf + row * (D * 2) + c, p.v + o0 + off + i * 32, ok0);
                copy_async16(dst + kHalf + (row + 8u) * (D * 2) + c, p.v + o1 + off + i * 32, ok1);
            }
            in_slot = in_slot + 1u == kRing ? 0u : in_slot + 1u;
            in += kAttWarps;
            look_up();
        }
        copy_commit();
    };
    look_up();
#pragma unroll
    for (int i = 0; i < kRing; ++i) issue();

    uint4 q[kN][kBlocks];                                    // this lane's parts of rows `row` and, with kN 2, `row + 8`
#pragma unroll
    for (int r = 0; r < kN; ++r) {
        uint32_t rb, rh;
        place(row + r * 8u, rb, rh);
        const uint16_t *from = p.q + (int64_t)rb * p.q_row + (int64_t)rh * p.q_head + quad * 8u;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) q[r][i] = row + r * 8u < n_rows ? __ldg(reinterpret_cast<const uint4 *>(from + i * 32)) : make_uint4(0u, 0u, 0u, 0u);
    }
    // of the rows 8 r + 2 quad + c: the largest score so far, this lane's share of the weights; their sums, dimensions 16 j + row and + 8
    float o[kN][D / 16][4], m[kN][2], l[kN][2];
#pragma unroll
    for (int r = 0; r < kN; ++r) {
        m[r][0] = m[r][1] = -INFINITY; l[r][0] = l[r][1] = 0.0f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[r][j][0] = o[r][j][1] = o[r][j][2] = o[r][j][3] = 0.0f;
    }
    uint32_t slot = 0u;
    for (uint32_t st = warp; st < stages; st += kAttWarps) {
        copy_wait<kRing - 1>();
        __syncwarp();
        const uint32_t src = base + slot * kStage;
        slot = slot + 1u == kRing ? 0u : slot + 1u;
        float s[kN][4];                                      // keys `row` (0, 1) and `row + 8` (2, 3) for two rows
#pragma unroll
        for (int r = 0; r < kN; ++r) s[r][0] = s[r][1] = s[r][2] = s[r][3] = 0.0f;
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const uint4 ka = ld_shared16(src + (i * 2) * 512u + lane * 16u), kb = ld_shared16(src + (i * 2 + 1) * 512u + lane * 16u);
#pragma unroll
            for (int r = 0; r < kN; ++r) {
                Ty::mma(s[r], ka.x, kb.x, ka.y, kb.y, q[r][i].x, q[r][i].y);
                Ty::mma(s[r], ka.z, kb.z, ka.w, kb.w, q[r][i].z, q[r][i].w);
            }
        }
        const uint32_t key = begin + st * kStageKeys + row;
        const bool in0 = key < end, in1 = key + 8u < end;
        // the running maximum of each row; while it is -inf there is nothing to scale and every weight is 0
        float top[kN][2];
        bool more = false;
#pragma unroll
        for (int r = 0; r < kN; ++r)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                s[r][c] = in0 ? s[r][c] * p.scale_log2 : -INFINITY;
                s[r][c + 2] = in1 ? s[r][c + 2] * p.scale_log2 : -INFINITY;
                top[r][c] = fmaxf(s[r][c], s[r][c + 2]);
            }
#pragma unroll
        for (int x = 4; x < 32; x <<= 1)
#pragma unroll
            for (int r = 0; r < kN; ++r)
#pragma unroll
                for (int c = 0; c < 2; ++c) top[r][c] = fmaxf(top[r][c], __shfl_xor_sync(0xffffffffu, top[r][c], x));
#pragma unroll
        for (int r = 0; r < kN; ++r) more |= top[r][0] > m[r][0] || top[r][1] > m[r][1];
        if (__any_sync(0xffffffffu, more)) {
#pragma unroll
            for (int r = 0; r < kN; ++r) {
                float f[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float n = fmaxf(m[r][c], top[r][c]);
                    f[c] = n == -INFINITY ? 1.0f : exp2_fast(m[r][c] - n);
                    m[r][c] = n; l[r][c] *= f[c];
                }
#pragma unroll
                for (int j = 0; j < D / 16; ++j) { o[r][j][0] *= f[0]; o[r][j][1] *= f[1]; o[r][j][2] *= f[0]; o[r][j][3] *= f[1]; }
            }
        }
        // The weights as a B operand (keys, then rows), each as the sum of two numbers of the values' type: rounding them once would cost as
        // much again as rounding the output does.  The first is rounded down and the second is positive where the weight is, so that
        // both take an infinite value the same way.
        uint32_t hi[kN][2], lo[kN][2];
#pragma unroll
        for (int r = 0; r < kN; ++r) {
            const float z0 = m[r][0] == -INFINITY ? 0.0f : m[r][0] - Ty::kLift, z1 = m[r][1] == -INFINITY ? 0.0f : m[r][1] - Ty::kLift;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float a = exp2_fast(s[r][2 * k] - z0), b = exp2_fast(s[r][2 * k + 1] - z1);
                l[r][0] += a; l[r][1] += b;
                const uint32_t h = Ty::pack_down(a, b);
                const float2 back = Ty::unpack(h);
                hi[r][k] = transpose_tile(h);
                lo[r][k] = transpose_tile(Ty::pack(fmaxf(a - back.x, fminf(a, Ty::kTiny)), fmaxf(b - back.y, fminf(b, Ty::kTiny))));
            }
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            uint32_t v0, v1, v2, v3;
            const uint32_t kr = (lane & 7u) + (lane >> 4) * 8u, c = j * 2u + ((lane >> 3) & 1u);
            load_tiles_t(src + kHalf + kr * (D * 2) + ((c ^ (kr & 7u)) * 16u), v0, v1, v2, v3);
#pragma unroll
            for (int r = 0; r < kN; ++r) {
                Ty::mma(o[r][j], v0, v1, v2, v3, hi[r][0], hi[r][1]);
                Ty::mma(o[r][j], v0, v1, v2, v3, lo[r][0], lo[r][1]);
            }
        }
        __syncwarp();                                        // every lane has read the values that the next copies replace
        issue();
    }
#pragma unroll
    for (int x = 4; x < 32; x <<= 1)
#pragma unroll
        for (int r = 0; r < kN; ++r)
#pragma unroll
            for (int c = 0; c < 2; ++c) l[r][c] += __shfl_xor_sync(0xffffffffu, l[r][c], x);
    copy_wait<0>();
    const bool none = __any_sync(0xffffffffu, bad);          // a page that is none: the rows have no answer
    __syncthreads();                                         // the rings are empty: their memory holds the warps' sums
    float *os = reinterpret_cast<float *>(smem);
    __shared__ float2 ml[kAttWarps][kRows];
    constexpr int kPitch = D + 4;
    static_assert((size_t)kAttWarps * kRows * kPitch * 4 <= kAttSmem<D>, "the warps' sums");
#pragma unroll
    for (int r = 0; r < kN; ++r) {
        float *to = os + ((size_t)warp * kRows + r * 8 + quad * 2) * kPitch + row;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) { to[j * 16] = o[r][j][0]; to[kPitch + j * 16] = o[r][j][1]; to[j * 16 + 8] = o[r][j][2]; to[kPitch + j * 16 + 8] = o[r][j][3]; }
#pragma unroll
        for (int c = 0; c < 2; ++c) if (row == 0u) ml[warp][r * 8 + quad * 2 + c] = make_float2(m[r][c] - Ty::kLift, none ? __int_as_float(0x7fc00000) : l[r][c]);
    }
    __syncthreads();
    constexpr int kLanes = D / 4;                            // threads a row, four dimensions each
    const uint32_t col = threadIdx.x % kLanes;
    for (uint32_t r = threadIdx.x / kLanes; r < n_rows; r += kAttThreads / kLanes) {
        float M = -INFINITY, L = 0.0f;
#pragma unroll
        for (int w = 0; w < kAttWarps; ++w) M = fmaxf(M, ml[w][r].x);
        const float z = M == -INFINITY ? 0.0f : M;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < kAttWarps; ++w) {
            const float f = exp2_fast(ml[w][r].x - z);
            const float4 x = *reinterpret_cast<const float4 *>(os + ((size_t)w * kRows + r) * kPitch + col * 4u);
            L += f * ml[w][r].y; v.x += f * x.x; v.y += f * x.y; v.z += f * x.z; v.w += f * x.w;
        }
        uint32_t rb, rh;
        place(r, rb, rh);
        const size_t n = (size_t)rb * p.Hq + rh;
        if (p.pieces == 1u) {
            const float inv = L == 0.0f ? 0.0f : 1.0f / L;   // nothing to attend to: zeros
            uint2 w2 = make_uint2(Ty::pack(v.x * inv, v.y * inv), Ty::pack(v.z * inv, v.w * inv));
            *reinterpret_cast<uint2 *>(p.out + (int64_t)rb * p.out_row + (int64_t)rh * p.out_head + col * 4u) = w2;
            if (p.lse && col == 0u) p.lse[n] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
        } else {
            const size_t rows = (size_t)p.B * p.Hq;
            if (L != 0.0f) *reinterpret_cast<float4 *>(p.part_o + (slot_out * rows + n) * D + col * 4u) = v;
            if (col == 0u) p.part_ml[slot_out * rows + n] = make_float2(M, L);
        }
    }
    // What joins the pieces waits for this kernel only: its last block ends after the prefix's.  (Not every block: they would keep their SMs.)
    if (p.behind && blockIdx.x == gridDim.x - 1u) pdl_wait();
}

// Joins the rows' pieces: kPer warps a row.  First the pieces' shares of the whole, exp2(m - M), by a thread each; then their sums, four or eight
// of a warp's pieces on their way at a time.
constexpr int kJoinWarps = 8;
constexpr uint32_t kMostPieces = 1024;                      // of a row (attention_pieces makes fewer)
template <class Ty, int D, int kPer>
__global__ void __launch_bounds__(kJoinWarps * 32)
k_attend_join(const __grid_constant__ AttnDev p) {
    constexpr int kRows = kJoinWarps / kPer, kEach = D / 32, kOn = kPer == kJoinWarps ? 8 : 4;
    __shared__ float share[kRows][kMostPieces / kRows], red[kJoinWarps][2], so[kJoinWarps][D];
    const uint32_t lane = lane_id(), warp = threadIdx.x >> 5, group = warp / kPer, part = warp % kPer;
    const size_t rows = (size_t)p.B * p.Hq;
    const uint32_t n = blockIdx.x * kRows + group;
    const bool there = n < rows;
    float *f = share[group];
    pdl_wait();
    float M = -INFINITY, L = 0.0f;
    if (there)
        for (uint32_t s = part * 32u + lane; s < p.pieces; s += kPer * 32u) {
            float2 ml;
            asm volatile("ld.global.cg.v2.f32 {%0,%1}, [%2];" : "=f"(ml.x), "=f"(ml.y) : "l"(p.part_ml + s * rows + n));
            if (ml.y == 0.0f) ml.x = -INFINITY;              // an empty piece
            const float N = fmaxf(M, ml.x), z = N == -INFINITY ? 0.0f : N;
            L = L * exp2_fast(M - z) + ml.y * exp2_fast(ml.x - z);
            M = N; f[s] = ml.x;
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xffffffffu, M, o), l2 = __shfl_xor_sync(0xffffffffu, L, o), N = fmaxf(M, m2), z = N == -INFINITY ? 0.0f : N;
        L = L * exp2_fast(M - z) + l2 * exp2_fast(m2 - z);
        M = N;
    }
    if (lane == 0u) { red[warp][0] = M; red[warp][1] = L; }
    __syncthreads();
    M = -INFINITY; L = 0.0f;
#pragma unroll
    for (int w = 0; w < kPer; ++w) M = fmaxf(M, red[group * kPer + w][0]);
    const float z = M == -INFINITY ? 0.0f : M;
#pragma unroll
    for (int w = 0; w < kPer; ++w) L += exp2_fast(red[group * kPer + w][0] - z) * red[group * kPer + w][1];
    float v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = 0.0f;
    if (there)
        for (uint32_t s0 = part; s0 < p.pieces; s0 += kPer * kOn) {
            float x[kOn][kEach], g[kOn];
#pragma unroll
            for (int k = 0; k < kOn; ++k) {
                const uint32_t s = s0 + k * kPer;
                g[k] = s < p.pieces ? exp2_fast(f[s] - z) : 0.0f;
                const float *from = p.part_o + (s * rows + n) * D + lane * kEach;
#pragma unroll
                for (int i = 0; i < kEach; ++i) x[k][i] = 0.0f;
                if (g[k] != 0.0f) {
                    if (kEach == 4) asm volatile("ld.global.cg.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x[k][0]), "=f"(x[k][1]), "=f"(x[k][kEach - 2]), "=f"(x[k][kEach - 1]) : "l"(from));
                    else asm volatile("ld.global.cg.v2.f32 {%0,%1}, [%2];" : "=f"(x[k][0]), "=f"(x[k][1]) : "l"(from));
                }
            }
#pragma unroll
            for (int k = 0; k < kOn; ++k)
#pragma unroll
                for (int i = 0; i < kEach; ++i) v[i] += g[k] * x[k][i];
        }
#pragma unroll
    for (int i = 0; i < kEach; ++i) so[warp][lane * kEach + i] = v[i];
    __syncthreads();
    if (!there) return;
    const uint32_t b = n / p.Hq, h = n - b * p.Hq;
    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
    for (uint32_t d = (part * 32u + lane) * 2u; d < (uint32_t)D; d += kPer * 64u) {
        float a0 = 0.0f, a1 = 0.0f;
#pragma unroll
        for (int w = 0; w < kPer; ++w) { a0 += so[group * kPer + w][d]; a1 += so[group * kPer + w][d + 1u]; }
        *reinterpret_cast<uint32_t *>(p.out + (int64_t)b * p.out_row + (int64_t)h * p.out_head + d) = L == 0.0f ? 0u : Ty::pack(a0 * inv, a1 * inv);
    }
    if (p.lse && part == 0u && lane == 0u) p.lse[n] = L == 0.0f ? -INFINITY : (M + log2f(L)) * 0.69314718055994531f;
}

// The records of what a step reads: every page of the prefix once, keys then values, then every request's own pages; the places of pages
// that a request does not have hold records of one byte at address 0, outside every range.
__global__ void __launch_bounds__(256)
k_attend_accesses(const __grid_constant__ AttnDev p, uint32_t prefix_slots, uint32_t own_slots, uint32_t page_bytes, int64_t issue_ns, int64_t gap_ns,
                  hbf_access_t *acc, uint64_t n) {
    for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256u) {
        const uint64_t page = i >> 1;
        int32_t id = -1;
        if (page < prefix_slots) id = p.prefix_pages[page];
        else {
            const uint64_t k = page - prefix_slots;
            const uint32_t b = (uint32_t)(k / own_slots), s = (uint32_t)(k - (uint64_t)b * own_slots);
            const int32_t len = p.own_len ? p.own_len[b] : 0;
            if (len > 0 && (uint32_t)len <= p.max_own && s * p.page_tokens < (uint32_t)len) id = p.own_pages[(size_t)b * p.own_stride + s];
        }
        hbf_access_t v = {0, issue_ns + (int64_t)i * gap_ns, 1, 0};
        if ((uint32_t)id < p.n_pages) {
            v.addr = (uint64_t)(uintptr_t)((i & 1u ? p.v : p.k) + (int64_t)id * p.page_stride);
            v.bytes = page_bytes;
        }
        acc[i] = v;
    }
}

static bool kv_ok(const hbf_kv_t &c) {
    if (c.n_pages == 0 || c.n_pages > 0x7fffffffu || c.page_tokens == 0 || c.page_tokens > (1u << 20) || c.kv_heads == 0 || c.kv_heads > 1024u) return false;
    if ((c.head_dim != 64 && c.head_dim != 128) || c.dtype > HBF_FP16) return false;
    return c.page_stride >= 0 && c.slot_stride >= 0 && c.head_stride >= 0 && c.page_stride % 8 == 0 && c.slot_stride % 8 == 0 && c.head_stride % 8 == 0;
}
static bool attention_ok(const hbf_attention_t *a) {
    if (!a || !kv_ok(a->kv) || a->q_heads == 0 || a->q_heads % a->kv.kv_heads || a->q_heads > 65536u || a->batch > 65536u) return false;
    if (a->prefix_len > HBF_ATTENTION_MAX_LEN || a->max_own_len > HBF_ATTENTION_MAX_LEN || !(a->scale - a->scale == 0.0f)) return false;
    return (uint64_t)a->batch * a->q_heads <= (1u << 22);
}
static bool attention_pointers_ok(const hbf_attention_t *a) {
    if (!a->kv.k || !a->kv.v || (uintptr_t)a->kv.k % 16 || (uintptr_t)a->kv.v % 16) return false;
    if (a->prefix_len && (!a->prefix_pages || (uintptr_t)a->prefix_pages % 4)) return false;
    if (a->max_own_len && (!a->own_pages || !a->own_len || (uintptr_t)a->own_pages % 4 || (uintptr_t)a->own_len % 4)) return false;
    if (a->max_own_len && (uint64_t)a->own_pages_stride * a->kv.page_tokens < a->max_own_len) return false;
    return true;
}

// Whether the prefix goes through k_attend, which reads it again, from L2, for every 16 rows: while that is no more than kPrefixAgain bytes
// in all, it costs less than the further launch and the longer start of k_prefix_tiles (8 MB: 12.1 to 14.1 us against 14.5 to 21.2; 32 MB 16.5
// and 18.5 against 16.5 and 20.8; 64 MB 20.6, 21.4 and 20.6 against 18.5, 20.6 and 22.6; 192 MB 36.8 against 28.8).
constexpr uint64_t kPrefixAgain = 48ull << 20;
static bool prefix_small(const hbf_attention_t *a) {
    const uint64_t rows = (uint64_t)a->batch * (a->q_heads / a->kv.kv_heads);
    return rows <= 16u || (rows + 15u) / 16u * a->kv.kv_heads * a->prefix_len * a->kv.head_dim * 4u <= kPrefixAgain;
}

static uint32_t up_to(uint32_t v, uint32_t m) { return (v + m - 1u) / m * m; }

// How the keys are cut.  A piece costs its start-up (about 2 us to the first values) and d * 4 bytes a row to join.  The prefix: as long as
// leaves about two blocks an SM, which are resident at once (one request behind 8K tokens 12.0 us, with four 14.5).  The requests' own, whose
// lengths differ: shorter ones, so that the blocks that are done take others' (128 requests with up to 2,048 130 us with pieces of 512 at
// most, with 1,024 132, with 256 133).  At least 64 keys, a multiple of 64.
static void attention_pieces(const hbf_attention_t *a, uint32_t n_sm, AttnDev &p) {
    const uint32_t G = p.G, blocks = 2u * n_sm;
    // rows of a tile of k_attend: eight, or sixteen where more come together
    const bool small = prefix_small(a);
    p.rows = G > 8u || (small && a->prefix_len && p.B * G > 8u) ? 16u : 8u;
    p.prefix_rows = small ? p.rows : 256u;
    p.row_tiles = (p.B * G + p.prefix_rows - 1u) / p.prefix_rows;
    p.group_tiles = (G + p.rows - 1u) / p.rows;
    p.prefix_pieces = 0u; p.prefix_chunk = 64u;
    if (a->prefix_len && p.B) {
        // (k_prefix_tiles: a block an SM, tiles of 128 keys)
        const uint32_t step = p.prefix_rows == 256u ? 128u : 64u, there = p.prefix_rows == 256u ? n_sm : blocks;
        const uint32_t pairs = p.row_tiles * p.Hk, most = (a->prefix_len + step - 1u) / step;
        const uint32_t want = there <= pairs ? 1u : there / pairs < kMostPieces / 4u ? there / pairs : kMostPieces / 4u;
        p.prefix_chunk = up_to((a->prefix_len + (want < most ? want : most) - 1u) / (want < most ? want : most), step);
        p.prefix_pieces = (a->prefix_len + p.prefix_chunk - 1u) / p.prefix_chunk;
    }
    p.own_pieces = 0u; p.own_chunk = 64u;
    if (a->max_own_len && p.B) {
        const uint64_t lists = (uint64_t)p.B * p.Hk * p.group_tiles;
        const uint64_t want = lists < 2u * blocks ? 2u * blocks / lists : 1u;
        uint64_t chunk = (a->max_own_len + want - 1u) / want;
        chunk = chunk < 64u ? 64u : chunk > 512u ? 512u : chunk;
        const uint64_t least = ((uint64_t)a->max_own_len + kMostPieces / 4u - 1u) / (kMostPieces / 4u);
        if (chunk < least) chunk = least;
        p.own_chunk = up_to((uint32_t)chunk, 64u);
        p.own_pieces = (a->max_own_len + p.own_chunk - 1u) / p.own_chunk;
    }
    p.n_prefix_items = p.prefix_pieces * p.row_tiles * p.Hk;
    p.pieces = p.own_pieces + p.prefix_pieces;
}

static AttnDev attention_dev(const hbf_attention_t *a, uint32_t n_sm) {
    AttnDev p = {};
    p.k = static_cast<const uint16_t *>(a->kv.k); p.v = static_cast<const uint16_t *>(a->kv.v);
    p.page_stride = a->kv.page_stride; p.slot_stride = a->kv.slot_stride; p.head_stride = a->kv.head_stride;
    p.n_pages = a->kv.n_pages; p.Hk = a->kv.kv_heads; p.Hq = a->q_heads; p.G = p.Hq / p.Hk; p.B = a->batch;
    p.page_tokens = a->kv.page_tokens; p.div_page = make_div32(p.page_tokens); p.div_g = make_div32(p.G);
    p.q = static_cast<const uint16_t *>(a->q); p.q_row = a->q_row_stride; p.q_head = a->q_head_stride;
    p.out = static_cast<uint16_t *>(a->out); p.out_row = a->out_row_stride; p.out_head = a->out_head_stride;
    p.lse = a->lse; p.scale_log2 = a->scale * 1.4426950408889634f;
    p.prefix_len = a->prefix_len; p.max_own = a->max_own_len; p.own_stride = a->own_pages_stride;
    p.prefix_pages = a->prefix_pages; p.own_pages = a->own_pages; p.own_len = a->own_len;
    p.polls = g_operator_polls.load(std::memory_order_relaxed);
    attention_pieces(a, n_sm, p);
    return p;
}
static size_t attention_bytes(const AttnDev &p, uint32_t dim) {
    if (p.pieces <= 1u || p.B == 0u) return 256u;
    return ((size_t)p.pieces * p.B * p.Hq * (dim * 4u + 8u) + 255u) / 256u * 256u;
}

template <class Ty, int D>
static cudaError_t launch_attention(AttnDev p, bool bf16, cudaStream_t st) {
    const bool tiles = p.prefix_rows == 256u && p.n_prefix_items;
    AttnDev own = p;
    if (tiles) { own.n_prefix_items = 0u; own.behind = 1u; }
    const uint64_t items = own.n_prefix_items + (uint64_t)p.B * p.Hk * p.group_tiles * p.own_pieces;
    cudaError_t e = cudaSuccess;
    // The requests' own keys go to the SMs that the prefix's blocks leave free, and to the others as those end.  k_attend, launched to overlap
    // k_prefix_tiles, reads nothing of its and writes other places, so its blocks need no pdl_wait of their own; but the join waits for k_attend only, so
    // k_attend's last block waits for the prefix, and k_attend is done only when that is.  (k_prefix_tiles itself is launched behind all that came before.)
    if (tiles && (e = launch_prefix_tiles(p, D, bf16, st)) != cudaSuccess) return e;
    if (items) {
        const auto attend = p.rows == 8u ? k_attend<Ty, D, 1> : k_attend<Ty, D, 2>;
        if ((e = ensure_dyn_smem((const void *)attend, kAttSmem<D>)) != cudaSuccess) return e;
        if (tiles) e = launch_pdl(attend, (unsigned)items, kAttThreads, kAttSmem<D>, st, own);
        else { attend<<<(unsigned)items, kAttThreads, kAttSmem<D>, st>>>(own); e = cudaGetLastError(); }
        g_kernel_launches += 1;
        if (e != cudaSuccess) return e;
    }
    if (p.pieces == 1u) return e;
    g_kernel_launches += 1;
    // many rows: two warps each, else eight.  The whole call with two and with eight, 8K keys in common and 512 of each: 512 rows 22.8 and 19.3 us,
    // 1,024 28.4 and 24.9, 1,280 29.9 and 30.8, 2,048 35.5 and 38.7, 4,096 55.4 and 66.8; 32K in common 1,280 rows 49.7 and 49.3; none 36.6 and 38.6.
    const uint32_t per = p.B * p.Hq > 1024u && p.pieces <= kMostPieces / 4u ? 2u : kJoinWarps, rows = kJoinWarps / per;
    const auto join = per == 2u ? k_attend_join<Ty, D, 2> : k_attend_join<Ty, D, kJoinWarps>;
    const uint32_t blocks = (p.B * p.Hq + rows - 1u) / rows;
    if (p.pieces == 0u) { join<<<blocks, kJoinWarps * 32, 0, st>>>(p); return cudaGetLastError(); }
    return launch_pdl(join, blocks, kJoinWarps * 32, 0, st, p);
}

}  // namespace hbf

using namespace hbf;

extern "C" int hbf_debug_operator_waits(int32_t poll_limit) {
    g_operator_polls.store(poll_limit < 0 ? kBarPolls : (uint32_t)poll_limit, std::memory_order_relaxed);
    return HBF_OK;
}

extern "C" size_t hbf_attention_workspace_bytes(const hbf_attention_t *a) {
    uint32_t n_sm = 0;
    if (!attention_ok(a) || sm_count(&n_sm) != HBF_OK) return 0;
    return attention_bytes(attention_dev(a, n_sm), a->kv.head_dim);
}

extern "C" int hbf_prefix_attention(const hbf_attention_t *a, void *d_workspace, size_t workspace_bytes, void *cuda_stream) {
    if (!attention_ok(a)) return HBF_E_INVAL;
    if (a->batch == 0) return HBF_OK;
    if (!attention_pointers_ok(a) || !a->q || !a->out || (uintptr_t)a->q % 16 || (uintptr_t)a->out % 16 || (uintptr_t)a->lse % 4) return HBF_E_INVAL;
    if (a->q_row_stride % 8 || a->q_head_stride % 8 || a->out_row_stride % 8 || a->out_head_stride % 8) return HBF_E_INVAL;
    if ((a->batch > 1 && a->out_row_stride == 0) || (a->q_heads > 1 && a->out_head_stride == 0)) return HBF_E_INVAL;      // rows on top of each other
    uint32_t n_sm = 0;
    const int rc = device_of(a->kv.k, &n_sm);
    if (rc != HBF_OK) return rc;
    AttnDev p = attention_dev(a, n_sm);
    if ((uint64_t)p.B * p.Hk * p.group_tiles * p.own_pieces + p.n_prefix_items > 0x7fffffffull) return HBF_E_INVAL;
    if (!d_workspace || (uintptr_t)d_workspace % 256 || workspace_bytes < attention_bytes(p, a->kv.head_dim)) return HBF_E_WORKSPACE;
    p.part_o = static_cast<float *>(d_workspace);
    p.part_ml = reinterpret_cast<float2 *>(p.part_o + (size_t)p.pieces * p.B * p.Hq * a->kv.head_dim);
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e;
    if (a->kv.dtype == HBF_BF16) e = a->kv.head_dim == 128 ? launch_attention<Bf16, 128>(p, true, st) : launch_attention<Bf16, 64>(p, true, st);
    else e = a->kv.head_dim == 128 ? launch_attention<Fp16, 128>(p, false, st) : launch_attention<Fp16, 64>(p, false, st);
    return e == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}

static uint64_t attention_records(const hbf_attention_t *a) {
    const uint64_t own = (a->max_own_len + a->kv.page_tokens - 1) / a->kv.page_tokens, prefix = (a->prefix_len + a->kv.page_tokens - 1) / a->kv.page_tokens;
    return 2 * (prefix + own * a->batch);
}
extern "C" uint64_t hbf_attention_access_count(const hbf_attention_t *a) { return attention_ok(a) ? attention_records(a) : 0; }

extern "C" int hbf_attention_accesses(const hbf_attention_t *a, int64_t issue_ns, int64_t gap_ns, hbf_access_t *d_acc, uint64_t n, void *cuda_stream) {
    if (!attention_ok(a) || issue_ns < 0 || gap_ns < 0 || n != attention_records(a) || n > HBF_MAX_BATCH) return HBF_E_INVAL;
    // a page is one stretch of memory, slots and heads side by side in either order
    const int64_t dim = a->kv.head_dim, slots = a->kv.page_tokens, heads = a->kv.kv_heads;
    const bool by_slot = a->kv.head_stride == dim && a->kv.slot_stride == dim * heads, by_head = a->kv.slot_stride == dim && a->kv.head_stride == dim * slots;
    const int64_t bytes = dim * slots * heads * 2;
    if ((!by_slot && !by_head) || bytes > 0xffffffffll) return HBF_E_INVAL;
    if (n == 0) return HBF_OK;
    if (!attention_pointers_ok(a) || !d_acc || (uintptr_t)d_acc % 8) return HBF_E_INVAL;
    uint32_t n_sm = 0;
    const int rc = device_of(a->kv.k, &n_sm);
    if (rc != HBF_OK) return rc;
    const uint32_t own = (uint32_t)((a->max_own_len + slots - 1) / slots), prefix = (uint32_t)((a->prefix_len + slots - 1) / slots);
    const uint64_t blocks = (n + 255) / 256;
    k_attend_accesses<<<(unsigned)(blocks < 8u * n_sm ? blocks : 8u * n_sm), 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        attention_dev(a, n_sm), prefix, own ? own : 1u, (uint32_t)bytes, issue_ns, gap_ns, d_acc, n);
    g_kernel_launches += 1;
    return cudaGetLastError() == cudaSuccess ? HBF_OK : HBF_E_CUDA;
}
