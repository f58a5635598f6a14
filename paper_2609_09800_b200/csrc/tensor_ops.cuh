// Device helpers of the operators of a served layer: 16-bit types by their tag, m16n8k16 products with 32-bit sums, asynchronous
// 16-byte copies to shared memory, and exact division by a small run-time constant.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "device_utils.cuh"

namespace hbf {

struct Bf16 {
    using type = __nv_bfloat16;
    static __device__ __forceinline__ type from(float f) { return __float2bfloat16_rn(f); }
    static __device__ __forceinline__ float to(type v) { return __bfloat162float(v); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ uint32_t pack_down(float lo, float hi) {       // towards zero
        uint32_t u; asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo)); return u;
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&u)); }
    // attention's weights: how many powers of two above 1 the largest is put, and a number that is next to nothing beside it
    static constexpr float kLift = 0.0f, kTiny = 1.17549435e-38f;
    static __device__ __forceinline__ void mma(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};
struct Fp16 {
    using type = __half;
    static __device__ __forceinline__ type from(float f) { return __float2half_rn(f); }
    static __device__ __forceinline__ float to(type v) { return __half2float(v); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
    static __device__ __forceinline__ uint32_t pack_down(float lo, float hi) {
        uint32_t u; asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo)); return u;
    }
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2 *>(&u)); }
    // fp16 ends at 2^-24: from 2^14 down, weights of 2^-38 of the largest still count, and a long sequence may hold very many
    static constexpr float kLift = 14.0f, kTiny = 5.9604645e-8f;
    static __device__ __forceinline__ void mma(float *c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    }
};

// 16 bytes to shared memory, past L1; with ok false zeros are written and nothing is read.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
// the same through L1, for what other warps of the block read too
__device__ __forceinline__ void copy_async16_shared(uint32_t dst, const void *src, bool ok) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Barriers in shared memory that count arrivals and the bytes of asynchronous copies; bulk copies that report to them.
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_init_done() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_arrive_bytes(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// Waits for the phase of the given parity to end.  false: it had not after `polls` polls (1 at least; a poll sleeps for up to some 1.6 us), or another
// thread of the block gave up a wait, or `live` says that this one did before.  Who gives up says so in gave_up (in shared memory, 0 at first)
// before anything else.  From then on a thread neither issues copies or products nor says that any are there, and the block's results are
// NaN; at its end the block waits for what is still on its way (wait_for_own).  A block that is to give up at once begins with `live` false.
// (The loop's form counts: the limit or the flag looked at before the first poll, or a poll told to sleep for 1 us at most, were 2 to 9 % of a
// layer of experts for 64 tokens, 163 to 174 us against 160; `live` not known to be true at first 25 % of k_prefix_tiles.)
constexpr uint32_t kBarPolls = 1u << 20;
__device__ __forceinline__ bool bar_poll(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0u;
}
__device__ __forceinline__ uint32_t ld_flag(uint32_t a) { uint32_t v; asm volatile("ld.volatile.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory"); return v; }
__device__ __forceinline__ void st_flag(uint32_t a, uint32_t v) { asm volatile("st.volatile.shared.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, bool live, uint32_t polls, uint32_t gave_up) {
    if (!live) return false;
    uint32_t i = 0;
#pragma unroll 1
    do {
        if (__builtin_expect(bar_poll(bar, parity), 1)) return true;
        if (ld_flag(gave_up)) return false;
    } while (++i != polls);
    st_flag(gave_up, 1u);
    return false;
}
// For what was issued by the block itself and ends whatever others do: bounded all the same.
__device__ __forceinline__ void wait_for_own(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t i = 0; i < kBarPolls; ++i) if (bar_poll(bar, parity)) return;
}
__device__ __forceinline__ void barrier_of(uint32_t id, uint32_t threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

__device__ __forceinline__ uint4 ld_shared16(uint32_t a) {
    uint4 v; asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory"); return v;
}
// four 8x8 tiles of 16-bit values, transposed: lane l gives the address of row l % 8 of tile l / 8
__device__ __forceinline__ void load_tiles_t(uint32_t a, uint32_t &r0, uint32_t &r1, uint32_t &r2, uint32_t &r3) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3) : "r"(a) : "memory");
}
// an 8x8 tile of 16-bit values that lies in registers as a product's sums do (row lane / 4, columns 2 (lane % 4) and the next), transposed
__device__ __forceinline__ uint32_t transpose_tile(uint32_t a) { uint32_t d; asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a)); return d; }
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// n / d for n, d < 2^31: with l = ceil(log2 d) and m = floor(2^(31+l) / d) + 1 < 2^32, n / d = (n * m) >> (31 + l), exact since
// n * (m * d - 2^(31+l)) <= n * d < 2^(31+l).
struct Div32 { uint32_t magic, shift; };
__host__ __device__ inline Div32 make_div32(uint32_t d) {
    uint32_t l = 0; while ((1ull << l) < d) ++l;
    Div32 r; r.shift = 31 + l;
    r.magic = (uint32_t)((1ull << (31 + l)) / d + 1ull);
    return r;
}
__device__ __forceinline__ uint32_t div32(uint32_t n, const Div32 &d) { return (uint32_t)(((uint64_t)n * d.magic) >> d.shift); }

// ---- host -----------------------------------------------------------------------------------------------
// Polls of a wait in the tensor-memory kernels; a test may lower it (hbf_debug_operator_waits).
inline std::atomic<uint32_t> g_operator_polls{kBarPolls};
// The current device's number of SMs, asked once per device.
inline int sm_count(uint32_t *n_sm) {
    static std::atomic<int> known[64] = {};
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return HBF_E_CUDA;
    if (dev < 0 || dev >= 64) return HBF_E_INVAL;
    n = known[dev].load(std::memory_order_relaxed);
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return HBF_E_CUDA;
        known[dev].store(n, std::memory_order_relaxed);
    }
    *n_sm = (uint32_t)n;
    return HBF_OK;
}
// The operators run on the current device: memory of another one is refused, as is host memory.
inline int device_of(const void *p, uint32_t *n_sm) {
    cudaPointerAttributes at = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaPointerGetAttributes(&at, p) != cudaSuccess) { (void)cudaGetLastError(); return HBF_E_CUDA; }
    if ((at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) || at.device != dev) return HBF_E_INVAL;
    return sm_count(n_sm);
}

}  // namespace hbf
