// The 5th-generation tensor cores: matrices in shared memory as they read them, products into tensor memory, loads and stores of it.
#pragma once
#include <cuda.h>

#include "tensor_ops.cuh"

namespace hbf {

// matrices in shared memory: rows of 64 values (128 bytes) in groups of eight, 16-byte columns permuted by the row's number, the next 64 values of
// all rows behind.  Rows as the products' rows or columns (the sum along a row): `next8` is the way to the next eight rows; the sum along
// the rows' numbers: also `next64` to the next 64 values.
struct TileDesc {
    uint32_t lo, hi;
    __device__ __forceinline__ TileDesc(uint32_t addr, uint32_t next64, uint32_t next8)
        : lo((addr >> 4) | (next64 >> 4) << 16), hi(next8 >> 4 | 1u << 14 | 2u << 29) {}
    __device__ __forceinline__ uint64_t at(uint32_t bytes) const {           // (shared memory ends below 2^18: no carry into the next field)
        uint64_t d; asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo + (bytes >> 4)), "r"(hi)); return d;
    }
};
__device__ __forceinline__ uint32_t product_desc(bool bf16, bool b_by_rows, uint32_t m, uint32_t n) {
    const uint32_t type = bf16 ? 1u : 0u;
    return 1u << 4 | type << 7 | type << 10 | (b_by_rows ? 1u << 16 : 0u) | (n >> 3) << 17 | (m >> 4) << 24;
}
__device__ __forceinline__ void product_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void product_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
    asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void products_arrive(uint32_t bar) {              // when all products issued so far are done
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define HBF_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define HBF_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of this warp's 32 lanes of tensor memory, a lane a thread
__device__ __forceinline__ void tensor_load(uint32_t addr, uint32_t (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : HBF_R8(v, 0), HBF_R8(v, 8), HBF_R8(v, 16), HBF_R8(v, 24) : "r"(addr));
}
__device__ __forceinline__ void tensor_loaded(uint32_t (&v)[32]) {           // (the values may be used behind this)
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+r"(v[i]));
}
__device__ __forceinline__ void tensor_store16(uint32_t addr, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), HBF_I8(v, 0), HBF_I8(v, 8) : "memory");
}
__device__ __forceinline__ void tensor_load16(uint32_t addr, uint32_t (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];" : HBF_R8(v, 0), HBF_R8(v, 8) : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) asm volatile("" : "+r"(v[i]));
}
__device__ __forceinline__ void tensor_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tensor_alloc(uint32_t where, uint32_t columns) {             // by one whole warp; the address goes to shared memory
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tensor_free(uint32_t addr, uint32_t columns) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}

// The driver's call that makes tensor maps, asked for once; nullptr: there is none.
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                 CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
    static std::atomic<void *> known{nullptr};
    void *f = known.load(std::memory_order_relaxed);
    if (f) return reinterpret_cast<EncodeTiled>(f);
    cudaDriverEntryPointQueryResult how;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess || how != cudaDriverEntryPointSuccess) return nullptr;
    known.store(f, std::memory_order_relaxed);
    return reinterpret_cast<EncodeTiled>(f);
}

}  // namespace hbf
