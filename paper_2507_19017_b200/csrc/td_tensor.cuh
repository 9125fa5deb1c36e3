// Matrix products on the tensor memory: 128 rows at a time, issued by one thread, operands in shared memory in rows of 128
// bytes whose 16-byte vectors are exchanged (vector v of row r lies at v ^ (r & 7)), or (the left one) in tensor memory.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

namespace td {

// ---- barriers that the products arrive at ----
__device__ __forceinline__ void product_bar_init(uint32_t bar) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
// Waits, with a limit, until the phase of this parity is over.
__device__ __forceinline__ bool product_wait(uint32_t bar, uint32_t parity) {
    constexpr uint32_t kPolls = 1u << 16;
    for (uint32_t i = 0; i < kPolls; ++i) {
        uint32_t ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}
// The barrier is arrived at when all products issued so far are done.
__device__ __forceinline__ void product_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ---- tensor memory ----
__device__ __forceinline__ void tensor_alloc(uint32_t to, uint32_t columns) {          // by a warp; the address goes to shared memory
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tensor_free(uint32_t at, uint32_t columns) {           // by the same warp
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tensor_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// What the threads wrote to shared memory is there for the products.
__device__ __forceinline__ void shared_for_products() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 16 columns of the lane's row, from the address (row << 16 | column; a warp reaches the rows 32 (warp % 4) ..).
__device__ __forceinline__ void tensor_load16(uint32_t (&r)[16], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at));
}
__device__ __forceinline__ void tensor_store16(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}

// ---- products ----
// A matrix in shared memory at `at` (a multiple of 16 bytes inside a region aligned to 1024): `eights` bytes from 8 rows to the next 8,
// `across` bytes from 64 columns to the next 64 where the columns are the long side.
__device__ __forceinline__ uint64_t shared_matrix(uint32_t at, uint32_t eights, uint32_t across) {
    return (uint64_t)(at >> 4 & 0x3fffu) | (uint64_t)(across >> 4) << 16 | (uint64_t)(eights >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// The kind of c (128 x n, float) = or += a (128 x 16) b, a and b of T.  turned: b lies with its columns side by side.
template <typename T> struct ProductType;
template <> struct ProductType<__half> { static constexpr uint32_t kBits = 0; };
template <> struct ProductType<__nv_bfloat16> { static constexpr uint32_t kBits = 1u << 7 | 1u << 10; };
template <typename T>
__device__ __forceinline__ constexpr uint32_t product_kind(uint32_t n, bool turned) {
    return 1u << 4 | ProductType<T>::kBits | (turned ? 1u << 16 : 0u) | n >> 3 << 17 | 128u >> 4 << 24;
}
__device__ __forceinline__ void product(uint32_t c, uint64_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(c), "l"(a), "l"(b), "r"(kind), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void product_from_tensor(uint32_t c, uint32_t a, uint64_t b, uint32_t kind, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(c), "r"(a), "l"(b), "r"(kind), "r"((uint32_t)add) : "memory");
}

}  // namespace td
