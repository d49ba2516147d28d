// What the kernels on the tensor cores share: barriers with bounded waits,
// shared-memory matrices, tensor memory, tensor copies.
#pragma once

#include <cuda.h>

#include "cpdp_layers.cuh"

namespace cpdp {

// The bounded waits that ran out in the kernels of another file since the last call, and sets its count to 0.
cudaError_t take_loss_timeouts(unsigned long long* count);

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_tiled() {
    static const EncodeTiled f = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
            r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return f;
}

#ifdef __CUDACC__
namespace {

#ifdef CPDP_CHECKED
constexpr unsigned long long kWaitLimitNs = 200000000ull;
#else
constexpr unsigned long long kWaitLimitNs = 2000000000ull;
#endif

__device__ unsigned long long wait_timeouts;  // of this file's kernels

__device__ __forceinline__ uint32_t smem_at(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ void barrier_init(uint64_t* b, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* b) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_at(b)) : "memory");
}
// Whether the phase is done, after waiting in hardware for up to `ns`.
__device__ __forceinline__ bool barrier_done(uint64_t* b, uint32_t parity, uint32_t ns) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(smem_at(b)), "r"(parity), "r"(ns)
        : "memory");
    return done != 0;
}
// False, counted and noted in the block's `failed`, where the phase does not end within the limit.
__device__ __noinline__ bool barrier_wait_long(uint64_t* b, uint32_t parity, int* failed) {
    const unsigned long long start = now_ns();
    while (!barrier_done(b, parity, 100000u))
        if (now_ns() - start > kWaitLimitNs) {
            atomicAdd(&wait_timeouts, 1ull);
            *static_cast<volatile int*>(failed) = 1;
            return false;
        }
    return true;
}
__device__ __forceinline__ bool barrier_wait(uint64_t* b, uint32_t parity, int* failed) {
    return barrier_done(b, parity, 100000u) || barrier_wait_long(b, parity, failed);
}

// 16 columns of the warp's 32 lanes of tensor memory; there once the wait is over.
__device__ __forceinline__ void read_sums(uint32_t at, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at)
        : "memory");
}
// The loads' results are operands, so that nothing uses them before.
__device__ __forceinline__ void wait_read(uint32_t (&r)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}

}  // namespace
#endif

}  // namespace cpdp
