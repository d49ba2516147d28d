// The weight gradient dW = dy^T x^ from activations held in 8 bits
// (include/cpdp_layers.h).
#include <atomic>
#include <cuda.h>

#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

// dW = dy^T x^ is bound by shared memory: a step of 64 tokens takes the tensor
// core 512 clocks, and 768 times 128 bytes move for it (48 KB of operands read,
// 32 KB of dy and 16 KB of x^ written). 2 x 16,384 tokens, 2,048 -> 8,192: 809 us,
// 1,359 TFLOP/s, to either type; 8 x 3,152, 384 -> 1,536 (144 blocks): 35 us.
//
// One block computes 128 (i) x 256 (o) of dW, transposed on the tensor cores:
// the accumulator's 128 lanes are neighbouring i, so that a warp's stores of
// one column are 32 neighbours of dW's row. Tokens pass in steps of 64 through
// a ring of shared-memory slots. Both operands have the tokens, the axis summed
// over, as their slow axis; a slot holds them as rows of 64 elements (128
// bytes) per token in the 128-byte swizzle, one block of rows per 64 columns:
//   dy   bfloat16, by one tensor copy per block of rows
//   x^   made by converting warps from codes and exponents, each thread one
//        block of 32 features of one token: exact in bfloat16. Groups of eight
//        warps take the steps in turn: one group needs 900 clocks for a step
//        (wait, convert, store, hand over), the tensor core 512.
// One thread issues the matrix instructions. The tensor core cuts its float32
// sums off where others round them, always towards 0. In one chain that grows
// with the tokens: where all products have one sign dW came out 0.4 % too small
// at 2^18 tokens and 4 % at 2^22, more than a bfloat16 output's own rounding. So
// a chunk of kChunk steps is summed at a time, and the chunks are added up,
// rounded to nearest: the first chunk's sums lie in one half of tensor memory,
// the others' in turn in the other, from where four adding warps add them to the
// first half. The next chunk waits for that, while the slots are filled (0.9 us
// per chunk; 2 x 16,384 tokens, 2,048 -> 8,192 in one chain took 783 us). The
// converting warps add the last chunk as they write dW. 2,048 tokens of one sign
// lose 2e-6, of both signs 5e-7 of dW.
constexpr int kTileI = 128, kTileO = 256, kStep = 64, kSlots = 4;
constexpr int kGroupWarps = 8, kGroups = 2, kConvertWarps = kGroupWarps * kGroups;
constexpr int kCopyWarp = kConvertWarps, kMultiplyWarp = kConvertWarps + 1, kAddWarp = kConvertWarps + 2;  // the first of four
constexpr int kThreads = (kAddWarp + 4) * 32;
constexpr int kChunk = 32;  // steps
constexpr int kBlockBytes = kStep * 128;                               // a step's rows of 64 elements
constexpr int kXBytes = kTileI / 64 * kBlockBytes, kDyBytes = kTileO / 64 * kBlockBytes, kSlotBytes = kXBytes + kDyBytes;
constexpr int kSmemBytes = kSlots * kSlotBytes + 1024;  // and room to align the slots
constexpr int kAhead = 2;                               // of its steps whose codes a group loads ahead
#ifdef CPDP_CHECKED
constexpr unsigned long long kWaitLimitNs = 200000000ull;
// A step whose dy is never copied, so that waits run out; -1: none. Debug build only.
__device__ int dropped_step = -1;
#else
constexpr unsigned long long kWaitLimitNs = 2000000000ull;
#endif
static_assert(kStep * kTileI == kGroupWarps * 32 * kBlock8, "one block of features per converting thread and step");

__device__ unsigned long long wait_timeouts;

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

// A matrix in shared memory whose rows of 64 elements run along the summed
// axis: blocks of columns kBlockBytes apart, groups of 8 rows 1,024 bytes
// apart, 128-byte swizzle.
__device__ __forceinline__ uint64_t matrix_at(uint32_t address) {
    return static_cast<uint64_t>((address & 0x3ffffu) >> 4) | static_cast<uint64_t>(kBlockBytes >> 4) << 16 |
           static_cast<uint64_t>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// float32 sums, both operands bfloat16 with the summed axis slow, 128 x 256.
constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | (kTileO / 8) << 17 | (kTileI / 16) << 24;

__device__ __forceinline__ void multiply(uint32_t sums, uint64_t a, uint64_t b, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(sums),
        "l"(a), "l"(b), "r"(kInstruction), "r"(add ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void arrive_when_multiplied(uint64_t* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
// 16 columns of the warp's 32 lanes; there once the wait is over.
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
__device__ __forceinline__ void store_sums(uint32_t at, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(at),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// The sum of 16 columns at `a` and at `b`.
__device__ __forceinline__ void add_sums(uint32_t a, uint32_t b, uint32_t (&r)[16]) {
    uint32_t more[16];
    read_sums(a, r);
    read_sums(b, more);
    wait_read(r);
    wait_read(more);
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(more[i]));
}

__device__ __forceinline__ uint32_t sub_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t mul_pair(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Four codes as bfloat16 times `unit` (a pair of the same power of two). With
// a code's lower seven bits n and its sign s, 0x4300 | n is 128 + n and
// 0x4300 | 0x80 s is 128 or 256, so their difference is the code; every step
// is exact.
__device__ __forceinline__ uint2 values_of(uint32_t codes, uint32_t unit) {
    const uint32_t low = codes & 0x7f7f7f7fu, sign = codes & 0x80808080u, k = 0x43434343u;
    return make_uint2(mul_pair(sub_pair(__byte_perm(low, k, 0x4140), __byte_perm(sign, k, 0x4140)), unit),
                      mul_pair(sub_pair(__byte_perm(low, k, 0x4342), __byte_perm(sign, k, 0x4342)), unit));
}

struct Codes {
    uint4 half[2];
    uint32_t byte;
};

struct WeightGradient {
    const int8_t* codes;
    const uint8_t* exponents;
    int64_t M;
    int O, I, W, blocks;  // blocks of 32 features in a row of x^
    int64_t split_steps;  // of a part of the tokens; more than one: parts [part][W][O][I] of float32
    void* out;
    int64_t out_worker, out_split;
};

// Columns [first, first + count) of dW, the warp's 32 lanes of i: the sums of
// the first chunk and, where there are several, of the others; zeros where
// there are none.
template <typename G>
__device__ __forceinline__ void write_out(const WeightGradient& p, uint32_t sums, int chunks, int i0, int o0, int first, int count, G* out) {
    const int quarter = threadIdx.x / 32 % 4 * 32, i = i0 + quarter + static_cast<int>(threadIdx.x % 32);
    const int end = min(p.O - o0, first + count);
    G* to = out + (int64_t)(o0 + first) * p.I + i;
#pragma unroll 1
    for (int o = first; o < end; o += 16, to += (int64_t)16 * p.I) {
        const uint32_t at = sums + (quarter << 16) + o;
        uint32_t v[16] = {};
        if (chunks > 1) {
            add_sums(at, at + kTileO, v);
        } else if (chunks > 0) {
            read_sums(at, v);
            wait_read(v);
        }
        if (i < p.I)
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (o + j < end) to[(int64_t)j * p.I] = from_float<G>(__uint_as_float(v[j]));
        __syncwarp();
    }
}

// G: the output's type.
template <typename G>
__global__ void __launch_bounds__(kThreads, 1)
weight_gradient_kernel(const __grid_constant__ CUtensorMap map, WeightGradient p) {
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kSlots], empty[kSlots], summed[2], added, complete, drained;
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;  // a wait of the block ran out
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t slots = (smem_at(raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kSlots; ++s) {
            barrier_init(&full[s], kGroupWarps + 1);
            barrier_init(&empty[s], 1);
        }
        for (int h = 0; h < 2; ++h) barrier_init(&summed[h], 1);
        barrier_init(&added, 4);
        barrier_init(&complete, 4);
        barrier_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMultiplyWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tensor_memory)), "r"(2 * kTileO)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t sums = tensor_memory;
    layer_begin();

    const int i0 = blockIdx.x * kTileI, o0 = blockIdx.y * kTileO;
    const int w = blockIdx.z % p.W, split = blockIdx.z / p.W;
    const int64_t first = split * p.split_steps * kStep;
    const int64_t tokens = min(p.M - first, p.split_steps * kStep);
    const int steps = static_cast<int>((tokens + kStep - 1) / kStep), chunks = (steps + kChunk - 1) / kChunk;

    G* const out0 = static_cast<G*>(p.out) + split * p.out_split + w * p.out_worker;
    if (warp == kCopyWarp) {
        if (lane == 0) {
            int k = 0;
            for (; k < steps; ++k) {
                const int s = k % kSlots;
                if (k >= kSlots && !barrier_wait(&empty[s], (k / kSlots - 1) & 1, &failed)) break;
#ifdef CPDP_CHECKED
                if (k == *static_cast<volatile int*>(&dropped_step)) continue;
#endif
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(&full[s])), "r"(kDyBytes) : "memory");
                for (int c = 0; c < kTileO / 64; ++c)
                    asm volatile(
                        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                            slots + s * kSlotBytes + kXBytes + c * kBlockBytes),
                        "l"(&map), "r"(o0 + c * 64), "r"(static_cast<int>(first) + k * kStep), "r"(w), "r"(smem_at(&full[s]))
                        : "memory");
            }
            // no copy may be in flight when the block ends, also where a wait ran out
            for (int q = max(k - kSlots, 0); q < k; ++q) barrier_wait(&full[q % kSlots], q / kSlots & 1, &failed);
        }
    } else if (warp == kMultiplyWarp) {
        if (lane == 0) {
            bool ok = true;
            for (int c = 0; c < chunks && ok; ++c) {
                const int end = min((c + 1) * kChunk, steps);
                if (c >= 2) ok = barrier_wait(&added, c & 1, &failed);  // the chunk before is out of the way
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                for (int k = c * kChunk; k < end && ok; ++k) {
                    const int s = k % kSlots;
                    ok = barrier_wait(&full[s], k / kSlots & 1, &failed);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t a = matrix_at(slots + s * kSlotBytes), b = matrix_at(slots + s * kSlotBytes + kXBytes);
#pragma unroll
                    for (int q = 0; q < kStep / 16; ++q)
                        multiply(sums + (c > 0 ? kTileO : 0), a + q * (2048 >> 4), b + q * (2048 >> 4), k > c * kChunk || q > 0);
                    arrive_when_multiplied(&empty[s]);
                }
                arrive_when_multiplied(&summed[c % 2]);
            }
            // nor a product
            arrive_when_multiplied(&drained);
            barrier_wait(&drained, 0, &failed);
        }
    } else if (warp >= kAddWarp) {
        // Every chunk's sums are waited for in turn. Two barriers take turns: the second chunk does not wait for this
        // warp, so one barrier could be two phases on before it looks.
        bool ok = true;
        for (int c = 0; c < chunks && ok; ++c) {
            ok = __all_sync(~0u, barrier_wait(&summed[c % 2], c / 2 & 1, &failed));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (c == 0 || c == chunks - 1) continue;
            const uint32_t at = sums + (warp % 4 * 32 << 16);
#pragma unroll 2
            for (int o = 0; o < kTileO; o += 16) {
                uint32_t v[16];
                add_sums(at + o, at + kTileO + o, v);
                store_sums(at + o, v);
            }
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) barrier_arrive(&added);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(&complete);
    } else {
        // thread: token 8 * (its warp in the group) + lane / 4 of the step, features 32 * (lane % 4) + 0..31 of the tile
        const int token = warp % kGroupWarps * 8 + lane / 4, quarter = lane % 4, block = i0 / kBlock8 + quarter;
        // rows of 64 elements are two blocks of 32; the two rows' threads store their 16-byte pieces in another
        // order, so that eight neighbouring threads meet in no bank
        const int swap = quarter / 2;
        const uint32_t row = slots + (quarter / 2) * kBlockBytes + token * 128;
        uint32_t piece[4];  // where the four 16-byte pieces go
#pragma unroll
        for (int k = 0; k < 4; ++k) piece[k] = row + (((quarter % 2 * 4 + (k ^ swap * 2)) ^ token % 8) << 4);
        // the thread's next step, its codes and its exponent
        const int64_t at = (w * p.M + first + warp / kGroupWarps * kStep + token) * p.blocks + block;
        const uint4* next_codes = reinterpret_cast<const uint4*>(p.codes + at * kBlock8) + swap;
        const uint8_t* next_byte = p.exponents + at;
        const int64_t down = (int64_t)kGroups * kStep * p.blocks;
        const int other = swap ? -1 : 1;
        int left = block < p.blocks ? static_cast<int>(tokens) - token - warp / kGroupWarps * kStep : 0;  // > 0: there is a token
        const auto load = [&]() {
            Codes c{};
            if (left > 0) {
                c.half[0] = *next_codes;
                c.half[1] = next_codes[other];
                c.byte = *next_byte;
            }
            left -= kGroups * kStep;
            next_codes += down * (kBlock8 / 16);
            next_byte += down;
            return c;
        };
        Codes ahead[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) ahead[u] = load();
        bool ok = true;
        for (int k0 = warp / kGroupWarps; k0 < steps && ok; k0 += kAhead * kGroups) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int k = k0 + u * kGroups, s = k % kSlots;
                if (k >= steps || !ok) break;
                const Codes c = ahead[u];
                ahead[u] = load();
                if (k >= kSlots) ok = __all_sync(~0u, barrier_wait(&empty[s], (k / kSlots - 1) & 1, &failed));
                if (!ok) break;
                // a block with an infinite or NaN value reads as NaN
                const uint32_t unit = c.byte == 255u ? 0x7fc07fc0u : c.byte << 7 | c.byte << 23;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint2 lo = values_of(e == 0 ? c.half[h].x : c.half[h].z, unit);
                        const uint2 hi = values_of(e == 0 ? c.half[h].y : c.half[h].w, unit);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(piece[h * 2 + e] + s * kSlotBytes),
                                     "r"(lo.x), "r"(lo.y), "r"(hi.x), "r"(hi.y)
                                     : "memory");
                    }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(&full[s]);
            }
        }
        constexpr int kPart = kTileO * 4 / kConvertWarps;
        __all_sync(~0u, barrier_wait(&complete, 0, &failed));
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        write_out(p, sums, chunks, i0, o0, warp / 4 * kPart, kPart, out0);
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (warp == kMultiplyWarp) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sums), "r"(2 * kTileO));
    }
    // what a block makes whose wait ran out is not dW: it says so
    if (failed)
        for (int k = threadIdx.x; k < kTileI * kTileO; k += kThreads) {
            const int i = i0 + k % kTileI, o = o0 + k / kTileI;
            if (i < p.I && o < p.O) out0[(int64_t)o * p.I + i] = from_float<G>(__uint_as_float(0x7fc00000u));
        }
}

// dy as the tensor copies need it: bfloat16 rows at multiples of 16 bytes. A
// warp per row, 8 elements per lane and turn: out of five neighbouring 32-bit
// words where a bfloat16 row starts between words. Only words that hold
// elements of the row are read; 23 us for 77 MB, 6.7 TB/s; with
// one store of 4 bytes per turn, out of two words, 52.
template <typename T>
__global__ void __launch_bounds__(256)
align_kernel(const T* dy, int64_t dy_worker, int64_t dy_row, int64_t M, int64_t rows, int O, int pitch, uint4* out) {
    layer_begin();
    const int lane = threadIdx.x % 32, pieces = pitch / 8;
    for (int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; row < rows; row += (int64_t)gridDim.x * 8) {
        const int64_t w = row / M;
        const T* p = dy + w * dy_worker + (row - w * M) * dy_row;
        uint4* to = out + row * pieces;
        if constexpr (sizeof(T) == 4) {
#pragma unroll 2
            for (int k = lane; k < pieces; k += 32) {
                uint32_t v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int o = k * 8 + e * 2;
                    const __nv_bfloat162 both = __floats2bfloat162_rn(o < O ? load_once(p + o) : 0.f, o + 1 < O ? load_once(p + o + 1) : 0.f);
                    v[e] = *reinterpret_cast<const uint32_t*>(&both);
                }
                to[k] = make_uint4(v[0], v[1], v[2], v[3]);
            }
        } else {
            const int between = reinterpret_cast<uintptr_t>(p) % 4 != 0;
            const uint32_t* q = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
            const int held = (O + between + 1) / 2;  // words that hold the row's elements
            const uint32_t take = between ? 0x5432u : 0x3210u;
#pragma unroll 2
            for (int k = lane; k < pieces; k += 32) {
                uint32_t a[5];
#pragma unroll
                for (int e = 0; e < 5; ++e) a[e] = k * 4 + e < held ? q[k * 4 + e] : 0u;
                to[k] = make_uint4(__byte_perm(a[0], a[1], take), __byte_perm(a[1], a[2], take), __byte_perm(a[2], a[3], take),
                                   __byte_perm(a[3], a[4], take));
            }
        }
    }
}

// The sum of the splits' parts, in their order; DRAM or L2.
template <typename G>
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float* parts, int splits, int64_t per_worker, int64_t all, G* dW, int64_t dW_worker) {
    layer_begin();
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        float s = 0.f;
        for (int k = 0; k < splits; ++k) s += load_once(parts + k * all + at);
        const int64_t w = at / per_worker;
        dW[w * dW_worker + (at - w * per_worker)] = from_float<G>(s);
    }
}

// How the tokens are split: the number of parts that takes least time, by the
// turns that the blocks take on the SMs. A step of a block takes 0.36 us, its
// start and end 4; parts cost their writing and reading at 4 TB/s and a launch.
struct Splits {
    int count;
    int64_t each;  // steps of a part
};
Splits splits_of(int W, int64_t M, int O, int I) {
    const int64_t steps = ceil_div(M, kStep), tiles = ceil_div(I, kTileI) * ceil_div(O, kTileO) * W;
    Splits best{1, steps};
    double least = 0;
    const int64_t most = ceil_div(2 * kSMs, tiles);  // beyond two turns there is nothing to gain
    for (int64_t count = 1; count <= most && (count == 1 || count * 4 <= steps); ++count) {
        const int64_t each = ceil_div(steps, count), parts = each > 0 ? ceil_div(steps, each) : 1;
        double us = static_cast<double>(ceil_div(tiles * parts, kSMs)) * (each * 0.36 + 4.0);
        if (parts > 1) us += 3.0 + 2e-6 * parts * W * O * I;
        if (count == 1 || us < least) {
            least = us;
            best = {static_cast<int>(parts), each};
        }
    }
    return best;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
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

}  // namespace
}  // namespace cpdp

using namespace cpdp;

static cpdp_status check_weight_gradient(int W, int64_t M, int O, int I) {
    CPDP_TRY(check_sizes(W, M, O));
    CPDP_TRY(check_sizes(W, M, I));
    CPDP_TRY(check_sizes(W, O, I));
    if (M > kLayerMaxRows - kStep) return layer_error(CPDP_EINVAL, "M=%lld is at most 2^31 - 65", (long long)M);
    const int64_t tiles_o = ceil_div(O, kTileO), splits = splits_of(W, M, O, I).count;
    if (tiles_o > 65535 || splits * W > 65535)
        return layer_error(CPDP_EINVAL, "W=%d, M=%lld, O=%d: more blocks than a launch takes", W, (long long)M, O);
    return CPDP_OK;
}

// Whether the tensor copies can read dy where it is. A stride that no index
// uses does not matter.
static bool in_place(const void* dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dtype, int W, int64_t M, int O) {
    return dtype == CPDP_BF16 && aligned_to(dy, 16) && (M <= 1 || (dy_row % 8 == 0 && dy_row >= O)) &&
           (W <= 1 || (dy_worker % 8 == 0 && dy_worker > 0));
}
static size_t parts_bytes(int W, int64_t M, int O, int I) {
    const int count = splits_of(W, M, O, I).count;
    return count > 1 ? ceil_div(static_cast<int64_t>(count) * W * O * I * 4, 16) * 16 : 0;
}
static int64_t pitch_of(int O) { return ceil_div(O, 8) * 8; }

size_t cpdp_weight_gradient_workspace(const void* dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dy_dtype, int W, int64_t M, int O,
                                      int I) {
    if (check_weight_gradient(W, M, O, I) != CPDP_OK) return 0;
    const size_t copy = in_place(dy, dy_worker, dy_row, dy_dtype, W, M, O) ? 0 : static_cast<size_t>(W) * M * pitch_of(O) * 2;
    return parts_bytes(W, M, O, I) + copy;
}

cpdp_status cpdp_weight_gradient(const void* dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dy_dtype,
                                 const int8_t* codes, const uint8_t* exponents, int W, int64_t M, int O, int I, void* dW,
                                 int64_t dW_worker, cpdp_dtype dW_dtype, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    CPDP_TRY(check_weight_gradient(W, M, O, I));
    if (!known_dtype(dy_dtype) || !known_dtype(dW_dtype))
        return layer_error(CPDP_EINVAL, "unknown dtype: dy's is %d, dW's %d", (int)dy_dtype, (int)dW_dtype);
    CPDP_TRY(check_array("dy", dy, M > 0, dtype_size(dy_dtype), dy_worker, dy_row));
    CPDP_TRY(check_array("codes", codes, M > 0, 16));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("dW", dW, true, dtype_size(dW_dtype), dW_worker));
    CPDP_TRY(check_apart("dW", W, dW_worker, (int64_t)O * I));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_weight_gradient_workspace(dy, dy_worker, dy_row, dy_dtype, W, M, O, I)));
    const Splits sp = splits_of(W, M, O, I);
    const bool parts = sp.count > 1;
    WeightGradient p{};
    p.codes = codes, p.exponents = exponents;
    p.M = M, p.O = O, p.I = I, p.W = W, p.blocks = static_cast<int>(ceil_div(I, kBlock8));
    p.split_steps = sp.each;
    p.out = parts ? workspace : dW;
    p.out_worker = parts ? (int64_t)O * I : dW_worker;
    p.out_split = (int64_t)W * O * I;

    CUtensorMap map{};
    if (M > 0) {
        int64_t rows = dy_row, workers = dy_worker;
        if (!in_place(dy, dy_worker, dy_row, dy_dtype, W, M, O)) {
            char* copy = static_cast<char*>(workspace) + parts_bytes(W, M, O, I);
            const int64_t all = W * M, blocks = ceil_div(all, 8) < kSMs * 8 ? ceil_div(all, 8) : kSMs * 8;
            const auto align = [&](auto* in) {
                return launch_layer(align_kernel<std::remove_const_t<std::remove_pointer_t<decltype(in)>>>, static_cast<unsigned>(blocks), 256,
                                    0, stream, in, dy_worker, dy_row, M, all, O, static_cast<int>(pitch_of(O)),
                                    reinterpret_cast<uint4*>(copy));
            };
            CPDP_TRY(layer_launched(dy_dtype == CPDP_F32 ? align(static_cast<const float*>(dy)) : align(static_cast<const __nv_bfloat16*>(dy)),
                                    "cpdp_weight_gradient"));
            dy = copy, rows = pitch_of(O), workers = rows * M;
        }
        if (M == 1) rows = pitch_of(O);  // strides that no index uses
        if (W == 1) workers = rows * M;
        const EncodeTiled encode = encode_tiled();
        if (encode == nullptr) return layer_error(CPDP_ECUDA, "the CUDA driver has no cuTensorMapEncodeTiled");
        const cuuint64_t dims[3] = {(cuuint64_t)O, (cuuint64_t)M, (cuuint64_t)W}, strides[2] = {(cuuint64_t)rows * 2, (cuuint64_t)workers * 2};
        const cuuint32_t box[3] = {64, kStep, 1}, one[3] = {1, 1, 1};
        const CUresult r = encode(&map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(dy), dims, strides, box, one,
                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
        if (r != CUDA_SUCCESS) return layer_error(CPDP_ECUDA, "cuTensorMapEncodeTiled: error %d", (int)r);
    }
    const dim3 grid(ceil_div(I, kTileI), ceil_div(O, kTileO), sp.count * W);
    const auto typed = [&](auto g) {
        using G = decltype(g);
        static std::atomic<uint64_t> allowed{0};  // the devices on which this kernel has been allowed its shared memory
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        const uint64_t bit = device < 64 ? uint64_t(1) << device : 0;
        if (e == cudaSuccess && (allowed.load() & bit) == 0) {
            e = cudaFuncSetAttribute(weight_gradient_kernel<G>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemBytes);
            if (e == cudaSuccess) allowed |= bit;
        }
        return e != cudaSuccess ? e : launch_layer(weight_gradient_kernel<G>, grid, kThreads, kSmemBytes, stream, map, p);
    };
    CPDP_TRY(layer_launched(parts || dW_dtype == CPDP_F32 ? typed(0.f) : typed(__nv_bfloat16{}), "cpdp_weight_gradient"));
    if (!parts) return CPDP_OK;
    const int64_t per_worker = (int64_t)O * I, all = per_worker * W;
    const unsigned blocks = static_cast<unsigned>(ceil_div(all, 256) < kSMs * 8 ? ceil_div(all, 256) : kSMs * 8);
    const auto sum = [&](auto* out) {
        return launch_layer(sum_parts_kernel<std::remove_pointer_t<decltype(out)>>, blocks, 256, 0, stream, static_cast<const float*>(workspace),
                            sp.count, per_worker, all, out, dW_worker);
    };
    return layer_launched(dW_dtype == CPDP_F32 ? sum(static_cast<float*>(dW)) : sum(static_cast<__nv_bfloat16*>(dW)), "cpdp_weight_gradient");
}

#ifdef CPDP_CHECKED
extern "C" cpdp_status cpdp_layer_drop_step(int step) {
    return layer_launched(cudaMemcpyToSymbol(dropped_step, &step, sizeof step), "cpdp_layer_drop_step");
}
#endif

cpdp_status cpdp_layer_timeouts(int64_t* count) {
    if (count == nullptr) return layer_error(CPDP_EINVAL, "count is NULL");
    unsigned long long seen = 0, zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&seen, wait_timeouts, sizeof seen);
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(wait_timeouts, &zero, sizeof zero);
    *count = static_cast<int64_t>(seen);
    return layer_launched(e, "cpdp_layer_timeouts");
}
