// Softmax cross entropy over a vocabulary, from the activations and the head's
// weight, without the logits in memory (include/cpdp_layers.h).
#include <algorithm>

#include "cpdp_tensor.cuh"

namespace cpdp {
namespace {

// All of it is products on the tensor cores, C[a][b] = sum over k of A[a][k] B[b][k]:
//   logits   a: tokens, b: words, k: features; an epilogue leaves each row's
//            maximum and sum of exponentials over 128 words
//   again    the same in the backward pass; the epilogue leaves
//            d = dloss (exp(l - lse) - onehot), for a piece of the vocabulary
//   dx       a: features, b: tokens, k: words of the piece
//   dweight  a: features, b: words of the piece, k: tokens
// One block per SM walks tiles of 128 (a) x 256 (b). k passes in steps of 64
// through a ring of shared-memory slots, filled by tensor copies; one thread
// issues the matrix instructions. Sums alternate between the halves of tensor
// memory, so that a tile's epilogue runs while the next one is multiplied. The
// accumulator's 128 lanes are a: a thread of the logits' epilogue holds 128 words
// of one token, and the products that are written out have their contiguous
// axis there, so that a warp's store is of 32 neighbours at any alignment.
//
// The tensor core cuts its float32 sums off where others round them, always
// towards 0: chunks of some steps are summed at a time and added up, rounded to
// nearest, in the epilogue's registers. Chunks of 32 steps lose 3.6e-7 of lse at
// 2,048 features and, float32 operands, 8e-7 of a loss at 771; chunks of 4 lose
// 5e-8 and 7e-8, chunks of 2 4e-8 and 6e-8. Forwards (2 x 4,096 tokens, 2,048
// features, 50,000 words, bfloat16): 1,082 us in chunks of 4, 989 in chunks of 8,
// 969 in chunks of 32 and 1,397 in chunks of 2.
constexpr int kTileA = 128, kTileB = 256, kStep = 64, kSlots = 4;
constexpr int kEpilogueWarps = 8, kCopyWarp = 8, kMultiplyWarp = 9, kThreads = 10 * 32;
constexpr int kHalf = kTileB / 2;  // columns of a thread
constexpr int kChunk = 4;  // steps
constexpr int kABytes = kTileA * kStep * 2, kBBytes = kTileB * kStep * 2, kSlotBytes = kABytes + kBBytes;
constexpr int kBlockBytes = kStep * 128;  // 64 columns of an operand that has k as its slow axis
constexpr int kSmemBytes = kSlots * kSlotBytes + 1024;
constexpr int kGroup = 8;  // neighbouring tiles along b that pass before the next along a
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float power(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Float32 operands are held as three bfloat16 planes, each the rounded rest of
// those before it: 24 bits. Six products of planes, k passing once for each,
// leave out what is below 2^-24 of a product.
constexpr int kPlanes = 3, kPlaneProducts = 6;
struct Planes {
    int products;   // of planes
    uint32_t a, b;  // which, four bits each, the first lowest
};
constexpr Planes kOnePlane{1, 0, 0}, kThreePlanes{kPlaneProducts, 0x021010u, 0x201100u};  // 00, 10, 01, 11, 20, 02
// d, the gradient of the logits, is float32 whatever the operands' type: three planes of it with the one of a bfloat16
// operand. In one plane, which takes a third of the products' time, it is the whole error of float32 gradients, 2.2e-4
// of dweight's norm at 512 tokens, 128 features and 8,192 words, and in two 2.5e-6 at 64 words; in three 3.6e-7. (2 x 4,096
// tokens, 2,048 features, 50,000 words, backwards: 8.7 ms, in one plane 3.4.)
constexpr Planes kThreeOfD{kPlanes, 0x000u, 0x210u};

#ifdef CPDP_CHECKED
// A block's step that is never copied, so that waits run out; -1: none. Debug build only.
__device__ int dropped_step = -1;
#endif

struct Product {
    int W, tiles_a, tiles_b, splits;
    int steps;                   // of k, which passes once for each product of planes
    Planes planes;
    int each;                    // steps of a split
    int a_k, b_at;               // where k begins in a, and the tiles in b
};

struct Tile {
    int w, split, a, b;
};
__device__ __forceinline__ int64_t tiles_of(const Product& p) { return (int64_t)p.W * p.splits * p.tiles_a * p.tiles_b; }
// Groups of tiles along b, so that the tiles in work at a time share operands in L2.
__device__ __forceinline__ Tile tile_of(const Product& p, int64_t i) {
    const int64_t per = (int64_t)p.tiles_a * p.tiles_b;
    const int batch = static_cast<int>(i / per);
    const int64_t j = i - batch * per;
    const int group = static_cast<int>(j / ((int64_t)p.tiles_a * kGroup)), first = group * kGroup, wide = min(kGroup, p.tiles_b - first);
    const int64_t in = j - (int64_t)group * p.tiles_a * kGroup;
    const int a = static_cast<int>(in / wide);
    return {batch % p.W, batch / p.W, a, first + static_cast<int>(in - (int64_t)a * wide)};
}

template <bool SLOW>  // whether k is the operand's slow axis
__device__ __forceinline__ uint64_t matrix_at(uint32_t address) {
    return static_cast<uint64_t>((address & 0x3ffffu) >> 4) | static_cast<uint64_t>(SLOW ? kBlockBytes >> 4 : 1) << 16 |
           static_cast<uint64_t>(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
template <bool A_SLOW, bool B_SLOW>
constexpr uint32_t kInstruction = 1u << 4 | 1u << 7 | 1u << 10 | (A_SLOW ? 1u << 15 : 0u) | (B_SLOW ? 1u << 16 : 0u) | (kTileB / 8) << 17 |
                                  (kTileA / 16) << 24;

__device__ __forceinline__ void multiply(uint32_t sums, uint64_t a, uint64_t b, uint32_t instruction, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(sums),
        "l"(a), "l"(b), "r"(instruction), "r"(add ? 1u : 0u)
        : "memory");
}
__device__ __forceinline__ void arrive_when_multiplied(uint64_t* b) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(b)) : "memory");
}
// One copy per operand and step (boxes of 64 columns one by one took a sixth longer): an operand that has k as its slow
// axis is a tensor of groups of 64 columns, each group's rows one after another in shared memory.
template <bool SLOW>
__device__ __forceinline__ void copy_operand(uint32_t to, const CUtensorMap* map, int at, int k, int w, int plane, uint64_t* full) {
    if constexpr (SLOW)
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(to),
            "l"(map), "r"(0), "r"(k), "r"(at / 64), "r"(w), "r"(plane), "r"(smem_at(full))
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
            "l"(map), "r"(k), "r"(at), "r"(w), "r"(plane), "r"(smem_at(full))
            : "memory");
}

// E: the epilogue. run(v, w, split, a, b) takes 128 sums of lane a, columns b to b + 127.
template <bool A_SLOW, bool B_SLOW, typename E>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, Product p, E epilogue) {
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t full[kSlots], empty[kSlots], summed[2], taken[2], drained;
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;  // a wait of the block ran out
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t slots = (smem_at(raw) + 1023u) & ~1023u;
    if (threadIdx.x == 0) {
        failed = 0;
        for (int s = 0; s < kSlots; ++s) {
            barrier_init(&full[s], 1);
            barrier_init(&empty[s], 1);
        }
        for (int h = 0; h < 2; ++h) {
            barrier_init(&summed[h], 1);
            barrier_init(&taken[h], kEpilogueWarps);
        }
        barrier_init(&drained, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kMultiplyWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tensor_memory)), "r"(2 * kTileB)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t sums = tensor_memory;
    layer_begin();

    const int64_t tiles = tiles_of(p);
    const auto range = [&](const Tile& t, int& first, int& count) {
        first = t.split * p.each;
        count = min(p.steps * p.planes.products - first, p.each);
    };
    if (warp == kCopyWarp) {
        if (lane == 0) {
            int64_t n = 0;  // steps copied
            bool ok = true;
            for (int64_t i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
                const Tile t = tile_of(p, i);
                int first, count;
                range(t, first, count);
                for (int k = 0; k < count; ++k, ++n) {
                    const int s = static_cast<int>(n % kSlots);
                    ok = n < kSlots || barrier_wait(&empty[s], (n / kSlots - 1) & 1, &failed);
                    if (!ok) break;
#ifdef CPDP_CHECKED
                    if (n == *static_cast<volatile int*>(&dropped_step)) continue;
#endif
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(&full[s])), "r"(kSlotBytes) : "memory");
                    const int pass = (first + k) / p.steps, at = (first + k - pass * p.steps) * kStep;
                    const uint32_t slot = slots + s * kSlotBytes;
                    copy_operand<A_SLOW>(slot, &map_a, t.a * kTileA, p.a_k + at, t.w, p.planes.a >> 4 * pass & 15, &full[s]);
                    copy_operand<B_SLOW>(slot + kABytes, &map_b, p.b_at + t.b * kTileB, at, t.w, p.planes.b >> 4 * pass & 15,
                                                 &full[s]);
                }
            }
            // no copy may be in flight when the block ends, also where a wait ran out
            for (int64_t q = n > kSlots ? n - kSlots : 0; q < n; ++q) barrier_wait(&full[q % kSlots], q / kSlots & 1, &failed);
        }
    } else if (warp == kMultiplyWarp) {
        if (lane == 0) {
            int64_t n = 0, c = 0;  // steps and chunks multiplied
            bool ok = true;
            for (int64_t i = blockIdx.x; i < tiles && ok; i += gridDim.x) {
                int first, count;
                range(tile_of(p, i), first, count);
                for (int k0 = 0; k0 < count && ok; k0 += kChunk, ++c) {
                    const int half = c & 1, end = min(k0 + kChunk, count);
                    if (c >= 2) ok = barrier_wait(&taken[half], (c / 2 - 1) & 1, &failed);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int k = k0; k < end && ok; ++k, ++n) {
                        const int s = static_cast<int>(n % kSlots);
                        ok = barrier_wait(&full[s], n / kSlots & 1, &failed);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t a = matrix_at<A_SLOW>(slots + s * kSlotBytes), b = matrix_at<B_SLOW>(slots + s * kSlotBytes + kABytes);
#pragma unroll
                        for (int q = 0; q < kStep / 16; ++q)
                            multiply(sums + half * kTileB, a + q * (A_SLOW ? 2048 >> 4 : 32 >> 4), b + q * (B_SLOW ? 2048 >> 4 : 32 >> 4),
                                     kInstruction<A_SLOW, B_SLOW>, k > k0 || q > 0);
                        arrive_when_multiplied(&empty[s]);
                    }
                    if (ok) arrive_when_multiplied(&summed[half]);  // else nobody is told that the sums are there
                }
            }
            // nor a product
            arrive_when_multiplied(&drained);
            barrier_wait(&drained, 0, &failed);
        }
    } else {
        const int quarter = warp % 4 * 32, side = warp / 4 * kHalf;
        int64_t c = 0;
        bool ok = true;
        for (int64_t i = blockIdx.x; i < tiles; i += gridDim.x) {
            const Tile t = tile_of(p, i);
            int first, count;
            range(t, first, count);
            float v[kHalf];
            if (count <= 0)
#pragma unroll
                for (int j = 0; j < kHalf; ++j) v[j] = 0.f;
            for (int k0 = 0; k0 < count && ok; k0 += kChunk, ++c) {
                const int half = c & 1;
                ok = __all_sync(~0u, barrier_wait(&summed[half], c / 2 & 1, &failed));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t at = sums + half * kTileB + (quarter << 16) + side;
#pragma unroll
                for (int j = 0; j < kHalf; j += 32) {
                    uint32_t lo[16], hi[16];
                    read_sums(at + j, lo);
                    read_sums(at + j + 16, hi);
                    wait_read(lo);
                    wait_read(hi);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        v[j + e] = k0 == 0 ? __uint_as_float(lo[e]) : v[j + e] + __uint_as_float(lo[e]);
                        v[j + 16 + e] = k0 == 0 ? __uint_as_float(hi[e]) : v[j + 16 + e] + __uint_as_float(hi[e]);
                    }
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(&taken[half]);
            }
            // what a block makes whose wait ran out is not the product: from there on it says so
            if (!ok)
#pragma unroll
                for (int j = 0; j < kHalf; ++j) v[j] = __uint_as_float(0x7fc00000u);
            epilogue.run(v, t.w, t.split, t.a * kTileA + quarter + lane, t.b * kTileB + side);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (warp == kMultiplyWarp) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(sums), "r"(2 * kTileB));
    }
}

// Of 128 neighbouring logits of a token: their maximum and the sum of
// exp(l - maximum), for the words that there are; and the target's logit.
struct RowSums {
    const int64_t* targets;
    float2* parts;  // [blocks of 128 words][W * M]
    float* chosen;  // [W * M]
    int64_t M, rows;
    int V;
    __device__ __forceinline__ void run(const float (&v)[kHalf], int w, int, int a, int b) const {
        const int there = V - b;
        float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < kHalf; ++j) top[j % 4] = fmaxf(top[j % 4], j < there ? v[j] : -INFINITY);
        const float most = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
        const float base = isinf(most) ? 0.f : most;  // an infinite one leaves infinity or 0, as the formula has it
        float sum[4] = {};
#pragma unroll
        for (int j = 0; j < kHalf; ++j) {
            const float e = power((v[j] - base) * kLog2e);  // the difference first: 1 for the largest itself, however large
            sum[j % 4] += j < there ? e : 0.f;
        }
        const bool real = a < M;
        const int64_t row = w * M + a;
        const int64_t target = real ? targets[row] - b : -1;
        const bool mine = target >= 0 && target < kHalf && target < there;
        if (__any_sync(~0u, mine)) {
            float l = 0.f;
#pragma unroll
            for (int j = 0; j < kHalf; ++j) l = j == target ? v[j] : l;
            if (mine) chosen[row] = l;
        }
        if (real) parts[(int64_t)(b / kHalf) * rows + row] = make_float2(most == INFINITY ? 0.f : most, (sum[0] + sum[1]) + (sum[2] + sum[3]));
    }
};

// The same for float32 operands and few tokens, where making the planes of weight takes longer than all else: sums of
// float32 products. A block takes 128 words and kTokens tokens; its warps 8 words at a time, lanes side by side along the
// features, V of them together per lane. Up to 8 tokens it is bound by reading weight (seven workers' 4 tokens, 3,840 features,
// 3,589 words: 97 us for 368 with planes), then by the multiplications and x's loads (six workers' 19 tokens, 2,176
// features, 9,310 words: 251 for 448). At 32 tokens, 1,024 features and 32,768 words it takes 115 us for 126, at 771 features,
// off 16 bytes, and 10,007 words of two workers 90 for 82: the limit lies below that.
constexpr int kFewTokens = 24, kTokens = 8, kWordsAtOnce = 8;
// A step of the sums over lanes: half of the 2 HALF sums that are left go to the lane HALF / 2 away. Where the rest begins.
template <int HALF>
__device__ __forceinline__ int hand_over(float (&sum)[kWordsAtOnce * kTokens], int lane) {
    const bool high = lane & HALF / 2;
#pragma unroll
    for (int k = 0; k < HALF; ++k) {
        const float send = high ? sum[k] : sum[k + HALF], keep = high ? sum[k + HALF] : sum[k];
        sum[k] = keep + __shfl_xor_sync(~0u, send, HALF / 2);
    }
    return high ? HALF : 0;
}
template <int V>
__global__ void __launch_bounds__(256, 2)
few_tokens_kernel(const float* x, int64_t x_worker, int64_t x_row, const float* weight, int64_t weight_worker, int64_t weight_row,
                  const int64_t* targets, int M, int words, int D, float2* parts, float* chosen, int64_t rows) {
    layer_begin();
    __shared__ float logits[kTokens][kHalf + 1];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, w = blockIdx.z, first = blockIdx.y * kTokens, b = blockIdx.x * kHalf;
    const float* xs[kTokens];
#pragma unroll
    for (int j = 0; j < kTokens; ++j) xs[j] = x + w * x_worker + min(first + j, M - 1) * x_row;
    for (int at = warp * 16; at < warp * 16 + 16 && b + at < words; at += kWordsAtOnce) {
        const float* ws[kWordsAtOnce];
#pragma unroll
        for (int i = 0; i < kWordsAtOnce; ++i) ws[i] = weight + w * weight_worker + min(b + at + i, words - 1) * weight_row;
        float sum[kWordsAtOnce * kTokens] = {};
        for (int k = lane * V; k < D; k += 32 * V) {
            Piece<float, V> v[kWordsAtOnce];
#pragma unroll
            for (int i = 0; i < kWordsAtOnce; ++i)
                if constexpr (V == 1)
                    v[i].v = 0.f, v[i].load(ws[i] + k, true);
                else
                    v[i].load(ws[i] + k);
#pragma unroll
            for (int j = 0; j < kTokens; ++j) {
                float a[V];
                if constexpr (V == 4) {
                    const float4 four = *reinterpret_cast<const float4*>(xs[j] + k);
                    a[0] = four.x, a[1] = four.y, a[2] = four.z, a[3] = four.w;
                } else {
                    a[0] = xs[j][k];
                }
#pragma unroll
                for (int i = 0; i < kWordsAtOnce; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) sum[i * kTokens + j] = fmaf(v[i].get(e), a[e], sum[i * kTokens + j]);
            }
        }
        int mine = hand_over<32>(sum, lane);  // one after another
        mine += hand_over<16>(sum, lane);
        mine += hand_over<8>(sum, lane);
        mine += hand_over<4>(sum, lane);
        mine += hand_over<2>(sum, lane);  // two are left to a lane
#pragma unroll
        for (int k = 0; k < 2; ++k) logits[(mine + k) % kTokens][at + (mine + k) / kTokens] = sum[k];
    }
    __syncthreads();
    const int m = first + warp;  // a warp's token
    if (m >= M) return;
    const int64_t row = (int64_t)w * M + m, target = targets[row] - b;
    const int there = min(words - b, kHalf);
    float most = -INFINITY, all = 0.f;
    for (int j = lane; j < there; j += 32) most = fmaxf(most, logits[warp][j]);
#pragma unroll
    for (int k = 16; k > 0; k /= 2) most = fmaxf(most, __shfl_xor_sync(~0u, most, k));
    const float base = isinf(most) ? 0.f : most;
    for (int j = lane; j < there; j += 32) all += power((logits[warp][j] - base) * kLog2e);
#pragma unroll
    for (int k = 16; k > 0; k /= 2) all += __shfl_xor_sync(~0u, all, k);
    if (lane > 0) return;
    if (target >= 0 && target < there) chosen[row] = logits[warp][target];
    parts[(int64_t)blockIdx.x * rows + row] = make_float2(most == INFINITY ? 0.f : most, all);
}

// lse and loss of each token from its parts: ROWS tokens per block, whose other threads share the parts.
template <int ROWS>
__global__ void __launch_bounds__(256)
finish_rows_kernel(const float2* parts, const float* chosen, const int64_t* targets, int64_t rows, int blocks, int V, float* loss, float* lse) {
    layer_begin();
    constexpr int kShares = 256 / ROWS;
    __shared__ float2 shared[kShares][ROWS];
    const int in = threadIdx.x % ROWS, share = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + in;
    const bool real = row < rows;
    float most = -INFINITY, sum = 0.f;
    const auto add = [&](float2 p) {
        if (p.y == 0.f) return;  // nothing there: words beyond the last, or logits of -infinity
        const float next = fmaxf(most, p.x);
        sum = sum * power((most - next) * kLog2e) + p.y * power((p.x - next) * kLog2e);
        most = next;
    };
    if (real)
#pragma unroll 8
        for (int k = share; k < blocks; k += kShares) add(parts[(int64_t)k * rows + row]);
    shared[share][in] = make_float2(most, sum);
#pragma unroll
    for (int half = kShares / 2; half > 0; half /= 2) {
        __syncthreads();
        if (share < half) {
            add(shared[share + half][in]);
            shared[share][in] = make_float2(most, sum);
        }
    }
    if (share == 0 && real) {
        const float l = most + logf(sum);
        const int64_t t = targets[row];
        lse[row] = l;
        loss[row] = t < 0 ? 0.f : t >= V ? __uint_as_float(0x7fc00000u) : l - chosen[row];
    }
}

// The gradient of a token's logits, d = dloss (exp(l - lse) - onehot), in three
// planes of bfloat16 (the type of the products' operands).
struct LogitGradients {
    const int64_t* targets;
    const float *lse, *dloss;
    __nv_bfloat16* d;  // [plane][W][M][pitch]
    int64_t M, plane, pitch;
    int V, first;      // the piece's first word
    __device__ __forceinline__ void run(float (&v)[kHalf], int w, int, int a, int b) const {
        if (a >= M) return;
        const int64_t row = w * M + a, target = targets[row];
        const bool ignored = target < 0;
        const float l = target >= V ? __uint_as_float(0x7fc00000u) : lse[row], scale = ignored ? 0.f : dloss[row];
        const int64_t hot = target - first - b;
        __nv_bfloat16* to = d + row * pitch + b;
#pragma unroll
        for (int j = 0; j < kHalf; j += 16) {  // 32 bytes, a whole sector of L2; the pitch is of whole ones
            float g[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float p = power((v[j + e] - l) * kLog2e) - (j + e == hot ? 1.f : 0.f);
                g[e] = ignored ? 0.f : p * scale;
            }
            if (b + j < pitch)
#pragma unroll
            for (int q = 0; q < kPlanes; ++q) {
                uint32_t v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = cpdp::pack(g[2 * e], g[2 * e + 1]);
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + q * plane + j), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                             "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                             : "memory");
                if (q + 1 < kPlanes)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float held = __bfloat162float(__float2bfloat16_rn(g[e]));
                        g[e] = isfinite(held) ? g[e] - held : 0.f;
                    }
            }
        }
    }
};

// C written out, [b][a] with a contiguous; 0 in the rows of ignored tokens (targets not NULL). Or as a part of a sum
// (float32, of a split), which may be added to what is there.
template <typename G>
struct WriteOut {
    G* out;
    int64_t worker, split, row;
    const int64_t* targets;
    int a_extent, b_extent, add;
    __device__ __forceinline__ void run(const float (&v)[kHalf], int w, int s, int a, int b) const {
        // which of the columns' tokens are ignored: a load beside each store would wait for the store before it
        uint32_t ignored[kHalf / 32] = {};
        if (targets != nullptr)
#pragma unroll
            for (int j = 0; j < kHalf / 32; ++j) {
                const int at = b + j * 32 + static_cast<int>(threadIdx.x % 32);
                ignored[j] = __ballot_sync(~0u, at < b_extent && targets[(int64_t)w * b_extent + at] < 0);
            }
        const int there = a < a_extent ? b_extent - b : 0;
        G* to = out + w * worker + s * split + b * row + a;
        if (sizeof(G) == 4 && add) {  // one addition to each element per launch: the order is that of the launches
#pragma unroll
            for (int j = 0; j < kHalf; ++j, to += row)
                if (j < there) asm volatile("red.global.add.f32 [%0], %1;" ::"l"(to), "f"(v[j]) : "memory");
        } else {
#pragma unroll
            for (int j = 0; j < kHalf; ++j, to += row)
                if (j < there) *to = from_float<G>(ignored[j / 32] >> j % 32 & 1 ? 0.f : v[j]);
        }
    }
};

// The sum of the splits' parts [split][W][rows][D], in their order; 0 in ignored tokens' rows. A warp per 128
// neighbouring elements of a row, V of them together per lane: with a warp per row, 1,034 rows of 771 in 8 parts took
// 51 us.
constexpr int kSummed = 128;
template <typename G, int V>
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float* parts, int splits, int64_t rows_each, int64_t rows, int D, const int64_t* targets, G* out, int64_t worker) {
    layer_begin();
    constexpr int kPieces = kSummed / 32 / V;
    const int lane = threadIdx.x % 32, chunks = (D + kSummed - 1) / kSummed;
    const int64_t all = rows * D, tasks = rows * chunks;
    for (int64_t task = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; task < tasks; task += (int64_t)gridDim.x * 8) {
        const int64_t r = task / chunks, w = r / rows_each;
        const int k0 = static_cast<int>(task - r * chunks) * kSummed + lane * V;
        const bool ignored = targets != nullptr && targets[r] < 0;
        const float* p = parts + r * D + k0;
        G* to = out + w * worker + (r - w * rows_each) * D + k0;
        float s[kPieces][V] = {};
        if (V == 1 || k0 < D)  // one piece per lane, or pieces that are loaded where they are there
#pragma unroll 4
            for (int i = 0; i < splits; ++i)
#pragma unroll
                for (int q = 0; q < kPieces; ++q) {
                    Piece<float, V> v{};
                    if constexpr (V == 1)
                        v.load(p + i * all + q * 32, k0 + q * 32 < D);
                    else
                        v.load(p + i * all);
#pragma unroll
                    for (int e = 0; e < V; ++e) s[q][e] += v.get(e);
                }
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
#pragma unroll
            for (int e = 0; e < V; ++e) s[q][e] = ignored ? 0.f : s[q][e];
            if (k0 + q * 32 < D) store_piece<V>(to + q * 32, s[q]);
        }
    }
}

// An operand as the tensor copies need it: bfloat16 rows at multiples of 16
// bytes, [plane][W][rows][pitch], zeros in the rows of ignored tokens. Eight
// elements per thread and turn.
template <typename T, int PLANES>
__global__ void __launch_bounds__(256)
pack_kernel(const T* x, int64_t worker, int64_t stride, int64_t rows_each, int64_t rows, int D, int pitch, const int64_t* targets,
            __nv_bfloat16* out) {
    layer_begin();
    const int lane = threadIdx.x % 32;
    for (int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; row < rows; row += (int64_t)gridDim.x * 8) {
        const int64_t w = row / rows_each;
        const T* p = x + w * worker + (row - w * rows_each) * stride;
        const bool there = targets == nullptr || targets[row] >= 0;
        __nv_bfloat16* to = out + row * pitch;
#pragma unroll 2
        for (int k = lane * 8; k < pitch; k += 256) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                Piece<T, 1> one{};
                one.load(p + k + e, there && k + e < D);
                v[e] = one.get(0);
            }
#pragma unroll
            for (int q = 0; q < PLANES; ++q) {
                float held[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    // the largest float32 numbers would round to infinity: bfloat16's largest stands in, the next plane holds the rest
                    const float most = 3.38953139e38f, there = fminf(fmaxf(v[e], -most), most);
                    held[e] = PLANES > 1 && isfinite(v[e]) ? there : v[e];
                }
                store_piece<8>(to + q * rows * pitch + k, held);
                if (q + 1 < PLANES)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float rest = v[e] - __bfloat162float(__float2bfloat16_rn(held[e]));
                        v[e] = isfinite(v[e]) ? rest : 0.f;
                    }
            }
        }
    }
}

// -- the host's side -------------------------------------------------------------------------------------------------

constexpr int64_t kPieceBytes = int64_t(1) << 30;  // of d at a time

int64_t padded(int64_t bytes) { return ceil_div(bytes, 256) * 256; }
int64_t pitch_of(int64_t n) { return ceil_div(n, 64) * 64; }  // whole groups of columns

// How k is split among blocks: the number of parts that takes least time, by
// the turns that the tiles take on the SMs. A step of a tile takes 0.36 us, its
// start and end 3; parts cost their writing and reading at 4 TB/s and a launch.
struct Splits {
    int count, each;
};
Splits splits_of(int64_t tiles, int64_t steps, int64_t outputs) {
    Splits best{1, static_cast<int>(steps)};
    double least = 0;
    const int64_t most = std::max<int64_t>(ceil_div(2 * kSMs, tiles), tiles < 8 * kSMs ? 4 : 1);
    for (int64_t count = 1; count <= most && (count == 1 || count * 4 <= steps); ++count) {
        const int64_t each = std::max<int64_t>(ceil_div(steps, count), 1), parts = std::max<int64_t>(ceil_div(steps, each), 1);
        double us = static_cast<double>(ceil_div(tiles * parts, kSMs)) * (each * 0.36 + 3.0);
        if (parts > 1) us += 3.0 + 2e-6 * parts * outputs;
        if (count == 1 || us < least) least = us, best = {static_cast<int>(parts), static_cast<int>(each)};
    }
    return best;
}

// What a call computes from its sizes.
struct Plan {
    int planes;                        // of the operands
    Planes products, d_products;       // with the operands, and with d
    int64_t x_copy, weight_copy;       // bytes of the copies that the tensor copies read; 0: in place
    int64_t weight_columns;            // the same in the backward pass, which takes weight by whole groups of columns too
    bool few;                          // forward: float32 products, without planes
    int64_t parts, chosen;             // forward
    int words, pieces;                 // of a piece, and how many
    int64_t pitch, d;                  // of d, and its bytes
    Splits dx, dweight;
    int64_t dx_parts, dweight_parts;   // bytes; 0: written in place
    int64_t forward, backward;         // bytes in all
};

bool in_place(const void* p, int64_t worker, int64_t row, cpdp_dtype dtype, int W, int64_t rows, int64_t D) {
    return dtype == CPDP_BF16 && aligned_to(p, 16) && (rows <= 1 || (row % 8 == 0 && row >= D && row < (int64_t(1) << 38))) &&
           (W <= 1 || (worker % 8 == 0 && worker > 0 && worker < (int64_t(1) << 38)));
}

Plan plan_of(const void* x, int64_t x_worker, int64_t x_row, const void* weight, int64_t weight_worker, int64_t weight_row, cpdp_dtype dtype,
             int W, int64_t M, int V, int D) {
    Plan p{};
    p.planes = dtype == CPDP_F32 ? kPlanes : 1;
    p.products = dtype == CPDP_F32 ? kThreePlanes : kOnePlane;
    p.d_products = dtype == CPDP_F32 ? kThreePlanes : kThreeOfD;
    const int64_t pitch = pitch_of(D), packed = padded(p.planes * W * M * pitch * 2);
    p.x_copy = in_place(x, x_worker, x_row, dtype, W, M, D) ? 0 : packed;
    p.weight_copy = in_place(weight, weight_worker, weight_row, dtype, W, V, D) ? 0 : padded(p.planes * W * (int64_t)V * pitch * 2);
    p.weight_columns = p.weight_copy || D % 64 == 0 ? p.weight_copy : padded(W * (int64_t)V * pitch * 2);
    const int64_t rows = W * M;
    p.parts = padded(ceil_div(V, kTileB) * 2 * rows * 8);
    p.chosen = padded(rows * 4);
    if (dtype == CPDP_F32 && M <= kFewTokens) p.x_copy = p.weight_copy = 0, p.few = true;
    p.forward = p.x_copy + p.weight_copy + p.parts + p.chosen;

    const int64_t fit = std::max<int64_t>(kPieceBytes / (kPlanes * 2 * std::max<int64_t>(rows, 1)), kTileB);
    p.pieces = static_cast<int>(ceil_div(V, fit));
    p.words = static_cast<int>(std::min<int64_t>(ceil_div(ceil_div(V, p.pieces), kTileB) * kTileB, ceil_div(V, kTileB) * kTileB));
    p.pieces = static_cast<int>(ceil_div(V, p.words));
    p.pitch = pitch_of(std::min(p.words, V));
    p.d = padded(kPlanes * rows * p.pitch * 2) + 16;  // room to begin at 32 bytes
    const int64_t tiles_d = ceil_div(D, kTileA);
    p.dx = splits_of(W * tiles_d * ceil_div(M, kTileB), ceil_div(std::min(p.words, V), kStep) * p.d_products.products, rows * D);
    p.dweight = splits_of(W * tiles_d * ceil_div(std::min(p.words, V), kTileB), ceil_div(M, kStep) * p.d_products.products, (int64_t)W * std::min(p.words, V) * D);
    p.dx_parts = p.dx.count > 1 || p.pieces > 1 ? padded(p.dx.count * rows * D * 4) : 0;
    p.dweight_parts = p.dweight.count > 1 ? padded((int64_t)p.dweight.count * W * std::min(p.words, V) * D * 4) : 0;
    p.backward = packed + p.weight_columns + p.d + p.dx_parts + p.dweight_parts;
    return p;
}

// A matrix [plane][W][rows][columns] of bfloat16 and the box that a copy takes of it.
cpdp_status encode(CUtensorMap* map, const void* p, int64_t columns, int64_t rows, int W, int planes, int64_t row, int64_t worker, int64_t plane,
                   int box_rows) {
    const EncodeTiled f = encode_tiled();
    if (f == nullptr) return layer_error(CPDP_ECUDA, "the CUDA driver has no cuTensorMapEncodeTiled");
    if (rows <= 1) row = pitch_of(columns);  // strides that no index uses
    if (W <= 1) worker = row * rows;
    if (planes <= 1) plane = worker * W;
    const cuuint64_t dims[4] = {(cuuint64_t)columns, (cuuint64_t)rows, (cuuint64_t)W, (cuuint64_t)planes},
                     strides[3] = {(cuuint64_t)row * 2, (cuuint64_t)worker * 2, (cuuint64_t)plane * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return layer_error(CPDP_ECUDA, "cuTensorMapEncodeTiled: error %d", (int)r);
    return CPDP_OK;
}

// The same by groups of 64 columns, of which a box takes `box_columns` in kStep rows. What lies beside the columns of a
// last, partial group is read, and must be there; no product that is kept uses it.
cpdp_status encode_columns(CUtensorMap* map, const void* p, int64_t columns, int64_t rows, int W, int planes, int64_t row, int64_t worker,
                           int64_t plane, int box_columns) {
    const EncodeTiled f = encode_tiled();
    if (f == nullptr) return layer_error(CPDP_ECUDA, "the CUDA driver has no cuTensorMapEncodeTiled");
    if (rows <= 1) row = pitch_of(columns);
    if (W <= 1) worker = row * rows;
    if (planes <= 1) plane = worker * W;
    const cuuint64_t dims[5] = {64, (cuuint64_t)rows, (cuuint64_t)ceil_div(columns, 64), (cuuint64_t)W, (cuuint64_t)planes},
                     strides[4] = {(cuuint64_t)row * 2, 128, (cuuint64_t)worker * 2, (cuuint64_t)plane * 2};
    const cuuint32_t box[5] = {64, kStep, (cuuint32_t)box_columns / 64, 1, 1}, one[5] = {1, 1, 1, 1, 1};
    const CUresult r = f(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void*>(p), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                         CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return layer_error(CPDP_ECUDA, "cuTensorMapEncodeTiled: error %d", (int)r);
    return CPDP_OK;
}

template <bool A_SLOW, bool B_SLOW, typename E>
cpdp_status multiply_all(const CUtensorMap& a, const CUtensorMap& b, const Product& p, const E& epilogue, void* stream, const char* what) {
    const int64_t tiles = (int64_t)p.W * p.splits * p.tiles_a * p.tiles_b;
    cudaError_t e = allow_shared_memory<product_kernel<A_SLOW, B_SLOW, E>>(kSmemBytes);
    if (e == cudaSuccess)
        e = launch_layer(product_kernel<A_SLOW, B_SLOW, E>, static_cast<unsigned>(std::min<int64_t>(tiles, kSMs)), kThreads, kSmemBytes, stream, a, b, p,
                         epilogue);
    return layer_launched(e, what);
}

Product product(int W, int64_t a, int64_t b, int64_t k, const Planes& planes, Splits s = {1, 0}) {
    Product p{};
    p.W = W;
    p.tiles_a = static_cast<int>(ceil_div(a, kTileA)), p.tiles_b = static_cast<int>(ceil_div(b, kTileB));
    p.steps = static_cast<int>(ceil_div(k, kStep)), p.planes = planes;
    p.splits = s.count, p.each = s.each > 0 ? s.each : p.steps * planes.products;
    return p;
}

cpdp_status pack(const void* x, int64_t worker, int64_t stride, cpdp_dtype dtype, int W, int64_t rows_each, int D, const int64_t* targets, void* out,
                 void* stream, const char* what) {
    const int64_t rows = W * rows_each;
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(ceil_div(rows, 8), kSMs * 8));
    const int pitch = static_cast<int>(pitch_of(D));
    auto* to = static_cast<__nv_bfloat16*>(out);
    return layer_launched(dtype == CPDP_F32
                              ? launch_layer(pack_kernel<float, kPlanes>, blocks, 256, 0, stream, static_cast<const float*>(x), worker, stride,
                                             rows_each, rows, D, pitch, targets, to)
                              : launch_layer(pack_kernel<__nv_bfloat16, 1>, blocks, 256, 0, stream, static_cast<const __nv_bfloat16*>(x), worker,
                                             stride, rows_each, rows, D, pitch, targets, to),
                          what);
}

cpdp_status check_loss(const void* x, int64_t x_worker, int64_t x_row, const void* weight, int64_t weight_worker, int64_t weight_row, cpdp_dtype dtype,
                       int W, int64_t M, int V, int D, const int64_t* targets) {
    CPDP_TRY(check_sizes(W, M, D));
    CPDP_TRY(check_sizes(W, V, D));
    CPDP_TRY(check_sizes(W, M, V));
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    if (V < 1 || V > kLayerMaxFeatures || M > kLayerMaxFeatures)
        return layer_error(CPDP_EINVAL, "V=%d must be in [1, 2^30] and M=%lld at most 2^30", V, (long long)M);
    CPDP_TRY(check_array("x", x, M > 0, dtype_size(dtype), x_worker, x_row));
    CPDP_TRY(check_array("weight", weight, true, dtype_size(dtype), weight_worker, weight_row));
    return check_array("targets", targets, M > 0, 8);
}

}  // namespace

#ifdef CPDP_CHECKED
extern "C" cpdp_status cpdp_layer_drop_loss_step(int step) {
    return layer_launched(cudaMemcpyToSymbol(dropped_step, &step, sizeof step), "cpdp_layer_drop_loss_step");
}
#endif

cudaError_t take_loss_timeouts(unsigned long long* count) {
    unsigned long long zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(count, wait_timeouts, sizeof *count);
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(wait_timeouts, &zero, sizeof zero);
    return e;
}

}  // namespace cpdp

using namespace cpdp;

static bool loss_sizes(int W, int64_t M, int V, int D) {
    return check_sizes(W, M, D) == CPDP_OK && check_sizes(W, V, D) == CPDP_OK && check_sizes(W, M, V) == CPDP_OK && V >= 1 &&
           V <= kLayerMaxFeatures && M <= kLayerMaxFeatures;
}

size_t cpdp_linear_cross_entropy_workspace(const void* x, int64_t x_worker, int64_t x_row, const void* weight, int64_t weight_worker,
                                           int64_t weight_row, cpdp_dtype dtype, int W, int64_t M, int V, int D) {
    if (!loss_sizes(W, M, V, D) || M == 0) return 0;
    return plan_of(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D).forward;
}

size_t cpdp_linear_cross_entropy_backward_workspace(const void* x, int64_t x_worker, int64_t x_row, const void* weight, int64_t weight_worker,
                                                    int64_t weight_row, cpdp_dtype dtype, int W, int64_t M, int V, int D) {
    if (!loss_sizes(W, M, V, D) || M == 0) return 0;
    return plan_of(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D).backward;
}

namespace {
struct Where {
    const void* p;
    int64_t worker, row, plane;
};
}  // namespace

cpdp_status cpdp_linear_cross_entropy(const void* x, int64_t x_worker, int64_t x_row, const void* weight, int64_t weight_worker,
                                      int64_t weight_row, const int64_t* targets, cpdp_dtype dtype, int W, int64_t M, int V, int D, float* loss,
                                      float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    constexpr const char* what = "cpdp_linear_cross_entropy";
    CPDP_TRY(check_loss(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D, targets));
    CPDP_TRY(check_array("loss", loss, M > 0, 4));
    CPDP_TRY(check_array("lse", lse, M > 0, 4));
    if (M == 0) return CPDP_OK;
    const Plan plan = plan_of(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D);
    CPDP_TRY(check_workspace(workspace, workspace_bytes, plan.forward));
    const int64_t pitch = pitch_of(D), rows = W * M;
    char* at = static_cast<char*>(workspace);
    Where xs{x, x_worker, x_row, 0}, ws{weight, weight_worker, weight_row, 0};
    if (plan.x_copy) {
        CPDP_TRY(pack(x, x_worker, x_row, dtype, W, M, D, nullptr, at, stream, what));
        xs = {at, M * pitch, pitch, rows * pitch};
        at += plan.x_copy;
    }
    if (plan.weight_copy) {
        CPDP_TRY(pack(weight, weight_worker, weight_row, dtype, W, V, D, nullptr, at, stream, what));
        ws = {at, V * pitch, pitch, (int64_t)W * V * pitch};
        at += plan.weight_copy;
    }
    auto* parts = reinterpret_cast<float2*>(at);
    auto* chosen = reinterpret_cast<float*>(at + plan.parts);
    if (plan.few) {
        const auto fours = [&](const void* p, int64_t worker, int64_t row) { return aligned_to(p, 16) && worker % 4 == 0 && row % 4 == 0; };
        const bool wide = D % 4 == 0 && fours(x, x_worker, x_row) && fours(weight, weight_worker, weight_row);
        const dim3 grid(static_cast<unsigned>(ceil_div(V, kTileB) * 2), static_cast<unsigned>(ceil_div(M, kTokens)), W);
        CPDP_TRY(layer_launched(launch_layer(wide ? few_tokens_kernel<4> : few_tokens_kernel<1>, grid, 256, 0, stream, static_cast<const float*>(x),
                                             x_worker, x_row, static_cast<const float*>(weight), weight_worker, weight_row, targets,
                                             static_cast<int>(M), V, D, parts, chosen, rows),
                                what));
    } else {
        CUtensorMap a, b;
        CPDP_TRY(encode(&a, xs.p, D, M, W, plan.planes, xs.row, xs.worker, xs.plane, kTileA));
        CPDP_TRY(encode(&b, ws.p, D, V, W, plan.planes, ws.row, ws.worker, ws.plane, kTileB));
        CPDP_TRY((multiply_all<false, false>(a, b, product(W, M, V, D, plan.products), RowSums{targets, parts, chosen, M, rows, V}, stream,
                                             what)));
    }
    const auto finish = [&](auto kernel, int each) {
        return launch_layer(kernel, static_cast<unsigned>(ceil_div(rows, each)), 256, 0, stream, static_cast<const float2*>(parts),
                            static_cast<const float*>(chosen), targets, rows, static_cast<int>(ceil_div(V, kTileB) * 2), V, loss, lse);
    };
    // few tokens: few blocks, and long sums for each of their threads
    return layer_launched(rows < kSMs * 32 ? finish(finish_rows_kernel<4>, 4) : finish(finish_rows_kernel<32>, 32), what);
}

template <typename G>
static cudaError_t sum_parts(const float* parts, int splits, int64_t rows_each, int W, int D, const int64_t* targets, G* out, int64_t worker,
                             void* stream) {
    const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(ceil_div(rows_each * W * ceil_div(D, kSummed), 8), kSMs * 8));
    const bool fours = D % 4 == 0 && aligned_to(out, 4 * sizeof(G)) && (W == 1 || worker % 4 == 0);
    return launch_layer(fours ? sum_parts_kernel<G, 4> : sum_parts_kernel<G, 1>, blocks, 256, 0, stream, parts, splits, rows_each, rows_each * W, D,
                        targets, out, worker);
}

template <typename G>
static cpdp_status zero_rows(G* out, int64_t worker, int W, int64_t each, void* stream) {
    for (int w = 0; w < W; ++w) {
        const cudaError_t e = cudaMemsetAsync(out + w * worker, 0, each * sizeof(G), static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return layer_launched(e, "cpdp_linear_cross_entropy_backward");
    }
    return CPDP_OK;
}

cpdp_status cpdp_linear_cross_entropy_backward(const float* dloss, const void* x, int64_t x_worker, int64_t x_row, const void* weight,
                                               int64_t weight_worker, int64_t weight_row, const int64_t* targets, const float* lse,
                                               cpdp_dtype dtype, int W, int64_t M, int V, int D, void* dx, void* dweight, int64_t dweight_worker,
                                               cpdp_dtype dweight_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    constexpr const char* what = "cpdp_linear_cross_entropy_backward";
    CPDP_TRY(check_loss(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D, targets));
    if (!known_dtype(dweight_dtype)) return layer_error(CPDP_EINVAL, "unknown dtype of dweight: %d", (int)dweight_dtype);
    CPDP_TRY(check_array("dloss", dloss, M > 0, 4));
    CPDP_TRY(check_array("lse", lse, M > 0, 4));
    CPDP_TRY(check_array("dx", dx, M > 0, dtype_size(dtype)));
    CPDP_TRY(check_array("dweight", dweight, true, dtype_size(dweight_dtype), dweight_worker));
    CPDP_TRY(check_apart("dweight", W, dweight_worker, (int64_t)V * D));
    if (M == 0)
        return dweight_dtype == CPDP_F32 ? zero_rows(static_cast<float*>(dweight), dweight_worker, W, (int64_t)V * D, stream)
                                         : zero_rows(static_cast<__nv_bfloat16*>(dweight), dweight_worker, W, (int64_t)V * D, stream);
    const Plan plan = plan_of(x, x_worker, x_row, weight, weight_worker, weight_row, dtype, W, M, V, D);
    CPDP_TRY(check_workspace(workspace, workspace_bytes, plan.backward));
    const int64_t pitch = pitch_of(D), rows = W * M;
    char* at = static_cast<char*>(workspace);
    // x with zeros for ignored tokens: what lies there must not reach dweight
    CPDP_TRY(pack(x, x_worker, x_row, dtype, W, M, D, targets, at, stream, what));
    const Where xs{at, M * pitch, pitch, rows * pitch};
    at += padded(plan.planes * rows * pitch * 2);
    Where ws{weight, weight_worker, weight_row, 0};
    if (plan.weight_columns) {
        CPDP_TRY(pack(weight, weight_worker, weight_row, dtype, W, V, D, nullptr, at, stream, what));
        ws = {at, V * pitch, pitch, (int64_t)W * V * pitch};
        at += plan.weight_columns;
    }
    auto* d = reinterpret_cast<__nv_bfloat16*>((reinterpret_cast<uintptr_t>(at) + 31) & ~uintptr_t(31));
    auto* dx_parts = reinterpret_cast<float*>(at + plan.d);
    auto* dweight_parts = reinterpret_cast<float*>(at + plan.d + plan.dx_parts);

    CUtensorMap x_rows, x_columns, w_rows, w_columns, d_rows, d_columns;
    CPDP_TRY(encode(&x_rows, xs.p, D, M, W, plan.planes, xs.row, xs.worker, xs.plane, kTileA));
    CPDP_TRY(encode_columns(&x_columns, xs.p, D, M, W, plan.planes, xs.row, xs.worker, xs.plane, kTileA));
    CPDP_TRY(encode(&w_rows, ws.p, D, V, W, plan.planes, ws.row, ws.worker, ws.plane, kTileB));
    CPDP_TRY(encode_columns(&w_columns, ws.p, D, V, W, plan.planes, ws.row, ws.worker, ws.plane, kTileA));
    for (int piece = 0; piece < plan.pieces; ++piece) {
        const int first = piece * plan.words, words = std::min(plan.words, V - first);
        const int64_t plane = rows * plan.pitch;
        CPDP_TRY(encode(&d_rows, d, words, M, W, kPlanes, plan.pitch, M * plan.pitch, plane, kTileB));
        CPDP_TRY(encode_columns(&d_columns, d, words, M, W, kPlanes, plan.pitch, M * plan.pitch, plane, kTileB));
        Product p = product(W, M, words, D, plan.products);
        p.b_at = first;
        CPDP_TRY((multiply_all<false, false>(x_rows, w_rows, p, LogitGradients{targets, lse, dloss, d, M, plane, plan.pitch, V, first}, stream, what)));

        p = product(W, D, M, words, plan.d_products, plan.dx);
        p.splits = static_cast<int>(ceil_div(p.steps * p.planes.products, p.each));  // a last piece may have fewer words
        p.a_k = first;
        if (plan.dx_parts) {
            CPDP_TRY((multiply_all<true, false>(w_columns, d_rows, p,
                                                WriteOut<float>{dx_parts, M * D, rows * D, D, nullptr, D, (int)M, piece > 0}, stream, what)));
        } else {
            const auto write = [&](auto* out) {
                using G = std::remove_pointer_t<decltype(out)>;
                return multiply_all<true, false>(w_columns, d_rows, p, WriteOut<G>{out, M * D, 0, D, targets, D, (int)M, 0}, stream, what);
            };
            CPDP_TRY(dtype == CPDP_F32 ? write(static_cast<float*>(dx)) : write(static_cast<__nv_bfloat16*>(dx)));
        }

        p = product(W, D, words, M, plan.d_products, plan.dweight);
        const int64_t part = (int64_t)words * D;
        if (plan.dweight_parts) {
            CPDP_TRY((multiply_all<true, true>(x_columns, d_columns, p,
                                               WriteOut<float>{dweight_parts, part, W * part, D, nullptr, D, words, 0}, stream, what)));
            const auto sum = [&](auto* out) { return sum_parts(dweight_parts, p.splits, words, W, D, nullptr, out + (int64_t)first * D, dweight_worker, stream); };
            CPDP_TRY(layer_launched(dweight_dtype == CPDP_F32 ? sum(static_cast<float*>(dweight)) : sum(static_cast<__nv_bfloat16*>(dweight)), what));
        } else {
            const auto write = [&](auto* out) {
                using G = std::remove_pointer_t<decltype(out)>;
                return multiply_all<true, true>(x_columns, d_columns, p,
                                                WriteOut<G>{out + (int64_t)first * D, dweight_worker, 0, D, nullptr, D, words, 0}, stream, what);
            };
            CPDP_TRY(dweight_dtype == CPDP_F32 ? write(static_cast<float*>(dweight)) : write(static_cast<__nv_bfloat16*>(dweight)));
        }
    }
    if (!plan.dx_parts) return CPDP_OK;
    const auto sum = [&](auto* out) { return sum_parts(dx_parts, plan.dx.count, M, W, D, targets, out, M * D, stream); };
    return layer_launched(dtype == CPDP_F32 ? sum(static_cast<float*>(dx)) : sum(static_cast<__nv_bfloat16*>(dx)), what);
}
