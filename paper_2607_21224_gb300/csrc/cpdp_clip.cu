// Gradient norms over the workers' rows and their clipping
// (include/cpdp_layers.h).
#include <algorithm>
#include <type_traits>

#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

// norm = sqrt(sum(g^2)) of a row, out = g * min(1, max_norm / norm). Both passes
// are bound by memory. The first leaves each block's part of the sum; in the
// second every block adds up its row's parts, in their order, and walks its own
// part of the row from the end, so that it begins with what is still in L2; what
// it writes is marked to leave L2 first. Rows that fill L2 together pass one group
// after another: 8 rows of 95 MB (float32) take 335 us, all in one launch of each
// pass 376, and 396 without the marks; two passes over memory would be 336, and
// reading and writing everything once 224.
constexpr int kThreads = 256, kVectors = 4;  // 16 bytes each, per thread and turn
constexpr int kMostParts = 8 * kSMs;

// Squares of float32 overflow from 1.8e19 on and vanish below 1e-23. Sums of
// squares of values times 2^-96 and 2^96 stand in there.
constexpr float kDown = 0x1p-96f, kUp = 0x1p96f;
struct Squares {
    float mid, down, up;
    __device__ __forceinline__ void add(float g) {
        mid = fmaf(g, g, mid);
        down = fmaf(g * kDown, g * kDown, down);
        up = fmaf(g * kUp, g * kUp, up);
    }
    __device__ __forceinline__ void add(const Squares& o) { mid += o.mid, down += o.down, up += o.up; }
};
__device__ __forceinline__ Squares over_warp(Squares s) {
#pragma unroll
    for (int d = 16; d > 0; d /= 2)
        s.add({__shfl_xor_sync(~0u, s.mid, d), __shfl_xor_sync(~0u, s.down, d), __shfl_xor_sync(~0u, s.up, d)});
    return s;
}
__device__ __forceinline__ Squares over_block(Squares s) {
    __shared__ Squares warps[kThreads / 32];
    s = over_warp(s);
    __syncthreads();
    if (threadIdx.x % 32 == 0) warps[threadIdx.x / 32] = s;
    __syncthreads();
    s = warps[0];
#pragma unroll
    for (int i = 1; i < kThreads / 32; ++i) s.add(warps[i]);
    return s;
}
// NaN where one is in the row, infinity where the norm is above the float32 range.
__device__ __forceinline__ float norm_of(const Squares& s) {
    if (s.mid >= 0x1p-90f && s.mid <= 0x1p100f) return sqrtf(s.mid);
    if (s.mid < 0x1p-90f) return sqrtf(s.up) * kDown;
    return sqrtf(s.down) * kUp;  // infinite and NaN sums too
}

// A row in 16-byte pieces: elements before the first whole piece, the pieces, and the elements after them.
template <typename T>
constexpr int kEach = 16 / sizeof(T);
template <typename T>
struct Row {
    int64_t head, pieces;
    __device__ __forceinline__ Row(const T* p, int64_t n) {
        const int64_t before = ((16 - reinterpret_cast<uintptr_t>(p) % 16) % 16) / sizeof(T);
        head = before < n ? before : n;
        pieces = (n - head) / kEach<T>;
    }
};

template <typename T>
__global__ void __launch_bounds__(kThreads)
norms_kernel(const T* grads, int64_t worker, int64_t n, Squares* parts) {
    layer_begin();
    const T* g = grads + blockIdx.y * worker;
    const Row<T> row(g, n);
    Squares s{};
    constexpr int64_t kTurn = kThreads * kVectors;
    for (int64_t i = blockIdx.x * kTurn; i < row.pieces; i += gridDim.x * kTurn) {
        Piece<T, kEach<T>> v[kVectors];
#pragma unroll
        for (int k = 0; k < kVectors; ++k) {
            const int64_t at = i + k * kThreads + threadIdx.x;
            if (at < row.pieces) v[k].v = *reinterpret_cast<const decltype(v[k].v)*>(g + row.head + at * kEach<T>);
        }
        Squares turn{};
#pragma unroll
        for (int k = 0; k < kVectors; ++k)
            if (i + k * kThreads + threadIdx.x < row.pieces)
#pragma unroll
                for (int e = 0; e < kEach<T>; ++e) turn.add(v[k].get(e));
        s.add(turn);
    }
    if (blockIdx.x == 0 && threadIdx.x < kEach<T>) {
        const int64_t after = row.head + row.pieces * kEach<T> + threadIdx.x;
        if (threadIdx.x < row.head) s.add(to_float(g[threadIdx.x]));
        if (after < n) s.add(to_float(g[after]));
    }
    s = over_block(s);
    if (threadIdx.x == 0) parts[blockIdx.y * gridDim.x + blockIdx.x] = s;
}

__device__ __forceinline__ void store_streaming(float* p, const float (&v)[4]) {
    __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
}
__device__ __forceinline__ void store_streaming(__nv_bfloat16* p, const float (&v)[8]) {
    __stcs(reinterpret_cast<uint4*>(p), make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7])));
}

// ALIGNED: rows of out lie in 16 bytes as those of grads do.
template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads)
clip_kernel(const T* grads, int64_t worker, int64_t n, const Squares* parts, int count, float max_norm, float* norms, T* out, int64_t out_worker) {
    layer_begin();
    Squares s{};
    for (int i = threadIdx.x; i < count; i += kThreads) s.add(parts[blockIdx.y * count + i]);
    const float norm = norm_of(over_block(s));
    if (blockIdx.x == 0 && threadIdx.x == 0) norms[blockIdx.y] = norm;
    // an infinite max_norm is above every norm, infinity and NaN too
    const float ratio = max_norm / norm;
    // a ratio near the end of the float32 range would have few bits, or none: 2^112 of it, and the products times 2^-112
    // (max_norm is below 2^8 then, and what is scaled below 2^120)
    const bool tiny = ratio < 0x1p-120f && norm < INFINITY;
    const float scale = ratio > 1.f || isinf(max_norm) ? 1.f : tiny ? max_norm * 0x1p112f / norm : ratio, after_scale = tiny ? 0x1p-112f : 1.f;
    const T* g = grads + blockIdx.y * worker;
    T* to = out + blockIdx.y * out_worker;
    const bool keep = scale == 1.f;  // as they lie in memory, whatever NaN's bits
    if (g == to && keep) return;
    const auto scaled = [&](T x) { return keep ? x : from_float<T>(to_float(x) * scale * after_scale); };
    const Row<T> row(g, n);
    constexpr int64_t kTurn = kThreads * kVectors;
    if constexpr (ALIGNED) {
        // the block's own turns of the first pass, the last first
        const int64_t turns = (row.pieces + kTurn - 1) / kTurn, own = (turns - blockIdx.x + gridDim.x - 1) / gridDim.x;
        for (int64_t turn = blockIdx.x + (own - 1) * gridDim.x; turn >= 0; turn -= gridDim.x) {
            Piece<T, kEach<T>> v[kVectors];
#pragma unroll
            for (int k = 0; k < kVectors; ++k) {
                const int64_t at = turn * kTurn + k * kThreads + threadIdx.x;
                if (at < row.pieces) v[k].load(g + row.head + at * kEach<T>);
            }
#pragma unroll
            for (int k = 0; k < kVectors; ++k) {
                const int64_t at = turn * kTurn + k * kThreads + threadIdx.x;
                float x[kEach<T>];
#pragma unroll
                for (int e = 0; e < kEach<T>; ++e) x[e] = v[k].get(e) * scale * after_scale;
                if (at < row.pieces) {
                    if (keep)
                        __stcs(reinterpret_cast<decltype(v[k].v)*>(to + row.head + at * kEach<T>), v[k].v);
                    else
                        store_streaming(to + row.head + at * kEach<T>, x);
                }
            }
        }
        if (blockIdx.x == 0 && threadIdx.x < kEach<T>) {
            const int64_t after = row.head + row.pieces * kEach<T> + threadIdx.x;
            if (threadIdx.x < row.head) to[threadIdx.x] = scaled(g[threadIdx.x]);
            if (after < n) to[after] = scaled(g[after]);
        }
    } else {
        const int64_t turns = (n + kThreads - 1) / kThreads;
#pragma unroll 4
        for (int64_t turn = turns - 1 - blockIdx.x; turn >= 0; turn -= gridDim.x) {
            const int64_t at = turn * kThreads + threadIdx.x;
            if (at < n) to[at] = scaled(g[at]);
        }
    }
}

// Blocks of a row, at most kMostParts: one turn each where that is not more than run at once.
int parts_of(int W, int64_t N) {
    const int64_t turns = ceil_div(N * 4, kThreads * kVectors * 16), most = ceil_div(kMostParts, W);
    return static_cast<int>(std::max<int64_t>(std::min(turns, most), 1));
}

// Rows of one launch of each pass: all, or as many as L2 may hold.
constexpr int64_t kHeld = int64_t(96) << 20;
int group_of(int W, int64_t N, int64_t size) {
    return static_cast<int>(N > 0 && W > kHeld / (N * size) ? std::max<int64_t>(kHeld / (N * size), 1) : W);
}

cpdp_status check_clip(int W, int64_t N) {
    if (W < 1 || W > 4096) return layer_error(CPDP_EINVAL, "W=%d must be in [1, 4096]", W);
    if (N < 0 || N > kLayerMaxElements / W) return layer_error(CPDP_EINVAL, "W=%d, N=%lld: W * N must be in [0, 2^40]", W, (long long)N);
    return CPDP_OK;
}

// Whether rows of `size` bytes at a and at b overlap, where they are not the same ones. Rows of one stride may lie between
// each other.
bool rows_meet(uintptr_t a, int64_t a_stride, uintptr_t b, int64_t b_stride, int W, int64_t size) {
    if (size == 0 || a == b) return false;
    const int64_t a_span = (W - 1) * a_stride + size, b_span = (W - 1) * b_stride + size;
    if (a + a_span <= b || b + b_span <= a) return false;
    if (W == 1 || a_stride != b_stride) return true;
    const int64_t after = a < b ? (b - a) % a_stride : a_stride - (a - b) % a_stride;  // from a row of a to the next one of b
    return after < size || after > a_stride - size;
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

size_t cpdp_clip_gradients_workspace(int W, int64_t N) {
    return check_clip(W, N) != CPDP_OK ? 0 : ceil_div((static_cast<int64_t>(W) * parts_of(W, N) + kMostParts) * sizeof(Squares), 16) * 16;
}

cpdp_status cpdp_clip_gradients(const void* grads, int64_t grads_worker, cpdp_dtype dtype, int W, int64_t N, float max_norm, float* norms,
                                void* out, int64_t out_worker, void* workspace, size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_clip(W, N));
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    if (!(max_norm > 0.f)) return layer_error(CPDP_EINVAL, "max_norm=%g must be above 0", (double)max_norm);
    const int64_t e = dtype_size(dtype);
    CPDP_TRY(check_array("grads", grads, N > 0, e, grads_worker));
    CPDP_TRY(check_array("norms", norms, true, 4));
    CPDP_TRY(check_array("out", out, N > 0, e, out_worker));
    CPDP_TRY(check_apart("out", W, out_worker, N));
    if (out == grads && W > 1 && out_worker != grads_worker)
        return layer_error(CPDP_EINVAL, "out is grads with another stride: %lld, not %lld", (long long)out_worker, (long long)grads_worker);
    if (rows_meet(reinterpret_cast<uintptr_t>(grads), grads_worker * e, reinterpret_cast<uintptr_t>(out), out_worker * e, W, N * e))
        return layer_error(CPDP_EINVAL, "rows of out (%p) overlap rows of grads (%p) and are not the same", out, grads);
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_clip_gradients_workspace(W, N)));
    auto* parts = static_cast<Squares*>(workspace);
    const bool aligned = (reinterpret_cast<uintptr_t>(grads) - reinterpret_cast<uintptr_t>(out)) % 16 == 0 &&
                         (W == 1 || (grads_worker - out_worker) * e % 16 == 0);
    const int together = group_of(W, N, e);
    const auto go = [&](auto* all) {
        using T = std::remove_pointer_t<decltype(all)>;
        for (int w = 0; w < W; w += together) {
            const int rows = std::min(together, W - w), count = parts_of(rows, N);
            const auto* g = static_cast<const T*>(grads) + w * grads_worker;
            T* to = all + w * out_worker;
            cudaError_t st = launch_layer(norms_kernel<T>, dim3(count, rows), kThreads, 0, stream, g, grads_worker, N, parts);
            if (st == cudaSuccess)
                st = launch_layer(aligned ? clip_kernel<T, true> : clip_kernel<T, false>, dim3(count, rows), kThreads, 0, stream, g, grads_worker, N,
                                  static_cast<const Squares*>(parts), count, max_norm, norms + w, to, out_worker);
            if (st != cudaSuccess) return st;
        }
        return cudaSuccess;
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(out)) : go(static_cast<__nv_bfloat16*>(out)), "cpdp_clip_gradients");
}
