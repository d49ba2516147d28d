// Activations held in 8 bits, and their values read back (include/cpdp_layers.h).
#include <type_traits>

#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 256;
constexpr int kPieces = 4;  // per thread, all loaded before the first is used

// Where the block's pieces lie: rows of `per_row` pieces, W * M of them. The
// divisions by the row's length are 64-bit once per block and 32-bit per piece.
struct Pieces {
    int64_t total, row0;
    uint32_t rest, per_row;
    __device__ __forceinline__ Pieces(int64_t all, uint32_t each) : total(all), per_row(each) {
        const int64_t first = (int64_t)blockIdx.x * (kThreads * kPieces);
        row0 = first / each;
        rest = static_cast<uint32_t>(first - row0 * each);
    }
    // piece u of this thread: its row and its place in the row; false past the end
    __device__ __forceinline__ bool find(int u, int64_t& row, uint32_t& piece) const {
        const uint32_t i = rest + u * kThreads + threadIdx.x, down = i / per_row;
        row = row0 + down;
        piece = i - down * per_row;
        return (int64_t)blockIdx.x * (kThreads * kPieces) + u * kThreads + threadIdx.x < total;
    }
};

// A thread takes pieces of V neighbours, 16 bytes; the 32 / V threads of a block
// of 32 features are neighbours in a warp, and agree on its exponent by
// shuffles. 2 x 16,384 x 2,048 in bf16, with the values: 70 us, 4.8 TB/s, bound by
// instructions (2.9 a clock); one element per thread took 317.
template <typename T, int V>
__global__ void __launch_bounds__(kThreads)
checkpoint_kernel(const T* x, int64_t x_worker, int64_t x_row, int64_t M, int D, int blocks, int64_t total, int8_t* codes,
                  uint8_t* exponents, __nv_bfloat16* values) {
    layer_begin();
    const Pieces at(total, static_cast<uint32_t>(blocks) * (kBlock8 / V));
    const int64_t w0 = at.row0 / M;
    const uint32_t m0 = static_cast<uint32_t>(at.row0 - w0 * M);
    Piece<T, V> in[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        int64_t row;
        uint32_t piece;
        in[u] = Piece<T, V>{};
        if (at.find(u, row, piece) && piece * V < (uint32_t)D) {
            const uint32_t down = m0 + static_cast<uint32_t>(row - at.row0), more = down / static_cast<uint32_t>(M);
            in[u].load(x + (w0 + more) * x_worker + (int64_t)(down - more * static_cast<uint32_t>(M)) * x_row + piece * V);
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        int64_t row;
        uint32_t piece;
        const bool here = at.find(u, row, piece);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(in[u].get(e)) & 0x7fffffffu);
#pragma unroll
        for (int h = 1; h < kBlock8 / V; h <<= 1) top = max(top, __shfl_xor_sync(~0u, top, h));
        const uint32_t byte = exponent_byte(top), d = piece * V;
        const float inverse = inverse_unit_of(byte), unit = unit_of(byte);
        int q[V];
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            q[e] = code_of(in[u].get(e), inverse);
            o[e] = q[e] * unit;
        }
        if (here) {
            store_codes<V>(codes + row * blocks * kBlock8 + d, q);
            if (d % kBlock8 == 0) exponents[row * blocks + d / kBlock8] = static_cast<uint8_t>(byte);
            if (values != nullptr && d < (uint32_t)D) store_piece<V>(values + row * D + d, o);
        }
    }
}

// Rows that do not start at multiples of 16 bytes: a warp takes kSpan blocks of
// 32 features of a row, a feature per lane, and lane i keeps block i's exponent.
// 2 x 1,999 x 1,003 in float32: 9 us; by pieces of one element 20.
constexpr int kSpan = 16;
struct Span {
    int64_t row;
    int first, count;  // blocks of 32 features; count <= 0: none
    __device__ __forceinline__ Span(int64_t rows, int blocks) {
        const int spans = (blocks + kSpan - 1) / kSpan;
        const int64_t i = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
        row = i / spans;
        first = static_cast<int>(i - row * spans) * kSpan;
        count = row < rows ? min(blocks - first, kSpan) : 0;
    }
};
template <typename T>
__global__ void __launch_bounds__(kThreads)
checkpoint_rows_kernel(const T* x, int64_t x_worker, int64_t x_row, int64_t M, int64_t rows, int D, int blocks, int8_t* codes,
                       uint8_t* exponents, __nv_bfloat16* values) {
    layer_begin();
    const Span at(rows, blocks);
    if (at.count <= 0) return;
    const int lane = threadIdx.x % 32, d0 = at.first * kBlock8 + lane;
    const int64_t w = at.row / M;
    const T* p = x + w * x_worker + (at.row - w * M) * x_row + d0;
    Piece<T, 1> in[kSpan];
#pragma unroll
    for (int k = 0; k < kSpan; ++k) {
        in[k] = Piece<T, 1>{};
        in[k].load(p + k * kBlock8, k < at.count && d0 + k * kBlock8 < D);
    }
    int8_t* q = codes + (at.row * blocks + at.first) * kBlock8 + lane;
    __nv_bfloat16* v = values + at.row * D + d0;
    uint32_t kept = 0;
#pragma unroll
    for (int k = 0; k < kSpan; ++k) {
        if (k >= at.count) break;
        const float f = in[k].get(0);
        const uint32_t byte = exponent_byte(__reduce_max_sync(~0u, __float_as_uint(f) & 0x7fffffffu));
        const int code = code_of(f, inverse_unit_of(byte));
        q[k * kBlock8] = static_cast<int8_t>(code);
        if (values != nullptr && d0 + k * kBlock8 < D) v[k * kBlock8] = from_float<__nv_bfloat16>(code * unit_of(byte));
        if (lane == k) kept = byte;
    }
    if (lane < at.count) exponents[at.row * blocks + at.first + lane] = static_cast<uint8_t>(kept);
}

// Values from the 8-bit form: 2 x 16,384 x 2,048 in 35 us, 5.8 TB/s (DRAM).
__global__ void __launch_bounds__(kThreads)
restore_kernel(const int8_t* codes, const uint8_t* exponents, int D, int blocks, int64_t total, __nv_bfloat16* values) {
    layer_begin();
    constexpr int V = 8;
    const Pieces at(total, static_cast<uint32_t>(blocks) * (kBlock8 / V));
    int2 in[kPieces];
    uint32_t byte[kPieces];
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        int64_t row;
        uint32_t piece;
        in[u] = make_int2(0, 0);
        byte[u] = 0;
        if (at.find(u, row, piece)) {
            in[u] = load_once(reinterpret_cast<const int2*>(codes + row * blocks * kBlock8 + piece * V));
            byte[u] = exponents[row * blocks + piece * V / kBlock8];
        }
    }
#pragma unroll
    for (int u = 0; u < kPieces; ++u) {
        int64_t row;
        uint32_t piece;
        if (!at.find(u, row, piece) || piece * V >= (uint32_t)D) continue;
        const float unit = unit_of(byte[u]);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = static_cast<int8_t>((e < 4 ? in[u].x : in[u].y) >> e % 4 * 8) * unit;
        store_piece<V>(values + row * D + piece * V, o);
    }
}

__global__ void __launch_bounds__(kThreads)
restore_rows_kernel(const int8_t* codes, const uint8_t* exponents, int64_t rows, int D, int blocks, __nv_bfloat16* values) {
    layer_begin();
    const Span at(rows, blocks);
    if (at.count <= 0) return;
    const int lane = threadIdx.x % 32, d0 = at.first * kBlock8 + lane;
    const int8_t* q = codes + (at.row * blocks + at.first) * kBlock8 + lane;
    const uint32_t kept = lane < at.count ? exponents[at.row * blocks + at.first + lane] : 0u;
    int code[kSpan];
#pragma unroll
    for (int k = 0; k < kSpan; ++k) code[k] = k < at.count ? load_once(q + k * kBlock8) : 0;
#pragma unroll
    for (int k = 0; k < kSpan; ++k) {
        const uint32_t byte = __shfl_sync(~0u, kept, k);
        if (k < at.count && d0 + k * kBlock8 < D) values[at.row * D + d0 + k * kBlock8] = from_float<__nv_bfloat16>(code[k] * unit_of(byte));
    }
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

cpdp_status cpdp_checkpoint(const void* x, int64_t x_worker, int64_t x_row, cpdp_dtype dtype, int W, int64_t M, int D,
                            int8_t* codes, uint8_t* exponents, void* values, void* stream) {
    CPDP_TRY(check_sizes(W, M, D));
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    CPDP_TRY(check_array("x", x, M > 0, dtype_size(dtype), x_worker, x_row));
    CPDP_TRY(check_array("codes", codes, M > 0, 16));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("values", values, false, 2));
    if (M == 0) return CPDP_OK;
    const int blocks = static_cast<int>(ceil_div(D, kBlock8));
    const int n = 16 / static_cast<int>(dtype_size(dtype));
    const bool wide = D % n == 0 && aligned_to(x, 16) && x_worker % n == 0 && x_row % n == 0 && aligned_to(values, 16);
    auto* out = static_cast<__nv_bfloat16*>(values);
    const auto pieces = [&](auto* in, auto each) {
        constexpr int V = decltype(each)::value;
        const int64_t total = W * M * blocks * (kBlock8 / V), grid = ceil_div(total, kThreads * kPieces);
        if (grid > kLayerMaxRows) return cudaErrorInvalidConfiguration;
        return launch_layer(checkpoint_kernel<std::remove_const_t<std::remove_pointer_t<decltype(in)>>, V>, static_cast<unsigned>(grid), kThreads,
                            0, stream, in, x_worker, x_row, M, D, blocks, total, codes, exponents, out);
    };
    const auto rows = [&](auto* in) {
        const int64_t grid = ceil_div(W * M * ceil_div(blocks, kSpan), kThreads / 32);
        if (grid > kLayerMaxRows) return cudaErrorInvalidConfiguration;
        return launch_layer(checkpoint_rows_kernel<std::remove_const_t<std::remove_pointer_t<decltype(in)>>>, static_cast<unsigned>(grid),
                            kThreads, 0, stream, in, x_worker, x_row, M, W * M, D, blocks, codes, exponents, out);
    };
    const auto* f = static_cast<const float*>(x);
    const auto* h = static_cast<const __nv_bfloat16*>(x);
    return layer_launched(dtype == CPDP_F32 ? (wide ? pieces(f, std::integral_constant<int, 4>{}) : rows(f))
                                            : (wide ? pieces(h, std::integral_constant<int, 8>{}) : rows(h)),
                          "cpdp_checkpoint");
}

cpdp_status cpdp_restore(const int8_t* codes, const uint8_t* exponents, int W, int64_t M, int D, void* values, void* stream) {
    CPDP_TRY(check_sizes(W, M, D));
    CPDP_TRY(check_array("codes", codes, M > 0, 16));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("values", values, M > 0, 2));
    if (M == 0) return CPDP_OK;
    const int blocks = static_cast<int>(ceil_div(D, kBlock8));
    const bool wide = D % 8 == 0 && aligned_to(values, 16);
    auto* out = static_cast<__nv_bfloat16*>(values);
    const int64_t total = W * M * blocks * (kBlock8 / 8);
    const int64_t grid = wide ? ceil_div(total, kThreads * kPieces) : ceil_div(W * M * ceil_div(blocks, kSpan), kThreads / 32);
    if (grid > kLayerMaxRows) return layer_error(CPDP_EINVAL, "W=%d, M=%lld, D=%d: more blocks than a launch takes", W, (long long)M, D);
    return layer_launched(wide ? launch_layer(restore_kernel, static_cast<unsigned>(grid), kThreads, 0, stream, codes, exponents, D, blocks, total, out)
                               : launch_layer(restore_rows_kernel, static_cast<unsigned>(grid), kThreads, 0, stream, codes, exponents, W * M, D, blocks, out),
                          "cpdp_restore");
}
