// Activations held in 8 bits, and their values read back (include/cpdp_layers.h).
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

// A thread takes pieces of V neighbours; the 32 / V threads of a block of 32
// features are neighbours in a warp, and agree on its exponent by shuffles.
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
        if constexpr (V == 1)
            top = __reduce_max_sync(~0u, top);
        else
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

template <int V>
__global__ void __launch_bounds__(kThreads)
restore_kernel(const int8_t* codes, const uint8_t* exponents, int D, int blocks, int64_t total, __nv_bfloat16* values) {
    layer_begin();
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
            const int8_t* p = codes + row * blocks * kBlock8 + piece * V;
            if constexpr (V == 8)
                in[u] = __ldcs(reinterpret_cast<const int2*>(p));
            else
                in[u].x = __ldcs(p) & 255;
            byte[u] = __ldg(exponents + row * blocks + piece * V / kBlock8);
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
    const auto go = [&](auto kernel, auto* in, int V) {
        const int64_t total = W * M * blocks * (kBlock8 / V), grid = ceil_div(total, kThreads * kPieces);
        if (grid > kLayerMaxRows) return cudaErrorInvalidConfiguration;
        return launch_layer(kernel, static_cast<unsigned>(grid), kThreads, 0, stream, in, x_worker, x_row, M, D, blocks, total, codes, exponents,
                            static_cast<__nv_bfloat16*>(values));
    };
    const auto* f = static_cast<const float*>(x);
    const auto* h = static_cast<const __nv_bfloat16*>(x);
    return layer_launched(dtype == CPDP_F32 ? (wide ? go(checkpoint_kernel<float, 4>, f, 4) : go(checkpoint_kernel<float, 1>, f, 1))
                                            : (wide ? go(checkpoint_kernel<__nv_bfloat16, 8>, h, 8) : go(checkpoint_kernel<__nv_bfloat16, 1>, h, 1)),
                          "cpdp_checkpoint");
}

cpdp_status cpdp_restore(const int8_t* codes, const uint8_t* exponents, int W, int64_t M, int D, void* values, void* stream) {
    CPDP_TRY(check_sizes(W, M, D));
    CPDP_TRY(check_array("codes", codes, M > 0, 16));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("values", values, M > 0, 2));
    if (M == 0) return CPDP_OK;
    const int blocks = static_cast<int>(ceil_div(D, kBlock8));
    const auto go = [&](auto kernel, int V) {
        const int64_t total = W * M * blocks * (kBlock8 / V), grid = ceil_div(total, kThreads * kPieces);
        if (grid > kLayerMaxRows) return cudaErrorInvalidConfiguration;
        return launch_layer(kernel, static_cast<unsigned>(grid), kThreads, 0, stream, codes, exponents, D, blocks, total,
                            static_cast<__nv_bfloat16*>(values));
    };
    return layer_launched(D % 8 == 0 && aligned_to(values, 16) ? go(restore_kernel<8>, 8) : go(restore_kernel<1>, 1), "cpdp_restore");
}
