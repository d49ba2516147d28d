// Activations held in 8 bits, and their values read back (include/cpdp_layers.h).
#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 256;

// One warp per block of 32 features.
template <typename T>
__global__ void __launch_bounds__(kThreads)
checkpoint_kernel(const T* x, int64_t x_worker, int64_t x_row, int64_t M, int D, int blocks, int64_t total, int8_t* codes,
                  uint8_t* exponents, __nv_bfloat16* values) {
    layer_begin();
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (at >= total) return;
    const int64_t row = at / blocks, w = row / M, m = row - w * M;
    const int d = static_cast<int>(at - row * blocks) * kBlock8 + threadIdx.x % 32;
    const float v = d < D ? to_float(x[w * x_worker + m * x_row + d]) : 0.f;
    const uint32_t e = exponent_byte(__reduce_max_sync(~0u, __float_as_uint(v) & 0x7fffffffu));
    const int q = code_of(v, inverse_unit_of(e));
    codes[at * kBlock8 + threadIdx.x % 32] = static_cast<int8_t>(q);
    if (threadIdx.x % 32 == 0) exponents[at] = static_cast<uint8_t>(e);
    if (values != nullptr && d < D) values[row * D + d] = from_float<__nv_bfloat16>(q * unit_of(e));
}

__global__ void __launch_bounds__(kThreads)
restore_kernel(const int8_t* codes, const uint8_t* exponents, int D, int blocks, int64_t total, __nv_bfloat16* values) {
    layer_begin();
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 32) + threadIdx.x / 32;
    if (at >= total) return;
    const int64_t row = at / blocks;
    const int d = static_cast<int>(at - row * blocks) * kBlock8 + threadIdx.x % 32;
    if (d < D) values[row * D + d] = from_float<__nv_bfloat16>(codes[at * kBlock8 + threadIdx.x % 32] * unit_of(exponents[at]));
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
    const int64_t total = W * M * blocks;
    const unsigned grid = static_cast<unsigned>(ceil_div(total, kThreads / 32));
    auto* out = static_cast<__nv_bfloat16*>(values);
    const cudaError_t launched =
        dtype == CPDP_F32 ? launch_layer(checkpoint_kernel<float>, grid, kThreads, 0, stream, static_cast<const float*>(x), x_worker,
                                         x_row, M, D, blocks, total, codes, exponents, out)
                          : launch_layer(checkpoint_kernel<__nv_bfloat16>, grid, kThreads, 0, stream,
                                         static_cast<const __nv_bfloat16*>(x), x_worker, x_row, M, D, blocks, total, codes,
                                         exponents, out);
    return layer_launched(launched, "cpdp_checkpoint");
}

cpdp_status cpdp_restore(const int8_t* codes, const uint8_t* exponents, int W, int64_t M, int D, void* values, void* stream) {
    CPDP_TRY(check_sizes(W, M, D));
    CPDP_TRY(check_array("codes", codes, M > 0, 16));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("values", values, M > 0, 2));
    if (M == 0) return CPDP_OK;
    const int blocks = static_cast<int>(ceil_div(D, kBlock8));
    const int64_t total = W * M * blocks;
    return layer_launched(launch_layer(restore_kernel, static_cast<unsigned>(ceil_div(total, kThreads / 32)), kThreads, 0, stream,
                                       codes, exponents, D, blocks, total, static_cast<__nv_bfloat16*>(values)),
                          "cpdp_restore");
}
