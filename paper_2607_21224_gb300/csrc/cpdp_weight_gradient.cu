// The weight gradient dW = dy^T x^ from activations held in 8 bits
// (include/cpdp_layers.h).
#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

// 64 x 64 of dW per block, 4 x 4 per thread.
template <typename T, typename G>
__global__ void __launch_bounds__(kThreads)
weight_gradient_kernel(const T* dy, int64_t dy_worker, int64_t dy_row, const int8_t* codes, const uint8_t* exponents,
                       int64_t M, int O, int I, G* dW, int64_t dW_worker) {
    layer_begin();
    __shared__ float a[kDepth][kTile], b[kDepth][kTile];
    const int64_t w = blockIdx.z;
    const int o0 = blockIdx.y * kTile, i0 = blockIdx.x * kTile, blocks = (I + kBlock8 - 1) / kBlock8;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float acc[4][4] = {};
    for (int64_t m0 = 0; m0 < M; m0 += kDepth) {
        for (int k = threadIdx.x; k < kDepth * kTile; k += kThreads) {
            const int64_t m = m0 + k / kTile;
            const int o = o0 + k % kTile, i = i0 + k % kTile;
            a[k / kTile][k % kTile] =
                m < M && o < O ? to_float(__float2bfloat16_rn(to_float(dy[w * dy_worker + m * dy_row + o]))) : 0.f;
            b[k / kTile][k % kTile] = m < M && i < I ? codes[(w * M + m) * blocks * kBlock8 + i] *
                                                           unit_of(exponents[(w * M + m) * blocks + i / kBlock8])
                                                     : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int r = 0; r < 4; ++r)
                for (int c = 0; c < 4; ++c) acc[r][c] += a[k][ty * 4 + r] * b[k][tx * 4 + c];
        __syncthreads();
    }
    for (int r = 0; r < 4; ++r)
        for (int c = 0; c < 4; ++c)
            if (o0 + ty * 4 + r < O && i0 + tx * 4 + c < I)
                dW[w * dW_worker + (int64_t)(o0 + ty * 4 + r) * I + i0 + tx * 4 + c] = from_float<G>(acc[r][c]);
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

size_t cpdp_weight_gradient_workspace(int W, int64_t M, int O, int I) {
    (void)W, (void)M, (void)O, (void)I;
    return 0;
}

cpdp_status cpdp_weight_gradient(const void* dy, int64_t dy_worker, int64_t dy_row, cpdp_dtype dy_dtype,
                                 const int8_t* codes, const uint8_t* exponents, int W, int64_t M, int O, int I, void* dW,
                                 int64_t dW_worker, cpdp_dtype dW_dtype, void* workspace, size_t workspace_bytes,
                                 void* stream) {
    CPDP_TRY(check_sizes(W, M, O));
    CPDP_TRY(check_sizes(W, M, I));
    CPDP_TRY(check_sizes(W, O, I));
    if (!known_dtype(dy_dtype) || !known_dtype(dW_dtype))
        return layer_error(CPDP_EINVAL, "unknown dtype: dy's is %d, dW's %d", (int)dy_dtype, (int)dW_dtype);
    CPDP_TRY(check_array("dy", dy, M > 0, dtype_size(dy_dtype), dy_worker, dy_row));
    CPDP_TRY(check_array("codes", codes, M > 0, 1));
    CPDP_TRY(check_array("exponents", exponents, M > 0, 1));
    CPDP_TRY(check_array("dW", dW, true, dtype_size(dW_dtype), dW_worker));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_weight_gradient_workspace(W, M, O, I)));
    const dim3 grid(ceil_div(I, kTile), ceil_div(O, kTile), W);
    const auto go = [&](auto* g, auto* out) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(g)>>;
        using G = std::remove_pointer_t<decltype(out)>;
        return launch_layer(weight_gradient_kernel<T, G>, grid, kThreads, 0, stream, g, dy_worker, dy_row, codes, exponents, M, O, I, out, dW_worker);
    };
    const auto typed = [&](auto* out) {
        return dy_dtype == CPDP_F32 ? go(static_cast<const float*>(dy), out) : go(static_cast<const __nv_bfloat16*>(dy), out);
    };
    return layer_launched(dW_dtype == CPDP_F32 ? typed(static_cast<float*>(dW)) : typed(static_cast<__nv_bfloat16*>(dW)),
                          "cpdp_weight_gradient");
}
