// Sums of the parts that blocks leave of small gradients.
#pragma once

#include "cpdp_layers.cuh"

namespace cpdp {

// A worker's gradients: up to three arrays, one after another in a part.
struct SumsOut {
    void* out[3];
    int64_t worker[3], size[3];
};

#ifdef __CUDACC__
namespace {

// out = the sum of a worker's parts [W][parts][n], in an order fixed by their
// number: 32 neighbouring values per block, every eighth part to a warp.
template <typename G>
__global__ void __launch_bounds__(256)
sum_gradients_kernel(const float* parts, int count, int64_t n, unsigned blocks, SumsOut o) {
    layer_begin();
    __shared__ float shared[8][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t w = blockIdx.x / blocks;
    int64_t at = (int64_t)(blockIdx.x % blocks) * 32 + lane;
    float s = 0.f;
    if (at < n)
#pragma unroll 4
        for (int k = warp; k < count; k += 8) s += parts[(w * count + k) * n + at];
    shared[warp][lane] = s;
    __syncthreads();
    if (warp > 0 || at >= n) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) s += shared[k][lane];
#pragma unroll
    for (int a = 0; a < 3; ++a) {
        if (at >= 0 && at < o.size[a]) static_cast<G*>(o.out[a])[w * o.worker[a] + at] = from_float<G>(s);
        at -= o.size[a];
    }
}

cudaError_t sum_gradients(const float* parts, int count, int W, const SumsOut& o, cpdp_dtype dtype, void* stream) {
    const int64_t n = o.size[0] + o.size[1] + o.size[2];
    if (ceil_div(n, 32) > kLayerMaxRows / W) return cudaErrorInvalidConfiguration;
    const unsigned blocks = static_cast<unsigned>(ceil_div(n, 32));
    return dtype == CPDP_F32 ? launch_layer(sum_gradients_kernel<float>, blocks * W, 256, 0, stream, parts, count, n, blocks, o)
                             : launch_layer(sum_gradients_kernel<__nv_bfloat16>, blocks * W, 256, 0, stream, parts, count, n, blocks, o);
}

}  // namespace
#endif

}  // namespace cpdp
