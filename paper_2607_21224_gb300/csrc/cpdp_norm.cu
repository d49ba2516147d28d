// Residual addition and root-mean-square norm for W workers, with an optional
// 8-bit output, and its backward pass (include/cpdp_layers.h).
#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v) {
    __shared__ float part[kThreads / 32];
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    __syncthreads();
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = v;
    __syncthreads();
    float s = 0.f;
    for (int i = 0; i < kThreads / 32; ++i) s += part[i];
    return s;
}

struct NormIn {
    const void* p;
    int64_t worker, row;
};

// One block per row.
template <typename T, bool CHECKPOINT>
__global__ void __launch_bounds__(kThreads)
norm_forward_kernel(NormIn x, NormIn residual, const float* weight, int64_t weight_worker, int64_t M, int D, float eps,
                    void* y, void* s, int8_t* codes, uint8_t* exponents) {
    layer_begin();
    const int64_t m = blockIdx.x, w = blockIdx.y, row = w * M + m;
    const T* xr = static_cast<const T*>(x.p) + w * x.worker + m * x.row;
    const T* rr = static_cast<const T*>(residual.p) + w * residual.worker + m * residual.row;
    const float* wt = weight + w * weight_worker;
    float sum = 0.f;
    for (int d = threadIdx.x; d < D; d += kThreads) {
        float v = to_float(xr[d]);
        if (residual.p != nullptr) {
            const T r = from_float<T>(v + to_float(rr[d]));
            static_cast<T*>(s)[row * D + d] = r;
            v = to_float(r);
        }
        sum += v * v;
    }
    const float k = rsqrtf(block_sum(sum) / D + eps);
    const int blocks = (D + kBlock8 - 1) / kBlock8;
    for (int d = threadIdx.x; d < blocks * kBlock8; d += kThreads) {
        float v = 0.f;
        if (d < D) {
            v = to_float(xr[d]);
            if (residual.p != nullptr) v = to_float(from_float<T>(v + to_float(rr[d])));
            v = v * k * wt[d];
        }
        if (CHECKPOINT) {
            const uint32_t top = __reduce_max_sync(~0u, __float_as_uint(v) & 0x7fffffffu);
            const uint32_t e = exponent_byte(top);
            const int q = code_of(v, inverse_unit_of(e));
            codes[row * blocks * kBlock8 + d] = static_cast<int8_t>(q);
            if (threadIdx.x % 32 == 0) exponents[row * blocks + d / kBlock8] = static_cast<uint8_t>(e);
            if (d < D) static_cast<__nv_bfloat16*>(y)[row * D + d] = from_float<__nv_bfloat16>(q * unit_of(e));
        } else if (d < D) {
            static_cast<T*>(y)[row * D + d] = from_float<T>(v);
        }
    }
}

// One block per row; the row's scale goes to `scale` for the weight's gradient.
template <typename T>
__global__ void __launch_bounds__(kThreads)
norm_backward_kernel(NormIn dy, NormIn s, NormIn ds, const float* weight, int64_t weight_worker, int64_t M, int D,
                     float eps, void* dx, float* scale) {
    layer_begin();
    const int64_t m = blockIdx.x, w = blockIdx.y, row = w * M + m;
    const T* g = static_cast<const T*>(dy.p) + w * dy.worker + m * dy.row;
    const T* sr = static_cast<const T*>(s.p) + w * s.worker + m * s.row;
    const T* dr = static_cast<const T*>(ds.p) + w * ds.worker + m * ds.row;
    const float* wt = weight + w * weight_worker;
    float squares = 0.f, dot = 0.f;
    for (int d = threadIdx.x; d < D; d += kThreads) {
        const float v = to_float(sr[d]);
        squares += v * v;
        dot += to_float(g[d]) * wt[d] * v;
    }
    squares = block_sum(squares);
    dot = block_sum(dot);
    const float k = rsqrtf(squares / D + eps);
    const float c = k * k * k * (dot / D);
    if (threadIdx.x == 0) scale[row] = k;
    for (int d = threadIdx.x; d < D; d += kThreads) {
        const float through = ds.p != nullptr ? to_float(dr[d]) : 0.f;
        static_cast<T*>(dx)[row * D + d] = from_float<T>(through + k * to_float(g[d]) * wt[d] - c * to_float(sr[d]));
    }
}

template <typename T, typename G>
__global__ void __launch_bounds__(kThreads)
norm_weight_kernel(NormIn dy, NormIn s, const float* scale, int64_t M, int D, G* dweight, int64_t dweight_worker) {
    layer_begin();
    const int d = blockIdx.x * kThreads + threadIdx.x;
    const int64_t w = blockIdx.y;
    if (d >= D) return;
    float sum = 0.f;
    for (int64_t m = 0; m < M; ++m)
        sum += to_float(static_cast<const T*>(dy.p)[w * dy.worker + m * dy.row + d]) *
               to_float(static_cast<const T*>(s.p)[w * s.worker + m * s.row + d]) * scale[w * M + m];
    dweight[w * dweight_worker + d] = from_float<G>(sum);
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

static cpdp_status check_norm(int W, int64_t M, int D, cpdp_dtype dtype, float eps) {
    CPDP_TRY(check_sizes(W, M, D));
    if (D > CPDP_NORM_MAX_FEATURES)
        return layer_error(CPDP_EINVAL, "a norm's rows have at most %d features, not %d", CPDP_NORM_MAX_FEATURES, D);
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    if (!(eps > 0.f) || eps > 3.0e38f) return layer_error(CPDP_EINVAL, "eps=%g must be positive and finite", (double)eps);
    return CPDP_OK;
}

cpdp_status cpdp_add_rmsnorm(const void* x, int64_t x_worker, int64_t x_row, const void* residual,
                             int64_t residual_worker, int64_t residual_row, const float* weight, int64_t weight_worker,
                             cpdp_dtype dtype, int W, int64_t M, int D, float eps, void* y, void* s, int8_t* codes,
                             uint8_t* exponents, void* stream) {
    CPDP_TRY(check_norm(W, M, D, dtype, eps));
    const int64_t e = dtype_size(dtype);
    const bool some = M > 0;
    CPDP_TRY(check_array("x", x, some, e, x_worker, x_row));
    CPDP_TRY(check_array("residual", residual, false, e, residual_worker, residual_row));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("y", y, some, codes != nullptr ? 2 : e));
    CPDP_TRY(check_array("s", s, some && residual != nullptr, e));
    if (some && residual == nullptr && s != nullptr) return layer_error(CPDP_EINVAL, "s is x where there is no residual: pass NULL");
    if ((codes == nullptr) != (exponents == nullptr))
        return layer_error(CPDP_EINVAL, "codes and exponents go together: one of them is NULL");
    CPDP_TRY(check_array("codes", codes, false, 16));
    if (!some) return CPDP_OK;
    const NormIn xi{x, x_worker, x_row}, ri{residual, residual_worker, residual_row};
    const dim3 grid(static_cast<unsigned>(M), W);
    const auto go = [&](auto kernel) {
        return launch_layer(kernel, grid, kThreads, 0, stream, xi, ri, weight, weight_worker, M, D, eps, y, s, codes, exponents);
    };
    const cudaError_t launched =
        dtype == CPDP_F32 ? (codes ? go(norm_forward_kernel<float, true>) : go(norm_forward_kernel<float, false>))
                          : (codes ? go(norm_forward_kernel<__nv_bfloat16, true>) : go(norm_forward_kernel<__nv_bfloat16, false>));
    return layer_launched(launched, "cpdp_add_rmsnorm");
}

size_t cpdp_add_rmsnorm_backward_workspace(int W, int64_t M, int D) {
    if (check_norm(W, M, D, CPDP_F32, 1.f) != CPDP_OK) return 0;
    return static_cast<size_t>(W) * M * 4;
}

cpdp_status cpdp_add_rmsnorm_backward(const void* dy, int64_t dy_worker, int64_t dy_row, const void* s, int64_t s_worker,
                                      int64_t s_row, const void* ds, int64_t ds_worker, int64_t ds_row,
                                      const float* weight, int64_t weight_worker, cpdp_dtype dtype, int W, int64_t M,
                                      int D, float eps, void* dx, void* dweight, int64_t dweight_worker,
                                      cpdp_dtype dweight_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_norm(W, M, D, dtype, eps));
    const int64_t e = dtype_size(dtype);
    const bool some = M > 0;
    CPDP_TRY(check_array("dy", dy, some, e, dy_worker, dy_row));
    CPDP_TRY(check_array("s", s, some, e, s_worker, s_row));
    CPDP_TRY(check_array("ds", ds, false, e, ds_worker, ds_row));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("dx", dx, some, e));
    if (!known_dtype(dweight_dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d of dweight", (int)dweight_dtype);
    CPDP_TRY(check_array("dweight", dweight, true, dtype_size(dweight_dtype), dweight_worker));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_add_rmsnorm_backward_workspace(W, M, D)));
    const NormIn gi{dy, dy_worker, dy_row}, si{s, s_worker, s_row}, di{ds, ds_worker, ds_row};
    float* scale = static_cast<float*>(workspace);
    if (some) {
        const auto go = [&](auto kernel) {
            return launch_layer(kernel, dim3(static_cast<unsigned>(M), W), kThreads, 0, stream, gi, si, di, weight, weight_worker, M, D, eps, dx, scale);
        };
        CPDP_TRY(layer_launched(dtype == CPDP_F32 ? go(norm_backward_kernel<float>) : go(norm_backward_kernel<__nv_bfloat16>),
                                "cpdp_add_rmsnorm_backward"));
    }
    const auto go = [&](auto kernel, auto* out) {
        return launch_layer(kernel, dim3(ceil_div(D, kThreads), W), kThreads, 0, stream, gi, si, scale, M, D, out, dweight_worker);
    };
    const auto typed = [&](auto* out) {
        using G = std::remove_pointer_t<decltype(out)>;
        return dtype == CPDP_F32 ? go(norm_weight_kernel<float, G>, out) : go(norm_weight_kernel<__nv_bfloat16, G>, out);
    };
    return layer_launched(dweight_dtype == CPDP_F32 ? typed(static_cast<float*>(dweight)) : typed(static_cast<__nv_bfloat16*>(dweight)),
                          "cpdp_add_rmsnorm_backward");
}
