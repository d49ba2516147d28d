// The gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) v_t, its backward
// pass and its single step (include/cpdp_layers.h).
#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 128;

struct SeqIn {
    const void* p;
    int64_t seq, step;
};

// a = sigmoid(x) and 1 - a, both to a few ulps: neither is formed as a
// difference from 1.
__device__ __forceinline__ void gate_of(float x, float& a, float& rest) {
    const float t = expf(-fabsf(x)), r = 1.f / (1.f + t);
    a = x >= 0.f ? r : t * r;
    rest = x >= 0.f ? t * r : r;
}

template <typename T>
__device__ __forceinline__ float at(const SeqIn& x, int64_t b, int64_t t, int d) {
    return to_float(static_cast<const T*>(x.p)[b * x.seq + t * x.step + d]);
}

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t b, int64_t T_) {
    return lengths == nullptr ? T_ : min(max((int64_t)lengths[b], (int64_t)0), T_);
}

// One thread per channel, through all steps.
template <typename T>
__global__ void __launch_bounds__(kThreads)
recurrence_kernel(SeqIn gate, SeqIn value, int64_t T_, int D, const float* h0, const int32_t* lengths, T* h, float* h_last,
                  float* carry) {
    layer_begin();
    const int64_t b = blockIdx.y;
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= D) return;
    const int64_t n = length_of(lengths, b, T_), carries = (T_ + CPDP_CARRY_STEPS - 1) / CPDP_CARRY_STEPS;
    float state = h0 != nullptr ? h0[b * D + d] : 0.f;
    for (int64_t t = 0; t < T_; ++t) {
        if (t < n) {
            if (carry != nullptr && t % CPDP_CARRY_STEPS == 0) carry[(b * carries + t / CPDP_CARRY_STEPS) * D + d] = state;
            float a, rest;
            gate_of(at<T>(gate, b, t, d), a, rest);
            state = a * state + rest * at<T>(value, b, t, d);
        }
        h[(b * T_ + t) * D + d] = from_float<T>(t < n ? state : 0.f);
    }
    h_last[b * D + d] = state;
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
recurrence_backward_kernel(SeqIn dh, SeqIn gate, SeqIn value, int64_t T_, int D, const float* carry, const float* dh_last,
                           const int32_t* lengths, T* dgate, T* dvalue, int64_t grad_seq, int64_t grad_step, float* dh0) {
    layer_begin();
    __shared__ float states[CPDP_CARRY_STEPS][kThreads];
    const int64_t b = blockIdx.y;
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= D) return;
    const int64_t n = length_of(lengths, b, T_), carries = (T_ + CPDP_CARRY_STEPS - 1) / CPDP_CARRY_STEPS;
    float flow = dh_last != nullptr ? dh_last[b * D + d] : 0.f;  // a_(t+1) G_(t+1)
    for (int64_t t = n; t < T_; ++t) dgate[b * grad_seq + t * grad_step + d] = dvalue[b * grad_seq + t * grad_step + d] = from_float<T>(0.f);
    for (int64_t c = (n + CPDP_CARRY_STEPS - 1) / CPDP_CARRY_STEPS - 1; c >= 0; --c) {
        const int64_t first = c * CPDP_CARRY_STEPS, end = min(n, first + CPDP_CARRY_STEPS);
        float state = carry[(b * carries + c) * D + d], a, rest;
        for (int64_t t = first; t < end; ++t) {
            states[t - first][threadIdx.x] = state;
            gate_of(at<T>(gate, b, t, d), a, rest);
            state = a * state + rest * at<T>(value, b, t, d);
        }
        for (int64_t t = end - 1; t >= first; --t) {
            gate_of(at<T>(gate, b, t, d), a, rest);
            const float g = at<T>(dh, b, t, d) + flow;
            dvalue[b * grad_seq + t * grad_step + d] = from_float<T>(rest * g);
            dgate[b * grad_seq + t * grad_step + d] =
                from_float<T>(g * (states[t - first][threadIdx.x] - at<T>(value, b, t, d)) * a * rest);
            flow = a * g;
        }
    }
    if (dh0 != nullptr) dh0[b * D + d] = flow;
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
recurrence_step_kernel(const T* gate, int64_t gate_seq, const T* value, int64_t value_seq, int D, float* state, T* h) {
    layer_begin();
    const int64_t b = blockIdx.y;
    const int d = blockIdx.x * kThreads + threadIdx.x;
    if (d >= D) return;
    float a, rest;
    gate_of(to_float(gate[b * gate_seq + d]), a, rest);
    const float next = a * state[b * D + d] + rest * to_float(value[b * value_seq + d]);
    state[b * D + d] = next;
    h[b * D + d] = from_float<T>(next);
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

static cpdp_status check_recurrence(int B, int64_t T, int D, cpdp_dtype dtype) {
    if (B < 0 || B > 65535) return layer_error(CPDP_EINVAL, "B=%d must be in [0, 65535]", B);
    CPDP_TRY(check_sizes(1, T, D));
    if (B > 0) {
        if (T > kLayerMaxRows / B || (T > 0 && D > kLayerMaxElements / (B * T)))
            return layer_error(CPDP_EINVAL, "B=%d, T=%lld, D=%d: B * T is at most 2^31 - 1 and all elements at most 2^40", B, (long long)T, D);
    }
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    return CPDP_OK;
}

size_t cpdp_gated_recurrence_workspace(int B, int64_t T, int D) {
    (void)B, (void)T, (void)D;
    return 0;
}

cpdp_status cpdp_gated_recurrence(const void* gate, int64_t gate_seq, int64_t gate_step, const void* value,
                                  int64_t value_seq, int64_t value_step, cpdp_dtype dtype, int B, int64_t T, int D,
                                  const float* h0, const int32_t* lengths, void* h, float* h_last, float* carry,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_recurrence(B, T, D, dtype));
    const int64_t e = dtype_size(dtype);
    const bool some = B > 0 && T > 0;
    CPDP_TRY(check_array("gate", gate, some, e, gate_seq, gate_step));
    CPDP_TRY(check_array("value", value, some, e, value_seq, value_step));
    CPDP_TRY(check_array("h0", h0, false, 4));
    CPDP_TRY(check_array("lengths", lengths, false, 4));
    CPDP_TRY(check_array("h", h, some, e));
    CPDP_TRY(check_array("h_last", h_last, B > 0, 4));
    CPDP_TRY(check_array("carry", carry, false, 4));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_gated_recurrence_workspace(B, T, D)));
    if (B == 0) return CPDP_OK;
    const SeqIn g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const dim3 grid(ceil_div(D, kThreads), B);
    return layer_launched(dtype == CPDP_F32 ? launch_layer(recurrence_kernel<float>, grid, kThreads, 0, stream, g, v, T, D, h0, lengths,
                                                           static_cast<float*>(h), h_last, carry)
                                            : launch_layer(recurrence_kernel<__nv_bfloat16>, grid, kThreads, 0, stream, g, v, T, D, h0,
                                                           lengths, static_cast<__nv_bfloat16*>(h), h_last, carry),
                          "cpdp_gated_recurrence");
}

cpdp_status cpdp_gated_recurrence_backward(const void* dh, int64_t dh_seq, int64_t dh_step, const void* gate,
                                           int64_t gate_seq, int64_t gate_step, const void* value, int64_t value_seq,
                                           int64_t value_step, cpdp_dtype dtype, int B, int64_t T, int D,
                                           const float* carry, const float* dh_last, const int32_t* lengths, void* dgate,
                                           void* dvalue, int64_t grad_seq, int64_t grad_step, float* dh0, void* workspace,
                                           size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_recurrence(B, T, D, dtype));
    const int64_t e = dtype_size(dtype);
    const bool some = B > 0 && T > 0;
    CPDP_TRY(check_array("dh", dh, some, e, dh_seq, dh_step));
    CPDP_TRY(check_array("gate", gate, some, e, gate_seq, gate_step));
    CPDP_TRY(check_array("value", value, some, e, value_seq, value_step));
    CPDP_TRY(check_array("carry", carry, some, 4));
    CPDP_TRY(check_array("dh_last", dh_last, false, 4));
    CPDP_TRY(check_array("lengths", lengths, false, 4));
    CPDP_TRY(check_array("dgate", dgate, some, e, grad_seq, grad_step));
    CPDP_TRY(check_array("dvalue", dvalue, some, e));
    CPDP_TRY(check_array("dh0", dh0, false, 4));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_gated_recurrence_workspace(B, T, D)));
    if (B == 0) return CPDP_OK;
    const SeqIn o{dh, dh_seq, dh_step}, g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const dim3 grid(ceil_div(D, kThreads), B);
    const auto go = [&](auto* dg, auto* dv) {
        using E = std::remove_pointer_t<decltype(dg)>;
        return launch_layer(recurrence_backward_kernel<E>, grid, kThreads, 0, stream, o, g, v, T, D, carry, dh_last, lengths, dg, dv,
                            grad_seq, grad_step, dh0);
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(dgate), static_cast<float*>(dvalue))
                                            : go(static_cast<__nv_bfloat16*>(dgate), static_cast<__nv_bfloat16*>(dvalue)),
                          "cpdp_gated_recurrence_backward");
}

cpdp_status cpdp_gated_recurrence_step(const void* gate, int64_t gate_seq, const void* value, int64_t value_seq,
                                       cpdp_dtype dtype, int B, int D, float* state, void* h, void* stream) {
    CPDP_TRY(check_recurrence(B, 1, D, dtype));
    const int64_t e = dtype_size(dtype);
    CPDP_TRY(check_array("gate", gate, B > 0, e, gate_seq));
    CPDP_TRY(check_array("value", value, B > 0, e, value_seq));
    CPDP_TRY(check_array("state", state, B > 0, 4));
    CPDP_TRY(check_array("h", h, B > 0, e));
    if (B == 0) return CPDP_OK;
    const dim3 grid(ceil_div(D, kThreads), B);
    const auto go = [&](auto* out) {
        using E = std::remove_pointer_t<decltype(out)>;
        return launch_layer(recurrence_step_kernel<E>, grid, kThreads, 0, stream, static_cast<const E*>(gate), gate_seq,
                            static_cast<const E*>(value), value_seq, D, state, out);
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(h)) : go(static_cast<__nv_bfloat16*>(h)),
                          "cpdp_gated_recurrence_step");
}
