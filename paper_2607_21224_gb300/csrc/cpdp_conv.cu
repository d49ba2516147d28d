// The short causal convolution y_t = silu(bias + sum_k weight_k x_(t-K+1+k)),
// its backward pass and its single step (include/cpdp_layers.h).
#include <algorithm>
#include <type_traits>

#include "cpdp_gates.cuh"
#include "cpdp_sums.cuh"

namespace cpdp {
namespace {

// A sequence's inputs with the K - 1 before it: e_0 .. e_(T+K-2), e_(K-1) = x_0,
// and v_t = bias + sum_k weight_k e_(t+k). A thread walks a stretch of steps of V
// neighbouring channels (16 or 8 bytes; 1 where rows are not whole pieces), with
// the last K - 1 inputs in registers, two channels to a pair, and some rows on
// their way. Both passes are bound by memory: rows of 16 bytes per thread eight
// ahead, in the backward pass four of x and dy of 8 bytes, at as many threads as
// that leaves (eight ahead at three quarters of the threads: 3 us more of 36).
constexpr int kThreads = 128, kForwardAhead = 8, kBackwardAhead = 4;
constexpr int kForwardBlocks = 4, kBackwardBlocks = 4;  // per SM
constexpr int kMostTaps = CPDP_CONV_MAX_TAPS;

// V neighbouring elements as they lie in memory, loaded where they are there; else 0. Predicates, not branches: see load_once.
template <typename T, int V>
struct Few {
    static constexpr int kBytes = V * sizeof(T), kWords = (kBytes + 3) / 4, P = (V + 1) / 2;
    uint32_t w[kWords];
    __device__ __forceinline__ void load(const T* p, bool there) {
        const uint32_t on = there ? 1u : 0u;
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = 0u;
        if constexpr (kBytes == 16)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t@p ld.global.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                         : "+r"(w[0]), "+r"(w[1]), "+r"(w[2]), "+r"(w[3])
                         : "l"(p), "r"(on)
                         : "memory");
        else if constexpr (kBytes == 8)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %3, 0;\n\t@p ld.global.v2.u32 {%0, %1}, [%2];\n\t}"
                         : "+r"(w[0]), "+r"(w[1])
                         : "l"(p), "r"(on)
                         : "memory");
        else if constexpr (kBytes == 4)
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(w[0]) : "l"(p), "r"(on) : "memory");
        else
            asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u16 %0, [%1];\n\t}" : "+r"(w[0]) : "l"(p), "r"(on) : "memory");
    }
    __device__ __forceinline__ void get(Pair (&v)[P]) const {
        if constexpr (V == 1) {
            v[0] = pair(sizeof(T) == 4 ? __uint_as_float(w[0]) : __uint_as_float(w[0] << 16), 0.f);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                v[i] = sizeof(T) == 4 ? pair(__uint_as_float(w[2 * i % kWords]), __uint_as_float(w[(2 * i + 1) % kWords]))
                                      : pair(__uint_as_float(w[i % kWords] << 16), __uint_as_float(w[i % kWords] & 0xffff0000u));
        }
    }
};
template <typename T, int V>
__device__ __forceinline__ void store_few(T* p, const Pair (&v)[(V + 1) / 2]) {
    if constexpr (V == 1) {
        *p = from_float<T>(floats(v[0]).x);
    } else {
        float x[V];
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = i % 2 ? floats(v[i / 2]).y : floats(v[i / 2]).x;
        store_piece<V>(p, x);
    }
}

struct Conv {
    const void* x;
    int64_t x_seq, x_step;
    const float *weight, *bias;
    int64_t weight_worker, bias_worker;
    const void* state;         // [B][K - 1][D]; NULL: zeros
    const int32_t* lengths;
    int B, T, D, each;         // sequences of a worker
    int steps, stretches;      // steps of a stretch
};

// The weights of a thread's channels. They lie together in memory, at any alignment; the warp's lanes read them side by
// side and hand them over through shared memory (each reading its own took two thirds of a forward pass).
template <int V, int K>
struct TapsShared {
    static constexpr int kEach = V * (K + 1);
    float v[32][kEach | 1];
};
template <typename T, int V, int K>
struct Taps {
    static constexpr int P = (V + 1) / 2;
    Pair w[K][P], bias[P];
    // All lanes of the warp; `live`: the lane has channels.
    __device__ __forceinline__ Taps(const Conv& p, int worker, int d, bool live, TapsShared<V, K>& s) {
        const int lane = threadIdx.x % 32;
        const int64_t weights = worker * p.weight_worker + (int64_t)d * K, biases = worker * p.bias_worker + d;
        const unsigned there = __ballot_sync(~0u, live);
        const auto fetch = [&](const float* from, int64_t at, auto many, int to) {
            constexpr int COUNT = decltype(many)::value;
            float v[COUNT];
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int whose = (i * 32 + lane) / COUNT;
                const int64_t start = __shfl_sync(~0u, at, whose);
                v[i] = there >> whose & 1 ? from[start + (i * 32 + lane) % COUNT] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < COUNT; ++i) s.v[(i * 32 + lane) / COUNT][to + (i * 32 + lane) % COUNT] = v[i];
        };
        fetch(p.weight, weights, std::integral_constant<int, V * K>{}, 0);
        fetch(p.bias, biases, std::integral_constant<int, V>{}, V * K);
        __syncwarp();
        const float* own = s.v[lane];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            constexpr int next = V > 1;
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][i] = pair(own[2 * i * K + k], next ? own[(2 * i + next) * K + k] : 0.f);
            bias[i] = pair(own[V * K + 2 * i], next ? own[V * K + 2 * i + next] : 0.f);
        }
    }
    __device__ __forceinline__ Pair sum(const Pair (&e)[K][P], int i) const {
        Pair v = bias[i];
#pragma unroll
        for (int k = 0; k < K; ++k) v = fma2(w[k][i], e[k][i], v);
        return v;
    }
};

// The inputs of one sequence and the thread's channels; `n` steps are there.
template <typename T, int V, int K>
struct Inputs {
    const T *x, *state;
    int64_t step;
    int D, n;
    __device__ __forceinline__ Inputs(const Conv& p, int64_t b, int d)
        : x(static_cast<const T*>(p.x) + b * p.x_seq + d), state(p.state == nullptr ? nullptr : static_cast<const T*>(p.state) + b * (K - 1) * p.D + d),
          step(p.x_step), D(p.D), n(p.lengths == nullptr ? p.T : min(max(p.lengths[b], 0), p.T)) {}
    // e_k, 0 behind the last
    __device__ __forceinline__ void get(Pair (&v)[(V + 1) / 2], int e) const {
        Few<T, V> f;
        if (e < K - 1)
            f.load(state + (int64_t)e * D, state != nullptr);
        else
            f.load(x + (int64_t)(e - (K - 1)) * step, e - (K - 1) < n);
        f.get(v);
    }
    // x of step t
    __device__ __forceinline__ void row(Few<T, V>& f, int t) const { f.load(x + t * step, t < n); }
};

template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads, kForwardBlocks)
conv_kernel(Conv p, T* y, T* last) {
    layer_begin();
    constexpr int P = (V + 1) / 2;
    __shared__ TapsShared<V, K> shared[kThreads / 32];
    const int64_t columns = p.D / V, i = (int64_t)blockIdx.x * kThreads + threadIdx.x, row = i / columns;
    const bool live = row / p.stretches < p.B;
    const int64_t b = live ? row / p.stretches : 0;
    const int d = static_cast<int>(i - row * columns) * V, stretch = live ? static_cast<int>(row - b * p.stretches) : 0;
    const Inputs<T, V, K> in(p, b, d);
    const int first = stretch * p.steps, end = live ? min(first + p.steps, p.T) : 0, inside = min(end, in.n);
    Few<T, V> next[kForwardAhead];
#pragma unroll
    for (int r = 0; r < kForwardAhead; ++r) in.row(next[r], first + r < inside ? first + r : in.n);
    Pair e[K][P];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) in.get(e[k], first + k);
    const Taps<T, V, K> taps(p, static_cast<int>(b / p.each), d, live, shared[threadIdx.x / 32]);
    if (!live) return;
    T* to = y + (b * p.T + first) * p.D + d;
    for (int t = first; t < inside; t += kForwardAhead) {
#pragma unroll
        for (int r = 0; r < kForwardAhead; ++r) {
            Pair out[P];
            next[r].get(e[K - 1]);
            in.row(next[r], t + r + kForwardAhead < inside ? t + r + kForwardAhead : in.n);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                const Pair v = taps.sum(e, i);
                out[i] = mul2(v, sigmoid(v));
#pragma unroll
                for (int k = 0; k + 1 < K; ++k) e[k][i] = e[k + 1][i];
            }
            if (t + r < inside) store_few<T, V>(to, out);
            to += p.D;
        }
    }
    const Pair none[P] = {};
    to = y + (b * p.T + max(first, inside)) * p.D + d;
    for (int t = max(first, inside); t < end; ++t, to += p.D) store_few<T, V>(to, none);
    if (stretch == 0 && last != nullptr)
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            in.get(e[0], in.n + k);
            store_few<T, V>(last + (b * (K - 1) + k) * p.D + d, e[0]);
        }
}

struct ConvGradients {
    const void* dy;
    int64_t dy_seq, dy_step;
    const void* dlast;  // [B][K - 1][D]; NULL: 0
    void *dx, *dstate;  // dstate NULL: not wanted
    float* parts;       // [W][parts][D K + D]
    int part_count, lanes, groups;  // lanes side by side, and groups of them per row
};

// With dv_t = dy_t silu'(v_t): de_e = sum_k weight_k dv_(e-k), of which the first
// K - 1 are the state's; dweight_k = sum_t dv_t e_(t+k). A stretch makes the dv
// of the K - 1 steps before it again. Teams of `lanes` threads take the
// stretches of a worker's sequences in turn; the block adds its teams' sums of
// dweight and dbias up.
template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads, kBackwardBlocks)
conv_backward_kernel(Conv p, ConvGradients g) {
    layer_begin();
    __shared__ union {
        float sums[kThreads][V * (K + 1) + 1];
        TapsShared<V, K> taps[kThreads / 32];
    } shared_memory;
    auto& shared = shared_memory.sums;
    constexpr int P = (V + 1) / 2;
    const int lane = threadIdx.x % g.lanes, team = threadIdx.x / g.lanes, teams = kThreads / g.lanes;
    const int group = blockIdx.x % g.groups, rest = blockIdx.x / g.groups, part = rest % g.part_count, worker = rest / g.part_count;
    const int d = (group * g.lanes + lane) * V;
    const bool live = d < p.D;
    Pair dw[K][P] = {}, db[P] = {};
    const Taps<T, V, K> taps(p, worker, d, live, shared_memory.taps[threadIdx.x / 32]);
    __syncthreads();  // before the sums take the same memory
    if (live) {
        const int items = p.each * p.stretches;
        for (int item = part * teams + team; item < items; item += g.part_count * teams) {
            const int64_t b = (int64_t)worker * p.each + item / p.stretches;
            const Inputs<T, V, K> in(p, b, d);
            const T* dy = static_cast<const T*>(g.dy) + b * g.dy_seq + d;
            const int first = item % p.stretches * p.steps, end = min(first + p.steps, p.T + K - 1);
            const int from = max(first - (K - 1), 0), inside = min(end, in.n);
            Few<T, V> next[kBackwardAhead], next_dy[kBackwardAhead];
            const auto fetch = [&](int r, int t) {
                in.row(next[r], t < end ? t : in.n);
                next_dy[r].load(dy + t * g.dy_step, t < inside);
            };
#pragma unroll
            for (int r = 0; r < kBackwardAhead; ++r) fetch(r, from + r);
            Pair e[K][P] = {}, dv[K][P] = {};  // dv[k]: of step t - k
            if (in.n > 0)
#pragma unroll
                for (int k = 0; k < K - 1; ++k) in.get(e[k], from + k);
            // WHOLE: every step of the turn and every row that it fetches is the stretch's own and inside, so nothing is
            // compared (both passes of 128 x 197 x 768 in bfloat16: 57.7 us for 61.1, in float32 82 for 89; of 64 x 300 x 771
            // 80 for 100; the same in the forward pass: 0.3 us)
            const auto turn = [&](int t0, auto known) {
                constexpr bool WHOLE = decltype(known)::value;
#pragma unroll
                for (int r = 0; r < kBackwardAhead; ++r) {
                    const int t = t0 + r;
                    Pair out[P], dy_r[P];
                    next[r].get(e[K - 1]);
                    next_dy[r].get(dy_r);
                    if constexpr (WHOLE) {
                        next[r].load(in.x + (t + kBackwardAhead) * in.step, true);
                        next_dy[r].load(dy + (t + kBackwardAhead) * g.dy_step, true);
                    } else {
                        fetch(r, t + kBackwardAhead);
                    }
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const Pair v = taps.sum(e, i);
#pragma unroll
                        for (int k = K - 1; k > 0; --k) dv[k][i] = dv[k - 1][i];
                        dv[0][i] = mul2(dy_r[i], silu_slope(v, sigmoid(v)));
                        if (!WHOLE) dv[0][i] = where(t < inside, dv[0][i]);
                        const Pair own = WHOLE ? dv[0][i] : where(t >= first, dv[0][i]);
                        db[i] = add2(db[i], own);
                        out[i] = mul2(taps.w[0][i], dv[0][i]);
                        dw[0][i] = fma2(own, e[0][i], dw[0][i]);
#pragma unroll
                        for (int k = 1; k < K; ++k) {
                            dw[k][i] = fma2(own, e[k][i], dw[k][i]);
                            out[i] = fma2(taps.w[k][i], dv[k][i], out[i]);
                        }
#pragma unroll
                        for (int k = 0; k + 1 < K; ++k) e[k][i] = e[k + 1][i];
                    }
                    if (!WHOLE && g.dlast != nullptr && t >= in.n && t < in.n + K - 1) {
                        Few<T, V> f;
                        Pair more[P];
                        f.load(static_cast<const T*>(g.dlast) + (b * (K - 1) + t - in.n) * p.D + d, true);
                        f.get(more);
#pragma unroll
                        for (int i = 0; i < P; ++i) out[i] = add2(out[i], more[i]);
                    }
                    if (WHOLE || (t >= first && t < end)) {
                        if (WHOLE || t >= K - 1)
                            store_few<T, V>(static_cast<T*>(g.dx) + (b * p.T + t - (K - 1)) * p.D + d, out);
                        else if (g.dstate != nullptr)
                            store_few<T, V>(static_cast<T*>(g.dstate) + (b * (K - 1) + t) * p.D + d, out);
                    }
                }
            };
            for (int t0 = from; t0 < end; t0 += kBackwardAhead) {
                if (t0 >= max(first, K - 1) && t0 + 2 * kBackwardAhead <= inside)
                    turn(t0, std::true_type{});
                else
                    turn(t0, std::false_type{});
            }
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const auto half = [&](Pair v) { return i % 2 ? floats(v).y : floats(v).x; };
#pragma unroll
        for (int k = 0; k < K; ++k) shared[threadIdx.x][i * K + k] = half(dw[k][i / 2]);
        shared[threadIdx.x][V * K + i] = half(db[i / 2]);
    }
    __syncthreads();
    if (team > 0 || !live) return;
    float* to = g.parts + ((int64_t)worker * g.part_count + part) * p.D * (K + 1);
#pragma unroll 1
    for (int j = 0; j < V * (K + 1); ++j) {
        float s = shared[lane][j];
        for (int k = 1; k < teams; ++k) s += shared[k * g.lanes + lane][j];
        to[j < V * K ? (int64_t)d * K + j : (int64_t)p.D * K + d + j - V * K] = s;
    }
}

// One step, a channel per thread: the launch.
template <typename T, int K>
__global__ void __launch_bounds__(kThreads)
conv_step_kernel(Conv p, T* state, T* y) {
    layer_begin();
    __shared__ TapsShared<1, K> shared[kThreads / 32];
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = i / p.D;
    const bool live = b < p.B;
    const int d = static_cast<int>(i - b * p.D);
    const Taps<T, 1, K> taps(p, static_cast<int>(b / p.each), d, live, shared[threadIdx.x / 32]);
    if (!live) return;
    T* s = state + b * (K - 1) * p.D + d;
    T e[K];
#pragma unroll
    for (int k = 0; k < K - 1; ++k) e[k] = s[(int64_t)k * p.D];
    e[K - 1] = static_cast<const T*>(p.x)[b * p.x_seq + d];
    Pair held[K][1];
#pragma unroll
    for (int k = 0; k < K; ++k) held[k][0] = pair(to_float(e[k]), 0.f);
    const Pair v = taps.sum(held, 0);
#pragma unroll
    for (int k = 0; k < K - 1; ++k) s[(int64_t)k * p.D] = e[k + 1];
    y[i] = from_float<T>(floats(mul2(v, sigmoid(v))).x);
}

cpdp_status check_conv(int W, int B, int64_t T, int D, int K, cpdp_dtype dtype) {
    if (B < 0) return layer_error(CPDP_EINVAL, "B=%d must be >= 0", B);
    CPDP_TRY(check_sizes(1, T, D));
    if (W < 1 || W > 4096 || B % W != 0) return layer_error(CPDP_EINVAL, "W=%d must be in [1, 4096] and divide B=%d", W, B);
    if (K < 2 || K > kMostTaps) return layer_error(CPDP_EINVAL, "K=%d must be in [2, %d]", K, kMostTaps);
    if (T > int64_t(1) << 30) return layer_error(CPDP_EINVAL, "T=%lld is at most 2^30", (long long)T);
    if (B > 0 && (T + K > kLayerMaxRows / B || D > kLayerMaxElements / (B * (T + K))))
        return layer_error(CPDP_EINVAL, "B=%d, T=%lld, D=%d: B * (T + K) is at most 2^31 - 1 and all elements at most 2^40", B, (long long)T, D);
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    return CPDP_OK;
}

// Steps of a stretch of the forward pass: as many stretches as run at once.
int stretch_of(int64_t T, int64_t rows) {
    const int64_t count = std::max<int64_t>((int64_t)kSMs * kForwardBlocks * kThreads / std::max<int64_t>(rows, 1), 1);
    return static_cast<int>(std::min<int64_t>(std::max<int64_t>(ceil_div(ceil_div(T, count), kForwardAhead), 1) * kForwardAhead, 128));
}

// Whether rows of an array are whole pieces of `bytes`.
bool in_pieces(const void* p, int64_t size, int64_t a, int64_t b, int64_t bytes) {
    return aligned_to(p, bytes) && a * size % bytes == 0 && b * size % bytes == 0;
}

struct Spread {
    int steps, stretches, lanes, groups, parts;
};
// Of the backward pass: as many blocks as run at once, and stretches that make the teams' turns come out even; a stretch
// costs some steps of its own.
Spread spread_of(int W, int B, int64_t T, int D, int K, int V) {
    Spread s{};
    const int64_t columns = ceil_div(D, V), rows = T + K - 1, each = B / W;
    s.lanes = 1;
    while (s.lanes < 32 && s.lanes < columns) s.lanes *= 2;
    s.groups = static_cast<int>(ceil_div(columns, s.lanes));
    const int64_t most = std::max<int64_t>(kSMs * kBackwardBlocks / ((int64_t)s.groups * W), 1), teams = most * (kThreads / s.lanes);
    int64_t least = -1;
    for (int64_t walked = 2 * kBackwardAhead; walked <= 32 * kBackwardAhead; walked += kBackwardAhead) {  // with the K - 1 steps before a stretch
        const int64_t steps = walked - (K - 1), stretches = ceil_div(rows, steps), cost = ceil_div(each * stretches, teams) * (walked + kBackwardAhead);
        if (least < 0 || cost < least) least = cost, s.steps = static_cast<int>(steps), s.stretches = static_cast<int>(stretches);
    }
    s.parts = static_cast<int>(std::max<int64_t>(std::min(ceil_div(each * s.stretches, kThreads / s.lanes), most), 1));
    return s;
}

template <typename F>
cudaError_t with_taps(int K, F&& f) {
    return K == 2 ? f(std::integral_constant<int, 2>{}) : K == 3 ? f(std::integral_constant<int, 3>{}) : f(std::integral_constant<int, 4>{});
}

Conv conv_of(const void* x, int64_t x_seq, int64_t x_step, const float* weight, int64_t weight_worker, const float* bias, int64_t bias_worker,
             const void* state, const int32_t* lengths, int W, int B, int64_t T, int D) {
    Conv p{};
    p.x = x, p.x_seq = x_seq, p.x_step = x_step;
    p.weight = weight, p.weight_worker = weight_worker, p.bias = bias, p.bias_worker = bias_worker;
    p.state = state, p.lengths = lengths;
    p.B = B, p.T = static_cast<int>(T), p.D = D, p.each = B / W;
    return p;
}

template <typename T>
constexpr int kWide = 16 / sizeof(T);  // channels of a thread of the forward pass
constexpr int kWideBackward = 4;

}  // namespace
}  // namespace cpdp

using namespace cpdp;

cpdp_status cpdp_causal_conv(const void* x, int64_t x_seq, int64_t x_step, const float* weight, int64_t weight_worker, const float* bias,
                             int64_t bias_worker, const void* state, const int32_t* lengths, cpdp_dtype dtype, int W, int B, int64_t T, int D,
                             int K, void* y, void* last, void* stream) {
    CPDP_TRY(check_conv(W, B, T, D, K, dtype));
    const int64_t e = dtype_size(dtype);
    CPDP_TRY(check_array("x", x, B > 0 && T > 0, e, x_seq, x_step));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("bias", bias, true, 4, bias_worker));
    CPDP_TRY(check_array("state", state, false, e));
    CPDP_TRY(check_array("lengths", lengths, false, 4));
    CPDP_TRY(check_array("y", y, B > 0 && T > 0, e));
    CPDP_TRY(check_array("last", last, false, e));
    if (B == 0) return CPDP_OK;
    Conv p = conv_of(x, x_seq, x_step, weight, weight_worker, bias, bias_worker, state, lengths, W, B, T, D);
    const bool wide = D * e % 16 == 0 && in_pieces(x, e, x_seq, x_step, 16) && aligned_to(y, 16) && aligned_to(state, 16) && aligned_to(last, 16);
    const auto go = [&](auto* out, auto many) {
        using E = std::remove_pointer_t<decltype(out)>;
        constexpr int V = decltype(many)::value;
        const int64_t columns = D / V;
        p.steps = stretch_of(T, (int64_t)B * columns);
        p.stretches = static_cast<int>(std::max<int64_t>(ceil_div(T, p.steps), 1));
        const int64_t blocks = ceil_div((int64_t)B * p.stretches * columns, kThreads);
        if (blocks > kLayerMaxRows) return cudaErrorInvalidConfiguration;
        return with_taps(K, [&](auto taps) {
            return launch_layer(conv_kernel<E, V, decltype(taps)::value>, static_cast<unsigned>(blocks), kThreads, 0, stream, p, out, static_cast<E*>(last));
        });
    };
    const auto typed = [&](auto* out) {
        return wide ? go(out, std::integral_constant<int, kWide<std::remove_pointer_t<decltype(out)>>>{}) : go(out, std::integral_constant<int, 1>{});
    };
    return layer_launched(dtype == CPDP_F32 ? typed(static_cast<float*>(y)) : typed(static_cast<__nv_bfloat16*>(y)), "cpdp_causal_conv");
}

size_t cpdp_causal_conv_backward_workspace(int W, int B, int64_t T, int D, int K) {
    if (check_conv(W, B, T, D, K, CPDP_F32) != CPDP_OK || B == 0) return 0;
    const int parts = std::max(spread_of(W, B, T, D, K, 1).parts, spread_of(W, B, T, D, K, kWideBackward).parts);
    return ceil_div((int64_t)W * parts * D * (K + 1) * 4, 16) * 16;
}

cpdp_status cpdp_causal_conv_backward(const void* dy, int64_t dy_seq, int64_t dy_step, const void* x, int64_t x_seq, int64_t x_step,
                                      const float* weight, int64_t weight_worker, const float* bias, int64_t bias_worker, const void* state,
                                      const void* dlast, const int32_t* lengths, cpdp_dtype dtype, int W, int B, int64_t T, int D, int K, void* dx,
                                      void* dstate, void* dweight, int64_t dweight_worker, void* dbias, int64_t dbias_worker,
                                      cpdp_dtype dweight_dtype, void* workspace, size_t workspace_bytes, void* stream) {
    CPDP_TRY(check_conv(W, B, T, D, K, dtype));
    if (!known_dtype(dweight_dtype)) return layer_error(CPDP_EINVAL, "unknown dtype of dweight and dbias: %d", (int)dweight_dtype);
    const int64_t e = dtype_size(dtype);
    const bool some = B > 0 && T > 0;
    CPDP_TRY(check_array("dy", dy, some, e, dy_seq, dy_step));
    CPDP_TRY(check_array("x", x, some, e, x_seq, x_step));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("bias", bias, true, 4, bias_worker));
    CPDP_TRY(check_array("state", state, false, e));
    CPDP_TRY(check_array("dlast", dlast, false, e));
    CPDP_TRY(check_array("lengths", lengths, false, 4));
    CPDP_TRY(check_array("dx", dx, some, e));
    CPDP_TRY(check_array("dstate", dstate, false, e));
    CPDP_TRY(check_array("dweight", dweight, true, dtype_size(dweight_dtype), dweight_worker));
    CPDP_TRY(check_array("dbias", dbias, true, dtype_size(dweight_dtype), dbias_worker));
    CPDP_TRY(check_apart("dweight", W, dweight_worker, (int64_t)D * K));
    CPDP_TRY(check_apart("dbias", W, dbias_worker, D));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_causal_conv_backward_workspace(W, B, T, D, K)));
    const SumsOut sums{{dweight, dbias, nullptr}, {dweight_worker, dbias_worker, 0}, {(int64_t)D * K, D, 0}};
    if (B == 0) return layer_launched(sum_gradients(nullptr, 0, W, sums, dweight_dtype, stream), "cpdp_causal_conv_backward");
    Conv p = conv_of(x, x_seq, x_step, weight, weight_worker, bias, bias_worker, state, lengths, W, B, T, D);
    ConvGradients g{};
    g.dy = dy, g.dy_seq = dy_seq, g.dy_step = dy_step, g.dlast = dlast, g.dx = dx, g.dstate = dstate;
    g.parts = static_cast<float*>(workspace);
    const int64_t piece = kWideBackward * e;
    const bool wide = D % kWideBackward == 0 && in_pieces(x, e, x_seq, x_step, piece) && in_pieces(dy, e, dy_seq, dy_step, piece) &&
                      aligned_to(state, piece) && aligned_to(dlast, piece) && aligned_to(dx, piece) && aligned_to(dstate, piece);
    const Spread s = spread_of(W, B, T, D, K, wide ? kWideBackward : 1);
    if ((int64_t)s.groups * s.parts * W > kLayerMaxRows) return layer_error(CPDP_EINVAL, "W=%d, D=%d: more blocks than a launch takes", W, D);
    p.steps = s.steps, p.stretches = s.stretches;
    g.lanes = s.lanes, g.groups = s.groups, g.part_count = s.parts;
    const auto go = [&](auto* in, auto many) {
        using E = std::remove_const_t<std::remove_pointer_t<decltype(in)>>;
        return with_taps(K, [&](auto taps) {
            return launch_layer(conv_backward_kernel<E, decltype(many)::value, decltype(taps)::value>, static_cast<unsigned>((int64_t)s.groups * s.parts * W),
                                kThreads, 0, stream, p, g);
        });
    };
    const auto typed = [&](auto* in) { return wide ? go(in, std::integral_constant<int, kWideBackward>{}) : go(in, std::integral_constant<int, 1>{}); };
    CPDP_TRY(layer_launched(dtype == CPDP_F32 ? typed(static_cast<const float*>(x)) : typed(static_cast<const __nv_bfloat16*>(x)),
                            "cpdp_causal_conv_backward"));
    return layer_launched(sum_gradients(g.parts, s.parts, W, sums, dweight_dtype, stream), "cpdp_causal_conv_backward");
}

cpdp_status cpdp_causal_conv_step(const void* x, int64_t x_seq, const float* weight, int64_t weight_worker, const float* bias, int64_t bias_worker,
                                  cpdp_dtype dtype, int W, int B, int D, int K, void* state, void* y, void* stream) {
    CPDP_TRY(check_conv(W, B, 1, D, K, dtype));
    const int64_t e = dtype_size(dtype);
    CPDP_TRY(check_array("x", x, B > 0, e, x_seq));
    CPDP_TRY(check_array("weight", weight, true, 4, weight_worker));
    CPDP_TRY(check_array("bias", bias, true, 4, bias_worker));
    CPDP_TRY(check_array("state", state, B > 0, e));
    CPDP_TRY(check_array("y", y, B > 0, e));
    if (B == 0) return CPDP_OK;
    const Conv p = conv_of(x, x_seq, 0, weight, weight_worker, bias, bias_worker, nullptr, nullptr, W, B, 1, D);
    const int64_t blocks = ceil_div((int64_t)B * D, kThreads);
    if (blocks > kLayerMaxRows) return layer_error(CPDP_EINVAL, "B=%d, D=%d: more blocks than a launch takes", B, D);
    const auto go = [&](auto* out) {
        using E = std::remove_pointer_t<decltype(out)>;
        return with_taps(K, [&](auto taps) {
            return launch_layer(conv_step_kernel<E, decltype(taps)::value>, static_cast<unsigned>(blocks), kThreads, 0, stream, p, static_cast<E*>(state), out);
        });
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(y)) : go(static_cast<__nv_bfloat16*>(y)), "cpdp_causal_conv_step");
}
