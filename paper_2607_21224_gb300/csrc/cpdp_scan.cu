// The selective state space scan h_t = exp(-dt exp(a_log)) h_(t-1) + dt u_t b_t,
// y_t = (sum_n c_t h_t + skip u_t) silu(z_t), dt = softplus(delta + bias), its
// backward pass and its single step (include/cpdp_layers.h).
#include <algorithm>
#include <type_traits>

#include "cpdp_gates.cuh"
#include "cpdp_sums.cuh"

namespace cpdp {
namespace {

// A warp takes kColumn neighbouring channels of a sequence (a column) with all
// of their states, which are registers: S neighbouring lanes share the states of
// C channels, each 4 of every channel's. So a sum over states passes through S
// lanes, one over channels (the gradients of b and c) through 32 / S, after C
// channels were added up in registers; S = C = 4 at 16 states takes the fewest
// steps between lanes. Channels lie in pairs of registers, states apart.
//
// Chunks of R steps: their inputs are taken by lanes side by side along the
// channels, two neighbours each, which make dt and dt u; these go through shared
// memory to the walk and the walk's sums back.
template <int S_, int C_>
struct Shape {
    static constexpr int S = S_, C = C_, P = C / 2, kColumn = 32 / S * C, kStates = 4 * S;
};
constexpr int R = CPDP_CARRY_STEPS;
constexpr int kBackwardWarps = 4;  // of a block of the backward pass, at most
constexpr int kAtOnce = 4;  // steps of the forward walk
constexpr int kForwardBlocks = 12, kBackwardBlocks = 3;  // per SM
constexpr float kLn2f = kLn2;

struct Rows {
    const void* p;
    int64_t seq, step;
};

struct Scan {
    Rows u, delta, z, b, c;  // z.p NULL: no gate
    const float *a_log, *skip, *bias;
    int64_t a_worker, skip_worker, bias_worker;
    const int32_t* lengths;
    int B, T, D, N, each;    // sequences of a worker
    int groups;              // columns of a sequence
    // Steps in `count` segments of `steps` (a multiple of R) where there are few columns: a first pass makes each
    // segment's map of the state, exp(A sum(dt)) h + what the segment adds, a second one composes those before its own.
    int count, steps;
    Pair* maps;              // [column][segment][P * 5][32 lanes]
};

// Where `there`, else 0; ALL: there. Predicates, not branches: see load_once.
template <bool ALL>
__device__ __forceinline__ float load_if(const void* p, bool there) {
    float v = 0.f;
    if constexpr (ALL)
        asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.f32 %0, [%1];\n\t}" : "+f"(v) : "l"(p), "r"(there ? 1u : 0u) : "memory");
    return v;
}
template <bool ALL>
__device__ __forceinline__ uint32_t load_word_if(const void* p, bool there) {
    uint32_t v = 0;
    if constexpr (ALL)
        asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u32 %0, [%1];\n\t}" : "+r"(v) : "l"(p), "r"(there ? 1u : 0u) : "memory");
    return v;
}
template <bool ALL>
__device__ __forceinline__ uint32_t load_half_if(const void* p, bool there) {
    uint32_t v = 0;
    if constexpr (ALL)
        asm volatile("ld.global.u16 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.u16 %0, [%1];\n\t}" : "+r"(v) : "l"(p), "r"(there ? 1u : 0u) : "memory");
    return v;
}
template <bool ALL>
__device__ __forceinline__ Pair load_pair_if(const void* p, bool there) {
    Pair v = 0;
    if constexpr (ALL)
        asm volatile("ld.global.b64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.b64 %0, [%1];\n\t}" : "+l"(v) : "l"(p), "r"(there ? 1u : 0u) : "memory");
    return v;
}

// Two neighbouring elements as they lie in memory. WIDE: at a multiple of their size; the second is there where the first
// is. ALL: both are.
template <typename T, bool WIDE>
struct Two;
template <>
struct Two<float, true> {
    Pair v;
    template <bool ALL>
    __device__ __forceinline__ void load(const float* p, bool first, bool) {
        v = load_pair_if<ALL>(p, first);
    }
    __device__ __forceinline__ Pair get() const { return v; }
};
template <>
struct Two<float, false> {
    float x, y;
    template <bool ALL>
    __device__ __forceinline__ void load(const float* p, bool first, bool second) {
        x = load_if<ALL>(p, first), y = load_if<ALL>(p + 1, second);
    }
    __device__ __forceinline__ Pair get() const { return pair(x, y); }
};
template <>
struct Two<__nv_bfloat16, true> {
    uint32_t v;
    template <bool ALL>
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool first, bool) {
        v = load_word_if<ALL>(p, first);
    }
    __device__ __forceinline__ Pair get() const { return pair(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
};
template <>
struct Two<__nv_bfloat16, false> {
    uint32_t x, y;
    template <bool ALL>
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool first, bool second) {
        x = load_half_if<ALL>(p, first), y = load_half_if<ALL>(p + 1, second);
    }
    __device__ __forceinline__ Pair get() const { return pair(__uint_as_float(x << 16), __uint_as_float(y << 16)); }
};
template <bool WIDE>
__device__ __forceinline__ void store_two(float* p, Pair both, bool second) {
    const float2 v = floats(both);
    if (WIDE) {
        *reinterpret_cast<Pair*>(p) = both;
    } else {
        p[0] = v.x;
        if (second) p[1] = v.y;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store_two(__nv_bfloat16* p, Pair both, bool second) {
    const float2 v = floats(both);
    if (WIDE) {
        *reinterpret_cast<__nv_bfloat162*>(p) = __float22bfloat162_rn(v);
    } else {
        p[0] = __float2bfloat16_rn(v.x);
        if (second) p[1] = __float2bfloat16_rn(v.y);
    }
}

// softplus(x) = max(x, 0) + log(1 + t) with t = e^-|x|, and sigmoid(x). With s = t / (2 + t), at most 1/3,
// log(1 + t) = 2 artanh(s) = 2 s (1 + s^2 / 3 + s^4 / 5 + ...), of which seven terms leave out 1.4e-8.
template <typename T>
__device__ __forceinline__ Pair softplus(Pair x) {
    const float2 v = floats(x);
    const Pair t = exp_of_minus<T>(v);
    const float2 d = floats(add2(t, twice(2.f)));
    const Pair s = mul2(t, pair(reciprocal(d.x), reciprocal(d.y))), q = mul2(s, s);
    Pair sum = fma2(q, twice(1.f / 13.f), twice(1.f / 11.f));
    sum = fma2(q, sum, twice(1.f / 9.f));
    sum = fma2(q, sum, twice(1.f / 7.f));
    sum = fma2(q, sum, twice(1.f / 5.f));
    sum = fma2(q, sum, twice(1.f / 3.f));
    sum = fma2(q, sum, kOnes);
    return fma2(add2(s, s), sum, pair(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}

// The decays 2^(dt A) of two channels, A = -exp(a_log) log2(e). The instruction's
// powers came out 1.9e-8 of themselves too small on average for exponents from
// -0.5 to -0.001 (a million exponents against 64 bits; 3.5e-8 root mean square),
// which slow decays add up over their steps: 2.5e-6 of the states after 197 steps.
// The exponent makes up for it, with an addition that the product has for nothing.
constexpr float kPowerBias = 2.7e-8f;  // 1.9e-8 / ln 2
__device__ __forceinline__ Pair decay_of(Pair dt, Pair A) {
    const float2 x = floats(fma2(dt, A, twice(kPowerBias)));
    return pair(power_of_minus(-x.x), power_of_minus(-x.y));
}
// A of a state's a_log, without the sign. Above 88.7 exp leaves float32; the largest number stands in there, which leaves
// no state where dt is not 0, and 1 of it, not NaN, where dt is 0 (below 2^-126, or behind the last step).
__device__ __forceinline__ float rate_of(float a_log) {
    const float r = kLog2eHigh * expf(a_log);
    return isinf(r) ? 3.40282347e38f : r;
}
// sum + x, with what the addition rounds off kept for the next one (Kahan's compensated sum). A segment's sum of dt, by
// whose decay a state crosses the segment, has a term for every chunk; equal terms round the same way each time (one
// float32 sum of 9,400 steps was off by 2.3e-5, of 75,000 by 7e-4).
__device__ __forceinline__ void add_up(Pair& sum, Pair& lost, Pair x) {
    const Pair y = add2(x, lost), next = add2(sum, y);
    lost = fma2(fma2(sum, kMinusOnes, next), kMinusOnes, y);
    sum = next;
}
__device__ __forceinline__ Pair shuffle(Pair v, int mask) { return __shfl_xor_sync(~0u, v, mask); }

// The lane's place in the walk: states 4 q .. 4 q + 3 of C channels, pairs and states in an order of the lane's own, so
// that what a sum between lanes keeps and what it sends lie in the same registers of every lane.
template <typename X>
struct Lane {
    int lane, q, g, turn, channel;  // channel: of the column, the lane's first
    __device__ __forceinline__ Lane()
        : lane(threadIdx.x % 32), q(lane % X::S), g(lane / X::S), turn((g & 1) << 1), channel(g * X::C) {}
    __device__ __forceinline__ int pair_at(int p) const { return X::P == 2 ? channel + 2 * (p ^ (q & 1)) : channel; }
    __device__ __forceinline__ bool sums_up() const { return q < 2 * X::P; }  // the others of the group have the same sums
    __device__ __forceinline__ int summed_state() const { return 4 * q + turn + (g >> 1 & 1); }
    // Of sums of pairs over states, the channel's whose sum the lane gets.
    __device__ __forceinline__ int summed_channel() const {
        return X::P == 2 ? channel + 2 * (q & 1) + (q >> 1 & 1) : channel + (q & 1);
    }
};
// Sums over the S lanes of a group.
template <typename X>
__device__ __forceinline__ float over_states(const Lane<X>& l, const Pair (&v)[X::P]) {
    if constexpr (X::P == 2) {
        const float2 r = floats(add2(v[0], shuffle(v[1], 1)));
        const bool high = l.q & 2;
        float s = (high ? r.y : r.x) + __shfl_xor_sync(~0u, high ? r.x : r.y, 2);
        if constexpr (X::S == 8) s += __shfl_xor_sync(~0u, s, 4);
        return s;
    } else {
        const float2 r = floats(v[0]);
        const bool high = l.q & 1;
        float s = (high ? r.y : r.x) + __shfl_xor_sync(~0u, high ? r.x : r.y, 1);
#pragma unroll
        for (int k = 2; k < X::S; k *= 2) s += __shfl_xor_sync(~0u, s, k);
        return s;
    }
}
// Sums over the groups of lanes: of x and y for the lane's 4 states (in its order). The lane gets that of state
// summed_state(); of x, of y where `second`, or of both (S = 8).
template <typename X>
__device__ __forceinline__ float2 over_channels(const Lane<X>& l, const float (&x)[4], const float (&y)[4]) {
    const auto add = [](float keep, float send, int mask) { return keep + __shfl_xor_sync(~0u, send, mask); };
    const float x0 = add(x[0], x[2], X::S), x1 = add(x[1], x[3], X::S), y0 = add(y[0], y[2], X::S), y1 = add(y[1], y[3], X::S);
    const bool odd = l.g & 2;
    const float xs = add(odd ? x1 : x0, odd ? x0 : x1, 2 * X::S), ys = add(odd ? y1 : y0, odd ? y0 : y1, 2 * X::S);
    if constexpr (X::S == 8) {
        return make_float2(xs, ys);
    } else {
        const bool second = l.g & 4;
        float s = add(second ? ys : xs, second ? xs : ys, 4 * X::S);
        if constexpr (X::S == 2) s += __shfl_xor_sync(~0u, s, 16);
        return make_float2(s, s);
    }
}

// 4 neighbouring values of two channels' rows [channel][N] of float32, in the lane's order, from and to memory.
template <typename X>
struct States {
    int first, N, turn;
    bool quads;  // N a multiple of 4 and rows at multiples of 16 bytes
    __device__ __forceinline__ States(const Lane<X>& l, int n, bool aligned, bool turned)
        : first(4 * l.q), N(n), turn(turned ? l.turn : 0), quads(aligned) {}
    __device__ __forceinline__ void row(const float* p, bool there, float (&v)[4]) const {
        float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
        if (quads) {
            if (there && first < N) f = *reinterpret_cast<const float4*>(p + first);
        } else if (there) {
            if (first < N) f.x = p[first];
            if (first + 1 < N) f.y = p[first + 1];
            if (first + 2 < N) f.z = p[first + 2];
            if (first + 3 < N) f.w = p[first + 3];
        }
        if (turn) f = make_float4(f.z, f.w, f.x, f.y);
        v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
    }
    __device__ __forceinline__ void put_row(float* p, bool there, const float (&v)[4]) const {
        if (!there) return;
        float4 f = make_float4(v[0], v[1], v[2], v[3]);
        if (turn) f = make_float4(f.z, f.w, f.x, f.y);
        if (quads) {
            if (first < N) *reinterpret_cast<float4*>(p + first) = f;
        } else {
            if (first < N) p[first] = f.x;
            if (first + 1 < N) p[first + 1] = f.y;
            if (first + 2 < N) p[first + 2] = f.z;
            if (first + 3 < N) p[first + 3] = f.w;
        }
    }
    __device__ __forceinline__ void get(const float* p, bool first_there, bool second_there, Pair (&v)[4]) const {
        float x[4], y[4];
        row(p, first_there, x);
        row(p + N, second_there, y);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = pair(x[j], y[j]);
    }
    __device__ __forceinline__ void put(float* p, bool first_there, bool second_there, const Pair (&v)[4]) const {
        float x[4], y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = floats(v[j]).x, y[j] = floats(v[j]).y;
        put_row(p, first_there, x);
        put_row(p + N, second_there, y);
    }
};

template <typename X>
__device__ __forceinline__ void rates(const Scan& s, const Lane<X>& l, int b, int first_channel, bool turned, Pair (&A)[X::P][4]) {
    const States<X> states(l, s.N, false, turned);
    const float* rows = s.a_log + b / s.each * s.a_worker;
#pragma unroll
    for (int p = 0; p < X::P; ++p) {
        const int d = first_channel + l.pair_at(p);
        float x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            states.row(rows + (int64_t)(d + i) * s.N, d + i < s.D, x[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = 4 * l.q + (turned ? j ^ l.turn : j);
                x[i][j] = d + i < s.D && n < s.N ? -rate_of(x[i][j]) : 0.f;  // 0: a state that stays 0
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) A[p][j] = pair(x[0][j], x[1][j]);
    }
}

// h before the task's segment: the maps of those before it applied to h.
template <typename X>
__device__ __forceinline__ void state_before(const Scan& s, int64_t column, int order, const Pair (&A)[X::P][4], Pair (&h)[X::P][4]) {
    const Pair* maps = s.maps + column * s.count * (X::P * 5 * 32) + threadIdx.x % 32;
#pragma unroll 4
    for (int i = 0; i < order; ++i, maps += X::P * 5 * 32)
#pragma unroll
        for (int p = 0; p < X::P; ++p) {
            const Pair dt = maps[(p * 5 + 4) * 32];
#pragma unroll
            for (int j = 0; j < 4; ++j) h[p][j] = fma2(decay_of(dt, A[p][j]), h[p][j], maps[(p * 5 + j) * 32]);
        }
}
template <typename X>
__device__ __forceinline__ void put_map(const Scan& s, int64_t column, int order, const Pair (&h)[X::P][4], const Pair (&dt)[X::P]) {
    Pair* maps = s.maps + (column * s.count + order) * (X::P * 5 * 32) + threadIdx.x % 32;
#pragma unroll
    for (int p = 0; p < X::P; ++p) {
#pragma unroll
        for (int j = 0; j < 4; ++j) maps[(p * 5 + j) * 32] = h[p][j];
        maps[(p * 5 + 4) * 32] = dt[p];
    }
}

// Who takes which of a chunk's inputs: two neighbouring channels (or states) of every kDown-th step per lane.
template <int COUNT>  // channels or states
struct Side {
    static constexpr int kLanes = COUNT / 2 < 32 ? COUNT / 2 : 32, kDown = 32 / kLanes, kItems = R / kDown;
    int at, row;
    __device__ __forceinline__ Side() : at(threadIdx.x % 32 % kLanes * 2), row(threadIdx.x % 32 / kLanes) {}
};
// An array's rows from the segment's first step on, and the lane's place in them. The rows' addresses are the same for
// all lanes, and a lane's offset from them fits 32 bits.
template <typename T>
struct Place {
    const T* rows;
    int64_t step;
    uint32_t offset;
    template <int COUNT>
    __device__ __forceinline__ Place(const Rows& r, int64_t b, int64_t first, int64_t column, const Side<COUNT>& side)
        : rows(r.p == nullptr ? nullptr : static_cast<const T*>(r.p) + b * r.seq + first * r.step + column), step(r.step),
          offset(static_cast<uint32_t>(side.row * r.step + side.at)) {}
    __device__ __forceinline__ const T* at(int64_t t) const { return rows + t * step + offset; }
};
template <typename T, bool WIDE, int COUNT>
struct Wide {
    Two<T, WIDE> v[Side<COUNT>::kItems];
    // From step t on; of `rows` steps and `there` channels. ALL: there are all.
    template <bool ALL>
    __device__ __forceinline__ void load(const Side<COUNT>& side, const Place<T>& p, int64_t t, int rows, int there) {
#pragma unroll
        for (int i = 0; i < Side<COUNT>::kItems; ++i) {
            const bool row = ALL || side.row + i * Side<COUNT>::kDown < rows;
            v[i].template load<ALL>(p.at(t + i * Side<COUNT>::kDown), row && side.at < there, row && side.at + 1 < there);
        }
    }
};

template <typename X>
struct alignas(16) ForwardShared {
    float dt[R][X::kColumn], x[R][X::kColumn], sum[R][X::kColumn];
    float b[R][X::kStates], c[R][X::kStates];
};

// MAPS: the first pass, which makes the segment's map.
template <typename T, bool WIDE, bool MAPS, typename X>
__global__ void __launch_bounds__(32, kForwardBlocks)
scan_kernel(Scan s, const float* h0, T* y, float* last, float* carry, bool quads) {
    layer_begin();
    __shared__ ForwardShared<X> m;
    const Lane<X> l;
    const Side<X::kColumn> side;
    const Side<X::kStates> few;
    const int64_t column = blockIdx.x / s.count;
    const int order = static_cast<int>(blockIdx.x - column * s.count), b = static_cast<int>(column / s.groups);
    if (MAPS && order == s.count - 1) return;  // nobody asks for the last one
    const int d0 = static_cast<int>(column - (int64_t)b * s.groups) * X::kColumn, channels = s.D - d0, worker = b / s.each;
    const int n = s.lengths == nullptr ? s.T : min(max(s.lengths[b], 0), s.T);
    const int first = order * s.steps, end = min(first + s.steps, s.T), inside = min(max(n - first, 0), max(end - first, 0));
    const Place<T> u(s.u, b, first, d0, side), delta(s.delta, b, first, d0, side), z(s.z, b, first, d0, side);
    const Place<T> bs(s.b, b, first, 0, few), cs(s.c, b, first, 0, few);
    const bool gated = s.z.p != nullptr, whole = channels >= X::kColumn && s.N == X::kStates;

    Wide<T, WIDE, X::kColumn> next_u, next_delta, next_z;
    Wide<T, WIDE, X::kStates> next_b, next_c;
    const auto fetch = [&](int t) {
        const int rows = inside - t;
        const auto load = [&](auto known) {
            constexpr bool ALL = decltype(known)::value;
            next_u.template load<ALL>(side, u, t, rows, channels);
            next_delta.template load<ALL>(side, delta, t, rows, channels);
            if (!MAPS && gated) next_z.template load<ALL>(side, z, t, rows, channels);
            next_b.template load<ALL>(few, bs, t, rows, s.N);
            if (!MAPS) next_c.template load<ALL>(few, cs, t, rows, s.N);
        };
        if (whole && rows >= R)
            load(std::true_type{});
        else
            load(std::false_type{});
    };
    fetch(0);

    const States<X> states(l, s.N, quads, false);
    Pair A[X::P][4], h[X::P][4], sum_dt[X::P], lost[X::P], chunk_dt[X::P];
    rates<X>(s, l, b, d0, false, A);
#pragma unroll
    for (int p = 0; p < X::P; ++p) {
        sum_dt[p] = lost[p] = chunk_dt[p] = kZeros;
#pragma unroll
        for (int j = 0; j < 4; ++j) h[p][j] = kZeros;
        const int d = l.pair_at(p);
        if (h0 != nullptr && !MAPS) states.get(h0 + ((int64_t)b * s.D + d0 + d) * s.N, d < channels, d + 1 < channels, h[p]);
    }
    if (!MAPS && s.count > 1) state_before<X>(s, column, order, A, h);
    const bool live = side.at < channels, second = side.at + 1 < channels;
    const auto weight = [&](const float* p, int64_t stride) {
        const float* at = p + worker * stride + d0 + side.at;
        return pair(live ? at[0] : 0.f, second ? at[1] : 0.f);
    };
    const Pair bias = weight(s.bias, s.bias_worker), skip = MAPS ? kZeros : weight(s.skip, s.skip_worker);
    float* carries = carry == nullptr ? nullptr : carry + (((int64_t)b * ((s.T + R - 1) / R) + first / R) * s.D + d0) * s.N;
    const Rows out_rows{y, (int64_t)s.T * s.D, s.D};
    const Place<T> out(out_rows, b, first, d0, side);

    for (int t = 0; t < inside; t += R) {
        const int rows = min(inside - t, R);
        const Wide<T, WIDE, X::kColumn> now_u = next_u, now_z = next_z;
#pragma unroll
        for (int i = 0; i < side.kItems; ++i) {
            const int r = side.row + i * side.kDown;
            const Pair dt = softplus<T>(add2(next_delta.v[i].get(), bias));
            *reinterpret_cast<Pair*>(&m.dt[r][side.at]) = dt;
            *reinterpret_cast<Pair*>(&m.x[r][side.at]) = mul2(dt, now_u.v[i].get());
        }
#pragma unroll
        for (int i = 0; i < few.kItems; ++i) {
            const int r = few.row + i * few.kDown;
            *reinterpret_cast<Pair*>(&m.b[r][few.at]) = next_b.v[i].get();
            if (!MAPS) *reinterpret_cast<Pair*>(&m.c[r][few.at]) = next_c.v[i].get();
        }
        __syncwarp();
        if (t + R < inside) fetch(t + R);
        if (!MAPS && carries != nullptr) {
#pragma unroll
            for (int p = 0; p < X::P; ++p) {
                const int d = l.pair_at(p);
                states.put(carries + (int64_t)d * s.N, d < channels, d + 1 < channels, h[p]);
            }
            carries += (int64_t)s.D * s.N;
        }
        // `many` steps at a time, then their sums: what goes to shared memory in between would hold up the next step's loads
        const auto walk = [&](int r0, auto many) {
            constexpr int COUNT = decltype(many)::value;
            Pair sum[COUNT][X::P];
#pragma unroll
            for (int e = 0; e < COUNT; ++e) {
                const int r = r0 + e;
                Pair dt[X::P], x[X::P];
#pragma unroll
                for (int p = 0; p < X::P; ++p) {
                    dt[p] = *reinterpret_cast<const Pair*>(&m.dt[r][l.pair_at(p)]);
                    x[p] = *reinterpret_cast<const Pair*>(&m.x[r][l.pair_at(p)]);
                    sum[e][p] = kZeros;
                    if (MAPS) chunk_dt[p] = add2(chunk_dt[p], dt[p]);
                }
                const float4 b4 = *reinterpret_cast<const float4*>(&m.b[r][4 * l.q]);
                const float4 c4 = MAPS ? b4 : *reinterpret_cast<const float4*>(&m.c[r][4 * l.q]);
                const float vb[4] = {b4.x, b4.y, b4.z, b4.w}, vc[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int p = 0; p < X::P; ++p) {
                        h[p][j] = fma2(decay_of(dt[p], A[p][j]), h[p][j], mul2(x[p], twice(vb[j])));
                        if (!MAPS) sum[e][p] = fma2(h[p][j], twice(vc[j]), sum[e][p]);
                    }
            }
            if constexpr (!MAPS) {
                float all[COUNT];
#pragma unroll
                for (int e = 0; e < COUNT; ++e) all[e] = over_states<X>(l, sum[e]);
                if (l.sums_up())
#pragma unroll
                    for (int e = 0; e < COUNT; ++e) m.sum[r0 + e][l.summed_channel()] = all[e];
            }
        };
        if (rows == R) {
#pragma unroll 1
            for (int r = 0; r < R; r += kAtOnce) walk(r, std::integral_constant<int, kAtOnce>{});
        } else {
#pragma unroll 1
            for (int r = 0; r < rows; ++r) walk(r, std::integral_constant<int, 1>{});
        }
        __syncwarp();
        if constexpr (MAPS) {
#pragma unroll
            for (int p = 0; p < X::P; ++p) {
                add_up(sum_dt[p], lost[p], chunk_dt[p]);
                chunk_dt[p] = kZeros;
            }
        } else {
#pragma unroll
            for (int i = 0; i < side.kItems; ++i) {
                const int r = side.row + i * side.kDown;
                Pair v = fma2(skip, now_u.v[i].get(), *reinterpret_cast<const Pair*>(&m.sum[r][side.at]));
                if (gated) {
                    const Pair vz = now_z.v[i].get();
                    v = mul2(v, mul2(vz, sigmoid(vz)));
                }
                if (live && (rows == R || r < rows)) store_two<WIDE>(const_cast<T*>(out.at(t + i * side.kDown)), v, second);
            }
            __syncwarp();
        }
    }
    if constexpr (MAPS) {
        put_map<X>(s, column, order, h, sum_dt);
    } else {
        if (live)
            for (int t = inside; t + side.row < end - first; t += side.kDown) store_two<WIDE>(const_cast<T*>(out.at(t)), kZeros, second);
        if (n > first ? n <= end : n == 0 && first == 0)
#pragma unroll
            for (int p = 0; p < X::P; ++p) {
                const int d = l.pair_at(p);
                states.put(last + ((int64_t)b * s.D + d0 + d) * s.N, d < channels, d + 1 < channels, h[p]);
            }
    }
}

struct ScanGradients {
    Rows dy;
    const float *carry, *dlast;
    void *du, *ddelta, *dz;
    float* dh0;
    float* small;   // [B][segments][D N + D + D]: dA, dskip, dbias
    float* few;     // [blocks of columns][B][T][2 kStates]: dc, db
    int blocks;     // of columns per sequence
};

template <typename X>
struct BackwardWarp {
    ulonglong2 h[R / 2][X::P * 2][32];                             // states before every second step
    float dt[R][X::kColumn], x[R][X::kColumn], gy[R][X::kColumn];  // then what the walk sums up
    float sums[R][2 * X::kStates];                                 // dc, db
};
template <typename X>
struct BackwardShared {
    float b[R][X::kStates], c[R][X::kStates];
    BackwardWarp<X> warps[kBackwardWarps];
};

// Backward pass, from the last step to the first. f_t, the gradient of h_t, is
// g_t + c_t gy_t with g_t = a_(t+1) f_(t+1), gy = dy silu(z). A chunk's states
// are made again from the carry and kept at every second step; the walk back
// makes those between, two steps at a time.
template <typename T, bool WIDE, typename X>
__global__ void __launch_bounds__(kBackwardWarps * 32, kBackwardBlocks)
scan_backward_kernel(Scan s, ScanGradients g, bool quads) {
    layer_begin();
    extern __shared__ __align__(16) uint8_t raw[];
    auto& shared = *reinterpret_cast<BackwardShared<X>*>(raw);
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32;
    auto& m = shared.warps[warp];
    const Lane<X> l;
    const Side<X::kColumn> side;
    const Side<X::kStates> few;
    const int lane = l.lane;
    const int64_t per = (int64_t)g.blocks * s.count, b64 = blockIdx.x / per;
    const int b = static_cast<int>(b64), rest = static_cast<int>(blockIdx.x - b64 * per), order = rest % s.count, block = rest / s.count;
    const int group = block * warps + warp, d0 = group * X::kColumn, channels = s.D - d0, worker = b / s.each;
    const int64_t column = b64 * s.groups + group;
    const bool works = group < s.groups, gated = s.z.p != nullptr;
    const int n = s.lengths == nullptr ? s.T : min(max(s.lengths[b], 0), s.T);
    const int segment = s.count - 1 - order;
    const int first = segment * s.steps, end = min(first + s.steps, s.T), inside = min(max(n - first, 0), max(end - first, 0));
    const Place<T> u(s.u, b, first, d0, side), delta(s.delta, b, first, d0, side), z(s.z, b, first, d0, side), dy(g.dy, b, first, d0, side);
    const Place<T> bs(s.b, b, first, 0, few), cs(s.c, b, first, 0, few);

    const States<X> states(l, s.N, quads, true);
    Pair A[X::P][4], flow[X::P][4], dA[X::P][4];
#pragma unroll
    for (int p = 0; p < X::P; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j) A[p][j] = flow[p][j] = dA[p][j] = kZeros;
    const bool live = works && side.at < channels, second = works && side.at + 1 < channels;
    const auto weight = [&](const float* p, int64_t stride) {
        const float* at = p + worker * stride + d0 + side.at;
        return pair(live ? at[0] : 0.f, second ? at[1] : 0.f);
    };
    const Pair bias = weight(s.bias, s.bias_worker), skip = weight(s.skip, s.skip_worker);
    Pair dskip = kZeros, dbias = kZeros;
    if (works) {
        rates<X>(s, l, b, d0, true, A);
#pragma unroll
        for (int p = 0; p < X::P; ++p) {
            const int d = l.pair_at(p);
            if (g.dlast != nullptr) states.get(g.dlast + ((int64_t)b * s.D + d0 + d) * s.N, d < channels, d + 1 < channels, flow[p]);
        }
        if (s.count > 1) state_before<X>(s, column, order, A, flow);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
            for (int k = lane; k < 2 * X::kStates; k += 32) m.sums[r][k] = 0.f;
    }
    const Rows out_rows{nullptr, (int64_t)s.T * s.D, s.D};
    const auto place = [&](void* p) { return Place<T>(Rows{p, out_rows.seq, out_rows.step}, b, first, d0, side); };
    const Place<T> du = place(g.du), ddelta = place(g.ddelta), dz = place(g.dz);
    const auto store = [&](const Place<T>& p, int t, Pair v) { store_two<WIDE>(const_cast<T*>(p.at(t)), v, second); };
    if (live)
        for (int t = inside; t + side.row < end - first; t += side.kDown) {
            store(du, t, kZeros);
            store(ddelta, t, kZeros);
            if (gated) store(dz, t, kZeros);
        }

    for (int t = (inside - 1) / R * R; t >= 0 && inside > 0; t -= R) {
        const int rows = min(inside - t, R), pairs = (rows + 1) / 2;
        Wide<T, WIDE, X::kColumn> in_u, in_delta, in_z, in_dy;
        Pair h[X::P][4], dts[side.kItems];
        // b and c for the block, the rest for the warp
        if (warp == warps - 1) {
            Wide<T, WIDE, X::kStates> in_b, in_c;
            in_b.template load<false>(few, bs, t, rows, s.N);
            in_c.template load<false>(few, cs, t, rows, s.N);
#pragma unroll
            for (int i = 0; i < few.kItems; ++i) {
                const int r = few.row + i * few.kDown;
                *reinterpret_cast<Pair*>(&shared.b[r][few.at]) = in_b.v[i].get();
                *reinterpret_cast<Pair*>(&shared.c[r][few.at]) = in_c.v[i].get();
            }
        }
        if (works) {
            const auto load = [&](auto known) {
                constexpr bool ALL = decltype(known)::value;
                in_delta.template load<ALL>(side, delta, t, rows, channels);
                in_dy.template load<ALL>(side, dy, t, rows, channels);
                in_u.template load<ALL>(side, u, t, rows, channels);
                if (gated) in_z.template load<ALL>(side, z, t, rows, channels);
            };
            if (rows == R && channels >= X::kColumn)
                load(std::true_type{});
            else
                load(std::false_type{});
            const float* carries = g.carry + (((int64_t)b * ((s.T + R - 1) / R) + (first + t) / R) * s.D + d0) * s.N;
#pragma unroll
            for (int p = 0; p < X::P; ++p) {
                const int d = l.pair_at(p);
                states.get(carries + (int64_t)d * s.N, d < channels, d + 1 < channels, h[p]);
            }
#pragma unroll
            for (int i = 0; i < side.kItems; ++i) {
                const int r = side.row + i * side.kDown;
                dts[i] = softplus<T>(add2(in_delta.v[i].get(), bias));
                if (rows < R && r >= rows) dts[i] = kZeros;
                Pair gy = in_dy.v[i].get();
                if (gated) gy = mul2(gy, mul2(in_z.v[i].get(), sigmoid(in_z.v[i].get())));
                *reinterpret_cast<Pair*>(&m.dt[r][side.at]) = dts[i];
                *reinterpret_cast<Pair*>(&m.x[r][side.at]) = mul2(dts[i], in_u.v[i].get());
                *reinterpret_cast<Pair*>(&m.gy[r][side.at]) = gy;
            }
        }
        __syncthreads();
        if (works) {
            // two of the lane's states, in its order
            const auto two_of = [&](const float (&v)[R][X::kStates], int r, int half) {
                return *reinterpret_cast<const float2*>(&v[r][4 * l.q + (2 * half ^ l.turn)]);
            };
            for (int k = 0; k < pairs; ++k) {
#pragma unroll
                for (int p = 0; p < X::P; ++p)
#pragma unroll
                    for (int j = 0; j < 4; j += 2) m.h[k][p * 2 + j / 2][lane] = make_ulonglong2(h[p][j], h[p][j + 1]);
                if (k + 1 == pairs) break;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 2 * k + e;
                    Pair dt[X::P], x[X::P];
#pragma unroll
                    for (int p = 0; p < X::P; ++p) {
                        dt[p] = *reinterpret_cast<const Pair*>(&m.dt[r][l.pair_at(p)]);
                        x[p] = *reinterpret_cast<const Pair*>(&m.x[r][l.pair_at(p)]);
                    }
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const float2 vb = two_of(shared.b, r, half);
#pragma unroll
                        for (int p = 0; p < X::P; ++p) {
                            h[p][2 * half] = fma2(decay_of(dt[p], A[p][2 * half]), h[p][2 * half], mul2(x[p], twice(vb.x)));
                            h[p][2 * half + 1] = fma2(decay_of(dt[p], A[p][2 * half + 1]), h[p][2 * half + 1], mul2(x[p], twice(vb.y)));
                        }
                    }
                }
            }
            for (int k = pairs - 1; k >= 0; --k) {
                Pair dt[2][X::P], x[2][X::P], gy[2][X::P], through[2][X::P], reach[2][X::P], sum[2][X::P];
                float dc[2][4], db[2][4];
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int p = 0; p < X::P; ++p) {
                        dt[e][p] = *reinterpret_cast<const Pair*>(&m.dt[2 * k + e][l.pair_at(p)]);
                        x[e][p] = *reinterpret_cast<const Pair*>(&m.x[2 * k + e][l.pair_at(p)]);
                        gy[e][p] = *reinterpret_cast<const Pair*>(&m.gy[2 * k + e][l.pair_at(p)]);
                        through[e][p] = reach[e][p] = sum[e][p] = kZeros;
                    }
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float2 vb[2], vc[2];
                    ulonglong2 kept[X::P];
#pragma unroll
                    for (int e = 0; e < 2; ++e) vb[e] = two_of(shared.b, 2 * k + e, half), vc[e] = two_of(shared.c, 2 * k + e, half);
#pragma unroll
                    for (int p = 0; p < X::P; ++p) kept[p] = m.h[k][p * 2 + half][lane];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int j = 2 * half + i;
                        Pair to_c[2] = {kZeros, kZeros}, to_b[2] = {kZeros, kZeros}, b2[2], c2[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) b2[e] = twice(i ? vb[e].y : vb[e].x), c2[e] = twice(i ? vc[e].y : vc[e].x);
#pragma unroll
                        for (int p = 0; p < X::P; ++p) {
                            Pair at[3], a[2];
                            at[0] = i ? kept[p].y : kept[p].x;
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                a[e] = decay_of(dt[e][p], A[p][j]);
                                at[e + 1] = fma2(a[e], at[e], mul2(x[e][p], b2[e]));
                            }
#pragma unroll
                            for (int e = 1; e >= 0; --e) {
                                const Pair f = fma2(gy[e][p], c2[e], flow[p][j]);
                                to_c[e] = fma2(at[e + 1], gy[e][p], to_c[e]);
                                to_b[e] = fma2(f, x[e][p], to_b[e]);
                                through[e][p] = fma2(f, b2[e], through[e][p]);
                                sum[e][p] = fma2(at[e + 1], c2[e], sum[e][p]);
                                flow[p][j] = mul2(f, a[e]);
                                const Pair r = mul2(flow[p][j], at[e]);
                                reach[e][p] = fma2(r, A[p][j], reach[e][p]);
                                dA[p][j] = fma2(r, dt[e][p], dA[p][j]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            dc[e][j] = floats(to_c[e]).x + floats(to_c[e]).y;
                            db[e][j] = floats(to_b[e]).x + floats(to_b[e]).y;
                        }
                    }
                }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = 2 * k + e, d = l.summed_channel(), state = l.summed_state();
                    const float all_through = over_states<X>(l, through[e]), all_reach = over_states<X>(l, reach[e]), all = over_states<X>(l, sum[e]);
                    if (l.sums_up()) m.dt[r][d] = all_through, m.x[r][d] = all_reach, m.gy[r][d] = all;
                    const float2 both = over_channels<X>(l, dc[e], db[e]);
                    if constexpr (X::S == 8)
                        m.sums[r][state] = both.x, m.sums[r][X::kStates + state] = both.y;
                    else if (X::S == 4 || l.g < 8)
                        m.sums[r][(l.g & 4 ? X::kStates : 0) + state] = both.x;
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < side.kItems; ++i) {
                const int r = side.row + i * side.kDown, at = t + i * side.kDown;
                const Pair through = *reinterpret_cast<const Pair*>(&m.dt[r][side.at]), reach = *reinterpret_cast<const Pair*>(&m.x[r][side.at]);
                const Pair sum = *reinterpret_cast<const Pair*>(&m.gy[r][side.at]), vu = in_u.v[i].get(), vdy = in_dy.v[i].get();
                Pair gy = vdy;
                const bool here = live && (rows == R || r < rows);
                if (gated) {
                    const Pair vz = in_z.v[i].get();
                    const Pair gate = sigmoid(vz);
                    gy = mul2(vdy, mul2(vz, gate));
                    if (here) store(dz, at, mul2(mul2(vdy, silu_slope(vz, gate)), fma2(skip, vu, sum)));
                }
                const Pair dbase = mul2(fma2(through, vu, mul2(reach, twice(kLn2f))), sigmoid(add2(in_delta.v[i].get(), bias)));
                if (here) {
                    store(du, at, fma2(through, dts[i], mul2(skip, gy)));
                    store(ddelta, at, dbase);
                    dskip = fma2(gy, vu, dskip);
                    dbias = add2(dbias, dbase);
                }
            }
        }
        __syncthreads();
        float* to = g.few + (((int64_t)block * s.B + b) * s.T + first + t) * (2 * X::kStates);
        for (int i = threadIdx.x; i < rows * 2 * X::kStates; i += blockDim.x) {
            float v = (&shared.warps[0].sums[0][0])[i];
            for (int w = 1; w < warps; ++w) v += (&shared.warps[w].sums[0][0])[i];
            to[i] = v;
        }
    }
    if (!works) return;
    const int64_t each = (int64_t)s.D * (s.N + 2);
    float* small = g.small + ((int64_t)b * s.count + segment) * each;
    const States<X> unaligned(l, s.N, false, true);
#pragma unroll
    for (int p = 0; p < X::P; ++p) {
        const int d = l.pair_at(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) dA[p][j] = mul2(mul2(dA[p][j], A[p][j]), twice(kLn2f));
        unaligned.put(small + (int64_t)(d0 + d) * s.N, d < channels, d + 1 < channels, dA[p]);
        if (g.dh0 != nullptr && segment == 0) states.put(g.dh0 + ((int64_t)b * s.D + d0 + d) * s.N, d < channels, d + 1 < channels, flow[p]);
    }
#pragma unroll
    for (int down = side.kLanes; down < 32; down *= 2) {
        dskip = add2(dskip, shuffle(dskip, down));
        dbias = add2(dbias, shuffle(dbias, down));
    }
    if (side.row == 0 && live) {
        float* to = small + (int64_t)s.D * s.N + d0 + side.at;
        to[0] = floats(dskip).x, to[s.D] = floats(dbias).x;
        if (second) to[1] = floats(dskip).y, to[s.D + 1] = floats(dbias).y;
    }
}

// The segments' maps of what flows back.
template <typename T, bool WIDE, typename X>
__global__ void __launch_bounds__(32, kForwardBlocks)
scan_backward_maps_kernel(Scan s, Rows grads) {
    layer_begin();
    __shared__ ForwardShared<X> m;
    const Lane<X> l;
    const Side<X::kColumn> side;
    const Side<X::kStates> few;
    const int64_t column = blockIdx.x / s.count;
    const int order = static_cast<int>(blockIdx.x - column * s.count), b = static_cast<int>(column / s.groups);
    if (order == s.count - 1) return;
    const int d0 = static_cast<int>(column - (int64_t)b * s.groups) * X::kColumn, channels = s.D - d0, worker = b / s.each;
    const int n = s.lengths == nullptr ? s.T : min(max(s.lengths[b], 0), s.T);
    const int first = (s.count - 1 - order) * s.steps, end = min(first + s.steps, s.T), inside = min(max(n - first, 0), max(end - first, 0));
    const Place<T> delta(s.delta, b, first, d0, side), z(s.z, b, first, d0, side), dy(grads, b, first, d0, side), cs(s.c, b, first, 0, few);
    const bool gated = s.z.p != nullptr, whole = channels >= X::kColumn && s.N == X::kStates;
    Wide<T, WIDE, X::kColumn> next_delta, next_z, next_dy;
    Wide<T, WIDE, X::kStates> next_c;
    const auto fetch = [&](int t) {
        const int rows = inside - t;
        const auto load = [&](auto known) {
            constexpr bool ALL = decltype(known)::value;
            next_delta.template load<ALL>(side, delta, t, rows, channels);
            if (gated) next_z.template load<ALL>(side, z, t, rows, channels);
            next_dy.template load<ALL>(side, dy, t, rows, channels);
            next_c.template load<ALL>(few, cs, t, rows, s.N);
        };
        if (whole && rows >= R)
            load(std::true_type{});
        else
            load(std::false_type{});
    };
    if (inside > 0) fetch((inside - 1) / R * R);
    Pair A[X::P][4], flow[X::P][4], sum_dt[X::P], lost[X::P], chunk_dt[X::P];
    rates<X>(s, l, b, d0, false, A);
#pragma unroll
    for (int p = 0; p < X::P; ++p) {
        sum_dt[p] = lost[p] = chunk_dt[p] = kZeros;
#pragma unroll
        for (int j = 0; j < 4; ++j) flow[p][j] = kZeros;
    }
    const float* at = s.bias + worker * s.bias_worker + d0 + side.at;
    const Pair bias = pair(side.at < channels ? at[0] : 0.f, side.at + 1 < channels ? at[1] : 0.f);
    for (int t = (inside - 1) / R * R; t >= 0 && inside > 0; t -= R) {
        const int rows = min(inside - t, R);
#pragma unroll
        for (int i = 0; i < few.kItems; ++i) *reinterpret_cast<Pair*>(&m.c[few.row + i * few.kDown][few.at]) = next_c.v[i].get();
#pragma unroll
        for (int i = 0; i < side.kItems; ++i) {
            const int r = side.row + i * side.kDown;
            Pair gy = next_dy.v[i].get();
            if (gated) gy = mul2(gy, mul2(next_z.v[i].get(), sigmoid(next_z.v[i].get())));
            *reinterpret_cast<Pair*>(&m.dt[r][side.at]) = softplus<T>(add2(next_delta.v[i].get(), bias));
            *reinterpret_cast<Pair*>(&m.x[r][side.at]) = gy;
        }
        __syncwarp();
        if (t > 0) fetch(t - R);
        const auto step = [&](int r) {
            Pair dt[X::P], gy[X::P];
#pragma unroll
            for (int p = 0; p < X::P; ++p) {
                dt[p] = *reinterpret_cast<const Pair*>(&m.dt[r][l.pair_at(p)]);
                gy[p] = *reinterpret_cast<const Pair*>(&m.x[r][l.pair_at(p)]);
                chunk_dt[p] = add2(chunk_dt[p], dt[p]);
            }
            const float4 c4 = *reinterpret_cast<const float4*>(&m.c[r][4 * l.q]);
            const float vc[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int p = 0; p < X::P; ++p) flow[p][j] = mul2(decay_of(dt[p], A[p][j]), fma2(gy[p], twice(vc[j]), flow[p][j]));
        };
        if (rows == R) {
#pragma unroll 4
            for (int r = R - 1; r >= 0; --r) step(r);
        } else {
#pragma unroll 1
            for (int r = rows - 1; r >= 0; --r) step(r);
        }
#pragma unroll
        for (int p = 0; p < X::P; ++p) {
            add_up(sum_dt[p], lost[p], chunk_dt[p]);
            chunk_dt[p] = kZeros;
        }
        __syncwarp();
    }
    // what reads it has two of the lane's states in another order
#pragma unroll
    for (int p = 0; p < X::P; ++p)
        if (l.turn) {
            const Pair a = flow[p][0], b = flow[p][1];
            flow[p][0] = flow[p][2], flow[p][1] = flow[p][3], flow[p][2] = a, flow[p][3] = b;
        }
    put_map<X>(s, column, order, flow, sum_dt);
}

// db and dc: the sum of the blocks' parts, 0 beyond a length.
template <typename T>
__global__ void __launch_bounds__(256)
sum_few_kernel(const float* parts, int blocks, int B, int T_, int N, int states, const int32_t* lengths, T* db, T* dc) {
    layer_begin();
    const int64_t all = (int64_t)B * T_ * N, one = (int64_t)B * T_ * 2 * states;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / N, b = row / T_;
        const int k = static_cast<int>(i - row * N), t = static_cast<int>(row - b * T_);
        float vc = 0.f, vb = 0.f;
        if (lengths == nullptr || t < lengths[b]) {
            const float* p = parts + row * 2 * states + k;
#pragma unroll 4
            for (int g = 0; g < blocks; ++g) {
                vc += p[g * one];
                vb += p[g * one + states];
            }
        }
        dc[i] = from_float<T>(vc);
        db[i] = from_float<T>(vb);
    }
}

// One step: 4 states of a channel per thread, S threads to a channel. States move as in a pass, to the bit: the decays are
// its, with the power's bias made up for, which generated tokens would add up otherwise (1.9e-8 of a slow state each).
template <typename T, int S>
__global__ void __launch_bounds__(128)
scan_step_kernel(Scan s, float* h, T* y) {
    layer_begin();
    const int64_t i = ((int64_t)blockIdx.x * 128 + threadIdx.x) / S, b = i / s.D;
    const bool there = b < s.B;
    const int d = static_cast<int>(i - b * s.D), q = threadIdx.x % S, worker = static_cast<int>(b / s.each);
    float sum = 0.f, u = 0.f;
    if (there) {
        u = to_float(static_cast<const T*>(s.u.p)[b * s.u.seq + d]);
        const float raw = to_float(static_cast<const T*>(s.delta.p)[b * s.delta.seq + d]) + s.bias[worker * s.bias_worker + d];
        const float dt = floats(softplus<T>(pair(raw, 0.f))).x, x = dt * u;
        const float* a = s.a_log + worker * s.a_worker + (int64_t)d * s.N;
        float* state = h + i * s.N;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = 4 * q + j;
            if (n < s.N) {
                const float decay = floats(decay_of(pair(dt, 0.f), pair(-rate_of(a[n]), 0.f))).x;
                const float vb = to_float(static_cast<const T*>(s.b.p)[b * s.b.seq + n]), vc = to_float(static_cast<const T*>(s.c.p)[b * s.c.seq + n]);
                const float next = fmaf(decay, state[n], x * vb);
                state[n] = next;
                sum = fmaf(next, vc, sum);
            }
        }
    }
#pragma unroll
    for (int k = 1; k < S; k *= 2) sum += __shfl_xor_sync(~0u, sum, k);
    if (!there || q > 0) return;
    float v = fmaf(s.skip[worker * s.skip_worker + d], u, sum);
    if (s.z.p != nullptr) {
        const float z = to_float(static_cast<const T*>(s.z.p)[b * s.z.seq + d]);
        v *= z * floats(sigmoid(pair(z, 0.f))).x;
    }
    y[i] = from_float<T>(v);
}

// -- the host's side -------------------------------------------------------------------------------------------------

cpdp_status check_scan(int W, int B, int64_t T, int D, int N, cpdp_dtype dtype) {
    if (B < 0) return layer_error(CPDP_EINVAL, "B=%d must be >= 0", B);
    CPDP_TRY(check_sizes(1, T, D));
    if (W < 1 || W > 4096 || B % W != 0) return layer_error(CPDP_EINVAL, "W=%d must be in [1, 4096] and divide B=%d", W, B);
    if (N < 1 || N > CPDP_SCAN_MAX_STATES) return layer_error(CPDP_EINVAL, "N=%d must be in [1, %d]", N, CPDP_SCAN_MAX_STATES);
    if (T > int64_t(1) << 30) return layer_error(CPDP_EINVAL, "T=%lld is at most 2^30", (long long)T);
    if (B > 0) {
        if (T > kLayerMaxRows / B || (T > 0 && D > kLayerMaxElements / 64 / (B * T)))
            return layer_error(CPDP_EINVAL, "B=%d, T=%lld, D=%d: B * T is at most 2^31 - 1 and all elements at most 2^34", B, (long long)T, D);
        if (ceil_div(D, 8) > (kLayerMaxRows >> 6) / B) return layer_error(CPDP_EINVAL, "B=%d, D=%d: more blocks than a launch takes", B, D);
    }
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    return CPDP_OK;
}

template <bool BACKWARD, typename F>
auto with_shape(int N, F&& f) {
    if constexpr (BACKWARD)
        return N <= 8 ? f(Shape<2, 2>{}) : N <= 16 ? f(Shape<4, 2>{}) : f(Shape<8, 2>{});
    else
        return N <= 8 ? f(Shape<2, 2>{}) : N <= 16 ? f(Shape<4, 4>{}) : f(Shape<8, 4>{});
}

struct Plan {
    int groups, column, states;   // columns of a sequence, channels of one, padded states
    int count, steps;             // segments
    int warps, blocks;            // of the backward pass: of a block, and blocks of columns per sequence
    int64_t maps, few, small;     // bytes
};
// `warps`: as many as run at once on the GPU.
Plan plan_of(int B, int64_t T, int D, int N, int64_t warps, bool backward) {
    Plan p{};
    const auto shaped = [&](auto x) { return p.column = decltype(x)::kColumn, p.states = decltype(x)::kStates, decltype(x)::P; };
    const int pairs = backward ? with_shape<true>(N, shaped) : with_shape<false>(N, shaped);
    p.groups = static_cast<int>(ceil_div(D, p.column));
    const int64_t columns = (int64_t)B * p.groups;
    int64_t count = columns * 3 <= warps ? warps / std::max<int64_t>(columns, 1) : 1;
    count = std::max<int64_t>(std::min(count, T / (4 * R)), 1);
    p.steps = static_cast<int>(ceil_div(ceil_div(std::max<int64_t>(T, 1), count), R) * R);
    p.count = static_cast<int>(std::max<int64_t>(ceil_div(T, p.steps), 1));
    p.maps = p.count > 1 ? columns * p.count * pairs * 5 * 32 * 8 : 0;
    if (backward) {
        p.warps = 1;
        for (int w = 2; w <= kBackwardWarps; ++w)
            if (ceil_div(p.groups, w) * w <= ceil_div(p.groups, p.warps) * p.warps + p.groups / 16) p.warps = w;
        p.blocks = static_cast<int>(ceil_div(p.groups, p.warps));
        p.few = ceil_div((int64_t)p.blocks * B * T * 2 * p.states * 4, 16) * 16;
        p.small = ceil_div((int64_t)B * p.count * D * (N + 2) * 4, 16) * 16;
    }
    return p;
}
Plan forward_plan(int B, int64_t T, int D, int N) { return plan_of(B, T, D, N, kSMs * kForwardBlocks, false); }
Plan backward_plan(int B, int64_t T, int D, int N) { return plan_of(B, T, D, N, kSMs * kBackwardBlocks * kBackwardWarps, true); }

bool pairs_at(const Rows& r, int64_t e) { return aligned_to(r.p, 2 * e) && r.seq % 2 == 0 && r.step % 2 == 0; }

cpdp_status check_step(const Rows& r, int64_t T) {  // a lane's offset from rows is held in 32 bits
    if (T > 1 && r.step >= int64_t(1) << 28) return layer_error(CPDP_EINVAL, "step strides (%lld) must be below 2^28", (long long)r.step);
    return CPDP_OK;
}

cpdp_status check_inputs(const Scan& s, int64_t e, bool some) {
    CPDP_TRY(check_array("u", s.u.p, some, e, s.u.seq, s.u.step));
    CPDP_TRY(check_array("delta", s.delta.p, some, e, s.delta.seq, s.delta.step));
    CPDP_TRY(check_array("z", s.z.p, false, e, s.z.seq, s.z.step));
    CPDP_TRY(check_array("b", s.b.p, some, e, s.b.seq, s.b.step));
    CPDP_TRY(check_array("c", s.c.p, some, e, s.c.seq, s.c.step));
    for (const Rows* r : {&s.u, &s.delta, &s.z, &s.b, &s.c}) CPDP_TRY(check_step(*r, s.T));
    CPDP_TRY(check_array("a_log", s.a_log, true, 4, s.a_worker));
    CPDP_TRY(check_array("skip", s.skip, true, 4, s.skip_worker));
    CPDP_TRY(check_array("bias", s.bias, true, 4, s.bias_worker));
    return check_array("lengths", s.lengths, false, 4);
}

Scan scan_of(const cpdp_scan_inputs& in, int W, int B, int64_t T, int D, int N) {
    Scan s{};
    s.u = {in.u, in.u_seq, in.u_step}, s.delta = {in.delta, in.delta_seq, in.delta_step}, s.z = {in.z, in.z_seq, in.z_step};
    s.b = {in.b, in.b_seq, in.b_step}, s.c = {in.c, in.c_seq, in.c_step};
    s.a_log = in.a_log, s.a_worker = in.a_log_worker, s.skip = in.skip, s.skip_worker = in.skip_worker, s.bias = in.bias, s.bias_worker = in.bias_worker;
    s.lengths = in.lengths;
    s.B = B, s.T = static_cast<int>(T), s.D = D, s.N = N, s.each = B / W;
    return s;
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

size_t cpdp_selective_scan_workspace(int B, int64_t T, int D, int N) {
    return check_scan(1, B, T, D, N, CPDP_F32) != CPDP_OK || B == 0 ? 0 : forward_plan(B, T, D, N).maps;
}

size_t cpdp_selective_scan_backward_workspace(int B, int64_t T, int D, int N) {
    if (check_scan(1, B, T, D, N, CPDP_F32) != CPDP_OK || B == 0) return 0;
    const Plan p = backward_plan(B, T, D, N);
    return p.maps + p.few + p.small;
}

cpdp_status cpdp_selective_scan(const cpdp_scan_inputs* inputs, cpdp_dtype dtype, int W, int B, int64_t T, int D, int N, const float* h0, void* y,
                                float* last, float* carry, void* workspace, size_t workspace_bytes, void* stream) {
    constexpr const char* what = "cpdp_selective_scan";
    CPDP_TRY(check_scan(W, B, T, D, N, dtype));
    if (inputs == nullptr) return layer_error(CPDP_EINVAL, "inputs is NULL");
    Scan s = scan_of(*inputs, W, B, T, D, N);
    const int64_t e = dtype_size(dtype);
    const bool some = B > 0 && T > 0;
    CPDP_TRY(check_inputs(s, e, some));
    CPDP_TRY(check_array("h0", h0, false, 4));
    CPDP_TRY(check_array("y", y, some, e));
    CPDP_TRY(check_array("last", last, B > 0, 4));
    CPDP_TRY(check_array("carry", carry, false, 4));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_selective_scan_workspace(B, T, D, N)));
    if (B == 0) return CPDP_OK;
    const Plan plan = forward_plan(B, T, D, N);
    s.groups = plan.groups, s.count = plan.count, s.steps = plan.steps, s.maps = static_cast<Pair*>(workspace);
    const bool quads = N % 4 == 0 && aligned_to(h0, 16) && aligned_to(last, 16) && aligned_to(carry, 16);
    const bool wide = D % 2 == 0 && pairs_at(s.u, e) && pairs_at(s.delta, e) && pairs_at(s.z, e) && N % 2 == 0 && pairs_at(s.b, e) && pairs_at(s.c, e) &&
                      aligned_to(y, 2 * e);
    const unsigned blocks = static_cast<unsigned>((int64_t)B * plan.groups * plan.count);
    const auto go = [&](auto* out, auto two) {
        using E = std::remove_pointer_t<decltype(out)>;
        constexpr bool WIDE = decltype(two)::value;
        return with_shape<false>(N, [&](auto shape) {
            using X = decltype(shape);
            if (plan.count > 1) {
                const cudaError_t first = launch_layer(scan_kernel<E, WIDE, true, X>, blocks, 32, 0, stream, s, h0, out, last, carry, quads);
                if (first != cudaSuccess) return first;
            }
            return launch_layer(scan_kernel<E, WIDE, false, X>, blocks, 32, 0, stream, s, h0, out, last, carry, quads);
        });
    };
    const auto typed = [&](auto* out) { return wide ? go(out, std::true_type{}) : go(out, std::false_type{}); };
    return layer_launched(dtype == CPDP_F32 ? typed(static_cast<float*>(y)) : typed(static_cast<__nv_bfloat16*>(y)), what);
}

cpdp_status cpdp_selective_scan_backward(const void* dy, int64_t dy_seq, int64_t dy_step, const cpdp_scan_inputs* inputs, cpdp_dtype dtype, int W,
                                         int B, int64_t T, int D, int N, const float* carry, const float* dlast, void* du, void* ddelta, void* dz,
                                         void* db, void* dc, float* dh0, void* da_log, int64_t da_log_worker, void* dskip, int64_t dskip_worker,
                                         void* dbias, int64_t dbias_worker, cpdp_dtype dweight_dtype, void* workspace, size_t workspace_bytes,
                                         void* stream) {
    constexpr const char* what = "cpdp_selective_scan_backward";
    CPDP_TRY(check_scan(W, B, T, D, N, dtype));
    if (inputs == nullptr) return layer_error(CPDP_EINVAL, "inputs is NULL");
    if (!known_dtype(dweight_dtype)) return layer_error(CPDP_EINVAL, "unknown dtype of the weights' gradients: %d", (int)dweight_dtype);
    Scan s = scan_of(*inputs, W, B, T, D, N);
    const int64_t e = dtype_size(dtype), grad = dtype_size(dweight_dtype);
    const bool some = B > 0 && T > 0;
    CPDP_TRY(check_array("dy", dy, some, e, dy_seq, dy_step));
    CPDP_TRY(check_inputs(s, e, some));
    CPDP_TRY(check_step({dy, dy_seq, dy_step}, T));
    CPDP_TRY(check_array("carry", carry, some, 4));
    CPDP_TRY(check_array("dlast", dlast, false, 4));
    CPDP_TRY(check_array("du", du, some, e));
    CPDP_TRY(check_array("ddelta", ddelta, some, e));
    CPDP_TRY(check_array("dz", dz, some && s.z.p != nullptr, e));
    CPDP_TRY(check_array("db", db, some, e));
    CPDP_TRY(check_array("dc", dc, some, e));
    CPDP_TRY(check_array("dh0", dh0, false, 4));
    CPDP_TRY(check_array("da_log", da_log, true, grad, da_log_worker));
    CPDP_TRY(check_array("dskip", dskip, true, grad, dskip_worker));
    CPDP_TRY(check_array("dbias", dbias, true, grad, dbias_worker));
    CPDP_TRY(check_apart("da_log", W, da_log_worker, (int64_t)D * N));
    CPDP_TRY(check_apart("dskip", W, dskip_worker, D));
    CPDP_TRY(check_apart("dbias", W, dbias_worker, D));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_selective_scan_backward_workspace(B, T, D, N)));
    const SumsOut sums{{da_log, dskip, dbias}, {da_log_worker, dskip_worker, dbias_worker}, {(int64_t)D * N, D, D}};
    if (B == 0) return layer_launched(sum_gradients(nullptr, 0, W, sums, dweight_dtype, stream), what);
    const Plan plan = backward_plan(B, T, D, N);
    s.groups = plan.groups, s.count = plan.count, s.steps = plan.steps, s.maps = static_cast<Pair*>(workspace);
    ScanGradients g{};
    g.dy = {dy, dy_seq, dy_step}, g.carry = carry, g.dlast = dlast, g.du = du, g.ddelta = ddelta, g.dz = dz, g.dh0 = dh0;
    g.few = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.maps);
    g.small = reinterpret_cast<float*>(static_cast<char*>(workspace) + plan.maps + plan.few);
    g.blocks = plan.blocks;
    const bool quads = N % 4 == 0 && aligned_to(carry, 16) && aligned_to(dlast, 16) && aligned_to(dh0, 16);
    const bool wide = D % 2 == 0 && pairs_at(s.u, e) && pairs_at(s.delta, e) && pairs_at(s.z, e) && pairs_at(g.dy, e) && N % 2 == 0 &&
                      pairs_at(s.b, e) && pairs_at(s.c, e) && aligned_to(du, 2 * e) &&
                      aligned_to(ddelta, 2 * e) && aligned_to(dz, 2 * e);
    const auto go = [&](auto* out, auto two) {
        using E = std::remove_pointer_t<decltype(out)>;
        constexpr bool WIDE = decltype(two)::value;
        return with_shape<true>(N, [&](auto shape) {
            using X = decltype(shape);
            if (plan.count > 1) {
                const cudaError_t first = launch_layer(scan_backward_maps_kernel<E, WIDE, X>, static_cast<unsigned>((int64_t)B * plan.groups * plan.count),
                                                       32, 0, stream, s, g.dy);
                if (first != cudaSuccess) return first;
            }
            const int smem = static_cast<int>(sizeof(BackwardShared<X>) - (kBackwardWarps - plan.warps) * sizeof(BackwardWarp<X>));
            const cudaError_t allowed = allow_shared_memory<scan_backward_kernel<E, WIDE, X>>(sizeof(BackwardShared<X>));
            if (allowed != cudaSuccess) return allowed;
            return launch_layer(scan_backward_kernel<E, WIDE, X>, static_cast<unsigned>((int64_t)B * plan.blocks * plan.count), plan.warps * 32, smem,
                                stream, s, g, quads);
        });
    };
    const auto typed = [&](auto* out) { return wide ? go(out, std::true_type{}) : go(out, std::false_type{}); };
    CPDP_TRY(layer_launched(dtype == CPDP_F32 ? typed(static_cast<float*>(du)) : typed(static_cast<__nv_bfloat16*>(du)), what));
    if (T > 0) {
        const unsigned blocks = static_cast<unsigned>(std::min<int64_t>(ceil_div((int64_t)B * T * N, 256), kSMs * 8));
        const auto sum = [&](auto* out) {
            using E = std::remove_pointer_t<decltype(out)>;
            return launch_layer(sum_few_kernel<E>, blocks, 256, 0, stream, static_cast<const float*>(g.few), plan.blocks, B, static_cast<int>(T), N,
                                plan.states, s.lengths, out, static_cast<E*>(dc));
        };
        CPDP_TRY(layer_launched(dtype == CPDP_F32 ? sum(static_cast<float*>(db)) : sum(static_cast<__nv_bfloat16*>(db)), what));
    }
    return layer_launched(sum_gradients(g.small, B / W * plan.count, W, sums, dweight_dtype, stream), what);
}

cpdp_status cpdp_selective_scan_step(const cpdp_scan_inputs* inputs, cpdp_dtype dtype, int W, int B, int D, int N, float* state, void* y, void* stream) {
    CPDP_TRY(check_scan(W, B, 1, D, N, dtype));
    if (inputs == nullptr) return layer_error(CPDP_EINVAL, "inputs is NULL");
    const Scan s = scan_of(*inputs, W, B, 1, D, N);
    const int64_t e = dtype_size(dtype);
    CPDP_TRY(check_inputs(s, e, B > 0));
    CPDP_TRY(check_array("state", state, B > 0, 4));
    CPDP_TRY(check_array("y", y, B > 0, e));
    if (B == 0) return CPDP_OK;
    const auto go = [&](auto* out) {
        using E = std::remove_pointer_t<decltype(out)>;
        return with_shape<false>(N, [&](auto shape) {
            constexpr int S = decltype(shape)::S;
            return launch_layer(scan_step_kernel<E, S>, static_cast<unsigned>(ceil_div((int64_t)B * D * S, 128)), 128, 0, stream, s, state, out);
        });
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(y)) : go(static_cast<__nv_bfloat16*>(y)), "cpdp_selective_scan_step");
}
