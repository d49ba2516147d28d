// The gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) v_t, its backward
// pass and its single step (include/cpdp_layers.h).
#include <type_traits>

#include "cpdp_layers.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 128;   // of the single step's kernel
constexpr int kWarps = 8;       // of a tile: each takes R consecutive steps
constexpr int kChannels = 64;   // of a tile: two per lane
constexpr int kForwardSteps = 16, kBackwardSteps = 8;  // R
constexpr int kForwardTile = kWarps * kForwardSteps, kBackwardTile = kWarps * kBackwardSteps;
constexpr int kGroup = 16;      // tiles between two published states
constexpr int kSpinLimit = 1 << 22;
static_assert(kBackwardTile == CPDP_CARRY_STEPS, "a backward tile starts from a carry");
static_assert(kForwardTile % CPDP_CARRY_STEPS == 0 && CPDP_CARRY_STEPS % kForwardSteps == 0, "carries fall on warps' first steps");

__device__ unsigned long long wait_timeouts;  // bounded waits that ran out

struct SeqIn {
    const void* p;
    int64_t seq, step;
};

// a = sigmoid(x) and 1 - a, neither formed as a difference from 1. With
// t = e^-|x| in [0, 1] they are 1 / (1 + t) and t / (1 + t). The power is 2^p of
// the rounded product p = |x| log2(e), so t's relative error is some ulps and
// grows with |x| (1e-6 at 16, where t itself is 1e-7). The scans are bound by
// the instructions that they issue: exact range reduction and division, with
// their cases for tiny numbers, took 2.5 times as many.
__device__ __forceinline__ void gate_of(float x, float& a, float& rest) {
    float t, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(-1.44269504f * fabsf(x)));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + t));
    const float q = t * r;
    a = x >= 0.f ? r : q;
    rest = x >= 0.f ? q : r;
}

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t b, int64_t steps) {
    return lengths == nullptr ? steps : min(max((int64_t)lengths[b], (int64_t)0), steps);
}

// Two neighbouring channels as they lie in memory. PAIR: one load or store,
// possible where D and the strides are even and the pointers aligned to two
// elements; else element by element, `second` telling whether there are two.
template <typename T>
struct Two;
template <>
struct Two<float> {
    float2 v;
    __device__ __forceinline__ float2 get() const { return v; }
};
template <>
struct Two<__nv_bfloat16> {
    uint32_t v;
    __device__ __forceinline__ float2 get() const { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
};
template <bool PAIR>
__device__ __forceinline__ Two<float> load_two(const float* p, bool second) {
    if (PAIR) return {__ldcs(reinterpret_cast<const float2*>(p))};
    return {make_float2(__ldcs(p), second ? __ldcs(p + 1) : 0.f)};
}
template <bool PAIR>
__device__ __forceinline__ Two<__nv_bfloat16> load_two(const __nv_bfloat16* p, bool second) {
    if (PAIR) return {__ldcs(reinterpret_cast<const uint32_t*>(p))};
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
    return {static_cast<uint32_t>(__ldcs(q)) | (second ? static_cast<uint32_t>(__ldcs(q + 1)) << 16 : 0u)};
}
template <bool PAIR>
__device__ __forceinline__ void store_two(float* p, float2 v, bool second) {
    if (PAIR) {
        *reinterpret_cast<float2*>(p) = v;
    } else {
        p[0] = v.x;
        if (second) p[1] = v.y;
    }
}
template <bool PAIR>
__device__ __forceinline__ void store_two(__nv_bfloat16* p, float2 v, bool second) {
    if (PAIR) {
        *reinterpret_cast<__nv_bfloat162*>(p) = __float22bfloat162_rn(v);
    } else {
        p[0] = __float2bfloat16_rn(v.x);
        if (second) p[1] = __float2bfloat16_rn(v.y);
    }
}

// x -> a x + b for two channels, and one such map after another.
struct Map {
    float2 a, b;
};
__device__ __forceinline__ float2 apply(const Map& m, float2 x) { return make_float2(fmaf(m.a.x, x.x, m.b.x), fmaf(m.a.y, x.y, m.b.y)); }
__device__ __forceinline__ Map then(const Map& first, const Map& second) {
    return {make_float2(second.a.x * first.a.x, second.a.y * first.a.y), apply(second, first.b)};
}

// What tiles tell each other, in the workspace: for every tile and channel its
// map (a, b) in one 64-bit word, and for every group of tiles and channel the
// state after it in 32 bits. All ones means "not there yet" (the workspace is
// set to that before the launch); no arithmetic makes that NaN, and a value
// that has it is stored as the usual NaN. A word is written whole, so the
// readers need no flag and no fence.
struct Exchange {
    unsigned* ticket;
    uint64_t* maps;    // [B][tiles][channels]
    uint32_t* states;  // [B][groups][channels]
    int tiles, groups, channels;  // channels: a multiple of kChannels
};

__device__ __forceinline__ uint32_t told(float x) {
    const uint32_t u = __float_as_uint(x);
    return u == 0xffffffffu ? 0x7fffffffu : u;
}
__device__ __forceinline__ void tell_map(uint64_t* p, const Map& m) {
    const uint64_t x = (uint64_t)told(m.a.x) << 32 | __float_as_uint(m.b.x), y = (uint64_t)told(m.a.y) << 32 | __float_as_uint(m.b.y);
    asm volatile("st.relaxed.gpu.global.v2.b64 [%0], {%1, %2};" ::"l"(p), "l"(x), "l"(y) : "memory");
}
__device__ __forceinline__ void tell_state(uint32_t* p, float2 s) {
    asm volatile("st.relaxed.gpu.global.v2.b32 [%0], {%1, %2};" ::"l"(p), "r"(told(s.x)), "r"(told(s.y)) : "memory");
}
// The waits are bounded: one that runs out is counted and answers NaN. Tiles
// take tickets in the order of their dependences, so what a tile waits for
// comes from blocks that are running or done.
__device__ __forceinline__ Map hear_map(const uint64_t* p) {
    uint64_t x, y;
    for (int i = 0; i < kSpinLimit; ++i) {
        asm volatile("ld.relaxed.gpu.global.v2.b64 {%0, %1}, [%2];" : "=l"(x), "=l"(y) : "l"(p) : "memory");
        if ((x >> 32) != 0xffffffffu && (y >> 32) != 0xffffffffu)
            return {make_float2(__uint_as_float(x >> 32), __uint_as_float(y >> 32)), make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)y))};
    }
    atomicAdd(&wait_timeouts, 1ull);
    const float nan = __uint_as_float(0x7fffffffu);
    return {make_float2(nan, nan), make_float2(nan, nan)};
}
__device__ __forceinline__ float2 hear_state(const uint32_t* p) {
    uint32_t x, y;
    for (int i = 0; i < kSpinLimit; ++i) {
        asm volatile("ld.relaxed.gpu.global.v2.b32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "l"(p) : "memory");
        if (x != 0xffffffffu && y != 0xffffffffu) return make_float2(__uint_as_float(x), __uint_as_float(y));
    }
    atomicAdd(&wait_timeouts, 1ull);
    return make_float2(__uint_as_float(0x7fffffffu), __uint_as_float(0x7fffffffu));
}

// The state before the `order`-th tile of a sequence, counted from where the
// scan starts; tile_at(i) is the i-th tile's index, `start` the scan's first
// state. The group's earlier tiles are heard by all warps, two each, and the
// group before by the last one; the maps are applied in the scan's order, so
// the result does not depend on which tile was ready when.
template <typename TileAt>
__device__ __forceinline__ float2 state_before(const Exchange& x, int64_t b, int channel, int order, TileAt tile_at, float2 start,
                                               Map (*maps)[32], float2* state) {
    constexpr int kEach = kGroup / kWarps;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, first = order - order % kGroup, group = order / kGroup;
    Map m{make_float2(1.f, 1.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = first + warp * kEach + i;
        if (at < order) m = then(m, hear_map(x.maps + ((int64_t)b * x.tiles + tile_at(at)) * x.channels + channel));
    }
    maps[warp][lane] = m;
    if (warp == kWarps - 1)
        state[lane] = group > 0 ? hear_state(x.states + ((int64_t)b * x.groups + group - 1) * x.channels + channel) : start;
    __syncthreads();
    float2 s = state[lane];
    const int heard = (order - first + kEach - 1) / kEach;
    for (int i = 0; i < heard; ++i) s = apply(maps[i][lane], s);
    return s;
}

// The block's place: tiles in the order of the scan, all sequences and
// channels of one before the next.
struct Place {
    int order, channel;
    int64_t b;
};
__device__ __forceinline__ Place take_place(const Exchange& x, int columns) {
    __shared__ unsigned ticket;
    unsigned id = blockIdx.x;
    if (x.tiles > 1) {
        if (threadIdx.x == 0) ticket = atomicAdd(x.ticket, 1u) + 1u;  // from all ones
        __syncthreads();
        id = ticket;
    }
    const int per = x.channels / kChannels, c = id % columns;
    return {static_cast<int>(id / columns), c % per * kChannels + static_cast<int>(threadIdx.x % 32) * 2, c / per};
}

// Forward pass: one block per tile of kForwardTile steps and 64 channels, R
// steps of a pair of channels per thread, read once and kept in registers. A
// tile's steps compose to one map of the state; the warps exchange theirs in
// shared memory, the tiles through `x`, and with the state before its steps
// each thread runs through them again.
template <typename T, bool PAIR>
__global__ void __launch_bounds__(kWarps * 32, 2)
recurrence_kernel(SeqIn gate, SeqIn value, int64_t steps, int D, const float* h0, const int32_t* lengths, T* h, float* h_last,
                  float* carry, Exchange x, int columns) {
    layer_begin();
    constexpr int R = kForwardSteps;
    __shared__ Map own[kWarps][32], heard[kWarps][32];
    __shared__ float2 state[32];
    const Place at = take_place(x, columns);
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = at.channel;
    const bool live = c < D, second = c + 1 < D;
    const int64_t n = length_of(lengths, at.b, steps), tile0 = (int64_t)at.order * kForwardTile, t0 = tile0 + warp * R;
    const int inside = static_cast<int>(min(max(n - t0, (int64_t)0), (int64_t)R));  // of the thread's steps
    const int written = static_cast<int>(min(max(steps - t0, (int64_t)0), (int64_t)R));
    T* out = h + (at.b * steps + t0) * D + c;
    if (tile0 >= n && at.order > 0) {  // wholly beyond the length: nothing to hear or to tell
        if (live)
            for (int r = 0; r < written; ++r) store_two<PAIR>(out + (int64_t)r * D, make_float2(0.f, 0.f), second);
        return;
    }
    // whether all steps and channels of the warp are there: no tests in the loops then
    const bool whole_warp = inside == R && c - 2 * lane + kChannels <= D;
    float2 a[R], u[R];
    const auto load = [&](auto known) {
        constexpr bool ALL = decltype(known)::value;
        Two<T> graw[R], vraw[R];
        const T* g = static_cast<const T*>(gate.p) + at.b * gate.seq + t0 * gate.step + c;
        const T* v = static_cast<const T*>(value.p) + at.b * value.seq + t0 * value.step + c;
#pragma unroll
        for (int r = 0; r < R; ++r, g += gate.step, v += value.step)
            if (ALL || (live && r < inside)) {
                graw[r] = load_two<PAIR>(g, ALL || second);
                vraw[r] = load_two<PAIR>(v, ALL || second);
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            a[r] = make_float2(1.f, 1.f);
            u[r] = make_float2(0.f, 0.f);
            if (ALL || (live && r < inside)) {
                const float2 gr = graw[r].get(), vr = vraw[r].get();
                float2 rest;
                gate_of(gr.x, a[r].x, rest.x);
                gate_of(gr.y, a[r].y, rest.y);
                u[r] = make_float2(rest.x * vr.x, rest.y * vr.y);
            }
        }
    };
    if (whole_warp)
        load(std::true_type{});
    else
        load(std::false_type{});
    Map m{a[0], u[0]};
#pragma unroll
    for (int r = 1; r < R; ++r) m = then(m, Map{a[r], u[r]});
    own[warp][lane] = m;
    __syncthreads();
    const bool more = n > tile0 + kForwardTile;  // a later tile has steps
    Map whole = own[0][lane];
    if (more && warp == 0) {
        for (int i = 1; i < kWarps; ++i) whole = then(whole, own[i][lane]);
        tell_map(x.maps + (at.b * x.tiles + at.order) * x.channels + c, whole);
    }
    const float2 start = h0 != nullptr && live ? make_float2(h0[at.b * D + c], second ? h0[at.b * D + c + 1] : 0.f) : make_float2(0.f, 0.f);
    float2 s = start;
    if (at.order > 0) s = state_before(x, at.b, c, at.order, [](int i) { return i; }, start, heard, state);
    if (more && warp == 0 && at.order % kGroup == kGroup - 1)
        tell_state(x.states + (at.b * x.groups + at.order / kGroup) * x.channels + c, apply(whole, s));
    for (int i = 0; i < warp; ++i) s = apply(own[i][lane], s);
    if (!live) return;
    if (carry != nullptr && inside > 0 && t0 % CPDP_CARRY_STEPS == 0) {
        const int64_t carries = (steps + CPDP_CARRY_STEPS - 1) / CPDP_CARRY_STEPS;
        store_two<false>(carry + (at.b * carries + t0 / CPDP_CARRY_STEPS) * D + c, s, second);
    }
    const bool last = inside > 0 && t0 + inside == n;
    if (n == 0 && warp == 0) store_two<false>(h_last + at.b * D + c, start, second);
    if (whole_warp) {
#pragma unroll
        for (int r = 0; r < R; ++r, out += D) {
            s = apply(Map{a[r], u[r]}, s);
            store_two<PAIR>(out, s, true);
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r, out += D) {
            s = apply(Map{a[r], u[r]}, s);  // beyond the length the identity
            if (r < written) store_two<PAIR>(out, r < inside ? s : make_float2(0.f, 0.f), second);
        }
    }
    if (last) store_two<false>(h_last + at.b * D + c, s, second);
}

// Backward pass, tiles of kBackwardTile steps from the last to the first. What
// flows from step t to t - 1 is f_t = a_t (dh_t + f_(t+1)), a map like the
// state's, scanned the other way. The states inside the tile are made again
// from the carry at its first step: reading the stored h would bring its
// rounding into dgate, and more bytes.
template <typename T, bool PAIR>
__global__ void __launch_bounds__(kWarps * 32, 2)
recurrence_backward_kernel(SeqIn dh, SeqIn gate, SeqIn value, int64_t steps, int D, const float* carry, const float* dh_last,
                           const int32_t* lengths, T* dgate, T* dvalue, int64_t grad_seq, int64_t grad_step, float* dh0, Exchange x,
                           int columns) {
    layer_begin();
    constexpr int R = kBackwardSteps;
    __shared__ Map own[kWarps][32], heard[kWarps][32];
    __shared__ float2 flows[kWarps][32], state[32];
    const Place at = take_place(x, columns);
    const int tile = x.tiles - 1 - at.order;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = at.channel;
    const bool live = c < D, second = c + 1 < D;
    const int64_t n = length_of(lengths, at.b, steps), tile0 = (int64_t)tile * kBackwardTile, t0 = tile0 + warp * R;
    const int inside = static_cast<int>(min(max(n - t0, (int64_t)0), (int64_t)R));
    const int written = static_cast<int>(min(max(steps - t0, (int64_t)0), (int64_t)R));
    const int64_t first_out = at.b * grad_seq + t0 * grad_step + c;
    if (tile0 >= n && tile > 0) {
        if (live)
            for (int r = 0; r < written; ++r) {
                store_two<PAIR>(dgate + first_out + r * grad_step, make_float2(0.f, 0.f), second);
                store_two<PAIR>(dvalue + first_out + r * grad_step, make_float2(0.f, 0.f), second);
            }
        return;
    }
    const bool whole_warp = inside == R && c - 2 * lane + kChannels <= D;
    Two<T> vraw[R], oraw[R];
    float2 a[R], rest[R];
    const auto load = [&](auto known) {
        constexpr bool ALL = decltype(known)::value;
        Two<T> graw[R];
        const T* g = static_cast<const T*>(gate.p) + at.b * gate.seq + t0 * gate.step + c;
        const T* v = static_cast<const T*>(value.p) + at.b * value.seq + t0 * value.step + c;
        const T* o = static_cast<const T*>(dh.p) + at.b * dh.seq + t0 * dh.step + c;
#pragma unroll
        for (int r = 0; r < R; ++r, g += gate.step, v += value.step, o += dh.step) {
            if (!ALL) vraw[r] = oraw[r] = Two<T>{};
            if (ALL || (live && r < inside)) {
                graw[r] = load_two<PAIR>(g, ALL || second);
                vraw[r] = load_two<PAIR>(v, ALL || second);
                oraw[r] = load_two<PAIR>(o, ALL || second);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            a[r] = make_float2(1.f, 1.f);
            rest[r] = make_float2(0.f, 0.f);
            if (ALL || (live && r < inside)) {
                const float2 gr = graw[r].get();
                gate_of(gr.x, a[r].x, rest[r].x);
                gate_of(gr.y, a[r].y, rest[r].y);
            }
        }
    };
    if (whole_warp)
        load(std::true_type{});
    else
        load(std::false_type{});
    // the thread's steps as a map of the state (forwards) and of the flow (backwards)
    Map m{make_float2(1.f, 1.f), make_float2(0.f, 0.f)};
    float2 flow = make_float2(0.f, 0.f);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float2 v = vraw[r].get();
        m = then(m, Map{a[r], make_float2(rest[r].x * v.x, rest[r].y * v.y)});
    }
#pragma unroll
    for (int r = R - 1; r >= 0; --r) {
        const float2 o = oraw[r].get();
        flow = make_float2(a[r].x * (o.x + flow.x), a[r].y * (o.y + flow.y));
    }
    own[warp][lane] = m;
    flows[warp][lane] = flow;
    __syncthreads();
    const int last_tile = n > 0 ? static_cast<int>((n - 1) / kBackwardTile) : 0, order = last_tile - tile;
    Map whole{own[kWarps - 1][lane].a, flows[kWarps - 1][lane]};
    if (tile > 0 && warp == 0) {
        for (int i = kWarps - 2; i >= 0; --i) whole = then(whole, Map{own[i][lane].a, flows[i][lane]});
        tell_map(x.maps + (at.b * x.tiles + tile) * x.channels + c, whole);
    }
    const float2 start = dh_last != nullptr && live ? make_float2(dh_last[at.b * D + c], second ? dh_last[at.b * D + c + 1] : 0.f)
                                                    : make_float2(0.f, 0.f);
    flow = start;
    if (order > 0) flow = state_before(x, at.b, c, order, [=](int i) { return last_tile - i; }, start, heard, state);
    if (tile > 0 && warp == 0 && order % kGroup == kGroup - 1)
        tell_state(x.states + (at.b * x.groups + order / kGroup) * x.channels + c, apply(whole, flow));
    if (!live) return;
    float2 s = make_float2(0.f, 0.f);
    if (n > 0) {
        const int64_t carries = (steps + CPDP_CARRY_STEPS - 1) / CPDP_CARRY_STEPS;
        const float* p = carry + (at.b * carries + tile) * D + c;
        s = make_float2(p[0], second ? p[1] : 0.f);
    }
    for (int i = 0; i < warp; ++i) s = apply(own[i][lane], s);
    for (int i = kWarps - 1; i > warp; --i) flow = apply(Map{own[i][lane].a, flows[i][lane]}, flow);
    float2 away[R];  // h_(t-1) - v_t
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float2 v = vraw[r].get();
        away[r] = make_float2(s.x - v.x, s.y - v.y);
        s = apply(Map{a[r], make_float2(rest[r].x * v.x, rest[r].y * v.y)}, s);
    }
    const auto finish = [&](auto known) {
        constexpr bool ALL = decltype(known)::value;
        T *dg = dgate + first_out + (R - 1) * grad_step, *dv = dvalue + first_out + (R - 1) * grad_step;
#pragma unroll
        for (int r = R - 1; r >= 0; --r, dg -= grad_step, dv -= grad_step) {
            const float2 o = oraw[r].get(), g = make_float2(o.x + flow.x, o.y + flow.y);
            flow = make_float2(a[r].x * g.x, a[r].y * g.y);
            const bool in = ALL || r < inside;
            if (ALL || r < written) {
                const float2 x = make_float2(rest[r].x * g.x, rest[r].y * g.y), zero = make_float2(0.f, 0.f);
                store_two<PAIR>(dv, in ? x : zero, ALL || second);
                store_two<PAIR>(dg, in ? make_float2(x.x * away[r].x * a[r].x, x.y * away[r].y * a[r].y) : zero, ALL || second);
            }
        }
    };
    if (whole_warp)
        finish(std::true_type{});
    else
        finish(std::false_type{});
    if (dh0 != nullptr && tile == 0 && warp == 0) store_two<false>(dh0 + at.b * D + c, flow, second);
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

// The workspace: a ticket, then the tiles' maps, then the groups' states.
static size_t lay_out(int B, int64_t T, int D, int tile, void* workspace, Exchange* x) {
    const int64_t tiles = ceil_div(T, tile), groups = ceil_div(tiles, kGroup), channels = ceil_div(D, kChannels) * kChannels;
    const int64_t maps = B * tiles * channels, states = B * groups * channels;
    if (x != nullptr) {
        char* p = static_cast<char*>(workspace);
        *x = Exchange{reinterpret_cast<unsigned*>(p), reinterpret_cast<uint64_t*>(p + 16),
                      reinterpret_cast<uint32_t*>(p + 16 + 8 * maps), (int)tiles, (int)groups, (int)channels};
    }
    return tiles > 1 && B > 0 ? static_cast<size_t>(16 + 8 * maps + 4 * states) : 0;
}

size_t cpdp_gated_recurrence_workspace(int B, int64_t T, int D) {
    if (check_recurrence(B, T, D, CPDP_F32) != CPDP_OK) return 0;
    return lay_out(B, T, D, kBackwardTile, nullptr, nullptr);
}

cpdp_status cpdp_layer_timeouts(int64_t* count) {
    if (count == nullptr) return layer_error(CPDP_EINVAL, "count is NULL");
    unsigned long long seen = 0, zero = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&seen, wait_timeouts, sizeof seen);
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(wait_timeouts, &zero, sizeof zero);
    unsigned long long others = 0;
    if (e == cudaSuccess) e = take_weight_gradient_timeouts(&others);
    *count = static_cast<int64_t>(seen + others);
    return layer_launched(e, "cpdp_layer_timeouts");
}

// The exchange of one pass, its words set to "not there yet".
static cpdp_status begin_exchange(int B, int64_t T, int D, int tile, void* workspace, size_t workspace_bytes, void* stream, Exchange* x) {
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_gated_recurrence_workspace(B, T, D)));
    const size_t used = lay_out(B, T, D, tile, workspace, x);
    const int64_t blocks = int64_t(x->tiles > 0 ? x->tiles : 1) * B * (x->channels / kChannels);
    if (blocks > kLayerMaxRows)
        return layer_error(CPDP_EINVAL, "B=%d, T=%lld, D=%d: more than 2^31 - 1 blocks", B, (long long)T, D);
    if (used > 0) return layer_launched(cudaMemsetAsync(workspace, 0xff, used, static_cast<cudaStream_t>(stream)), "setting the workspace");
    return CPDP_OK;
}

static unsigned blocks_of(const Exchange& x, int B) {
    return static_cast<unsigned>(x.tiles > 0 ? x.tiles : 1) * B * (x.channels / kChannels);
}

// Whether pairs of channels can be moved as one: D even, and every array's
// pointer and strides in whole pairs.
static bool even(const void* p, int64_t size, int64_t a, int64_t b) { return aligned_to(p, 2 * size) && a % 2 == 0 && b % 2 == 0; }

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
    Exchange x;
    if (B == 0) return CPDP_OK;
    CPDP_TRY(begin_exchange(B, T, D, kForwardTile, workspace, workspace_bytes, stream, &x));
    const SeqIn g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const bool pair = D % 2 == 0 && even(gate, e, gate_seq, gate_step) && even(value, e, value_seq, value_step) && even(h, e, 0, 0);
    const unsigned blocks = blocks_of(x, B);
    const auto go = [&](auto kernel, auto* out) {
        return launch_layer(kernel, blocks, kWarps * 32, 0, stream, g, v, T, D, h0, lengths, out, h_last, carry, x,
                            B * (x.channels / kChannels));
    };
    const auto typed = [&](auto* out) {
        using E = std::remove_pointer_t<decltype(out)>;
        return pair ? go(recurrence_kernel<E, true>, out) : go(recurrence_kernel<E, false>, out);
    };
    return layer_launched(dtype == CPDP_F32 ? typed(static_cast<float*>(h)) : typed(static_cast<__nv_bfloat16*>(h)), "cpdp_gated_recurrence");
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
    Exchange x;
    if (B == 0) return CPDP_OK;
    CPDP_TRY(begin_exchange(B, T, D, kBackwardTile, workspace, workspace_bytes, stream, &x));
    if (x.tiles == 0) x.tiles = 1;  // no steps: one tile passes dh_last on to dh0
    const SeqIn o{dh, dh_seq, dh_step}, g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const bool pair = D % 2 == 0 && even(dh, e, dh_seq, dh_step) && even(gate, e, gate_seq, gate_step) &&
                      even(value, e, value_seq, value_step) && even(dgate, e, grad_seq, grad_step) && even(dvalue, e, 0, 0);
    const unsigned blocks = blocks_of(x, B);
    const auto go = [&](auto kernel, auto* dg, auto* dv) {
        return launch_layer(kernel, blocks, kWarps * 32, 0, stream, o, g, v, T, D, carry, dh_last, lengths, dg, dv, grad_seq, grad_step,
                            dh0, x, B * (x.channels / kChannels));
    };
    const auto typed = [&](auto* dg, auto* dv) {
        using E = std::remove_pointer_t<decltype(dg)>;
        return pair ? go(recurrence_backward_kernel<E, true>, dg, dv) : go(recurrence_backward_kernel<E, false>, dg, dv);
    };
    return layer_launched(dtype == CPDP_F32 ? typed(static_cast<float*>(dgate), static_cast<float*>(dvalue))
                                            : typed(static_cast<__nv_bfloat16*>(dgate), static_cast<__nv_bfloat16*>(dvalue)),
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
