// The gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) v_t, its backward
// pass and its single step (include/cpdp_layers.h).
#include <type_traits>

#include "cpdp_gates.cuh"

namespace cpdp {
namespace {

constexpr int kThreads = 128;       // of the single step's kernel
constexpr int kWarps = 4;           // per block of the scans where they work together
constexpr int kChannels = 64;       // per warp: two per lane
constexpr int R = CPDP_CARRY_STEPS; // steps of a chunk
// Slots of a warp's ring of chunks, and the warps per SM that registers and
// shared memory then allow: 8 warps with two chunks each in flight reach the
// memory's rate.
constexpr int kForwardRing = 3;
template <typename T>
constexpr int kBackwardRing = sizeof(T) == 2 ? 3 : 2;
template <typename T>
constexpr int kForwardWarps = sizeof(T) == 2 ? 16 : 8;
template <typename T>
constexpr int kBackwardWarps = sizeof(T) == 2 ? 12 : 8;

struct SeqIn {
    const void* p;
    int64_t seq, step;
};

// A lane's two channels. WIDE, where every row starts at a multiple of 16
// bytes: neighbours, moved together. Else 32 apart, moved one by one, each with
// the other lanes' next to it.
template <bool WIDE>
__device__ __forceinline__ int first_channel(int lane) { return WIDE ? 2 * lane : lane; }
template <bool WIDE>
constexpr int kSecond = WIDE ? 1 : 32;

__device__ __forceinline__ Pair pair_at(const float* p) { return *reinterpret_cast<const Pair*>(p); }
__device__ __forceinline__ Pair pair_at(const __nv_bfloat16* p) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    return pair(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <bool WIDE>
__device__ __forceinline__ void store_two(float* p, Pair both, bool second) {
    const float2 v = floats(both);
    if (WIDE) {
        *reinterpret_cast<Pair*>(p) = both;
    } else {
        p[0] = v.x;
        if (second) p[32] = v.y;
    }
}
template <bool WIDE>
__device__ __forceinline__ void store_two(__nv_bfloat16* p, Pair both, bool second) {
    const float2 v = floats(both);
    if (WIDE) {
        *reinterpret_cast<__nv_bfloat162*>(p) = __float22bfloat162_rn(v);
    } else {
        p[0] = __float2bfloat16_rn(v.x);
        if (second) p[32] = __float2bfloat16_rn(v.y);
    }
}
// Two float32 channels that need not be aligned.
template <bool WIDE>
__device__ __forceinline__ Pair load_state(const float* p, bool second) { return pair(p[0], second ? p[kSecond<WIDE>] : 0.f); }
template <bool WIDE>
__device__ __forceinline__ void store_state(float* p, Pair s, bool second) {
    const float2 v = floats(s);
    p[0] = v.x;
    if (second) p[kSecond<WIDE>] = v.y;
}

// x -> a x + b for two channels, and one such map after another.
struct alignas(16) Map {
    Pair a, b;
};
constexpr Map kSame{kOnes, kZeros};
__device__ __forceinline__ Pair apply(const Map& m, Pair x) { return fma2(m.a, x, m.b); }
__device__ __forceinline__ Map then(const Map& first, const Map& second) {
    return {mul2(second.a, first.a), apply(second, first.b)};
}

// How the scans are shared out. A warp takes 64 channels of a sequence (a
// column) and walks a segment of its steps, the state in registers. Where
// there are columns enough, a segment is the whole sequence. Else the steps are
// split into `count` segments (1, 2 or a multiple of 4) of `steps` (a
// multiple of R): a first pass makes each segment's map of the state, a second
// one composes the maps before its segment and walks. `order` counts segments
// from where the scan starts.
struct Segments {
    int count, steps, groups;  // groups of channels per sequence
    int64_t columns;
    Map* maps;                 // [columns][count][32 lanes]
};
struct Task {
    int64_t column;
    int b, channel, order;
};
__device__ __forceinline__ Task task_of(const Segments& x) {
    const int64_t i = (int64_t)blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32, column = i / x.count;
    const int b = static_cast<int>(column / x.groups);
    return {column, b, static_cast<int>(column - (int64_t)b * x.groups) * kChannels, static_cast<int>(i - column * x.count)};
}

// The state before the task's segment: the maps of the segments before it
// applied to `start`, in an order fixed by their number. Those before the
// block's first are composed by its warps together.
__device__ __forceinline__ Pair state_before(const Segments& x, const Task& task, Pair start) {
    __shared__ Map parts[kWarps][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, first = x.count >= kWarps ? task.order - warp : 0;
    const Map* maps = x.maps + task.column * x.count * 32 + lane;
    Pair s = start;
    if (first > 0) {  // the same for all warps of the block
        const int each = (first + kWarps - 1) / kWarps, end = min(first, (warp + 1) * each);
        Map m = kSame;
#pragma unroll 8
        for (int i = warp * each; i < end; ++i) m = then(m, maps[i * 32]);
        parts[warp][lane] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWarps; ++i) s = apply(parts[i][lane], s);
    }
#pragma unroll 8
    for (int i = first; i < task.order; ++i) s = apply(maps[i * 32], s);
    return s;
}

// A chunk of R steps of the warp's channels, brought by asynchronous 16-byte
// copies into the warp's ring in shared memory, some chunks before its use.
// Where rows do not start at multiples of 16 bytes, the copies start at the
// multiple before (the same 16 bytes hold the row's first element), and a row
// has its first element that much further in its slot.
template <typename T, bool WIDE>
constexpr int kRowBytes = kChannels * sizeof(T) + (WIDE ? 0 : 16);
template <typename T, bool WIDE>
constexpr int kChunkBytes = R * kRowBytes<T, WIDE>;

__device__ __forceinline__ void copy_16(uint32_t to, const void* from, int bytes) {  // the rest of the 16 is set to 0
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
template <typename T, bool WIDE>
__device__ __forceinline__ void fill(uint8_t* to, const T* from, int64_t step, int rows, int channels) {
    const int lane = threadIdx.x % 32;
    const uint32_t slot = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if constexpr (WIDE) {
        constexpr int each = 16 / sizeof(T), per_row = kChannels / each, down = 32 / per_row;  // rows per round
        const int c = lane % per_row * each, r0 = lane / per_row;
        const bool there = c < channels;
        const T* p = from + r0 * step + c;
        const uint32_t at = slot + (r0 * kChannels + c) * sizeof(T);
#pragma unroll
        for (int k = 0; k < R / down; ++k, p += down * step) {
            const bool here = there && r0 + k * down < rows;
            copy_16(at + k * down * kRowBytes<T, true>, here ? p : from, here ? 16 : 0);
        }
    } else {
        constexpr int per_row = kRowBytes<T, false> / 16, all = R * per_row;
        const int width = min(channels, kChannels) * static_cast<int>(sizeof(T));
#pragma unroll
        for (int k = 0; k < (all + 31) / 32; ++k) {
            const int i = k * 32 + lane, r = i / per_row, piece = i % per_row;
            if (k * 32 + 32 > all && i >= all) break;
            const uintptr_t row = reinterpret_cast<uintptr_t>(from + min(r, rows - 1) * step), first = (row & ~uintptr_t(15)) + piece * 16;
            const int bytes = r < rows ? static_cast<int>(min(max((int64_t)(row + width - first), (int64_t)0), (int64_t)16)) : 0;
            copy_16(slot + i * 16, reinterpret_cast<const void*>(bytes > 0 ? first : row & ~uintptr_t(15)), bytes);
        }
    }
}
__device__ __forceinline__ void end_fill() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LATER>
__device__ __forceinline__ void wait_filled() {
    asm volatile("cp.async.wait_group %0;" ::"n"(LATER) : "memory");
    __syncwarp();
}

// The lane's channels of a chunk in its slot.
template <typename T, bool WIDE>
struct Chunk {
    const uint8_t* slot;
    uint32_t shift, each;  // of the first row, and from row to row
    __device__ __forceinline__ Chunk(const uint8_t* at, const T* from, int64_t step)
        : slot(at + first_channel<WIDE>(threadIdx.x % 32) * sizeof(T)), shift(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(from))),
          each(static_cast<uint32_t>(step) * sizeof(T)) {}
    __device__ __forceinline__ Pair get(int r) const {
        if constexpr (WIDE) {
            return pair_at(reinterpret_cast<const T*>(slot + r * kRowBytes<T, true>));
        } else {
            const T* p = reinterpret_cast<const T*>(slot + r * kRowBytes<T, false> + ((shift + r * each) & 15u));
            return pair(to_float(p[0]), to_float(p[32]));
        }
    }
};

// Forward pass: chunks of R steps pass through the warp's ring of shared
// memory; the only chain from step to step is one fused multiply-add.
// MAPS: the first pass, which makes the segment's map. In bf16, 64 x 1,024 x
// 1,024 (1,024 columns) take 72 us, 5.6 TB/s, 16 instructions per element;
// 65,536 x 1,024 (16 columns in 152 segments) 45 us for the maps and 64 for the
// rest, both at 6 TB/s of what they read and write. With fewer than 8 warps per
// SM the chunks' latency shows: 128 x 197 x 384 (5 warps) 18 us, 3.2 TB/s.
template <typename T, bool WIDE, bool MAPS>
__global__ void __launch_bounds__(kWarps * 32, kForwardWarps<T> / kWarps)
recurrence_kernel(SeqIn gate, SeqIn value, int steps, int D, const float* h0, const int32_t* lengths, T* h, float* h_last,
                  float* carry, Segments x) {
    layer_begin();
    constexpr int kRing = kForwardRing, kChunk = kChunkBytes<T, WIDE>;
    extern __shared__ __align__(16) uint8_t inputs[];
    const int lane = threadIdx.x % 32;
    uint8_t* const ring = inputs + threadIdx.x / 32 * (kRing * 2 * kChunk);
    const Task task = task_of(x);
    if (task.column >= x.columns) return;
    if (MAPS && task.order == x.count - 1) return;  // nobody asks for the last one
    const int c = task.channel + first_channel<WIDE>(lane), n = lengths == nullptr ? steps : min(max(lengths[task.b], 0), steps);
    const int first = task.order * x.steps, end = min(first + x.steps, steps), inside = min(max(n - first, 0), end - first);
    const bool live = c < D, second = c + kSecond<WIDE> < D;
    const T* g = static_cast<const T*>(gate.p) + task.b * gate.seq + first * gate.step + task.channel;
    const T* v = static_cast<const T*>(value.p) + task.b * value.seq + first * value.step + task.channel;
    const auto fetch = [&](int k) {
        const int t = k * R;
        if (t < inside) {
            uint8_t* to = ring + k % kRing * (2 * kChunk);
            fill<T, WIDE>(to, g + t * gate.step, gate.step, inside - t, D - task.channel);
            fill<T, WIDE>(to + kChunk, v + t * value.step, value.step, inside - t, D - task.channel);
        }
        end_fill();
    };
#pragma unroll
    for (int k = 0; k < kRing - 1; ++k) fetch(k);
    Pair s = kZeros;
    Map m = kSame;
    if constexpr (!MAPS) {
        if (h0 != nullptr && live) s = load_state<WIDE>(h0 + (int64_t)task.b * D + c, second);
        if (x.count > 1) s = state_before(x, task, s);
    }
    T* out = h + ((int64_t)task.b * steps + first) * D + c;
    float* carries = carry + ((int64_t)task.b * ((steps + R - 1) / R) + first / R) * D + c;
    for (int k = 0; k * R < inside; ++k) {
        const int t = k * R, rows = inside - t;
        wait_filled<kRing - 2>();
        fetch(k + kRing - 1);  // into the slot of the chunk before
        const uint8_t* slot = ring + k % kRing * (2 * kChunk);
        const Chunk<T, WIDE> gs(slot, g + t * gate.step, gate.step), vs(slot + kChunk, v + t * value.step, value.step);
        if (!MAPS && carry != nullptr && live) {
            store_two<WIDE>(carries, s, second);
            carries += D;
        }
        // FULL: all R steps are inside. Else those beyond are the identity; a
        // break there would leave nothing to overlap, 250 clocks a step.
        const auto walk = [&](auto known) {
            constexpr bool FULL = decltype(known)::value;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                Map one;
                Pair rest;
                gate_of<T>(gs.get(r), one.a, rest);
                one.b = mul2(rest, vs.get(r));
                if (!FULL && r >= rows) one = kSame;
                if constexpr (MAPS) {
                    m = then(m, one);
                } else {
                    s = apply(one, s);
                    if (live && (FULL || r < rows)) store_two<WIDE>(out + (int64_t)r * D, s, second);
                }
            }
            out += (int64_t)min(rows, R) * D;
        };
        if (rows >= R)
            walk(std::true_type{});
        else
            walk(std::false_type{});
        __syncwarp();
    }
    if constexpr (MAPS) {
        x.maps[(task.column * x.count + task.order) * 32 + lane] = m;
    } else if (live) {
        for (int t = inside; t < end - first; ++t, out += D) store_two<WIDE>(out, kZeros, second);
        if (n > first ? n <= end : n == 0 && first == 0) store_state<WIDE>(h_last + (int64_t)task.b * D + c, s, second);
    }
}

// Backward pass, from the last step to the first. What flows from step t to
// t - 1 is f_t = a_t (dh_t + f_(t+1)), a map like the state's. The states
// inside a chunk are made again from the carry at its first step: reading the
// stored h would bring its rounding into dgate, and more bytes. The same sizes
// as above: 115 us, 5.8 TB/s; 42 and 110; 27 us, 3.6 TB/s. Blocks of fewer
// registers, 16 warps per SM, spilled and took twice as long.
template <typename T, bool WIDE, bool MAPS>
__global__ void __launch_bounds__(kWarps * 32, kBackwardWarps<T> / kWarps)
recurrence_backward_kernel(SeqIn dh, SeqIn gate, SeqIn value, int steps, int D, const float* carry, const float* dh_last,
                           const int32_t* lengths, T* dgate, T* dvalue, int64_t grad_seq, int64_t grad_step, float* dh0, Segments x) {
    layer_begin();
    constexpr int kRing = kBackwardRing<T>, kChunk = kChunkBytes<T, WIDE>, kArrays = MAPS ? 2 : 3;
    extern __shared__ __align__(16) uint8_t inputs[];
    const int lane = threadIdx.x % 32;
    uint8_t* const ring = inputs + threadIdx.x / 32 * (kRing * kArrays * kChunk);
    const Task task = task_of(x);
    if (task.column >= x.columns) return;
    if (MAPS && task.order == x.count - 1) return;
    const int c = task.channel + first_channel<WIDE>(lane), n = lengths == nullptr ? steps : min(max(lengths[task.b], 0), steps);
    const int first = (x.count - 1 - task.order) * x.steps, end = min(first + x.steps, steps), inside = min(max(n - first, 0), max(end - first, 0));
    const bool live = c < D, second = c + kSecond<WIDE> < D, all_channels = task.channel + kChannels <= D;
    const T* g = static_cast<const T*>(gate.p) + task.b * gate.seq + first * gate.step + task.channel;
    const T* v = static_cast<const T*>(value.p) + task.b * value.seq + first * value.step + task.channel;
    const T* o = static_cast<const T*>(dh.p) + task.b * dh.seq + first * dh.step + task.channel;
    const int chunks = (inside + R - 1) / R;
    const auto fetch = [&](int i) {  // the i-th chunk from the end
        const int t = (chunks - 1 - i) * R;
        if (i < chunks) {
            uint8_t* to = ring + i % kRing * (kArrays * kChunk);
            fill<T, WIDE>(to, g + t * gate.step, gate.step, inside - t, D - task.channel);
            fill<T, WIDE>(to + kChunk, o + t * dh.step, dh.step, inside - t, D - task.channel);
            if constexpr (!MAPS) fill<T, WIDE>(to + 2 * kChunk, v + t * value.step, value.step, inside - t, D - task.channel);
        }
        end_fill();
    };
#pragma unroll
    for (int i = 0; i < kRing - 1; ++i) fetch(i);
    Pair flow = kZeros;
    Map m = kSame;
    if constexpr (!MAPS) {
        if (dh_last != nullptr && live) flow = load_state<WIDE>(dh_last + (int64_t)task.b * D + c, second);
        if (x.count > 1) flow = state_before(x, task, flow);
    }
    const int64_t out0 = task.b * grad_seq + first * grad_step + c;
    if (!MAPS && live)
        for (int64_t t = inside; t < end - first; ++t) {
            store_two<WIDE>(dgate + out0 + t * grad_step, kZeros, second);
            store_two<WIDE>(dvalue + out0 + t * grad_step, kZeros, second);
        }
    const float* carries = carry + ((int64_t)task.b * ((steps + R - 1) / R) + first / R) * D + c;
    for (int i = 0; i < chunks; ++i) {
        const int t = (chunks - 1 - i) * R, rows = inside - t;
        Pair s = kZeros;
        if (!MAPS && live) {
            const float* p = carries + (int64_t)(t / R) * D;
            s = load_state<WIDE>(p, second);
        }
        wait_filled<kRing - 2>();
        fetch(i + kRing - 1);
        const uint8_t* slot = ring + i % kRing * (kArrays * kChunk);
        const Chunk<T, WIDE> gs(slot, g + t * gate.step, gate.step), os(slot + kChunk, o + t * dh.step, dh.step),
            vs(slot + 2 * kChunk, v + t * value.step, value.step);
        const auto walk = [&](auto known, auto every) {
            constexpr bool FULL = decltype(known)::value;
            if constexpr (MAPS) {
#pragma unroll
                for (int r = R - 1; r >= 0; --r) {
                    Pair a, rest;
                    gate_of<T>(gs.get(r), a, rest);
                    if (!FULL && r >= rows) a = kOnes;  // dh is 0 there
                    m = Map{mul2(a, m.a), mul2(a, add2(os.get(r), m.b))};
                }
            } else {
                constexpr bool ALL = FULL && decltype(every)::value;
                Pair a[R], rest[R], away[R];  // away: (h_(t-1) - v_t) a_t
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    gate_of<T>(gs.get(r), a[r], rest[r]);
                    if (!FULL && r >= rows) a[r] = kOnes, rest[r] = kZeros;
                    const Pair vr = vs.get(r);
                    away[r] = mul2(fma2(vr, kMinusOnes, s), a[r]);
                    s = fma2(a[r], s, mul2(rest[r], vr));
                }
                T *dg = dgate + out0 + (t + R - 1) * grad_step, *dv = dvalue + out0 + (t + R - 1) * grad_step;
#pragma unroll
                for (int r = R - 1; r >= 0; --r, dg -= grad_step, dv -= grad_step) {
                    const Pair both = add2(os.get(r), flow), y = mul2(rest[r], both);
                    flow = mul2(a[r], both);
                    if (ALL || (live && (FULL || r < rows))) {
                        store_two<WIDE>(dv, y, second);
                        store_two<WIDE>(dg, mul2(y, away[r]), second);
                    }
                }
            }
        };
        if (rows >= R && all_channels)
            walk(std::true_type{}, std::true_type{});
        else if (rows >= R)
            walk(std::true_type{}, std::false_type{});
        else
            walk(std::false_type{}, std::false_type{});
        __syncwarp();
    }
    if constexpr (MAPS)
        x.maps[(task.column * x.count + task.order) * 32 + lane] = m;
    else if (dh0 != nullptr && first == 0 && live)
        store_state<WIDE>(dh0 + (int64_t)task.b * D + c, flow, second);
}

// One step, an element per thread: the launch (2.6 us a call from the host).
template <typename T>
__global__ void __launch_bounds__(kThreads)
recurrence_step_kernel(const T* gate, int64_t gate_seq, const T* value, int64_t value_seq, int D, unsigned per, float* state, T* h) {
    layer_begin();
    const int64_t b = blockIdx.x / per;  // `per` blocks to a sequence
    const int d = blockIdx.x % per * kThreads + threadIdx.x;
    if (d >= D) return;
    Pair a, rest;
    gate_of<T>(pair(to_float(gate[b * gate_seq + d]), 0.f), a, rest);
    const float next = fmaf(floats(a).x, state[b * D + d], floats(rest).x * to_float(value[b * value_seq + d]));
    state[b * D + d] = next;
    h[b * D + d] = from_float<T>(next);
}

}  // namespace
}  // namespace cpdp

using namespace cpdp;

static cpdp_status check_recurrence(int B, int64_t T, int D, cpdp_dtype dtype) {
    if (B < 0) return layer_error(CPDP_EINVAL, "B=%d must be >= 0", B);
    CPDP_TRY(check_sizes(1, T, D));
    if (T > int64_t(1) << 30) return layer_error(CPDP_EINVAL, "T=%lld is at most 2^30", (long long)T);
    if (B > 0) {
        if (T > kLayerMaxRows / B || (T > 0 && D > kLayerMaxElements / (B * T)))
            return layer_error(CPDP_EINVAL, "B=%d, T=%lld, D=%d: B * T is at most 2^31 - 1 and all elements at most 2^40", B, (long long)T, D);
        if (ceil_div(D, kChannels) > kLayerMaxRows / B)
            return layer_error(CPDP_EINVAL, "B=%d, D=%d: more blocks than a launch takes", B, D);
    }
    if (!known_dtype(dtype)) return layer_error(CPDP_EINVAL, "unknown dtype %d", (int)dtype);
    return CPDP_OK;
}

// Segments for B sequences of T steps and D channels, of a kernel that runs
// `warps` warps per SM. A split costs a second reading of two inputs, so it has
// to gain more than that: 3 columns per SM go half as fast unsplit as 8. Below,
// as many warps as run at once (more would wait for a second turn), of at least
// 4 chunks each.
static Segments segments_of(int B, int64_t T, int D, int warps) {
    const int64_t groups = ceil_div(D, kChannels), columns = B * groups;
    int64_t count = columns > 0 && columns < 3 * kSMs ? int64_t(warps) * kSMs / columns : 1;
    if (count > T / (4 * R)) count = T / (4 * R);
    count = count < 2 ? 1 : count < 4 ? 2 : count / 4 * 4;
    const int64_t steps = ceil_div(ceil_div(T > 0 ? T : 1, count), R) * R;
    return {static_cast<int>(count), static_cast<int>(steps), static_cast<int>(groups), columns, nullptr};
}

size_t cpdp_gated_recurrence_workspace(int B, int64_t T, int D) {
    if (check_recurrence(B, T, D, CPDP_F32) != CPDP_OK) return 0;
    const Segments x = segments_of(B, T, D, kForwardWarps<__nv_bfloat16>);  // the most warps: the most segments
    return x.count > 1 ? static_cast<size_t>(x.columns) * x.count * 32 * sizeof(Map) : 0;
}

// Whether an array's rows start at multiples of 16 bytes.
static bool in_pieces(const void* p, int64_t size, int64_t a, int64_t b) {
    return aligned_to(p, 16) && a * size % 16 == 0 && b * size % 16 == 0;
}

template <typename... KArgs, typename... Args>
static cudaError_t launch_walk(void (*kernel)(KArgs...), const Segments& x, size_t warp_smem, void* stream, Args... args) {
    // blocks whose warps do not work together are single warps, which share out best: 768 columns in blocks of
    // 4 left 112 SMs with 4 warps and 40 with 8
    const int warps = x.count > 1 ? kWarps : 1;
    const size_t smem = warps * warp_smem;
    // what a launch may have without asking is enough for single warps
    const cudaError_t e =
        smem <= 32 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    return e != cudaSuccess ? e : launch_layer(kernel, static_cast<unsigned>(ceil_div(x.columns * x.count, warps)), warps * 32, smem, stream, args..., x);
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
    Segments x = segments_of(B, T, D, dtype == CPDP_F32 ? kForwardWarps<float> : kForwardWarps<__nv_bfloat16>);
    x.maps = static_cast<Map*>(workspace);
    const SeqIn g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const bool wide = D * e % 16 == 0 && in_pieces(gate, e, gate_seq, gate_step) && in_pieces(value, e, value_seq, value_step) &&
                      aligned_to(h, 16) && aligned_to(carry, 8);
    const auto go = [&](auto* out, auto rows) {
        using E = std::remove_pointer_t<decltype(out)>;
        constexpr bool WIDE = decltype(rows)::value;
        const auto pass = [&](auto kernel) {
            return launch_walk(kernel, x, kForwardRing * 2 * kChunkBytes<E, WIDE>, stream, g, v, static_cast<int>(T), D, h0,
                               lengths, out, h_last, carry);
        };
        const cudaError_t first = x.count > 1 ? pass(recurrence_kernel<E, WIDE, true>) : cudaSuccess;
        return first != cudaSuccess ? first : pass(recurrence_kernel<E, WIDE, false>);
    };
    const auto typed = [&](auto* out) { return wide ? go(out, std::true_type{}) : go(out, std::false_type{}); };
    const cudaError_t launched = dtype == CPDP_F32 ? typed(static_cast<float*>(h)) : typed(static_cast<__nv_bfloat16*>(h));
    return layer_launched(launched, "cpdp_gated_recurrence");
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
    if (some && !nested(B, grad_seq, T, grad_step, D) && !nested(T, grad_step, B, grad_seq, D))
        return layer_error(CPDP_EINVAL, "dgate and dvalue: rows of %d elements at strides of %lld and %lld overlap", D, (long long)grad_seq,
                           (long long)grad_step);
    CPDP_TRY(check_array("dh0", dh0, false, 4));
    CPDP_TRY(check_workspace(workspace, workspace_bytes, cpdp_gated_recurrence_workspace(B, T, D)));
    if (B == 0) return CPDP_OK;
    Segments x = segments_of(B, T, D, dtype == CPDP_F32 ? kBackwardWarps<float> : kBackwardWarps<__nv_bfloat16>);
    x.maps = static_cast<Map*>(workspace);
    const SeqIn o{dh, dh_seq, dh_step}, g{gate, gate_seq, gate_step}, v{value, value_seq, value_step};
    const bool wide = D * e % 16 == 0 && in_pieces(dh, e, dh_seq, dh_step) && in_pieces(gate, e, gate_seq, gate_step) &&
                      in_pieces(value, e, value_seq, value_step) && in_pieces(dgate, e, grad_seq, grad_step) && aligned_to(dvalue, 16);
    const auto go = [&](auto* dg, auto rows) {
        using E = std::remove_pointer_t<decltype(dg)>;
        constexpr bool WIDE = decltype(rows)::value;
        const auto pass = [&](auto kernel, int arrays) {
            return launch_walk(kernel, x, kBackwardRing<E> * arrays * kChunkBytes<E, WIDE>, stream, o, g, v,
                               static_cast<int>(T), D, carry, dh_last, lengths, dg, static_cast<E*>(dvalue), grad_seq, grad_step, dh0);
        };
        const cudaError_t first = x.count > 1 ? pass(recurrence_backward_kernel<E, WIDE, true>, 2) : cudaSuccess;
        return first != cudaSuccess ? first : pass(recurrence_backward_kernel<E, WIDE, false>, 3);
    };
    const auto typed = [&](auto* dg) { return wide ? go(dg, std::true_type{}) : go(dg, std::false_type{}); };
    const cudaError_t launched = dtype == CPDP_F32 ? typed(static_cast<float*>(dgate)) : typed(static_cast<__nv_bfloat16*>(dgate));
    return layer_launched(launched, "cpdp_gated_recurrence_backward");
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
    const unsigned per = static_cast<unsigned>(ceil_div(D, kThreads));
    const auto go = [&](auto* out) {
        using E = std::remove_pointer_t<decltype(out)>;
        return launch_layer(recurrence_step_kernel<E>, per * B, kThreads, 0, stream, static_cast<const E*>(gate), gate_seq,
                            static_cast<const E*>(value), value_seq, D, per, state, out);
    };
    return layer_launched(dtype == CPDP_F32 ? go(static_cast<float*>(h)) : go(static_cast<__nv_bfloat16*>(h)),
                          "cpdp_gated_recurrence_step");
}
