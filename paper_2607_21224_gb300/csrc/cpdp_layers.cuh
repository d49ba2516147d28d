// What the files of the worker-batched layers (include/cpdp_layers.h) share:
// argument checks, launches, and loads and stores of the two element types.
#pragma once

#include <cstdint>
#include <cuda_runtime.h>
#include <cuda_bf16.h>

#include "cpdp_layers.h"

namespace cpdp {

// The message of a failed call that has no context (cpdp_last_error(NULL)); returns `st`.
cpdp_status layer_error(cpdp_status st, const char* fmt, ...);
// CPDP_OK, or CPDP_ECUDA with the launch's error (else one that the runtime recorded).
cpdp_status layer_launched(cudaError_t launched, const char* what);

constexpr int64_t kLayerMaxElements = int64_t(1) << 40;
constexpr int64_t kLayerMaxRows = (int64_t(1) << 31) - 1;
constexpr int64_t kLayerMaxFeatures = int64_t(1) << 30;
constexpr int kSMs = 152;
constexpr int kBlock8 = 32;  // features that share an exponent

__host__ __device__ constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline bool known_dtype(cpdp_dtype t) { return t == CPDP_F32 || t == CPDP_BF16; }
inline int64_t dtype_size(cpdp_dtype t) { return t == CPDP_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// W, M and D of an array [W][M][D].
inline cpdp_status check_sizes(int W, int64_t M, int64_t D) {
    if (W < 1 || W > 4096) return layer_error(CPDP_EINVAL, "W=%d must be in [1, 4096]", W);
    if (M < 0 || D < 1 || D > kLayerMaxFeatures)
        return layer_error(CPDP_EINVAL, "rows (%lld) must be >= 0 and features (%lld) in [1, 2^30]", (long long)M, (long long)D);
    if (M > kLayerMaxRows / W || (M > 0 && D > kLayerMaxElements / (W * M)))
        return layer_error(CPDP_EINVAL, "W=%d, rows=%lld, features=%lld: W * rows is at most 2^31 - 1 and all elements at most 2^40",
                           W, (long long)M, (long long)D);
    return CPDP_OK;
}

// An array that the call needs (`wanted`: it has elements): not NULL, aligned to its element, strides >= 0.
inline cpdp_status check_array(const char* name, const void* p, bool wanted, int64_t size, int64_t stride_a = 0,
                               int64_t stride_b = 0) {
    if (p == nullptr && wanted) return layer_error(CPDP_EINVAL, "%s is NULL", name);
    if (!aligned_to(p, size)) return layer_error(CPDP_EALIGN, "%s %p is not aligned to its %d-byte elements", name, p, (int)size);
    if (stride_a < 0 || stride_b < 0 || stride_a > kLayerMaxElements || stride_b > kLayerMaxElements)
        return layer_error(CPDP_EINVAL, "%s: strides %lld and %lld must be in [0, 2^40]", name, (long long)stride_a, (long long)stride_b);
    return CPDP_OK;
}

// Parts of an output, `size` elements each and `stride` apart, that different blocks write.
inline cpdp_status check_apart(const char* name, int64_t count, int64_t stride, int64_t size) {
    if (count > 1 && stride < size)
        return layer_error(CPDP_EINVAL, "%s: parts of %lld elements at a stride of %lld overlap", name, (long long)size, (long long)stride);
    return CPDP_OK;
}
// Whether n rows of `inner` elements of stride lie between neighbours of stride `outer`.
inline bool nested(int64_t count, int64_t outer, int64_t n, int64_t inner, int64_t size) {
    return (n <= 1 || inner >= size) && (count <= 1 || (outer >= size && (n <= 1 || n - 1 <= (outer - size) / inner)));
}

inline cpdp_status check_workspace(const void* p, size_t bytes, size_t needed) {
    if (needed == 0) return CPDP_OK;
    if (p == nullptr || bytes < needed)
        return layer_error(CPDP_EINVAL, "workspace of %zu bytes: %zu are needed", p == nullptr ? size_t(0) : bytes, needed);
    if (!aligned_to(p, 16)) return layer_error(CPDP_EALIGN, "workspace %p is not 16-byte aligned", p);
    return CPDP_OK;
}

#define CPDP_TRY(call)                               \
    do {                                             \
        const cpdp_status try_st = (call);           \
        if (try_st != CPDP_OK) return try_st;        \
    } while (0)

// Launch with programmatic dependent launch: the grid may begin while the one
// before it on the stream drains, and every kernel waits for that one's
// completion (layer_begin) before it touches memory.
template <typename... KArgs, typename... Args>
cudaError_t launch_layer(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, void* stream, Args... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

#ifdef __CUDACC__
__device__ __forceinline__ void layer_begin() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// Loads of what is read once, first out of L2. The launch before on the stream
// may have written it while this grid's blocks were already there, so loads here
// are coherent ones and stay below layer_begin's wait: volatile, with a memory
// clobber (or plain C++ loads), never ld.global.nc, whose contents must not
// change while a kernel runs.
__device__ __forceinline__ float load_once(const float* p) {
    float v;
    asm volatile("ld.global.cs.f32 %0, [%1];" : "=f"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ float4 load_once(const float4* p) {
    float4 v;
    asm volatile("ld.global.cs.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ uint4 load_once(const uint4* p) {
    uint4 v;
    asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int2 load_once(const int2* p) {
    int2 v;
    asm volatile("ld.global.cs.v2.s32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int load_once(const int8_t* p) {
    int v;
    asm volatile("ld.global.cs.s8 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
// Single elements where `there`; else v stays as it is. Predicates, not branches: loads in stretches of code of their own
// do not overlap (rows of bfloat16 off 16 bytes took 2 to 4 times as long). A bfloat16's bits go to a register of their
// own: a 16-bit variable shares one with another, and waits for that one's load.
__device__ __forceinline__ void load_once(float& v, const float* p, bool there) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.cs.f32 %0, [%1];\n\t}"
                 : "+f"(v)
                 : "l"(p), "r"(there ? 1u : 0u)
                 : "memory");
}
__device__ __forceinline__ void load_once(uint32_t& v, const __nv_bfloat16* p, bool there) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\t@p ld.global.cs.u16 %0, [%1];\n\t}"
                 : "+r"(v)
                 : "l"(p), "r"(there ? 1u : 0u)
                 : "memory");
}

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// The exponent byte of a block of 8-bit values whose largest magnitude is
// `top`, given as its bits: e = the least with top <= 127 * 2^e. top = m * 2^k
// with m in [1, 2), 127 = 1.984375 * 2^6, so e is k - 6 or, above 1.984375,
// k - 5: an integer addition to the bits carries into the exponent exactly
// there. 255 where top is infinite or NaN.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t top_bits) {
    if (top_bits >= 0x7f800000u) return 255u;
    const int k = static_cast<int>((top_bits + 0x0001ffffu) >> 23);  // k + 127, one more above 1.984375
    return static_cast<uint32_t>(min(max(k - 6, 1), 248));
}
// 2^e and 2^-e of an exponent byte; NaN and 0 for 255.
__device__ __forceinline__ float unit_of(uint32_t byte) { return __uint_as_float(byte == 255u ? 0x7fc00000u : byte << 23); }
__device__ __forceinline__ float inverse_unit_of(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0u : (254u - byte) << 23);
}
// The code of x in units of 1 / inverse (0 where x is not finite and the block reads back as NaN).
__device__ __forceinline__ int code_of(float x, float inverse) {
    return max(-127, min(127, __float2int_rn(x * inverse)));
}
// V neighbouring elements of a row as they lie in memory: 16 bytes' worth,
// or one, which is loaded where it is there.
template <typename T, int V>
struct Piece;
template <>
struct Piece<float, 4> {
    float4 v;
    __device__ __forceinline__ float get(int e) const { return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w; }
    __device__ __forceinline__ void load(const float* p) { v = load_once(reinterpret_cast<const float4*>(p)); }
};
template <>
struct Piece<__nv_bfloat16, 8> {
    uint4 v;
    __device__ __forceinline__ float get(int e) const {
        const uint32_t u = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w;
        return __uint_as_float(e % 2 ? u & 0xffff0000u : u << 16);
    }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = load_once(reinterpret_cast<const uint4*>(p)); }
};
template <>
struct Piece<float, 1> {
    float v;
    __device__ __forceinline__ float get(int) const { return v; }
    __device__ __forceinline__ void load(const float* p, bool there) { load_once(v, p, there); }
};
template <>
struct Piece<__nv_bfloat16, 1> {
    uint32_t v;
    __device__ __forceinline__ float get(int) const { return __uint_as_float(v << 16); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool there) { load_once(v, p, there); }
};

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <int V>
__device__ __forceinline__ void store_piece(float* p, const float* v) {
    if constexpr (V == 4)
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else
        *p = v[0];
}
template <int V>
__device__ __forceinline__ void store_piece(__nv_bfloat16* p, const float* v) {
    if constexpr (V == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(pack(v[0], v[1]), pack(v[2], v[3]), pack(v[4], v[5]), pack(v[6], v[7]));
    else if constexpr (V == 4)
        *reinterpret_cast<uint2*>(p) = make_uint2(pack(v[0], v[1]), pack(v[2], v[3]));
    else
        *p = __float2bfloat16_rn(v[0]);
}
template <int V>
__device__ __forceinline__ void store_codes(int8_t* p, const int* q) {
    const auto word = [](const int* c) { return (c[0] & 255) | (c[1] & 255) << 8 | (c[2] & 255) << 16 | c[3] << 24; };
    if constexpr (V == 8)
        *reinterpret_cast<int2*>(p) = make_int2(word(q), word(q + 4));
    else if constexpr (V == 4)
        *reinterpret_cast<int*>(p) = word(q);
    else
        *p = static_cast<int8_t>(q[0]);
}
#endif

}  // namespace cpdp
