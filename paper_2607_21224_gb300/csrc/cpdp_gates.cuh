// Arithmetic of the layers that walk along time: pairs of floats, the sigmoid.
#pragma once

#include "cpdp_layers.cuh"

#ifdef __CUDACC__
namespace cpdp {
namespace {

// Two floats in a pair of registers, for the instructions that work on both.
using Pair = unsigned long long;
constexpr Pair kOnes = 0x3f8000003f800000ull, kZeros = 0, kMinusOnes = 0xbf800000bf800000ull;
__device__ __forceinline__ Pair pair(float x, float y) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p) : "f"(x), "f"(y));
    return p;
}
__device__ __forceinline__ float2 floats(Pair p) {
    float2 v;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// a = sigmoid(x) and 1 - a, neither formed as a difference from 1. With
// t = e^-|x| in [0, 1] they are 1 / (1 + t) and t / (1 + t); below 1e-38 t is 0.
// The power is 2^-p of the rounded product p = |x| log2(e). What the rounding
// left out makes t's relative error grow with |x| (1e-6 at 16, 4e-6 at 80). For
// float32 gates t is multiplied by e^r, r = p ln 2 - |x|, of which 1 + r is
// enough (1 to 5 % of a scan's time). bfloat16 gates, whose own spacing is 30,000
// times that, go without (it took 3 to 15 %). The scans are bound by the
// instructions that they issue: exact range reduction and division, with their
// cases for tiny numbers, took 2.5 times as many.
constexpr float kLog2eHigh = 1.44269502162933349609375f, kLog2eLow = 1.92596303e-8f, kLn2 = 0.693147180559945309f;  // High: the float32
__device__ __forceinline__ float power_of_minus(float p) {
    float t;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(-p));
    return t;
}
__device__ __forceinline__ float size_of(float x) {  // beyond 128 t is 0 all the same, and r stays finite; NaN stays NaN
    float m;
    asm("min.NaN.f32 %0, %1, 0f43000000;" : "=f"(m) : "f"(fabsf(x)));
    return m;
}
__device__ __forceinline__ Pair twice(float x) { return pair(x, x); }
template <typename T>
__device__ __forceinline__ Pair exp_of_minus(float2 x) {
    if constexpr (sizeof(T) == 2) {
        return pair(power_of_minus(kLog2eHigh * fabsf(x.x)), power_of_minus(kLog2eHigh * fabsf(x.y)));
    } else {
        const Pair m = pair(size_of(x.x), size_of(x.y)), p = mul2(m, twice(kLog2eHigh));
        const Pair t = pair(power_of_minus(floats(p).x), power_of_minus(floats(p).y));
        const Pair rounded = fma2(m, twice(-kLog2eHigh), p);  // exact
        return fma2(t, fma2(rounded, twice(kLn2), mul2(m, twice(-kLog2eLow * kLn2))), t);
    }
}
__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// T: the gates' type.
template <typename T>
__device__ __forceinline__ void gate_of(Pair gates, Pair& a, Pair& rest) {
    const float2 x = floats(gates);
    const Pair t = exp_of_minus<T>(x);
    const float2 s = floats(add2(t, kOnes)), r = make_float2(reciprocal(s.x), reciprocal(s.y)), q = floats(mul2(t, pair(r.x, r.y)));
    a = pair(x.x >= 0.f ? r.x : q.x, x.y >= 0.f ? r.y : q.y);
    rest = pair(x.x >= 0.f ? q.x : r.x, x.y >= 0.f ? q.y : r.y);
}

// x or 0. Not a branch around what makes x, which ?: became where that is short (a backward pass of the convolution
// took 62 us for 48).
__device__ __forceinline__ Pair where(bool there, Pair x) {
    Pair r;
    asm("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %2, 0;\n\tselp.b64 %0, %1, 0, p;\n\t}" : "=l"(r) : "l"(x), "r"(there ? 1u : 0u));
    return r;
}
// sigmoid(x) alone, as 1 / (1 + 2^(-x log2(e))): 6 instructions for both, where gate_of takes some 20. The power's
// argument is rounded, which is |x| 2^-24 of the result; below -88 the power is infinite and the result 0.
__device__ __forceinline__ Pair sigmoid(Pair x) {
    const float2 p = floats(mul2(x, twice(kLog2eHigh))), s = floats(add2(pair(power_of_minus(p.x), power_of_minus(p.y)), kOnes));
    return pair(reciprocal(s.x), reciprocal(s.y));
}
// The slope of x sigmoid(x), a = sigmoid(x): a (1 + x (1 - a)).
__device__ __forceinline__ Pair silu_slope(Pair x, Pair a) { return mul2(a, fma2(x, fma2(a, kMinusOnes, kOnes), kOnes)); }

}  // namespace
}  // namespace cpdp
#endif
