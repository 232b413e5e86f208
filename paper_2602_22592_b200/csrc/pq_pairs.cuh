#pragma once
#include "pq_kernels.cuh"

namespace pq {

// Pairs of fp32 numbers, as bf16 words unpack into them; every operation rounds each of the two once.  (The packed f32x2 instructions took
// an eighth fewer instructions and the same time: norms backward of 8192 x 2048 50.4 against 49.9 us.)
struct F2 { float x, y; };
__device__ __forceinline__ F2 f2(float lo, float hi) { return F2{lo, hi}; }
__device__ __forceinline__ F2 f2(float x) { return F2{x, x}; }
__device__ __forceinline__ void get(const F2& a, float& lo, float& hi) { lo = a.x; hi = a.y; }
__device__ __forceinline__ F2 operator*(const F2& a, const F2& b) { return F2{__fmul_rn(a.x, b.x), __fmul_rn(a.y, b.y)}; }
__device__ __forceinline__ F2 operator+(const F2& a, const F2& b) { return F2{__fadd_rn(a.x, b.x), __fadd_rn(a.y, b.y)}; }
__device__ __forceinline__ F2 fma2(const F2& a, const F2& b, const F2& c) { return F2{__fmaf_rn(a.x, b.x, c.x), __fmaf_rn(a.y, b.y, c.y)}; }
__device__ __forceinline__ float both(const F2& a) { return a.x + a.y; }

}  // namespace pq
