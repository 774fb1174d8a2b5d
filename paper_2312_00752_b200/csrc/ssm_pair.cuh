// Arithmetic on one value (float) or on two at once (float2, whose sums and products are single packed instructions).
#pragma once

#include "ssm_common.cuh"

namespace ssm {
#ifdef __CUDACC__
__device__ __forceinline__ float vmul(float a, float b) { return a * b; }
__device__ __forceinline__ float2 vmul(float2 a, float2 b) { return f2mul(a, b); }
__device__ __forceinline__ float vadd(float a, float b) { return a + b; }
__device__ __forceinline__ float2 vadd(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float vfma(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ float2 vfma(float2 a, float2 b, float2 c) { return f2fma(a, b, c); }
template <class F>
__device__ __forceinline__ F vset(float v);
template <>
__device__ __forceinline__ float vset<float>(float v) { return v; }
template <>
__device__ __forceinline__ float2 vset<float2>(float v) { return make_float2(v, v); }
template <class Op>
__device__ __forceinline__ float vmap(float a, Op&& op) { return op(a); }
template <class Op>
__device__ __forceinline__ float2 vmap(float2 a, Op&& op) { return make_float2(op(a.x), op(a.y)); }
template <class Op>
__device__ __forceinline__ float vmap(float a, float b, float c, Op&& op) { return op(a, b, c); }
template <class Op>
__device__ __forceinline__ float2 vmap(float2 a, float2 b, float2 c, Op&& op) { return make_float2(op(a.x, b.x, c.x), op(a.y, b.y, c.y)); }

template <class F>
constexpr int kWidth = sizeof(F) / sizeof(float);
#endif
}  // namespace ssm
