// The gates of the gated linear recurrence (include/ssm_gated.h), on one channel (float) or a pair of channels (float2, whose
// sums and products issue two-wide), and what its kernels share.
#pragma once

#include <cfloat>

#include "ssm_common.cuh"
#include "ssm_gated.h"

namespace ssm {

struct GatedParams {
  const void* x;
  const void* gate;
  const void* in_gate;    // decay form
  const float* A;         // decay form
  const uint8_t* reset;   // null: none
  const float* h0;        // null: zero
  void* y;                // forward; null: not wanted (the states alone are)
  float* h_last;          // null: not wanted
  float* states;          // [batch][nck][D] state before every kGatedSteps-th step; forward: null if not wanted
  const void* dy;         // backward
  const float* dh_last;   // null: zero
  void* dx;
  void* dgate;
  void* din_gate;
  float* dA_part;         // [parts][D]
  float* dh0;             // null: not wanted
  int64_t ld_x, ld_gate, ld_in, ld_dx, ld_dgate, ld_din;   // distance of rows, in elements
  int batch, L, D, nck;
  int tiles;              // groups of channels of one batch entry
};

#ifdef __CUDACC__
// ------------------------------------------------------------------------------------------- one channel or two
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

// `F` of adjacent channels as they lie in memory
template <typename IO, class F>
struct Lane;
template <>
struct Lane<float, float> {
  using Raw = float;
  static __device__ __forceinline__ float open(float r) { return r; }
  static __device__ __forceinline__ float close(float v) { return v; }
};
template <>
struct Lane<float, float2> {
  using Raw = float2;
  static __device__ __forceinline__ float2 open(float2 r) { return r; }
  static __device__ __forceinline__ float2 close(float2 v) { return v; }
};
template <>
struct Lane<__nv_bfloat16, float> {
  using Raw = unsigned short;
  static __device__ __forceinline__ float open(unsigned short r) { return __uint_as_float((uint32_t)r << 16); }
  static __device__ __forceinline__ unsigned short close(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
};
template <>
struct Lane<__nv_bfloat16, float2> {
  using Raw = uint32_t;
  static __device__ __forceinline__ float2 open(uint32_t r) { return make_float2(bf16lo(r), bf16hi(r)); }
  static __device__ __forceinline__ uint32_t close(float2 v) {
    const __nv_bfloat162 r = __floats2bfloat162_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&r);
  }
};

// ------------------------------------------------------------------------------------------------------------- gates
__device__ __forceinline__ float rsqrt_approx(float v) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// sigma(z) and 1 - sigma(z).  Where g = sigma(z) is small, 1 - g is near 1 and the subtraction rounds it without bias, which
// matters where it is the retention, since its error multiplies over the 1 / g steps that the state remembers; where g is
// large 1 - g would cancel, and e / (1 + e) does not (e may be infinite, then g is 0).
template <class F>
__device__ __forceinline__ void gate_pair(F z, F& g, F& og) {
  const F e = vmap(vmul(z, vset<F>(-kLog2e)), [](float v) { return ex2_approx(v); });
  g = vmap(vadd(e, vset<F>(1.f)), [](float v) { return rcp_approx(v); });
  const F near = vfma(g, vset<F>(-1.f), vset<F>(1.f)), far = vmul(e, g);
  og = vmap(g, near, far, [](float v, float n, float f) { return v < 0.5f ? n : f; });
}

// a = exp(v) and 1 - a for v <= 0: 1 - a = -expm1(v) by its series up to |v| < 1/4 (relative remainder 0.25^6 / 5040 = 5e-8)
template <class F>
__device__ __forceinline__ void decay_pair(F v, F& a, F& oa) {
  F s = vfma(v, vset<F>(1.f / 720.f), vset<F>(1.f / 120.f));
  s = vfma(v, s, vset<F>(1.f / 24.f));
  s = vfma(v, s, vset<F>(1.f / 6.f));
  s = vfma(v, s, vset<F>(0.5f));
  s = vfma(v, s, vset<F>(1.f));
  const F near = vmul(vmul(v, vset<F>(-1.f)), s);
  const F ex = vmap(vmul(v, vset<F>(kLog2e)), [](float w) { return ex2_approx(w); });
  const F far = vfma(ex, vset<F>(-1.f), vset<F>(1.f));
  oa = vmap(v, near, far, [](float w, float n, float f) { return fabsf(w) < 0.25f ? n : f; });
  a = vmap(v, vfma(near, vset<F>(-1.f), vset<F>(1.f)), ex, [](float w, float n, float f) { return fabsf(w) < 0.25f ? n : f; });
}

// The same for -1 <= A <= 0, with w = -v in [0, 1]: (1 - exp(-w)) / w by its Chebyshev interpolation of degree 6 (relative error
// 3e-9), no special-function operation and no case distinction.
template <class F>
__device__ __forceinline__ void decay_pair_small(F w, F& a, F& oa) {
  F s = vfma(w, vset<F>(1.29076311e-4f), vset<F>(-1.30077498e-3f));
  s = vfma(w, s, vset<F>(8.27550516e-3f));
  s = vfma(w, s, vset<F>(-4.16468494e-2f));
  s = vfma(w, s, vset<F>(1.66663408e-1f));
  s = vfma(w, s, vset<F>(-4.99999791e-1f));
  s = vfma(w, s, vset<F>(1.f));
  oa = vmul(w, s);
  a = vfma(oa, vset<F>(-1.f), vset<F>(1.f));
}

// 1 - a^2 = oa (2 - oa).  The least normal number keeps its reciprocal root finite where a = 1: that meets rho or A, which is 0
// there, and the root itself is 1e-19 instead of 0.
template <class F>
__device__ __forceinline__ F one_minus_square(F oa) {
  return vfma(oa, vfma(oa, vset<F>(-1.f), vset<F>(2.f)), vset<F>(FLT_MIN));
}

// One step of the forward recurrence: retention a and input u.  SMALL: -1 <= A <= 0, and A comes negated.
// The special-function unit, four lanes a cycle, limits bf16 io next to the memory, so beta and the input gate come from
// one operation: with f = 1 + exp(-in_gate), m2 rsqrt(m2 f^2) = sqrt(m2) / f = beta iota (f^2 may be infinite: then it is 0).
template <bool DECAY, bool SMALL, class F>
__device__ __forceinline__ void step_inputs(F x, F gate, F in_gate, F A, F& a, F& u) {
  F g;
  if constexpr (!DECAY) {
    gate_pair(gate, g, a);
    u = vmul(g, x);
  } else {
    F oa;
    g = vmap(vadd(vmap(vmul(gate, vset<F>(-kLog2e)), [](float v) { return ex2_approx(v); }), vset<F>(1.f)), [](float v) { return rcp_approx(v); });
    const F f = vadd(vmap(vmul(in_gate, vset<F>(-kLog2e)), [](float v) { return ex2_approx(v); }), vset<F>(1.f));
    if constexpr (SMALL) decay_pair_small(vmul(g, A), a, oa);
    else decay_pair(vmul(g, A), a, oa);
    const F m2 = one_minus_square(oa);
    u = vmul(vmul(m2, vmap(vmul(vmul(m2, f), f), [](float v) { return rsqrt_approx(v); })), x);
  }
}
#endif

// ------------------------------------------------------------------------------------------------------------ launches
// Steps of one warp in a tile, and between two saved states.
constexpr int kGatedSteps = 16;

// unit: bytes (16, 4 or, for bf16, 2) whose multiples the io pointers and the distances of rows are, D too
cudaError_t launch_gated_fwd(const GatedParams& p, int io_dtype, bool decay, int unit, cudaStream_t s);

}  // namespace ssm
