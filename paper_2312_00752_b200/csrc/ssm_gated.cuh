// The gates of the gated linear recurrence (include/ssm_gated.h): what a step does to the state, and what its gradients need.
#pragma once

#include "ssm_common.cuh"
#include "ssm_gated.h"

namespace ssm {

// Steps between two saved states.
constexpr int kGatedCkptSteps = 16;

struct GatedParams {
  const void* x;
  const void* gate;
  const void* in_gate;    // decay form
  const float* A;         // decay form
  const uint8_t* reset;   // null: none
  const float* h0;        // null: zero
  void* y;                // forward; null: not wanted (the states alone are)
  float* h_last;          // null: not wanted
  float* states;          // [batch][nck][D] state before every kGatedCkptSteps-th step; forward: null if not wanted
  const void* dy;         // backward
  const float* dh_last;   // null: zero
  void* dx;
  void* dgate;
  void* din_gate;
  float* dA_part;         // [parts][D]
  float* dh0;             // null: not wanted
  int64_t ld_x, ld_gate, ld_in, ld_dx, ld_dgate, ld_din;   // distance of rows, in elements
  int batch, L, D, nck;
};

// One step of one channel.  a: what is kept of the state, u: what comes in.
//   convex: a = 1 - g.  Where g is small a is near 1 and the subtraction rounds it without bias, which matters, since the
//   error of a multiplies over the 1 / g steps that the state remembers; where g is large 1 - g would cancel, and the
//   quotient's other part e / (1 + e) is exact.
//   decay: m = 1 - a = -expm1(v), v = rho A, by its series up to |v| < 1/4 (relative remainder 0.25^6 / 5040 = 5e-8), and
//   1 - a^2 = m (2 - m) without cancellation.
struct Gates {
  float a, u;
  float g, og;       // the gate (g or rho) and 1 - g
  float iota, oi;    // decay: the input gate and 1 - iota
  float beta;        // decay: sqrt(1 - a^2)
  float m2;          // decay: 1 - a^2
};

__device__ __forceinline__ void gate_pair(float z, float& g, float& og) {   // sigma(z) and 1 - sigma(z)
  const float e = ex2_approx(-kLog2e * z);
  g = rcp_approx(1.f + e);
  og = g < 0.5f ? 1.f - g : e * g;      // (e may be infinite, then g is 0)
}

__device__ __forceinline__ float one_minus_exp(float v) {
  float s = fmaf(v, 1.f / 720.f, 1.f / 120.f);
  s = fmaf(v, s, 1.f / 24.f);
  s = fmaf(v, s, 1.f / 6.f);
  s = fmaf(v, s, 0.5f);
  s = fmaf(v, s, 1.f);
  return fabsf(v) < 0.25f ? -v * s : 1.f - ex2_approx(kLog2e * v);
}

__device__ __forceinline__ float sqrt_approx(float v) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float rsqrt_approx(float v) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

template <bool DECAY>
__device__ __forceinline__ Gates gates(float x, float gate, float in_gate, float A) {
  Gates r;
  gate_pair(gate, r.g, r.og);
  if constexpr (!DECAY) {
    r.a = r.og;
    r.u = r.g * x;
  } else {
    const float v = r.g * A;
    const float m = one_minus_exp(v);
    r.a = fabsf(v) < 0.25f ? 1.f - m : ex2_approx(kLog2e * v);
    r.m2 = m * (2.f - m);
    gate_pair(in_gate, r.iota, r.oi);
    r.beta = sqrt_approx(r.m2);
    r.u = r.beta * r.iota * x;
  }
  return r;
}

}  // namespace ssm
