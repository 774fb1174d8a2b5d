// Gated linear recurrence, forward, backward and one step of decoding.  See include/ssm_gated.h for the definition.
#include "ssm_gated.cuh"

namespace ssm {

namespace {

constexpr int kThreads = 128;

template <typename IO>
__device__ __forceinline__ float at(const void* base, int64_t row, int64_t ld, int d) {
  return io_to_float<IO>(static_cast<const IO*>(base)[row * ld + d]);
}
template <typename IO>
__device__ __forceinline__ void put(void* base, int64_t row, int64_t ld, int d, float v) {
  static_cast<IO*>(base)[row * ld + d] = float_to_io<IO>(v);
}

// One step, with what its gradients need: the gate g (or rho) and 1 - g, the input gate and 1 - iota, beta = sqrt(1 - a^2).
struct Gates {
  float a, u, g, og, iota, oi, beta, inv;
};
template <bool DECAY>
__device__ __forceinline__ Gates gates(float x, float gate, float in_gate, float A) {
  Gates r{};
  gate_pair(gate, r.g, r.og);
  r.a = r.og;
  r.u = r.g * x;
  if constexpr (DECAY) {
    float oa;
    decay_pair(r.g * A, r.a, oa);
    gate_pair(in_gate, r.iota, r.oi);
    const float m2 = one_minus_square(oa);
    r.inv = rsqrt_approx(m2);
    r.beta = m2 * r.inv;
    r.u = r.beta * r.iota * x;
  }
  return r;
}

template <typename IO, bool DECAY>
__global__ void __launch_bounds__(kThreads) ssm_gated_bwd_kernel(const GatedParams p) {
  dependency_wait();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= (int64_t)p.batch * p.D) return;
  const int b = (int)(i / p.D), d = (int)(i % p.D);
  const float A = DECAY ? p.A[d] : 0.f;
  float carry = p.dh_last != nullptr ? p.dh_last[i] : 0.f;   // a[t+1] mu[t+1]
  float dA = 0.f;
  for (int k0 = p.nck - 1; k0 >= 0; --k0) {
    const int t0 = k0 * kGatedSteps, n = min(kGatedSteps, p.L - t0);
    float before[kGatedSteps];     // the state that each step starts from
    float h = p.states[((int64_t)b * p.nck + k0) * p.D + d];
#pragma unroll
    for (int j = 0; j < kGatedSteps; ++j) {
      if (j < n) {
        const int64_t row = (int64_t)b * p.L + t0 + j;
        const Gates k = gates<DECAY>(at<IO>(p.x, row, p.ld_x, d), at<IO>(p.gate, row, p.ld_gate, d),
                                     DECAY ? at<IO>(p.in_gate, row, p.ld_in, d) : 0.f, A);
        before[j] = p.reset != nullptr && p.reset[row] ? 0.f : h;
        h = p.reset != nullptr && p.reset[row] ? k.u : fmaf(k.a, h, k.u);
      }
    }
#pragma unroll
    for (int j = kGatedSteps - 1; j >= 0; --j) {
      if (j < n) {
        const int64_t row = (int64_t)b * p.L + t0 + j;
        const float x = at<IO>(p.x, row, p.ld_x, d);
        const Gates k = gates<DECAY>(x, at<IO>(p.gate, row, p.ld_gate, d), DECAY ? at<IO>(p.in_gate, row, p.ld_in, d) : 0.f, A);
        const float mu = at<IO>(p.dy, row, p.D, d) + carry;
        if constexpr (DECAY) {
          const float m = mu * k.a * fmaf(-k.a * k.iota, x * k.inv, before[j]);
          put<IO>(p.dx, row, p.ld_dx, d, mu * k.beta * k.iota);
          put<IO>(p.din_gate, row, p.ld_din, d, mu * k.u * k.oi);
          put<IO>(p.dgate, row, p.ld_dgate, d, m * A * k.g * k.og);
          dA = fmaf(m, k.g, dA);
        } else {
          put<IO>(p.dx, row, p.ld_dx, d, mu * k.g);
          put<IO>(p.dgate, row, p.ld_dgate, d, mu * (x - before[j]) * k.g * k.og);
        }
        carry = p.reset != nullptr && p.reset[row] ? 0.f : mu * k.a;
      }
    }
  }
  if (p.dh0 != nullptr) p.dh0[i] = carry;
  if (DECAY) p.dA_part[i] = dA;
}

// dA[d]: the parts in ascending order
__global__ void __launch_bounds__(kThreads) ssm_gated_reduce_kernel(const float* __restrict__ part, int parts, int D,
                                                                  float* __restrict__ dA) {
  dependency_wait();
  const int d = blockIdx.x * kThreads + threadIdx.x;
  if (d >= D) return;
  float s = 0.f;
  for (int q = 0; q < parts; ++q) s += part[(size_t)q * D + d];
  dA[d] = s;
}

// ------------------------------------------------------------------------------------------------------------ one step
template <typename IO, bool DECAY>
__global__ void __launch_bounds__(kThreads) ssm_gated_step_kernel(const GatedParams p, float* __restrict__ hbuf) {
  dependency_wait();
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= (int64_t)p.batch * p.D) return;
  const int b = (int)(i / p.D), d = (int)(i % p.D);
  const Gates k = gates<DECAY>(at<IO>(p.x, b, p.ld_x, d), at<IO>(p.gate, b, p.ld_gate, d),
                               DECAY ? at<IO>(p.in_gate, b, p.ld_in, d) : 0.f, DECAY ? p.A[d] : 0.f);
  const float h = p.reset != nullptr && p.reset[b] ? k.u : fmaf(k.a, hbuf[i], k.u);
  hbuf[i] = h;
  put<IO>(p.y, b, p.D, d, h);
}

template <typename... P, typename... A>
cudaError_t launch_channels(void (*kernel)(P...), const GatedParams& p, cudaStream_t s, const A&... args) {
  return launch_dependent(kernel, (unsigned)(((int64_t)p.batch * p.D + kThreads - 1) / kThreads), kThreads, 0, 1, s, args...);
}

// ------------------------------------------------------------------------------------------------------- host side
bool decay(const ssm_gated_problem_t& p) { return p.flags & SSM_GATED_FLAG_DECAY; }
size_t esize(const ssm_gated_problem_t& p) { return p.io_dtype == SSM_BF16 ? 2 : 4; }
int64_t row_distance(int64_t ld, int D) { return ld == 0 ? D : ld; }

ssm_status_t validate(const ssm_gated_problem_t* p) {
  if (p == nullptr || p->batch < 1 || p->L < 1 || p->D < 1) return SSM_ERR_INVALID_ARG;
  if (p->flags & ~(uint32_t)(SSM_GATED_FLAG_DECAY | SSM_GATED_FLAG_SAVE_STATES)) return SSM_ERR_INVALID_ARG;
  if (p->io_dtype != SSM_F32 && p->io_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)p->batch * p->L;
  if (p->D > INT64_MAX / 8 / rows) return SSM_ERR_UNSUPPORTED;
  for (int64_t ld : {p->ld_x, p->ld_gate, p->ld_in_gate, p->ld_dx, p->ld_dgate, p->ld_din_gate}) {
    if (ld != 0 && ld < p->D) return SSM_ERR_INVALID_ARG;
    if (ld > INT64_MAX / 8 / rows) return SSM_ERR_INVALID_ARG;    // (byte offsets stay within 63 bits)
  }
  if (!decay(*p) && (p->ld_in_gate != 0 || p->ld_din_gate != 0)) return SSM_ERR_INVALID_ARG;
  if (p->D > 1 << 28) return SSM_ERR_UNSUPPORTED;                // (a row's bytes fit 32 bits)
  // blocks of the grids, 32 channels of one batch entry at the least
  if ((int64_t)p->batch * (((int64_t)p->D + 31) / 32) > INT32_MAX / 16) return SSM_ERR_UNSUPPORTED;
  if (p->L > INT32_MAX - 65536) return SSM_ERR_UNSUPPORTED;     // (steps of a round past the end)
  return SSM_OK;
}

bool aligned(const void* q, size_t a) { return reinterpret_cast<uintptr_t>(q) % a == 0; }

GatedParams params(const ssm_gated_problem_t& p) {
  GatedParams g{};
  g.batch = p.batch;
  g.L = p.L;
  g.D = p.D;
  g.nck = (p.L + kGatedSteps - 1) / kGatedSteps;
  g.ld_x = row_distance(p.ld_x, p.D);
  g.ld_gate = row_distance(p.ld_gate, p.D);
  g.ld_in = row_distance(p.ld_in_gate, p.D);
  g.ld_dx = row_distance(p.ld_dx, p.D);
  g.ld_dgate = row_distance(p.ld_dgate, p.D);
  g.ld_din = row_distance(p.ld_din_gate, p.D);
  return g;
}

size_t state_bytes(const ssm_gated_problem_t& p) {
  return (size_t)p.batch * ((p.L + kGatedSteps - 1) / kGatedSteps) * p.D * sizeof(float);
}
size_t round16(size_t n) { return (n + 15) / 16 * 16; }

template <typename IO>
cudaError_t launch_backward(const GatedParams& p, bool dec, cudaStream_t s) {
  return dec ? launch_channels(ssm_gated_bwd_kernel<IO, true>, p, s, p) : launch_channels(ssm_gated_bwd_kernel<IO, false>, p, s, p);
}
template <typename IO>
cudaError_t launch_step(const GatedParams& p, float* h, bool dec, cudaStream_t s) {
  return dec ? launch_channels(ssm_gated_step_kernel<IO, true>, p, s, p, h) : launch_channels(ssm_gated_step_kernel<IO, false>, p, s, p, h);
}

// The largest unit that every row begins and ends on; for bf16 pairs of channels need pairs of float32 parameters and states too.
int unit(const ssm_gated_problem_t& p, const GatedParams& g) {
  const size_t esz = esize(p);
  uintptr_t bits = (uintptr_t)(g.D | g.ld_x | g.ld_gate | g.ld_in | g.ld_dx | g.ld_dgate | g.ld_din) * esz;
  for (const void* q : {g.x, g.gate, g.in_gate, (const void*)g.y, g.dy, (const void*)g.dx, (const void*)g.dgate, (const void*)g.din_gate})
    bits |= reinterpret_cast<uintptr_t>(q);
  if (esz == 2)
    for (const float* q : {g.A, g.h0, (const float*)g.h_last, (const float*)g.states, g.dh_last, (const float*)g.dA_part, (const float*)g.dh0})
      if (!aligned(q, 8)) return 2;
  return bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 2;
}

ssm_status_t status(cudaError_t e) { return e == cudaSuccess ? SSM_OK : SSM_ERR_CUDA; }

}  // namespace

}  // namespace ssm

using namespace ssm;

extern "C" {

size_t ssm_gated_saved_state_bytes(const ssm_gated_problem_t* p) { return validate(p) == SSM_OK ? state_bytes(*p) : 0; }

ssm_status_t ssm_gated_fwd(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate, const float* A,
                           const uint8_t* reset, const float* h0, void* y, float* h_last, float* saved_states,
                           void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool dec = decay(*p), save = p->flags & SSM_GATED_FLAG_SAVE_STATES;
  if (!x || !gate || !y || dec != (in_gate != nullptr) || dec != (A != nullptr) || save != (saved_states != nullptr))
    return SSM_ERR_INVALID_ARG;
  const size_t esz = esize(*p);
  for (const void* q : {x, gate, in_gate, (const void*)y})
    if (!aligned(q, esz)) return SSM_ERR_INVALID_ARG;
  for (const float* q : {A, h0, (const float*)h_last, (const float*)saved_states})
    if (!aligned(q, 4)) return SSM_ERR_INVALID_ARG;
  GatedParams g = params(*p);
  g.x = x;
  g.gate = gate;
  g.in_gate = in_gate;
  g.A = A;
  g.reset = reset;
  g.h0 = h0;
  g.y = y;
  g.h_last = h_last;
  g.states = saved_states;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return status(launch_gated_fwd(g, p->io_dtype, dec, unit(*p, g), s));
}

size_t ssm_gated_bwd_workspace_bytes(const ssm_gated_problem_t* p) {
  if (validate(p) != SSM_OK) return 0;
  const size_t parts = decay(*p) ? (size_t)p->batch * p->D * sizeof(float) : 0;
  return round16(parts) + (p->flags & SSM_GATED_FLAG_SAVE_STATES ? 0 : state_bytes(*p));
}

ssm_status_t ssm_gated_bwd(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate, const float* A,
                           const uint8_t* reset, const float* h0, const void* dy, const float* dh_last,
                           const float* saved_states, void* dx, void* dgate, void* din_gate, float* dA, float* dh0,
                           void* workspace, size_t workspace_bytes, void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool dec = decay(*p), saved = p->flags & SSM_GATED_FLAG_SAVE_STATES;
  if (!x || !gate || !dy || !dx || !dgate || dec != (in_gate != nullptr) || dec != (A != nullptr) ||
      dec != (din_gate != nullptr) || dec != (dA != nullptr) || saved != (saved_states != nullptr))
    return SSM_ERR_INVALID_ARG;
  const size_t esz = esize(*p);
  for (const void* q : {x, gate, in_gate, dy, (const void*)dx, (const void*)dgate, (const void*)din_gate})
    if (!aligned(q, esz)) return SSM_ERR_INVALID_ARG;
  for (const float* q : {A, h0, dh_last, saved_states, (const float*)dA, (const float*)dh0})
    if (!aligned(q, 4)) return SSM_ERR_INVALID_ARG;
  const size_t need = ssm_gated_bwd_workspace_bytes(p);
  if (need > 0 && (workspace == nullptr || !aligned(workspace, 16) || workspace_bytes < need)) return SSM_ERR_WORKSPACE;
  GatedParams g = params(*p);
  g.x = x;
  g.gate = gate;
  g.in_gate = in_gate;
  g.A = A;
  g.reset = reset;
  g.h0 = h0;
  g.dA_part = static_cast<float*>(workspace);
  g.states = const_cast<float*>(saved_states);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool bf16 = p->io_dtype == SSM_BF16;
  if (!saved) {
    g.states = reinterpret_cast<float*>(static_cast<char*>(workspace) + round16(dec ? (size_t)p->batch * p->D * sizeof(float) : 0));
    if (launch_gated_fwd(g, p->io_dtype, dec, unit(*p, g), s) != cudaSuccess) return SSM_ERR_CUDA;
  }
  g.dy = dy;
  g.dh_last = dh_last;
  g.dx = dx;
  g.dgate = dgate;
  g.din_gate = din_gate;
  g.dh0 = dh0;
  const cudaError_t e = bf16 ? launch_backward<__nv_bfloat16>(g, dec, s) : launch_backward<float>(g, dec, s);
  if (e != cudaSuccess) return SSM_ERR_CUDA;
  if (!dec) return SSM_OK;
  return status(launch_dependent(ssm_gated_reduce_kernel, (p->D + kThreads - 1) / kThreads, kThreads, 0, 1, s, g.dA_part, p->batch,
                                 p->D, dA));
}

ssm_status_t ssm_gated_step(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate, const float* A,
                            const uint8_t* reset, float* h, void* y, void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool dec = decay(*p);
  if (p->L != 1 || (p->flags & SSM_GATED_FLAG_SAVE_STATES) || !x || !gate || !h || !y || dec != (in_gate != nullptr) ||
      dec != (A != nullptr))
    return SSM_ERR_INVALID_ARG;
  const size_t esz = esize(*p);
  for (const void* q : {x, gate, in_gate, (const void*)y})
    if (!aligned(q, esz)) return SSM_ERR_INVALID_ARG;
  if (!aligned(A, 4) || !aligned(h, 4)) return SSM_ERR_INVALID_ARG;
  GatedParams g = params(*p);
  g.x = x;
  g.gate = gate;
  g.in_gate = in_gate;
  g.A = A;
  g.reset = reset;
  g.y = y;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return status(p->io_dtype == SSM_BF16 ? launch_step<__nv_bfloat16>(g, h, dec, s) : launch_step<float>(g, h, dec, s));
}

}  // extern "C"
