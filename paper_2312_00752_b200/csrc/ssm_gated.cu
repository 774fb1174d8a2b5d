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
  float a, u;
  step_inputs<DECAY, false>(at<IO>(p.x, b, p.ld_x, d), at<IO>(p.gate, b, p.ld_gate, d), DECAY ? at<IO>(p.in_gate, b, p.ld_in, d) : 0.f,
                            DECAY ? p.A[d] : 0.f, a, u);
  const float h = p.reset != nullptr && p.reset[b] ? u : fmaf(a, hbuf[i], u);
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
  if (p->flags & ~(uint32_t)(SSM_GATED_FLAG_DECAY | SSM_GATED_FLAG_SAVE_STATES | SSM_GATED_FLAG_TEST_WITHHOLD)) return SSM_ERR_INVALID_ARG;
  if (p->io_dtype != SSM_F32 && p->io_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  const int64_t rows = (int64_t)p->batch * p->L;
  if (p->D > 1 << 28 || rows > INT64_MAX >> 32) return SSM_ERR_UNSUPPORTED;   // (byte offsets stay within 63 bits)
  for (int64_t ld : {p->ld_x, p->ld_gate, p->ld_in_gate, p->ld_dx, p->ld_dgate, p->ld_din_gate}) {
    if (ld != 0 && ld < p->D) return SSM_ERR_INVALID_ARG;
    if (ld > 1 << 28) return SSM_ERR_UNSUPPORTED;                 // (a row's bytes fit 32 bits)
  }
  if (!decay(*p) && (p->ld_in_gate != 0 || p->ld_din_gate != 0)) return SSM_ERR_INVALID_ARG;
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
  g.withhold = p.flags & SSM_GATED_FLAG_TEST_WITHHOLD ? 1 : 0;
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
size_t part_bytes(const ssm_gated_problem_t& p) { return decay(p) ? (size_t)p.batch * kGatedCluster * p.D * sizeof(float) : 0; }
size_t round16(size_t n) { return (n + 15) / 16 * 16; }

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
  return round16(part_bytes(*p)) + (p->flags & SSM_GATED_FLAG_SAVE_STATES ? 0 : state_bytes(*p));
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
  if (!saved) {
    g.states = reinterpret_cast<float*>(static_cast<char*>(workspace) + round16(part_bytes(*p)));
    if (launch_gated_fwd(g, p->io_dtype, dec, unit(*p, g), s) != cudaSuccess) return SSM_ERR_CUDA;
  }
  g.dy = dy;
  g.dh_last = dh_last;
  g.dx = dx;
  g.dgate = dgate;
  g.din_gate = din_gate;
  g.dh0 = dh0;
  int parts = 0;
  if (launch_gated_bwd(g, p->io_dtype, dec, unit(*p, g), &parts, s) != cudaSuccess) return SSM_ERR_CUDA;
  if (!dec) return SSM_OK;
  return status(launch_dependent(ssm_gated_reduce_kernel, (p->D + kThreads - 1) / kThreads, kThreads, 0, 1, s, g.dA_part, parts,
                                 p->D, dA));
}

ssm_status_t ssm_gated_step(const ssm_gated_problem_t* p, const void* x, const void* gate, const void* in_gate, const float* A,
                            const uint8_t* reset, float* h, void* y, void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool dec = decay(*p);
  if (p->L != 1 || (p->flags & ~(uint32_t)SSM_GATED_FLAG_DECAY) || !x || !gate || !h || !y || dec != (in_gate != nullptr) ||
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
