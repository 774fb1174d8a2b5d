// Norm of rows (layer norm, or without mean and bias) with the residual add in front of it, forward and backward.  See
// include/ssm_norm.h for the definition.
#include "ssm_common.cuh"
#include "ssm_norm.h"

namespace ssm {

namespace {

constexpr int kNormThreads = 256;

struct NormParams {
  const void* x;
  const void* residual;      // null: none
  const float* weight;
  const float* bias;         // null: none
  void* y;
  void* residual_out;        // null: not wanted
  float* stats;              // null: not wanted (forward)
  const void* s;             // backward
  const void* dy;
  const void* dresidual_out; // null: none
  void* dx;
  void* dresidual;           // null: not wanted
  float* dw_part;            // [parts][D]
  float* db_part;            // [parts][D]; null: none
  int64_t rows;
  int D, rms;
  float eps;
  int rows_per_part;
};

// the sum over a block, in every thread
__device__ __forceinline__ float block_sum(float v, float* scratch) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  __syncthreads();
  if (threadIdx.x % 32 == 0) scratch[threadIdx.x / 32] = v;
  __syncthreads();
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kNormThreads / 32; ++w) v += scratch[w];
  return v;
}

template <typename IO, typename RES>
__global__ void __launch_bounds__(kNormThreads) ssm_norm_fwd_kernel(const NormParams p) {
  __shared__ float scratch[kNormThreads / 32];
  dependency_wait();
  const int64_t row = blockIdx.x;
  const IO* x = static_cast<const IO*>(p.x) + row * p.D;
  const RES* res = p.residual != nullptr ? static_cast<const RES*>(p.residual) + row * p.D : nullptr;
  auto sum_at = [&](int d) {
    const float v = io_to_float<IO>(x[d]);
    return res == nullptr ? v : io_to_float<RES>(float_to_io<RES>(v + io_to_float<RES>(res[d])));
  };
  float m = 0.f;
  if (!p.rms) {
    for (int d = threadIdx.x; d < p.D; d += kNormThreads) m += sum_at(d);
    m = block_sum(m, scratch) / p.D;
  }
  float q = 0.f;
  for (int d = threadIdx.x; d < p.D; d += kNormThreads) {
    const float c = sum_at(d) - m;
    q = fmaf(c, c, q);
  }
  const float r = rsqrtf(block_sum(q, scratch) / p.D + p.eps);
  for (int d = threadIdx.x; d < p.D; d += kNormThreads) {
    const float s = sum_at(d);
    static_cast<IO*>(p.y)[row * p.D + d] = float_to_io<IO>(fmaf((s - m) * r, p.weight[d], p.bias != nullptr ? p.bias[d] : 0.f));
    if (p.residual_out != nullptr) static_cast<RES*>(p.residual_out)[row * p.D + d] = float_to_io<RES>(s);
  }
  if (p.stats != nullptr && threadIdx.x == 0) {
    p.stats[2 * row] = m;
    p.stats[2 * row + 1] = r;
  }
}

template <typename IO, typename RES>
__global__ void __launch_bounds__(kNormThreads) ssm_norm_bwd_kernel(const NormParams p) {
  __shared__ float scratch[kNormThreads / 32];
  dependency_wait();
  const int64_t row = blockIdx.x;
  const RES* s = static_cast<const RES*>(p.s) + row * p.D;
  const IO* dy = static_cast<const IO*>(p.dy) + row * p.D;
  const float m = p.stats[2 * row], r = p.stats[2 * row + 1];
  float c1 = 0.f, c2 = 0.f;
  for (int d = threadIdx.x; d < p.D; d += kNormThreads) {
    const float q = io_to_float<IO>(dy[d]) * p.weight[d];
    c1 += q;
    c2 = fmaf(q, (io_to_float<RES>(s[d]) - m) * r, c2);
  }
  c1 = p.rms ? 0.f : block_sum(c1, scratch) / p.D;
  c2 = block_sum(c2, scratch) / p.D;
  for (int d = threadIdx.x; d < p.D; d += kNormThreads) {
    const float q = io_to_float<IO>(dy[d]) * p.weight[d];
    const float xh = (io_to_float<RES>(s[d]) - m) * r;
    float ds = r * (q - c1 - xh * c2);
    if (p.dresidual_out != nullptr) ds += io_to_float<RES>(static_cast<const RES*>(p.dresidual_out)[row * p.D + d]);
    static_cast<IO*>(p.dx)[row * p.D + d] = float_to_io<IO>(ds);
    if (p.dresidual != nullptr) static_cast<RES*>(p.dresidual)[row * p.D + d] = float_to_io<RES>(ds);
  }
}

// partial sums of dweight and dbias over `rows_per_part` rows
template <typename IO, typename RES>
__global__ void __launch_bounds__(kNormThreads) ssm_norm_params_kernel(const NormParams p) {
  dependency_wait();
  const int d = blockIdx.x * kNormThreads + threadIdx.x;
  if (d >= p.D) return;
  const int64_t r0 = (int64_t)blockIdx.y * p.rows_per_part, r1 = min(p.rows, r0 + p.rows_per_part);
  float dw = 0.f, db = 0.f;
  for (int64_t row = r0; row < r1; ++row) {
    const float g = io_to_float<IO>(static_cast<const IO*>(p.dy)[row * p.D + d]);
    dw = fmaf(g, (io_to_float<RES>(static_cast<const RES*>(p.s)[row * p.D + d]) - p.stats[2 * row]) * p.stats[2 * row + 1], dw);
    db += g;
  }
  p.dw_part[(size_t)blockIdx.y * p.D + d] = dw;
  if (p.db_part != nullptr) p.db_part[(size_t)blockIdx.y * p.D + d] = db;
}

// dweight and dbias: the parts in ascending order
__global__ void __launch_bounds__(kNormThreads) ssm_norm_reduce_kernel(const float* __restrict__ dw_part, const float* __restrict__ db_part, int parts,
                                                                     int D, float* __restrict__ dw, float* __restrict__ db) {
  dependency_wait();
  const int d = blockIdx.x * kNormThreads + threadIdx.x;
  if (d >= D) return;
  float a = 0.f, b = 0.f;
  for (int q = 0; q < parts; ++q) {
    a += dw_part[(size_t)q * D + d];
    if (db_part != nullptr) b += db_part[(size_t)q * D + d];
  }
  dw[d] = a;
  if (db != nullptr) db[d] = b;
}

// ------------------------------------------------------------------------------------------------------- host side
constexpr int kMaxParts = 296;

ssm_status_t validate(const ssm_norm_problem_t* p) {
  if (p == nullptr || p->rows < 1 || p->D < 1) return SSM_ERR_INVALID_ARG;
  if (p->flags & ~(uint32_t)(SSM_NORM_FLAG_RMS | SSM_NORM_FLAG_HAS_BIAS | SSM_NORM_FLAG_HAS_RESIDUAL)) return SSM_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f && p->eps <= 3.0e38f)) return SSM_ERR_INVALID_ARG;
  if (p->io_dtype != SSM_F32 && p->io_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  if (p->residual_dtype != SSM_F32 && p->residual_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  if (p->residual_dtype != p->io_dtype) {
    if (!(p->flags & SSM_NORM_FLAG_HAS_RESIDUAL)) return SSM_ERR_INVALID_ARG;
    if (p->residual_dtype != SSM_F32) return SSM_ERR_UNSUPPORTED;
  }
  if (p->rows > INT32_MAX) return SSM_ERR_UNSUPPORTED;
  return SSM_OK;
}

size_t esize(int dtype) { return dtype == SSM_BF16 ? 2 : 4; }
bool aligned(const void* q, size_t a) { return reinterpret_cast<uintptr_t>(q) % a == 0; }
int parts_of(const ssm_norm_problem_t& p) { return (int)(p.rows < kMaxParts ? p.rows : kMaxParts); }
ssm_status_t status(cudaError_t e) { return e == cudaSuccess ? SSM_OK : SSM_ERR_CUDA; }

template <typename IO, typename RES>
cudaError_t launch_backward(const NormParams& p, int parts, cudaStream_t s) {
  cudaError_t e = launch_dependent(ssm_norm_bwd_kernel<IO, RES>, (unsigned)p.rows, kNormThreads, 0, 1, s, p);
  if (e != cudaSuccess) return e;
  return launch_dependent(ssm_norm_params_kernel<IO, RES>, dim3((p.D + kNormThreads - 1) / kNormThreads, parts), kNormThreads, 0, 1, s, p);
}

}  // namespace

}  // namespace ssm

using namespace ssm;

extern "C" {

ssm_status_t ssm_norm_fwd(const ssm_norm_problem_t* p, const void* x, const void* residual, const float* weight,
                          const float* bias, void* y, void* residual_out, float* stats, void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool res = p->flags & SSM_NORM_FLAG_HAS_RESIDUAL, has_bias = p->flags & SSM_NORM_FLAG_HAS_BIAS;
  if (!x || !weight || !y || res != (residual != nullptr) || has_bias != (bias != nullptr) || (!res && residual_out))
    return SSM_ERR_INVALID_ARG;
  const size_t esz = esize(p->io_dtype), rsz = esize(p->residual_dtype);
  if (!aligned(x, esz) || !aligned(y, esz) || !aligned(residual, rsz) || !aligned(residual_out, rsz)) return SSM_ERR_INVALID_ARG;
  if (!aligned(weight, 4) || !aligned(bias, 4) || !aligned(stats, 4)) return SSM_ERR_INVALID_ARG;
  NormParams n{};
  n.x = x;
  n.residual = residual;
  n.weight = weight;
  n.bias = bias;
  n.y = y;
  n.residual_out = residual_out;
  n.stats = stats;
  n.rows = p->rows;
  n.D = p->D;
  n.rms = p->flags & SSM_NORM_FLAG_RMS ? 1 : 0;
  n.eps = p->eps;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (p->io_dtype == SSM_F32) return status(launch_dependent(ssm_norm_fwd_kernel<float, float>, (unsigned)p->rows, kNormThreads, 0, 1, s, n));
  if (p->residual_dtype == SSM_F32)
    return status(launch_dependent(ssm_norm_fwd_kernel<__nv_bfloat16, float>, (unsigned)p->rows, kNormThreads, 0, 1, s, n));
  return status(launch_dependent(ssm_norm_fwd_kernel<__nv_bfloat16, __nv_bfloat16>, (unsigned)p->rows, kNormThreads, 0, 1, s, n));
}

size_t ssm_norm_bwd_workspace_bytes(const ssm_norm_problem_t* p) {
  if (validate(p) != SSM_OK) return 0;
  return (size_t)parts_of(*p) * p->D * sizeof(float) * (p->flags & SSM_NORM_FLAG_HAS_BIAS ? 2 : 1);
}

ssm_status_t ssm_norm_bwd(const ssm_norm_problem_t* p, const void* sum, const float* weight, const void* dy, const float* stats,
                          const void* dresidual_out, void* dx, void* dresidual, float* dweight, float* dbias, void* workspace,
                          size_t workspace_bytes, void* stream) {
  const ssm_status_t st = validate(p);
  if (st != SSM_OK) return st;
  const bool res = p->flags & SSM_NORM_FLAG_HAS_RESIDUAL, has_bias = p->flags & SSM_NORM_FLAG_HAS_BIAS;
  if (!sum || !weight || !dy || !stats || !dx || !dweight || has_bias != (dbias != nullptr) || (!res && dresidual_out) ||
      (p->residual_dtype == p->io_dtype && dresidual))
    return SSM_ERR_INVALID_ARG;
  const size_t esz = esize(p->io_dtype), rsz = esize(p->residual_dtype);
  if (!aligned(dy, esz) || !aligned(dx, esz)) return SSM_ERR_INVALID_ARG;
  for (const void* q : {sum, dresidual_out, (const void*)dresidual})
    if (!aligned(q, rsz)) return SSM_ERR_INVALID_ARG;
  for (const float* q : {weight, stats, (const float*)dweight, (const float*)dbias})
    if (!aligned(q, 4)) return SSM_ERR_INVALID_ARG;
  if (workspace == nullptr || !aligned(workspace, 16) || workspace_bytes < ssm_norm_bwd_workspace_bytes(p)) return SSM_ERR_WORKSPACE;
  NormParams n{};
  const int parts = parts_of(*p);
  n.s = sum;
  n.weight = weight;
  n.dy = dy;
  n.stats = const_cast<float*>(stats);
  n.dresidual_out = dresidual_out;
  n.dx = dx;
  n.dresidual = dresidual;
  n.dw_part = static_cast<float*>(workspace);
  n.db_part = has_bias ? n.dw_part + (size_t)parts * p->D : nullptr;
  n.rows = p->rows;
  n.D = p->D;
  n.rms = p->flags & SSM_NORM_FLAG_RMS ? 1 : 0;
  n.rows_per_part = (int)((p->rows + parts - 1) / parts);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t e;
  if (p->io_dtype == SSM_F32) e = launch_backward<float, float>(n, parts, s);
  else if (p->residual_dtype == SSM_F32) e = launch_backward<__nv_bfloat16, float>(n, parts, s);
  else e = launch_backward<__nv_bfloat16, __nv_bfloat16>(n, parts, s);
  if (e != cudaSuccess) return SSM_ERR_CUDA;
  return status(launch_dependent(ssm_norm_reduce_kernel, (p->D + kNormThreads - 1) / kNormThreads, kNormThreads, 0, 1, s, n.dw_part, n.db_part,
                                 parts, p->D, dweight, dbias));
}

}  // extern "C"
