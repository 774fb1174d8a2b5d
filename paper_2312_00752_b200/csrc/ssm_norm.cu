// Norm of rows (layer norm, or without mean and bias) with the residual add in front of it, forward and backward.  See
// include/ssm_norm.h for the definition.
#include "ssm_common.cuh"
#include "ssm_norm.h"

namespace ssm {

namespace {

constexpr int kNormThreads = 256;      // of the kernels for rows that do not fit a block's registers

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
  int rows_per_part;         // (the kernels for long rows)
  int group;                 // threads of a row: a power of two up to 32, or a multiple of 32 that is the whole block
};


// ------------------------------------------------------------------------------------------------------ rows in registers
// A group of threads holds a row: NV vectors of VE adjacent elements a thread, vector k of thread j at (k group + j) VE, so that the
// group's accesses are contiguous.  VE is 16 bytes of io, or one element where the rows do not allow such accesses.
template <typename T, int VE>
struct Row {   // VE elements of type T
  T v[VE];
};
template <typename T, int VE>
__device__ __forceinline__ void load(Row<T, VE>& r, const void* base, int64_t at) {
  const T* q = static_cast<const T*>(base) + at;
  if constexpr (VE * sizeof(T) % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)(VE * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(r.v)[i] = reinterpret_cast<const uint4*>(q)[i];
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) r.v[i] = q[i];
  }
}
template <typename T, int VE>
__device__ __forceinline__ void store(const Row<T, VE>& r, void* base, int64_t at) {
  T* q = static_cast<T*>(base) + at;
  if constexpr (VE * sizeof(T) % 16 == 0) {
#pragma unroll
    for (int i = 0; i < (int)(VE * sizeof(T) / 16); ++i) reinterpret_cast<uint4*>(q)[i] = reinterpret_cast<const uint4*>(r.v)[i];
  } else {
#pragma unroll
    for (int i = 0; i < VE; ++i) q[i] = r.v[i];
  }
}

constexpr int kMaxWarps = 32;
// threads of a block, by vectors a thread: what the registers allow
constexpr int fwd_threads(int VE, int NV) { return VE == 8 && NV == 4 ? 768 : 1024; }
constexpr int bwd_threads(int VE, int NV) {
  if (VE == 1) return 768;
  if (VE == 4) return NV == 1 ? 1024 : NV == 2 ? 640 : 384;
  return NV == 1 ? 768 : NV == 2 ? 384 : 256;
}

// sums of N values over the group, in every thread of it; s_sum: [2][kMaxWarps][N], `turn` alternates from call to call
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int group, float (*s_sum)[kMaxWarps][N], int turn) {
  for (int o = (group < 32 ? group : 32) / 2; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(~0u, v[i], o);
  if (group > 32) {
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) s_sum[turn][threadIdx.x / 32][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < group / 32; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += s_sum[turn][w][i];
  }
}

template <typename IO, typename RES, int VE, int NV>
__global__ void __launch_bounds__(fwd_threads(VE, NV)) ssm_norm_rows_fwd_kernel(const NormParams p) {
  __shared__ float s_sum[2][kMaxWarps][1];
  const int group = p.group, j = threadIdx.x % group;
  const int64_t here = (int64_t)blockIdx.x * (blockDim.x / group) + threadIdx.x / group;
  const bool live = here < p.rows;
  const int64_t at0 = (live ? here : 0) * p.D;          // (groups past the last row run along on the first)
  dependency_wait();
  const bool add = p.residual != nullptr;
  Row<IO, VE> x[NV];
  Row<RES, VE> s[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D) {
      load(x[k], p.x, at0 + c);
      if (add) load(s[k], p.residual, at0 + c);
    }
  }
  float sum[1] = {0.f};
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D) {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float v = io_to_float<IO>(x[k].v[i]);
        s[k].v[i] = float_to_io<RES>(add ? v + io_to_float<RES>(s[k].v[i]) : v);
        sum[0] += io_to_float<RES>(s[k].v[i]);
      }
      if (p.residual_out != nullptr && live) store(s[k], p.residual_out, at0 + c);
    }
  }
  float m = 0.f;
  if (!p.rms) {
    group_sum(sum, group, s_sum, 0);
    m = sum[0] / (float)p.D;
  }
  sum[0] = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if ((k * group + j) * VE < p.D)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        const float c = io_to_float<RES>(s[k].v[i]) - m;
        sum[0] = fmaf(c, c, sum[0]);
      }
  group_sum(sum, group, s_sum, 1);
  const float r = rsqrtf(sum[0] / (float)p.D + p.eps);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D && live) {
      Row<float, VE> w, b;
      Row<IO, VE> y;
      load(w, p.weight, c);
      if (p.bias != nullptr) load(b, p.bias, c);
#pragma unroll
      for (int i = 0; i < VE; ++i)
        y.v[i] = float_to_io<IO>(fmaf((io_to_float<RES>(s[k].v[i]) - m) * r, w.v[i], p.bias != nullptr ? b.v[i] : 0.f));
      store(y, p.y, at0 + c);
    }
  }
  if (p.stats != nullptr && j == 0 && live) {
    p.stats[2 * here] = m;
    p.stats[2 * here + 1] = r;
  }
}

// Rows blockIdx.x (blockDim.x / group) + .., one grid of groups apart; the thread's columns stay the same, so dweight and dbias are
// summed in registers over all its rows, then over the groups of the block in order, and written as one part per block.  The next
// row is loaded before this one is reduced.
template <typename IO, typename RES, int VE, int NV, bool BIAS>
__global__ void __launch_bounds__(bwd_threads(VE, NV)) ssm_norm_rows_bwd_kernel(const NormParams p) {
  __shared__ float s_sum[2][kMaxWarps][2];
  extern __shared__ float s_part[];                      // groups of 32 threads or fewer: [groups][D]
  const int group = p.group, j = threadIdx.x % group;
  const int groups = blockDim.x / group;
  const int64_t apart = (int64_t)gridDim.x * groups;
  const int64_t first = (int64_t)blockIdx.x * groups;    // (the block's groups run the same number of turns)
  int64_t here = first + threadIdx.x / group;
  dependency_wait();
  float dw[NV][VE], db[BIAS ? NV : 1][BIAS ? VE : 1];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      dw[k][i] = 0.f;
      if constexpr (BIAS) db[k][i] = 0.f;
    }
  Row<RES, VE> s[NV], sn[NV];
  Row<IO, VE> g[NV], gn[NV];
  float m = 0.f, r = 0.f, mn = 0.f, rn = 0.f;
  auto fetch = [&](int64_t row) {
    if (row < p.rows) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (c < p.D) {
          load(sn[k], p.s, row * p.D + c);
          load(gn[k], p.dy, row * p.D + c);
        }
      }
      mn = p.stats[2 * row];
      rn = p.stats[2 * row + 1];
    }
  };
  fetch(here);
  const float over = 1.f / (float)p.D;
  int turn = 0;
  for (int64_t row0 = first; row0 < p.rows; row0 += apart, here += apart, turn ^= 1) {
    const bool live = here < p.rows;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      s[k] = sn[k];
      g[k] = gn[k];
    }
    m = mn;
    r = rn;
    Row<RES, VE> add[NV];
    if (p.dresidual_out != nullptr && live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (c < p.D) load(add[k], p.dresidual_out, here * p.D + c);
      }
    }
    fetch(here + apart);
    float sum[2] = {0.f, 0.f};
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (c < p.D) {
          Row<float, VE> w;
          load(w, p.weight, c);
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            const float gy = io_to_float<IO>(g[k].v[i]), q = gy * w.v[i], xh = (io_to_float<RES>(s[k].v[i]) - m) * r;
            sum[0] += q;
            sum[1] = fmaf(q, xh, sum[1]);
            dw[k][i] = fmaf(gy, xh, dw[k][i]);
            if constexpr (BIAS) db[k][i] += gy;
          }
        }
      }
    }
    group_sum(sum, group, s_sum, turn);
    const float c1 = p.rms ? 0.f : sum[0] * over, c2 = sum[1] * over;
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (c < p.D) {
          Row<float, VE> w;
          load(w, p.weight, c);
          Row<IO, VE> dx;
          Row<RES, VE> dr;
#pragma unroll
          for (int i = 0; i < VE; ++i) {
            const float q = io_to_float<IO>(g[k].v[i]) * w.v[i], xh = (io_to_float<RES>(s[k].v[i]) - m) * r;
            float ds = r * (q - c1 - xh * c2);
            if (p.dresidual_out != nullptr) ds += io_to_float<RES>(add[k].v[i]);
            dx.v[i] = float_to_io<IO>(ds);
            dr.v[i] = float_to_io<RES>(ds);
          }
          store(dx, p.dx, here * p.D + c);
          if (p.dresidual != nullptr) store(dr, p.dresidual, here * p.D + c);
        }
      }
    }
  }
  auto put = [&](float* out, auto& v) {                  // the block's sum of the groups' v
    if (groups == 1) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
#pragma unroll
        for (int i = 0; i < VE; ++i)
          if (c + i < p.D) out[c + i] = v[k][i];
      }
      return;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * group + j) * VE;
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (c + i < p.D) s_part[threadIdx.x / group * p.D + c + i] = v[k][i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.D; c += blockDim.x) {
      float a = s_part[c];
      for (int q = 1; q < groups; ++q) a += s_part[q * p.D + c];
      out[c] = a;
    }
  };
  put(p.dw_part + (size_t)blockIdx.x * p.D, dw);
  if constexpr (BIAS) put(p.db_part + (size_t)blockIdx.x * p.D, db);
}

// dweight and dbias from the blocks' parts, in a fixed order: 32 columns a block, its slices of threads take every kSlices-th part
constexpr int kSlices = 8;
__global__ void __launch_bounds__(32 * kSlices) ssm_norm_parts_kernel(const float* __restrict__ dw_part, const float* __restrict__ db_part, int parts,
                                                                    int D, float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float s_sum[kSlices][32];
  dependency_wait();
  const int lane = threadIdx.x % 32, slice = threadIdx.x / 32;
  const int d = blockIdx.x * 32 + lane;
  const float* part = blockIdx.y == 0 ? dw_part : db_part;
  float a = 0.f;
  if (d < D) {
#pragma unroll 8
    for (int q = slice; q < parts; q += kSlices) a += part[(size_t)q * D + d];
  }
  s_sum[slice][lane] = a;
  __syncthreads();
  if (slice == 0 && d < D) {
#pragma unroll
    for (int q = 1; q < kSlices; ++q) a += s_sum[q][lane];
    (blockIdx.y == 0 ? dw : db)[d] = a;
  }
}

// ------------------------------------------------------------------------------------------------------------- long rows
// (read again from the caches in every pass)
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

// ------------------------------------------------------------------------------------------------------- host side
constexpr int kMaxParts = 148 * 4;

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

// How a row is spread: NV vectors a thread, the fewest lanes idle, more vectors a thread where that is even.  0: it does not fit.
struct Spread {
  int nv, group;
};
constexpr int kMostNv = 4;
Spread spread(int D, int VE, int (*most_threads)(int, int)) {
  const int vecs = (D + VE - 1) / VE;
  Spread best{0, 0};
  long long best_slots = 0;
  for (int nv = kMostNv; nv >= 1; --nv) {
    int g = (vecs + nv - 1) / nv;
    if (g > 32) g = (g + 31) / 32 * 32;
    else
      while (g & (g - 1)) ++g;
    if (g > most_threads(VE, nv)) continue;
    const long long slots = (long long)nv * g;
    if (best.nv == 0 || slots < best_slots) {
      best = {nv, g};
      best_slots = slots;
    }
  }
  return best;
}
int block_threads(int group) { return group > 32 ? group : 128; }

template <typename IO, typename RES, int VE, int NV>
cudaError_t launch_fwd_rows(const NormParams& p, cudaStream_t s) {
  const int threads = block_threads(p.group), rows = threads / p.group;
  return launch_dependent(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV>, (unsigned)((p.rows + rows - 1) / rows), threads, 0, 1, s, p);
}

template <typename IO, typename RES, int VE>
cudaError_t launch_fwd_ve(NormParams p, cudaStream_t s) {
  const Spread sp = spread(p.D, VE, fwd_threads);
  p.group = sp.group;
  switch (sp.nv) {
    case 1: return launch_fwd_rows<IO, RES, VE, 1>(p, s);
    case 2: return launch_fwd_rows<IO, RES, VE, 2>(p, s);
    case 3: return launch_fwd_rows<IO, RES, VE, 3>(p, s);
    case 4: return launch_fwd_rows<IO, RES, VE, 4>(p, s);
    default: return launch_dependent(ssm_norm_fwd_kernel<IO, RES>, (unsigned)p.rows, kNormThreads, 0, 1, s, p);
  }
}

template <typename IO, typename RES, int VE, int NV, bool BIAS>
cudaError_t launch_bwd_rows(const NormParams& p, int* parts, cudaStream_t s) {
  const auto kernel = ssm_norm_rows_bwd_kernel<IO, RES, VE, NV, BIAS>;
  const int threads = block_threads(p.group), rows = threads / p.group;
  const size_t smem = rows > 1 ? 128 * VE * NV * sizeof(float) : 0;     // rows p.D at most
  KernelLimits lim;
  const cudaError_t e = kernel_limits(reinterpret_cast<const void*>(kernel), threads, smem, &lim);
  if (e != cudaSuccess) return e;
  long long blocks = (p.rows + rows - 1) / rows;
  const long long most = (long long)lim.sms * lim.per_sm;
  if (blocks > most) blocks = most;
  if (blocks > kMaxParts) blocks = kMaxParts;
  *parts = (int)blocks;
  NormParams q = p;
  if constexpr (BIAS) q.db_part = q.dw_part + (size_t)blocks * p.D;
  return launch_dependent(kernel, (unsigned)blocks, threads, smem, 1, s, q);
}
template <typename IO, typename RES, int VE, int NV>
cudaError_t launch_bwd_nv(const NormParams& p, bool bias, int* parts, cudaStream_t s) {
  return bias ? launch_bwd_rows<IO, RES, VE, NV, true>(p, parts, s) : launch_bwd_rows<IO, RES, VE, NV, false>(p, parts, s);
}

template <typename IO, typename RES, int VE>
cudaError_t launch_bwd_ve(NormParams p, bool bias, int* parts, cudaStream_t s) {
  const Spread sp = spread(p.D, VE, bwd_threads);
  p.group = sp.group;
  switch (sp.nv) {
    case 1: return launch_bwd_nv<IO, RES, VE, 1>(p, bias, parts, s);
    case 2: return launch_bwd_nv<IO, RES, VE, 2>(p, bias, parts, s);
    case 3: return launch_bwd_nv<IO, RES, VE, 3>(p, bias, parts, s);
    case 4: return launch_bwd_nv<IO, RES, VE, 4>(p, bias, parts, s);
    default: break;
  }
  *parts = (int)(p.rows < kMaxParts ? p.rows : kMaxParts);
  p.rows_per_part = (int)((p.rows + *parts - 1) / *parts);
  if (bias) p.db_part = p.dw_part + (size_t)*parts * p.D;
  const cudaError_t e = launch_dependent(ssm_norm_bwd_kernel<IO, RES>, (unsigned)p.rows, kNormThreads, 0, 1, s, p);
  if (e != cudaSuccess) return e;
  return launch_dependent(ssm_norm_params_kernel<IO, RES>, dim3((p.D + kNormThreads - 1) / kNormThreads, *parts), kNormThreads, 0, 1, s, p);
}

// whether rows are whole 16 bytes at aligned pointers
template <typename IO>
bool wide(const NormParams& p) {
  uintptr_t bits = (uintptr_t)p.D * sizeof(IO);
  for (const void* q : {p.x, p.residual, (const void*)p.weight, (const void*)p.bias, (const void*)p.y, (const void*)p.residual_out, p.s, p.dy,
                        p.dresidual_out, (const void*)p.dx, (const void*)p.dresidual})
    bits |= reinterpret_cast<uintptr_t>(q);
  return bits % 16 == 0;
}

template <typename IO, typename RES>
cudaError_t launch_forward(const NormParams& p, cudaStream_t s) {
  return wide<IO>(p) ? launch_fwd_ve<IO, RES, 16 / sizeof(IO)>(p, s) : launch_fwd_ve<IO, RES, 1>(p, s);
}
template <typename IO, typename RES>
cudaError_t launch_backward(const NormParams& p, bool bias, int* parts, cudaStream_t s) {
  return wide<IO>(p) ? launch_bwd_ve<IO, RES, 16 / sizeof(IO)>(p, bias, parts, s) : launch_bwd_ve<IO, RES, 1>(p, bias, parts, s);
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
  if (p->io_dtype == SSM_F32) return status(launch_forward<float, float>(n, s));
  return status(p->residual_dtype == SSM_F32 ? launch_forward<__nv_bfloat16, float>(n, s) : launch_forward<__nv_bfloat16, __nv_bfloat16>(n, s));
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
  n.s = sum;
  n.weight = weight;
  n.dy = dy;
  n.stats = const_cast<float*>(stats);
  n.dresidual_out = dresidual_out;
  n.dx = dx;
  n.dresidual = dresidual;
  n.dw_part = static_cast<float*>(workspace);
  n.rows = p->rows;
  n.D = p->D;
  n.rms = p->flags & SSM_NORM_FLAG_RMS ? 1 : 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int parts = 0;
  cudaError_t e;
  if (p->io_dtype == SSM_F32) e = launch_backward<float, float>(n, has_bias, &parts, s);
  else if (p->residual_dtype == SSM_F32) e = launch_backward<__nv_bfloat16, float>(n, has_bias, &parts, s);
  else e = launch_backward<__nv_bfloat16, __nv_bfloat16>(n, has_bias, &parts, s);
  if (e != cudaSuccess) return SSM_ERR_CUDA;
  return status(launch_dependent(ssm_norm_parts_kernel, dim3((p->D + 31) / 32, has_bias ? 2 : 1), 32 * kSlices, 0, 1, s, n.dw_part,
                                 n.dw_part + (size_t)parts * p->D, parts, p->D, dweight, dbias));
}

}  // extern "C"
