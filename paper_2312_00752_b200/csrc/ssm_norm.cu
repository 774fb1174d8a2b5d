// Norm of rows (layer norm, or without mean and bias) with the residual add in front of it, forward and backward.  See
// include/ssm_norm.h for the definition.
#include <cmath>
#include <type_traits>

#include "ssm_common.cuh"
#include "ssm_norm.h"
#include "ssm_pair.cuh"

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
  int withhold;              // test hook: the ring's first row stays incomplete, and is waited for briefly
  int group;                 // threads of a row: a power of two up to 32, or a multiple of 32 that is the whole block
};


// ------------------------------------------------------------------------------------------------------ rows in registers
// A group of threads holds a row: NV vectors of VE adjacent elements a thread, vector k of thread j at (k group + j) VE, so that the
// group's accesses are contiguous.  VE is 16 bytes of io, a pair of bf16 or one element, as the rows allow.
template <int VE>
using Val = typename std::conditional<VE == 1, float, float2>::type;   // what arithmetic is done on
template <int VE>
constexpr int kVals = VE == 1 ? 1 : VE / 2;
__device__ __forceinline__ float total(float v) { return v; }
__device__ __forceinline__ float total(float2 v) { return v.x + v.y; }

template <typename T, int VE>
struct Row {   // VE elements of type T as they lie in memory
  static constexpr int kBytes = VE * (int)sizeof(T);
  using Word = typename std::conditional<VE == 1, T, typename std::conditional<kBytes == 4, uint32_t, typename std::conditional<kBytes == 8, uint2, uint4>::type>::type>::type;
  static constexpr int kWords = kBytes <= 16 ? 1 : kBytes / 16;
  Word w[kWords];
  // Global memory; 32 bytes move at once: two accesses of 16 would each touch every second 16 bytes of the lines, and the float32
  // parameters of bf16 rows were what the L1's data path spent most of its time on (8192 x 5120 layer norm forward 41 us, 36 so).
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const Word* q = reinterpret_cast<const Word*>(static_cast<const T*>(base) + at);
    if constexpr (VE > 1 && kWords == 2) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y), "=r"(w[1].z), "=r"(w[1].w)
                   : "l"(q));
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = q[i];
    }
  }
  __device__ __forceinline__ void load_shared(const T* base, int at) {
    const Word* q = reinterpret_cast<const Word*>(base + at);
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = q[i];
  }
  __device__ __forceinline__ void store(void* base, int64_t at) const {
    Word* q = reinterpret_cast<Word*>(static_cast<T*>(base) + at);
    if constexpr (VE > 1 && kWords == 2) {
      asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(w[0].x), "r"(w[0].y), "r"(w[0].z), "r"(w[0].w), "r"(w[1].x),
                   "r"(w[1].y), "r"(w[1].z), "r"(w[1].w), "l"(q)
                   : "memory");
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) q[i] = w[i];
    }
  }
  __device__ __forceinline__ void get(Val<VE> (&v)[kVals<VE>]) const {
    if constexpr (VE == 1) {
      v[0] = io_to_float<T>(w[0]);
    } else if constexpr (kBytes == 4) {
      v[0] = make_float2(bf16lo(w[0]), bf16hi(w[0]));
    } else if constexpr (kBytes == 8) {
      v[0] = make_float2(__uint_as_float(w[0].x), __uint_as_float(w[0].y));
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint32_t r[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
        if constexpr (sizeof(T) == 4) {
          v[2 * i] = make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
          v[2 * i + 1] = make_float2(__uint_as_float(r[2]), __uint_as_float(r[3]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) v[4 * i + j] = make_float2(bf16lo(r[j]), bf16hi(r[j]));
        }
      }
    }
  }
  __device__ __forceinline__ void set(const Val<VE> (&v)[kVals<VE>]) {   // rounded to T
    if constexpr (VE == 1) {
      w[0] = float_to_io<T>(v[0]);
    } else if constexpr (kBytes == 4) {
      const __nv_bfloat162 c = __floats2bfloat162_rn(v[0].x, v[0].y);
      w[0] = *reinterpret_cast<const uint32_t*>(&c);
    } else if constexpr (kBytes == 8) {
      w[0] = make_uint2(__float_as_uint(v[0].x), __float_as_uint(v[0].y));
    } else {
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        uint32_t r[4];
        if constexpr (sizeof(T) == 4) {
          w[i] = make_uint4(__float_as_uint(v[2 * i].x), __float_as_uint(v[2 * i].y), __float_as_uint(v[2 * i + 1].x), __float_as_uint(v[2 * i + 1].y));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 c = __floats2bfloat162_rn(v[4 * i + j].x, v[4 * i + j].y);
            r[j] = *reinterpret_cast<const uint32_t*>(&c);
          }
          w[i] = make_uint4(r[0], r[1], r[2], r[3]);
        }
      }
    }
  }
};

// the thread within its group, the group within the block, groups of a block
__device__ __forceinline__ int lane_of(int group) { return group > 32 ? threadIdx.x : threadIdx.x & (group - 1); }
__device__ __forceinline__ int group_index(int group) { return group > 32 ? 0 : threadIdx.x >> (31 - __clz(group)); }
__device__ __forceinline__ int groups_of(int group) { return group > 32 ? 1 : blockDim.x >> (31 - __clz(group)); }

constexpr int kMaxWarps = 32;
// threads of a block, by vectors a thread: what the registers allow
constexpr int fwd_threads(int VE, int NV) { return VE * NV > 48 ? 384 : VE * NV > 16 ? 512 : 1024; }
constexpr int bwd_threads(int VE, int NV) {
  if (VE <= 2) return NV == 8 ? 512 : 768;
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

// MODE: 1 a residual is added, 2 there is a bias, 4 look at the pointers (the tests, and the residual's rounding where there is none,
// were a tenth of the instructions of a row)
template <typename IO, typename RES, int VE, int NV, int MODE>
__global__ void __launch_bounds__(fwd_threads(VE, NV)) ssm_norm_rows_fwd_kernel(const NormParams p) {
  __shared__ float s_sum[2][kMaxWarps][1];
  const int group = p.group, j = lane_of(group);
  const int64_t here = (int64_t)blockIdx.x * groups_of(group) + group_index(group);
  const bool live = here < p.rows;
  const int64_t at0 = (live ? here : 0) * p.D;          // (groups past the last row run along on the first)
  dependency_wait();
  const bool add = MODE & 4 ? p.residual != nullptr : MODE & 1, bias = MODE & 4 ? p.bias != nullptr : (MODE & 2) != 0;
  const bool keep = add && p.residual_out != nullptr && live;
  Row<IO, VE> x[NV];
  Row<RES, VE> s[NV];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D) {
      x[k].load(p.x, at0 + c);
      if (add) s[k].load(p.residual, at0 + c);
    }
  }
  using F = Val<VE>;
  constexpr int M = kVals<VE>;
  F acc = vset<F>(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D) {
      F v[M], a[M];
      x[k].get(v);
      if (add) {
        s[k].get(a);
#pragma unroll
        for (int i = 0; i < M; ++i) v[i] = vadd(v[i], a[i]);
      }
      s[k].set(v);
      if (add) s[k].get(v);
#pragma unroll
      for (int i = 0; i < M; ++i) acc = vadd(acc, v[i]);
      if (keep) s[k].store(p.residual_out, at0 + c);
    }
  }
  const float over = 1.f / (float)p.D;
  float m = 0.f, sum[1] = {total(acc)};
  if (!p.rms) {
    group_sum(sum, group, s_sum, 0);
    m = sum[0] * over;
  }
  const F off = vset<F>(-m);
  acc = vset<F>(0.f);
#pragma unroll
  for (int k = 0; k < NV; ++k)
    if ((k * group + j) * VE < p.D) {
      F v[M];
      s[k].get(v);
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const F c = vadd(v[i], off);
        acc = vfma(c, c, acc);
      }
    }
  sum[0] = total(acc);
  group_sum(sum, group, s_sum, 1);
  const float r = rsqrtf(fmaf(sum[0], over, p.eps));
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
    if (c < p.D && live) {
      Row<float, VE> w, b;
      Row<IO, VE> y;
      F v[M], wv[M], bv[M];
      s[k].get(v);
      w.load(p.weight, c);
      w.get(wv);
      if (bias) {
        b.load(p.bias, c);
        b.get(bv);
      }
#pragma unroll
      for (int i = 0; i < M; ++i) {
        const F xh = vmul(vadd(v[i], off), vset<F>(r));
        v[i] = bias ? vfma(xh, wv[i], bv[i]) : vmul(xh, wv[i]);
      }
      y.set(v);
      y.store(p.y, at0 + c);
    }
  }
  if (p.stats != nullptr && j == 0 && live) {
    p.stats[2 * here] = m;
    p.stats[2 * here + 1] = r;
  }
}

// the sum of a block's groups' column sums v, in order; s_part: [groups][D] where there is more than one
template <int VE, int NV>
__device__ __forceinline__ void block_parts(float* __restrict__ out, const Val<VE> (&v)[NV][kVals<VE>], int D, int group, float* s_part) {
  const int j = lane_of(group), groups = groups_of(group);
  if (groups > 1) __syncthreads();
  float* to = groups > 1 ? s_part + group_index(group) * D : out;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * group + j) * VE;
#pragma unroll
    for (int i = 0; i < kVals<VE>; ++i)
      if (c < D) *reinterpret_cast<Val<VE>*>(to + c + i * kWidth<Val<VE>>) = v[k][i];
  }
  if (groups == 1) return;
  __syncthreads();
  for (int c = threadIdx.x; c < D; c += blockDim.x) {
    float a = s_part[c];
    for (int q = 1; q < groups; ++q) a += s_part[q * D + c];
    out[c] = a;
  }
}

// Rows blockIdx.x (blockDim.x / group) + .., one grid of groups apart; the thread's columns stay the same, so dweight and dbias are
// summed in registers over all its rows, then over the groups of the block in order, and written as one part per block.  The next
// row is loaded before this one is reduced.
template <typename IO, typename RES, int VE, int NV, bool BIAS, bool FULL>
__global__ void __launch_bounds__(bwd_threads(VE, NV)) ssm_norm_rows_bwd_kernel(const NormParams p) {
  __shared__ float s_sum[2][kMaxWarps][2];
  extern __shared__ float s_part[];                      // groups of 32 threads or fewer: [groups][D]
  const int group = p.group, j = lane_of(group);
  const int groups = groups_of(group);
  const int64_t apart = (int64_t)gridDim.x * groups;
  const int64_t first = (int64_t)blockIdx.x * groups;    // (the block's groups run the same number of turns)
  int64_t here = first + group_index(group);
  const bool arrives = p.dresidual_out != nullptr, both = p.dresidual != nullptr;
  dependency_wait();
  using F = Val<VE>;
  constexpr int M = kVals<VE>;
  F dw[NV][M], db[BIAS ? NV : 1][M];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < M; ++i) {
      dw[k][i] = vset<F>(0.f);
      if constexpr (BIAS) db[k][i] = vset<F>(0.f);
    }
  Row<RES, VE> s[NV], sn[NV];
  Row<IO, VE> g[NV], gn[NV];
  float m = 0.f, r = 0.f, mn = 0.f, rn = 0.f;
  auto fetch = [&](int64_t row) {
    if (row < p.rows) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (FULL || c < p.D) {
          sn[k].load(p.s, row * p.D + c);
          gn[k].load(p.dy, row * p.D + c);
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
    if (arrives && live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (FULL || c < p.D) add[k].load(p.dresidual_out, here * p.D + c);
      }
    }
    fetch(here + apart);
    const F off = vset<F>(-m);
    F acc0 = vset<F>(0.f), acc1 = vset<F>(0.f);
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (FULL || c < p.D) {
          Row<float, VE> w;
          F wv[M], sv[M], yv[M];
          w.load(p.weight, c);
          w.get(wv);
          s[k].get(sv);
          g[k].get(yv);
#pragma unroll
          for (int i = 0; i < M; ++i) {
            const F q = vmul(yv[i], wv[i]), xh = vmul(vadd(sv[i], off), vset<F>(r));
            acc0 = vadd(acc0, q);
            acc1 = vfma(q, xh, acc1);
            dw[k][i] = vfma(yv[i], xh, dw[k][i]);
            if constexpr (BIAS) db[k][i] = vadd(db[k][i], yv[i]);
          }
        }
      }
    }
    float sum[2] = {total(acc0), total(acc1)};
    group_sum(sum, group, s_sum, turn);
    const float c1 = p.rms ? 0.f : sum[0] * over, c2 = sum[1] * over;
    if (live) {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int c = (k * group + j) * VE;
        if (FULL || c < p.D) {
          Row<float, VE> w;
          F wv[M], sv[M], yv[M];
          w.load(p.weight, c);
          w.get(wv);
          s[k].get(sv);
          g[k].get(yv);
#pragma unroll
          for (int i = 0; i < M; ++i) {
            const F xh = vmul(vadd(sv[i], off), vset<F>(r));
            sv[i] = vfma(vmul(yv[i], wv[i]), vset<F>(r), vfma(xh, vset<F>(-r * c2), vset<F>(-r * c1)));
          }
          if (arrives) {
            F av[M];
            add[k].get(av);
#pragma unroll
            for (int i = 0; i < M; ++i) sv[i] = vadd(sv[i], av[i]);
          }
          Row<IO, VE> dx;
          dx.set(sv);
          dx.store(p.dx, here * p.D + c);
          if (both) {
            Row<RES, VE> dr;
            dr.set(sv);
            dr.store(p.dresidual, here * p.D + c);
          }
        }
      }
    }
  }
  block_parts<VE, NV>(p.dw_part + (size_t)blockIdx.x * p.D, dw, p.D, group, s_part);
  if constexpr (BIAS) block_parts<VE, NV>(p.db_part + (size_t)blockIdx.x * p.D, db, p.D, group, s_part);
}

// ------------------------------------------------------------------------------------------------- rows through a ring
// The same for long rows of whole 16 bytes, with the whole block on one row: its tensors are brought to shared memory `stages` rows
// ahead, each by one bulk copy, which keeps enough bytes under way without a register for them.
__device__ __forceinline__ unsigned shared_address(const void* q) { return (unsigned)__cvta_generic_to_shared(q); }
__device__ __forceinline__ void bulk_load(const void* dst, const void* src, unsigned bytes, const uint64_t* barrier) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_address(dst)), "l"(src), "r"(bytes),
               "r"(shared_address(barrier))
               : "memory");
}
__device__ __forceinline__ void expect(const uint64_t* barrier, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(barrier)), "r"(bytes) : "memory");
}
// Waits for a row.  Its copies are under way when the wait begins, so that it ends; the limit (4 s) is for a fault elsewhere.  A thread that
// has given up waits and fetches no more, and makes NaN of its columns: of dx from this row on (of the whole row, by the sums), of
// its share of dweight and dbias.
constexpr int kWaitLimit = 1 << 20, kWithheldLimit = 1000;
__device__ __forceinline__ bool wait_full(const uint64_t* barrier, unsigned phase, int limit) {
  for (int i = 0; i < limit; ++i) {
    unsigned done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done)
                 : "r"(shared_address(barrier)), "r"(phase)
                 : "memory");
    if (done) return true;
  }
  return false;
}
constexpr int kMostStages = 4;

template <typename IO, typename RES, int VE, int NV, bool BIAS, bool FULL>
__global__ void __launch_bounds__(bwd_threads(VE, NV)) ssm_norm_ring_bwd_kernel(const NormParams p, int stages) {
  using F = Val<VE>;
  constexpr int M = kVals<VE>;
  __shared__ float s_sum[2][kMaxWarps][2];
  __shared__ uint64_t s_full[kMostStages];
  extern __shared__ __align__(128) char s_ring[];
  const int group = p.group, j = threadIdx.x;
  const bool add = p.dresidual_out != nullptr, both = p.dresidual != nullptr;
  const int sbytes = p.D * (int)sizeof(RES), ybytes = p.D * (int)sizeof(IO), bytes = sbytes + ybytes + (add ? sbytes : 0);
  if (threadIdx.x == 0) set_up_barriers(s_full, stages);
  __syncthreads();
  dependency_wait();
  const int limit = p.withhold ? kWithheldLimit : kWaitLimit;
  auto fill = [&](int64_t row, int stage) {                // thread 0
    if (row >= p.rows) return;
    char* dst = s_ring + stage * bytes;
    expect(&s_full[stage], bytes);
    bulk_load(dst, static_cast<const RES*>(p.s) + row * p.D, sbytes, &s_full[stage]);
    if (!(p.withhold && row < gridDim.x)) bulk_load(dst + sbytes, static_cast<const IO*>(p.dy) + row * p.D, ybytes, &s_full[stage]);
    if (add) bulk_load(dst + sbytes + ybytes, static_cast<const RES*>(p.dresidual_out) + row * p.D, sbytes, &s_full[stage]);
  };
  if (threadIdx.x == 0)
    for (int i = 0; i < stages - 1; ++i) fill(blockIdx.x + (int64_t)i * gridDim.x, i);
  F dw[NV][M], db[BIAS ? NV : 1][M];
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int i = 0; i < M; ++i) {
      dw[k][i] = vset<F>(0.f);
      if constexpr (BIAS) db[k][i] = vset<F>(0.f);
    }
  int stage = 0, turn = 0;
  unsigned phase = 0;
  const float over = 1.f / (float)p.D;
  int gave_up = 0;                                         // 1 + 2 stage + phase of the wait that ran out
  float mn = p.stats[2 * (int64_t)blockIdx.x], rn = p.stats[2 * (int64_t)blockIdx.x + 1];
  for (int64_t here = blockIdx.x; here < p.rows; here += gridDim.x, turn ^= 1) {
    const float m = mn, r = rn;
    if (here + gridDim.x < p.rows) {
      mn = p.stats[2 * (here + gridDim.x)];
      rn = p.stats[2 * (here + gridDim.x) + 1];
    }
    const char* at = s_ring + stage * bytes;
    const RES* bs = reinterpret_cast<const RES*>(at);
    const IO* by = reinterpret_cast<const IO*>(at + sbytes);
    const RES* ba = reinterpret_cast<const RES*>(at + sbytes + ybytes);
    if (gave_up == 0 && !wait_full(&s_full[stage], phase, limit)) gave_up = 1 + 2 * stage + (int)phase;
    const bool there = gave_up == 0;
    const F off = vset<F>(-m);
    F acc0 = vset<F>(there ? 0.f : NAN), acc1 = acc0;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * group + j) * VE;
      if (FULL || c < p.D) {
        Row<float, VE> w;
        Row<RES, VE> s;
        Row<IO, VE> y;
        F wv[M], sv[M], yv[M];
        w.load(p.weight, c);
        w.get(wv);
        s.load_shared(bs, c);
        s.get(sv);
        y.load_shared(by, c);
        y.get(yv);
#pragma unroll
        for (int i = 0; i < M; ++i) {
          const F q = vmul(yv[i], wv[i]), xh = vmul(vadd(sv[i], off), vset<F>(r));
          acc0 = vadd(acc0, q);
          acc1 = vfma(q, xh, acc1);
          dw[k][i] = vfma(yv[i], xh, dw[k][i]);
          if constexpr (BIAS) db[k][i] = vadd(db[k][i], yv[i]);
        }
      }
    }
    float sum[2] = {total(acc0), total(acc1)};
    group_sum(sum, group, s_sum, turn);
    // every thread is past the row before this one: its place is free
    if (threadIdx.x == 0 && there) fill(here + (int64_t)(stages - 1) * gridDim.x, stage == 0 ? stages - 1 : stage - 1);
    const float c1 = p.rms ? (there ? 0.f : NAN) : sum[0] * over, c2 = sum[1] * over;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * group + j) * VE;
      if (FULL || c < p.D) {
        Row<float, VE> w;
        Row<RES, VE> s;
        Row<IO, VE> y;
        F wv[M], sv[M], yv[M];
        w.load(p.weight, c);
        w.get(wv);
        s.load_shared(bs, c);
        s.get(sv);
        y.load_shared(by, c);
        y.get(yv);
#pragma unroll
        for (int i = 0; i < M; ++i) {
          const F xh = vmul(vadd(sv[i], off), vset<F>(r));
          sv[i] = vfma(vmul(yv[i], wv[i]), vset<F>(r), vfma(xh, vset<F>(-r * c2), vset<F>(-r * c1)));
        }
        if (add) {
          F av[M];
          s.load_shared(ba, c);
          s.get(av);
#pragma unroll
          for (int i = 0; i < M; ++i) sv[i] = vadd(sv[i], av[i]);
        }
        y.set(sv);
        y.store(p.dx, here * p.D + c);
        if (both) {
          s.set(sv);
          s.store(p.dresidual, here * p.D + c);
        }
      }
    }
    if (++stage == stages) {
      stage = 0;
      phase ^= 1;
    }
  }
  if (gave_up > 0) {
    // (thread 0: the copies under way were of this stage's row and of the stages - 2 after it)
    for (int i = 0; threadIdx.x == 0 && i < stages - 1; ++i) {
      const int at = (gave_up - 1) / 2 + i, back = at < stages ? at : at - stages;
      wait_full(&s_full[back], (unsigned)(((gave_up - 1) & 1) ^ (at < stages ? 0 : 1)), limit);
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < M; ++i) {
        dw[k][i] = vset<F>(NAN);
        if constexpr (BIAS) db[k][i] = vset<F>(NAN);
      }
  }
  block_parts<VE, NV>(p.dw_part + (size_t)blockIdx.x * p.D, dw, p.D, group, nullptr);
  if constexpr (BIAS) block_parts<VE, NV>(p.db_part + (size_t)blockIdx.x * p.D, db, p.D, group, nullptr);
}

// dweight and dbias from the blocks' parts, in a fixed order: 32 columns a block, its slices of threads take every kSlices-th part
constexpr int kSlices = 32;
__global__ void __launch_bounds__(32 * kSlices) ssm_norm_parts_kernel(const float* __restrict__ dw_part, const float* __restrict__ db_part, int parts,
                                                                    int D, float* __restrict__ dw, float* __restrict__ db) {
  __shared__ float s_sum[kSlices][32];
  dependency_wait();
  const int lane = threadIdx.x % 32, slice = threadIdx.x / 32;
  const int d = blockIdx.x * 32 + lane;
  const float* part = blockIdx.y == 0 ? dw_part : db_part;
  float a = 0.f;
  if (d < D) {
#pragma unroll 10
    for (int q = slice; q < parts; q += kSlices) a += part[(size_t)q * D + d];
  }
  s_sum[slice][lane] = a;
  __syncthreads();
  if (slice == 0 && d < D) {
    a = 0.f;
#pragma unroll
    for (int q = 0; q < kSlices; ++q) a += s_sum[q][lane];
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
  if (p->flags & ~(uint32_t)(SSM_NORM_FLAG_RMS | SSM_NORM_FLAG_HAS_BIAS | SSM_NORM_FLAG_HAS_RESIDUAL | SSM_NORM_FLAG_TEST_WITHHOLD)) return SSM_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f && p->eps <= 3.0e38f)) return SSM_ERR_INVALID_ARG;
  if (p->io_dtype != SSM_F32 && p->io_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  if (p->residual_dtype != SSM_F32 && p->residual_dtype != SSM_BF16) return SSM_ERR_UNSUPPORTED;
  if (p->residual_dtype != p->io_dtype) {
    if (!(p->flags & SSM_NORM_FLAG_HAS_RESIDUAL)) return SSM_ERR_INVALID_ARG;
    if (p->residual_dtype != SSM_F32) return SSM_ERR_UNSUPPORTED;
  }
  if (p->rows > INT32_MAX || p->D > 1 << 28) return SSM_ERR_UNSUPPORTED;   // (blocks of a grid; a row's columns, and a step past them, fit 32 bits)
  return SSM_OK;
}

size_t esize(int dtype) { return dtype == SSM_BF16 ? 2 : 4; }
bool aligned(const void* q, size_t a) { return reinterpret_cast<uintptr_t>(q) % a == 0; }
int parts_of(const ssm_norm_problem_t& p) { return (int)(p.rows < kMaxParts ? p.rows : kMaxParts); }
ssm_status_t status(cudaError_t e) { return e == cudaSuccess ? SSM_OK : SSM_ERR_CUDA; }

// How a row is spread over a group: NV vectors a thread.  0: it does not fit.
struct Spread {
  int nv, group;
};
int group_of(int vecs, int nv) {
  int g = (vecs + nv - 1) / nv;
  if (g > 32) return (g + 31) / 32 * 32;
  while (g & (g - 1)) ++g;
  return g;
}
// The most vectors a thread, of `most_nv` down, that leave no more than a tenth of the lanes idle beyond the least possible: the
// sums over a group cost more the more warps it has (8192 x 5120 bf16 layer norm forward with 5, 4, 2, 1 vectors: 40, 45, 62, 93 us).
Spread spread(int D, int VE, int most_nv, int (*most_threads)(int, int)) {
  const int vecs = (D + VE - 1) / VE;
  long long least = 0;
  for (int pass = 0; pass < 2; ++pass)
    for (int nv : {8, 5, 4, 3, 2, 1}) {
      if (nv > most_nv || (nv == 5 && most_threads == bwd_threads)) continue;
      const int g = group_of(vecs, nv);
      if (g > most_threads(VE, nv)) continue;
      const long long slots = (long long)nv * g;
      if (pass == 0) least = least == 0 || slots < least ? slots : least;
      else if (10 * slots <= 11 * least) return {nv, g};
    }
  return {0, 0};
}
// The ring's: the fewest vectors a thread, of those that leave the fewest lanes idle, with groups of at most 256 threads.
Spread ring_spread(int D, int VE) {
  const int vecs = (D + VE - 1) / VE;
  Spread best{0, 0};
  for (int nv = 1; nv <= 4; ++nv) {
    const int g = group_of(vecs, nv);
    if (g <= 256 && (best.nv == 0 || nv * g < best.nv * best.group)) best = {nv, g};
  }
  return best;
}
// no lane of the group idle: the backward kernels go without their tests of columns (3 to 5 %; the forward one keeps them, it
// holds the parameters in registers too early without: 8192 x 5120 42 us against 36)
bool even(const NormParams& p, int VE, int NV) { return p.D == NV * p.group * VE; }
int block_threads(int group) { return group > 32 ? group : 128; }

template <typename IO, typename RES, int VE, int NV>
cudaError_t launch_fwd_rows(const NormParams& p, cudaStream_t s) {
  const int threads = block_threads(p.group), rows = threads / p.group;
  const unsigned blocks = (unsigned)((p.rows + rows - 1) / rows);
  auto launch = [&](auto kernel) { return launch_dependent(kernel, blocks, threads, 0, 1, s, p); };
  if constexpr (VE > 2) {
    if (p.residual != nullptr)
      return p.bias != nullptr ? launch(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV, 3>) : launch(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV, 1>);
    if constexpr (std::is_same<IO, RES>::value)
      return p.bias != nullptr ? launch(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV, 2>) : launch(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV, 0>);
    return cudaErrorInvalidValue;                          // (a residual's type is that of x without one)
  } else {
    return launch(ssm_norm_rows_fwd_kernel<IO, RES, VE, NV, 4>);
  }
}

template <typename IO, typename RES, int VE>
cudaError_t launch_fwd_ve(NormParams p, cudaStream_t s) {
  // (single elements of long rows: the kernel for long rows is faster, bf16 8192 x 2561 37 us against 52)
  const Spread sp = VE == 1 && p.D > 2048 ? Spread{0, 0} : spread(p.D, VE, VE <= 2 ? 8 : sizeof(IO) == sizeof(RES) ? 5 : 4, fwd_threads);
  p.group = sp.group;
  switch (sp.nv) {
    case 1: return launch_fwd_rows<IO, RES, VE, 1>(p, s);
    case 2: return launch_fwd_rows<IO, RES, VE, 2>(p, s);
    case 3: return launch_fwd_rows<IO, RES, VE, 3>(p, s);
    case 4: return launch_fwd_rows<IO, RES, VE, 4>(p, s);
    case 5: return launch_fwd_rows<IO, RES, VE, 5>(p, s);
    case 8:
      if constexpr (VE <= 2) return launch_fwd_rows<IO, RES, VE, 8>(p, s);
      [[fallthrough]];
    default: return launch_dependent(ssm_norm_fwd_kernel<IO, RES>, (unsigned)p.rows, kNormThreads, 0, 1, s, p);
  }
}

// Rows of a block's ring: two at least, and more where the most blocks of an SM (eight) that have two leave room for them.
constexpr int kSharedBytes = 224 << 10;
int ring_stages(size_t bytes) {
  for (int blocks = 8; blocks >= 1; --blocks)
    for (int n = kMostStages; n >= 2; --n)
      if (blocks * (n * bytes + 2048) <= kSharedBytes) return n;
  return 0;
}
static_assert(2 * 4 * 256 * 8 * (4 + 2 + 4) + 2048 <= kSharedBytes && 2 * 4 * 256 * 4 * (4 + 4 + 4) + 2048 <= kSharedBytes,
              "two of the longest rows that ring_spread allows fit");

template <typename IO, typename RES, int VE, int NV, bool BIAS>
cudaError_t launch_bwd_ring(const NormParams& p, int* parts, cudaStream_t s) {
  const auto kernel = even(p, VE, NV) ? ssm_norm_ring_bwd_kernel<IO, RES, VE, NV, BIAS, true> : ssm_norm_ring_bwd_kernel<IO, RES, VE, NV, BIAS, false>;
  const size_t bytes = (size_t)p.D * (sizeof(IO) + (p.dresidual_out != nullptr ? 2 : 1) * sizeof(RES));
  const int stages = ring_stages(bytes);
  KernelLimits lim;
  const cudaError_t e = kernel_limits(reinterpret_cast<const void*>(kernel), p.group, stages * bytes, &lim);
  if (e != cudaSuccess) return e;
  const long long most = (long long)lim.sms * lim.per_sm, blocks = p.rows < most ? p.rows : most;
  *parts = (int)(blocks < kMaxParts ? blocks : kMaxParts);
  NormParams q = p;
  if constexpr (BIAS) q.db_part = q.dw_part + (size_t)*parts * p.D;
  return launch_dependent(kernel, (unsigned)*parts, p.group, stages * bytes, 1, s, q, stages);
}

template <typename IO, typename RES, int VE, int NV, bool BIAS>
cudaError_t launch_bwd_rows(const NormParams& p, int* parts, cudaStream_t s) {
  const auto kernel = even(p, VE, NV) ? ssm_norm_rows_bwd_kernel<IO, RES, VE, NV, BIAS, true> : ssm_norm_rows_bwd_kernel<IO, RES, VE, NV, BIAS, false>;
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
cudaError_t launch_bwd_nv(const NormParams& p, bool bias, bool ring, int* parts, cudaStream_t s) {
  if constexpr (VE > 2 && NV <= 4) {
    if (ring) return bias ? launch_bwd_ring<IO, RES, VE, NV, true>(p, parts, s) : launch_bwd_ring<IO, RES, VE, NV, false>(p, parts, s);
  }
  if constexpr (VE <= 2 || NV <= 2)
    return bias ? launch_bwd_rows<IO, RES, VE, NV, true>(p, parts, s) : launch_bwd_rows<IO, RES, VE, NV, false>(p, parts, s);
  return cudaErrorInvalidValue;
}

// Up to 192 threads of two vectors a row's next one waits in registers; where a row is longer the sums take so many that the ring
// is faster (layer norm with bias, 8192 rows of bf16: 5120 columns 66 us against 97, 4096 64 against 74, 2560 45 against 40).
template <typename IO, typename RES, int VE>
cudaError_t launch_bwd_ve(NormParams p, bool bias, int* parts, cudaStream_t s) {
  const bool ring = VE > 2 && p.D > 2 * 192 * VE;
  const Spread sp = ring ? ring_spread(p.D, VE) : spread(p.D, VE, VE <= 2 ? 8 : 2, bwd_threads);
  p.group = sp.group;
  switch (sp.nv) {
    case 1: return launch_bwd_nv<IO, RES, VE, 1>(p, bias, ring, parts, s);
    case 2: return launch_bwd_nv<IO, RES, VE, 2>(p, bias, ring, parts, s);
    case 3: return launch_bwd_nv<IO, RES, VE, 3>(p, bias, ring, parts, s);
    case 4: return launch_bwd_nv<IO, RES, VE, 4>(p, bias, ring, parts, s);
    case 8:
      if constexpr (VE <= 2) return launch_bwd_nv<IO, RES, VE, 8>(p, bias, false, parts, s);
      break;
    default: break;
  }
  *parts = (int)(p.rows < kMaxParts ? p.rows : kMaxParts);
  p.rows_per_part = (int)((p.rows + *parts - 1) / *parts);
  if (bias) p.db_part = p.dw_part + (size_t)*parts * p.D;
  const cudaError_t e = launch_dependent(ssm_norm_bwd_kernel<IO, RES>, (unsigned)p.rows, kNormThreads, 0, 1, s, p);
  if (e != cudaSuccess) return e;
  return launch_dependent(ssm_norm_params_kernel<IO, RES>, dim3((p.D + kNormThreads - 1) / kNormThreads, *parts), kNormThreads, 0, 1, s, p);
}

// Whether rows are whole `bytes` of io, at pointers that are aligned to an access: so many bytes, twice as many where a float32
// goes with a bf16.
template <typename IO, typename RES>
bool whole(const NormParams& p, int bytes) {
  uintptr_t bits = (uintptr_t)p.D * sizeof(IO);
  for (const void* q : {p.x, (const void*)p.y, p.dy, (const void*)p.dx}) bits |= reinterpret_cast<uintptr_t>(q);
  for (const void* q : {p.residual, (const void*)p.residual_out, p.s, p.dresidual_out, (const void*)p.dresidual})
    bits |= reinterpret_cast<uintptr_t>(q) * sizeof(IO) / sizeof(RES);
  for (const void* q : {(const void*)p.weight, (const void*)p.bias}) bits |= reinterpret_cast<uintptr_t>(q) * sizeof(IO) / sizeof(float);
  return bits % bytes == 0;
}

template <typename IO, typename RES>
cudaError_t launch_forward(const NormParams& p, cudaStream_t s) {
  if (whole<IO, RES>(p, 16)) return launch_fwd_ve<IO, RES, 16 / sizeof(IO)>(p, s);
  if constexpr (sizeof(IO) == 2)
    if (whole<IO, RES>(p, 4)) return launch_fwd_ve<IO, RES, 2>(p, s);
  return launch_fwd_ve<IO, RES, 1>(p, s);
}
template <typename IO, typename RES>
cudaError_t launch_backward(const NormParams& p, bool bias, int* parts, cudaStream_t s) {
  if (whole<IO, RES>(p, 16)) return launch_bwd_ve<IO, RES, 16 / sizeof(IO)>(p, bias, parts, s);
  if constexpr (sizeof(IO) == 2)
    if (whole<IO, RES>(p, 4)) return launch_bwd_ve<IO, RES, 2>(p, bias, parts, s);
  return launch_bwd_ve<IO, RES, 1>(p, bias, parts, s);
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
  n.withhold = p->flags & SSM_NORM_FLAG_TEST_WITHHOLD ? 1 : 0;
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
