// The gates of the gated linear recurrence (include/ssm_gated.h), on one channel (float) or a pair of channels (float2, whose
// sums and products issue two-wide), and what its kernels share.
#pragma once

#include <cfloat>

#include "ssm_common.cuh"
#include "ssm_gated.h"
#include "ssm_pair.cuh"

namespace ssm {

constexpr int kGatedSteps = 8;     // steps between two saved states
constexpr int kGatedCluster = 16;  // blocks of a cluster at most

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
  int withhold;           // test hook: the first block of a cluster has given up from the start, the others wait briefly
};

#ifdef __CUDACC__
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

// The same for -1 <= A <= 0, with w = -v in [0, 1]: (1 - exp(-w)) / w by its Chebyshev interpolation of degree 6, the constant
// term set to 1 (relative error 2.4e-8 at w = 1, less elsewhere: below half a unit), no special-function operation and no case distinction.
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
// one operation: with f = 1 + exp(-in_gate), m2 rsqrt(m2 f^2) = sqrt(m2) / f = beta iota (f^2 is infinite below an
// in_gate of -44 or less: then it is 0 instead of 1e-19 or less; the backward pass has iota by itself).
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
// ---------------------------------------------------------------------------------------------------- runs of steps
// What a run of steps does to the state that enters it: h -> P h + S.
template <class F>
struct alignas(2 * sizeof(F)) Affine {
  F P, S;
};

// the state behind a run of steps; RESET: P = 0 lets nothing pass
template <bool RESET, class F>
__device__ __forceinline__ F apply(const Affine<F>& k, F h) {
  const F r = vfma(k.P, h, k.S);
  if constexpr (!RESET) return r;
  return vmap(k.P, k.S, r, [](float P, float s, float v) { return P == 0.f ? s : v; });
}
template <bool RESET, class F>
__device__ __forceinline__ Affine<F> then(const Affine<F>& first, const Affine<F>& second) {
  Affine<F> r;
  r.S = apply<RESET>(second, first.S);
  r.P = vmul(second.P, first.P);
  if constexpr (RESET)
    r.P = vmap(r.P, first.P, second.P, [](float v, float a, float b) { return a == 0.f || b == 0.f ? 0.f : fmaxf(v, FLT_MIN); });
  else
    r.P = vmap(r.P, [](float v) { return fmaxf(v, FLT_MIN); });
  return r;
}

// --------------------------------------------------------------------------------------- between the blocks of a cluster
__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_size() {
  unsigned r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned shared_address(const void* q) { return (unsigned)__cvta_generic_to_shared(q); }
__device__ __forceinline__ unsigned remote_address(const void* local, unsigned rank) {   // the same place in block `rank`
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(shared_address(local)), "r"(rank));
  return r;
}
// A store into another block's shared memory that counts its bytes at a barrier there: the reader waits for the bytes, and the
// writer for nothing.  (A barrier of the whole cluster with its release waits for every store of y under way and every copy: 1.5
// of the 9.6 cycles between two instructions of a warp.)
__device__ __forceinline__ void send(unsigned to, unsigned barrier, const Affine<float>& v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to), "f"(v.P), "f"(v.S), "r"(barrier) : "memory");
}
__device__ __forceinline__ void send(unsigned to, unsigned barrier, const Affine<float2>& v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to), "f"(v.P.x), "f"(v.P.y),
               "f"(v.S.x), "f"(v.S.y), "r"(barrier)
               : "memory");
}
__device__ __forceinline__ void barrier_expect(const void* barrier, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(shared_address(barrier)), "r"(bytes) : "memory");
}
// Waits for the bytes of a phase.  The blocks of a cluster run at the same time and send before they wait, so that every wait
// ends; the limit (4 us a turn, 4 s) keeps a fault elsewhere from holding the GPU.  False: it was reached.  A thread that has given
// up sets its limit to 0.  It waits no more than one turn, expects no further bytes (the phase is still open) and sends none, so that
// the others give up as well, and the bytes that arrive uncounted are those of a round or two.  From there on its carry is NaN, which
// stays by itself but where a reset lets nothing pass, and its block stays until the others have left or given up too.
constexpr int kWaitLimit = 1 << 20, kWithheldLimit = 1000;
__device__ __forceinline__ bool barrier_wait(const void* barrier, unsigned phase, int limit) {
  int i = 0;
  do {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(shared_address(barrier)), "r"(phase)
        : "memory");
    if (done) return true;
  } while (++i < limit);
  return false;
}

__device__ __forceinline__ void cp_async4(void* dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(shared_address(dst)), "l"(src), "r"(valid ? 4 : 0) : "memory");
}


// Launches `kernel` with clusters of `c` blocks.  More than eight need the kernel's leave, and where a device has no room for
// them eight it is; *c: what it came to.
template <typename Kernel>
inline cudaError_t launch_gated(Kernel kernel, long long groups, int threads, size_t smem, int* c, cudaStream_t s, const GatedParams& p) {
  if (*c > 8) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess) e = launch_dependent(kernel, (unsigned)(groups * *c), threads, smem, *c, s, p);
    if (e == cudaSuccess) return e;
    (void)cudaGetLastError();
    *c = 8;
  }
  return launch_dependent(kernel, (unsigned)(groups * *c), threads, smem, *c, s, p);
}
#endif

// ------------------------------------------------------------------------------------------------------------ launches

// unit: bytes (16, 4 or, for bf16, 2) whose multiples the io pointers and the distances of rows are, D too
cudaError_t launch_gated_fwd(const GatedParams& p, int io_dtype, bool decay, int unit, cudaStream_t s);
// parts: how many rows of dA_part were written
cudaError_t launch_gated_bwd(const GatedParams& p, int io_dtype, bool decay, int unit, int* parts, cudaStream_t s);
// Blocks of a cluster that shares the tiles (of `tile_steps` each) of a group of channels; `groups` of them, `resident` blocks at once.
int choose_gated_cluster(long long groups, long long steps, int tile_steps, long long resident);

}  // namespace ssm
