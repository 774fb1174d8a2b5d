// Forward kernel of the gated linear recurrence (include/ssm_gated.h).
//
// What a step does to a state is affine, h -> a h + u, and so is what a run of steps does: h -> P h + S.  A block owns 32
// lanes of channels (one or two each) and walks the sequence in tiles; in a tile every one of its warps takes kGatedSteps
// adjacent steps, forms their a and u once, in registers, and their (P, S).  The warps' pairs meet in shared memory, each warp
// folds those before it onto the state that entered the tile, and runs its steps again from there, which is one multiply-add
// each.  So x and the gates are read once and y written once, and a warp's loads for the next tile are under way while it does.
// Where the channels alone do not fill the GPU, the blocks of a cluster take adjacent tiles of the same channels and hand
// their tile's (P, S) to one another through distributed shared memory: one cluster barrier a round, nothing waits on memory.
//
// P may underflow although no retention is zero, and zero times an infinite state would be NaN where the steps one by one
// keep it infinite: it is held at the least normal number, 2^-126 of the state at most, far below its rounding.  A step that
// resets makes P exactly zero, and zero stands for "nothing of the state passes", infinite or not.
#include <cfloat>

#include "ssm_gated.cuh"

namespace ssm {

namespace {

constexpr int S = kGatedSteps;
constexpr int W = 8;                 // warps of a block
constexpr int kTile = S * W;         // steps of a tile
constexpr int kMaxCluster = 8;

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
// stores to the same place in the shared memory of block `rank` of the cluster
__device__ __forceinline__ unsigned remote_address(const void* local, unsigned rank) {
  unsigned r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((unsigned)__cvta_generic_to_shared(local)), "r"(rank));
  return r;
}
__device__ __forceinline__ void remote_store(unsigned address, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(address), "f"(v) : "memory");
}
__device__ __forceinline__ void remote_store(unsigned address, float2 v) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(address), "f"(v.x), "f"(v.y) : "memory");
}

template <class F>
struct Affine {
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

template <typename IO, class F, bool DECAY, bool RESET>
__global__ void __launch_bounds__(32 * W) ssm_gated_fwd_kernel(const GatedParams p) {
  using Io = Lane<IO, F>;
  using Raw = typename Io::Raw;
  constexpr int V = kWidth<F>;
  __shared__ Affine<F> s_warp[2][W][32];
  __shared__ Affine<F> s_block[2][kMaxCluster][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int C = (int)cluster_size(), rank = (int)cluster_rank();
  const int tile = (int)(blockIdx.x / (unsigned)C);
  const int b = tile / p.tiles;
  const int d = ((tile - b * p.tiles) * 32 + lane) * V;
  const bool live = d < p.D;
  const int dc = live ? d : 0;                       // (lanes past the last channel run along on the first)
  const int64_t row0 = (int64_t)b * p.L;
  dependency_wait();

  const IO* __restrict__ px = static_cast<const IO*>(p.x) + row0 * p.ld_x + dc;
  const IO* __restrict__ pg = static_cast<const IO*>(p.gate) + row0 * p.ld_gate + dc;
  const IO* __restrict__ pi = DECAY ? static_cast<const IO*>(p.in_gate) + row0 * p.ld_in + dc : nullptr;
  const uint8_t* __restrict__ pr = RESET ? p.reset + row0 : nullptr;
  IO* __restrict__ py = static_cast<IO*>(p.y) + row0 * p.D + dc;
  F A = vset<F>(0.f);
  if constexpr (DECAY) A = *reinterpret_cast<const F*>(p.A + dc);
  F carry = vset<F>(0.f);                            // the state that enters the round
  if (p.h0 != nullptr) carry = *reinterpret_cast<const F*>(p.h0 + (int64_t)b * p.D + dc);

  Raw rx[S], rg[S], ri[DECAY ? S : 1];
  unsigned cut = 0;                                  // bit u: step u of this warp resets
  auto fetch = [&](int t0) {
    const int n = min(S, p.L - t0);
    if (n <= 0) return;
    const IO *qx = px + t0 * p.ld_x, *qg = pg + t0 * p.ld_gate, *qi = DECAY ? pi + t0 * p.ld_in : nullptr;
#pragma unroll
    for (int u = 0; u < S; ++u) {
      if (u < n) {
        rx[u] = *reinterpret_cast<const Raw*>(qx + u * p.ld_x);
        rg[u] = *reinterpret_cast<const Raw*>(qg + u * p.ld_gate);
        if constexpr (DECAY) ri[u] = *reinterpret_cast<const Raw*>(qi + u * p.ld_in);
      }
    }
    if constexpr (RESET) cut = __ballot_sync(~0u, lane < n && pr[t0 + min(lane, n - 1)] != 0);
  };

  const int rounds = (p.L + kTile * C - 1) / (kTile * C);
  fetch((rank * W + w) * S);
  for (int r = 0; r < rounds; ++r) {
    const int t0 = ((r * C + rank) * W + w) * S;
    const int n = min(S, p.L - t0);                  // steps of this warp (not above zero: none)
    F a[S], u[S];
    Affine<F> mine{vset<F>(1.f), vset<F>(0.f)};
    const unsigned cuts = RESET ? cut : 0u;
#pragma unroll
    for (int k = 0; k < S; ++k) {
      if (k < n) {
        step_inputs<DECAY>(Io::open(rx[k]), Io::open(rg[k]), DECAY ? Io::open(ri[DECAY ? k : 0]) : vset<F>(0.f), A, a[k], u[k]);
        if (RESET && (cuts >> k & 1)) {
          mine = {vset<F>(0.f), u[k]};
        } else {
          mine.S = vfma(a[k], mine.S, u[k]);
          mine.P = vmul(a[k], mine.P);
        }
      }
    }
    if (!RESET || cuts == 0) mine.P = vmap(mine.P, [](float v) { return fmaxf(v, FLT_MIN); });
    if (r + 1 < rounds) fetch(t0 + kTile * C);

    const int half = r & 1;
    s_warp[half][w][lane] = mine;
    __syncthreads();
    F h;
    if (C == 1) {
      h = carry;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if (j == w) h = carry;
        carry = apply<RESET>(s_warp[half][j][lane], carry);
      }
    } else {
      Affine<F> before{vset<F>(1.f), vset<F>(0.f)}, all = s_warp[half][0][lane];
#pragma unroll
      for (int j = 1; j < W; ++j) {
        if (j == w) before = all;
        all = then<RESET>(all, s_warp[half][j][lane]);
      }
      if (w < C) {                                   // warp w tells block w
        const unsigned to = remote_address(&s_block[half][rank][lane], w);
        remote_store(to, all.P);
        remote_store(to + sizeof(F), all.S);
      }
      cluster_sync();
      F in = carry;
      for (int j = 0; j < C; ++j) {
        if (j == rank) in = carry;
        carry = apply<RESET>(s_block[half][j][lane], carry);
      }
      h = w == 0 ? in : apply<RESET>(before, in);
    }

    if (live && n > 0) {
      if (p.states != nullptr) *reinterpret_cast<F*>(p.states + ((int64_t)b * p.nck + t0 / S) * p.D + d) = h;
      IO* __restrict__ qy = py + (int64_t)t0 * p.D;
      if (p.y != nullptr) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
          if (k < n) {
            h = RESET && (cuts >> k & 1) ? u[k] : vfma(a[k], h, u[k]);
            *reinterpret_cast<Raw*>(qy + (int64_t)k * p.D) = Io::close(h);
          }
        }
      }
    }
  }
  if (p.h_last != nullptr && live && w == 0 && rank == 0) *reinterpret_cast<F*>(p.h_last + (int64_t)b * p.D + d) = carry;
}

// Blocks of a cluster.  Blocks run in ceil(blocks / resident) turns of ceil(L / (cluster kTile)) rounds each.
int choose_cluster(long long tiles, int L, long long resident) {
  int best = 1;
  long long best_cost = -1;
  for (int c = 1; c <= kMaxCluster; c *= 2) {
    const long long rounds = (L + (long long)kTile * c - 1) / ((long long)kTile * c);
    const long long cost = (tiles * c + resident - 1) / resident * (rounds * (c > 1 ? 10 : 9) + 10);
    if (best_cost < 0 || cost < best_cost) {
      best_cost = cost;
      best = c;
    }
  }
  return best;
}

template <typename IO, class F, bool DECAY, bool RESET>
cudaError_t launch(GatedParams p, cudaStream_t s) {
  const auto kernel = ssm_gated_fwd_kernel<IO, F, DECAY, RESET>;
  p.tiles = (p.D + 32 * kWidth<F> - 1) / (32 * kWidth<F>);
  KernelLimits lim;
  const cudaError_t e = kernel_limits(reinterpret_cast<const void*>(kernel), 32 * W, 0, &lim);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.tiles * p.batch;
  const int c = choose_cluster(tiles, p.L, (long long)lim.sms * lim.per_sm);
  return launch_dependent(kernel, (unsigned)(tiles * c), 32 * W, 0, c, s, p);
}

template <typename IO, class F>
cudaError_t launch_form(const GatedParams& p, bool decay, cudaStream_t s) {
  if (p.reset != nullptr) return decay ? launch<IO, F, true, true>(p, s) : launch<IO, F, false, true>(p, s);
  return decay ? launch<IO, F, true, false>(p, s) : launch<IO, F, false, false>(p, s);
}

}  // namespace

cudaError_t launch_gated_fwd(const GatedParams& p, int io_dtype, bool decay, bool wide, cudaStream_t s) {
  if (io_dtype == SSM_BF16) return wide ? launch_form<__nv_bfloat16, float2>(p, decay, s) : launch_form<__nv_bfloat16, float>(p, decay, s);
  return wide ? launch_form<float, float2>(p, decay, s) : launch_form<float, float>(p, decay, s);
}

}  // namespace ssm
