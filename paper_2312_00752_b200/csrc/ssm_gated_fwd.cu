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
#include <type_traits>

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

// The inputs of a warp's steps on their way from global memory: kStages buffers of the warp's own in shared memory, filled by
// asynchronous copies of COPY bytes (16: a row of the warp's channels is cut among its lanes; otherwise every lane copies what it
// will read itself), or, for COPY = 0, elements too small for such copies, registers.
constexpr int kStages = 2;

__device__ __forceinline__ void copy_own(void* dst, const void* src, int bytes, std::integral_constant<int, 4>) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"((unsigned)__cvta_generic_to_shared(dst)), "l"(src), "r"(bytes) : "memory");
}

template <typename IO, class F, bool DECAY, int COPY>
struct Feed {
  using Raw = typename Lane<IO, F>::Raw;
  static constexpr int kTensors = DECAY ? 3 : 2;
  static constexpr int kRow = 32 * (int)sizeof(Raw);              // bytes of a row of the warp's channels
  static constexpr int kBytes = COPY > 0 ? kStages * kTensors * S * kRow : 0;   // of shared memory for a warp

  const IO* base[kTensors];   // this lane's first element (COPY = 16: of the chunk it copies) in the first row
  int64_t ld[kTensors];
  char* buf;
  int lane, live;             // live: the lane's channels (chunk) exist

  __device__ __forceinline__ void init(const GatedParams& p, int64_t row0, int d0, char* smem, int lane_) {
    lane = lane_;
    buf = smem;
    const int at = COPY == 16 ? d0 + (lane * 16 % kRow) / (int)sizeof(IO) : d0 + lane * kWidth<F>;
    live = at < p.D;
    const int64_t c = live ? at : 0;
    const void* const ptr[3] = {p.x, p.gate, p.in_gate};
    const int64_t lds[3] = {p.ld_x, p.ld_gate, p.ld_in};
#pragma unroll
    for (int i = 0; i < kTensors; ++i) {
      ld[i] = lds[i];
      base[i] = static_cast<const IO*>(ptr[i]) + row0 * ld[i] + c;
    }
  }
  // starts the copies of n rows (at most S) from t0 into buffer `stage`
  __device__ __forceinline__ void issue(int t0, int n, int stage) {
    if constexpr (COPY > 0) {
      constexpr int kLanes = COPY == 16 ? kRow / 16 : 32;         // lanes for one row
#pragma unroll
      for (int i = 0; i < kTensors; ++i) {
        char* dst = buf + (stage * kTensors + i) * S * kRow;
#pragma unroll
        for (int k = 0; k < S / (32 / kLanes); ++k) {
          const int row = k * (32 / kLanes) + lane / kLanes;
          const bool ok = live && row < n;
          const IO* src = base[i] + (ok ? (t0 + row) * ld[i] : 0);
          if constexpr (COPY == 16) cp_async16(dst + row * kRow + lane % kLanes * 16, src, ok);
          else copy_own(dst + row * kRow + lane * 4, src, ok ? 4 : 0, std::integral_constant<int, 4>{});
        }
      }
    }
    if constexpr (COPY > 0) cp_async_commit();
  }
  __device__ __forceinline__ void arrive() {   // the older of the two buffers under way is there
    if constexpr (COPY > 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ void release() {  // every lane has read its values
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ F get(int i, int k, int t0, int stage) const {
    if constexpr (COPY > 0) {
      return Lane<IO, F>::open(*reinterpret_cast<const Raw*>(buf + ((stage * kTensors + i) * S + k) * kRow + lane * (int)sizeof(Raw)));
    } else {
      return Lane<IO, F>::open(*reinterpret_cast<const Raw*>(base[i] + (t0 + k) * ld[i]));
    }
  }
};

template <typename IO, class F, bool DECAY, bool RESET, int COPY>
__global__ void __launch_bounds__(32 * W) ssm_gated_fwd_kernel(const GatedParams p) {
  using Io = Lane<IO, F>;
  using Raw = typename Io::Raw;
  using In = Feed<IO, F, DECAY, COPY>;
  constexpr int V = kWidth<F>;
  extern __shared__ __align__(16) char s_feed[];
  __shared__ Affine<F> s_warp[2][W][32];
  __shared__ Affine<F> s_block[2][kMaxCluster][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int C = (int)cluster_size(), rank = (int)cluster_rank();
  const int tile = (int)(blockIdx.x / (unsigned)C);
  const int b = tile / p.tiles;
  const int d0 = (tile - b * p.tiles) * 32 * V, d = d0 + lane * V;
  const bool live = d < p.D;
  const int64_t row0 = (int64_t)b * p.L;
  const int rounds = (p.L + kTile * C - 1) / (kTile * C);
  const int step = kTile * C;                        // from a tile to the next one of this block
  int t0 = (rank * W + w) * S;                       // this warp's first step in the round
  In in;
  in.init(p, row0, d0, s_feed + w * In::kBytes, lane);
  dependency_wait();

  in.issue(t0, p.L - t0, 0);
  in.issue(t0 + step, p.L - t0 - step, 1);
  // bytes of the mask: those of the step after the next are loaded where those of this one are looked at
  const uint8_t* __restrict__ pr = RESET ? p.reset + row0 : nullptr;
  auto mask_at = [&](int t) -> unsigned { return RESET && lane < S && t + lane < p.L ? pr[t + lane] : 0u; };
  unsigned mask0 = mask_at(t0), mask1 = mask_at(t0 + step);
  F A = vset<F>(0.f), carry = vset<F>(0.f);          // carry: the state that enters the round
  if (live) {
    if constexpr (DECAY) A = *reinterpret_cast<const F*>(p.A + d);
    if (p.h0 != nullptr) carry = *reinterpret_cast<const F*>(p.h0 + (int64_t)b * p.D + d);
  }

  for (int r = 0; r < rounds; ++r, t0 += step) {
    const int n = p.L - t0;                          // steps left from this warp's first one on (S or more: all of its)
    const int half = r & 1;
    F a[S], u[S];
    Affine<F> mine{vset<F>(1.f), vset<F>(0.f)};
    const unsigned cuts = RESET ? __ballot_sync(~0u, mask0 != 0) : 0u;   // bit k: step k of this warp resets
    mask0 = mask1;
    mask1 = mask_at(t0 + 2 * step);
    in.arrive();
    auto read = [&](auto all) {
#pragma unroll
      for (int k = 0; k < S; ++k) {
        if (decltype(all)::value || k < n) {
          step_inputs<DECAY>(in.get(0, k, t0, half), in.get(1, k, t0, half), DECAY ? in.get(DECAY ? 2 : 0, k, t0, half) : vset<F>(0.f), A, a[k], u[k]);
          if (RESET && (cuts >> k & 1)) {
            mine = {vset<F>(0.f), u[k]};
          } else {
            mine.S = vfma(a[k], mine.S, u[k]);
            mine.P = vmul(a[k], mine.P);
          }
        }
      }
    };
    if (n >= S) read(std::true_type{});
    else if (n > 0) read(std::false_type{});
    in.release();
    in.issue(t0 + 2 * step, n - 2 * step, half);
    if (!RESET || cuts == 0) mine.P = vmap(mine.P, [](float v) { return fmaxf(v, FLT_MIN); });

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
      F enter = carry;
      for (int j = 0; j < C; ++j) {
        if (j == rank) enter = carry;
        carry = apply<RESET>(s_block[half][j][lane], carry);
      }
      h = w == 0 ? enter : apply<RESET>(before, enter);
    }

    if (live && n > 0) {
      if (p.states != nullptr) *reinterpret_cast<F*>(p.states + ((int64_t)b * p.nck + t0 / S) * p.D + d) = h;
      if (p.y != nullptr) {
        IO* __restrict__ py = static_cast<IO*>(p.y) + (row0 + t0) * p.D + d;
        auto write = [&](auto all) {
#pragma unroll
          for (int k = 0; k < S; ++k) {
            if (decltype(all)::value || k < n) {
              h = RESET && (cuts >> k & 1) ? u[k] : vfma(a[k], h, u[k]);
              *reinterpret_cast<Raw*>(py) = Io::close(h);
              py += p.D;
            }
          }
        };
        if (n >= S) write(std::true_type{});
        else write(std::false_type{});
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

template <typename IO, class F, bool DECAY, bool RESET, int COPY>
cudaError_t launch(GatedParams p, cudaStream_t s) {
  const auto kernel = ssm_gated_fwd_kernel<IO, F, DECAY, RESET, COPY>;
  constexpr size_t smem = (size_t)W * Feed<IO, F, DECAY, COPY>::kBytes;
  p.tiles = (p.D + 32 * kWidth<F> - 1) / (32 * kWidth<F>);
  KernelLimits lim;
  const cudaError_t e = kernel_limits(reinterpret_cast<const void*>(kernel), 32 * W, smem, &lim);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.tiles * p.batch;
  const int c = choose_cluster(tiles, p.L, (long long)lim.sms * lim.per_sm);
  return launch_dependent(kernel, (unsigned)(tiles * c), 32 * W, smem, c, s, p);
}

template <typename IO, class F, int COPY>
cudaError_t launch_form(const GatedParams& p, bool decay, cudaStream_t s) {
  if (p.reset != nullptr) return decay ? launch<IO, F, true, true, COPY>(p, s) : launch<IO, F, false, true, COPY>(p, s);
  return decay ? launch<IO, F, true, false, COPY>(p, s) : launch<IO, F, false, false, COPY>(p, s);
}

}  // namespace

// Pairs of bf16 channels per lane (a row of a warp is a 128-byte line either way); float32 io has twice the bytes for the same
// arithmetic and does without packed instructions.
cudaError_t launch_gated_fwd(const GatedParams& p, int io_dtype, bool decay, int unit, cudaStream_t s) {
  if (io_dtype == SSM_BF16) {
    if (unit == 16) return launch_form<__nv_bfloat16, float2, 16>(p, decay, s);
    return unit >= 4 ? launch_form<__nv_bfloat16, float2, 4>(p, decay, s) : launch_form<__nv_bfloat16, float, 0>(p, decay, s);
  }
  return unit == 16 ? launch_form<float, float, 16>(p, decay, s) : launch_form<float, float, 4>(p, decay, s);
}

}  // namespace ssm
