// Backward kernel of the gated linear recurrence (include/ssm_gated.h).
//
// The adjoint runs the other way and is affine like the forward recurrence: what leaves a run of steps towards the past is
// P c + R for what enters it from the future, c.  So the kernel is laid out like the forward one (ssm_gated_fwd.cu): a block walks
// tiles of 32 lanes of channels from the end of the sequence, every warp has kGatedSteps adjacent steps in registers, the warps' (P, R)
// meet in shared memory and those of the blocks of a cluster in one another's.  A warp's steps begin at a saved state, from which
// it runs the recurrence forward for the states that the gradients need; the gates are formed once, and what the gradients need of
// them waits in registers until the adjoint arrives.
//
// Decay form, with w = beta iota and inv = 1 / beta kept: iota = w inv, u / (1 - a^2) = iota inv x, so that
//     dx = mu w,  din_gate = dx x (1 - iota),  m = mu a (h[t-1] - a iota inv x),  dgate = m rho A (1 - rho),  dA = sum m rho
// take no special-function operation beyond the five of the gates.
//
// What bounds it: 10 or 14 bytes an element and the saved states, about 120 instructions for a pair of channels in the decay form,
// and the registers of what waits for the adjoint: ten values a step and pair, 168 in all, three blocks an SM ((8, 2048, 2560) bf16
// 155 us, 57 % of the copy bandwidth; four blocks of 128 registers 226, two 200; with A < -1 164).  The convex form keeps six and runs four
// blocks ((4, 2048, 5120) bf16 97 us, 66 %).
#include <cmath>
#include <type_traits>

#include "ssm_gated.cuh"

namespace ssm {

namespace {

constexpr int S = kGatedSteps;
constexpr int W = 4;                 // warps of a block
constexpr int kTile = S * W;

// The inputs of a warp's steps: a tile ahead, in two buffers of the warp's own in shared memory (see Feed in ssm_gated_fwd.cu; for
// COPY = 0 they pass through registers on the way there).
template <typename IO, class F, bool DECAY, int COPY>
struct Feed {
  using Raw = typename Lane<IO, F>::Raw;
  static constexpr int kTensors = DECAY ? 4 : 3;                        // x, gate, dy, in_gate
  static constexpr int kRow = 32 * (int)sizeof(Raw);
  static constexpr int kStage = kTensors * S * kRow;
  static constexpr int kBytes = 2 * kStage;
  static constexpr int kLanes = COPY == 16 ? kRow / 16 : 32;
  static constexpr int kRows = 32 / kLanes;

  const char* next[kTensors];   // this lane's first element (or chunk) in its first row of the next tile to fetch
  unsigned ld[kTensors];        // bytes
  char* buf;
  int lane;
  bool live;
  Raw raw[COPY > 0 ? 1 : kTensors][COPY > 0 ? 1 : S];

  __device__ __forceinline__ void init(const GatedParams& p, int64_t row, int d0, char* smem, int lane_) {
    lane = lane_;
    buf = smem;
    const int at = d0 + (COPY == 16 ? lane % kLanes * (16 / (int)sizeof(IO)) : lane * kWidth<F>);
    live = at < p.D;
    const void* const ptr[4] = {p.x, p.gate, p.dy, p.in_gate};
    const int64_t lds[4] = {p.ld_x, p.ld_gate, p.D, p.ld_in};
#pragma unroll
    for (int i = 0; i < kTensors; ++i) {
      ld[i] = (unsigned)(lds[i] * (int)sizeof(IO));
      next[i] = static_cast<const char*>(ptr[i]) + (row + lane / kLanes) * (int64_t)ld[i] + (live ? at : 0) * (int)sizeof(IO);
    }
  }
  template <bool ALL>
  __device__ __forceinline__ void rows(int n, int stage) {
#pragma unroll
    for (int i = 0; i < kTensors; ++i) {
#pragma unroll(COPY == 4 && sizeof(IO) == 2 ? 4 : S / kRows)   // (pairs of bf16: all eight need more registers than there are)
      for (int k = 0; k < S / kRows; ++k) {
        const int row = k * kRows + lane / kLanes;
        const char* src = next[i] + (uint64_t)ld[i] * (k * kRows);
        if constexpr (COPY > 0) {
          char* dst = buf + stage * kStage + (i * S + row) * kRow + lane % kLanes * COPY;
          const bool ok = live && (ALL || row < n);
          const char* from = ALL || row < n ? src : next[i];     // (not read where the row is not one)
          if constexpr (COPY == 16) cp_async16(dst, from, ok);
          else cp_async4(dst, from, ok);
        } else if (ALL || row < n) {
          raw[i][k] = *reinterpret_cast<const Raw*>(src);
        }
      }
    }
  }
  // fetches the next tile, n rows of it, and moves back by `step` rows
  __device__ __forceinline__ void issue(int n, int stage, int step) {
    if (n >= S) rows<true>(n, stage);
    else if (n > 0) rows<false>(n, stage);
    if constexpr (COPY > 0) cp_async_commit();
#pragma unroll
    for (int i = 0; i < kTensors; ++i) next[i] -= (uint64_t)ld[i] * step;
  }
  __device__ __forceinline__ void arrive(int stage) {
    if constexpr (COPY > 0) {
      asm volatile("cp.async.wait_group 1;" ::: "memory");
    } else {
#pragma unroll
      for (int i = 0; i < kTensors; ++i)
#pragma unroll
        for (int k = 0; k < S; ++k) *reinterpret_cast<Raw*>(buf + stage * kStage + (i * S + k) * kRow + lane * (int)sizeof(Raw)) = raw[i][k];
    }
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ void release() {
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ F get(int i, int k, int stage) const {
    return Lane<IO, F>::open(*reinterpret_cast<const Raw*>(buf + stage * kStage + (i * S + k) * kRow + lane * (int)sizeof(Raw)));
  }
};

// 1 - g of a gate g = sigma(z).  Where g is near 1 the difference cancels: its absolute error is up to 2.5 * 2^-25 (the sum 1 + e, the
// reciprocal and the difference are rounded), which is 3e-5 of it at z = kOpen, a hundredth of a bf16's rounding, and all of it at 17.
// e g has no such limit and takes another exponential (exact).  float32 io always forms it so where g is not small (it has twice the
// bytes to wait for).  With bf16 a warp looks for gates above kOpen among its own first: (8, 2048, 2560) 155 us where it finds none,
// 180 where every one is (154 and 181 if it never or always formed them so).
// CLAMP: e is held finite instead of the difference taken where g is small (g is 0 where that matters, and the gradients are products
// with it); 180 us against 187, but not for rows of pairs of bf16, (2, 2048, 1026) 33.5 against 31.6.
constexpr float kOpen = 6.f;
template <bool CLAMP, class F, class Exact>
__device__ __forceinline__ F rest(F z, F g, Exact exact) {   // exact: bool, or known when compiled
  const F near = vfma(g, vset<F>(-1.f), vset<F>(1.f));
  if constexpr (std::is_same<Exact, bool>::value) {
    if (!exact) return near;
  } else if constexpr (!Exact::value) {
    return near;
  }
  const F v = vmul(z, vset<F>(-kLog2e));
  if constexpr (CLAMP) return vmul(vmap(v, [](float v) { return ex2_approx(fminf(v, 126.f)); }), g);
  const F far = vmul(vmap(v, [](float v) { return ex2_approx(v); }), g);
  return vmap(g, near, far, [](float v, float n, float f) { return v < 0.5f ? n : f; });
}

template <typename IO, class F, bool DECAY, bool RESET, int COPY>
__global__ void __launch_bounds__(32 * W, DECAY ? 3 : 4) ssm_gated_bwd_kernel(const GatedParams p) {
  using Io = Lane<IO, F>;
  using Raw = typename Io::Raw;
  using In = Feed<IO, F, DECAY, COPY>;
  using Yes = std::true_type;
  using No = std::false_type;
  constexpr int V = kWidth<F>;
  constexpr int kAhead = COPY > 0 ? 2 : 1;           // tiles fetched before the first is looked at
  constexpr bool kLook = DECAY && sizeof(IO) == 2;   // whether a gate is above kOpen is asked
  constexpr bool kClamp = kLook && COPY == 16;
  extern __shared__ __align__(16) char s_feed[];
  __shared__ Affine<F> s_warp[2][W][32];
  __shared__ Affine<F> s_block[2][kGatedCluster][32];
  __shared__ uint64_t s_there[2];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int C = (int)cluster_size(), rank = (int)cluster_rank();
  const int tile = (int)(blockIdx.x / (unsigned)C);
  const int b = tile / p.tiles;
  const int d0 = (tile - b * p.tiles) * 32 * V, d = d0 + lane * V;
  const bool live = d < p.D;
  const int64_t row0 = (int64_t)b * p.L;
  const int rounds = (p.nck + W * C - 1) / (W * C);
  int q = p.nck - 1 - (rank * W + w);                // this warp's run of steps in the round: from the end towards 0, then below
  const int step = W * C;
  if (C > 1) {
    if (threadIdx.x == 0) set_up_barriers(s_there, 2);
    cluster_sync();
  }
  In in;
  in.init(p, row0 + (int64_t)q * S, d0, s_feed + w * In::kBytes, lane);
  dependency_wait();
  auto rows_of = [&](int k) { return k < 0 ? 0 : min(S, p.L - k * S); };

#pragma unroll
  for (int i = 0; i < kAhead; ++i) in.issue(rows_of(q - i * step), i, step * S);
  const uint8_t* __restrict__ pr = RESET ? p.reset + row0 : nullptr;
  auto mask_at = [&](int k) -> unsigned { return RESET && lane < rows_of(k) ? pr[k * S + lane] : 0u; };
  unsigned mask0 = mask_at(q), mask1 = mask_at(q - step);
  const float* __restrict__ ps = p.states + (int64_t)b * p.nck * p.D + d;
  auto state_at = [&](int k) { return live && k >= 0 ? *reinterpret_cast<const F*>(ps + (int64_t)k * p.D) : vset<F>(0.f); };
  F h0 = state_at(q), h1 = state_at(q - step);       // saved states of this run and the next
  F A = vset<F>(0.f), carry = vset<F>(0.f), dA = vset<F>(0.f);   // carry: what enters the round from the future
  int limit = !p.withhold ? kWaitLimit : rank > 0 ? kWithheldLimit : 0;   // of the waits; 0: one has been given up
  if (live) {
    if constexpr (DECAY) A = *reinterpret_cast<const F*>(p.A + d);
    if (p.dh_last != nullptr) carry = *reinterpret_cast<const F*>(p.dh_last + (int64_t)b * p.D + d);
  }
  bool small = false;                                // -1 <= A <= 0 in all of the warp's channels
  if constexpr (DECAY) {
    bool mine = true;
    vmap(A, [&](float v) { mine = mine && v >= -1.f && v <= 0.f; return v; });
    small = __all_sync(~0u, mine);
  }

  for (int r = 0; r < rounds; ++r, q -= step) {
    const int n = rows_of(q);
    const int half = r & 1, stage = COPY > 0 ? half : 0;
    // of each step: retention, state before it, and convex: g; decay: rho, w = beta iota, inv = 1 / beta
    F a[S], before[S], g[S], wi[DECAY ? S : 1], inv[DECAY ? S : 1];
    Affine<F> mine{vset<F>(1.f), vset<F>(0.f)};
    F most = vset<F>(0.f);                           // of the gates
    const unsigned cuts = RESET ? __ballot_sync(~0u, mask0 != 0) : 0u;
    mask0 = mask1;
    mask1 = mask_at(q - 2 * step);
    F h = h0;
    h0 = h1;
    h1 = state_at(q - 2 * step);
    in.arrive(stage);
    if constexpr (COPY == 0) in.issue(rows_of(q - step), 0, step * S);

    auto gates = [&](auto all_steps, auto small_A) {
      constexpr bool SMALL = decltype(small_A)::value;
      const F At = SMALL ? vmul(A, vset<F>(-1.f)) : A;
#pragma unroll
      for (int k = 0; k < S; ++k) {
        if (decltype(all_steps)::value || k < n) {
          const F x = in.get(0, k, stage), z = in.get(1, k, stage);
          F u;
          if constexpr (!DECAY) {
            gate_pair(z, g[k], a[k]);
            u = vmul(g[k], x);
          } else {
            F oa;
            g[k] = vmap(vadd(vmap(vmul(z, vset<F>(-kLog2e)), [](float v) { return ex2_approx(v); }), vset<F>(1.f)), [](float v) { return rcp_approx(v); });
            const F zi = in.get(DECAY ? 3 : 0, k, stage);
            if constexpr (kLook) most = vmap(most, z, zi, [](float v, float p, float q) { return fmaxf(v, fmaxf(p, q)); });
            const F iota = vmap(vadd(vmap(vmul(zi, vset<F>(-kLog2e)), [](float v) { return ex2_approx(v); }), vset<F>(1.f)),
                                [](float v) { return rcp_approx(v); });
            if constexpr (SMALL) decay_pair_small(vmul(g[k], At), a[k], oa);
            else decay_pair(vmul(g[k], At), a[k], oa);
            const F m2 = one_minus_square(oa);
            inv[k] = vmap(m2, [](float v) { return rsqrt_approx(v); });
            wi[k] = vmul(vmul(m2, inv[k]), iota);
            u = vmul(wi[k], x);
          }
          const bool cut = RESET && (cuts >> k & 1);
          before[k] = cut ? vset<F>(0.f) : h;
          h = cut ? u : vfma(a[k], h, u);
        }
      }
      // what enters from the future, through these steps
#pragma unroll
      for (int k = S - 1; k >= 0; --k) {
        if (decltype(all_steps)::value || k < n) {
          if (RESET && (cuts >> k & 1)) {
            mine = {vset<F>(0.f), vset<F>(0.f)};
          } else {
            mine.S = vmul(a[k], vadd(in.get(2, k, stage), mine.S));
            mine.P = vmul(a[k], mine.P);
          }
        }
      }
    };
    if (n >= S) {
      if (DECAY && small) gates(Yes{}, Yes{});
      else gates(Yes{}, No{});
    } else if (n > 0) {
      if (DECAY && small) gates(No{}, Yes{});
      else gates(No{}, No{});
    }
    if (!RESET || cuts == 0) mine.P = vmap(mine.P, [](float v) { return fmaxf(v, FLT_MIN); });

    s_warp[half][w][lane] = mine;
    if (C > 1 && threadIdx.x == 0 && limit > 0) barrier_expect(&s_there[half], C * 32 * sizeof(Affine<F>));
    __syncthreads();
    F c;
    if (C == 1) {
      c = carry;
#pragma unroll
      for (int j = 0; j < W; ++j) {
        if (j == w) c = carry;
        carry = apply<RESET>(s_warp[half][j][lane], carry);
      }
    } else {
      Affine<F> ahead{vset<F>(1.f), vset<F>(0.f)};
      if (w > 0) ahead = s_warp[half][0][lane];
#pragma unroll
      for (int j = 1; j < W - 1; ++j)
        if (j < w) ahead = then<RESET>(ahead, s_warp[half][j][lane]);
      if (w == W - 1 && limit > 0) {
        const Affine<F> all = then<RESET>(ahead, mine);
        for (int j = 0; j < C; ++j) send(remote_address(&s_block[half][rank][lane], j), remote_address(&s_there[half], j), all);
      }
      if (!barrier_wait(&s_there[half], r >> 1 & 1, limit)) {
        limit = 0;
        carry = vset<F>(NAN);
      }
      F enter = carry;
      for (int j = 0; j < C; ++j) {
        if (j == rank) enter = carry;
        carry = apply<RESET>(s_block[half][j][lane], carry);
      }
      c = w == 0 ? enter : apply<RESET>(ahead, enter);
      if (RESET && limit == 0) c = carry = vset<F>(NAN);
    }

    if (n > 0) {
      const int64_t row = row0 + (int64_t)q * S;
      const unsigned lx = (unsigned)(p.ld_dx * (int)sizeof(IO)), lg = (unsigned)(p.ld_dgate * (int)sizeof(IO)), li = (unsigned)(p.ld_din * (int)sizeof(IO));
      char* const ox = reinterpret_cast<char*>(static_cast<IO*>(p.dx) + row * p.ld_dx + d);
      char* const og = reinterpret_cast<char*>(static_cast<IO*>(p.dgate) + row * p.ld_dgate + d);
      char* const oi = DECAY ? reinterpret_cast<char*>(static_cast<IO*>(p.din_gate) + row * p.ld_din + d) : nullptr;
      auto gradients = [&](auto all_steps, auto exact) {
#pragma unroll
        for (int k = S - 1; k >= 0; --k) {
          if (decltype(all_steps)::value || k < n) {
            const F x = in.get(0, k, stage), mu = vadd(in.get(2, k, stage), c);
            const F back = vmul(mu, a[k]);           // a mu
            F dx, dg, di = vset<F>(0.f);
            if constexpr (!DECAY) {
              dx = vmul(mu, g[k]);
              dg = vmul(vmul(back, g[k]), vfma(before[k], vset<F>(-1.f), x));
            } else {
              const F iota = vmul(wi[k], inv[k]);
              dx = vmul(mu, wi[k]);
              di = vmul(vmul(dx, x), rest<kClamp>(in.get(DECAY ? 3 : 0, k, stage), iota, exact));
              const F m = vmul(vmul(back, vfma(vmul(a[k], vset<F>(-1.f)), vmul(vmul(iota, inv[k]), x), before[k])), g[k]);   // m rho
              dA = vadd(dA, m);
              dg = vmul(vmul(m, A), rest<kClamp>(in.get(1, k, stage), g[k], exact));
            }
            if (live) {
              *reinterpret_cast<Raw*>(ox + (uint64_t)lx * k) = Io::close(dx);
              *reinterpret_cast<Raw*>(og + (uint64_t)lg * k) = Io::close(dg);
              if constexpr (DECAY) *reinterpret_cast<Raw*>(oi + (uint64_t)li * k) = Io::close(di);
            }
            c = RESET && (cuts >> k & 1) ? vset<F>(0.f) : back;
          }
        }
      };
      if constexpr (kLook) {
        bool open = false;
        vmap(most, [&](float v) { open = open || v > kOpen; return v; });
        open = __any_sync(~0u, open);
        // Rows of whole 16 bytes take a body for either case (asked step by step 170 us instead of 156); for others, whose copies are
        // four times as many instructions, two bodies are the longer way ((2, 2048, 1026) 33 us against 31.5).
        if (n < S) gradients(No{}, open);
        else if constexpr (COPY != 16) gradients(Yes{}, open);
        else if (open) gradients(Yes{}, Yes{});
        else gradients(Yes{}, No{});
      } else {
        if (n >= S) gradients(Yes{}, Yes{});
        else gradients(No{}, Yes{});
      }
    }
    in.release();
    if constexpr (COPY > 0) in.issue(rows_of(q - 2 * step), half, step * S);
  }
  if (__any_sync(~0u, limit == 0)) cluster_sync();       // (waits for the blocks that have not left)
  if (p.dh0 != nullptr && live && w == 0 && rank == 0) *reinterpret_cast<F*>(p.dh0 + (int64_t)b * p.D + d) = carry;
  if constexpr (DECAY) {                             // the warps' sums of dA, in order
    __syncthreads();
    s_warp[0][w][lane].P = dA;
    __syncthreads();
    if (w == 0 && live) {
#pragma unroll
      for (int j = 1; j < W; ++j) dA = vadd(dA, s_warp[0][j][lane].P);
      *reinterpret_cast<F*>(p.dA_part + ((int64_t)b * C + rank) * p.D + d) = dA;
    }
  }
}

template <typename IO, class F, bool DECAY, bool RESET, int COPY>
cudaError_t launch(GatedParams p, int* parts, cudaStream_t s) {
  const auto kernel = ssm_gated_bwd_kernel<IO, F, DECAY, RESET, COPY>;
  constexpr size_t smem = (size_t)W * Feed<IO, F, DECAY, COPY>::kBytes;
  p.tiles = (p.D + 32 * kWidth<F> - 1) / (32 * kWidth<F>);
  KernelLimits lim;
  const cudaError_t e = kernel_limits(reinterpret_cast<const void*>(kernel), 32 * W, smem, &lim);
  if (e != cudaSuccess) return e;
  const long long tiles = (long long)p.tiles * p.batch;
  int c = choose_gated_cluster(tiles, p.L, kTile, (long long)lim.sms * lim.per_sm);
  const cudaError_t launched = launch_gated(kernel, tiles, 32 * W, smem, &c, s, p);
  *parts = p.batch * c;
  return launched;
}

template <typename IO, class F, int COPY>
cudaError_t launch_form(const GatedParams& p, bool decay, int* parts, cudaStream_t s) {
  if (p.reset != nullptr) return decay ? launch<IO, F, true, true, COPY>(p, parts, s) : launch<IO, F, false, true, COPY>(p, parts, s);
  return decay ? launch<IO, F, true, false, COPY>(p, parts, s) : launch<IO, F, false, false, COPY>(p, parts, s);
}

}  // namespace

cudaError_t launch_gated_bwd(const GatedParams& p, int io_dtype, bool decay, int unit, int* parts, cudaStream_t s) {
  if (io_dtype == SSM_BF16) {
    if (unit == 16) return launch_form<__nv_bfloat16, float2, 16>(p, decay, parts, s);
    return unit >= 4 ? launch_form<__nv_bfloat16, float2, 4>(p, decay, parts, s) : launch_form<__nv_bfloat16, float, 0>(p, decay, parts, s);
  }
  return unit == 16 ? launch_form<float, float, 16>(p, decay, parts, s) : launch_form<float, float, 4>(p, decay, parts, s);
}

}  // namespace ssm
