// Forward kernel of the gated linear recurrence (include/ssm_gated.h).
//
// What a step does to a state is affine, h -> a h + u, and so is what a run of steps does: h -> P h + S.  A block owns 32
// lanes of channels (one or two each) and walks the sequence in tiles; in a tile every one of its warps takes 16
// adjacent steps, forms their a and u once, in registers, and their (P, S).  The warps' pairs meet in shared memory, each warp
// folds those before it onto the state that entered the tile, and runs its steps again from there, which is one multiply-add
// each.  So x and the gates are read once and y written once, and a warp's loads for the next tile are under way while it does.
// Where the channels alone do not fill the GPU evenly, the blocks of a cluster take adjacent tiles of the same channels and
// send their tile's (P, S) into one another's shared memory, once a round.
//
// What bounds it: 6 (convex) or 8 (decay) bytes an element, 2 or 4 special-function operations and about 43 or 59 instructions for a
// pair of channels.  (4, 2048, 5120) bf16: convex 52 us, 74 % of the copy bandwidth, lost in the balance of its blocks ((4, 2048,
// 9472), whose groups of channels fill the GPU exactly, 91 %); decay 77 us, 67 %, fixed latencies at 9.6 warps an SM (162 registers; no pipe is above 50 %).
// A channel with A < -1 sends its warp through the general form of the gates: (8, 2048, 2560) 90 us instead of 77.
//
// P may underflow although no retention is zero, and zero times an infinite state would be NaN where the steps one by one
// keep it infinite: it is held at the least normal number, 2^-126 of the state at most, far below its rounding.  A step that
// resets makes P exactly zero, and zero stands for "nothing of the state passes", infinite or not.
#include <cmath>
#include <type_traits>

#include "ssm_gated.cuh"

namespace ssm {

namespace {

constexpr int S = 16;                // steps of a warp in a tile (8, with more warps an SM: decay 80 us against 76)
constexpr int W = 4;                 // warps of a block (8: 86)
constexpr int kTile = S * W;         // steps of a tile

// The inputs of a warp's steps on their way from global memory, a tile ahead: two buffers of half the steps each, of the warp's own
// in shared memory, that asynchronous copies of COPY bytes fill again as soon as they are read (16: a row of the warp's channels is cut
// among its lanes; 4: every lane copies what it will read itself); or, for COPY = 0, elements too small for such copies, registers.
template <typename IO, class F, bool DECAY, int COPY>
struct Feed {
  using Raw = typename Lane<IO, F>::Raw;
  static constexpr int kTensors = DECAY ? 3 : 2;
  static constexpr int kRow = 32 * (int)sizeof(Raw);                    // bytes of a row of the warp's channels
  static constexpr int kBytes = COPY > 0 ? kTensors * S * kRow : 0;     // of shared memory for a warp
  static constexpr int kLanes = COPY == 16 ? kRow / 16 : 32;            // lanes that copy a row
  static constexpr int kRows = 32 / kLanes;                             // rows that the warp copies at once

  const char* next[kTensors];   // this lane's first element (or chunk) in its first row of the next half to fetch
  int64_t ld[kTensors];         // bytes
  char* buf;
  int lane;
  bool live;                    // the lane's channels (or chunk) exist
  Raw raw[COPY > 0 ? 1 : kTensors][COPY > 0 ? 1 : S];

  __device__ __forceinline__ void init(const GatedParams& p, int64_t row, int d0, char* smem, int lane_) {
    lane = lane_;
    buf = smem;
    const int at = d0 + (COPY == 16 ? lane % kLanes * (16 / (int)sizeof(IO)) : lane * kWidth<F>);
    live = at < p.D;
    const void* const ptr[3] = {p.x, p.gate, p.in_gate};
    const int64_t lds[3] = {p.ld_x, p.ld_gate, p.ld_in};
#pragma unroll
    for (int i = 0; i < kTensors; ++i) {
      ld[i] = lds[i] * (int)sizeof(IO);
      next[i] = static_cast<const char*>(ptr[i]) + (row + lane / kLanes) * ld[i] + (live ? at : 0) * (int)sizeof(IO);
    }
  }
  template <int HALF, bool ALL>
  __device__ __forceinline__ void rows(int n) {
#pragma unroll
    for (int i = 0; i < kTensors; ++i) {
      const char* src = next[i];
#pragma unroll(COPY == 4 ? 4 : S / 2 / kRows)
      for (int k = 0; k < S / 2 / kRows; ++k, src += kRows * ld[i]) {
        const int row = k * kRows + lane / kLanes;
        if constexpr (COPY > 0) {
          char* dst = buf + ((i * 2 + HALF) * (S / 2) + row) * kRow + lane % kLanes * COPY;
          const bool ok = live && (ALL || row < n);
          const char* from = ALL || row < n ? src : next[i];     // (not read where the row is not one)
          if constexpr (COPY == 16) cp_async16(dst, from, ok);
          else cp_async4(dst, from, ok);
        } else if (ALL || row < n) {
          raw[i][HALF * (S / 2) + k] = *reinterpret_cast<const Raw*>(src);
        }
      }
    }
  }
  // fetches the next half of a tile, n rows (S / 2 at most), and moves on by `step` rows
  template <int HALF>
  __device__ __forceinline__ void issue(int n, int step) {
    if (n >= S / 2) rows<HALF, true>(n);
    else if (n > 0) rows<HALF, false>(n);
    if constexpr (COPY > 0) cp_async_commit();
#pragma unroll
    for (int i = 0; i < kTensors; ++i) next[i] += step * ld[i];
  }
  __device__ __forceinline__ void arrive() {   // the older half under way is there
    if constexpr (COPY > 0) asm volatile("cp.async.wait_group 1;" ::: "memory");
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ void release() {  // every lane has read its values
    if constexpr (COPY == 16) __syncwarp();
  }
  __device__ __forceinline__ Raw get(int i, int k) const {   // step k of the tile
    if constexpr (COPY > 0) return *reinterpret_cast<const Raw*>(buf + (i * S + k) * kRow + lane * (int)sizeof(Raw));
    else return raw[i][k];
  }
};

// Blocks of an SM: the decay form wants the registers of three ((2, 8192, 2560) bf16 84 us with four, 75 with three), with a
// mask it is faster with four ((8, 2048, 2560) 84 us, 91 with three), as is the convex form.
template <typename IO, class F, bool DECAY, bool RESET, int COPY>
__global__ void __launch_bounds__(32 * W, DECAY && !RESET ? 3 : 4) ssm_gated_fwd_kernel(const GatedParams p) {
  using Io = Lane<IO, F>;
  using Raw = typename Io::Raw;
  using In = Feed<IO, F, DECAY, COPY>;
  constexpr int V = kWidth<F>;
  extern __shared__ __align__(16) char s_feed[];
  __shared__ Affine<F> s_warp[2][W][32];
  __shared__ Affine<F> s_block[2][kGatedCluster][32];
  __shared__ uint64_t s_there[2];                    // one barrier for each half of s_block
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
  if (C > 1) {
    if (threadIdx.x == 0) set_up_barriers(s_there, 2);
    cluster_sync();                                  // (every block is there, its barriers set up)
  }
  In in;
  in.init(p, row0 + t0, d0, s_feed + w * In::kBytes, lane);
  dependency_wait();

  in.template issue<0>(p.L - t0, S / 2);
  in.template issue<1>(p.L - t0 - S / 2, step - S / 2);
  // bytes of the mask: those of the tile after the next are loaded where those of this one are looked at
  const uint8_t* __restrict__ pr = RESET ? p.reset + row0 : nullptr;
  auto mask_at = [&](int t) -> unsigned { return RESET && lane < S && t + lane < p.L ? pr[t + lane] : 0u; };
  unsigned mask0 = mask_at(t0), mask1 = mask_at(t0 + step);
  F A = vset<F>(0.f), carry = vset<F>(0.f);          // carry: the state that enters the round
  int limit = !p.withhold ? kWaitLimit : rank > 0 ? kWithheldLimit : 0;   // of the waits; 0: one has been given up
  if (live) {
    if constexpr (DECAY) A = *reinterpret_cast<const F*>(p.A + d);
    if (p.h0 != nullptr) carry = *reinterpret_cast<const F*>(p.h0 + (int64_t)b * p.D + d);
  }
  bool small = false;                                // -1 <= A <= 0 in all of the warp's channels
  if constexpr (DECAY) {
    bool mine = true;
    vmap(A, [&](float v) { mine = mine && v >= -1.f && v <= 0.f; return v; });
    small = __all_sync(~0u, mine);
  }

  for (int r = 0; r < rounds; ++r, t0 += step) {
    const int n = p.L - t0;                          // steps left from this warp's first one on (S or more: all of its)
    const int half = r & 1;
    F a[S], u[S];
    Affine<F> mine{vset<F>(1.f), vset<F>(0.f)};
    const unsigned cuts = RESET ? __ballot_sync(~0u, mask0 != 0) : 0u;   // bit k: step k of this warp resets
    mask0 = mask1;
    mask1 = mask_at(t0 + 2 * step);
    auto read = [&](auto first, auto all_steps, auto small_A) {   // steps first .. first + S / 2
      constexpr bool SMALL = decltype(small_A)::value;
      const F At = SMALL ? vmul(A, vset<F>(-1.f)) : A;
#pragma unroll
      for (int k = decltype(first)::value; k < decltype(first)::value + S / 2; ++k) {
        if (decltype(all_steps)::value || k < n) {
          const F x = Io::open(in.get(0, k));
          step_inputs<DECAY, SMALL>(x, Io::open(in.get(1, k)), DECAY ? Io::open(in.get(DECAY ? 2 : 0, k)) : x, At, a[k], u[k]);
          if (RESET && (cuts >> k & 1)) {
            mine = {vset<F>(0.f), u[k]};
          } else {
            mine.S = vfma(a[k], mine.S, u[k]);
            mine.P = vmul(a[k], mine.P);
          }
        }
      }
    };
    using Yes = std::true_type;
    using No = std::false_type;
    auto read_half = [&](auto first) {
      if (n >= S) {
        if (DECAY && small) read(first, Yes{}, Yes{});
        else read(first, Yes{}, No{});
      } else if (n > 0) {
        if (DECAY && small) read(first, No{}, Yes{});
        else read(first, No{}, No{});
      }
      in.release();
    };
    in.arrive();
    read_half(std::integral_constant<int, 0>{});
    in.template issue<0>(n - step, S / 2);
    in.arrive();
    read_half(std::integral_constant<int, S / 2>{});
    in.template issue<1>(n - step - S / 2, step - S / 2);
    if (!RESET || cuts == 0) mine.P = vmap(mine.P, [](float v) { return fmaxf(v, FLT_MIN); });

    s_warp[half][w][lane] = mine;
    if (C > 1 && threadIdx.x == 0 && limit > 0) barrier_expect(&s_there[half], C * 32 * sizeof(Affine<F>));
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
      Affine<F> before{vset<F>(1.f), vset<F>(0.f)};
      if (w > 0) before = s_warp[half][0][lane];
#pragma unroll
      for (int j = 1; j < W - 1; ++j)
        if (j < w) before = then<RESET>(before, s_warp[half][j][lane]);
      if (w == W - 1 && limit > 0) {
        const Affine<F> all = then<RESET>(before, mine);
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
      h = w == 0 ? enter : apply<RESET>(before, enter);
      if (RESET && limit == 0) h = carry = vset<F>(NAN);
    }

    if (live && n > 0) {
      float* __restrict__ keep = p.states != nullptr ? p.states + ((int64_t)b * p.nck + t0 / kGatedSteps) * p.D + d : nullptr;
      if (keep != nullptr || p.y != nullptr) {
        char* __restrict__ py = reinterpret_cast<char*>(static_cast<IO*>(p.y) + (row0 + t0) * p.D + d);
        const unsigned ld = (unsigned)p.D * (unsigned)sizeof(IO);
        auto write = [&](auto all_steps) {
#pragma unroll
          for (int k = 0; k < S; ++k) {
            if (decltype(all_steps)::value || k < n) {
              if (k % kGatedSteps == 0 && keep != nullptr) *reinterpret_cast<F*>(keep + (int64_t)(k / kGatedSteps) * p.D) = h;
              h = RESET && (cuts >> k & 1) ? u[k] : vfma(a[k], h, u[k]);
              if (p.y != nullptr) *reinterpret_cast<Raw*>(py + (uint64_t)ld * k) = Io::close(h);
            }
          }
        };
        if (n >= S) write(Yes{});
        else write(No{});
      }
    }
  }
  if (__any_sync(~0u, limit == 0)) cluster_sync();       // (waits for the blocks that have not left)
  if (p.h_last != nullptr && live && w == 0 && rank == 0) *reinterpret_cast<F*>(p.h_last + (int64_t)b * p.D + d) = carry;
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
  int c = choose_gated_cluster(tiles, p.L, kTile, (long long)lim.sms * lim.per_sm);
  return launch_gated(kernel, tiles, 32 * W, smem, &c, s, p);
}

template <typename IO, class F, int COPY>
cudaError_t launch_form(const GatedParams& p, bool decay, cudaStream_t s) {
  if (p.reset != nullptr) return decay ? launch<IO, F, true, true, COPY>(p, s) : launch<IO, F, false, true, COPY>(p, s);
  return decay ? launch<IO, F, true, false, COPY>(p, s) : launch<IO, F, false, false, COPY>(p, s);
}

}  // namespace

// A block takes a round's time and a half to get going, and the last blocks run faster when they are few, so that blocks in
// 2.2 turns cost less than in three: 0.3 of the whole turns and 0.7 of the exact ones fit what clusters of 1 to 8 blocks measured
// on 21 shapes of both kernels (the choice is 1 % off the best on the average, 6 % at most; clusters of two powers alone were 4 %
// and 20 %).  Clusters lie within a GPC and leave places unused: per cent of the SMs' places that they can take, measured with four blocks
// an SM; for the kernels with three it is an estimate ((1, 131072, 1536) runs in clusters of 12).
int choose_gated_cluster(long long groups, long long steps, int tile_steps, long long resident) {
  constexpr struct {
    int blocks, share;
  } kSizes[] = {{1, 100}, {2, 100}, {3, 95}, {4, 95}, {5, 93}, {6, 94}, {7, 90}, {8, 91}, {10, 92}, {12, 84}, {16, 80}};
  int best = 1;
  double best_cost = -1.;
  for (const auto& k : kSizes) {
    const long long places = resident * k.share / 100 / k.blocks;      // clusters at once
    if (places < 1) continue;
    const long long rounds = (steps + (long long)tile_steps * k.blocks - 1) / ((long long)tile_steps * k.blocks);
    const double exact = (double)groups / (double)places, whole = (double)((groups + places - 1) / places);
    const double turns = 0.3 * whole + 0.7 * exact;
    const double cost = (turns < 1. ? 1. : turns) * ((double)rounds + 1.5);
    if (best_cost < 0. || cost < best_cost) {
      best_cost = cost;
      best = k.blocks;
    }
  }
  return best;
}

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
