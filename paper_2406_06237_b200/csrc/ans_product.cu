// Matrix product with its epilogue on the tensor cores:
//   Y[m][n] = act(x_scale[m] * w_scale[n] * sum_k X[m][k] W[n][k] + bias[n]) + residual[m][n]
//
// The operands are exchanged, Y^T = W X^T: 128 features of W are the 128-lane operand and the tokens
// (rows of X) the columns, so that a call with few tokens uses matrix instructions with few columns
// and reads W, which is what such a call is made of, in full tiles.  Both operands come by TMA in
// 128-byte rows (64 bf16 or 128 e4m3) into a ring of stages; one thread issues tcgen05.mma; sums
// stay in tensor memory in fp32.  Teams of four warps take them out: a thread holds one feature, so a warp's
// block of 32 tokens goes through its own 4 KB of shared memory (fp32, token-major) and leaves in rows of 32
// features, where the epilogue's operands (bias, scales of W) are constants of a thread and residual and
// Y are read and written in whole sectors.
//
// Two forms:
//   split:  one tile of 128 features x BN tokens a cluster of S CTAs; each sums a part of K and writes its sums of
//           every token into the shared memory of the CTA that finishes the token, which adds the S parts in the
//           order of the ranks: no workspace, no atomics, results do not vary from run to run.  Weights
//           that the caller calls settled are fetched before the work queued ahead is done.
//   whole:  persistent; a CTA (or a pair of CTAs on one tile of 256 features, cta_group::2) takes tile after
//           tile, the accumulators are double-buffered so that one tile's epilogue runs under the next one's products.
// Every wait is bounded; one that runs out sets ANS_STATUS_COPY_TIMEOUT and the kernel runs to its end.
#include <cuda.h>

#include <cmath>

#include <initializer_list>
#include <type_traits>

#include "ans_tensor.cuh"

namespace ansb {

using namespace ten;

constexpr uint32_t kPrRow = 128;                      // bytes of K per stage and row
constexpr uint32_t kPrFeatures = 128;                 // features of a CTA's tile

struct PrArgs {
  const float* x_scales; const float* w_scales; const float* bias;
  const void* residual; void* y;
  uint64_t residual_stride, y_stride;
  uint32_t M, N, steps;                               // steps: stages of K
  uint32_t tiles_f, tiles_t;
  int32_t activation;
  uint32_t settled;                                   // W may be read before the work queued ahead is done
  uint32_t wide;                                      // four features of Y (and residual) can be accessed at once
  uint32_t* status;
};

// NT times BN tokens a tile, BN a matrix instruction; CG CTAs on it; SPLIT: K is dealt over a cluster.
template <uint32_t BN, uint32_t NT, uint32_t CG, bool SPLIT>
struct PrShape {
  static constexpr uint32_t kTokens = NT * BN;        // of a tile
  static constexpr uint32_t kW = kPrFeatures * kPrRow;
  static constexpr uint32_t kBlockX = BN / CG * kPrRow;  // a pair's CTAs hold half of the tokens each
  static constexpr uint32_t kX = NT * kBlockX;
  static constexpr uint32_t kStage = kW + kX;
  static constexpr uint32_t kTeams = NT == 2u ? 4u : SPLIT && BN <= 64u ? 1u : 2u;    // teams of four epilogue warps, each with its part of the tokens
  // tokens that an epilogue warp takes out at a time, of its 32 features, and the bytes of such a block
  static constexpr uint32_t kBlock = NT == 2u || BN < 32u ? 16u : 32u;
  static constexpr uint32_t kScratch = kBlock * 32u * 4u;
  static constexpr uint32_t kTma = 4u * kTeams, kMma = kTma + 1u;     // the warps after them: copies, matrix instructions
  static constexpr uint32_t kThreads = 32u * (kMma + 1u);
  // whole: a block for each epilogue warp; split: what the cluster's CTAs send to this one
  static constexpr uint32_t kStagingBytes = SPLIT ? BN * kPrFeatures * 4u : 4u * kTeams * kScratch;
  // Up to 64 tokens a CTA takes half of an SM's shared memory at most, so that the next call's CTAs can start
  // beside it and fetch their weights; with more the ring has to be long enough for the matrix instructions' pace.
  static constexpr uint32_t kRoom = SPLIT && BN <= 64u ? 112u * 1024u : 227u * 1024u;
  static constexpr uint32_t kFit = (kRoom - 1024u - 512u - kStagingBytes) / kStage;
  static constexpr uint32_t kStages = kFit > 8u ? 8u : kFit;
  static constexpr uint32_t kAccs = SPLIT || kTokens > 256u ? 1u : 2u;  // tiles' accumulators in tensor memory
  static constexpr uint32_t kCols = kAccs * kTokens < 32u ? 32u : kAccs * kTokens;
  static constexpr uint32_t kSmem = 1024u + kStages * kStage + kStagingBytes + 512u;
};

// 2^x and 1/x to about 2^-22, subnormal results as zero
__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float inverse_fast(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The activation of N values; one branch for all of them.  All but relu are v * (a distribution function of v), with
// the function's small side computed as such: no difference of near-equal numbers.
template <uint32_t N>
__device__ __forceinline__ void activate(float (&v)[N], int32_t act) {
  switch (act) {
    case ANS_ACT_RELU:
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];            // a NaN stays
      break;
    case ANS_ACT_GELU:
      // Abramowitz and Stegun 7.1.26: erfc(z) = (a1 t + ... + a5 t^5) exp(-z^2) + e, t = 1 / (1 + p z), |e| <= 1.5e-7,
      // z = |v| / sqrt 2; the coefficients are halved
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) {
        const float z = fabsf(v[i]) * 0.70710678118654752f;
        const float t = inverse_fast(fmaf(0.3275911f, z, 1.f));
        float q = fmaf(0.5307027145f, t, -0.7265760135f);
        q = fmaf(q, t, 0.7107068705f);
        q = fmaf(q, t, -0.142248368f);
        q = fmaf(q, t, 0.127414796f);
        q = q * t * exp2_fast(z * z * -1.44269504089f);
        v[i] = v[i] * (v[i] < 0.f ? q : 1.f - q);
      }
      break;
    case ANS_ACT_GELU_TANH:
      // (1 + tanh u) / 2 = 1 / (1 + exp(-2u)); 2 sqrt(2 / pi) log2(e) = 2.3022082
#pragma unroll
      for (uint32_t i = 0; i < N; ++i)
        v[i] = v[i] * inverse_fast(1.f + exp2_fast(v[i] * fmaf(-0.10294324f * v[i], v[i], -2.30220820f)));
      break;
    case ANS_ACT_SILU:
#pragma unroll
      for (uint32_t i = 0; i < N; ++i) v[i] = v[i] * inverse_fast(1.f + exp2_fast(v[i] * -1.44269504089f));
      break;
    default: break;
  }
}

// The epilogue's constants of a thread: its four features f .. f + 3.
struct PrColumns {
  float bias[4], scale[4];
  __device__ __forceinline__ void load(const PrArgs& a, uint32_t f) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const bool in = f + i < a.N;
      bias[i] = a.bias && in ? *(a.bias + f + i) : 0.f;
      scale[i] = a.w_scales && in ? *(a.w_scales + f + i) : 1.f;
    }
  }
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// What the epilogue reads for features f .. f + 3 of the T tokens m, m + step, ... before `end`: the tokens' scales, and
// the residual where four features can be accessed at once.  Fetched ahead of the sums, without a branch between the
// loads (a token past the end stands for the last one).
template <uint32_t T, bool YF32>
struct PrAhead {
  uint4 r[T];                                          // bf16: x and y
  float xs[T];
  __device__ __forceinline__ void fetch(const PrArgs& a, uint32_t m, uint32_t step, uint32_t end, uint32_t f) {
#pragma unroll
    for (uint32_t j = 0; j < T; ++j) xs[j] = 1.f;
    if (m >= end) return;
    if (a.x_scales) {
#pragma unroll
      for (uint32_t j = 0; j < T; ++j) xs[j] = a.x_scales[min(m + j * step, end - 1u)];
    }
    if (a.residual && a.wide && f + 4 <= a.N) {
#pragma unroll
      for (uint32_t j = 0; j < T; ++j) {
        const uint64_t at = uint64_t(min(m + j * step, end - 1u)) * a.residual_stride + f;
        if constexpr (YF32) {
          r[j] = *reinterpret_cast<const uint4*>(static_cast<const float*>(a.residual) + at);
        } else {
          const uint2 q = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.residual) + at);
          r[j].x = q.x;
          r[j].y = q.y;
        }
      }
    }
  }
};

// Features f .. f + 3 of the T tokens m, m + step, ..., sums in v (four a token): scales, bias, activation,
// residual, one rounding, store.  Tokens from `end` on are left alone.
template <uint32_t T, bool YF32>
__device__ __forceinline__ void finish(const PrArgs& a, const PrColumns& c, const PrAhead<T, YF32>& p, uint32_t m, uint32_t step, uint32_t end,
                                       uint32_t f, float (&v)[4 * T]) {
  using Y = std::conditional_t<YF32, float, __nv_bfloat16>;
  if (f >= a.N || m >= end) return;
#pragma unroll
  for (uint32_t j = 0; j < T; ++j) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) v[4 * j + i] = fmaf(v[4 * j + i], p.xs[j] * c.scale[i], c.bias[i]);
  }
  activate<4 * T>(v, a.activation);
  Y* const y = static_cast<Y*>(a.y) + uint64_t(m) * a.y_stride + f;
  const uint64_t down = uint64_t(step) * a.y_stride;
  if (a.wide && f + 4 <= a.N) {
    if (a.residual) {
#pragma unroll
      for (uint32_t j = 0; j < T; ++j) {
        v[4 * j] += YF32 ? __uint_as_float(p.r[j].x) : bf16_lo(p.r[j].x);
        v[4 * j + 1] += YF32 ? __uint_as_float(p.r[j].y) : bf16_hi(p.r[j].x);
        v[4 * j + 2] += YF32 ? __uint_as_float(p.r[j].z) : bf16_lo(p.r[j].y);
        v[4 * j + 3] += YF32 ? __uint_as_float(p.r[j].w) : bf16_hi(p.r[j].y);
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < T; ++j) {
      uint4 u;
      if constexpr (YF32) {
        u = make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
      } else {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v[4 * j], v[4 * j + 1]), hi = __floats2bfloat162_rn(v[4 * j + 2], v[4 * j + 3]);
        u.x = *reinterpret_cast<const uint32_t*>(&lo);
        u.y = *reinterpret_cast<const uint32_t*>(&hi);
      }
      if (m + j * step < end) {
        if constexpr (YF32) *reinterpret_cast<uint4*>(y + j * down) = u;
        else *reinterpret_cast<uint2*>(y + j * down) = make_uint2(u.x, u.y);
      }
    }
  } else {
    const Y* const r = static_cast<const Y*>(a.residual) + uint64_t(m) * a.residual_stride + f;
    const uint64_t r_down = uint64_t(step) * a.residual_stride;
#pragma unroll
    for (uint32_t j = 0; j < T; ++j) {
      if (m + j * step >= end) break;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) {
        if (f + i >= a.N) break;
        const float u = a.residual ? v[4 * j + i] + static_cast<float>(r[j * r_down + i]) : v[4 * j + i];
        if constexpr (YF32) y[j * down + i] = u; else y[j * down + i] = __float2bfloat16_rn(u);
      }
    }
  }
}

// tile number -> tile of features, tile of tokens: groups of 8 feature tiles, so that the tiles in flight
// at one time share their operands in L2
__device__ __forceinline__ void tile_at(const PrArgs& a, uint32_t tile, uint32_t& tf, uint32_t& tt) {
  const uint32_t per = 8u * a.tiles_t, g = tile / per, in = tile - g * per;
  const uint32_t wide = min(8u, a.tiles_f - g * 8u);
  tt = in / wide;
  tf = g * 8u + (in - tt * wide);
}

template <uint32_t BN, uint32_t NT, uint32_t CG, bool F8, bool SPLIT, bool YF32>
__global__ void __launch_bounds__(PrShape<BN, NT, CG, SPLIT>::kThreads, 1)
ans_product_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const PrArgs a) {
  using S = PrShape<BN, NT, CG, SPLIT>;
  constexpr uint32_t kPerRow = F8 ? 128u : 64u;                        // elements of a stage's row
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t staging = base + S::kStages * S::kStage;
  const uint32_t bars = staging + S::kStagingBytes;
  const uint32_t full = bars, empty = bars + 8u * S::kStages, acc_full = bars + 16u * S::kStages, acc_empty = acc_full + 8u * S::kAccs;
  const uint32_t slot = acc_empty + 8u * S::kAccs;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint32_t rank = SPLIT || CG == 2 ? cluster_rank() : 0u;
  uint32_t ranks = 1;
  if constexpr (SPLIT) asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const uint32_t share = BN / ranks;                                   // split: tokens that a rank finishes; powers of two all
  uint32_t bad = 0;
  if constexpr (!SPLIT) let_next_start();

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < S::kStages; ++s) { bar_init(full + 8u * s, 1); bar_init(empty + 8u * s, 1); }
    for (uint32_t s = 0; s < S::kAccs; ++s) { bar_init(acc_full + 8u * s, 1); bar_init(acc_empty + 8u * s, 4u * S::kTeams * CG); }
    bar_init_fence();
  }
  if (warp == S::kMma) tmem_alloc<CG>(slot, S::kCols);
  if (threadIdx.x == 32u * S::kTma && a.steps) { map_prefetch(&w_map); map_prefetch(&x_map); }
  fence_before();
  if constexpr (CG == 2) cluster_sync(); else __syncthreads();
  if (SPLIT && ranks > 1) cluster_arrive();                            // waited for before the first store into another CTA
  fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

  // this CTA's tiles, and its part of K
  const uint32_t tiles = a.tiles_f * a.tiles_t;
  const uint32_t team = SPLIT ? blockIdx.x / ranks : blockIdx.x / CG, teams = SPLIT ? tiles : gridDim.x / CG;
  const uint32_t k0 = SPLIT ? static_cast<uint32_t>(uint64_t(a.steps) * rank / ranks) : 0u;
  const uint32_t k1 = SPLIT ? static_cast<uint32_t>(uint64_t(a.steps) * (rank + 1u) / ranks) : a.steps;

  // split: the tokens that this CTA finishes, and the first of a warp's
  constexpr uint32_t kEach = BN < 64u ? 2u : 4u;                       // tokens of a warp at a time
  uint32_t f_mine = 0, first = 0, here = 0;
  PrColumns own;
  PrAhead<kEach, YF32> mine;
  if constexpr (SPLIT) {
    uint32_t tf, tt;
    tile_at(a, team, tf, tt);
    const uint32_t live = min(BN, a.M - tt * BN);
    f_mine = tf * kPrFeatures + 4u * lane;
    first = tt * BN + rank * share;
    here = live > rank * share ? min(share, live - rank * share) : 0u;
  }

  if (warp == S::kTma) {
    if (lane == 0) {
      uint32_t n = 0, early = 0;                                       // stages filled so far; those with W alone
      if (SPLIT && a.settled) {
        uint32_t tf, tt;
        tile_at(a, team, tf, tt);
        early = min(S::kStages, k1 - k0);
        for (uint32_t s = 0; s < early; ++s) {
          bar_expect(full + 8u * s, S::kStage);
          tile_load<false>(base + s * S::kStage, &w_map, full + 8u * s, (k0 + s) * kPerRow, tf * kPrFeatures);
        }
      }
      wait_for_previous();
      for (uint32_t tile = team; tile < tiles; tile += teams) {
        uint32_t tf, tt;
        tile_at(a, tile, tf, tt);
        const uint32_t f = (tf * CG + (CG == 2 ? rank : 0u)) * kPrFeatures, t = tt * S::kTokens + (CG == 2 ? rank * (BN / 2u) : 0u);
        for (; n < early; ++n) tile_load<false>(base + n * S::kStage + S::kW, &x_map, full + 8u * n, (k0 + n) * kPerRow, t);
        for (uint32_t k = k0 + early; k < k1; ++k, ++n) {
          const uint32_t s = n % S::kStages, round = n / S::kStages;
          if (round && !bar_wait(empty + 8u * s, (round - 1u) & 1u, bad)) break;
          if (CG == 1 || rank == 0) bar_expect(full + 8u * s, CG * S::kStage);
          const uint32_t at = base + s * S::kStage;
          tile_load<CG == 2>(at, &w_map, full + 8u * s, k * kPerRow, f);
#pragma unroll
          for (uint32_t h = 0; h < NT; ++h)
            tile_load<CG == 2>(at + S::kW + h * S::kBlockX, &x_map, full + 8u * s, k * kPerRow, t + h * BN);
        }
        if (bad) break;
      }
      // The next call's CTAs come up while the last stages are worked on and the parts are added; earlier they would fetch
      // settled weights against this call's own and be idle at its end.
      if constexpr (SPLIT) let_next_start();
      // no copy may be in flight when the CTA ends: every filled stage has to be seen full or free
      for (uint32_t i = n > S::kStages ? n - S::kStages : 0u; i < n; ++i)
        bar_wait(empty + 8u * (i % S::kStages), (i / S::kStages) & 1u, bad);
    }
  } else if (warp == S::kMma) {
    if (lane == 0 && (CG == 1 || rank == 0)) {
      constexpr uint32_t idesc = instruction<F8>(kPrFeatures * CG, BN);
      wait_for_previous();                                             // the limits of the waits below are for this call's own work
      uint32_t n = 0, it = 0;
      for (uint32_t tile = team; tile < tiles; tile += teams, ++it) {
        const uint32_t acc = it % S::kAccs, round = it / S::kAccs;
        if (round && !bar_wait(acc_empty + 8u * acc, (round - 1u) & 1u, bad)) break;
        fence_after();
        for (uint32_t k = k0; k < k1; ++k, ++n) {
          const uint32_t s = n % S::kStages;
          if (!bar_wait(full + 8u * s, (n / S::kStages) & 1u, bad)) break;
          fence_after();
          const uint64_t dw = operand(base + s * S::kStage), dx = operand(base + s * S::kStage + S::kW);
#pragma unroll
          for (uint32_t j = 0; j < 4; ++j)                             // 32 bytes of K an instruction
            if constexpr (NT == 1) {
              mma<CG, F8>(tmem + acc * S::kTokens, dw + 2u * j, dx + 2u * j, idesc, (k > k0 || j) ? 1u : 0u);
            } else {                                                   // both halves of the tokens against one read of W (1 % at 8192^3)
              mma<CG, F8, 1>(tmem, dw + 2u * j, dx + 2u * j, idesc, (k > k0 || j) ? 1u : 0u);
              mma<CG, F8, 2>(tmem + BN, dw + 2u * j, dx + (S::kBlockX >> 4) + 2u * j, idesc, (k > k0 || j) ? 1u : 0u);
            }
          mma_commit<CG>(empty + 8u * s);
        }
        mma_commit<CG>(acc_full + 8u * acc);
        if (bad) break;
      }
    }
  } else {
    wait_for_previous();
    if constexpr (SPLIT) {                                             // under way while the sums are made
      own.load(a, f_mine);
      mine.fetch(a, first + warp, 4u * S::kTeams, first + here, f_mine);
    }
    const uint32_t part = warp >> 2, quarter = warp & 3u;              // which tokens, which features
    uint32_t it = 0;
    for (uint32_t tile = team; tile < tiles; tile += teams, ++it) {
      uint32_t tf, tt;
      tile_at(a, tile, tf, tt);
      const uint32_t f = (tf * CG + (CG == 2 ? rank : 0u)) * kPrFeatures + quarter * 32u + 4u * (lane & 7u), t0 = tt * S::kTokens;
      const uint32_t live = min(S::kTokens, a.M - t0);                         // tokens of the tile
      const uint32_t acc = it % S::kAccs;
      constexpr uint32_t kStep = S::kBlock;
      const uint32_t row = lane >> 3;
      PrColumns columns;
      PrAhead<kStep / 4u, YF32> next;                                  // a block ahead of the sums
      if constexpr (!SPLIT) {
        columns.load(a, f);
        next.fetch(a, t0 + part * kStep + row, 4u, t0 + live, f);
      }
      if (lane == 0) bar_wait(acc_full + 8u * acc, (it / S::kAccs) & 1u, bad);   // one lane polls
      __syncwarp();
      fence_after();
      if (SPLIT && ranks > 1) cluster_wait();
      const uint32_t from = tmem + ((quarter * 32u) << 16) + acc * S::kTokens;
      // a warp's block goes through its own scratch (split: in the ring, which is done with) into rows of 32 features:
      // lane: four features of token 4 i + lane / 8
      const uint32_t scratch = SPLIT ? base + warp * S::kScratch : staging + warp * S::kScratch;
#pragma unroll 1
      for (uint32_t c = part * kStep; c < live; c += S::kTeams * kStep) {
        uint32_t v[kStep];
        __syncwarp();
        tmem_load(from + c, v);
        const PrAhead<kStep / 4u, YF32> now = next;
        if constexpr (!SPLIT) next.fetch(a, t0 + c + S::kTeams * kStep + row, 4u, t0 + live, f);
        tmem_wait();
        if (k1 == k0) {                                                // K = 0: nothing was accumulated
#pragma unroll
          for (uint32_t i = 0; i < kStep; ++i) v[i] = 0u;
        }
        __syncwarp();                                                  // the block before is read
#pragma unroll
        for (uint32_t i = 0; i < kStep; ++i)
          asm volatile("st.shared.u32 [%0], %1;" :: "r"(scratch + i * 128u + lane * 4u), "r"(v[i]) : "memory");
        __syncwarp();
        float q[kStep];
#pragma unroll
        for (uint32_t i = 0; i < kStep / 4u; ++i)
          asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(q[4 * i]), "=f"(q[4 * i + 1]), "=f"(q[4 * i + 2]), "=f"(q[4 * i + 3])
                       : "r"(scratch + i * 512u + lane * 16u));
        if constexpr (SPLIT) {                                         // to the tokens' ranks
#pragma unroll
          for (uint32_t i = 0; i < kStep / 4u; ++i) {
            const uint32_t t = c + 4u * i + row;
            if (t < live)
              asm volatile(
                  "{\n\t.reg .b32 p;\n\t"
                  "mapa.shared::cluster.u32 p, %0, %1;\n\t"
                  "st.shared::cluster.v4.f32 [p], {%2, %3, %4, %5};\n\t}"
                  :: "r"(staging + ((rank * share + (t & (share - 1u))) * kPrFeatures + quarter * 32u + (lane & 7u) * 4u) * 4u), "r"(t / share),
                     "f"(q[4 * i]), "f"(q[4 * i + 1]), "f"(q[4 * i + 2]), "f"(q[4 * i + 3]) : "memory");
          }
        } else {
          finish<kStep / 4u, YF32>(a, columns, now, t0 + c + row, 4u, t0 + live, f, q);
        }
      }
      if constexpr (!SPLIT) {
        fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_at(acc_empty + 8u * acc, CG == 2 ? 0u : rank);
      }
    }
  }
  __syncwarp();

  if constexpr (SPLIT) {
    if (warp >= S::kTma && ranks > 1) cluster_wait();
    if (ranks > 1) cluster_sync(); else __syncthreads();               // all parts are in place
    if (warp < S::kTma) {
      constexpr uint32_t kWarps = 4u * S::kTeams;
      for (uint32_t l = warp; l < here; l += kWarps * kEach) {
        float v[4 * kEach];
#pragma unroll
        for (uint32_t i = 0; i < 4 * kEach; ++i) v[i] = 0.f;
        for (uint32_t r = 0; r < ranks; ++r) {
          float q[4 * kEach];
#pragma unroll
          for (uint32_t j = 0; j < kEach; ++j)
            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                         : "=f"(q[4 * j]), "=f"(q[4 * j + 1]), "=f"(q[4 * j + 2]), "=f"(q[4 * j + 3])
                         : "r"(staging + ((r * share + min(l + kWarps * j, here - 1u)) * kPrFeatures + 4u * lane) * 4u));
#pragma unroll
          for (uint32_t i = 0; i < 4 * kEach; ++i) v[i] += q[i];
        }
        const PrAhead<kEach, YF32> now = mine;
        mine.fetch(a, first + l + kWarps * kEach, kWarps, first + here, f_mine);
        finish<kEach, YF32>(a, own, now, first + l, kWarps, first + here, f_mine, v);
      }
    }
  }
  fence_before();
  if constexpr (CG == 2) cluster_sync(); else __syncthreads();         // nothing of the pair's other CTA is under way any more
  if (warp == S::kMma) {
    fence_after();
    tmem_free<CG>(tmem, S::kCols);
  }
  bad = __any_sync(kAll, bad);
  if (lane == 0 && bad) atomicOr(a.status, ANS_STATUS_COPY_TIMEOUT);
}

// Rows that start anywhere, elements `step` apart, into rows that start on 16 bytes, zeros behind their ends, of one matrix or of
// two in one launch: 16 bytes of a row a thread, element by element (the elements' neighbours come out of L1).  5 TB/s read and
// written at 8192 x 8191 in bf16.  T: an element's bits; UNIT: all steps are 1.
struct PrRows {
  const void* from; uint64_t stride, step;
  uint4* to;
  uint32_t rows, blocks;
};
template <typename T, bool UNIT>
__global__ void __launch_bounds__(256) ans_product_rows_kernel(const PrRows first, const PrRows second, uint32_t k, uint32_t pieces) {
  constexpr uint32_t kIn = 16 / sizeof(T);
  let_next_start();
  const bool one = blockIdx.x < first.blocks;
  const PrRows& a = one ? first : second;
  const uint64_t i = uint64_t(blockIdx.x - (one ? 0u : first.blocks)) * 256u + threadIdx.x;
  wait_for_previous();
  const uint64_t row = i / pieces;
  if (row >= a.rows) return;
  const uint32_t e = static_cast<uint32_t>(i - row * pieces) * kIn;
  const T* const p = static_cast<const T*>(a.from) + row * a.stride + (UNIT ? e : e * a.step);
  T v[kIn];
#pragma unroll
  for (uint32_t j = 0; j < kIn; ++j) v[j] = e + j < k ? p[UNIT ? j : j * a.step] : T(0);
  uint4 out;
  uint32_t* const w = &out.x;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j) {
    w[j] = 0;
#pragma unroll
    for (uint32_t b = 0; b < kIn / 4; ++b) w[j] |= uint32_t(v[j * (kIn / 4) + b]) << (8 * sizeof(T) * b);
  }
  a.to[i] = out;
}

// ---- host side -----------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return f;
}

// rows x k of 1- or 2-byte elements in boxes of 128 bytes x box_rows; what lies outside reads as zeros
static int make_map(CUtensorMap* map, const void* p, uint32_t rows, uint32_t k, uint64_t stride, bool f8, uint32_t box_rows) {
  const EncodeTiled encode = encode_tiled();
  if (!encode) return cuda_fail(cudaErrorNotSupported);
  const uint64_t size = f8 ? 1 : 2;
  const cuuint64_t dims[2] = {k, rows};
  const cuuint64_t strides[1] = {rows > 1 ? stride * size : (k * size + 15) & ~uint64_t(15)};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(kPrRow / size), box_rows}, step[2] = {1, 1};
  const CUresult rc = encode(map, f8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims,
                             strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return rc == CUDA_SUCCESS ? ANS_OK : cuda_fail(cudaErrorInvalidValue);
}

template <uint32_t BN, uint32_t NT, uint32_t CG, bool F8, bool SPLIT, bool YF32>
static int launch_form(const ans_product_desc& d, PrArgs a, uint32_t cluster, int sms, cudaStream_t st) {
  using S = PrShape<BN, NT, CG, SPLIT>;
  CUtensorMap w_map{}, x_map{};                       // k = 0: not used
  if (d.k) {
    int rc = make_map(&w_map, d.d_w, d.n, d.k, d.w_stride, F8, kPrFeatures);
    if (rc == ANS_OK) rc = make_map(&x_map, d.d_x, d.m, d.k, d.x_stride, F8, BN / CG);
    if (rc != ANS_OK) return rc;
  }
  a.tiles_f = (d.n + CG * kPrFeatures - 1) / (CG * kPrFeatures);
  a.tiles_t = (d.m + S::kTokens - 1) / S::kTokens;
  const uint64_t tiles = uint64_t(a.tiles_f) * a.tiles_t;
  if (tiles * cluster > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const uint32_t teams = SPLIT ? static_cast<uint32_t>(tiles)
                               : static_cast<uint32_t>(tiles < uint64_t(sms) / CG ? tiles : uint64_t(sms) / CG);
  constexpr auto kernel = ans_product_kernel<BN, NT, CG, F8, SPLIT, YF32>;
  const int allowed = allow_smem<kernel>(S::kSmem);
  if (allowed != ANS_OK) return allowed;
  const uint32_t together = SPLIT ? cluster : CG;
  return launch(kernel, dim3(teams * together), dim3(S::kThreads), S::kSmem, st, together, w_map, x_map, a);
}

template <uint32_t BN, uint32_t NT, uint32_t CG, bool F8, bool SPLIT>
static int launch_product(const ans_product_desc& d, const PrArgs& a, uint32_t cluster, int sms, cudaStream_t st) {
  return d.y_dtype == ANS_F32 ? launch_form<BN, NT, CG, F8, SPLIT, true>(d, a, cluster, sms, st)
                              : launch_form<BN, NT, CG, F8, SPLIT, false>(d, a, cluster, sms, st);
}

// What a form takes, in us, by a model fitted to sweeps on a B200 (both types, 1 to 4096 tokens, 1000 to 8192
// features, K of 512 to 8192), of which the order of the forms is used: about 2 us for the launch and its way to the first
// stage, the stages at the rate at which a CTA takes them in, and the tile's end.  A CTA takes in its ring every 1.36 us, the way
// from memory, and an SM 118 GB/s at most.  It has no term for DRAM, so a call bound by W's bytes takes longer than
// it says (1 x 8192 x 8192 in bf16 23.3 us, by the model 13.2; 16 x 8192 x 8192 in e4m3 14.4, by the model 8.2).
struct PrChoice {
  float us = 1e30f;
  uint32_t tokens = 0, split = 0;                      // split = 0: the whole form
};

static uint32_t stages_of(const ans_product_desc& d) { return static_cast<uint32_t>((uint64_t(d.k) * (d.dtype == ANS_E4M3 ? 1 : 2) + kPrRow - 1) / kPrRow); }

// The split form: every CTA one part of one tile; two CTAs an SM up to 64 tokens.
template <uint32_t BN>
static void weigh_split(const ans_product_desc& d, uint32_t steps, int sms, PrChoice& best) {
  using S = PrShape<BN, 1, 1, true>;
  constexpr float kEnd = BN == 16 ? 1.2f : BN == 32 ? 1.5f : BN == 64 ? 2.8f : 3.5f;
  constexpr float kRing = S::kStages * S::kStage / 1.36e3f;           // GB/s
  const uint64_t tiles = uint64_t((d.n + 127) / 128) * ((d.m + BN - 1) / BN), slots = uint64_t(sms) * (BN <= 64 ? 2 : 1);
  // Clusters of 8 with an SM for each CTA do not all fit the GPU's groups of SMs at once: 100 x 2048 x 8192 24 us against
  // 15 in fours.
  for (uint32_t split = 1; split <= (BN <= 64 ? 8u : 4u) && (split == 1 || split <= steps); split *= 2) {
    const uint64_t ctas = tiles * split, waves = (ctas + slots - 1) / slots;
    const uint64_t beside = waves > 1 ? slots / sms : (ctas + sms - 1) / sms;   // CTAs of an SM
    const float rate = fminf(kRing, 118.f / beside);
    const float us = 2.f + waves * (kEnd + (steps + split - 1) / split * (S::kStage / 1e3f) / rate);
    if (us < best.us) best = {us, BN, split};
  }
}

static PrChoice choose(const ans_product_desc& d, int sms) {
  const uint32_t steps = stages_of(d);
  PrChoice best;
  weigh_split<16>(d, steps, sms, best);
  if (d.m > 16) weigh_split<32>(d, steps, sms, best);
  if (d.m > 32) weigh_split<64>(d, steps, sms, best);
  if (d.m > 64) weigh_split<128>(d, steps, sms, best);
  if (d.m > 64 && sms > 1) {
    // The whole forms on pairs of SMs: a stage of 256 tokens 0.31 us, of 512 tokens 0.55 us (they read W once for both
    // halves and move a quarter less into shared memory, but nothing runs under a tile's end): 8192^3 in bf16 power-
    // capped 830 us in 512s, 900 in 256s; 4096 x 4096 x 1024 43 and 38.
    const uint64_t pairs = sms / 2, wide_f = (d.n + 255) / 256;
    auto rounds = [&](uint32_t tokens) { return static_cast<float>((wide_f * ((d.m + tokens - 1) / tokens) + pairs - 1) / pairs); };
    const float us256 = 6.5f + rounds(256) * steps * 0.31f, us512 = 3.5f + rounds(512) * (steps * 0.55f + 5.f);
    if (us256 < best.us) best = {us256, 256, 0};
    if (us512 < best.us) best = {us512, 512, 0};
  }
  return best;
}

template <bool F8>
static int launch_choice(const ans_product_desc& d, const PrArgs& a, int sms, cudaStream_t st) {
  const PrChoice best = choose(d, sms);
  switch (best.tokens) {
    case 16: return launch_product<16, 1, 1, F8, true>(d, a, best.split, sms, st);
    case 32: return launch_product<32, 1, 1, F8, true>(d, a, best.split, sms, st);
    case 64: return launch_product<64, 1, 1, F8, true>(d, a, best.split, sms, st);
    case 128: return launch_product<128, 1, 1, F8, true>(d, a, best.split, sms, st);
    case 256: return launch_product<256, 1, 2, F8, false>(d, a, 1, sms, st);
    default: return launch_product<256, 2, 2, F8, false>(d, a, 1, sms, st);
  }
}

}  // namespace ansb

using namespace ansb;

// whether TMA can read a matrix's rows
static bool rows_fit(const void* p, uint64_t stride, uint32_t rows, uint64_t es) {
  return !(reinterpret_cast<uintptr_t>(p) & 15) && (rows <= 1 || !((stride * es) & 15));
}
static uint64_t room_row(uint32_t k, uint64_t es) { return (k * es + 15) & ~uint64_t(15); }
// bytes of the room for W, which comes first, and for X
static uint64_t room_w(const ans_product_desc& d, uint64_t es) {
  return !(d.flags & ANS_PRODUCT_WEIGHTS_ANYWHERE) || rows_fit(d.d_w, d.w_stride, d.n, es) ? 0 : d.n * room_row(d.k, es);
}
static uint64_t room_x(const ans_product_desc& d, uint64_t es) {
  return rows_fit(d.d_x, d.x_stride, d.m, es) ? 0 : d.m * room_row(d.k, es);
}

static int lay_out(PrRows first, PrRows second, uint32_t k, uint64_t es, cudaStream_t st) {
  const uint64_t pieces = room_row(k, es) / 16;
  uint64_t blocks = 0;
  for (PrRows* r : {&first, &second}) {
    const uint64_t own = (r->rows * pieces + 255) / 256;
    blocks += own;
    if (blocks > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
    r->blocks = static_cast<uint32_t>(own);
  }
  const bool unit = first.step == 1 && (second.step == 1 || !second.rows);
  auto* const kernel = es == 1 ? (unit ? ans_product_rows_kernel<uint8_t, true> : ans_product_rows_kernel<uint8_t, false>)
                               : (unit ? ans_product_rows_kernel<uint16_t, true> : ans_product_rows_kernel<uint16_t, false>);
  return launch(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, 1, first, second, k, static_cast<uint32_t>(pieces));
}

ANS_EXPORT int ans_product_rows(const void* d_from, uint64_t stride, uint64_t step, uint32_t rows, uint32_t k, int dtype, void* d_to, void* stream) {
  ApiRange range("ans_product_rows");
  if (dtype != ANS_BF16 && dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  constexpr uint64_t kFar = uint64_t(1) << 36;
  if (rows > (1u << 30) || k > (1u << 22) || stride > kFar || step > kFar) return ANS_ERR_UNSUPPORTED;
  if (rows == 0 || k == 0) return ANS_OK;
  const uint64_t es = dtype == ANS_E4M3 ? 1 : 2;
  if (!d_from || !d_to || (reinterpret_cast<uintptr_t>(d_from) & (es - 1)) || (reinterpret_cast<uintptr_t>(d_to) & 15)) return ANS_ERR_INVALID_ARG;
  return lay_out({d_from, stride, step, static_cast<uint4*>(d_to), rows, 0}, {}, k, es, static_cast<cudaStream_t>(stream));
}

ANS_EXPORT int ans_product_room_bytes(const ans_product_desc* h_desc, size_t* h_bytes_out) {
  if (!h_desc || !h_bytes_out) return ANS_ERR_INVALID_ARG;
  if (h_desc->dtype != ANS_BF16 && h_desc->dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  const uint64_t es = h_desc->dtype == ANS_E4M3 ? 1 : 2;
  *h_bytes_out = room_w(*h_desc, es) + room_x(*h_desc, es);
  return ANS_OK;
}

ANS_EXPORT int ans_product_form(const ans_product_desc* h_desc, uint32_t* h_tokens, uint32_t* h_parts) {
  if (!h_desc || !h_tokens || !h_parts) return ANS_ERR_INVALID_ARG;
  if (h_desc->dtype != ANS_BF16 && h_desc->dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  *h_tokens = *h_parts = 0;
  if (h_desc->m == 0 || h_desc->n == 0) return ANS_OK;
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != ANS_OK) return rc;
  const PrChoice best = choose(*h_desc, sms);
  *h_tokens = best.tokens;
  *h_parts = best.split;
  return ANS_OK;
}

ANS_EXPORT int ans_product(const ans_product_desc* h_desc, uint32_t* d_status, void* stream) {
  ApiRange range("ans_product");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  ans_product_desc d = *h_desc;
  if (d.dtype != ANS_BF16 && d.dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  if (d.y_dtype != ANS_BF16 && d.y_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (d.flags & ~(ANS_PRODUCT_WEIGHTS_SETTLED | ANS_PRODUCT_WEIGHTS_ANYWHERE)) return ANS_ERR_UNSUPPORTED;
  if (d.activation < ANS_ACT_NONE || d.activation > ANS_ACT_SILU) return ANS_ERR_UNSUPPORTED;
  constexpr uint32_t kMost = 1u << 30;
  if (d.m > kMost || d.n > kMost || d.k > (1u << 22)) return ANS_ERR_UNSUPPORTED;
  if (d.m == 0 || d.n == 0) return ANS_OK;
  if (!d.d_y || (d.k && (!d.d_x || !d.d_w))) return ANS_ERR_INVALID_ARG;
  const uint64_t es = d.dtype == ANS_E4M3 ? 1 : 2, ys = d.y_dtype == ANS_F32 ? 4 : 2;
  const bool anywhere = d.flags & ANS_PRODUCT_WEIGHTS_ANYWHERE;
  if ((reinterpret_cast<uintptr_t>(d.d_w) & (anywhere ? es - 1 : 15)) || (reinterpret_cast<uintptr_t>(d.d_x) & (es - 1))) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d.d_y) | reinterpret_cast<uintptr_t>(d.d_residual)) & (ys - 1)) return ANS_ERR_INVALID_ARG;
  for (const float* p : {d.d_x_scales, d.d_w_scales, d.d_bias})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kFar = uint64_t(1) << 36;
  if (d.k && d.m > 1 && (d.x_stride < d.k || d.x_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.k && d.n > 1 && (d.w_stride < d.k || (!anywhere && (d.w_stride * es) % 16) || d.w_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.m > 1 && (d.y_stride < d.n || d.y_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.m > 1 && d.d_residual && (d.residual_stride < d.n || d.residual_stride > kFar)) return ANS_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const uint64_t for_w = d.k ? room_w(d, es) : 0, for_x = d.k ? room_x(d, es) : 0;
  if (for_w + for_x) {
    if (!d.d_room || d.room_bytes < for_w + for_x) return ANS_ERR_BUFFER_TOO_SMALL;
    if (reinterpret_cast<uintptr_t>(d.d_room) & 15) return ANS_ERR_INVALID_ARG;
    PrRows w{}, x{};
    if (for_w) w = {d.d_w, d.w_stride, 1, static_cast<uint4*>(d.d_room), d.n, 0};
    if (for_x) x = {d.d_x, d.x_stride, 1, reinterpret_cast<uint4*>(static_cast<char*>(d.d_room) + for_w), d.m, 0};
    const int rc = for_w ? lay_out(w, x, d.k, es, st) : lay_out(x, w, d.k, es, st);
    if (rc != ANS_OK) return rc;
    const uint64_t stride = room_row(d.k, es) / es;
    if (for_w) { d.d_w = w.to; d.w_stride = stride; d.flags &= ~ANS_PRODUCT_WEIGHTS_SETTLED; }      // written just ahead
    if (for_x) { d.d_x = x.to; d.x_stride = stride; }
  }
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc != ANS_OK) return rc;
  PrArgs a{};
  a.x_scales = d.d_x_scales; a.w_scales = d.d_w_scales; a.bias = d.d_bias;
  a.residual = d.d_residual; a.y = d.d_y; a.residual_stride = d.residual_stride; a.y_stride = d.y_stride;
  a.M = d.m; a.N = d.n; a.steps = stages_of(d);
  a.activation = d.activation;
  a.settled = (d.flags & ANS_PRODUCT_WEIGHTS_SETTLED) != 0;
  auto four = [&](const void* p, uint64_t stride) { return !p || !((reinterpret_cast<uintptr_t>(p) | (d.m > 1 ? stride * ys : 0)) & (4 * ys - 1)); };
  a.wide = four(d.d_y, d.y_stride) && four(d.d_residual, d.residual_stride);
  a.status = d_status;
  return d.dtype == ANS_E4M3 ? launch_choice<true>(d, a, sms, st) : launch_choice<false>(d, a, sms, st);
}
