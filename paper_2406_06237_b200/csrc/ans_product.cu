// Matrix product with its epilogue on the tensor cores:
//   Y[m][n] = act(x_scale[m] * w_scale[n] * sum_k X[m][k] W[n][k] + bias[n]) + residual[m][n]
//
// The operands are exchanged, Y^T = W X^T: 128 features of W are the 128-lane operand and the tokens
// (rows of X) the columns, so that a call with few tokens uses matrix instructions with few columns
// and reads W, which is what such a call is made of, in full tiles.  Both operands come by TMA in
// 128-byte rows (64 bf16 or 128 e4m3) into a ring of stages; one thread issues tcgen05.mma; sums
// stay in tensor memory in fp32.  Four warps take them out: a thread holds one feature, so a block of
// tokens goes through shared memory (fp32, token-major) and leaves in rows of 128 features, where
// the epilogue's operands (bias, scales of W) are constants of a thread and residual and Y are
// read and written in whole sectors.
//
// Two forms:
//   split:  one tile of 128 features x BN tokens a cluster of S CTAs; each sums a part of K, then each
//           takes some of the tokens and adds the S partial sums out of the others' shared memory, in
//           the order of the ranks: no workspace, no atomics, results do not vary from run to run.
//   whole:  persistent; a CTA (or a pair of CTAs on one tile of 256 features, cta_group::2) takes tile after
//           tile, the accumulators are double-buffered so that one tile's epilogue runs under the next one's products.
// Every wait is bounded; one that runs out sets ANS_STATUS_COPY_TIMEOUT and the kernel runs to its end.
#include <cuda.h>

#include <initializer_list>

#include "ans_tensor.cuh"

namespace ansb {

using namespace ten;

constexpr uint32_t kPrRow = 128;                      // bytes of K per stage and row
constexpr uint32_t kPrFeatures = 128;                 // features of a CTA's tile
constexpr uint32_t kPrThreads = 192;                  // warps 0-3: epilogue; 4: TMA; 5: matrix instructions
constexpr uint32_t kPrBlock = 32;                     // tokens of an epilogue block
constexpr uint32_t kPrStaging = kPrBlock * kPrFeatures * 4;

struct PrArgs {
  const float* x_scales; const float* w_scales; const float* bias;
  const void* residual; void* y;
  uint64_t residual_stride, y_stride;
  uint32_t M, N, steps;                               // steps: stages of K
  uint32_t tiles_f, tiles_t;
  int32_t activation;
  uint32_t y_f32;
  uint32_t wide;                                      // four features of Y (and residual) can be accessed at once
  uint32_t* status;
};

// BN tokens a tile; CG CTAs on it; SPLIT: K is dealt over a cluster.
template <uint32_t BN, uint32_t CG, bool SPLIT>
struct PrShape {
  static constexpr uint32_t kW = kPrFeatures * kPrRow;
  static constexpr uint32_t kX = BN / CG * kPrRow;    // a pair's CTAs hold half of the tokens each
  static constexpr uint32_t kStage = kW + kX;
  static constexpr uint32_t kStagingBytes = SPLIT ? 0u : 2u * kPrStaging;
  static constexpr uint32_t kFit = (227u * 1024u - 1024u - 512u - kStagingBytes) / kStage;
  static constexpr uint32_t kStages = kFit > 8u ? 8u : kFit;
  static constexpr uint32_t kAccs = SPLIT ? 1u : 2u;  // accumulators in tensor memory
  static constexpr uint32_t kCols = kAccs * BN < 32u ? 32u : kAccs * BN;
  static constexpr uint32_t kSmem = 1024u + kStages * kStage + kStagingBytes + 512u;
  static_assert(!SPLIT || BN * kPrFeatures * 4u <= kStages * kStage, "partial sums fit the ring");
};

__device__ __forceinline__ float activate(float v, int32_t act) {
  switch (act) {
    case ANS_ACT_RELU: return v < 0.f ? 0.f : v;                       // a NaN stays
    case ANS_ACT_GELU: return 0.5f * v * (1.f + erff(v * 0.70710678118654752f));
    case ANS_ACT_GELU_TANH: {
      // (1 + tanh u) / 2 = 1 / (1 + exp(-2u)): no difference of near-equal numbers
      const float u = 1.5957691216057308f * v * fmaf(0.044715f * v, v, 1.f);
      return v / (1.f + __expf(-u));
    }
    case ANS_ACT_SILU: return v / (1.f + __expf(-v));
    default: return v;
  }
}

// The epilogue's constants of a thread: its four features f .. f + 3.
struct PrColumns {
  float bias[4], scale[4];
  __device__ __forceinline__ void load(const PrArgs& a, uint32_t f) {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
      const bool in = f + i < a.N;
      bias[i] = a.bias && in ? __ldg(a.bias + f + i) : 0.f;
      scale[i] = a.w_scales && in ? __ldg(a.w_scales + f + i) : 1.f;
    }
  }
};

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Features f .. f + 3 of token m, sums in v: scales, bias, activation, residual, one rounding, store.
__device__ __forceinline__ void finish(const PrArgs& a, const PrColumns& c, uint32_t m, uint32_t f, float (&v)[4]) {
  const float xs = a.x_scales ? __ldg(a.x_scales + m) : 1.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = activate(fmaf(v[i], xs * c.scale[i], c.bias[i]), a.activation);
  const uint64_t at = uint64_t(m) * a.y_stride + f, rat = uint64_t(m) * a.residual_stride + f;
  if (a.y_f32) {
    float* y = static_cast<float*>(a.y) + at;
    const float* r = static_cast<const float*>(a.residual) + rat;
    if (a.wide && f + 4 <= a.N) {
      if (a.residual) {
        const float4 q = *reinterpret_cast<const float4*>(r);
        v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
      }
      *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (f + i < a.N) y[i] = a.residual ? v[i] + r[i] : v[i];
    }
  } else {
    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(a.y) + at;
    const __nv_bfloat16* r = static_cast<const __nv_bfloat16*>(a.residual) + rat;
    if (a.wide && f + 4 <= a.N) {
      if (a.residual) {
        const uint2 q = *reinterpret_cast<const uint2*>(r);
        v[0] += bf16_lo(q.x); v[1] += bf16_hi(q.x); v[2] += bf16_lo(q.y); v[3] += bf16_hi(q.y);
      }
      const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
      *reinterpret_cast<uint2*>(y) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i)
        if (f + i < a.N) y[i] = __float2bfloat16_rn(a.residual ? v[i] + __bfloat162float(r[i]) : v[i]);
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

template <uint32_t BN, uint32_t CG, bool F8, bool SPLIT>
__global__ void __launch_bounds__(kPrThreads, 1)
ans_product_kernel(const __grid_constant__ CUtensorMap w_map, const __grid_constant__ CUtensorMap x_map, const PrArgs a) {
  using S = PrShape<BN, CG, SPLIT>;
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
  uint32_t bad = 0;

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < S::kStages; ++s) { bar_init(full + 8u * s, 1); bar_init(empty + 8u * s, 1); }
    for (uint32_t s = 0; s < S::kAccs; ++s) { bar_init(acc_full + 8u * s, 1); bar_init(acc_empty + 8u * s, 4u * CG); }
    bar_init_fence();
  }
  if (warp == 5) tmem_alloc<CG>(slot, S::kCols);
  if (threadIdx.x == 128 && a.steps) { map_prefetch(&w_map); map_prefetch(&x_map); }
  fence_before();
  if constexpr (SPLIT || CG == 2) cluster_sync(); else __syncthreads();
  fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

  // this CTA's tiles, and its part of K
  const uint32_t tiles = a.tiles_f * a.tiles_t;
  const uint32_t team = SPLIT ? blockIdx.x / ranks : blockIdx.x / CG, teams = SPLIT ? tiles : gridDim.x / CG;
  const uint32_t k0 = SPLIT ? static_cast<uint32_t>(uint64_t(a.steps) * rank / ranks) : 0u;
  const uint32_t k1 = SPLIT ? static_cast<uint32_t>(uint64_t(a.steps) * (rank + 1u) / ranks) : a.steps;

  if (warp == 4) {
    if (lane == 0) {
      uint32_t n = 0;                                                  // stages filled so far
      for (uint32_t tile = team; tile < tiles; tile += teams) {
        uint32_t tf, tt;
        tile_at(a, tile, tf, tt);
        const uint32_t f = (tf * CG + (CG == 2 ? rank : 0u)) * kPrFeatures, t = tt * BN + (CG == 2 ? rank * (BN / 2u) : 0u);
        for (uint32_t k = k0; k < k1; ++k, ++n) {
          const uint32_t s = n % S::kStages, round = n / S::kStages;
          if (round && !bar_wait(empty + 8u * s, (round - 1u) & 1u, bad)) break;
          if (CG == 1 || rank == 0) bar_expect(full + 8u * s, CG * S::kStage);
          const uint32_t at = base + s * S::kStage;
          tile_load<CG == 2>(at, &w_map, full + 8u * s, k * kPerRow, f);
          tile_load<CG == 2>(at + S::kW, &x_map, full + 8u * s, k * kPerRow, t);
        }
        if (bad) break;
      }
      // no copy may be in flight when the CTA ends: every filled stage has to be seen full or free
      for (uint32_t i = n > S::kStages ? n - S::kStages : 0u; i < n; ++i)
        bar_wait(empty + 8u * (i % S::kStages), (i / S::kStages) & 1u, bad);
    }
  } else if (warp == 5) {
    if (lane == 0 && (CG == 1 || rank == 0)) {
      constexpr uint32_t idesc = instruction<F8>(kPrFeatures * CG, BN);
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
            mma<CG, F8>(tmem + acc * BN, dw + 2u * j, dx + 2u * j, idesc, (k > k0 || j) ? 1u : 0u);
          mma_commit<CG>(empty + 8u * s);
        }
        mma_commit<CG>(acc_full + 8u * acc);
        if (bad) break;
      }
    }
  } else {
    uint32_t it = 0;
    for (uint32_t tile = team; tile < tiles; tile += teams, ++it) {
      uint32_t tf, tt;
      tile_at(a, tile, tf, tt);
      const uint32_t f = (tf * CG + (CG == 2 ? rank : 0u)) * kPrFeatures + 4u * lane, t0 = tt * BN;
      const uint32_t live = min(BN, a.M - t0);                         // tokens of the tile
      const uint32_t acc = it % S::kAccs;
      PrColumns columns;
      columns.load(a, f);
      bar_wait(acc_full + 8u * acc, (it / S::kAccs) & 1u, bad);
      __syncwarp();
      fence_after();
      const uint32_t from = tmem + ((warp * 32u) << 16) + acc * BN;
      constexpr uint32_t kStep = BN < kPrBlock ? BN : kPrBlock;        // tokens taken out at a time
#pragma unroll 1
      for (uint32_t c = 0; c < BN; c += kStep) {
        if (c >= live) break;
        uint32_t v[kStep / 16][16];
#pragma unroll
        for (uint32_t h = 0; h < kStep / 16u; ++h) tmem_load16(from + c + 16u * h, v[h]);
        tmem_wait();
        if (k1 == k0) {                                                // K = 0: nothing was accumulated
#pragma unroll
          for (uint32_t h = 0; h < kStep / 16u; ++h)
#pragma unroll
            for (uint32_t i = 0; i < 16; ++i) v[h][i] = 0u;
        }
        const uint32_t to = SPLIT ? base + c * (kPrFeatures * 4u) : staging + ((c / kPrBlock) & 1u) * kPrStaging;
#pragma unroll
        for (uint32_t h = 0; h < kStep / 16u; ++h)
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i)
            asm volatile("st.shared.u32 [%0], %1;" :: "r"(to + ((16u * h + i) * kPrFeatures + warp * 32u + lane) * 4u), "r"(v[h][i]) : "memory");
        if constexpr (!SPLIT) {
          asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll 2
          for (uint32_t i = 0; i < kStep / 4u; ++i) {
            const uint32_t t = warp * (kStep / 4u) + i;
            if (c + t < live) {
              float q[4];
              asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                           : "=f"(q[0]), "=f"(q[1]), "=f"(q[2]), "=f"(q[3]) : "r"(to + (t * kPrFeatures + 4u * lane) * 4u));
              if (f < a.N) finish(a, columns, t0 + c + t, f, q);
            }
          }
        }
      }
      if constexpr (!SPLIT) {
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (CG == 2) bar_arrive_at(acc_empty + 8u * acc, 0); else bar_arrive_at(acc_empty + 8u * acc, rank);
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");                 // the staging blocks are free
      }
    }
  }
  __syncwarp();

  if constexpr (SPLIT) {
    cluster_sync();                                                    // the partial sums of all ranks are in place
    if (warp < 4) {
      uint32_t tf, tt;
      tile_at(a, team, tf, tt);
      const uint32_t f = tf * kPrFeatures + 4u * lane, t0 = tt * BN, live = min(BN, a.M - t0);
      PrColumns columns;
      columns.load(a, f);
      for (uint32_t t = rank * 4u + warp; t < live; t += 4u * ranks) {
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t r = 0; r < ranks; ++r) {
          float q0, q1, q2, q3;
          asm volatile(
              "{\n\t.reg .b32 p;\n\t"
              "mapa.shared::cluster.u32 p, %4, %5;\n\t"
              "ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [p];\n\t}"
              : "=f"(q0), "=f"(q1), "=f"(q2), "=f"(q3) : "r"(base + (t * kPrFeatures + 4u * lane) * 4u), "r"(r) : "memory");
          v[0] += q0; v[1] += q1; v[2] += q2; v[3] += q3;
        }
        if (f < a.N) finish(a, columns, t0 + t, f, v);
      }
    }
  }
  fence_before();
  if constexpr (SPLIT || CG == 2) cluster_sync(); else __syncthreads();   // others' shared memory is read, theirs signals ours
  if (warp == 5) {
    fence_after();
    tmem_free<CG>(tmem, S::kCols);
  }
  bad = __any_sync(kAll, bad);
  if (lane == 0 && bad) atomicOr(a.status, ANS_STATUS_COPY_TIMEOUT);
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

template <uint32_t BN, uint32_t CG, bool F8, bool SPLIT>
static int launch_product(const ans_product_desc& d, PrArgs a, uint32_t cluster, int sms, cudaStream_t st) {
  using S = PrShape<BN, CG, SPLIT>;
  CUtensorMap w_map{}, x_map{};                       // k = 0: not used
  if (d.k) {
    int rc = make_map(&w_map, d.d_w, d.n, d.k, d.w_stride, F8, kPrFeatures);
    if (rc == ANS_OK) rc = make_map(&x_map, d.d_x, d.m, d.k, d.x_stride, F8, BN / CG);
    if (rc != ANS_OK) return rc;
  }
  a.tiles_f = (d.n + CG * kPrFeatures - 1) / (CG * kPrFeatures);
  a.tiles_t = (d.m + BN - 1) / BN;
  const uint64_t tiles = uint64_t(a.tiles_f) * a.tiles_t;
  if (tiles * cluster > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const uint32_t teams = SPLIT ? static_cast<uint32_t>(tiles)
                               : static_cast<uint32_t>(tiles < uint64_t(sms) / CG ? tiles : uint64_t(sms) / CG);
  auto* kernel = ans_product_kernel<BN, CG, F8, SPLIT>;
  ANSB_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::kSmem)));
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(teams * (SPLIT ? cluster : CG));
  cfg.blockDim = dim3(kPrThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = SPLIT ? cluster : CG;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ANSB_CUDA(cudaLaunchKernelEx(&cfg, kernel, w_map, x_map, a));
  return ANS_OK;
}

template <bool F8>
static int choose_product(const ans_product_desc& d, const PrArgs& a, int sms, cudaStream_t st) {
  // Few tiles: K is split so that all SMs have a part of the work, at least two stages each.
  auto split_of = [&](uint32_t bn) {
    const uint64_t tiles = uint64_t((d.n + 127) / 128) * ((d.m + bn - 1) / bn);
    uint32_t s = 1;
    while (s < 8 && tiles * s * 2 <= uint64_t(sms) && a.steps >= 4 * s) s *= 2;
    return s;
  };
  if (d.m <= 16) return launch_product<16, 1, F8, true>(d, a, split_of(16), sms, st);
  if (d.m <= 32) return launch_product<32, 1, F8, true>(d, a, split_of(32), sms, st);
  if (d.m <= 64) return launch_product<64, 1, F8, true>(d, a, split_of(64), sms, st);
  const uint64_t tiles = uint64_t((d.n + 127) / 128) * ((d.m + 127) / 128);
  if (tiles <= uint64_t(sms)) return launch_product<128, 1, F8, true>(d, a, split_of(128), sms, st);
  return launch_product<256, 2, F8, false>(d, a, 1, sms, st);
}

}  // namespace ansb

using namespace ansb;

ANS_EXPORT int ans_product(const ans_product_desc* h_desc, uint32_t* d_status, void* stream) {
  ApiRange range("ans_product");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  const ans_product_desc& d = *h_desc;
  if (d.dtype != ANS_BF16 && d.dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  if (d.y_dtype != ANS_BF16 && d.y_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (d.activation < ANS_ACT_NONE || d.activation > ANS_ACT_SILU) return ANS_ERR_UNSUPPORTED;
  constexpr uint32_t kMost = 1u << 30;
  if (d.m > kMost || d.n > kMost || d.k > (1u << 22)) return ANS_ERR_UNSUPPORTED;
  if (d.m == 0 || d.n == 0) return ANS_OK;
  if (!d.d_y || (d.k && (!d.d_x || !d.d_w))) return ANS_ERR_INVALID_ARG;
  const uint64_t es = d.dtype == ANS_E4M3 ? 1 : 2, ys = d.y_dtype == ANS_F32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(d.d_x) | reinterpret_cast<uintptr_t>(d.d_w)) & 15) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d.d_y) | reinterpret_cast<uintptr_t>(d.d_residual)) & (ys - 1)) return ANS_ERR_INVALID_ARG;
  for (const float* p : {d.d_x_scales, d.d_w_scales, d.d_bias})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kFar = uint64_t(1) << 36;
  if (d.k && d.m > 1 && (d.x_stride < d.k || (d.x_stride * es) % 16 || d.x_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.k && d.n > 1 && (d.w_stride < d.k || (d.w_stride * es) % 16 || d.w_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.m > 1 && (d.y_stride < d.n || d.y_stride > kFar)) return ANS_ERR_INVALID_ARG;
  if (d.m > 1 && d.d_residual && (d.residual_stride < d.n || d.residual_stride > kFar)) return ANS_ERR_INVALID_ARG;
  int dev = 0, sms = 0;
  ANSB_CUDA(cudaGetDevice(&dev));
  ANSB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  PrArgs a{};
  a.x_scales = d.d_x_scales; a.w_scales = d.d_w_scales; a.bias = d.d_bias;
  a.residual = d.d_residual; a.y = d.d_y; a.residual_stride = d.residual_stride; a.y_stride = d.y_stride;
  a.M = d.m; a.N = d.n; a.steps = static_cast<uint32_t>((d.k * es + kPrRow - 1) / kPrRow);
  a.activation = d.activation;
  a.y_f32 = d.y_dtype == ANS_F32;
  auto four = [&](const void* p, uint64_t stride) { return !p || !((reinterpret_cast<uintptr_t>(p) | (d.m > 1 ? stride * ys : 0)) & (4 * ys - 1)); };
  a.wide = four(d.d_y, d.y_stride) && four(d.d_residual, d.residual_stride);
  a.status = d_status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return d.dtype == ANS_E4M3 ? choose_product<true>(d, a, sms, st) : choose_product<false>(d, a, sms, st);
}
