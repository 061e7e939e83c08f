// Low-rank adapters of many requests beside a projection that they share:
//   out[t] = y[t] + scales[i] * x_scales[t] * (x[t] A_i^T) B_i^T,   i the adapter of row t's request.
//
// For more rows than requests two kernels, both over tiles of 16 or 32 rows of one request: the first sums h = x A^T (mma.sync,
// fp32) over a part of the inputs, up to eight parts a tile, into the caller's room; the second adds the parts in their order and
// streams y through the product with B.  With a rank of 16, 8192 inputs and as many outputs in bf16, a row alone has 0.9 operations
// for each byte that must be moved, 64 rows of a request 9 and any number under 11: bound by the bytes, so the plain matrix instructions are enough.  h meets B as the sum of two bf16 numbers, h = hi + lo,
// |h - hi - lo| <= 2^-17 |h|: a second product, which costs less than the rounding of h to 8 bits would lose.
//
// 5507 rows of 8192 in e4m3, rank 32, 8192 outputs take 62 us, 19 of them the first kernel and 43 the second (4.2 TB/s of y and out;
// bound by latency and by issue at 16 warps an SM, 45 % of its issue slots used).  What made it that:
//   equal shares of the work for as many blocks as fit the GPU (80.5 us with a block for each tile and part: waves that end
//   half filled; rows without an adapter counted in both kernels: 65.3), at a cost of 1 us where there are a few rows;
//   h as an operand in registers and four groups of y on their way (75.4 with h read from shared memory for every group, three
//   blocks an SM and two groups of y);
//   a form without questions at each access for rows without a ragged edge (EXACT; 91 to 81 us when it came).
// One kernel with a cluster a tile, whose blocks exchange h through shared memory, took 118: 54 us of it were the blocks'
// starts, barriers and exchanges, eight times as many as there are tiles.
//
// The order of the inputs in a product is free, so a lane takes 16 bytes of a row at once; the columns of a product with B stand
// for outputs such that a lane has 8 neighbouring ones.
#include <cuda_fp16.h>

#include <algorithm>
#include <initializer_list>

#include "ans_adapters.cuh"

namespace ansb {
namespace blk {

template <int R, int MT>
struct AdShape {
  static constexpr uint32_t kRows = 16 * MT;
  static constexpr uint32_t kSums = kRows * R;                       // of h
  static constexpr uint32_t kHRow = R + 8, kPart = kRows * (R + 8);  // elements of a row of h, of a warp's sums; + 8: eight rows in different banks
  static constexpr uint32_t kDownSmem = kAdWarps * kPart * 4;
  // a warp's ring of groups of 32 outputs of y: four groups in bf16, two in fp32
  static constexpr uint32_t kGroup = kRows * 32 * 2, kRing = 4 * kGroup;
  static constexpr uint32_t kUpSmem = 2 * kRows * kHRow * 2 + kAdWarps * kRing;
};

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {       // onto zeros
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// two e4m3 values as bf16 (exact)
__device__ __forceinline__ uint32_t open_e4m3(uint32_t two) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(two), __NV_E4M3);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  return pack_bf16(f.x, f.y);
}
// 16 bytes of a row of bf16 or e4m3 elements from element e on; zeros from element n on.  VEC: the row starts on 16 bytes and n is a
// multiple of 16 bytes.
template <typename T, bool VEC>
__device__ __forceinline__ uint4 piece_of(const T* row, uint32_t e, uint32_t n, bool live) {
  uint4 v = make_uint4(0, 0, 0, 0);
  if (!live) return v;
  if constexpr (VEC) {
    if (e < n) v = *reinterpret_cast<const uint4*>(row + e);
  } else {
    constexpr uint32_t kIn = 16 / sizeof(T);
    uint32_t* const w = &v.x;
#pragma unroll
    for (uint32_t i = 0; i < kIn; ++i)
      if (e + i < n) w[i / (kIn / 4)] |= static_cast<uint32_t>(row[e + i]) << (8 * sizeof(T) * (i % (kIn / 4)));
  }
  return v;
}

// Tiles of ROWS rows, request by request, and the steps that each takes, of a unit of inputs or a group of outputs for each
// warp, make a call's work in a row, which is cut into equal parts for as many blocks as there are, so that none waits for
// a last wave: a block has the end of a tile and the
// beginning of the next one, say.  first[s], in shared memory: tiles before request s's, and returned all of them; x: those that have
// an adapter, which are the first kernel's; y: those that get outputs, the second one's.  The first kernel has no place for y's.
template <uint32_t ROWS>
__device__ __forceinline__ uint2 ad_tiles(const AdArgs& a, uint32_t* first_x, uint32_t* first_y, bool tell) {
  __shared__ uint2 part[kAdWarps];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  uint2 total = make_uint2(0, 0);
  bool bad = false;
  for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += kAdThreads) {
    const uint32_t s = s0 + threadIdx.x;
    uint2 own = make_uint2(0, 0);
    if (s < a.n_seqs) {
      const int32_t r0 = a.starts[s], r1 = a.starts[s + 1], i = a.which[s];
      if (r0 < 0 || r1 < r0 || static_cast<uint32_t>(r1) > a.rows) {
        bad = true;
      } else {
        const bool none = i < 0 || static_cast<uint32_t>(i) >= a.count;
        bad |= r1 > r0 && i >= 0 && none;
        const uint32_t tiles = (static_cast<uint32_t>(r1 - r0) + ROWS - 1) / ROWS;
        own = make_uint2(none ? 0u : tiles, none && a.out == a.y ? 0u : tiles);
      }
    }
    uint2 x = own;
#pragma unroll
    for (uint32_t step = 1; step < 32; step *= 2) {
      const uint2 from = make_uint2(__shfl_up_sync(kAll, x.x, step), __shfl_up_sync(kAll, x.y, step));
      if (lane >= step) { x.x += from.x; x.y += from.y; }
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    uint2 before = total;
#pragma unroll
    for (uint32_t w = 0; w < kAdWarps; ++w) {
      const uint2 of = part[w];
      if (w < warp) { before.x += of.x; before.y += of.y; }
      total.x += of.x;
      total.y += of.y;
    }
    if (s < a.n_seqs) {
      first_x[s] = before.x + x.x - own.x;
      if (first_y) first_y[s] = before.y + x.y - own.y;
    }
    if (s0 + kAdThreads < a.n_seqs) __syncthreads();   // the warps' sums are read
  }
  if (threadIdx.x == 0) {
    first_x[a.n_seqs] = total.x;
    if (first_y) first_y[a.n_seqs] = total.y;
  }
  if (tell && bad) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
  __syncthreads();
  return total;
}
// the last request that has begun with or before the tile; first[0] <= tile < first[n]
__device__ __forceinline__ uint32_t ad_request(const uint32_t* first, uint32_t n, uint32_t tile) {
  uint32_t s = 0;
  while (n - s > 1) {
    const uint32_t mid = (s + n) / 2;
    if (first[mid] <= tile) s = mid; else n = mid;
  }
  return s;
}
// Block b's share of `all` steps, `each` of them a tile: from step `in` of `tile` on, `left` of them (fewer than 2^32: a step has 4096
// elements of y, or of x, which are in memory).  And the block that has step x.
struct AdShare { uint32_t tile, in, left; };
__device__ __forceinline__ AdShare ad_share(uint64_t all, uint32_t each, uint32_t blocks, uint32_t b) {
  const uint64_t from = all * b / blocks, tile = from / each;
  return {static_cast<uint32_t>(tile), static_cast<uint32_t>(from - tile * each), static_cast<uint32_t>(all * (b + 1u) / blocks - from)};
}
__device__ __forceinline__ uint32_t ad_block_of(uint64_t all, uint32_t blocks, uint64_t x) { return static_cast<uint32_t>(((x + 1u) * blocks + all - 1u) / all - 1u); }
// Blocks that x A^T is dealt to, so that a tile's steps lie in `most` blocks at most: as many for each tile, or else shares of at
// least 1 / (most - 1) of a tile, which begin in at most most - 1 places behind a tile's first step.
__device__ __forceinline__ uint32_t ad_down_blocks(uint32_t grid, uint32_t most, uint32_t tiles, uint32_t steps) {
  const uint64_t even = uint64_t(tiles) * min(most, steps);
  return static_cast<uint32_t>(even <= grid ? even : min(uint64_t(grid), uint64_t(tiles) * (most - 1u)));
}

// R: the rank, rounded up to 16, 32, 64 or 128; MT: 16 rows each; most: parts of a tile's sums.
template <int R, int MT, bool F8, bool VEC>
__global__ void __launch_bounds__(kAdThreads, R * MT >= 128 ? 1 : 2) ans_adapters_down_kernel(const AdArgs a, const uint32_t most) {
  using S = AdShape<R, MT>;
  using X = std::conditional_t<F8, uint8_t, uint16_t>;
  constexpr uint32_t kUnit = F8 ? 64 : 32, kLane = kUnit / 4, kSteps = kUnit / 16;     // inputs of a unit, of a lane, products
  constexpr int NT = R / 8;
  constexpr int kAhead = MT * R <= 16 ? (F8 ? 2 : 4) : MT * R <= 64 && !F8 ? 2 : 1;    // units whose loads are under way together
  extern __shared__ __align__(16) uint8_t smem[];
  float* const parts = reinterpret_cast<float*>(smem);               // [warp][row][R + 8]
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
  let_next_start();
  wait_for_previous();
  uint32_t* const first = reinterpret_cast<uint32_t*>(smem + S::kDownSmem);             // [n_seqs + 1]
  const uint32_t tiles = ad_tiles<S::kRows>(a, first, nullptr, blockIdx.x == 0).x, units = (a.n_in + kUnit - 1) / kUnit;
  const uint32_t steps = (units + kAdWarps - 1) / kAdWarps, blocks = ad_down_blocks(gridDim.x, most, tiles, steps);
  if (blockIdx.x >= blocks) return;
  const uint64_t all = uint64_t(tiles) * steps;
  AdShare share = ad_share(all, steps, blocks, blockIdx.x);
  uint32_t s = ad_request(first, a.n_seqs, share.tile);
  for (; share.left; ++share.tile, share.in = 0) {
    const uint32_t tile = share.tile, count = min(steps - share.in, share.left);
    const uint32_t u0 = kAdWarps * share.in, u1 = min(units, u0 + kAdWarps * count);
    share.left -= count;
    while (first[s + 1] <= tile) ++s;
    const uint32_t i = a.which[s];
    const uint32_t r0 = (tile - first[s]) * S::kRows, live = min(S::kRows, static_cast<uint32_t>(a.starts[s + 1] - a.starts[s]) - r0);
    const uint64_t begin = uint64_t(a.starts[s]) + r0;

    float c[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) c[m][n][0] = c[m][n][1] = c[m][n][2] = c[m][n][3] = 0.f;
    const X* x[MT][2];                                               // the lane's rows
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (uint32_t h = 0; h < 2; ++h) x[m][h] = reinterpret_cast<const X*>(a.x) + (begin + min(16u * m + 8u * h + g, live - 1u)) * a.x_stride;
    const uint16_t* const down = reinterpret_cast<const uint16_t*>(a.a) + (uint64_t(i) * a.rank + min(g, a.rank - 1u)) * a.n_in;
    for (uint32_t u = u0 + warp; u < u1; u += kAdWarps * kAhead) {
      uint4 xf[kAhead][MT][2], af[kAhead][NT][kLane / 8];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const uint32_t now = u + kAdWarps * k, e = now * kUnit + t * kLane;
        const bool in = now < u1;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (uint32_t h = 0; h < kLane / 8; ++h)
            af[k][n][h] = piece_of<uint16_t, VEC>(down + 8u * n * a.n_in, e + 8u * h, a.n_in, in && 8u * n + g < a.rank);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (uint32_t h = 0; h < 2; ++h) xf[k][m][h] = piece_of<X, VEC>(x[m][h], e, a.n_in, in && 16u * m + 8u * h + g < live);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
#pragma unroll
        for (uint32_t j = 0; j < kSteps; ++j) {
          uint32_t xw[MT][4];
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t* const w = &xf[k][m][h].x;
              if constexpr (F8) {
                xw[m][h] = open_e4m3(w[j] & 0xFFFFu);
                xw[m][h + 2] = open_e4m3(w[j] >> 16);
              } else {
                xw[m][h] = w[2 * j];
                xw[m][h + 2] = w[2 * j + 1];
              }
            }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const uint32_t* const w = &af[k][n][j / 2].x;
            const uint32_t b0 = w[2 * (j % 2)], b1 = w[2 * (j % 2) + 1];
#pragma unroll
            for (int m = 0; m < MT; ++m) mma_bf16(c[m][n], xw[m][0], xw[m][1], xw[m][2], xw[m][3], b0, b1);
          }
        }
    }
    float* const to = parts + warp * S::kPart;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        *reinterpret_cast<float2*>(to + (16 * m + g) * (R + 8) + 8 * n + 2 * t) = make_float2(c[m][n][0], c[m][n][1]);
        *reinterpret_cast<float2*>(to + (16 * m + g + 8) * (R + 8) + 8 * n + 2 * t) = make_float2(c[m][n][2], c[m][n][3]);
      }
    __syncthreads();
    const uint32_t part = blockIdx.x - ad_block_of(all, blocks, uint64_t(tile) * steps);
    float* const h = a.room + (uint64_t(part) * a.rows + begin) * R;
#pragma unroll
    for (uint32_t n = 0; n < S::kSums / kAdThreads; ++n) {
      const uint32_t e = threadIdx.x + n * kAdThreads;
      if (e / R >= live) break;
      float sum = 0.f;
#pragma unroll
      for (uint32_t w = 0; w < kAdWarps; ++w) sum += parts[w * S::kPart + (e / R) * (R + 8) + e % R];
      h[e] = e % R < a.rank ? sum : 0.f;                 // not what the zeros behind the rank make of an infinity
    }
    __syncthreads();                                     // the warps' sums are read
  }
}

// `most` and `down`: of the kernel before, its parts of a tile's sums and its grid.  EXACT: the rank is R, outputs come in whole groups of 32, and B, y
// and out can be accessed 8 and 16 bytes at a time: addresses are then constants apart and nothing is asked.
template <int R, int MT, bool EXACT>
__global__ void __launch_bounds__(kAdThreads, 2) ans_adapters_up_kernel(const AdArgs a, const uint32_t most, const uint32_t down, const uint32_t down_steps) {
  using S = AdShape<R, MT>;
  constexpr int KT = R / 16;
  extern __shared__ __align__(16) uint8_t smem[];
  __nv_bfloat16* const high = reinterpret_cast<__nv_bfloat16*>(smem);
  __nv_bfloat16* const low = high + S::kRows * S::kHRow;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
  uint8_t* const ring = reinterpret_cast<uint8_t*>(low + S::kRows * S::kHRow) + warp * S::kRing;
  let_next_start();
  wait_for_previous();
  uint32_t* const first_down = reinterpret_cast<uint32_t*>(smem + S::kUpSmem);          // [n_seqs + 1]
  uint32_t* const first = first_down + a.n_seqs + 1;                                   // [n_seqs + 1]
  const uint2 counts = ad_tiles<S::kRows>(a, first_down, first, false);
  const uint32_t tiles = counts.y, groups = (a.n_out + 31u) / 32u;
  const uint32_t steps = (groups + kAdWarps - 1) / kAdWarps;
  const uint64_t all = uint64_t(tiles) * steps;
  const uint32_t blocks = static_cast<uint32_t>(min(uint64_t(gridDim.x), all));
  if (blockIdx.x >= blocks) return;
  const uint32_t down_blocks = ad_down_blocks(down, most, counts.x, down_steps);
  AdShare share = ad_share(all, steps, blocks, blockIdx.x);
  uint32_t s = ad_request(first, a.n_seqs, share.tile);
  for (; share.left; ++share.tile, share.in = 0) {
    const uint32_t tile = share.tile, count = min(steps - share.in, share.left);
    const uint32_t o0 = kAdWarps * share.in, o1 = min(groups, o0 + kAdWarps * count);
    share.left -= count;
    while (first[s + 1] <= tile) ++s;
    const int32_t i = a.which[s];
    const bool none = i < 0 || static_cast<uint32_t>(i) >= a.count;
    const uint32_t r0 = (tile - first[s]) * S::kRows, live = min(S::kRows, static_cast<uint32_t>(a.starts[s + 1] - a.starts[s]) - r0);
    const uint64_t begin = uint64_t(a.starts[s]) + r0;

    // rows of B for group o: column g of product j stands for output 32 o + 8 (g / 2) + 2 j + g % 2, and products k take
    // elements t R / 4 + 4 k and on of a row
    const uint32_t b_out = 8u * (g >> 1) + (g & 1u), b_in = t * (R / 4), b_row = EXACT ? R : a.rank;
    const __nv_bfloat16* const b_lane = a.b + (uint64_t(none ? 0 : i) * a.n_out + b_out) * b_row + b_in;
    auto load_b = [&](uint32_t o, uint32_t (&f)[4][KT][2]) {
      const __nv_bfloat16* const rows = b_lane + uint64_t(o) * (32u * b_row);
      const bool ours = o < o1 && !none;
      const uint32_t left = ours ? a.n_out - 32u * o : 0u;             // outputs from the group's first on
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const __nv_bfloat16* const row = rows + 2u * j * b_row;
#pragma unroll
        for (uint32_t k = 0; k < KT; ++k) {
          if constexpr (EXACT) {
            if (ours) {
              const uint2 u = *reinterpret_cast<const uint2*>(row + 4u * k);
              f[j][k][0] = u.x; f[j][k][1] = u.y;
            }
          } else {
            const bool in = b_out + 2u * j < left;
            f[j][k][0] = f[j][k][1] = 0u;
            if (a.b_wide) {
              if (in && b_in + 4u * k < a.rank) {
                const uint2 u = *reinterpret_cast<const uint2*>(row + 4u * k);
                f[j][k][0] = u.x; f[j][k][1] = u.y;
              }
            } else {
#pragma unroll
              for (uint32_t h = 0; h < 4; ++h)
                if (in && b_in + 4u * k + h < a.rank)
                  f[j][k][h / 2] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(row)[4u * k + h]) << (16 * (h % 2));
            }
          }
        }
      }
    };
    // groups of y: 16 bytes a lane and copy, a group ring slot a commit
    const uint32_t y_shift = a.y_f32 ? 3u : 2u, y_size = a.y_f32 ? 4u : 2u;        // 2^y_shift pieces of 16 bytes a row
    const uint32_t slot_bytes = S::kRows << (y_shift + 4u), slots = S::kRing / slot_bytes;
    const uint8_t* const y = static_cast<const uint8_t*>(a.y) + begin * a.y_stride * y_size;
    uint8_t* const out = static_cast<uint8_t*>(a.out) + begin * a.out_stride * y_size;
    const uint32_t y_row = lane >> y_shift, y_at = 16u * (lane & ((1u << y_shift) - 1u)), y_rows = 32u >> y_shift;
    const uint64_t y_down = y_rows * a.y_stride * y_size;
    const uint8_t* const y_lane = y + y_row * a.y_stride * y_size + y_at;
    const uint32_t ring_lane = smem_addr(ring) + lane * 16u;
    const bool whole = live == S::kRows;
    auto fetch_y = [&](uint32_t o, uint32_t slot) {
      const uint64_t across = uint64_t(32u * y_size) * o;
      if ((EXACT || a.y_wide) && o < o1 && (EXACT || across + y_at + 16u <= uint64_t(a.n_out) * y_size)) {
        const uint8_t* from = y_lane + across;
        uint32_t to = ring_lane + slot * slot_bytes;
        if (EXACT && whole && y_shift == 2) {
#pragma unroll
          for (uint32_t n = 0; n < S::kRows / 8; ++n, from += y_down, to += 512u)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
        } else {
          for (uint32_t row = y_row; row < live; row += y_rows, from += y_down, to += 512u)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory");
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (uint32_t n = 0; n < slots; ++n) fetch_y(o0 + warp + kAdWarps * n, n);
    constexpr uint32_t kBs = R <= 32 ? 2 : 1;                          // groups whose rows of B are loaded ahead
    uint32_t bf[kBs][4][KT][2];
#pragma unroll
    for (uint32_t n = 0; n < kBs; ++n) load_b(o0 + warp + kAdWarps * n, bf[n]);

    __syncthreads();                                     // the rows of h before are read
    if (!none) {
      const float scale = a.scales ? a.scales[i] : 1.f;
      const float* const h = a.room + begin * R;
      const uint64_t all_steps = uint64_t(counts.x) * down_steps, step = uint64_t(first_down[s] + (tile - first[s])) * down_steps;
      const uint32_t sums = ad_block_of(all_steps, down_blocks, step + down_steps - 1u) - ad_block_of(all_steps, down_blocks, step) + 1u;
#pragma unroll
      for (uint32_t n = 0; n < S::kSums / kAdThreads; ++n) {
        const uint32_t e = threadIdx.x + n * kAdThreads, row = e / R, k = e % R;
        float v[8], sum = 0.f;                                         // of all parts, under way together
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) v[p] = p < sums && row < live ? h[uint64_t(p) * a.rows * R + e] : 0.f;
#pragma unroll
        for (uint32_t p = 0; p < 8; ++p) sum += v[p];
        sum *= a.x_scales && row < live ? a.x_scales[begin + row] * scale : scale;
        constexpr float kMost = 3.3895313892515355e38f;                // the largest bf16 number: what is finite stays so
        const __nv_bfloat16 hi = __float2bfloat16_rn(isfinite(sum) ? fminf(fmaxf(sum, -kMost), kMost) : sum);
        const float rest = sum - __bfloat162float(hi);
        high[row * S::kHRow + k] = hi;
        low[row * S::kHRow + k] = __float2bfloat16_rn(isfinite(rest) ? rest : 0.f);
      }
      __syncthreads();
    }

    // h as the operand, in registers where they hold it
    constexpr bool kHeld = MT * R <= 64;
    uint2 held[kHeld ? MT : 1][kHeld ? KT : 1][4];
    auto operand_of = [&](uint32_t m, uint32_t k, uint2 (&v)[4]) {
      const uint32_t up = (16u * m + g) * S::kHRow + t * (R / 4) + 4u * k, dn = up + 8u * S::kHRow;
      v[0] = *reinterpret_cast<const uint2*>(low + up); v[1] = *reinterpret_cast<const uint2*>(low + dn);
      v[2] = *reinterpret_cast<const uint2*>(high + up); v[3] = *reinterpret_cast<const uint2*>(high + dn);
    };
    if constexpr (kHeld)
      if (!none)
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int k = 0; k < KT; ++k) operand_of(m, k, held[m][k]);

    uint32_t slot = 0;
    uint8_t* out_lane = out + (g * a.out_stride + 8u * t) * y_size + uint64_t(32u * y_size) * (o0 + warp);
    const uint64_t out_down = 8u * a.out_stride * y_size;
#pragma unroll 1
    for (uint32_t first = o0 + warp; first < o1; first += kAdWarps * kBs) {
#pragma unroll
      for (uint32_t n = 0; n < kBs; ++n, out_lane += 32u * y_size * kAdWarps) {
        const uint32_t o = first + kAdWarps * n;
        if (o >= o1) break;
        const uint32_t at = 32u * o + 8u * t;                          // the lane's outputs: at .. at + 7
        const bool wide = EXACT || (a.y_wide && at + 8 <= a.n_out);
        if (slots == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        const uint8_t* const staged = ring + slot * slot_bytes;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          float d[4][4];
          if (!none) {
#pragma unroll
            for (uint32_t k = 0; k < KT; ++k) {
              uint2 v[4];
              if constexpr (kHeld) {
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = held[m][k][q];
              } else {
                operand_of(m, k, v);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                if (k == 0) mma_bf16_first(d[j], v[0].x, v[1].x, v[0].y, v[1].y, bf[n][j][k][0], bf[n][j][k][1]);
                else mma_bf16(d[j], v[0].x, v[1].x, v[0].y, v[1].y, bf[n][j][k][0], bf[n][j][k][1]);
              }
#pragma unroll
              for (int j = 0; j < 4; ++j) mma_bf16(d[j], v[2].x, v[3].x, v[2].y, v[3].y, bf[n][j][k][0], bf[n][j][k][1]);
            }
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t r = 16u * m + 8u * h + g;
            if (r >= live) continue;
            float v[8];
            uint8_t* const p = out_lane + (2 * m + h) * out_down;
            if (wide) {
              const uint4* const q = reinterpret_cast<const uint4*>(staged) + ((r * 4u + t) << (y_shift - 2u));
              if (a.y_f32) {
                const uint4 w = q[0], z = q[1];
                v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
                v[4] = __uint_as_float(z.x); v[5] = __uint_as_float(z.y); v[6] = __uint_as_float(z.z); v[7] = __uint_as_float(z.w);
              } else {
                const uint4 u = q[0];
                const uint32_t* const w = &u.x;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  v[2 * k] = __uint_as_float(w[k] << 16);
                  v[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
                }
              }
              if (!none)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  v[2 * j] += d[j][2 * h];
                  v[2 * j + 1] += d[j][2 * h + 1];
                }
              if (a.y_f32) {
                reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
              } else {
                *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
              }
            } else {
              const uint8_t* const q = y + (r * a.y_stride + at) * y_size;
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (at + k < a.n_out) {
                  float u = a.y_f32 ? reinterpret_cast<const float*>(q)[k] : __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(q)[k]);
                  if (!none) u += d[k / 2][2 * h + k % 2];
                  if (a.y_f32) reinterpret_cast<float*>(p)[k] = u;
                  else reinterpret_cast<__nv_bfloat16*>(p)[k] = __float2bfloat16_rn(u);
                }
            }
          }
        }
        __syncwarp();
        load_b(o + kAdWarps * kBs, bf[n]);
        fetch_y(o + kAdWarps * slots, slot);
        slot = slot + 1u == slots ? 0u : slot + 1u;
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// What a call with more rows than requests launches.
struct AdPlan {
  int r, mt;                         // the rank as the kernels have it, and 16 rows each
  uint32_t down, up;                 // blocks
  uint32_t most;                     // parts of a tile's sums
  size_t room;
};
static AdPlan plan_adapters(const ans_adapters_desc& d, int sms) {
  AdPlan p{};
  p.r = d.rank <= 16 ? 16 : d.rank <= 32 ? 32 : d.rank <= 64 ? 64 : 128;
  // tiles of 16 rows where requests have about as many, else of 32, if registers hold their sums
  p.mt = p.r == 128 || uint64_t(d.rows) <= 16ull * d.n_seqs ? 1 : 2;
  const uint64_t tiles = d.rows / (16u * p.mt) + d.n_seqs;
  // as many blocks as have their places on the GPU at once, as far as there are steps for them and not more than 8 parts of
  // a tile's inputs
  p.up = static_cast<uint32_t>(std::min<uint64_t>(uint64_t(sms) * 2, tiles * ((d.n_out + 32 * kAdWarps - 1) / (32 * kAdWarps))));
  p.down = uint64_t(sms) * (p.r * p.mt >= 128 ? 1 : 2);
  p.most = static_cast<uint32_t>(std::min<uint64_t>(p.down / tiles + 2, 8));
  p.down = static_cast<uint32_t>(std::min<uint64_t>(p.down, tiles * p.most));
  p.room = size_t(p.most) * d.rows * p.r * sizeof(float);
  return p;
}

template <int R, int MT, bool F8, bool VEC>
static int launch_down(const AdArgs& a, const AdPlan& p, cudaStream_t st) {
  using S = AdShape<R, MT>;
  constexpr auto kernel = ans_adapters_down_kernel<R, MT, F8, VEC>;
  const int rc = allow_smem<kernel>(S::kDownSmem + 4 * (ANS_MAX_SEQS + 1));
  return rc == ANS_OK ? launch(kernel, dim3(p.down), dim3(kAdThreads), S::kDownSmem + 4 * (a.n_seqs + 1), st, 1, a, p.most) : rc;
}
template <int R, int MT, bool EXACT>
static int launch_up(const AdArgs& a, const AdPlan& p, uint32_t steps, cudaStream_t st) {
  using S = AdShape<R, MT>;
  constexpr auto kernel = ans_adapters_up_kernel<R, MT, EXACT>;
  const int rc = allow_smem<kernel>(S::kUpSmem + 8 * (ANS_MAX_SEQS + 1));
  return rc == ANS_OK ? launch(kernel, dim3(p.up), dim3(kAdThreads), S::kUpSmem + 8 * (a.n_seqs + 1), st, 1, a, p.most, p.down, steps) : rc;
}
template <int R, int MT>
static int launch_both(const AdArgs& a, const AdPlan& p, bool f8, bool vec, cudaStream_t st) {
  const int rc = f8 ? (vec ? launch_down<R, MT, true, true>(a, p, st) : launch_down<R, MT, true, false>(a, p, st))
              : (vec ? launch_down<R, MT, false, true>(a, p, st) : launch_down<R, MT, false, false>(a, p, st));
  if (rc != ANS_OK) return rc;
  const uint32_t inputs = (f8 ? 64u : 32u) * kAdWarps, steps = (a.n_in + inputs - 1) / inputs;       // as the first kernel has them
  return a.rank == R && a.n_out % 32 == 0 && a.b_wide && a.y_wide ? launch_up<R, MT, true>(a, p, steps, st) : launch_up<R, MT, false>(a, p, steps, st);
}
static int launch_tiles_of(const AdArgs& a, const AdPlan& p, bool f8, bool vec, cudaStream_t st) {
  switch (p.r) {
    case 16: return p.mt == 1 ? launch_both<16, 1>(a, p, f8, vec, st) : launch_both<16, 2>(a, p, f8, vec, st);
    case 32: return p.mt == 1 ? launch_both<32, 1>(a, p, f8, vec, st) : launch_both<32, 2>(a, p, f8, vec, st);
    case 64: return p.mt == 1 ? launch_both<64, 1>(a, p, f8, vec, st) : launch_both<64, 2>(a, p, f8, vec, st);
    default: return launch_both<128, 1>(a, p, f8, vec, st);
  }
}

}  // namespace blk
}  // namespace ansb

using namespace ansb;
using namespace ansb::blk;

ANS_EXPORT int ans_adapters_room_bytes(const ans_adapters_desc* h_desc, size_t* h_bytes_out) {
  if (!h_desc || !h_bytes_out) return ANS_ERR_INVALID_ARG;
  if (h_desc->rank == 0 || h_desc->n_in == 0) return ANS_ERR_INVALID_ARG;
  if (h_desc->rank > 128 || h_desc->n_seqs > ANS_MAX_SEQS || h_desc->rows > 0x7FFFFFFFu || h_desc->n_in > (1u << 22) || h_desc->n_out > (1u << 30)) return ANS_ERR_UNSUPPORTED;
  *h_bytes_out = 0;
  if (h_desc->rows <= h_desc->n_seqs || h_desc->n_seqs == 0 || h_desc->n_out == 0) return ANS_OK;
  int sms = 0;
  const int rc = sm_count(&sms);
  if (rc == ANS_OK) *h_bytes_out = plan_adapters(*h_desc, sms).room;
  return rc;
}

ANS_EXPORT int ans_adapters(const ans_adapters_desc* h_desc, uint32_t* d_status, void* stream) {
  ApiRange range("ans_adapters");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  const ans_adapters_desc& d = *h_desc;
  if (d.x_dtype != ANS_BF16 && d.x_dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  if (d.y_dtype != ANS_BF16 && d.y_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (d.rank == 0 || d.n_in == 0) return ANS_ERR_INVALID_ARG;
  if (d.rank > 128 || d.n_seqs > ANS_MAX_SEQS || d.rows > 0x7FFFFFFFu || d.n_in > (1u << 22) || d.n_out > (1u << 30) || d.count > 0x7FFFFFFFu) return ANS_ERR_UNSUPPORTED;
  if (d.rows == 0 || d.n_seqs == 0 || d.n_out == 0) return ANS_OK;
  if (!d.d_x || !d.d_y || !d.d_out || !d.d_which || !d.d_starts || (d.count && (!d.d_a || !d.d_b))) return ANS_ERR_INVALID_ARG;
  const uint64_t xs = d.x_dtype == ANS_E4M3 ? 1 : 2, ys = d.y_dtype == ANS_F32 ? 4 : 2;
  if (reinterpret_cast<uintptr_t>(d.d_x) & (xs - 1) || (reinterpret_cast<uintptr_t>(d.d_y) | reinterpret_cast<uintptr_t>(d.d_out)) & (ys - 1) ||
      (reinterpret_cast<uintptr_t>(d.d_a) | reinterpret_cast<uintptr_t>(d.d_b)) & 1)
    return ANS_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(d.d_x_scales), static_cast<const void*>(d.d_scales), static_cast<const void*>(d.d_which),
                        static_cast<const void*>(d.d_starts)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kFar = uint64_t(1) << 36;
  if (d.rows > 1 && (d.x_stride < d.n_in || d.y_stride < d.n_out || d.out_stride < d.n_out)) return ANS_ERR_INVALID_ARG;
  if (d.rows > 1 && d.d_y == d.d_out && d.y_stride != d.out_stride) return ANS_ERR_INVALID_ARG;
  if (d.x_stride > kFar || d.y_stride > kFar || d.out_stride > kFar) return ANS_ERR_UNSUPPORTED;
  AdArgs a{};
  a.x = static_cast<const uint8_t*>(d.d_x); a.x_scales = d.d_x_scales; a.y = d.d_y; a.out = d.d_out;
  a.a = static_cast<const __nv_bfloat16*>(d.d_a); a.b = static_cast<const __nv_bfloat16*>(d.d_b); a.scales = d.d_scales;
  a.which = d.d_which; a.starts = d.d_starts;
  a.x_stride = d.x_stride; a.y_stride = d.y_stride; a.out_stride = d.out_stride;
  a.rows = d.rows; a.n_seqs = d.n_seqs; a.count = d.count; a.rank = d.rank; a.n_in = d.n_in; a.n_out = d.n_out;
  a.status = d_status;
  const uint64_t many = d.rows > 1;
  const bool vec = !((reinterpret_cast<uintptr_t>(d.d_x) | (many * d.x_stride * xs) | reinterpret_cast<uintptr_t>(d.d_a) | (uint64_t(d.n_in) * 2) |
                      (uint64_t(d.n_in) * xs)) & 15);
  a.b_run = !((reinterpret_cast<uintptr_t>(d.d_b) | (uint64_t(d.n_out) * d.rank * 2)) & 15);
  a.b_wide = d.rank % 4 == 0 && !(reinterpret_cast<uintptr_t>(d.d_b) & 7);
  a.y_wide = !((reinterpret_cast<uintptr_t>(d.d_y) | reinterpret_cast<uintptr_t>(d.d_out) | (many * d.y_stride * ys) | (many * d.out_stride * ys)) & 15);
  a.y_f32 = ys == 4;
  int sms = 0;
  const int asked = sm_count(&sms);
  if (asked != ANS_OK) return asked;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (d.rows <= d.n_seqs) return launch_adapters_rows(a, d.x_dtype == ANS_E4M3, vec, sms, st);
  const AdPlan p = plan_adapters(d, sms);
  if (!d.d_room || d.room_bytes < p.room) return ANS_ERR_BUFFER_TOO_SMALL;
  if (reinterpret_cast<uintptr_t>(d.d_room) & 15) return ANS_ERR_INVALID_ARG;
  a.room = static_cast<float*>(d.d_room);
  return launch_tiles_of(a, p, d.x_dtype == ANS_E4M3, vec, st);
}
