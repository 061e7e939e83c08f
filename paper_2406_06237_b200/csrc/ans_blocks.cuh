// What the kernels on a block-scaled cache share: the batch, the sequences' ranges, codes opened to fp16.
#pragma once

#include <cuda_fp16.h>

#include "ans_tensor.cuh"

namespace ansb {
namespace blk {

using namespace ten;

constexpr float kLeastScale = 9.094947017729282e-13f;  // 2^-40

struct Batch {
  const int32_t* tables; uint64_t table_stride; uint32_t table_pages;
  uint32_t n_seqs, rows;
  const int32_t* lengths; const int32_t* starts;
};
struct Cache {
  int8_t* codes[2];                  // [0]: keys, [1]: values
  float* scales[2];
  uint32_t n_pages, page_size, heads, dim;
};

// A sequence's rows and tokens, as far as they can be used: `fits` is false where they do not lie in the batch.
struct Range {
  uint32_t row, fresh, length;       // first row, new tokens, tokens
  bool fits;
};
__device__ __forceinline__ Range range_of(const Batch& b, uint32_t s) {
  const int32_t r0 = b.starts[s], r1 = b.starts[s + 1], len = b.lengths[s];
  Range r;
  r.fits = r0 >= 0 && r1 >= r0 && static_cast<uint32_t>(r1) <= b.rows && len >= 0;
  r.row = r0;
  r.fresh = r.fits ? r1 - r0 : 0u;
  r.length = len;
  return r;
}

// Of places dealt out so that sequence s has starts[s] / per + each * s and on (times `share` first): the sequence of place `at`, for a
// whole warp.  All starts of up to 1024 sequences are asked for together: one trip to memory, where halving would take one a step.
__device__ __forceinline__ uint32_t sequence_at(const int32_t* starts, uint32_t n, uint32_t share, uint32_t per, uint32_t each, uint32_t at) {
  const uint32_t lane = threadIdx.x & 31u;
  uint32_t count = 0;                                  // of sequences that begin at or before the place: they come first
  for (uint32_t s0 = 0; s0 < n; s0 += 1024) {
    uint32_t here = 0;
#pragma unroll 8
    for (uint32_t s = s0 + lane; s < min(s0 + 1024u, n); s += 32)
      here += static_cast<uint32_t>(uint64_t(max(starts[s], 0)) * share / per) + each * s <= at ? 1u : 0u;
    here = __reduce_add_sync(kAll, here);
    count += here;
    if (here < min(1024u, n - s0)) break;
  }
  return count ? count - 1u : 0u;
}

// Four codes in a word, opened to two pairs of fp16: 0x6400 | u is 1024 + u, u = code + 128.
__device__ __forceinline__ __half2 less_1152(uint32_t w) {
  return __hsub2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0x6480)));
}
__device__ __forceinline__ uint32_t open_low(uint32_t offset_codes) {            // bytes 0 and 1
  const __half2 h = less_1152(__byte_perm(offset_codes, 0x64646464u, 0x4140));
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t open_high(uint32_t offset_codes) {           // bytes 2 and 3
  const __half2 h = less_1152(__byte_perm(offset_codes, 0x64646464u, 0x4342));
  return *reinterpret_cast<const uint32_t*>(&h);
}

// 2^x to about 2^-22 of it
__device__ __forceinline__ float exp2_near(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_near(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A block's scale as the formulas use it: at least 2^-40, NaN where it is NaN.
__device__ __forceinline__ float usable(float scale) { return scale < kLeastScale ? kLeastScale : scale; }

// ---- host side -----------------------------------------------------------------------------
int check_block_cache(const ans_block_cache_desc& d, Cache& c);
int check_batch(const ans_batch_desc& d, Batch& b);

}  // namespace blk
}  // namespace ansb
