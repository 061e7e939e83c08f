// What the two attention kernels share: the call's arguments and the formulas of the softmax.
//
// With s_i = scale * log2(e) * (q . k_i), k_i = kscale_i * kcode_i, v_i = vscale_i * vcode_i, the output is
//   sum_i 2^(s_i) vscale_i vcode_i / sum_i 2^(s_i).
// The scales of values go into the exponent: e_i = log2(vscale_i), M = max_i (s_i + e_i), and
//   P_i = 2^(s_i + e_i - M + kUp),   out = 2^kSum * sum_i P_i vcode_i / L,   L = 2^(kUp + kSum) * sum_i 2^(s_i - M) = sum_i P_i 2^(kSum - e_i),
// so that the matrix instructions meet small integers (codes, exact in fp16) with P_i <= 2^kUp in fp16, whose relative error of
// 2^-11 then reaches down to 2^-(14 + kUp) of the largest term, and no product with a scale is rounded on its own.  Scales that
// the cache's write makes are powers of two, so e_i is an integer and the terms of L are exact multiples of P_i.
// L adds the P_i before they are rounded to fp16.
//
// e_i is -40 to 128.  2^(kSum - e_i) is then a normal number, and L one of 2^-101 to 2^105 (2^30 tokens).  As a P_i below fp32's range
// may still count in L, where the largest e is far above its own (a block of zeros beside values of 1e30), blocks whose e is kApart below the
// largest one met so far add 2^(s_i - M + kUp + kSum) to L by an exponential of their own: what is lost elsewhere is under 2^-40 of the largest
// term of L.  For the same reason L goes to another M by two factors of half the exponent.
// A block of 16 tokens lies in one page, so both scales are constants of such a block.
#pragma once

#include "ans_blocks.cuh"

namespace ansb {
namespace blk {

constexpr float kUp = 14.f;
constexpr float kSum = 20.f, kFromSum = 1048576.f;     // 2^kSum
constexpr float kApart = 90.f;
constexpr float kLowest = -3.402823466e38f;

struct AttendArgs {
  Cache c;
  Batch b;
  const __nv_bfloat16* q; __nv_bfloat16* out;
  uint64_t q_token, q_head, out_token, out_head;       // strides, elements
  uint32_t share, window, causal;
  uint32_t share_by, share_shift;                      // x / share = x * share_by >> share_shift, x < 2^31
  uint32_t out_wide;                                   // eight values of out can be stored at once
  float scale2;                                        // scale * log2(e)
  uint32_t least, most;                                // a kernel takes sequences of least .. most rows (new tokens * share)
  float* parts;                                        // partial results: see the kernels
  uint32_t* status;
};

// A row of a sequence (new token * share + query of the head): its token.  With k the bits of share - 1, share_by = ceil(2^(31 + k) / share) and
// share_shift = 31 + k the quotient is exact: the product is off by x * (less than share) < 2^(31 + k).
__device__ __forceinline__ uint32_t token_of(const AttendArgs& a, uint32_t row) {
  return static_cast<uint32_t>(uint64_t(row) * a.share_by >> a.share_shift);
}

// The tokens that new token i of a sequence sees are [first, end).
struct Seen { int32_t first, end; };
__device__ __forceinline__ Seen seen_by(const AttendArgs& a, int32_t old, int32_t length, uint32_t i) {
  Seen r;
  r.end = a.causal ? max(min(old + static_cast<int32_t>(i) + 1, length), 0) : length;
  r.first = a.window && static_cast<uint32_t>(r.end) > a.window ? r.end - static_cast<int32_t>(a.window) : 0;
  return r;
}

// The exponent by which a row of queries is brought to a largest magnitude in [1, 2), from that magnitude's bits: row = 2^e * (1 .. 2).
// An infinity or a NaN stays one.
__device__ __forceinline__ int32_t exponent_of(uint32_t top) { return min(max(static_cast<int32_t>(top >> 23), 1), 253) - 127; }
__device__ __forceinline__ float power_of(int32_t e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace blk
}  // namespace ansb
