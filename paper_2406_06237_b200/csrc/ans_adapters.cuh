// The arguments of the adapters' kernels.
#pragma once

#include "ans_blocks.cuh"

namespace ansb {
namespace blk {

struct AdArgs {
  const uint8_t* x; const float* x_scales; const void* y; void* out;
  const __nv_bfloat16* a; const __nv_bfloat16* b; const float* scales;
  const int32_t* which; const int32_t* starts;
  uint64_t x_stride, y_stride, out_stride;
  uint32_t rows, n_seqs, count, rank, n_in, n_out;
  uint32_t b_run;                    // runs of 32 rows of B start on 16 bytes
  uint32_t b_wide, y_wide;           // four elements of B, eight of y and out can be accessed at once
  uint32_t y_f32;                    // y and out in fp32, else bf16
  float* room;                       // [part of the inputs][row][rank as the kernels have it]
  uint32_t* status;
};

constexpr uint32_t kAdWarps = 8, kAdThreads = 32 * kAdWarps;

// for batches of about a row a request; vec: rows of x and of A can be read 8 elements at a time
int launch_adapters_rows(const AdArgs& a, bool f8, bool vec, int sms, cudaStream_t st);

}  // namespace blk
}  // namespace ansb
