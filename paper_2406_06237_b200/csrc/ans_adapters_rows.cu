// Low-rank adapters for single rows (a decode step): out[t] = y[t] + scales[i] * x_scales[t] * (x[t] A_i^T) B_i^T.
//
// All there is to do is to read A_i and B_i, so everything is asked for at once: a cluster of blocks has a row, each block a part of
// the inputs and a part of the outputs; its part of B goes into shared memory (cp.async) while its part of A is multiplied out of registers.
// One multiply-add an element on the plain units, in fp32: with one row the matrix instructions would work on 15 rows of zeros
// and cost more instructions around them than they save.  The blocks' sums meet through distributed shared memory in the order of the ranks.
// 64 rows of 8192 inputs and 8192 outputs at rank 16 (36 MB of adapters): 12.9 us, 6.3 of which an empty launch of the
// same clusters takes; one row 5.0.
#include <cuda_fp16.h>

#include "ans_adapters.cuh"

namespace ansb {
namespace blk {

constexpr uint32_t kArRing = 8192;                     // bytes of B of a warp: groups of 32 outputs, 64 * rank bytes each

__device__ __forceinline__ void open8(const uint4& w, float (&v)[8]) {           // eight bf16
  const uint32_t* const e = &w.x;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(e[k] << 16);
    v[2 * k + 1] = __uint_as_float(e[k] & 0xFFFF0000u);
  }
}
template <bool VEC>
__device__ __forceinline__ uint4 eight_of(const uint16_t* p, uint32_t e, uint32_t n) {           // elements e .. e + 7 of n, then zeros
  uint4 w = make_uint4(0, 0, 0, 0);
  if constexpr (VEC) {
    if (e < n) w = *reinterpret_cast<const uint4*>(p + e);
  } else {
    uint32_t* const u = &w.x;
#pragma unroll
    for (uint32_t k = 0; k < 8; ++k)
      if (e + k < n) u[k / 2] |= static_cast<uint32_t>(p[e + k]) << (16 * (k % 2));
  }
  return w;
}

// The lane's output of a group of 32: rows of B of P pieces of 16 bytes lie one after the other, a lane takes piece lane % P of the rows
// lane / P + 32 / P j, in the order in which they lie, and the P lanes of a row exchange their sums until each has a row's.
template <uint32_t P>
__device__ __forceinline__ float across(const uint8_t* rows, uint32_t lane, const float (&hp)[8]) {
  float sum[P];
#pragma unroll
  for (uint32_t j = 0; j < P; ++j) {
    float z[8];
    open8(*reinterpret_cast<const uint4*>(rows + lane * 16u + j * 512u), z);
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int n = 0; n < 8; n += 2) {
      s = fmaf(hp[n], z[n], s);
      u = fmaf(hp[n + 1], z[n + 1], u);
    }
    sum[j] = s + u;
  }
#pragma unroll
  for (uint32_t n = P / 2; n >= 1; n /= 2)             // lane bit n: which half of the rows it goes on with
#pragma unroll
    for (uint32_t k = 0; k < n; ++k) {
      const bool up = lane & n;
      const float give = up ? sum[k] : sum[k + n], keep = up ? sum[k + n] : sum[k];
      sum[k] = keep + __shfl_xor_sync(kAll, give, n);
    }
  // lane l has row l / P + 32 / P (l % P): its own output's is with lane (l % (32 / P)) P + l / (32 / P)
  return P == 1 ? sum[0] : __shfl_sync(kAll, sum[0], (lane % (32u / P)) * P + lane / (32u / P));
}

template <bool F8, bool VEC>
__global__ void __launch_bounds__(kAdThreads, 2) ans_adapters_rows_kernel(const AdArgs a) {
  constexpr uint32_t kUnit = 256, kRows = 16;          // inputs of a warp, rows of A at a time
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float parts[kAdWarps][128], mine[128];
  __shared__ __align__(16) float h[128];
  constexpr uint32_t kYs = 8;
  __shared__ uint32_t ahead[kYs][kAdThreads];          // y of a warp's next groups, of each lane its own
  __shared__ uint32_t s_seq;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  uint32_t ranks;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const uint32_t rank = cluster_rank(), row = blockIdx.x / ranks;
  let_next_start();
  wait_for_previous();
  if (warp == 0) {
    uint32_t count = 0;                                // of requests that begin at or before the row; those before them have ended
    for (uint32_t s0 = 0; s0 < a.n_seqs; s0 += 1024) {
      uint32_t here = 0;
#pragma unroll 8
      for (uint32_t s = s0 + lane; s < min(s0 + 1024u, a.n_seqs); s += 32) here += a.starts[s] <= static_cast<int32_t>(row) ? 1u : 0u;
      here = __reduce_add_sync(kAll, here);
      count += here;
      if (here < min(1024u, a.n_seqs - s0)) break;
    }
    if (lane == 0) s_seq = count ? count - 1u : 0u;
  }
  __syncthreads();
  const uint32_t s = s_seq;
  const int32_t r0 = a.starts[s], r1 = a.starts[s + 1], last = a.starts[a.n_seqs];
  int32_t i = a.which[s];
  if (row == 0 && rank == 0) {                         // what does not fit is found by one block
    bool bad = last < 0 || static_cast<uint32_t>(last) > a.rows;
    for (uint32_t k = threadIdx.x; k < a.n_seqs; k += kAdThreads) bad |= a.starts[k] < 0 || a.starts[k + 1] < a.starts[k];
    if (bad) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
  }
  // the same for the whole cluster
  if (r0 < 0 || static_cast<int32_t>(row) < r0 || static_cast<int32_t>(row) >= r1 || static_cast<uint32_t>(r1) > a.rows) return;
  if (i >= 0 && static_cast<uint32_t>(i) >= a.count) {
    if (rank == 0 && threadIdx.x == 0) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
    i = -1;
  }
  const bool none = i < 0;
  if (none && a.out == a.y) return;

  // B: a group of 32 outputs is one run of 64 * rank bytes
  const uint32_t groups = (a.n_out + 31u) / 32u, bytes = 64u * a.rank, slots = kArRing / bytes;
  const uint32_t o0 = static_cast<uint32_t>(uint64_t(groups) * rank / ranks), o1 = static_cast<uint32_t>(uint64_t(groups) * (rank + 1u) / ranks);
  const __nv_bfloat16* const b = a.b + uint64_t(max(i, 0)) * a.n_out * a.rank;
  uint8_t* const ring = smem + warp * kArRing;
  const bool staged = !none && a.b_run;
  auto fetch = [&](uint32_t o, uint32_t slot) {
    if (staged && o < o1) {
      const uint8_t* const from = reinterpret_cast<const uint8_t*>(b) + uint64_t(o) * bytes;
      const uint32_t have = static_cast<uint32_t>(min(uint64_t(bytes), (uint64_t(a.n_out) - 32u * o) * a.rank * 2u));
      const uint32_t to = smem_addr(ring) + slot * bytes;
      for (uint32_t at = lane * 16u; at < have; at += 512u)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to + at), "l"(from + at), "r"(min(16u, have - at)) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  for (uint32_t n = 0; n < slots; ++n) fetch(o0 + warp + kAdWarps * n, n);
  // y of the lane's output in a warp's next kYs groups
  const uint32_t size = a.y_f32 ? 4u : 2u;
  const uint8_t* const y = static_cast<const uint8_t*>(a.y) + row * a.y_stride * size;
  uint8_t* const out = static_cast<uint8_t*>(a.out) + row * a.out_stride * size;
  uint32_t ys[kYs];
  auto y_of = [&](uint32_t o) {
    const uint32_t at = 32u * o + lane;
    if (o >= o1 || at >= a.n_out) return 0u;
    return a.y_f32 ? reinterpret_cast<const uint32_t*>(y)[at] : static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(y)[at]);
  };
#pragma unroll
  for (uint32_t n = 0; n < kYs; ++n) ys[n] = y_of(o0 + warp + kAdWarps * n);

  if (!none) {
    const uint32_t units = (a.n_in + kUnit - 1) / kUnit;
    const uint32_t u0 = static_cast<uint32_t>(uint64_t(units) * rank / ranks), u1 = static_cast<uint32_t>(uint64_t(units) * (rank + 1u) / ranks);
    const uint16_t* const down = reinterpret_cast<const uint16_t*>(a.a) + uint64_t(i) * a.rank * a.n_in;
    const uint8_t* const x = a.x + row * a.x_stride * (F8 ? 1 : 2);
    const float factor = (a.scales ? a.scales[i] : 1.f) * (a.x_scales ? a.x_scales[row] : 1.f);
    for (uint32_t k0 = 0; k0 < a.rank; k0 += kRows) {
      float sum[kRows];
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) sum[k] = 0.f;
      for (uint32_t u = u0 + warp; u < u1; u += kAdWarps) {
        const uint32_t e = u * kUnit + lane * 8u;
        uint4 w[kRows];
#pragma unroll
        for (uint32_t k = 0; k < kRows; ++k)
          w[k] = k0 + k < a.rank ? eight_of<VEC>(down + uint64_t(k0 + k) * a.n_in, e, a.n_in) : make_uint4(0, 0, 0, 0);
        float v[8];
        if constexpr (F8) {
          uint32_t q[2] = {0, 0};
          if constexpr (VEC) {
            if (e < a.n_in) {
              const uint2 z = *reinterpret_cast<const uint2*>(x + e);
              q[0] = z.x; q[1] = z.y;
            }
          } else {
#pragma unroll
            for (uint32_t k = 0; k < 8; ++k)
              if (e + k < a.n_in) q[k / 4] |= static_cast<uint32_t>(x[e + k]) << (8 * (k % 4));
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const __half2_raw z = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(q[k / 2] >> (16 * (k % 2))), __NV_E4M3);
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&z));
            v[2 * k] = f.x;
            v[2 * k + 1] = f.y;
          }
        } else {
          open8(eight_of<VEC>(reinterpret_cast<const uint16_t*>(x), e, a.n_in), v);
        }
#pragma unroll
        for (uint32_t k = 0; k < kRows; ++k) {
          float z[8];
          open8(w[k], z);
#pragma unroll
          for (int n = 0; n < 8; ++n) sum[k] = fmaf(v[n], z[n], sum[k]);
        }
      }
      // sixteen sums over 32 lanes: halves are exchanged, so that a lane has one at the end
#pragma unroll
      for (uint32_t step = 16, n = kRows / 2; n >= 1; step /= 2, n /= 2) {
#pragma unroll
        for (uint32_t k = 0; k < n; ++k) {
          const bool up = lane & step;
          const float give = up ? sum[k] : sum[k + n], keep = up ? sum[k + n] : sum[k];
          sum[k] = keep + __shfl_xor_sync(kAll, give, step);
        }
      }
      sum[0] += __shfl_xor_sync(kAll, sum[0], 1);
      if (!(lane & 1u)) parts[warp][k0 + (lane >> 1)] = sum[0];       // lane bits 4 .. 1: the row, most significant first
    }
    __syncthreads();
    if (threadIdx.x < 128) {
      float sum = 0.f;
      if (threadIdx.x < a.rank)
#pragma unroll
        for (uint32_t w = 0; w < kAdWarps; ++w) sum += parts[w][threadIdx.x];
      mine[threadIdx.x] = sum;
    }
    if (ranks > 1) cluster_sync(); else __syncthreads();
    if (threadIdx.x < 128) {
      float v[8], sum = 0.f;
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r)
        if (r < ranks)
          asm volatile("{\n\t.reg .b32 p;\n\tmapa.shared::cluster.u32 p, %1, %2;\n\tld.shared::cluster.f32 %0, [p];\n\t}"
                       : "=f"(v[r]) : "r"(smem_addr(mine + threadIdx.x)), "r"(r));
#pragma unroll
      for (uint32_t r = 0; r < 8; ++r)
        if (r < ranks) sum += v[r];
      h[threadIdx.x] = sum * factor;
    }
    __syncthreads();
    if (ranks > 1) cluster_arrive();                                 // this block has read the others' sums
  }

  const uint32_t pieces = a.rank % 8 == 0 ? a.rank / 8u : 0u;
  float hp[8];                                         // of the lane's piece
#pragma unroll
  for (uint32_t k = 0; k < 8; ++k) hp[k] = none || !pieces ? 0.f : h[(lane % pieces) * 8u + k];
  uint32_t slot = 0;
  for (uint32_t first = o0 + warp; first < o1; first += kAdWarps * kYs) {
#pragma unroll
    for (uint32_t n = 0; n < kYs; ++n) ahead[n][threadIdx.x] = ys[n];
#pragma unroll
    for (uint32_t n = 0; n < kYs; ++n) ys[n] = y_of(first + kAdWarps * (kYs + n));
#pragma unroll 1                                                     // short code: most of it runs once a block, out of a cold instruction cache
    for (uint32_t n = 0; n < kYs; ++n) {
      const uint32_t o = first + kAdWarps * n, at = 32u * o + lane;
      if (o >= o1) break;
      const bool in = at < a.n_out;
      float v = a.y_f32 ? __uint_as_float(ahead[n][threadIdx.x]) : __uint_as_float(ahead[n][threadIdx.x] << 16);
      // all but the slots behind this one may be on their way: waits for a few are kinds of instruction
      if (slots >= 8) asm volatile("cp.async.wait_group 7;" ::: "memory");
      else if (slots >= 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
      else if (slots >= 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
      else asm volatile("cp.async.wait_group 0;" ::: "memory");
      __syncwarp();
      const uint8_t* const rows = ring + slot * bytes;
      if (none) {
      } else if (staged && pieces == 1) {
        v += across<1>(rows, lane, hp);
      } else if (staged && pieces == 2) {
        v += across<2>(rows, lane, hp);
      } else if (staged && pieces == 4) {
        v += across<4>(rows, lane, hp);
      } else if (staged && pieces == 8) {
        v += across<8>(rows, lane, hp);
      } else if (in) {
        const uint16_t* const far = reinterpret_cast<const uint16_t*>(b) + uint64_t(at) * a.rank;
        const uint16_t* const near = reinterpret_cast<const uint16_t*>(rows) + lane * a.rank;
        float sum = 0.f;
        for (uint32_t k = 0; k < a.rank; ++k) sum = fmaf(h[k], __uint_as_float(static_cast<uint32_t>(staged ? near[k] : far[k]) << 16), sum);
        v += sum;
      }
      if (in) {
        if (a.y_f32) reinterpret_cast<float*>(out)[at] = v;
        else reinterpret_cast<__nv_bfloat16*>(out)[at] = __float2bfloat16_rn(v);
      }
      __syncwarp();
      fetch(o + kAdWarps * slots, slot);
      slot = slot + 1u == slots ? 0u : slot + 1u;
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (!none && ranks > 1) cluster_wait();                            // nobody reads this block's sums any more
}

template <bool F8, bool VEC>
static int launch_rows_of(const AdArgs& a, uint32_t ranks, cudaStream_t st) {
  constexpr auto kernel = ans_adapters_rows_kernel<F8, VEC>;
  constexpr size_t kSmem = kAdWarps * kArRing;
  const int rc = allow_smem<kernel>(kSmem);
  return rc == ANS_OK ? launch(kernel, dim3(a.rows * ranks), dim3(kAdThreads), kSmem, st, ranks, a) : rc;
}
int launch_adapters_rows(const AdArgs& a, bool f8, bool vec, int sms, cudaStream_t st) {
  // as many blocks a row as have their places on the GPU at once, two an SM; at most 8
  uint32_t ranks = 8;
  while (ranks > 1 && uint64_t(a.rows) * ranks > 2ull * sms) ranks /= 2;
  if (f8) return vec ? launch_rows_of<true, true>(a, ranks, st) : launch_rows_of<true, false>(a, ranks, st);
  return vec ? launch_rows_of<false, true>(a, ranks, st) : launch_rows_of<false, false>(a, ranks, st);
}

}  // namespace blk
}  // namespace ansb
