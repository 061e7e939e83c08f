// Writing into a paged cache in 8 bits with one scale for each block (page) and head.
//
// The scale is the least power of two s >= 2^-40 with max|x| <= 127 s.  With max|x| = m 2^e, 1 <= m < 2, that is 2^(e - 6)
// if m <= 127/64 and 2^(e - 5) otherwise: exponent arithmetic on the bits, no logarithm.  As dividing by a power of two is exact,
// a code rint(x / s) rounds once, and codes are a function of the values alone, whatever the order or the precision of the
// arithmetic; codes that are rounded to a larger scale are shifted by whole bits.  What that costs is up to one bit of a block's 7
// (half a bit on average); what it saves beside the exactness is most of the rescaling, since a scale grows only
// past a power of two.
//
// A block of threads has one (sequence, page, head) of the keys or of the values: the new values' largest magnitude, the scale,
// the codes.  The values are held in registers between the two, 64 a thread (32 in fp32), by as many threads as that takes for a
// page, 128 to 512; what a larger page has more is read again.  8194 tokens of 8 heads of 128 in pages of 64: 15.0 us held, 18.0 read
// again when held it was 15.1; 8000 in pages of 128 14.4, and 23.0 by 128 threads that also waited for the old scale first; 1750 of 4 heads of 256 in fp32 in pages of
// 128 6.7 and 17.1.  Bound by issue (61 % of the slots) and the blocks' own beginnings where prompts are written, by latency (numbers of
// the sequence, page number, values, codes: four trips) for single tokens.  Both keys and values by one block took 16.5 for the 15.1.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ans_blocks.cuh"

namespace ansb {
namespace blk {

struct BlockWriteArgs {
  Cache c;
  Batch b;
  const void* x[2];
  uint64_t token_stride[2], head_stride[2];
  uint32_t wide[2];                  // eight values can be loaded at once
  uint32_t* status;
};

// Eight values from p on, as they lie, and as fp32.
template <typename T> struct Eight { uint32_t w[2 * sizeof(T)]; };
template <typename T>
__device__ __forceinline__ Eight<T> load8(const T* p, uint32_t wide) {
  Eight<T> s;
  if (wide) {
#pragma unroll
    for (uint32_t h = 0; h < sizeof(T) / 2; ++h) {
      const uint4 u = reinterpret_cast<const uint4*>(p)[h];
      s.w[4 * h] = u.x; s.w[4 * h + 1] = u.y; s.w[4 * h + 2] = u.z; s.w[4 * h + 3] = u.w;
    }
  } else if constexpr (sizeof(T) == 2) {
    const uint16_t* e = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) s.w[i] = e[2 * i] | static_cast<uint32_t>(e[2 * i + 1]) << 16;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) s.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
  }
  return s;
}
template <typename T>
__device__ __forceinline__ float value_of(const Eight<T>& s, int i) {
  if constexpr (sizeof(T) == 2) return __uint_as_float(i % 2 ? s.w[i / 2] & 0xFFFF0000u : s.w[i / 2] << 16);
  else return __uint_as_float(s.w[i]);
}

// The scale for a largest magnitude, given as its bits; NaN for an infinity or a NaN.
__device__ __forceinline__ float scale_for(uint32_t top) {
  if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  const int32_t e = static_cast<int32_t>(top >> 23) - ((top & 0x7FFFFFu) <= 0x7E0000u ? 6 : 5);      // m <= 127/64 = 1.984375
  return __uint_as_float(static_cast<uint32_t>(max(e, 127 - 40)) << 23);
}

// the low bytes of eight words
__device__ __forceinline__ uint2 packed(const uint32_t (&w)[8]) {
  uint2 out;
  out.x = __byte_perm(__byte_perm(w[0], w[1], 0x40), __byte_perm(w[2], w[3], 0x40), 0x5410);
  out.y = __byte_perm(__byte_perm(w[4], w[5], 0x40), __byte_perm(w[6], w[7], 0x40), 0x5410);
  return out;
}

// rint(x / scale) to nearest even for any scale, |x / scale| < 127.5, in the low bits.  x * per rounds to the quotient's neighbour at most, and
// what a whole number of steps leaves of x is exact: x itself, or a number of up to 2^24 units in the last place of x or scale.
__device__ __forceinline__ uint32_t code_of(float x, float scale, float per) {
  const float near = rintf(x * per), rest = fmaf(-near, scale, x), half = 0.5f * scale;
  const bool odd = static_cast<int32_t>(near) & 1;
  const float by = fabsf(rest) > half || (fabsf(rest) == half && odd) ? copysignf(1.f, rest) : 0.f;
  return static_cast<uint32_t>(static_cast<int32_t>(near + by));
}

// gridDim.x: at least the pages that can get tokens: sequence s has places starts[s] / P + 2 s and on, of which there are at
// least m / P + 2 before the next one's, and m new tokens lie in at most m / P + 2 pages.
// THREADS: so that a page is held, if 512 can.  Blocks an SM: registers for all loads of the held values at once; left to the compiler,
// 1600 rows of 4 x 256 in fp32 take 8.6 us, so 6.7, 8194 tokens of 8 x 128 16.1 and 15.0.
template <typename T, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == 128 ? 7 : THREADS == 256 ? 4 : 1) ans_block_write_kernel(const BlockWriteArgs a) {
  let_next_start();
  __shared__ uint32_t s_top[THREADS / 32], s_seq;
  const uint32_t P = a.c.page_size, head = blockIdx.y, which = blockIdx.z, lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  wait_for_previous();
  if (warp == 0) {
    const uint32_t found = sequence_at(a.b.starts, a.b.n_seqs, 1u, P, 2u, blockIdx.x);
    if (lane == 0) s_seq = found;
  }
  __syncthreads();
  const uint32_t s = s_seq;
  const Range r = range_of(a.b, s);
  const bool first = blockIdx.x == 0 && head == 0 && which == 0;
  if (first) {                                         // what does not fit is found by one block
    bool bad = false;
    for (uint32_t i = threadIdx.x; i < a.b.n_seqs; i += THREADS) {
      const Range q = range_of(a.b, i);
      bad |= !q.fits || q.fresh > q.length || q.length > uint64_t(a.b.table_pages) * P;
    }
    if (bad) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
  }
  if (!r.fits || r.fresh == 0 || r.fresh > r.length) return;
  const uint32_t old = r.length - r.fresh, place = r.row / P + 2u * s;
  if (blockIdx.x < place) return;
  const uint64_t page_in = uint64_t(old / P) + (blockIdx.x - place), begin = page_in * P;
  if (begin >= r.length || page_in >= a.b.table_pages) return;
  const int32_t page = a.b.tables[s * a.b.table_stride + page_in];
  if (page < 0 || static_cast<uint32_t>(page) >= a.c.n_pages) {
    if (threadIdx.x == 0) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
    return;
  }
  const uint32_t from = old > begin ? static_cast<uint32_t>(old - begin) : 0u;          // the block's new tokens: [from, to)
  const uint32_t to = static_cast<uint32_t>(min(uint64_t(P), r.length - begin));
  const uint32_t dim = a.c.dim, across = dim / 8u, pieces = (to - from) * across;
  const T* const x = static_cast<const T*>(a.x[which]) + (r.row + (begin + from - old)) * a.token_stride[which] + head * a.head_stride[which];
  const uint64_t block = uint64_t(page) * a.c.heads + head;
  int8_t* const codes = a.c.codes[which] + block * P * dim;
  float* const scale_at = a.c.scales[which] + block;
  const float lay = from ? *scale_at : 0.f;           // looked at behind the values, so as not to be waited for here

  // a thread's pieces of eight values: token t, values c .. c + 7, the next one THREADS pieces on
  const uint32_t down = THREADS / across, right = THREADS % across, t0 = threadIdx.x / across, c0 = threadIdx.x % across;
  auto move = [&](uint32_t& t, uint32_t& c) {
    t += down;
    c += right;
    if (c >= across) { c -= across; ++t; }
  };
  constexpr uint32_t kHeld = 16 / sizeof(T);
  Eight<T> held[kHeld];
  uint32_t top = 0;
  auto look = [&](const Eight<T>& s) {
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(value_of<T>(s, k)) & 0x7FFFFFFFu);
  };
  uint32_t t = t0, c = c0;
#pragma unroll
  for (uint32_t n = 0; n < kHeld; ++n, move(t, c))
    if (t < to - from) held[n] = load8(x + t * a.token_stride[which] + 8u * c, a.wide[which]);
  for (; t < to - from; move(t, c)) look(load8(x + t * a.token_stride[which] + 8u * c, a.wide[which]));
#pragma unroll
  for (uint32_t n = 0; n < kHeld; ++n)
    if (threadIdx.x + n * THREADS < pieces) look(held[n]);
  top = __reduce_max_sync(kAll, top);
  if (lane == 0) s_top[warp] = top;
  __syncthreads();                                     // the old scale is read
#pragma unroll
  for (uint32_t i = 0; i < THREADS / 32; ++i) top = max(top, s_top[i]);
  float scale = scale_for(top);
  const float before = usable(lay);
  if (from) {
    if (isnan(before)) scale = before;
    else if (before > scale) scale = before;
  }
  if (threadIdx.x == 0) *scale_at = scale;
  const bool sound = !isnan(scale);
  const float per = 1.f / scale;                       // exact: a power of two, but for scales that others have written (code_of)
  constexpr float kMagic = 12582912.f;                 // 1.5 * 2^23: rint(v) in the low bits of v + kMagic, |v| < 2^22
  auto put = [&](const Eight<T>& s) {
    uint32_t w[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) w[k] = sound ? __float_as_uint(fmaf(value_of<T>(s, k), per, kMagic)) : 0u;
    *reinterpret_cast<uint2*>(codes + (from + t) * dim + 8u * c) = packed(w);
  };
  t = t0;
  c = c0;
#pragma unroll
  for (uint32_t n = 0; n < kHeld; ++n, move(t, c))
    if (t < to - from) put(held[n]);
  for (; t < to - from; move(t, c)) put(load8(x + t * a.token_stride[which] + 8u * c, a.wide[which]));
  if (from && sound && scale > before) {               // the tokens before them, rounded to the larger scale
    const float shrink = before * per;
    for (uint32_t i = threadIdx.x; i < from * across; i += THREADS) {
      uint32_t* const p = reinterpret_cast<uint32_t*>(codes + i * 8u);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t q = p[h];
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = __float_as_uint(fmaf(static_cast<float>(static_cast<int8_t>(q >> (8 * j))), shrink, kMagic));
        p[h] = __byte_perm(__byte_perm(w[0], w[1], 0x40), __byte_perm(w[2], w[3], 0x40), 0x5410);
      }
    }
  }
  // A scale of others' holds what there is (one that grows is a power of two): a thread's codes once more, out of values read again.  Here, and
  // rolled, it leaves the registers of what comes before alone.
  if (sound && (__float_as_uint(scale) & 0x7FFFFFu)) {
#pragma unroll 1
    for (uint32_t i = threadIdx.x; i < pieces; i += THREADS) {
      const Eight<T> s = load8(x + i / across * a.token_stride[which] + 8u * (i % across), a.wide[which]);
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) w[k] = code_of(value_of<T>(s, k), scale, per);
      *reinterpret_cast<uint2*>(codes + from * dim + 8u * i) = packed(w);
    }
  }
}

int check_block_cache(const ans_block_cache_desc& d, Cache& c) {
  if (d.page_size == 0 || d.heads == 0 || d.head_dim == 0) return ANS_ERR_INVALID_ARG;
  if (d.page_size % 16 || d.page_size > 256 || d.head_dim % 16 || d.head_dim > 256) return ANS_ERR_UNSUPPORTED;
  if (d.heads > 65535u || d.n_pages > 0x7FFFFFFFu) return ANS_ERR_UNSUPPORTED;
  if (d.n_pages && (!d.d_k_codes || !d.d_v_codes || !d.d_k_scales || !d.d_v_scales)) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d.d_k_codes) | reinterpret_cast<uintptr_t>(d.d_v_codes) | reinterpret_cast<uintptr_t>(d.d_k_scales) |
       reinterpret_cast<uintptr_t>(d.d_v_scales)) & 15)
    return ANS_ERR_INVALID_ARG;
  c.codes[0] = d.d_k_codes; c.codes[1] = d.d_v_codes;
  c.scales[0] = d.d_k_scales; c.scales[1] = d.d_v_scales;
  c.n_pages = d.n_pages; c.page_size = d.page_size; c.heads = d.heads; c.dim = d.head_dim;
  return ANS_OK;
}

int check_batch(const ans_batch_desc& d, Batch& b) {
  if (d.n_seqs > ANS_MAX_SEQS || d.rows > 0x7FFFFFFFu || d.table_pages > (1u << 27) || d.table_stride > (uint64_t(1) << 40)) return ANS_ERR_UNSUPPORTED;
  if (d.n_seqs && d.rows && (!d.d_lengths || !d.d_starts || (!d.d_tables && d.table_pages))) return ANS_ERR_INVALID_ARG;
  if (d.n_seqs > 1 && d.table_stride < d.table_pages) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d.d_tables) | reinterpret_cast<uintptr_t>(d.d_lengths) | reinterpret_cast<uintptr_t>(d.d_starts)) & 3)
    return ANS_ERR_INVALID_ARG;
  b.tables = d.d_tables; b.table_stride = d.table_stride; b.table_pages = d.table_pages;
  b.n_seqs = d.n_seqs; b.rows = d.rows; b.lengths = d.d_lengths; b.starts = d.d_starts;
  return ANS_OK;
}

}  // namespace blk
}  // namespace ansb

using namespace ansb;
using namespace ansb::blk;

ANS_EXPORT int ans_block_cache_write(const ans_block_cache_desc* h_cache, const ans_batch_desc* h_batch, const void* d_k, const void* d_v,
                                     int dtype, uint64_t k_token_stride, uint64_t k_head_stride, uint64_t v_token_stride,
                                     uint64_t v_head_stride, uint32_t* d_status, void* stream) {
  ApiRange range("ans_block_cache_write");
  if (!h_cache || !h_batch || !d_status) return ANS_ERR_INVALID_ARG;
  BlockWriteArgs a{};
  int rc = check_block_cache(*h_cache, a.c);
  if (rc == ANS_OK) rc = check_batch(*h_batch, a.b);
  if (rc != ANS_OK) return rc;
  if (dtype != ANS_BF16 && dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (a.b.n_seqs == 0 || a.b.rows == 0) return ANS_OK;
  if (!d_k || !d_v) return ANS_ERR_INVALID_ARG;
  const uint64_t size = dtype == ANS_BF16 ? 2 : 4;
  if ((reinterpret_cast<uintptr_t>(d_k) % size) || (reinterpret_cast<uintptr_t>(d_v) % size)) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kMost = uint64_t(1) << 40;
  if (k_token_stride > kMost || k_head_stride > kMost || v_token_stride > kMost || v_head_stride > kMost) return ANS_ERR_UNSUPPORTED;
  a.x[0] = d_k; a.x[1] = d_v;
  a.token_stride[0] = k_token_stride; a.token_stride[1] = v_token_stride;
  a.head_stride[0] = k_head_stride; a.head_stride[1] = v_head_stride;
  for (int w = 0; w < 2; ++w)
    a.wide[w] = !((reinterpret_cast<uintptr_t>(a.x[w]) | (a.token_stride[w] * size) | (a.head_stride[w] * size)) & 15);
  a.status = d_status;
  const uint64_t places = a.b.rows / a.c.page_size + 2ull * a.b.n_seqs;
  if (places > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(places), a.c.heads, 2);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // what a block writes if the sequences share the rows evenly: single tokens into large pages need few threads (64 in pages of
  // 128 x 256: 6.2 us, with 512 threads 26)
  const uint32_t values = std::min(a.c.page_size, a.b.rows / a.b.n_seqs) * a.c.dim, per_thread = dtype == ANS_BF16 ? 64u : 32u;
  auto go = [&](auto threads) {
    constexpr uint32_t kThreads = threads();
    return dtype == ANS_BF16 ? launch(ans_block_write_kernel<__nv_bfloat16, kThreads>, grid, dim3(kThreads), 0, st, 1, a)
                             : launch(ans_block_write_kernel<float, kThreads>, grid, dim3(kThreads), 0, st, 1, a);
  };
  if (values <= 128u * per_thread) return go(std::integral_constant<uint32_t, 128>{});
  if (values <= 256u * per_thread) return go(std::integral_constant<uint32_t, 256>{});
  return go(std::integral_constant<uint32_t, 512>{});
}
