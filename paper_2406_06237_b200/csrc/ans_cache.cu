// A paged cache of keys and values, quantised with a zero-point as it is written and read back by pages.
//
// Per group of values of one (token, head), L = 2^b - 1, u = 1 / L, lo = min(x, 0), hi = max(x, 0):
//   scale = max(hi * u - lo * u, 2^-126),  zero = rint(-lo / scale),  code = clamp(rint(x / scale) + zero, 0, L)
// and back  scale * (code - zero).  The results are those of IEEE divisions, so codes are a function of the
// values alone and equal on every device and in any IEEE restatement.
//
// Both directions are bound by memory.  Writing takes eight values a thread (16 bytes of bf16), reading sixteen.
#include <cmath>
#include <initializer_list>

#include "ans_tensor.cuh"

namespace ansb {

struct CacheArgs {
  uint8_t* codes[2];                 // [0]: keys, [1]: values
  float* scales[2];
  uint8_t* zeros[2];
  uint64_t slots;                    // n_pages * page_size
  uint32_t page_size, n_pages, heads, head_dim, group;
};

struct WriteArgs {
  CacheArgs c;
  const void* x[2];
  uint64_t token_stride[2], head_stride[2];
  const int64_t* slot;
  uint64_t tokens;
  uint32_t* status;
  uint32_t wide[2];                  // every run of 8 values starts on 16 bytes
};

// LANES (a power of two) lanes per group, eight values each, lanes past group / 8 idle.  blockIdx.y: keys or values.
template <typename T, int BITS, int LANES>
__global__ void __launch_bounds__(256) ans_cache_write_kernel(const WriteArgs a) {
  ten::let_next_start();
  const uint32_t which = blockIdx.y;
  const uint32_t lane = threadIdx.x % LANES;
  const uint32_t per_head = a.c.head_dim / a.c.group, per_token = a.c.heads * per_head;
  const uint64_t unit = (uint64_t(blockIdx.x) * 256u + threadIdx.x) / LANES;      // (token, head, group)
  const uint64_t token = unit / per_token;
  const uint32_t in_token = static_cast<uint32_t>(unit - token * per_token);
  int64_t slot = -1;
  ten::wait_for_previous();
  if (token < a.tokens) {
    slot = a.slot[token];
    if (slot >= 0 && static_cast<uint64_t>(slot) >= a.c.slots) {
      if (lane == 0 && in_token == 0 && which == 0) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
      slot = -1;
    }
  }
  const uint32_t head = in_token / per_head, g = in_token - head * per_head;
  const bool live = slot >= 0 && lane * 8u < a.c.group;
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = 0.f;
  if (live) {
    const T* p = static_cast<const T*>(a.x[which]) + token * a.token_stride[which] + head * a.head_stride[which] + g * a.c.group + lane * 8u;
    if (a.wide[which]) {
      if constexpr (sizeof(T) == 2) {
        const uint4 u = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          v[2 * j] = __uint_as_float(w[j] << 16);
          v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
      } else {
        const float4 q0 = reinterpret_cast<const float4*>(p)[0], q1 = reinterpret_cast<const float4*>(p)[1];
        v[0] = q0.x; v[1] = q0.y; v[2] = q0.z; v[3] = q0.w; v[4] = q1.x; v[5] = q1.y; v[6] = q1.z; v[7] = q1.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = static_cast<float>(p[i]);
    }
  }
  float lo = 0.f, hi = 0.f;
  bool odd = false;                                       // an infinity or a NaN
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, v[i]);
    hi = fmaxf(hi, v[i]);
    odd |= !(fabsf(v[i]) < INFINITY);
  }
  if (odd) hi = INFINITY;
#pragma unroll
  for (int d = LANES / 2; d; d >>= 1) {
    lo = fminf(lo, __shfl_xor_sync(ten::kAll, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(ten::kAll, hi, d));
  }
  if (!live) return;
  constexpr float L = static_cast<float>((1 << BITS) - 1);
  const uint64_t param = (uint64_t(slot) * a.c.heads + head) * per_head + g;
  float scale = fmaxf(hi * (1.f / L) - lo * (1.f / L), 1.17549435e-38f);
  float zero = fminf(rintf(-lo / scale), L);
  const float inverse = 1.f / scale;
  uint32_t code[8];
  if (hi < INFINITY) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      // v * (1 / scale) is within 2^-14 of v / scale, whose magnitude is at most 255: only near a tie between two codes
      // is the division itself needed
      const float q = v[i] * inverse;
      float n = rintf(q);
      if (fabsf(fabsf(q - n) - 0.5f) < 0.0001f) n = rintf(v[i] / scale);
      code[i] = static_cast<uint32_t>(fminf(fmaxf(n + zero, 0.f), L));
    }
  } else {
    scale = __uint_as_float(0x7FC00000u);
    zero = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) code[i] = 0;
  }
  const uint64_t at = param * a.c.group + lane * 8u;      // the first code's number in the whole array
  if constexpr (BITS == 8) {
    uint2 w;
    w.x = code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24;
    w.y = code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24;
    *reinterpret_cast<uint2*>(a.c.codes[which] + at) = w;
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= code[i] << (4 * i);
    *reinterpret_cast<uint32_t*>(a.c.codes[which] + at / 2) = w;
  }
  if (lane == 0) {
    a.c.scales[which][param] = scale;
    a.c.zeros[which][param] = static_cast<uint8_t>(zero);
  }
}

struct ReadArgs {
  CacheArgs c;
  const int32_t* tables;
  uint64_t table_stride;
  uint32_t table_pages;
  const int32_t* starts;
  uint32_t n_seqs;
  uint64_t rows;
  void* out[2];
  uint32_t* status;
};

constexpr uint32_t kReadRows = 64;    // rows of a block at most

// scale * (code - zero).  The ends of a group's range lie up to half a step outside its values, so that with
// values near the type's largest the product can pass it: such a result is that largest value.  A NaN stays.
// raised: 2^23 + code as a float; below: 2^23 + zero.  Their difference is exact.
template <typename T>
__device__ __forceinline__ float value_of(uint32_t raised, float below, float scale) {
  const float v = scale * (__uint_as_float(raised) - below);
  const float most = __uint_as_float(sizeof(T) == 2 ? 0x7F7F0000u : 0x7F7FFFFFu);
  float r;
  asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(r) : "f"(v), "f"(most));   // the smaller magnitude, v's sign
  return r;
}

// The last s in 0 .. n - 1 with starts[s] <= row (0 if there is none): a warp looks at 32 places at a time.
__device__ __forceinline__ uint32_t sequence_of(const int32_t* starts, uint32_t n, int64_t row, uint32_t lane) {
  uint32_t lo = 0, hi = n;                                // the answer lies in [lo, hi)
  while (hi - lo > 1) {
    const uint32_t step = (hi - lo + 31u) / 32u, at = lo + lane * step;
    const uint32_t below = __ballot_sync(ten::kAll, at < hi && static_cast<int64_t>(starts[at]) <= row);
    const uint32_t last = below ? 31u - __clz(below) : 0u;
    lo += last * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// A block reads `some` output rows of keys or of values (blockIdx.y).  First the slots of its rows: two warps find the
// sequences of the first and the last row, between which, most often nowhere, the others' lie.  Then
// sixteen values a thread, four of them under way at a time.
template <typename T, int BITS>
__global__ void __launch_bounds__(256) ans_cache_read_kernel(const ReadArgs a, const uint32_t some) {
  __shared__ int64_t s_slot[kReadRows];                   // -1: zeros, -2: not written
  __shared__ uint32_t s_seq[2];
  ten::let_next_start();
  const uint32_t which = blockIdx.y, warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const uint64_t row0 = uint64_t(blockIdx.x) * some;
  ten::wait_for_previous();
  const int64_t last = min(static_cast<int64_t>(a.starts[a.n_seqs]), static_cast<int64_t>(a.rows));   // rows to write
  if (warp < 2) {
    const uint32_t s = sequence_of(a.starts, a.n_seqs, static_cast<int64_t>(row0) + (warp ? some - 1 : 0), lane);
    if (lane == 0) s_seq[warp] = s;
  }
  __syncthreads();
  if (threadIdx.x < some) {
    const int64_t row = static_cast<int64_t>(row0 + threadIdx.x);
    int64_t slot = -2;
    if (row < last) {
      uint32_t lo = s_seq[0], hi = max(s_seq[0], s_seq[1]) + 1;
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (static_cast<int64_t>(a.starts[mid]) <= row) lo = mid; else hi = mid;
      }
      const int64_t pos = row - a.starts[lo];
      slot = -1;
      if (pos >= 0) {
        const uint32_t in = static_cast<uint32_t>(pos) / a.c.page_size;
        if (in < a.table_pages) {
          const int32_t page = a.tables[lo * a.table_stride + in];
          if (page >= 0 && static_cast<uint32_t>(page) < a.c.n_pages)
            slot = int64_t(page) * a.c.page_size + (static_cast<uint32_t>(pos) - in * a.c.page_size);
        }
      }
      if (slot < 0 && which == 0) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
    }
    if (row == 0 && which == 0 && static_cast<int64_t>(a.starts[a.n_seqs]) > static_cast<int64_t>(a.rows)) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
    s_slot[threadIdx.x] = slot;
  }
  __syncthreads();
  const uint32_t width = a.c.heads * a.c.head_dim, units = width / 16u, per_row = width / a.c.group;
  constexpr uint32_t kAhead = 4;
  for (uint32_t i0 = threadIdx.x; i0 < some * units; i0 += 256u * kAhead) {
    uint32_t w[kAhead][BITS / 2];
    float scale[kAhead];
    uint32_t zero[kAhead];
    int64_t slot[kAhead];
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      const uint32_t i = i0 + j * 256u;
      slot[j] = -2;
      if (i < some * units) {
        const uint32_t r = i / units, e = (i - r * units) * 16u;
        slot[j] = s_slot[r];
        if (slot[j] >= 0) {
          const uint64_t at = uint64_t(slot[j]) * width + e, param = uint64_t(slot[j]) * per_row + e / a.c.group;
          if constexpr (BITS == 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(a.c.codes[which] + at);
            w[j][0] = u.x; w[j][1] = u.y; w[j][2] = u.z; w[j][3] = u.w;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(a.c.codes[which] + at / 2);
            w[j][0] = u.x; w[j][1] = u.y;
          }
          scale[j] = *(a.c.scales[which] + param);
          zero[j] = *(a.c.zeros[which] + param);
        }
      }
    }
#pragma unroll
    for (uint32_t j = 0; j < kAhead; ++j) {
      if (slot[j] == -2) continue;
      const uint32_t i = i0 + j * 256u, r = i / units, e = (i - r * units) * 16u;
      float v[16];
      if (slot[j] >= 0) {
        const float below = 8388608.f + static_cast<float>(zero[j]);
#pragma unroll
        for (uint32_t n = 0; n < 16; ++n) {
          const uint32_t raised = BITS == 8 ? __byte_perm(w[j][n / 4], 0x4B000000u, 0x7540u + n % 4)
                                            : ((w[j][n / 8] >> (4 * (n % 8))) & 15u) | 0x4B000000u;
          v[n] = value_of<T>(raised, below, scale[j]);
        }
      } else {
#pragma unroll
        for (uint32_t n = 0; n < 16; ++n) v[n] = 0.f;
      }
      const uint64_t to = (row0 + r) * width + e;
      if constexpr (sizeof(T) == 2) {
        uint32_t o[8];
#pragma unroll
        for (uint32_t n = 0; n < 8; ++n) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * n], v[2 * n + 1]);
          o[n] = *reinterpret_cast<const uint32_t*>(&b);
        }
        uint4* p = reinterpret_cast<uint4*>(static_cast<T*>(a.out[which]) + to);
        p[0] = make_uint4(o[0], o[1], o[2], o[3]);
        p[1] = make_uint4(o[4], o[5], o[6], o[7]);
      } else {
        float4* p = reinterpret_cast<float4*>(static_cast<T*>(a.out[which]) + to);
#pragma unroll
        for (uint32_t n = 0; n < 4; ++n) p[n] = make_float4(v[4 * n], v[4 * n + 1], v[4 * n + 2], v[4 * n + 3]);
      }
    }
  }
}

static int check_cache(const ans_cache_desc& d, CacheArgs& c) {
  if (d.bitwidth != 8 && d.bitwidth != 4) return ANS_ERR_UNSUPPORTED;
  if (d.group < 16 || d.group > 256 || d.group % 16 || d.head_dim == 0 || d.head_dim % d.group) return ANS_ERR_UNSUPPORTED;
  if (d.heads == 0 || d.page_size == 0) return ANS_ERR_INVALID_ARG;
  if (uint64_t(d.heads) * d.head_dim > (1u << 20) || d.n_pages > 0x7FFFFFFFu || d.page_size > (1u << 20)) return ANS_ERR_UNSUPPORTED;
  if (d.n_pages && (!d.d_k_codes || !d.d_v_codes || !d.d_k_scales || !d.d_v_scales || !d.d_k_zeros || !d.d_v_zeros)) return ANS_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(d.d_k_codes), static_cast<const void*>(d.d_v_codes),
                        static_cast<const void*>(d.d_k_scales), static_cast<const void*>(d.d_v_scales)})
    if (reinterpret_cast<uintptr_t>(p) & 15) return ANS_ERR_INVALID_ARG;
  c.codes[0] = d.d_k_codes; c.codes[1] = d.d_v_codes;
  c.scales[0] = d.d_k_scales; c.scales[1] = d.d_v_scales;
  c.zeros[0] = d.d_k_zeros; c.zeros[1] = d.d_v_zeros;
  c.slots = uint64_t(d.n_pages) * d.page_size;
  c.page_size = d.page_size; c.n_pages = d.n_pages; c.heads = d.heads; c.head_dim = d.head_dim; c.group = d.group;
  return ANS_OK;
}

template <typename T, int BITS>
static int launch_write(const WriteArgs& a, cudaStream_t st) {
  const uint32_t need = a.c.group / 8u;
  const uint32_t lanes = need <= 2 ? 2 : need <= 4 ? 4 : need <= 8 ? 8 : need <= 16 ? 16 : 32;
  const uint64_t units = a.tokens * a.c.heads * (a.c.head_dim / a.c.group);
  const uint64_t blocks = (units * lanes + 255) / 256;
  if (blocks > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks), 2);
  switch (lanes) {
    case 2: return ten::launch(ans_cache_write_kernel<T, BITS, 2>, grid, dim3(256), 0, st, 1, a);
    case 4: return ten::launch(ans_cache_write_kernel<T, BITS, 4>, grid, dim3(256), 0, st, 1, a);
    case 8: return ten::launch(ans_cache_write_kernel<T, BITS, 8>, grid, dim3(256), 0, st, 1, a);
    case 16: return ten::launch(ans_cache_write_kernel<T, BITS, 16>, grid, dim3(256), 0, st, 1, a);
    default: return ten::launch(ans_cache_write_kernel<T, BITS, 32>, grid, dim3(256), 0, st, 1, a);
  }
}

}  // namespace ansb

using namespace ansb;

ANS_EXPORT int ans_cache_write(const ans_cache_desc* h_desc, const void* d_k, const void* d_v, int dtype, uint64_t tokens,
                               uint64_t k_token_stride, uint64_t k_head_stride, uint64_t v_token_stride,
                               uint64_t v_head_stride, const int64_t* d_slots, uint32_t* d_status, void* stream) {
  ApiRange range("ans_cache_write");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  WriteArgs a{};
  const int rc = check_cache(*h_desc, a.c);
  if (rc != ANS_OK) return rc;
  if (dtype != ANS_BF16 && dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (tokens == 0) return ANS_OK;
  if (!d_k || !d_v || !d_slots || (reinterpret_cast<uintptr_t>(d_slots) & 7)) return ANS_ERR_INVALID_ARG;
  const uint64_t size = dtype == ANS_BF16 ? 2 : 4;
  if ((reinterpret_cast<uintptr_t>(d_k) % size) || (reinterpret_cast<uintptr_t>(d_v) % size)) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kMost = uint64_t(1) << 40;
  if (tokens > kMost || k_token_stride > kMost || k_head_stride > kMost || v_token_stride > kMost || v_head_stride > kMost)
    return ANS_ERR_UNSUPPORTED;
  a.x[0] = d_k; a.x[1] = d_v;
  a.token_stride[0] = k_token_stride; a.token_stride[1] = v_token_stride;
  a.head_stride[0] = k_head_stride; a.head_stride[1] = v_head_stride;
  a.slot = d_slots; a.tokens = tokens; a.status = d_status;
  for (int w = 0; w < 2; ++w)
    a.wide[w] = !((reinterpret_cast<uintptr_t>(a.x[w]) | (a.token_stride[w] * size) | (a.head_stride[w] * size)) & 15);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (dtype == ANS_BF16) return h_desc->bitwidth == 8 ? launch_write<__nv_bfloat16, 8>(a, st) : launch_write<__nv_bfloat16, 4>(a, st);
  return h_desc->bitwidth == 8 ? launch_write<float, 8>(a, st) : launch_write<float, 4>(a, st);
}

ANS_EXPORT int ans_cache_read(const ans_cache_desc* h_desc, const int32_t* d_tables, uint64_t table_stride,
                              uint32_t table_pages, uint32_t n_seqs, const int32_t* d_starts, uint64_t rows, void* d_k_out,
                              void* d_v_out, int out_dtype, uint32_t* d_status, void* stream) {
  ApiRange range("ans_cache_read");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  ReadArgs a{};
  const int rc = check_cache(*h_desc, a.c);
  if (rc != ANS_OK) return rc;
  if (out_dtype != ANS_BF16 && out_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (rows == 0 || n_seqs == 0) return ANS_OK;
  if ((!d_tables && table_pages) || !d_starts || !d_k_out || !d_v_out) return ANS_ERR_INVALID_ARG;
  if (n_seqs > 1 && table_stride < table_pages) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d_k_out) | reinterpret_cast<uintptr_t>(d_v_out)) & 15) return ANS_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d_tables) | reinterpret_cast<uintptr_t>(d_starts)) & 3) return ANS_ERR_INVALID_ARG;
  if (rows > 0x7FFFFFFFull || n_seqs > 0x7FFFFFFFu || table_stride > (uint64_t(1) << 40)) return ANS_ERR_UNSUPPORTED;
  a.tables = d_tables; a.table_stride = table_stride; a.table_pages = table_pages; a.starts = d_starts; a.n_seqs = n_seqs; a.rows = rows;
  a.out[0] = d_k_out; a.out[1] = d_v_out; a.status = d_status;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // rows of a block: enough blocks for eight on each SM, up to 64 rows each, over which a block's look-up is spread
  int dev = 0, sms = 0;
  ANSB_CUDA(cudaGetDevice(&dev));
  ANSB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  const uint64_t share = rows / (4u * static_cast<uint64_t>(sms));
  const uint32_t some = share < 4 ? 4u : share > kReadRows ? kReadRows : static_cast<uint32_t>(share);
  const dim3 grid(static_cast<unsigned>((rows + some - 1) / some), 2);
  if (out_dtype == ANS_BF16)
    return h_desc->bitwidth == 8 ? ten::launch(ans_cache_read_kernel<__nv_bfloat16, 8>, grid, dim3(256), 0, st, 1, a, some)
                                 : ten::launch(ans_cache_read_kernel<__nv_bfloat16, 4>, grid, dim3(256), 0, st, 1, a, some);
  return h_desc->bitwidth == 8 ? ten::launch(ans_cache_read_kernel<float, 8>, grid, dim3(256), 0, st, 1, a, some)
                               : ten::launch(ans_cache_read_kernel<float, 4>, grid, dim3(256), 0, st, 1, a, some);
}
