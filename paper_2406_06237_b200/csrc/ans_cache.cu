// A paged cache of keys and values, quantised with a zero-point as it is written and read back by pages.
//
// Per group of values of one (token, head), L = 2^b - 1, u = 1 / L, lo = min(x, 0), hi = max(x, 0):
//   scale = max(hi * u - lo * u, 2^-126),  zero = rint(-lo / scale),  code = clamp(rint(x / scale) + zero, 0, L)
// and back  scale * (code - zero).  The results are those of IEEE divisions, so codes are a function of the
// values alone and equal on every device and in any IEEE restatement.
//
// A thread has sixteen values of one group.  Reading is bound by memory: 64 sequences of about 1500 tokens (8 heads of 128, 8 bits)
// 72 us, 91 % of the rate of a copy with the step's write before it.  Writing is bound by instruction issue: 10240 tokens
// of the same heads in 4 bits, groups of 32, 17 us where the bytes take 8; two 16-byte loads a lane, the next piece's under way
// while one is quantised.
#include <cmath>
#include <initializer_list>

#include "ans_tensor.cuh"

namespace ansb {

using namespace ten;

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
  uint32_t wide[2];                  // every run of 16 values starts on 32 bytes: 2; on 16: 1
};

// the least and the largest of three, NaN if one of them is
__device__ __forceinline__ float least(float a, Two b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(low(b)), "f"(high(b)));
  return r;
}
__device__ __forceinline__ float largest(float a, Two b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(low(b)), "f"(high(b)));
  return r;
}

// Sixteen values from p on, as they lie, and opened.  wide: 2: on 32 bytes, 1: on 16, 0: on a value.
template <typename T> struct Sixteen { uint32_t w[4 * sizeof(T)]; };
template <typename T>
__device__ __forceinline__ Sixteen<T> load16(const T* p, uint32_t wide) {
  Sixteen<T> s;
  constexpr int kParts = sizeof(T) / 2;                   // 32 bytes each
#pragma unroll
  for (int h = 0; h < kParts; ++h) {
    uint32_t* const w = s.w + 8 * h;
    const uint4* q = reinterpret_cast<const uint4*>(p) + 2 * h;
    if (wide == 2) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(q) : "memory");
    } else if (wide == 1) {
      const uint4 a = q[0], b = q[1];
      w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    } else {
      const uint16_t* e = reinterpret_cast<const uint16_t*>(p) + 16 * h;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (kParts == 1) w[i] = e[2 * i] | static_cast<uint32_t>(e[2 * i + 1]) << 16;
        else w[i] = reinterpret_cast<const uint32_t*>(p)[8 * h + i];
      }
    }
  }
  return s;
}
template <typename T>
__device__ __forceinline__ void open16(const Sixteen<T>& s, Two (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (sizeof(T) == 2) v[i] = two(__uint_as_float(s.w[i] << 16), __uint_as_float(s.w[i] & 0xFFFF0000u));
    else v[i] = two(__uint_as_float(s.w[2 * i]), __uint_as_float(s.w[2 * i + 1]));
  }
}

// LANES (a power of two) lanes per group, sixteen values each, lanes past group / 16 idle.  blockIdx.y: keys or values.
// A block's piece of work is blockDim.y tokens, or a part of one token that has more threads' work than a block; it takes
// piece after piece and loads the next one's values before it quantises one's.
template <typename T, int BITS, int LANES>
__global__ void __launch_bounds__(256) ans_cache_write_kernel(const WriteArgs a) {
  let_next_start();
  const uint32_t which = blockIdx.y;
  const uint32_t per_head = a.c.head_dim / a.c.group, per_token = a.c.heads * per_head;
  const uint32_t lane = threadIdx.x % LANES;
  constexpr float L = static_cast<float>((1 << BITS) - 1);
  const uint32_t parts = (per_token * LANES + blockDim.x - 1) / blockDim.x;   // of a token
  const uint64_t pieces = (a.tokens + blockDim.y - 1) / blockDim.y * parts;
  wait_for_previous();
  struct Piece { Sixteen<T> s; int64_t slot; uint32_t unit; bool live; };
  // a (head, group)'s values within a token; the same for all pieces where a piece is whole tokens
  auto inside = [&](uint32_t unit) {
    const uint32_t head = unit / per_head, g = unit - head * per_head;
    return head * a.head_stride[which] + (g * a.c.group + lane * 16u);
  };
  const uint32_t unit0 = threadIdx.x / LANES;
  const bool live0 = unit0 < per_token && lane * 16u < a.c.group;
  const T* const x0 = static_cast<const T*>(a.x[which]) + inside(unit0);
  auto fetch = [&](uint64_t piece) {
    Piece p;
    uint64_t token = piece * blockDim.y + threadIdx.y;
    const T* from = x0;
    p.unit = unit0;
    p.live = live0;
    if (parts > 1) {
      const uint64_t tokens = piece / parts;
      token = tokens * blockDim.y + threadIdx.y;
      p.unit = (static_cast<uint32_t>(piece - tokens * parts) * blockDim.x + threadIdx.x) / LANES;
      p.live = p.unit < per_token && lane * 16u < a.c.group;
      from = static_cast<const T*>(a.x[which]) + inside(p.unit);
    }
    p.slot = -1;
    p.live = p.live && token < a.tokens;
    p.s = Sixteen<T>{};
    if (p.live) {
      p.slot = a.slot[token];
      p.s = load16(from + token * a.token_stride[which], a.wide[which]);
    }
    return p;
  };
  Piece next = fetch(blockIdx.x);
  for (uint64_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {     // the same trips for all of the block
    const Piece now = next;
    next = fetch(piece + gridDim.x);
    int64_t slot = now.slot;
    const bool live = now.live;
    const uint32_t unit = now.unit;
    if (slot >= 0 && static_cast<uint64_t>(slot) >= a.c.slots) {
      if (which == 0 && unit == 0 && lane == 0) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
      slot = -1;
    }
    Two v[8];
    open16(now.s, v);
    float lo = 0.f, hi = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      lo = least(lo, v[i]);
      hi = largest(hi, v[i]);
    }
#pragma unroll
    for (int d = LANES / 2; d; d >>= 1) {
      const float l = __shfl_xor_sync(kAll, lo, d), h = __shfl_xor_sync(kAll, hi, d);
      lo = least(lo, two(l, l));
      hi = largest(hi, two(h, h));
    }
    if (!live || slot < 0) continue;
    const bool finite = lo > -INFINITY && hi < INFINITY;  // neither infinite nor NaN
    float scale = fmaxf(hi * (1.f / L) - lo * (1.f / L), 1.17549435e-38f);
    // The quotients x / scale, correctly rounded (Markstein, 1990): with the correctly rounded reciprocal y of the
    // divisor, q = x y is at most a unit off, its remainder r = x - q * scale is exact, and q + r y rounds to the
    // quotient, as long as r is no subnormal number.  Ties between codes are common (bf16 values, few levels), so
    // a product by y alone would not do.  Adding 1.5 * 2^23 rounds to a whole number, in the sum's low bits.
    const float inverse = __frcp_rn(scale);
    constexpr float kWhole = 12582912.f;
    const Two y = two(inverse, inverse), s = two(-scale, -scale), up = two(kWhole, kWhole);
    auto quotient = [&](Two x) {
      const Two q = mul2(x, y);
      return fma2(fma2(q, s, x), y, q);
    };
    float zero = rintf(low(quotient(two(-lo, -lo))));
    Two m[8];
    if (scale > 1e-27f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = add2(quotient(v[i]), up);
    } else {
      zero = rintf(-lo / scale);
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = add2(two(rintf(low(v[i]) / scale), rintf(high(v[i]) / scale)), up);
    }
    zero = fminf(zero, L);
    // no code is under 0: values are at least lo, and zero is what -lo rounds to
    const int raise = static_cast<int>(zero) - __float_as_int(kWhole);
    uint32_t w[BITS / 2];
#pragma unroll
    for (int i = 0; i < BITS / 2; ++i) {
      w[i] = 0;
#pragma unroll
      for (int j = 0; j < 32 / BITS; ++j) {
        const Two pair = m[(i * (32 / BITS) + j) / 2];
        const int code = min(__float_as_int(j & 1 ? high(pair) : low(pair)) + raise, (1 << BITS) - 1);
        w[i] |= static_cast<uint32_t>(code) << (BITS * j);
      }
    }
    if (!finite) {
      scale = __uint_as_float(0x7FC00000u);
      zero = 0.f;
#pragma unroll
      for (int i = 0; i < BITS / 2; ++i) w[i] = 0;
    }
    const uint64_t param = uint64_t(slot) * per_token + unit;
    const uint64_t at = param * a.c.group + lane * 16u;   // the first code's number in the whole array
    if constexpr (BITS == 8) *reinterpret_cast<uint4*>(a.c.codes[which] + at) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(a.c.codes[which] + at / 2) = make_uint2(w[0], w[1]);
    if (lane == 0) {
      a.c.scales[which][param] = scale;
      a.c.zeros[which][param] = static_cast<uint8_t>(zero);
    }
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
  uint32_t wide;                     // outputs on 32 bytes
};

constexpr uint32_t kReadRows = 256;   // rows of a block at most

// Sixteen codes in w to scale * (code - zero), two at a time: a code set under the exponent of 2^23 is 2^23 + code * 16^k
// (k: its place among the four nibbles of a half word; 0 for whole bytes), from which 2^23 + zero * 16^k is
// subtracted without error, and scale / 16^k, exact too where it is no subnormal number, gives the product's one rounding.
template <int BITS>
__device__ __forceinline__ void open_codes(const uint32_t (&w)[BITS / 2], uint32_t zero, float scale, Two (&v)[8]) {
  constexpr float kRaise = 8388608.f;
  const float z = static_cast<float>(zero);
  if constexpr (BITS == 8) {
    const Two below = two(-kRaise - z, -kRaise - z), s = two(scale, scale);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const Two raised = two(__uint_as_float(__byte_perm(w[n / 2], 0x4B000000u, 0x7540u + (2 * n) % 4)),
                             __uint_as_float(__byte_perm(w[n / 2], 0x4B000000u, 0x7540u + (2 * n + 1) % 4)));
      v[n] = mul2(add2(raised, below), s);
    }
  } else {
    const Two below[2] = {two(-kRaise - z, -kRaise - 16.f * z), two(-kRaise - 256.f * z, -kRaise - 4096.f * z)};
    const Two s[2] = {two(scale, scale * 0.0625f), two(scale * 0.00390625f, scale * 0.000244140625f)};
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const uint32_t h = n & 2 ? w[n / 4] >> 16 : w[n / 4];
      const uint32_t mask = n & 1 ? 0xF00u : 0xFu;
      const Two raised = two(__uint_as_float((h & mask) | 0x4B000000u), __uint_as_float((h & (mask << 4)) | 0x4B000000u));
      v[n] = mul2(add2(raised, below[n & 1]), s[n & 1]);
    }
  }
}
// The same for scales of any size.  The ends of a group's range lie up to half a step outside its values, so that
// with values near the type's largest the product can pass it: such a result is that largest value.  A NaN stays.
template <typename T, int BITS>
__device__ __forceinline__ void open_any(const uint32_t (&w)[BITS / 2], uint32_t zero, float scale, Two (&v)[8]) {
  const float most = __uint_as_float(sizeof(T) == 2 ? 0x7F7F0000u : 0x7F7FFFFFu);
  float f[16];
#pragma unroll
  for (int n = 0; n < 16; ++n) {
    const uint32_t code = BITS == 8 ? (w[n / 4] >> (8 * (n % 4))) & 255u : (w[n / 8] >> (4 * (n % 8))) & 15u;
    f[n] = scale * static_cast<float>(static_cast<int>(code) - static_cast<int>(zero));
    asm("min.NaN.xorsign.abs.f32 %0, %1, %2;" : "=f"(f[n]) : "f"(f[n]), "f"(most));   // the smaller magnitude, the value's sign
  }
#pragma unroll
  for (int n = 0; n < 8; ++n) v[n] = two(f[2 * n], f[2 * n + 1]);
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
// sixteen values a thread, always of the same columns, four rows under way at a time.
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
  const uint32_t across = min(units, 256u), down = 256u / across;        // threads over a row, rows at a time
  const uint32_t r0 = threadIdx.x / across;
  if (r0 >= down) return;
  constexpr uint32_t kAhead = 4;
  for (uint32_t c = threadIdx.x - r0 * across; c < units; c += across) {
    const uint32_t e = c * 16u, group = e / a.c.group;
    const uint8_t* const codes = a.c.codes[which] + (BITS == 8 ? e : e / 2);
    const float* const scales = a.c.scales[which] + group;
    const uint8_t* const zeros = a.c.zeros[which] + group;
    T* const out = static_cast<T*>(a.out[which]) + row0 * width + e;
    for (uint32_t r = r0; r < some; r += kAhead * down) {
      uint32_t w[kAhead][BITS / 2], zero[kAhead];
      float scale[kAhead];
      bool to[kAhead];
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) {
        const uint32_t at = r + j * down;
        const int64_t slot = at < some ? s_slot[at] : -2;
        to[j] = slot != -2;
        scale[j] = 0.f;                                   // no page: zeros
        zero[j] = 0;
#pragma unroll
        for (int i = 0; i < BITS / 2; ++i) w[j][i] = 0;
        if (slot >= 0) {
          const uint8_t* const p = codes + uint64_t(slot) * (BITS == 8 ? width : width / 2);
          if constexpr (BITS == 8) {
            const uint4 u = *reinterpret_cast<const uint4*>(p);
            w[j][0] = u.x; w[j][1] = u.y; w[j][2] = u.z; w[j][3] = u.w;
          } else {
            const uint2 u = *reinterpret_cast<const uint2*>(p);
            w[j][0] = u.x; w[j][1] = u.y;
          }
          scale[j] = scales[uint64_t(slot) * per_row];
          zero[j] = zeros[uint64_t(slot) * per_row];
        }
      }
#pragma unroll
      for (uint32_t j = 0; j < kAhead; ++j) {
        if (!to[j]) continue;
        Two v[8];
        if (scale[j] == 0.f || (scale[j] > 1e-33f && scale[j] < 1e36f)) open_codes<BITS>(w[j], zero[j], scale[j], v);
        else open_any<T, BITS>(w[j], zero[j], scale[j], v);
        T* const p = out + uint64_t(r + j * down) * width;
        if constexpr (sizeof(T) == 2) {
          uint32_t o[8];
#pragma unroll
          for (uint32_t n = 0; n < 8; ++n) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(low(v[n]), high(v[n]));
            o[n] = *reinterpret_cast<const uint32_t*>(&b);
          }
          if (a.wide) {
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         :: "l"(p), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
          } else {
            reinterpret_cast<uint4*>(p)[0] = make_uint4(o[0], o[1], o[2], o[3]);
            reinterpret_cast<uint4*>(p)[1] = make_uint4(o[4], o[5], o[6], o[7]);
          }
        } else {
#pragma unroll
          for (uint32_t n = 0; n < 4; ++n)
            reinterpret_cast<float4*>(p)[n] = make_float4(low(v[2 * n]), high(v[2 * n]), low(v[2 * n + 1]), high(v[2 * n + 1]));
        }
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
  const uint32_t need = a.c.group / 16u;
  const uint32_t lanes = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : need <= 8 ? 8 : 16;
  const uint32_t threads = a.c.heads * (a.c.head_dim / a.c.group) * lanes;        // of a token
  const uint32_t across = threads >= 256 ? 256u : 32u % threads == 0 ? threads : (threads + 31u) / 32u * 32u;
  const dim3 block(across, 256u / across);
  const uint64_t pieces = (a.tokens + block.y - 1) / block.y * ((threads + block.x - 1) / block.x);
  int sms = 0;
  const int asked = ten::sm_count(&sms);
  if (asked != ANS_OK) return asked;
  // up to five blocks an SM, keys and values together (what registers hold)
  const uint64_t most = 5ull * sms / 2;
  const dim3 grid(static_cast<unsigned>(pieces < most ? pieces : most), 2);
  switch (lanes) {
    case 1: return ten::launch(ans_cache_write_kernel<T, BITS, 1>, grid, block, 0, st, 1, a);
    case 2: return ten::launch(ans_cache_write_kernel<T, BITS, 2>, grid, block, 0, st, 1, a);
    case 4: return ten::launch(ans_cache_write_kernel<T, BITS, 4>, grid, block, 0, st, 1, a);
    case 8: return ten::launch(ans_cache_write_kernel<T, BITS, 8>, grid, block, 0, st, 1, a);
    default: return ten::launch(ans_cache_write_kernel<T, BITS, 16>, grid, block, 0, st, 1, a);
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
    {
      const uint64_t places = reinterpret_cast<uintptr_t>(a.x[w]) | (a.token_stride[w] * size) | (a.head_stride[w] * size);
      a.wide[w] = !(places & 31) ? 2 : !(places & 15) ? 1 : 0;
    }
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
  a.wide = !((reinterpret_cast<uintptr_t>(d_k_out) | reinterpret_cast<uintptr_t>(d_v_out)) & 31);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  // Rows of a block: enough blocks for eight on each SM, up to 64 rows each, over which a block's look-up is spread; of
  // narrow rows as many as give its threads four pieces each.
  int sms = 0;
  const int asked = ten::sm_count(&sms);
  if (asked != ANS_OK) return asked;
  const uint64_t share = rows / (4u * static_cast<uint64_t>(sms));
  uint32_t some = share < 4 ? 4u : share > 64 ? 64u : static_cast<uint32_t>(share);
  const uint32_t units = a.c.heads * a.c.head_dim / 16u;
  uint64_t full = 1024u / units < kReadRows ? 1024u / units : kReadRows;
  if (full > 2 * rows / sms) full = 2 * rows / sms;                   // but not fewer blocks than SMs
  if (some < full) some = static_cast<uint32_t>(full);
  const dim3 grid(static_cast<unsigned>((rows + some - 1) / some), 2);
  if (out_dtype == ANS_BF16)
    return h_desc->bitwidth == 8 ? ten::launch(ans_cache_read_kernel<__nv_bfloat16, 8>, grid, dim3(256), 0, st, 1, a, some)
                                 : ten::launch(ans_cache_read_kernel<__nv_bfloat16, 4>, grid, dim3(256), 0, st, 1, a, some);
  return h_desc->bitwidth == 8 ? ten::launch(ans_cache_read_kernel<float, 8>, grid, dim3(256), 0, st, 1, a, some)
                               : ten::launch(ans_cache_read_kernel<float, 4>, grid, dim3(256), 0, st, 1, a, some);
}
