// Root-mean-square norm of rows, with the residual's addition before it and bf16, fp32 or 8-bit output.
//
//   h = x + r,   y = h * rsqrt(mean h^2 + eps) * w,   s = max(max|y| / 448, 2^-126),   q = e4m3(y / s)
//
// One pass: a row is read once, lives in registers in fp32, and is written once.  The largest |y| needs no
// second pass over the row: it is rsqrt(...) times the largest |h w|, so the sum of squares and the
// maximum are reduced together, behind one barrier.
//
// Squares leave fp32's range long before the values do.  A row whose sum of squares is infinite, or (where eps is too
// small to matter) next to nothing, is noted, and the threads that had it compute it again at their end, element by
// element in units of 2^76 or 2^-76 (powers of two change no rounding).  The note costs other rows 0 to 3 %, narrow ones more (60000 x
// 128: 16.1 to 18.4 us); the same in the middle of their work cost 1 to 6 %, and 20.2 us.
//
// Bound by memory for all but few or unaligned rows: 16384 x 8192 in bf16 with residual to e4m3 169 us, 5.6 TB/s, 85 % of the
// rate of a copy; 8192 x 4096 from fp32 to bf16 32 us, 95 %; one row of 8192 2.8 us, its own latency; 5000 x 7777 in bf16
// (rows off 16 bytes) 65 us, 73 %.
#include <cmath>
#include <type_traits>

#include "ans_tensor.cuh"

namespace ansb {

struct NormArgs {
  const char* x; const char* r; const void* w;
  char* out; float* scales; char* sum;
  const char* x_end; const char* r_end;        // the ends of the last rows
  uint64_t rows;
  uint64_t x_step, r_step, out_step, sum_step; // bytes from a row to the next
  uint32_t width;
  float eps, part;        // part: 1 / width
  float low;              // a sum of squares under this is taken again in smaller units; 0: none is, eps covers them
  uint32_t in_place;      // the sum is stored over x or r
  uint32_t together;      // the rows of all matrices start equally far from a 16-byte boundary
  uint32_t shift;         // the most that a row starts past such a boundary, in elements
  uint32_t w_f32;         // type of w
  uint32_t w_vec;         // w on a 16-byte boundary
};

using namespace ten;

// ---- elements of a type, one by one and a vector at a time -------------------------------------
// A vector is 16 bytes of x: E = 8 elements of bf16, 4 of fp32.
__device__ __forceinline__ uint4 load_once(const void* p) {        // past L1, which is left to the weight
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
  return r;
}
__device__ __forceinline__ Two open(uint32_t w) { return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ void open(const uint4& u, Two (&v)[4]) {            // bf16
  v[0] = open(u.x); v[1] = open(u.y); v[2] = open(u.z); v[3] = open(u.w);
}
__device__ __forceinline__ void open(const uint4& u, Two (&v)[2]) {            // fp32
  v[0] = two(__uint_as_float(u.x), __uint_as_float(u.y));
  v[1] = two(__uint_as_float(u.z), __uint_as_float(u.w));
}
template <typename T>
__device__ __forceinline__ float one(const void* p, int i) { return static_cast<float>(static_cast<const T*>(p)[i]); }
template <typename T>
__device__ __forceinline__ void put1(void* p, int i, float v) {
  if constexpr (sizeof(T) == 1) static_cast<uint8_t*>(p)[i] = static_cast<uint8_t>(__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3));
  else if constexpr (sizeof(T) == 2) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  else static_cast<float*>(p)[i] = v;
}
template <typename T>
__device__ __forceinline__ void copy1(void* to, int i, const void* from, int j) {
  using Bits = std::conditional_t<sizeof(T) == 1, uint8_t, std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t>>;
  static_cast<Bits*>(to)[i] = static_cast<const Bits*>(from)[j];
}
template <typename T, int H>
__device__ __forceinline__ void put_all(void* p, int i, const Two (&v)[H]) {
  if constexpr (sizeof(T) == 4) {
    float4* f = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
#pragma unroll
    for (int j = 0; j < H / 2; ++j) f[j] = make_float4(low(v[2 * j]), high(v[2 * j]), low(v[2 * j + 1]), high(v[2 * j + 1]));
  } else if constexpr (sizeof(T) == 2) {
    uint32_t w[H];
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(low(v[j]), high(v[j]));
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
    if constexpr (H == 4) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(p) + i) = make_uint2(w[0], w[1]);
  } else {
    uint32_t w[H / 2];
#pragma unroll
    for (int j = 0; j < H / 2; ++j) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(low(v[2 * j]), high(v[2 * j])), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(low(v[2 * j + 1]), high(v[2 * j + 1])), __NV_SATFINITE, __NV_E4M3);
      w[j] = lo | (hi << 16);
    }
    if constexpr (H == 4) *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p) + i) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(p) + i) = w[0];
  }
}

// The vectors at a row's ends, and all vectors where the matrices' rows are not equally aligned: element by
// element, elements e .. e + 2 H - 1 of a row of `width`, those outside it as zeros.  Not inlined: rare, and long.
template <int H> struct Pairs { Two v[H]; };
template <typename T, int H>
__device__ __noinline__ Pairs<H> gather(const void* row, int e, int width) {
  float f[2 * H];
#pragma unroll
  for (int i = 0; i < 2 * H; ++i) f[i] = static_cast<unsigned>(e + i) < static_cast<unsigned>(width) ? one<T>(row, e + i) : 0.f;
  Pairs<H> p;
#pragma unroll
  for (int i = 0; i < H; ++i) p.v[i] = two(f[2 * i], f[2 * i + 1]);
  return p;
}
template <typename T, int H>
__device__ __noinline__ void scatter(void* row, int e, int width, Pairs<H> f) {
#pragma unroll
  for (int i = 0; i < 2 * H; ++i)
    if (static_cast<unsigned>(e + i) < static_cast<unsigned>(width)) put1<T>(row, e + i, i & 1 ? high(f.v[i / 2]) : low(f.v[i / 2]));
}

// The weights e .. e + 2 H - 1.  aligned: e is a multiple of 2 H and all of them lie in the row.
template <int H>
__device__ __forceinline__ Pairs<H> weights(const NormArgs& a, int e, bool aligned) {
  Pairs<H> p;
  if (!a.w) {
#pragma unroll
    for (int i = 0; i < H; ++i) p.v[i] = two(1.f, 1.f);
  } else if (!a.w_vec || !aligned) {
    if (a.w_f32) return gather<float, H>(a.w, e, static_cast<int>(a.width));
    const int e0 = e & ~7, by = e & 7;
    if (!a.w_vec || e < 0 || e0 + 16 > static_cast<int>(a.width)) return gather<__nv_bfloat16, H>(a.w, e, static_cast<int>(a.width));
    // the two aligned vectors around them, moved down by `by` elements
    const uint4* q = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.w) + e0);
    const uint4 lo = q[0], hi = q[1];
    uint32_t c[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int j = 0; j < 6; ++j) c[j] = by & 4 ? c[j + 2] : c[j];
#pragma unroll
    for (int j = 0; j < 5; ++j) c[j] = by & 2 ? c[j + 1] : c[j];
#pragma unroll
    for (int i = 0; i < H; ++i) p.v[i] = open(by & 1 ? __funnelshift_r(c[i], c[i + 1], 16) : c[i]);
  } else if (a.w_f32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(a.w) + e);
#pragma unroll
    for (int i = 0; i < H / 2; ++i) {
      const float4 u = q[i];
      p.v[2 * i] = two(u.x, u.y);
      p.v[2 * i + 1] = two(u.z, u.w);
    }
  } else if constexpr (H == 4) {
    open(*reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.w) + e), p.v);
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.w) + e);
    p.v[0] = open(u.x);
    p.v[1] = open(u.y);
  }
  return p;
}

constexpr uint32_t kNormWarps = 32;
constexpr float kUp = 75557863725914323419136.f, kDown = 1.f / kUp;      // 2^76, 2^-76
constexpr size_t kNormRing = 216 * 1024;         // bytes of an SM's rings

// an 8-bit row's scale from its largest magnitude
__device__ __forceinline__ float scale_of(float amax) {
  return amax != amax ? amax : fmaxf(amax * (1.f / 448.f), 1.17549435e-38f);                 // fmaxf alone would drop a NaN
}

// What the kernels share of a row: thread t of its T threads holds the V vectors of E elements t, t + T, ...
// Where rows start `phase` elements past a 16-byte boundary, vector 0 starts `phase` elements before the
// row, so that every vector is aligned.  EVEN: all rows start on a boundary and are whole vectors.
template <typename TX, typename TO, int V, bool EVEN>
struct NormRow {
  static constexpr int E = 16 / sizeof(TX), H = E / 2;
  const NormArgs& a;
  int t, T, width, phase;
  bool edge;                       // among the first or last rows, whose end vectors can reach past the matrices
  const char* x; const char* r; char* out; char* sum;          // the row
  const char* x0; const char* r0; char* out0; char* sum0;      // the thread's vector 0 of it
  char* ends;                      // this warp's 128 bytes of shared memory for the row's end vectors: two of h, two of y
  __device__ __forceinline__ NormRow(const NormArgs& args, uint32_t thread, uint32_t threads, char* scratch)
      : a(args), t(static_cast<int>(thread)), T(static_cast<int>(threads)), width(static_cast<int>(args.width)), phase(0), edge(true), ends(scratch) {}
  __device__ __forceinline__ void at(uint64_t row) {
    x = a.x + row * a.x_step;
    r = a.r + row * a.r_step;
    out = a.out + row * a.out_step;
    sum = a.sum + row * a.sum_step;
    if constexpr (EVEN) {                                         // these are the thread's vector 0 from here on
      x += t * 16;
      r += t * 16;
      sum += t * 16;
      out += t * E * int(sizeof(TO));
    }
    settle(row);
  }
  __device__ __forceinline__ void settle(uint64_t row) {
    if constexpr (!EVEN) {
      phase = a.shift ? static_cast<int>((reinterpret_cast<uintptr_t>(x) / sizeof(TX)) & (E - 1u)) : 0;
      edge = row < E || row + E >= a.rows;
    }
    const int at0 = EVEN ? 0 : first(0);
    x0 = x + at0 * int(sizeof(TX));
    r0 = r + at0 * int(sizeof(TX));
    sum0 = sum + at0 * int(sizeof(TX));
    out0 = out + at0 * int(sizeof(TO));
  }
  __device__ __forceinline__ int first(int j) const { return (t + j * T) * E - phase; }   // a vector's first element
  __device__ __forceinline__ bool some(int j) const { return first(j) < width; }
  __device__ __forceinline__ bool whole(int j) const { return EVEN ? some(j) : a.together && first(j) >= 0 && first(j) + E <= width; }
  __device__ __forceinline__ const char* place(const char* row0, int j) const { return row0 + j * T * 16; }
  // Whether vector j can be loaded as one: it holds some of the row, and nothing from before the matrices' first
  // element or past their last one (what belongs to the rows next to this one is dropped).
  __device__ __forceinline__ bool loads(int j) const {
    if constexpr (EVEN) return some(j);
    if (!a.together || !some(j)) return false;
    return !edge || loads_at_edge(j);
  }
  __device__ __forceinline__ bool loads_at_edge(int j) const {
    return place(x0, j) >= a.x && place(x0, j) + 16 <= a.x_end && (!a.r || (place(r0, j) >= a.r && place(r0, j) + 16 <= a.r_end));
  }
  // h = x + r from the loaded vectors; h stored; its sum of squares
  __device__ __forceinline__ float add(const uint4 (&xs)[V], const uint4 (&rs)[V], Two (&h)[V][H]) const {
    Two total = two(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
      if (EVEN || loads(j)) {
        open(xs[j], h[j]);
        if (a.r) {
          Two u[H];
          open(rs[j], u);
#pragma unroll
          for (int i = 0; i < H; ++i) h[j][i] = add2(h[j][i], u[i]);
        }
        if constexpr (!EVEN) {
          if (some(j) && !whole(j)) {
#pragma unroll
            for (int i = 0; i < H; ++i)
              h[j][i] = two(static_cast<unsigned>(first(j) + 2 * i) < static_cast<unsigned>(width) ? low(h[j][i]) : 0.f,
                            static_cast<unsigned>(first(j) + 2 * i + 1) < static_cast<unsigned>(width) ? high(h[j][i]) : 0.f);
          }
        }
      } else {
        Pairs<H> f{};
        if (some(j)) f = gather<TX, H>(x, first(j), width);
#pragma unroll
        for (int i = 0; i < H; ++i) h[j][i] = f.v[i];
        if (a.r && some(j)) {
          const Pairs<H> g = gather<TX, H>(r, first(j), width);
#pragma unroll
          for (int i = 0; i < H; ++i) h[j][i] = add2(h[j][i], g.v[i]);
        }
      }
      if (a.sum) put<TX, 0>(sum, sum0, j, h[j]);
#pragma unroll
      for (int i = 0; i < H; ++i) total = fma2(h[j][i], h[j][i], total);
    }
    return low(total) + high(total);
  }
  // Vector j of a matrix; an end vector waits in slot SLOT (or the one after it) of the warp's scratch.
  template <typename T2, int SLOT>
  __device__ __forceinline__ void put(char* row, char* row0, int j, const Two (&v)[H]) const {
    if (whole(j)) {
      put_all<T2, H>(row0 + j * T * (E * int(sizeof(T2))), 0, v);
    } else if (!EVEN && some(j)) {
      if (a.together) {
        put_all<T2, H>(ends + 32 * (SLOT + (first(j) < 0 ? 0 : 1)), 0, v);
      } else {
        Pairs<H> f;
#pragma unroll
        for (int i = 0; i < H; ++i) f.v[i] = v[i];
        scatter<T2, H>(row, first(j), width, f);
      }
    }
  }
  // The end vectors out of the scratch, an element a lane: lanes 0-7 h's first, 8-15 h's last, 16-23 y's first, 24-31 y's last.
  __device__ __forceinline__ void put_ends() const {
    if constexpr (!EVEN) {
      if (!a.together) return;
      bool head = false, tail = false;
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const bool part = some(j) && !whole(j);
        head |= part && first(j) < 0;
        tail |= part && first(j) >= 0;
      }
      head = __any_sync(ten::kAll, head);
      tail = __any_sync(ten::kAll, tail);
      if (head || tail) {
        __syncwarp();
        const int lane = t & 31, i = lane & 7, last = lane & 8;
        const int e = (last ? (width + phase - 1) & ~(E - 1) : 0) - phase + i;
        const char* const from = ends + 32 * (lane >> 3);
        if (i < E && static_cast<unsigned>(e) < static_cast<unsigned>(width) && (last ? tail : head)) {
          if (lane >= 16) copy1<TO>(out, e, from, i);
          else if (a.sum) copy1<TX>(sum, e, from, i);
        }
        __syncwarp();
      }
    }
  }
  // h * w in place of h, and for an 8-bit output the largest of |h w|
  static __device__ __forceinline__ float scale(Two (&h)[H], const Two (&w)[H], float top) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      h[i] = mul2(h[i], w[i]);
      if constexpr (sizeof(TO) == 1) top = larger(top, h[i]);
    }
    return top;
  }
  // over a row's threads; s_*: a place for each warp, free when this is called.  Magnitudes compare like their bits, NaN above all.
  __device__ __forceinline__ void reduce(float& total, float& top, float* s_sum, float* s_top) const {
    constexpr bool k8 = sizeof(TO) == 1;
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(ten::kAll, total, d);
    if (k8) top = __uint_as_float(__reduce_max_sync(ten::kAll, __float_as_uint(top)));
    if (T > 32) {
      const int warps = T >> 5, lane = t & 31;
      if (lane == 0) {
        s_sum[t >> 5] = total;
        if (k8) s_top[t >> 5] = top;
      }
      if (t >= warps && t < 8) {
        s_sum[t] = 0.f;
        if (k8) s_top[t] = 0.f;
      }
      __syncthreads();
      if (warps <= 8) {                                           // the same eight words for every thread: no second round of shuffles
        const float4 p = reinterpret_cast<const float4*>(s_sum)[0], q = reinterpret_cast<const float4*>(s_sum)[1];
        total = ((p.x + p.y) + (p.z + p.w)) + ((q.x + q.y) + (q.z + q.w));
        if (k8) {
          const uint4 u = reinterpret_cast<const uint4*>(s_top)[0], v = reinterpret_cast<const uint4*>(s_top)[1];
          top = __uint_as_float(max(max(max(u.x, u.y), max(u.z, u.w)), max(max(v.x, v.y), max(v.z, v.w))));
        }
      } else {
        total = lane < warps ? s_sum[lane] : 0.f;
#pragma unroll
        for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(ten::kAll, total, d);
        if (k8) top = __uint_as_float(__reduce_max_sync(ten::kAll, lane < warps ? __float_as_uint(s_top[lane]) : 0u));
      }
    }
  }
  __device__ __forceinline__ void store(uint64_t row, Two (&h)[V][H], float total, float top) const {
    float f = rsqrtf(fmaf(total, a.part, a.eps));
    if constexpr (sizeof(TO) == 1) {
      const float s = scale_of(f * top);
      if (t == 0) a.scales[row] = s;
      const float back = __frcp_rn(s);                            // at most 2^126
      if (!(f * back < INFINITY) && back < INFINITY) {            // tiny rows: not in one factor
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
          for (int i = 0; i < H; ++i) h[j][i] = mul2(h[j][i], two(f, f));
        f = 1.f;
      }
      f *= back;
    }
    const Two ff = two(f, f);
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int i = 0; i < H; ++i) h[j][i] = mul2(h[j][i], ff);
      put<TO, 2>(out, out0, j, h[j]);
    }
  }
};

// Whether a row's sum of squares is out of range.  A NaN is not: its row is NaN whatever the units.
__device__ __forceinline__ bool out_of_range(const NormArgs& a, float total) { return total == INFINITY || total < a.low; }

// A row again if its sum of squares is out of range (or within 1 %: the sums' order differs here, and values may be
// the stored ones), by the threads that had it.  Values are x + r, or the stored sum where that is exact (fp32) or lies over one of them.
template <typename TX, typename TO>
__device__ __noinline__ void redo(const NormArgs& a, uint64_t row, int t, int T, float* s_sum, float* s_top) {
  using Row = NormRow<TX, TO, 1, false>;
  const Row n(a, t, T, nullptr);
  const char* const x = a.x + row * a.x_step;
  const char* const r = a.r + row * a.r_step;
  const char* const sum = a.sum + row * a.sum_step;
  char* const out = a.out + row * a.out_step;
  const int width = static_cast<int>(a.width);
  const bool stored = a.sum && (sizeof(TX) == 4 || a.in_place);
  auto value = [&](int e) { return stored ? one<TX>(sum, e) : a.r ? one<TX>(x, e) + one<TX>(r, e) : one<TX>(x, e); };
  auto sync = [&] { if (T > 32) __syncthreads(); else __syncwarp(); };
  sync();                                                         // what the row's threads stored is seen; the places are free
  float total = 0.f, top = 0.f;
  for (int e = t; e < width; e += T) { const float v = value(e); total = fmaf(v, v, total); }
  n.reduce(total, top, s_sum, s_top);
  if (!(total > 3.37e38f || total < 1.01f * a.low)) return;
  const float unit = total < 1.f ? kUp : kDown;
  auto weighed = [&](int e) {
    const float w = !a.w ? 1.f : a.w_f32 ? one<float>(a.w, e) : one<__nv_bfloat16>(a.w, e);
    return value(e) * unit * w;
  };
  total = 0.f;
  for (int e = t; e < width; e += T) {
    const float v = value(e) * unit;
    total = fmaf(v, v, total);
    if constexpr (sizeof(TO) == 1) { const float u = weighed(e); top = larger(top, two(u, u)); }
  }
  sync();
  n.reduce(total, top, s_sum, s_top);
  float f = rsqrtf(fmaf(total, a.part, a.eps * unit * unit)), back = 1.f;
  if constexpr (sizeof(TO) == 1) {
    const float s = scale_of(f * top);
    if (t == 0) a.scales[row] = s;
    back = __frcp_rn(s);
  }
  for (int e = t; e < width; e += T) put1<TO>(out, e, weighed(e) * f * back);
  sync();
}

// A block a row: for few rows, where a row's own latency counts, and for rows that the rings below do not fit.
template <typename TX, typename TO, int V, int MOST>
__global__ void __launch_bounds__(MOST) ans_rms_norm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ __align__(16) float s_sum[kNormWarps], s_top[kNormWarps];
  __shared__ uint4 s_ends[kNormWarps][8];
  ten::let_next_start();
  using Row = NormRow<TX, TO, V, false>;
  Row n(a, threadIdx.x, blockDim.x, reinterpret_cast<char*>(s_ends[threadIdx.x >> 5]));
  n.at(blockIdx.x);
  ten::wait_for_previous();
  uint4 x[V], r[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    x[j] = r[j] = make_uint4(0u, 0u, 0u, 0u);
    if (n.loads(j)) {
      x[j] = load_once(n.place(n.x0, j));
      if (a.r) r[j] = load_once(n.place(n.r0, j));
    }
  }
  auto weight = [&](int j) { return n.some(j) ? weights<Row::H>(a, n.first(j), !n.phase && n.whole(j)) : Pairs<Row::H>{}; };
  Two h[V][Row::H];
  float total, top = 0.f;
  if constexpr (V == 1) {                                         // its load is under way with the row's
    const Pairs<Row::H> w = weight(0);
    total = n.add(x, r, h);
    top = n.scale(h[0], w.v, top);
  } else {
    total = n.add(x, r, h);
#pragma unroll
    for (int j = 0; j < V; ++j) top = n.scale(h[j], weight(j).v, top);
  }
  n.reduce(total, top, s_sum, s_top);
  n.store(blockIdx.x, h, total, top);
  n.put_ends();
  if (out_of_range(a, total)) redo<TX, TO>(a, blockIdx.x, threadIdx.x, blockDim.x, s_sum, s_top);
}

// Persistent: blockDim = (threads of a row, rows of a block); a block takes row after row.  Every thread copies its
// own vectors of the rows to come into a ring of `depth` rows in shared memory (cp.async), so memory is
// read on while a row is reduced and written; a thread reads only what it copied, and a row of one warp needs no
// barrier at all.  Even rows: a weight in bf16 stays in registers.  Others, whose vectors start at any element: the
// weight lies in shared memory, element e at [e % E][e / E], where a warp's reads of any alignment meet no conflict.
template <typename TX, typename TO, int V, int MOST, bool EVEN>
__global__ void __launch_bounds__(MOST) ans_rms_norm_ring_kernel(const __grid_constant__ NormArgs a, const uint32_t depth) {
  extern __shared__ uint4 ring[];
  __shared__ __align__(16) float s_sum[2][kNormWarps], s_top[2][kNormWarps];
  __shared__ uint4 s_ends[EVEN ? 1 : kNormWarps][8];
  __shared__ uint32_t s_again[kNormWarps];
  ten::let_next_start();
  using Row = NormRow<TX, TO, V, EVEN>;
  constexpr int E = Row::E, H = Row::H;
  const uint32_t t = threadIdx.x, T = blockDim.x, y = threadIdx.y, Y = blockDim.y;
  const uint32_t per_row = (a.r ? 2u : 1u) * V * T;               // vectors of a row in the ring
  const uint32_t mine = ten::smem_addr(ring + size_t(y) * depth * per_row + t), ring_end = mine + depth * per_row * 16u;
  float* const s_w = reinterpret_cast<float*>(ring + size_t(Y) * depth * per_row);
  const uint32_t w_base = ten::smem_addr(s_w);
  const uint32_t w_pitch = a.width / E + 3u;                      // elements -E .. width + E and more
  const uint64_t step = uint64_t(gridDim.x) * Y;                  // rows from a block's row to its next, and their bytes
  const uint64_t x_on = step * a.x_step, r_on = step * a.r_step, out_on = step * a.out_step, sum_on = step * a.sum_step;
  uint64_t row = uint64_t(blockIdx.x) * Y + y;
  ten::wait_for_previous();

  char* const scratch = reinterpret_cast<char*>(s_ends[EVEN ? 0 : (y * T + t) >> 5]);
  Row ahead(a, t, T, scratch), n(a, t, T, scratch);               // the row that is fetched next, the row at hand
  ahead.at(row);
  n.at(row);
  uint64_t ahead_row = row;
  auto fetch = [&](uint32_t to) {
    if (ahead_row < a.rows) {
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!ahead.loads(j)) continue;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + j * T * 16u), "l"(ahead.place(ahead.x0, j)) : "memory");
        if (a.r) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + (V + j) * T * 16u), "l"(ahead.place(ahead.r0, j)) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    ahead_row += step;
    ahead.x += x_on;
    ahead.r += r_on;
    ahead.settle(ahead_row);
  };
  uint32_t spare = mine;                                          // the place for the next fetch
  for (uint32_t i = 0; i + 1 < depth; ++i, spare += per_row * 16u) fetch(spare);

  const bool keep = EVEN && a.w && !a.w_f32;
  uint2 kept[V][H / 2];
  if constexpr (EVEN) {
#pragma unroll
    for (int j = 0; j < V; ++j)
      if (keep && n.some(j)) {
#pragma unroll
        for (int i = 0; i < H / 2; ++i) kept[j][i] = reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.w) + n.first(j))[i];
      }
  } else {
    for (uint32_t i = y * T + t; i < E * w_pitch; i += T * Y) {
      const int e = static_cast<int>(i) - E;
      float w = 0.f;
      if (static_cast<unsigned>(e) < a.width) w = !a.w ? 1.f : a.w_f32 ? one<float>(a.w, e) : one<__nv_bfloat16>(a.w, e);
      s_w[(i % E) * w_pitch + i / E] = w;
    }
    __syncthreads();
  }

  uint32_t from = mine, odd = 0;
  uint32_t* const again = &s_again[(y * T + t) >> 5];
  *again = 0u;
  __syncwarp();
  for (uint64_t base = uint64_t(blockIdx.x) * Y; base < a.rows; base += step) {   // the same trips for all of the block
    fetch(spare);
    spare += per_row * 16u;
    if (spare == ring_end) spare = mine;
    switch (depth) {                                              // all but the last depth - 1 copies are there
      case 2: asm volatile("cp.async.wait_group 1;" ::: "memory"); break;
      case 3: asm volatile("cp.async.wait_group 2;" ::: "memory"); break;
      case 4: asm volatile("cp.async.wait_group 3;" ::: "memory"); break;
      case 5: asm volatile("cp.async.wait_group 4;" ::: "memory"); break;
      default: asm volatile("cp.async.wait_group 5;" ::: "memory"); break;
    }
    const bool live = row < a.rows;
    Two h[V][H];
    float total = 0.f, top = 0.f;
    if (live) {
      uint4 x[V], r[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        x[j] = r[j] = make_uint4(0u, 0u, 0u, 0u);
        if (n.loads(j)) {
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x[j].x), "=r"(x[j].y), "=r"(x[j].z), "=r"(x[j].w)
                       : "r"(from + j * T * 16u) : "memory");
          if (a.r)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[j].x), "=r"(r[j].y), "=r"(r[j].z), "=r"(r[j].w)
                         : "r"(from + (V + j) * T * 16u) : "memory");
        }
      }
      total = n.add(x, r, h);
      uint32_t w_at[E];                                           // element i of a vector at [(i - phase) % E][vector + 1 + (i - phase) / E]
      if constexpr (!EVEN) {
#pragma unroll
        for (int i = 0; i < E; ++i) w_at[i] = w_base + (((i - n.phase) & (E - 1)) * w_pitch + (i < n.phase ? 0u : 1u) + t) * 4u;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if (!n.some(j)) continue;
        Pairs<H> w;
        if constexpr (EVEN) {
          if (keep) {
#pragma unroll
            for (int i = 0; i < H / 2; ++i) { w.v[2 * i] = open(kept[j][i].x); w.v[2 * i + 1] = open(kept[j][i].y); }
          } else {
            w = weights<H>(a, n.first(j), true);
          }
        } else {
          float f[E];
#pragma unroll
          for (int i = 0; i < E; ++i) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[i]) : "r"(w_at[i] + j * T * 4u));
#pragma unroll
          for (uint32_t i = 0; i < H; ++i) w.v[i] = two(f[2 * i], f[2 * i + 1]);
        }
        top = n.scale(h[j], w.v, top);
      }
    }
    n.reduce(total, top, s_sum[odd], s_top[odd]);
    if (live) {
      n.store(row, h, total, top);
      n.put_ends();
      if (out_of_range(a, total)) *again = 1u;
    }
    from += per_row * 16u;
    if (from == ring_end) from = mine;
    odd ^= 1u;
    row += step;
    n.x += x_on;
    n.r += r_on;
    n.out += out_on;
    n.sum += sum_on;
    n.settle(row);
  }
  __syncwarp();
  if (*again)                                                      // the row's threads alike
    for (row = uint64_t(blockIdx.x) * Y + y; row < a.rows; row += step) redo<TX, TO>(a, row, t, T, s_sum[0], s_top[0]);
}

// `blocks` blocks an SM split its shared memory; a ring of two to six rows
template <typename TX>
static size_t weight_bytes(const NormArgs& a) { return size_t(a.width / (16 / sizeof(TX)) + 3) * (16 / sizeof(TX)) * 4; }
template <typename TX, typename TO, int V, int MOST, bool EVEN>
static int launch_ring(const NormArgs& a, dim3 block, uint32_t blocks, int sms, cudaStream_t st) {
  const size_t row = size_t(a.r ? 2 : 1) * V * 16 * block.x * block.y;
  const size_t rest = EVEN ? 0 : weight_bytes<TX>(a);
  constexpr auto kernel = ans_rms_norm_ring_kernel<TX, TO, V, MOST, EVEN>;
  while (blocks > 1 && blocks * (2 * row + rest) > kNormRing) --blocks;
  uint32_t depth = static_cast<uint32_t>((kNormRing / blocks - rest) / row);
  if (depth > 6) depth = 6;
  const size_t smem = depth * row + rest;
  const int rc = ten::allow_smem<kernel>(kNormRing);
  if (rc != ANS_OK) return rc;
  const uint64_t need = (a.rows + block.y - 1) / block.y, have = uint64_t(sms) * blocks;
  return ten::launch(kernel, dim3(static_cast<unsigned>(need < have ? need : have)), block, smem, st, 1, a, depth);
}

template <typename TX, typename TO, bool EVEN>
static int launch_norm(const NormArgs& a, int sms, cudaStream_t st) {
  constexpr uint32_t E = 16 / sizeof(TX), kTwice = sizeof(TX) / 2;   // fp32: twice the vectors for a row
  const uint32_t vectors = (a.width + a.shift + E - 1) / E;
  auto threads = [&](uint32_t v) { return dim3(((vectors + v - 1) / v + 31) / 32 * 32); };
  // The ring.  Even rows: a warp a row up to 128 vectors; a block a row where a block has at least two of them to read ahead:
  // 1100 x 8192 13 us, 16 without, 400 x 8192 6.8 with and without.  Rows off 16 bytes spend their time on their ends and
  // on the weight's place, which the ring's few threads make longer: it takes the narrowest (100000 x 111 52 us, 104 with a
  // block a row; but 20000 x 333 28 and 22) and the widest (3000 x 16001 86 and 100 us; but 16000 x 2047 74 and 55).
  const dim3 warps(32, 8);
  if (vectors <= 32) return launch_ring<TX, TO, 1, 256, EVEN>(a, warps, EVEN ? 4 : 3, sms, st);
  if constexpr (EVEN) {
    if (vectors <= 64) return launch_ring<TX, TO, 2, 256, true>(a, warps, 3, sms, st);
    if (vectors <= 128) return launch_ring<TX, TO, 4, 256, true>(a, warps, kTwice == 2 ? 3 : 2, sms, st);
  }
  constexpr int V = 4 * kTwice;
  const dim3 block = threads(V);
  const uint32_t blocks = 512 / block.x;
  const size_t bytes = size_t(vectors + 256) * 16 * (a.r ? 2 : 1);   // of a row in the ring, at most
  const size_t rest = EVEN ? 0 : weight_bytes<TX>(a);
  if (vectors <= 2048 * kTwice && (EVEN || vectors > 1024) && a.rows >= (EVEN ? 2u : 6u) * uint64_t(sms) * blocks && 2 * bytes + rest <= kNormRing)
    return launch_ring<TX, TO, V, 512, EVEN>(a, block, blocks, sms, st);
  if (a.rows > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const dim3 rows(static_cast<unsigned>(a.rows));
  // One vector a thread while all rows' blocks are on the SMs at once (1344 threads of it an SM), else two: 500 x 2047 3.2 and
  // 4.2 us, 1537 x 2047 7.7 and 6.7, 1500 x 8192 28 and 21.
  if (vectors <= 1024 && a.rows > uint64_t(sms) * (1344u / threads(1).x)) return ten::launch(ans_rms_norm_kernel<TX, TO, 2, 512>, rows, threads(2), 0, st, 1, a);
  if (vectors <= 1024) return ten::launch(ans_rms_norm_kernel<TX, TO, 1, 1024>, rows, threads(1), 0, st, 1, a);
  if (vectors <= 2048 * kTwice) return ten::launch(ans_rms_norm_kernel<TX, TO, 4 * kTwice, 512>, rows, threads(4 * kTwice), 0, st, 1, a);
  return ten::launch(ans_rms_norm_kernel<TX, TO, 8 * kTwice, 576>, rows, threads(8 * kTwice), 0, st, 1, a);
}

template <typename TX>
static int launch_norm_out(const NormArgs& a, int out_dtype, int sms, cudaStream_t st) {
  const bool even = a.together && !a.shift && a.width % (16 / sizeof(TX)) == 0 && (!a.w || a.w_vec);
  if (out_dtype == ANS_E4M3) return even ? launch_norm<TX, __nv_fp8_e4m3, true>(a, sms, st) : launch_norm<TX, __nv_fp8_e4m3, false>(a, sms, st);
  if (out_dtype == ANS_F32) return even ? launch_norm<TX, float, true>(a, sms, st) : launch_norm<TX, float, false>(a, sms, st);
  return even ? launch_norm<TX, __nv_bfloat16, true>(a, sms, st) : launch_norm<TX, __nv_bfloat16, false>(a, sms, st);
}

}  // namespace ansb

using namespace ansb;

ANS_EXPORT int ans_rms_norm(const ans_norm_desc* h_desc, void* stream) {
  ApiRange range("ans_rms_norm");
  if (!h_desc) return ANS_ERR_INVALID_ARG;
  const ans_norm_desc& d = *h_desc;
  if (d.x_dtype != ANS_BF16 && d.x_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (d.weight_dtype != ANS_BF16 && d.weight_dtype != ANS_F32) return ANS_ERR_UNSUPPORTED;
  if (d.out_dtype != ANS_BF16 && d.out_dtype != ANS_F32 && d.out_dtype != ANS_E4M3) return ANS_ERR_UNSUPPORTED;
  if (d.width > 32768) return ANS_ERR_UNSUPPORTED;
  if (!(d.eps >= 0.f) || !std::isfinite(d.eps)) return ANS_ERR_INVALID_ARG;
  if (d.rows == 0 || d.width == 0) return ANS_OK;
  if (!d.d_x || !d.d_out || (d.out_dtype == ANS_E4M3 && !d.d_scales)) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kMost = uint64_t(1) << 40;
  if (d.rows > kMost) return ANS_ERR_UNSUPPORTED;
  const uint64_t strides[4] = {d.x_stride, d.d_residual ? d.residual_stride : d.width, d.out_stride, d.d_sum ? d.sum_stride : d.width};
  for (uint64_t s : strides)
    if (d.rows > 1 && (s < d.width || s > kMost)) return ANS_ERR_INVALID_ARG;
  const int xs = d.x_dtype == ANS_F32 ? 4 : 2, os = d.out_dtype == ANS_F32 ? 4 : d.out_dtype == ANS_BF16 ? 2 : 1;
  // the place of a matrix's first row past a whole vector, in elements, and its rows' step; 99: not even on an element
  const unsigned E = 16 / xs;
  auto place = [&](const void* p, int size) { const uintptr_t u = reinterpret_cast<uintptr_t>(p); return u % size ? 99u : unsigned(u / size % E); };
  const unsigned at = place(d.d_x, xs);
  if (at == 99 || place(d.d_out, os) == 99 || (d.d_residual && place(d.d_residual, xs) == 99) || (d.d_sum && place(d.d_sum, xs) == 99))
    return ANS_ERR_INVALID_ARG;
  if (d.d_weight && place(d.d_weight, d.weight_dtype == ANS_F32 ? 4 : 2) == 99) return ANS_ERR_INVALID_ARG;
  auto same = [&](const void* p, int size, uint64_t stride) {
    return !p || (place(p, size) == at && (d.rows == 1 || stride % E == d.x_stride % E));
  };
  NormArgs a{};
  a.x = static_cast<const char*>(d.d_x); a.r = static_cast<const char*>(d.d_residual); a.w = d.d_weight;
  a.out = static_cast<char*>(d.d_out); a.scales = d.d_scales; a.sum = static_cast<char*>(d.d_sum);
  a.rows = d.rows; a.width = d.width; a.eps = d.eps;
  a.x_step = d.x_stride * xs; a.out_step = d.out_stride * os;
  if (a.r) a.r_step = d.residual_stride * xs;
  if (a.sum) a.sum_step = d.sum_stride * xs;
  a.x_end = a.x + (d.rows - 1) * a.x_step + uint64_t(d.width) * xs;
  a.r_end = a.r + (d.rows - 1) * a.r_step + uint64_t(d.width) * xs;
  a.part = 1.f / static_cast<float>(d.width);
  constexpr float kLittle = 7.8886091e-31f;                         // 2^-100: squares that vanish (2^-149 each) are nothing beside it
  a.low = d.eps < kLittle ? kLittle : 0.f;
  a.in_place = a.sum && (a.sum == a.x || a.sum == a.r);
  a.together = same(d.d_residual, xs, d.residual_stride) && same(d.d_out, os, d.out_stride) && same(d.d_sum, xs, d.sum_stride);
  a.shift = a.together && (at || (d.rows > 1 && d.x_stride % E)) ? E - 1 : 0u;
  a.w_f32 = d.weight_dtype == ANS_F32;
  a.w_vec = !(reinterpret_cast<uintptr_t>(d.d_weight) & 15);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int sms = 0;
  const int rc = ten::sm_count(&sms);
  if (rc != ANS_OK) return rc;
  return d.x_dtype == ANS_F32 ? launch_norm_out<float>(a, d.out_dtype, sms, st) : launch_norm_out<__nv_bfloat16>(a, d.out_dtype, sms, st);
}
