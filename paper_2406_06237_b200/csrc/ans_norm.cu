// Root-mean-square norm of rows, with the residual's addition before it and bf16, fp32 or 8-bit output.
//
//   h = x + r,   y = h * rsqrt(mean h^2 + eps) * w,   s = max(max|y| / 448, 2^-126),   q = e4m3(y / s)
//
// One pass: a row is read once, lives in registers in fp32, and is written once.  The largest |y| needs no
// second pass over the row: it is rsqrt(...) times the largest |h w|, so the sum of squares and the
// maximum are reduced together, behind one barrier.
#include <cmath>
#include <type_traits>

#include "ans_tensor.cuh"

namespace ansb {

struct NormArgs {
  const void* x; const void* r; const void* w;
  void* out; float* scales; void* sum;
  uint64_t rows, x_stride, r_stride, out_stride, sum_stride;
  uint32_t width;
  float eps;
  uint32_t together;      // the rows of all matrices start equally far from a 16-byte boundary
  uint32_t shift;         // the most that a row starts past such a boundary, in elements
  uint32_t w_f32;         // type of w
  uint32_t w_vec;         // w on a 16-byte boundary
};

// Elements of a type one by one and eight at a time.  Eight are loaded as they lie (Raw), so that all of a
// thread's loads are under way before the first value is used; they bypass L1, which is left to the weight.
template <typename T> struct Elem;
template <int N> struct Raw { uint4 q[N]; };
template <int N>
__device__ __forceinline__ Raw<N> load_once(const void* p) {
  Raw<N> r;
#pragma unroll
  for (int i = 0; i < N; ++i)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.q[i].x), "=r"(r.q[i].y), "=r"(r.q[i].z), "=r"(r.q[i].w) : "l"(static_cast<const uint4*>(p) + i) : "memory");
  return r;
}
template <> struct Elem<__nv_bfloat16> {
  using Eight = Raw<1>;
  static __device__ __forceinline__ float one(const void* p, uint64_t i) {
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  }
  static __device__ __forceinline__ const void* at(const void* p, uint64_t i) { return static_cast<const __nv_bfloat16*>(p) + i; }
  static __device__ __forceinline__ void open(const Eight& u, float (&v)[8]) {
    const uint32_t w[4] = {u.q[0].x, u.q[0].y, u.q[0].z, u.q[0].w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[2 * j] = __uint_as_float(w[j] << 16);
      v[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void put(void* p, uint64_t i, float v) {
    static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
  }
  static __device__ __forceinline__ void put8(void* p, uint64_t i, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p) + i) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Elem<float> {
  using Eight = Raw<2>;
  static __device__ __forceinline__ float one(const void* p, uint64_t i) { return static_cast<const float*>(p)[i]; }
  static __device__ __forceinline__ const void* at(const void* p, uint64_t i) { return static_cast<const float*>(p) + i; }
  static __device__ __forceinline__ void open(const Eight& u, float (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[4 * j] = __uint_as_float(u.q[j].x);
      v[4 * j + 1] = __uint_as_float(u.q[j].y);
      v[4 * j + 2] = __uint_as_float(u.q[j].z);
      v[4 * j + 3] = __uint_as_float(u.q[j].w);
    }
  }
  static __device__ __forceinline__ void put(void* p, uint64_t i, float v) { static_cast<float*>(p)[i] = v; }
  static __device__ __forceinline__ void put8(void* p, uint64_t i, const float (&v)[8]) {
    float4* f = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    f[0] = make_float4(v[0], v[1], v[2], v[3]);
    f[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
};
template <> struct Elem<__nv_fp8_e4m3> {
  static __device__ __forceinline__ void put(void* p, uint64_t i, float v) {
    static_cast<uint8_t*>(p)[i] = static_cast<uint8_t>(__nv_cvt_float_to_fp8(v, __NV_SATFINITE, __NV_E4M3));
  }
  static __device__ __forceinline__ void put8(void* p, uint64_t i, const float (&v)[8]) {
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j], v[4 * j + 1]), __NV_SATFINITE, __NV_E4M3);
      const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * j + 2], v[4 * j + 3]), __NV_SATFINITE, __NV_E4M3);
      w[j] = lo | (hi << 16);
    }
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p) + i) = make_uint2(w[0], w[1]);
  }
};

// Elements i .. i + 7 of w, i any number in 0 .. width - 8.
__device__ __forceinline__ void weight8(const NormArgs& a, int i, float (&w)[8]) {
  if (!a.w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 1.f;
    return;
  }
  if (a.w_vec && !(i & 7)) {
    if (a.w_f32) {
      const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(a.w) + i);
      const float4 p = *f, q = f[1];
      w[0] = p.x; w[1] = p.y; w[2] = p.z; w[3] = p.w; w[4] = q.x; w[5] = q.y; w[6] = q.z; w[7] = q.w;
    } else {
      Raw<1> u;
      u.q[0] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.w) + i);
      Elem<__nv_bfloat16>::open(u, w);
    }
    return;
  }
  const int i0 = i & ~7, by = i & 7;
  if (a.w_vec && !a.w_f32 && i0 + 16 <= static_cast<int>(a.width)) {
    // the two aligned vectors around it, moved down by `by` elements (the same for the whole row)
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.w) + i0);
    const uint4 lo = p[0], hi = p[1];
    uint32_t c[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
    if (by & 4) {
#pragma unroll
      for (int j = 0; j < 6; ++j) c[j] = c[j + 2];
    }
    if (by & 2) {
#pragma unroll
      for (int j = 0; j < 6; ++j) c[j] = c[j + 1];
    }
    if (by & 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j) c[j] = __funnelshift_r(c[j], c[j + 1], 16);
    }
    Raw<1> u;
    u.q[0] = make_uint4(c[0], c[1], c[2], c[3]);
    Elem<__nv_bfloat16>::open(u, w);
    return;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) w[j] = a.w_f32 ? Elem<float>::one(a.w, i + j) : Elem<__nv_bfloat16>::one(a.w, i + j);
}

constexpr uint32_t kNormWarps = 32;

// blockDim = (threads of a row, rows of a block); a row of at most one warp needs no barrier.
// Thread t of a row holds the V vectors of 8 elements t, t + T, ...  Where rows start `phase` elements
// past a 16-byte boundary, vector 0 starts `phase` elements before the row, so that every vector is
// aligned; the first and the last, and all of them where the matrices' rows are not equally aligned,
// are read and written element by element.
template <typename TX, typename TO, int V, int MOST>
__global__ void __launch_bounds__(MOST) ans_rms_norm_kernel(const NormArgs a) {
  __shared__ float s_sum[kNormWarps];
  __shared__ uint32_t s_top[kNormWarps];
  ten::let_next_start();
  const uint64_t row = uint64_t(blockIdx.x) * blockDim.y + threadIdx.y;
  const uint32_t T = blockDim.x, t = threadIdx.x;
  const bool live = row < a.rows;
  const uint64_t xo = row * a.x_stride, ro = row * a.r_stride, oo = row * a.out_stride, so = row * a.sum_stride;
  const int width = static_cast<int>(a.width);
  const int phase = a.together ? static_cast<int>((reinterpret_cast<uintptr_t>(a.x) / sizeof(TX) + xo) & 7u) : 0;
  auto first = [&](int j) { return static_cast<int>(t + j * T) * 8 - phase; };             // the vector's first element
  auto whole = [&](int j) { return a.together && first(j) >= 0 && first(j) + 8 <= width; };
  ten::wait_for_previous();

  typename Elem<TX>::Eight x[V], r[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    x[j] = {}; r[j] = {};
    if (live && whole(j)) {
      x[j] = load_once<sizeof(TX) / 2>(Elem<TX>::at(a.x, xo + first(j)));
      if (a.r) r[j] = load_once<sizeof(TX) / 2>(Elem<TX>::at(a.r, ro + first(j)));
    }
  }
  float h[V][8];
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float u[8];
    Elem<TX>::open(x[j], h[j]);
    Elem<TX>::open(r[j], u);
    if (a.r) {
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] += u[i];
    }
    if (live && whole(j)) {
      if (a.sum) Elem<TX>::put8(a.sum, so + first(j), h[j]);
    } else if (live && first(j) < width) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = first(j) + i;
        if (e >= 0 && e < width) {
          h[j][i] = Elem<TX>::one(a.x, xo + e);
          if (a.r) h[j][i] += Elem<TX>::one(a.r, ro + e);
          if (a.sum) Elem<TX>::put(a.sum, so + e, h[j][i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(h[j][i], h[j][i], sum);
  }

  // h * w in place of h; the largest of |h w| as bits: of two non-negative floats the larger has the larger bits, NaN above all
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < V; ++j) {
    float w[8];
    if (whole(j)) {
      weight8(a, first(j), w);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = first(j) + i;
        w[i] = 1.f;
        if (a.w && e >= 0 && e < width) w[i] = a.w_f32 ? Elem<float>::one(a.w, e) : Elem<__nv_bfloat16>::one(a.w, e);
      }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      h[j][i] *= w[i];
      top = max(top, __float_as_uint(h[j][i]) & 0x7FFFFFFFu);
    }
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(ten::kAll, sum, d);
  top = __reduce_max_sync(ten::kAll, top);
  if (T > 32) {
    const uint32_t warps = T >> 5, lane = t & 31u;
    if (lane == 0) { s_sum[t >> 5] = sum; s_top[t >> 5] = top; }
    __syncthreads();
    sum = lane < warps ? s_sum[lane] : 0.f;
    top = lane < warps ? s_top[lane] : 0u;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(ten::kAll, sum, d);
    top = __reduce_max_sync(ten::kAll, top);
  }
  if (!live) return;
  const float f = 1.f / sqrtf(sum / static_cast<float>(width) + a.eps);
  float back = 1.f;
  constexpr bool k8 = std::is_same<TO, __nv_fp8_e4m3>::value;
  if constexpr (k8) {
    const float amax = f * __uint_as_float(top);
    const float s = amax != amax ? amax : fmaxf(amax / 448.f, 1.17549435e-38f);   // fmaxf alone would drop a NaN
    if (t == 0) a.scales[row] = s;
    back = 1.f / s;                                               // at most 2^126: f / s at once could overflow
  }
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = k8 ? h[j][i] * f * back : h[j][i] * f;
    if (whole(j)) {
      Elem<TO>::put8(a.out, oo + first(j), h[j]);
    } else if (first(j) < width) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = first(j) + i;
        if (e >= 0 && e < width) Elem<TO>::put(a.out, oo + e, h[j][i]);
      }
    }
  }
}

template <typename TX, typename TO>
static int launch_norm(const NormArgs& a, int sms, cudaStream_t st) {
  const uint32_t vectors = (a.width + a.shift + 7u) / 8u;
  constexpr uint32_t kWide = sizeof(TX) == 2 ? 4 : 2;             // vectors a thread: 64 bytes of x
  if (vectors <= 128) {                                           // a warp a row
    const uint64_t blocks = (a.rows + 7) / 8;
    if (blocks > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
    const dim3 grid(static_cast<unsigned>(blocks)), block(32, 8);
    if (vectors <= 32) return ten::launch(ans_rms_norm_kernel<TX, TO, 1, 256>, grid, block, 0, st, 1, a);
    if (vectors <= 64) return ten::launch(ans_rms_norm_kernel<TX, TO, 2, 256>, grid, block, 0, st, 1, a);
    return ten::launch(ans_rms_norm_kernel<TX, TO, 4, 256>, grid, block, 0, st, 1, a);
  }
  if (a.rows > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(a.rows));
  auto threads = [&](uint32_t v) { return dim3(((vectors + v - 1) / v + 31) / 32 * 32); };
  // Few rows: as many threads as a row has vectors; many: as many loads a thread as registers hold.
  if (vectors <= 1024 && a.rows <= 2ull * sms) return ten::launch(ans_rms_norm_kernel<TX, TO, 1, 1024>, grid, threads(1), 0, st, 1, a);
  if (vectors <= 512 * kWide) return ten::launch(ans_rms_norm_kernel<TX, TO, kWide, 512>, grid, threads(kWide), 0, st, 1, a);
  if (vectors <= 2048) return ten::launch(ans_rms_norm_kernel<TX, TO, 4, 512>, grid, threads(4), 0, st, 1, a);
  return ten::launch(ans_rms_norm_kernel<TX, TO, 8, 576>, grid, threads(8), 0, st, 1, a);
}

template <typename TX>
static int launch_norm_out(const NormArgs& a, int out_dtype, int sms, cudaStream_t st) {
  if (out_dtype == ANS_E4M3) return launch_norm<TX, __nv_fp8_e4m3>(a, sms, st);
  if (out_dtype == ANS_F32) return launch_norm<TX, float>(a, sms, st);
  return launch_norm<TX, __nv_bfloat16>(a, sms, st);
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
  // the place of a matrix's first row past a multiple of 8 elements, and its rows' step modulo 8; 99: not even on an element
  auto place = [](const void* p, int size) { const uintptr_t u = reinterpret_cast<uintptr_t>(p); return u % size ? 99u : unsigned(u / size % 8); };
  const unsigned at = place(d.d_x, xs);
  if (at == 99 || place(d.d_out, os) == 99 || (d.d_residual && place(d.d_residual, xs) == 99) || (d.d_sum && place(d.d_sum, xs) == 99))
    return ANS_ERR_INVALID_ARG;
  if (d.d_weight && place(d.d_weight, d.weight_dtype == ANS_F32 ? 4 : 2) == 99) return ANS_ERR_INVALID_ARG;
  auto same = [&](const void* p, int size, uint64_t stride) {
    return !p || (place(p, size) == at && (d.rows == 1 || stride % 8 == d.x_stride % 8));
  };
  NormArgs a{};
  a.x = d.d_x; a.r = d.d_residual; a.w = d.d_weight; a.out = d.d_out; a.scales = d.d_scales; a.sum = d.d_sum;
  a.rows = d.rows; a.width = d.width; a.eps = d.eps;
  a.x_stride = d.x_stride; a.r_stride = d.residual_stride; a.out_stride = d.out_stride; a.sum_stride = d.sum_stride;
  a.together = same(d.d_residual, xs, d.residual_stride) && same(d.d_out, os, d.out_stride) && same(d.d_sum, xs, d.sum_stride);
  a.shift = a.together && (at || (d.rows > 1 && d.x_stride % 8)) ? 7u : 0u;
  a.w_f32 = d.weight_dtype == ANS_F32;
  a.w_vec = !(reinterpret_cast<uintptr_t>(d.d_weight) & 15);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int dev = 0, sms = 0;
  ANSB_CUDA(cudaGetDevice(&dev));
  ANSB_CUDA(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev));
  return d.x_dtype == ANS_F32 ? launch_norm_out<float>(a, d.out_dtype, sms, st) : launch_norm_out<__nv_bfloat16>(a, d.out_dtype, sms, st);
}
