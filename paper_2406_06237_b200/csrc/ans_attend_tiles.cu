// Attention over the block-scaled cache for many queries a head of the cache (prompts, chunks of prompts), on the
// fifth-generation tensor cores.
//
// A block of threads has a tile of rows (new tokens x query heads of one head of the cache), one or two halves of 128, and
// goes over the tokens that they see, 64 at a time.  Its warps:
//   4 converters:   codes from global memory, opened to fp16, into shared memory as operands (four stages of K and V, two
//                   for 256 dimensions);
//   1 for scales:   of the runs of 16 tokens, as the softmax uses them;
//   1 issuer:       S = Q K^T into tensor memory, then O += P V with P out of tensor memory;
//   4 a half:       the softmax of a row a thread: S out of tensor memory, P over it as fp16, O rescaled there when the row's
//                   maximum has grown by more than 2^kSlack since it was last.
// V is the operand as it lies in the cache, tokens x dimensions ("MN-major"), so nothing is transposed.
//
// For 64 tokens of 128 dimensions the two halves' four products take 1024 clocks of the tensor pipe and their 16384
// exponentials as many (16 a clock).  What bounds is neither but a half's own chain, about 2100 clocks: S out of tensor
// memory, the row's maximum, exponentials, P back, each waiting for the one before with one warp a scheduler and half.  A
// prompt of 4096 (32 query heads on 8, D = 128) takes 176 us, 780 TFLOP/s of the products that causal order leaves; five chunks
// of 1229 to 2048 behind 3601 to 6001 cached ones 900 us, 820 (172 and 875 before runs could count apart in the sum, ans_attend.cuh).  The prompt
// takes 144 with D = 64 and 400 with D = 256, whose one half has nothing beside its chain and whose registers spill (492 bytes a thread; 12
// with D = 128, none with 64).  Blocks of 128 tokens with one place for S and two stages took 184 and
// 938 for 172 and 875.  Measured and not taken: a part of the exponentials by a polynomial on the plain units (170 and 868 for the 172 and 875 at best), 16
// softmax warps with half a row a thread (a tenth slower), an issuer that takes whichever product is ready (the same).
//
// A half has two places for S, in turn, with a barrier for S and one for P each: a warp whose rows need no rescaling may be
// a block ahead of another of its half, and must not count for it.  S of block n + 2 goes over P of block n: the products of
// one issuer are done in order, and P's was issued before.  O is rescaled when the products of the block before are done,
// which a barrier tells.  Where there are fewer tiles than SMs, several blocks have parts of a tile's tokens and a second
// kernel joins them.
#include <algorithm>
#include <type_traits>

#include "ans_attend.cuh"
#include "ans_attend_tiles.cuh"

namespace ansb {
namespace blk {

constexpr float kUpTile = 7.f, kSlack = 8.f;           // P <= 2^15
constexpr float kLeastFactor = 1e-38f;                 // of S, so that -inf times it is -inf
constexpr uint32_t kAtSoft = 8, kAtOpen = 4, kAtIssue = kAtSoft + kAtOpen, kAtScales = kAtIssue + 1;   // warps: softmax, converters, issuer, scales
constexpr uint32_t kAtThreads = 32 * (kAtScales + 1);

template <int D>
struct AtShape {
  static constexpr uint32_t kHalves = D <= 128 ? 2 : 1;
  static constexpr uint32_t kRows = 128 * kHalves;
  static constexpr uint32_t kTokens = 64;                              // of a block
  static constexpr uint32_t kPanels = D / 64;                          // of 64 dimensions, 128 bytes
  static constexpr uint32_t kQPanel = 128 * 128, kPanel = kTokens * 128;
  static constexpr uint32_t kQ = kHalves * kPanels * kQPanel;
  static constexpr uint32_t kTile = kPanels * kPanel;                  // K or V of a block
  static constexpr uint32_t kStages = D == 256 ? 2 : 4;
  static constexpr uint32_t kSubs = kTokens / 16;                      // runs of 16 tokens, each in one page
  static constexpr uint32_t kMeta = kStages * kSubs * 16;
  static constexpr uint32_t kBars = 8 * (4 * kStages + 5 * kHalves + 2);
  static constexpr uint32_t kSmem = 1024 + kQ + 2 * kStages * kTile + kMeta + kBars + 16;
  static constexpr uint32_t kOwn = kTokens / kAtOpen, kRuns = kOwn / 16;         // tokens and runs of a converter's warp
  static constexpr uint32_t kPieces = kOwn / 8 * kPanels;              // of 16 codes, of a converter's lane
  static constexpr uint32_t kS = 0, kO = 256;                          // columns in tensor memory: a half's two blocks of S, 64 apart; O; halves 128 and D apart
};

__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
               "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
               :: "r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
                  "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
                  "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
                  "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]));
}
__device__ __forceinline__ void tmem_load4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// operand of tokens x dimensions with the dimensions contiguous: 64 of them in 128 bytes, 8 tokens in 1024, panels `panel` bytes apart
__device__ __forceinline__ uint64_t operand_across(uint32_t addr, uint32_t panel) {
  return uint64_t((addr & 0x3FFFFu) >> 4) | (uint64_t(panel >> 4) << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
// fp16 operands, sums in fp32; B across: its N contiguous
__host__ __device__ constexpr uint32_t instruction_half(uint32_t n, bool across) {
  return (1u << 4) | (across ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}
// One lane of a warp that runs together issues: so the operands stay in uniform registers, and an instruction costs a few
// clocks of issue where a single lane's branch costs 130, twice what the instruction takes on the tensor pipe.
__device__ __forceinline__ uint32_t elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void mma_smem(uint32_t chosen, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(chosen) : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t chosen, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
               "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(chosen) : "memory");
}
__device__ __forceinline__ void commit(uint32_t chosen, uint32_t bar) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
               "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" :: "r"(bar), "r"(chosen) : "memory");
}
__device__ __forceinline__ float largest3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// columns outside [lo, hi) as tokens that are not seen
template <uint32_t N>
__device__ __forceinline__ void hide(uint32_t (&v)[N], int32_t lo, int32_t hi) {
#pragma unroll
  for (int32_t c = 0; c < static_cast<int32_t>(N); ++c)
    if (c < lo || c >= hi) v[c] = 0xFF800000u;
}

// A tile: rows [r0, r0 + live) of a sequence's new tokens x share, and the blocks of tokens that they see.
struct AtTile {
  uint32_t row, fresh, r0, live;
  int32_t old, length;
  uint32_t b0, b1;                                     // blocks of kTokens
};

template <int D>
__global__ void __launch_bounds__(kAtThreads, 1) ans_attend_tiles_kernel(const AttendArgs a, const uint32_t splits) {
  using S = AtShape<D>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_addr(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = q_at + S::kQ, v_at = k_at + S::kStages * S::kTile, meta = v_at + S::kStages * S::kTile;
  const uint32_t bars = meta + S::kMeta;
  const uint32_t k_full = bars, k_empty = k_full + 8 * S::kStages, v_full = k_empty + 8 * S::kStages, v_empty = v_full + 8 * S::kStages;
  const uint32_t s_full = v_empty + 8 * S::kStages, p_full = s_full + 16 * S::kHalves, o_done = p_full + 16 * S::kHalves, q_full = o_done + 8 * S::kHalves, o_full = q_full + 8;
  const uint32_t slot = o_full + 8;
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  uint32_t bad = 0;
  __shared__ uint32_t s_seq;
  const float4* const scales = reinterpret_cast<const float4*>(smem_raw + (meta - smem_addr(smem_raw)));

  if (threadIdx.x == 0) {
    for (uint32_t s = 0; s < S::kStages; ++s) {
      bar_init(k_full + 8 * s, kAtOpen); bar_init(k_empty + 8 * s, 1);
      bar_init(v_full + 8 * s, kAtOpen + 1); bar_init(v_empty + 8 * s, 1);
    }
    for (uint32_t h = 0; h < S::kHalves; ++h) { bar_init(s_full + 16 * h, 1); bar_init(s_full + 16 * h + 8, 1); bar_init(p_full + 16 * h, 4); bar_init(p_full + 16 * h + 8, 4); bar_init(o_done + 8 * h, 1); }
    bar_init(q_full, 4 * S::kHalves);
    bar_init(o_full, 1);
    bar_init_fence();
  }
  if (warp == kAtIssue) tmem_alloc<1>(slot, 512);
  let_next_start();
  wait_for_previous();
  // tiles: sequence s has starts[s] * share / rows + s and on; those that see most come first
  const uint32_t behind = blockIdx.x / a.c.heads, head = blockIdx.x - behind * a.c.heads, x = gridDim.x / a.c.heads - 1u - behind;
  if (warp == 0) {
    const uint32_t found = sequence_at(a.b.starts, a.b.n_seqs, a.share, S::kRows, 1u, x);
    if (lane == 0) s_seq = found;
  }
  fence_before();
  __syncthreads();
  fence_after();
  uint32_t tmem;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(tmem) : "r"(slot));

  const uint32_t s = s_seq;
  AtTile T;
  const Range r = range_of(a.b, s);
  const uint32_t rows = r.fresh * a.share;
  uint32_t blocks = 0;                                 // of this block of threads
  uint32_t first = 0;
  bool mine = false;
  {
    const uint32_t place = static_cast<uint32_t>(uint64_t(r.row) * a.share / S::kRows) + s;
    const uint64_t held = min(uint64_t(a.b.table_pages) * a.c.page_size, uint64_t(kAtLongest));
    T.row = r.row; T.fresh = r.fresh;
    T.length = static_cast<int32_t>(min(uint64_t(max(static_cast<int32_t>(r.length), 0)), held));
    T.old = static_cast<int32_t>(r.length) - static_cast<int32_t>(r.fresh);
    const uint64_t r0 = uint64_t(x - place) * S::kRows;
    mine = r.fits && x >= place && rows >= a.least && rows <= a.most && r0 < rows;
    if (x == 0 && head == 0 && blockIdx.z == 0) {      // what does not fit is found by one block
      bool wrong = false;
      for (uint32_t i = threadIdx.x; i < a.b.n_seqs; i += kAtThreads) {
        const Range o = range_of(a.b, i);
        wrong |= !o.fits || (o.fresh && o.length > held);
      }
      if (wrong) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
    }
    if (mine) {
      T.r0 = static_cast<uint32_t>(r0);
      T.live = min(S::kRows, rows - T.r0);
      const Seen top = seen_by(a, T.old, T.length, token_of(a, T.r0)), end = seen_by(a, T.old, T.length, token_of(a, T.r0 + T.live - 1u));
      T.b0 = static_cast<uint32_t>(top.first) / S::kTokens;
      T.b1 = (static_cast<uint32_t>(end.end) + S::kTokens - 1) / S::kTokens;
      if (T.b1 < T.b0) T.b1 = T.b0;
      const uint32_t all = T.b1 - T.b0;
      first = T.b0 + static_cast<uint32_t>(uint64_t(all) * blockIdx.z / splits);
      blocks = T.b0 + static_cast<uint32_t>(uint64_t(all) * (blockIdx.z + 1u) / splits) - first;
    }
  }
  const uint32_t halves = mine && T.live > 128u ? S::kHalves : 1u;
  const int32_t* const table = a.b.tables + s * a.b.table_stride;

  if (mine && warp < kAtSoft) {
    // ---- softmax: a row a thread
    const uint32_t half = warp >> 2, row = T.r0 + threadIdx.x;
    if (half < halves) {
      const bool live = threadIdx.x < T.live;
      const uint32_t i = token_of(a, live ? row : T.r0), j = (live ? row : T.r0) - i * a.share;
      // the queries of this warp's 32 rows, kPer lanes a row
      constexpr uint32_t kPer = D / 8 < 32 ? D / 8 : 32, kAtOnce = 32 / kPer;
      uint32_t my_top = 0;
      {
        const uint32_t d = (lane % kPer) * 8u;
        uint4 w[32 / kAtOnce];                         // all under way together
#pragma unroll
        for (uint32_t n = 0; n < 32 / kAtOnce; ++n) {
          const uint32_t in_tile = warp * 32u + n * kAtOnce + lane / kPer;
          w[n] = make_uint4(0, 0, 0, 0);
          if (in_tile < T.live && d < a.c.dim) {
            const uint32_t at = T.r0 + in_tile, token = token_of(a, at);
            w[n] = *reinterpret_cast<const uint4*>(a.q + (T.row + token) * a.q_token + (head * a.share + (at - token * a.share)) * a.q_head + d);
          }
        }
#pragma unroll
        for (uint32_t n = 0; n < 32 / kAtOnce; ++n) {
          uint32_t* const e = &w[n].x;
          uint32_t top = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) top = max(top, max((e[k] << 16) & 0x7FFFFFFFu, e[k] & 0x7FFF0000u));
#pragma unroll
          for (uint32_t step = 1; step < kPer; step *= 2) top = max(top, __shfl_xor_sync(kAll, top, step));
#pragma unroll
          for (uint32_t k = 0; k < kAtOnce; ++k) {
            const uint32_t of = __shfl_sync(kAll, top, k * kPer);
            if (lane == n * kAtOnce + k) my_top = of;
          }
          const float down = power_of(-exponent_of(top)) * (a.scale2 < 0.f ? -1.f : 1.f);      // the scale's sign goes to the queries
#pragma unroll
          for (int k = 0; k < 4; ++k) e[k] = pack_half(__uint_as_float(e[k] << 16) * down, __uint_as_float(e[k] & 0xFFFF0000u) * down);
          const uint32_t in_half = (warp * 32u + n * kAtOnce + lane / kPer) & 127u;
          const uint32_t to = q_at + (half * S::kPanels + d / 64u) * S::kQPanel + in_half * 128u + (((d / 8u) & 7u) ^ (in_half & 7u)) * 16u;
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(to), "r"(e[0]), "r"(e[1]), "r"(e[2]), "r"(e[3]) : "memory");
        }
      }
      const float factor = fabsf(a.scale2) * power_of(exponent_of(my_top));
      fence_operands();
      __syncwarp();
      if (lane == 0) arrive(q_full);
      const Seen seen = seen_by(a, T.old, T.length, i);
      const int32_t all_lo = __reduce_max_sync(kAll, seen.first), all_hi = __reduce_min_sync(kAll, seen.end);
      const uint32_t lanes = (warp & 3u) << 21;        // this warp's 32 lanes of tensor memory
      const uint32_t s_both = tmem + lanes + S::kS + half * 128u, o_at = tmem + lanes + S::kO + half * D;
      float top = kLowest, sum = 0.f;
      for (uint32_t n = 0; n < blocks; ++n) {
        const uint32_t stage = n % S::kStages;
        const uint32_t s_at = s_both + (n & 1u) * 64u;
        bar_wait(s_full + 16 * half + 8 * (n & 1u), (n >> 1) & 1u, bad);
        bar_wait(v_full + 8 * stage, (n / S::kStages) & 1u, bad);      // the scales
        __syncwarp();
        fence_after();
        const int32_t t0 = static_cast<int32_t>((first + n) * S::kTokens), lo = seen.first - t0, hi = seen.end - t0;
        const bool inside = t0 >= all_lo && t0 + static_cast<int32_t>(S::kTokens) <= all_hi;
        // of a run of 16 tokens: s_i + e_i = S_i f + e, and what p_i counts for in the sum
        auto run = [&](uint32_t b, float& f, float& e, float& back) {
          const float4 m = scales[stage * S::kSubs + b];
          f = fmaxf(factor * m.x, kLeastFactor);
          e = m.y;
          back = m.z;
        };
        uint32_t v[S::kTokens];
#pragma unroll
        for (uint32_t c = 0; c < S::kTokens; c += 32) tmem_load(s_at + c, *reinterpret_cast<uint32_t(*)[32]>(v + c));
        tmem_wait();
        if (!inside) hide(v, lo, hi);
        // the maximum, of S by runs, as f is positive
        float best = kLowest;
#pragma unroll
        for (uint32_t b = 0; b < S::kSubs; ++b) {
          float m = __uint_as_float(v[16 * b]), f, e, back;
          run(b, f, e, back);
#pragma unroll
          for (uint32_t k = 1; k < 15; k += 2) m = largest3(m, __uint_as_float(v[16 * b + k]), __uint_as_float(v[16 * b + k + 1]));
          best = fmaxf(best, fmaf(fmaxf(m, __uint_as_float(v[16 * b + 15])), f, e));
        }
        if (__any_sync(kAll, best > top + kSlack)) {
          const float now = fmaxf(top, best), by_half = exp2_near(0.5f * (top - now)), shrink = by_half * by_half;
          top = now;
          sum = sum * by_half * by_half;
          if (n) {
            bar_wait(o_done + 8 * half, (n - 1u) & 1u, bad);           // the products before are done; the next ones wait for P
            __syncwarp();
            fence_after();
#pragma unroll 1
            for (uint32_t c = 0; c < D; c += 32) {
              uint32_t o[32];
              tmem_load(o_at + c, o);
              tmem_wait();
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * shrink);
              tmem_store(o_at + c, o);
            }
          }
        }
        // Runs that count in the sum by exponentials of their own, a few columns of S at a time: out of the registers of v this would cost heads
        // of 256 dimensions their registers (1500 rows 69.8 us, so 49.4).
        if (__any_sync(kAll, scales[stage * S::kSubs].w != 0.f)) {
#pragma unroll 1
          for (uint32_t c = 0; c < S::kTokens; c += 4) {
            const float4 m = scales[stage * S::kSubs + c / 16u];
            if (m.w < 2.f) continue;
            uint32_t now[4];
            tmem_load4(s_at + c, now);
            tmem_wait();
            hide(now, lo - static_cast<int32_t>(c), hi - static_cast<int32_t>(c));
            const float f = fmaxf(factor * m.x, kLeastFactor), less = kUpTile + kSum - top;
#pragma unroll
            for (uint32_t k = 0; k < 4; ++k) sum += exp2_near(fmaf(__uint_as_float(now[k]), f, less));
          }
        }
        // one stretch of code without branches, so that the runs' chains of instructions run beside each other
        auto weigh = [&](auto all_seen) {
          const float less = kUpTile - top;
#pragma unroll
          for (uint32_t b = 0; b < S::kSubs; ++b) {
            float f, e, back;
            run(b, f, e, back);
            const float add = e + less;
            const Two ff = two(f, f), aa = two(add, add);
            uint32_t (&now)[16] = *reinterpret_cast<uint32_t(*)[16]>(v + 16 * b);
#pragma unroll
            for (uint32_t k = 0; k < 16; k += 2) {
              const Two y = fma2(two(__uint_as_float(now[k]), __uint_as_float(now[k + 1])), ff, aa);
              now[k] = __float_as_uint(low(y));
              now[k + 1] = __float_as_uint(high(y));
            }
            // what is not seen is hidden again, also from a scale that is NaN
            if constexpr (!decltype(all_seen)::value) hide(now, lo - static_cast<int32_t>(16 * b), hi - static_cast<int32_t>(16 * b));
            Two part[2] = {0, 0};
#pragma unroll
            for (uint32_t k = 0; k < 16; k += 2) {
              const float p0 = exp2_near(__uint_as_float(now[k])), p1 = exp2_near(__uint_as_float(now[k + 1]));
              part[(k / 2) % 2] = add2(part[(k / 2) % 2], two(p0, p1));
              v[8 * b + k / 2] = pack_half(p0, p1);
            }
            const Two both = add2(part[0], part[1]);
            sum = fmaf(low(both) + high(both), back, sum);
          }
        };
        if (inside) weigh(std::true_type{}); else weigh(std::false_type{});
        tmem_store(s_at, *reinterpret_cast<uint32_t(*)[32]>(v));       // P over S, which has been read
        tmem_stored();
        fence_before();
        __syncwarp();
        if (lane == 0) arrive(p_full + 16 * half + 8 * (n & 1u));
      }
      bar_wait(o_full, 0u, bad);
      __syncwarp();
      fence_after();
      const float f = sum == 0.f ? 0.f : kFromSum / sum;
      const uint32_t heads = a.share * a.c.heads;
      const uint64_t part = (uint64_t(blockIdx.z) * a.b.rows + T.row + i) * heads + head * a.share + j;
      if (splits > 1 && live) reinterpret_cast<float2*>(a.parts + uint64_t(splits) * a.b.rows * heads * D)[part] = make_float2(top, sum);
      // Rows leave through the stages of K and V, which are done with, 8 KB a warp: 128 bytes of a row a step, its 16-byte pieces
      // in the places where eight rows meet different banks.
      const uint32_t own = k_at + warp * 8192u;
      static_assert(2 * S::kStages * S::kTile >= 8 * 8192, "");
      constexpr uint32_t kStep = 64;                   // dimensions: as bf16 128 bytes, or as fp32 two lines of 128
      const uint8_t* const own_p = smem_raw + (own - smem_addr(smem_raw));
      // eight lanes a row, rows lane / 8, lane / 8 + 4, ...
      const uint32_t piece = lane & 7u;
      uint64_t goes[8];                                // elements from the start of out or of the parts
#pragma unroll
      for (uint32_t k = 0; k < 8; ++k) {
        const uint32_t at = T.r0 + min(warp * 32u + 4u * k + lane / 8u, T.live - 1u), token = token_of(a, at), h = head * a.share + (at - token * a.share);
        goes[k] = splits > 1 ? ((uint64_t(blockIdx.z) * a.b.rows + T.row + token) * heads + h) * D + 4u * piece
                             : (T.row + token) * a.out_token + h * a.out_head + 8u * piece;
      }
#pragma unroll 1
      for (uint32_t c = 0; c < D; c += kStep) {
        uint32_t o[64];
        tmem_load(o_at + c, *reinterpret_cast<uint32_t(*)[32]>(o));
        tmem_load(o_at + c + 32, *reinterpret_cast<uint32_t(*)[32]>(o + 32));
        tmem_wait();
        if (!blocks) {
#pragma unroll
          for (int k = 0; k < 64; ++k) o[k] = 0u;
        }
        if (splits > 1) {
#pragma unroll
          for (uint32_t k = 0; k < 16; ++k)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(own + (k / 8) * 4096u + lane * 128u + ((k ^ lane) & 7u) * 16u), "r"(o[4 * k]),
                         "r"(o[4 * k + 1]), "r"(o[4 * k + 2]), "r"(o[4 * k + 3]) : "memory");
        } else {
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) {
            uint32_t w[4];
#pragma unroll
            for (uint32_t x = 0; x < 4; ++x) {
              const __nv_bfloat162 b = __floats2bfloat162_rn(__uint_as_float(o[8 * k + 2 * x]) * f, __uint_as_float(o[8 * k + 2 * x + 1]) * f);
              w[x] = *reinterpret_cast<const uint32_t*>(&b);
            }
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(own + lane * 128u + ((k ^ lane) & 7u) * 16u), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                         "r"(w[3]) : "memory");
          }
        }
        __syncwarp();
        for (uint32_t line = 0; line < (splits > 1 ? 2u : 1u); ++line) {
          uint4 w[8];
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) {
            const uint32_t r = 4u * k + lane / 8u;
            w[k] = *reinterpret_cast<const uint4*>(own_p + line * 4096u + r * 128u + ((piece ^ r) & 7u) * 16u);
          }
#pragma unroll
          for (uint32_t k = 0; k < 8; ++k) {
            if (warp * 32u + 4u * k + lane / 8u >= T.live) continue;
            if (splits > 1) {
              *reinterpret_cast<uint4*>(a.parts + goes[k] + c + line * 32u) = w[k];
            } else if (c + 8u * piece < a.c.dim) {
              __nv_bfloat16* const to = a.out + goes[k] + c;
              if (a.out_wide) {
                *reinterpret_cast<uint4*>(to) = w[k];
              } else {
                uint32_t* const p = reinterpret_cast<uint32_t*>(to);
                p[0] = w[k].x; p[1] = w[k].y; p[2] = w[k].z; p[3] = w[k].w;
              }
            }
          }
        }
        __syncwarp();
      }
    }
  } else if (mine && warp < kAtIssue) {
    // ---- converters: a warp has kOwn tokens of every block, one or two runs of 16
    // A lane has piece lane % 4 (16 codes) of each panel of every eighth token: the two chunks of 8 dimensions that it becomes have the
    // same places in every panel and every eight tokens, and four lanes by two tokens write to different banks.
    const uint32_t w = warp - kAtSoft, row0 = lane / 4u, c = lane % 4u;
    const uint32_t line = (w * S::kOwn + row0) * 128u, place0 = line + ((2u * c) ^ (row0 & 7u)) * 16u, place1 = line + ((2u * c + 1u) ^ (row0 & 7u)) * 16u;
    const uint64_t from = uint64_t(row0) * a.c.dim + c * 16u;
    // page numbers are asked for a block ahead of their codes, those a block ahead of their use
    int32_t page[S::kRuns];
    uint32_t offset[S::kRuns];                         // of a run in its page
    auto ask = [&](uint32_t block) {
#pragma unroll
      for (uint32_t r = 0; r < S::kRuns; ++r) {
        const uint32_t token = block * S::kTokens + w * S::kOwn + 16u * r, p_in = token / a.c.page_size;
        offset[r] = token - p_in * a.c.page_size;
        page[r] = -1;
        if (block < first + blocks && token < static_cast<uint32_t>(T.length)) page[r] = table[p_in];
      }
    };
    uint64_t where[S::kRuns];
    bool used[S::kRuns];
    auto take = [&]() {
#pragma unroll
      for (uint32_t r = 0; r < S::kRuns; ++r) {
        used[r] = page[r] >= 0 && static_cast<uint32_t>(page[r]) < a.c.n_pages;
        where[r] = from + ((uint64_t(max(page[r], 0)) * a.c.heads + head) * a.c.page_size + offset[r]) * a.c.dim;
      }
    };
    uint4 codes[2][S::kPieces];                        // piece i: panel i % kPanels, tokens row0 + 8 (i / kPanels)
    auto load = [&](uint32_t which) {
#pragma unroll
      for (uint32_t i = 0; i < S::kPieces; ++i) {
        const uint32_t down = 8u * (i / S::kPanels), p = i % S::kPanels, r = down / 16u;
        codes[which][i] = make_uint4(0, 0, 0, 0);
        if (used[r] && p * 64u + c * 16u < a.c.dim)
          codes[which][i] = *reinterpret_cast<const uint4*>(a.c.codes[which] + where[r] + (down % 16u) * a.c.dim + p * 64u);
      }
    };
    auto open = [&](uint32_t which, uint32_t to) {
#pragma unroll
      for (uint32_t i = 0; i < S::kPieces; ++i) {
        const uint32_t* const x = &codes[which][i].x;
        uint32_t h[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t u = x[k] ^ 0x80808080u;
          h[2 * k] = open_low(u);
          h[2 * k + 1] = open_high(u);
        }
        const uint32_t at = to + (i % S::kPanels) * S::kPanel + 8u * (i / S::kPanels) * 128u;
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at + place0), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at + place1), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7]) : "memory");
      }
    };
    ask(first);
    take();
    load(0);
    load(1);
    ask(first + 1);
    for (uint32_t n = 0; n < blocks; ++n) {
      const uint32_t stage = n % S::kStages, round = n / S::kStages;
      take();
      ask(first + n + 2);
      if (round) bar_wait(k_empty + 8 * stage, (round - 1u) & 1u, bad);
      open(0, k_at + stage * S::kTile);
      fence_operands();
      __syncwarp();
      if (lane == 0) arrive(k_full + 8 * stage);
      load(0);
      if (round) bar_wait(v_empty + 8 * stage, (round - 1u) & 1u, bad);
      open(1, v_at + stage * S::kTile);
      fence_operands();
      __syncwarp();
      if (lane == 0) arrive(v_full + 8 * stage);
      load(1);
    }
  } else if (mine && warp == kAtScales) {
    // ---- scales: lane b has run b of every block
    float ks, e, back, high = -INFINITY;               // high: the largest e so far
    auto look = [&](uint32_t block) {
      const uint32_t token = block * S::kTokens + lane * 16u;
      ks = 1.f; e = -INFINITY; back = 0.f;             // not there: not seen
      if (lane < S::kSubs && block < first + blocks && token < static_cast<uint32_t>(T.length)) {
        const int32_t page = table[token / a.c.page_size];
        if (page >= 0 && static_cast<uint32_t>(page) < a.c.n_pages) {
          const uint64_t at = uint64_t(page) * a.c.heads + head;
          ks = usable(a.c.scales[0][at]);
          e = log2_near(usable(a.c.scales[1][at]));
          if (isnan(ks)) e = ks;
          back = isnan(e) ? 1.f : exp2_near(kSum - e);                 // where e is NaN, so is what is summed
        } else if (token + 16u > static_cast<uint32_t>(seen_by(a, T.old, T.length, token_of(a, T.r0)).first)) {       // what the window has left need not be there
          atomicOr(a.status, ANS_STATUS_BAD_PAGE);
        }
      }
    };
    for (uint32_t n = 0; n < blocks; ++n) {
      const uint32_t stage = n % S::kStages, round = n / S::kStages;
      look(first + n);
      float top = e;
#pragma unroll
      for (uint32_t step = 1; step < S::kSubs; step *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, step));
      high = fmaxf(high, top);
      const bool apart = e + kApart < high && e > kLowest;
      if (apart) back = 0.f;
      const float how = (__any_sync(kAll, apart) ? 1.f : 0.f) + (apart ? 1.f : 0.f);          // 1: a run of the block is, 2: this one
      if (round) bar_wait(v_empty + 8 * stage, (round - 1u) & 1u, bad);
      if (lane < S::kSubs)
        asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(meta + (stage * S::kSubs + lane) * 16u), "f"(ks), "f"(e), "f"(back), "f"(how) : "memory");
      __syncwarp();
      if (lane == 0) arrive(v_full + 8 * stage);
    }
  } else if (mine) {
    if (warp == kAtIssue) {
      // ---- issuer: the whole warp waits, one lane issues
      const uint32_t me = elect();
      constexpr uint32_t is = instruction_half(S::kTokens, false), io = instruction_half(D, true);
      auto scores = [&](uint32_t h, uint32_t n) {
        const uint32_t stage = n % S::kStages;
#pragma unroll
        for (uint32_t p = 0; p < S::kPanels; ++p) {
          const uint64_t dq = operand(q_at + (h * S::kPanels + p) * S::kQPanel), dk = operand(k_at + stage * S::kTile + p * S::kPanel);
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) mma_smem(me, tmem + S::kS + h * 128u + (n & 1u) * 64u, dq + 2u * k, dk + 2u * k, is, p || k);
        }
        commit(me, s_full + 16 * h + 8 * (n & 1u));
      };
      auto outputs = [&](uint32_t h, uint32_t n) {
        const uint64_t dv = operand_across(v_at + n % S::kStages * S::kTile, S::kPanel);
        const uint32_t p = tmem + S::kS + h * 128u + (n & 1u) * 64u;
#pragma unroll
        for (uint32_t k = 0; k < S::kTokens / 16; ++k)
          mma_tmem(me, tmem + S::kO + h * D, p + 8u * k, dv + uint64_t(k * 2048u >> 4), io, n || k);
        commit(me, o_done + 8 * h);
      };
      for (uint32_t h = 0; h < S::kHalves; ++h)
        if (h >= halves) for (uint32_t i = 0; i < 4; ++i) { if (lane == 0) arrive(q_full); }            // a half without rows
      bar_wait(q_full, 0u, bad);
      // S of the next block is made while the softmax of this one runs
      if (blocks) {
        bar_wait(k_full, 0u, bad);
        fence_after();
        for (uint32_t h = 0; h < halves; ++h) scores(h, 0);
        commit(me, k_empty);
      }
      for (uint32_t n = 0; n < blocks; ++n) {
        const uint32_t stage = n % S::kStages, next = (n + 1) % S::kStages;
        for (uint32_t h = 0; h < halves; ++h) {
          if (n + 1 < blocks) {
            if (h == 0) bar_wait(k_full + 8 * next, ((n + 1) / S::kStages) & 1u, bad);
            fence_after();
            scores(h, n + 1);
            if (h + 1 == halves) commit(me, k_empty + 8 * next);
          }
          if (h == 0) bar_wait(v_full + 8 * stage, (n / S::kStages) & 1u, bad);
          bar_wait(p_full + 16 * h + 8 * (n & 1u), (n >> 1) & 1u, bad);
          fence_after();
          outputs(h, n);
          if (h + 1 == halves) commit(me, v_empty + 8 * stage);
        }
      }
      commit(me, o_full);
      bar_wait(o_full, 0u, bad);                       // nothing is under way any more
    }
  }
  fence_before();
  __syncthreads();
  if (warp == kAtIssue) {
    fence_after();
    tmem_free<1>(tmem, 512);
  }
  bad = __any_sync(kAll, bad);
  if (lane == 0 && bad) atomicOr(a.status, ANS_STATUS_COPY_TIMEOUT);
}

// Joins the parts of every row of the sequences that the tiles kernel had: a warp a row and head.
template <int D>
__global__ void __launch_bounds__(256) ans_attend_tiles_join_kernel(const AttendArgs a, const uint32_t splits) {
  let_next_start();
  wait_for_previous();
  const uint32_t lane = threadIdx.x & 31u, heads = a.share * a.c.heads;
  const uint64_t at = uint64_t(blockIdx.x) * 8u + (threadIdx.x >> 5);
  if (at >= uint64_t(a.b.rows) * heads) return;
  const uint32_t row = static_cast<uint32_t>(at / heads), head = static_cast<uint32_t>(at - uint64_t(row) * heads);
  uint32_t lo = 0, hi = a.b.n_seqs;                    // the last sequence that does not start behind the row
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (a.b.starts[mid] <= static_cast<int32_t>(row)) lo = mid; else hi = mid;
  }
  const Range r = range_of(a.b, lo);
  const uint64_t rows = uint64_t(r.fresh) * a.share;
  if (!r.fits || row < r.row || row - r.row >= r.fresh || rows < a.least || rows > a.most) return;
  const uint64_t all = uint64_t(a.b.rows) * heads;
  const float2* const ml = reinterpret_cast<const float2*>(a.parts + splits * all * D);
  float most = kLowest, sum = 0.f;
  for (uint32_t z = 0; z < splits; ++z) most = fmaxf(most, ml[z * all + at].x);
  float x[D / 32];
#pragma unroll
  for (int k = 0; k < D / 32; ++k) x[k] = 0.f;
#pragma unroll 2
  for (uint32_t z = 0; z < splits; ++z) {
    const float2 m = ml[z * all + at];
    const float half = exp2_near(0.5f * (m.x - most)), f = half * half;
    sum = fmaf(half, half * m.y, sum);
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
      const float2 v = *reinterpret_cast<const float2*>(a.parts + (z * all + at) * D + 64 * k + 2 * lane);
      x[2 * k] = fmaf(f, v.x, x[2 * k]);
      x[2 * k + 1] = fmaf(f, v.y, x[2 * k + 1]);
    }
  }
  const float f = sum == 0.f ? 0.f : kFromSum / sum;
  __nv_bfloat16* const to = a.out + row * a.out_token + head * a.out_head;
#pragma unroll
  for (int k = 0; k < D / 64; ++k) {
    const uint32_t d = 64u * k + 2u * lane;
    if (d < a.c.dim) *reinterpret_cast<__nv_bfloat162*>(to + d) = __floats2bfloat162_rn(x[2 * k] * f, x[2 * k + 1] * f);
  }
}

// ---- host side -----------------------------------------------------------------------------
template <int D>
static void plan_tiles_shape(const AttendArgs& a, int sms, AtPlan& p) {
  using S = AtShape<D>;
  const uint64_t rows = uint64_t(a.b.rows) * a.share;
  p.tiles = static_cast<uint32_t>(rows / S::kRows + a.b.n_seqs);
  // Parts: as many as there are SMs for, of 512 tokens at least, 16 at most.  100 tokens (4 query heads a head, D = 128) behind 700, 1500 and 3000 of 2
  // heads take 25, 25 and 25 us, undivided 25, 40 and 67; with parts of 128 tokens 17, 20 and 21, of 1024 25, 40 and 33.  Behind 64000 of 8, 2 and 1
  // heads 155, 93 and 90 us; with up to 8 parts 172, 163 and 159, with up to 37 155, 58 and 54.
  const uint64_t units = std::max<uint64_t>((rows + S::kRows - 1) / S::kRows * a.c.heads, 1);
  const uint64_t most = uint64_t(a.b.table_pages) * a.c.page_size / 512;
  p.splits = static_cast<uint32_t>(std::max<uint64_t>(std::min<uint64_t>({uint64_t(sms) / units, most, 16}), 1));
  p.room = p.splits > 1 ? size_t(p.splits) * a.b.rows * a.share * a.c.heads * (D + 2) * sizeof(float) : 0;
}
void plan_tiles(const AttendArgs& a, int sms, AtPlan& p) {
  if (a.c.dim <= 64) plan_tiles_shape<64>(a, sms, p);
  else if (a.c.dim <= 128) plan_tiles_shape<128>(a, sms, p);
  else plan_tiles_shape<256>(a, sms, p);
}

template <int D>
static int launch_tiles_shape(const AttendArgs& a, const AtPlan& p, cudaStream_t st) {
  using S = AtShape<D>;
  constexpr auto kernel = ans_attend_tiles_kernel<D>;
  static_assert(S::kSmem <= 227 * 1024, "");
  if (uint64_t(a.c.heads) * p.tiles > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  int rc = allow_smem<kernel>(S::kSmem);
  if (rc == ANS_OK) rc = launch(kernel, dim3(a.c.heads * p.tiles, 1, p.splits), dim3(kAtThreads), S::kSmem, st, 1, a, p.splits);
  if (rc == ANS_OK && p.splits > 1) {
    const uint64_t blocks = (uint64_t(a.b.rows) * a.share * a.c.heads + 7) / 8;
    rc = launch(ans_attend_tiles_join_kernel<D>, dim3(static_cast<unsigned>(blocks)), dim3(256), 0, st, 1, a, p.splits);
  }
  return rc;
}
int launch_tiles(const AttendArgs& a, const AtPlan& p, cudaStream_t st) {
  if (a.c.dim <= 64) return launch_tiles_shape<64>(a, p, st);
  if (a.c.dim <= 128) return launch_tiles_shape<128>(a, p, st);
  return launch_tiles_shape<256>(a, p, st);
}

}  // namespace blk
}  // namespace ansb
