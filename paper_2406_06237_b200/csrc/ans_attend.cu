// Attention over the block-scaled cache for few queries a head of the cache (single tokens, short runs of new tokens), whose
// cost is reading the cache once.
//
// Warps read 16 tokens at a time, keys and values, into their own rings in shared memory (cp.async), open the codes to
// fp16 in registers and use them as the 16-row operand of mma.sync: S^T = K Q^T (16 tokens x 8 queries), O^T = V^T P^T.
// At this operand size the tensor pipe is at a third and DRAM is what is left, while tcgen05 would ask for the opened codes in
// shared memory, 4 bytes more of traffic there for each byte read.
//
// The order of dimensions in a product of S is free, so a lane takes 16 bytes of a row of K at once; so is the order in which the
// rows of O^T stand for dimensions, so a lane takes 16 bytes of four rows of V and pairs their bytes.  P^T comes out of S^T by a
// transpose of 8 x 8 blocks in registers.
//
// Work is cut into chunks of 128 tokens of one (sequence, head, group of queries), all chunks of the call in a row are dealt
// evenly over the blocks that fit the GPU at once, and what a block has of a unit that others have parts of goes to a
// workspace, which a second kernel joins in the order of the blocks: results do not depend on timing.
//
// Measured: one new token each of 64 requests with 762 to 1500 cached (32 query heads on 8, D = 128; 149 MB) 41.8 us, 3.6 TB/s;
// one request of 32768 tokens 21.9 us.  What bounds is the issue of instructions and their latency at 4 warps a scheduler (52 % of the issue
// slots): over inputs that pass L2 several times the two take 39.6 and 19.9 us without the copies, 32.7 and 18.1 without the
// arithmetic, 21.4 and 10.6 without both (the requests' numbers, tables, scales, the units' beginnings and ends), 37.9 and 17.2 without the join.
// That a tile may count apart in the sum (ans_attend.cuh) costs 1 of the first.  Not faster: two runs of 16 tokens at a time a warp
// (45.3 and 39.2 when the first was 44.3: fewer bytes under way), dealing over warps instead of blocks (42.5 and 23.4: more parts to join).
#include <cmath>

#include <algorithm>

#include "ans_attend.cuh"
#include "ans_attend_tiles.cuh"

namespace ansb {
namespace blk {

constexpr uint32_t kArWarps = 8, kArThreads = 32 * kArWarps, kArChunk = 16 * kArWarps, kArStages = 3;

template <int D, int NT>
struct ArShape {
  static constexpr uint32_t kQueries = 8 * NT;
  static constexpr uint32_t kStage = 16 * D * 2;                      // a warp's keys and values
  static constexpr uint32_t kRing = kArWarps * kArStages * kStage;
  static constexpr uint32_t kRow = D + 4;                             // floats of a query's sums in shared memory
  static constexpr uint32_t kSums = kArWarps * kQueries * kRow * 4;
  static constexpr uint32_t kBody = kRing > kSums ? kRing : kSums;
  // then: where a warp's tiles lie and their scales, the warps' maxima and sums, the sequences' first chunks
  static constexpr uint32_t kMeta = kArWarps * 64 * 16;
  static constexpr uint32_t kMl = kArWarps * kQueries * 8 + kQueries * 8 + kArWarps * kQueries * 4;
  static constexpr uint32_t kSmem = kBody + kMeta + kMl;              // + 4 (n + 1)
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from, uint32_t bytes) {       // bytes: 16, or 0 for zeros
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
  return v;
}
__device__ __forceinline__ uint2 lds8(uint32_t at) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
  return v;
}

// Where 16-byte piece c of row `row` lies in a stage: K: pieces of neighbouring rows in different halves of 128 bytes, V: of
// every other row in different 16 bytes, which is how the lanes of a quarter-warp take them.
template <int D> __device__ __forceinline__ uint32_t k_piece(uint32_t row, uint32_t c) {
  return row * D + (D >= 128 ? c ^ ((row & 1u) << 2) : c) * 16u;
}
template <int D> __device__ __forceinline__ uint32_t v_piece(uint32_t row, uint32_t c) {
  return row * D + (D >= 128 ? c ^ (row & 7u) : c ^ ((row >> 1) & 3u)) * 16u;
}

// A sequence's units and chunks.
struct ArSeq {
  uint32_t row, fresh;
  int32_t old, length;                                 // old: tokens before the new ones (negative: some rows see nothing)
  uint32_t first, begin, chunks, groups;               // first token that a row sees, and its chunk's, chunks of a unit, groups of queries
};
template <uint32_t QUERIES>
__device__ __forceinline__ ArSeq ar_sequence(const AttendArgs& a, uint32_t s, bool& bad) {
  const Range r = range_of(a.b, s);
  ArSeq q;
  q.row = r.row;
  q.fresh = r.fresh;
  const uint64_t held = min(uint64_t(a.b.table_pages) * a.c.page_size, uint64_t(kAtLongest));
  bad |= !r.fits || (r.fresh && r.length > held);
  q.length = static_cast<int32_t>(min(uint64_t(max(static_cast<int32_t>(r.length), 0)), held));
  q.old = static_cast<int32_t>(r.length) - static_cast<int32_t>(r.fresh);
  const uint64_t rows = uint64_t(r.fresh) * a.share;
  q.groups = rows >= a.least && rows <= a.most ? static_cast<uint32_t>((rows + QUERIES - 1) / QUERIES) : 0u;
  q.first = static_cast<uint32_t>(max(seen_by(a, q.old, q.length, 0).first, 0));
  q.begin = q.first / kArChunk * kArChunk;
  const uint32_t tokens = q.length > static_cast<int32_t>(q.begin) ? q.length - q.begin : 0u;
  q.chunks = max((tokens + kArChunk - 1) / kArChunk, 1u);
  return q;
}

constexpr uint32_t kArMost = 0x7FFFFFFFu;              // chunks of a call stop here
__device__ __forceinline__ uint32_t ar_plus(uint32_t x, uint32_t y) { return min(x + y, kArMost); }

// The workspace: a record for each block, then for each block two slots of kQueries x (D sums, maximum, sum).
struct ArRecord { uint32_t seq, unit, last, live; };

// EXACT: heads are of D dimensions, so that a tile's 16 pieces lie constants apart.
template <int D, int NT, bool EXACT>
__global__ void __launch_bounds__(kArThreads, D * NT <= 128 ? 2 : 1) ans_attend_rows_kernel(const AttendArgs a) {
  using S = ArShape<D, NT>;
  constexpr uint32_t Q = S::kQueries;
  extern __shared__ __align__(128) uint8_t smem[];
  const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, t = lane & 3u;
  float* const sums = reinterpret_cast<float*>(smem);
  uint4* const tiles = reinterpret_cast<uint4*>(smem + S::kBody) + warp * 64;           // of chunk c: [c % 64] {place in the codes, kscale, log2 vscale}; kscale < 0: counts apart
  float2* const ml = reinterpret_cast<float2*>(smem + S::kBody + S::kMeta);            // [warp][query] {maximum, sum}
  float2* const total_ml = ml + kArWarps * Q;                                          // [query]
  float* const weight = reinterpret_cast<float*>(total_ml + Q);                        // [warp][query]
  uint32_t* const first = reinterpret_cast<uint32_t*>(smem + S::kSmem);                // [n + 1]
  __shared__ uint32_t part[kArWarps];
  __shared__ float highest[kArWarps];                  // of a warp's unit: the largest log2 vscale so far
  const uint32_t ring = smem_addr(smem) + warp * kArStages * S::kStage;
  const uint32_t n = a.b.n_seqs;
  let_next_start();
  wait_for_previous();

  // chunks of all sequences, summed
  uint32_t total = 0;
  bool bad = false;
  for (uint32_t s0 = 0; s0 < n; s0 += kArThreads) {
    const uint32_t s = s0 + threadIdx.x;
    uint32_t x = 0;
    if (s < n) {
      const ArSeq q = ar_sequence<Q>(a, s, bad);
      x = static_cast<uint32_t>(min(uint64_t(q.groups) * q.chunks * a.c.heads, uint64_t(kArMost)));
    }
    const uint32_t own = x;
#pragma unroll
    for (uint32_t step = 1; step < 32; step *= 2) {
      const uint32_t from = __shfl_up_sync(kAll, x, step);
      if (lane >= step) x = ar_plus(x, from);
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    uint32_t before = total;
#pragma unroll
    for (uint32_t w = 0; w < kArWarps; ++w) {
      if (w == warp && s < n) first[s] = ar_plus(before, x - own);     // x - own: exact unless the sums have stopped
      before = ar_plus(before, part[w]);
    }
    total = before;
    __syncthreads();
  }
  if (threadIdx.x == 0) first[n] = total;
  if (blockIdx.x == 0 && (bad || total == kArMost)) atomicOr(a.status, ANS_STATUS_BAD_PAGE);
  if (total == kArMost) total = 0;
  __syncthreads();
  const uint32_t blocks = min(gridDim.x, total);
  ArRecord* const record = reinterpret_cast<ArRecord*>(a.parts) + blockIdx.x;
  if (blockIdx.x >= blocks) {
    if (a.parts && threadIdx.x == 0) *record = ArRecord{0, 0, 0, 0};
    return;
  }
  float* const slots = a.parts + gridDim.x * (sizeof(ArRecord) / 4);
  uint32_t at = static_cast<uint32_t>(uint64_t(total) * blockIdx.x / blocks);
  const uint32_t end = static_cast<uint32_t>(uint64_t(total) * (blockIdx.x + 1u) / blocks);
  ArRecord mine{0, 0, 0, 0};

  uint32_t s = 0;
  {
    uint32_t hi = n;
    while (hi - s > 1) {                               // the last s with first[s] <= at: it has chunks
      const uint32_t mid = (s + hi) / 2;
      if (first[mid] <= at) s = mid; else hi = mid;
    }
  }
  while (at < end) {
    while (first[s + 1] <= at) ++s;
    bool unused = false;
    const ArSeq q = ar_sequence<Q>(a, s, unused);
    const uint32_t unit = (at - first[s]) / q.chunks, c0 = at - first[s] - unit * q.chunks;
    const uint32_t c1 = min(q.chunks, c0 + (end - at));
    const uint32_t head = unit / q.groups, group = unit - head * q.groups;
    const uint32_t rows = q.fresh * a.share, r0 = group * Q, live = min(Q, rows - r0);
    const int32_t* const table = a.b.tables + s * a.b.table_stride;

    // this warp's tokens: 16 of each chunk; where a tile begins in the codes, and its scales, for 32 chunks at a time: the places
    // first, so that copies begin while the scales are on their way
    uint32_t known = c0, scaled = c0;                  // chunks before them have their places, their scales in the table
    const uint32_t dim = EXACT ? D : a.c.dim;
    float k_of = 0.f, v_of = 0.f;
    highest[warp] = -INFINITY;
    __syncwarp();
    auto scales = [&]() {
      if (scaled == known) return;
      float* const to = reinterpret_cast<float*>(tiles + (scaled + lane) % 64u);
      const float k = usable(k_of), e = log2_near(usable(v_of));
      float top = fmaxf(e, highest[warp]);
#pragma unroll
      for (uint32_t step = 1; step < 32; step *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, step));
      highest[warp] = top;
      to[2] = e + kApart < top ? -k : k;
      to[3] = e;
      scaled = known;
      __syncwarp();
    };
    auto look = [&]() {
      scales();
      const uint32_t c = known + lane, token = q.begin + c * kArChunk + warp * 16u;
      uint64_t where = ~uint64_t(0);                   // not there
      if (c < c1 && token < static_cast<uint32_t>(q.length) && token + 16u > q.first) {          // what the window has left need not be there
        const uint32_t in = token / a.c.page_size;
        const int32_t page = table[in];
        if (page >= 0 && static_cast<uint32_t>(page) < a.c.n_pages) {
          const uint64_t block = uint64_t(page) * a.c.heads + head;
          where = (block * a.c.page_size + (token - in * a.c.page_size)) * dim;
          k_of = a.c.scales[0][block];
          v_of = a.c.scales[1][block];
        } else {
          atomicOr(a.status, ANS_STATUS_BAD_PAGE);
        }
      }
      *reinterpret_cast<uint2*>(tiles + c % 64u) = make_uint2(static_cast<uint32_t>(where), static_cast<uint32_t>(where >> 32));
      known += 32u;
      __syncwarp();
    };
    // a lane's pieces of a tile: D / 32 of 16 codes of K and of V, kDown rows apart
    constexpr uint32_t kDown = 512 / D;
    const uint32_t row0 = lane / (D / 16), x0 = lane % (D / 16), lane_at = row0 * dim + x0 * 16u, in = x0 * 16u < dim ? 16u : 0u;
    auto fetch = [&](uint32_t c, uint32_t stage) {     // chunk c's tile into a stage
      if (c < c1) {
        if (c >= known) look();
        const uint2 tile = *reinterpret_cast<const uint2*>(tiles + c % 64u);
        if ((tile.x & tile.y) != 0xFFFFFFFFu) {
          const uint64_t at = (uint64_t(tile.y) << 32 | tile.x) + (EXACT || in ? lane_at : 0u);
          const int8_t* const k = a.c.codes[0] + at;
          const int8_t* const v = a.c.codes[1] + at;
          const uint32_t to = ring + stage * S::kStage;
#pragma unroll
          for (uint32_t i = 0; i < D / 32; ++i) {
            const uint32_t row = row0 + kDown * i, far = EXACT || in ? kDown * i * dim : 0u;
            copy16(to + k_piece<D>(row, x0), k + far, EXACT ? 16u : in);
            copy16(to + 16u * D + v_piece<D>(row, x0), v + far, EXACT ? 16u : in);
          }
        }
      }
      copies_end();
    };
    // queries, on their way with the first tiles: column g of each 8; row r of the group is new token (r0 + r) / share, query head
    // (r0 + r) % share of the head
    uint4 qw[NT][D / 32];
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const uint32_t r = 8u * m + g;
      const uint32_t i = token_of(a, r0 + min(r, live - 1u)), j = (r0 + min(r, live - 1u)) - i * a.share;
      const __nv_bfloat16* const from = a.q + (q.row + i) * a.q_token + (head * a.share + j) * a.q_head;
#pragma unroll
      for (uint32_t x = 0; x < D / 32; ++x) {          // 8 values: half x % 2 of dims 64 (x / 2) + 16 t
        const uint32_t d = 64u * (x / 2) + 16u * t + 8u * (x % 2);
        qw[m][x] = make_uint4(0, 0, 0, 0);
        if (d < dim && r < live) qw[m][x] = *reinterpret_cast<const uint4*>(from + d);
      }
    }
#pragma unroll
    for (uint32_t i = 0; i + 1 < kArStages; ++i) fetch(c0 + i, i);

    uint32_t qf[NT][D / 16][2];
    float factor[NT][2];                               // of the lane's columns 2t and 2t + 1 of S^T
    int32_t lo[NT][2], hi[NT][2];
    int32_t all_lo = 0, all_hi = 0x7FFFFFFF, any_hi = 0;     // tokens that all rows see, and end of those that one does
#pragma unroll
    for (int m = 0; m < NT; ++m) {
      const uint4 (&w)[D / 32] = qw[m];
      uint32_t top = 0;
#pragma unroll
      for (uint32_t x = 0; x < D / 32; ++x) {
        const uint32_t* const e = &w[x].x;
#pragma unroll
        for (int k = 0; k < 4; ++k) top = max(top, max((e[k] << 16) & 0x7FFFFFFFu, e[k] & 0x7FFF0000u));
      }
      top = max(top, __shfl_xor_sync(kAll, top, 1));
      top = max(top, __shfl_xor_sync(kAll, top, 2));
      const int32_t up = exponent_of(top);
      const float down = power_of(-up);
#pragma unroll
      for (uint32_t x = 0; x < D / 32; ++x) {
        const uint32_t* const e = &w[x].x;
        uint32_t h[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = pack_half(__uint_as_float(e[k] << 16) * down, __uint_as_float(e[k] & 0xFFFF0000u) * down);
        // product 4 (x / 2) + j takes bytes 4 j .. 4 j + 3 of a lane's 16 of K
        const uint32_t k = 4u * (x / 2) + 2u * (x % 2);
        qf[m][k][0] = h[0]; qf[m][k][1] = h[1];
        qf[m][k + 1][0] = h[2]; qf[m][k + 1][1] = h[3];
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        factor[m][e] = a.scale2 * power_of(__shfl_sync(kAll, up, (2u * t + e) * 4u));
        const uint32_t col = 8u * m + 2u * t + e;
        const Seen v = seen_by(a, q.old, q.length, token_of(a, r0 + min(col, live - 1u)));
        lo[m][e] = v.first;
        hi[m][e] = v.end;
        all_lo = max(all_lo, v.first);
        all_hi = min(all_hi, v.end);
        any_hi = max(any_hi, v.end);
      }
    }
    all_lo = __reduce_max_sync(kAll, all_lo);
    all_hi = __reduce_min_sync(kAll, all_hi);
    any_hi = __reduce_max_sync(kAll, any_hi);

    float o[NT][D / 16][4];
    float top[NT][2], sum[NT][2];
#pragma unroll
    for (int m = 0; m < NT; ++m) {
#pragma unroll
      for (int k = 0; k < D / 16; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][k][e] = 0.f;
      top[m][0] = top[m][1] = kLowest;
      sum[m][0] = sum[m][1] = 0.f;
    }

    uint32_t stage = 0;
    for (uint32_t c = c0; c < c1; ++c) {
      fetch(c + kArStages - 1u, stage == 0 ? kArStages - 1u : stage - 1u);
      if (c >= scaled) scales();
      copies_wait<kArStages - 1>();
      __syncwarp();
      const int32_t token = static_cast<int32_t>(q.begin + c * kArChunk + warp * 16u);
      const uint4 tile = tiles[c % 64u];
      if ((tile.x & tile.y) != 0xFFFFFFFFu && token < any_hi) {
        const uint32_t keys = ring + stage * S::kStage, values = keys + 16u * D;
        float sc[NT][4];
#pragma unroll
        for (int m = 0; m < NT; ++m) sc[m][0] = sc[m][1] = sc[m][2] = sc[m][3] = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < D / 64; ++i) {
          const uint4 x = lds16(keys + k_piece<D>(g, 4u * i + t)), y = lds16(keys + k_piece<D>(g + 8u, 4u * i + t));
          const uint32_t* const xw = &x.x;
          const uint32_t* const yw = &y.x;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t u = xw[j] ^ 0x80808080u, v = yw[j] ^ 0x80808080u;
            const uint32_t a0 = open_low(u), a1 = open_low(v), a2 = open_high(u), a3 = open_high(v);
#pragma unroll
            for (int m = 0; m < NT; ++m) mma16(sc[m], a0, a1, a2, a3, qf[m][4 * i + j][0], qf[m][4 * i + j][1]);
          }
        }
        const float e = __uint_as_float(tile.w), back = __uint_as_float(tile.z) < 0.f ? 0.f : exp2_near(kSum - e);
        const bool inside = token >= all_lo && token + 16 <= all_hi;
        uint32_t p[NT][2];
#pragma unroll
        for (int m = 0; m < NT; ++m) {
          float best[2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {                // columns 2t + k: values k (token g) and k + 2 (token g + 8)
            const float f = factor[m][k] * fabsf(__uint_as_float(tile.z));
            sc[m][k] = fmaf(sc[m][k], f, e);
            sc[m][k + 2] = fmaf(sc[m][k + 2], f, e);
            if (!inside) {
              const int32_t x = token + static_cast<int32_t>(g), y = x + 8;
              if (x < lo[m][k] || x >= hi[m][k]) sc[m][k] = -INFINITY;
              if (y < lo[m][k] || y >= hi[m][k]) sc[m][k + 2] = -INFINITY;
            }
            best[k] = fmaxf(sc[m][k], sc[m][k + 2]);
          }
#pragma unroll
          for (uint32_t step = 4; step < 32; step *= 2) {
            best[0] = fmaxf(best[0], __shfl_xor_sync(kAll, best[0], step));
            best[1] = fmaxf(best[1], __shfl_xor_sync(kAll, best[1], step));
          }
          if (__any_sync(kAll, best[0] > top[m][0] || best[1] > top[m][1])) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float now = fmaxf(top[m][k], best[k]), half = exp2_near(0.5f * (top[m][k] - now)), shrink = half * half;
              top[m][k] = now;
              sum[m][k] = sum[m][k] * half * half;
#pragma unroll
              for (int d = 0; d < D / 16; ++d) {
                o[m][d][k] *= shrink;
                o[m][d][k + 2] *= shrink;
              }
            }
          }
          float pr[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) pr[k] = exp2_near(sc[m][k] - (top[m][k & 1] - kUp));
          // a row that sees none of the tile's tokens is left alone, also where the tile's scale is NaN
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const float add = pr[k] + pr[k + 2];
            if (add != 0.f) sum[m][k] = fmaf(add, back, sum[m][k]);
          }
          p[m][0] = transpose8(pack_half(pr[0], pr[1]));
          p[m][1] = transpose8(pack_half(pr[2], pr[3]));
        }
        if (__any_sync(kAll, __uint_as_float(tile.z) < 0.f)) {         // the same for all lanes, which the vote tells the compiler
#pragma unroll
          for (int m = 0; m < NT; ++m)
#pragma unroll
            for (int k = 0; k < 2; ++k) sum[m][k] += exp2_near(sc[m][k] - e + (kUp + kSum - top[m][k])) + exp2_near(sc[m][k + 2] - e + (kUp + kSum - top[m][k]));
        }
        // values: rows 2t, 2t + 1, 2t + 8, 2t + 9
        constexpr int kWords = D / 32;                 // of a row, for this lane
        uint32_t v[4][kWords];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t row = 2u * t + (k & 1u) + (k >= 2 ? 8u : 0u);
          if constexpr (D == 64) {
            const uint2 u = lds8(values + v_piece<D>(row, g >> 1) + (g & 1u) * 8u);
            v[k][0] = u.x; v[k][1] = u.y;
          } else {
#pragma unroll
            for (int i = 0; i < kWords / 4; ++i) {
              const uint4 u = lds16(values + v_piece<D>(row, g + 8u * i));
              v[k][4 * i] = u.x; v[k][4 * i + 1] = u.y; v[k][4 * i + 2] = u.z; v[k][4 * i + 3] = u.w;
            }
          }
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k][w] ^= 0x80808080u;
#pragma unroll
          for (int h = 0; h < 2; ++h) {                // bytes 2 h and 2 h + 1 of the word
            const uint32_t pair0 = __byte_perm(v[0][w], v[1][w], h ? 0x7362 : 0x5140), pair1 = __byte_perm(v[2][w], v[3][w], h ? 0x7362 : 0x5140);
            const uint32_t a0 = open_low(pair0), a1 = open_high(pair0), a2 = open_low(pair1), a3 = open_high(pair1);
#pragma unroll
            for (int m = 0; m < NT; ++m) mma16(o[m][2 * w + h], a0, a1, a2, a3, p[m][0], p[m][1]);
          }
        }
      }
      __syncwarp();
      stage = stage + 1 == kArStages ? 0u : stage + 1u;
    }
    copies_wait<0>();
    __syncthreads();                                   // the rings are read

    // the warps' parts
#pragma unroll
    for (int m = 0; m < NT; ++m) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float x = sum[m][k];
#pragma unroll
        for (uint32_t step = 4; step < 32; step *= 2) x += __shfl_xor_sync(kAll, x, step);
        const uint32_t r = 8u * m + 2u * t + k;
        if (g == 0) ml[warp * Q + r] = make_float2(top[m][k], x);
        float* const to = sums + (warp * Q + r) * S::kRow;
#pragma unroll
        for (int w = 0; w < D / 32; ++w) {
          const uint32_t d = D == 64 ? 8u * g + 4u * w : 128u * (w / 4) + 16u * g + 4u * (w % 4);
          *reinterpret_cast<float4*>(to + d) = make_float4(o[m][2 * w][k], o[m][2 * w][k + 2], o[m][2 * w + 1][k], o[m][2 * w + 1][k + 2]);
        }
      }
    }
    __syncthreads();
    if (threadIdx.x < Q) {
      float most = kLowest, all = 0.f;
      for (uint32_t w = 0; w < kArWarps; ++w) most = fmaxf(most, ml[w * Q + threadIdx.x].x);
      for (uint32_t w = 0; w < kArWarps; ++w) {
        const float2 x = ml[w * Q + threadIdx.x];
        const float half = exp2_near(0.5f * (x.x - most));
        weight[w * Q + threadIdx.x] = half * half;
        all = fmaf(half, half * x.y, all);
      }
      total_ml[threadIdx.x] = make_float2(most, all);
    }
    __syncthreads();
    const bool whole = c0 == 0 && c1 == q.chunks;
    float* const slot = slots + uint64_t(2u * blockIdx.x + (c0 == 0 ? 1u : 0u)) * Q * (D + 2);
    for (uint32_t i = threadIdx.x; i < live * (D / 4); i += kArThreads) {
      const uint32_t r = i / (D / 4), d = i % (D / 4) * 4u;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (uint32_t w = 0; w < kArWarps; ++w) {
        const float f = weight[w * Q + r];
        const float4 y = *reinterpret_cast<const float4*>(sums + (w * Q + r) * S::kRow + d);
        x.x = fmaf(f, y.x, x.x); x.y = fmaf(f, y.y, x.y); x.z = fmaf(f, y.z, x.z); x.w = fmaf(f, y.w, x.w);
      }
      if (whole) {
        if (d < a.c.dim) {
          const float l = total_ml[r].y, f = l == 0.f ? 0.f : kFromSum / l;
          const uint32_t row = token_of(a, r0 + r), j = (r0 + r) - row * a.share;
          __nv_bfloat162* const to = reinterpret_cast<__nv_bfloat162*>(a.out + (q.row + row) * a.out_token + (head * a.share + j) * a.out_head + d);
          to[0] = __floats2bfloat162_rn(x.x * f, x.y * f);
          to[1] = __floats2bfloat162_rn(x.z * f, x.w * f);
        }
      } else {
        *reinterpret_cast<float2*>(slot + r * D + d) = make_float2(x.x, x.y);
        *reinterpret_cast<float2*>(slot + r * D + d + 2) = make_float2(x.z, x.w);
      }
    }
    if (!whole && threadIdx.x < live) *reinterpret_cast<float2*>(slot + Q * D + 2 * threadIdx.x) = total_ml[threadIdx.x];
    if (!whole && c0 == 0) {
      // the unit's last chunk is in the last block whose first chunk is not behind it
      const uint64_t x = uint64_t(first[s]) + uint64_t(unit) * q.chunks + q.chunks;
      mine = ArRecord{s, unit, static_cast<uint32_t>((x * blocks + total - 1) / total - 1), 1u};
    }
    __syncthreads();                                   // the sums are read: the rings may be filled
    at += c1 - c0;
  }
  if (a.parts && threadIdx.x == 0) *record = mine;
}

// Joins the parts of the units that begin in one block and end in another: blockIdx.x has the unit that this record names, blockIdx.y a row
// of it, whose slots the block's warps share (ALONE: four rows, a warp each).
constexpr uint32_t kAjWarps = 4;
template <int D, int NT, bool ALONE>
__global__ void __launch_bounds__(32 * kAjWarps) ans_attend_join_kernel(const AttendArgs a, uint32_t blocks) {
  constexpr uint32_t Q = 8 * NT, kMany = 4, kTogether = D == 256 ? 4 : 8;
  __shared__ float2 found[kAjWarps][32 * kMany];       // {slot's number, weight} of a warp
  __shared__ float2 parts_ml[kAjWarps];
  __shared__ __align__(16) float parts[kAjWarps][D];
  let_next_start();
  wait_for_previous();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const ArRecord rec = reinterpret_cast<const ArRecord*>(a.parts)[blockIdx.x];
  if (!rec.live) return;
  const float* const slots = a.parts + blocks * (sizeof(ArRecord) / 4);
  bool unused = false;
  const ArSeq q = ar_sequence<Q>(a, rec.seq, unused);
  const uint32_t head = rec.unit / q.groups, group = rec.unit - head * q.groups, count = rec.last - blockIdx.x + 1u;
  const uint32_t rows = q.fresh * a.share, r0 = group * Q, live = min(Q, rows - r0);
  auto slot = [&](uint32_t b) { return 2u * (blockIdx.x + b) + (b == 0 ? 1u : 0u); };
  constexpr uint32_t kShare = ALONE ? 1 : kAjWarps;  // warps of a row
  const uint32_t part = ALONE ? 0u : warp;
  for (uint32_t r = ALONE ? blockIdx.y * kAjWarps + warp : blockIdx.y; r < live; r += gridDim.y * (kAjWarps / kShare)) {
    float most = kLowest, all = 0.f, x[D / 32];
#pragma unroll
    for (int k = 0; k < D / 32; ++k) x[k] = 0.f;
    const uint32_t b1 = count * (part + 1u) / kShare;
    for (uint32_t b0 = count * part / kShare; b0 < b1; b0 += 32 * kMany) {
      float2 m[kMany];
#pragma unroll
      for (uint32_t k = 0; k < kMany; ++k) {
        const uint32_t b = b0 + 32u * k + lane;
        m[k] = b < b1 ? *reinterpret_cast<const float2*>(slots + uint64_t(slot(b)) * Q * (D + 2) + Q * D + 2 * r) : make_float2(kLowest, 0.f);
      }
      float top = most;
#pragma unroll
      for (uint32_t k = 0; k < kMany; ++k) top = fmaxf(top, m[k].x);
#pragma unroll
      for (uint32_t step = 1; step < 32; step *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, step));
      const float half = exp2_near(0.5f * (most - top)), shrink = half * half;
      most = top;
      all = all * half * half;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) x[k] *= shrink;
      uint32_t have = 0;
      float own = 0.f;
#pragma unroll
      for (uint32_t k = 0; k < kMany; ++k) {
        const bool some = m[k].y != 0.f;             // a NaN counts
        const uint32_t some_of = __ballot_sync(kAll, some);
        const float half = exp2_near(0.5f * (m[k].x - most));
        if (some) {
          found[warp][have + __popc(some_of & ((1u << lane) - 1u))] = make_float2(__uint_as_float(slot(b0 + 32u * k + lane)), half * half);
          own = fmaf(half, half * m[k].y, own);
        }
        have += __popc(some_of);
      }
#pragma unroll
      for (uint32_t step = 1; step < 32; step *= 2) own += __shfl_xor_sync(kAll, own, step);
      all += own;
      __syncwarp();
      for (uint32_t e = 0; e < have; e += kTogether) {
        float v[kTogether][D / 32], w[kTogether];
#pragma unroll
        for (uint32_t z = 0; z < kTogether; ++z) {
          const float2 of = found[warp][min(e + z, have - 1u)];
          w[z] = of.y;
          const float* const at = slots + uint64_t(__float_as_uint(of.x)) * Q * (D + 2) + r * D + 2 * lane;
#pragma unroll
          for (int k = 0; k < D / 64; ++k) {
            const float2 y = *reinterpret_cast<const float2*>(at + 64 * k);
            v[z][2 * k] = y.x;
            v[z][2 * k + 1] = y.y;
          }
        }
#pragma unroll
        for (uint32_t z = 0; z < kTogether; ++z)
          if (e + z < have)
#pragma unroll
            for (int k = 0; k < D / 32; ++k) x[k] = fmaf(w[z], v[z][k], x[k]);
      }
      __syncwarp();
    }
    const uint32_t row = token_of(a, r0 + r), j = (r0 + r) - row * a.share;
    __nv_bfloat16* const to = a.out + (q.row + row) * a.out_token + (head * a.share + j) * a.out_head;
    if constexpr (ALONE) {
      const float f = all == 0.f ? 0.f : kFromSum / all;
#pragma unroll
      for (int k = 0; k < D / 64; ++k) {
        const uint32_t d = 64u * k + 2u * lane;
        if (d < a.c.dim) *reinterpret_cast<__nv_bfloat162*>(to + d) = __floats2bfloat162_rn(x[2 * k] * f, x[2 * k + 1] * f);
      }
      continue;
    }
    if (lane == 0) parts_ml[warp] = make_float2(most, all);
#pragma unroll
    for (int k = 0; k < D / 64; ++k) *reinterpret_cast<float2*>(&parts[warp][64 * k + 2 * lane]) = make_float2(x[2 * k], x[2 * k + 1]);
    __syncthreads();
    most = kLowest;
    all = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < kAjWarps; ++w) most = fmaxf(most, parts_ml[w].x);
    float f[kAjWarps];
#pragma unroll
    for (uint32_t w = 0; w < kAjWarps; ++w) {
      const float half = exp2_near(0.5f * (parts_ml[w].x - most));
      f[w] = half * half;
      all = fmaf(half, half * parts_ml[w].y, all);
    }
    const float over = all == 0.f ? 0.f : kFromSum / all;
    for (uint32_t d = 2u * threadIdx.x; d < a.c.dim; d += 64 * kAjWarps) {
      float y0 = 0.f, y1 = 0.f;
#pragma unroll
      for (uint32_t w = 0; w < kAjWarps; ++w) {
        y0 = fmaf(f[w], parts[w][d], y0);
        y1 = fmaf(f[w], parts[w][d + 1], y1);
      }
      *reinterpret_cast<__nv_bfloat162*>(to + d) = __floats2bfloat162_rn(y0 * over, y1 * over);
    }
    __syncthreads();
  }
  }

// ---- host side -----------------------------------------------------------------------------
struct ArPlan {
  uint32_t tiles;                                      // queries in eights
  uint32_t blocks;
  bool join;                                           // a unit may lie in several blocks
  uint32_t units, rows;                                // by the caller's numbers: units, rows of a unit
  size_t room;
};

template <int D, int NT>
static void plan_shape(const AttendArgs& a, uint32_t longest, int sms, ArPlan& p) {
  using S = ArShape<D, NT>;
  const uint64_t tokens = uint64_t(a.b.table_pages) * a.c.page_size;
  const uint64_t chunks = std::max<uint64_t>((tokens + kArChunk - 1) / kArChunk, 1);
  const uint64_t groups = (uint64_t(longest) * a.share + S::kQueries - 1) / S::kQueries;
  const uint64_t all = std::min<uint64_t>(chunks, 1u << 20) * a.b.n_seqs * a.c.heads * std::min<uint64_t>(std::max<uint64_t>(groups, 1), 1u << 20);
  p.blocks = static_cast<uint32_t>(std::min<uint64_t>(all, uint64_t(sms) * (D * NT <= 128 ? 2 : 1)));
  p.join = chunks > 1;
  p.tiles = NT;
  p.units = static_cast<uint32_t>(std::min<uint64_t>(groups * a.c.heads * a.b.n_seqs, 1u << 28));
  p.rows = static_cast<uint32_t>(std::min<uint64_t>(uint64_t(longest) * a.share, S::kQueries));
  p.room = p.join ? size_t(p.blocks) * (sizeof(ArRecord) + 2 * S::kQueries * (D + 2) * sizeof(float)) : 0;
}

template <int D, int NT>
static int launch_rows(const AttendArgs& a, const ArPlan& p, cudaStream_t st) {
  using S = ArShape<D, NT>;
  constexpr size_t most = S::kSmem + 4 * (ANS_MAX_SEQS + 1);
  static_assert(most <= 227 * 1024, "");
  const size_t smem = S::kSmem + 4 * (size_t(a.b.n_seqs) + 1);
  int rc;
  if (a.c.dim == D) {
    rc = allow_smem<ans_attend_rows_kernel<D, NT, true>>(most);
    if (rc == ANS_OK) rc = launch(ans_attend_rows_kernel<D, NT, true>, dim3(p.blocks), dim3(kArThreads), smem, st, 1, a);
  } else {
    rc = allow_smem<ans_attend_rows_kernel<D, NT, false>>(most);
    if (rc == ANS_OK) rc = launch(ans_attend_rows_kernel<D, NT, false>, dim3(p.blocks), dim3(kArThreads), smem, st, 1, a);
  }
  if (rc != ANS_OK || !p.join) return rc;
  // a warp a row where units lie in few blocks, up to 8 on average
  rc = p.blocks <= 8 * p.units ? launch(ans_attend_join_kernel<D, NT, true>, dim3(p.blocks, (p.rows + kAjWarps - 1) / kAjWarps), dim3(32 * kAjWarps), 0, st, 1, a, p.blocks)
                               : launch(ans_attend_join_kernel<D, NT, false>, dim3(p.blocks, p.rows), dim3(32 * kAjWarps), 0, st, 1, a, p.blocks);
  return rc;
}

static int check_attend(const ans_block_cache_desc& c, const ans_batch_desc& b, const ans_attend_desc& d, AttendArgs& a) {
  int rc = check_block_cache(c, a.c);
  if (rc == ANS_OK) rc = check_batch(b, a.b);
  if (rc != ANS_OK) return rc;
  if (d.q_heads == 0 || d.q_heads % a.c.heads) return ANS_ERR_INVALID_ARG;
  if (d.q_heads / a.c.heads > 128 || uint64_t(a.b.rows) * (d.q_heads / a.c.heads) > 0x7FFFFFFFull) return ANS_ERR_UNSUPPORTED;
  a.scale2 = static_cast<float>(d.scale * 1.4426950408889634);
  if (!std::isfinite(a.scale2)) return ANS_ERR_INVALID_ARG;
  if (a.b.n_seqs == 0 || a.b.rows == 0) return ANS_OK;
  if (!d.d_q || !d.d_out || (reinterpret_cast<uintptr_t>(d.d_q) & 15) || (reinterpret_cast<uintptr_t>(d.d_out) & 3)) return ANS_ERR_INVALID_ARG;
  if ((d.q_token_stride | d.q_head_stride) & 7 || (d.out_token_stride | d.out_head_stride) & 1) return ANS_ERR_INVALID_ARG;
  constexpr uint64_t kFar = uint64_t(1) << 40;
  if (d.q_token_stride > kFar || d.q_head_stride > kFar || d.out_token_stride > kFar || d.out_head_stride > kFar) return ANS_ERR_UNSUPPORTED;
  a.q = static_cast<const __nv_bfloat16*>(d.d_q); a.out = static_cast<__nv_bfloat16*>(d.d_out);
  a.q_token = d.q_token_stride; a.q_head = d.q_head_stride; a.out_token = d.out_token_stride; a.out_head = d.out_head_stride;
  if (d.d_q == d.d_out && (d.q_token_stride != d.out_token_stride || d.q_head_stride != d.out_head_stride)) return ANS_ERR_INVALID_ARG;
  a.share = d.q_heads / a.c.heads;
  uint32_t bits = 0;
  while ((1u << bits) < a.share) ++bits;
  a.share_shift = 31 + bits;
  a.share_by = static_cast<uint32_t>(((uint64_t(1) << a.share_shift) + a.share - 1) / a.share);
  a.window = std::min<uint32_t>(d.window, 0x7FFFFFFFu);
  a.causal = d.causal != 0;
  a.out_wide = !((reinterpret_cast<uintptr_t>(d.d_out) | (d.out_token_stride | d.out_head_stride) * 2) & 15);
  return ANS_OK;
}

// What a call launches: the kernel of this file for sequences of up to kBorder rows (new tokens x share), the tiles for
// the others; one of them alone where the caller's numbers say that no sequence needs the other.  The two by the rows of a head, us, this kernel
// and the tiles; 16 sequences of 2000 tokens, 64 of 500, one of 16000, 8 heads:
//   D = 64:   16 rows  23  51    28  51    18  25      32 rows   33  53    44  53   23  25      64 rows   55  56    77  58   33  26
//   D = 128:  16 rows  30  64    41  62    21  29      32 rows   49  66    67  63   29  29      64 rows   87  70   128  70   43  31
//   D = 256:  16 rows  58 100    77  99    33  44      32 rows  102 104   140 104   52  44      64 rows  186  86   274 114   87  47
// So 32 is the last number of rows at which this kernel is as fast or nearly so for D = 64 and 128; for D = 256, whose groups have 8 queries, 16 would be.
constexpr uint32_t kBorder = 32;
struct AttendPlan {
  bool with_rows, with_tiles;
  ArPlan rows;
  AtPlan tiles;
  size_t room;
};
template <typename F>
static int for_shape(uint32_t dim, uint32_t tiles, F&& f) {
  if (dim <= 64) return tiles == 1 ? f(std::integral_constant<int, 64>{}, std::integral_constant<int, 1>{}) : f(std::integral_constant<int, 64>{}, std::integral_constant<int, 2>{});
  if (dim <= 128) return tiles == 1 ? f(std::integral_constant<int, 128>{}, std::integral_constant<int, 1>{}) : f(std::integral_constant<int, 128>{}, std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 256>{}, std::integral_constant<int, 1>{});
}
static int plan_attend(const AttendArgs& a, uint32_t longest, AttendPlan& p) {
  int sms = 0;
  int rc = sm_count(&sms);
  if (rc != ANS_OK) return rc;
  if (longest == 0 || longest > a.b.rows) longest = a.b.rows;
  const uint64_t most = uint64_t(longest) * a.share;
  p.with_tiles = most > kBorder;
  p.with_rows = !p.with_tiles || (a.b.n_seqs > 1 && a.share <= kBorder);          // a single token has `share` rows
  // Groups of 8 queries or of 16: 16 queries in one group and in two take, for the sequences above, 23 and 25, 28 and 32, 18 and 17 us (D = 64), 30 and
  // 34, 41 and 45, 21 and 22 (D = 128); 4 queries in a group of 16 and of 8 21 and 17, 25 and 20, 14 and 12; 28 and 24, 37 and 27, 19 and 15.
  if (p.with_rows)                                     // beside the tiles, most others are single tokens
    rc = for_shape(a.c.dim, (p.with_tiles ? a.share : most) <= 8 ? 1 : 2, [&](auto d, auto nt) {
      plan_shape<d(), nt()>(a, p.with_tiles ? std::max(kBorder / a.share, 1u) : longest, sms, p.rows);
      return int(ANS_OK);
    });
  if (p.with_tiles) plan_tiles(a, sms, p.tiles);
  p.room = std::max(p.rows.room, p.tiles.room);        // the two kernels follow each other
  return rc;
}

}  // namespace blk
}  // namespace ansb

using namespace ansb;
using namespace ansb::blk;

ANS_EXPORT int ans_attend_room_bytes(const ans_block_cache_desc* h_cache, const ans_batch_desc* h_batch, const ans_attend_desc* h_desc,
                                     size_t* h_bytes_out) {
  if (!h_cache || !h_batch || !h_desc || !h_bytes_out) return ANS_ERR_INVALID_ARG;
  AttendArgs a{};
  int rc = check_attend(*h_cache, *h_batch, *h_desc, a);
  if (rc != ANS_OK) return rc;
  *h_bytes_out = 0;
  if (a.b.n_seqs == 0 || a.b.rows == 0) return ANS_OK;
  AttendPlan p{};
  rc = plan_attend(a, h_desc->longest, p);
  if (rc == ANS_OK) *h_bytes_out = p.room;
  return rc;
}

ANS_EXPORT int ans_attend(const ans_block_cache_desc* h_cache, const ans_batch_desc* h_batch, const ans_attend_desc* h_desc, uint32_t* d_status,
                          void* stream) {
  ApiRange range("ans_attend");
  if (!h_cache || !h_batch || !h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  AttendArgs a{};
  int rc = check_attend(*h_cache, *h_batch, *h_desc, a);
  if (rc != ANS_OK || a.b.n_seqs == 0 || a.b.rows == 0) return rc;
  a.status = d_status;
  AttendPlan p{};
  rc = plan_attend(a, h_desc->longest, p);
  if (rc != ANS_OK) return rc;
  if (p.room) {
    if (!h_desc->d_room || h_desc->room_bytes < p.room) return ANS_ERR_BUFFER_TOO_SMALL;
    if (reinterpret_cast<uintptr_t>(h_desc->d_room) & 15) return ANS_ERR_INVALID_ARG;
    a.parts = static_cast<float*>(h_desc->d_room);
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (p.with_tiles) {
    a.least = p.with_rows ? kBorder + 1 : 1;
    a.most = 0xFFFFFFFFu;
    rc = launch_tiles(a, p.tiles, st);
    if (rc != ANS_OK || !p.with_rows) return rc;
  }
  a.least = 1;
  a.most = p.with_tiles ? kBorder : 0xFFFFFFFFu;
  return for_shape(a.c.dim, p.rows.tiles, [&](auto d, auto nt) { return launch_rows<d(), nt()>(a, p.rows, st); });
}
