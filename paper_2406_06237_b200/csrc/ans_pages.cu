// Block tables, slot maps and row ranges of a batch from its requests' lengths.
//
// With b_s = cached, m_s = new tokens and P the page size, request s lacks w_s = ceil((b_s + m_s) / P) - ceil(b_s / P) pages;
// its rows start at sum_{r<s} m_r and its new pages at sum_{r<s} w_r of the free list.  Three sums over the requests, then every
// row and every page finds its request in them.  A token's page is known without the table being written first:
// it is either one that the request had or an entry of the free list.
//
// Each block makes the sums by itself (they are what a row's search needs, in shared memory) and takes a part of the rows and of the
// pages.  Where lengths lie over cached, or taken over taken, something has to stand between the last read of the requests'
// numbers and the first write: the blocks are then one cluster of up to 8 with its barrier; no workspace, no second launch.  A small
// call is bound by latency (3.1 us: launch, one trip for the numbers, the sums, one trip for the pages, the stores), and so is a large one: two
// trips of the sums, ten steps of the search, the pages (158 thousand rows of 700 requests 5.8 us on all SMs, 36 % of the issue slots used;
// in place 36, as eight SMs do the work).
#include <algorithm>
#include <initializer_list>

#include "ans_tensor.cuh"

namespace ansb {

using namespace ten;

constexpr uint32_t kPgThreads = 512, kPgAhead = 8;   // rows of a thread whose pages are asked for together
constexpr uint32_t kPgMost = 0x7FFFFFFFu;              // sums stop here, which no batch that fits reaches

// sums that stop at kPgMost: associative for numbers up to it
__device__ __forceinline__ uint32_t plus(uint32_t a, uint32_t b) { return min(a + b, kPgMost); }

// the last s with sums[s] <= at, given that sums[0] <= at < sums[n]
__device__ __forceinline__ uint32_t place_in(const uint32_t* sums, uint32_t n, uint32_t at) {
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (sums[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

// x / page_size = x * by >> shift, x < 2^31: exact with k the bits of page_size - 1, by = ceil(2^(31 + k) / page_size), shift = 31 + k
struct PgDivide { uint32_t by, shift; };

__global__ void __launch_bounds__(kPgThreads) ans_page_tables_kernel(const ans_pages_desc d, const PgDivide p, const uint32_t together, uint32_t* status) {
  extern __shared__ uint32_t smem[];
  uint32_t* const rows = smem;                         // [n + 1] sums of new tokens
  uint32_t* const more = rows + d.n_seqs + 1;          // [n + 1] sums of new pages
  uint32_t* const had = more + d.n_seqs + 1;           // [n] cached tokens
  __shared__ uint32_t part[3][kPgThreads / 32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, n = d.n_seqs;
  const uint32_t blocks = gridDim.x, rank = blockIdx.x;
  auto pages_of = [&](uint32_t x) { return static_cast<uint32_t>(uint64_t(x) * p.by >> p.shift); };          // whole ones
  auto pages_for = [&](uint32_t x) { const uint32_t n = pages_of(x); return n + (n * d.page_size != x ? 1u : 0u); };
  let_next_start();
  wait_for_previous();

  const int32_t taken0 = *d.d_taken;
  uint32_t base[3] = {0, 0, 0};                        // new tokens, new pages, tokens of the requests before
  bool bad = taken0 < 0 || static_cast<uint32_t>(taken0) > d.n_free;
  // Lengths and their sums are kept by the thread that made them until all blocks have read (one trip of the loop: the
  // usual case), else made again behind the barrier.
  uint32_t my_cached = 0, my_end = 0;
  for (uint32_t s0 = 0; s0 < n; s0 += kPgThreads) {
    const uint32_t s = s0 + threadIdx.x;
    uint32_t v[3] = {0, 0, 0}, cached = 0;
    if (s < n) {
      const int32_t c = d.d_cached[s], m = d.d_new[s];
      const uint32_t b = max(c, 0), a = plus(b, max(m, 0));
      const uint32_t held = pages_for(b), need = pages_for(a);
      bad |= c < 0 || m < 0 || a == kPgMost || need > d.table_pages;
      v[0] = max(m, 0);
      v[1] = need - held;
      v[2] = a;
      cached = b;
    }
    uint32_t x[3] = {v[0], v[1], v[2]};
#pragma unroll
    for (uint32_t step = 1; step < 32; step *= 2) {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const uint32_t from = __shfl_up_sync(kAll, x[k], step);
        if (lane >= step) x[k] = plus(x[k], from);
      }
    }
    if (lane == 31) { part[0][warp] = x[0]; part[1][warp] = x[1]; part[2][warp] = x[2]; }
    __syncthreads();
    uint32_t before[3], all[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {                      // every warp sums the warps' totals by itself
      uint32_t t = lane < kPgThreads / 32 ? part[k][lane] : 0u;
#pragma unroll
      for (uint32_t step = 1; step < kPgThreads / 32; step *= 2) {
        const uint32_t from = __shfl_up_sync(kAll, t, step);
        if (lane >= step) t = plus(t, from);
      }
      all[k] = __shfl_sync(kAll, t, kPgThreads / 32 - 1);
      before[k] = __shfl_sync(kAll, t, (warp - 1u) & 31u);
      if (warp == 0) before[k] = 0;
      before[k] = plus(before[k], base[k]);
      base[k] = plus(base[k], all[k]);
      x[k] = plus(x[k], before[k]);                    // with this request
    }
    if (s < n) { rows[s + 1] = x[0]; more[s + 1] = x[1]; had[s] = cached; }
    my_cached = cached;
    my_end = x[2];
    __syncthreads();
  }
  if (threadIdx.x == 0) rows[0] = more[0] = 0;
  const uint32_t total = base[0], pages = base[1];
  bad |= total > d.rows || base[2] == kPgMost || (!bad && pages > d.n_free - static_cast<uint32_t>(taken0));
  bad = __syncthreads_or(bad);
  // A request's own numbers are read again below; what overwrites them waits for the other blocks.
  const int32_t* const free_from = d.d_free + taken0;

  // rows: a warp takes 32 at a time, kPgAhead times together, and moves on in the sums from the request of the last ones
  const uint32_t warps = blocks * (kPgThreads / 32), each = (d.rows + 32 * warps - 1) / (32 * warps) * 32;
  const uint64_t r0 = uint64_t(rank * (kPgThreads / 32) + warp) * each, r1 = min(r0 + each, uint64_t(d.rows));
  uint32_t s = 0;
  for (uint64_t at = r0 + lane; at < r1; at += 32 * kPgAhead) {
    int32_t page[kPgAhead];
    uint32_t in[kPgAhead], position[kPgAhead];
    bool live[kPgAhead];
#pragma unroll
    for (uint32_t k = 0; k < kPgAhead; ++k) {
      const uint64_t mine = at + 32 * k;
      const uint32_t row = static_cast<uint32_t>(mine);
      live[k] = !bad && mine < r1 && row < total;
      page[k] = -1;
      in[k] = position[k] = 0;
      if (live[k]) {
        if (mine < r0 + 32) s = place_in(rows, n, row);
        else while (rows[s + 1] <= row) ++s;
        const uint32_t c = had[s], pos = c + (row - rows[s]), number = pages_of(pos), held = pages_for(c);
        page[k] = number < held ? d.d_tables[s * d.table_stride + number] : free_from[more[s] + (number - held)];
        in[k] = pos - number * d.page_size;
        position[k] = pos;
      }
    }
#pragma unroll
    for (uint32_t k = 0; k < kPgAhead; ++k) {
      const uint64_t mine = at + 32 * k;
      if (mine >= r1) break;
      int64_t slot = int64_t(page[k]) * d.page_size + in[k];
      if (page[k] < 0 || slot > int64_t(kPgMost)) {
        slot = -1;
        if (live[k]) atomicOr(status, ANS_STATUS_BAD_PAGE);
      }
      d.d_slots[mine] = slot;
      d.d_positions[mine] = static_cast<int32_t>(position[k]);
    }
  }
  // pages
  if (!bad) {
    uint32_t q = 0;
    bool first = true;
    for (uint32_t at = rank * kPgThreads + threadIdx.x; at < pages; at += blocks * kPgThreads) {
      if (first) q = place_in(more, n, at);
      else while (more[q + 1] <= at) ++q;
      first = false;
      const uint32_t held = pages_for(had[q]);
      d.d_tables[q * d.table_stride + held + (at - more[q])] = free_from[at];
    }
  }
  if (together) cluster_sync(); else __syncthreads();                // nobody reads what is written below any more

  if (rank == 0) {
    if (n <= kPgThreads && !bad) {
      if (threadIdx.x < n) {
        const uint32_t t = threadIdx.x;
        d.d_starts[t + 1] = static_cast<int32_t>(rows[t + 1]);
        d.d_lengths[t] = static_cast<int32_t>(my_cached + (rows[t + 1] - rows[t]));
        d.d_ends[t + 1] = static_cast<int32_t>(my_end);
      }
      if (threadIdx.x == 0) { d.d_starts[0] = 0; d.d_ends[0] = 0; }
    } else {
      if (threadIdx.x == 0) { d.d_starts[0] = 0; d.d_ends[0] = 0; }
      uint32_t end = 0;
      for (uint32_t s0 = 0; s0 < n; s0 += kPgThreads) {
        const uint32_t t = s0 + threadIdx.x;
        uint32_t length = 0;
        if (t < n) length = plus(max(d.d_cached[t], 0), bad ? 0u : rows[t + 1] - rows[t]);
        uint32_t x = length;
#pragma unroll
        for (uint32_t step = 1; step < 32; step *= 2) {
          const uint32_t from = __shfl_up_sync(kAll, x, step);
          if (lane >= step) x = plus(x, from);
        }
        if (lane == 31) part[0][warp] = x;
        __syncthreads();
        uint32_t sum = lane < kPgThreads / 32 ? part[0][lane] : 0u;
#pragma unroll
        for (uint32_t step = 1; step < kPgThreads / 32; step *= 2) {
          const uint32_t from = __shfl_up_sync(kAll, sum, step);
          if (lane >= step) sum = plus(sum, from);
        }
        const uint32_t all = __shfl_sync(kAll, sum, kPgThreads / 32 - 1);
        uint32_t before = __shfl_sync(kAll, sum, (warp - 1u) & 31u);
        if (warp == 0) before = 0;
        if (t < n) {
          // a negative number of cached tokens stays as it is where the batch is refused
          d.d_lengths[t] = bad ? d.d_cached[t] : static_cast<int32_t>(length);
          d.d_starts[t + 1] = bad ? 0 : static_cast<int32_t>(rows[t + 1]);
          d.d_ends[t + 1] = static_cast<int32_t>(plus(plus(end, before), x));
        }
        end = plus(end, all);
        __syncthreads();
      }
    }
    if (threadIdx.x == 0) {
      *d.d_taken_out = bad ? taken0 : static_cast<int32_t>(taken0 + pages);
      if (bad) atomicOr(status, ANS_STATUS_BAD_PAGE);
    }
  }
}

}  // namespace ansb

using namespace ansb;

ANS_EXPORT int ans_page_tables(const ans_pages_desc* h_desc, uint32_t* d_status, void* stream) {
  ApiRange range("ans_page_tables");
  if (!h_desc || !d_status) return ANS_ERR_INVALID_ARG;
  const ans_pages_desc& d = *h_desc;
  if (d.page_size == 0) return ANS_ERR_INVALID_ARG;
  if (d.n_seqs > ANS_MAX_SEQS || d.page_size > (1u << 20) || d.rows > kPgMost || d.n_free > kPgMost || d.table_pages > kPgMost ||
      d.table_stride > (uint64_t(1) << 40))
    return ANS_ERR_UNSUPPORTED;
  if (d.n_seqs && (!d.d_cached || !d.d_new || !d.d_lengths || (!d.d_tables && d.table_pages) || (!d.d_free && d.n_free))) return ANS_ERR_INVALID_ARG;
  if (!d.d_taken || !d.d_taken_out || !d.d_starts || !d.d_ends || (d.rows && (!d.d_slots || !d.d_positions))) return ANS_ERR_INVALID_ARG;
  if (d.n_seqs > 1 && d.table_stride < d.table_pages) return ANS_ERR_INVALID_ARG;
  for (const void* p : {static_cast<const void*>(d.d_cached), static_cast<const void*>(d.d_new), static_cast<const void*>(d.d_free),
                        static_cast<const void*>(d.d_taken), static_cast<const void*>(d.d_tables), static_cast<const void*>(d.d_starts),
                        static_cast<const void*>(d.d_lengths), static_cast<const void*>(d.d_ends), static_cast<const void*>(d.d_positions),
                        static_cast<const void*>(d.d_taken_out)})
    if (reinterpret_cast<uintptr_t>(p) & 3) return ANS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(d.d_slots) & 7) return ANS_ERR_INVALID_ARG;
  uint32_t bits = 0;
  while ((1u << bits) < d.page_size) ++bits;
  const PgDivide p{static_cast<uint32_t>(((uint64_t(1) << (31 + bits)) + d.page_size - 1) / d.page_size), 31 + bits};
  int sms = 0;
  const int asked = sm_count(&sms);
  if (asked != ANS_OK) return asked;
  const bool over = d.d_lengths == d.d_cached || d.d_taken_out == d.d_taken;
  const uint64_t work = std::max<uint64_t>(d.rows, d.n_seqs) / (2 * kPgThreads);
  uint32_t blocks = static_cast<uint32_t>(std::min<uint64_t>(std::max<uint64_t>(work, 1), sms));
  if (over) blocks = blocks < 2 ? 1 : blocks < 4 ? 2 : blocks < 8 ? 4 : 8;
  const size_t smem = 3 * (size_t(d.n_seqs) + 1) * sizeof(uint32_t);
  const int rc = allow_smem<ans_page_tables_kernel>(3 * (ANS_MAX_SEQS + 1) * sizeof(uint32_t));
  if (rc != ANS_OK) return rc;
  return launch(ans_page_tables_kernel, dim3(blocks), dim3(kPgThreads), smem, static_cast<cudaStream_t>(stream), over ? blocks : 1, d, p, over && blocks > 1 ? 1u : 0u, d_status);
}
