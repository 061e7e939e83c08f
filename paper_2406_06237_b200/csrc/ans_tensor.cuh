// What the kernels on matrices share: mbarriers with bounded waits, TMA tiles, tcgen05, small numerics.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <atomic>
#include <utility>

#include "ans_common.cuh"

namespace ansb {
namespace ten {

constexpr uint32_t kAll = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t smem_addr(const void* p) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// ---- launches that overlap their ends ------------------------------------------------------
// Every kernel lets the next one on its stream be set up while it runs, and touches no global memory
// before the work queued ahead of it is complete, but for weights that the caller calls settled.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// What a launch needs to know of the current device, asked once: both are properties of the device or of the kernel on
// it for as long as the process lives.
constexpr int kDevices = 64;
inline int sm_count(int* sms) {
  static std::atomic<int> known[kDevices];
  int dev = 0;
  ANSB_CUDA(cudaGetDevice(&dev));
  const bool keep = dev >= 0 && dev < kDevices;
  if (keep && (*sms = known[dev].load(std::memory_order_relaxed)) > 0) return ANS_OK;
  ANSB_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
  if (keep) known[dev].store(*sms, std::memory_order_relaxed);
  return ANS_OK;
}
template <auto KERNEL>
inline int allow_smem(size_t most) {
  static std::atomic<bool> done[kDevices];
  int dev = 0;
  ANSB_CUDA(cudaGetDevice(&dev));
  const bool keep = dev >= 0 && dev < kDevices;
  if (keep && done[dev].load(std::memory_order_relaxed)) return ANS_OK;
  ANSB_CUDA(cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most)));
  if (keep) done[dev].store(true, std::memory_order_relaxed);
  return ANS_OK;
}

template <typename... P, typename... A>
inline int launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, uint32_t cluster, A&&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, std::forward<A>(args)...);
  return e == cudaSuccess ? ANS_OK : cuda_fail(e);
}

// ---- mbarriers ---------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_init_fence() {
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// arrive on the barrier at the same offset in CTA `rank` of the cluster
__device__ __forceinline__ void bar_arrive_at(uint32_t bar, uint32_t rank) {
  asm volatile(
      "{\n\t.reg .b32 r;\n\t"
      "mapa.shared::cluster.u32 r, %0, %1;\n\t"
      "mbarrier.arrive.release.cluster.shared::cluster.b64 _, [r];\n\t}"
      :: "r"(bar), "r"(rank) : "memory");
}
// A wait with a limit of about 0.1 s; `bad` is set when it runs out, and a thread whose `bad` is set
// looks only once from then on, so that a broken run ends soon.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, uint32_t& bad) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  if (done) return true;
  const long long t0 = clock64();
  for (;;) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity), "r"(20000u) : "memory");   // asleep for up to 20 us
    if (done) return true;
    if (bad || clock64() - t0 > 200000000ll) { bad = 1; return false; }
  }
}

// ---- two floats at a time ------------------------------------------------------------------
using Two = unsigned long long;
__device__ __forceinline__ Two two(float a, float b) {
  Two r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float low(Two v) { return __uint_as_float(static_cast<uint32_t>(v)); }
__device__ __forceinline__ float high(Two v) { return __uint_as_float(static_cast<uint32_t>(v >> 32)); }
__device__ __forceinline__ Two add2(Two a, Two b) {
  Two r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
  Two r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
  Two r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
// the largest magnitude, NaN above all
__device__ __forceinline__ float larger(float top, Two v) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(top), "f"(low(v)), "f"(high(v)));
  return r;
}

// ---- clusters ----------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// the two halves of cluster_sync
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// ---- TMA: a box of 128 bytes x rows from a row-major matrix, 128-byte swizzle ---------------
// PAIR: the bytes are counted on the barrier of the CTA pair's first CTA.
template <bool PAIR>
__device__ __forceinline__ void tile_load(uint32_t dst, const void* map, uint32_t bar, uint32_t x, uint32_t y) {
  if constexpr (PAIR)
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        :: "r"(dst), "l"(map), "r"(bar & 0xFEFFFFFFu), "r"(x), "r"(y) : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        :: "r"(dst), "l"(map), "r"(bar), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void map_prefetch(const void* map) {
  asm volatile("prefetch.tensormap [%0];" :: "l"(map) : "memory");
}

// ---- tcgen05 -----------------------------------------------------------------------------
// shared-memory operand descriptor of a K-major tile of 128-byte rows with the 128-byte swizzle:
// 8-row groups 1024 bytes apart
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
  return uint64_t((addr & 0x3FFFFu) >> 4) | (uint64_t(1) << 16) | (uint64_t(1024 >> 4) << 32) |
         (uint64_t(1) << 46) | (uint64_t(2) << 61);
}
// instruction descriptor: D in 32 bits, both operands K-major; bf16 (kind::f16) or e4m3 (kind::f8f6f4)
template <bool F8>
__host__ __device__ constexpr uint32_t instruction(uint32_t m, uint32_t n) {
  return (1u << 4) | (F8 ? 0u : (1u << 7) | (1u << 10)) | ((n >> 3) << 17) | ((m >> 4) << 24);
}
// D += A B.  REUSE: 0: A is read for this instruction alone; 1: and kept for the next one; 2: the kept A is used, the last time
#define ANSB_MMA(GROUP, KIND, COLLECT)                                                                    \
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"                                          \
               "tcgen05.mma.cta_group::" GROUP ".kind::" KIND COLLECT " [%0], %1, %2, %3, p;\n\t}"        \
               :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory")
template <uint32_t CG, bool F8, int REUSE = 0>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CG == 1) {
    static_assert(REUSE == 0, "");
    if constexpr (F8) ANSB_MMA("1", "f8f6f4", ""); else ANSB_MMA("1", "f16", "");
  } else if constexpr (REUSE == 0) {
    if constexpr (F8) ANSB_MMA("2", "f8f6f4", ""); else ANSB_MMA("2", "f16", "");
  } else if constexpr (REUSE == 1) {
    if constexpr (F8) ANSB_MMA("2", "f8f6f4", ".collector::a::fill"); else ANSB_MMA("2", "f16", ".collector::a::fill");
  } else {
    if constexpr (F8) ANSB_MMA("2", "f8f6f4", ".collector::a::lastuse"); else ANSB_MMA("2", "f16", ".collector::a::lastuse");
  }
}
#undef ANSB_MMA
// arrive on `bar` (CG = 2: on it in both CTAs of the pair) when the matrix instructions issued so far are done
template <uint32_t CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
  else
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
        :: "r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
}
template <uint32_t CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols) {
  if constexpr (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <uint32_t CG>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t cols) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(cols) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 16 or 32 columns of this warp's 32 lanes; the values are there after tmem_wait()
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
               "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
                 "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
                 "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
               : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

}  // namespace ten
}  // namespace ansb
