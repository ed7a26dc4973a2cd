// Barriers in shared memory, and the copies that they count.
#pragma once
#include <cstdint>

#include <cuda.h>
#include <cuda_runtime.h>

namespace lba {

// cuTensorMapEncodeTiled, asked for once; null where the driver has none
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled tensor_map_encoder() {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return (EncodeTiled)f;
  }();
  return fn;
}

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void mbar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
// true in one lane of a converged warp; the compiler then knows that operands of what follows are the same for all active lanes, where
// a lane chosen by its number had each copy cost some hundred clocks of issue
__device__ __forceinline__ bool elected() {
  uint32_t d;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(d));
  return d;
}
// announces bytes; the first form also arrives
__device__ __forceinline__ void mbar_arrive_expect(uint32_t bar, int bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, int bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Every wait ends: after WAIT_LIMIT, or soon where `dead` says that another of the CTA's has run out; then `dead` is set.  The clock is looked
// at once in 64 tries, each of which may take its time.
constexpr uint64_t WAIT_LIMIT = 10000000000ull;  // ns
__device__ __forceinline__ uint64_t wall_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
template <typename Try>
__device__ __forceinline__ bool wait_until(Try there, volatile int* dead) {
  uint64_t end = 0;
  for (uint32_t i = 1;; ++i) {
    if (there()) return true;
    if (i & 63) continue;
    const uint64_t now = wall_ns();
    if (end == 0) end = now + WAIT_LIMIT;
    if (*dead) return false;
    if (now >= end) {
      *dead = 1;
      return false;
    }
  }
}
// Waits for the phase of the given parity.  Returns whether it ended.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {
  return wait_until([&] {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
  }, dead);
}
// the same for a barrier that the other CTA of a cluster arrives at too
__device__ __forceinline__ bool mbar_wait_cluster(uint32_t bar, uint32_t parity, volatile int* dead) {
  return wait_until([&] {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
        : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
  }, dead);
}
// Where a wait ran out, copies may still be on their way into the CTA's shared memory, which the next CTA on this SM gets: they land
// within microseconds, and nothing counts them any more.
__device__ __forceinline__ void let_copies_land() {
#pragma unroll 1
  for (int i = 0; i < 10000; ++i) __nanosleep(1000);
}
// one box of a two-dimensional tensor map
__device__ __forceinline__ void tensor_load(uint32_t dst, const void* map, int x, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

}  // namespace lba
