// Barriers in shared memory that count arrivals and bytes, and stores to the
// shared memory of another block of the cluster that count as bytes there.
#pragma once

#include "internal.cuh"

#ifdef __CUDACC__
namespace adapm {
namespace {

__device__ __forceinline__ uint32_t shared_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Nanoseconds that a try may sleep: a warp that polls takes issue slots from those that work.
constexpr uint32_t kPatience = 100000;
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(kPatience)
      : "memory");
  return done != 0;
}
__device__ __forceinline__ uint64_t now_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}
// Waits for a phase of a barrier, two seconds at most; false: it gave up.
// nap: nanoseconds of sleep between tries, for those that need not be the first to know.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t nap = 0) {
  if (barrier_try(bar, parity)) return true;
  const uint64_t start = now_ns();
  for (uint32_t i = 1;; ++i) {
    if (nap > 0) __nanosleep(nap);
    if (barrier_try(bar, parity)) return true;
    if ((i & 15u) == 0u && now_ns() - start > 2000000000ull) return false;
  }
}

// The address of the same place in block `rank` of the cluster.
__device__ __forceinline__ uint32_t shared_of(uint32_t at, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
  return r;
}
// 16 bytes to another block's shared memory; they count at a barrier there.
// Unlike a store and a cluster barrier behind it, this waits for no earlier store.
__device__ __forceinline__ void store_and_count(uint32_t at, float4 v, uint32_t bar) {
  asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(at),
               "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(bar)
               : "memory");
}

}  // namespace
}  // namespace adapm
#endif
