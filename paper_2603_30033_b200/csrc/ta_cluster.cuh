// Exchange between the CTAs of a cluster through distributed shared memory.
//
// A receiver's mbarrier is told once how many bytes an exchange will bring (expect_tx) before the cluster's start
// barrier; senders store with st.async, whose bytes complete on that mbarrier, and the receiver waits for its phase 0.
// That is one way through the cluster and no fence, where a cluster barrier costs the fence over all remote stores and
// a round of arrivals (join kernel of the paged step, cluster barriers against this: one-pool step 32.7 -> 32.1 us,
// long batch 142.0 -> 141.5, document 87.6 -> 87.3, system prompt 45.9 -> 46.1).  Each buffer and mbarrier is used once
// per launch.  A CTA may leave when it has received everything that is sent to it (stay_for, where a wait ran out).
#pragma once

#include "ta_common.cuh"
#include "ta_sm100.cuh"

namespace ta {
namespace cluster {

__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
using sm100::smem_u32;
__device__ __forceinline__ uint32_t map_rank(const void* own, uint32_t rank) {      // `own`'s counterpart in CTA `rank`
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(own)), "r"(rank));
  return a;
}
// Sends values to the counterpart of `own` in CTA `rank`; their bytes complete on that CTA's barrier.
__device__ __forceinline__ void send(const float* own, uint32_t rank, uint64_t* bar, float v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.f32 [%0], %1, [%2];"
               ::"r"(map_rank(own, rank)), "f"(v), "r"(map_rank(bar, rank)) : "memory");
}
__device__ __forceinline__ void send2(const float* own, uint32_t rank, uint64_t* bar, float2 v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];"
               ::"r"(map_rank(own, rank)), "f"(v.x), "f"(v.y), "r"(map_rank(bar, rank)) : "memory");
}
__device__ __forceinline__ void send4(const float* own, uint32_t rank, uint64_t* bar, float4 v) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
               ::"r"(map_rank(own, rank)), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w), "r"(map_rank(bar, rank)) : "memory");
}
__device__ __forceinline__ bool received_now(uint64_t* bar) {
  uint32_t ok;
  asm volatile(
      "{\n"
      ".reg .pred p;\n"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], 0;\n"
      "selp.u32 %0, 1, 0, p;\n"
      "}\n"
      : "=r"(ok)
      : "r"(smem_u32(bar))
      : "memory");
  return ok != 0;
}
// Waits for everything that one exchange sends to this CTA.  Bounded: a wait that runs out is flagged and returns
// false, and the CTA goes on (every CTA sends whatever happens, so that no other one is left waiting), its result void.
__device__ __forceinline__ bool received(uint64_t* bar, unsigned int* err, long long budget_cycles = sm100::kWaitBudgetCycles) {
  if (received_now(bar)) return true;
  const long long t0 = clock64();
  while (!received_now(bar))
    if (clock64() - t0 > budget_cycles) {
      atomicOr(err, (unsigned)TA_DEVERR_WAIT_TIMEOUT);
      return false;
    }
  return true;
}
// For a thread whose wait ran out, before it ends: it stays, and its CTA's shared memory with it, until the late bytes
// have come, so that nothing is stored to a CTA that has gone.  They do come: a sender sends after sitting out its own
// waits, of which it has a few.
__device__ __forceinline__ void stay_for(uint64_t* bar) {
  const long long t0 = clock64();
  while (!received_now(bar) && clock64() - t0 < 8 * sm100::kWaitBudgetCycles) {}
}
}  // namespace cluster
}  // namespace ta
