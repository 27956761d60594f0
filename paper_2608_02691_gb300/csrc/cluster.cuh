// Thread-block clusters: rank, barrier, loads from another CTA's shared memory.
#pragma once

#include <stdint.h>

namespace optr {

__device__ __forceinline__ int cluster_rank_of() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}

__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// All threads of the cluster's CTAs.
__device__ __forceinline__ void cluster_barrier() {
  cluster_arrive();
  cluster_wait();
}

// The word at x (this CTA's shared memory) of the CTA of that rank.
__device__ __forceinline__ uint32_t cluster_ld32(const void* x, int rank) {
  uint32_t v;
  asm volatile("{\n .reg .u32 r;\n mapa.shared::cluster.u32 r, %1, %2;\n"
               " ld.shared::cluster.u32 %0, [r];\n}\n"
               : "=r"(v) : "r"((uint32_t)__cvta_generic_to_shared(x)), "r"(rank) : "memory");
  return v;
}
__device__ __forceinline__ unsigned long long cluster_ld64(const void* x, int rank) {
  unsigned long long v;
  asm volatile("{\n .reg .u32 r;\n mapa.shared::cluster.u32 r, %1, %2;\n"
               " ld.shared::cluster.u64 %0, [r];\n}\n"
               : "=l"(v) : "r"((uint32_t)__cvta_generic_to_shared(x)), "r"(rank) : "memory");
  return v;
}

}  // namespace optr
