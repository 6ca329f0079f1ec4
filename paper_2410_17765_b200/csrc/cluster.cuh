// Rows shared out over the blocks of a thread-block cluster: their barrier, and one another's shared memory.
#pragma once
#include <cstdint>

#include "ptx.cuh"

namespace cpmtp {
namespace cluster {

typedef unsigned long long u64;
constexpr int kMostCtas = 8;

// Shared memory of another block may be touched once that block has begun.  A kernel whose first access to it has no barrier of the cluster before it
// tells the others that it is there, does what it can alone, and waits for them before that access.
__device__ __forceinline__ void tell_begun(int ctas) {
  if (ctas > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void await_begun(int ctas) {
  if (ctas > 1) {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}
__device__ __forceinline__ void sync_row(int ctas) {
  if (ctas == 1) {
    __syncthreads();
  } else {
    __syncwarp();                                             // (a warp arrives as a whole)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
}
// The address in block `cta` of the cluster of what `p` is here.
__device__ __forceinline__ uint32_t remote(const void* p, int cta) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(ptx::smem_u32(p)), "r"(cta));
  return r;
}
__device__ __forceinline__ void store_remote(const void* p, int cta, u64 v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(remote(p, cta)), "l"(v) : "memory");
}
__device__ __forceinline__ u64 load_remote64(const void* p, int cta) {
  u64 v;
  asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(remote(p, cta)) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t load_remote32(const void* p, int cta) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote(p, cta)) : "memory");
  return v;
}

// Unsigned keys in the order of fp32 numbers.
__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);     // (-0 as +0)
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

}  // namespace cluster
}  // namespace cpmtp
