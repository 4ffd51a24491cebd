// CTAs of a cluster: their barrier, and what one writes in another's shared memory.
#pragma once

#include "gar_device.cuh"

namespace gar {

__device__ __forceinline__ int cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}
// All threads of all CTAs; what they have written, also to global memory, is seen after the wait.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() { cluster_arrive(), cluster_wait(); }

// The address of CTA `rank`'s own p.
__device__ __forceinline__ uint32_t in_cta(const void *p, int rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return r;
}
__device__ __forceinline__ void store_in_cta(int *p, int rank, int x) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(in_cta(p, rank)), "r"(x) : "memory");
}
__device__ __forceinline__ void store_in_cta(float2 *p, int rank, float2 x) {
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(in_cta(p, rank)), "f"(x.x), "f"(x.y) : "memory");
}
__device__ __forceinline__ int load_from_cta(const int *p, int rank) {
  int x;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(in_cta(p, rank)) : "memory");
  return x;
}

// launch() in clusters of `ctas` CTAs.
template <typename... P, typename... A>
int launch_clusters(const char *what, void (*kernel)(P...), int64_t blocks, int ctas, int threads, gar_stream_t stream,
                    const A &...args) {
  cudaLaunchAttribute attribute[2]{};
  attribute[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attribute[0].val.programmaticStreamSerializationAllowed = 1;
  attribute[1].id = cudaLaunchAttributeClusterDimension;
  attribute[1].val.clusterDim.x = (unsigned)ctas, attribute[1].val.clusterDim.y = attribute[1].val.clusterDim.z = 1;
  cudaLaunchConfig_t config{};
  config.gridDim = dim3((unsigned)blocks), config.blockDim = dim3((unsigned)threads);
  config.stream = (cudaStream_t)stream, config.attrs = attribute, config.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&config, kernel, args...);
  return e == cudaSuccess ? (int)GAR_OK : cuda_fail(e, what);
}

}  // namespace gar
