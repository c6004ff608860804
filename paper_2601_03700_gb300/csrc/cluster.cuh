// Thread-block clusters: rank, barrier, stores to and loads from the other CTAs' shared memory, the launch.
#pragma once
#include "common.cuh"

#include <atomic>

namespace adept {

__device__ __forceinline__ int cluster_rank() {
  int r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ int cluster_size() {
  int n;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
  return n;
}
// All threads of the cluster, converged warps; orders their global and shared memory accesses.
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The same in two halves.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_map(const void* p, int rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  return a;
}
// *p of the cluster's CTA `rank` = v.
__device__ __forceinline__ void cluster_store(int* p, int rank, int v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(cluster_map(p, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_store(long long* p, int rank, long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_map(p, rank)), "l"(v) : "memory");
}

// Lets a kernel run in clusters of 16, once per device (Tag: a type of the kernel's own).
template <typename Tag, typename K>
inline cudaError_t cluster16_once(K* kernel) {
  static std::atomic<unsigned long long> done{0};   // bit per device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev < 64 ? 1ull << dev : 0;
  if (bit && (done.load() & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e == cudaSuccess) done.fetch_or(bit);
  return e;
}

// Clusters of `ctas` CTAs of a kernel (no dynamic shared memory) that an idle GPU holds at once, 0 where not one or where that cannot be
// told; asked for once per device (Tag: a type of the kernel's own; ctas: a power of two up to 16).
template <typename Tag, typename K>
inline int clusters_at_once(K* kernel, int ctas, int threads) {
  static std::atomic<int> known[64][5];   // one more than there are; 0: not asked yet
  int at = 0, dev = 0;
  while (1 << at < ctas) ++at;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  int n = dev < 64 ? known[dev][at].load() : 0;
  if (n > 0) return n - 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3((unsigned)threads);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)ctas;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;   // (not kept: it may have been for a moment)
  }
  if (n < 0) n = 0;
  if (dev < 64) known[dev][at].store(n + 1);
  return n;
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, int cluster, int block, size_t smem, cudaStream_t st, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = g_pdl ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
}

}  // namespace adept
