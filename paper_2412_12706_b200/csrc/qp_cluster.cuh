// Host side of the kernels that choose their cluster size by what fits on the device.
#pragma once

#include <mutex>

#include "qp_common.cuh"

namespace qp {

// What a kernel needs before its first launch on a device, and how many clusters of 1 .. max_cluster CTAs of it fit there at once:
// active[1 .. max_cluster].  Done and asked by the first call only; active[0] != 0 once all of it is there, so a host thread that
// comes meanwhile waits, and reads whole answers.  cfg: block, shared memory and stream of the launch.
template <typename K>
cudaError_t clusters_that_fit(K kernel, cudaLaunchConfig_t cfg, int max_cluster, int* active) {
  if (__atomic_load_n(&active[0], __ATOMIC_ACQUIRE)) return cudaSuccess;
  static std::mutex mu;
  std::lock_guard<std::mutex> lock(mu);
  if (__atomic_load_n(&active[0], __ATOMIC_RELAXED)) return cudaSuccess;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)cfg.dynamicSmemBytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  for (int c = 1; c <= max_cluster && e == cudaSuccess; ++c) {
    cfg.gridDim = dim3(c);
    attr[0].val.clusterDim.x = c;
    e = cudaOccupancyMaxActiveClusters(&active[c], kernel, &cfg);
  }
  if (e == cudaSuccess) __atomic_store_n(&active[0], 1, __ATOMIC_RELEASE);
  return e;
}

}  // namespace qp
