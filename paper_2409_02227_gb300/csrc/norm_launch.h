// Launches of the norms' kernels: early start, clusters, large shared memory.
#pragma once

#include <cuda_runtime.h>

#include <map>
#include <mutex>
#include <set>
#include <string>
#include <tuple>
#include <utility>

namespace goldy {

struct NormKernel {
  const void* fn;
  int threads, teams, per_sm;      // per_sm: CTAs resident
  size_t smem;
};

struct NormLaunch {
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];

  NormLaunch(unsigned grid, unsigned threads, size_t smem, void* stream, unsigned cluster = 1) {
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
  }
  NormLaunch(const NormLaunch&) = delete;
  cudaError_t run(const void* fn, void** args) { return cudaLaunchKernelExC(&cfg, fn, args); }
};

// Clusters of a kernel that the device holds at once (a GPC's SMs need not make
// whole clusters), asked for once.
inline cudaError_t resident_clusters(int device, const NormKernel& k, int cluster, int* n) {
  static std::mutex mu;
  static std::map<std::tuple<int, const void*, int>, int> known;
  std::lock_guard<std::mutex> lock(mu);
  const auto key = std::make_tuple(device, k.fn, cluster);
  const auto it = known.find(key);
  if (it != known.end()) {
    *n = it->second;
    return cudaSuccess;
  }
  NormLaunch l(unsigned(cluster), unsigned(k.threads), k.smem, nullptr, unsigned(cluster));
  const cudaError_t e = cudaOccupancyMaxActiveClusters(n, k.fn, &l.cfg);
  if (e == cudaSuccess) known[key] = *n;
  return e;
}

// Opts a kernel into more than 48 KB of shared memory, once per device.
inline cudaError_t allow_smem(int device, const NormKernel& k) {
  if (k.smem <= 40 * 1024) return cudaSuccess;     // with the kernel's static part below 48 KB
  static std::mutex mu;
  static std::set<std::pair<int, const void*>> done;
  std::lock_guard<std::mutex> lock(mu);
  if (done.count({device, k.fn})) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, int(k.smem));
  if (e == cudaSuccess) done.insert({device, k.fn});
  return e;
}

}  // namespace goldy
