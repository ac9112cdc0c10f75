// What the layer operators' host code shares: argument helpers and a launch
// whose kernel may begin while the one before it on the stream still runs (it
// waits for that one before it touches global memory).
#pragma once

#include <cuda_runtime.h>

#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"

namespace goldy {

inline bool on_boundary(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
inline goldy_status invalid(const std::string& why) { return fail(GOLDY_ERR_INVALID_ARG, why); }
inline size_t element_size(int dtype) { return dtype == GOLDY_F32 ? 4 : 2; }

// rows of `ld` elements: more than 2^60 are beyond any memory
inline bool too_far(int64_t rows, int64_t ld) { return rows > 0 && ld > (int64_t(1) << 60) / rows; }

inline goldy_status check_workspace(const char* what, const void* workspace, size_t bytes, size_t need) {
  if (!workspace || !on_boundary(workspace, 256))
    return invalid(std::string(what) + ": the workspace must be a 256-byte aligned device pointer");
  if (bytes < need)
    return fail(GOLDY_ERR_NOMEM, std::string(what) + ": workspace of " + std::to_string(bytes) + " bytes, " +
                                     std::to_string(need) + " needed");
  return GOLDY_OK;
}

inline goldy_status launch_layer(const char* what, const void* fn, int64_t grid, int threads, size_t smem, void* stream,
                                 void** args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(grid));
  cfg.blockDim = dim3(unsigned(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelExC(&cfg, fn, args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string(what) + " launch: " + cudaGetErrorString(e));
  return GOLDY_OK;
}

}  // namespace goldy
