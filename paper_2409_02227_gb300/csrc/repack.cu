// Copies bf16 matrices whose rows do not start on 16-byte boundaries into
// padded ones (rows rounded up to 8 elements), for the tensor-memory
// accelerator.  One read and one write of the operand; used only where a row
// stride is not a multiple of 8.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

struct RepackParams {
  const uint16_t* from;
  uint4* to;
  int64_t rows, ld, batch_stride;      // source rows of one matrix, strides in elements
  int64_t vecs;                        // 16-byte pieces of all padded rows
  int32_t cols, row_vecs;
};

__global__ void __launch_bounds__(256) repack_kernel(const RepackParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < p.vecs; i += int64_t(gridDim.x) * 256) {
    const int64_t line = i / p.row_vecs;
    const int c = int(i - line * p.row_vecs) * 8;
    const uint16_t* from = p.from + (line / p.rows) * p.batch_stride + (line % p.rows) * p.ld + c;
    uint32_t v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < p.cols ? from[k] : 0u;
    p.to[i] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
  }
}

}  // namespace

goldy_status launch_repack(const LayerContext& ctx, const void* from, void* to, int64_t batch, int64_t rows,
                           int64_t cols, int64_t ld, int64_t batch_stride, void* stream) {
  RepackParams p;
  p.from = static_cast<const uint16_t*>(from);
  p.to = static_cast<uint4*>(to);
  p.rows = rows;
  p.ld = ld;
  p.batch_stride = batch_stride;
  p.cols = int32_t(cols);
  p.row_vecs = int32_t(ceil_div(cols, 8));
  p.vecs = batch * rows * p.row_vecs;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(std::max<int64_t>(1, std::min<int64_t>(ceil_div(p.vecs, 256), int64_t(ctx.sm_count) * 8))));
  cfg.blockDim = dim3(256);
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* args[] = {&p};
  const cudaError_t e = cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(&repack_kernel), args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("operand copy launch: ") + cudaGetErrorString(e));
  return GOLDY_OK;
}

}  // namespace goldy
