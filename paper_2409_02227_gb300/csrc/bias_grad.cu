// Bias gradient of a linear layer, with the activation's gradient fused in:
//   dZ = dY * act'(Z)  (bf16, when Z is given),  db[e] = sum of dZ (or dY) over the rows of group e.
//
// HBM-bound: dY (and Z) are read once, dZ is written once.  A CTA sums a slice
// of the rows for 64 columns: a warp covers 4 rows of 128 bytes per access (8
// columns per lane), 8 warps 32 rows, kPasses such accesses in flight.  Per
// group that its slice meets it writes one fp32 partial row.  Slice s and group
// e use partial row s + e: along increasing rows slice and group numbers only
// grow, so the sums are distinct.  The last slice to arrive at a column block
// adds the partials in slice order.  Sums are fp32 in a fixed order (a lane's
// rows, lanes, warps, slices), taken before dZ is rounded.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kCols = 64;          // columns per CTA
constexpr int kWarps = 8;
constexpr int kLines = kWarps * 4; // rows per pass of a CTA
constexpr int kPasses = 8;         // passes in flight (half with an activation)
constexpr int kMinRows = 32;       // rows per slice, at least
constexpr int kTargetCtas = 608;   // 4 per SM
constexpr int kStaged = 128;       // partial rows that the last CTA takes into shared memory at once

int slices_for(int64_t rows, int64_t cols) {
  const int64_t blocks = std::max<int64_t>(1, ceil_div(cols, kCols));
  const int64_t want = std::max<int64_t>(1, kTargetCtas / blocks);
  return int(std::max<int64_t>(1, std::min<int64_t>(want, ceil_div(rows, kMinRows))));
}

template <bool ACT>
__global__ void __launch_bounds__(kWarps * 32, 4) bias_grad_kernel(const BiasGradParams p) {
  constexpr int kUnroll = ACT ? kPasses / 2 : kPasses;
  __shared__ float part[kStaged][kCols];
  __shared__ unsigned arrived;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int line = threadIdx.x >> 3;               // row of a pass
  const int c0 = blockIdx.x * kCols;
  const int col = c0 + (threadIdx.x & 7) * 8;
  const int n = max(0, min(8, p.cols - col));
  const bool vec = p.vec && n == 8;
  const int height = (p.rows + p.slices - 1) / p.slices;
  const int row_lo = min(p.rows, int(blockIdx.y) * height), row_hi = min(p.rows, row_lo + height);

  // (a plain load: the kernel before may have written the offsets after this one
  // began, which the read-only data path does not allow)
  auto first_row = [&](int e) { return p.offsets ? min(max(p.offsets[e], 0), p.rows) : (e == 0 ? 0 : p.rows); };
  // the first group that ends behind row_lo: all ends are read at once (a
  // search would wait for one after the other)
  int e = 0;
  if (p.offsets)
    for (int g = 0; g < p.groups; g += kWarps * 32) {
      const int at = g + int(threadIdx.x);
      e += __syncthreads_count(at < p.groups && first_row(at + 1) <= row_lo);
    }
  for (; e < p.groups; ++e) {
    const int a = max(first_row(e), row_lo), b = min(first_row(e + 1), row_hi);
    if (first_row(e) >= row_hi) break;
    if (a >= b) continue;
    float sum[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) sum[k] = 0.0f;
    auto row = [&](const void* base, int64_t ld, int r) {
      return static_cast<const uint16_t*>(base) + int64_t(r) * ld + col;
    };
    if (vec) {
      for (int r0 = a + line; r0 < b; r0 += kUnroll * kLines) {
        uint4 y[kUnroll], z[kUnroll];
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
          const int r = r0 + i * kLines;
          y[i] = make_uint4(0, 0, 0, 0);
          if (r < b) y[i] = *reinterpret_cast<const uint4*>(row(p.dy, p.lddy, r));
          if (ACT && r < b) z[i] = *reinterpret_cast<const uint4*>(row(p.z, p.ldz, r));
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
          const int r = r0 + i * kLines;
          float f[8];
          unpack8(y[i], f);
          if (ACT && r < b) {
            float g[8];
            unpack8(z[i], g);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] *= act_slope(g[k], p.act);
            *reinterpret_cast<uint4*>(const_cast<uint16_t*>(row(p.dz, p.lddz, r))) = pack8(f);
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) sum[k] += f[k];
        }
      }
    } else {
      for (int r = a + line; r < b; r += kLines) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k >= n) break;
          float f = load_bf16(row(p.dy, p.lddy, r), k);
          if (ACT) {
            f *= act_slope(load_bf16(row(p.z, p.ldz, r), k), p.act);
            store_bf16(const_cast<uint16_t*>(row(p.dz, p.lddz, r)), k, f);
          }
          sum[k] += f;
        }
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {                  // the warp's 4 lines
      sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], 8);
      sum[k] += __shfl_xor_sync(0xFFFFFFFFu, sum[k], 16);
    }
    if ((threadIdx.x & 24) == 0) {
#pragma unroll
      for (int k = 0; k < 8; ++k) part[threadIdx.x >> 5][(threadIdx.x & 7) * 8 + k] = sum[k];
    }
    __syncthreads();
    if (threadIdx.x < kCols && c0 + int(threadIdx.x) < p.cols) {
      float s = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) s += part[w][threadIdx.x];
      __stcg(p.part + int64_t(blockIdx.y + e) * p.cols + c0 + threadIdx.x, s);
    }
    __syncthreads();
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) arrived = atomicAdd(p.cnt + blockIdx.x, 1u);
  __syncthreads();
  if (arrived != unsigned(p.slices - 1)) return;
  __threadfence();
  if (threadIdx.x == 0) p.cnt[blockIdx.x] = 0u;
  // the sum of 12 partial rows i, i + step, ... below `end`, in flight together
  auto partials = [&](int i, int step, int end, int g) {
    const int col_at = c0 + int(threadIdx.x) % kCols;
    float t[12], s = 0.0f;
#pragma unroll
    for (int k = 0; k < 12; ++k)
      t[k] = i + k * step < end ? __ldcg(p.part + int64_t(i + k * step + g) * p.cols + col_at) : 0.0f;
#pragma unroll
    for (int k = 0; k < 12; ++k) s += t[k];
    return s;
  };
  // Four threads per column share the groups, or the slices of a single one.
  constexpr int kShare = kWarps * 32 / kCols, kFirst = 6;
  const int mine = threadIdx.x / kCols, c = c0 + int(threadIdx.x) % kCols;
  if (p.groups == 1) {
    float s = 0.0f;
    // only the slices that the group's rows lie in have written a partial row
    const int a = first_row(0), b = first_row(1);
    if (c < p.cols && a < b) {
      const int used = (b - 1) / height + 1;
      for (int i0 = a / height + mine; i0 < used; i0 += 12 * kShare) s += partials(i0, kShare, used, 0);
    }
    part[mine][threadIdx.x % kCols] = s;
    __syncthreads();
    if (mine == 0 && c < p.cols) {
#pragma unroll
      for (int i = 1; i < kShare; ++i) s += part[i][threadIdx.x];
      p.db[c] = p.accumulate ? p.db[c] + s : s;
    }
    return;
  }
  // Few partial rows are all read at once, and each group's range is worked out by
  // one thread: the sums are then short loops over shared memory (8192 x 1024, 64
  // groups: 15.2 us the call; with ranges and loads group after group 18.4).
  const int rows_used = p.slices + p.groups;
  if (rows_used <= kStaged) {
#pragma unroll
    for (int i = 0; i < kStaged / kShare; ++i) {
      const int r = mine + i * kShare;
      if (r < rows_used && c < p.cols) part[r][threadIdx.x % kCols] = __ldcg(p.part + int64_t(r) * p.cols + c);
    }
    __shared__ int2 range[kStaged];                // a group's partial rows
    if (int(threadIdx.x) < p.groups) {
      const int g = threadIdx.x, a = first_row(g), b = first_row(g + 1);
      range[g] = a < b ? make_int2(a / height + g, (b - 1) / height + g) : make_int2(0, -1);
    }
    __syncthreads();
    if (c >= p.cols) return;
    for (int g = mine; g < p.groups; g += kShare) {
      const int2 r = range[g];
      float s = 0.0f;
      for (int i = r.x; i <= r.y; ++i) s += part[i][threadIdx.x % kCols];
      float* to = p.db + int64_t(g) * p.cols + c;
      *to = p.accumulate ? *to + s : s;
    }
    return;
  }
  if (c >= p.cols) return;
  for (int g0 = mine; g0 < p.groups; g0 += 4 * kShare) {
    // four groups at a time, their first kFirst partials in flight together
    int i[4], last[4];
    float s[4], t[4][kFirst];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int g = g0 + k * kShare;
      const int a = g < p.groups ? first_row(g) : 0, b = g < p.groups ? first_row(g + 1) : 0;
      i[k] = a < b ? a / height : 0;
      last[k] = a < b ? (b - 1) / height : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int j = 0; j < kFirst; ++j)
        t[k][j] = i[k] + j <= last[k] ? __ldcg(p.part + int64_t(i[k] + j + g0 + k * kShare) * p.cols + c) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      s[k] = t[k][0];
#pragma unroll
      for (int j = 1; j < kFirst; ++j) s[k] += t[k][j];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int g = g0 + k * kShare;
      if (g >= p.groups) break;
      for (int j = i[k] + kFirst; j <= last[k]; j += 12) s[k] += partials(j, 1, last[k] + 1, g);
      float* to = p.db + int64_t(g) * p.cols + c;
      *to = p.accumulate ? *to + s[k] : s[k];
    }
  }
}

goldy_status bad(const std::string& why) { return fail(GOLDY_ERR_INVALID_ARG, why); }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

struct BiasCall {
  BiasGradParams p;
  void* stream;
};

goldy_status launch_bias_grad(const LayerContext&, void* arg) {
  BiasCall& call = *static_cast<BiasCall*>(arg);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(ceil_div(call.p.cols, kCols)), unsigned(call.p.slices));
  cfg.blockDim = dim3(kWarps * 32);
  cfg.stream = static_cast<cudaStream_t>(call.stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* args[] = {&call.p};
  const void* fn = call.p.z ? reinterpret_cast<const void*>(&bias_grad_kernel<true>)
                            : reinterpret_cast<const void*>(&bias_grad_kernel<false>);
  const cudaError_t e = cudaLaunchKernelExC(&cfg, fn, args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("bias gradient launch: ") + cudaGetErrorString(e));
  return GOLDY_OK;
}

}  // namespace

size_t bias_grad_part_bytes(const goldy_linear_desc& d) {
  if (d.out == 0) return 0;
  return size_t(slices_for(d.rows, d.out) + std::max(1, d.groups)) * size_t(d.out) * sizeof(float);
}

}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_linear_bias_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* dY,
                                               const void* Z, void* dZ, float* db, int accumulate, void* workspace,
                                               size_t workspace_bytes, void* stream) try {
  goldy_status st = check_linear(desc);
  if (st == GOLDY_OK) st = check_offsets(*desc, offsets);
  if (st != GOLDY_OK) return st;
  if (accumulate != 0 && accumulate != 1) return bad("linear layer: accumulate must be 0 or 1");
  if ((Z != nullptr) != (dZ != nullptr)) return bad("linear layer: Z and dZ come together");
  if (Z && desc->act == GOLDY_ACT_NONE) return bad("linear layer: Z given, but act is GOLDY_ACT_NONE");
  if (desc->out == 0) return ok();
  if (ceil_div(desc->out, kCols) > int64_t(kLayerCounterBytes / sizeof(unsigned)))
    return fail(GOLDY_ERR_UNSUPPORTED, "bias gradient: too many columns");
  if (!db || !aligned(db, 4)) return bad("linear layer: db null or misaligned");
  const int64_t ldy = stride_or_dense(desc->ldy, desc->out, GOLDY_BF16);
  const int64_t ldz = stride_or_dense(desc->ldz, desc->out, GOLDY_BF16);
  if (desc->rows > 0 && (!dY || !aligned(dY, 2) || !aligned(Z, 2) || !aligned(dZ, 2)))
    return bad("linear layer: dY null, or dY, Z or dZ misaligned");
  if (Z && ldz < desc->out) return bad("linear layer: the row stride of Z is smaller than its row");
  const size_t need = kLayerCounterBytes + bias_grad_part_bytes(*desc);
  if (!workspace || !aligned(workspace, 256)) return bad("linear layer: the workspace must be a 256-byte aligned device pointer");
  if (workspace_bytes < need)
    return fail(GOLDY_ERR_NOMEM, "linear layer: workspace of " + std::to_string(workspace_bytes) + " bytes, " +
                                     std::to_string(need) + " needed");
  BiasCall call{};
  BiasGradParams& p = call.p;
  p.dy = dY;
  p.z = Z;
  p.dz = dZ;
  p.db = db;
  p.offsets = offsets;
  p.cnt = static_cast<unsigned*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kLayerCounterBytes);
  p.lddy = ldy;
  p.ldz = ldz;
  p.lddz = ldy;
  p.rows = int32_t(desc->rows);
  p.cols = int32_t(desc->out);
  p.groups = std::max(1, desc->groups);
  p.act = desc->act;
  p.slices = slices_for(desc->rows, desc->out);
  p.vec = aligned(dY, 16) && ldy % 8 == 0 && (!Z || (aligned(Z, 16) && ldz % 8 == 0 && aligned(dZ, 16)));
  p.accumulate = accumulate;
  call.stream = stream;
  st = with_layer_context(stream, launch_bias_grad, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
