// Internal types of the layer operators (linear-layer products, bias
// gradient, layer norm): kernel parameter blocks shared by the host code and
// the kernels, and the launch context the launch manager provides.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/goldy.h"

namespace goldy {

// ---- launch context (runtime.cu) --------------------------------------------
typedef CUresult (*TensorMapEncodeFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                      const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                      CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                      CUtensorMapFloatOOBfill);
struct LayerContext {
  int device;             // current device
  int sm_count;           // SMs the stream may use (its partition's, or the device's)
  bool whole;             // that is all of the device's
  int* err_word;          // the kernels' error word (goldy_device_error)
  TensorMapEncodeFn encode;
};
// Run `body(ctx, arg)` with the SM partition of `stream` (if it has one)
// current on this thread.
goldy_status with_layer_context(void* stream, goldy_status (*body)(const LayerContext&, void*), void* arg);

// What an entry point answers when C++ raised an exception inside it (host
// memory for an error text or a table): nothing is thrown across the ABI.
goldy_status layer_exception();

// One workspace serves every layer operator: a fixed counter area in front
// (zero between calls), fp32 partial results behind it.
constexpr size_t kLayerCounterBytes = 64 * 1024;

// ---- linear-layer products (linear_kernel.cuh, linear.cu) -------------------
// All three passes compute C[r][c] with c, the contiguous index of C, along
// the tensor cores' M dimension and r along their N dimension:
//   forward      C = Y  (rows x out): c an output feature, r a row, reduction over input features
//   input grad   C = dX (rows x in):  c an input feature,  r a row, reduction over output features
//   weight grad  C = dW (in x out):   c an output feature, r an input feature, reduction over rows
constexpr int kLinForward = 0;
constexpr int kLinInputGrad = 1;
constexpr int kLinWeightGrad = 2;
// results of the kernels
constexpr int kLinBf16 = 0;
constexpr int kLinF32 = 1;
constexpr int kLinBf16Long = 2;           // weight gradient over more than kLinLongRows rows
constexpr int kLinEpiWarps = 12;
// a load warp, an MMA warp, the epilogue's, and the weight gradient's mending warp
constexpr int lin_threads(int pass) { return (2 + kLinEpiWarps + (pass == kLinWeightGrad ? 1 : 0)) * 32; }
constexpr int kLinStageK = 64;            // reduction elements per pipeline stage
constexpr int kLinMaxStages = 12;
constexpr int kLinRowBand = 8;            // row tiles walked before the next column tile
// rows per tile of an fp32 result: its sums take registers, and 256 rows' did
// not fit (spilled: 2048 x 8192 input gradient over 2048 columns 57 us, now 53)
constexpr int kLinMaxTileF32 = 192;
constexpr int kLinPromote = 12;           // stages accumulated in tensor memory for fp32 results
constexpr int kLinPromoteLong = 128;      // and for long bf16 ones, whose sums may spill: rarely touched
// rows from which a bf16 weight gradient is summed that way too: the accumulator's
// truncation, 1e-9 per row, is then 6% of a rounding to bf16 (1024 x 1024 over 65537
// rows: 95 us, in one accumulator 88; 192-row tiles without spills 124)
constexpr int64_t kLinLongRows = 65536;
constexpr int kLinSmemBudget = 232448;    // 227 KB

// n / d for 0 <= n < 2^31 as the high half of n * mul, mul = floor(2^64 / d) + 1.
struct LinDivisor {
  uint64_t mul;
  int32_t one;             // d = 1
  int32_t pad;
};
inline LinDivisor lin_divisor(uint32_t d) { return {d > 1 ? ~uint64_t(0) / d + 1 : 0, d == 1, 0}; }

struct LinearParams {
  CUtensorMap ta;          // operand along c (weights, or dY of the weight gradient)
  CUtensorMap tb;          // operand along r, one box per full tile
  CUtensorMap tb_part;     // the same in boxes of part_box rows, for narrower tiles
  const int* offsets;      // groups + 1 row offsets, or null
  int32_t groups;          // >= 1
  int32_t rows;            // rows of X and Y
  int32_t size_c;          // columns of C
  int32_t size_r;          // rows of C (weight gradient), else = rows
  int32_t red;             // reduction length (forward, input gradient)
  int32_t tile_r;          // rows of C per tile, at most
  int32_t tiles_c;         // column tiles
  int32_t split;           // reduction split over this many units
  LinDivisor div_split, div_band;   // by split; by kLinRowBand * tiles_c
  int32_t stages;
  int32_t stage_bytes;
  int32_t part_box;        // rows per box of tb_part
  int32_t part_chunks;     // 8-row chunks per epilogue warp in a partial
  int32_t bias_f32;
  int32_t vec;             // bf16 results, residual and Z allow 4-byte accesses
  int32_t loads;           // 0: empty reduction, no tensor maps
  void* c;
  int64_t ldc, c_group;    // row stride and group stride of C (group stride: weight gradient)
  const void* bias;        // [groups][size_c] or null
  const void* res;         // added to the result, same type and layout rules as C, or null
  int64_t ldr, r_group;
  const void* z_in;        // bf16: multiply by act'(z_in) instead of applying act
  void* z_out;             // bf16: receives the value before act
  int64_t ldz;
  float* part;             // split partials
  unsigned* cnt;           // arrival counters, zero between calls
  int* err;
};
static_assert(sizeof(LinearParams) <= 4096, "kernel parameter block");

// ---- bias gradient and layer norm -------------------------------------------
struct BiasGradParams {
  const void* dy;
  const void* z;           // null: no activation gradient
  void* dz;
  float* db;               // [groups][cols]
  const int* offsets;
  float* part;
  unsigned* cnt;
  int64_t lddy, ldz, lddz;
  int32_t rows, cols, groups, act, slices, vec, accumulate;
};

// Argument checks shared by the linear-layer entry points (linear.cu), and the
// bias gradient's workspace behind the counters (bias_grad.cu).
// A row stride of 0 stands for dense rows; bf16 rows are then padded to 16 bytes.
inline int64_t dense_stride(int64_t width, int dtype) { return dtype == GOLDY_BF16 ? (width + 7) / 8 * 8 : width; }
inline int64_t stride_or_dense(int64_t ld, int64_t width, int dtype) { return ld ? ld : dense_stride(width, dtype); }
// `batch` bf16 matrices with any strides -> packed ones with rows of ceil(cols / 8) * 8 (repack.cu).
goldy_status launch_repack(const LayerContext& ctx, const void* from, void* to, int64_t batch, int64_t rows,
                           int64_t cols, int64_t ld, int64_t batch_stride, void* stream);
goldy_status check_linear(const goldy_linear_desc* d);
goldy_status check_offsets(const goldy_linear_desc& d, const int32_t* offsets);
size_t bias_grad_part_bytes(const goldy_linear_desc& d);

struct NormParams {
  const void* x;
  const void* dy;
  const void* gamma;       // null: 1
  const void* beta;        // null: 0
  void* out;               // Y, or dX
  float* mean;             // forward: written, may be null
  float* rstd;
  float* part;             // backward: [CTA or cluster][2][n] partial dgamma, dbeta (null: not wanted)
  float* dgamma;
  float* dbeta;
  int32_t accumulate;
  int64_t ldx, ldy;        // row strides: X and dX; Y and dY
  int64_t rows;
  int32_t n;
  int32_t param_f32;
  float eps;
  float inv_n;
  int32_t cluster;         // CTAs that share a row, each with `seg` of its columns (the last with the rest)
  int32_t seg;
};

}  // namespace goldy
