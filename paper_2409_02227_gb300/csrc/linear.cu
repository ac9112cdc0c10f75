// Host side of the linear-layer operators: argument checks, tensor maps, the
// choice of tile and split, launches.  Nothing here allocates device memory
// or synchronises; the choice is a pure function of the descriptor, so that
// goldy_linear_query can size the workspace without a device.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <mutex>
#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"

namespace goldy {

// linear_kernels.cu, compiled once per pass and activation
const void* linear_kernel_p0_a0(int pair, int out);
const void* linear_kernel_p0_a1(int pair, int out);
const void* linear_kernel_p0_a2(int pair, int out);
const void* linear_kernel_p0_a3(int pair, int out);
const void* linear_kernel_p0_a4(int pair, int out);
const void* linear_kernel_p1_a0(int pair, int out);
const void* linear_kernel_p1_a1(int pair, int out);
const void* linear_kernel_p1_a2(int pair, int out);
const void* linear_kernel_p1_a3(int pair, int out);
const void* linear_kernel_p1_a4(int pair, int out);
const void* linear_kernel_p2_a0(int pair, int out);

namespace {

const void* linear_kernel_fn(int pass, int act, int pair, int out) {
  typedef const void* (*Pick)(int, int);
  static const Pick picks[2][5] = {
      {linear_kernel_p0_a0, linear_kernel_p0_a1, linear_kernel_p0_a2, linear_kernel_p0_a3, linear_kernel_p0_a4},
      {linear_kernel_p1_a0, linear_kernel_p1_a1, linear_kernel_p1_a2, linear_kernel_p1_a3, linear_kernel_p1_a4}};
  return (pass == kLinWeightGrad ? linear_kernel_p2_a0 : picks[pass][act])(pair, out);
}

constexpr int64_t kMaxDim = (int64_t(1) << 31) - 1024;   // TMA coordinates are 32-bit
constexpr int kModelSms = 152;                           // SMs the choice is made for (a partition's calls take it too)
constexpr int kMaxDevices = 64;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
size_t type_bytes(int dtype) { return dtype == GOLDY_F32 ? 4 : 2; }

struct LinShape {
  int pass;
  int64_t rows, size_c, size_r, red;   // size_r: rows, or input features (weight grad); red as in LinearParams
  int groups;
  int out_dtype;
};

LinShape shape_of(const goldy_linear_desc& d, int pass) {
  LinShape s;
  s.pass = pass;
  s.rows = d.rows;
  s.groups = std::max(1, d.groups);
  s.size_c = pass == kLinInputGrad ? d.in : d.out;
  s.size_r = pass == kLinWeightGrad ? d.in : d.rows;
  s.red = pass == kLinForward ? d.in : pass == kLinInputGrad ? d.out : d.rows;
  s.out_dtype = pass == kLinForward ? d.y_dtype : pass == kLinInputGrad ? d.dx_dtype : d.dw_dtype;
  return s;
}

// What the kernel makes of a shape's result.
int result_of(const LinShape& s) {
  if (s.out_dtype == GOLDY_F32) return kLinF32;
  return s.pass == kLinWeightGrad && s.rows > kLinLongRows ? kLinBf16Long : kLinBf16;
}

struct LinChoice {
  int pair, tile_r, split;
  int64_t max_tiles;       // upper bound over all group sizes
  size_t part_bytes;       // workspace behind the counters
};

int part_chunks(int tile_r) { return int(ceil_div(ceil_div(tile_r, 8), kLinEpiWarps / 4)); }

// Time model of a launch in ns, fitted to the times of 46 shapes (1 to 8192
// rows, 64 to 8192 features, 0 to 64 groups, all passes) under every tile and
// split.  With the kernels as they are now the choice is 4% slower than the best
// measured one on average over these and over 46 other shapes, 34% at worst (8 rows
// of 16 groups, 328 -> 5440 features, where a split of 8 is best).
//   A 64-deep stage of an nw-row tile costs the largest of its tensor time, the
//   issue of its copies and products, and its operands' trip from L2.
//   A unit costs its stages or, if longer, draining its accumulator; the last
//   drain is not hidden.
//   A split adds its partials' trip through L2.
// Group sizes are on the device, so groups are taken as equal.
constexpr double kTensorNs = 1.04;       // per row of a stage
constexpr double kIssueNs = 93.0, kIssuePairNs = 333.0;
constexpr double kSmRate = 102.0, kL2Rate = 15655.0;   // bytes per ns into one SM, into all
constexpr double kDrainNs = 8.7, kUnitNs = 654.0;      // per row of a tile; per unit
constexpr double kSplitNs = 771.0, kSplitEachNs = 195.0, kSplitRowNs = 2.0;

LinChoice choose(const LinShape& s) {
  struct Candidate { int pair, tile_r; };
  static const Candidate cand[] = {{1, 256}, {1, 224}, {1, 192}, {1, 128}, {1, 64}, {0, 256}, {0, 128}, {0, 64}, {0, 32}, {0, 16}};
  const bool wgrad = s.pass == kLinWeightGrad;
  const int64_t live = std::max<int64_t>(1, wgrad ? s.groups : std::min<int64_t>(s.groups, s.rows));
  const int64_t r_rows = wgrad ? s.size_r : ceil_div(std::max<int64_t>(s.rows, 1), live);
  const int64_t red = wgrad ? ceil_div(std::max<int64_t>(s.rows, 1), live) : s.red;
  const int64_t kbs = std::max<int64_t>(1, ceil_div(red, kLinStageK));
  LinChoice best{0, 16, 1, 0, 0};
  double best_t = -1.0;
  for (const Candidate& c : cand) {
    if (s.out_dtype == GOLDY_F32 && c.tile_r > kLinMaxTileF32) continue;
    const int gran = c.pair ? 32 : 16, ctas = c.pair ? 2 : 1;
    const int64_t w = ceil_div(ceil_div(r_rows, ceil_div(r_rows, c.tile_r)), gran) * gran;
    const int64_t tiles_c = ceil_div(s.size_c, 128 * ctas);
    const int64_t tiles = live * ceil_div(r_rows, w) * tiles_c;
    const int64_t workers = kModelSms / ctas;
    // tiles over all groups, at most: each group may end in a partial tile
    const int64_t most = (wgrad || s.groups == 1 ? s.groups * ceil_div(s.size_r, c.tile_r)
                                                 : s.rows / c.tile_r + std::min<int64_t>(s.groups, s.rows)) * tiles_c;
    for (int split = 1; split <= 8; split *= 2) {
      // splits fill idle SMs; their counters have a fixed place in the workspace
      if (split > 1 && (tiles * split > 2 * workers || split > kbs ||
                        size_t(most) * ctas * kLinEpiWarps * sizeof(unsigned) > kLayerCounterBytes))
        break;
      const double rows = double(w), waves = double(ceil_div(tiles * split, workers));
      const double rate = std::min(kSmRate, kL2Rate / double(std::min<int64_t>(tiles * split, workers) * ctas));
      const double stage = std::max({rows * kTensorNs, c.pair ? kIssuePairNs : kIssueNs,
                                     (16384.0 + rows * 128 / ctas) / rate});
      double t = waves * std::max(double(ceil_div(kbs, split)) * stage, rows * kDrainNs + kUnitNs) + rows * kDrainNs;
      if (split > 1) t += kSplitNs + kSplitEachNs * split + kSplitRowNs * rows * (split + 1);
      if (best_t < 0 || t < best_t) {
        best_t = t;
        best.pair = c.pair;
        best.tile_r = c.tile_r;
        best.split = split;
        best.max_tiles = most;
      }
    }
  }
  best.part_bytes = best.split > 1 ? size_t(best.max_tiles) * best.split * (best.pair ? 2 : 1) * kLinEpiWarps *
                                         part_chunks(best.tile_r) * 1024
                                   : 0;
  return best;
}

goldy_status bad(const std::string& why) { return fail(GOLDY_ERR_INVALID_ARG, why); }

bool is_dtype(int t) { return t == GOLDY_BF16 || t == GOLDY_F32; }

// A bf16 operand of a product: `batch` matrices of rows x cols.  The tensor
// memory accelerator reads it in place if its rows start on 16-byte
// boundaries, else a padded copy in the workspace.
struct Operand {
  const void* ptr;
  int64_t batch, rows, cols, ld, stride;
  bool copied() const { return ld % 8 != 0 || (batch > 1 && stride % 8 != 0); }
  size_t copy_bytes() const {
    if (!copied()) return 0;
    return (size_t(batch) * size_t(rows) * size_t(dense_stride(cols, GOLDY_BF16)) * 2 + 255) & ~size_t(255);
  }
};

Operand operand_x(const goldy_linear_desc& d, const void* x) {
  const int64_t ld = stride_or_dense(d.ldx, d.in, GOLDY_BF16);
  return {x, 1, d.rows, d.in, ld, d.rows * ld};
}
Operand operand_dy(const goldy_linear_desc& d, const void* dy) {
  const int64_t ld = stride_or_dense(d.ldy, d.out, GOLDY_BF16);
  return {dy, 1, d.rows, d.out, ld, d.rows * ld};
}
int64_t weight_stride(const goldy_linear_desc& d, int64_t ldw) { return d.stride_w ? d.stride_w : d.in * ldw; }
Operand operand_w(const goldy_linear_desc& d, const void* w) {
  const int64_t ld = stride_or_dense(d.ldw, d.out, GOLDY_BF16);
  return {w, std::max(1, d.groups), d.in, d.out, ld, d.groups > 1 ? weight_stride(d, ld) : d.in * ld};
}
// the operands along c and along r of a pass
void operands_of(const goldy_linear_desc& d, int pass, const void* p_ptr, const void* q_ptr, Operand (&o)[2]) {
  o[0] = pass == kLinWeightGrad ? operand_dy(d, p_ptr) : operand_w(d, p_ptr);
  o[1] = pass == kLinInputGrad ? operand_dy(d, q_ptr) : operand_x(d, q_ptr);
}

goldy_status check_operand(const Operand& o, const char* name) {
  if (!o.ptr || !aligned(o.ptr, o.copied() ? 2 : 16))
    return bad(std::string("linear layer: ") + name + (o.copied() ? " null or misaligned" : " must be a 16-byte aligned device pointer"));
  return GOLDY_OK;
}

// Tensor map of an operand, boxes of box_rows rows x 64 elements, 128-byte
// swizzled.
goldy_status encode(const LayerContext& ctx, CUtensorMap* m, const Operand& o, int box_rows) {
  cuuint64_t dims[3] = {cuuint64_t(o.cols), cuuint64_t(o.rows), cuuint64_t(o.batch)};
  cuuint64_t strides[2] = {cuuint64_t(o.ld) * 2, cuuint64_t(o.stride) * 2};
  cuuint32_t box[3] = {64, cuuint32_t(box_rows), 1};
  cuuint32_t one[3] = {1, 1, 1};
  const CUresult r = ctx.encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.ptr), dims, strides, box,
                                one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(GOLDY_ERR_CUDA, "cuTensorMapEncodeTiled failed with code " + std::to_string(int(r)));
  return GOLDY_OK;
}

goldy_status set_smem(const LayerContext& ctx, const void* fn, int pass, int act, int pair, int out) {
  static std::mutex mu;
  static bool done[kMaxDevices][3][5][2][3] = {};
  std::lock_guard<std::mutex> lock(mu);
  bool& d = done[ctx.device][pass][act][pair][out];
  if (!d) {
    const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kLinSmemBudget);
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
    d = true;
  }
  return GOLDY_OK;
}

struct LinCall {
  LinShape s;
  Operand o[2];            // along c: W, or dY; along r: X, dY, or X
  LinearParams prm;        // epilogue fields filled in by the entry point
  int act;                 // of the result, or whose slope the result is multiplied by
  void* workspace;
  size_t workspace_bytes;
  void* stream;
};

goldy_status launch_linear(const LayerContext& ctx, void* arg) {
  LinCall& call = *static_cast<LinCall*>(arg);
  const LinShape& s = call.s;
  LinearParams& p = call.prm;
  const LinChoice c = choose(s);
  if (c.max_tiles * c.split > kMaxDim) return fail(GOLDY_ERR_UNSUPPORTED, "linear layer: too many output tiles");
  Operand* const o = call.o;
  const size_t copy_bytes = s.red > 0 ? o[0].copy_bytes() + o[1].copy_bytes() : 0;
  if (c.split > 1 || copy_bytes > 0) {
    if (!call.workspace || !aligned(call.workspace, 256))
      return bad("linear layer: the workspace must be a 256-byte aligned device pointer");
    const size_t need = kLayerCounterBytes + c.part_bytes + copy_bytes;
    if (call.workspace_bytes < need)
      return fail(GOLDY_ERR_NOMEM, "linear layer: workspace of " + std::to_string(call.workspace_bytes) + " bytes, " +
                                       std::to_string(need) + " needed");
    char* ws = static_cast<char*>(call.workspace);
    p.cnt = reinterpret_cast<unsigned*>(ws);
    p.part = reinterpret_cast<float*>(ws + kLayerCounterBytes);
    ws += kLayerCounterBytes + c.part_bytes;
    for (int i = 0; i < 2 && copy_bytes > 0; ++i) {
      const size_t bytes = o[i].copy_bytes();
      if (bytes == 0) continue;
      goldy_status st = launch_repack(ctx, o[i].ptr, ws, o[i].batch, o[i].rows, o[i].cols, o[i].ld, o[i].stride, call.stream);
      if (st != GOLDY_OK) return st;
      o[i].ptr = ws;
      o[i].ld = dense_stride(o[i].cols, GOLDY_BF16);
      o[i].stride = o[i].rows * o[i].ld;
      ws += bytes;
    }
  }
  const bool wgrad = s.pass == kLinWeightGrad;
  const int ctas = c.pair ? 2 : 1;
  p.groups = s.groups;
  p.rows = int32_t(s.rows);
  p.size_c = int32_t(s.size_c);
  p.size_r = int32_t(s.size_r);
  p.red = int32_t(s.red);
  p.tile_r = c.tile_r;
  p.tiles_c = int32_t(ceil_div(s.size_c, 128 * ctas));
  p.split = c.split;
  p.div_split = lin_divisor(unsigned(c.split));
  p.div_band = lin_divisor(unsigned(kLinRowBand) * unsigned(p.tiles_c));
  p.part_box = std::min(32, c.tile_r / ctas);
  p.part_chunks = part_chunks(c.tile_r);
  p.loads = s.red > 0 ? 1 : 0;
  const int b_rows = wgrad ? int(ceil_div(c.tile_r / ctas, 64)) * 64 : c.tile_r / ctas;
  p.stage_bytes = 128 * kLinStageK * 2 + b_rows * kLinStageK * 2;
  const int fixed = 2048;      // alignment of the tiles; barriers
  p.stages = std::min<int>(kLinMaxStages, (kLinSmemBudget - fixed) / p.stage_bytes);
  p.err = ctx.err_word;
  if (p.loads) {
    goldy_status st;
    st = encode(ctx, &p.ta, o[0], s.pass == kLinInputGrad ? 128 : kLinStageK);
    if (st == GOLDY_OK) st = encode(ctx, &p.tb, o[1], wgrad ? kLinStageK : c.tile_r / ctas);
    if (st == GOLDY_OK && !wgrad) st = encode(ctx, &p.tb_part, o[1], p.part_box);
    if (st != GOLDY_OK) return st;
  }
  const int out = result_of(s);
  const void* fn = linear_kernel_fn(s.pass, call.act, c.pair, out);
  goldy_status st = set_smem(ctx, fn, s.pass, call.act, c.pair, out);
  if (st != GOLDY_OK) return st;
  const int64_t units = c.max_tiles * c.split;
  const int64_t workers = std::max<int64_t>(1, std::min<int64_t>(units, ctx.sm_count / ctas));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(unsigned(workers * ctas));
  cfg.blockDim = dim3(unsigned(lin_threads(s.pass)));
  cfg.dynamicSmemBytes = size_t(fixed + p.stages * p.stage_bytes);
  cfg.stream = static_cast<cudaStream_t>(call.stream);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.numAttrs = 1;
  if (c.pair) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  cfg.attrs = attr;
  void* args[] = {&p};
  const cudaError_t e = cudaLaunchKernelExC(&cfg, fn, args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("linear layer launch: ") + cudaGetErrorString(e));
  return GOLDY_OK;
}

// Fields of the result and what is added to it, common to the passes.
goldy_status set_result(LinearParams& p, const LinShape& s, void* C, int64_t ldc, const void* R, int64_t ldr,
                        const char* name) {
  const size_t es = type_bytes(s.out_dtype);
  if (!C || !aligned(C, es)) return bad(std::string("linear layer: ") + name + " null or misaligned");
  ldr = stride_or_dense(ldr, s.size_c, s.out_dtype);
  if (R && (!aligned(R, es) || ldr < s.size_c)) return bad("linear layer: residual misaligned or its row stride too small");
  p.c = C;
  p.ldc = ldc;
  p.res = R;
  p.ldr = ldr;
  p.vec = aligned(C, 4) && ldc % 2 == 0 && (!R || (aligned(R, 4) && ldr % 2 == 0));
  return GOLDY_OK;
}

goldy_status set_saved(LinearParams& p, const LinShape& s, const void* Z, int64_t ldz) {
  ldz = stride_or_dense(ldz, s.size_c, GOLDY_BF16);
  if (!aligned(Z, 2) || ldz < s.size_c) return bad("linear layer: Z misaligned or its row stride too small");
  p.ldz = ldz;
  p.vec = p.vec && aligned(Z, 4) && ldz % 2 == 0;
  return GOLDY_OK;
}

}  // namespace

goldy_status layer_exception() {
  try {
    return fail(GOLDY_ERR_NOMEM, "out of host memory");
  } catch (...) {
    return GOLDY_ERR_NOMEM;
  }
}

goldy_status check_linear(const goldy_linear_desc* d) {
  if (!d) return bad("null descriptor");
  if (d->rows < 0 || d->in < 0 || d->out < 0 || d->rows > kMaxDim || d->in > kMaxDim || d->out > kMaxDim)
    return bad("linear layer: a size is negative or too large");
  if (d->groups < 0 || d->groups > GOLDY_MAX_GROUPS) return bad("linear layer: groups out of range");
  if ((d->ldx && d->ldx < d->in) || (d->lddx && d->lddx < d->in) || (d->ldw && d->ldw < d->out) ||
      (d->ldy && d->ldy < d->out) || d->ldz < 0 || d->ldr < 0)
    return bad("linear layer: a row stride is smaller than its row");
  if (d->ldx > kMaxDim || d->lddx > kMaxDim || d->ldw > kMaxDim || d->ldy > kMaxDim || d->ldz > kMaxDim || d->ldr > kMaxDim)
    return bad("linear layer: a row stride is too large");
  if (d->stride_w < 0 || (d->groups > 1 && d->stride_w && d->stride_w < d->in * stride_or_dense(d->ldw, d->out, GOLDY_BF16)))
    return bad("linear layer: stride_w is smaller than in * ldw");
  // no array has more elements than this; sums of sizes then stay far from 64 bits
  const double most = double(int64_t(1) << 46), rows = double(d->rows);
  const int64_t ldw = stride_or_dense(d->ldw, d->out, GOLDY_BF16);
  const double weights = d->groups > 1 && d->stride_w ? double(d->stride_w) : double(d->in) * double(ldw);
  if (weights * std::max(1, d->groups) > most || rows * double(std::max({d->in, d->ldx, d->lddx})) > most ||
      rows * double(std::max({d->out, d->ldy, d->ldz, d->ldr})) > most)
    return bad("linear layer: an array is too large");
  if (d->act < GOLDY_ACT_NONE || d->act > GOLDY_ACT_SILU || d->act_x < GOLDY_ACT_NONE || d->act_x > GOLDY_ACT_SILU)
    return bad("linear layer: unknown activation");
  if (!is_dtype(d->y_dtype) || !is_dtype(d->dx_dtype) || !is_dtype(d->dw_dtype) || !is_dtype(d->bias_dtype))
    return fail(GOLDY_ERR_UNSUPPORTED, "linear layer: types are GOLDY_BF16 or GOLDY_F32");
  if (d->reserved != 0) return bad("linear layer: reserved must be 0");
  return GOLDY_OK;
}

goldy_status check_offsets(const goldy_linear_desc& d, const int32_t* offsets) {
  if (d.groups > 0 && (!offsets || !aligned(offsets, 4)))
    return bad("linear layer: grouped rows need offsets (groups + 1 device integers)");
  if (d.groups == 0 && offsets) return bad("linear layer: offsets given, but the descriptor has no groups");
  return GOLDY_OK;
}

}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_linear_query(const goldy_linear_desc* desc, size_t* workspace_bytes) try {
  goldy_status st = check_linear(desc);
  if (st != GOLDY_OK) return st;
  if (!workspace_bytes) return bad("null argument");
  size_t part = 0;
  for (int pass = 0; pass < 3; ++pass) {
    const LinShape s = shape_of(*desc, pass);
    if (s.size_c == 0 || s.size_r == 0) continue;
    Operand o[2];
    operands_of(*desc, pass, nullptr, nullptr, o);
    part = std::max(part, choose(s).part_bytes + o[0].copy_bytes() + o[1].copy_bytes());
  }
  part = std::max(part, bias_grad_part_bytes(*desc));
  *workspace_bytes = part > 0 ? kLayerCounterBytes + part : 0;
  return ok();
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_linear_forward(const goldy_linear_desc* desc, const int32_t* offsets, const void* X,
                                             const void* W, const void* bias, const void* R, void* Z, void* Y,
                                             void* workspace, size_t workspace_bytes, void* stream) try {
  goldy_status st = check_linear(desc);
  if (st == GOLDY_OK) st = check_offsets(*desc, offsets);
  if (st != GOLDY_OK) return st;
  LinCall call{};
  call.s = shape_of(*desc, kLinForward);
  operands_of(*desc, kLinForward, W, X, call.o);
  if (call.s.size_c == 0 || call.s.size_r == 0) return ok();
  if (call.s.red > 0) {
    st = check_operand(call.o[0], "W");
    if (st == GOLDY_OK) st = check_operand(call.o[1], "X");
    if (st != GOLDY_OK) return st;
  }
  LinearParams& p = call.prm;
  st = set_result(p, call.s, Y, stride_or_dense(desc->ldy, desc->out, desc->y_dtype), R, desc->ldr, "Y");
  if (st == GOLDY_OK && Z) st = set_saved(p, call.s, Z, desc->ldz);
  if (st != GOLDY_OK) return st;
  if (bias && !aligned(bias, type_bytes(desc->bias_dtype))) return bad("linear layer: bias misaligned");
  p.z_out = Z;
  p.bias = bias;
  p.bias_f32 = desc->bias_dtype == GOLDY_F32;
  call.act = desc->act;
  p.offsets = offsets;
  call.workspace = workspace;
  call.workspace_bytes = workspace_bytes;
  call.stream = stream;
  st = with_layer_context(stream, launch_linear, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_linear_input_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* dY,
                                                const void* W, const void* Z, const void* R, void* dX, void* workspace,
                                                size_t workspace_bytes, void* stream) try {
  goldy_status st = check_linear(desc);
  if (st == GOLDY_OK) st = check_offsets(*desc, offsets);
  if (st != GOLDY_OK) return st;
  if (desc->act_x != GOLDY_ACT_NONE && !Z) return bad("linear layer: the activation's gradient needs Z");
  if (desc->act_x == GOLDY_ACT_NONE && Z) return bad("linear layer: Z given, but act_x is GOLDY_ACT_NONE");
  LinCall call{};
  call.s = shape_of(*desc, kLinInputGrad);
  operands_of(*desc, kLinInputGrad, W, dY, call.o);
  if (call.s.size_c == 0 || call.s.size_r == 0) return ok();
  if (call.s.red > 0) {
    st = check_operand(call.o[0], "W");
    if (st == GOLDY_OK) st = check_operand(call.o[1], "dY");
    if (st != GOLDY_OK) return st;
  }
  LinearParams& p = call.prm;
  st = set_result(p, call.s, dX, stride_or_dense(desc->lddx, desc->in, desc->dx_dtype), R, desc->ldr, "dX");
  if (st == GOLDY_OK && Z) st = set_saved(p, call.s, Z, desc->ldz);
  if (st != GOLDY_OK) return st;
  p.z_in = Z;
  call.act = desc->act_x;
  p.offsets = offsets;
  call.workspace = workspace;
  call.workspace_bytes = workspace_bytes;
  call.stream = stream;
  st = with_layer_context(stream, launch_linear, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_linear_weight_grad(const goldy_linear_desc* desc, const int32_t* offsets, const void* X,
                                                 const void* dY, void* dW, int accumulate, void* workspace,
                                                 size_t workspace_bytes, void* stream) try {
  goldy_status st = check_linear(desc);
  if (st == GOLDY_OK) st = check_offsets(*desc, offsets);
  if (st != GOLDY_OK) return st;
  if (accumulate != 0 && accumulate != 1) return bad("linear layer: accumulate must be 0 or 1");
  LinCall call{};
  call.s = shape_of(*desc, kLinWeightGrad);
  operands_of(*desc, kLinWeightGrad, dY, X, call.o);
  if (call.s.size_c == 0 || call.s.size_r == 0) return ok();
  if (call.s.red > 0) {
    st = check_operand(call.o[0], "dY");
    if (st == GOLDY_OK) st = check_operand(call.o[1], "X");
    if (st != GOLDY_OK) return st;
  }
  LinearParams& p = call.prm;
  const int64_t ldw = stride_or_dense(desc->ldw, desc->out, desc->dw_dtype);
  st = set_result(p, call.s, dW, ldw, accumulate ? dW : nullptr, ldw, "dW");
  if (st != GOLDY_OK) return st;
  p.c_group = p.r_group = desc->groups > 1 ? weight_stride(*desc, ldw) : 0;
  p.vec = p.vec && p.c_group % 2 == 0;
  p.offsets = offsets;
  call.workspace = workspace;
  call.workspace_bytes = workspace_bytes;
  call.stream = stream;
  st = with_layer_context(stream, launch_linear, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
