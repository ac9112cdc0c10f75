// A block's output joined to the residual stream through a norm, a gate and the
// stream's scale, with the next block's norm at once, forwards and backwards.
//
//   S = alpha X + gate N_f(F),  Y = N_y(S),  N(v) = xhat gamma + beta,  xhat = (v - mean) rstd
//   backwards, with N'(g) = rstd (g - [layer: sum(g) / n] - xhat sum(g xhat) / n):
//   T = dS + N_y'(dY gamma_y),  dX = alpha T,  dF = N_f'(T gate gamma_f)
//   A = sum over rows of T xhat_f,  B = sum of T,  C = sum of dY xhat_y,  D = sum of dY:
//   dgate = gamma_f A + beta_f B,  dgamma_f = gate A,  dbeta_f = gate B,  dgamma_y = C,  dbeta_y = D
//
// HBM-bound: two arrays are read and two written (backwards four and two), each
// once.  As in the layer norm, teams of 32 to 512 threads hold rows in registers (16
// values per thread, backwards 8: four sums per column stay there too) with the
// next rows on their way into shared memory, and rows too long for a team are
// shared by clusters.  Forwards the parameters are folded, gate gamma_f and gate
// beta_f, so that four vectors fit the registers (16384 x 4096 bf16: 89 us, 6.0
// TB/s).  Backwards the second sums of a row and the first of the next one are
// exchanged at one barrier (16384 x 2048 bf16: 77 us, 5.2 TB/s; with a barrier for
// each 110), and the arithmetic is in pairs (one by one: 90); instructions issue in
// 59% of the slots, and the 16 warps per SM that the sums leave room for do not hide
// the rest, their own latencies.  A cluster's
// warps tell one another their sums directly, and the next row is asked for before
// the answer is waited for (4096 x 8192 backwards: 104 us; sums joined in each CTA
// first: 123).  The CTAs' partial rows are summed in CTA order by a second kernel.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>
#include <utility>

#include "residual_norm_kernel.cuh"

namespace goldy {
namespace {

constexpr int kStreamThreads = 512;
constexpr int kBwdCtas = 152;          // CTAs of a backward launch, at most: one partial row each

template <typename T>
__device__ __forceinline__ float elem(const void* base, int64_t i) {
  return sizeof(T) == 2 ? load_bf16(base, i) : static_cast<const float*>(base)[i];
}
template <typename T>
__device__ __forceinline__ void put(void* base, int64_t i, float v) {
  if (sizeof(T) == 2) store_bf16(base, i, v);
  else static_cast<float*>(base)[i] = v;
}

// Sum of two values over the CTA (every thread gets both).
__device__ __forceinline__ float2 cta_sum(float a, float b, float2* slots) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    a += __shfl_xor_sync(0xFFFFFFFFu, a, d);
    b += __shfl_xor_sync(0xFFFFFFFFu, b, d);
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = make_float2(a, b);
  __syncthreads();
  float2 r = make_float2(0.0f, 0.0f);
#pragma unroll
  for (int i = 0; i < kStreamThreads / 32; ++i) {
    r.x += slots[i].x;
    r.y += slots[i].y;
  }
  return r;
}

// Mean and rstd of n values at(c) over the CTA.
template <typename F>
__device__ __forceinline__ float2 statistics(int kind, int n, float inv_n, float eps, float2* slots, F at) {
  float mean = 0.0f;
  if (kind == GOLDY_NORM_LAYER) {
    float s = 0.0f;
    for (int c = threadIdx.x; c < n; c += kStreamThreads) s += at(c);
    mean = cta_sum(s, 0.0f, slots).x * inv_n;
  }
  float m2 = 0.0f;
  for (int c = threadIdx.x; c < n; c += kStreamThreads) {
    const float d = at(c) - mean;
    m2 = fmaf(d, d, m2);
  }
  return make_float2(mean, rsqrtf(fmaf(cta_sum(m2, 0.0f, slots).x, inv_n, eps)));
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads) residual_norm_forward_stream_kernel(const ResidualNormParams p) {
  __shared__ float2 slots[kStreamThreads / 32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    float2 sf = make_float2(0.0f, 1.0f), sy = sf;
    auto f_at = [&](int c) { return elem<T>(p.f, row * p.ldf + c); };
    if (p.norm_f != GOLDY_NORM_NONE) sf = statistics(p.norm_f, p.n, p.inv_n, p.eps, slots, f_at);
    auto s_at = [&](int c) {
      const float v = fmaf((f_at(c) - sf.x) * sf.y, param_at(p.gamma_f, p.param_f32, c, 1.0f),
                           param_at(p.beta_f, p.param_f32, c, 0.0f));
      return fmaf(param_at(p.gate, p.param_f32, c, 1.0f), v, p.alpha * elem<T>(p.x, row * p.ldx + c));
    };
    if (p.norm_y != GOLDY_NORM_NONE) sy = statistics(p.norm_y, p.n, p.inv_n, p.eps, slots, s_at);
    // the only pass that writes: each thread what it alone reads in this pass
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
      const float s = s_at(c);
      put<T>(p.s, row * p.lds + c, s);
      if (p.y)
        put<T>(p.y, row * p.ldy + c, fmaf((s - sy.x) * sy.y, param_at(p.gamma_y, p.param_f32, c, 1.0f),
                                          param_at(p.beta_y, p.param_f32, c, 0.0f)));
    }
    if (threadIdx.x == 0 && p.stats) {
      if (p.norm_f == GOLDY_NORM_LAYER) p.stats[row] = sf.x;
      if (p.norm_f != GOLDY_NORM_NONE) p.stats[p.rows + row] = sf.y;
      if (p.norm_y == GOLDY_NORM_LAYER) p.stats[2 * p.rows + row] = sy.x;
      if (p.norm_y != GOLDY_NORM_NONE) p.stats[3 * p.rows + row] = sy.y;
    }
    __syncthreads();                               // before the slots are used again
  }
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads) residual_norm_backward_stream_kernel(const ResidualNormParams p) {
  __shared__ float2 slots[kStreamThreads / 32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  float* part = p.part ? p.part + int64_t(blockIdx.x) * kSums * p.n : nullptr;
  if (part)
    for (int64_t c = threadIdx.x; c < int64_t(kSums) * p.n; c += kStreamThreads) part[c] = 0.0f;
  __syncthreads();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const float mf = p.norm_f == GOLDY_NORM_LAYER ? p.stats[row] : 0.0f;
    const float rf = p.norm_f != GOLDY_NORM_NONE ? p.stats[p.rows + row] : 1.0f;
    const float my = p.norm_y == GOLDY_NORM_LAYER ? p.stats[2 * p.rows + row] : 0.0f;
    const float ry = p.norm_y != GOLDY_NORM_NONE ? p.stats[3 * p.rows + row] : 1.0f;
    auto yhat = [&](int c) { return (elem<T>(p.s_in, row * p.lds + c) - my) * ry; };
    auto fhat = [&](int c) { return (elem<T>(p.f, row * p.ldf + c) - mf) * rf; };
    auto dy_at = [&](int c) { return elem<T>(p.dy, row * p.ldy + c); };
    float2 sy = make_float2(0.0f, 0.0f), sf = sy;
    if (p.dy) {
      for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
        const float g = dy_at(c) * param_at(p.gamma_y, p.param_f32, c, 1.0f);
        sy.x += g;
        sy.y = fmaf(g, yhat(c), sy.y);
      }
      sy = cta_sum(sy.x, sy.y, slots);
      sy.x = p.norm_y == GOLDY_NORM_LAYER ? sy.x * p.inv_n : 0.0f;
      sy.y *= p.inv_n;
    }
    auto t_at = [&](int c) {
      float t = p.ds ? elem<T>(p.ds, row * p.lds + c) : 0.0f;
      if (p.dy) t += ry * (dy_at(c) * param_at(p.gamma_y, p.param_f32, c, 1.0f) - sy.x - yhat(c) * sy.y);
      return t;
    };
    auto u_at = [&](int c, float t) {
      return t * param_at(p.gate, p.param_f32, c, 1.0f) * param_at(p.gamma_f, p.param_f32, c, 1.0f);
    };
    if (p.norm_f != GOLDY_NORM_NONE) {
      for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
        const float u = u_at(c, t_at(c));
        sf.x += u;
        sf.y = fmaf(u, fhat(c), sf.y);
      }
      sf = cta_sum(sf.x, sf.y, slots);
      sf.x = p.norm_f == GOLDY_NORM_LAYER ? sf.x * p.inv_n : 0.0f;
      sf.y *= p.inv_n;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
      const float t = t_at(c), h = fhat(c);
      const float df = rf * (u_at(c, t) - sf.x - h * sf.y);
      if (part) {
        part[c] = fmaf(t, h, part[c]);
        part[p.n + c] += t;
        if (p.dy) {
          part[2 * int64_t(p.n) + c] = fmaf(dy_at(c), yhat(c), part[2 * int64_t(p.n) + c]);
          part[3 * int64_t(p.n) + c] += dy_at(c);
        }
      }
      put<T>(p.s, row * p.ldx + c, p.alpha * t);
      put<T>(p.y, row * p.ldf + c, df);
    }
  }
}

// ---- gradients of the parameters --------------------------------------------------

// The parameters' gradients from the CTAs' partial rows, in CTA order: of 32
// columns, eight warps per sum take every eighth row, all in flight together, and
// the warps are added in order.
constexpr int kReduceWarps = 8;
constexpr int kReduceRows = (kBwdCtas + kReduceWarps - 1) / kReduceWarps;
__global__ void __launch_bounds__(kSums * kReduceWarps * 32) residual_norm_reduce_kernel(const ResidualNormParams p) {
  __shared__ float s[kSums][kReduceWarps][32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, q = w / kReduceWarps, k = w % kReduceWarps;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float v = 0.0f, t[kReduceRows];
#pragma unroll
  for (int i = 0; i < kReduceRows; ++i) {
    const int r = k + i * kReduceWarps;
    t[i] = r < p.parts && c < p.n ? __ldcg(p.part + (int64_t(r) * kSums + q) * p.n + c) : 0.0f;
  }
#pragma unroll
  for (int i = 0; i < kReduceRows; ++i) v += t[i];
  s[q][k][lane] = v;
  __syncthreads();
  if (w != 0 || c >= p.n) return;
  float all[kSums];
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    all[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < kReduceWarps; ++j) all[i] += s[i][j][lane];
  }
  give_gradients(p, c, all[0], all[1], all[2], all[3]);
}

// ---- host ---------------------------------------------------------------------

// Threads per row; 0: the row streams.  `cluster` CTAs of kMaxTeam threads share a
// row that is too long for one.
ResidualNormShape shape_for(const goldy_residual_norm_desc& d, bool backward, RowMode mode) {
  const int64_t vals = backward ? kBwdVals : kFwdVals, most = kMaxTeam * vals;
  // (a framed row begins inside its first block)
  const int64_t wide = d.n + (mode == kFramedRows ? 16 / int64_t(element_size(d.dtype)) - 1 : 0);
  int team = int(std::max<int64_t>(1, ceil_div(wide, 32 * vals))) * 32, cluster = 1;
  // as many warps as the row takes up to 8, then 16 (16384 x 1111 bf16: 42 us, backwards
  // 77; with powers of two 65 and 112); forwards 7 leave too little of the SM (8192 x
  // 3333: 58 us, with 8 53); a power of two for rows that lie anyhow
  if (team > 256) team = kMaxTeam;
  if (team == 224 && !backward) team = 256;
  if (mode == kAnyRows)
    while (team & (team - 1)) team += 32;
  while (cluster < kMaxCluster && cluster * most < wide) cluster *= 2;
  if (cluster * most < wide) return {0, 1, 0};
  return {cluster > 1 ? kMaxTeam : team, cluster, int(ceil_div(ceil_div(wide, cluster), 8) * 8)};      // whole pieces
}

// Partial rows of a backward launch, at most: CTAs, or clusters of them.
int64_t stream_parts(const goldy_residual_norm_desc& d) {
  return std::max<int64_t>(1, std::min<int64_t>(kBwdCtas, d.rows));
}
// Rows per team up to which one CTA does them all: a further kernel that sums
// partial rows costs more.
constexpr int kAloneRows = 2;
int64_t team_parts(const goldy_residual_norm_desc& d, const ResidualNormShape& s) {
  const int64_t teams = s.cluster > 1 ? 1 : bwd_threads(s.team) / s.team;
  if (d.rows <= kAloneRows * teams) return 1;      // no second kernel
  return std::min<int64_t>(kBwdCtas / s.cluster, ceil_div(d.rows, teams));
}
size_t backward_bytes(const goldy_residual_norm_desc& d) {
  int64_t parts = 0;
  for (const RowMode mode : {kWholeRows, kFramedRows, kAnyRows}) {
    const ResidualNormShape s = shape_for(d, true, mode);
    // (inside an SM partition rows stream where clusters would share them)
    parts = std::max(parts, s.team == 0 || s.cluster > 1 ? stream_parts(d) : team_parts(d, s));
  }
  return kLayerCounterBytes + size_t(parts) * kSums * size_t(d.n) * sizeof(float);
}

bool is_kind(int k) { return k == GOLDY_NORM_NONE || k == GOLDY_NORM_LAYER || k == GOLDY_NORM_RMS; }

goldy_status check_residual_norm(const goldy_residual_norm_desc* d) {
  if (!d) return invalid("null descriptor");
  if (d->rows < 0 || d->n < 0 || d->n > (int64_t(1) << 30)) return invalid("residual norm: a size is negative or too large");
  if (d->ldx < d->n || d->ldf < d->n || d->lds < d->n || d->ldy < d->n)
    return invalid("residual norm: a row stride is smaller than its row");
  if (too_far(d->rows, d->ldx) || too_far(d->rows, d->ldf) || too_far(d->rows, d->lds) || too_far(d->rows, d->ldy) ||
      d->rows > (int64_t(1) << 40))
    return invalid("residual norm: an array is beyond any memory");
  if ((d->dtype != GOLDY_BF16 && d->dtype != GOLDY_F32) || (d->param_dtype != GOLDY_BF16 && d->param_dtype != GOLDY_F32))
    return fail(GOLDY_ERR_UNSUPPORTED, "residual norm: types are GOLDY_BF16 or GOLDY_F32");
  if (!is_kind(d->norm_f) || !is_kind(d->norm_y)) return invalid("residual norm: norm_f or norm_y out of range");
  if (!(d->eps >= 0.0f) || d->eps > 1e30f) return invalid("residual norm: eps must be finite and not negative");
  if (!std::isfinite(d->alpha)) return invalid("residual norm: alpha must be finite");
  if (d->reserved != 0) return invalid("residual norm: reserved must be 0");
  return GOLDY_OK;
}

// Parameters, or gradients, of norms that are there, on their boundaries.
goldy_status check_params(const goldy_residual_norm_desc& d, const goldy_residual_norm_params& p, size_t size) {
  if (d.norm_f == GOLDY_NORM_NONE && (p.gamma_f || p.beta_f))
    return invalid("residual norm: gamma_f or beta_f given, but norm_f is GOLDY_NORM_NONE");
  if (d.norm_y == GOLDY_NORM_NONE && (p.gamma_y || p.beta_y))
    return invalid("residual norm: gamma_y or beta_y given, but norm_y is GOLDY_NORM_NONE");
  for (const void* q : {p.gate, p.gamma_f, p.beta_f, p.gamma_y, p.beta_y})
    if (!on_boundary(q, size)) return invalid("residual norm: a parameter or gradient is misaligned");
  return GOLDY_OK;
}

struct ResidualNormCall {
  ResidualNormParams p;
  const goldy_residual_norm_desc* d;
  bool backward;
  RowMode mode;
  int period;            // framed rows: that many rows apart they begin alike
  void* stream;
};

NormKernel kernel_for(const ResidualNormCall& call, const ResidualNormShape& shape, RowMode mode) {
  const goldy_residual_norm_desc& d = *call.d;
  const bool f32 = d.dtype == GOLDY_F32, full = d.norm_f != GOLDY_NORM_NONE && d.norm_y != GOLDY_NORM_NONE && call.p.ds;
  if (shape.team == 0)
    return {call.backward ? (f32 ? reinterpret_cast<const void*>(&residual_norm_backward_stream_kernel<float>)
                                 : reinterpret_cast<const void*>(&residual_norm_backward_stream_kernel<uint16_t>))
                          : (f32 ? reinterpret_cast<const void*>(&residual_norm_forward_stream_kernel<float>)
                                 : reinterpret_cast<const void*>(&residual_norm_forward_stream_kernel<uint16_t>)),
            kStreamThreads, 1, 4, 0};
  static ResidualNormPick* const picks[2][2][3] = {
      {{residual_norm_forward_bf16_0, residual_norm_forward_bf16_1, residual_norm_forward_bf16_2},
       {residual_norm_forward_f32_0, residual_norm_forward_f32_1, residual_norm_forward_f32_2}},
      {{residual_norm_backward_bf16_0, residual_norm_backward_bf16_1, residual_norm_backward_bf16_2},
       {residual_norm_backward_f32_0, residual_norm_backward_f32_1, residual_norm_backward_f32_2}}};
  return picks[call.backward][f32][mode](shape, full);
}

// CTAs, or clusters of them, all resident (`cap` are), every team with rows of its own
int64_t groups_for(const ResidualNormCall& call, const ResidualNormShape& shape, const NormKernel& k, int64_t cap) {
  const goldy_residual_norm_desc& d = *call.d;
  int64_t groups = std::min(cap, ceil_div(d.rows, int64_t(k.teams)));
  if (call.backward) groups = shape.team == 0 ? stream_parts(d) : team_parts(d, shape);
  if (shape.cluster > 1) groups = std::min(groups, cap);
  return std::max<int64_t>(1, groups);
}

goldy_status launch_residual_norm(const LayerContext& ctx, void* arg) {
  ResidualNormCall& call = *static_cast<ResidualNormCall*>(arg);
  const goldy_residual_norm_desc& d = *call.d;
  RowMode mode = call.mode;
  ResidualNormShape shape;
  NormKernel k;
  int64_t groups = 0;
  for (;; mode = kAnyRows) {
    shape = shape_for(d, call.backward, mode);
    // which SMs a partition has, and so whether a cluster fits into it, is not known
    if (!ctx.whole && shape.cluster > 1) shape = {0, 1, 0};
    if (mode == kFramedRows) {
      // a frame may take a larger team than the row: in bf16 it pays all the same
      // (16384 x 1023 backwards 74 us, in the general way 96; x 511 49 and 59), and
      // forwards in fp32 (8192 x 511 17 and 26), but not backwards in fp32, where
      // single elements cost less (8192 x 1023 62 and 51)
      const ResidualNormShape any = shape_for(d, call.backward, kAnyRows);
      const bool grown = shape.team > any.team && call.backward && d.dtype == GOLDY_F32;
      if (shape.team == 0 || shape.cluster > any.cluster || grown) continue;
    }
    k = kernel_for(call, shape, mode);
    int64_t cap = int64_t(ctx.sm_count) * k.per_sm;            // CTAs, or clusters, resident at once
    if (shape.cluster > 1) {
      cudaError_t e = allow_smem(ctx.device, k);
      int most = 0;
      if (e == cudaSuccess) e = resident_clusters(ctx.device, k, shape.cluster, &most);
      if (e == cudaSuccess && most < 1) e = cudaErrorInvalidClusterSize;
      if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("residual norm, clusters: ") + cudaGetErrorString(e));
      cap = std::min<int64_t>(cap / shape.cluster, most);
    }
    groups = groups_for(call, shape, k, cap);
    if (mode != kFramedRows) break;
    // a team with several rows has them a whole number of periods apart
    while (groups > 0 && groups * k.teams < d.rows && groups * k.teams % call.period != 0) --groups;
    if (groups > 0) break;
  }
  cudaError_t e = allow_smem(ctx.device, k);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
  call.p.cluster = shape.cluster;
  call.p.seg = shape.seg;
  call.p.parts = int32_t(groups);
  void* args[] = {&call.p};
  e = NormLaunch(unsigned(groups * shape.cluster), unsigned(k.threads), k.smem, call.stream, unsigned(shape.cluster)).run(k.fn, args);
  if (e == cudaSuccess && call.p.part && (groups > 1 || shape.team == 0))
    e = NormLaunch(unsigned(ceil_div(d.n, 32)), kSums * kReduceWarps * 32, 0, call.stream)
            .run(reinterpret_cast<const void*>(&residual_norm_reduce_kernel), args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("residual norm launch: ") + cudaGetErrorString(e));
  return GOLDY_OK;
}

// How the arrays' rows lie (the parameters are read one by one but for whole rows).
void row_mode(ResidualNormCall& call, const goldy_residual_norm_desc& d, const goldy_residual_norm_params& given,
              std::initializer_list<std::pair<const void*, int64_t>> arrays) {
  const int64_t size = int64_t(element_size(d.dtype)), per = 16 / size;
  bool whole = d.n % per == 0, alike = true;
  const auto& f = *arrays.begin();                 // F, which is always there
  for (const auto& a : arrays) {
    if (!a.first) continue;
    whole = whole && on_boundary(a.first, 16) && a.second % per == 0;
    alike = alike && reinterpret_cast<uintptr_t>(a.first) % 16 == reinterpret_cast<uintptr_t>(f.first) % 16 &&
            a.second % per == f.second % per;
  }
  for (const void* q : {given.gate, given.gamma_f, given.beta_f, given.gamma_y, given.beta_y}) whole = whole && on_boundary(q, 16);
  call.mode = whole ? kWholeRows : alike ? kFramedRows : kAnyRows;
  call.period = 1;                                 // per / gcd(stride, per)
  while (f.second * call.period % per != 0) call.period *= 2;
}

void common_params(ResidualNormCall& call, const goldy_residual_norm_desc& d, const goldy_residual_norm_params& given) {
  ResidualNormParams& p = call.p;
  call.d = &d;
  p.gate = given.gate;
  p.gamma_f = given.gamma_f;
  p.beta_f = given.beta_f;
  p.gamma_y = given.gamma_y;
  p.beta_y = given.beta_y;
  p.rows = d.rows;
  p.ldx = d.ldx;
  p.ldf = d.ldf;
  p.lds = d.lds;
  p.ldy = d.ldy;
  p.n = int32_t(d.n);
  p.param_f32 = d.param_dtype == GOLDY_F32;
  p.norm_f = d.norm_f;
  p.norm_y = d.norm_y;
  p.eps = d.eps;
  p.alpha = d.alpha;
  p.inv_n = float(1.0 / double(d.n));
}

}  // namespace
}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_residual_norm_query(const goldy_residual_norm_desc* desc, size_t* workspace_bytes) try {
  const goldy_status st = check_residual_norm(desc);
  if (st != GOLDY_OK) return st;
  if (!workspace_bytes) return invalid("null argument");
  *workspace_bytes = desc->n > 0 ? backward_bytes(*desc) : 0;
  return ok();
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_residual_norm_forward(const goldy_residual_norm_desc* desc,
                                                    const goldy_residual_norm_params* params, const void* X,
                                                    const void* F, void* S, void* Y, float* stats, void* stream) try {
  goldy_status st = check_residual_norm(desc);
  if (st != GOLDY_OK) return st;
  const goldy_residual_norm_params given = params ? *params : goldy_residual_norm_params{};
  st = check_params(*desc, given, element_size(desc->param_dtype));
  if (st != GOLDY_OK) return st;
  if ((Y != nullptr) != (desc->norm_y != GOLDY_NORM_NONE) && desc->rows > 0 && desc->n > 0)
    return invalid("residual norm: Y is null exactly when norm_y is GOLDY_NORM_NONE");
  if (desc->rows == 0 || desc->n == 0) return ok();
  if (!X || !F || !S) return invalid("residual norm: X, F and S are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(X, es) || !on_boundary(F, es) || !on_boundary(S, es) || !on_boundary(Y, es) || !on_boundary(stats, 4))
    return invalid("residual norm: a pointer is misaligned");
  if (S == Y) return invalid("residual norm: S and Y are one array");
  if ((S == X && desc->lds != desc->ldx) || (S == F && desc->lds != desc->ldf) || (Y == X && desc->ldy != desc->ldx) ||
      (Y == F && desc->ldy != desc->ldf))
    return invalid("residual norm: a result is an input, with another stride");
  ResidualNormCall call{};
  common_params(call, *desc, given);
  call.p.x = X;
  call.p.f = F;
  call.p.s = S;
  call.p.y = Y;
  call.p.stats = stats;
  row_mode(call, *desc, given, {{F, desc->ldf}, {X, desc->ldx}, {S, desc->lds}, {Y, desc->ldy}});
  call.stream = stream;
  st = with_layer_context(stream, launch_residual_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_residual_norm_backward(const goldy_residual_norm_desc* desc,
                                                     const goldy_residual_norm_params* params, const void* dY,
                                                     const void* dS, const void* F, const void* S, const float* stats,
                                                     void* dX, void* dF, const goldy_residual_norm_params* grads,
                                                     int accumulate, void* workspace, size_t workspace_bytes,
                                                     void* stream) try {
  goldy_status st = check_residual_norm(desc);
  if (st != GOLDY_OK) return st;
  if (accumulate != 0 && accumulate != 1) return invalid("residual norm: accumulate must be 0 or 1");
  const goldy_residual_norm_params given = params ? *params : goldy_residual_norm_params{};
  const goldy_residual_norm_params want = grads ? *grads : goldy_residual_norm_params{};
  st = check_params(*desc, given, element_size(desc->param_dtype));
  if (st == GOLDY_OK) st = check_params(*desc, want, sizeof(float));
  if (st != GOLDY_OK) return st;
  if (desc->n == 0) return ok();
  const bool sums = want.gate || want.gamma_f || want.beta_f || want.gamma_y || want.beta_y;
  if (desc->rows == 0 && !sums) return ok();
  if (desc->rows > 0) {
    if ((dY != nullptr) != (desc->norm_y != GOLDY_NORM_NONE))
      return invalid("residual norm: dY is null exactly when norm_y is GOLDY_NORM_NONE");
    if (!dY && !dS) return invalid("residual norm: dY or dS is needed");
    const bool norms = desc->norm_f != GOLDY_NORM_NONE || desc->norm_y != GOLDY_NORM_NONE;
    if (!F || (dY && !S) || !dX || !dF || (norms && !stats))
      return invalid("residual norm: F, S, stats, dX and dF are needed");
  }
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(dY, es) || !on_boundary(dS, es) || !on_boundary(F, es) || !on_boundary(S, es) || !on_boundary(dX, es) ||
      !on_boundary(dF, es) || !on_boundary(stats, 4))
    return invalid("residual norm: a pointer is misaligned");
  if (desc->rows > 0 && dX == dF) return invalid("residual norm: dX and dF are one array");
  const std::pair<const void*, int64_t> from[] = {{dY, desc->ldy}, {dS, desc->lds}, {F, desc->ldf}, {S, desc->lds}};
  for (const auto& a : from)
    if (a.first && ((dX == a.first && desc->ldx != a.second) || (dF == a.first && desc->ldf != a.second)))
      return invalid("residual norm: a result is an input, with another stride");
  if (sums) {
    st = check_workspace("residual norm", workspace, workspace_bytes, backward_bytes(*desc));
    if (st != GOLDY_OK) return st;
  }
  ResidualNormCall call{};
  common_params(call, *desc, given);
  call.backward = true;
  call.p.dy = dY;
  call.p.ds = dS;
  call.p.f = F;
  call.p.s_in = S;
  call.p.stats = const_cast<float*>(stats);
  call.p.s = dX;
  call.p.y = dF;
  call.p.part = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kLayerCounterBytes) : nullptr;
  call.p.dgate = static_cast<float*>(want.gate);
  call.p.dgamma_f = static_cast<float*>(want.gamma_f);
  call.p.dbeta_f = static_cast<float*>(want.beta_f);
  call.p.dgamma_y = static_cast<float*>(want.gamma_y);
  call.p.dbeta_y = static_cast<float*>(want.beta_y);
  call.p.accumulate = accumulate;
  row_mode(call, *desc, given, {{F, desc->ldf}, {dY, desc->ldy}, {dS, desc->lds}, {dY ? S : nullptr, desc->lds},
                                {dX, desc->ldx}, {dF, desc->ldf}});
  call.stream = stream;
  st = with_layer_context(stream, launch_residual_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
