// A block's output joined to the residual stream through a norm, a gate and the
// stream's scale, with the next block's norm at once, forwards and backwards.
//
//   S = alpha X + gate N_f(F),  Y = N_y(S),  N(v) = xhat gamma + beta,  xhat = (v - mean) rstd
//   backwards, with N'(g) = rstd (g - [layer: sum(g) / n] - xhat sum(g xhat) / n):
//   T = dS + N_y'(dY gamma_y),  dX = alpha T,  dF = N_f'(T gate gamma_f)
//   A = sum over rows of T xhat_f,  B = sum of T,  C = sum of dY xhat_y,  D = sum of dY:
//   dgate = gamma_f A + beta_f B,  dgamma_f = gate A,  dbeta_f = gate B,  dgamma_y = C,  dbeta_y = D
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "layer_launch.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kStreamThreads = 512;
constexpr int kBwdCtas = 152;          // CTAs of a backward launch, at most: one partial row each
constexpr int kSums = 4;               // A, B, C, D

struct ResidualNormParams {
  const void* x;
  const void* f;
  const void* dy;            // backward, null without a norm
  const void* ds;            // may be null
  const void* s_in;          // backward
  void* s;                   // S, or dX
  void* y;                   // Y, or dF
  const void* gate;
  const void* gamma_f;
  const void* beta_f;
  const void* gamma_y;
  const void* beta_y;
  float* stats;              // [4][rows], may be null forwards
  float* part;               // backward: [CTA][kSums][n]
  int64_t rows, ldx, ldf, lds, ldy;
  int32_t n, param_f32, norm_f, norm_y;
  float eps, alpha, inv_n;
};

struct ReduceParams {
  const float* part;
  const void* gate;
  const void* gamma_f;
  const void* beta_f;
  float* dgate;
  float* dgamma_f;
  float* dbeta_f;
  float* dgamma_y;
  float* dbeta_y;
  int32_t n, parts, accumulate, param_f32;
};

__device__ __forceinline__ float param_at(const void* p, int f32, int i, float absent) {
  if (!p) return absent;
  return f32 ? static_cast<const float*>(p)[i] : load_bf16(p, i);
}
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

// The parameters' gradients from the CTAs' partial rows, in CTA order: 8 warps
// take every eighth row of 32 columns' four sums, then the warps in order.
constexpr int kReduceWarps = 8;
__global__ void __launch_bounds__(kReduceWarps * 32) residual_norm_reduce_kernel(const ReduceParams p) {
  __shared__ float s[kReduceWarps][kSums][32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float v[kSums] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < p.n)
    for (int r = w; r < p.parts; r += kReduceWarps)
#pragma unroll
      for (int i = 0; i < kSums; ++i) v[i] += __ldcg(p.part + (int64_t(r) * kSums + i) * p.n + c);
#pragma unroll
  for (int i = 0; i < kSums; ++i) s[w][i][lane] = v[i];
  __syncthreads();
  if (w != 0 || c >= p.n) return;
#pragma unroll
  for (int i = 0; i < kSums; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < kReduceWarps; ++k) v[i] += s[k][i][lane];
  }
  const float gate = param_at(p.gate, p.param_f32, int(c), 1.0f);
  auto give = [&](float* to, float g) {
    if (to) to[c] = p.accumulate ? to[c] + g : g;
  };
  give(p.dgate, fmaf(param_at(p.gamma_f, p.param_f32, int(c), 1.0f), v[0], param_at(p.beta_f, p.param_f32, int(c), 0.0f) * v[1]));
  give(p.dgamma_f, gate * v[0]);
  give(p.dbeta_f, gate * v[1]);
  give(p.dgamma_y, v[2]);
  give(p.dbeta_y, v[3]);
}

// ---- host ---------------------------------------------------------------------

int64_t backward_parts(const goldy_residual_norm_desc& d) {
  return std::max<int64_t>(1, std::min<int64_t>(kBwdCtas, d.rows));
}
size_t backward_bytes(const goldy_residual_norm_desc& d) {
  return kLayerCounterBytes + size_t(backward_parts(d)) * kSums * size_t(d.n) * sizeof(float);
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
  ReduceParams r;
  const goldy_residual_norm_desc* d;
  bool backward;
  void* stream;
};

goldy_status launch_residual_norm(const LayerContext& ctx, void* arg) {
  ResidualNormCall& call = *static_cast<ResidualNormCall*>(arg);
  const goldy_residual_norm_desc& d = *call.d;
  const bool f32 = d.dtype == GOLDY_F32;
  void* args[] = {&call.p};
  const void* fn;
  int64_t grid;
  if (call.backward) {
    fn = f32 ? reinterpret_cast<const void*>(&residual_norm_backward_stream_kernel<float>)
             : reinterpret_cast<const void*>(&residual_norm_backward_stream_kernel<uint16_t>);
    grid = backward_parts(d);
  } else {
    fn = f32 ? reinterpret_cast<const void*>(&residual_norm_forward_stream_kernel<float>)
             : reinterpret_cast<const void*>(&residual_norm_forward_stream_kernel<uint16_t>);
    grid = std::min<int64_t>(d.rows, int64_t(ctx.sm_count) * 4);
  }
  const goldy_status st = launch_layer("residual norm", fn, grid, kStreamThreads, 0, call.stream, args);
  if (st != GOLDY_OK || !call.p.part) return st;
  call.r.parts = int32_t(grid);
  void* rargs[] = {&call.r};
  return launch_layer("residual norm", reinterpret_cast<const void*>(&residual_norm_reduce_kernel), ceil_div(d.n, 32),
                      kReduceWarps * 32, 0, call.stream, rargs);
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
  ReduceParams& r = call.r;
  r.part = call.p.part;
  r.gate = given.gate;
  r.gamma_f = given.gamma_f;
  r.beta_f = given.beta_f;
  r.dgate = static_cast<float*>(want.gate);
  r.dgamma_f = static_cast<float*>(want.gamma_f);
  r.dbeta_f = static_cast<float*>(want.beta_f);
  r.dgamma_y = static_cast<float*>(want.gamma_y);
  r.dbeta_y = static_cast<float*>(want.beta_y);
  r.n = int32_t(desc->n);
  r.accumulate = accumulate;
  r.param_f32 = desc->param_dtype == GOLDY_F32;
  call.stream = stream;
  st = with_layer_context(stream, launch_residual_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
