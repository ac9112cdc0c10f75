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
#include <initializer_list>
#include <string>
#include <utility>

#include "layer_launch.h"
#include "layer_math.cuh"
#include "norm_launch.h"
#include "norm_rows.cuh"
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
  int32_t cluster;           // CTAs that share a row, each with `seg` of its columns (the last with the rest)
  int32_t seg;
  // the parameters' gradients (backward)
  float* dgate;
  float* dgamma_f;
  float* dbeta_f;
  float* dgamma_y;
  float* dbeta_y;
  int32_t accumulate, parts;
};

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

// ---- rows in registers ----------------------------------------------------------

constexpr int kMaxTeam = 512;
constexpr int kFwdThreads = 256;       // per CTA, at least the team
constexpr int kBwdThreads = 512;
constexpr int kFwdVals = 16;           // values of a row per thread
constexpr int kBwdVals = 8;
constexpr int kFwdDepth = 3;           // rows in a thread's ring
// (backwards a row's F and dS stay until the row after it has come in)
template <typename T> __host__ __device__ constexpr int bwd_depth() { return sizeof(T) == 2 ? 4 : 3; }

// The parameters' gradients of column c from its four sums.
__device__ __forceinline__ void give_gradients(const ResidualNormParams& p, int64_t c, float a, float b, float cc, float d) {
  const float gate = param_at(p.gate, p.param_f32, int(c), 1.0f);
  auto give = [&](float* to, float g) {
    if (to) to[c] = p.accumulate ? to[c] + g : g;
  };
  give(p.dgate, fmaf(param_at(p.gamma_f, p.param_f32, int(c), 1.0f), a, param_at(p.beta_f, p.param_f32, int(c), 0.0f) * b));
  give(p.dgamma_f, gate * a);
  give(p.dbeta_f, gate * b);
  give(p.dgamma_y, cc);
  give(p.dbeta_y, d);
}

template <typename T, int TEAM, bool VEC, bool WIDE>
__global__ void __launch_bounds__(TEAM > kFwdThreads ? TEAM : kFwdThreads, TEAM > kFwdThreads ? 1 : 2)
residual_norm_forward_kernel(const ResidualNormParams p) {
  constexpr int THREADS = TEAM > kFwdThreads ? TEAM : kFwdThreads, TEAMS = THREADS / TEAM, VALS = kFwdVals;
  constexpr int WARPS = TEAM / 32, D = kFwdDepth;
  using R = NormRow<T, VALS, TEAM, THREADS, VEC, WIDE>;
  __shared__ float4 slot[2][2][TEAMS][WARPS];      // per row, norm and warp: sum, M2, elements, mean
  __shared__ float4 part[2][2][WIDE ? kMaxCluster : 1];
  extern __shared__ __align__(16) uint8_t ring[];  // D rows of F, D of X
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  // WIDE: this CTA's n columns from c0 on, of rows that a cluster shares
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0, c0 = WIDE ? rank * p.seg : 0;
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  const T* const f_in = static_cast<const T*>(p.f) + c0;
  const T* const x_in = static_cast<const T*>(p.x) + c0;
  T* const s_out = static_cast<T*>(p.s) + c0;
  T* const y_out = static_cast<T*>(p.y) + c0;
  if (WIDE) ptx::cluster_sync_all();               // the others have started
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(groups) * TEAMS;
  int64_t row = int64_t(group) * TEAMS + team;
  if (row >= p.rows) return;                       // whole teams only
  auto fetch = [&](int d, int64_t r) {
    if (r < p.rows) {
      R::fetch(ring + 2 * d * R::RING_BYTES, f_in, r, p.ldf, n, t);
      R::fetch(ring + (2 * d + 1) * R::RING_BYTES, x_in, r, p.ldx, n, t);
    }
    copy_commit();
  };
#pragma unroll
  for (int d = 0; d < D - 1; ++d) fetch(d, row + d * step);
  // gate * N_f(v) = xhat * a + b: two parameters instead of three
  float a[VALS], b[VALS], gamma[VALS], beta[VALS];
  int mine = 0;                                    // values this thread has
#pragma unroll
  for (int i = 0; i < R::SLOTS; ++i) {
    if (!R::in(i, t, n)) {
#pragma unroll
      for (int k = i * R::PER; k < (i + 1) * R::PER; ++k) a[k] = b[k] = gamma[k] = beta[k] = 0.0f;
      continue;
    }
    const int c = c0 + R::col(i, t), k0 = i * R::PER;
    load_params<R::PER, VEC>(p.gate, p.param_f32, c, c0 + n, 1.0f, gamma + k0);
    load_params<R::PER, VEC>(p.gamma_f, p.param_f32, c, c0 + n, 1.0f, a + k0);
    load_params<R::PER, VEC>(p.beta_f, p.param_f32, c, c0 + n, 0.0f, b + k0);
#pragma unroll
    for (int k = k0; k < k0 + R::PER; ++k) a[k] *= gamma[k], b[k] *= gamma[k];
    load_params<R::PER, VEC>(p.gamma_y, p.param_f32, c, c0 + n, 1.0f, gamma + k0);
    load_params<R::PER, VEC>(p.beta_y, p.param_f32, c, c0 + n, 0.0f, beta + k0);
    mine += R::whole(i, t, n) ? R::PER : n - R::col(i, t);
  }
  const float warp_n = warp_sum(float(mine));
  const float warp_inv = warp_n > 0.0f ? 1.0f / warp_n : 0.0f;
  int at = 0, ahead = D - 1;                       // ring places of this row and of the one fetched now
  for (int flip = 0; row < p.rows; row += step, flip ^= 1) {
    // xhat of the values in v, which are 0 outside the row and stay 0 there
    // (a layer norm's as differences from the warp's mean first)
    auto normalise = [&](int kind, int which, float (&v)[VALS]) {
      if (kind == GOLDY_NORM_NONE) return;
      float s = 0.0f, wm = 0.0f;
      if (kind == GOLDY_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < VALS; ++j) s += v[j];
        s = warp_sum(s);
        wm = s * warp_inv;
#pragma unroll
        for (int i = 0; i < R::SLOTS; ++i) {
          if (!R::in(i, t, n)) continue;
#pragma unroll
          for (int k = 0; k < R::PER; ++k) {
            float& e = v[i * R::PER + k];
            e = R::whole(i, t, n) || R::col(i, t) + k < n ? e - wm : 0.0f;
          }
        }
      }
      float m2 = 0.0f;
#pragma unroll
      for (int j = 0; j < VALS; ++j) m2 = fmaf(v[j], v[j], m2);
      m2 = warp_sum(m2);
      float mean = wm;
      if (WARPS > 1) {
        if (lane == 0) slot[flip][which][team][w] = make_float4(s, m2, warp_n, wm);
        team_sync<TEAM, THREADS>(team);
        const float4 o = slot[flip][which][team][lane & (WARPS - 1)];
        float total = 0.0f;
        if (kind == GOLDY_NORM_LAYER) {
          total = lanes_sum<WARPS>(o.x);
          mean = total * (WIDE ? 1.0f / float(n) : p.inv_n);
        }
        const float d = o.w - mean;
        m2 = lanes_sum<WARPS>(fmaf(o.z * d, d, o.y));
        if (WIDE) {                                // the same once more, over the cluster's CTAs in order
          tell_cluster(part[flip][which], rank, p.cluster, make_float4(total, m2, float(n), mean));
          float all = 0.0f;
          for (int k = 0; k < p.cluster; ++k) all += part[flip][which][k].x;
          mean = all * p.inv_n;
          m2 = 0.0f;
          for (int k = 0; k < p.cluster; ++k) {
            const float4 q = part[flip][which][k];
            const float e = q.w - mean;
            m2 += fmaf(q.z * e, e, q.y);
          }
        }
      }
      const float rstd = rsqrtf(fmaf(m2, p.inv_n, p.eps)), shift = (wm - mean) * rstd;
#pragma unroll
      for (int i = 0; i < R::SLOTS; ++i) {
        if (!R::in(i, t, n)) continue;
#pragma unroll
        for (int j = i * R::PER; j < (i + 1) * R::PER; ++j) v[j] = fmaf(v[j], rstd, shift);
      }
      if (t == 0 && rank == 0 && p.stats) {
        if (kind == GOLDY_NORM_LAYER) p.stats[2 * which * p.rows + row] = mean;
        p.stats[(2 * which + 1) * p.rows + row] = rstd;
      }
    };
    fetch(ahead, row + (D - 1) * step);
    copy_wait<D - 1>();
    if (R::SHIFT) team_sync<TEAM, THREADS>(team);
    float v[VALS], x[VALS];
    R::values(ring + 2 * at * R::RING_BYTES, f_in, row, p.ldf, n, t, v);
    R::values(ring + (2 * at + 1) * R::RING_BYTES, x_in, row, p.ldx, n, t, x);
    // (SHIFT: the ring's place is used again when every piece has been read, which
    // the barriers of the norms make sure of, if there is one)
    if (R::SHIFT && (WARPS == 1 || (p.norm_f == GOLDY_NORM_NONE && p.norm_y == GOLDY_NORM_NONE))) team_sync<TEAM, THREADS>(team);
    at = at + 1 == D ? 0 : at + 1;
    ahead = ahead + 1 == D ? 0 : ahead + 1;
    normalise(p.norm_f, 0, v);
#pragma unroll
    for (int j = 0; j < VALS; ++j) v[j] = fmaf(v[j], a[j], fmaf(p.alpha, x[j], b[j]));
    R::store(s_out, row, p.lds, n, t, v);
    if (p.norm_y == GOLDY_NORM_NONE) continue;
    normalise(p.norm_y, 1, v);
#pragma unroll
    for (int j = 0; j < VALS; ++j) v[j] = fmaf(v[j], gamma[j], beta[j]);
    R::store(y_out, row, p.ldy, n, t, v);
  }
}

// FULL: both norms and dS are there.
template <typename T, int TEAM, bool VEC, bool WIDE, bool FULL>
__global__ void __launch_bounds__(kBwdThreads) residual_norm_backward_kernel(const ResidualNormParams p) {
  constexpr int TEAMS = kBwdThreads / TEAM, WARPS = TEAM / 32, VALS = kBwdVals, D = bwd_depth<T>();
  using R = NormRow<T, VALS, TEAM, kBwdThreads, VEC, WIDE>;
  __shared__ float4 slot[2][TEAMS][WARPS];
  __shared__ float4 part[2][WIDE ? kMaxCluster : 1];
  extern __shared__ __align__(16) uint8_t ring[];  // D rows of F, S, dY and dS each; at the end the CTA's sums
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0, c0 = WIDE ? rank * p.seg : 0;
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  const T* const f_in = static_cast<const T*>(p.f) + c0;
  const T* const s_in = static_cast<const T*>(p.s_in) + c0;
  const T* const dy_in = static_cast<const T*>(p.dy) + c0;
  const T* const ds_in = static_cast<const T*>(p.ds) + c0;
  T* const dx_out = static_cast<T*>(p.s) + c0;
  T* const df_out = static_cast<T*>(p.y) + c0;
  const bool has_y = FULL || p.norm_y != GOLDY_NORM_NONE, has_f = FULL || p.norm_f != GOLDY_NORM_NONE;
  const bool has_ds = FULL || p.ds != nullptr;
  const float layer_f = p.norm_f == GOLDY_NORM_LAYER ? p.inv_n : 0.0f, layer_y = p.norm_y == GOLDY_NORM_LAYER ? p.inv_n : 0.0f;
  if (WIDE) ptx::cluster_sync_all();               // the others have started
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(groups) * TEAMS, row0 = int64_t(group) * TEAMS + team;
  int left = row0 < p.rows ? int((p.rows - row0 - 1) / step) + 1 : 0;    // rows of this team (memory holds fewer than 2^31)
  // pointers run along: of the row fetched next, of the row whose dX and dF are next
  const T* f_at = f_in + row0 * p.ldf;
  const T* s_at = s_in + row0 * p.lds;
  const T* dy_at = dy_in + row0 * p.ldy;
  const T* ds_at = ds_in + row0 * p.lds;
  T* dx_at = dx_out + row0 * p.ldx;
  T* df_at = df_out + row0 * p.ldf;
  const int64_t step_f = step * p.ldf, step_s = step * p.lds, step_y = step * p.ldy, step_x = step * p.ldx;
  auto fetch = [&](int d, bool there) {
    if (there) {
      uint8_t* to = ring + 4 * d * R::RING_BYTES;
      R::fetch(to, f_at, n, t);
      if (has_y) {
        R::fetch(to + R::RING_BYTES, s_at, n, t);
        R::fetch(to + 2 * R::RING_BYTES, dy_at, n, t);
      }
      if (has_ds) R::fetch(to + 3 * R::RING_BYTES, ds_at, n, t);
    }
    f_at += step_f;
    s_at += step_s;
    dy_at += step_y;
    ds_at += step_s;
    copy_commit();
  };
  // a row's statistics, one per lane: mean and rstd of N_f, of N_y
  const int which = lane & 3;
  const bool mine = which == 0 ? p.norm_f == GOLDY_NORM_LAYER : which == 1 ? has_f : which == 2 ? p.norm_y == GOLDY_NORM_LAYER : has_y;
  const float* stats_at = p.stats + which * p.rows + row0;
  auto next_stats = [&](bool there) {
    const float v = mine && there ? *stats_at : float(which & 1);
    stats_at += step;
    return v;
  };
  auto stat = [&](float v, int q) { return __shfl_sync(0xFFFFFFFFu, v, q); };
#pragma unroll
  for (int d = 0; d < D - 1; ++d) fetch(d, left > d);
  float now = next_stats(left > 0), next = next_stats(left > 1);
  // values in pairs: half the instructions
  constexpr int PAIRS = VALS / 2;
  uint64_t gf[PAIRS], gy[PAIRS], sum[kSums][PAIRS];      // gate * gamma_f, gamma_y; 0 outside the row
  {
    float a[VALS], b[VALS], c[VALS];
#pragma unroll
    for (int i = 0; i < R::SLOTS; ++i) {
      const int k0 = i * R::PER, at = c0 + R::col(i, t);
      if (R::in(i, t, n)) {
        load_params<R::PER, VEC>(p.gate, p.param_f32, at, c0 + n, 1.0f, a + k0);
        load_params<R::PER, VEC>(p.gamma_f, p.param_f32, at, c0 + n, 1.0f, b + k0);
        load_params<R::PER, VEC>(p.gamma_y, p.param_f32, at, c0 + n, 1.0f, c + k0);
      } else {
#pragma unroll
        for (int k = k0; k < k0 + R::PER; ++k) a[k] = b[k] = c[k] = 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      gf[j] = mul2(two(a[2 * j], a[2 * j + 1]), two(b[2 * j], b[2 * j + 1]));
      gy[j] = two(c[2 * j], c[2 * j + 1]);
#pragma unroll
      for (int q = 0; q < kSums; ++q) sum[q][j] = two(0.0f);
    }
  }
  // A row takes two sums one after the other: (1) of dY gamma_y and its product
  // with xhat_y, which T needs, (2) of T gate gamma_f and its product with xhat_f,
  // which dF needs.  The second ones of a row and the first ones of the next row
  // are exchanged together: one barrier per row, and each phase has another row's
  // arithmetic beside it.
  uint64_t g[PAIRS], hy[PAIRS], u[PAIRS], h[PAIRS];
  float s1x, s1y, s2x = 0.0f, s2y = 0.0f;          // partial sums, then the rows'
  auto both = [](uint64_t v) {
    const float2 f = apart(v);
    return f.x + f.y;
  };
  float ry = 1.0f;                                 // rstd of N_y of the row that first() has seen
  int64_t row = row0;                              // (SHIFT: whose rows start anywhere)
  auto first = [&](const uint8_t* from, bool there, int64_t r, float st) {
    s1x = s1y = 0.0f;
    if (!has_y || !there) return;
    float v[VALS], d[VALS];
    R::values(from + R::RING_BYTES, R::SHIFT ? s_in + r * p.lds : nullptr, n, t, v);
    R::values(from + 2 * R::RING_BYTES, R::SHIFT ? dy_in + r * p.ldy : nullptr, n, t, d);
    ry = stat(st, 3);
    // the mean is subtracted before the scale: rows far from zero keep their
    // digits; columns outside the row have dY = gamma = 0 and add nothing
    const uint64_t off = two(-stat(st, 2)), scale = two(ry);
    uint64_t a = two(0.0f), b = a;
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      hy[j] = mul2(add2(two(v[2 * j], v[2 * j + 1]), off), scale);
      const uint64_t dy = two(d[2 * j], d[2 * j + 1]);
      sum[2][j] = fma2(dy, hy[j], sum[2][j]);
      sum[3][j] = add2(sum[3][j], dy);
      g[j] = mul2(dy, gy[j]);
      a = add2(a, g[j]);
      b = fma2(g[j], hy[j], b);
    }
    s1x = both(a);
    s1y = both(b);
  };
  auto exchange = [&](int flip) {
    const float4 v = warp_sum4(s1x, s1y, s2x, s2y, lane, WARPS > 1 ? reinterpret_cast<float*>(&slot[flip][team][w]) : nullptr);
    float4 r = v;
    if (WARPS > 1) {
      team_sync<TEAM, kBwdThreads>(team);
      if (WARPS <= 4) {
        r = slot[flip][team][0];
#pragma unroll
        for (int k = 1; k < WARPS; ++k) {
          const float4 o = slot[flip][team][k];
          r.x += o.x, r.y += o.y, r.z += o.z, r.w += o.w;
        }
      } else {
        const float4 o = slot[flip][team][lane & (WARPS - 1)];
        r = make_float4(lanes_sum<WARPS>(o.x), lanes_sum<WARPS>(o.y), lanes_sum<WARPS>(o.z), lanes_sum<WARPS>(o.w));
      }
      if (WIDE) {
        tell_cluster(part[flip], rank, p.cluster, r);
        r = part[flip][0];
        for (int k = 1; k < p.cluster; ++k) {
          const float4 o = part[flip][k];
          r.x += o.x, r.y += o.y, r.z += o.z, r.w += o.w;
        }
      }
    } else if (R::SHIFT) {
      __syncwarp();
    }
    s1x = r.x, s1y = r.y, s2x = r.z, s2y = r.w;
  };
  float last_rf = 0.0f;                            // of the row whose dF is left
  auto finish = [&]() {
    const uint64_t less = two(-s2x * layer_f * last_rf), slope = two(-s2y * p.inv_n * last_rf), scale = two(last_rf);
    float v[VALS];
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      const float2 f = apart(has_f ? fma2(h[j], slope, fma2(u[j], scale, less)) : u[j]);
      v[2 * j] = f.x;
      v[2 * j + 1] = f.y;
    }
    R::store(df_at, n, t, v);
    df_at += step_f;
  };
  int at = 0, ahead = D - 1;
  bool begun = false;
  if (left > 0) {                                  // whole teams, and whole clusters
    copy_wait<D - 2>();
    if (R::SHIFT) team_sync<TEAM, kBwdThreads>(team);
    first(ring, true, row, now);
    exchange(1);
  }
  for (int flip = 0; left > 0; --left, row += step, flip ^= 1) {
    fetch(ahead, left > D - 1);                    // where the row before this one was
    const float later = next_stats(left > 2);
    copy_wait<D - 2>();
    if (R::SHIFT) team_sync<TEAM, kBwdThreads>(team);
    if (begun) finish();
    begun = true;
    // T, dX, and what dF needs
    const uint8_t* from = ring + 4 * at * R::RING_BYTES;
    at = at + 1 == D ? 0 : at + 1;
    ahead = ahead + 1 == D ? 0 : ahead + 1;
    float tt[VALS], v[VALS];
    if (has_ds) {
      R::values(from + 3 * R::RING_BYTES, R::SHIFT ? ds_in + row * p.lds : nullptr, n, t, tt);
    } else {
#pragma unroll
      for (int j = 0; j < VALS; ++j) tt[j] = 0.0f;
    }
    R::values(from, R::SHIFT ? f_in + row * p.ldf : nullptr, n, t, v);
    last_rf = stat(now, 1);
    const uint64_t less = two(-s1x * layer_y * ry), slope = two(-s1y * p.inv_n * ry), by = two(ry);
    const uint64_t off = two(-stat(now, 0)), scale = two(last_rf), alpha = two(p.alpha);
    uint64_t a = two(0.0f), b = a;
#pragma unroll
    for (int j = 0; j < PAIRS; ++j) {
      uint64_t d = two(tt[2 * j], tt[2 * j + 1]);
      if (has_y) d = add2(d, fma2(hy[j], slope, fma2(g[j], by, less)));
      h[j] = mul2(add2(two(v[2 * j], v[2 * j + 1]), off), scale);
      sum[0][j] = fma2(d, h[j], sum[0][j]);
      sum[1][j] = add2(sum[1][j], d);
      u[j] = mul2(d, gf[j]);
      a = add2(a, u[j]);
      b = fma2(u[j], h[j], b);
      const float2 f = apart(mul2(d, alpha));
      tt[2 * j] = f.x;
      tt[2 * j + 1] = f.y;
    }
    s2x = both(a);
    s2y = both(b);
    R::store(dx_at, n, t, tt);
    dx_at += step_x;
    now = next;
    next = later;
    first(ring + 4 * at * R::RING_BYTES, left > 1, row + step, now);
    exchange(flip);
  }
  if (begun) finish();
  if (!p.part) return;
  // the teams' sums go through shared memory, in column order, to be added in
  // team order
  float* sums = reinterpret_cast<float*>(ring);    // [teams][kSums][column]
  constexpr int ALL = TEAM * VALS;
  copy_wait<0>();
  __syncthreads();
#pragma unroll
  for (int i = 0; i < R::SLOTS; ++i)
#pragma unroll
    for (int q = 0; q < kSums; ++q)
#pragma unroll
      for (int k = 0; k < R::PER; ++k) {
        const float2 f = apart(sum[q][(i * R::PER + k) / 2]);
        sums[(team * kSums + q) * ALL + R::col(i, t) + k] = (i * R::PER + k) & 1 ? f.y : f.x;
      }
  __syncthreads();
  float* to = p.part + int64_t(group) * kSums * p.n + c0;
  for (int c = threadIdx.x; c < n; c += kBwdThreads) {
    float v[kSums];
#pragma unroll
    for (int q = 0; q < kSums; ++q) {
      v[q] = 0.0f;
#pragma unroll
      for (int k = 0; k < TEAMS; ++k) v[q] += sums[(k * kSums + q) * ALL + c];
    }
    if (groups > 1) {
#pragma unroll
      for (int q = 0; q < kSums; ++q) __stcg(to + int64_t(q) * p.n + c, v[q]);
    } else {                                       // this CTA's sums are the result
      give_gradients(p, c0 + c, v[0], v[1], v[2], v[3]);
    }
  }
}

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

// Threads per row; 0: the row streams.  `cluster` CTAs of kMaxTeam threads share
// a row that is too long for one.
struct NormShape {
  int team, cluster, seg;
};
NormShape shape_for(const goldy_residual_norm_desc& d, bool backward) {
  const int64_t vals = backward ? kBwdVals : kFwdVals;
  int team = 32;
  while (team < kMaxTeam && team * vals < d.n) team *= 2;
  int cluster = 1;
  while (cluster < kMaxCluster && cluster * team * vals < d.n) cluster *= 2;
  if (cluster * team * vals < d.n) return {0, 1, 0};
  return {team, cluster, int(ceil_div(ceil_div(d.n, cluster), 8) * 8)};     // whole pieces
}

// Partial rows of a backward launch, at most: CTAs, or clusters of them.
int64_t stream_parts(const goldy_residual_norm_desc& d) {
  return std::max<int64_t>(1, std::min<int64_t>(kBwdCtas, d.rows));
}
// Rows per team up to which one CTA does them all: a further kernel that sums
// partial rows costs more.
constexpr int kAloneRows = 2;
int64_t team_parts(const goldy_residual_norm_desc& d, const NormShape& s) {
  const int64_t teams = s.cluster > 1 ? 1 : kBwdThreads / s.team;
  if (d.rows <= kAloneRows * teams) return 1;      // no second kernel
  return std::min<int64_t>(kBwdCtas / s.cluster, ceil_div(d.rows, teams));
}
size_t backward_bytes(const goldy_residual_norm_desc& d) {
  const NormShape s = shape_for(d, true);
  // (inside an SM partition rows stream where clusters would share them)
  const int64_t parts = s.team == 0 || s.cluster > 1 ? stream_parts(d) : team_parts(d, s);
  return kLayerCounterBytes + size_t(parts) * kSums * size_t(d.n) * sizeof(float);
}

template <typename T, int TEAM, bool VEC, bool WIDE = false>
NormKernel pick(bool backward, bool full) {
  if (backward) {
    using R = NormRow<T, kBwdVals, TEAM, kBwdThreads, VEC, WIDE>;
    return {full ? reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, VEC, WIDE, VEC>)
                 : reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, VEC, WIDE, false>), kBwdThreads,
            kBwdThreads / TEAM, 1,
            std::max(size_t(4) * bwd_depth<T>() * R::RING_BYTES, size_t(kSums) * kBwdThreads * kBwdVals * sizeof(float))};
  }
  constexpr int THREADS = TEAM > kFwdThreads ? TEAM : kFwdThreads;
  using R = NormRow<T, kFwdVals, TEAM, THREADS, VEC, WIDE>;
  return {reinterpret_cast<const void*>(&residual_norm_forward_kernel<T, TEAM, VEC, WIDE>), THREADS, THREADS / TEAM,
          TEAM > kFwdThreads ? 1 : 2, size_t(2) * kFwdDepth * R::RING_BYTES};
}
template <typename T, bool VEC>
NormKernel pick_shape(const NormShape& s, bool backward, bool full) {
  if (s.cluster > 1) return pick<T, kMaxTeam, VEC, true>(backward, full);
  switch (s.team) {
    case 32: return pick<T, 32, VEC>(backward, full);
    case 64: return pick<T, 64, VEC>(backward, full);
    case 128: return pick<T, 128, VEC>(backward, full);
    case 256: return pick<T, 256, VEC>(backward, full);
    case 512: return pick<T, 512, VEC>(backward, full);
    default:
      return {backward ? reinterpret_cast<const void*>(&residual_norm_backward_stream_kernel<T>)
                       : reinterpret_cast<const void*>(&residual_norm_forward_stream_kernel<T>),
              kStreamThreads, 1, 4, 0};
  }
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
  bool backward, vec;
  void* stream;
};

goldy_status launch_residual_norm(const LayerContext& ctx, void* arg) {
  ResidualNormCall& call = *static_cast<ResidualNormCall*>(arg);
  const goldy_residual_norm_desc& d = *call.d;
  NormShape shape = shape_for(d, call.backward);
  // which SMs a partition has, and so whether a cluster fits into it, is not known
  if (!ctx.whole && shape.cluster > 1) shape = {0, 1, 0};
  const int cluster = shape.cluster;
  NormKernel k;
  const bool full = call.vec && d.norm_f != GOLDY_NORM_NONE && d.norm_y != GOLDY_NORM_NONE && call.p.ds;
  if (d.dtype == GOLDY_F32)
    k = call.vec ? pick_shape<float, true>(shape, call.backward, full) : pick_shape<float, false>(shape, call.backward, full);
  else
    k = call.vec ? pick_shape<uint16_t, true>(shape, call.backward, full)
                 : pick_shape<uint16_t, false>(shape, call.backward, full);
  cudaError_t e = allow_smem(ctx.device, k);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
  int64_t cap = int64_t(ctx.sm_count) * k.per_sm;              // CTAs, or clusters, resident at once
  if (cluster > 1) {
    int most = 0;
    e = resident_clusters(ctx.device, k, cluster, &most);
    if (e == cudaSuccess && most < 1) e = cudaErrorInvalidClusterSize;
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("residual norm, clusters: ") + cudaGetErrorString(e));
    cap = std::min<int64_t>(cap / cluster, most);
  }
  // all resident, every team with rows of its own
  int64_t groups = std::min(cap, ceil_div(d.rows, int64_t(k.teams)));
  if (call.backward) groups = shape.team == 0 ? stream_parts(d) : team_parts(d, shape);
  if (cluster > 1) groups = std::min(groups, cap);
  groups = std::max<int64_t>(1, groups);
  call.p.cluster = cluster;
  call.p.seg = shape.seg;
  call.p.parts = int32_t(groups);
  void* args[] = {&call.p};
  e = NormLaunch(unsigned(groups * cluster), unsigned(k.threads), k.smem, call.stream, unsigned(cluster)).run(k.fn, args);
  if (e == cudaSuccess && call.p.part && (groups > 1 || shape.team == 0))
    e = NormLaunch(unsigned(ceil_div(d.n, 32)), kSums * kReduceWarps * 32, 0, call.stream)
            .run(reinterpret_cast<const void*>(&residual_norm_reduce_kernel), args);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("residual norm launch: ") + cudaGetErrorString(e));
  return GOLDY_OK;
}

// 16-byte accesses: whole vectors in every row, rows, bases and parameters on
// vector boundaries
bool whole_vectors(const goldy_residual_norm_desc& d, const goldy_residual_norm_params& given,
                   std::initializer_list<std::pair<const void*, int64_t>> arrays) {
  const int64_t per = d.dtype == GOLDY_F32 ? 4 : 8;
  if (d.n % per != 0) return false;
  for (const auto& a : arrays)
    if (a.first && (!on_boundary(a.first, 16) || a.second % per != 0)) return false;
  for (const void* q : {given.gate, given.gamma_f, given.beta_f, given.gamma_y, given.beta_y})
    if (!on_boundary(q, 16)) return false;
  return true;
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
  call.vec = whole_vectors(*desc, given, {{X, desc->ldx}, {F, desc->ldf}, {S, desc->lds}, {Y, desc->ldy}});
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
  call.vec = whole_vectors(*desc, given, {{dY, desc->ldy}, {dS, desc->lds}, {F, desc->ldf}, {dY ? S : nullptr, desc->lds},
                                          {dX, desc->ldx}, {dF, desc->ldf}});
  call.stream = stream;
  st = with_layer_context(stream, launch_residual_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
