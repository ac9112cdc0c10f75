// Layer norm over the last dimension, forwards and backwards.
//
//   y = (x - mean) rstd gamma + beta,  mean = sum(x) / n,  rstd = 1 / sqrt(sum((x - mean)^2) / n + eps)
//   g = dy gamma, xhat = (x - mean) rstd:
//   dx = rstd (g - sum(g) / n - xhat sum(g xhat) / n),  dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//
// HBM-bound: x (and dy) read once, y (or dx) written once.  A team of threads
// holds a row in registers, 16 values per thread (team of 32 to 512 threads by
// the row's length), so both statistics passes of the forward direction and
// the two sums of the backward direction cost no second read; the next row's
// loads are issued before the current row's sums meet.  gamma and beta stay in
// registers over all rows of a team.  The variance is a sum of squared
// differences from each warp's own mean, warps combined by
// M2 = sum(M2_w + n_w (mean_w - mean)^2): no cancellation, one barrier.
// Backward, each thread owns its columns for all rows of its team and keeps
// dgamma and dbeta in registers; the teams of a CTA combine in shared memory,
// one fp32 partial row per CTA goes to the workspace, and a second small kernel
// sums the partial rows in CTA order.  Nothing depends on the order of arrival.
// Rows over 8192 elements stream through three (two) reads of the row instead.
#include <cuda_runtime.h>

#include <algorithm>
#include <cstring>
#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kVals = 16;           // values of a row per thread
constexpr int kMaxTeam = 512;
constexpr int kStreamThreads = 512;
constexpr int kFwdThreads = 256;    // per CTA, at least the team
constexpr int kBwdThreads = 512;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

__device__ __forceinline__ float param_at(const void* p, int f32, int i, float absent) {
  if (!p) return absent;
  return f32 ? static_cast<const float*>(p)[i] : load_bf16(p, i);
}

// A team's row in registers.  VEC: 16-byte accesses, columns (i * TEAM + t) *
// per + k for the thread's i-th vector of `per` elements; otherwise single
// elements, columns i * TEAM + t.
template <typename T, int TEAM, bool VEC>
struct Row {
  static constexpr int PER = VEC ? 16 / int(sizeof(T)) : 1;
  static constexpr int SLOTS = kVals / PER;
  static __device__ __forceinline__ int col(int slot, int t) { return (slot * TEAM + t) * PER; }

  // raw bits as loaded; converted when the row is used, so that a row in
  // flight takes as few registers as it can
  static constexpr int WORDS = VEC ? SLOTS * 4 : SLOTS;
  uint32_t raw[WORDS];

  __device__ __forceinline__ void load(const void* base, int64_t row, int64_t ld, int n, int t) {
    const T* at = static_cast<const T*>(base) + row * ld;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int c = col(s, t);
      if (VEC) {
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < n) v = __ldcs(reinterpret_cast<const uint4*>(at + c));
        raw[s * 4] = v.x, raw[s * 4 + 1] = v.y, raw[s * 4 + 2] = v.z, raw[s * 4 + 3] = v.w;
      } else {
        raw[s] = 0;
        if (c < n) {
          if (sizeof(T) == 2) raw[s] = uint32_t(reinterpret_cast<const uint16_t*>(at)[c]) << 16;
          else raw[s] = reinterpret_cast<const uint32_t*>(at)[c];
        }
      }
    }
  }
  __device__ __forceinline__ void values(float (&f)[kVals]) const {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      if (!VEC) {
        f[s] = __uint_as_float(raw[s]);
      } else if (sizeof(T) == 2) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f[(s * 4 + k) * 2] = bf16_lo(raw[s * 4 + k]);
          f[(s * 4 + k) * 2 + 1] = bf16_hi(raw[s * 4 + k]);
        }
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[s * 4 + k] = __uint_as_float(raw[s * 4 + k]);
      }
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t row, int64_t ld, int n, int t,
                                               const float (&f)[kVals]) {
    T* at = static_cast<T*>(base) + row * ld;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int c = col(s, t);
      if (c >= n) continue;
      if (!VEC) {
        if (sizeof(T) == 2) store_bf16(at, c, f[s]);
        else reinterpret_cast<float*>(at)[c] = f[s];
      } else if (sizeof(T) == 2) {
        __stcs(reinterpret_cast<uint4*>(at + c),
               make_uint4(pack_bf16(f[s * 8], f[s * 8 + 1]), pack_bf16(f[s * 8 + 2], f[s * 8 + 3]),
                          pack_bf16(f[s * 8 + 4], f[s * 8 + 5]), pack_bf16(f[s * 8 + 6], f[s * 8 + 7])));
      } else {
        __stcs(reinterpret_cast<float4*>(at + c), make_float4(f[s * 4], f[s * 4 + 1], f[s * 4 + 2], f[s * 4 + 3]));
      }
    }
  }
  // columns of this thread inside the row, and of value j
  static __device__ __forceinline__ bool inside(int j, int t, int n) { return col(j / PER, t) + j % PER < n; }
};

// Barrier of one team: a warp needs none, the whole CTA has barrier 0.
template <int TEAM, int THREADS>
__device__ __forceinline__ void team_sync(int team) {
  if (TEAM == 32) __syncwarp();
  else if (TEAM == THREADS) __syncthreads();
  else ptx::named_bar_sync(uint32_t(team + 1), TEAM);
}

template <typename T, int TEAM, bool VEC>
__global__ void __launch_bounds__(TEAM > kFwdThreads ? TEAM : kFwdThreads)
norm_forward_kernel(const NormParams p) {
  constexpr int THREADS = TEAM > kFwdThreads ? TEAM : kFwdThreads;
  constexpr int TEAMS = THREADS / TEAM;
  constexpr int WARPS = TEAM / 32;
  using R = Row<T, TEAM, VEC>;
  __shared__ float4 slot[2][TEAMS][WARPS];         // per warp: sum, M2, elements, mean
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5;
  const int n = p.n;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(gridDim.x) * TEAMS;
  int64_t row = int64_t(blockIdx.x) * TEAMS + team;
  if (row >= p.rows) return;                       // whole teams only
  R next;
  next.load(p.x, row, p.ldx, n, t);
  float gamma[kVals], beta[kVals];
  int mine = 0;                                    // values this thread has
#pragma unroll
  for (int j = 0; j < kVals; ++j) {
    const bool in = R::inside(j, t, n);
    gamma[j] = in ? param_at(p.gamma, p.param_f32, R::col(j / R::PER, t) + j % R::PER, 1.0f) : 0.0f;
    beta[j] = in ? param_at(p.beta, p.param_f32, R::col(j / R::PER, t) + j % R::PER, 0.0f) : 0.0f;
    mine += in;
  }
  const float warp_n = warp_sum(float(mine));
  const float warp_inv = warp_n > 0.0f ? 1.0f / warp_n : 0.0f;
  for (int flip = 0; row < p.rows; row += step, flip ^= 1) {
    float x[kVals];
    next.values(x);
    if (row + step < p.rows) next.load(p.x, row + step, p.ldx, n, t);
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < kVals; ++j) s += x[j];     // zeros outside the row
    s = warp_sum(s);
    const float wm = s * warp_inv;
    float m2 = 0.0f;
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
      const float d = R::inside(j, t, n) ? x[j] - wm : 0.0f;
      m2 = fmaf(d, d, m2);
    }
    m2 = warp_sum(m2);
    float mean = wm;
    if (WARPS > 1) {
      if ((t & 31) == 0) slot[flip][team][w] = make_float4(s, m2, warp_n, wm);
      team_sync<TEAM, THREADS>(team);
      float total = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) total += slot[flip][team][i].x;
      mean = total * p.inv_n;
      m2 = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float4 o = slot[flip][team][i];
        const float d = o.w - mean;
        m2 += fmaf(o.z * d, d, o.y);
      }
    }
    const float rstd = rsqrtf(fmaf(m2, p.inv_n, p.eps));
#pragma unroll
    for (int j = 0; j < kVals; ++j) x[j] = fmaf((x[j] - mean) * rstd, gamma[j], beta[j]);
    R::store(p.out, row, p.ldy, n, t, x);
    if (t == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

template <typename T, int TEAM, bool VEC>
__global__ void __launch_bounds__(kBwdThreads) norm_backward_kernel(const NormParams p) {
  constexpr int TEAMS = kBwdThreads / TEAM;
  constexpr int WARPS = TEAM / 32;
  using R = Row<T, TEAM, VEC>;
  __shared__ float2 slot[2][TEAMS][WARPS];
  extern __shared__ float sums[];                  // [2][TEAM * kVals]
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5;
  const int n = p.n;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(gridDim.x) * TEAMS;
  int64_t row = int64_t(blockIdx.x) * TEAMS + team;
  R nx, ny;
  float mean = 0.0f, rstd = 0.0f;
  auto fetch = [&](int64_t r) {
    nx.load(p.x, r, p.ldx, n, t);
    ny.load(p.dy, r, p.ldy, n, t);
    mean = __ldg(p.mean + r);
    rstd = __ldg(p.rstd + r);
  };
  if (row < p.rows) fetch(row);
  float gamma[kVals], dg[kVals], db[kVals];
#pragma unroll
  for (int j = 0; j < kVals; ++j) {
    gamma[j] = R::inside(j, t, n) ? param_at(p.gamma, p.param_f32, R::col(j / R::PER, t) + j % R::PER, 1.0f) : 0.0f;
    dg[j] = db[j] = 0.0f;
  }
  for (int flip = 0; row < p.rows; row += step, flip ^= 1) {
    float x[kVals], y[kVals];
    nx.values(x);
    ny.values(y);
    const float m = mean, rs = rstd;
    if (row + step < p.rows) fetch(row + step);
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int j = 0; j < kVals; ++j) {
      x[j] = R::inside(j, t, n) ? (x[j] - m) * rs : 0.0f;      // xhat
      dg[j] = fmaf(y[j], x[j], dg[j]);
      db[j] += y[j];
      y[j] *= gamma[j];
      s1 += y[j];
      s2 = fmaf(y[j], x[j], s2);
    }
    s1 = warp_sum(s1);
    s2 = warp_sum(s2);
    if (WARPS > 1) {
      if ((t & 31) == 0) slot[flip][team][w] = make_float2(s1, s2);
      team_sync<TEAM, kBwdThreads>(team);
      s1 = s2 = 0.0f;
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float2 o = slot[flip][team][i];
        s1 += o.x;
        s2 += o.y;
      }
    }
    s1 *= p.inv_n;
    s2 *= p.inv_n;
#pragma unroll
    for (int j = 0; j < kVals; ++j) x[j] = rs * (y[j] - s1 - x[j] * s2);
    R::store(p.out, row, p.ldx, n, t, x);
  }
  if (!p.part) return;
  // teams of the CTA, in order
  for (int k = 0; k < TEAMS; ++k) {
    if (team == k) {
#pragma unroll
      for (int j = 0; j < kVals; ++j) {
        float* a = sums + j * TEAM + t;
        a[0] = k == 0 ? dg[j] : a[0] + dg[j];
        a[TEAM * kVals] = k == 0 ? db[j] : a[TEAM * kVals] + db[j];
      }
    }
    __syncthreads();
  }
  float* to = p.part + int64_t(blockIdx.x) * 2 * n;
  for (int i = threadIdx.x; i < TEAM * kVals; i += kBwdThreads) {
    const int j = i / TEAM, tt = i % TEAM;
    const int c = R::col(j / R::PER, tt) + j % R::PER;
    if (c < n) {
      __stcg(to + c, sums[i]);
      __stcg(to + n + c, sums[TEAM * kVals + i]);
    }
  }
}

// ---- rows that do not fit in a team's registers -------------------------------

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
  a = warp_sum(a);
  b = warp_sum(b);
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

template <typename T>
__global__ void __launch_bounds__(kStreamThreads) norm_forward_stream_kernel(const NormParams p) {
  __shared__ float2 slots[kStreamThreads / 32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const int64_t at = row * p.ldx;
    float s = 0.0f;
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) s += elem<T>(p.x, at + c);
    const float mean = cta_sum(s, 0.0f, slots).x * p.inv_n;
    float m2 = 0.0f;
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
      const float d = elem<T>(p.x, at + c) - mean;
      m2 = fmaf(d, d, m2);
    }
    const float rstd = rsqrtf(fmaf(cta_sum(m2, 0.0f, slots).x, p.inv_n, p.eps));
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads)
      put<T>(p.out, row * p.ldy + c, fmaf((elem<T>(p.x, at + c) - mean) * rstd, param_at(p.gamma, p.param_f32, c, 1.0f),
                                          param_at(p.beta, p.param_f32, c, 0.0f)));
    if (threadIdx.x == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kStreamThreads) norm_backward_stream_kernel(const NormParams p) {
  __shared__ float2 slots[kStreamThreads / 32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  float* part = p.part ? p.part + int64_t(blockIdx.x) * 2 * p.n : nullptr;
  bool first = true;
  for (int64_t row = blockIdx.x; row < p.rows || first; row += gridDim.x) {
    if (row >= p.rows) {                           // a CTA without rows has a zero partial
      for (int c = threadIdx.x; part && c < 2 * p.n; c += kStreamThreads) part[c] = 0.0f;
      break;
    }
    const float m = p.mean[row], rs = p.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
      const float g = elem<T>(p.dy, row * p.ldy + c) * param_at(p.gamma, p.param_f32, c, 1.0f);
      s1 += g;
      s2 = fmaf(g, (elem<T>(p.x, row * p.ldx + c) - m) * rs, s2);
    }
    float2 s = cta_sum(s1, s2, slots);
    s.x *= p.inv_n;
    s.y *= p.inv_n;
    for (int c = threadIdx.x; c < p.n; c += kStreamThreads) {
      const float dy = elem<T>(p.dy, row * p.ldy + c);
      const float xhat = (elem<T>(p.x, row * p.ldx + c) - m) * rs;
      if (part) {                                  // this thread's columns in this CTA's partial row
        part[c] = first ? dy * xhat : fmaf(dy, xhat, part[c]);
        part[p.n + c] = first ? dy : part[p.n + c] + dy;
      }
      put<T>(p.out, row * p.ldx + c, rs * (dy * param_at(p.gamma, p.param_f32, c, 1.0f) - s.x - xhat * s.y));
    }
    first = false;
  }
}

// dgamma and dbeta from the CTAs' partial rows: a warp per 32 columns of the
// 2 n, 8 warps taking every eighth partial row, then the warps in order.
constexpr int kReduceWarps = 8;
__global__ void __launch_bounds__(kReduceWarps * 32)
norm_reduce_kernel(const float* part, float* dgamma, float* dbeta, int n, int rows, int accumulate) {
  __shared__ float s[kReduceWarps][32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float v = 0.0f;
  if (c < 2 * int64_t(n)) {
#pragma unroll 4
    for (int r = w; r < rows; r += kReduceWarps) v += __ldcg(part + int64_t(r) * 2 * n + c);
  }
  s[w][lane] = v;
  __syncthreads();
  if (w != 0 || c >= 2 * int64_t(n)) return;
  v = 0.0f;
#pragma unroll
  for (int i = 0; i < kReduceWarps; ++i) v += s[i][lane];
  float* to = c < n ? dgamma : dbeta;
  if (!to) return;
  to += c < n ? c : c - n;
  *to = accumulate ? *to + v : v;
}

// ---- host ------------------------------------------------------------------------

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
goldy_status bad(const std::string& why) { return fail(GOLDY_ERR_INVALID_ARG, why); }

int team_for(int64_t n) {
  int team = 32;
  while (team < kMaxTeam && int64_t(team) * kVals < n) team *= 2;
  return int64_t(team) * kVals >= n ? team : 0;    // 0: the row streams
}

struct Kernel {
  const void* fn;
  int threads, teams;
  size_t smem;
};

template <typename T, int TEAM, bool VEC>
Kernel pick(bool backward) {
  if (backward)
    return {reinterpret_cast<const void*>(&norm_backward_kernel<T, TEAM, VEC>), kBwdThreads, kBwdThreads / TEAM,
            size_t(2) * TEAM * kVals * sizeof(float)};
  const int threads = std::max(TEAM, kFwdThreads);
  return {reinterpret_cast<const void*>(&norm_forward_kernel<T, TEAM, VEC>), threads, threads / TEAM, 0};
}

template <typename T, bool VEC>
Kernel pick_team(int team, bool backward) {
  switch (team) {
    case 32: return pick<T, 32, VEC>(backward);
    case 64: return pick<T, 64, VEC>(backward);
    case 128: return pick<T, 128, VEC>(backward);
    case 256: return pick<T, 256, VEC>(backward);
    case 512: return pick<T, 512, VEC>(backward);
    default:
      return {backward ? reinterpret_cast<const void*>(&norm_backward_stream_kernel<T>)
                       : reinterpret_cast<const void*>(&norm_forward_stream_kernel<T>),
              kStreamThreads, 1, 0};
  }
}

Kernel kernel_for(const goldy_layernorm_desc& d, bool vec, bool backward) {
  const int team = team_for(d.n);
  if (d.dtype == GOLDY_F32) return vec ? pick_team<float, true>(team, backward) : pick_team<float, false>(team, backward);
  return vec ? pick_team<uint16_t, true>(team, backward) : pick_team<uint16_t, false>(team, backward);
}

// CTAs of a backward launch: one partial row each
constexpr int kBwdCtas = 152;      // one per SM
int backward_ctas(const goldy_layernorm_desc& d) {
  const int team = team_for(d.n);
  const int64_t teams = team ? kBwdThreads / team : 1;
  return int(std::max<int64_t>(1, std::min<int64_t>(kBwdCtas, ceil_div(d.rows, teams))));
}

goldy_status check_norm(const goldy_layernorm_desc* d) {
  if (!d) return bad("null descriptor");
  if (d->rows < 0 || d->n < 0 || d->n > (int64_t(1) << 30)) return bad("layer norm: a size is negative or too large");
  if (d->ldx < d->n || d->ldy < d->n) return bad("layer norm: a row stride is smaller than its row");
  if ((d->dtype != GOLDY_BF16 && d->dtype != GOLDY_F32) || (d->param_dtype != GOLDY_BF16 && d->param_dtype != GOLDY_F32))
    return fail(GOLDY_ERR_UNSUPPORTED, "layer norm: types are GOLDY_BF16 or GOLDY_F32");
  if (!(d->eps >= 0.0f) || d->eps > 1e30f) return bad("layer norm: eps must be finite and not negative");
  if (d->reserved != 0) return bad("layer norm: reserved must be 0");
  return GOLDY_OK;
}

struct NormCall {
  NormParams p;
  const goldy_layernorm_desc* d;
  bool vec, backward;
  float *dgamma, *dbeta;
  int accumulate;
  void* stream;
};

cudaError_t launch(const void* fn, unsigned grid, unsigned threads, size_t smem, void* stream, void** args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelExC(&cfg, fn, args);
}

goldy_status launch_norm(const LayerContext& ctx, void* arg) {
  NormCall& call = *static_cast<NormCall*>(arg);
  const Kernel k = kernel_for(*call.d, call.vec, call.backward);
  cudaError_t e = cudaSuccess;
  if (k.smem > 48 * 1024) e = cudaFuncSetAttribute(k.fn, cudaFuncAttributeMaxDynamicSharedMemorySize, int(k.smem));
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
  unsigned grid;
  if (call.backward) {
    grid = unsigned(backward_ctas(*call.d));
  } else {
    // 2048 threads per SM, every team with rows of its own
    const int64_t cap = int64_t(ctx.sm_count) * (2048 / k.threads);
    grid = unsigned(std::max<int64_t>(1, std::min<int64_t>(cap, ceil_div(call.d->rows, k.teams))));
  }
  void* args[] = {&call.p};
  if (call.d->rows > 0 || call.backward) {
    e = launch(k.fn, grid, unsigned(k.threads), k.smem, call.stream, args);
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("layer norm launch: ") + cudaGetErrorString(e));
  }
  if (call.backward && call.p.part) {
    int n = int(call.d->n), rows = int(grid);
    void* rargs[] = {&call.p.part, &call.dgamma, &call.dbeta, &n, &rows, &call.accumulate};
    e = launch(reinterpret_cast<const void*>(&norm_reduce_kernel), unsigned(ceil_div(2 * call.d->n, 32)),
               kReduceWarps * 32, 0, call.stream, rargs);
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("layer norm launch: ") + cudaGetErrorString(e));
  }
  return GOLDY_OK;
}

// 16-byte accesses: whole vectors in every row (a team's last vector may not
// reach past the row), rows and bases on vector boundaries
bool vectors(const goldy_layernorm_desc& d, const void* a, const void* b, const void* c) {
  const int64_t per = d.dtype == GOLDY_F32 ? 4 : 8;
  return d.n % per == 0 && d.ldx % per == 0 && d.ldy % per == 0 && aligned(a, 16) && aligned(b, 16) && aligned(c, 16);
}

size_t backward_bytes(const goldy_layernorm_desc& d) {
  return kLayerCounterBytes + size_t(backward_ctas(d)) * 2 * size_t(d.n) * sizeof(float);
}

void common_params(NormParams& p, const goldy_layernorm_desc& d) {
  p.ldx = d.ldx;
  p.ldy = d.ldy;
  p.rows = d.rows;
  p.n = int32_t(d.n);
  p.param_f32 = d.param_dtype == GOLDY_F32;
  p.eps = d.eps;
  p.inv_n = float(1.0 / double(d.n));
}

}  // namespace
}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_layernorm_query(const goldy_layernorm_desc* desc, size_t* workspace_bytes) {
  goldy_status st = check_norm(desc);
  if (st != GOLDY_OK) return st;
  if (!workspace_bytes) return bad("null argument");
  *workspace_bytes = desc->n > 0 ? backward_bytes(*desc) : 0;
  return ok();
}

extern "C" goldy_status goldy_layernorm_forward(const goldy_layernorm_desc* desc, const void* X, const void* gamma,
                                                const void* beta, void* Y, float* mean, float* rstd, void* stream) {
  goldy_status st = check_norm(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->n == 0) return ok();
  const size_t es = desc->dtype == GOLDY_F32 ? 4 : 2, ps = desc->param_dtype == GOLDY_F32 ? 4 : 2;
  if (!X || !Y || !aligned(X, es) || !aligned(Y, es)) return bad("layer norm: X or Y null or misaligned");
  if (!aligned(gamma, ps) || !aligned(beta, ps) || !aligned(mean, 4) || !aligned(rstd, 4))
    return bad("layer norm: gamma, beta, mean or rstd misaligned");
  NormCall call{};
  call.d = desc;
  call.vec = vectors(*desc, X, Y, nullptr);
  call.stream = stream;
  common_params(call.p, *desc);
  call.p.x = X;
  call.p.gamma = gamma;
  call.p.beta = beta;
  call.p.out = Y;
  call.p.mean = mean;
  call.p.rstd = rstd;
  st = with_layer_context(stream, launch_norm, &call);
  return st == GOLDY_OK ? ok() : st;
}

extern "C" goldy_status goldy_layernorm_backward(const goldy_layernorm_desc* desc, const void* dY, const void* X,
                                                 const void* gamma, const float* mean, const float* rstd, void* dX,
                                                 float* dgamma, float* dbeta, int accumulate, void* workspace,
                                                 size_t workspace_bytes, void* stream) {
  goldy_status st = check_norm(desc);
  if (st != GOLDY_OK) return st;
  if (accumulate != 0 && accumulate != 1) return bad("layer norm: accumulate must be 0 or 1");
  if (desc->n == 0) return ok();
  const bool sums = dgamma || dbeta;
  if (desc->rows == 0 && !sums) return ok();
  const size_t es = desc->dtype == GOLDY_F32 ? 4 : 2, ps = desc->param_dtype == GOLDY_F32 ? 4 : 2;
  if (desc->rows > 0 && (!X || !dY || !dX || !mean || !rstd))
    return bad("layer norm: X, dY, dX, mean and rstd are needed");
  if (!aligned(X, es) || !aligned(dY, es) || !aligned(dX, es) || !aligned(gamma, ps) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4))
    return bad("layer norm: a pointer is misaligned");
  if (sums) {
    if (!workspace || !aligned(workspace, 256))
      return bad("layer norm: the workspace must be a 256-byte aligned device pointer");
    if (workspace_bytes < backward_bytes(*desc))
      return fail(GOLDY_ERR_NOMEM, "layer norm: workspace of " + std::to_string(workspace_bytes) + " bytes, " +
                                       std::to_string(backward_bytes(*desc)) + " needed");
  }
  NormCall call{};
  call.d = desc;
  call.vec = vectors(*desc, X, dY, dX);
  call.backward = true;
  call.dgamma = dgamma;
  call.dbeta = dbeta;
  call.accumulate = accumulate;
  call.stream = stream;
  common_params(call.p, *desc);
  call.p.x = X;
  call.p.dy = dY;
  call.p.gamma = gamma;
  call.p.out = dX;
  call.p.mean = const_cast<float*>(mean);
  call.p.rstd = const_cast<float*>(rstd);
  call.p.part = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kLayerCounterBytes) : nullptr;
  st = with_layer_context(stream, launch_norm, &call);
  return st == GOLDY_OK ? ok() : st;
}
