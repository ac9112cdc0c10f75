// Layer norm over the last dimension, forwards and backwards.
//
//   y = (x - mean) rstd gamma + beta,  mean = sum(x) / n,  rstd = 1 / sqrt(sum((x - mean)^2) / n + eps)
//   g = dy gamma, xhat = (x - mean) rstd:
//   dx = rstd (g - sum(g) / n - xhat sum(g xhat) / n),  dgamma = sum over rows of dy xhat,  dbeta = sum over rows of dy
//
// HBM-bound: x (and dy) read once, y (or dx) written once.  A team of 32 to 512
// threads, by the row's length, holds a row in registers (16 or 32 values per
// thread), so both statistics passes of the forward direction and the two sums of
// the backward direction cost no second read.  The next rows are on their way
// meanwhile: each thread copies its own pieces into shared memory with cp.async
// and reads back only those, so that rows in flight take no registers and need no
// barrier (but for bf16 rows off 16-byte boundaries, see NormRow).  gamma and beta
// stay in registers.
// The variance is a sum of squared differences from each warp's own mean,
// warps combined by M2 = sum(M2_w + n_w (mean_w - mean)^2): no cancellation,
// one barrier per row.  Backward, each thread owns its columns for all rows of
// its team and keeps dgamma and dbeta in registers; the teams of a CTA combine
// in shared memory, one fp32 partial row per CTA goes to the workspace, and a
// second small kernel sums the partial rows in CTA order.  Nothing depends on
// the order of arrival.  Rows too long for a team are shared by a cluster of 2 to
// 8 CTAs, which exchange their statistics through distributed shared memory,
// one cluster barrier per row (8192 rows of 12288, bf16: backwards 187 us, and
// 1176 when such rows streamed; 2048 rows of 65536 forwards 154 and 471 us);
// rows too long for 8 CTAs (131072 elements, backwards 65536), and those of
// clusters inside an SM partition, stream through three (two) reads instead.
#include <cuda_runtime.h>

#include <algorithm>
#include <string>

#include "goldy_internal.h"
#include "layer_internal.h"
#include "layer_math.cuh"
#include "norm_launch.h"
#include "norm_rows.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kMaxTeam = 512;
constexpr int kStreamThreads = 512;
constexpr int kFwdThreads = 256;    // per CTA, at least the team
constexpr int kBwdThreads = 512;
// Values of a row per thread: 16 up to 256 threads (4096 values; 16384 rows of
// 4096 take 44 us, with 32 values 50), then 32 (8192 rows of 8192: 44 us, with
// 16 values and 512 threads 55).
constexpr int kFwdVals = 16, kFwdMoreVals = 32;
constexpr int kFwdTeam = 256;
constexpr int kBwdVals = 16;
constexpr int kFwdDepth = 3;        // rows in a thread's ring
// CTAs of a backward launch: one partial row each
constexpr int kBwdCtas = 152;      // one per SM
template <typename T> __host__ __device__ constexpr int bwd_depth() { return sizeof(T) == 2 ? 3 : 2; }

template <int TEAM, int VALS, bool VEC>
struct FwdShape {
  static constexpr int THREADS = TEAM > kFwdThreads ? TEAM : kFwdThreads;
  static constexpr int TEAMS = THREADS / TEAM;
  static constexpr int CTAS = VALS > 16 || !VEC ? 512 / THREADS : 3;   // per SM, by registers
};

template <typename T, int TEAM, int VALS, bool VEC, bool WIDE>
__global__ void __launch_bounds__(FwdShape<TEAM, VALS, VEC>::THREADS, FwdShape<TEAM, VALS, VEC>::CTAS)
norm_forward_kernel(const NormParams p) {
  constexpr int THREADS = FwdShape<TEAM, VALS, VEC>::THREADS, TEAMS = FwdShape<TEAM, VALS, VEC>::TEAMS;
  constexpr int WARPS = TEAM / 32, D = kFwdDepth;
  using R = NormRow<T, VALS, TEAM, THREADS, VEC, WIDE>;
  __shared__ float4 slot[2][TEAMS][WARPS];         // per warp: sum, M2, elements, mean
  __shared__ float4 part[2][WIDE ? kMaxCluster : 1];   // per CTA of the cluster: the same
  extern __shared__ __align__(16) uint8_t ring[];
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  // WIDE: this CTA's n columns from c0 on, of rows that a cluster shares
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0, c0 = WIDE ? rank * p.seg : 0;
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  const T* const in = static_cast<const T*>(p.x) + c0;
  T* const out = static_cast<T*>(p.out) + c0;
  if (WIDE) ptx::cluster_sync_all();               // the others have started
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(groups) * TEAMS;
  int64_t row = int64_t(group) * TEAMS + team;
  if (row >= p.rows) return;                       // whole teams only
#pragma unroll
  for (int d = 0; d < D - 1; ++d) {
    if (row + d * step < p.rows) R::fetch(ring + d * R::RING_BYTES, in, row + d * step, p.ldx, n, t);
    copy_commit();
  }
  float gamma[VALS], beta[VALS];
  int mine = 0;                                    // values this thread has
#pragma unroll
  for (int i = 0; i < R::SLOTS; ++i) {
    if (!R::in(i, t, n)) continue;
    load_params<R::PER, VEC>(p.gamma, p.param_f32, c0 + R::col(i, t), c0 + n, 1.0f, gamma + i * R::PER);
    load_params<R::PER, VEC>(p.beta, p.param_f32, c0 + R::col(i, t), c0 + n, 0.0f, beta + i * R::PER);
    mine += R::whole(i, t, n) ? R::PER : n - R::col(i, t);
  }
  const float warp_n = warp_sum(float(mine));
  const float warp_inv = warp_n > 0.0f ? 1.0f / warp_n : 0.0f;
  int at = 0, ahead = D - 1;                       // ring places of this row and of the one fetched now
  for (int flip = 0; row < p.rows; row += step, flip ^= 1) {
    if (row + (D - 1) * step < p.rows) R::fetch(ring + ahead * R::RING_BYTES, in, row + (D - 1) * step, p.ldx, n, t);
    copy_commit();
    copy_wait<D - 1>();
    if (R::SHIFT) team_sync<TEAM, THREADS>(team);
    float x[VALS];
    R::values(ring + at * R::RING_BYTES, in, row, p.ldx, n, t, x);
    at = at + 1 == D ? 0 : at + 1;
    ahead = ahead + 1 == D ? 0 : ahead + 1;
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < VALS; ++j) s += x[j];      // zeros outside the row
    s = warp_sum(s);
    const float wm = s * warp_inv;
    float m2 = 0.0f;
#pragma unroll
    for (int i = 0; i < R::SLOTS; ++i) {
      if (!R::in(i, t, n)) continue;
      if (!R::whole(i, t, n)) {
#pragma unroll
        for (int k = 0; k < R::PER; ++k)
          if (R::col(i, t) + k >= n) x[i * R::PER + k] = wm;
      }
#pragma unroll
      for (int k = 0; k < R::PER; ++k) {
        x[i * R::PER + k] -= wm;                   // differences from the warp's mean from here on
        m2 = fmaf(x[i * R::PER + k], x[i * R::PER + k], m2);
      }
    }
    m2 = warp_sum(m2);
    float mean = wm;
    if (WARPS > 1) {
      if (lane == 0) slot[flip][team][w] = make_float4(s, m2, warp_n, wm);
      team_sync<TEAM, THREADS>(team);
      const float4 o = slot[flip][team][lane & (WARPS - 1)];
      const float total = lanes_sum<WARPS>(o.x);
      mean = total * (WIDE ? 1.0f / float(n) : p.inv_n);
      const float d = o.w - mean;
      m2 = lanes_sum<WARPS>(fmaf(o.z * d, d, o.y));
      if (WIDE) {                                  // the same once more, over the cluster's CTAs in order
        tell_cluster(part[flip], rank, p.cluster, make_float4(total, m2, float(n), mean));
        float all = 0.0f;
        for (int k = 0; k < p.cluster; ++k) all += part[flip][k].x;
        mean = all * p.inv_n;
        m2 = 0.0f;
        for (int k = 0; k < p.cluster; ++k) {
          const float4 o = part[flip][k];
          const float d = o.w - mean;
          m2 += fmaf(o.z * d, d, o.y);
        }
      }
    }
    const float rstd = rsqrtf(fmaf(m2, p.inv_n, p.eps));
    const float shift = (wm - mean) * rstd;
#pragma unroll
    for (int i = 0; i < R::SLOTS; ++i) {
      if (!R::in(i, t, n)) continue;
#pragma unroll
      for (int j = i * R::PER; j < (i + 1) * R::PER; ++j) x[j] = fmaf(fmaf(x[j], rstd, shift), gamma[j], beta[j]);
    }
    R::store(out, row, p.ldy, n, t, x);
    if (t == 0 && rank == 0) {
      if (p.mean) p.mean[row] = mean;
      if (p.rstd) p.rstd[row] = rstd;
    }
  }
}

template <typename T, int TEAM, bool VEC, bool WIDE>
__global__ void __launch_bounds__(kBwdThreads) norm_backward_kernel(const NormParams p) {
  constexpr int TEAMS = kBwdThreads / TEAM, WARPS = TEAM / 32, VALS = kBwdVals, D = bwd_depth<T>();
  using R = NormRow<T, VALS, TEAM, kBwdThreads, VEC, WIDE>;
  __shared__ float2 slot[2][TEAMS][WARPS];
  __shared__ float4 part[2][WIDE ? kMaxCluster : 1];
  extern __shared__ __align__(16) uint8_t ring[];  // D rows of x, D of dy; at the end the CTA's sums
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0, c0 = WIDE ? rank * p.seg : 0;
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  const T* const in = static_cast<const T*>(p.x) + c0;
  const T* const dy = static_cast<const T*>(p.dy) + c0;
  T* const out = static_cast<T*>(p.out) + c0;
  if (WIDE) ptx::cluster_sync_all();               // the others have started
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(groups) * TEAMS;
  int64_t row = int64_t(group) * TEAMS + team;
  auto fetch = [&](int d, int64_t r) {
    if (r < p.rows) {
      R::fetch(ring + 2 * d * R::RING_BYTES, in, r, p.ldx, n, t);
      R::fetch(ring + (2 * d + 1) * R::RING_BYTES, dy, r, p.ldy, n, t);
    }
    copy_commit();
  };
#pragma unroll
  for (int d = 0; d < D - 1; ++d) fetch(d, row + d * step);
  float mean = 0.0f, rstd = 0.0f;
  if (row < p.rows) {
    mean = p.mean[row];
    rstd = p.rstd[row];
  }
  // in pairs (8192 rows of 8192: 75 us; one by one 89, at 24 instructions per
  // element); columns outside the row have dy = gamma = 0 and add nothing
  uint64_t gamma[VALS / 2], dg2[VALS / 2], db2[VALS / 2];
  {
    float f[VALS];
#pragma unroll
    for (int i = 0; i < R::SLOTS; ++i) {
      if (R::in(i, t, n)) {
        load_params<R::PER, VEC>(p.gamma, p.param_f32, c0 + R::col(i, t), c0 + n, 1.0f, f + i * R::PER);
      } else {
#pragma unroll
        for (int k = 0; k < R::PER; ++k) f[i * R::PER + k] = 0.0f;
      }
    }
#pragma unroll
    for (int j = 0; j < VALS / 2; ++j) {
      gamma[j] = two(f[2 * j], f[2 * j + 1]);
      dg2[j] = db2[j] = two(0.0f);
    }
  }
  int at = 0, ahead = D - 1;
  for (int flip = 0; row < p.rows; row += step, flip ^= 1) {
    fetch(ahead, row + (D - 1) * step);
    const float m = mean, rs = rstd;
    if (row + step < p.rows) {
      mean = p.mean[row + step];
      rstd = p.rstd[row + step];
    }
    copy_wait<D - 1>();
    if (R::SHIFT) team_sync<TEAM, kBwdThreads>(team);
    float x[VALS], y[VALS];
    R::values(ring + 2 * at * R::RING_BYTES, in, row, p.ldx, n, t, x);
    R::values(ring + (2 * at + 1) * R::RING_BYTES, dy, row, p.ldy, n, t, y);
    at = at + 1 == D ? 0 : at + 1;
    ahead = ahead + 1 == D ? 0 : ahead + 1;
    // xhat = (x - mean) rstd: in fma(x, rstd, -mean * rstd) the rounding of
    // mean * rstd would enter every element (a row 2000 deviations from zero:
    // gamma's gradient off by 1e-4 of its terms).  The mean is subtracted first;
    // rows that a cluster shares add what that rounding took instead, as exact and
    // as many instructions, for which the compiler finds the better schedule (8192
    // rows of 12288, bf16: 187 us, subtracted first 258; 4096 of 32768: 232, 311)
    const float mr = m * rs;
    const uint64_t scale = two(rs), off = two(WIDE ? -mr : -m), lost = two(fmaf(-m, rs, mr));
    uint64_t xhat[VALS / 2], g[VALS / 2], sum1 = two(0.0f), sum2 = sum1;
#pragma unroll
    for (int j = 0; j < VALS / 2; ++j) {
      const uint64_t v = two(x[2 * j], x[2 * j + 1]);
      xhat[j] = WIDE ? add2(fma2(v, scale, off), lost) : mul2(add2(v, off), scale);
      const uint64_t d = two(y[2 * j], y[2 * j + 1]);
      dg2[j] = fma2(d, xhat[j], dg2[j]);
      db2[j] = add2(db2[j], d);
      g[j] = mul2(d, gamma[j]);
      sum1 = add2(sum1, g[j]);
      sum2 = fma2(g[j], xhat[j], sum2);
    }
    const float2 a1 = apart(sum1), a2 = apart(sum2);
    const float both = warp_sum2(a1.x + a1.y, a2.x + a2.y, lane);
    float s1, s2;
    if (WARPS == 1) {
      s1 = __shfl_sync(0xFFFFFFFFu, both, 0);
      s2 = __shfl_sync(0xFFFFFFFFu, both, 16);
    } else {
      if ((lane & 15) == 0) reinterpret_cast<float*>(&slot[flip][team][w])[lane >> 4] = both;
      team_sync<TEAM, kBwdThreads>(team);
      if (WARPS <= 4) {
        s1 = s2 = 0.0f;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
          s1 += slot[flip][team][k].x;
          s2 += slot[flip][team][k].y;
        }
      } else {
        const float2 o = slot[flip][team][lane & (WARPS - 1)];
        s1 = lanes_sum<WARPS>(o.x);
        s2 = lanes_sum<WARPS>(o.y);
      }
      if (WIDE) {
        tell_cluster(part[flip], rank, p.cluster, make_float4(s1, s2, 0.0f, 0.0f));
        s1 = s2 = 0.0f;
        for (int k = 0; k < p.cluster; ++k) {
          s1 += part[flip][k].x;
          s2 += part[flip][k].y;
        }
      }
    }
    const uint64_t less = two(-s1 * p.inv_n * rs), slope = two(-s2 * p.inv_n * rs);
#pragma unroll
    for (int j = 0; j < VALS / 2; ++j) {
      const float2 v = apart(fma2(xhat[j], slope, fma2(g[j], scale, less)));
      x[2 * j] = v.x;
      x[2 * j + 1] = v.y;
    }
    R::store(out, row, p.ldx, n, t, x);
  }
  if (!p.part) return;
  // the teams' sums go through shared memory, in column order, to be added in
  // team order
  float* sums = reinterpret_cast<float*>(ring);    // [teams][dgamma, dbeta][column]
  constexpr int ALL = TEAM * VALS;
  copy_wait<0>();
  __syncthreads();
  float dg[VALS], db[VALS];
#pragma unroll
  for (int j = 0; j < VALS / 2; ++j) {
    const float2 a = apart(dg2[j]), b = apart(db2[j]);
    dg[2 * j] = a.x, dg[2 * j + 1] = a.y, db[2 * j] = b.x, db[2 * j + 1] = b.y;
  }
#pragma unroll
  for (int i = 0; i < R::SLOTS; ++i) {
    float* at = sums + team * 2 * ALL + R::col(i, t);
    if (R::PER == 1) {
      at[0] = dg[i];
      at[ALL] = db[i];
    } else {
#pragma unroll
      for (int k = 0; k < R::PER; k += 4) {
        const int j = i * R::PER + k;
        *reinterpret_cast<float4*>(at + k) = make_float4(dg[j], dg[(j + 1) % VALS], dg[(j + 2) % VALS], dg[(j + 3) % VALS]);
        *reinterpret_cast<float4*>(at + ALL + k) = make_float4(db[j], db[(j + 1) % VALS], db[(j + 2) % VALS], db[(j + 3) % VALS]);
      }
    }
  }
  __syncthreads();
  float* to = p.part + int64_t(group) * 2 * p.n + c0;
#pragma unroll 4
  for (int c = threadIdx.x; c < n; c += kBwdThreads) {
    float g = 0.0f, b = 0.0f;
#pragma unroll
    for (int k = 0; k < TEAMS; ++k) {
      g += sums[k * 2 * ALL + c];
      b += sums[k * 2 * ALL + ALL + c];
    }
    if (groups > 1) {
      __stcg(to + c, g);
      __stcg(to + p.n + c, b);
    } else {                                       // this CTA's sums are the result
      if (p.dgamma) p.dgamma[c0 + c] = p.accumulate ? p.dgamma[c0 + c] + g : g;
      if (p.dbeta) p.dbeta[c0 + c] = p.accumulate ? p.dbeta[c0 + c] + b : b;
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
      for (int64_t c = threadIdx.x; part && c < 2 * int64_t(p.n); c += kStreamThreads) part[c] = 0.0f;
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
constexpr int kReduceRows = (kBwdCtas + kReduceWarps - 1) / kReduceWarps;
__global__ void __launch_bounds__(kReduceWarps * 32)
norm_reduce_kernel(const float* part, float* dgamma, float* dbeta, int n, int rows, int accumulate) {
  __shared__ float s[kReduceWarps][32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t c = int64_t(blockIdx.x) * 32 + lane;
  float v = 0.0f;
  if (c < 2 * int64_t(n)) {
    // all of a warp's rows in flight together (a loop's remainder would wait
    // for them one by one: 8 us for 152 rows instead of 4)
    for (int r0 = w; r0 < rows; r0 += kReduceRows * kReduceWarps) {
      float t[kReduceRows];
#pragma unroll
      for (int i = 0; i < kReduceRows; ++i) {
        const int r = r0 + i * kReduceWarps;
        t[i] = r < rows ? __ldcg(part + int64_t(r) * 2 * n + c) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kReduceRows; ++i) v += t[i];
    }
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

// Threads per row at 16 values each (forwards, more than kFwdTeam stand for half
// as many with 32); 0: the row streams.  `cluster` CTAs of kMaxTeam threads
// share a row that is too long for one.
struct NormShape {
  int team, cluster, seg;
};
NormShape shape_for(const goldy_layernorm_desc& d, bool backward) {
  const int most = backward ? kMaxTeam : 2 * kMaxTeam;
  const int64_t vals = backward ? kBwdVals : kFwdVals;
  int team = 32;
  while (team < most && team * vals < d.n) team *= 2;
  int cluster = 1;
  while (cluster < kMaxCluster && cluster * team * vals < d.n) cluster *= 2;
  if (cluster * team * vals < d.n) return {0, 1, 0};
  const int64_t seg = ceil_div(ceil_div(d.n, cluster), 8) * 8;     // whole pieces
  return {team, cluster, int(seg)};
}

template <typename T, int TEAM, int VALS, bool VEC, bool WIDE = false>
NormKernel pick_forward() {
  using S = FwdShape<TEAM, VALS, VEC>;
  using R = NormRow<T, VALS, TEAM, S::THREADS, VEC, WIDE>;
  return {reinterpret_cast<const void*>(&norm_forward_kernel<T, TEAM, VALS, VEC, WIDE>), S::THREADS, S::TEAMS, S::CTAS,
          size_t(kFwdDepth) * R::RING_BYTES};
}
template <typename T, int TEAM, bool VEC, bool WIDE = false>
NormKernel pick_backward() {
  using R = NormRow<T, kBwdVals, TEAM, kBwdThreads, VEC, WIDE>;
  return {reinterpret_cast<const void*>(&norm_backward_kernel<T, TEAM, VEC, WIDE>), kBwdThreads, kBwdThreads / TEAM, 1,
          std::max(size_t(2) * bwd_depth<T>() * R::RING_BYTES, size_t(2) * kBwdThreads * kBwdVals * sizeof(float))};
}

template <typename T, int TEAM, bool VEC>
NormKernel pick(bool backward) {
  if (backward) return pick_backward<T, TEAM, VEC>();
  if constexpr (TEAM > kFwdTeam) return pick_forward<T, TEAM / 2, kFwdMoreVals, VEC>();
  else return pick_forward<T, TEAM, kFwdVals, VEC>();
}

template <typename T, bool VEC>
NormKernel pick_shape(const NormShape& s, bool backward) {
  if (s.cluster > 1)
    return backward ? pick_backward<T, kMaxTeam, VEC, true>() : pick_forward<T, kMaxTeam, kFwdMoreVals, VEC, true>();
  switch (s.team) {
    case 32: return pick<T, 32, VEC>(backward);
    case 64: return pick<T, 64, VEC>(backward);
    case 128: return pick<T, 128, VEC>(backward);
    case 256: return pick<T, 256, VEC>(backward);
    case 512: return pick<T, 512, VEC>(backward);
    case 2 * kMaxTeam: return pick_forward<T, kMaxTeam, kFwdMoreVals, VEC>();
    default:
      return {backward ? reinterpret_cast<const void*>(&norm_backward_stream_kernel<T>)
                       : reinterpret_cast<const void*>(&norm_forward_stream_kernel<T>),
              kStreamThreads, 1, 4, 0};
  }
}

NormKernel kernel_for(const goldy_layernorm_desc& d, const NormShape& s, bool vec, bool backward) {
  if (d.dtype == GOLDY_F32) return vec ? pick_shape<float, true>(s, backward) : pick_shape<float, false>(s, backward);
  return vec ? pick_shape<uint16_t, true>(s, backward) : pick_shape<uint16_t, false>(s, backward);
}

// Rows per team up to which one CTA does them all: a further kernel that sums
// partial rows costs 3.4 us, a further row of a team about 1.
constexpr int kAloneRows = 3;
// CTAs, or clusters of them, of a backward launch
int backward_groups(const goldy_layernorm_desc& d) {
  const NormShape s = shape_for(d, true);
  if (s.team == 0) return int(std::max<int64_t>(1, std::min<int64_t>(kBwdCtas, d.rows)));
  const int64_t teams = s.cluster > 1 ? 1 : kBwdThreads / s.team;
  if (d.rows <= kAloneRows * teams) return 1;      // no second kernel
  return int(std::min<int64_t>(kBwdCtas / s.cluster, ceil_div(d.rows, teams)));
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
  NormShape shape;
  void* stream;
};

goldy_status launch_norm(const LayerContext& ctx, void* arg) {
  NormCall& call = *static_cast<NormCall*>(arg);
  // which SMs a partition has, and so whether a cluster fits into it, is not known
  if (!ctx.whole && call.shape.cluster > 1) call.shape = {0, 1, 0};
  const int cluster = call.shape.cluster;
  const NormKernel k = kernel_for(*call.d, call.shape, call.vec, call.backward);
  cudaError_t e = allow_smem(ctx.device, k);
  if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
  int64_t cap = int64_t(ctx.sm_count) * k.per_sm;              // CTAs, or clusters, resident at once
  if (cluster > 1) {
    int most = 0;
    e = resident_clusters(ctx.device, k, cluster, &most);
    if (e == cudaSuccess && most < 1) e = cudaErrorInvalidClusterSize;
    if (e != cudaSuccess)
      return fail(GOLDY_ERR_CUDA, std::string("layer norm, clusters: ") + cudaGetErrorString(e));
    cap = std::min<int64_t>(cap / cluster, most);
  }
  // all resident, every team with rows of its own
  int64_t groups = call.backward ? backward_groups(*call.d) : std::min(cap, ceil_div(call.d->rows, int64_t(k.teams)));
  if (cluster > 1) groups = std::min(groups, cap);
  groups = std::max<int64_t>(1, groups);
  void* args[] = {&call.p};
  if (call.d->rows > 0 || call.backward) {
    e = NormLaunch(unsigned(groups * cluster), unsigned(k.threads), k.smem, call.stream, unsigned(cluster)).run(k.fn, args);
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("layer norm launch: ") + cudaGetErrorString(e));
  }
  if (call.backward && call.p.part && (groups > 1 || call.shape.team == 0)) {
    int n = int(call.d->n), rows = int(groups);
    void* rargs[] = {&call.p.part, &call.p.dgamma, &call.p.dbeta, &n, &rows, &call.p.accumulate};
    e = NormLaunch(unsigned(ceil_div(2 * call.d->n, 32)), kReduceWarps * 32, 0, call.stream)
            .run(reinterpret_cast<const void*>(&norm_reduce_kernel), rargs);
    if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("layer norm launch: ") + cudaGetErrorString(e));
  }
  return GOLDY_OK;
}

// 16-byte accesses: whole vectors in every row (a team's last vector may not
// reach past the row), rows and bases on vector boundaries
bool vectors(const goldy_layernorm_desc& d, const void* a, const void* b, const void* c, const void* gamma,
             const void* beta) {
  const int64_t per = d.dtype == GOLDY_F32 ? 4 : 8;
  return d.n % per == 0 && d.ldx % per == 0 && d.ldy % per == 0 && aligned(a, 16) && aligned(b, 16) && aligned(c, 16) &&
         aligned(gamma, 16) && aligned(beta, 16);
}

size_t backward_bytes(const goldy_layernorm_desc& d) {
  return kLayerCounterBytes + size_t(backward_groups(d)) * 2 * size_t(d.n) * sizeof(float);
}

void common_params(NormParams& p, const goldy_layernorm_desc& d, const NormShape& s) {
  p.cluster = s.cluster;
  p.seg = s.seg;
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

extern "C" goldy_status goldy_layernorm_query(const goldy_layernorm_desc* desc, size_t* workspace_bytes) try {
  goldy_status st = check_norm(desc);
  if (st != GOLDY_OK) return st;
  if (!workspace_bytes) return bad("null argument");
  *workspace_bytes = desc->n > 0 ? backward_bytes(*desc) : 0;
  return ok();
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_layernorm_forward(const goldy_layernorm_desc* desc, const void* X, const void* gamma,
                                                const void* beta, void* Y, float* mean, float* rstd, void* stream) try {
  goldy_status st = check_norm(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->n == 0) return ok();
  const size_t es = desc->dtype == GOLDY_F32 ? 4 : 2, ps = desc->param_dtype == GOLDY_F32 ? 4 : 2;
  if (!X || !Y || !aligned(X, es) || !aligned(Y, es)) return bad("layer norm: X or Y null or misaligned");
  if (!aligned(gamma, ps) || !aligned(beta, ps) || !aligned(mean, 4) || !aligned(rstd, 4))
    return bad("layer norm: gamma, beta, mean or rstd misaligned");
  NormCall call{};
  call.d = desc;
  call.vec = vectors(*desc, X, Y, nullptr, gamma, beta);
  call.shape = shape_for(*desc, false);
  call.stream = stream;
  common_params(call.p, *desc, call.shape);
  call.p.x = X;
  call.p.gamma = gamma;
  call.p.beta = beta;
  call.p.out = Y;
  call.p.mean = mean;
  call.p.rstd = rstd;
  st = with_layer_context(stream, launch_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_layernorm_backward(const goldy_layernorm_desc* desc, const void* dY, const void* X,
                                                 const void* gamma, const float* mean, const float* rstd, void* dX,
                                                 float* dgamma, float* dbeta, int accumulate, void* workspace,
                                                 size_t workspace_bytes, void* stream) try {
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
  call.vec = vectors(*desc, X, dY, dX, gamma, nullptr);
  call.shape = shape_for(*desc, true);
  call.backward = true;
  call.stream = stream;
  common_params(call.p, *desc, call.shape);
  call.p.x = X;
  call.p.dy = dY;
  call.p.gamma = gamma;
  call.p.out = dX;
  call.p.mean = const_cast<float*>(mean);
  call.p.rstd = const_cast<float*>(rstd);
  call.p.dgamma = dgamma;
  call.p.dbeta = dbeta;
  call.p.accumulate = accumulate;
  call.p.part = sums ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kLayerCounterBytes) : nullptr;
  st = with_layer_context(stream, launch_norm, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}
