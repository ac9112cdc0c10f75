// The residual norms' kernels that hold rows in registers (see residual_norm.cu for
// the mathematics).
#pragma once

#include <cuda_runtime.h>

#include <algorithm>

#include "layer_launch.h"
#include "layer_math.cuh"
#include "norm_launch.h"
#include "norm_rows.cuh"
#include "sm103_ptx.cuh"

namespace goldy {

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

// Threads per row (0: the row streams).  `cluster` CTAs of kMaxTeam threads share a
// row that is too long for one, `seg` columns each.
struct ResidualNormShape {
  int team, cluster, seg;
};

// How rows lie: in whole blocks of 16 bytes; all arrays' rows r the same number of
// elements behind a block's start, a number that comes again every few rows, so that
// a team whose rows are that far apart has its parameters, sums and data in one
// frame (bf16, 16384 rows of 1999: 66 us, backwards 104, in the ways for rows that
// lie anyhow 78 and 184; of 201: 16 and 23, then 34 and 34); or anyhow.
enum RowMode { kWholeRows = 0, kFramedRows = 1, kAnyRows = 2 };

// The kernel for a shape, per direction, type and mode (residual_norm_kernels.cu).
// full: both norms and dS are there (backwards).
using ResidualNormPick = NormKernel(const ResidualNormShape& s, bool full);
ResidualNormPick residual_norm_forward_bf16_0, residual_norm_forward_bf16_1, residual_norm_forward_bf16_2;
ResidualNormPick residual_norm_forward_f32_0, residual_norm_forward_f32_1, residual_norm_forward_f32_2;
ResidualNormPick residual_norm_backward_bf16_0, residual_norm_backward_bf16_1, residual_norm_backward_bf16_2;
ResidualNormPick residual_norm_backward_f32_0, residual_norm_backward_f32_1, residual_norm_backward_f32_2;

constexpr int kMaxTeam = 512;
constexpr int kFwdVals = 16;           // values of a row per thread
constexpr int kBwdVals = 8;
// Threads of a CTA: whole teams, 512 per SM together (128 registers each).
__host__ __device__ constexpr int fwd_threads(int team) { return team > 256 ? team : 256 % team ? team : 256; }
__host__ __device__ constexpr int bwd_threads(int team) { return team * (512 / team); }

constexpr int kFwdDepth = 3;           // rows in a thread's ring
// where the row after one has to come in before its place is used again
template <typename T> __host__ __device__ constexpr int norm_depth() { return sizeof(T) == 2 ? 4 : 3; }

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

// Elements that row r of an array starts behind a block's start.
template <typename T>
__device__ __forceinline__ int frame_of(const void* base, int64_t row, int64_t ld) {
  return int((reinterpret_cast<uintptr_t>(base) / sizeof(T) + uint64_t(row) * uint64_t(ld)) % (16 / sizeof(T)));
}

template <typename T, int TEAM, RowMode MODE, bool WIDE>
__global__ void __launch_bounds__(fwd_threads(TEAM), 512 / fwd_threads(TEAM))
residual_norm_forward_kernel(const ResidualNormParams p) {
  constexpr int THREADS = fwd_threads(TEAM), TEAMS = THREADS / TEAM, VALS = kFwdVals;
  constexpr int WARPS = TEAM / 32, D = WIDE ? norm_depth<T>() : kFwdDepth;
  constexpr bool VEC = MODE == kWholeRows, FRAME = MODE == kFramedRows;
  using R = NormRow<T, VALS, TEAM, THREADS, VEC || FRAME, WIDE, FRAME>;
  // per row, norm and warp (WIDE: of all CTAs that share the row): sum, M2, elements, mean
  __shared__ float4 slot[2][2][WIDE ? kMaxCluster : TEAMS][WARPS];
  extern __shared__ __align__(16) uint8_t ring[];  // D rows of F, D of X
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  // this CTA's n columns, from column c0 of the row on (of a frame: from its first
  // block on, the row's first element being the frame's element lo)
  const int frame = FRAME ? frame_of<T>(p.f, int64_t(group) * TEAMS + team, p.ldf) : 0;
  const int c0 = (WIDE ? rank * p.seg : 0) - frame, lo = rank == 0 ? frame : 0;
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n - c0;
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
    const int c = c0 + R::col(i, t), k0 = i * R::PER, end = c0 + n;
    load_params<R::PER, VEC>(p.gate, p.param_f32, c, end, 1.0f, gamma + k0);
    load_params<R::PER, VEC>(p.gamma_f, p.param_f32, c, end, 1.0f, a + k0);
    load_params<R::PER, VEC>(p.beta_f, p.param_f32, c, end, 0.0f, b + k0);
#pragma unroll
    for (int k = k0; k < k0 + R::PER; ++k) a[k] *= gamma[k], b[k] *= gamma[k];
    load_params<R::PER, VEC>(p.gamma_y, p.param_f32, c, end, 1.0f, gamma + k0);
    load_params<R::PER, VEC>(p.beta_y, p.param_f32, c, end, 0.0f, beta + k0);
    mine += R::count(i, t, n, lo);
  }
  const float warp_n = warp_sum(float(mine));
  const float warp_inv = warp_n > 0.0f ? 1.0f / warp_n : 0.0f;
  if constexpr (!WIDE) {
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
              e = R::complete(i, t, n, lo) || R::inside(i, k, t, n, lo) ? e - wm : 0.0f;
            }
          }
        }
        float m2 = 0.0f;
#pragma unroll
        for (int j = 0; j < VALS; ++j) m2 = fmaf(v[j], v[j], m2);
        m2 = warp_sum(m2);
        float mean = wm;
        if (WARPS > 1) {
          const float4 o = make_float4(s, m2, warp_n, wm);
          [[maybe_unused]] float total = 0.0f;
          if (lane == 0) slot[flip][which][team][w] = o;
          team_sync<TEAM, THREADS>(team);
          if constexpr ((WARPS & (WARPS - 1)) == 0) {
            const float4 q = slot[flip][which][team][lane & (WARPS - 1)];
            if (kind == GOLDY_NORM_LAYER) mean = lanes_sum<WARPS>(q.x) * p.inv_n;
            const float d = q.w - mean;
            m2 = lanes_sum<WARPS>(fmaf(q.z * d, d, q.y));
          } else {
            if (kind == GOLDY_NORM_LAYER) {
#pragma unroll
              for (int k = 0; k < WARPS; ++k) total += slot[flip][which][team][k].x;
              mean = total * p.inv_n;
            }
            m2 = 0.0f;
#pragma unroll
            for (int k = 0; k < WARPS; ++k) {
              const float4 q = slot[flip][which][team][k];
              const float d = q.w - mean;
              m2 += fmaf(q.z * d, d, q.y);
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
      R::values(ring + 2 * at * R::RING_BYTES, f_in + row * p.ldf, n, t, v, lo);
      R::values(ring + (2 * at + 1) * R::RING_BYTES, x_in + row * p.ldx, n, t, x, lo);
      // (SHIFT: the ring's place is used again when every piece has been read, which
      // the barriers of the norms make sure of, if there is one)
      if (R::SHIFT && (WARPS == 1 || (p.norm_f == GOLDY_NORM_NONE && p.norm_y == GOLDY_NORM_NONE))) team_sync<TEAM, THREADS>(team);
      at = at + 1 == D ? 0 : at + 1;
      ahead = ahead + 1 == D ? 0 : ahead + 1;
      normalise(p.norm_f, 0, v);
#pragma unroll
      for (int j = 0; j < VALS; ++j) v[j] = fmaf(v[j], a[j], fmaf(p.alpha, x[j], b[j]));
      R::store(s_out + row * p.lds, n, t, v, lo);
      if (p.norm_y == GOLDY_NORM_NONE) continue;
      normalise(p.norm_y, 1, v);
#pragma unroll
      for (int j = 0; j < VALS; ++j) v[j] = fmaf(v[j], gamma[j], beta[j]);
      R::store(y_out + row * p.ldy, n, t, v, lo);
    }
  } else {
    // A row takes the statistics of F, then those of S.  The first of a row and the
    // second of the row before it are exchanged together: one cluster barrier per row,
    // and each phase has another row's arithmetic beside it (8192 x 12288 bf16: 261 us,
    // one after the other 334; a team's own barrier is not worth it: 16384 x 2048 48
    // and 44, 16384 x 1999 85 and 66).
    struct Sums {
      float s, m2, wm;                               // of a warp: sum, squares about its mean, mean (RMS: about 0)
    };
    auto sums_of = [&](int kind, const float (&v)[VALS]) {
      Sums r = {0.0f, 0.0f, 0.0f};
      if (kind == GOLDY_NORM_NONE) return r;
      if (kind == GOLDY_NORM_RMS) {                  // (zeros outside the row)
#pragma unroll
        for (int j = 0; j < VALS; ++j) r.m2 = fmaf(v[j], v[j], r.m2);
      } else {
#pragma unroll
        for (int j = 0; j < VALS; ++j) r.s += v[j];
        r.s = warp_sum(r.s);
        r.wm = r.s * warp_inv;
#pragma unroll
        for (int i = 0; i < R::SLOTS; ++i) {
          if (!R::in(i, t, n)) continue;
          const bool complete = R::complete(i, t, n, lo);
#pragma unroll
          for (int k = 0; k < R::PER; ++k) {
            const float d = complete || R::inside(i, k, t, n, lo) ? v[i * R::PER + k] - r.wm : 0.0f;
            r.m2 = fmaf(d, d, r.m2);
          }
        }
      }
      r.m2 = warp_sum(r.m2);
      return r;
    };
    Sums sf = {0.0f, 0.0f, 0.0f}, sy = sf;           // what is sent
    float2 of = make_float2(0.0f, 1.0f), oy = of;    // mean and rstd that come of it
    auto send = [&](int flip) {
      tell_cluster_warp<WARPS>(&slot[flip][0][0][0], rank, p.cluster, w, lane, make_float4(sf.s, sf.m2, warp_n, sf.wm));
      tell_cluster_warp<WARPS>(&slot[flip][1][0][0], rank, p.cluster, w, lane, make_float4(sy.s, sy.m2, warp_n, sy.wm));
      tell_cluster_begin();
    };
    auto receive = [&](int flip) {
      tell_cluster_end();
      auto joined = [&](int kind, int which) {
        if (kind == GOLDY_NORM_NONE) return make_float2(0.0f, 1.0f);
        const float4* all = &slot[flip][which][0][0];
        float mean = 0.0f, m2 = 0.0f;
        if (kind == GOLDY_NORM_LAYER) {
          for (int k = lane; k < p.cluster * WARPS; k += 32) mean += all[k].x;
          mean = warp_sum(mean) * p.inv_n;
        }
        for (int k = lane; k < p.cluster * WARPS; k += 32) {
          const float4 q = all[k];
          const float d = q.w - mean;
          m2 += fmaf(q.z * d, d, q.y);
        }
        return make_float2(mean, rsqrtf(fmaf(warp_sum(m2), p.inv_n, p.eps)));
      };
      of = joined(p.norm_f, 0);
      oy = joined(p.norm_y, 1);
    };
    auto keep = [&](int kind, int which, int64_t r, const float2& o) {
      if (t != 0 || rank != 0 || !p.stats || kind == GOLDY_NORM_NONE) return;
      if (kind == GOLDY_NORM_LAYER) p.stats[2 * which * p.rows + r] = o.x;
      p.stats[(2 * which + 1) * p.rows + r] = o.y;
    };
    float v[VALS];                                   // S of the row whose Y is left
    auto finish = [&](int64_t r) {
      if (p.norm_y == GOLDY_NORM_NONE) return;
      keep(p.norm_y, 1, r, oy);
      const float shift = -oy.x;
#pragma unroll
      for (int j = 0; j < VALS; ++j) v[j] = fmaf((v[j] + shift) * oy.y, gamma[j], beta[j]);
      R::store(y_out + r * p.ldy, n, t, v, lo);
    };
    auto first = [&](const uint8_t* from, int64_t r) {
      if (p.norm_f == GOLDY_NORM_NONE || r >= p.rows) return;
      float f[VALS];
      R::values(from, f_in + r * p.ldf, n, t, f, lo);
      sf = sums_of(p.norm_f, f);
    };
    // where threads read one another's pieces of the row that makes place for the next
    // one, the barrier has to lie before that is asked for
    constexpr bool LATE = !R::SHIFT;
    const int64_t row0 = row;
    int at = 0, ahead = D - 1, last_flip = 0;
    copy_wait<D - 2>();
    if (R::SHIFT) team_sync<TEAM, THREADS>(team);
    first(ring, row);
    send(1);
    if (!LATE) receive(1);
    for (int flip = 0; row < p.rows; row += step, last_flip = flip, flip ^= 1) {
      fetch(ahead, row + (D - 1) * step);            // where the row before this one was
      copy_wait<D - 2>();
      if (R::SHIFT) team_sync<TEAM, THREADS>(team);
      if (LATE) receive(flip ^ 1);
      if (row != row0) finish(row - step);
      keep(p.norm_f, 0, row, of);
      const uint8_t* from = ring + 2 * at * R::RING_BYTES;
      at = at + 1 == D ? 0 : at + 1;
      ahead = ahead + 1 == D ? 0 : ahead + 1;
      float x[VALS];
      R::values(from, f_in + row * p.ldf, n, t, v, lo);
      R::values(from + R::RING_BYTES, x_in + row * p.ldx, n, t, x, lo);
      // (the mean is subtracted before the scale: rows far from zero keep their digits)
      const float shift = -of.x;
#pragma unroll
      for (int j = 0; j < VALS; ++j) v[j] = fmaf((v[j] + shift) * of.y, a[j], fmaf(p.alpha, x[j], b[j]));
      R::store(s_out + row * p.lds, n, t, v, lo);
      sy = sums_of(p.norm_y, v);
      first(ring + 2 * at * R::RING_BYTES, row + step);
      send(flip);
      if (!LATE) receive(flip);
    }
    if (LATE) receive(last_flip);
    finish(row - step);
  }
}

// FULL: both norms and dS are there.
template <typename T, int TEAM, RowMode MODE, bool WIDE, bool FULL>
__global__ void __launch_bounds__(bwd_threads(TEAM)) residual_norm_backward_kernel(const ResidualNormParams p) {
  constexpr int THREADS = bwd_threads(TEAM), TEAMS = THREADS / TEAM, WARPS = TEAM / 32, VALS = kBwdVals, D = norm_depth<T>();
  constexpr bool VEC = MODE == kWholeRows, FRAME = MODE == kFramedRows;
  using R = NormRow<T, VALS, TEAM, THREADS, VEC || FRAME, WIDE, FRAME>;
  __shared__ float4 slot[2][WIDE ? kMaxCluster : TEAMS][WARPS];
  extern __shared__ __align__(16) uint8_t ring[];  // D rows of F, S, dY and dS each; at the end the CTA's sums
  const int team = threadIdx.x / TEAM, t = threadIdx.x % TEAM, w = t >> 5, lane = t & 31;
  const int rank = WIDE ? int(ptx::cluster_ctarank()) : 0;
  const int group = WIDE ? int(blockIdx.x) / p.cluster : int(blockIdx.x);
  const int groups = WIDE ? int(gridDim.x) / p.cluster : int(gridDim.x);
  const int frame = FRAME ? frame_of<T>(p.f, int64_t(group) * TEAMS + team, p.ldf) : 0;
  const int c0 = (WIDE ? rank * p.seg : 0) - frame, lo = rank == 0 ? frame : 0;     // as forwards
  const int n = WIDE ? min(p.seg, p.n - c0) : p.n - c0;
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
  const typename R::Masks masks(t, n, lo);
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
      const int k0 = i * R::PER, at = c0 + R::col(i, t), end = c0 + n;
      if (R::in(i, t, n)) {
        load_params<R::PER, VEC>(p.gate, p.param_f32, at, end, 1.0f, a + k0);
        load_params<R::PER, VEC>(p.gamma_f, p.param_f32, at, end, 1.0f, b + k0);
        load_params<R::PER, VEC>(p.gamma_y, p.param_f32, at, end, 1.0f, c + k0);
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
    R::values(from + R::RING_BYTES, R::SHIFT ? s_in + r * p.lds : nullptr, n, t, v, masks);
    R::values(from + 2 * R::RING_BYTES, R::SHIFT ? dy_in + r * p.ldy : nullptr, n, t, d, masks);
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
  auto send = [&](int flip) {
    if (WIDE) {
      tell_cluster_warp<WARPS>(&slot[flip][0][0], rank, p.cluster, w, lane, warp_sum4(s1x, s1y, s2x, s2y, lane, nullptr));
      tell_cluster_begin();
    } else if (WARPS > 1) {
      warp_sum4(s1x, s1y, s2x, s2y, lane, reinterpret_cast<float*>(&slot[flip][team][w]));
    } else {
      const float4 r = warp_sum4(s1x, s1y, s2x, s2y, lane, nullptr);
      s1x = r.x, s1y = r.y, s2x = r.z, s2y = r.w;
    }
  };
  auto receive = [&](int flip) {
    if (WARPS == 1) {
      if (R::SHIFT) __syncwarp();
      return;
    }
    float4 r;
    if (WIDE) {
      tell_cluster_end();
      const float4* all = &slot[flip][0][0];
      r = all[lane];                               // (at least two CTAs of 16 warps)
      for (int k = lane + 32; k < p.cluster * WARPS; k += 32) {
        const float4 o = all[k];
        r.x += o.x, r.y += o.y, r.z += o.z, r.w += o.w;
      }
      r = make_float4(warp_sum(r.x), warp_sum(r.y), warp_sum(r.z), warp_sum(r.w));
    } else {
      team_sync<TEAM, THREADS>(team);
      if (WARPS < 8) {
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
    }
    s1x = r.x, s1y = r.y, s2x = r.z, s2y = r.w;
  };
  // between the two the next row is asked for; where threads read one another's
  // pieces of the row that makes place for it, the barrier has to lie before that
  constexpr bool LATE = !R::SHIFT;
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
    R::store(df_at, n, t, v, lo);
    df_at += step_f;
  };
  int at = 0, ahead = D - 1;
  bool begun = false;
  if (left > 0) {                                  // whole teams, and whole clusters
    copy_wait<D - 2>();
    if (R::SHIFT) team_sync<TEAM, THREADS>(team);
    first(ring, true, row, now);
    send(1);
    if (!LATE) receive(1);
  }
  int last_flip = 0;
  for (int flip = 0; left > 0; --left, row += step, last_flip = flip, flip ^= 1) {
    fetch(ahead, left > D - 1);                    // where the row before this one was
    const float later = next_stats(left > 2);
    copy_wait<D - 2>();
    if (R::SHIFT) team_sync<TEAM, THREADS>(team);
    if (LATE) receive(flip ^ 1);
    if (begun) finish();
    begun = true;
    // T, dX, and what dF needs
    const uint8_t* from = ring + 4 * at * R::RING_BYTES;
    at = at + 1 == D ? 0 : at + 1;
    ahead = ahead + 1 == D ? 0 : ahead + 1;
    float tt[VALS], v[VALS];
    if (has_ds) {
      R::values(from + 3 * R::RING_BYTES, R::SHIFT ? ds_in + row * p.lds : nullptr, n, t, tt, masks);
    } else {
#pragma unroll
      for (int j = 0; j < VALS; ++j) tt[j] = 0.0f;
    }
    R::values(from, R::SHIFT ? f_in + row * p.ldf : nullptr, n, t, v, masks);
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
    R::store(dx_at, n, t, tt, lo);
    dx_at += step_x;
    now = next;
    next = later;
    first(ring + 4 * at * R::RING_BYTES, left > 1, row + step, now);
    send(flip);
    if (!LATE) receive(flip);
  }
  if (begun) {
    if (LATE) receive(last_flip);
    finish();
  }
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
  float* to = p.part + int64_t(group) * kSums * p.n;
  int from[TEAMS];                                 // where column 0 of the teams' rows is in their sums
#pragma unroll
  for (int k = 0; k < TEAMS; ++k)
    from[k] = (FRAME ? frame_of<T>(p.f, int64_t(group) * TEAMS + k, p.ldf) : 0) - (WIDE ? rank * p.seg : 0);
  for (int c = max(c0, 0) + int(threadIdx.x); c < c0 + n; c += THREADS) {
    float v[kSums];
#pragma unroll
    for (int q = 0; q < kSums; ++q) {
      v[q] = 0.0f;
#pragma unroll
      for (int k = 0; k < TEAMS; ++k) v[q] += sums[(k * kSums + q) * ALL + c + from[k]];
    }
    if (groups > 1) {
#pragma unroll
      for (int q = 0; q < kSums; ++q) __stcg(to + int64_t(q) * p.n + c, v[q]);
    } else {                                       // this CTA's sums are the result
      give_gradients(p, c, v[0], v[1], v[2], v[3]);
    }
  }
}

}  // namespace goldy
