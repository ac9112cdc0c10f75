// Linear-layer products with fused epilogues, plain or grouped by expert.
//
// One persistent tcgen05 kernel computes C[r][c] = sum_k P[c][k] Q[r][k] for
// the three passes of a linear layer Y = act(X W + b) + R:
//   forward      C = X W,    P = W^T (c contiguous in memory), Q = X
//   input grad   C = dY W^T, P = W (k contiguous),             Q = dY
//   weight grad  C = X^T dY, P = dY^T (c contiguous), Q = X^T (r contiguous)
// c, the contiguous index of C, lies along the tensor cores' M (128 lanes of
// tensor memory per CTA) and r along N, for every pass.  With ragged groups
// (rows offsets[e] .. offsets[e+1]-1 belong to expert e) r is the ragged axis
// of the first two passes: N is an operand of the instruction, so a tile of w
// rows costs ceil(w / 16) * 16 columns of tensor work whatever the group
// sizes, a single token included, and no row is padded or copied in memory.
// In the weight gradient the ragged axis is the reduction: a group's last
// stage may hold rows of the next group, which the load warp zeroes in shared
// memory before handing the stage on (zero times whatever the neighbour holds
// would not do: 0 * inf is NaN).
//
// PAIR: a cluster of two CTAs computes 256 columns x up to 256 rows with
// cta_group::2 MMAs (each CTA stages its 128 columns of P and half of Q's
// rows: 32 KB per 64-deep stage for 128 x 256 x 64 multiply-adds per SM).
// Without PAIR one CTA computes 128 columns x tile_r rows; the reduction may
// be split over several units whose fp32 partials the last one to arrive sums
// in split order (workspace), so results do not depend on the order of
// arrival.
//
// Roles (320 threads): warp 0 loads by TMA, warp 1 issues the MMAs, warps 2-9
// drain the accumulator (double buffered in tensor memory): each takes every
// second 32-row chunk of its 32 lanes through a 4 KB transposing buffer, so
// that global accesses run along c (64-byte bf16 or 128-byte fp32 segments)
// and bias, activation, its gradient, residual and the saved pre-activation
// cost no further pass over C.
//
// OUT_F32: the tensor cores add into fp32 accumulators with truncation, a
// relative error of about 1e-9 per reduction element (4.4e-6 at 4096,
// measured against fp64).  fp32 results therefore leave tensor memory every
// kLinPromote stages (512 elements) and are summed in registers with rounding
// to nearest: 5e-7 at any length.  bf16 results (relative rounding 2^-8) keep
// the whole sum in tensor memory.
//
// Every wait is bounded; a wait that runs out sets the error word and the
// kernel ends.
#pragma once

#include "go_kernel.cuh"
#include "layer_internal.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {

// Arrive on an mbarrier of a CTA of the cluster and add `bytes` to what its
// phase waits for.
__device__ __forceinline__ void mbar_arrive_expect_tx_remote(uint32_t cluster_addr, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.release.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(cluster_addr),
               "r"(bytes)
               : "memory");
}

// One unit of work: a tile of C, or one split of its reduction.
struct LinUnit {
  int e;           // group
  int r0;          // first row of C (forward, input grad: absolute; weight grad: input feature)
  int w;           // rows of the tile
  int nw;          // the same, rounded up to the instruction's N
  int c0;          // first column of C
  int k0, red;     // first reduction row and reduction length (weight grad), 0 and length otherwise
  int kb0, kb1;    // stages of 64 reduction elements
  int tile, s;     // index of the tile over all groups, split
};

// Walks the units of a launch in increasing order.  All lanes of a warp call
// it together; groups are looked up 32 at a time (offsets clamped to
// [0, rows] and taken as non-decreasing, so that no offsets make a launch
// leave its buffers).
template <int PASS, bool PAIR>
struct LinWalk {
  static constexpr int G = PAIR ? 32 : 16;     // granularity of N
  const LinearParams& p;
  const int lane;
  int e0 = 0, begin = 0, prev = 0;             // window of 32 groups: first, units before it, row before it
  int start = 0, cnt = 0, incl = 0;            // this lane's group: first row, rows, units up to its end
  bool loaded = false;

  __device__ LinWalk(const LinearParams& params, int lane_id) : p(params), lane(lane_id) {}

  __device__ static int width(int rows, int tile_r) {
    if (rows <= 0) return G;
    const int n = (rows + tile_r - 1) / tile_r;      // equal tiles
    return ((rows + n - 1) / n + G - 1) / G * G;
  }
  __device__ int group_units(int rows) const {
    if (rows <= 0) return 0;
    const int w = width(rows, p.tile_r);
    return (rows + w - 1) / w * p.tiles_c * p.split;
  }
  __device__ void load_window() {
    const int e = e0 + lane;
    int o = 0, o1 = 0;
    if (e < p.groups) {
      o = min(max(__ldg(p.offsets + e), 0), p.rows);
      o1 = min(max(__ldg(p.offsets + e + 1), 0), p.rows);
    }
    int m = max(o, prev);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int t = __shfl_up_sync(0xFFFFFFFFu, m, d);
      if (lane >= d) m = max(m, t);
    }
    start = m;
    cnt = e < p.groups ? max(o1 - m, 0) : 0;
    int u = group_units(cnt);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int t = __shfl_up_sync(0xFFFFFFFFu, u, d);
      if (lane >= d) u += t;
    }
    incl = begin + u;
    loaded = true;
  }

  // Unit u (not below the last one asked for); false past the end.
  __device__ bool find(int u, LinUnit& t) {
    int rows, local;
    if (PASS == kLinWeightGrad) {
      const int per = group_units(p.size_r);
      t.e = u / per;
      if (t.e >= p.groups) return false;
      local = u - t.e * per;
      rows = p.size_r;
      int a = 0, b = p.rows;
      if (p.offsets) {
        a = min(max(__ldg(p.offsets + t.e), 0), p.rows);
        b = min(max(__ldg(p.offsets + t.e + 1), a), p.rows);
      }
      t.k0 = a;
      t.red = max(b - a, 0);
      t.r0 = 0;
    } else {
      if (p.offsets) {
        if (!loaded) load_window();
        int last;
        while (u >= (last = __shfl_sync(0xFFFFFFFFu, incl, 31))) {
          if (e0 + 32 >= p.groups) return false;
          prev = __shfl_sync(0xFFFFFFFFu, start + cnt, 31);
          begin = last;
          e0 += 32;
          load_window();
        }
        const int j = __ffs(__ballot_sync(0xFFFFFFFFu, u < incl)) - 1;
        rows = __shfl_sync(0xFFFFFFFFu, cnt, j);
        t.r0 = __shfl_sync(0xFFFFFFFFu, start, j);
        local = u - (__shfl_sync(0xFFFFFFFFu, incl, j) - group_units(rows));
        t.e = e0 + j;
      } else {
        rows = p.rows;
        t.r0 = 0;
        t.e = 0;
        local = u;
        if (u >= group_units(rows)) return false;
      }
      t.k0 = 0;
      t.red = p.red;
    }
    t.tile = u / p.split;
    const int w = width(rows, p.tile_r);
    const int n_r = (rows + w - 1) / w;
    const int i = local / p.split;
    t.s = local - i * p.split;
    const int band = i / (kLinRowBand * p.tiles_c);
    const int rem = i - band * kLinRowBand * p.tiles_c;
    const int in_band = min(kLinRowBand, n_r - band * kLinRowBand);
    const int tc = rem / in_band;
    const int tr = band * kLinRowBand + rem - tc * in_band;
    t.r0 += tr * w;
    t.w = min(w, rows - tr * w);
    t.nw = (t.w + G - 1) / G * G;
    t.c0 = tc * (PAIR ? 256 : 128);
    const int kbs = (t.red + kLinStageK - 1) / kLinStageK;
    t.kb0 = int(int64_t(kbs) * t.s / p.split);
    t.kb1 = int(int64_t(kbs) * (t.s + 1) / p.split);
    return true;
  }
};

// A 32 x 32 fp32 block in shared memory, 128 bytes per row of C, 16-byte
// pieces permuted by row so that neither the column-wise writes nor the
// row-wise reads collide in a bank.
__device__ __forceinline__ uint32_t lin_stage_addr(uint32_t base, int row, int piece) {
  return base + uint32_t(row * 128 + ((piece ^ (row & 7)) << 4));
}

// Bounded wait of a whole warp, with one answer for all lanes.
__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, ptx::mbar_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ bool lin_wait_cluster(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, ptx::mbar_wait_cluster(bar, parity, abort_flag));
}

// What a warp adds to 8 consecutive columns; loaded once per unit.
struct LinBias {
  float v[8];
};

template <int PASS>
__device__ __forceinline__ void lin_load_bias(const LinearParams& p, int e, int col, LinBias& b) {
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    b.v[k] = 0.0f;
    if (PASS == kLinForward && p.bias && col + k < p.size_c) {
      const int64_t i = int64_t(e) * p.size_c + col + k;
      b.v[k] = p.bias_f32 ? static_cast<const float*>(p.bias)[i] : load_bf16(p.bias, i);
    }
  }
}

// Epilogue of one 32-row chunk: v[j] is row j of this lane's column.  After
// the transposition a lane has 8 consecutive columns of 4 rows, 8 apart.  What
// the rows need from memory (saved pre-activation, residual) is asked for
// first, all 4 rows at once, so that its latency is paid once per chunk.
__device__ __forceinline__ void lin_transpose(uint32_t buf, int lane, const float (&v)[32]) {
  __syncwarp();
#pragma unroll
  for (int j = 0; j < 32; ++j) {
    const uint32_t a = lin_stage_addr(buf, j, lane >> 2) + uint32_t((lane & 3) * 4);
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v[j]) : "memory");
  }
  __syncwarp();
}
__device__ __forceinline__ void lin_transposed(uint32_t buf, int lane, int row, const LinBias& bias, float (&f)[8]) {
  const float4 a = ptx::ld_shared_v4(lin_stage_addr(buf, row, (lane & 3) * 2));
  const float4 b = ptx::ld_shared_v4(lin_stage_addr(buf, row, (lane & 3) * 2 + 1));
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] += bias.v[k];
}

// Whole 16-byte accesses: every tensor of the epilogue on 16-byte boundaries,
// 32 whole columns.  bf16 results.
template <int PASS, int ACT>
__device__ __forceinline__ void lin_finish_fast(const LinearParams& p, const LinUnit& t, uint32_t buf, int lane,
                                                int row0, int col, const LinBias& bias, const float (&v)[32]) {
  const int sub = lane >> 2;
  const int64_t r0 = int64_t(t.r0) + row0 + sub;
  const int left = t.w - row0 - sub;               // row i * 8 of this lane exists if i * 8 < left
  const int64_t c_at = int64_t(t.e) * p.c_group + r0 * p.ldc + col;
  const int64_t q_at = int64_t(t.e) * p.r_group + r0 * p.ldr + col;
  constexpr bool SLOPE = PASS == kLinInputGrad && ACT != GOLDY_ACT_NONE;
  uint4 z[4], q[4];
  if (SLOPE) {
    const uint16_t* from = static_cast<const uint16_t*>(p.z_in) + r0 * p.ldz + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i * 8 < left) z[i] = __ldg(reinterpret_cast<const uint4*>(from + i * 8 * p.ldz));
  }
  if (p.res) {
    const uint16_t* from = static_cast<const uint16_t*>(p.res) + q_at;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i * 8 < left) q[i] = *reinterpret_cast<const uint4*>(from + i * 8 * p.ldr);
  }
  lin_transpose(buf, lane, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i * 8 >= left) break;
    float f[8];
    lin_transposed(buf, lane, i * 8 + sub, bias, f);
    if (PASS == kLinForward && p.z_out)
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.z_out) + (r0 + i * 8) * p.ldz + col) = pack8(f);
    if (SLOPE) {
      float zf[8];
      unpack8(z[i], zf);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] *= act_slope(zf[k], ACT);
    } else if (PASS == kLinForward) {
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = act_value(f[k], ACT);
    }
    if (p.res) {
      float qf[8];
      unpack8(q[i], qf);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] += qf[k];
    }
    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.c) + c_at + i * 8 * p.ldc) = pack8(f);
  }
}

// The same for fp32 results, rolled up: the sums of the chunks still to come
// occupy the registers.
template <int PASS>
__device__ __forceinline__ void lin_finish_f32(const LinearParams& p, const LinUnit& t, uint32_t buf, int lane,
                                               int row0, int col, const LinBias& bias) {
  const int sub = lane >> 2;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + sub;
    if (row0 + row >= t.w) break;
    const int64_t r = int64_t(t.r0) + row0 + row;
    float4 q0 = make_float4(0.0f, 0.0f, 0.0f, 0.0f), q1 = q0;
    if (PASS != kLinWeightGrad && p.res) {
      const float* from = static_cast<const float*>(p.res) + r * p.ldr + col;
      q0 = *reinterpret_cast<const float4*>(from);
      q1 = *reinterpret_cast<const float4*>(from + 4);
    }
    float f[8];
    lin_transposed(buf, lane, row, bias, f);
    if (PASS == kLinForward) {
      if (p.z_out) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.z_out) + r * p.ldz + col) = pack8(f);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = act_value(f[k], p.act);
    }
    if (PASS == kLinInputGrad && p.z_in) {
      float zf[8];
      unpack8(__ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.z_in) + r * p.ldz + col)), zf);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] *= act_slope(zf[k], p.act);
    }
    float* c = static_cast<float*>(p.c) + int64_t(t.e) * p.c_group + r * p.ldc + col;
    *reinterpret_cast<float4*>(c) = make_float4(f[0] + q0.x, f[1] + q0.y, f[2] + q0.z, f[3] + q0.w);
    *reinterpret_cast<float4*>(c + 4) = make_float4(f[4] + q1.x, f[5] + q1.y, f[6] + q1.z, f[7] + q1.w);
  }
}

// Any alignment and the columns at C's edge, element by element.
template <int PASS, bool OUT_F32>
__device__ __noinline__ void lin_finish_slow(const LinearParams& p, int e, int first_row, int rows, uint32_t buf,
                                             int lane, int col) {
  const int sub = lane >> 2;
  const int n_col = min(8, p.size_c - col);
  LinBias bias;
  lin_load_bias<PASS>(p, e, col, bias);
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + sub;
    if (row >= rows) break;
    const int64_t r = int64_t(first_row) + row;
    float f[8];
    lin_transposed(buf, lane, row, bias, f);
    const int64_t c_at = int64_t(e) * p.c_group + r * p.ldc + col;
    const int64_t q_at = int64_t(e) * p.r_group + r * p.ldr + col;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (k >= n_col) break;
      float v = f[k];
      if (PASS == kLinForward) {
        if (p.z_out) store_bf16(p.z_out, r * p.ldz + col + k, v);
        v = act_value(v, p.act);
      } else if (PASS == kLinInputGrad && p.z_in) {
        v *= act_slope(load_bf16(p.z_in, r * p.ldz + col + k), p.act);
      }
      if (p.res && !(OUT_F32 && PASS == kLinWeightGrad))
        v += OUT_F32 ? static_cast<const float*>(p.res)[q_at + k] : load_bf16(p.res, q_at + k);
      if (OUT_F32) static_cast<float*>(p.c)[c_at + k] = v;
      else store_bf16(p.c, c_at + k, v);
    }
  }
}

template <int PASS, bool OUT_F32>
__device__ __forceinline__ void lin_finish_chunk(const LinearParams& p, const LinUnit& t, uint32_t buf, int lane,
                                                 int row0, int col0, const LinBias& bias, const float (&v)[32]) {
  const int col = col0 + (lane & 3) * 8;           // this lane's 8 columns
  if (!p.vec || col0 + 32 > p.size_c) {
    lin_transpose(buf, lane, v);
    if (col < p.size_c) lin_finish_slow<PASS, OUT_F32>(p, t.e, t.r0 + row0, t.w - row0, buf, lane, col);
    return;
  }
  if (OUT_F32) {
    lin_transpose(buf, lane, v);
    lin_finish_f32<PASS>(p, t, buf, lane, row0, col, bias);
    return;
  }
  switch (PASS == kLinWeightGrad ? GOLDY_ACT_NONE : p.act) {
    case GOLDY_ACT_RELU: lin_finish_fast<PASS, GOLDY_ACT_RELU>(p, t, buf, lane, row0, col, bias, v); break;
    case GOLDY_ACT_GELU: lin_finish_fast<PASS, GOLDY_ACT_GELU>(p, t, buf, lane, row0, col, bias, v); break;
    case GOLDY_ACT_GELU_TANH: lin_finish_fast<PASS, GOLDY_ACT_GELU_TANH>(p, t, buf, lane, row0, col, bias, v); break;
    case GOLDY_ACT_SILU: lin_finish_fast<PASS, GOLDY_ACT_SILU>(p, t, buf, lane, row0, col, bias, v); break;
    default: lin_finish_fast<PASS, GOLDY_ACT_NONE>(p, t, buf, lane, row0, col, bias, v);
  }
}

template <int PASS, bool PAIR, bool OUT_F32>
__global__ void __launch_bounds__(kLinThreads, 1) linear_kernel(const __grid_constant__ LinearParams p) {
  constexpr bool A_MN = PASS != kLinInputGrad;         // P contiguous along c
  constexpr bool B_MN = PASS == kLinWeightGrad;        // Q contiguous along r
  constexpr bool TAIL = PASS == kLinWeightGrad;        // ragged reduction
  constexpr int ACC = 2;
  constexpr int A_BYTES = 128 * kLinStageK * 2;
  constexpr int CTAS = PAIR ? 2 : 1;
  constexpr uint32_t TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int stages = p.stages;
  const uint32_t stage_bytes = uint32_t(p.stage_bytes);
  uint8_t* staging = smem + size_t(stages) * stage_bytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(staging + kLinStagingBytes);
  uint64_t* full = bars;                               // pair: used in the even CTA only
  uint64_t* empty = bars + kLinMaxStages;
  uint64_t* tfull = bars + 2 * kLinMaxStages;
  uint64_t* tempty = tfull + ACC;
  uint64_t* drain = tempty + ACC;
  uint64_t* tail = drain + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(tail + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const uint32_t tiles = ptx::smem_u32(smem);
  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const uint32_t rank = PAIR ? (ptx::cluster_ctarank() & 1u) : 0u;
  const bool lead = rank == 0;
  const int worker = PAIR ? int(blockIdx.x >> 1) : int(blockIdx.x);
  const int n_workers = PAIR ? int(gridDim.x >> 1) : int(gridDim.x);

  if (threadIdx.x == 0) {
    if (p.loads) {
      ptx::prefetch_tensormap(&p.ta);
      ptx::prefetch_tensormap(&p.tb);
      if (!B_MN) ptx::prefetch_tensormap(&p.tb_part);
    }
    for (int s = 0; s < stages; ++s) {
      // the weight gradient's pair counts both CTAs' load warps in
      ptx::mbar_init(ptx::smem_u32(&full[s]), (PAIR && TAIL) ? 2 : 1);
      ptx::mbar_init(ptx::smem_u32(&empty[s]), 1);
    }
    for (int a = 0; a < ACC; ++a) {
      ptx::mbar_init(ptx::smem_u32(&tfull[a]), 1);
      ptx::mbar_init(ptx::smem_u32(&tempty[a]), kLinEpiWarps * CTAS);
    }
    ptx::mbar_init(ptx::smem_u32(drain), 1);
    ptx::mbar_init(ptx::smem_u32(tail), 1);
    *abort_flag = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async_smem();
  }
  if (warp == 1) {
    if (PAIR) {
      ptx::tmem_alloc_pair(ptx::smem_u32(tmem_slot), TMEM_COLS);
      ptx::tmem_relinquish_pair();
    } else {
      ptx::tmem_alloc(ptx::smem_u32(tmem_slot), TMEM_COLS);
      ptx::tmem_relinquish();
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (PAIR) {
    ptx::cluster_sync_all();                           // the peer's barriers and tensor memory are ready
    ptx::tc_fence_after();
  }
  const uint32_t tmem_base = *tmem_slot;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();                                 // inputs and offsets may come from the previous kernel

  LinWalk<PASS, PAIR> walk(p, lane);
  LinUnit t;

  if (warp == 0) {
    // -------------------------------------------------------------- loads
    int stage = 0;
    uint32_t phase = 0, issued = 0, last_phase = 0, tail_phase = 0;
    bool ok = true;
    for (int u = worker; ok && walk.find(u, t); u += n_workers) {
      const int half = t.nw / CTAS;                    // rows of Q this CTA stages
      const int r0 = t.r0 + int(rank) * half;
      const int c0 = t.c0 + int(rank) * 128;
      const bool full_box = !B_MN && t.nw == p.tile_r;
      const int boxes = B_MN ? (half + 63) / 64 : full_box ? 1 : (half + p.part_box - 1) / p.part_box;
      const uint32_t box_bytes = B_MN ? 8192u : uint32_t(full_box ? half : p.part_box) * 128u;
      const uint32_t bytes = A_BYTES + boxes * box_bytes;
      for (int kb = t.kb0; kb < t.kb1; ++kb) {
        if ((issued >> stage & 1) && !lin_wait(ptx::smem_u32(&empty[stage]), phase ^ 1, abort_flag)) {
          ok = false;
          break;
        }
        const uint32_t fb_local = ptx::smem_u32(&full[stage]);
        const uint32_t fb = PAIR ? ptx::map_to_rank(fb_local, 0) : fb_local;
        const uint32_t as = tiles + stage * stage_bytes;
        const uint32_t bs = as + A_BYTES;
        const int k = t.k0 + kb * kLinStageK;
        // rows of the next group behind this group's last one
        const int valid = t.red - kb * kLinStageK;
        const bool fix = TAIL && valid < kLinStageK && t.k0 + t.red < p.rows;
        if (lane == 0) {
          uint32_t bar = fb;
          if (fix) {
            bar = ptx::smem_u32(tail);
            ptx::mbar_arrive_expect_tx(bar, bytes);
            if (PAIR) bar = ptx::map_to_rank(bar, rank);
          } else if (!PAIR) {
            ptx::mbar_arrive_expect_tx(fb_local, bytes);
          } else if (TAIL) {
            mbar_arrive_expect_tx_remote(fb, bytes);
          } else if (lead) {
            ptx::mbar_arrive_expect_tx(fb_local, 2 * bytes);
          }
          auto load = [&](uint32_t dst, const void* map, int x, int y, int z) {
            if (PAIR) ptx::tma_load_3d_pair(dst, map, bar, x, y, z);
            else ptx::tma_load_3d(dst, map, bar, x, y, z);
          };
          const int e = PASS == kLinWeightGrad ? 0 : t.e;
          if (A_MN) {
            load(as, &p.ta, c0, k, e);
            load(as + 8192, &p.ta, c0 + 64, k, e);
          } else {
            load(as, &p.ta, k, c0, e);
          }
          if (B_MN) {
            for (int b = 0; b < boxes; ++b) load(bs + b * 8192, &p.tb, r0 + b * 64, k, 0);
          } else if (full_box) {
            load(bs, &p.tb, k, r0, 0);
          } else {
            for (int b = 0; b < boxes; ++b) load(bs + b * box_bytes, &p.tb_part, k, r0 + b * p.part_box, 0);
          }
        }
        issued |= 1u << stage;
        last_phase = (last_phase & ~(1u << stage)) | (phase << stage);
        if (TAIL && fix) {
          ok = lin_wait(ptx::smem_u32(tail), tail_phase, nullptr);
          tail_phase ^= 1;
          // lines of 128 bytes, one per reduction row, in 8 KB blocks of 64 columns
          const int lines = kLinStageK - valid;
          for (int i = lane; i < (2 + boxes) * lines * 8; i += 32) {
            const int blk = i / (lines * 8), o = i - blk * lines * 8;
            ptx::st_shared_v4(as + blk * 8192 + valid * 128 + o * 16, 0, 0, 0, 0);
          }
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            if (PAIR) ptx::mbar_arrive_remote_release(fb);
            else ptx::mbar_arrive(fb_local);
          }
          if (!ok) break;
        }
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
    if (!ok && lane == 0) raise_error(p.err, abort_flag, kErrProducerWait);
    // every stage filled must have been consumed (and, for a pair, both CTAs'
    // commits landed) before the CTA may leave
    if (lane == 0) {
      const uint64_t t0 = ptx::global_timer();
      for (int s = 0; s < stages; ++s) {
        if (!(issued >> s & 1)) continue;
        while (!ptx::mbar_try_wait(ptx::smem_u32(&empty[s]), (last_phase >> s) & 1)) {
          if (ptx::global_timer() - t0 > ptx::kWaitLimitNs) {
            raise_error(p.err, abort_flag, kErrProducerWait);
            break;
          }
        }
      }
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- MMAs
    if (lead) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0, acc_used = 0;
      bool ok = true, any = false;
      for (int u = worker; ok && walk.find(u, t); u += n_workers) {
        const uint32_t idesc = ptx::make_idesc_bf16(128 * CTAS, 16, A_MN, B_MN) + (uint32_t((t.nw - 16) >> 3) << 17);
        for (int kb = t.kb0; kb < t.kb1;) {
          const int stop = OUT_F32 ? min(kb + kLinPromote, t.kb1) : t.kb1;
          if (acc_used >> acc & 1) {
            const uint32_t b = ptx::smem_u32(&tempty[acc]);
            ok = PAIR ? lin_wait_cluster(b, acc_phase ^ 1, abort_flag) : lin_wait(b, acc_phase ^ 1, abort_flag);
            if (!ok) break;
          }
          acc_used |= 1u << acc;
          ptx::tc_fence_after();
          const uint32_t d = tmem_base + uint32_t(acc * 256);
          bool fresh = true;
          for (; kb < stop; ++kb) {
            const uint32_t b = ptx::smem_u32(&full[stage]);
            ok = (PAIR && TAIL) ? lin_wait_cluster(b, phase, abort_flag) : lin_wait(b, phase, abort_flag);
            if (!ok) break;
            ptx::tc_fence_after();
            if (lane == 0) {
              const uint32_t as = tiles + stage * stage_bytes;
              const uint32_t bs = as + A_BYTES;
#pragma unroll
              for (int kk = 0; kk < 4; ++kk) {
                const uint64_t ad = A_MN ? ptx::make_sdesc_sw128(as + kk * 2048, 8192, 1024)
                                         : ptx::make_sdesc_sw128(as + kk * 32, 16, 1024);
                const uint64_t bd = B_MN ? ptx::make_sdesc_sw128(bs + kk * 2048, 8192, 1024)
                                         : ptx::make_sdesc_sw128(bs + kk * 32, 16, 1024);
                const uint32_t add = (!fresh || kk > 0) ? 1u : 0u;
                if (PAIR) ptx::mma_bf16_pair(d, ad, bd, idesc, add);
                else ptx::mma_bf16(d, ad, bd, idesc, add);
              }
              if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(&empty[stage]), 0x3);
              else ptx::mma_commit(ptx::smem_u32(&empty[stage]));
            }
            __syncwarp();
            fresh = false;
            any = true;
            if (++stage == stages) {
              stage = 0;
              phase ^= 1;
            }
          }
          if (!ok) break;
          if (lane == 0) {
            if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(&tfull[acc]), 0x3);
            else ptx::mma_commit(ptx::smem_u32(&tfull[acc]));
          }
          __syncwarp();
          if (++acc == ACC) {
            acc = 0;
            acc_phase ^= 1;
          }
        }
      }
      if (!ok && lane == 0) {
        raise_error(p.err, abort_flag, kErrMmaWait);
        if (any) {
          if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(drain), 0x1);
          else ptx::mma_commit(ptx::smem_u32(drain));
          ptx::mbar_wait(ptx::smem_u32(drain), 0, nullptr);
        }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue
    const int ew = warp - 2;
    const int q = warp & 3;                            // lanes of tensor memory this warp may read
    const int side = ew >> 2;                          // takes chunks side, side + 2, ...
    const uint32_t buf = ptx::smem_u32(staging) + uint32_t(ew * 4096);
    int acc = 0;
    uint32_t acc_phase = 0;
    bool ok = true;
    auto next_acc = [&]() {
      if (++acc == ACC) {
        acc = 0;
        acc_phase ^= 1;
      }
    };
    auto release = [&]() {                             // this warp has read accumulator `acc`
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        const uint32_t b = ptx::smem_u32(&tempty[acc]);
        if (PAIR) ptx::mbar_arrive_remote_release(ptx::map_to_rank(b, 0));
        else ptx::mbar_arrive(b);
      }
    };
    for (int u = worker; ok && walk.find(u, t); u += n_workers) {
      const int col0 = t.c0 + int(rank) * 128 + q * 32;
      LinBias bias;
      lin_load_bias<PASS>(p, t.e, col0 + (lane & 3) * 8, bias);
      const uint32_t lanes = tmem_base + (uint32_t(q * 32) << 16);
      const bool split = p.split > 1;
      float* part = p.part + ((size_t(t.tile) * p.split * CTAS + rank) * kLinEpiWarps + ew) * (size_t(p.part_chunks) * 1024);
      const size_t split_stride = size_t(CTAS) * kLinEpiWarps * p.part_chunks * 1024;
      auto publish = [&](int i, int chunk, const float (&v)[32]) {
        float* to = part + t.s * split_stride + size_t(i) * 1024 + lane;
#pragma unroll
        for (int j = 0; j < 32; ++j)
          if (chunk * 32 + j < t.w) __stcg(to + j * 32, v[j]);
      };
      bool last = true;
      if (OUT_F32) {
        float sum[4][32];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 32; ++j) {
            sum[i][j] = 0.0f;
            // a gradient that is added to starts from it (split 0 does), read
            // while the tensor cores work
            const int row = (side + 2 * i) * 32 + j;
            if (PASS == kLinWeightGrad && p.res && t.s == 0 && row < t.w && col0 + lane < p.size_c)
              sum[i][j] = static_cast<const float*>(p.res)[int64_t(t.e) * p.r_group + (int64_t(t.r0) + row) * p.ldr +
                                                           col0 + lane];
          }
        for (int kb = t.kb0; kb < t.kb1; kb += kLinPromote) {
          ok = lin_wait(ptx::smem_u32(&tfull[acc]), acc_phase, abort_flag);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int chunk = side + 2 * i;
            if (chunk * 32 < t.nw) {
              uint32_t raw[32];
              ptx::tmem_ld_32x32b_x32(lanes + uint32_t(acc * 256 + chunk * 32), raw);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 32; ++j) sum[i][j] += __uint_as_float(raw[j]);
            }
          }
          release();
          next_acc();
        }
        if (!ok) break;
        if (!split) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int chunk = side + 2 * i;
            if (chunk * 32 < t.w) lin_finish_chunk<PASS, OUT_F32>(p, t, buf, lane, chunk * 32, col0, bias, sum[i]);
          }
          continue;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if ((side + 2 * i) * 32 < t.w) publish(i, side + 2 * i, sum[i]);
      }
      const bool some = !OUT_F32 && t.kb1 > t.kb0;     // the result is in accumulator `acc`
      if (some) {
        ok = lin_wait(ptx::smem_u32(&tfull[acc]), acc_phase, abort_flag);
        if (!ok) break;
        ptx::tc_fence_after();
      }
      auto read_acc = [&](int chunk, float (&v)[32]) {
        if (some) {
          uint32_t raw[32];
          ptx::tmem_ld_32x32b_x32(lanes + uint32_t(acc * 256 + chunk * 32), raw);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(raw[j]);
          // the accumulator is free once its last chunk is in registers
          if ((chunk + 2) * 32 >= t.w) release();
        } else {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0.0f;
        }
      };
      unsigned* cnt = p.cnt + (size_t(t.tile) * CTAS + rank) * kLinEpiWarps + ew;
      if (split) {
        if (!OUT_F32) {
#pragma unroll 1
          for (int i = 0; (side + 2 * i) * 32 < t.w; ++i) {
            float v[32];
            read_acc(side + 2 * i, v);
            publish(i, side + 2 * i, v);
          }
        }
        __threadfence();
        __syncwarp();
        unsigned old = 0;
        if (lane == 0) old = atomicAdd(cnt, 1u);
        last = __shfl_sync(0xFFFFFFFFu, old, 0) == unsigned(p.split - 1);
        if (last) __threadfence();
      }
      // the last of the splits to arrive at this warp's part of the tile sums
      // all of them in split order and leaves the counter at zero
#pragma unroll 1
      for (int i = 0; last && (side + 2 * i) * 32 < t.w; ++i) {
        const int chunk = side + 2 * i;
        float v[32];
        if (split) {
#pragma unroll
          for (int j = 0; j < 32; ++j) v[j] = 0.0f;
#pragma unroll 1
          for (int s = 0; s < p.split; ++s) {
            const float* from = part + s * split_stride + size_t(i) * 1024 + lane;
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (chunk * 32 + j < t.w) v[j] += __ldcg(from + j * 32);
          }
        } else {
          read_acc(chunk, v);
        }
        lin_finish_chunk<PASS, OUT_F32>(p, t, buf, lane, chunk * 32, col0, bias, v);
      }
      if (split && last && lane == 0) *cnt = 0u;
      if (some) {
        if (side * 32 >= t.w) release();               // no chunk of this warp's
        next_acc();
      }
    }
    if (!ok && lane == 0) raise_error(p.err, abort_flag, kErrEpilogueWait);
  }

  __syncthreads();
  if (PAIR) ptx::cluster_sync_all();                   // the peer may still signal this CTA's barriers
  if (warp == 1) {
    __syncwarp();
    ptx::tc_fence_after();
    if (PAIR) ptx::tmem_dealloc_pair(tmem_base, TMEM_COLS);
    else ptx::tmem_dealloc(tmem_base, TMEM_COLS);
  }
}

}  // namespace goldy
