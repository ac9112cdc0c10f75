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
// stage may hold rows of the next group, which a further warp zeroes in
// shared memory before the stage is used (zero times whatever the neighbour holds
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
// Roles: warp 0 loads by TMA, warp 1 issues the MMAs, the other warps drain
// the accumulator (double buffered in tensor memory) straight from registers
// to C, and bias, activation, its gradient, residual and the saved
// pre-activation cost no further pass over C.
//
// OUT_F32: the tensor cores add into fp32 accumulators with truncation, a
// relative error of about 1e-9 per reduction element (4.4e-6 at 4096,
// measured against fp64).  fp32 results therefore leave tensor memory every
// kLinPromote stages (768 elements) and are summed in registers with rounding
// to nearest: off by 2.3e-7 (256 elements) to 7.4e-7 (262144), an fp32 product by 1.1e-7
// to 4.6e-7, of the result's norm for normal inputs.  (Parts of 512 elements are good to 5e-7, but
// the drain of a tile, 3.6 us, then holds its accumulator past the next tile's
// first part: 58 against 53 us for a 2048 x 8192 gradient over 2048 rows.)  bf16
// results (relative rounding 2^-8) keep the whole sum in tensor memory, but for weight
// gradients over more than kLinLongRows rows, which are PROMOTEd like fp32 ones, in
// parts of 8192 rows: a million rows would lose 1e-3 of their sum.
//
// A launch begins while the kernel before it still runs, so nothing that one may
// have written (offsets, Z, R) goes through the read-only data path, which
// wants data that does not change while the kernel lives: plain loads behind
// griddepcontrol.wait.
//
// Every wait is bounded; a wait that runs out sets the error word and the
// kernel ends.
#pragma once

#include "go_kernel.cuh"
#include "layer_internal.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {

// Arrive on an mbarrier of a CTA of the cluster, ordering no memory but this
// CTA's: all a drained accumulator needs (tcgen05 fences order the reads of
// tensor memory).  A release at cluster scope would wait for the warp's stores
// to C, about a microsecond per tile.
__device__ __forceinline__ void lin_arrive_remote(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}

// True in one lane of a converged warp; `leader` gets that lane's number.  The
// copies, MMAs and commits stand under this predicate, not under lane == 0:
// they take their operands from registers shared by the warp, and only here
// does the compiler know that one lane runs them.  Under lane == 0 each became
// a loop over the lanes, some 70 cycles apiece, and no tile, however narrow,
// took less than 290 ns per 64-deep stage.
__device__ __forceinline__ bool lin_elect(int& leader) {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync %0|p, 0xFFFFFFFF;\n\tselp.u32 %1, 1, 0, p;\n\t}"
               : "=r"(leader), "=r"(one));
  return one != 0;
}

// One K = 16 step of a product, operands by the low words of their shared-memory
// descriptors (the address in 16-byte units and the leading offset); the high
// words are constant, which leaves an addition per step to the issuing lane.
template <bool PAIR>
__device__ __forceinline__ void lin_mma(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t add) {
  constexpr uint32_t HI = (1024u >> 4) | (1u << 14) | (2u << 29);   // 8-row groups 1024 bytes apart, version 1, 128-byte swizzle
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(add), "r"(HI)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(add), "r"(HI)
        : "memory");
}

// Whether the phase with parity `parity` has completed, without waiting.
__device__ __forceinline__ bool lin_test(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}

// A value that all lanes share, in a form that the compiler knows to be shared.
__device__ __forceinline__ int lin_shared(int x) { return __shfl_sync(0xFFFFFFFFu, x, 0); }

// Bounded wait for the phase with parity `parity`, false if it gave up (the
// limit, or another role's abort flag).  The timer is read at every 64th poll.
// (Arrivals over tensor memory are ordered by the tcgen05 fences; CLUSTER adds
// acquire at cluster scope for the peer's shared memory.)
template <bool CLUSTER = false>
__device__ __forceinline__ bool lin_wait(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
  uint64_t t0 = 0;
  for (uint32_t n = 1;; ++n) {
    if (CLUSTER ? ptx::mbar_try_wait_acq_cluster(bar, parity) : ptx::mbar_try_wait(bar, parity)) return true;
    if ((n & 63) != 0) continue;
    if (abort_flag != nullptr && *abort_flag) return false;
    const uint64_t now = ptx::global_timer();
    if (t0 == 0) t0 = now;
    else if (now - t0 > ptx::kWaitLimitNs) return false;
  }
}
// The same for a whole warp, with one answer for all lanes.
template <bool CLUSTER = false>
__device__ __forceinline__ bool lin_wait_warp(uint32_t bar, uint32_t parity, const volatile int* abort_flag) {
  return __all_sync(0xFFFFFFFFu, lin_wait<CLUSTER>(bar, parity, abort_flag));
}

// Stages per accumulator of a promoted result: equal parts of at most MOST.
template <int MOST>
__device__ __forceinline__ int lin_promote(int kbs) {
  const int parts = (kbs + MOST - 1) / MOST;
  return parts > 1 ? int(unsigned(kbs + parts - 1) / unsigned(parts)) : kbs;
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

__device__ __forceinline__ int lin_div(int n, const LinDivisor& d) {
  return d.one ? n : int(__umul64hi(uint64_t(unsigned(n)), d.mul));
}

// Walks the units of a launch in increasing order.  All lanes of a warp call
// it together; groups are looked up 32 at a time (offsets clamped to
// [0, rows] and taken as non-decreasing, so that no offsets make a launch
// leave its buffers).  Every warp of every role walks, so a step within a
// group has no division.
template <int PASS, bool PAIR>
struct LinWalk {
  static constexpr int G = PAIR ? 32 : 16;     // granularity of N
  const LinearParams& p;
  const int lane;
  // the current group: its units, rows, tile height, row tiles, and 2^32 over
  // the tiles of its last band
  int e = 0, first = 0, end = 0, start = 0, rows = 0, w = 0, n_r = 0;
  unsigned last_inv = 0;
  // forward and input gradient: a window of 32 groups, one per lane
  int e0 = 0, begin = 0, prev = 0;             // its first group, units and rows before it
  int my_start = 0, my_rows = 0, my_end = 0;   // this lane's group: first row, rows, end of its units

  __device__ LinWalk(const LinearParams& params, int lane_id) : p(params), lane(lane_id) {
    if (PASS == kLinWeightGrad || !p.offsets) {
      rows = PASS == kLinWeightGrad ? p.size_r : p.rows;
      end = set_group();
    } else {
      load_window();
    }
  }

  __device__ static int width(int rows, int tile_r) {
    if (rows <= 0) return G;
    const int n = int((unsigned(rows) + tile_r - 1) / unsigned(tile_r));      // equal tiles
    return int((unsigned(rows) + n - 1) / unsigned(n) + G - 1) / G * G;
  }
  // tile height and count of the current group from its rows; returns its units
  __device__ int set_group() {
    w = width(rows, p.tile_r);
    n_r = int((unsigned(rows) + w - 1) / unsigned(w));
    const int rest = n_r % kLinRowBand;
    last_inv = rest > 1 ? 0xFFFFFFFFu / unsigned(rest) + 1u : 0u;
    return n_r * p.tiles_c * p.split;
  }
  __device__ void load_window() {
    const int g = e0 + lane;
    int o = 0, o1 = 0;
    if (g < p.groups) {
      o = min(max(p.offsets[g], 0), p.rows);
      o1 = min(max(p.offsets[g + 1], 0), p.rows);
    }
    int m = max(o, prev);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int t = __shfl_up_sync(0xFFFFFFFFu, m, d);
      if (lane >= d) m = max(m, t);
    }
    my_start = m;
    my_rows = g < p.groups ? max(o1 - m, 0) : 0;
    const int mw = width(my_rows, p.tile_r);
    int u = int((unsigned(my_rows) + mw - 1) / unsigned(mw)) * p.tiles_c * p.split;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int t = __shfl_up_sync(0xFFFFFFFFu, u, d);
      if (lane >= d) u += t;
    }
    my_end = begin + u;
  }

  // Unit u (not below the last one asked for); false past the end.
  __device__ __forceinline__ bool find(int u, LinUnit& t) {
    if (PASS == kLinWeightGrad) {
      while (u >= end) {
        if (++e >= p.groups) return false;
        const int units = end - first;
        first = end;
        end += units;
      }
      int a = 0, b = p.rows;
      if (p.offsets) {
        a = min(max(p.offsets[e], 0), p.rows);
        b = min(max(p.offsets[e + 1], a), p.rows);
      }
      t.k0 = a;
      t.red = b - a;
    } else {
      if (u >= end) {
        if (!p.offsets) return false;
        int last;
        while (u >= (last = __shfl_sync(0xFFFFFFFFu, my_end, 31))) {
          if (e0 + 32 >= p.groups) return false;
          prev = __shfl_sync(0xFFFFFFFFu, my_start + my_rows, 31);
          begin = last;
          e0 += 32;
          load_window();
        }
        const int j = __ffs(__ballot_sync(0xFFFFFFFFu, u < my_end)) - 1;
        e = e0 + j;
        start = __shfl_sync(0xFFFFFFFFu, my_start, j);
        rows = __shfl_sync(0xFFFFFFFFu, my_rows, j);
        end = __shfl_sync(0xFFFFFFFFu, my_end, j);
        first = end - set_group();
      }
      t.k0 = 0;
      t.red = p.red;
    }
    t.e = e;
    const int local = u - first;
    const int i = lin_div(local, p.div_split);
    t.s = local - i * p.split;
    t.tile = lin_div(u, p.div_split);
    const int band = lin_div(i, p.div_band);
    const int rem = i - band * kLinRowBand * p.tiles_c;
    const int in_band = min(kLinRowBand, n_r - band * kLinRowBand);
    const int tc = in_band == kLinRowBand ? rem / kLinRowBand : in_band == 1 ? rem : int(__umulhi(unsigned(rem), last_inv));
    const int tr = band * kLinRowBand + rem - tc * in_band;
    t.r0 = start + tr * w;
    t.w = min(w, rows - tr * w);
    t.nw = (t.w + G - 1) / G * G;
    t.c0 = tc * (PAIR ? 256 : 128);
    const int kbs = (t.red + kLinStageK - 1) / kLinStageK;
    t.kb0 = lin_div(kbs * t.s, p.div_split);
    t.kb1 = lin_div(kbs * (t.s + 1), p.div_split);
    return true;
  }
};

// Brings `bytes` from `at` on into L2.
__device__ __forceinline__ void lin_prefetch(const char* at, int bytes) {
  for (int i = 0; i < bytes; i += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(at + i));
  asm volatile("prefetch.global.L2 [%0];" ::"l"(at + bytes - 1));
}

// 8 accumulator columns of this warp's 32 lanes: tensor memory -> registers,
// and back.
__device__ __forceinline__ void lin_tmem_load(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr)
               : "memory");
}
__device__ __forceinline__ void lin_tmem_store(uint32_t taddr, const float (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "f"(v[0]),
               "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
               : "memory");
}
__device__ __forceinline__ void lin_tmem_store_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// Transposes the 2 x 2 block of bf16 values that an even lane and the odd lane
// next to it hold: (rows j, j + 1 of one column) <-> (two columns of one row,
// the even lane's row j, the odd lane's row j + 1).
__device__ __forceinline__ uint32_t lin_trade(uint32_t x, int odd) {
  const uint32_t y = __shfl_xor_sync(0xFFFFFFFFu, x, 1);
  return __byte_perm(x, y, odd ? 0x3276 : 0x5410);
}

// Drains this warp's part of a tile: 32 columns, one per lane, in chunks of 8
// rows (chunks side, side + SIDES, ...).  The arithmetic is per column; bf16
// values meet memory two columns at a time (PAIRS: rows on 4-byte boundaries
// and 32 whole columns), so that an access covers two 64-byte row segments;
// fp32 rows are 128-byte segments as they are.  The next chunk's accumulator
// columns, saved pre-activations and residuals are on their way while a chunk
// is finished.  The loop body is kept short: unrolled over 32 rows, the same
// work waited for instructions (5.5 us a tile instead of 2).
constexpr int kLinSides = kLinEpiWarps / 4;

constexpr int kLinNo = 0, kLinYes = 1, kLinMaybe = 2;

// What a drain needs.
struct LinDrain {
  char* c;                 // this lane's first element of C, of R, and of Z
  const char* q;
  char* z;
  int64_t c_step, q_step, z_step;   // bytes between the rows that it takes in turn
  const float* part;       // splits' partials (null: the accumulator)
  int64_t split_stride;
  int split;
  uint32_t cols;           // the accumulator's first column
  uint32_t release;        // barrier of the accumulator's drain
  int rows, side, lane;
  float bias;
  bool some;               // the sum is in the accumulator
  bool save, has_q;        // Z is written; there is an R
  bool in;                 // this lane's column exists
};

template <int PASS, bool PAIR, bool OUT_F32, int ACT, bool PAIRS, int RES_IS>
__device__ __forceinline__ void lin_drain(LinDrain d) {
  constexpr bool SLOPE = PASS == kLinInputGrad && ACT != GOLDY_ACT_NONE;
  constexpr int N = PAIRS ? 4 : 8;                 // accesses per chunk and array
  constexpr int DOWN = PAIRS ? 2 : 1;              // rows between them
  constexpr bool AHEAD = PAIRS || OUT_F32;         // else loaded where they are used (edges, odd strides)
  const bool RES = RES_IS == kLinMaybe ? d.has_q : RES_IS == kLinYes;
  const bool SAVE = PASS == kLinForward && d.save;
  const int odd = PAIRS ? (d.lane & 1) : 0;
  const int rows = d.in ? d.rows - odd : 0;        // this lane stores chunk-relative row i while i < rows - chunk * 8
  const int chunks = (d.rows + 7) / 8;
  const char* z_at = d.z;

  uint32_t z[N], q[N], an[8];
  // what a chunk needs from memory, asked for as soon as the last chunk's has
  // been used: nothing is copied, for a copy would wait for the load
  auto fetch_z = [&](int chunk) {
    const int left = chunk < chunks ? rows - chunk * 8 : 0;
    if (SLOPE) {
#pragma unroll
      for (int i = 0; i < N; ++i, z_at += d.z_step)
        if (DOWN * i < left)
          z[i] = PAIRS ? *reinterpret_cast<const uint32_t*>(z_at) : uint32_t(*reinterpret_cast<const uint16_t*>(z_at));
      z_at += (kLinSides - 1) * N * d.z_step;
    }
  };
  auto fetch_q = [&](int chunk) {
    const int left = chunk < chunks ? rows - chunk * 8 : 0;
    if (RES) {
#pragma unroll
      for (int i = 0; i < N; ++i, d.q += d.q_step)
        if (DOWN * i < left)
          q[i] = PAIRS || OUT_F32 ? *reinterpret_cast<const uint32_t*>(d.q)
                                  : uint32_t(*reinterpret_cast<const uint16_t*>(d.q));
      d.q += (kLinSides - 1) * N * d.q_step;
    }
  };
  auto release = [&]() {                           // this warp has read the accumulator
    ptx::tc_fence_before();
    __syncwarp();
    if (d.lane == 0) {
      if (PAIR) lin_arrive_remote(d.release);
      else ptx::mbar_arrive(d.release);
    }
  };
  if (AHEAD) {
    fetch_z(d.side);
    fetch_q(d.side);
  }
  if (d.some && d.side < chunks) lin_tmem_load(d.cols + uint32_t(d.side * 8), an);
#pragma unroll 1
  for (int chunk = d.side; chunk < chunks; chunk += kLinSides) {
    const int left = rows - chunk * 8;
    if (!AHEAD) fetch_z(chunk);
    float v[8];
    uint64_t slope[4];
    if (SLOPE) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w = PAIRS ? lin_trade(z[i], odd) : (z[(2 * i) % N] & 0xFFFFu) | (z[(2 * i + 1) % N] << 16);
        slope[i] = act_slope2(two(bf16_lo(w), bf16_hi(w)), ACT);
      }
    }
    if (AHEAD) fetch_z(chunk + kLinSides);
    if (d.some) {
      ptx::tmem_ld_wait();
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(an[j]);
      if (chunk + kLinSides < chunks) lin_tmem_load(d.cols + uint32_t((chunk + kLinSides) * 8), an);
      else release();                              // the last chunk is in registers
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = 0.0f;
      if (d.part) {                                // in the splits' order
        const float* from = d.part + (chunk / kLinSides) * 256 + d.lane;
#pragma unroll 4
        for (int s = 0; s < d.split; ++s) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] += __ldcg(from + s * d.split_stride + j * 32);
        }
      }
    }
    if (PASS == kLinForward) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += d.bias;
    }
    if (SAVE) {
#pragma unroll
      for (int i = 0; i < N; ++i, d.z += d.z_step) {
        if (PAIRS) {
          const uint32_t w = lin_trade(pack_bf16(v[2 * i], v[2 * i + 1]), odd);
          if (2 * i < left) *reinterpret_cast<uint32_t*>(d.z) = w;
        } else if (i < left) {
          store_bf16(d.z, 0, v[i]);
        }
      }
      d.z += (kLinSides - 1) * N * d.z_step;
    }
    if (SLOPE || (PASS == kLinForward && ACT != GOLDY_ACT_NONE)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint64_t pair = two(v[2 * i], v[2 * i + 1]);
        pair = SLOPE ? mul2(pair, slope[i]) : act_value2(pair, ACT);
        const float2 r = apart(pair);
        v[2 * i] = r.x;
        v[2 * i + 1] = r.y;
      }
    }
    if (!AHEAD) fetch_q(chunk);
    if (RES) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (PAIRS) {
          const uint32_t w = lin_trade(q[i], odd);
          v[2 * i] += bf16_lo(w);
          v[2 * i + 1] += bf16_hi(w);
        } else {
          v[i] += OUT_F32 ? __uint_as_float(q[i]) : bf16_lo(q[i]);
        }
      }
    }
    if (AHEAD) fetch_q(chunk + kLinSides);
#pragma unroll
    for (int i = 0; i < N; ++i, d.c += d.c_step) {
      if (PAIRS) {
        const uint32_t w = lin_trade(pack_bf16(v[2 * i], v[2 * i + 1]), odd);
        if (2 * i < left) *reinterpret_cast<uint32_t*>(d.c) = w;
      } else if (i < left) {
        if (OUT_F32) *reinterpret_cast<float*>(d.c) = v[i];
        else store_bf16(d.c, 0, v[i]);
      }
    }
    d.c += (kLinSides - 1) * N * d.c_step;
  }
}

template <int PASS, bool PAIR, bool OUT_F32, int ACT, bool PAIRS>
__device__ __forceinline__ void lin_drain_as(const LinearParams& p, const LinUnit& t, int col0, LinDrain d) {
  constexpr int64_t ES = OUT_F32 ? 4 : 2;
  const int odd = PAIRS ? (d.lane & 1) : 0;
  const int col = col0 + d.lane - odd;
  const int64_t r = int64_t(t.r0) + d.side * 8 + odd;
  const int64_t down = PAIRS ? 2 : 1;
  const void* z = PASS == kLinInputGrad ? p.z_in : p.z_out;
  d.in = col < p.size_c;
  d.c = static_cast<char*>(p.c) + (int64_t(t.e) * p.c_group + r * p.ldc + col) * ES;
  d.q = static_cast<const char*>(p.res) + (int64_t(t.e) * p.r_group + r * p.ldr + col) * ES;
  d.z = static_cast<char*>(const_cast<void*>(z)) + (r * p.ldz + col) * 2;
  d.c_step = down * p.ldc * ES;
  d.q_step = down * p.ldr * ES;
  d.z_step = down * p.ldz * 2;
  d.save = p.z_out != nullptr;
  d.has_q = p.res != nullptr;
  // a drain of its own with a residual where that costs no registers
  if (PASS == kLinInputGrad || !PAIRS) lin_drain<PASS, PAIR, OUT_F32, ACT, PAIRS, kLinMaybe>(d);
  else if (p.res) lin_drain<PASS, PAIR, OUT_F32, ACT, PAIRS, kLinYes>(d);
  else lin_drain<PASS, PAIR, OUT_F32, ACT, PAIRS, kLinNo>(d);
}

template <int PASS, int ACT, bool PAIR, bool OUT_F32, bool PROMOTE>
__global__ void __launch_bounds__(lin_threads(PASS), 1) linear_kernel(const __grid_constant__ LinearParams p) {
  constexpr bool A_MN = PASS != kLinInputGrad;         // P contiguous along c
  constexpr bool B_MN = PASS == kLinWeightGrad;        // Q contiguous along r
  constexpr bool TAIL = PASS == kLinWeightGrad;        // ragged reduction
  constexpr int PART = OUT_F32 ? kLinPromote : kLinPromoteLong;   // PROMOTE: stages per accumulator, at most
  constexpr int ACC = 2;
  constexpr int A_BYTES = 128 * kLinStageK * 2;
  constexpr int CTAS = PAIR ? 2 : 1;
  constexpr uint32_t TMEM_COLS = 512;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const int stages = p.stages;
  const uint32_t stage_bytes = uint32_t(p.stage_bytes);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + size_t(stages) * stage_bytes);
  uint64_t* full = bars;                               // pair: used in the even CTA only
  uint64_t* empty = bars + kLinMaxStages;
  uint64_t* tfull = bars + 2 * kLinMaxStages;
  uint64_t* tempty = tfull + ACC;
  uint64_t* drain = tempty + ACC;
  uint64_t* tail = drain + 1;                          // a group's last, ragged stage has landed in this CTA
  uint64_t* peer = tail + kLinMaxStages;               // even CTA: the odd CTA has zeroed its part of one
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(peer + kLinMaxStages);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const uint32_t tiles = ptx::smem_u32(smem);
  const int warp = lin_shared(threadIdx.x >> 5);
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
      ptx::mbar_init(ptx::smem_u32(&full[s]), 1);
      ptx::mbar_init(ptx::smem_u32(&empty[s]), 1);
      if (TAIL) {
        ptx::mbar_init(ptx::smem_u32(&tail[s]), 1);
        ptx::mbar_init(ptx::smem_u32(&peer[s]), 1);
      }
    }
    for (int a = 0; a < ACC; ++a) {
      ptx::mbar_init(ptx::smem_u32(&tfull[a]), 1);
      ptx::mbar_init(ptx::smem_u32(&tempty[a]), kLinEpiWarps * CTAS);
    }
    ptx::mbar_init(ptx::smem_u32(drain), 1);
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
  const uint32_t tmem_base = uint32_t(lin_shared(int(*tmem_slot)));
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();                                 // inputs and offsets may come from the previous kernel

  LinWalk<PASS, PAIR> walk(p, lane);
  LinUnit t;
  // weight gradient: the unit's last stage holds rows of the next group behind
  // this one's last
  auto ragged = [&]() {
    return TAIL && t.kb1 > t.kb0 && t.red < t.kb1 * kLinStageK && t.k0 + t.red < p.rows;
  };

  if (warp == 0) {
    // -------------------------------------------------------------- loads
    int stage = 0;
    uint32_t phase = 0, issued = 0, last_phase = 0;
    bool ok = true;
    for (int u = worker; ok && walk.find(u, t); u += n_workers) {
      t.e = lin_shared(t.e), t.r0 = lin_shared(t.r0), t.nw = lin_shared(t.nw), t.c0 = lin_shared(t.c0);
      t.k0 = lin_shared(t.k0), t.red = lin_shared(t.red), t.kb0 = lin_shared(t.kb0), t.kb1 = lin_shared(t.kb1);
      const int half = t.nw / CTAS;                    // rows of Q this CTA stages
      const int r0 = t.r0 + int(rank) * half;
      const int c0 = t.c0 + int(rank) * 128;
      const bool full_box = !B_MN && t.nw == p.tile_r;
      const int boxes = B_MN ? (half + 63) / 64 : full_box ? 1 : (half + p.part_box - 1) / p.part_box;
      const uint32_t box_bytes = B_MN ? 8192u : uint32_t(full_box ? half : p.part_box) * 128u;
      const uint32_t bytes = A_BYTES + boxes * box_bytes;
      const int e = PASS == kLinWeightGrad ? 0 : t.e;
      // one lane: starts a stage's copies, which complete on `bar`
      auto fill = [&](int kb, uint32_t bar) {
        const uint32_t as = tiles + stage * stage_bytes;
        const uint32_t bs = as + A_BYTES;
        const int k = t.k0 + kb * kLinStageK;
        auto load = [&](uint32_t dst, const void* map, int x, int y, int z) {
          if (PAIR) ptx::tma_load_3d_pair(dst, map, bar, x, y, z);
          else ptx::tma_load_3d(dst, map, bar, x, y, z);
        };
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
      };
      auto claim_stage = [&]() {
        if (issued >> stage & 1) ok = lin_wait(ptx::smem_u32(&empty[stage]), phase ^ 1, abort_flag);
        issued |= 1u << stage;
        return ok;
      };
      auto next_stage = [&]() {
        last_phase = (last_phase & ~(1u << stage)) | (phase << stage);
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
      };
      const int whole = ragged() ? t.kb1 - 1 : t.kb1;
      int leader;
      if (lin_elect(leader)) {
        for (int kb = t.kb0; kb < t.kb1; ++kb) {
          if (!claim_stage()) break;
          if (TAIL && kb >= whole) {                   // lands on this CTA's own barrier, to be mended
            const uint32_t tb = ptx::smem_u32(&tail[stage]);
            ptx::mbar_arrive_expect_tx(tb, bytes);
            fill(kb, PAIR ? ptx::map_to_rank(tb, rank) : tb);
          } else {
            const uint32_t fb = ptx::smem_u32(&full[stage]);
            if (lead) ptx::mbar_arrive_expect_tx(fb, CTAS * bytes);
            fill(kb, PAIR ? ptx::map_to_rank(fb, 0) : fb);   // a pair's copies complete in the even CTA
          }
          next_stage();
        }
      }
      __syncwarp();
      ok = __shfl_sync(0xFFFFFFFFu, ok, leader);
      // the tile's rows of Z and R come into L2 while its products, and the
      // drain of the tile before, are under way (a warp's 32 columns and its
      // neighbours' fill whole lines)
      if (PASS == kLinInputGrad ? (p.z_in || p.res) : p.res != nullptr) {
        const int first = t.c0 + int(rank) * 128, last = min(first + 128, p.size_c) - 1;
        for (int row = lane; row < t.w && last >= first; row += 32) {
          const int64_t r = int64_t(t.r0) + row;
          if (PASS == kLinInputGrad && p.z_in)
            lin_prefetch(static_cast<const char*>(p.z_in) + (r * p.ldz + first) * 2, (last - first + 1) * 2);
          if (p.res) {
            constexpr int ES = OUT_F32 ? 4 : 2;
            lin_prefetch(static_cast<const char*>(p.res) + (int64_t(t.e) * p.r_group + r * p.ldr + first) * ES,
                         (last - first + 1) * ES);
          }
        }
      }
    }
    if (!ok && lane == 0) raise_error(p.err, abort_flag, kErrProducerWait);
    // every stage filled must have been consumed (and, for a pair, both CTAs'
    // commits landed) before the CTA may leave
    int leader;
    if (lin_elect(leader)) {
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
      int stage = 0, acc = 0, leader = 0;
      uint32_t phase = 0, acc_phase = 0, acc_used = 0;
      bool ok = true, any = false, ready = false;      // `any` and the ring's state: the elected lane's
      const uint32_t full_at = ptx::smem_u32(full), words = stage_bytes >> 4;
      const uint32_t a_base = (tiles >> 4) | (uint32_t((A_MN ? 8192 : 16) >> 4) << 16);
      const uint32_t b_base = ((tiles + A_BYTES) >> 4) | (uint32_t((B_MN ? 8192 : 16) >> 4) << 16);
      for (int u = worker; ok && walk.find(u, t); u += n_workers) {
        const int nw = lin_shared(t.nw), kb0 = lin_shared(t.kb0), kb1 = lin_shared(t.kb1);
        const uint32_t idesc = ptx::make_idesc_bf16(128 * CTAS, 16, A_MN, B_MN) + (uint32_t((nw - 16) >> 3) << 17);
        const int step = PROMOTE ? lin_promote<PART>(kb1 - kb0) : kb1 - kb0;
        if (lin_elect(leader)) {
          ready = false;
          for (int kb = kb0; kb < kb1;) {
            const int stop = min(kb + step, kb1);
            if (acc_used >> acc & 1) {
              ok = lin_wait<PAIR>(ptx::smem_u32(&tempty[acc]), acc_phase ^ 1, abort_flag);
              if (!ok) break;
            }
            acc_used |= 1u << acc;
            ptx::tc_fence_after();
            const uint32_t d = tmem_base + uint32_t(acc * 256);
            uint32_t add = 0;
            for (; kb < stop; ++kb) {
              if (!ready) ok = lin_wait(full_at + stage * 8, phase, abort_flag);
              if (!ok) break;
              ptx::tc_fence_after();
              const uint32_t a_lo = a_base + stage * words, b_lo = b_base + stage * words;
#pragma unroll
              for (int kk = 0; kk < 4; ++kk)
                lin_mma<PAIR>(d, a_lo + kk * (A_MN ? 2048 : 32) / 16, b_lo + kk * (B_MN ? 2048 : 32) / 16, idesc,
                              kk > 0 ? 1u : add);
              if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(&empty[stage]), 0x3);
              else ptx::mma_commit(ptx::smem_u32(&empty[stage]));
              add = 1;
              any = true;
              if (++stage == stages) {
                stage = 0;
                phase ^= 1;
              }
              ready = lin_test(full_at + stage * 8, phase);   // the answer arrives behind the loop's end
            }
            if (!ok) break;
            if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(&tfull[acc]), 0x3);
            else ptx::mma_commit(ptx::smem_u32(&tfull[acc]));
            if (++acc == ACC) {
              acc = 0;
              acc_phase ^= 1;
            }
          }
        }
        __syncwarp();
        ok = __shfl_sync(0xFFFFFFFFu, ok, leader);
      }
      if (!ok) {
        if (lane == 0) raise_error(p.err, abort_flag, kErrMmaWait);
        if (lin_elect(leader) && any) {
          if (PAIR) ptx::mma_commit_pair_multicast(ptx::smem_u32(drain), 0x1);
          else ptx::mma_commit(ptx::smem_u32(drain));
          lin_wait(ptx::smem_u32(drain), 0, nullptr);
        }
        __syncwarp();
      }
    }
  } else if (TAIL && warp == 2 + kLinEpiWarps) {
    // -------------------------------------------------------------- mending
    // A ragged stage lands on this CTA's own barrier.  The warp zeroes what is
    // behind the group's last row (lines of 128 bytes, one per reduction row,
    // in 8 KB blocks of 64 columns) and then hands the stage to the MMAs.
    // A warp of its own: the load warp would stop loading meanwhile, and the
    // MMA warp multiplying (43 against 38 us for 8 groups of about 1000 rows,
    // 2048 x 1024 each).
    int stage = 0;
    uint32_t tail_phase = 0;
    bool ok = true;
    for (int u = worker; ok && walk.find(u, t); u += n_workers) {
      const int kbs = t.kb1 - t.kb0;
      if (ragged()) {
        const int at = (stage + kbs - 1) % stages;
        const uint32_t parity = tail_phase >> at & 1;
        tail_phase ^= 1u << at;
        ok = lin_wait_warp(ptx::smem_u32(&tail[at]), parity, abort_flag);
        const uint32_t as = tiles + at * stage_bytes;
        const int valid = t.red - (t.kb1 - 1) * kLinStageK;
        const int pieces = (kLinStageK - valid) * 8;
        const int blocks = 2 + (t.nw / CTAS + 63) / 64;
        for (int b = 0; b < blocks; ++b)
          for (int i = lane; i < pieces; i += 32) ptx::st_shared_v4(as + b * 8192 + valid * 128 + i * 16, 0, 0, 0, 0);
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (PAIR && lead && ok) ok = lin_wait_warp<true>(ptx::smem_u32(&peer[at]), parity, abort_flag);
        if (lane == 0) {
          if (lead) ptx::mbar_arrive(ptx::smem_u32(&full[at]));
          else ptx::mbar_arrive_remote_release(ptx::map_to_rank(ptx::smem_u32(&peer[at]), 0));
        }
      }
      stage = (stage + kbs) % stages;
    }
    if (!ok && lane == 0) raise_error(p.err, abort_flag, kErrProducerWait);
  } else {
    // ------------------------------------------------------------ epilogue
    constexpr int MOST = ((OUT_F32 ? kLinMaxTileF32 : 256) / 8 + kLinSides - 1) / kLinSides;   // 8-row chunks of a tile per warp
    const int ew = warp - 2;
    const int q = warp & 3;                            // lanes of tensor memory this warp may read
    const int side = ew >> 2;                          // takes chunks side, side + kLinSides, ...
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
        if (PAIR) lin_arrive_remote(ptx::map_to_rank(b, 0));
        else ptx::mbar_arrive(b);
      }
    };
    for (int u = worker; ok && walk.find(u, t); u += n_workers) {
      const int col0 = t.c0 + int(rank) * 128 + q * 32;
      float bias = 0.0f;
      if (PASS == kLinForward && p.bias && col0 + lane < p.size_c) {
        const int64_t at = int64_t(t.e) * p.size_c + col0 + lane;
        bias = p.bias_f32 ? static_cast<const float*>(p.bias)[at] : load_bf16(p.bias, at);
      }
      const int chunks = (t.w + 7) / 8;
      const bool some = t.kb1 > t.kb0;                 // else the sum is empty and no accumulator is used
      const bool split = p.split > 1;
      uint32_t cols = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(acc * 256);
      if (PROMOTE && t.kb1 - t.kb0 > PART) {
        // sum the accumulators of some PART stages each.  An fp32 weight
        // gradient is stored from here, starting from what it is added to, so
        // that the last accumulator is free at once; other totals go back into
        // the last one's tensor memory, where the code below finds them.
        const int step = lin_promote<PART>(t.kb1 - t.kb0);
        const bool direct = PASS == kLinWeightGrad && OUT_F32 && !split;
        const int64_t c_step = p.ldc * 4;
        char* c_out = static_cast<char*>(p.c) + (int64_t(t.e) * p.c_group + (int64_t(t.r0) + side * 8) * p.ldc + col0 + lane) * 4;
        const int c_rows = col0 + lane < p.size_c ? t.w - side * 8 : 0;
        float sum[MOST][8];
#pragma unroll
        for (int i = 0; i < MOST; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[i][j] = 0.0f;
        if (direct && p.res) {
          const char* from = c_out;
#pragma unroll
          for (int i = 0; i < MOST; ++i, from += (kLinSides - 1) * 8 * c_step)
#pragma unroll
            for (int j = 0; j < 8; ++j, from += c_step)
              if (i * kLinSides * 8 + j < c_rows) sum[i][j] = *reinterpret_cast<const float*>(from);
        }
        for (int kb = t.kb0; kb < t.kb1; kb += step) {
          ok = lin_wait_warp(ptx::smem_u32(&tfull[acc]), acc_phase, abort_flag);
          if (!ok) break;
          ptx::tc_fence_after();
          cols = tmem_base + (uint32_t(q * 32) << 16) + uint32_t(acc * 256);
#pragma unroll
          for (int i = 0; i < MOST; ++i) {
            const int chunk = side + kLinSides * i;
            if (chunk < chunks) {
              uint32_t raw[8];
              lin_tmem_load(cols + uint32_t(chunk * 8), raw);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 8; ++j) sum[i][j] += __uint_as_float(raw[j]);
            }
          }
          if (direct || kb + step < t.kb1) {
            release();
            next_acc();
          }
        }
        if (!ok) break;
        if (direct) {
#pragma unroll
          for (int i = 0; i < MOST; ++i, c_out += (kLinSides - 1) * 8 * c_step)
#pragma unroll
            for (int j = 0; j < 8; ++j, c_out += c_step)
              if (i * kLinSides * 8 + j < c_rows) *reinterpret_cast<float*>(c_out) = sum[i][j];
          continue;
        }
#pragma unroll
        for (int i = 0; i < MOST; ++i)
          if (side + kLinSides * i < chunks) lin_tmem_store(cols + uint32_t((side + kLinSides * i) * 8), sum[i]);
        lin_tmem_store_wait();
      } else if (some) {
        ok = lin_wait_warp(ptx::smem_u32(&tfull[acc]), acc_phase, abort_flag);
        if (!ok) break;
        ptx::tc_fence_after();
      }
      // partials of this warp's part of the tile: [split][chunk][row][column]
      float* part = p.part + ((size_t(t.tile) * p.split * CTAS + rank) * kLinEpiWarps + ew) * (size_t(p.part_chunks) * 256);
      const size_t split_stride = size_t(CTAS) * kLinEpiWarps * p.part_chunks * 256;
      if (split) {
#pragma unroll 1
        for (int chunk = side; chunk < chunks; chunk += kLinSides) {
          uint32_t raw[8];
          if (some) {
            lin_tmem_load(cols + uint32_t(chunk * 8), raw);
            ptx::tmem_ld_wait();
          }
          float* to = part + t.s * split_stride + (chunk / kLinSides) * 256 + lane;
#pragma unroll
          for (int j = 0; j < 8; ++j) __stcg(to + j * 32, some ? __uint_as_float(raw[j]) : 0.0f);
        }
        if (some) {
          release();
          next_acc();
        }
        // the last of the splits to arrive sums all of them in split order and
        // leaves the counter at zero
        unsigned* cnt = p.cnt + (size_t(t.tile) * CTAS + rank) * kLinEpiWarps + ew;
        __threadfence();
        __syncwarp();
        unsigned old = 0;
        if (lane == 0) {
          old = atomicAdd(cnt, 1u);
          if (old == unsigned(p.split - 1)) *cnt = 0u;
        }
        if (__shfl_sync(0xFFFFFFFFu, old, 0) != unsigned(p.split - 1)) continue;
        __threadfence();
      }
      const bool from_acc = some && !split;
      LinDrain d;
      d.part = split ? part : nullptr;
      d.split_stride = int64_t(split_stride);
      d.split = p.split;
      d.cols = cols;
      d.release = PAIR ? ptx::map_to_rank(ptx::smem_u32(&tempty[acc]), 0) : ptx::smem_u32(&tempty[acc]);
      d.rows = t.w;
      d.side = side;
      d.lane = lane;
      d.bias = bias;
      d.some = from_acc;
      if (!OUT_F32 && p.vec && col0 + 32 <= p.size_c)
        lin_drain_as<PASS, PAIR, OUT_F32, ACT, !OUT_F32>(p, t, col0, d);
      else
        lin_drain_as<PASS, PAIR, OUT_F32, ACT, false>(p, t, col0, d);
      if (from_acc) {
        if (side >= chunks) release();                 // no chunk of this warp's
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
