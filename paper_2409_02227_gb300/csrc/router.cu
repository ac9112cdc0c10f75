// A router: the k largest of each row's logits, their softmax weights, and the
// logits' gradient.
//
//   weight of a chosen expert e = scale exp(l_e - m) / sum exp(l - m),  m the row's largest logit
//   dl_e = p_e (g_e - sum over e of g p),  p the softmax, g_e = scale * dweight where e was chosen, else 0
//
// Keys are unsigned integers in the order of the numbers.  Up to 8 of up to 256
// experts: see below.  Otherwise a warp holds a row in registers, consecutive logits
// per lane; each choice is one maximum over the warp, and the lowest lane that has
// it has the lowest index too.  Rows of more than 1024 logits are read again from
// the cache for every choice instead: the next one is the largest (key, lowest
// index) behind the last.
//
// A row is read once (and its gradient written once), but what bounds the kernels is
// comparisons for the choice (their unit is busy for two thirds of the time), and
// backwards the latency of the chosen logits, asked for when their ids have come
// (32768 x 128 fp32, 8 chosen: 10.4 us forwards and 6.2 backwards with the logits in
// the L2 cache, 14.7 and 10.6 from DRAM; floors 2.8 and 5.2.  bf16: 7.7 and 5.8).
#include <cuda_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "layer_launch.h"
#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kWarps = 8;
constexpr unsigned kAll = 0xFFFFFFFFu;
constexpr uint32_t kClosed = 0x007FFFFFu;          // the key of -infinity

struct RouterParams {
  const void* logits;
  int32_t* ids;
  float* weights;            // forward
  const float* dweights;     // backward
  void* dlogits;
  int64_t rows, ld, ldd;
  int32_t experts, k, over;
  int32_t vec, vec_d;        // rows of logits, of dlogits, on vector boundaries
  float scale;
};

// Unsigned keys in the order of the numbers: -0 as 0, every NaN the largest.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);
  return v != v ? 0xFFFFFFFFu : b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ float sum_of(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

template <typename T>
__device__ __forceinline__ float logit_at(const void* p, int64_t i) {
  return sizeof(T) == 2 ? load_bf16(p, i) : static_cast<const float*>(p)[i];
}
template <typename T>
__device__ __forceinline__ void put_logit(void* p, int64_t i, float v) {
  if (sizeof(T) == 2) store_bf16(p, i, v);
  else static_cast<float*>(p)[i] = v;
}

// Logits VPL * lane .. VPL * lane + VPL - 1 of a row, -infinity behind its end.
template <typename T, int VPL>
__device__ __forceinline__ void load_row(const void* base, int64_t at, int experts, int lane, int vec, float (&f)[VPL]) {
  const int c = lane * VPL;
  constexpr int PER = VPL * int(sizeof(T)) >= 16 ? 16 / int(sizeof(T)) : VPL;     // per access
  const char* from = static_cast<const char*>(base) + (at + c) * int64_t(sizeof(T));
#pragma unroll
  for (int i = 0; i < VPL; i += PER) {
    if (vec && c + i + PER <= experts) {
      constexpr int BYTES = PER * int(sizeof(T));
      uint32_t w[4];
      if constexpr (BYTES == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(from + i * sizeof(T));
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
      } else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(from + i * sizeof(T));
        w[0] = v.x, w[1] = v.y;
      } else if constexpr (BYTES == 4) {
        w[0] = *reinterpret_cast<const uint32_t*>(from + i * sizeof(T));
      } else {
        w[0] = *reinterpret_cast<const uint16_t*>(from + i * sizeof(T));
      }
#pragma unroll
      for (int j = 0; j < PER; ++j)
        f[i + j] = sizeof(T) == 4 ? __uint_as_float(w[j % 4]) : j & 1 ? bf16_hi(w[j / 2 % 4]) : bf16_lo(w[j / 2 % 4]);
    } else {
#pragma unroll
      for (int j = 0; j < PER; ++j) f[i + j] = c + i + j < experts ? logit_at<T>(base, at + c + i + j) : -INFINITY;
    }
  }
}

// One row by a warp.
template <typename T, int VPL>
__device__ __forceinline__ void forward_row(const RouterParams& p, int64_t row, int lane) {
  const int64_t at = row * p.ld;
  uint32_t key[VPL > 0 ? VPL : 1];
  float total = 0.0f;
  if constexpr (VPL > 0) {
    float f[VPL];
    load_row<T, VPL>(p.logits, at, p.experts, lane, p.vec, f);
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = key_of(f[i]);
  }
  uint32_t mine = kClosed, first = kClosed, last = 0xFFFFFFFFu;
  int last_at = -1, found = 0;
  for (int j = 0; j < p.k; ++j) {
    uint32_t best = kClosed;
    int best_at = 0;
    if constexpr (VPL > 0) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) best = max(best, key[i]);
    } else {
      for (int c = lane; c < p.experts; c += 32) {
        const uint32_t v = key_of(logit_at<T>(p.logits, at + c));
        if ((v < last || (v == last && c > last_at)) && v > best) best = v, best_at = c;
      }
    }
    const uint32_t m = __reduce_max_sync(kAll, best);
    if (m <= kClosed) break;                     // no open expert is left
    if (j == 0) {
      first = m;
      if (p.over == GOLDY_ROUTER_ALL) {
        const float top = value_of(m);
        if constexpr (VPL > 0) {
#pragma unroll
          for (int i = 0; i < VPL; ++i) total += expf(value_of(key[i]) - top);
        } else {
          for (int c = lane; c < p.experts; c += 32) total += expf(logit_at<T>(p.logits, at + c) - top);
        }
        total = sum_of(total);
      }
    }
    if constexpr (VPL > 0) {
      const int winner = __ffs(int(__ballot_sync(kAll, best == m))) - 1;
      if (lane == winner) {
        bool open = true;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
          if (open && key[i] == m) {
            open = false;
            key[i] = kClosed;
            p.ids[row * p.k + j] = lane * VPL + i;
          }
        }
      }
    } else {
      last = m;
      last_at = int(__reduce_min_sync(kAll, best == m ? unsigned(best_at) : 0xFFFFFFFFu));
      if (lane == 0) p.ids[row * p.k + j] = last_at;
    }
    if (lane == j) mine = m;
    ++found;
  }
  float e = lane < found ? expf(value_of(mine) - value_of(first)) : 0.0f;
  if (p.over == GOLDY_ROUTER_CHOSEN) total = sum_of(e);
  if (lane < p.k) {
    p.weights[row * p.k + lane] = lane < found ? p.scale * (e / total) : 0.0f;
    if (lane >= found) p.ids[row * p.k + lane] = -1;
  }
}

template <typename T, int VPL>
__global__ void __launch_bounds__(kWarps * 32) router_forward_kernel(const RouterParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(gridDim.x) * kWarps;
  for (int64_t row = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); row < p.rows; row += step)
    forward_row<T, VPL>(p, row, threadIdx.x & 31);
}

template <typename T, int VPL>
__global__ void __launch_bounds__(kWarps * 32) router_backward_kernel(const RouterParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t step = int64_t(gridDim.x) * kWarps;
  const bool all = p.over == GOLDY_ROUTER_ALL;
  for (int64_t row = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); row < p.rows; row += step) {
    const int64_t at = row * p.ld, to = row * p.ldd;
    float f[VPL > 0 ? VPL : 1];
    if constexpr (VPL > 0) load_row<T, VPL>(p.logits, at, p.experts, lane, p.vec, f);
    // this lane's slot
    int id = lane < p.k ? p.ids[row * p.k + lane] : -1;
    if (id < 0 || id >= p.experts) id = -1;
    float g = id >= 0 ? p.scale * p.dweights[row * p.k + lane] : 0.0f;
    const float l = id >= 0 ? logit_at<T>(p.logits, at + id) : -INFINITY;
    // an expert that is named again: the lowest slot takes all its gradients
    const unsigned same = __match_any_sync(kAll, id >= 0 ? id : -1 - lane);
    const bool owner = id >= 0 && (same & ((1u << lane) - 1)) == 0;
    if (__any_sync(kAll, id >= 0 && !owner)) {
      float all_g = 0.0f;
      for (int j = 0; j < p.k; ++j) {
        const float gj = __shfl_sync(kAll, g, j);
        if (same >> j & 1) all_g += gj;
      }
      g = all_g;
    }
    // the largest logit, and the sum of the exponentials
    uint32_t best = owner ? key_of(l) : kClosed;
    if (all) {
      if constexpr (VPL > 0) {
#pragma unroll
        for (int i = 0; i < VPL; ++i) best = max(best, key_of(f[i]));
      } else {
        for (int c = lane; c < p.experts; c += 32) best = max(best, key_of(logit_at<T>(p.logits, at + c)));
      }
    }
    const uint32_t first = __reduce_max_sync(kAll, best);
    const float top = first == kClosed ? 0.0f : value_of(first);
    float e = owner ? expf(l - top) : 0.0f, total = 0.0f;
    if (!all) {
      total = e;
    } else if constexpr (VPL > 0) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        f[i] = expf(f[i] - top);
        total += f[i];
      }
    } else {
      for (int c = lane; c < p.experts; c += 32) total += expf(logit_at<T>(p.logits, at + c) - top);
    }
    total = sum_of(total);
    const float inv = first == kClosed ? 0.0f : 1.0f / total;
    const float prob = e * inv;
    const float dot = sum_of(owner ? g * prob : 0.0f);
    if constexpr (VPL > 0) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int c = lane * VPL + i;
        if (c < p.experts) put_logit<T>(p.dlogits, to + c, all ? f[i] * inv * -dot : 0.0f);
      }
    } else {
      for (int c = lane; c < p.experts; c += 32)
        put_logit<T>(p.dlogits, to + c, all ? expf(logit_at<T>(p.logits, at + c) - top) * inv * -dot : 0.0f);
    }
    __syncwarp();                                  // behind the others' zeros
    if (owner) put_logit<T>(p.dlogits, to + id, prob * (g - dot));
  }
}

// ---- up to 8 of up to 256 experts: eight lanes per row ---------------------------
// Four rows per warp share every instruction (a warp per row: 32768 x 128 forwards
// and backwards 32 us, now 17).  A lane sorts its keys eight at a time,
// and lists are merged (the larger of A[i] and B[7 - i] are the eight largest of
// both, in an order that three steps of compare and exchange sort): first those of
// a lane, then those of the eight lanes, after which every lane knows the row's
// eight largest keys.  bf16 logits leave room for the index in the key; of fp32
// logits, a lane that holds one of them finds its slot by its key, and where two of
// these are equal the team looks for the lowest index slot by slot (32768 x 128
// fp32 forwards: 10.4 us, logits that hold bf16 values 14.7).

constexpr int kTeam = 8;
constexpr int kTop = 8;

__device__ __forceinline__ void order(uint32_t& a, uint32_t& b) {
  const uint32_t hi = max(a, b);
  b = min(a, b);
  a = hi;
}
// falling order of eight keys that rise and fall once
__device__ __forceinline__ void sort_bitonic(uint32_t (&k)[kTop]) {
#pragma unroll
  for (int d = 4; d > 0; d /= 2)
#pragma unroll
    for (int i = 0; i < kTop; ++i)
      if ((i & d) == 0) order(k[i], k[i + d]);
}
// falling order of eight keys (Batcher's merge exchange, 19 comparisons)
__device__ __forceinline__ void sort8(uint32_t (&k)[kTop]) {
  order(k[0], k[1]), order(k[2], k[3]), order(k[4], k[5]), order(k[6], k[7]);
  order(k[0], k[2]), order(k[1], k[3]), order(k[4], k[6]), order(k[5], k[7]);
  order(k[1], k[2]), order(k[5], k[6]);
  order(k[0], k[4]), order(k[1], k[5]), order(k[2], k[6]), order(k[3], k[7]);
  order(k[2], k[4]), order(k[3], k[5]);
  order(k[1], k[2]), order(k[3], k[4]), order(k[5], k[6]);
}

// A lane's logits are those of pieces lane, lane + 8, ... of PIECE each.
template <typename T, int VPL>
struct Share {
  static constexpr int PIECE = 16 / int(sizeof(T)) < VPL ? 16 / int(sizeof(T)) : VPL;
  static __device__ __forceinline__ int index(int i, int lane) { return (i / PIECE * kTeam + lane) * PIECE + i % PIECE; }
  static __device__ __forceinline__ void load(const void* base, int64_t at, int experts, int lane, int vec, float (&f)[VPL]) {
#pragma unroll
    for (int i = 0; i < VPL; i += PIECE) {
      const int c = index(i, lane);
      if (vec && c + PIECE <= experts) {
        const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const char*>(base) + (at + c) * int64_t(sizeof(T)));
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < PIECE; ++j)
          f[i + j] = sizeof(T) == 4 ? __uint_as_float(w[j % 4]) : j & 1 ? bf16_hi(w[j / 2 % 4]) : bf16_lo(w[j / 2 % 4]);
      } else {
#pragma unroll
        for (int j = 0; j < PIECE; ++j) f[i + j] = c + j < experts ? logit_at<T>(base, at + c + j) : -INFINITY;
      }
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t at, int experts, int lane, int vec, const float (&f)[VPL]) {
#pragma unroll
    for (int i = 0; i < VPL; i += PIECE) {
      const int c = index(i, lane);
      if (vec && c + PIECE <= experts) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = sizeof(T) == 4 ? __float_as_uint(f[i + j]) : pack_bf16(f[(i + 2 * j) % VPL], f[(i + 2 * j + 1) % VPL]);
        *reinterpret_cast<uint4*>(static_cast<char*>(base) + (at + c) * int64_t(sizeof(T))) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
#pragma unroll
        for (int j = 0; j < PIECE; ++j)
          if (c + j < experts) put_logit<T>(base, at + c + j, f[i + j]);
      }
    }
  }
};

// exp(x) for x <= 0 (NaN stays NaN): exp(x) = 2^y exp(x - y ln 2) for any y, here x
// log2 e as it is rounded, which alone would cost |x| u and more.  What is left, r,
// is below 2^-15, so that 1 + r is its exponential; ln 2 is taken in two parts.
// Where r is no such number, x being infinite or far down, the power is 0.
// (32768 x 128 fp32: 10.4 us and, backwards, 6.2; without r 10.2 and 6.0, with expf 11.1 and 6.5.)
constexpr float kLn2 = 0.693147180559945309f, kLn2Rest = float(0.693147180559945309 - double(kLn2));
__device__ __forceinline__ uint64_t exp_below2(uint64_t x) {
  const uint64_t y = mul2(x, two(kLog2E));
  const float2 p = apart(y), r = apart(fma2(y, two(-kLn2Rest), fma2(y, two(-kLn2), x)));
  const uint64_t e = two(fast_exp2(p.x), fast_exp2(p.y));
  return fma2(e, two(fminf(r.x, 1.0f), fminf(r.y, 1.0f)), e);
}
__device__ __forceinline__ float exp_below(float x) {
  const float y = x * kLog2E, r = fmaf(y, -kLn2Rest, fmaf(y, -kLn2, x)), e = fast_exp2(y);
  return fmaf(e, fminf(r, 1.0f), e);
}
// f = exp(f - top), and their sum
template <int N>
__device__ __forceinline__ float exp_all(float (&f)[N], float top) {
  uint64_t sum = two(0.0f);
#pragma unroll
  for (int i = 0; i < N; i += 2) {
    const uint64_t e = exp_below2(add2(two(f[i], f[i + 1]), two(-top)));
    sum = add2(sum, e);
    const float2 v = apart(e);
    f[i] = v.x;
    f[i + 1] = v.y;
  }
  const float2 v = apart(sum);
  return v.x + v.y;
}
// sum over a team's lanes, to all of them
__device__ __forceinline__ float team_sum(float v) {
#pragma unroll
  for (int d = kTeam / 2; d > 0; d /= 2) v += __shfl_xor_sync(kAll, v, d);
  return v;
}

template <typename T, int VPL>
__global__ void __launch_bounds__(kWarps * 32, VPL > 16 ? 2 : 4) router_forward_small_kernel(const RouterParams p) {
  using S = Share<T, VPL>;
  constexpr bool INDEXED = sizeof(T) == 2;         // the key's lower half holds the index
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x & (kTeam - 1);
  const int64_t step = int64_t(gridDim.x) * (kWarps * 32 / kTeam);
  const int64_t first_row = int64_t(blockIdx.x) * (kWarps * 32 / kTeam) + (threadIdx.x / 32) * (32 / kTeam);
  for (int64_t row4 = first_row; row4 < p.rows; row4 += step) {    // the warp's four rows
    const int64_t row = row4 + (threadIdx.x & 31) / kTeam;
    const bool there = row < p.rows;
    const int64_t at = (there ? row : row4) * p.ld;
    float f[VPL];
    uint32_t key[VPL], best[kTop];
    S::load(p.logits, at, p.experts, lane, p.vec, f);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      key[i] = INDEXED ? (key_of(f[i]) & 0xFFFF0000u) | uint32_t(0xFFFF - S::index(i, lane)) : key_of(f[i]);
#pragma unroll
    for (int i0 = 0; i0 < VPL; i0 += kTop) {
      uint32_t k[kTop];
#pragma unroll
      for (int i = 0; i < kTop; ++i) k[i] = key[i0 + i];
      sort8(k);
      if (i0 == 0) {
#pragma unroll
        for (int i = 0; i < kTop; ++i) best[i] = k[i];
      } else {
#pragma unroll
        for (int i = 0; i < kTop; ++i) best[i] = max(best[i], k[kTop - 1 - i]);
        sort_bitonic(best);
      }
    }
#pragma unroll
    for (int d = 1; d < kTeam; d *= 2) {
      uint32_t k[kTop];
#pragma unroll
      for (int i = 0; i < kTop; ++i) k[i] = __shfl_xor_sync(kAll, best[kTop - 1 - i], d);
#pragma unroll
      for (int i = 0; i < kTop; ++i) best[i] = max(best[i], k[i]);
      sort_bitonic(best);
    }
    // open ones among the first k
    int found = 0;
    uint32_t least = 0xFFFFFFFFu;                  // the smallest chosen key
#pragma unroll
    for (int j = 0; j < kTop; ++j) {
      const bool open = j < p.k && (INDEXED ? best[j] >> 16 > kClosed >> 16 : best[j] > kClosed);
      found += open;
      least = open ? best[j] : least;
    }
    auto value = [](uint32_t k) {
      return INDEXED ? __uint_as_float(__float_as_uint(value_of(k)) & 0xFFFF0000u) : value_of(k);
    };
    const float top = found ? value(best[0]) : 0.0f;
    float total = 0.0f;
    if (p.over == GOLDY_ROUTER_ALL) {
      total = team_sum(exp_all(f, top));
    } else {
#pragma unroll
      for (int j = 0; j < kTop; ++j) total += j < found ? exp_below(value(best[j]) - top) : 0.0f;
    }
    const float share = p.scale / total;
    int32_t* ids = p.ids + row * p.k;
    float* weights = p.weights + row * p.k;
    if constexpr (INDEXED) {
      uint32_t k = best[0];
#pragma unroll
      for (int j = 1; j < kTop; ++j) k = lane == j ? best[j] : k;
      if (there && lane < p.k) {
        ids[lane] = lane < found ? int(0xFFFF - (k & 0xFFFFu)) : -1;
        weights[lane] = lane < found ? exp_below(value(k) - top) * share : 0.0f;
      }
    } else {
      uint32_t mine = 0;                           // this lane's chosen logits
#pragma unroll
      for (int i = 0; i < VPL; ++i) mine |= uint32_t(found > 0 && key[i] >= least) << i;
      int chosen = __popc(mine);
#pragma unroll
      for (int d = 1; d < kTeam; d *= 2) chosen += __shfl_xor_sync(kAll, chosen, d);
      bool twice = chosen != found;
#pragma unroll
      for (int j = 0; j + 1 < kTop; ++j) twice |= j + 1 < found && best[j] == best[j + 1];
      // slots of equal logits, and the last one where more logits than slots have its
      // key: by index, the lowest behind the one before
      uint32_t shared = 0;
      if (__any_sync(kAll, there && twice)) {
        int last = -1;
#pragma unroll
        for (int j = 0; j < kTop; ++j) {
          const bool again = j > 0 && best[j] == best[j > 0 ? j - 1 : 0];
          const bool is = j < found && (again || (j + 1 < found ? best[j] == best[j + 1 < kTop ? j + 1 : j] : chosen > found));
          if (!__any_sync(kAll, is)) continue;
          shared |= uint32_t(is) << j;
          if (!again) last = -1;
          int c = INT_MAX;
#pragma unroll
          for (int i = VPL - 1; i >= 0; --i)
            if (key[i] == best[j] && S::index(i, lane) > last) c = S::index(i, lane);
#pragma unroll
          for (int d = 1; d < kTeam; d *= 2) c = min(c, __shfl_xor_sync(kAll, c, d));
          last = c;
          if (there && is && lane == j) {
            ids[j] = c;
            weights[j] = exp_below(value(best[j]) - top) * share;
          }
        }
      }
      if (!there) mine = 0;
      while (mine) {
        const int c = S::index(__ffs(int(mine)) - 1, lane);
        mine &= mine - 1;
        const float v = logit_at<T>(p.logits, at + c);
        const uint32_t k = key_of(v);
        int slot = 0;
#pragma unroll
        for (int j = 0; j < kTop; ++j) slot += best[j] > k;
        if (shared >> slot & 1) continue;
        ids[slot] = c;
        weights[slot] = exp_below(v - top) * share;
      }
      if (there && lane >= found && lane < p.k) {
        ids[lane] = -1;
        weights[lane] = 0.0f;
      }
    }
  }
}

template <typename T, int VPL>
__global__ void __launch_bounds__(kWarps * 32, VPL > 16 ? 2 : VPL > 8 ? 4 : 6) router_backward_small_kernel(const RouterParams p) {
  using S = Share<T, VPL>;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x & (kTeam - 1);
  const int64_t step = int64_t(gridDim.x) * (kWarps * 32 / kTeam);
  const int64_t first_row = int64_t(blockIdx.x) * (kWarps * 32 / kTeam) + (threadIdx.x / 32) * (32 / kTeam);
  const bool all = p.over == GOLDY_ROUTER_ALL;
  for (int64_t row4 = first_row; row4 < p.rows; row4 += step) {
    const int64_t row = row4 + (threadIdx.x & 31) / kTeam;
    const bool there = row < p.rows;
    const int64_t at = (there ? row : row4) * p.ld;
    // this lane's slot
    int id = there && lane < p.k ? p.ids[row * p.k + lane] : -1;
    if (id < 0 || id >= p.experts) id = -1;
    float f[VPL];
    if (all) S::load(p.logits, at, p.experts, lane, p.vec, f);
    const float dw = id >= 0 ? p.scale * p.dweights[row * p.k + lane] : 0.0f;
    const float l = id >= 0 ? logit_at<T>(p.logits, at + id) : -INFINITY;
    // an expert that is named again: the lowest slot takes all its gradients
    float g = 0.0f, top = -INFINITY;
    bool owner = id >= 0;
#pragma unroll
    for (int j = 0; j < kTop; ++j) {
      const bool same = __shfl_sync(kAll, id, j, kTeam) == id;
      const float gj = __shfl_sync(kAll, dw, j, kTeam);
      if (same) g += gj;
      owner &= !(same && j < lane);
    }
    if (all) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) top = fmaxf(top, f[i]);
    } else {
      top = l;
    }
#pragma unroll
    for (int d = 1; d < kTeam; d *= 2) top = fmaxf(top, __shfl_xor_sync(kAll, top, d));
    const bool none = top == -INFINITY;            // (a NaN among the logits makes the sum NaN)
    if (none) top = 0.0f;
    const float e = owner ? exp_below(l - top) : 0.0f;
    float total = e;
    if (all) total = exp_all(f, top);
    total = team_sum(total);
    const float inv = none && total == 0.0f ? 0.0f : 1.0f / total, prob = e * inv;
    const float dot = team_sum(owner ? g * prob : 0.0f), back = -dot * inv;
    const int64_t to = row * p.ldd;
#pragma unroll
    for (int i = 0; i < VPL; ++i) f[i] = all ? f[i] * back : 0.0f;
    if (there) S::store(p.dlogits, to, p.experts, lane, p.vec_d, f);
    __syncwarp();                                  // behind the others' values
    if (owner) put_logit<T>(p.dlogits, to + id, prob * (g - dot));
  }
}

template <typename T, int VPL>
const void* pick(bool backward) {
  return backward ? reinterpret_cast<const void*>(&router_backward_kernel<T, VPL>)
                  : reinterpret_cast<const void*>(&router_forward_kernel<T, VPL>);
}
template <typename T>
const void* pick_width(int per_lane, bool backward) {
  switch (per_lane) {
    case 1: return pick<T, 1>(backward);
    case 2: return pick<T, 2>(backward);
    case 4: return pick<T, 4>(backward);
    case 8: return pick<T, 8>(backward);
    case 16: return pick<T, 16>(backward);
    case 32: return pick<T, 32>(backward);
    default: return pick<T, 0>(backward);
  }
}

template <typename T, int VPL>
const void* pick_small(bool backward) {
  return backward ? reinterpret_cast<const void*>(&router_backward_small_kernel<T, VPL>)
                  : reinterpret_cast<const void*>(&router_forward_small_kernel<T, VPL>);
}
template <typename T>
const void* pick_small_width(int experts, bool backward) {
  if (experts <= 8 * kTeam) return pick_small<T, 8>(backward);
  return experts <= 16 * kTeam ? pick_small<T, 16>(backward) : pick_small<T, 32>(backward);
}

struct RouterCall {
  RouterParams p;
  const void* fn;
  int64_t per_cta;           // rows
  void* stream;
};

goldy_status launch_router(const LayerContext& ctx, void* arg) {
  RouterCall& call = *static_cast<RouterCall*>(arg);
  const int64_t grid = std::min(ceil_div(call.p.rows, call.per_cta), int64_t(ctx.sm_count) * 8);
  void* args[] = {&call.p};
  return launch_layer("router", call.fn, grid, kWarps * 32, 0, call.stream, args);
}

goldy_status check_router(const goldy_router_desc* d) {
  if (!d) return invalid("null descriptor");
  if (d->rows < 0 || d->rows > (int64_t(1) << 40)) return invalid("router: rows is negative or too large");
  if (d->experts < 1 || d->experts > GOLDY_MAX_GROUPS) return invalid("router: experts out of range");
  if (d->k < 1 || d->k > d->experts || d->k > GOLDY_MAX_SLOTS) return invalid("router: k out of range");
  if (d->ld < d->experts || d->ldd < d->experts) return invalid("router: a row stride is smaller than its row");
  if (too_far(d->rows, d->ld) || too_far(d->rows, d->ldd)) return invalid("router: an array is beyond any memory");
  if (d->dtype != GOLDY_BF16 && d->dtype != GOLDY_F32)
    return fail(GOLDY_ERR_UNSUPPORTED, "router: logits are GOLDY_BF16 or GOLDY_F32");
  if (d->over != GOLDY_ROUTER_ALL && d->over != GOLDY_ROUTER_CHOSEN) return invalid("router: over out of range");
  if (!std::isfinite(d->scale)) return invalid("router: scale must be finite");
  if (d->reserved != 0) return invalid("router: reserved must be 0");
  return GOLDY_OK;
}

goldy_status run_router(const goldy_router_desc& d, RouterCall& call, const void* logits, bool backward, void* stream) {
  const bool f32 = d.dtype == GOLDY_F32, small = d.k <= kTop && d.experts <= 32 * kTeam;
  int per_lane = 1;
  while (per_lane < 64 && per_lane * 32 < d.experts) per_lane *= 2;
  const int64_t es = int64_t(element_size(d.dtype)), access = small ? 16 : std::min<int64_t>(16, per_lane * es);
  if (small) call.fn = f32 ? pick_small_width<float>(d.experts, backward) : pick_small_width<uint16_t>(d.experts, backward);
  else call.fn = f32 ? pick_width<float>(per_lane, backward) : pick_width<uint16_t>(per_lane, backward);
  call.per_cta = small ? kWarps * 32 / kTeam : kWarps;
  call.p.logits = logits;
  call.p.rows = d.rows;
  call.p.ld = d.ld;
  call.p.ldd = d.ldd;
  call.p.experts = d.experts;
  call.p.k = d.k;
  call.p.over = d.over;
  call.p.scale = d.scale;
  call.p.vec = on_boundary(logits, size_t(access)) && d.ld * es % access == 0;
  call.p.vec_d = on_boundary(call.p.dlogits, 16) && d.ldd * es % 16 == 0;
  call.stream = stream;
  const goldy_status st = with_layer_context(stream, launch_router, &call);
  return st == GOLDY_OK ? ok() : st;
}

}  // namespace
}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_router_forward(const goldy_router_desc* desc, const void* logits, int32_t* ids,
                                             float* weights, void* stream) try {
  const goldy_status st = check_router(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0) return ok();
  if (!logits || !ids || !weights) return invalid("router: logits, ids and weights are needed");
  if (!on_boundary(logits, element_size(desc->dtype)) || !on_boundary(ids, 4) || !on_boundary(weights, 4))
    return invalid("router: a pointer is misaligned");
  RouterCall call{};
  call.p.ids = ids;
  call.p.weights = weights;
  return run_router(*desc, call, logits, false, stream);
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_router_backward(const goldy_router_desc* desc, const void* logits, const int32_t* ids,
                                              const float* dweights, void* dlogits, void* stream) try {
  const goldy_status st = check_router(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0) return ok();
  if (!logits || !ids || !dweights || !dlogits) return invalid("router: logits, ids, dweights and dlogits are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(logits, es) || !on_boundary(dlogits, es) || !on_boundary(ids, 4) || !on_boundary(dweights, 4))
    return invalid("router: a pointer is misaligned");
  if (dlogits == logits && desc->ld != desc->ldd) return invalid("router: dlogits are the logits, with another stride");
  RouterCall call{};
  call.p.ids = const_cast<int32_t*>(ids);
  call.p.dweights = dweights;
  call.p.dlogits = dlogits;
  return run_router(*desc, call, logits, true, stream);
} catch (...) {
  return layer_exception();
}
