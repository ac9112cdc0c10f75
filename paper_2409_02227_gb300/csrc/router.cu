// A router: the k largest of each row's logits, their softmax weights, and the
// logits' gradient.
//
//   weight of a chosen expert e = scale exp(l_e - m) / sum exp(l - m),  m the row's largest logit
//   dl_e = p_e (g_e - sum over e of g p),  p the softmax, g_e = scale * dweight where e was chosen, else 0
//
// A warp holds a row in registers, consecutive logits per lane, as unsigned
// keys in the order of the numbers.  Each choice is one maximum over the warp;
// the lowest lane that has it has the lowest index too.  Rows of more than 1024
// logits are read again from the cache for every choice instead: the next one is
// the largest (key, lowest index) behind the last.
#include <cuda_runtime.h>

#include <algorithm>
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
  int32_t experts, k, over, vec;
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

template <typename T, int VPL>
__global__ void __launch_bounds__(kWarps * 32) router_forward_kernel(const RouterParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t step = int64_t(gridDim.x) * kWarps;
  for (int64_t row = int64_t(blockIdx.x) * kWarps + (threadIdx.x >> 5); row < p.rows; row += step) {
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

struct RouterCall {
  RouterParams p;
  const void* fn;
  void* stream;
};

goldy_status launch_router(const LayerContext& ctx, void* arg) {
  RouterCall& call = *static_cast<RouterCall*>(arg);
  const int64_t grid = std::min(ceil_div(call.p.rows, int64_t(kWarps)), int64_t(ctx.sm_count) * 8);
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
  int per_lane = 1;
  while (per_lane < 64 && per_lane * 32 < d.experts) per_lane *= 2;
  call.fn = d.dtype == GOLDY_F32 ? pick_width<float>(per_lane, backward) : pick_width<uint16_t>(per_lane, backward);
  const int64_t access = std::min<int64_t>(16, per_lane * int64_t(element_size(d.dtype)));
  call.p.logits = logits;
  call.p.rows = d.rows;
  call.p.ld = d.ld;
  call.p.ldd = d.ldd;
  call.p.experts = d.experts;
  call.p.k = d.k;
  call.p.over = d.over;
  call.p.scale = d.scale;
  call.p.vec = on_boundary(logits, size_t(access)) && d.ld * int64_t(element_size(d.dtype)) % access == 0;
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
