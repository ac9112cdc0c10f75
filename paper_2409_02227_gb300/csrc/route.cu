// Tokens sorted by expert and back.
//
//   sort       place[slot] = slots of smaller experts + slots of the same expert before it
//   dispatch   E[place[t, j]] = X[t]
//   combine    Y[t] = R[t] + sum_j w[t, j] E[place[t, j]]
//   its gradient  dE[place[t, j]] = w[t, j] dY[t],  dw[t, j] = dY[t] . E[place[t, j]]
//
// The sort is a counting sort over chunks of the slots: a first kernel counts
// each chunk's slots per expert, a second one adds up what lies before its
// chunk and walks the chunk's slots in order, a warp's 32 at a time; lanes with
// the same expert rank themselves by lane.  Slots without an expert are counted
// as one more expert behind the others.  A single chunk needs no first kernel.
// Nothing depends on an order of arrival.
//
// The rest is HBM-bound: a thread moves 16-byte blocks of a token's row, to all
// its places (dispatch: X is read once) or from all of them (combine).  The
// gradient takes a warp per slot, which also sums the dot product.
#include <cuda_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <mutex>
#include <set>
#include <utility>

#include "layer_launch.h"
#include "row_blocks.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr unsigned kAll = 0xFFFFFFFFu;

// ---- sort ---------------------------------------------------------------------

constexpr int kSortThreads = 512;
constexpr int kAlone = 4096;           // slots up to which one CTA sorts them
constexpr int kChunk = 2048;           // slots per CTA otherwise
constexpr int kMostChunks = 304;       // at most, then chunks grow
constexpr int kSortSmem = 200 * 1024;  // for the warps' counts

struct SortParams {
  const int32_t* ids;
  int32_t* offsets;
  int32_t* place;
  int32_t* source;       // may be null
  int32_t* counts;       // [chunks][groups + 1]; null: one chunk
  int32_t slots, groups, chunk, chunks;
  int32_t warps;         // that walk a chunk
};

__device__ __forceinline__ int group_of(const SortParams& p, int slot) {
  const int id = p.ids[slot];
  return id >= 0 && id < p.groups ? id : p.groups;
}

__global__ void __launch_bounds__(kSortThreads) route_count_kernel(const SortParams p) {
  extern __shared__ int32_t count[];
  ptx::griddep_launch_dependents();
  for (int g = threadIdx.x; g <= p.groups; g += kSortThreads) count[g] = 0;
  ptx::griddep_wait();
  __syncthreads();
  const int64_t lo = int64_t(blockIdx.x) * p.chunk, hi = min(int64_t(p.slots), lo + p.chunk);
  for (int64_t s = lo + threadIdx.x; s < hi; s += kSortThreads) atomicAdd(count + group_of(p, int(s)), 1);
  __syncthreads();
  int32_t* to = p.counts + int64_t(blockIdx.x) * (p.groups + 1);
  for (int g = threadIdx.x; g <= p.groups; g += kSortThreads) to[g] = count[g];
}

__global__ void __launch_bounds__(kSortThreads) route_place_kernel(const SortParams p) {
  extern __shared__ int32_t smem[];
  __shared__ int32_t warp_total[kSortThreads / 32];
  const int bins = p.groups + 1, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  int32_t* start = smem;                 // [bins + 1]: slots of smaller groups
  int32_t* next = smem + bins + 1;       // [warps][bins]: counts, then the next place
  ptx::griddep_launch_dependents();
  for (int i = threadIdx.x; i < p.warps * bins; i += kSortThreads) next[i] = 0;
  ptx::griddep_wait();
  __syncthreads();
  const int64_t lo = int64_t(blockIdx.x) * p.chunk, hi = min(int64_t(p.slots), lo + p.chunk);
  const int64_t share = (p.chunk / 32 + p.warps - 1) / p.warps * 32;       // slots per warp
  const int64_t from = min(hi, lo + warp * share), to = warp < p.warps ? min(hi, from + share) : from;
  for (int64_t s = from + lane; s < to; s += 32) atomicAdd(next + warp * bins + group_of(p, int(s)), 1);
  __syncthreads();
  // all slots of a group, and those of the chunks before
  for (int g = threadIdx.x; g < bins; g += kSortThreads) {
    int total = 0, before = 0;
    if (p.counts) {
      for (int c = 0; c < p.chunks; ++c) {
        const int n = p.counts[int64_t(c) * bins + g];
        if (c < int(blockIdx.x)) before += n;
        total += n;
      }
    } else {
      for (int w = 0; w < p.warps; ++w) total += next[w * bins + g];
    }
    start[g] = total;
    int at = before;
    for (int w = 0; w < p.warps; ++w) {
      const int n = next[w * bins + g];
      next[w * bins + g] = at;
      at += n;
    }
  }
  __syncthreads();
  // exclusive sums over the groups: consecutive ones per thread
  const int per = (bins + kSortThreads - 1) / kSortThreads, g0 = min(bins, int(threadIdx.x) * per), g1 = min(bins, g0 + per);
  int sum = 0;
  for (int g = g0; g < g1; ++g) sum += start[g];
  int up = sum;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int v = __shfl_up_sync(kAll, up, d);
    if (lane >= d) up += v;
  }
  if (lane == 31) warp_total[warp] = up;
  __syncthreads();
  int at = up - sum;
  for (int w = 0; w < warp; ++w) at += warp_total[w];
  for (int g = g0; g < g1; ++g) {
    const int n = start[g];
    start[g] = at;
    at += n;
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int g = threadIdx.x; g < bins; g += kSortThreads) p.offsets[g] = start[g];
  if (warp >= p.warps) return;
  int32_t* mine = next + warp * bins;
  for (int64_t s0 = from; s0 < to; s0 += 32) {
    const int64_t s = s0 + lane;
    const int g = s < to ? group_of(p, int(s)) : -1;
    const unsigned same = __match_any_sync(kAll, g);
    const int rank = __popc(same & ((1u << lane) - 1));
    const int base = g >= 0 ? mine[g] : 0;
    __syncwarp();
    if (g >= 0 && rank == 0) mine[g] = base + __popc(same);
    __syncwarp();
    if (g < 0) continue;
    const int at = start[g] + base + rank;
    const bool lost = g == p.groups;
    p.place[s] = lost ? -1 : at;
    if (p.source) p.source[at] = lost ? -1 : int(s);
  }
}

// ---- rows ---------------------------------------------------------------------

constexpr int kRowThreads = 256;
constexpr int kInFlight = 8;           // experts' rows that combine reads at once

struct RowParams {
  const void* tokens;    // X, or dY
  const void* experts;   // E
  const void* res;       // R
  void* out;             // E (dispatch), Y, or dE
  const int32_t* place;
  const float* weights;
  float* dweights;
  int64_t rows, ldx, lde, ldr;
  int32_t width, k, places;
  int32_t lanes_log;     // threads per row, log2
};

__device__ __forceinline__ int place_of(const RowParams& p, int64_t slot) {
  const int at = p.place[slot];
  return at >= 0 && at < p.places ? at : -1;
}

// Calls body(token, block) for this thread's blocks of its rows.
template <typename T, bool ALIGNED, typename F>
__device__ __forceinline__ void for_blocks(const RowParams& p, F body) {
  const int lanes = 1 << p.lanes_log, x = threadIdx.x & (lanes - 1);
  const int64_t per_cta = kRowThreads >> p.lanes_log;
  // a row that starts inside a block touches one more
  const int blocks = p.width / Block<T>::PER + (ALIGNED ? 0 : 2);
  for (int64_t t = int64_t(blockIdx.x) * per_cta + (threadIdx.x >> p.lanes_log); t < p.rows; t += int64_t(gridDim.x) * per_cta)
    for (int b = x; b < blocks; b += lanes) body(t, b);
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads) route_dispatch_kernel(const RowParams p) {
  using B = Block<T>;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for_blocks<T, ALIGNED>(p, [&](int64_t t, int b) {
    const T* x = static_cast<const T*>(p.tokens) + t * p.ldx;
    uint4 v;
    if (ALIGNED) v = B::template load<true>(x, b * B::PER, p.width);
    for (int j = 0; j < p.k; ++j) {
      const int at = place_of(p, t * p.k + j);
      if (at < 0) continue;
      T* e = static_cast<T*>(p.out) + int64_t(at) * p.lde;
      const int c = b * B::PER - (ALIGNED ? 0 : B::off(e));
      if (!ALIGNED) {
        if (c >= p.width) continue;
        v = B::template load<false>(x, c, p.width);
      }
      B::template store<ALIGNED>(e, c, p.width, v);
    }
  });
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads) route_combine_kernel(const RowParams p) {
  using B = Block<T>;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for_blocks<T, ALIGNED>(p, [&](int64_t t, int b) {
    T* y = static_cast<T*>(p.out) + t * p.ldx;
    const int c = b * B::PER - (ALIGNED ? 0 : B::off(y));
    if (!ALIGNED && c >= p.width) return;
    float sum[B::PER], f[B::PER];
#pragma unroll
    for (int i = 0; i < B::PER; ++i) sum[i] = 0.0f;
    for (int j0 = 0; j0 < p.k; j0 += kInFlight) {
      uint4 v[kInFlight];
      int at[kInFlight];
      float w[kInFlight];
#pragma unroll
      for (int j = 0; j < kInFlight; ++j) {
        const bool there = j0 + j < p.k;
        at[j] = there ? place_of(p, t * p.k + j0 + j) : -1;
        w[j] = there && p.weights ? p.weights[t * p.k + j0 + j] : 1.0f;
      }
#pragma unroll
      for (int j = 0; j < kInFlight; ++j)
        if (at[j] >= 0)
          v[j] = B::template load<ALIGNED>(static_cast<const T*>(p.experts) + int64_t(at[j]) * p.lde, c, p.width);
#pragma unroll
      for (int j = 0; j < kInFlight; ++j) {
        if (at[j] < 0) continue;
        B::unpack(v[j], f);
#pragma unroll
        for (int i = 0; i < B::PER; ++i) sum[i] = fmaf(w[j], f[i], sum[i]);
      }
    }
    if (p.res) {
      B::unpack(B::template load<ALIGNED>(static_cast<const T*>(p.res) + t * p.ldr, c, p.width), f);
#pragma unroll
      for (int i = 0; i < B::PER; ++i) sum[i] += f[i];
    }
    B::template store<ALIGNED>(y, c, p.width, B::pack(sum));
  });
}

template <typename T, bool ALIGNED, bool DOT>
__global__ void __launch_bounds__(kRowThreads) route_combine_grad_kernel(const RowParams p) {
  using B = Block<T>;
  constexpr int UNROLL = 4;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x & 31;
  const int64_t slots = p.rows * p.k, step = int64_t(gridDim.x) * (kRowThreads / 32);
  for (int64_t s = int64_t(blockIdx.x) * (kRowThreads / 32) + (threadIdx.x >> 5); s < slots; s += step) {
    const int at = place_of(p, s);
    if (at < 0) {
      if (DOT && lane == 0) p.dweights[s] = 0.0f;
      continue;
    }
    const T* dy = static_cast<const T*>(p.tokens) + s / p.k * p.ldx;
    const T* e = static_cast<const T*>(p.experts) + int64_t(at) * p.lde;
    T* de = static_cast<T*>(p.out) + int64_t(at) * p.lde;
    const float w = p.weights ? p.weights[s] : 1.0f;
    const int off = ALIGNED ? 0 : B::off(de);
    float dot = 0.0f;
    for (int c0 = lane * B::PER - off; c0 < p.width; c0 += UNROLL * 32 * B::PER) {
      uint4 g[UNROLL], v[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int c = c0 + u * 32 * B::PER;
        if (c >= p.width) continue;
        g[u] = B::template load<ALIGNED>(dy, c, p.width);
        if (DOT) v[u] = B::template load<ALIGNED>(e, c, p.width);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int c = c0 + u * 32 * B::PER;
        if (c >= p.width) continue;
        float f[B::PER], h[B::PER];
        B::unpack(g[u], f);
        if (DOT) B::unpack(v[u], h);
#pragma unroll
        for (int i = 0; i < B::PER; ++i) {
          if (DOT) dot = fmaf(f[i], h[i], dot);
          f[i] *= w;
        }
        B::template store<ALIGNED>(de, c, p.width, B::pack(f));
      }
    }
    if (DOT) {
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) dot += __shfl_xor_sync(kAll, dot, d);
      if (lane == 0) p.dweights[s] = dot;
    }
  }
}

// ---- host ---------------------------------------------------------------------

int64_t slots_of(const goldy_route_desc& d) { return d.rows * d.k; }
int64_t chunks_of(int64_t slots) {
  return slots <= kAlone ? 1 : std::min<int64_t>(kMostChunks, ceil_div(slots, int64_t(kChunk)));
}
size_t sort_bytes(const goldy_route_desc& d) {
  const int64_t chunks = chunks_of(slots_of(d));
  return chunks == 1 ? 0 : kLayerCounterBytes + size_t(chunks) * size_t(d.groups + 1) * sizeof(int32_t);
}

goldy_status check_route(const goldy_route_desc* d) {
  if (!d) return invalid("null descriptor");
  if (d->k < 1 || d->k > GOLDY_MAX_SLOTS) return invalid("route: k out of range");
  if (d->groups < 1 || d->groups > GOLDY_MAX_GROUPS) return invalid("route: groups out of range");
  if (d->rows < 0 || d->rows >= (int64_t(1) << 31) / d->k) return invalid("route: rows is negative or too large");
  if (d->width < 0 || d->width > (int64_t(1) << 30)) return invalid("route: width is negative or too large");
  if (d->ldx < d->width || d->lde < d->width || d->ldr < d->width)
    return invalid("route: a row stride is smaller than its row");
  if (too_far(d->rows, d->ldx) || too_far(slots_of(*d), d->lde) || too_far(d->rows, d->ldr))
    return invalid("route: an array is beyond any memory");
  if (d->dtype != GOLDY_BF16 && d->dtype != GOLDY_F32)
    return fail(GOLDY_ERR_UNSUPPORTED, "route: types are GOLDY_BF16 or GOLDY_F32");
  if (d->reserved != 0) return invalid("route: reserved must be 0");
  return GOLDY_OK;
}

struct SortCall {
  SortParams p;
  void* stream;
};

goldy_status launch_sort(const LayerContext& ctx, void* arg) {
  SortCall& call = *static_cast<SortCall*>(arg);
  SortParams& p = call.p;
  const int64_t bins = p.groups + 1;
  void* args[] = {&p};
  if (p.counts) {
    const goldy_status st = launch_layer("route sort", reinterpret_cast<const void*>(&route_count_kernel), p.chunks,
                                         kSortThreads, size_t(bins) * sizeof(int32_t), call.stream, args);
    if (st != GOLDY_OK) return st;
  }
  const void* fn = reinterpret_cast<const void*>(&route_place_kernel);
  const size_t smem = size_t(bins + 1 + p.warps * bins) * sizeof(int32_t);
  if (smem > 40 * 1024) {              // opted into once per device, with the largest size
    static std::mutex mu;
    static std::set<int> done;
    std::lock_guard<std::mutex> lock(mu);
    if (!done.count(ctx.device)) {
      const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 kSortSmem + (GOLDY_MAX_GROUPS + 2) * int(sizeof(int32_t)));
      if (e != cudaSuccess) return fail(GOLDY_ERR_CUDA, std::string("cudaFuncSetAttribute: ") + cudaGetErrorString(e));
      done.insert(ctx.device);
    }
  }
  return launch_layer("route sort", fn, p.chunks, kSortThreads, smem, call.stream, args);
}

struct RowCall {
  RowParams p;
  const void* fn;
  bool warp_per_slot;
  void* stream;
};

goldy_status launch_rows(const LayerContext& ctx, void* arg) {
  RowCall& call = *static_cast<RowCall*>(arg);
  const int64_t per_cta = call.warp_per_slot ? kRowThreads / 32 : kRowThreads >> call.p.lanes_log;
  const int64_t units = call.warp_per_slot ? call.p.rows * call.p.k : call.p.rows;
  const int64_t grid = std::min(ceil_div(units, per_cta), int64_t(ctx.sm_count) * 64);
  void* args[] = {&call.p};
  return launch_layer("route", call.fn, grid, kRowThreads, 0, call.stream, args);
}

goldy_status run_rows(const goldy_route_desc& d, RowCall& call, void* stream) {
  RowParams& p = call.p;
  p.rows = d.rows;
  p.ldx = d.ldx;
  p.lde = d.lde;
  p.ldr = d.ldr;
  p.width = int32_t(d.width);
  p.k = d.k;
  p.places = int32_t(slots_of(d));
  const int64_t blocks = d.width / (16 / int64_t(element_size(d.dtype))) + 2;
  while ((1 << p.lanes_log) < kRowThreads && (int64_t(1) << p.lanes_log) + 2 < blocks) ++p.lanes_log;
  call.stream = stream;
  const goldy_status st = with_layer_context(stream, launch_rows, &call);
  return st == GOLDY_OK ? ok() : st;
}

// every row whole blocks on their boundaries
bool in_blocks(const goldy_route_desc& d, std::initializer_list<std::pair<const void*, int64_t>> arrays) {
  const int64_t per = 16 / int64_t(element_size(d.dtype));
  if (d.width % per != 0) return false;
  for (const auto& a : arrays)
    if (a.first && (!on_boundary(a.first, 16) || a.second % per != 0)) return false;
  return true;
}

template <typename T>
const void* dispatch_fn(bool aligned) {
  return aligned ? reinterpret_cast<const void*>(&route_dispatch_kernel<T, true>)
                 : reinterpret_cast<const void*>(&route_dispatch_kernel<T, false>);
}
template <typename T>
const void* combine_fn(bool aligned) {
  return aligned ? reinterpret_cast<const void*>(&route_combine_kernel<T, true>)
                 : reinterpret_cast<const void*>(&route_combine_kernel<T, false>);
}
template <typename T>
const void* grad_fn(bool aligned, bool dot) {
  if (dot)
    return aligned ? reinterpret_cast<const void*>(&route_combine_grad_kernel<T, true, true>)
                   : reinterpret_cast<const void*>(&route_combine_grad_kernel<T, false, true>);
  return aligned ? reinterpret_cast<const void*>(&route_combine_grad_kernel<T, true, false>)
                 : reinterpret_cast<const void*>(&route_combine_grad_kernel<T, false, false>);
}

}  // namespace
}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_route_query(const goldy_route_desc* desc, size_t* workspace_bytes) try {
  const goldy_status st = check_route(desc);
  if (st != GOLDY_OK) return st;
  if (!workspace_bytes) return invalid("null argument");
  *workspace_bytes = sort_bytes(*desc);
  return ok();
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_route_sort(const goldy_route_desc* desc, const int32_t* ids, int32_t* offsets,
                                         int32_t* place, int32_t* source, void* workspace, size_t workspace_bytes,
                                         void* stream) try {
  goldy_status st = check_route(desc);
  if (st != GOLDY_OK) return st;
  if (!offsets || !on_boundary(offsets, 4)) return invalid("route: offsets null or misaligned");
  if (desc->rows > 0 && (!ids || !place)) return invalid("route: ids and place are needed");
  if (!on_boundary(ids, 4) || !on_boundary(place, 4) || !on_boundary(source, 4))
    return invalid("route: a pointer is misaligned");
  const size_t need = sort_bytes(*desc);
  if (need > 0) {
    st = check_workspace("route", workspace, workspace_bytes, need);
    if (st != GOLDY_OK) return st;
  }
  SortCall call{};
  SortParams& p = call.p;
  p.ids = ids;
  p.offsets = offsets;
  p.place = place;
  p.source = source;
  p.counts = need > 0 ? reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + kLayerCounterBytes) : nullptr;
  p.slots = int32_t(slots_of(*desc));
  p.groups = desc->groups;
  p.chunks = int32_t(chunks_of(p.slots));
  p.chunk = int32_t(ceil_div(std::max<int64_t>(1, ceil_div(p.slots, int64_t(p.chunks))), 32) * 32);
  p.warps = int32_t(std::min<int64_t>(kSortThreads / 32, kSortSmem / ((p.groups + 1) * int64_t(sizeof(int32_t)))));
  call.stream = stream;
  st = with_layer_context(stream, launch_sort, &call);
  return st == GOLDY_OK ? ok() : st;
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_route_dispatch(const goldy_route_desc* desc, const void* X, const int32_t* place, void* E,
                                             void* stream) try {
  const goldy_status st = check_route(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->width == 0) return ok();
  if (!X || !place || !E) return invalid("route: X, place and E are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(X, es) || !on_boundary(E, es) || !on_boundary(place, 4)) return invalid("route: a pointer is misaligned");
  RowCall call{};
  call.p.tokens = X;
  call.p.place = place;
  call.p.out = E;
  const bool aligned = in_blocks(*desc, {{X, desc->ldx}, {E, desc->lde}});
  call.fn = desc->dtype == GOLDY_F32 ? dispatch_fn<float>(aligned) : dispatch_fn<uint16_t>(aligned);
  return run_rows(*desc, call, stream);
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_route_combine(const goldy_route_desc* desc, const void* E, const int32_t* place,
                                            const float* weights, const void* R, void* Y, void* stream) try {
  const goldy_status st = check_route(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->width == 0) return ok();
  if (!E || !place || !Y) return invalid("route: E, place and Y are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(E, es) || !on_boundary(R, es) || !on_boundary(Y, es) || !on_boundary(place, 4) || !on_boundary(weights, 4))
    return invalid("route: a pointer is misaligned");
  if (R == Y && desc->ldr != desc->ldx) return invalid("route: R is Y, with another stride");
  RowCall call{};
  call.p.experts = E;
  call.p.place = place;
  call.p.weights = weights;
  call.p.res = R;
  call.p.out = Y;
  const bool aligned = in_blocks(*desc, {{E, desc->lde}, {R, desc->ldr}, {Y, desc->ldx}});
  call.fn = desc->dtype == GOLDY_F32 ? combine_fn<float>(aligned) : combine_fn<uint16_t>(aligned);
  return run_rows(*desc, call, stream);
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_route_combine_grad(const goldy_route_desc* desc, const void* dY, const void* E,
                                                 const int32_t* place, const float* weights, void* dE, float* dweights,
                                                 void* stream) try {
  const goldy_status st = check_route(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || (desc->width == 0 && !dweights)) return ok();
  if (!place || (desc->width > 0 && (!dY || !dE || (dweights && !E))))
    return invalid("route: dY, place, dE and, for dweights, E are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(dY, es) || !on_boundary(E, es) || !on_boundary(dE, es) || !on_boundary(place, 4) ||
      !on_boundary(weights, 4) || !on_boundary(dweights, 4))
    return invalid("route: a pointer is misaligned");
  RowCall call{};
  call.p.tokens = dY;
  call.p.experts = E;
  call.p.place = place;
  call.p.weights = weights;
  call.p.out = dE;
  call.p.dweights = dweights;
  call.warp_per_slot = true;
  const bool aligned = in_blocks(*desc, {{dY, desc->ldx}, {dweights ? E : nullptr, desc->lde}, {dE, desc->lde}});
  const bool dot = dweights != nullptr;
  call.fn = desc->dtype == GOLDY_F32 ? grad_fn<float>(aligned, dot) : grad_fn<uint16_t>(aligned, dot);
  return run_rows(*desc, call, stream);
} catch (...) {
  return layer_exception();
}
