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
// gradient takes 8 to 32 lanes per slot, which also sum the dot product.  bf16: 16384
// x 4096 to two places 57 us (7.0 TB/s, with the sort before it 66), 8192 x 8 x 2048
// back with weights and residual 54 (6.2 TB/s), its gradient 88 (6.5 TB/s).  Rows that
// start on any element take two blocks of the source per block of the result, 4 to 6
// more instructions per element pair, and partly written blocks (8192 x 8 x 1111: 46,
// 47 and 74 us, floors 27, 24 and 46).  The gradient's lanes also take a row in whole
// steps of 64 blocks and the slots in whole rounds (5000 x 3 x 1111: 21 us, floor
// 11.5; 72% of the lanes and 77% of the rounds are filled).  The placing kernel's
// every CTA adds up all chunks' counts, so that many slots over many experts cost by
// chunks x chunks x experts (262144 slots over 64 experts 18 us, 256 41, 4096 599).
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
constexpr int kAlone = 2048;           // slots up to which one CTA sorts them
constexpr int kChunk = 1024;           // slots per CTA otherwise
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
  int32_t share_log;     // lanes per group that add up the chunks, log2
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
  // all slots of a group, and those of the chunks before: `share_log` lanes per
  // group add up the chunks, four loads of each on their way at once
  if (p.counts) {
    const int lanes = 1 << p.share_log, x = threadIdx.x & (lanes - 1);
    for (int g = threadIdx.x >> p.share_log; (g & ~31) < bins; g += kSortThreads >> p.share_log) {     // whole warps
      int total = 0, before = 0;
      for (int c0 = x; c0 < p.chunks; c0 += 4 * lanes) {
        int n[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int c = c0 + i * lanes;
          n[i] = c < p.chunks && g < bins ? p.counts[int64_t(c) * bins + g] : 0;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (c0 + i * lanes < int(blockIdx.x)) before += n[i];
          total += n[i];
        }
      }
      for (int d = 1; d < lanes; d *= 2) {
        total += __shfl_xor_sync(kAll, total, d);
        before += __shfl_xor_sync(kAll, before, d);
      }
      if (g < bins && x == 0) {
        start[g] = total;
        int at = before;
        for (int w = 0; w < p.warps; ++w) {
          const int n = next[w * bins + g];
          next[w * bins + g] = at;
          at += n;
        }
      }
    }
  } else {
    for (int g = threadIdx.x; g < bins; g += kSortThreads) {
      int at = 0;
      for (int w = 0; w < p.warps; ++w) {
        const int n = next[w * bins + g];
        next[w * bins + g] = at;
        at += n;
      }
      start[g] = at;
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

constexpr int kRowThreads = 256;       // at most
constexpr int kDispatchBlocks = 2;     // of a row, on their way per thread
constexpr int kDispatchCtas = 5;       // per SM, by registers
constexpr int combine_ctas(int slots) { return slots > 2 ? 4 : 5; }
constexpr int kGradBlocks = 2;         // of dY, and as many of E (4, with 2 CTAs per SM: 74 us for 30000 x 150 to
                                       // four places, now 36)
constexpr int kGradCtas = 4;

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
  int32_t lanes, per_cta;  // threads per row, rows per CTA
};

__device__ __forceinline__ int valid_place(const RowParams& p, int at) { return unsigned(at) < unsigned(p.places) ? at : -1; }

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kRowThreads, kDispatchCtas) route_dispatch_kernel(const RowParams p) {
  using B = Block<T>;
  constexpr int BLOCKS = kDispatchBlocks;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int line = threadIdx.x / p.lanes, x = threadIdx.x % p.lanes, lanes = p.lanes;
  for (int64_t t = int64_t(blockIdx.x) * p.per_cta + line; t < p.rows; t += int64_t(gridDim.x) * p.per_cta) {
    const T* const from = static_cast<const T*>(p.tokens) + t * p.ldx;
    const int32_t* const place = p.place + t * p.k;
    if constexpr (ALIGNED) {
      const int blocks = p.width / B::PER;
      for (int b0 = x; b0 < blocks; b0 += lanes * BLOCKS) {
        uint4 v[BLOCKS];
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u)
          if (u == 0 || b0 + u * lanes < blocks) v[u] = reinterpret_cast<const uint4*>(from)[b0 + u * lanes];
        for (int j = 0; j < p.k; ++j) {
          const int at = valid_place(p, place[j]);
          if (at < 0) continue;
          uint4* e = reinterpret_cast<uint4*>(static_cast<T*>(p.out) + int64_t(at) * p.lde);
#pragma unroll
          for (int u = 0; u < BLOCKS; ++u)
            if (u == 0 || b0 + u * lanes < blocks) e[b0 + u * lanes] = v[u];
        }
      }
    } else {
      // places start on any element: a block of any of them lies in three of X
      const typename B::Source source(from, p.width, 0);
      const int blocks = B::count(from, p.width) + 1;
      for (int b = x; b < blocks; b += lanes) {
        uint4 v[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] = source.first[min(max(b + i - 1, 0), source.last)];
        for (int j = 0; j < p.k; ++j) {
          const int at = valid_place(p, place[j]);
          if (at < 0) continue;
          T* e = static_cast<T*>(p.out) + int64_t(at) * p.lde;
          const typename B::Source s(from, p.width, B::off(e));
          const int c = b * B::PER - B::off(e);
          if (c >= p.width) continue;
          B::template store<false>(e, c, p.width, shift_blocks(s.ahead ? v[0] : v[1], s.ahead ? v[1] : v[2], s.shift));
        }
      }
    }
  }
}

// SLOTS * BLOCKS blocks of experts' rows on their way at once.  (Copies of the next
// tokens' rows into shared memory or the L2 cache meanwhile took 112 and 99 us for
// 8192 tokens of 8 x 2048, this 52; 8 slots of one block 61.  Rows of 1111 elements,
// which start anywhere: 46 us, twice the floor, by instructions.)
template <typename T, bool ALIGNED, int SLOTS, int BLOCKS>
__global__ void __launch_bounds__(kRowThreads, combine_ctas(SLOTS)) route_combine_kernel(const RowParams p) {
  using B = Block<T>;
  constexpr int PAIRS = B::PER / 2;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int line = threadIdx.x / p.lanes, x = threadIdx.x % p.lanes, lanes = p.lanes;
  for (int64_t t = int64_t(blockIdx.x) * p.per_cta + line; t < p.rows; t += int64_t(gridDim.x) * p.per_cta) {
    T* const y = static_cast<T*>(p.out) + t * p.ldx;
    const int32_t* const place = p.place + t * p.k;
    const float* const weights = p.weights ? p.weights + t * p.k : nullptr;
    const int off = ALIGNED ? 0 : B::off(y), blocks = ALIGNED ? p.width / B::PER : B::count(y, p.width);
    auto source = [&](const T* row) {
      if constexpr (!ALIGNED) return typename B::Source(row, p.width, off);
      typename B::Source s;
      s.first = reinterpret_cast<const uint4*>(row);
      return s;
    };
    auto expert = [&](int at) { return source(static_cast<const T*>(p.experts) + int64_t(at) * p.lde); };
    for (int b0 = x; b0 < blocks; b0 += lanes * BLOCKS) {
      uint64_t sum[BLOCKS][PAIRS];
#pragma unroll
      for (int u = 0; u < BLOCKS; ++u)
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sum[u][i] = two(0.0f);
      auto inside = [&](int u) { return u == 0 || b0 + u * lanes < blocks; };
      auto add = [&](int u, const uint4& v, float w) {
        uint64_t f[PAIRS];
        B::pairs(v, f);
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) sum[u][i] = fma2(two(w), f[i], sum[u][i]);
      };
      for (int j0 = 0; j0 < p.k; j0 += SLOTS) {
        typename B::template Raw<ALIGNED> v[SLOTS][BLOCKS];
        int at[SLOTS];
        uint32_t shift[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) at[j] = j0 + j < p.k ? valid_place(p, place[j0 + j]) : -1;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
          if (at[j] < 0) continue;
          const typename B::Source s = expert(at[j]);
          shift[j] = s.shift;
#pragma unroll
          for (int u = 0; u < BLOCKS; ++u)
            if (inside(u)) v[j][u].load(s, b0 + u * lanes);
        }
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
          if (at[j] < 0) continue;
          const float w = weights ? weights[j0 + j] : 1.0f;
#pragma unroll
          for (int u = 0; u < BLOCKS; ++u) add(u, v[j][u].get(shift[j]), w);
        }
      }
      if (p.res) {
        const typename B::Source s = source(static_cast<const T*>(p.res) + t * p.ldr);
        typename B::template Raw<ALIGNED> v[BLOCKS];
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u)
          if (inside(u)) v[u].load(s, b0 + u * lanes);
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u) add(u, v[u].get(s.shift), 1.0f);
      }
#pragma unroll
      for (int u = 0; u < BLOCKS; ++u)
        if (inside(u)) B::template store<ALIGNED>(y, (b0 + u * lanes) * B::PER - off, p.width, B::pack(sum[u]));
    }
  }
}

// LANES threads per slot.
template <typename T, bool ALIGNED, bool DOT, int LANES>
__global__ void __launch_bounds__(kRowThreads, kGradCtas) route_combine_grad_kernel(const RowParams p) {
  using B = Block<T>;
  constexpr int BLOCKS = kGradBlocks, PAIRS = B::PER / 2, TEAMS = kRowThreads / LANES;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % LANES, slots = p.places;
  const int64_t step = int64_t(gridDim.x) * TEAMS;
  int64_t s = int64_t(blockIdx.x) * TEAMS + threadIdx.x / LANES;
  auto slot = [&](int64_t i, int& at, float& w) {
    at = i < slots ? valid_place(p, p.place[i]) : -1;
    w = i < slots && p.weights ? p.weights[i] : 1.0f;
  };
  int at, next_at;
  float w, next_w;
  slot(s, at, w);
  for (; __any_sync(kAll, s < slots); s += step, at = next_at, w = next_w) {       // whole warps: they add up together
    slot(s + step, next_at, next_w);
    uint64_t dot2 = two(0.0f);
    if (at >= 0) {
      const T* dy_row = static_cast<const T*>(p.tokens) + int64_t(uint32_t(s) / uint32_t(p.k)) * p.ldx;
      const T* e_row = static_cast<const T*>(p.experts) + int64_t(at) * p.lde;
      T* const de = static_cast<T*>(p.out) + int64_t(at) * p.lde;
      const int off = ALIGNED ? 0 : B::off(de), blocks = ALIGNED ? p.width / B::PER : B::count(de, p.width);
      typename B::Source dy, e;
      if constexpr (ALIGNED) {
        dy.first = reinterpret_cast<const uint4*>(dy_row);
        e.first = reinterpret_cast<const uint4*>(e_row);
      } else {
        dy = typename B::Source(dy_row, p.width, off);
        if (DOT) e = typename B::Source(e_row, p.width, off);
      }
      for (int b0 = lane; b0 < blocks; b0 += BLOCKS * LANES) {
        typename B::template Raw<ALIGNED> g[BLOCKS], v[BLOCKS];
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u) {
          const int b = b0 + u * LANES;
          if (u > 0 && b >= blocks) continue;
          g[u].load(dy, b);
          if (DOT) v[u].load(e, b);
        }
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u) {
          const int b = b0 + u * LANES, c = b * B::PER - off;
          if (u > 0 && b >= blocks) continue;
          uint64_t f[PAIRS], h[PAIRS];
          uint4 gv = g[u].get(dy.shift);
          if (DOT) {
            uint4 ev = v[u].get(e.shift);
            if (!ALIGNED && (c < 0 || c + B::PER > p.width)) {
              const uint4 m = B::inside(c, p.width);
              gv.x &= m.x, gv.y &= m.y, gv.z &= m.z, gv.w &= m.w;
              ev.x &= m.x, ev.y &= m.y, ev.z &= m.z, ev.w &= m.w;
            }
            B::pairs(ev, h);
          }
          B::pairs(gv, f);
#pragma unroll
          for (int i = 0; i < PAIRS; ++i) {
            if (DOT) dot2 = fma2(f[i], h[i], dot2);
            f[i] = mul2(f[i], two(w));
          }
          B::template store<ALIGNED>(de, c, p.width, B::pack(f));
        }
      }
    }
    if (DOT) {
      const float2 d2 = apart(dot2);
      float dot = d2.x + d2.y;
#pragma unroll
      for (int d = LANES / 2; d > 0; d >>= 1) dot += __shfl_xor_sync(kAll, dot, d);
      if (lane == 0 && s < slots) p.dweights[s] = dot;
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
  int64_t units;         // rows, or slots
  int per_cta, threads;
  int per_sm;            // CTAs, at most
  void* stream;
};

goldy_status launch_rows(const LayerContext& ctx, void* arg) {
  RowCall& call = *static_cast<RowCall*>(arg);
  const int64_t grid = std::min(ceil_div(call.units, int64_t(call.per_cta)), int64_t(ctx.sm_count) * call.per_sm);
  void* args[] = {&call.p};
  return launch_layer("route", call.fn, grid, call.threads, 0, call.stream, args);
}

int64_t row_blocks(const goldy_route_desc& d) { return std::max<int64_t>(1, ceil_div(d.width, 16 / int64_t(element_size(d.dtype)))); }

goldy_status run_rows(const goldy_route_desc& d, RowCall& call, void* stream) {
  RowParams& p = call.p;
  p.rows = d.rows;
  p.ldx = d.ldx;
  p.lde = d.lde;
  p.ldr = d.ldr;
  p.width = int32_t(d.width);
  p.k = d.k;
  p.places = int32_t(slots_of(d));
  call.stream = stream;
  const goldy_status st = with_layer_context(stream, launch_rows, &call);
  return st == GOLDY_OK ? ok() : st;
}

// Threads that share a token's row, each with `per_thread` blocks at once: equal
// shares, whatever their number (a row of 139 blocks in twos: 70 threads, three
// rows per CTA), not powers of two.  A row off its blocks' boundaries has one more.
void share_rows(const goldy_route_desc& d, RowCall& call, int per_thread, bool aligned) {
  const int64_t blocks = row_blocks(d) + (aligned ? 0 : 1), rounds = ceil_div(blocks, int64_t(kRowThreads) * per_thread);
  call.p.lanes = int32_t(ceil_div(blocks, rounds * per_thread));
  call.p.per_cta = kRowThreads / call.p.lanes;
  call.units = d.rows;
  call.per_cta = call.p.per_cta;
  call.threads = call.p.lanes * call.p.per_cta;
  // more CTAs than fit (16384 x 4096 to two places: 67 us, resident ones alone 75)
  call.per_sm = 64;
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
const void* combine_fn(bool aligned, int k) {
  if (!aligned) return reinterpret_cast<const void*>(&route_combine_kernel<T, false, 4, 1>);
  return k > 2 ? reinterpret_cast<const void*>(&route_combine_kernel<T, true, 4, 2>)
               : reinterpret_cast<const void*>(&route_combine_kernel<T, true, 2, 2>);
}
// Threads per slot: few blocks leave no work for a whole warp.
int grad_lanes(const goldy_route_desc& d) { return row_blocks(d) > 48 ? 32 : row_blocks(d) > 16 ? 16 : 8; }
template <typename T, int LANES>
const void* grad_fn(bool aligned, bool dot) {
  if (dot)
    return aligned ? reinterpret_cast<const void*>(&route_combine_grad_kernel<T, true, true, LANES>)
                   : reinterpret_cast<const void*>(&route_combine_grad_kernel<T, false, true, LANES>);
  return aligned ? reinterpret_cast<const void*>(&route_combine_grad_kernel<T, true, false, LANES>)
                 : reinterpret_cast<const void*>(&route_combine_grad_kernel<T, false, false, LANES>);
}
template <typename T>
const void* grad_fn(bool aligned, bool dot, int lanes) {
  switch (lanes) {
    case 32: return grad_fn<T, 32>(aligned, dot);
    case 16: return grad_fn<T, 16>(aligned, dot);
    default: return grad_fn<T, 8>(aligned, dot);
  }
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
  while (p.share_log < 5 && (int64_t(p.groups + 1) << p.share_log) < kSortThreads && (1 << p.share_log) < p.chunks) ++p.share_log;
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
  call.fn = desc->dtype == GOLDY_F32 ? dispatch_fn<uint32_t>(aligned) : dispatch_fn<uint16_t>(aligned);
  share_rows(*desc, call, aligned ? kDispatchBlocks : 1, aligned);
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
  call.fn = desc->dtype == GOLDY_F32 ? combine_fn<uint32_t>(aligned, desc->k) : combine_fn<uint16_t>(aligned, desc->k);
  share_rows(*desc, call, aligned ? 2 : 1, aligned);
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
  // (rows of no elements: only the zeros of dweights are written)
  const bool aligned =
      desc->width == 0 || in_blocks(*desc, {{dY, desc->ldx}, {dweights ? E : nullptr, desc->lde}, {dE, desc->lde}});
  const bool dot = dweights != nullptr;
  const int lanes = grad_lanes(*desc);
  call.fn = desc->dtype == GOLDY_F32 ? grad_fn<uint32_t>(aligned, dot, lanes) : grad_fn<uint16_t>(aligned, dot, lanes);
  call.units = slots_of(*desc);
  call.per_cta = kRowThreads / lanes;
  call.threads = kRowThreads;
  call.per_sm = kGradCtas;                         // resident: the next slot's place is read ahead
  return run_rows(*desc, call, stream);
} catch (...) {
  return layer_exception();
}
