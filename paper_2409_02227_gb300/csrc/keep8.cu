// Pre-activations kept in 8 bits, and what the backward pass needs of them.
//
//   e = the smallest power with (largest finite |z| of 32) <= 448 * 2^e, at least -127
//   q = e4m3(z / 2^e);  Z = q 2^e,  H = act(Z)
//
// With the largest |z| = m 2^E, 1 <= m < 2, e is E - 8 for m <= 1.75 and E - 7
// above: integer arithmetic on its bits.  Multiplying by a power of two is exact,
// so that q is rounded once.
//
// HBM-bound: Z is read once and its blocks are written once, or the reverse.  A
// thread takes 8 elements, four neighbours share a block and its scale (8192 x 8192
// bf16, kept and read back through gelu: 78 us, 6.9 TB/s, as some of the blocks are
// still in the L2 cache).
#include <cuda_runtime.h>

#include <algorithm>

#include "layer_launch.h"
#include "row_blocks.cuh"
#include "sm103_ptx.cuh"

namespace goldy {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock = GOLDY_KEEP8_BLOCK;
constexpr int kPer = 8;                          // elements per thread
constexpr int kShare = kBlock / kPer;            // threads per block
constexpr int kUnroll = 4;                       // pieces of 8 per thread and step, packing; half as many back
constexpr uint32_t kInfinity = 0x7F800000u;

struct KeepParams {
  const void* z_in;
  uint2* q;              // 8 bytes per thread
  uint8_t* scales;
  void* z;
  void* h;
  int64_t rows, ldz, ldh;
  int32_t n, blocks;
  int32_t lanes_log;     // threads per row, log2
  int64_t pieces;        // of 8 elements, where rows follow one another without a gap
};

// 2^i for -127 <= i <= 127
__device__ __forceinline__ float power(int i) { return __uint_as_float(i > -127 ? uint32_t(i + 127) << 23 : 1u << 22); }

__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(uint16_t(v)));
  float2 f;
  asm("{.reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi;}" : "=f"(f.x), "=f"(f.y) : "r"(r));
  return f;
}

// Four lanes' 8 elements each as a block: this lane's bytes, and e.
__device__ __forceinline__ uint2 quantise(float (&f)[kPer], int& e) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
  if (top >= kInfinity) {                          // an infinity or NaN among them
    top = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const uint32_t b = __float_as_uint(f[i]) & 0x7FFFFFFFu;
      if (b < kInfinity) top = max(top, b);
      else f[i] = __uint_as_float(0x7FFFFFFFu);
    }
  }
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
  top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
  e = max(-127, int(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u));
  const uint64_t scale = two(power(-e));
  uint32_t w[kPer / 2];
#pragma unroll
  for (int i = 0; i < kPer / 2; ++i) {
    const float2 v = apart(mul2(two(f[2 * i], f[2 * i + 1]), scale));
    w[i] = to_e4m3x2(v.x, v.y);
  }
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) keep8_pack_kernel(const KeepParams p) {
  using B = Block<T>;
  constexpr int LOADS = kPer / B::PER;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lanes = 1 << p.lanes_log, x = threadIdx.x & (lanes - 1);
  const int per_row = p.blocks * kShare;
  const int64_t per_cta = kThreads >> p.lanes_log;
  const int64_t rounds = (p.rows + per_cta - 1) / per_cta;
  for (int64_t r = blockIdx.x; r < rounds; r += gridDim.x) {
    const int64_t row = r * per_cta + (threadIdx.x >> p.lanes_log);
    const typename B::Source source(static_cast<const T*>(p.z_in) + min(row, p.rows - 1) * p.ldz, p.n, 0);
    for (int at0 = 0; at0 < per_row; at0 += lanes) {     // every thread of a warp goes along: they trade maxima
      const int at = at0 + x;
      typename B::template Raw<false> raw[LOADS];
#pragma unroll
      for (int i = 0; i < LOADS; ++i)
        if (at * kPer + i * B::PER < p.n) raw[i].load(source, at * LOADS + i);
      float f[kPer];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int c = at * kPer + i * B::PER;
        float g[B::PER];
        uint4 v = make_uint4(0, 0, 0, 0);
        if (c < p.n) {
          v = raw[i].get(source.shift);
          if (c + B::PER > p.n) {
            const uint4 m = B::inside(c, p.n);
            v.x &= m.x, v.y &= m.y, v.z &= m.z, v.w &= m.w;
          }
        }
        B::unpack(v, g);
#pragma unroll
        for (int j = 0; j < B::PER; ++j) f[i * B::PER + j] = g[j];
      }
      int e;
      const uint2 bytes = quantise(f, e);
      if (row >= p.rows || at >= per_row) continue;
      p.q[row * per_row + at] = bytes;
      if ((at & (kShare - 1)) == 0) p.scales[row * p.blocks + at / kShare] = uint8_t(e + 127);
    }
  }
}

// Rows without gaps and of whole blocks are one long row: several pieces per
// thread are on their way at once, and no index is more than a sum.
template <typename T>
__global__ void __launch_bounds__(kThreads) keep8_pack_flat_kernel(const KeepParams p) {
  using B = Block<T>;
  constexpr int LOADS = kPer / B::PER;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const uint4* z = static_cast<const uint4*>(p.z_in);
  const int64_t step = int64_t(gridDim.x) * kThreads * kUnroll;
  for (int64_t u0 = int64_t(blockIdx.x) * kThreads * kUnroll + threadIdx.x; (u0 & ~int64_t(31)) < p.pieces; u0 += step) {
    uint4 v[kUnroll][LOADS];
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int64_t u = u0 + k * kThreads;
#pragma unroll
      for (int i = 0; i < LOADS; ++i) v[k][i] = u < p.pieces ? __ldcs(z + u * LOADS + i) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kUnroll; ++k) {
      const int64_t u = u0 + k * kThreads;
      float f[kPer];
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        float g[B::PER];
        B::unpack(v[k][i], g);
#pragma unroll
        for (int j = 0; j < B::PER; ++j) f[i * B::PER + j] = g[j];
      }
      int e;
      const uint2 q = quantise(f, e);
      if (u >= p.pieces) continue;
      p.q[u] = q;
      if ((u & (kShare - 1)) == 0) p.scales[u / kShare] = uint8_t(e + 127);
    }
  }
}

__device__ __forceinline__ void restore(const uint2& v, int e, uint64_t (&f)[kPer / 2]) {
  const uint64_t scale = two(power(e - 127));
  const uint32_t w[4] = {v.x, v.x >> 16, v.y, v.y >> 16};
#pragma unroll
  for (int i = 0; i < kPer / 2; ++i) {
    const float2 g = from_e4m3x2(w[i]);
    f[i] = mul2(two(g.x, g.y), scale);
  }
}

__device__ __forceinline__ void singles(const uint64_t (&v)[kPer / 2], float (&f)[kPer]) {
#pragma unroll
  for (int i = 0; i < kPer / 2; ++i) {
    const float2 g = apart(v[i]);
    f[2 * i] = g.x;
    f[2 * i + 1] = g.y;
  }
}

// Rows that start anywhere are written in blocks of their own address: the bytes of
// a block lie in two neighbouring words of 8 (4, for fp32), under one scale or two.
template <typename T, int ACT, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) keep8_unpack_kernel(const KeepParams p) {
  using B = Block<T>;
  constexpr int PAIRS = B::PER / 2;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lanes = 1 << p.lanes_log, x = threadIdx.x & (lanes - 1), row_bytes = p.blocks * kBlock;
  const int64_t step = int64_t(gridDim.x) * (kThreads >> p.lanes_log);
  for (int64_t row = int64_t(blockIdx.x) * (kThreads >> p.lanes_log) + (threadIdx.x >> p.lanes_log); row < p.rows; row += step) {
    const uint8_t* const q = reinterpret_cast<const uint8_t*>(p.q) + row * row_bytes;
    const uint8_t* const scales = p.scales + row * p.blocks;
    // values c .. c + PER - 1 of the row, in pairs (those outside it are anything)
    auto values = [&](int c, uint64_t (&f)[PAIRS]) {
      if constexpr (ALIGNED) {                     // whole words under one scale
        const uint32_t* w = reinterpret_cast<const uint32_t*>(q + c);
        const uint32_t lo = w[0], hi = B::PER == 8 ? w[B::PER / 4 - 1] : lo;
        const uint64_t scale = two(power(int(scales[c / kBlock]) - 127));
        const uint32_t v[4] = {lo, lo >> 16, hi, hi >> 16};
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
          const float2 g = from_e4m3x2(v[i]);
          f[i] = mul2(two(g.x, g.y), scale);
        }
        return;
      }
      const int first = max(c, 0), last = min(c + B::PER, row_bytes) - 1;       // kept bytes, zeros behind the row's end
      const int w0 = first / 4, w1 = last / 4, at = c >= 0 ? c : first;
      uint32_t w[3];
      if constexpr (B::PER == 8) {
        const int mid = min(w0 + 1, w1);
        w[0] = reinterpret_cast<const uint32_t*>(q)[w0];
        w[1] = reinterpret_cast<const uint32_t*>(q)[mid];
        w[2] = reinterpret_cast<const uint32_t*>(q)[w1];
      } else {
        w[0] = reinterpret_cast<const uint32_t*>(q)[w0];
        w[1] = w[2] = reinterpret_cast<const uint32_t*>(q)[w1];
      }
      const uint32_t bits = uint32_t(at & 3) * 8u;
      uint32_t lo = __funnelshift_r(w[0], w[1], bits), hi = __funnelshift_r(w[1], w[2], bits);
      if (c < 0) {                                 // the row's first elements are the block's last
        const uint32_t up = uint32_t(-c) * 8u;
        const uint64_t v = up < 64 ? (uint64_t(w[1]) << 32 | w[0]) << up : 0;
        lo = uint32_t(v), hi = uint32_t(v >> 32);
      }
      const int s0 = first / kBlock, change = (s0 + 1) * kBlock - c;            // elements under the first scale
      const float a = power(int(scales[s0]) - 127), b = power(int(scales[last / kBlock]) - 127);
      const uint32_t v[4] = {lo, lo >> 16, hi, hi >> 16};
#pragma unroll
      for (int i = 0; i < PAIRS; ++i) {
        const float2 g = from_e4m3x2(v[i]);
        f[i] = mul2(two(g.x, g.y), two(2 * i < change ? a : b, 2 * i + 1 < change ? a : b));
      }
    };
    auto fill = [&](T* to, bool act) {
      const int off = ALIGNED ? 0 : B::off(to), blocks = B::count(to, p.n);
      for (int i = x; i < blocks; i += lanes) {
        uint64_t f[PAIRS];
        values(i * B::PER - off, f);
        if (act) {
#pragma unroll
          for (int k = 0; k < PAIRS; ++k) f[k] = act_value2(f[k], ACT);
        }
        B::template store<false>(to, i * B::PER - off, p.n, B::pack(f));
      }
    };
    T* const z = p.z ? static_cast<T*>(p.z) + row * p.ldz : nullptr;
    T* const h = p.h ? static_cast<T*>(p.h) + row * p.ldh : nullptr;
    if (z && h && (ALIGNED || B::off(z) == B::off(h))) {       // both from one reading
      const int off = ALIGNED ? 0 : B::off(z), blocks = B::count(z, p.n);
      for (int i = x; i < blocks; i += lanes) {
        uint64_t f[PAIRS];
        values(i * B::PER - off, f);
        B::template store<false>(z, i * B::PER - off, p.n, B::pack(f));
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) f[k] = act_value2(f[k], ACT);
        B::template store<false>(h, i * B::PER - off, p.n, B::pack(f));
      }
    } else {
      if (z) fill(z, false);
      if (h) fill(h, true);
    }
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) keep8_unpack_flat_kernel(const KeepParams p) {
  using B = Block<T>;
  constexpr int UNROLL = kUnroll / 2, STORES = kPer / B::PER;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int64_t step = int64_t(gridDim.x) * kThreads * UNROLL;
  for (int64_t u0 = int64_t(blockIdx.x) * kThreads * UNROLL + threadIdx.x; u0 < p.pieces; u0 += step) {
    uint2 q[UNROLL];
    int e[UNROLL];
#pragma unroll
    for (int k = 0; k < UNROLL; ++k) {
      const int64_t u = min(u0 + k * kThreads, p.pieces - 1);
      q[k] = __ldcs(p.q + u);
      e[k] = p.scales[u / kShare];
    }
#pragma unroll
    for (int k = 0; k < UNROLL; ++k) {
      const int64_t u = u0 + k * kThreads;
      if (u >= p.pieces) break;
      uint64_t v[kPer / 2];
      float f[kPer];
      auto put = [&](void* base) {
        singles(v, f);
#pragma unroll
        for (int i = 0; i < STORES; ++i) {
          float g[B::PER];
#pragma unroll
          for (int j = 0; j < B::PER; ++j) g[j] = f[i * B::PER + j];
          __stcs(static_cast<uint4*>(base) + u * STORES + i, B::pack(g));
        }
      };
      restore(q[k], e[k], v);
      if (p.z) put(p.z);
      if (!p.h) continue;
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) v[i] = act_value2(v[i], ACT);
      put(p.h);
    }
  }
}

template <typename T, int ACT>
const void* unpack_fn(bool flat, bool aligned) {
  if (flat) return reinterpret_cast<const void*>(&keep8_unpack_flat_kernel<T, ACT>);
  return aligned ? reinterpret_cast<const void*>(&keep8_unpack_kernel<T, ACT, true>)
                 : reinterpret_cast<const void*>(&keep8_unpack_kernel<T, ACT, false>);
}
template <typename T>
const void* unpack_fn(int act, bool flat, bool aligned) {
  switch (act) {
    case GOLDY_ACT_RELU: return unpack_fn<T, GOLDY_ACT_RELU>(flat, aligned);
    case GOLDY_ACT_GELU: return unpack_fn<T, GOLDY_ACT_GELU>(flat, aligned);
    case GOLDY_ACT_GELU_TANH: return unpack_fn<T, GOLDY_ACT_GELU_TANH>(flat, aligned);
    case GOLDY_ACT_SILU: return unpack_fn<T, GOLDY_ACT_SILU>(flat, aligned);
    default: return unpack_fn<T, GOLDY_ACT_NONE>(flat, aligned);
  }
}
template <typename T>
const void* pack_fn(bool flat) {
  return flat ? reinterpret_cast<const void*>(&keep8_pack_flat_kernel<T>) : reinterpret_cast<const void*>(&keep8_pack_kernel<T>);
}

struct KeepCall {
  KeepParams p;
  const void* fn;
  bool flat;
  int per_thread;        // pieces per step (flat)
  void* stream;
};

goldy_status launch_keep(const LayerContext& ctx, void* arg) {
  KeepCall& call = *static_cast<KeepCall*>(arg);
  const int64_t units = call.flat ? ceil_div(call.p.pieces, int64_t(kThreads) * call.per_thread)
                                  : ceil_div(call.p.rows, int64_t(kThreads >> call.p.lanes_log));
  const int64_t grid = std::min(units, int64_t(ctx.sm_count) * 32);
  void* args[] = {&call.p};
  return launch_layer("keep8", call.fn, grid, kThreads, 0, call.stream, args);
}

goldy_status check_keep(const goldy_keep8_desc* d) {
  if (!d) return invalid("null descriptor");
  if (d->rows < 0 || d->n < 0 || d->n > (int64_t(1) << 30)) return invalid("keep8: a size is negative or too large");
  if (d->ldz < d->n || d->ldh < d->n) return invalid("keep8: a row stride is smaller than its row");
  if (d->rows > (int64_t(1) << 40) || too_far(d->rows, d->ldz) || too_far(d->rows, d->ldh) || too_far(d->rows, d->n + kBlock))
    return invalid("keep8: an array is beyond any memory");
  if (d->dtype != GOLDY_BF16 && d->dtype != GOLDY_F32)
    return fail(GOLDY_ERR_UNSUPPORTED, "keep8: types are GOLDY_BF16 or GOLDY_F32");
  if (d->act < GOLDY_ACT_NONE || d->act > GOLDY_ACT_SILU) return invalid("keep8: act out of range");
  if (d->reserved != 0) return invalid("keep8: reserved must be 0");
  return GOLDY_OK;
}

goldy_status run_keep(const goldy_keep8_desc& d, KeepCall& call, bool pack, void* stream) {
  KeepParams& p = call.p;
  p.rows = d.rows;
  p.ldz = d.ldz;
  p.ldh = d.ldh;
  p.n = int32_t(d.n);
  p.blocks = int32_t(ceil_div(d.n, kBlock));
  while ((1 << p.lanes_log) < kThreads && (1 << p.lanes_log) < p.blocks * kShare) ++p.lanes_log;
  const int64_t per = 16 / int64_t(element_size(d.dtype));
  auto whole = [&](const void* a, int64_t ld) { return !a || (on_boundary(a, 16) && ld % per == 0); };
  auto packed = [&](const void* a, int64_t ld) { return !a || ld == d.n; };
  const bool aligned = whole(p.z_in, d.ldz) && whole(p.z, d.ldz) && whole(p.h, d.ldh);
  call.flat = aligned && d.n % kBlock == 0 && packed(p.z_in, d.ldz) && packed(p.z, d.ldz) && packed(p.h, d.ldh);
  p.pieces = d.rows * (d.n / kPer);
  call.per_thread = pack ? kUnroll : kUnroll / 2;
  const bool f32 = d.dtype == GOLDY_F32;
  if (pack) call.fn = f32 ? pack_fn<uint32_t>(call.flat) : pack_fn<uint16_t>(call.flat);
  else call.fn = f32 ? unpack_fn<uint32_t>(d.act, call.flat, aligned) : unpack_fn<uint16_t>(d.act, call.flat, aligned);
  call.stream = stream;
  const goldy_status st = with_layer_context(stream, launch_keep, &call);
  return st == GOLDY_OK ? ok() : st;
}

}  // namespace
}  // namespace goldy

using namespace goldy;

extern "C" goldy_status goldy_keep8_query(const goldy_keep8_desc* desc, size_t* q_bytes, size_t* scale_bytes) try {
  const goldy_status st = check_keep(desc);
  if (st != GOLDY_OK) return st;
  if (!q_bytes || !scale_bytes) return invalid("null argument");
  *scale_bytes = size_t(desc->rows) * size_t(ceil_div(desc->n, kBlock));
  *q_bytes = *scale_bytes * kBlock;
  return ok();
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_keep8_pack(const goldy_keep8_desc* desc, const void* Z, void* Q, void* scales,
                                         void* stream) try {
  const goldy_status st = check_keep(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->n == 0) return ok();
  if (!Z || !Q || !scales) return invalid("keep8: Z, Q and scales are needed");
  if (!on_boundary(Z, element_size(desc->dtype)) || !on_boundary(Q, 16)) return invalid("keep8: Z or Q misaligned");
  KeepCall call{};
  call.p.z_in = Z;
  call.p.q = static_cast<uint2*>(Q);
  call.p.scales = static_cast<uint8_t*>(scales);
  return run_keep(*desc, call, true, stream);
} catch (...) {
  return layer_exception();
}

extern "C" goldy_status goldy_keep8_unpack(const goldy_keep8_desc* desc, const void* Q, const void* scales, void* Z,
                                           void* H, void* stream) try {
  const goldy_status st = check_keep(desc);
  if (st != GOLDY_OK) return st;
  if (desc->rows == 0 || desc->n == 0) return ok();
  if (!Q || !scales || (!Z && !H)) return invalid("keep8: Q, scales and one of Z and H are needed");
  const size_t es = element_size(desc->dtype);
  if (!on_boundary(Z, es) || !on_boundary(H, es) || !on_boundary(Q, 16)) return invalid("keep8: a pointer is misaligned");
  if (Z == H) return invalid("keep8: Z and H are one array");
  KeepCall call{};
  call.p.q = static_cast<uint2*>(const_cast<void*>(Q));
  call.p.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
  call.p.z = Z;
  call.p.h = H;
  return run_keep(*desc, call, false, stream);
} catch (...) {
  return layer_exception();
}
