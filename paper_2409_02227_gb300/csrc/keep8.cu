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
// thread takes 8 elements, four neighbours share a block and its scale.
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
constexpr uint32_t kInfinity = 0x7F800000u;

struct KeepParams {
  const void* z_in;
  uint2* q;              // 8 bytes per thread
  uint8_t* scales;
  void* z;
  void* h;
  int64_t rows, ldz, ldh;
  int32_t n, blocks, vec;
  int32_t lanes_log;     // threads per row, log2
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

// 8 elements from column c on, 0 behind the row's end
template <typename T>
__device__ __forceinline__ void load8(const T* row, int c, int n, int vec, float (&f)[kPer]) {
  using B = Block<T>;
#pragma unroll
  for (int i = 0; i < kPer; i += B::PER) {
    float g[B::PER];
    B::unpack(vec && c + i + B::PER <= n ? B::template load<true>(row, c + i, n) : B::template load<false>(row, c + i, n), g);
#pragma unroll
    for (int j = 0; j < B::PER; ++j) f[i + j] = g[j];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* row, int c, int n, int vec, const float (&f)[kPer]) {
  using B = Block<T>;
#pragma unroll
  for (int i = 0; i < kPer; i += B::PER) {
    if (vec && c + i + B::PER <= n) {
      float g[B::PER];
#pragma unroll
      for (int j = 0; j < B::PER; ++j) g[j] = f[i + j];
      B::template store<true>(row, c + i, n, B::pack(g));
    } else {
#pragma unroll
      for (int j = 0; j < B::PER; ++j)
        if (c + i + j < n) B::put(row, c + i + j, f[i + j]);
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) keep8_pack_kernel(const KeepParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lanes = 1 << p.lanes_log, x = threadIdx.x & (lanes - 1);
  const int per_row = p.blocks * kShare;
  const int64_t per_cta = kThreads >> p.lanes_log;
  const int trips = (per_row + lanes - 1) >> p.lanes_log;
  const int64_t rounds = (p.rows + per_cta - 1) / per_cta;
  for (int64_t r = blockIdx.x; r < rounds; r += gridDim.x) {
    const int64_t row = r * per_cta + (threadIdx.x >> p.lanes_log);
    for (int trip = 0; trip < trips; ++trip) {      // every thread of a warp goes along: they trade maxima
      const int at = trip * lanes + x;
      const bool in = row < p.rows && at < per_row;
      float f[kPer];
#pragma unroll
      for (int i = 0; i < kPer; ++i) f[i] = 0.0f;
      if (in) load8<T>(static_cast<const T*>(p.z_in) + row * p.ldz, at * kPer, p.n, p.vec, f);
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kPer; ++i) top = max(top, __float_as_uint(f[i]) & 0x7FFFFFFFu);
      const bool odd = top >= kInfinity;            // an infinity or NaN among them
      if (odd) {
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
      const int e = max(-127, int(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u));
      const float scale = power(-e);
      uint32_t w[kPer / 2];
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) w[i] = to_e4m3x2(f[2 * i] * scale, f[2 * i + 1] * scale);
      if (!in) continue;
      p.q[row * per_row + at] = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
      if ((at & (kShare - 1)) == 0) p.scales[row * p.blocks + at / kShare] = uint8_t(e + 127);
    }
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads) keep8_unpack_kernel(const KeepParams p) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lanes = 1 << p.lanes_log, x = threadIdx.x & (lanes - 1);
  const int per_row = p.blocks * kShare, used = (p.n + kPer - 1) / kPer;
  const int64_t step = int64_t(gridDim.x) * (kThreads >> p.lanes_log);
  for (int64_t row = int64_t(blockIdx.x) * (kThreads >> p.lanes_log) + (threadIdx.x >> p.lanes_log); row < p.rows; row += step)
    for (int at = x; at < used; at += lanes) {
      const uint2 v = p.q[row * per_row + at];
      const float scale = power(int(p.scales[row * p.blocks + at / kShare]) - 127);
      const uint32_t w[4] = {v.x, v.x >> 16, v.y, v.y >> 16};
      float f[kPer];
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) {
        const float2 g = from_e4m3x2(w[i]);
        f[2 * i] = g.x * scale;
        f[2 * i + 1] = g.y * scale;
      }
      if (p.z) store8<T>(static_cast<T*>(p.z) + row * p.ldz, at * kPer, p.n, p.vec, f);
      if (!p.h) continue;
#pragma unroll
      for (int i = 0; i < kPer / 2; ++i) {
        const float2 g = apart(act_value2(two(f[2 * i], f[2 * i + 1]), ACT));
        f[2 * i] = g.x;
        f[2 * i + 1] = g.y;
      }
      store8<T>(static_cast<T*>(p.h) + row * p.ldh, at * kPer, p.n, p.vec, f);
    }
}

template <typename T>
const void* unpack_fn(int act) {
  switch (act) {
    case GOLDY_ACT_RELU: return reinterpret_cast<const void*>(&keep8_unpack_kernel<T, GOLDY_ACT_RELU>);
    case GOLDY_ACT_GELU: return reinterpret_cast<const void*>(&keep8_unpack_kernel<T, GOLDY_ACT_GELU>);
    case GOLDY_ACT_GELU_TANH: return reinterpret_cast<const void*>(&keep8_unpack_kernel<T, GOLDY_ACT_GELU_TANH>);
    case GOLDY_ACT_SILU: return reinterpret_cast<const void*>(&keep8_unpack_kernel<T, GOLDY_ACT_SILU>);
    default: return reinterpret_cast<const void*>(&keep8_unpack_kernel<T, GOLDY_ACT_NONE>);
  }
}

struct KeepCall {
  KeepParams p;
  const void* fn;
  void* stream;
};

goldy_status launch_keep(const LayerContext& ctx, void* arg) {
  KeepCall& call = *static_cast<KeepCall*>(arg);
  const int64_t grid = std::min(ceil_div(call.p.rows, int64_t(kThreads >> call.p.lanes_log)), int64_t(ctx.sm_count) * 32);
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

goldy_status run_keep(const goldy_keep8_desc& d, KeepCall& call, void* stream) {
  KeepParams& p = call.p;
  p.rows = d.rows;
  p.ldz = d.ldz;
  p.ldh = d.ldh;
  p.n = int32_t(d.n);
  p.blocks = int32_t(ceil_div(d.n, kBlock));
  while ((1 << p.lanes_log) < kThreads && (1 << p.lanes_log) < p.blocks * kShare) ++p.lanes_log;
  const int64_t per = 16 / int64_t(element_size(d.dtype));
  auto whole = [&](const void* a, int64_t ld) { return !a || (on_boundary(a, 16) && ld % per == 0); };
  p.vec = whole(p.z_in, d.ldz) && whole(p.z, d.ldz) && whole(p.h, d.ldh);
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
  call.fn = desc->dtype == GOLDY_F32 ? reinterpret_cast<const void*>(&keep8_pack_kernel<float>)
                                     : reinterpret_cast<const void*>(&keep8_pack_kernel<uint16_t>);
  return run_keep(*desc, call, stream);
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
  call.fn = desc->dtype == GOLDY_F32 ? unpack_fn<float>(desc->act) : unpack_fn<uint16_t>(desc->act);
  return run_keep(*desc, call, stream);
} catch (...) {
  return layer_exception();
}
