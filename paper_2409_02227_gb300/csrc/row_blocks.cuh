// Rows moved in 16-byte blocks whatever element they start on.  A row's result
// is written in the blocks of its own address; what goes into a block is loaded
// from two neighbouring blocks of a source that starts on another element and
// shifted into place.  Blocks that a row shares with its neighbours are written
// element by element.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "layer_math.cuh"

namespace goldy {

// 16 bytes from an address on any element's boundary: the aligned blocks that
// hold them, words picked by the address's low bits.
__device__ __forceinline__ uint4 load_block_any(const void* from) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(from);
  const uint4* base = reinterpret_cast<const uint4*>(a & ~uintptr_t(15));
  const uint32_t off = uint32_t(a) & 15u;
  const uint4 lo = base[0];
  if (off == 0) return lo;
  const uint4 hi = base[1];
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  if (off & 8u) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (off & 4u) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const uint32_t bits = (off & 3u) * 8u;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                    __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}

template <typename T>
struct Block {
  static constexpr int PER = 16 / int(sizeof(T));
  // elements that a row's address lies behind a block's start
  static __device__ __forceinline__ int off(const void* row) {
    return int(reinterpret_cast<uintptr_t>(row) & 15) / int(sizeof(T));
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[PER]) {
    if constexpr (sizeof(T) == 2) unpack8(v, f);
    else f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[PER]) {
    if constexpr (sizeof(T) == 2) return pack8(f);
    else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ float at(const T* row, int64_t c) {
    return sizeof(T) == 2 ? load_bf16(row, c) : reinterpret_cast<const float*>(row)[c];
  }
  static __device__ __forceinline__ void put(T* row, int64_t c, float v) {
    if (sizeof(T) == 2) store_bf16(row, c, v);
    else reinterpret_cast<float*>(row)[c] = v;
  }
  // Elements c .. c + PER - 1 of a row of n, 0 outside it; ALIGNED: inside, on a
  // block's boundary.
  template <bool ALIGNED>
  static __device__ __forceinline__ uint4 load(const T* row, int64_t c, int64_t n) {
    if (ALIGNED) return *reinterpret_cast<const uint4*>(row + c);
    if (c >= 0 && c + PER <= n) return load_block_any(row + c);
    float f[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) f[i] = c + i >= 0 && c + i < n ? at(row, c + i) : 0.0f;
    return pack(f);
  }
  // The same elements, on a block's boundary, written where they are inside.
  template <bool ALIGNED>
  static __device__ __forceinline__ void store(T* row, int64_t c, int64_t n, const uint4& v) {
    if (ALIGNED || (c >= 0 && c + PER <= n)) {
      *reinterpret_cast<uint4*>(row + c) = v;
      return;
    }
    float f[PER];
    unpack(v, f);
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (c + i >= 0 && c + i < n) put(row, c + i, f[i]);
  }
};

}  // namespace goldy
