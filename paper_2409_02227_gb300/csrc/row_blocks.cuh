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

// 16 bytes that start `off` bytes into two neighbouring blocks; off is one for a
// whole row, so that its threads take the same way.
__device__ __forceinline__ uint4 shift_blocks(const uint4& lo, const uint4& hi, uint32_t off) {
  const uint32_t bits = (off & 3u) * 8u;
  switch (off >> 2) {
    case 0:
      return make_uint4(__funnelshift_r(lo.x, lo.y, bits), __funnelshift_r(lo.y, lo.z, bits),
                        __funnelshift_r(lo.z, lo.w, bits), __funnelshift_r(lo.w, hi.x, bits));
    case 1:
      return make_uint4(__funnelshift_r(lo.y, lo.z, bits), __funnelshift_r(lo.z, lo.w, bits),
                        __funnelshift_r(lo.w, hi.x, bits), __funnelshift_r(hi.x, hi.y, bits));
    case 2:
      return make_uint4(__funnelshift_r(lo.z, lo.w, bits), __funnelshift_r(lo.w, hi.x, bits),
                        __funnelshift_r(hi.x, hi.y, bits), __funnelshift_r(hi.y, hi.z, bits));
    default:
      return make_uint4(__funnelshift_r(lo.w, hi.x, bits), __funnelshift_r(hi.x, hi.y, bits),
                        __funnelshift_r(hi.y, hi.z, bits), __funnelshift_r(hi.z, hi.w, bits));
  }
}

// T: uint16_t for bf16, uint32_t for fp32.
template <typename T>
struct Block {
  static constexpr int PER = 16 / int(sizeof(T));
  // elements that a row's address lies behind a block's start
  static __device__ __forceinline__ int off(const void* row) {
    return int(reinterpret_cast<uintptr_t>(row) & 15) / int(sizeof(T));
  }
  // blocks that a row of n > 0 elements lies in
  static __device__ __forceinline__ int count(const void* row, int n) { return (off(row) + n - 1) / PER + 1; }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[PER]) {
    if constexpr (sizeof(T) == 2) unpack8(v, f);
    else f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[PER]) {
    if constexpr (sizeof(T) == 2) return pack8(f);
    else return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  // the same in pairs
  static __device__ __forceinline__ void pairs(const uint4& v, uint64_t (&f)[PER / 2]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
      if constexpr (sizeof(T) == 2) f[i] = two(bf16_lo(w[i]), bf16_hi(w[i]));
      else f[i] = two(__uint_as_float(w[2 * i % 4]), __uint_as_float(w[(2 * i + 1) % 4]));
    }
  }
  static __device__ __forceinline__ uint4 pack(const uint64_t (&f)[PER / 2]) {
    float v[PER];
#pragma unroll
    for (int i = 0; i < PER / 2; ++i) {
      const float2 p = apart(f[i]);
      v[2 * i] = p.x;
      v[2 * i + 1] = p.y;
    }
    return pack(v);
  }
  // A row of n elements as the source of a result whose row starts `off` elements
  // behind a block's start: block b of the result holds the row's elements from
  // b * PER - off on, which lie in two neighbouring blocks of the source.
  struct Source {
    const uint4* first;      // the row's first block
    int last;                // its last one
    int ahead;               // result's block b starts in the source's block b + ahead,
    uint32_t shift;          // so many bytes in
    __device__ __forceinline__ Source() {}
    __device__ __forceinline__ Source(const T* row, int n, int off_result) {
      const uintptr_t a = reinterpret_cast<uintptr_t>(row);
      const uint32_t off_row = uint32_t(a & 15) / uint32_t(sizeof(T));
      const int d = int(off_row) - off_result;
      first = reinterpret_cast<const uint4*>(a & ~uintptr_t(15));
      last = int((off_row + uint32_t(n) - 1) / PER);
      ahead = d >> 31;
      shift = (uint32_t(d) & (PER - 1)) * uint32_t(sizeof(T));
    }
  };
  // What a block of the result is made from: loads alone, so that many are on
  // their way before the first is shifted into place.  Only blocks that hold some
  // of the row are read; elements of the result outside its row come out as anything.
  template <bool ALIGNED>
  struct Raw {
    uint4 v[ALIGNED ? 1 : 2];
    __device__ __forceinline__ void load(const Source& s, int b) {
      if (ALIGNED) {
        v[0] = s.first[b];
      } else {
        b += s.ahead;
        v[0] = s.first[uint32_t(max(b, 0))];
        if (s.shift) v[ALIGNED ? 0 : 1] = s.first[uint32_t(min(b + 1, s.last))];
      }
    }
    __device__ __forceinline__ uint4 get(uint32_t shift) const {
      if (ALIGNED) return v[0];
      return shift_blocks(v[0], v[ALIGNED ? 0 : 1], shift);
    }
  };
  // ones in the place of the elements inside a row of n (c: the first one's index)
  static __device__ __forceinline__ uint4 inside(int c, int n) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (sizeof(T) == 4) w[i] = uint32_t(c + i) < uint32_t(n) ? 0xFFFFFFFFu : 0u;
      else w[i] = (uint32_t(c + 2 * i) < uint32_t(n) ? 0xFFFFu : 0u) | (uint32_t(c + 2 * i + 1) < uint32_t(n) ? 0xFFFF0000u : 0u);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  // Elements c .. c + PER - 1 of a row of n, on a block's boundary, written where
  // they are inside.
  template <bool ALIGNED>
  static __device__ __forceinline__ void store(T* row, int c, int n, const uint4& v) {
    if (ALIGNED || (c >= 0 && c + PER <= n)) {
      *reinterpret_cast<uint4*>(row + c) = v;
      return;
    }
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < PER; ++i)
      if (uint32_t(c + i) < uint32_t(n)) row[c + i] = sizeof(T) == 4 ? T(w[i % 4]) : T(w[i / 2 % 4] >> (i & 1) * 16);
  }
};

}  // namespace goldy
