// What the norms share: rows held in a team of threads' registers, fetched ahead
// into shared memory, and the sums over a warp, a team and a cluster.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "layer_math.cuh"
#include "sm103_ptx.cuh"

namespace goldy {

constexpr int kMaxCluster = 8;      // CTAs that may share a row

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Sums of a and of b over the warp, in lanes 0 to 15 that of a, in the others
// that of b: half the exchanges of two sums.
__device__ __forceinline__ float warp_sum2(float a, float b, int lane) {
  const bool upper = lane & 16;
  float v = (upper ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : b, 16);
#pragma unroll
  for (int d = 8; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// Sums of four values over the warp, to all lanes, or, with an address in shared
// memory, to there: 6 exchanges instead of 20.
__device__ __forceinline__ float4 warp_sum4(float a, float b, float c, float d, int lane, float* to) {
  const bool upper = lane & 16, second = lane & 8;
  const float x = (upper ? c : a) + __shfl_xor_sync(0xFFFFFFFFu, upper ? a : c, 16);
  const float y = (upper ? d : b) + __shfl_xor_sync(0xFFFFFFFFu, upper ? b : d, 16);
  float v = (second ? y : x) + __shfl_xor_sync(0xFFFFFFFFu, second ? x : y, 8);
#pragma unroll
  for (int k = 4; k > 0; k >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, k);
  if (to) {
    if ((lane & 7) == 0) to[lane >> 3] = v;
    return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  return make_float4(__shfl_sync(0xFFFFFFFFu, v, 0), __shfl_sync(0xFFFFFFFFu, v, 8), __shfl_sync(0xFFFFFFFFu, v, 16),
                     __shfl_sync(0xFFFFFFFFu, v, 24));
}

__device__ __forceinline__ float param_at(const void* p, int f32, int i, float absent) {
  if (!p) return absent;
  return f32 ? static_cast<const float*>(p)[i] : load_bf16(p, i);
}

// Sum over groups of N consecutive lanes (N a power of two), to all of them.
template <int N>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int d = N / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  return v;
}

// PER parameters from index c on, 0 from n on and before 0; VEC: c + PER <= n, on a vector's
// boundary.  Plain loads, as of mean and rstd: the kernel before this one may have
// written them after this one began, which the read-only data path does not allow.
template <int PER, bool VEC>
__device__ __forceinline__ void load_params(const void* p, int f32, int c, int n, float absent, float* f) {
  if (!VEC || !p) {
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      if (!VEC && (c + k >= n || c + k < 0)) f[k] = 0.0f;
      else if (!p) f[k] = absent;
      else f[k] = f32 ? static_cast<const float*>(p)[c + k] : load_bf16(p, c + k);
    }
  } else if (f32) {
#pragma unroll
    for (int k = 0; k < PER; k += 4) {
      const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(p) + c + k);
      f[k] = v.x, f[(k + 1) % PER] = v.y, f[(k + 2) % PER] = v.z, f[(k + 3) % PER] = v.w;
    }
  } else if (PER == 8) {
    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + c);
    f[0] = bf16_lo(v.x), f[1 % PER] = bf16_hi(v.x), f[2 % PER] = bf16_lo(v.y), f[3 % PER] = bf16_hi(v.y);
    f[4 % PER] = bf16_lo(v.z), f[5 % PER] = bf16_hi(v.z), f[6 % PER] = bf16_lo(v.w), f[7 % PER] = bf16_hi(v.w);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + c);
    f[0] = bf16_lo(v.x), f[1 % PER] = bf16_hi(v.x), f[2 % PER] = bf16_lo(v.y), f[3 % PER] = bf16_hi(v.y);
  }
}

template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
  const uint32_t at = ptx::smem_u32(to);
  if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// A thread's share of a row, VALS values, in pieces: piece i of thread t starts
// at column (i * TEAM + t) * PER.  VEC: 16 bytes, inside the row or outside as a
// whole.  bf16 otherwise (odd lengths or strides, rows that start anywhere),
// SHIFT: 8 elements, maybe part of them outside, that lie in two 16-byte blocks.
// Whole blocks are copied, each by one thread of the team, and a thread picks its
// elements from its block and the next; a result's blocks are put together from
// a lane's and the lower lane's elements and stored whole, but for those that two
// warps or two rows share (16384 rows of 2047: 42 us, backwards 54; loading and
// storing single elements took 62 and 69, aligned words traded between lanes 57
// and 79).  What else a row's first and last block hold is read and ignored,
// never written.  fp32 otherwise: single elements (4096 rows of 4095: 29 us,
// backwards 50; in blocks 30 and 55).
// SURE: the first half of the pieces is inside whatever the row's length, as the
// host takes the smallest team that holds the row: no tests for those.
// FRAME (with VEC): the row starts `lo` elements behind a block's start, and so do
// all rows of the team and all arrays; columns are counted from the block's start,
// n is the row's end in that count, and only its first and last block are not whole.
template <typename T, int VALS, int TEAM, int THREADS, bool VEC, bool WIDE, bool FRAME = false>
struct NormRow {
  static constexpr bool SHIFT = !VEC && sizeof(T) == 2;
  static constexpr int PER = VEC ? 16 / int(sizeof(T)) : SHIFT ? 8 : 1;
  static constexpr int SLOTS = VALS / PER;
  static constexpr int PIECE = VEC || SHIFT ? 16 : 4;
  static constexpr int BLOCKS = SLOTS * TEAM + 1;  // SHIFT: of one row
  static constexpr int RING_BYTES = SHIFT ? THREADS / TEAM * BLOCKS * 16 : SLOTS * THREADS * PIECE;   // of one row per team
  static constexpr int SURE = TEAM > 32 && !WIDE && !FRAME ? SLOTS / 2 : 0;
  static __device__ __forceinline__ int col(int slot, int t) { return (slot * TEAM + t) * PER; }
  static __device__ __forceinline__ bool in(int slot, int t, int n) { return slot < SURE || col(slot, t) < n; }
  static __device__ __forceinline__ bool whole(int slot, int t, int n) {
    return !SHIFT || slot < SURE || col(slot, t) + PER <= n;
  }
  // elements lo <= col + k < n of a piece, and how many there are
  static __device__ __forceinline__ bool inside(int slot, int k, int t, int n, int lo) {
    return col(slot, t) + k < n && (!FRAME || col(slot, t) + k >= lo);
  }
  static __device__ __forceinline__ bool complete(int slot, int t, int n, int lo) {
    return FRAME ? col(slot, t) >= lo && col(slot, t) + PER <= n : whole(slot, t, n);
  }
  static __device__ __forceinline__ int count(int slot, int t, int n, int lo) {
    return complete(slot, t, n, lo) ? PER : min(col(slot, t) + PER, n) - (FRAME ? max(col(slot, t), lo) : col(slot, t));
  }
  // FRAME: ones in the place of a thread's elements, for its pieces' words
  struct Masks {
    uint4 m[FRAME ? SLOTS : 1];
    __device__ __forceinline__ Masks(int t, int n, int lo) {
      if constexpr (FRAME) {
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
          uint32_t w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if (sizeof(T) == 4) w[k] = inside(s, k, t, n, lo) ? 0xFFFFFFFFu : 0u;
            else w[k] = (inside(s, 2 * k, t, n, lo) ? 0xFFFFu : 0u) | (inside(s, 2 * k + 1, t, n, lo) ? 0xFFFF0000u : 0u);
          }
          m[s] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
  };
  // SHIFT: elements by which a row starts behind a block's start
  static __device__ __forceinline__ int shift(const T* at) { return int(reinterpret_cast<uintptr_t>(at) & 15) / 2; }
  // place in the ring of a thread's piece, or block
  static __device__ __forceinline__ int place(int slot, int t) {
    return SHIFT ? (int(threadIdx.x) / TEAM * BLOCKS + slot * TEAM + t) * 16 : (slot * THREADS + int(threadIdx.x)) * PIECE;
  }

  static __device__ __forceinline__ void fetch(uint8_t* ring, const void* base, int64_t row, int64_t ld, int n, int t) {
    fetch(ring, static_cast<const T*>(base) + row * ld, n, t);
  }
  static __device__ __forceinline__ void fetch(uint8_t* ring, const T* at, int n, int t) {
    const int off = SHIFT ? shift(at) : 0;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s)
      if (in(s, t, n + off)) copy_async<PIECE>(ring + place(s, t), at + col(s, t) - off);
    if (SHIFT && t == 0 && col(SLOTS, 0) < n + off) copy_async<PIECE>(ring + place(SLOTS, 0), at + col(SLOTS, 0) - off);
  }

  template <int OFF>
  static __device__ __forceinline__ void pick(const uint8_t* ring, int n, int t, float (&f)[VALS]) {
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const uint4 a = *reinterpret_cast<const uint4*>(ring + place(s, t));
      const uint4 b = OFF > 0 ? *reinterpret_cast<const uint4*>(ring + place(s, t) + 16) : a;
      const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
      for (int k = 0; k < 8; ++k) f[(s * PER + k) % VALS] = (OFF + k) & 1 ? bf16_hi(w[(OFF + k) / 2]) : bf16_lo(w[(OFF + k) / 2]);
      if (!whole(s, t, n)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (col(s, t) + k >= n) f[(s * PER + k) % VALS] = 0.0f;
      }
    }
  }
  // the row's values, 0 outside it (SHIFT: behind the team's barrier)
  static __device__ __forceinline__ void values(const uint8_t* ring, const void* base, int64_t row, int64_t ld, int n,
                                                int t, float (&f)[VALS]) {
    values(ring, static_cast<const T*>(base) + row * ld, n, t, f, 0);
  }
  // OUTSIDE: what tells the elements outside a frame's row, `lo` or masks (which cost
  // registers, but no way apart for the threads at the row's ends: backwards 16384 x
  // 1999 104 us, with lo 110; forwards 8192 x 3333 57, with lo 53)
  template <typename OUTSIDE>
  static __device__ __forceinline__ void values(const uint8_t* ring, const T* at, int n, int t, float (&f)[VALS], const OUTSIDE& out) {
    if constexpr (SHIFT) {
      switch (shift(at)) {
        case 0: pick<0>(ring, n, t, f); break;
        case 1: pick<1>(ring, n, t, f); break;
        case 2: pick<2>(ring, n, t, f); break;
        case 3: pick<3>(ring, n, t, f); break;
        case 4: pick<4>(ring, n, t, f); break;
        case 5: pick<5>(ring, n, t, f); break;
        case 6: pick<6>(ring, n, t, f); break;
        default: pick<7>(ring, n, t, f); break;
      }
    } else {
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        if (!in(s, t, n)) {
#pragma unroll
          for (int k = 0; k < PER; ++k) f[s * PER + k] = 0.0f;
        } else if (!VEC) {
          f[s] = *reinterpret_cast<const float*>(ring + place(s, t));
        } else {
          uint4 v = *reinterpret_cast<const uint4*>(ring + place(s, t));
          if constexpr (FRAME && sizeof(OUTSIDE) > sizeof(int))
            v.x &= out.m[s].x, v.y &= out.m[s].y, v.z &= out.m[s].z, v.w &= out.m[s].w;
          float* o = f + s * PER;
          if (sizeof(T) == 2) {
            o[0] = bf16_lo(v.x), o[1] = bf16_hi(v.x), o[2] = bf16_lo(v.y), o[3] = bf16_hi(v.y);
            o[4 % PER] = bf16_lo(v.z), o[5 % PER] = bf16_hi(v.z), o[6 % PER] = bf16_lo(v.w), o[7 % PER] = bf16_hi(v.w);
          } else {
            o[0] = __uint_as_float(v.x), o[1] = __uint_as_float(v.y), o[2] = __uint_as_float(v.z), o[3] = __uint_as_float(v.w);
          }
          if constexpr (FRAME && sizeof(OUTSIDE) == sizeof(int)) {
            if (!complete(s, t, n, out)) {
#pragma unroll
              for (int k = 0; k < PER; ++k)
                if (!inside(s, k, t, n, out)) o[k] = 0.0f;
            }
          }
        }
      }
    }
  }

  // SHIFT: `at` is OFF elements behind a block's start
  template <int OFF>
  static __device__ __forceinline__ void put(T* at, int n, int t, const float (&f)[VALS]) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int s = 0; s < SLOTS; ++s) {
      const int c = col(s, t);
      uint32_t w[8];                               // the lower lane's elements, then this lane's
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        w[4 + k] = pack_bf16(f[(s * PER + 2 * k) % VALS], f[(s * PER + 2 * k + 1) % VALS]);
        w[k] = 2 * k + 1 >= 8 - OFF ? __shfl_up_sync(0xFFFFFFFFu, w[4 + k], 1) : 0u;
      }
      uint32_t v[4];                               // elements 8 - OFF .. 15 - OFF of those
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int h = 8 - OFF + 2 * k;
        v[k] = h & 1 ? __byte_perm(w[h / 2], w[(h / 2 + 1) % 8], 0x5432) : w[(h / 2) % 8];
      }
      // blocks that this lane, and the next, store whole
      const bool own = (OFF == 0 || lane > 0) && (s < SURE || c + 8 - OFF <= n);
      const bool next = lane < 31 && (s < SURE || c + 16 - OFF <= n);
      if (own) __stcs(reinterpret_cast<uint4*>(at + c - OFF), make_uint4(v[0], v[1], v[2], v[3]));
      if (!own || (OFF > 0 && !next)) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if ((k < 8 - OFF ? !own : !next) && (s < SURE || c + k < n))
            reinterpret_cast<uint16_t*>(at)[c + k] = uint16_t(w[4 + k / 2] >> (k & 1) * 16);
      }
    }
  }
  // the row's results (all lanes of a warp)
  static __device__ __forceinline__ void store(void* base, int64_t row, int64_t ld, int n, int t, const float (&f)[VALS]) {
    store(static_cast<T*>(base) + row * ld, n, t, f);
  }
  static __device__ __forceinline__ void store(T* at, int n, int t, const float (&f)[VALS], int lo = 0) {
    if constexpr (SHIFT) {
      switch (shift(at)) {
        case 0: put<0>(at, n, t, f); break;
        case 1: put<1>(at, n, t, f); break;
        case 2: put<2>(at, n, t, f); break;
        case 3: put<3>(at, n, t, f); break;
        case 4: put<4>(at, n, t, f); break;
        case 5: put<5>(at, n, t, f); break;
        case 6: put<6>(at, n, t, f); break;
        default: put<7>(at, n, t, f); break;
      }
    } else {
#pragma unroll
      for (int s = 0; s < SLOTS; ++s) {
        if (!in(s, t, n)) continue;
        T* to = at + col(s, t);
        const float* v = f + s * PER;
        if (FRAME && !complete(s, t, n, lo)) {
#pragma unroll
          for (int k = 0; k < PER; ++k) {
            if (!inside(s, k, t, n, lo)) continue;
            if (sizeof(T) == 2) store_bf16(to, k, v[k]);
            else reinterpret_cast<float*>(to)[k] = v[k];
          }
        } else if (!VEC) {
          *reinterpret_cast<float*>(to) = v[0];
        } else if (sizeof(T) == 2) {
          __stcs(reinterpret_cast<uint4*>(to), make_uint4(pack_bf16(v[0], v[1 % PER]), pack_bf16(v[2 % PER], v[3 % PER]),
                                                          pack_bf16(v[4 % PER], v[5 % PER]), pack_bf16(v[6 % PER], v[7 % PER])));
        } else {
          __stcs(reinterpret_cast<float4*>(to), make_float4(v[0], v[1 % PER], v[2 % PER], v[3 % PER]));
        }
      }
    }
  }
};

// What a cluster's CTAs tell one another about a row: each writes its value
// into every CTA's place `rank`, in this CTA's shared memory at `to`.
__device__ __forceinline__ void tell_cluster(float4* to, int rank, int cluster, float4 v) {
  if (threadIdx.x < unsigned(cluster))
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(
                     ptx::map_to_rank(ptx::smem_u32(to + rank), threadIdx.x)),
                 "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
  ptx::cluster_sync_all();
}

// The same from warp to warp: warp w of CTA `rank` tells every CTA of the cluster
// its value (the same in all lanes), which one barrier later each has in
// slots[rank][w] of its own shared memory.  Work may lie between begin and end.
template <int WARPS>
__device__ __forceinline__ void tell_cluster_warp(float4* slots, int rank, int cluster, int w, int lane, float4 v) {
  if (lane < cluster)
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(
                     ptx::map_to_rank(ptx::smem_u32(slots + rank * WARPS + w), uint32_t(lane))),
                 "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
}
__device__ __forceinline__ void tell_cluster_begin() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void tell_cluster_end() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Barrier of one team: a warp needs none, the whole CTA has barrier 0.
template <int TEAM, int THREADS>
__device__ __forceinline__ void team_sync(int team) {
  if (TEAM == 32) __syncwarp();
  else if (TEAM == THREADS) __syncthreads();
  else ptx::named_bar_sync(uint32_t(team + 1), TEAM);
}

}  // namespace goldy
