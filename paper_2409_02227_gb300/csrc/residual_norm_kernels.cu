// The residual norms' kernels of one type (GOLDY_NORM_F32), direction
// (GOLDY_NORM_BACKWARD) and way rows lie (GOLDY_NORM_MODE), behind the function
// GOLDY_NORM_KERNEL.
#include "residual_norm_kernel.cuh"

namespace goldy {
namespace {

#if GOLDY_NORM_F32
using T = float;
#else
using T = uint16_t;
#endif

template <int TEAM, RowMode MODE, bool WIDE = false>
NormKernel pick(bool full) {
#if GOLDY_NORM_BACKWARD
  constexpr bool ALL = MODE != kAnyRows;           // rows that lie anyhow have one kernel for all cases
  constexpr int THREADS = bwd_threads(TEAM);
  using R = NormRow<T, kBwdVals, TEAM, THREADS, MODE != kAnyRows, WIDE, MODE == kFramedRows>;
  return {full ? reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, MODE, WIDE, ALL>)
               : reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, MODE, WIDE, false>),
          THREADS, THREADS / TEAM, 1,
          std::max(size_t(4) * norm_depth<T>() * R::RING_BYTES, size_t(kSums) * THREADS * kBwdVals * sizeof(float))};
#else
  constexpr int THREADS = fwd_threads(TEAM);
  using R = NormRow<T, kFwdVals, TEAM, THREADS, MODE != kAnyRows, WIDE, MODE == kFramedRows>;
  return {reinterpret_cast<const void*>(&residual_norm_forward_kernel<T, TEAM, MODE, WIDE>), THREADS, THREADS / TEAM,
          512 / THREADS, size_t(2) * (WIDE ? norm_depth<T>() : kFwdDepth) * R::RING_BYTES};
#endif
}

template <RowMode MODE>
NormKernel pick_team(const ResidualNormShape& s, bool full) {
  if constexpr (MODE != kAnyRows) {                // in between the powers of two
    switch (s.team) {
      case 96: return pick<96, MODE>(full);
      case 160: return pick<160, MODE>(full);
      case 192: return pick<192, MODE>(full);
#if GOLDY_NORM_BACKWARD
      case 224: return pick<224, MODE>(full);
#endif
      default: break;
    }
  }
  switch (s.team) {
    case 32: return pick<32, MODE>(full);
    case 64: return pick<64, MODE>(full);
    case 128: return pick<128, MODE>(full);
    case 256: return pick<256, MODE>(full);
    default: return pick<512, MODE>(full);
  }
}
template <RowMode MODE>
NormKernel pick_shape(const ResidualNormShape& s, bool full) {
  return s.cluster > 1 ? pick<kMaxTeam, MODE, true>(full) : pick_team<MODE>(s, full);
}

}  // namespace

NormKernel GOLDY_NORM_KERNEL(const ResidualNormShape& s, bool full) { return pick_shape<GOLDY_NORM_MODE>(s, full); }

}  // namespace goldy
