// The residual norms' kernels of one type (GOLDY_NORM_F32) and direction
// (GOLDY_NORM_BACKWARD).
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
  using R = NormRow<T, kBwdVals, TEAM, kBwdThreads, MODE != kAnyRows, WIDE, MODE == kFramedRows>;
  return {full ? reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, MODE, WIDE, ALL>)
               : reinterpret_cast<const void*>(&residual_norm_backward_kernel<T, TEAM, MODE, WIDE, false>),
          kBwdThreads, kBwdThreads / TEAM, 1,
          std::max(size_t(4) * bwd_depth<T>() * R::RING_BYTES, size_t(kSums) * kBwdThreads * kBwdVals * sizeof(float))};
#else
  constexpr int THREADS = TEAM > kFwdThreads ? TEAM : kFwdThreads;
  using R = NormRow<T, kFwdVals, TEAM, THREADS, MODE != kAnyRows, WIDE, MODE == kFramedRows>;
  return {reinterpret_cast<const void*>(&residual_norm_forward_kernel<T, TEAM, MODE, WIDE>), THREADS, THREADS / TEAM,
          TEAM > kFwdThreads ? 1 : 2, size_t(2) * kFwdDepth * R::RING_BYTES};
#endif
}

template <RowMode MODE>
NormKernel pick_team(const ResidualNormShape& s, bool full) {
  switch (s.team) {
    case 32: return pick<32, MODE>(full);
    case 64: return pick<64, MODE>(full);
    case 128: return pick<128, MODE>(full);
    case 256: return pick<256, MODE>(full);
    default: return pick<512, MODE>(full);
  }
}
NormKernel pick_shape(const ResidualNormShape& s, RowMode mode, bool full) {
  if (s.cluster > 1) return mode == kWholeRows ? pick<kMaxTeam, kWholeRows, true>(full) : pick<kMaxTeam, kAnyRows, true>(full);
  switch (mode) {
    case kWholeRows: return pick_team<kWholeRows>(s, full);
    case kFramedRows: return pick_team<kFramedRows>(s, full);
    default: return pick_team<kAnyRows>(s, full);
  }
}

}  // namespace

#if GOLDY_NORM_BACKWARD
#if GOLDY_NORM_F32
NormKernel residual_norm_backward_f32(const ResidualNormShape& s, RowMode mode, bool full) {
#else
NormKernel residual_norm_backward_bf16(const ResidualNormShape& s, RowMode mode, bool full) {
#endif
  return pick_shape(s, mode, full);
}
#else
#if GOLDY_NORM_F32
NormKernel residual_norm_forward_f32(const ResidualNormShape& s, RowMode mode) {
#else
NormKernel residual_norm_forward_bf16(const ResidualNormShape& s, RowMode mode) {
#endif
  return pick_shape(s, mode, false);
}
#endif

}  // namespace goldy
