// Instantiations of the linear-layer kernel, one translation unit per pass and
// activation (-DGOLDY_LINEAR_PASS=0, 1, 2 -DGOLDY_LINEAR_ACT=0 .. 4; the weight
// gradient has no activation).
#include "linear_kernel.cuh"

#define LIN_CAT_(a, b, c, d) a##b##c##d
#define LIN_CAT(a, b, c, d) LIN_CAT_(a, b, c, d)

namespace goldy {

// out: kLinBf16, kLinF32 or (weight gradient) kLinBf16Long
const void* LIN_CAT(linear_kernel_p, GOLDY_LINEAR_PASS, _a, GOLDY_LINEAR_ACT)(int pair, int out) {
  constexpr int P = GOLDY_LINEAR_PASS, A = GOLDY_LINEAR_ACT;
  if constexpr (P == kLinWeightGrad) {
    if (out == kLinBf16Long)
      return pair ? reinterpret_cast<const void*>(&linear_kernel<P, A, true, false, true>)
                  : reinterpret_cast<const void*>(&linear_kernel<P, A, false, false, true>);
  }
  if (pair)
    return out == kLinF32 ? reinterpret_cast<const void*>(&linear_kernel<P, A, true, true, true>)
                          : reinterpret_cast<const void*>(&linear_kernel<P, A, true, false, false>);
  return out == kLinF32 ? reinterpret_cast<const void*>(&linear_kernel<P, A, false, true, true>)
                        : reinterpret_cast<const void*>(&linear_kernel<P, A, false, false, false>);
}

}  // namespace goldy
