// Instantiations of the linear-layer kernel, one translation unit per pass
// (-DGOLDY_LINEAR_PASS=0, 1, 2).
#include "linear_kernel.cuh"

namespace goldy {

template <int PASS>
static const void* pick(int pair, int out_f32) {
  if (pair)
    return out_f32 ? reinterpret_cast<const void*>(&linear_kernel<PASS, true, true>)
                   : reinterpret_cast<const void*>(&linear_kernel<PASS, true, false>);
  return out_f32 ? reinterpret_cast<const void*>(&linear_kernel<PASS, false, true>)
                 : reinterpret_cast<const void*>(&linear_kernel<PASS, false, false>);
}

#if GOLDY_LINEAR_PASS == 0
const void* linear_kernel_forward(int pair, int out_f32) { return pick<kLinForward>(pair, out_f32); }
#elif GOLDY_LINEAR_PASS == 1
const void* linear_kernel_input_grad(int pair, int out_f32) { return pick<kLinInputGrad>(pair, out_f32); }
#else
const void* linear_kernel_weight_grad(int pair, int out_f32) { return pick<kLinWeightGrad>(pair, out_f32); }
#endif

}  // namespace goldy
