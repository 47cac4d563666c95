// The experts' first product with the gated activation, and its backward pass, in 8-bit floating point.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_swiglu_fp8(const ExpertGemm& g, bool vec, hipStream_t s) {
  using namespace expert;
  return pick_gemm<uint8_t, kInner, kInner, kSwiglu, false, true>(g, tile_size<uint8_t>(g), vec, s);
}

hipError_t launch_expert_swiglu_grad_fp8(const ExpertGemm& g, bool vec, hipStream_t s) {
  using namespace expert;
  return pick_gemm<uint8_t, kOuter, kInner, kSwigluGrad, false, true>(g, tile_size<uint8_t>(g), vec, s);
}

}  // namespace dol
