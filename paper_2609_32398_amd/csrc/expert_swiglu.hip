// The experts' first product with the gated activation, and its backward pass.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_swiglu(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s) {
  using namespace expert;
  if (dt == DO_F32) return pick_gemm<float, kInner, kInner, kSwiglu, false, true>(g, tile_size<float>(g), vec, s);
  return pick_gemm<uint16_t, kInner, kInner, kSwiglu, false, true>(g, tile_size<uint16_t>(g), vec, s);
}

hipError_t launch_expert_swiglu_grad(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s) {
  using namespace expert;
  if (dt == DO_F32) return pick_gemm<float, kOuter, kInner, kSwigluGrad, false, true>(g, tile_size<float>(g), vec, s);
  return pick_gemm<uint16_t, kOuter, kInner, kSwigluGrad, false, true>(g, tile_size<uint16_t>(g), vec, s);
}

}  // namespace dol
