// The experts' first product with the gated activation, and its backward pass.
// 524,288 rows of 128 experts, 2,048 -> 2 x 768 bf16: forward with the 8-bit checkpoint 3,300 to 3,380 us (980 to
// 1,000 TFLOP/s; 9 GB come from behind the L2 caches, where rows and weights are 2.9), backward 2,490 us (660): half of the forward's products, and 3.2 GB of 8-bit values in and
// gradients out at the tiles' ends, where the matrix cores wait.
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
