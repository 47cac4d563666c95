// Gradients of the experts' weights, fp32: sums over each expert's rows, in the order of the rows.
// 49,152 rows of 64 experts, 1,536 x 1,024: 1,160 us, 133 of the 155 TFLOP/s of a large matrix product.
// 3,074 rows of 8 experts, 333 x 517 (through registers): 48 us, against 30 for 352 x 512 in whole pieces: loads from odd addresses.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_weight_grad_f32(const ExpertGemm& g, bool big, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = big ? kBig : kSmall;
  const bool p = g.p_token != nullptr, q = g.q_token != nullptr;
  if (p && q) return pick_gemm<float, kOuter, kOuter, kWeightGrad, true, true>(g, size, vec, s);
  if (p) return pick_gemm<float, kOuter, kOuter, kWeightGrad, true, false>(g, size, vec, s);
  if (q) return pick_gemm<float, kOuter, kOuter, kWeightGrad, false, true>(g, size, vec, s);
  return pick_gemm<float, kOuter, kOuter, kWeightGrad>(g, size, vec, s);
}

}  // namespace dol
