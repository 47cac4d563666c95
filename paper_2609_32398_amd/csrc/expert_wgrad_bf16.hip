// Gradients of the experts' weights, bf16: sums over each expert's rows.  A block sums a tile over all
// rows of its expert in fp32, so that nothing is added up by atomics and the order is fixed.
// 524,288 rows of 128 experts, 1,536 x 2,048, one side by token: 3,460 to 3,640 us, 910 to 950 TFLOP/s; added to
// what dW holds, which is read along columns, 700 us more.  The tiles of an
// expert that run at one time read the same rows; what the L2 caches miss of that, 9 GB where 4 would
// do, and the operands' way to LDS bound it.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_weight_grad_bf16(const ExpertGemm& g, bool big, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = big ? kBig : kSmall;
  const bool p = g.p_token != nullptr, q = g.q_token != nullptr;
  if (p && q) return pick_gemm<uint16_t, kOuter, kOuter, kWeightGrad, true, true>(g, size, vec, s);
  if (p) return pick_gemm<uint16_t, kOuter, kOuter, kWeightGrad, true, false>(g, size, vec, s);
  if (q) return pick_gemm<uint16_t, kOuter, kOuter, kWeightGrad, false, true>(g, size, vec, s);
  return pick_gemm<uint16_t, kOuter, kOuter, kWeightGrad>(g, size, vec, s);
}

}  // namespace dol
