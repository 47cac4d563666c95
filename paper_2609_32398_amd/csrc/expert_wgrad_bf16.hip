// Gradients of the experts' weights, bf16: sums over each expert's rows.
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
