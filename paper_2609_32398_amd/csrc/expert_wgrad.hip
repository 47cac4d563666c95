// Gradients of the experts' weights: sums over each expert's rows.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_weight_grad(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s) {
  using namespace expert;
  const bool big = g.Pd > 128 && g.Qd > 64 && (int64_t)g.E * g.Pd * g.Qd >= int64_t(256) * 65536;
  if (dt == DO_F32) return pick_gemm<float, kOuter, kOuter, kWeightGrad>(g, big, vec, s);
  return pick_gemm<uint16_t, kOuter, kOuter, kWeightGrad>(g, big, vec, s);
}

}  // namespace dol
