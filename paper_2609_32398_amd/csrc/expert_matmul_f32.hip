// Products of rows with their expert's weights, and with the transposed weights, fp32.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_matmul_f32(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s) {
  using namespace expert;
  const bool big = big_tiles<float>(g);
  if (g.q_token != nullptr)
    return transposed ? pick_gemm<float, kOuter, kInner, kStore, false, true>(g, big, vec, s)
                      : pick_gemm<float, kInner, kInner, kStore, false, true>(g, big, vec, s);
  return transposed ? pick_gemm<float, kOuter, kInner, kStore>(g, big, vec, s)
                    : pick_gemm<float, kInner, kInner, kStore>(g, big, vec, s);
}

}  // namespace dol
