// Products of rows with their expert's weights, and with the transposed weights, fp32.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_matmul_f32(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = tile_size<float>(g);
  if (g.q_token != nullptr)
    return transposed ? pick_gemm<float, kOuter, kInner, kStore, false, true>(g, size, vec, s)
                      : pick_gemm<float, kInner, kInner, kStore, false, true>(g, size, vec, s);
  return transposed ? pick_gemm<float, kOuter, kInner, kStore>(g, size, vec, s)
                    : pick_gemm<float, kInner, kInner, kStore>(g, size, vec, s);
}

}  // namespace dol
