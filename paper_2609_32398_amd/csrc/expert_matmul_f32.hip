// Products of rows with their expert's weights, and with the transposed weights, fp32.
// 49,146 rows of 48 experts, 1,536 -> 1,024 transposed: 1,260 us, 123 of the 155 TFLOP/s of a large
// matrix product.
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
