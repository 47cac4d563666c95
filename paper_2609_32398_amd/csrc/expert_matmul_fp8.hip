// Products of rows with their expert's weights, and with the transposed weights, in 8-bit floating point.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_matmul_fp8(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = tile_size<uint8_t>(g);
  if (g.q_token != nullptr)
    return transposed ? pick_gemm<uint8_t, kOuter, kInner, kStore, false, true>(g, size, vec, s)
                      : pick_gemm<uint8_t, kInner, kInner, kStore, false, true>(g, size, vec, s);
  return transposed ? pick_gemm<uint8_t, kOuter, kInner, kStore>(g, size, vec, s)
                    : pick_gemm<uint8_t, kInner, kInner, kStore>(g, size, vec, s);
}

}  // namespace dol
