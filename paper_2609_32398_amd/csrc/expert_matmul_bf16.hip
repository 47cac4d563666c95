// Products of rows with their expert's weights, and with the transposed weights, bf16.
// 524,288 rows of 128 experts, 768 -> 2,048: 1,660 to 1,700 us, 970 to 990 TFLOP/s; transposed, 1,536 -> 2,048:
// 3,140 us, 1,050 TFLOP/s.  Bound by the operands' way to LDS.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

hipError_t launch_expert_matmul_bf16(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = tile_size<uint16_t>(g);
  if (g.q_token != nullptr)
    return transposed ? pick_gemm<uint16_t, kOuter, kInner, kStore, false, true>(g, size, vec, s)
                      : pick_gemm<uint16_t, kInner, kInner, kStore, false, true>(g, size, vec, s);
  return transposed ? pick_gemm<uint16_t, kOuter, kInner, kStore>(g, size, vec, s)
                    : pick_gemm<uint16_t, kInner, kInner, kStore>(g, size, vec, s);
}

}  // namespace dol
