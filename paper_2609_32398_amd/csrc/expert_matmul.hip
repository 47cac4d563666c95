// Products of rows with their expert's weights, and with the transposed weights.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

// Large tiles where an expert has rows for them on average, small ones else.
static bool big_tiles(const ExpertGemm& g) { return g.R / g.E >= 128; }

hipError_t launch_expert_matmul(const ExpertGemm& g, do_dtype dt, bool transposed, bool vec, hipStream_t s) {
  using namespace expert;
  const bool big = big_tiles(g);
  if (dt == DO_F32)
    return transposed ? pick_gemm<float, kOuter, kInner, kStore>(g, big, vec, s)
                      : pick_gemm<float, kInner, kInner, kStore>(g, big, vec, s);
  return transposed ? pick_gemm<uint16_t, kOuter, kInner, kStore>(g, big, vec, s)
                    : pick_gemm<uint16_t, kInner, kInner, kStore>(g, big, vec, s);
}

}  // namespace dol
