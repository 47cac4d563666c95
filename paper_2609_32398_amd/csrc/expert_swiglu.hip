// The experts' first product with the gated activation, and its backward pass.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

// Large tiles where an expert has rows for them on average, small ones else.
static bool big_tiles(const ExpertGemm& g) { return g.R / g.E >= 128; }

hipError_t launch_expert_swiglu(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s) {
  using namespace expert;
  if (dt == DO_F32) return pick_gemm<float, kInner, kInner, kSwiglu>(g, big_tiles(g), vec, s);
  return pick_gemm<uint16_t, kInner, kInner, kSwiglu>(g, big_tiles(g), vec, s);
}

hipError_t launch_expert_swiglu_grad(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s) {
  using namespace expert;
  if (dt == DO_F32) return pick_gemm<float, kOuter, kInner, kSwigluGrad>(g, big_tiles(g), vec, s);
  return pick_gemm<uint16_t, kOuter, kInner, kSwigluGrad>(g, big_tiles(g), vec, s);
}

}  // namespace dol
