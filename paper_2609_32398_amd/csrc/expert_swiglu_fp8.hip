// The experts' first product with the gated activation, and its backward pass, in 8-bit floating point.
//
// 524,288 rows of 128 experts, 2,048 -> 2 x 768: forward with the 8-bit checkpoint 1,700 to 1,800 us (1,830 to 1,940
// TFLOP/s; the bf16 kernel 3,300; a large library product of this shape runs at 2,510), matrix cores busy 43 %: a
// stage's 64 KiB take 1,600 of its 3,500 cycles on their way to LDS (40 bytes a cycle: what the vector cache holds on
// its way over the L2's latency), in which half of the waves multiply, and the others after them.  Backward 1,690 us:
// half of the products, and 3.6 GB of 8-bit values in and gradients out (740 us at the rate of a copy), with 33 vector
// instructions an activation.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

// The 32-row tile up to 112 rows an expert on average, since one with 64 rows of 256 fills a CU's LDS by itself: 8 of
// 64 experts a token, 2,048 -> 2 x 768, 32 rows against 256: 64 rows an expert 57 against 73 us (the 64-row tile 75),
// 96 rows 71 against 75 (73), 128 rows 89 against 77 (92), 256 rows 143 against 116 (144).  Rows that go through
// registers take the 64-row tile instead, whose loads are on their way together (their 256-row tile spills 14
// registers). However many rows an expert has, the large tiles also have to be 3/8 of the CUs, as fills() counts them,
// since one takes 27 us whether others run or not.  32 rows against 256 at 2,048 in the contraction, by large tiles
// over all experts: 1 to 48 of them 13 to 18 against 27 to 28 us, 64 (8 experts of 2,048 rows, 2 x 128) 31 against 29,
// 96 (one of 4,096, 2 x 768) 30 against 28, 128 (8 of 2,048, 2 x 256) 44 against 30, 192 58 against 33; 64 that are
// half empty (64 experts of 128 rows, 2 x 128) 18 against 29.
hipError_t launch_expert_swiglu_fp8(const ExpertGemm& g, bool vec, hipStream_t s) {
  using namespace expert;
  const int size = g.R / g.E >= 112 && fills<128>(g) ? kBig : vec ? kFew : kSmall;
  return pick_gemm<uint8_t, kInner, kInner, kSwiglu, false, true>(g, size, vec, s);
}

// 8 of 64 experts a token, 2,048 and 768 wide, 128 x 128 tiles against 128 x 64: 48 rows an expert 34 against 31 us, 64
// rows 35 against 46, 96 rows 36 against 44, 128 rows 54 against 49, 192 rows 60 against 68, 512 rows 127 against 161.
// 128 x 32 is not ahead below that: 4 rows 27.4 against 26.8, 16 rows 29.3 against 28.6.
hipError_t launch_expert_swiglu_grad_fp8(const ExpertGemm& g, bool vec, hipStream_t s) {
  using namespace expert;
  return pick_gemm<uint8_t, kOuter, kInner, kSwigluGrad, false, true>(g, g.R / g.E >= 64 ? kBig : kSmall, vec, s);
}

}  // namespace dol
