// Products of rows with their expert's weights, and with the transposed weights, in 8-bit floating point.
//
// 524,288 rows of 128 experts, 768 -> 2,048: 1,010 us, 1,630 TFLOP/s (the library on one product of this width:
// 1,660).  8,191 rows 2,048 -> 4,096: 64 us, 2,160 TFLOP/s (the library at 8,192^3: 2,650).  49,146 rows of 48
// experts, 1,536 -> 1,024 transposed: 98 us, 1,580 TFLOP/s, of which a fifth is the last round of its 864 tiles.  64
// tokens of 8 of 128 experts, 768 -> 2,048: 40 us, the weights at 5.0 TB/s.  524,288 rows taken from 65,536 tokens,
// 768 -> 2,048: 931 us where rows of their own take 989, since the 50 MB of tokens stay in the caches.  One matrix,
// 8,191 rows 4,096 -> 2,048 transposed: 61 us, 32,768 rows 224 us, 2,450 TFLOP/s (2,048 -> 4,096: 245).  Bound by the
// operands' way to LDS (a stage of 64 KiB and its products take 3,500 cycles, the products alone 2,048) and, at 768,
// by 5,300 cycles of outputs a tile.  Rows that go through registers (odd widths) spill 20 to 29 registers in the 256
// x 256 tiles, the transposed one with rows by token 6; 65,536 rows 1,003 -> 1,501: 331 us, 1,008 -> 1,504: 156.
#include <algorithm>

#include "expert_gemm.h"

namespace dol {

// By rows an expert on average as in bf16.  8 of 64 experts a token, 768 -> 2,048 and transposed 2,048 -> 768, 256 x 256
// tiles against 128 x 64: 96 rows 28 and 29 against 26 and 22 us, 128 rows 29 and 30 against 33 and 32, 256 rows 45 and
// 55 against 50 and 50, 512 rows 72 and 72 against 88 and 103; 128 x 32 against 128 x 64: 4 rows 18.9 and 18.4 against
// 19.2 and 19.0, 16 rows 19.3 and 19.3 against 19.7 and 19.9, 32 rows 21.5 and 21.9 against 20.4 and 20.3.
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
