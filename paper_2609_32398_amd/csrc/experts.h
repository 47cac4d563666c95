// Internal declarations of the experts' operators: the rows that a token's
// choices give, the products of those rows with their expert's weights, the
// gated activation between them, and activations held in 8 bits.
#pragma once

#include "common.h"

namespace dol {

constexpr int kAct8Group = 32;          // elements that share one exponent byte
constexpr int kFp8Block = 128;          // the same of 8-bit floating point (weights: 128 x 128)
constexpr int32_t kMaxWidth = 1 << 16;  // of a row of activations or weights
// Rows of a product: a tile's rows, a stage and a list of 1,024 tokens are added to a row's number in int32.
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1024;

// do_last_error of the calling thread, and the status itself.
do_status set_error(do_status st, const char* msg);

// The check-finite mode's scan of n scores (DO_OK where the mode is off).
do_status check_finite_scores(const void* scores, int64_t n, do_dtype dt, hipStream_t s);

// 512-token units are the work items of the row kernels; at most kRowChunks
// blocks take a contiguous range of them each.
constexpr int64_t kRowChunks = 512;
hipError_t launch_expert_rows(const u64* bits, int64_t N, int32_t E, int32_t k, int32_t* offsets, int32_t* row_token,
                              int32_t* token_row, int32_t* token_expert, uint32_t* counts, hipStream_t s);
hipError_t launch_expert_combine(const void* o, do_dtype dt, const int32_t* token_row, int64_t N, int32_t k, int64_t R,
                                 int32_t H, void* y, hipStream_t s);

hipError_t launch_act8_pack(const void* x, do_dtype dt, int64_t rows, int32_t W, int8_t* q, uint8_t* e, hipStream_t s);
hipError_t launch_act8_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int32_t W, void* x, do_dtype dt,
                              hipStream_t s);

// One product grouped by expert.  The result of a tile is D[p][q] = sum over
// the contraction of P[p] Q[q], p along a row of the output.
struct ExpertGemm {
  const void* P;           // weights [E][..][..], or the tokens' x for weight gradients
  const void* Q;           // activations
  const int32_t* offsets;  // [E + 1] rows of each expert
  const int32_t* p_token;  // nullable: P's (weight gradients) or Q's row r is row token[r] of the operand
  const int32_t* q_token;
  int64_t N;               // rows of a gathered operand
  int64_t R;               // rows
  int32_t E;
  int32_t Pd;              // extent of p: columns of the output (the gated activation: F)
  int32_t Qd;              // weight gradients: extent of q (rows of an expert's gradient)
  int32_t K;               // contraction (weight gradients: the rows of an expert)
  int32_t ldp, ldq;        // elements of a row of P and Q
  int32_t wide;            // rows taken by token span 4 GiB or more
  int32_t accumulate;      // weight gradients: add to what is there
  int32_t vec_out;         // rows of the outputs take 16-byte stores
  int32_t vec_q8;          // rows of the 8-bit values take 8-byte stores (forward) or 16-byte loads
  int32_t p_bf16;          // type of prob
  const void* prob;        // nullable [N][E] routing probabilities
  int8_t* q8;              // [R][2][F] 8-bit gate and up values (written, or read by the backward pass)
  uint8_t* e8;             // [R][2][G] their exponents
  void* out;
  void* out2;              // backward pass: the activations again
  const uint8_t* p_exp;    // 8-bit floating point: the operands' exponents (of the weights', and of the rows' blocks)
  const uint8_t* q_exp;
  uint8_t* h_exp;          // and those of the activations
  float* dp;               // backward pass: partial sums of the probabilities' gradient, [R][ceil(F / 64)]
};

hipError_t launch_expert_matmul_bf16(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s);
hipError_t launch_expert_matmul_f32(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s);
hipError_t launch_expert_weight_grad_bf16(const ExpertGemm& g, bool big, bool vec, hipStream_t s);
hipError_t launch_expert_weight_grad_f32(const ExpertGemm& g, bool big, bool vec, hipStream_t s);
hipError_t launch_expert_swiglu(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s);
// In 8 bits (p_exp, q_exp); offsets may be NULL: one expert with all R rows.
hipError_t launch_expert_matmul_fp8(const ExpertGemm& g, bool transposed, bool vec, hipStream_t s);
hipError_t launch_expert_swiglu_fp8(const ExpertGemm& g, bool vec, hipStream_t s);
hipError_t launch_expert_swiglu_grad_fp8(const ExpertGemm& g, bool vec, hipStream_t s);
// Matrices of weights [mats][O][I] (weights), or rows [mats * O][I], to 8 bits and back.
hipError_t launch_fp8_pack(const void* x, do_dtype dt, int64_t mats, int64_t O, int32_t I, bool weights, uint8_t* q,
                           uint8_t* e, hipStream_t s);
hipError_t launch_fp8_unpack(const uint8_t* q, const uint8_t* e, int64_t mats, int64_t O, int32_t I, bool weights,
                             void* x, do_dtype dt, hipStream_t s);
hipError_t launch_expert_swiglu_grad(const ExpertGemm& g, do_dtype dt, bool vec, hipStream_t s);
// 16 rows an expert or fewer on average.
inline bool few_rows(int64_t R, int32_t E) { return R / E <= 16; }
// Forward products (swiglu: with the gated activation) of whole pieces for few rows per expert.
hipError_t launch_expert_skinny(const ExpertGemm& g, do_dtype dt, bool swiglu, hipStream_t s);
// dp [N][E] (fp32 or bf16) from the partial sums: zero where a token has no row.
hipError_t launch_expert_dp(const float* part, int32_t nparts, int64_t R, const int32_t* token_row,
                            const int32_t* token_expert, int64_t N, int32_t k, int32_t E, void* dp, do_dtype dt,
                            hipStream_t s);

// The layer of a few tokens: a chosen expert, its first row and its tokens (bit t: token t).
struct Chosen {
  int32_t e, first;
  u64 tokens;
};
constexpr int kLayerTokens = 64;
struct LayerArgs {
  const void* x;          // [N][H]
  const void* scores;     // [N][E]
  const void* p;          // nullable [N][E]
  const void* w1;         // [E][2 F][H] and its exponents (8 bits)
  const void* w2;         // [E][H][F]
  const uint8_t* w1_exp;
  const uint8_t* w2_exp;
  void* y;                // [N][H]
  int32_t* n_chosen;      // workspace
  Chosen* chosen;
  int32_t* arrived;       // [ceil(H / 16)]
  float* parts;           // sums of the blocks that share a column tile
  void* h;                // activations, rows by expert
  int32_t N, E, k, H, F;
  int32_t ldh;            // elements of a row of h
  int32_t most;           // experts that can be chosen
  int32_t split;          // blocks that share a column tile of the second kernel
  int32_t scores_bf16, p_bf16;
};
// Rows of the activations are whole 16-byte pieces.
inline int32_t layer_row(do_dtype dt, int32_t F) { return dt == DO_F32 ? (F + 3) & ~3 : (F + 7) & ~7; }
int64_t expert_layer_bytes(do_dtype dt, int64_t N, int32_t E, int32_t k, int32_t H, int32_t F);
hipError_t launch_expert_layer(LayerArgs a, do_dtype dt, void* workspace, hipStream_t s);

// ---- bf16 and 8-bit conversions ---------------------------------------------

__device__ __forceinline__ float bf16_float(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// Two floats to bf16, each rounded to nearest even (NaN stays NaN), a in the low half.
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  v2bf v;
  v[0] = (__bf16)a;
  v[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint16_t bf16_bits(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

// Exponent byte of a group whose largest magnitude has the bit pattern m (sign
// clear): the least e >= -126 with amax <= 127 * 2^e, plus 127; 255 when the
// group holds an infinity or NaN.  127 * 2^e is 1.984375 * 2^(e + 6), whose
// mantissa bits are 0x7E0000.
__device__ __forceinline__ uint32_t act8_exponent(uint32_t m) {
  if (m >= 0x7F800000u) return 255u;
  const int e = (int)(m >> 23) - 6 + ((m & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
  return (uint32_t)(e < 1 ? 1 : e);
}
// 2^-e of an exponent byte; 0 for a group that is not finite, whose values are stored as 0.
__device__ __forceinline__ float act8_inverse(uint32_t byte) {
  return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
}
// 2^e; NaN for byte 255.  Byte 0 does not occur; it reads as 2^-127 would, flushed to 0.
__device__ __forceinline__ float act8_scale(uint32_t byte) {
  return byte == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(byte << 23);
}
// Four values x * 2^-e to the nearest integers, ties to even, one to a byte (x 2^-e
// is exact, or so small that it rounds to 0).  fma(x, 2^-e, 1.5 * 2^23) rounds
// once, at the unit, and its low byte is the integer in two's complement.
__device__ __forceinline__ uint32_t act8_round4(const float* x, float inv, uint32_t byte) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(__builtin_fmaf(x[i], inv, 12582912.0f));
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000C0Cu);
  return byte == 255u ? 0u : lo | hi;
}
// 8-bit floating point (e4m3: 3 bits after the leading one, 448 at most).  Exponent byte of a block whose largest
// magnitude has the bit pattern m: the least e >= -120 with amax <= 448 * 2^e, plus 127; 255 when it holds an infinity
// or NaN.  448 is 1.75 * 2^8, whose mantissa bits are 0x600000.  -120 leaves 2^-9 2^e, the least step, to fp32's range
// on both sides (2^-e is used too).
__device__ __forceinline__ uint32_t fp8_exponent(uint32_t m) {
  if (m >= 0x7F800000u) return 255u;
  const int e = (int)(m >> 23) - 8 + ((m & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)(e < 7 ? 7 : e);
}
__device__ __forceinline__ float fp8_inverse(uint32_t byte) { return act8_inverse(byte); }
__device__ __forceinline__ float fp8_scale(uint32_t byte) { return act8_scale(byte); }
// Four values within 448, each rounded once to e4m3 (nearest, ties to even), one to a byte; 0 in a block that is not
// finite.
__device__ __forceinline__ uint32_t fp8_round4(float a, float b, float c, float d, uint32_t byte) {
  int v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  return byte == 255u ? 0u : (uint32_t)v;
}

// Four 8-bit values times s = 2^e, exactly.
__device__ __forceinline__ void act8_values4(uint32_t q, float s, float* v) {
  const uint32_t u = q ^ 0x80808080u;  // + 128: unsigned bytes convert in one instruction
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ((float)((u >> (8 * i)) & 255u) - 128.0f) * s;
}

}  // namespace dol
