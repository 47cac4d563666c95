// Host side of the experts' entry points declared in include/doloss.h:
// argument validation and dispatch to the kernels.
#include <algorithm>
#include <initializer_list>

#include "experts.h"

#define DOLOSS_API extern "C" __attribute__((visibility("default")))

using dol::set_error;
using dol::u64;

namespace {

#define DO_TRY(expr)              \
  do {                            \
    const do_status st_ = (expr); \
    if (st_ != DO_OK) return st_; \
  } while (0)

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

do_status launched(hipError_t e) { return e == hipSuccess ? DO_OK : set_error(DO_ERR_HIP, hipGetErrorString(e)); }

do_status check_dtype(int dt) {
  if (dt != DO_F32 && dt != DO_BF16) return set_error(DO_ERR_UNSUPPORTED_DTYPE, "dtype must be DO_F32 or DO_BF16");
  return DO_OK;
}
size_t size_of(do_dtype dt) { return dt == DO_F32 ? 4 : 2; }

do_status check_ptr(const void* p, size_t align, const char* msg) {
  return p == nullptr || !aligned(p, align) ? set_error(DO_ERR_INVALID_ARG, msg) : DO_OK;
}

do_status check_experts(int64_t N, int32_t E, int32_t k) {
  if (E < 1 || E > dol::kMaxE) return set_error(DO_ERR_INVALID_ARG, "E must be in [1, 1024]");
  if (k < 1 || k > E) return set_error(DO_ERR_INVALID_ARG, "k must be in [1, E]");
  if (N < 1) return set_error(DO_ERR_INVALID_ARG, "N must be >= 1");
  if (N >= (int64_t(1) << 31) || N * k >= (int64_t(1) << 31))
    return set_error(DO_ERR_OVERFLOW, "N * k must be < 2^31 (rows are int32)");
  return DO_OK;
}
// most: rows of the products (dol::kMaxRows), or whatever int32 holds.
do_status check_rows(int64_t N, int64_t R, int32_t E, int64_t most = dol::kMaxRows) {
  if (E < 1 || E > dol::kMaxE) return set_error(DO_ERR_INVALID_ARG, "E must be in [1, 1024]");
  if (N < 1 || R < 1) return set_error(DO_ERR_INVALID_ARG, "N and R must be >= 1");
  if (N >= (int64_t(1) << 31) || R > most)
    return set_error(DO_ERR_OVERFLOW, "N must be < 2^31 and R at most 2^31 - 1024 (rows are int32)");
  return DO_OK;
}
do_status check_widths(int64_t R, int32_t E, std::initializer_list<int32_t> w) {
  int64_t tiles = 1;
  for (int32_t v : w) {
    if (v < 1 || v > dol::kMaxWidth) return set_error(DO_ERR_INVALID_ARG, "widths must be in [1, 65536]");
    tiles = std::max<int64_t>(tiles, (v + 63) / 64);
  }
  // the tile list of a product is counted in int32
  if ((R / 128 + E) * tiles >= (int64_t(1) << 31))
    return set_error(DO_ERR_OVERFLOW, "too many rows for rows of this width");
  return DO_OK;
}

// An operand of whole 16-byte pieces: its address and the length of its rows, and fewer than 2^32 pieces.
bool whole(const void* p, do_dtype dt, int32_t row, int64_t rows = 1) {
  return aligned(p, 16) && row * size_of(dt) % 16 == 0 && rows * (int64_t)(row * size_of(dt) / 16) < (int64_t(1) << 32);
}

// The same for weights whose rows are read along: one expert's byte offsets fit 32 bits too.
bool whole_expert(const void* w, do_dtype dt, int32_t row, int64_t rows) {
  return whole(w, dt, row) && rows * row * (int64_t)size_of(dt) < (int64_t(1) << 32);
}

// Whether there are few rows, and the experts that can have them are so few that their tiles of `cols`
// weight rows leave CUs idle, or, in fp32, whose matrix instructions take 16 times as long, fill them less
// than twice: then a tile's time counts, and it is shorter with a quarter of the contraction for each wave.
// Against the tiles that share LDS, 8 of 128 experts a token, 768 -> 2,048 and gated 2,048 -> 2 x 768, calls in
// a graph whose weights come from memory: bf16, 1 token 10.2 and 18.4 us against 13.8 and 31.8, 2 tokens (at the
// rule's edge) 16.3 and 29.9 against 15.8 and 34.7, 4 tokens (outside) 26.0 and 43.7 against 19.3 and 40.0;
// fp32, 1 token 18.7 and 35.1 against 34.4 and 83.7, 4 tokens (the edge) 49.6 and 84.0 against 57.4 and 139,
// 16 tokens (outside) 123 and 222 against 114 and 227.  Few experts keep within the rule up to 16 rows each on
// average, where some then have two tiles of 16 rows: 2 of 8 experts, 1,536 -> 4,096 and gated 2,048 -> 2 x 1,792,
// 64 tokens, bf16 38.1 and 42.6 us against 27.0 and 36.7 and fp32 74.6 and 84.9 against 64.2 and 84.6; 32 tokens
// 29.5 and 30.8 against 27.0 and 36.4 and 54.9 and 59.3 against 64.0 and 84.1.
bool few_tiles(do_dtype dt, int64_t R, int32_t E, int32_t width, int cols) {
  const int64_t tiles = std::min<int64_t>(R, E) * ((width + cols - 1) / cols);
  return dol::few_rows(R, E) && tiles <= (dt == DO_F32 ? 2 : 1) * dol::device_info().cu_count;
}

// Rows taken by token whose byte offsets pass 32 bits.
int32_t wide(do_dtype dt, int32_t row, int64_t rows) { return rows * row * (int64_t)size_of(dt) >= (int64_t(1) << 32); }

}  // namespace

DOLOSS_API int64_t do_expert_rows_workspace(int64_t N, int32_t E) {
  if (N < 1 || E < 1 || E > dol::kMaxE) return 0;
  const int64_t U = (N - 1) / 512 + 1;
  return U == 1 ? 0 : std::min<int64_t>(U, dol::kRowChunks) * E * (int64_t)sizeof(uint32_t);
}

DOLOSS_API do_status do_expert_rows(const uint64_t* bits, int64_t N, int32_t E, int32_t k, int32_t* offsets,
                                    int32_t* row_token, int32_t* token_row, int32_t* token_expert, void* workspace,
                                    int64_t workspace_bytes, hipStream_t stream) {
  DO_TRY(check_experts(N, E, k));
  DO_TRY(check_ptr(bits, 8, "bits is NULL or not 8-byte aligned"));
  DO_TRY(check_ptr(offsets, 4, "offsets is NULL or not 4-byte aligned"));
  DO_TRY(check_ptr(row_token, 4, "row_token is NULL or not 4-byte aligned"));
  DO_TRY(check_ptr(token_row, 4, "token_row is NULL or not 4-byte aligned"));
  DO_TRY(check_ptr(token_expert, 4, "token_expert is NULL or not 4-byte aligned"));
  const int64_t need = do_expert_rows_workspace(N, E);
  if (need > 0) {
    DO_TRY(check_ptr(workspace, 4, "workspace is NULL or not 4-byte aligned"));
    if (workspace_bytes < need)
      return set_error(DO_ERR_INVALID_ARG, "workspace is smaller than do_expert_rows_workspace(N, E)");
  }
  return launched(dol::launch_expert_rows(reinterpret_cast<const u64*>(bits), N, E, k, offsets, row_token, token_row,
                                          token_expert, static_cast<uint32_t*>(workspace), stream));
}

DOLOSS_API do_status do_expert_combine(const void* o, do_dtype dtype, const int32_t* token_row, int64_t N, int32_t k,
                                       int32_t H, void* y, hipStream_t stream) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_experts(N, dol::kMaxE, k));
  DO_TRY(check_widths(N, 1, {H}));
  DO_TRY(check_ptr(o, size_of(dtype), "o is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(token_row, 4, "token_row is NULL or not 4-byte aligned"));
  DO_TRY(check_ptr(y, size_of(dtype), "y is NULL or not aligned to its element size"));
  return launched(dol::launch_expert_combine(o, dtype, token_row, N, k, N * k, H, y, stream));
}

DOLOSS_API do_status do_expert_matmul(const void* x, const void* w, do_dtype dtype, const int32_t* offsets,
                                      const int32_t* row_token, int64_t N, int64_t R, int32_t E, int32_t O, int32_t I,
                                      int32_t transposed, void* y, hipStream_t stream) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_rows(N, R, E));
  DO_TRY(check_widths(R, E, {O, I}));
  DO_TRY(check_ptr(x, size_of(dtype), "x is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(w, size_of(dtype), "w is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(y, size_of(dtype), "y is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(offsets, 4, "offsets is NULL or not 4-byte aligned"));
  if (row_token != nullptr && !aligned(row_token, 4))
    return set_error(DO_ERR_INVALID_ARG, "row_token is not 4-byte aligned");
  const int32_t in = transposed ? O : I, out = transposed ? I : O;
  dol::ExpertGemm g{};
  g.P = w;
  g.Q = x;
  g.offsets = offsets;
  g.q_token = row_token;
  g.N = N;
  g.R = R;
  g.E = E;
  g.Pd = out;
  g.K = in;
  g.ldp = I;
  g.ldq = in;
  g.out = y;
  g.wide = row_token != nullptr && wide(dtype, in, N);
  g.vec_out = whole(y, dtype, out);
  const bool vec = (transposed ? whole(w, dtype, I) : whole_expert(w, dtype, I, O)) &&
                   whole(x, dtype, in, row_token != nullptr ? N : R);
  if (vec && !transposed && few_tiles(dtype, R, E, O, 128)) return launched(dol::launch_expert_skinny(g, dtype, false, stream));
  return launched((dtype == DO_F32 ? dol::launch_expert_matmul_f32 : dol::launch_expert_matmul_bf16)(
      g, transposed != 0, vec, stream));
}

DOLOSS_API do_status do_expert_weight_grad(const void* dy, const void* x, do_dtype dtype, const int32_t* offsets,
                                           const int32_t* dy_token, const int32_t* x_token, int64_t N, int64_t R,
                                           int32_t E, int32_t O, int32_t I, int32_t accumulate, float* dw,
                                           hipStream_t stream) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_rows(N, R, E));
  DO_TRY(check_widths(1, E, {O, I}));
  DO_TRY(check_ptr(dy, size_of(dtype), "dy is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(x, size_of(dtype), "x is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(dw, 4, "dw is NULL or not 4-byte aligned"));
  DO_TRY(check_ptr(offsets, 4, "offsets is NULL or not 4-byte aligned"));
  if ((dy_token != nullptr && !aligned(dy_token, 4)) || (x_token != nullptr && !aligned(x_token, 4)))
    return set_error(DO_ERR_INVALID_ARG, "dy_token / x_token is not 4-byte aligned");
  if ((int64_t)E * ((O + 63) / 64) * ((I + 63) / 64) >= (int64_t(1) << 31))
    return set_error(DO_ERR_OVERFLOW, "too many weights");
  dol::ExpertGemm g{};
  g.P = x;
  g.Q = dy;
  g.offsets = offsets;
  g.p_token = x_token;
  g.q_token = dy_token;
  g.N = N;
  g.R = R;
  g.E = E;
  g.Pd = I;
  g.Qd = O;
  g.ldp = I;
  g.ldq = O;
  g.accumulate = accumulate != 0;
  g.out = dw;
  g.wide = wide(dtype, std::max(O, I), N);
  g.vec_out = whole(dw, DO_F32, I);
  // Large tiles where there are enough of them for every CU and they are wider than a small one both ways.
  // Large against small: 64 experts of 1,536 x 1,024, 768 rows each, bf16 224 against 404 us and fp32 1,159
  // against 1,465; 16 of 1,024 x 1,024, 2,048 rows (just within the rule) 79 against 132 and 511 against 634;
  // 8 of them (outside) 112 against 124 and 973 against 621; 32 of 64 x 2,048, 8,192 rows (outside) 261
  // against 165 and 1,955 against 641.  Few rows do not change that: 128 of 1,536 x 2,048, whose 1.6 GB of
  // gradients bound it, 8 rows each 283 against 319 and 355 against 461, 128 rows 311 against 458 and 1,130
  // against 1,463; 16 of 1,024 x 1,024, one row each 17 against 20 and 23 against 26.
  const bool big = I > 128 && O > 64 && (int64_t)E * I * O >= int64_t(256) * 65536;
  return launched((dtype == DO_F32 ? dol::launch_expert_weight_grad_f32 : dol::launch_expert_weight_grad_bf16)(
      g, big, whole(x, dtype, I, std::max(N, R)) && whole(dy, dtype, O, std::max(N, R)), stream));
}

namespace {

// What do_expert_swiglu and do_expert_swiglu_grad check alike.
do_status check_swiglu(do_dtype dtype, const void* p, do_dtype p_dtype, const int32_t* offsets,
                       const int32_t* row_token, int64_t N, int64_t R, int32_t E, int32_t H, int32_t F) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_rows(N, R, E));
  DO_TRY(check_widths(R, E, {H, F}));
  if (p != nullptr) {
    DO_TRY(check_dtype(p_dtype));
    if (!aligned(p, size_of(p_dtype))) return set_error(DO_ERR_INVALID_ARG, "p is not aligned to its element size");
  }
  DO_TRY(check_ptr(offsets, 4, "offsets is NULL or not 4-byte aligned"));
  return check_ptr(row_token, 4, "row_token is NULL or not 4-byte aligned");
}

}  // namespace

DOLOSS_API do_status do_expert_swiglu(const void* x, const void* w1, do_dtype dtype, const void* p, do_dtype p_dtype,
                                      const int32_t* offsets, const int32_t* row_token, int64_t N, int64_t R,
                                      int32_t E, int32_t H, int32_t F, void* h, int8_t* q, uint8_t* e,
                                      hipStream_t stream) {
  DO_TRY(check_swiglu(dtype, p, p_dtype, offsets, row_token, N, R, E, H, F));
  DO_TRY(check_ptr(x, size_of(dtype), "x is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(w1, size_of(dtype), "w1 is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(h, size_of(dtype), "h is NULL or not aligned to its element size"));
  if ((q == nullptr) != (e == nullptr)) return set_error(DO_ERR_INVALID_ARG, "q and e are given together or not at all");
  dol::ExpertGemm g{};
  g.P = w1;
  g.Q = x;
  g.offsets = offsets;
  g.q_token = row_token;
  g.N = N;
  g.R = R;
  g.E = E;
  g.Pd = F;
  g.K = H;
  g.ldp = H;
  g.ldq = H;
  g.wide = wide(dtype, H, N);
  g.prob = p;
  g.p_bf16 = p_dtype == DO_BF16;
  g.q8 = q;
  g.e8 = e;
  g.out = h;
  g.vec_out = aligned(h, 16) && F % 8 == 0;
  g.vec_q8 = q != nullptr && aligned(q, 8) && F % 8 == 0;
  const bool vec = whole(x, dtype, H, N) && whole_expert(w1, dtype, H, 2 * (int64_t)F);
  if (vec && few_tiles(dtype, R, E, F, 64)) return launched(dol::launch_expert_skinny(g, dtype, true, stream));
  return launched(dol::launch_expert_swiglu(g, dtype, vec, stream));
}

DOLOSS_API int64_t do_expert_swiglu_grad_workspace(int64_t R, int32_t F) {
  return R < 1 || F < 1 ? 0 : R * ((F + 63) / 64) * (int64_t)sizeof(float);
}

DOLOSS_API do_status do_expert_swiglu_grad(const void* dy, const void* w2, do_dtype dtype, const void* p,
                                           do_dtype p_dtype, const int32_t* offsets, const int32_t* row_token,
                                           const int32_t* token_row, const int32_t* token_expert, int64_t N, int32_t E,
                                           int32_t k, int32_t H, int32_t F, const int8_t* q, const uint8_t* e,
                                           void* da, void* h, void* dp, void* workspace, int64_t workspace_bytes,
                                           hipStream_t stream) {
  DO_TRY(check_experts(N, E, k));
  const int64_t R = N * k;
  DO_TRY(check_swiglu(dtype, p, p_dtype, offsets, row_token, N, R, E, H, F));
  DO_TRY(check_ptr(dy, size_of(dtype), "dy is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(w2, size_of(dtype), "w2 is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(da, size_of(dtype), "da is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(h, size_of(dtype), "h is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(q, 1, "q is NULL"));
  DO_TRY(check_ptr(e, 1, "e is NULL"));
  if (dp != nullptr) {
    if (p == nullptr) return set_error(DO_ERR_INVALID_ARG, "dp is the gradient of p, which is NULL");
    if (!aligned(dp, size_of(p_dtype))) return set_error(DO_ERR_INVALID_ARG, "dp is not aligned to its element size");
    DO_TRY(check_ptr(token_row, 4, "token_row is NULL or not 4-byte aligned"));
    DO_TRY(check_ptr(token_expert, 4, "token_expert is NULL or not 4-byte aligned"));
    DO_TRY(check_ptr(workspace, 4, "workspace is NULL or not 4-byte aligned"));
    if (workspace_bytes < do_expert_swiglu_grad_workspace(R, F))
      return set_error(DO_ERR_INVALID_ARG, "workspace is smaller than do_expert_swiglu_grad_workspace(R, F)");
  }
  dol::ExpertGemm g{};
  g.P = w2;
  g.Q = dy;
  g.offsets = offsets;
  g.q_token = row_token;
  g.N = N;
  g.R = R;
  g.E = E;
  g.Pd = F;
  g.K = H;
  g.ldp = F;
  g.ldq = H;
  g.wide = wide(dtype, H, N);
  g.prob = p;
  g.p_bf16 = p_dtype == DO_BF16;
  g.q8 = const_cast<int8_t*>(q);
  g.e8 = const_cast<uint8_t*>(e);
  g.out = da;
  g.out2 = h;
  g.dp = dp != nullptr ? static_cast<float*>(workspace) : nullptr;
  g.vec_out = aligned(da, 16) && aligned(h, 16) && F % 8 == 0;
  g.vec_q8 = aligned(q, 16) && F % 16 == 0;
  DO_TRY(launched(dol::launch_expert_swiglu_grad(g, dtype, whole(dy, dtype, H, N) && whole(w2, dtype, F), stream)));
  if (dp == nullptr) return DO_OK;
  return launched(dol::launch_expert_dp(g.dp, (F + 63) / 64, R, token_row, token_expert, N, k, E, dp, p_dtype, stream));
}

DOLOSS_API do_status do_act8_pack(const void* x, do_dtype dtype, int64_t rows, int32_t W, int8_t* q, uint8_t* e,
                                  hipStream_t stream) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_rows(1, rows, 1, (int64_t(1) << 31) - 1));
  DO_TRY(check_widths(1, 1, {W}));
  DO_TRY(check_ptr(x, size_of(dtype), "x is NULL or not aligned to its element size"));
  DO_TRY(check_ptr(q, 1, "q is NULL"));
  DO_TRY(check_ptr(e, 1, "e is NULL"));
  return launched(dol::launch_act8_pack(x, dtype, rows, W, q, e, stream));
}

DOLOSS_API do_status do_act8_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int32_t W, void* x,
                                    do_dtype dtype, hipStream_t stream) {
  DO_TRY(check_dtype(dtype));
  DO_TRY(check_rows(1, rows, 1, (int64_t(1) << 31) - 1));
  DO_TRY(check_widths(1, 1, {W}));
  DO_TRY(check_ptr(q, 1, "q is NULL"));
  DO_TRY(check_ptr(e, 1, "e is NULL"));
  DO_TRY(check_ptr(x, size_of(dtype), "x is NULL or not aligned to its element size"));
  return launched(dol::launch_act8_unpack(q, e, rows, W, x, dtype, stream));
}
