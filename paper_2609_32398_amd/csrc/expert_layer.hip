// The whole layer of a few tokens (64 at most) in two kernels: y_t = sum over t's k best experts of
// W2_e h_te, h_te = p_te silu(g) u, (g, u) = W1_e x_t.
//
// The time is that of the chosen experts' weights coming from memory, each read once.  Both kernels feed the matrix
// instructions straight from memory: a wave's 64 lanes hold 16 bytes of 16 weight rows (64 bytes of each), and the
// tokens' values beside them; a lane's 16 bytes are one, two or four instructions' k, in the same order for both
// operands.  Weights in 8 bits become bf16 (or fp32) with their power of two in registers, exactly.
//
//   k_layer_up    Every block finds the k best experts of all tokens and, as N <= 64, holds an expert's tokens as one
//                 word of 64 bits.  The kernel without weights to speak of (64 and 8 wide) takes 4.2 us for the best of
//                 128 experts and 6.6 for the best 8, of one token and of 16; each further round 0.2 us (64 tokens
//                 0.85).  From 257 experts on a wave takes a token: 8 of 1,024 experts 11 us, of 64 tokens 91, and
//                 about 10 ms where 64 tokens take all 1,024.  Its tiles are 8 activations of an
//                 expert: their 8 gate and 8 up rows are the 16 rows of an instruction, its four waves take a quarter
//                 of H each.
//   k_layer_down  A block takes 16 columns of y and a share of the chosen experts: its waves take the experts in turn
//                 and add their tokens' sums in LDS, each wave in a place of its own, so that the order of a sum is
//                 fixed; the blocks of a column tile meet through memory.
//
// One token, 8 of 128 experts, 2,048 and 768 wide, bf16: 15.4 + 9.1 us, 6.6 + 3.8 of them without weights to speak of,
// so the 50 and 25 MB of weights come at 5.7 and 4.8 TB/s (reading 76 MB alone: 5.3).  16 tokens, 8 bits: 60 + 34 us
// (78 experts' 245 and 123 MB, 4.1 and 3.6 TB/s): waves that read more than others at the kernels' ends.  37 tokens of
// 6 of 48 experts, 1,000 and 333 wide, fp32: 40 to 43 + 27 to 28 us (128 and 64 MB, 3.0 and 2.3 TB/s).  Their rows are
// no multiples of 64 bytes, so that neighbours share pieces of a line (159 and 86 MB counted; 1,008 and 336 wide 147
// and 78 MB, 35 + 23 us).
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "experts.h"

namespace dol {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kUpWaves = 4, kDownWaves = 4;
constexpr int kTile = 16;     // rows and columns of a matrix instruction
constexpr int kActs = 8;      // activations of a tile
// The second kernel's column tiles are split over blocks, 16 at most, that have 64 KiB of weights or more each.  Against
// one block a column tile: 1 token bf16 24.3 against 26.7 us, 16 tokens 8 bits 92.5 against 137, 37 tokens fp32 71
// against 123, 64 tokens 8 bits 176 against 248.  With 32 KiB the same to 1 us, with 128 KiB 26.7, 92.6, 75.6 and 176.
constexpr int kMaxSplit = 16;
constexpr int kSplitBytes = 65536;

__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// What the two operands are made of.  T: activations (float, or uint16_t for bf16); W8: weights in 8 bits.
template <typename T, bool W8>
struct Form {
  static constexpr int W = W8 ? 16 : 16 / (int)sizeof(T);  // weights in a lane's 16 bytes
  static constexpr int X = W * (int)sizeof(T) / 16;        // 16-byte pieces of activations beside them
  static constexpr int P = W8 ? 2 : 1;                     // pieces of weights in a step: 8 bits, a block's 128
  static constexpr int piece = 4 * W;                      // k of four lanes' pieces
  static constexpr int step = P * piece;
  using Element = std::conditional_t<W8, uint8_t, T>;
  // steps that are on their way together, for NT tiles of activations: as many as leave four waves a SIMD, two at least.
  // Two of fp32 activations beside 8-bit weights do not fit: 8 to 21 registers spill with one tile, 61 to 65 with two
  // (16 tokens 162 us against 92 in bf16, 64 tokens 334 against 176, the fp32 matrix instructions included).  bf16 beside
  // 8-bit weights spills 2 in the first kernel of two tiles, nothing else does.
  template <int NT>
  static constexpr int ahead = std::max(2, std::min(8, 68 / (P * (4 + 4 * X * NT))));

  // acc[weight row 4 (lane / 16) + v][activation row lane % 16] += their products over the step's k
  static __device__ __forceinline__ v4f mul(v4u w, float s, const v4u* x, v4f acc) {
    if constexpr (W8 && sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        v4u b;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          b[2 * j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[2 * i + j], s, false));
          b[2 * j + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[2 * i + j], s, true));
        }
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, x[i]), acc, 0, 0, 0);
      }
    } else if constexpr (W8) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
        const float v[4] = {lo[0] * s, lo[1] * s, hi[0] * s, hi[1] * s};
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(v[j], __uint_as_float(x[i][j]), acc, 0, 0, 0);
      }
    } else if constexpr (sizeof(T) == 2) {
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, w), __builtin_bit_cast(v8bf, x[0]), acc, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), __uint_as_float(x[0][j]), acc, 0, 0, 0);
    }
    return acc;
  }
};

// 16 bytes at p, of any alignment to whole elements.
template <typename E>
__device__ __forceinline__ v4u piece(const E* p) {
  v4u v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// Weights pass the caches: each is read once.
template <typename E>
__device__ __forceinline__ v4u weights(const E* p) {
  typedef uint32_t v4u_any __attribute__((ext_vector_type(4), aligned(1)));
  return __builtin_nontemporal_load(reinterpret_cast<const v4u_any*>(p));
}
// The first n of a piece's elements, zeros behind.
template <typename E>
__device__ __forceinline__ v4u part(const E* p, int n) {
  constexpr int EL = 16 / (int)sizeof(E), PW = 4 / (int)sizeof(E);  // elements of a piece, of a word
  if (n >= EL) return piece(p);
  v4u v{0u, 0u, 0u, 0u};
#pragma unroll
  for (int i = 0; i < EL; ++i)
    if (i < n) {
      uint32_t u;
      if constexpr (sizeof(E) == 4)
        u = __float_as_uint(p[i]);
      else
        u = (uint32_t)p[i] << (8 * (int)sizeof(E) * (i % PW));
      v[i / PW] |= u;
    }
  return v;
}

// A wave's products over steps [s0, s1) of a contraction of K: w is the lane's weight row, e its blocks' exponents, x
// the lane's activation row of each of NT tiles.
template <typename T, bool W8, int NT>
__device__ __forceinline__ void multiply(const typename Form<T, W8>::Element* w, const uint8_t* e, const T* const* x,
                                         int K, int s0, int s1, int lane, v4f* acc) {
  using F = Form<T, W8>;
  constexpr int D = F::template ahead<NT>;
  const int full = min(s1, K / F::step), mine = (lane >> 4) * F::W;
  struct Step {
    v4u w[F::P], x[F::P][NT][F::X];
    uint32_t e;
  };
  // the lane's places in the step that is loaded next
  const typename F::Element* wp = w + s0 * F::step + mine;
  const uint8_t* ep = e + s0;
  const T* xp[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) xp[t] = x[t] + s0 * F::step + mine;
  auto load = [&](int u) {
    Step n;
#pragma unroll
    for (int q = 0; q < F::P; ++q) {
      const int k = u * F::step + q * F::piece;
      n.w[q] = weights(wp + k);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < F::X; ++i) n.x[q][t][i] = piece(xp[t] + k + i * (F::W / F::X));
    }
    n.e = W8 ? ep[u] : 0;
    return n;
  };
  auto on = [&](int steps) {
    wp += steps * F::step;
    ep += W8 ? steps : 0;
#pragma unroll
    for (int t = 0; t < NT; ++t) xp[t] += steps * F::step;
  };
  auto use = [&](const Step& n) {
    const float sc = W8 ? fp8_scale(n.e) : 1.0f;
#pragma unroll
    for (int q = 0; q < F::P; ++q)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t] = F::mul(n.w[q], sc, n.x[q][t], acc[t]);
  };
  int left = full - s0;
  if (left >= D) {  // D steps on their way at any time
    Step ring[D];
#pragma unroll
    for (int u = 0; u < D; ++u) ring[u] = load(u);
    on(D);
    for (left -= D; left >= D; left -= D) {
#pragma unroll
      for (int u = 0; u < D; ++u) {
        use(ring[u]);
        ring[u] = load(u);
      }
      on(D);
    }
#pragma unroll
    for (int u = 0; u < D; ++u) use(ring[u]);
  }
  if (left > 0) {  // fewer than D: as many again from the last one's place, which are not used
    Step some[D - 1];
#pragma unroll
    for (int u = 0; u < D - 1; ++u) some[u] = load(min(u, left - 1));
#pragma unroll
    for (int u = 0; u < D - 1; ++u)
      if (u < left) use(some[u]);
  }
  if (full < s1) {  // the last step, which ends inside
    const float sc = W8 ? fp8_scale(e[full]) : 1.0f;
#pragma unroll
    for (int q = 0; q < F::P; ++q) {
      const int k = full * F::step + q * F::piece + mine, n = K - k;
      const v4u wv = n > 0 ? part(w + k, n) : v4u{0u, 0u, 0u, 0u};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        v4u xv[F::X];
#pragma unroll
        for (int i = 0; i < F::X; ++i) {
          const int at = i * (F::W / F::X);
          xv[i] = n > at ? part(x[t] + k + at, n - at) : v4u{0u, 0u, 0u, 0u};
        }
        acc[t] = F::mul(wv, sc, xv, acc[t]);
      }
    }
  }
}

// A score's rank as a number above 0: NaN below all others, both zeros alike.
__device__ __forceinline__ uint32_t rank_of(float v) {
  const uint32_t b = __float_as_uint(v);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 1u;
  if ((b & 0x7FFFFFFFu) == 0u) return 0x80000000u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// A value of another lane of the row of 16, or (scans) of the rows before; lanes without one get 0.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false);
}
// op over the 16 lanes of a row, or all 64, in every lane.
template <int G, typename F>
__device__ __forceinline__ uint32_t over_group(uint32_t v, F&& op) {
  v = op(v, moved<0x128>(v));  // rotations of the row by 8, 4, 2 and 1
  v = op(v, moved<0x124>(v));
  v = op(v, moved<0x122>(v));
  v = op(v, moved<0x121>(v));
  if constexpr (G == 64) {
    auto of = [&](int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); };
    v = op(op(of(0), of(16)), op(of(32), of(48)));
  }
  return v;
}
// The sum of the lanes up to this one.
__device__ __forceinline__ uint32_t running_sum(uint32_t v) {
  v += moved<0x111>(v);  // shifts of the row by 1, 2, 4 and 8
  v += moved<0x112>(v);
  v += moved<0x114>(v);
  v += moved<0x118>(v);
  v += moved<0x142, 0xA>(v);  // the end of the row before to rows 1 and 3
  v += moved<0x143, 0xC>(v);  // that of row 1 to rows 2 and 3
  return v;
}

// The tokens of each expert among every token's k best: larger scores first, equal ones by the lower expert.  G lanes
// take a token, P experts each.  A round finds the largest of what is left, and who has it.
template <int G, int P, int THREADS>
__device__ __forceinline__ void choose(const LayerArgs& a, u64* tokens) {
  const int at = threadIdx.x % G;
  float next[P];  // the next token's scores
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const int64_t from = (int64_t)min(t, a.N - 1) * a.E + min(i * G + at, a.E - 1);
      next[i] = a.scores_bf16 ? bf16_float(static_cast<const uint16_t*>(a.scores)[from])
                              : static_cast<const float*>(a.scores)[from];
    }
  };
  load(threadIdx.x / G);
  for (int t = threadIdx.x / G; t < a.N; t += THREADS / G) {
    uint32_t key[P];
#pragma unroll
    for (int i = 0; i < P; ++i) key[i] = i * G + at < a.E ? rank_of(next[i]) : 0u;
    load(t + THREADS / G);
    for (int j = 0; j < a.k; ++j) {
      uint32_t top = key[0];
#pragma unroll
      for (int i = 1; i < P; ++i) top = max(top, key[i]);
      top = over_group<G>(top, [](uint32_t x, uint32_t y) { return max(x, y); });
      uint32_t won = ~0u;
#pragma unroll
      for (int i = P - 1; i >= 0; --i) won = key[i] == top ? (uint32_t)(i * G + at) : won;
      won = over_group<G>(won, [](uint32_t x, uint32_t y) { return min(x, y); });
#pragma unroll
      for (int i = 0; i < P; ++i) key[i] = won == (uint32_t)(i * G + at) ? 0u : key[i];
      if (at == 0) atomicOr(&tokens[won], (u64)1 << t);
    }
  }
}

// The n-th tokens of an expert, in a wave's own place in LDS: n < 64.
__device__ __forceinline__ void list_tokens(u64 tokens, int lane, uint8_t* list) {
  if (tokens >> lane & 1) list[__popcll(tokens & (((u64)1 << lane) - 1))] = (uint8_t)lane;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// Waves a SIMD to leave registers for.  (With one fewer, and as many more steps on their way, 16 tokens in 8 bits take 4 us
// more.)
template <int NT>
constexpr int kOccupancy = NT == 1 ? 4 : 3;

// NT: tiles of 16 tokens that share a pass over an expert's weights.
template <typename T, bool W8, int NT>
__global__ __launch_bounds__(kUpWaves* kWave, kOccupancy<NT>) void k_layer_up(const LayerArgs a) {
  using F = Form<T, W8>;
  constexpr int kThreads = kUpWaves * kWave;
  extern __shared__ __align__(16) char sm[];
  Chosen* chosen = reinterpret_cast<Chosen*>(sm);           // [E]
  u64* tokens = reinterpret_cast<u64*>(chosen + a.E);       // [E]
  __shared__ int32_t n_chosen;
  __shared__ uint8_t lists[kUpWaves][kWave];
  __shared__ __align__(16) v4f red[2][kUpWaves][NT][kWave];  // the waves' sums, lane by lane
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e < a.E; e += kThreads) tokens[e] = 0;
  __syncthreads();
  if (a.E <= 64)
    choose<16, 4, kThreads>(a, tokens);
  else if (a.E <= 128)
    choose<16, 8, kThreads>(a, tokens);
  else if (a.E <= 256)
    choose<16, 16, kThreads>(a, tokens);
  else
    choose<64, 16, kThreads>(a, tokens);
  __syncthreads();
  if (wave == 0) {
    int rows = 0, have = 0;
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      const int e = e0 + lane;
      const u64 mine = e < a.E ? tokens[e] : 0;
      const int own = __popcll(mine), n = (int)running_sum(own);
      const u64 some = __ballot(own > 0);
      if (own > 0) chosen[have + __popcll(some & (((u64)1 << lane) - 1))] = Chosen{e, rows + n - own, mine};
      rows += __builtin_amdgcn_readlane(n, 63);
      have += __popcll(some);
    }
    if (lane == 0) n_chosen = have;
  }
  __syncthreads();
  const int have = __builtin_amdgcn_readfirstlane(n_chosen);
  if (blockIdx.x == 0) {  // for the second kernel
    for (int i = tid; i < have; i += kThreads) a.chosen[i] = chosen[i];
    for (int i = tid; i < (a.H + kTile - 1) / kTile; i += kThreads) a.arrived[i] = 0;
    if (tid == 0) *a.n_chosen = have;
  }
  const int C = (a.F + kActs - 1) / kActs, steps = (a.H + F::step - 1) / F::step;
  const int s0 = wave * steps / kUpWaves, s1 = (wave + 1) * steps / kUpWaves;
  const int row = lane & 15;
  int turn = 0;
  for (int tile = blockIdx.x; tile < have * C; tile += gridDim.x) {
    const Chosen ch = chosen[tile / C];
    const int e = __builtin_amdgcn_readfirstlane(ch.e), f0 = tile % C * kActs;
    const int n = __builtin_amdgcn_readfirstlane(__popcll(ch.tokens));
    list_tokens(ch.tokens, lane, lists[wave]);
    // 8 gate rows, then the 8 up rows beside them
    const int64_t wr = min(f0 + (row & 7), a.F - 1) + (row >> 3) * (int64_t)a.F;
    const auto* w = static_cast<const typename F::Element*>(a.w1) + ((int64_t)e * 2 * a.F + wr) * a.H;
    const uint8_t* we = nullptr;
    if constexpr (W8) {
      const int64_t PB = (2 * (int64_t)a.F + kFp8Block - 1) / kFp8Block, KB = (a.H + kFp8Block - 1) / kFp8Block;
      we = a.w1_exp + (e * PB + wr / kFp8Block) * KB;
    }
    for (int r0 = 0; r0 < n; r0 += NT * kTile, turn ^= 1) {
      const T* x[NT];
      float p[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int64_t token = lists[wave][min(r0 + t * kTile + row, n - 1)];
        x[t] = static_cast<const T*>(a.x) + token * a.H;
        p[t] = a.p == nullptr ? 1.0f
               : a.p_bf16     ? bf16_float(static_cast<const uint16_t*>(a.p)[token * a.E + e])
                              : static_cast<const float*>(a.p)[token * a.E + e];
      }
      v4f acc[NT] = {};
      if (NT == 1 || n - r0 <= kTile)
        multiply<T, W8, 1>(w, we, x, a.H, s0, s1, lane, acc);
      else
        multiply<T, W8, NT>(w, we, x, a.H, s0, s1, lane, acc);
#pragma unroll
      for (int t = 0; t < NT; ++t) red[turn][wave][t][lane] = acc[t];
      __syncthreads();  // one a turn: the sums of the turn after next are written behind the next one
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (wave != t) continue;  // one wave for each tile of tokens
        v4f s = red[turn][0][t][lane];
#pragma unroll
        for (int v = 1; v < kUpWaves; ++v) s += red[turn][v][t][lane];
        // lanes 0 to 31 hold four gates of a token each, the lanes 32 on their ups
        const int r = r0 + t * kTile + row, c = f0 + (lane >> 4) * 4;
        float h[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          const float u = __shfl_xor(s[v], 32);
          h[v] = p[t] * (s[v] * sigmoid(s[v])) * u;
        }
        if (lane < 32 && r < n) {
          // rounded to bf16 as an operand of the second product, as do_expert_swiglu does; rows are whole pieces
          T* d = static_cast<T*>(a.h) + (int64_t)(ch.first + r) * a.ldh + c;
          if constexpr (sizeof(T) == 2) {
            if (c < a.ldh) *reinterpret_cast<v2u*>(d) = v2u{bf16_pair(h[0], h[1]), bf16_pair(h[2], h[3])};
          } else {
            if (c < a.ldh) *reinterpret_cast<v4f*>(d) = v4f{h[0], h[1], h[2], h[3]};
          }
        }
      }
    }
  }
}

// TOK: tokens at most.  gridDim.y blocks share a column tile: each adds up its part of the experts, and the last one
// to arrive adds the parts, in their order.
template <typename T, bool W8, int NT, int TOK>
__global__ __launch_bounds__(kDownWaves* kWave, kOccupancy<NT>) void k_layer_down(const LayerArgs a) {
  using F = Form<T, W8>;
  constexpr int kThreads = kDownWaves * kWave;
  extern __shared__ __align__(16) char sm[];
  Chosen* chosen = reinterpret_cast<Chosen*>(sm);
  __shared__ uint8_t lists[kDownWaves][kWave];
  __shared__ __align__(16) float sums[kDownWaves][TOK][kTile + 4];  // of a wave, by token and column
  __shared__ int32_t last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = lane & 15;
  const int have = *a.n_chosen, S = gridDim.y;
  // the list's end is not known yet: what lies behind it is loaded and not used
  for (int i = tid; i < a.most; i += kThreads) chosen[i] = a.chosen[i];
  for (int i = lane; i < TOK * (kTile + 4); i += kWave) (&sums[wave][0][0])[i] = 0.0f;
  __syncthreads();
  const int c0 = blockIdx.x * kTile;
  const int steps = (a.F + F::step - 1) / F::step, waves = S * kDownWaves;
  const int parts = max(1, min(steps, waves / have));  // of an expert's contraction
  for (int unit = blockIdx.y * kDownWaves + wave; unit < have * parts; unit += waves) {
    const Chosen ch = chosen[unit / parts];
    const int e = __builtin_amdgcn_readfirstlane(ch.e), part = __builtin_amdgcn_readfirstlane(unit % parts);
    const int n = __builtin_amdgcn_readfirstlane(__popcll(ch.tokens));
    const int s0 = part * steps / parts, s1 = (part + 1) * steps / parts;
    list_tokens(ch.tokens, lane, lists[wave]);
    const int64_t wr = min(c0 + row, a.H - 1);
    const auto* w = static_cast<const typename F::Element*>(a.w2) + ((int64_t)e * a.H + wr) * a.F;
    const uint8_t* we = nullptr;
    if constexpr (W8) {
      const int64_t PB = (a.H + kFp8Block - 1) / kFp8Block, KB = (a.F + kFp8Block - 1) / kFp8Block;
      we = a.w2_exp + (e * PB + wr / kFp8Block) * KB;
    }
    for (int r0 = 0; r0 < n; r0 += NT * kTile) {
      const T* x[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t)
        x[t] = static_cast<const T*>(a.h) + (int64_t)(ch.first + min(r0 + t * kTile + row, n - 1)) * a.ldh;
      v4f acc[NT] = {};
      if (NT == 1 || n - r0 <= kTile)
        multiply<T, W8, 1>(w, we, x, a.F, s0, s1, lane, acc);
      else
        multiply<T, W8, NT>(w, we, x, a.F, s0, s1, lane, acc);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int r = r0 + t * kTile + row;
        if (r < n) *reinterpret_cast<v4f*>(&sums[wave][lists[wave][r]][(lane >> 4) * 4]) += acc[t];
      }
    }
  }
  __syncthreads();
  float* parted = a.parts + (int64_t)blockIdx.x * S * a.N * kTile;
  const int all = a.N * kTile;
  auto store = [&](int i, float s) {
    const int t = i / kTile, c = c0 + i % kTile;
    if (c >= a.H) return;
    T* d = static_cast<T*>(a.y) + (int64_t)t * a.H + c;
    if constexpr (sizeof(T) == 2)
      *d = bf16_bits(s);
    else
      *d = s;
  };
  for (int i = tid; i < all; i += kThreads) {
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < kDownWaves; ++v) s += sums[v][i / kTile][i % kTile];
    if (S == 1)
      store(i, s);
    else
      __hip_atomic_store(parted + blockIdx.y * all + i, s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  if (S == 1) return;
  // The parts are stored and loaded past the L2 caches, which belong to an XCD each, so that they only have to be
  // done before the count: a fence would write a whole cache back (60 to 80 us more).
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (tid == 0)
    last = __hip_atomic_fetch_add(&a.arrived[blockIdx.x], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == S - 1;
  __syncthreads();
  if (!last) return;
  for (int i = tid; i < all; i += kThreads) {
    float v[kMaxSplit], s = 0.0f;  // all loaded before the first is used
#pragma unroll
    for (int u = 0; u < kMaxSplit; ++u)
      v[u] = __hip_atomic_load(parted + min(u, S - 1) * all + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int u = 0; u < kMaxSplit; ++u) s += u < S ? v[u] : 0.0f;
    store(i, s);
  }
}

template <typename T, bool W8, int NT>
hipError_t launch_up(const LayerArgs& a, hipStream_t s) {
  static std::atomic<int> per_cu[64];
  const DevInfo di = device_info();
  if (di.device < 0 || di.device >= 64) return hipErrorInvalidDevice;
  int occ = per_cu[di.device].load(std::memory_order_acquire);
  if (occ == 0) {
    const hipError_t e =
        hipOccupancyMaxActiveBlocksPerMultiprocessor(&occ, k_layer_up<T, W8, NT>, kUpWaves * kWave, 0);
    if (e != hipSuccess) return e;
    if (occ < 1) return hipErrorLaunchOutOfResources;
    per_cu[di.device].store(occ, std::memory_order_release);
  }
  // at most this many tiles: how many experts are chosen is only known on the device
  const int64_t tiles = (int64_t)a.most * ((a.F + kActs - 1) / kActs);
  hipLaunchKernelGGL((k_layer_up<T, W8, NT>), dim3((unsigned)std::min<int64_t>(tiles, (int64_t)occ * di.cu_count)),
                     dim3(kUpWaves * kWave), (size_t)a.E * (sizeof(Chosen) + sizeof(u64)), s, a);
  return hipGetLastError();
}

template <typename T, bool W8, int NT, int TOK>
hipError_t launch(const LayerArgs& a, hipStream_t s) {
  const hipError_t e = launch_up<T, W8, NT>(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_layer_down<T, W8, NT, TOK>), dim3((unsigned)((a.H + kTile - 1) / kTile), (unsigned)a.split),
                     dim3(kDownWaves * kWave), (size_t)a.most * sizeof(Chosen), s, a);
  return hipGetLastError();
}

template <typename T, bool W8>
hipError_t by_tokens(const LayerArgs& a, hipStream_t s) {
  return a.N <= 16 ? launch<T, W8, 1, 16>(a, s) : launch<T, W8, 2, 64>(a, s);
}

}  // namespace

// The workspace: how many experts are chosen, the list of them, how many blocks of a column tile have arrived, their
// sums, the activations.
namespace {
struct LayerSpace {
  int64_t chosen, arrived, parts, h, bytes;
};
LayerSpace layer_space(do_dtype dt, int64_t N, int32_t E, int32_t k, int32_t H, int32_t F) {
  auto up = [](int64_t n) { return (n + 15) & ~int64_t(15); };
  const int64_t rows = N * k, tiles = (H + kTile - 1) / kTile;
  LayerSpace w;
  w.chosen = 16;
  w.arrived = w.chosen + std::min<int64_t>(E, rows) * (int64_t)sizeof(Chosen);
  w.parts = w.arrived + up(tiles * 4);
  w.h = w.parts + tiles * kMaxSplit * N * kTile * 4;
  w.bytes = w.h + rows * layer_row(dt, F) * (dt == DO_F32 ? 4 : 2);
  return w;
}
}  // namespace

int64_t expert_layer_bytes(do_dtype dt, int64_t N, int32_t E, int32_t k, int32_t H, int32_t F) {
  return layer_space(dt, N, E, k, H, F).bytes;
}

hipError_t launch_expert_layer(LayerArgs a, do_dtype dt, void* workspace, hipStream_t s) {
  char* ws = static_cast<char*>(workspace);
  const LayerSpace w = layer_space(dt, a.N, a.E, a.k, a.H, a.F);
  a.n_chosen = reinterpret_cast<int32_t*>(ws);
  a.chosen = reinterpret_cast<Chosen*>(ws + w.chosen);
  a.arrived = reinterpret_cast<int32_t*>(ws + w.arrived);
  a.parts = reinterpret_cast<float*>(ws + w.parts);
  a.h = ws + w.h;
  a.ldh = layer_row(dt, a.F);
  a.most = (int32_t)std::min<int64_t>(a.E, (int64_t)a.N * a.k);
  // blocks that share a column tile of the second kernel: those that fit in all, each with 64 KiB of weights or more
  const int64_t tiles = (a.H + kTile - 1) / kTile;
  const int64_t bytes = (int64_t)a.most * kTile * a.F * (a.w1_exp != nullptr ? 1 : dt == DO_F32 ? 4 : 2);
  a.split = (int32_t)std::max<int64_t>(
      1, std::min({(int64_t)kMaxSplit, (a.N <= 16 ? 4 : 3) * (int64_t)device_info().cu_count / tiles, bytes / kSplitBytes}));
  const bool w8 = a.w1_exp != nullptr;
  if (dt == DO_F32) return w8 ? by_tokens<float, true>(a, s) : by_tokens<float, false>(a, s);
  return w8 ? by_tokens<uint16_t, true>(a, s) : by_tokens<uint16_t, false>(a, s);
}

}  // namespace dol
