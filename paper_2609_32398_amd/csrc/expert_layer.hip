// The whole layer of a few tokens (64 at most) in two kernels: y_t = sum over t's k best experts of
// W2_e h_te, h_te = p_te silu(g) u, (g, u) = W1_e x_t.
//
// The time is that of the chosen experts' weights coming from memory, each read once.  Both kernels feed the matrix
// instructions straight from memory: a wave's 64 lanes hold 16 bytes of 16 weight rows (64 bytes of each), and the
// tokens' values beside them; a lane's 16 bytes are one, two or four instructions' k, in the same order for both
// operands.  Weights in 8 bits become bf16 (or fp32) with their power of two in registers, exactly.
//
//   k_layer_up    Every block finds the k best experts of all tokens (a few thousand scores) and, as N <= 64, holds an
//                 expert's tokens as one word of 64 bits.  Its tiles are 8 activations of an expert: their 8 gate and 8
//                 up rows are the 16 rows of an instruction, its four waves take a quarter of H each.
//   k_layer_down  A block takes 16 columns of y and all chosen experts: its waves take the experts in turn and add
//                 their tokens' sums in LDS, each wave in a place of its own, so that the order of a sum is fixed.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "experts.h"

namespace dol {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kUpWaves = 4, kDownWaves = 8;
constexpr int kTile = 16;     // rows and columns of a matrix instruction
constexpr int kActs = 8;      // activations of a tile
constexpr int kAhead = 4;     // steps whose loads are issued together

__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// What the two operands are made of.  T: activations (float, or uint16_t for bf16); W8: weights in 8 bits.
template <typename T, bool W8>
struct Form {
  static constexpr int W = W8 ? 16 : 16 / (int)sizeof(T);  // weights in a lane's 16 bytes
  static constexpr int X = W * (int)sizeof(T) / 16;        // 16-byte pieces of activations beside them
  static constexpr int step = 4 * W;                       // k of a step
  using Element = std::conditional_t<W8, uint8_t, T>;

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
// the lane's activation row of each of nt (NT at most) tiles.
template <typename T, bool W8, int NT>
__device__ __forceinline__ void multiply(const typename Form<T, W8>::Element* w, const uint8_t* e, const T* const* x, int nt,
                                         int K, int s0, int s1, int lane, v4f* acc) {
  using F = Form<T, W8>;
  const int full = min(s1, K / F::step), mine = (lane >> 4) * F::W;
  for (int s = s0; s < full; s += kAhead) {
    v4u wv[kAhead], xv[kAhead][NT][F::X];
    uint32_t ev[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = min(s + u, full - 1) * F::step + mine;
      wv[u] = weights(w + k);
      if constexpr (W8) ev[u] = e[k / kFp8Block];
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < F::X; ++i) xv[u][t][i] = piece(x[t] + k + i * (F::W / F::X));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (s + u < full) {
        const float sc = W8 ? fp8_scale(ev[u]) : 1.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t)
          if (t < nt) acc[t] = F::mul(wv[u], sc, xv[u][t], acc[t]);
      }
    }
  }
  if (full < s1) {  // the last step, which ends inside
    const int k = full * F::step + mine, n = K - k;
    const v4u wv = n > 0 ? part(w + k, n) : v4u{0u, 0u, 0u, 0u};
    const float sc = W8 && n > 0 ? fp8_scale(e[k / kFp8Block]) : 1.0f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (t >= nt) continue;
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

// A score's rank as a number above 0: NaN below all others, both zeros alike.
__device__ __forceinline__ uint32_t rank_of(float v) {
  const uint32_t b = __float_as_uint(v);
  if ((b & 0x7FFFFFFFu) > 0x7F800000u) return 1u;
  if ((b & 0x7FFFFFFFu) == 0u) return 0x80000000u;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

template <int G>
__device__ __forceinline__ u64 largest_of_group(u64 v) {
#pragma unroll
  for (int d = 1; d < G; d <<= 1) {
    const u64 o = (u64)__shfl_xor((long long)v, d);
    v = o > v ? o : v;
  }
  return v;
}

// The tokens of each expert among every token's k best: larger scores first, equal ones by the lower expert.  G lanes
// take a token, 16 experts a lane at most.
template <int G, int THREADS>
__device__ __forceinline__ void choose(const LayerArgs& a, u64* tokens) {
  constexpr int P = 16;
  const int at = threadIdx.x % G;
  for (int t = threadIdx.x / G; t < a.N; t += THREADS / G) {
    uint32_t key[P];
    const int64_t row = (int64_t)t * a.E;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      key[i] = 0u;
      const int e = i * G + at;
      if (i * G < a.E && e < a.E)
        key[i] = rank_of(a.scores_bf16 ? bf16_float(static_cast<const uint16_t*>(a.scores)[row + e])
                                       : static_cast<const float*>(a.scores)[row + e]);
    }
    for (int j = 0; j < a.k; ++j) {
      uint32_t best = 0u, e = 0u;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const bool more = key[i] > best;
        best = more ? key[i] : best;
        e = more ? (uint32_t)(i * G + at) : e;
      }
      const u64 top = largest_of_group<G>((u64)best << 32 | (0xFFFFFFFFu - e));
      const uint32_t won = 0xFFFFFFFFu - (uint32_t)top;
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

template <typename T, bool W8, int NT>
__global__ __launch_bounds__(kUpWaves* kWave) void k_layer_up(const LayerArgs a) {
  using F = Form<T, W8>;
  constexpr int kThreads = kUpWaves * kWave;
  __shared__ u64 tokens[kMaxE];
  __shared__ Chosen chosen[kMaxE];
  __shared__ int32_t n_chosen;
  __shared__ uint8_t lists[kUpWaves][kWave];
  __shared__ __align__(16) float red[2][kUpWaves][NT][kTile][kTile + 4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int e = tid; e < a.E; e += kThreads) tokens[e] = 0;
  __syncthreads();
  if (a.E <= 256)
    choose<16, kThreads>(a, tokens);
  else
    choose<64, kThreads>(a, tokens);
  __syncthreads();
  if (wave == 0) {
    int rows = 0, have = 0;
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      const int e = e0 + lane;
      const u64 mine = e < a.E ? tokens[e] : 0;
      int n = __popcll(mine);
      const int own = n;
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(n, d);
        n += lane >= d ? o : 0;
      }
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
    if (tid == 0) *a.n_chosen = have;
  }
  const int C = (a.F + kActs - 1) / kActs, steps = (a.H + F::step - 1) / F::step;
  const int s0 = wave * steps / kUpWaves, s1 = (wave + 1) * steps / kUpWaves;
  const int row = lane & 15;
  int turn = 0;
  for (int tile = blockIdx.x; tile < have * C; tile += gridDim.x, turn ^= 1) {
    const Chosen ch = chosen[tile / C];
    const int e = __builtin_amdgcn_readfirstlane(ch.e), n = __popcll(ch.tokens), f0 = tile % C * kActs;
    list_tokens(ch.tokens, lane, lists[wave]);
    const int nt = (n + kTile - 1) / kTile;
    const T* x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
      x[t] = static_cast<const T*>(a.x) + (int64_t)lists[wave][min(t * kTile + row, n - 1)] * a.H;
    // 8 gate rows, then the 8 up rows beside them
    const int64_t wr = min(f0 + (row & 7), a.F - 1) + (row >> 3) * (int64_t)a.F;
    const auto* w = static_cast<const typename F::Element*>(a.w1) + ((int64_t)e * 2 * a.F + wr) * a.H;
    const uint8_t* we = nullptr;
    if constexpr (W8) {
      const int64_t PB = (2 * (int64_t)a.F + kFp8Block - 1) / kFp8Block, KB = (a.H + kFp8Block - 1) / kFp8Block;
      we = a.w1_exp + (e * PB + wr / kFp8Block) * KB;
    }
    v4f acc[NT] = {};
    multiply<T, W8, NT>(w, we, x, nt, a.H, s0, s1, lane, acc);
#pragma unroll
    for (int t = 0; t < NT; ++t)
      if (t < nt) *reinterpret_cast<v4f*>(&red[turn][wave][t][row][(lane >> 4) * 4]) = acc[t];
    __syncthreads();  // one a tile: the sums of the tile after next are written behind the next one
    for (int i = tid; i < nt * kTile * kActs; i += kThreads) {
      const int r = i / kActs, c = i % kActs;
      if (r >= n || f0 + c >= a.F) continue;
      float g = 0.0f, u = 0.0f;
#pragma unroll
      for (int v = 0; v < kUpWaves; ++v) {
        g += red[turn][v][r / kTile][r % kTile][c];
        u += red[turn][v][r / kTile][r % kTile][kActs + c];
      }
      float p = 1.0f;
      if (a.p != nullptr) {
        const int64_t at = (int64_t)lists[wave][r] * a.E + e;
        p = a.p_bf16 ? bf16_float(static_cast<const uint16_t*>(a.p)[at]) : static_cast<const float*>(a.p)[at];
      }
      const float h = p * (g * sigmoid(g)) * u;
      T* d = static_cast<T*>(a.h) + (int64_t)(ch.first + r) * a.ldh + f0 + c;
      // rounded to bf16 as an operand of the second product, as do_expert_swiglu does
      if constexpr (sizeof(T) == 2)
        *d = bf16_bits(h);
      else
        *d = h;
    }
  }
}

template <typename T, bool W8, int NT>
__global__ __launch_bounds__(kDownWaves* kWave) void k_layer_down(const LayerArgs a) {
  using F = Form<T, W8>;
  constexpr int kThreads = kDownWaves * kWave;
  __shared__ Chosen chosen[kMaxE];
  __shared__ uint8_t lists[kDownWaves][kWave];
  __shared__ __align__(16) float sums[kDownWaves][NT * kTile][kTile + 4];  // of a wave, by token and column
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, row = lane & 15;
  const int have = *a.n_chosen;
  for (int i = tid; i < have; i += kThreads) chosen[i] = a.chosen[i];
  for (int i = lane; i < NT * kTile * (kTile + 4); i += kWave) (&sums[wave][0][0])[i] = 0.0f;
  __syncthreads();
  const int c0 = blockIdx.x * kTile;
  const int steps = (a.F + F::step - 1) / F::step;
  const int parts = max(1, kDownWaves / have);  // of an expert's contraction
  for (int unit = wave; unit < have * parts; unit += kDownWaves) {
    const Chosen ch = chosen[unit / parts];
    const int e = __builtin_amdgcn_readfirstlane(ch.e), n = __popcll(ch.tokens), part = unit % parts;
    list_tokens(ch.tokens, lane, lists[wave]);
    const int nt = (n + kTile - 1) / kTile;
    const T* x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
      x[t] = static_cast<const T*>(a.h) + (int64_t)(ch.first + min(t * kTile + row, n - 1)) * a.ldh;
    const int64_t wr = min(c0 + row, a.H - 1);
    const auto* w = static_cast<const typename F::Element*>(a.w2) + ((int64_t)e * a.H + wr) * a.F;
    const uint8_t* we = nullptr;
    if constexpr (W8) {
      const int64_t PB = (a.H + kFp8Block - 1) / kFp8Block, KB = (a.F + kFp8Block - 1) / kFp8Block;
      we = a.w2_exp + (e * PB + wr / kFp8Block) * KB;
    }
    v4f acc[NT] = {};
    multiply<T, W8, NT>(w, we, x, nt, a.F, part * steps / parts, (part + 1) * steps / parts, lane, acc);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = t * kTile + row;
      if (r < n) {
        v4f* s = reinterpret_cast<v4f*>(&sums[wave][lists[wave][r]][(lane >> 4) * 4]);
        *s += acc[t];
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < a.N * kTile; i += kThreads) {
    const int t = i / kTile, c = i % kTile;
    if (c0 + c >= a.H) continue;
    float s = 0.0f;
#pragma unroll
    for (int v = 0; v < kDownWaves; ++v) s += sums[v][t][c];
    T* d = static_cast<T*>(a.y) + (int64_t)t * a.H + c0 + c;
    if constexpr (sizeof(T) == 2)
      *d = bf16_bits(s);
    else
      *d = s;
  }
}

template <typename T, bool W8, int NT>
hipError_t launch(const LayerArgs& a, hipStream_t s) {
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
  const int64_t tiles = std::min<int64_t>(a.E, (int64_t)a.N * a.k) * ((a.F + kActs - 1) / kActs);
  const unsigned up = (unsigned)std::min<int64_t>(tiles, (int64_t)occ * di.cu_count);
  hipLaunchKernelGGL((k_layer_up<T, W8, NT>), dim3(up), dim3(kUpWaves * kWave), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_layer_down<T, W8, NT>), dim3((unsigned)((a.H + kTile - 1) / kTile)), dim3(kDownWaves * kWave), 0,
                     s, a);
  return hipGetLastError();
}

template <typename T, bool W8>
hipError_t by_tokens(const LayerArgs& a, hipStream_t s) {
  return a.N <= 16 ? launch<T, W8, 1>(a, s) : a.N <= 32 ? launch<T, W8, 2>(a, s) : launch<T, W8, 4>(a, s);
}

}  // namespace

// The workspace: how many experts are chosen, the list of them, the activations.
int64_t expert_layer_bytes(do_dtype dt, int64_t N, int32_t E, int32_t k, int32_t F) {
  const int64_t rows = N * k;
  return 16 + std::min<int64_t>(E, rows) * (int64_t)sizeof(Chosen) + rows * layer_row(dt, F) * (dt == DO_F32 ? 4 : 2);
}

hipError_t launch_expert_layer(LayerArgs a, do_dtype dt, void* workspace, hipStream_t s) {
  char* ws = static_cast<char*>(workspace);
  a.n_chosen = reinterpret_cast<int32_t*>(ws);
  a.chosen = reinterpret_cast<Chosen*>(ws + 16);
  a.h = ws + 16 + std::min<int64_t>(a.E, (int64_t)a.N * a.k) * (int64_t)sizeof(Chosen);
  a.ldh = layer_row(dt, a.F);
  const bool w8 = a.w1_exp != nullptr;
  if (dt == DO_F32) return w8 ? by_tokens<float, true>(a, s) : by_tokens<float, false>(a, s);
  return w8 ? by_tokens<uint16_t, true>(a, s) : by_tokens<uint16_t, false>(a, s);
}

}  // namespace dol
