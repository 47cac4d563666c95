// Products for a handful of rows (one token, few experts): the forward product
// and the gated activation.
//
// A row of x meets 16 rows at most, and there are too few tiles to fill the CUs:
// the time is that of one tile, which is that of its share of the weights coming
// from memory.  A block takes 64 rows of an expert's weights and up to 16 rows of
// x; its four waves take a quarter of the contraction each and feed the matrix
// instructions straight from memory, without LDS or barriers: lane l holds 16
// bytes of row l % 16, a 128-byte line of 16 rows in two loads, and all of a
// line's ten loads are issued before the last line's are used.  The four partial
// results meet in LDS.
//
// One token, 8 of 128 experts, 768 -> 2,048 bf16: 8.8 us, of which the 25 MB of
// weights take 5 at the rate of a copy; the rest is a tile's latency.
#include <algorithm>
#include <type_traits>

#include "expert_gemm.h"

namespace dol {
namespace expert {
namespace {

constexpr int kRows = 16;     // of x in a tile
constexpr int kCols = 64;     // rows of the weights in a tile
constexpr int kWaves = 4;
typedef float v4acc __attribute__((ext_vector_type(4)));

template <typename T>
__device__ __forceinline__ v4acc mul16(v4u a, v4u b, v4acc c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  }
}

template <typename T, int EPI, bool GQ>
__global__ __launch_bounds__(kWaves* kWave) void k_expert_skinny(const ExpertGemm g) {
  __shared__ int32_t first[kMaxE + 1];
  __shared__ __align__(16) float red[kWaves][kRows][kCols + 4];
  constexpr int EL = Mma<T>::kElems, LINE = 128 / (int)sizeof(T);
  constexpr int BPo = EPI == kSwiglu ? kCols / 2 : kCols;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int PT = (g.Pd + BPo - 1) / BPo;
  if (wave == 0) {
    int carry = 0;
    for (int e0 = 0; e0 < g.E; e0 += kWave) {
      const int e = e0 + lane;
      int n = 0;
      if (e < g.E) {
        const int b = clip_rows(g.offsets[e], g.R), c = clip_rows(g.offsets[e + 1], g.R);
        n = c > b ? (c - b + kRows - 1) / kRows * PT : 0;
      }
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(n, d);
        n += lane >= d ? o : 0;
      }
      if (e < g.E) first[e + 1] = carry + n;
      carry += __builtin_amdgcn_readlane(n, 63);
    }
    if (lane == 0) first[0] = 0;
  }
  __syncthreads();
  const int tile = blockIdx.x;
  if (tile >= __builtin_amdgcn_readfirstlane(first[g.E])) return;
  int e = 0;
  for (int e0 = 0; e0 < g.E; e0 += kWave)
    e += __popcll(__ballot(e0 + lane < g.E && first[e0 + lane + 1] <= tile));
  e = __builtin_amdgcn_readfirstlane(e);
  const int i = tile - first[e], p0 = i % PT * BPo;
  const int r0 = clip_rows(g.offsets[e], g.R) + i / PT * kRows;
  const int rows = min(kRows, clip_rows(g.offsets[e + 1], g.R) - r0);

  // lane l: row l % 16 of each 16 weight rows and of x, 16 bytes l / 16 of each half line
  const int row = lane & 15, at = (lane >> 4) * EL;
  int64_t xr = r0 + min(row, rows - 1);
  if constexpr (GQ) {
    xr = clip_token(g.q_token[xr], (int32_t)(g.N - 1));
  }
  const T* x = static_cast<const T*>(g.Q) + xr * g.ldq;
  const T* we = static_cast<const T*>(g.P) + (int64_t)e * (EPI == kSwiglu ? 2 * g.Pd : g.Pd) * g.ldp;
  const T* wr[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    int64_t r;
    if constexpr (EPI == kSwiglu)  // 32 gate rows, then the up rows beside them
      r = min(p0 + (t & 1) * 16 + row, g.Pd - 1) + (int64_t)(t >> 1) * g.Pd;
    else
      r = min(p0 + t * 16 + row, g.Pd - 1);
    wr[t] = we + r * g.ldp;
  }
  const int lines = (g.K + LINE - 1) / LINE;
  const int l0 = wave * lines / kWaves, l1 = (wave + 1) * lines / kWaves;
  v4acc acc[4] = {};
  struct Line {
    v4u w[4][2], x[2];
  };
  auto load = [&](int l) {
    Line n;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = l * LINE + h * (LINE / 2) + at;
      const int kk = k < g.K ? k : 0;  // past the end: any place inside, and x as zeros
#pragma unroll
      for (int t = 0; t < 4; ++t) n.w[t][h] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(wr[t] + kk));
      n.x[h] = *reinterpret_cast<const v4u*>(x + kk);
      if (k >= g.K) {
        n.x[h] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
        for (int t = 0; t < 4; ++t) n.w[t][h] = v4u{0u, 0u, 0u, 0u};
      }
    }
    return n;
  };
  if (l0 < l1) {
    Line cur = load(l0);
    for (int l = l0; l < l1; ++l) {
      Line nxt;
      if (l + 1 < l1) nxt = load(l + 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = mul16<T>(cur.w[t][h], cur.x[h], acc[t]);
      cur = nxt;
    }
  }
  // accumulator v of tile t: weight row 16 t + 4 (lane / 16) + v, row lane % 16 of x
#pragma unroll
  for (int t = 0; t < 4; ++t) *reinterpret_cast<v4acc*>(&red[wave][row][t * 16 + (lane >> 4) * 4]) = acc[t];
  __syncthreads();
  const int orow = tid >> 4;  // 16 threads a row
  const int64_t r = r0 + orow;
  const bool live = orow < rows;
  if constexpr (EPI == kStore) {
    const int c = (tid & 15) * 4, n = min(4, g.Pd - p0 - c);
    v4f s = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) s += *reinterpret_cast<const v4f*>(&red[w][orow][c]);
    if (live && n > 0) store_four<T>(static_cast<T*>(g.out) + r * g.Pd + p0 + c, s, n, g.vec_out);
  } else {
    const int F = g.Pd, G = (F + kAct8Group - 1) / kAct8Group;
    const int c = (tid & 15) * 2, n = min(2, F - p0 - c);
    float a[2][2] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int v = 0; v < 2; ++v) a[half][v] += red[w][orow][half * 32 + c + v];
    const float p = live ? row_prob(g, r, e) : 0.0f;
    if (live) {
      T* h = static_cast<T*>(g.out) + r * F + p0 + c;
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        if (v >= n) continue;
        const float s = p * (a[0][v] * sigmoid(a[0][v])) * a[1][v];
        if constexpr (sizeof(T) == 2)
          h[v] = bf16_bits(s);
        else
          h[v] = s;
      }
    }
    if (g.q8 != nullptr) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        float z[4] = {n > 0 ? a[half][0] : 0.0f, n > 1 ? a[half][1] : 0.0f, 0.0f, 0.0f};
        uint32_t m = max(__float_as_uint(z[0]) & 0x7FFFFFFFu, __float_as_uint(z[1]) & 0x7FFFFFFFu);
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
        const uint32_t byte = act8_exponent(m);
        const uint32_t q = act8_round4(z, act8_inverse(byte), byte);
        if (live) {
          int8_t* d = g.q8 + (r * 2 + half) * F + p0 + c;
          if (n > 0) d[0] = (int8_t)q;
          if (n > 1) d[1] = (int8_t)(q >> 8);
          if (c == 0) g.e8[(r * 2 + half) * G + p0 / 32] = (uint8_t)byte;
        }
      }
    }
  }
}

template <typename T, int EPI, bool GQ>
hipError_t launch(const ExpertGemm& g, hipStream_t s) {
  constexpr int BPo = EPI == kSwiglu ? kCols / 2 : kCols;
  const int64_t PT = (g.Pd + BPo - 1) / BPo, tiles = PT * (g.R / kRows + std::min<int64_t>(g.E, g.R));
  if (tiles >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_expert_skinny<T, EPI, GQ>), dim3((unsigned)tiles), dim3(kWaves * kWave), 0, s, g);
  return hipGetLastError();
}

}  // namespace
}  // namespace expert

hipError_t launch_expert_skinny(const ExpertGemm& g, do_dtype dt, bool swiglu, hipStream_t s) {
  using namespace expert;
  if (swiglu) return dt == DO_F32 ? launch<float, kSwiglu, true>(g, s) : launch<uint16_t, kSwiglu, true>(g, s);
  if (g.q_token != nullptr)
    return dt == DO_F32 ? launch<float, kStore, true>(g, s) : launch<uint16_t, kStore, true>(g, s);
  return dt == DO_F32 ? launch<float, kStore, false>(g, s) : launch<uint16_t, kStore, false>(g, s);
}

}  // namespace dol
