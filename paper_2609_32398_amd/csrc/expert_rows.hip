// Rows by expert from the load signatures, and the sum of the experts' outputs
// over each token's rows.
//
// A token t of expert e is a row; the rows are ordered by expert and then by
// token, so the row of (t, e) is
//   offsets[e] + #{t' < t : f_e(t') = 1},
// a prefix count over the signature of e.  The signatures come in units of 512
// tokens, so one block takes whole units and one wave takes one 64-token word
// position of a unit: lane l is token 64 w + l, the word of an expert is the
// wave's mask of the tokens that chose it, and the place of a token among them
// is a population count below its lane.
//
// Bound by latency and launches up to some thousand tokens; beyond, by the
// scattered 4-byte stores of the three lists (12 N k bytes).
#include <algorithm>

#include "experts.h"

namespace dol {
namespace {

constexpr int kRowThreads = 512;  // eight waves: the eight words of a unit

__device__ __forceinline__ u64 lane_word(u64 v, int i) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, i);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), i);
  return ((u64)hi << 32) | lo;
}

// The masks of unit u: mask[e * 8 + w] = tokens of word w that chose e.  A
// token's choices past the k-th in expert order (never for Top-k signatures)
// and bits at or past N are left out, so no list can overflow.
__device__ __forceinline__ void unit_masks(const u64* bits, int64_t u, int64_t N, int32_t E, int32_t k, u64* mask) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = u * 512 + w * 64;
  const u64 live = t0 >= N ? 0 : (N - t0 >= 64 ? ~u64(0) : (u64(1) << (N - t0)) - 1);
  int have = 0;
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = e0 + lane;
    u64 mine = e < E && live != 0 ? bits[((u * E + e) << 3) + w] & live : 0;
    const int n = min(kWave, E - e0);
    for (int i = 0; i < n; ++i) {
      const u64 m = lane_word(mine, i);
      if (m == 0) continue;
      const bool take = ((m >> lane) & 1) != 0 && have < k;
      const u64 got = __ballot(take);
      have += take;
      if (got != m && lane == i) mine = got;
    }
    if (e < E) mask[e * 8 + w] = mine;
  }
}

// counts[c][e]: tokens of chunk c (units c U / C ..) with a row for e.
__global__ __launch_bounds__(kRowThreads) void k_row_counts(const u64* bits, int64_t N, int32_t E, int32_t k,
                                                            uint32_t* counts) {
  extern __shared__ u64 sm[];  // E * 8 masks
  const int64_t U = (N + 511) >> 9;
  const int64_t u0 = (int64_t)blockIdx.x * U / gridDim.x, u1 = (int64_t)(blockIdx.x + 1) * U / gridDim.x;
  uint32_t c[kMaxE / kRowThreads] = {};
  for (int64_t u = u0; u < u1; ++u) {
    unit_masks(bits, u, N, E, k, sm);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxE / kRowThreads; ++i) {
      const int e = threadIdx.x + i * kRowThreads;
      if (e < E)
        for (int w = 0; w < 8; ++w) c[i] += (uint32_t)__popcll(sm[e * 8 + w]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kMaxE / kRowThreads; ++i) {
    const int e = threadIdx.x + i * kRowThreads;
    if (e < E) counts[(int64_t)blockIdx.x * E + e] = c[i];
  }
}

// One block per chunk.  counts: of every chunk (k_row_counts); nullptr: one
// chunk of one unit, whose counts are taken here.
__global__ __launch_bounds__(kRowThreads) void k_rows(const u64* bits, int64_t N, int32_t E, int32_t k,
                                                      const uint32_t* counts, int32_t* offsets, int32_t* row_token,
                                                      int32_t* token_row, int32_t* token_expert) {
  extern __shared__ u64 sm[];  // E * 8 masks, then E next rows
  uint32_t* next = reinterpret_cast<uint32_t*>(sm + (size_t)E * 8);
  __shared__ uint32_t wsum[kRowThreads / kWave];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t U = (N + 511) >> 9;
  const int64_t u0 = (int64_t)blockIdx.x * U / gridDim.x, u1 = (int64_t)(blockIdx.x + 1) * U / gridDim.x;
  unit_masks(bits, u0, N, E, k, sm);
  __syncthreads();
  // loads of thread t's experts t, t + 512, and the rows that earlier chunks take of them
  uint32_t load[kMaxE / kRowThreads] = {}, before[kMaxE / kRowThreads] = {};
#pragma unroll
  for (int i = 0; i < kMaxE / kRowThreads; ++i) {
    const int e = threadIdx.x + i * kRowThreads;
    if (e < E) {
      if (counts == nullptr) {
        for (int v = 0; v < 8; ++v) load[i] += (uint32_t)__popcll(sm[e * 8 + v]);
      } else {
        for (int c = 0; c < (int)gridDim.x; ++c) {
          const uint32_t n = counts[(int64_t)c * E + e];
          load[i] += n;
          before[i] += c < (int)blockIdx.x ? n : 0u;
        }
      }
    }
  }
  // exclusive sum over the experts
  uint32_t carry = 0;
#pragma unroll
  for (int i = 0; i < kMaxE / kRowThreads; ++i) {
    uint32_t s = load[i];
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) {
      const uint32_t o = (uint32_t)__shfl_up((int)s, d);
      s += lane >= d ? o : 0u;
    }
    if (lane == 63) wsum[w] = s;
    __syncthreads();
    uint32_t base = carry, all = 0;
    for (int v = 0; v < kRowThreads / kWave; ++v) {
      base += v < w ? wsum[v] : 0u;
      all += wsum[v];
    }
    carry += all;
    const int e = threadIdx.x + i * kRowThreads;
    if (e < E) {
      next[e] = base + s - load[i] + before[i];
      if (blockIdx.x == 0) {
        offsets[e] = (int32_t)(base + s - load[i]);
        if (e == E - 1) offsets[E] = (int32_t)(base + s);
      }
    }
    __syncthreads();
  }
  for (int64_t u = u0; u < u1; ++u) {
    if (u != u0) {
      unit_masks(bits, u, N, E, k, sm);
      __syncthreads();
    }
    const int64_t t = u * 512 + w * 64 + lane;
    int have = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane;
      u64 mine = 0;
      uint32_t at = 0;
      if (e < E) {
        mine = sm[e * 8 + w];
        at = next[e];
        for (int v = 0; v < 8; ++v) at += v < w ? (uint32_t)__popcll(sm[e * 8 + v]) : 0u;
      }
      const int n = min(kWave, E - e0);
      for (int i = 0; i < n; ++i) {
        const u64 m = lane_word(mine, i);
        if (m == 0) continue;
        const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)at, i);
        if ((m >> lane) & 1) {
          const uint32_t r = first + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
          row_token[r] = (int32_t)t;
          token_row[t * k + have] = (int32_t)r;
          token_expert[t * k + have] = e0 + i;
          ++have;
        }
      }
    }
    if (t < N)
      for (; have < k; ++have) {
        token_row[t * k + have] = -1;
        token_expert[t * k + have] = -1;
      }
    if (u + 1 < u1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kMaxE / kRowThreads; ++i) {
        const int e = threadIdx.x + i * kRowThreads;
        if (e < E)
          for (int v = 0; v < 8; ++v) next[e] += (uint32_t)__popcll(sm[e * 8 + v]);
      }
      __syncthreads();
    }
  }
}

template <typename T>
__device__ __forceinline__ float as_float(T v);
template <>
__device__ __forceinline__ float as_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float as_float<uint16_t>(uint16_t v) { return bf16_float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ uint16_t from_float<uint16_t>(float v) { return bf16_bits(v); }

// y[t] = sum over the token's rows of o[row], in expert order, in fp32, rounded
// once.  One element per thread; rows of any width and alignment.
template <typename T>
__global__ __launch_bounds__(256) void k_combine(const T* o, const int32_t* token_row, int64_t N, int32_t k, int64_t R,
                                                 int32_t H, T* y) {
  for (int64_t t = blockIdx.x; t < N; t += gridDim.x) {
    for (int c = blockIdx.y * 256 + threadIdx.x; c < H; c += gridDim.y * 256) {
      float s = 0.0f;
      for (int j = 0; j < k; ++j) {
        const int64_t r = token_row[t * k + j];
        if (r >= 0 && r < R) s += as_float<T>(o[r * H + c]);
      }
      y[t * H + c] = from_float<T>(s);
    }
  }
}

// dp[t][e] of the token's rows: the partial sums in order; zero elsewhere.
template <typename T>
__global__ __launch_bounds__(256) void k_expert_dp(const float* part, int32_t nparts, int64_t R,
                                                   const int32_t* token_row, const int32_t* token_expert, int64_t N,
                                                   int32_t k, int32_t E, T* dp) {
  const int lane = threadIdx.x & 63;
  for (int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); t < N; t += (int64_t)gridDim.x * 4) {
    // lane j holds the token's j-th row and expert, 64 at a time; the wave then
    // writes the row of dp, each lane looking its columns up among them
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane;
      float v = 0.0f;
      for (int j = 0; j < k; ++j) {
        const int64_t r = token_row[t * k + j];
        const int te = token_expert[t * k + j];
        if (te == e && r >= 0 && r < R) {
          v = 0.0f;
          for (int i = 0; i < nparts; ++i) v += part[(int64_t)i * R + r];
        }
      }
      if (e < E) dp[t * E + e] = from_float<T>(v);
    }
  }
}

}  // namespace

hipError_t launch_expert_rows(const u64* bits, int64_t N, int32_t E, int32_t k, int32_t* offsets, int32_t* row_token,
                              int32_t* token_row, int32_t* token_expert, uint32_t* counts, hipStream_t s) {
  const int64_t U = (N + 511) / 512;
  const int64_t chunks = std::min<int64_t>(U, kRowChunks);
  const size_t masks = (size_t)E * 64, lds = masks + (size_t)E * 4;
  hipError_t e;
  if ((e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_rows), hipFuncAttributeMaxDynamicSharedMemorySize,
                               (int)lds)) != hipSuccess)
    return e;
  if (U > 1) {
    if ((e = hipFuncSetAttribute(reinterpret_cast<const void*>(k_row_counts),
                                 hipFuncAttributeMaxDynamicSharedMemorySize, (int)masks)) != hipSuccess)
      return e;
    hipLaunchKernelGGL(k_row_counts, dim3((unsigned)chunks), dim3(kRowThreads), masks, s, bits, N, E, k, counts);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_rows, dim3((unsigned)chunks), dim3(kRowThreads), lds, s, bits, N, E, k,
                     U > 1 ? counts : nullptr, offsets, row_token, token_row, token_expert);
  return hipGetLastError();
}

hipError_t launch_expert_combine(const void* o, do_dtype dt, const int32_t* token_row, int64_t N, int32_t k, int64_t R,
                                 int32_t H, void* y, hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>(N, 65536), (unsigned)((H + 255) / 256));
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_combine<float>, grid, dim3(256), 0, s, static_cast<const float*>(o), token_row, N, k, R, H,
                       static_cast<float*>(y));
  else
    hipLaunchKernelGGL(k_combine<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t*>(o), token_row, N, k,
                       R, H, static_cast<uint16_t*>(y));
  return hipGetLastError();
}

hipError_t launch_expert_dp(const float* part, int32_t nparts, int64_t R, const int32_t* token_row,
                            const int32_t* token_expert, int64_t N, int32_t k, int32_t E, void* dp, do_dtype dt,
                            hipStream_t s) {
  const dim3 grid((unsigned)std::min<int64_t>((N + 3) / 4, 65536));
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_expert_dp<float>, grid, dim3(256), 0, s, part, nparts, R, token_row, token_expert, N, k, E,
                       static_cast<float*>(dp));
  else
    hipLaunchKernelGGL(k_expert_dp<uint16_t>, grid, dim3(256), 0, s, part, nparts, R, token_row, token_expert, N, k,
                       E, static_cast<uint16_t*>(dp));
  return hipGetLastError();
}

}  // namespace dol
