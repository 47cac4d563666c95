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
// is a population count below its lane.  A bit transpose gives each lane its
// token's experts, of which it then visits only those that are set.
//
// Bound by latency and launches up to some thousand tokens (64 tokens of 8 of 128
// experts: one block, 6.5 us).  Beyond, by a row's place: a choice counts up to eight
// words of LDS, those of neighbouring experts 64 bytes apart, so that four banks serve a
// wave (561,000 conflict cycles at 65,536 tokens), and each block first adds up the
// counts of all blocks.  65,536 tokens: 128 blocks, 5 us for the counts of their units and
// 45 us for the rows, whose three lists are 6.8 MB in memory.
#include <algorithm>
#include <atomic>

#include "experts.h"

namespace dol {
namespace {

constexpr int kRowThreads = 512;  // eight waves: the eight words of a unit
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// 64 x 64 bit transpose across the lanes of a wave: bit t of lane e's word becomes
// bit e of lane t's.  Six exchanges of blocks of 32, 16, .. 1 bits between the
// lanes that differ in that bit.
__device__ __forceinline__ u64 transpose_bits(u64 v) {
  const int lane = threadIdx.x & 63;
  constexpr u64 low[6] = {0x5555555555555555ull, 0x3333333333333333ull, 0x0F0F0F0F0F0F0F0Full,
                          0x00FF00FF00FF00FFull, 0x0000FFFF0000FFFFull, 0x00000000FFFFFFFFull};
#pragma unroll
  for (int b = 5; b >= 0; --b) {
    const int d = 1 << b;
    const u64 o = ((u64)(uint32_t)__shfl_xor((int)(uint32_t)(v >> 32), d) << 32) |
                  (uint32_t)__shfl_xor((int)(uint32_t)v, d);
    v = (lane & d) ? (v & ~low[b]) | ((o & ~low[b]) >> d) : (v & low[b]) | ((o & low[b]) << d);
  }
  return v;
}

// The masks of unit u: mask[e * 8 + w] = tokens of word w that chose e; and
// chosen(i, v): v = the experts 64 i .. 64 i + 63 that the lane's token chose.
// A token's choices past the k-th in expert order (never for Top-k signatures)
// and bits at or past N are left out, so no list can overflow.
template <typename F>
__device__ __forceinline__ void unit_masks(const u64* bits, int64_t u, int64_t N, int32_t E, int32_t k, u64* mask,
                                           F&& chosen) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t0 = u * 512 + w * 64;
  const u64 live = t0 >= N ? 0 : (N - t0 >= 64 ? ~u64(0) : (u64(1) << (N - t0)) - 1);
  int left = k;
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = e0 + lane;
    u64 mine = e < E && live != 0 ? bits[((u * E + e) << 3) + w] & live : 0;
    u64 ex = transpose_bits(mine);
    const int n = __popcll(ex);
    if (__ballot(n > left) != 0) {  // some token has too many: keep its first ones
      for (int i = n; i > left; --i) ex &= ~(u64(1) << (63 - __clzll((long long)ex)));
      mine = transpose_bits(ex);
    }
    left -= __popcll(ex);
    if (e < E) mask[e * 8 + w] = mine;
    chosen(e0, ex);
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
    unit_masks(bits, u, N, E, k, sm, [](int, u64) {});
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
  u64 ex[kMaxE / kWave];  // the experts of the lane's token
  auto keep = [&](int e0, u64 v) {
#pragma unroll
    for (int i = 0; i < kMaxE / kWave; ++i) ex[i] = e0 == i * kWave ? v : ex[i];
  };
  unit_masks(bits, u0, N, E, k, sm, keep);
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
      unit_masks(bits, u, N, E, k, sm, keep);
      __syncthreads();
    }
    const int64_t t = u * 512 + w * 64 + lane;
    int have = 0;
#pragma unroll
    for (int i = 0; i < kMaxE / kWave; ++i) {
      if (i * kWave < E) {
        u64 v = ex[i];
        while (v != 0) {
          const int e = i * kWave + __ffsll((long long)v) - 1;
          v &= v - 1;
          uint32_t r = next[e] + (uint32_t)__popcll(sm[e * 8 + w] & ((u64(1) << lane) - 1));
          for (int x = 0; x < w; ++x) r += (uint32_t)__popcll(sm[e * 8 + x]);
          row_token[r] = (int32_t)t;
          token_row[t * k + have] = (int32_t)r;
          token_expert[t * k + have] = e;
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
// once.  One element per thread; rows of any width and alignment (65,536 tokens of 8
// rows of 2,047 bf16: 1,369 us, 1.8 TB/s, in loads of two bytes).
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

// The same for rows of whole 16-byte pieces: one piece per thread, the k rows'
// pieces in flight together.  Bound by memory: 65,536 tokens of 8 rows of 2,048
// bf16 move 2.42 GB in 406 us (6.0 TB/s, nine tenths of it reads).
template <typename T>
__global__ __launch_bounds__(256) void k_combine_pieces(const v4u* o, const int32_t* token_row, int64_t N, int32_t k,
                                                        int64_t R, int32_t pieces, v4u* y) {
  constexpr int EL = 16 / (int)sizeof(T);
  const int64_t total = N * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t t = total <= 0xFFFFFFFFll ? (uint32_t)i / (uint32_t)pieces : i / pieces;
    const int64_t c = i - t * pieces;
    float s[EL];
#pragma unroll
    for (int v = 0; v < EL; ++v) s[v] = 0.0f;
    for (int j0 = 0; j0 < k; j0 += 8) {
      v4u x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int64_t r = j0 + j < k ? token_row[t * k + j0 + j] : -1;
        x[j] = r >= 0 && r < R ? __builtin_nontemporal_load(o + r * pieces + c) : v4u{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int v = 0; v < EL; ++v) {
          if constexpr (sizeof(T) == 4)
            s[v] += __uint_as_float(x[j][v]);
          else
            s[v] += bf16_float((uint16_t)(x[j][v >> 1] >> (16 * (v & 1))));
        }
    }
    v4u out;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int v = 0; v < 4; ++v) out[v] = __float_as_uint(s[v]);
    } else {
#pragma unroll
      for (int v = 0; v < 4; ++v) out[v] = bf16_pair(s[2 * v], s[2 * v + 1]);
    }
    __builtin_nontemporal_store(out, y + i);
  }
}

// dp[t][e] of the token's rows: the partial sums in order; zero elsewhere.
// A block takes T tokens: their rows of dp in LDS, zeroed, a thread for each of
// the tokens' experts, and the rows written as they lie in memory.
template <typename T>
__global__ __launch_bounds__(256) void k_expert_dp(const float* part, int32_t parts, int64_t R,
                                                   const int32_t* token_row, const int32_t* token_expert, int64_t N,
                                                   int32_t k, int32_t E, int32_t tokens, T* dp) {
  extern __shared__ float rows[];  // [tokens][E]
  const int64_t t0 = (int64_t)blockIdx.x * tokens;
  const int n = (int)min((int64_t)tokens, N - t0);
  for (int i = threadIdx.x; i < n * E; i += 256) rows[i] = 0.0f;
  __syncthreads();
  for (int i = threadIdx.x; i < n * k; i += 256) {
    const int64_t r = token_row[t0 * k + i];
    const int e = token_expert[t0 * k + i];
    if (r >= 0 && r < R && e >= 0 && e < E) {
      float v = 0.0f;
      for (int p = 0; p < parts; ++p) v += part[r * parts + p];
      rows[i / k * E + e] = v;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * E; i += 256) dp[t0 * E + i] = from_float<T>(rows[i]);
}

// The kernels' LDS limits, for any E and once per device: a limit set for one call could be too small for
// another thread's.
hipError_t allow_lds() {
  static std::atomic<bool> done[64];
  const int device = device_info().device;
  if (device < 0 || device >= 64) return hipErrorInvalidDevice;
  if (done[device].load(std::memory_order_acquire)) return hipSuccess;
  for (const void* kern : {reinterpret_cast<const void*>(k_row_counts), reinterpret_cast<const void*>(k_rows)}) {
    const hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, kMaxE * (64 + 4));
    if (e != hipSuccess) return e;
  }
  done[device].store(true, std::memory_order_release);
  return hipSuccess;
}

}  // namespace

hipError_t launch_expert_rows(const u64* bits, int64_t N, int32_t E, int32_t k, int32_t* offsets, int32_t* row_token,
                              int32_t* token_row, int32_t* token_expert, uint32_t* counts, hipStream_t s) {
  const int64_t U = (N + 511) / 512;
  const int64_t chunks = std::min<int64_t>(U, kRowChunks);
  const size_t masks = (size_t)E * 64, lds = masks + (size_t)E * 4;
  hipError_t e = allow_lds();
  if (e != hipSuccess) return e;
  if (U > 1) {
    hipLaunchKernelGGL(k_row_counts, dim3((unsigned)chunks), dim3(kRowThreads), masks, s, bits, N, E, k, counts);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_rows, dim3((unsigned)chunks), dim3(kRowThreads), lds, s, bits, N, E, k,
                     U > 1 ? counts : nullptr, offsets, row_token, token_row, token_expert);
  return hipGetLastError();
}

hipError_t launch_expert_combine(const void* o, do_dtype dt, const int32_t* token_row, int64_t N, int32_t k, int64_t R,
                                 int32_t H, void* y, hipStream_t s) {
  const int el = dt == DO_F32 ? 4 : 8;
  if (H % el == 0 && ((reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(y)) & 15) == 0) {
    const int32_t pieces = H / el;
    const dim3 grid((unsigned)std::min<int64_t>((N * pieces + 255) / 256, 1 << 20));
    if (dt == DO_F32)
      hipLaunchKernelGGL(k_combine_pieces<float>, grid, dim3(256), 0, s, static_cast<const v4u*>(o), token_row, N, k,
                         R, pieces, static_cast<v4u*>(y));
    else
      hipLaunchKernelGGL(k_combine_pieces<uint16_t>, grid, dim3(256), 0, s, static_cast<const v4u*>(o), token_row, N,
                         k, R, pieces, static_cast<v4u*>(y));
    return hipGetLastError();
  }
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
  const int tokens = std::max(1, std::min(256 / k, 8192 / E));  // about one expert a thread, 32 KiB at most
  const dim3 grid((unsigned)((N + tokens - 1) / tokens));
  const size_t lds = (size_t)tokens * E * sizeof(float);
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_expert_dp<float>, grid, dim3(256), lds, s, part, nparts, R, token_row, token_expert, N, k, E,
                       tokens, static_cast<float*>(dp));
  else
    hipLaunchKernelGGL(k_expert_dp<uint16_t>, grid, dim3(256), lds, s, part, nparts, R, token_row, token_expert, N, k,
                       E, tokens, static_cast<uint16_t*>(dp));
  return hipGetLastError();
}

}  // namespace dol
