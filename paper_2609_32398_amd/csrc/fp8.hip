// 8-bit floating point: e4m3 values whose blocks share a power of two.  128 consecutive elements of a row are a block
// (weights: 128 x 128 of a matrix; the last block of a row or column may be short) with the least 2^e, e >= -120,
// that leaves them within 448, and each element is x 2^-e rounded to the nearest e4m3 value, ties to even.  x 2^-e is
// exact where it is not so small that it rounds to 0, so there is one rounding; q 2^e is exact in bf16 (4 significant
// bits, down to 2^-129).  A block with an infinity or NaN has exponent byte 255, zeros for values, and reads as NaN.
//
// Streaming passes bound by memory: 65,536 x 2,048 bf16 move 405 MB each way, packed in 70 us and unpacked in 69 (5.8
// TB/s); weights of 128 x 1,536 x 2,048 bf16 packed in 203 us (6.0 TB/s).  Rows of any width take the same path with
// loads of any alignment: 65,536 x 2,047 packed in 111 us and unpacked in 128.  37 x 1,001 fp32: 3.1 and 2.9 us.
#include <algorithm>

#include "experts.h"

namespace dol {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
constexpr int kThreads = 256;
constexpr int kPiece = 8;                        // elements of a thread's piece
constexpr int kLanes = kFp8Block / kPiece;       // threads of a row's block
constexpr int kRowsAtOnce = kThreads / kLanes;   // rows of a block of weights in one step

// Eight elements as they lie in memory.
template <typename T>
struct Raw {
  v4u v[sizeof(T) / 2];
  __device__ __forceinline__ float at(int i) const {
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(v[i >> 2][i & 3]);
    else
      return __uint_as_float((i & 1) ? v[0][i >> 1] & 0xFFFF0000u : v[0][i >> 1] << 16);
  }
  __device__ __forceinline__ uint32_t largest() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) m = max(m, __float_as_uint(at(i)) & 0x7FFFFFFFu);
    return m;
  }
};

// The first n of eight elements at p, of any alignment to whole elements; the others are zeros.
template <typename T, bool WHOLE>
__device__ __forceinline__ Raw<T> load_piece(const T* p, int n) {
  Raw<T> r;
  if (WHOLE || n >= kPiece) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
      if constexpr (WHOLE)
        r.v[i] = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p) + i);
      else
        __builtin_memcpy(&r.v[i], reinterpret_cast<const char*>(p) + 16 * i, 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.v[i] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
      if (i < n) {
        if constexpr (sizeof(T) == 4)
          r.v[i >> 2][i & 3] = __float_as_uint(p[i]);
        else
          r.v[0][i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
      }
  }
  return r;
}

template <typename T, bool WHOLE>
__device__ __forceinline__ void store_piece(uint8_t* q, const Raw<T>& r, int n, uint32_t byte) {
  const float inv = fp8_inverse(byte);
  const v2u o{fp8_round4(r.at(0) * inv, r.at(1) * inv, r.at(2) * inv, r.at(3) * inv, byte),
              fp8_round4(r.at(4) * inv, r.at(5) * inv, r.at(6) * inv, r.at(7) * inv, byte)};
  if (WHOLE) {
    __builtin_nontemporal_store(o, reinterpret_cast<v2u*>(q));
  } else if (n >= kPiece) {
    __builtin_memcpy(q, &o, 8);
  } else {
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
      if (i < n) q[i] = (uint8_t)(o[i >> 2] >> (8 * (i & 3)));
  }
}

// Rows: 16 threads a block.  WHOLE: rows of whole blocks at aligned addresses, so that blocks are consecutive.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_fp8_pack(const T* x, int64_t blocks, int32_t W, int32_t G, uint8_t* q,
                                                      uint8_t* e) {
  const int lane = threadIdx.x % kLanes;
  const int64_t step = (int64_t)gridDim.x * kRowsAtOnce;
  for (int64_t b = (int64_t)blockIdx.x * kRowsAtOnce + threadIdx.x / kLanes; b < blocks; b += step) {
    int64_t at = b * kFp8Block;
    int n = kPiece;
    if constexpr (!WHOLE) {
      const int64_t row = (b >> 32) ? b / G : (int64_t)((uint32_t)b / (uint32_t)G);
      const int c = (int)(b - row * G) * kFp8Block;
      n = W - c - lane * kPiece;
      at = row * W + c;
    }
    at += lane * kPiece;
    const Raw<T> r = load_piece<T, WHOLE>(x + at, n);
    uint32_t m = r.largest();
#pragma unroll
    for (int d = 1; d < kLanes; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    const uint32_t byte = fp8_exponent(m);
    store_piece<T, WHOLE>(q + at, r, n, byte);
    if (lane == 0) e[b] = (uint8_t)byte;
  }
}

// Weights: a block of threads takes a block of 128 x 128, held in registers between its largest magnitude and its
// rounding.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_fp8_pack_weights(const T* x, int64_t blocks, int32_t O, int32_t I, int32_t OB,
                                                              int32_t IB, uint8_t* q, uint8_t* e) {
  constexpr int N = kFp8Block / kRowsAtOnce;
  __shared__ uint32_t top[kThreads / kWave];
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int64_t mat = b / ((int64_t)OB * IB);
    const int in = (int)(b - mat * OB * IB), o0 = in / IB * kFp8Block, c0 = in % IB * kFp8Block;
    const int c = c0 + threadIdx.x % kLanes * kPiece, o = o0 + threadIdx.x / kLanes;
    const int64_t base = mat * O * I + c;
    const int n = I - c;
    Raw<T> r[N];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = o + i * kRowsAtOnce;
      r[i] = WHOLE || row < O ? load_piece<T, WHOLE>(x + base + (int64_t)row * I, n) : Raw<T>{};
    }
#pragma unroll
    for (int i = 0; i < N; ++i) m = max(m, r[i].largest());
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    __syncthreads();  // the last block's largest has been read
    if (threadIdx.x % kWave == 0) top[threadIdx.x / kWave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kThreads / kWave; ++i) m = max(m, top[i]);
    const uint32_t byte = fp8_exponent(m);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = o + i * kRowsAtOnce;
      if (WHOLE || row < O) store_piece<T, WHOLE>(q + base + (int64_t)row * I, r[i], n, byte);
    }
    if (threadIdx.x == 0) e[b] = (uint8_t)byte;
  }
}

__device__ __forceinline__ void fp8_values4(uint32_t q, float s, float* v) {
  typedef float v2f __attribute__((ext_vector_type(2)));
  const v2f lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  v[0] = lo[0] * s;
  v[1] = lo[1] * s;
  v[2] = hi[0] * s;
  v[3] = hi[1] * s;
}

// Back: a thread writes 16 bytes, so that a wave's stores are one run (with 16 elements a thread, in two stores, 65,536 x
// 2,048 bf16 took 98 us).  OB: 128 rows share an exponent (weights; 0: each row has its own).
template <typename T, bool WHOLE>
__global__ __launch_bounds__(kThreads) void k_fp8_unpack(const uint8_t* q, const uint8_t* e, int64_t pieces, int32_t P,
                                                        int32_t O, int32_t OB, int32_t I, int32_t G, T* x) {
  constexpr int EL = 16 / (int)sizeof(T);
  const int64_t step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < pieces; i += step) {
    const int64_t row = (i >> 32) ? i / P : (int64_t)((uint32_t)i / (uint32_t)P);
    const int c = (int)(i - row * P) * EL, n = I - c;
    int64_t er = row;
    if (OB) {
      const int64_t mat = (row >> 32) ? row / O : (int64_t)((uint32_t)row / (uint32_t)O);
      er = mat * OB + (row - mat * O) / kFp8Block;
    }
    const uint8_t* src = q + row * I + c;
    T* dst = x + row * I + c;
    uint32_t w[EL / 4] = {};
    if (WHOLE || n >= EL) {
      if constexpr (WHOLE && EL == 8) {
        const v2u v = __builtin_nontemporal_load(reinterpret_cast<const v2u*>(src));
        w[0] = v[0];
        w[1] = v[1];
      } else if constexpr (WHOLE) {
        w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(src));
      } else {
        __builtin_memcpy(w, src, EL);
      }
    } else {
#pragma unroll
      for (int k = 0; k < EL; ++k)
        if (k < n) w[k >> 2] |= (uint32_t)src[k] << (8 * (k & 3));
    }
    const float s = fp8_scale(e[er * G + c / kFp8Block]);
    float v[EL];
#pragma unroll
    for (int k = 0; k < EL / 4; ++k) fp8_values4(w[k], s, v + 4 * k);
    if (WHOLE || n >= EL) {
      v4u o;
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        if constexpr (sizeof(T) == 4)
          o[d] = __float_as_uint(v[d]);
        else
          o[d] = bf16_pair(v[2 * d], v[2 * d + 1]);
      }
      if constexpr (WHOLE)
        __builtin_nontemporal_store(o, reinterpret_cast<v4u*>(dst));
      else
        __builtin_memcpy(dst, &o, 16);
    } else {
#pragma unroll
      for (int k = 0; k < EL; ++k)
        if (k < n) {
          if constexpr (sizeof(T) == 4)
            dst[k] = v[k];
          else
            dst[k] = bf16_bits(v[k]);
        }
    }
  }
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename T>
hipError_t pack(const T* x, int64_t mats, int64_t O, int32_t I, bool weights, uint8_t* q, uint8_t* e, hipStream_t s) {
  const int32_t G = (I + kFp8Block - 1) / kFp8Block;
  const bool whole = aligned16(x) && aligned16(q) && I % kFp8Block == 0 && (!weights || O % kFp8Block == 0);
  if (weights) {
    const int64_t OB = (O + kFp8Block - 1) / kFp8Block, blocks = mats * OB * G;
    auto* kern = whole ? k_fp8_pack_weights<T, true> : k_fp8_pack_weights<T, false>;
    hipLaunchKernelGGL(kern, dim3((unsigned)std::min<int64_t>(blocks, 1 << 20)), dim3(kThreads), 0, s, x,
                       blocks, (int32_t)O, I, (int32_t)OB, G, q, e);
  } else {
    const int64_t blocks = mats * O * G;
    auto* kern = whole ? k_fp8_pack<T, true> : k_fp8_pack<T, false>;
    const dim3 grid((unsigned)std::min<int64_t>((blocks + kRowsAtOnce - 1) / kRowsAtOnce, 1 << 20));
    hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, x, blocks, I, G, q, e);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t unpack(const uint8_t* q, const uint8_t* e, int64_t mats, int64_t O, int32_t I, bool weights, T* x,
                  hipStream_t s) {
  constexpr int EL = 16 / (int)sizeof(T);
  const int32_t G = (I + kFp8Block - 1) / kFp8Block, P = (I + EL - 1) / EL;
  const int64_t pieces = mats * O * P;
  const bool whole = aligned16(x) && aligned16(q) && I % EL == 0;
  auto* kern = whole ? k_fp8_unpack<T, true> : k_fp8_unpack<T, false>;
  const dim3 grid((unsigned)std::min<int64_t>((pieces + kThreads - 1) / kThreads, 1 << 20));
  hipLaunchKernelGGL(kern, grid, dim3(kThreads), 0, s, q, e, pieces, P, weights ? (int32_t)O : 0,
                     weights ? (int32_t)((O + kFp8Block - 1) / kFp8Block) : 0, I, G, x);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_pack(const void* x, do_dtype dt, int64_t mats, int64_t O, int32_t I, bool weights, uint8_t* q,
                           uint8_t* e, hipStream_t s) {
  return dt == DO_F32 ? pack(static_cast<const float*>(x), mats, O, I, weights, q, e, s)
                      : pack(static_cast<const uint16_t*>(x), mats, O, I, weights, q, e, s);
}

hipError_t launch_fp8_unpack(const uint8_t* q, const uint8_t* e, int64_t mats, int64_t O, int32_t I, bool weights,
                             void* x, do_dtype dt, hipStream_t s) {
  return dt == DO_F32 ? unpack(q, e, mats, O, I, weights, static_cast<float*>(x), s)
                      : unpack(q, e, mats, O, I, weights, static_cast<uint16_t*>(x), s);
}

}  // namespace dol
