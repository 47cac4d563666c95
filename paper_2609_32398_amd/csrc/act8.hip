// Activations in 8 bits: 32 consecutive elements of a row share a power of two
// 2^e, the smallest (2^-126 at least) that leaves them within 127, and each is
// q = x 2^-e rounded to the nearest integer, ties to even.  x 2^-e is exact, so
// there is one rounding, and q 2^e has 7 significant bits: it is exact in bf16
// too.  A group with an infinity or NaN has exponent byte 255 and reads as NaN.
//
// Both directions are streaming passes bound by memory: 65,536 x 2,048 bf16
// move 407 MB each way, packed in 71 us (5.7 TB/s) and unpacked in 66 us.  Rows of
// any width go element by element: 65,536 x 2,047 packed in 283 us and unpacked in 245.
#include <algorithm>

#include "experts.h"

namespace dol {
namespace {

typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));

template <typename T>
__device__ __forceinline__ float load_elem(const T* p);
template <>
__device__ __forceinline__ float load_elem<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float load_elem<uint16_t>(const uint16_t* p) { return bf16_float(*p); }

// A half-wave per group, one element per lane: any width and alignment.
template <typename T>
__global__ __launch_bounds__(256) void k_act8_pack(const T* x, int64_t rows, int32_t W, int32_t G, int8_t* q,
                                                   uint8_t* e) {
  const int lane = threadIdx.x & 31;
  const int64_t groups = rows * G, step = (int64_t)gridDim.x * 8;
  for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += step) {
    const int64_t row = g / G;
    const int c = (int)(g - row * G) * kAct8Group + lane;
    const float v = c < W ? load_elem<T>(x + row * W + c) : 0.0f;
    uint32_t m = __float_as_uint(v) & 0x7FFFFFFFu;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    const uint32_t byte = act8_exponent(m);
    const float one[4] = {v, 0.0f, 0.0f, 0.0f};
    if (c < W) q[row * W + c] = (int8_t)act8_round4(one, act8_inverse(byte), byte);
    if (lane == 0) e[g] = (uint8_t)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_act8_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int32_t W,
                                                     int32_t G, T* x) {
  const int lane = threadIdx.x & 31;
  const int64_t groups = rows * G, step = (int64_t)gridDim.x * 8;
  for (int64_t g = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); g < groups; g += step) {
    const int64_t row = g / G;
    const int c = (int)(g - row * G) * kAct8Group + lane;
    if (c < W) {
      const float v = (float)q[row * W + c] * act8_scale(e[g]);
      if constexpr (sizeof(T) == 4)
        x[row * W + c] = v;
      else
        x[row * W + c] = bf16_bits(v);
    }
  }
}

// Rows of whole groups (W a multiple of 32, so that groups are consecutive in
// memory) at 16-byte aligned addresses.  Four lanes take a group, eight elements
// each.
template <typename T>
__global__ __launch_bounds__(256) void k_act8_pack_pieces(const T* x, int64_t groups, int8_t* q, uint8_t* e) {
  const int64_t n = groups * 4, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {  // n and step are multiples of 4
    float v[8];
    if constexpr (sizeof(T) == 4) {
      const v4u a = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(x) + 2 * i);
      const v4u b = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(x) + 2 * i + 1);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        v[c] = __uint_as_float(a[c]);
        v[4 + c] = __uint_as_float(b[c]);
      }
    } else {
      const v4u a = __builtin_nontemporal_load(reinterpret_cast<const v4u*>(x) + i);
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] = bf16_float((uint16_t)(a[c >> 1] >> (16 * (c & 1))));
    }
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) m = max(m, __float_as_uint(v[c]) & 0x7FFFFFFFu);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    m = max(m, (uint32_t)__shfl_xor((int)m, 2));
    const uint32_t byte = act8_exponent(m);
    const float inv = act8_inverse(byte);
    const v2u out = v2u{act8_round4(v, inv, byte), act8_round4(v + 4, inv, byte)};
    __builtin_nontemporal_store(out, reinterpret_cast<v2u*>(q) + i);
    if ((i & 3) == 0) e[i >> 2] = (uint8_t)byte;
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_act8_unpack_pieces(const int8_t* q, const uint8_t* e, int64_t groups, T* x) {
  const int64_t n = groups * 4, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
    const v2u a = __builtin_nontemporal_load(reinterpret_cast<const v2u*>(q) + i);
    const float s = act8_scale(e[i >> 2]);
    float v[8];
    act8_values4(a[0], s, v);
    act8_values4(a[1], s, v + 4);
    if constexpr (sizeof(T) == 4) {
      v4u b, c;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        b[k] = __float_as_uint(v[k]);
        c[k] = __float_as_uint(v[4 + k]);
      }
      __builtin_nontemporal_store(b, reinterpret_cast<v4u*>(x) + 2 * i);
      __builtin_nontemporal_store(c, reinterpret_cast<v4u*>(x) + 2 * i + 1);
    } else {
      v4u b;
#pragma unroll
      for (int k = 0; k < 4; ++k) b[k] = bf16_pair(v[2 * k], v[2 * k + 1]);
      __builtin_nontemporal_store(b, reinterpret_cast<v4u*>(x) + i);
    }
  }
}

bool whole_groups(const void* x, const int8_t* q, int32_t W) {
  return W % kAct8Group == 0 && (reinterpret_cast<uintptr_t>(x) & 15) == 0 && (reinterpret_cast<uintptr_t>(q) & 7) == 0;
}

}  // namespace

hipError_t launch_act8_pack(const void* x, do_dtype dt, int64_t rows, int32_t W, int8_t* q, uint8_t* e,
                            hipStream_t s) {
  const int32_t G = (W + kAct8Group - 1) / kAct8Group;
  if (whole_groups(x, q, W)) {
    const dim3 grid((unsigned)std::min<int64_t>((rows * G + 63) / 64, 1 << 20));
    if (dt == DO_F32)
      hipLaunchKernelGGL(k_act8_pack_pieces<float>, grid, dim3(256), 0, s, static_cast<const float*>(x), rows * G, q,
                         e);
    else
      hipLaunchKernelGGL(k_act8_pack_pieces<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t*>(x),
                         rows * G, q, e);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)std::min<int64_t>((rows * G + 7) / 8, 1 << 16));
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_act8_pack<float>, grid, dim3(256), 0, s, static_cast<const float*>(x), rows, W, G, q, e);
  else
    hipLaunchKernelGGL(k_act8_pack<uint16_t>, grid, dim3(256), 0, s, static_cast<const uint16_t*>(x), rows, W, G, q,
                       e);
  return hipGetLastError();
}

hipError_t launch_act8_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int32_t W, void* x, do_dtype dt,
                              hipStream_t s) {
  const int32_t G = (W + kAct8Group - 1) / kAct8Group;
  if (whole_groups(x, q, W)) {
    const dim3 grid((unsigned)std::min<int64_t>((rows * G + 63) / 64, 1 << 20));
    if (dt == DO_F32)
      hipLaunchKernelGGL(k_act8_unpack_pieces<float>, grid, dim3(256), 0, s, q, e, rows * G, static_cast<float*>(x));
    else
      hipLaunchKernelGGL(k_act8_unpack_pieces<uint16_t>, grid, dim3(256), 0, s, q, e, rows * G,
                         static_cast<uint16_t*>(x));
    return hipGetLastError();
  }
  const dim3 grid((unsigned)std::min<int64_t>((rows * G + 7) / 8, 1 << 16));
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_act8_unpack<float>, grid, dim3(256), 0, s, q, e, rows, W, G, static_cast<float*>(x));
  else
    hipLaunchKernelGGL(k_act8_unpack<uint16_t>, grid, dim3(256), 0, s, q, e, rows, W, G, static_cast<uint16_t*>(x));
  return hipGetLastError();
}

}  // namespace dol
