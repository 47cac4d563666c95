// Activations in 8 bits: 32 consecutive elements of a row share a power of two
// 2^e, the smallest (2^-126 at least) that leaves them within 127, and each is
// q = x 2^-e rounded to the nearest integer, ties to even.  x 2^-e is exact, so
// there is one rounding, and q 2^e has 7 significant bits: it is exact in bf16
// too.  A group with an infinity or NaN has exponent byte 255 and reads as NaN.
//
// Both directions are streaming passes bound by memory: 65,536 x 2,048 bf16
// move 407 MB each way.
#include <algorithm>

#include "experts.h"

namespace dol {
namespace {

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
    if (c < W) q[row * W + c] = (int8_t)act8_round(v, act8_inverse(byte), byte);
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

}  // namespace

hipError_t launch_act8_pack(const void* x, do_dtype dt, int64_t rows, int32_t W, int8_t* q, uint8_t* e,
                            hipStream_t s) {
  const int32_t G = (W + kAct8Group - 1) / kAct8Group;
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
  const dim3 grid((unsigned)std::min<int64_t>((rows * G + 7) / 8, 1 << 16));
  if (dt == DO_F32)
    hipLaunchKernelGGL(k_act8_unpack<float>, grid, dim3(256), 0, s, q, e, rows, W, G, static_cast<float*>(x));
  else
    hipLaunchKernelGGL(k_act8_unpack<uint16_t>, grid, dim3(256), 0, s, q, e, rows, W, G, static_cast<uint16_t*>(x));
  return hipGetLastError();
}

}  // namespace dol
