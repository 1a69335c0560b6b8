// Rows of a matrix to 8-bit integers with a scale each.  See include/embx_serving.h for the formulas.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/embx_serving.h"
#include "dense_device.hpp"
#include "serving.hpp"

namespace embx {
namespace {

// x / s to the nearest whole number, half to even, exactly: the product with the rounded reciprocal is off by less than one
// of the nearest, and what is left of x after it, x - r s, is exact near the borders (a multiple of the smaller operand's
// last place, and at most s), so that a comparison with s / 2 mends it.
__device__ inline float nearest(float x, float s, float inverse) {
  float r = rintf(x * inverse);
  const float left = 2.0f * fmaf(-r, s, x);
  const float one = copysignf(1.0f, left);
  if (fabsf(left) > s || (fabsf(left) == s && fabsf(rintf(r * 0.5f) * 2.0f - r) == 1.0f)) r += one;
  return r;
}

template <int TYPE>
__global__ __launch_bounds__(256) void quantize_rows(Quantize a) {
  using T = typename Elem<TYPE>::T;
  __shared__ uint32_t most[4];
  for (int64_t i = blockIdx.x; i < a.m; i += gridDim.x) {
    const T* const x = static_cast<const T*>(a.x) + i * a.ldx;
    uint32_t largest = 0;
    for (int j = threadIdx.x; j < a.k; j += 256) largest = max(largest, __float_as_uint(float(x[j])) & 0x7fffffffu);
    for (int step = 32; step > 0; step >>= 1) largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), step)));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = largest;
    __syncthreads();
    largest = max(max(most[0], most[1]), max(most[2], most[3]));
    const bool fine = largest < 0x7f800000u;
    const float s = fmaxf(__uint_as_float(largest) / 127.0f, 0x1p-126f), inverse = 1.0f / s;
    if (threadIdx.x == 0) a.scale[i] = fine ? s : __uint_as_float(0x7fc00000u);
    int8_t* const q = a.q + i * a.ldq;
    for (int j = threadIdx.x; j < a.padded; j += 256)
      q[j] = j < a.k && fine ? static_cast<int8_t>(nearest(float(x[j]), s, inverse)) : 0;
    __syncthreads();
  }
}

}  // namespace

int quantize_launch(int dtype, const Quantize& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const uint32_t grid = static_cast<uint32_t>(std::min<int64_t>(a.m, 65536));
  if (dtype == EMB_DTYPE_F32) quantize_rows<kDenseF32><<<grid, 256, 0, s>>>(a);
  else if (dtype == EMB_DTYPE_F16) quantize_rows<kDenseF16><<<grid, 256, 0, s>>>(a);
  else quantize_rows<kDenseBF16><<<grid, 256, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace embx
