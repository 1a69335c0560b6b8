// Device code that quantizes a row's elements: its scale, and whole numbers for it.
#ifndef EMBX_QUANTIZE_DEVICE_HPP
#define EMBX_QUANTIZE_DEVICE_HPP

#include "dense_device.hpp"

namespace embx {
namespace {

constexpr float kRound = 0x1.8p23f;   // a float with this added has its whole part, rounded half to even, in its low bits

// A row's scale from the largest of its magnitudes (by their bits: NaN is the largest); not `fine` where that is not finite.
struct Scale {
  float s, inverse;
  bool fine;

  __device__ static Scale of(float most) {
    Scale r;
    r.fine = most < __builtin_inff();   // (NaN is not)
    r.s = r.fine ? fmaxf(most / 127.0f, 0x1p-126f) : 1.0f;
    r.inverse = 1.0f / r.s;
    return r;
  }

  __device__ float stored() const { return fine ? s : __builtin_nanf(""); }

  // x / s to the nearest whole number, half to even, exactly, in the low 8 bits of the result: x times the rounded
  // reciprocal is off by less than one of the nearest, and what is left of x after it, x - r s, is exact near the borders
  // (a multiple of the smaller operand's last place, and at most s).  *far: whether that is s / 2 or more, for mend().
  __device__ uint32_t nearest(float x, bool* far) const {
    const float u = fmaf(x, inverse, kRound), left = fmaf(kRound - u, s, x);
    *far |= fabsf(left + left) >= s;
    return __float_as_uint(u);
  }

  __device__ uint32_t mend(float x) const {
    float u = fmaf(x, inverse, kRound);
    const float left = fmaf(kRound - u, s, x), twice = fabsf(left + left);
    if (twice > s || (twice == s && (__float_as_uint(u) & 1))) u += copysignf(1.0f, left);
    return __float_as_uint(u);
  }
};

// the low 8 bits of four values as one
__device__ inline uint32_t four(const uint32_t* u) {
  return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400), __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400), 0x05040100);
}

// eight values to whole numbers; a row that is not fine has zeros
__device__ inline void quantize8(const Scale& s, const float* x, uint32_t* out) {
  uint32_t u[8];
  bool far = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = s.nearest(x[e], &far);
  if (__any(far)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = s.mend(x[e]);
  }
  out[0] = s.fine ? four(u) : 0, out[1] = s.fine ? four(u + 4) : 0;
}

}  // namespace
}  // namespace embx
#endif
