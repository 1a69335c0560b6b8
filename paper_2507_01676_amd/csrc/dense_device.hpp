// Device code that the kernels of the dense layers and of their serving forms share: element types, activations,
// loads and stores of eight elements, matrix instructions.
#ifndef EMBX_DENSE_DEVICE_HPP
#define EMBX_DENSE_DEVICE_HPP

#include <hip/hip_runtime.h>

#include <type_traits>

#include "../../include/embx_dense.h"
#include "dense.hpp"

namespace embx {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int TYPE> struct Elem;
template <> struct Elem<kDenseF32> { using T = float; };
template <> struct Elem<kDenseF16> { using T = _Float16; using V = f16x8; };
template <> struct Elem<kDenseBF16> { using T = __bf16; using V = bf16x8; };
template <> struct Elem<kDenseI8> { using T = int8_t; };   // (of operands: results have a type of their own)

// Activations in 32 bits, from the hardware's exp2 and reciprocal (an ulp each).  exp(z) = 2^(z log2 e).  f32 carries the
// rest of that product, which would be up to |z| / 2^24 of the result, into a second factor 1 + rest ln 2 (two ulps in all).
// With FAR it forms small results 2^64 times as large first, as the hardware's are nought below the normal numbers (z <= 0
// there, and below -150 as at -150, where the result is nought and the rest still finite).  The 16-bit types round the rest
// away, and take the normal distribution function by formula 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical
// Functions (off by less than 1e-7, and of itself by 0.2% at z = -5 and 1% at -8), where f32 takes the library's erfc.
template <int TYPE, bool FAR = true>
__device__ inline float exp_f(float z) {
  if constexpr (TYPE != kDenseF32) return __builtin_amdgcn_exp2f(z * 1.44269504f);
  if constexpr (FAR) z = __builtin_elementwise_maximum(z, -150.0f);   // NaN passes
  const float hi = z * 1.44269504f, rest = fmaf(z, 1.92596299e-8f, fmaf(z, 1.44269504f, -hi)) * 0.69314718f;
  if constexpr (FAR) {
    const bool small = hi < -100.0f;
    const float e = __builtin_amdgcn_exp2f(hi + (small ? 64.0f : 0.0f));
    return fmaf(e, rest, e) * (small ? 0x1p-64f : 1.0f);
  }
  const float e = __builtin_amdgcn_exp2f(hi);
  return fmaf(e, rest, e);
}

template <int TYPE>
__device__ inline float rcp_f(float z) { return __builtin_amdgcn_rcpf(z); }

// In f32 from exp(-|z|), so that the reciprocal is never below the normal numbers (five ulps in all).  16 bits: nought below
// 2^-126.
template <int TYPE, bool FAR>
__device__ inline float sigmoid_f(float z) {
  if constexpr (TYPE != kDenseF32) return rcp_f<TYPE>(1.0f + exp_f<TYPE>(-z));
  const float t = exp_f<TYPE, FAR>(-fabsf(z)), r = rcp_f<TYPE>(1.0f + t);
  return z >= 0.0f ? r : t * r;
}

// the normal distribution function, and exp(-z^2 / 2) on the way
template <int TYPE>
__device__ inline float phi_f(float z, float* bell) {
  const float e = exp_f<TYPE>(-0.5f * z * z);
  *bell = e;
  if constexpr (TYPE == kDenseF32) {
    return 0.5f * erfcf(z * -0.70710678f);   // (1 + erf loses the small values of negative z)
  } else {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.0f));
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f) * t;
    const float tail = 0.5f * p * e;   // of |z|
    return z < 0.0f ? tail : 1.0f - tail;
  }
}

// dy act'(z); *value = act(z).  The sigmoid's slope is s(z) s(-z), with both from exp(-|z|): 1 - s(z) would
// lose all its digits where z is large.
template <int TYPE>
__device__ inline float slope_f(float dy, float z, int act, float* value) {
  switch (act) {
    case EMB_ACT_RELU:
      *value = z < 0.0f ? 0.0f : z;
      return z <= 0.0f ? 0.0f : dy;   // an infinite dy is not multiplied by 0
    case EMB_ACT_SIGMOID:
    case EMB_ACT_SILU: {
      const float t = exp_f<TYPE>(-fabsf(z)), r = rcp_f<TYPE>(1.0f + t), w = t * r;
      const float s = z >= 0.0f ? r : w, c = z >= 0.0f ? w : r;
      *value = act == EMB_ACT_SIGMOID ? s : z * s;
      return dy * (act == EMB_ACT_SIGMOID ? s * c : s * (1.0f + z * c));
    }
    case EMB_ACT_GELU: {
      float bell;
      const float p = phi_f<TYPE>(z, &bell);
      *value = z * p;
      return dy * (p + z * 0.39894228f * bell);
    }
    default:
      *value = z;
      return dy;
  }
}

// whether exp(-|z|) has small results among a wavefront's eights of values: asked of all at once, they hardly ever cost
// anything (f32 65536 x 512 x 64 with a sigmoid 59.4 us a call, with small results considered for each value 61.4)
template <int TYPE>
__device__ inline bool far_out(const float* z) {
  if constexpr (TYPE != kDenseF32) return false;
  float largest = fabsf(z[0]);
#pragma unroll
  for (int e = 1; e < 8; ++e) largest = fmaxf(largest, fabsf(z[e]));
  return __any(largest > 69.0f);
}

// the sigmoid of eight values, or (TIMES) each value times its
template <int TYPE, bool FAR, bool TIMES>
__device__ inline void sigmoid8(float* z) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float s = sigmoid_f<TYPE, FAR>(z[e]);
    z[e] = TIMES ? z[e] * s : s;
  }
}

// act of eight values: one branch
template <int TYPE>
__device__ inline void act8(float* z, int act) {
  float bell;
  switch (act) {
    case EMB_ACT_RELU:
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] = __builtin_elementwise_maximum(z[e], 0.0f);   // NaN passes
      break;
    case EMB_ACT_SIGMOID:
      if (far_out<TYPE>(z)) sigmoid8<TYPE, true, false>(z);
      else sigmoid8<TYPE, false, false>(z);
      break;
    case EMB_ACT_SILU:
      if (far_out<TYPE>(z)) sigmoid8<TYPE, true, true>(z);
      else sigmoid8<TYPE, false, true>(z);
      break;
    case EMB_ACT_GELU:
#pragma unroll
      for (int e = 0; e < 8; ++e) z[e] *= phi_f<TYPE>(z[e], &bell);
      break;
    default: break;
  }
}

// act of one f32 value
__device__ inline float act_f(float z, int act) {
  float bell;
  switch (act) {
    case EMB_ACT_RELU: return __builtin_elementwise_maximum(z, 0.0f);   // NaN passes
    case EMB_ACT_SIGMOID: return sigmoid_f<kDenseF32, true>(z);
    case EMB_ACT_SILU: return z * sigmoid_f<kDenseF32, true>(z);
    case EMB_ACT_GELU: return z * phi_f<kDenseF32>(z, &bell);
    default: return z;
  }
}

// Eight consecutive elements at p, of which n >= 1 are inside (the last one stands for the others); whole eights are read
// and written 16 bytes at a time at any alignment.
template <int TYPE>
__device__ inline void load8(const void* p, int n, float* v) {
  using T = typename Elem<TYPE>::T;
  T x[8];
  if (n == 8) {
    __builtin_memcpy(x, p, sizeof(x));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = float(static_cast<const T*>(p)[min(e, n - 1)]);
  }
}

template <int TYPE>
__device__ inline void store8(void* p, int n, const float* v) {
  using T = typename Elem<TYPE>::T;
  T x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = T(v[e]);
  if (n == 8) {
    __builtin_memcpy(p, x, sizeof(x));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n) static_cast<T*>(p)[e] = x[e];
  }
}

// Four sums.  Of 8-bit integers they are whole numbers, exact in 32 bits; until the epilogue turns them into f32 they pass
// through LDS and memory with their bits unchanged.
template <int TYPE> using Sums = std::conditional_t<TYPE == kDenseI8, i32x4, f32x4>;

// 64 bytes of the reduction of both operands, 16 of them in a lane
template <int TYPE>
__device__ inline Sums<TYPE> mfma16(s16x8 a, s16x8 b, Sums<TYPE> c) {
  if constexpr (TYPE == kDenseI8) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  } else {
    using V = typename Elem<TYPE>::V;
    if constexpr (TYPE == kDenseF16)
      return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
  }
}

// Copies up to three matrices to rows that start at multiples of 16 bytes and end in zeros up to a whole chunk: the
// tiles above read nothing else.  A wavefront takes 64 consecutive elements at a time, as rows that start anywhere
// are read fastest (16-byte loads at odd addresses measured 1.1 TB/s).  f16 65536 x 1001: 262 MB read and written in 60 us,
// 4.4 TB/s, with four rows of a thread under way (one: 81 us).
template <class E>
__device__ inline void pack_rows(const DensePack& p, uint32_t mat, uint32_t group) {
  constexpr uint32_t kChunk = 16 / sizeof(E);
  const uint32_t cols = p.cols[mat], padded = (cols + kChunk - 1) / kChunk * kChunk;
  const uint32_t rows = p.rows[mat];
  const E* src = static_cast<const E*>(p.src[mat]);
  E* dst = static_cast<E*>(p.dst[mat]);
  // as many rows side by side as 256 threads hold, four at a time
  const uint32_t wide = p.wide[mat], x = threadIdx.x % wide, y = threadIdx.x / wide, side = 256 / wide;
  const uint64_t step = uint64_t(p.groups) * side;
  for (uint32_t panel = 0; panel < padded; panel += kPanel, dst += p.panel[mat] - kPanel) {
    const uint32_t end = min(padded, panel + static_cast<uint32_t>(kPanel));
    for (uint64_t i = uint64_t(group) * side + y; i < rows; i += 4 * step)
#pragma unroll 2
      for (uint32_t j = panel + x; j < end; j += wide) {
        E v[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = src[min(i + r * step, uint64_t(rows) - 1) * p.lds[mat] + min(j, cols - 1)];
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (i + r * step < rows) dst[(i + r * step) * p.ldd[mat] + j] = j < cols ? v[r] : 0;
      }
  }
}

// Sixteen bytes at p at any alignment, of which those from `left` on (of what can be read there) are something else.
__device__ inline s16x8 load16(const int8_t* p, int64_t left) {
  s16x8 v;
  if (left >= 16) {
    __builtin_memcpy(&v, p, 16);
  } else {
    int8_t b[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) b[e] = p[min(int64_t(e), left - 1)];
    __builtin_memcpy(&v, b, 16);
  }
  return v;
}

// keeps `left` bytes of sixteen, zeros behind them
__device__ inline s16x8 keep16(s16x8 v, int left) {
  i32x4 w = __builtin_bit_cast(i32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int bytes = left - 4 * i;
    w[i] = bytes >= 4 ? w[i] : bytes <= 0 ? 0 : w[i] & static_cast<int>((1u << 8 * bytes) - 1);
  }
  return __builtin_bit_cast(s16x8, w);
}

// pack_rows of 8-bit integers, 16 bytes a thread: read at any alignment those run at a copy's rate (5.0 TB/s; 1 byte a
// thread at 1.2).
__device__ inline void pack_eights(const DensePack& p, uint32_t mat, uint32_t group) {
  const uint32_t cols = p.cols[mat], chunks = (cols + 15) / 16, rows = p.rows[mat];
  const int8_t* const src = static_cast<const int8_t*>(p.src[mat]);
  int8_t* const dst = static_cast<int8_t*>(p.dst[mat]);
  const int64_t last = int64_t(rows - 1) * p.lds[mat] + cols;   // bytes of the matrix
  const uint32_t wide = p.wide[mat], x = threadIdx.x % wide, y = threadIdx.x / wide, side = 256 / wide;
  const uint64_t step = uint64_t(p.groups) * side;
  for (uint64_t i = uint64_t(group) * side + y; i < rows; i += 4 * step)
    for (uint32_t j = x; j < chunks; j += wide) {
      s16x8 v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int64_t at = static_cast<int64_t>(min(i + r * step, uint64_t(rows) - 1)) * p.lds[mat] + j * 16;
        v[r] = load16(src + at, last - at);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (i + r * step < rows)
          *reinterpret_cast<s16x8*>(dst + static_cast<int64_t>(i + r * step) * p.ldd[mat] + j * 16) =
              keep16(v[r], static_cast<int>(min(16u, cols - j * 16)));
    }
}

}  // namespace
}  // namespace embx
#endif
