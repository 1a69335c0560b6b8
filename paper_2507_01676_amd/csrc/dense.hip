// Dense layers for gfx950 (MI355X): the matrix products of fully connected layers and gated
// feed-forward blocks, forward and backward.  See include/embx_dense.h for the formulas.
#include <hip/hip_runtime.h>

#include "../../include/embx_dense.h"
#include "dense.hpp"

#ifndef EMBX_DPART
#define EMBX_DPART -1
#endif
#define EMBX_HAS_DPART(p) (EMBX_DPART < 0 || EMBX_DPART == (p))

namespace embx {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int TYPE> struct Elem;
template <> struct Elem<kDenseF32> { using T = float; };
template <> struct Elem<kDenseF16> { using T = _Float16; using V = f16x8; };
template <> struct Elem<kDenseBF16> { using T = __bf16; using V = bf16x8; };

__device__ inline float sigmoid_f(float z) { return 1.0f / (1.0f + expf(-z)); }
__device__ inline float phi_f(float z) { return 0.5f * (1.0f + erff(z * 0.70710678f)); }

__device__ inline float act_f(float z, int act) {
  switch (act) {
    case EMB_ACT_RELU: return z < 0.0f ? 0.0f : z;   // NaN passes
    case EMB_ACT_SIGMOID: return sigmoid_f(z);
    case EMB_ACT_SILU: return z * sigmoid_f(z);
    case EMB_ACT_GELU: return z * phi_f(z);
    default: return z;
  }
}

// The sigmoid's slope is s(z) s(-z), with both from exp(-|z|): 1 - s(z) would lose all its digits
// where z is large.
__device__ inline float slope_f(float z, int act) {
  switch (act) {
    case EMB_ACT_RELU: return z <= 0.0f ? 0.0f : 1.0f;
    case EMB_ACT_SIGMOID:
    case EMB_ACT_SILU: {
      const float t = expf(-fabsf(z)), r = 1.0f / (1.0f + t), w = t * r;
      const float s = z >= 0.0f ? r : w, c = z >= 0.0f ? w : r;
      return act == EMB_ACT_SIGMOID ? s * c : s * (1.0f + z * c);
    }
    case EMB_ACT_GELU: return phi_f(z) + z * 0.39894228f * expf(-0.5f * z * z);
    default: return 1.0f;
  }
}

// ---------------------------------------------------------------- epilogue

// Stores one element of the result from its sums (s1: the up projection's).
template <int TYPE, int KIND>
__device__ inline void finish(const DenseGemm& g, int part, int i, int j, float s0, float s1) {
  using T = typename Elem<TYPE>::T;
  if constexpr (KIND == kForward || KIND == kGated) {
    if (g.bias[0]) s0 += float(static_cast<const T*>(g.bias[0])[j]);
    if (g.z[0]) static_cast<T*>(g.z[0])[i * g.ldz[0] + j] = T(s0);
    float y = act_f(s0, g.act);
    if constexpr (KIND == kGated) {
      if (g.bias[1]) s1 += float(static_cast<const T*>(g.bias[1])[j]);
      if (g.z[1]) static_cast<T*>(g.z[1])[i * g.ldz[1] + j] = T(s1);
      y *= s1;
    } else if (g.res) {
      y += float(static_cast<const T*>(g.res)[i * g.ldr + j]);
    }
    static_cast<T*>(g.c[0])[i * g.ldc[0] + j] = T(y);
  } else {
    static_cast<T*>(g.c[part])[i * g.ldc[part] + j] = T(s0);
  }
}

// ---------------------------------------------------------------- matrix products

constexpr int kBM = 64, kBN = 64, kBK = 32, kPad = 8;

// A tile of 64 x 64 results, four wavefronts of 32 x 32 each.
template <int TYPE, int KIND>
__global__ __launch_bounds__(256) void dense_tile(DenseGemm g) {
  using T = typename Elem<TYPE>::T;
  __shared__ T sa[kBM][kBK + kPad], sb[kBN][kBK + kPad];
  constexpr bool kGate = KIND == kGated;
  constexpr int kCols = kGate ? kBN / 2 : kBN;   // result columns of a tile
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int tiles_j = (g.nj + kCols - 1) / kCols;
  const int i0 = static_cast<int>(blockIdx.x / tiles_j) * kBM, j0 = static_cast<int>(blockIdx.x % tiles_j) * kCols;
  const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
  const int q = lane >> 4, c = lane & 15;
  const int bpart = KIND == kWeightGrad ? blockIdx.z : 0;
  f32x4 acc[2][2] = {};
  const int parts = KIND == kInputGrad ? g.parts : 1;
  for (int part = 0; part < parts; ++part) {
    const T* a = static_cast<const T*>(g.a[KIND == kWeightGrad ? bpart : part]);
    for (int r0 = 0; r0 < g.nr; r0 += kBK) {
      __syncthreads();
      for (int e = tid; e < kBM * kBK; e += 256) {
        if constexpr (KIND == kWeightGrad) {
          const int r = e / kBM, i = e % kBM;
          sa[i][r] = r0 + r < g.nr && i0 + i < g.ni ? a[(r0 + r) * g.lda + i0 + i] : T(0.0f);
        } else {
          const int i = e / kBK, r = e % kBK;
          sa[i][r] = r0 + r < g.nr && i0 + i < g.ni ? a[(i0 + i) * g.lda + r0 + r] : T(0.0f);
        }
      }
      for (int e = tid; e < kBN * kBK; e += 256) {
        if constexpr (KIND == kForward || KIND == kGated) {
          const int row = e / kBK, r = e % kBK;
          const int mat = kGate ? row / kCols : 0, j = row - mat * kCols;
          const T* b = static_cast<const T*>(g.b[mat]);
          sb[row][r] = r0 + r < g.nr && j0 + j < g.nj ? b[(j0 + j) * g.ldb[mat] + r0 + r] : T(0.0f);
        } else {
          const int r = e / kBN, j = e % kBN;
          const int mat = KIND == kInputGrad ? part : 0;
          const T* b = static_cast<const T*>(g.b[mat]);
          sb[j][r] = r0 + r < g.nr && j0 + j < g.nj ? b[(r0 + r) * g.ldb[mat] + j0 + j] : T(0.0f);
        }
      }
      __syncthreads();
#pragma unroll
      for (int fi = 0; fi < 2; ++fi)
#pragma unroll
        for (int fj = 0; fj < 2; ++fj) {
          const T* pa = sa[wi + fi * 16 + c];
          // gated: a wavefront's first fragment is of the gate, its second of the up projection
          const T* pb = kGate ? sb[fj * kCols + (wave & 1) * 16 + c] : sb[wj + fj * 16 + c];
          if constexpr (TYPE == kDenseF32) {
#pragma unroll
            for (int s = 0; s < kBK / 4; ++s)
              acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x4f32(pb[4 * s + q], pa[4 * s + q], acc[fi][fj], 0, 0, 0);
          } else {
            using V = typename Elem<TYPE>::V;
            const V va = *reinterpret_cast<const V*>(pa + 8 * q), vb = *reinterpret_cast<const V*>(pb + 8 * q);
            if constexpr (TYPE == kDenseF16)
              acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, va, acc[fi][fj], 0, 0, 0);
            else
              acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, va, acc[fi][fj], 0, 0, 0);
          }
        }
    }
  }
  // lane: result row i = c, columns 4 q .. 4 q + 3 of a fragment
#pragma unroll
  for (int fi = 0; fi < 2; ++fi)
#pragma unroll
    for (int fj = 0; fj < (kGate ? 1 : 2); ++fj)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = i0 + wi + fi * 16 + c;
        const int j = j0 + (kGate ? (wave & 1) * 16 : wj + fj * 16) + 4 * q + e;
        if (i < g.ni && j < g.nj) finish<TYPE, KIND>(g, bpart, i, j, acc[fi][fj][e], kGate ? acc[fi][1][e] : 0.0f);
      }
}

// ---------------------------------------------------------------- elementwise parts of the gradients

// dz (or dg and du) and sums of their columns over a block of rows: a thread per column
template <int TYPE>
__global__ __launch_bounds__(256) void dense_slope(DenseSlope s) {
  using T = typename Elem<TYPE>::T;
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= s.n) return;
  const int rows = (s.m + s.row_blocks - 1) / s.row_blocks;
  const int first = blockIdx.y * rows, end = min(s.m, first + rows);
  float sum0 = 0.0f, sum1 = 0.0f;
  for (int i = first; i < end; ++i) {
    const float dy = float(static_cast<const T*>(s.dy)[i * s.lddy + j]);
    float d0 = dy, d1 = 0.0f;
    if (s.z[0]) {
      const float z = float(static_cast<const T*>(s.z[0])[i * s.ldz[0] + j]);
      if (s.gated) {
        const float u = float(static_cast<const T*>(s.z[1])[i * s.ldz[1] + j]);
        d1 = dy * act_f(z, s.act);
        d0 = dy * u * slope_f(z, s.act);
      } else {
        d0 = s.act == EMB_ACT_RELU ? (z <= 0.0f ? 0.0f : dy) : dy * slope_f(z, s.act);
      }
    }
    if (s.dz[0]) static_cast<T*>(s.dz[0])[i * s.lddz + j] = T(d0);
    if (s.dz[1]) static_cast<T*>(s.dz[1])[i * s.lddz + j] = T(d1);
    sum0 += d0;
    sum1 += d1;
  }
  if (s.colsum[0]) s.colsum[0][int64_t(blockIdx.y) * s.n + j] = sum0;
  if (s.colsum[1]) s.colsum[1][int64_t(blockIdx.y) * s.n + j] = sum1;
}

template <int TYPE>
__global__ __launch_bounds__(256) void dense_colsum(const float* partial, int32_t blocks, int32_t n, void* out) {
  using T = typename Elem<TYPE>::T;
  const int j = blockIdx.x * 256 + threadIdx.x;
  if (j >= n) return;
  float sum = 0.0f;
  for (int b = 0; b < blocks; ++b) sum += partial[int64_t(b) * n + j];
  static_cast<T*>(out)[j] = T(sum);
}

template <int TYPE>
int gemm_launch(int kind, const DenseGemm& g, hipStream_t stream) {
  const int cols = kind == kGated ? kBN / 2 : kBN;
  const int64_t tiles = int64_t((g.ni + kBM - 1) / kBM) * ((g.nj + cols - 1) / cols);
  const dim3 grid(static_cast<uint32_t>(tiles), 1, kind == kWeightGrad ? g.parts : 1);
  switch (kind) {
    case kForward: dense_tile<TYPE, kForward><<<grid, 256, 0, stream>>>(g); break;
    case kGated: dense_tile<TYPE, kGated><<<grid, 256, 0, stream>>>(g); break;
    case kInputGrad: dense_tile<TYPE, kInputGrad><<<grid, 256, 0, stream>>>(g); break;
    default: dense_tile<TYPE, kWeightGrad><<<grid, 256, 0, stream>>>(g); break;
  }
  return hipGetLastError();
}

template <int TYPE>
int slope_launch(const DenseSlope& s, hipStream_t stream) {
  dense_slope<TYPE><<<dim3((s.n + 255) / 256, s.row_blocks), 256, 0, stream>>>(s);
  return hipGetLastError();
}

template <int TYPE>
int colsum_launch(const float* partial, int32_t blocks, int32_t n, void* out, hipStream_t stream) {
  dense_colsum<TYPE><<<(n + 255) / 256, 256, 0, stream>>>(partial, blocks, n, out);
  return hipGetLastError();
}

}  // namespace

#define EMBX_DENSE_TYPE(NAME, TYPE)                                                                     \
  int dense_gemm_##NAME(int kind, const DenseGemm& g, void* stream) {                                   \
    return gemm_launch<TYPE>(kind, g, static_cast<hipStream_t>(stream));                                \
  }                                                                                                     \
  int dense_slope_##NAME(const DenseSlope& s, void* stream) {                                           \
    return slope_launch<TYPE>(s, static_cast<hipStream_t>(stream));                                     \
  }                                                                                                     \
  int dense_colsum_##NAME(const float* p, int32_t blocks, int32_t n, void* out, void* stream) {         \
    return colsum_launch<TYPE>(p, blocks, n, out, static_cast<hipStream_t>(stream));                    \
  }

#if EMBX_HAS_DPART(0)
EMBX_DENSE_TYPE(f32, kDenseF32)
#endif
#if EMBX_HAS_DPART(1)
EMBX_DENSE_TYPE(f16, kDenseF16)
#endif
#if EMBX_HAS_DPART(2)
EMBX_DENSE_TYPE(bf16, kDenseBF16)
#endif

}  // namespace embx
