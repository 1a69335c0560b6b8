// A layer of experts for few rows on gfx950 (MI355X).  See include/embx_serving.h for the formulas.
//
// Three launches: the router (which experts a row takes, and their shares), the gate and up projections of each row's
// experts with the activation between them, and the down projection, which adds up a row's experts.  Rows and their
// experts are pairs ("uses"), number row * top_k + place; a workgroup finds the uses of an expert by itself, so nothing is
// sorted or counted in memory.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/embx_serving.h"
#include "dense_device.hpp"
#include "serving.hpp"

#ifndef EMBX_MPART
#define EMBX_MPART -1
#endif
#define EMBX_HAS_MPART(p) (EMBX_MPART < 0 || EMBX_MPART == (p))

namespace embx {
namespace {

// ---------------------------------------------------------------- router

// f64 to whole numbers of the same order; NaN above everything, both zeros alike
__device__ inline uint64_t order_of(double v) {
  if (v != v) return ~uint64_t(0);
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(v + 0.0));
  return b >> 63 ? ~b : b | uint64_t(1) << 63;
}

// A workgroup takes a row: a wavefront each expert's logit in turn, summed in 64 bits, then the first one the choice.
template <int TYPE>
__global__ __launch_bounds__(512) void moe_route(Moe a) {
  using T = typename Elem<TYPE>::T;
  __shared__ double logit[kMostExperts];
  __shared__ uint64_t key[kMostExperts];
  const int64_t i = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const T* const x = static_cast<const T*>(a.x) + i * a.ldx;
  for (int e = wave; e < a.experts; e += 8) {
    const T* const r = static_cast<const T*>(a.router) + e * a.ldr;
    double sum = 0.0;
    for (int j = lane; j < a.d; j += 64) sum = fma(double(float(x[j])), double(float(r[j])), sum);
    for (int step = 32; step > 0; step >>= 1) sum += __shfl_xor(sum, step);
    if (lane == 0) logit[e] = sum, key[e] = order_of(sum);
  }
  __syncthreads();
  if (wave != 0) return;
  int mine = 0;          // lane p: the expert in place p
  double first = 0.0;
  for (int place = 0; place < a.top_k; ++place) {
    uint64_t best = 0;   // (a key is never 0: that would be a NaN with its sign)
    int at = kMostExperts;
    for (int e = lane; e < a.experts; e += 64)
      if (key[e] > best) best = key[e], at = e;
    for (int step = 32; step > 0; step >>= 1) {
      const uint64_t other = __shfl_xor(static_cast<unsigned long long>(best), step);
      const int its = __shfl_xor(at, step);
      if (other > best || (other == best && its < at)) best = other, at = its;
    }
    if (place == 0) first = logit[at];
    if (lane == place) mine = at;
    if (lane == 0) key[at] = 0;
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  float total = 0.0f, e = 0.0f;
  if (lane < a.top_k) e = expf(static_cast<float>(logit[mine] - first));
  if (a.renormalize) {
    total = e;
  } else {
    for (int n = lane; n < a.experts; n += 64) total += expf(static_cast<float>(logit[n] - first));
  }
  for (int step = 32; step > 0; step >>= 1) total += __shfl_xor(total, step);
  if (lane < a.top_k) {
    a.chosen[i * a.top_k + lane] = mine;
    a.share[i * a.top_k + lane] = e / total;
  }
}

// ---------------------------------------------------------------- products

// A lane's elements of a step of the reduction: two times eight of 8-bit weights, one of others.
template <int TYPE>
struct Piece {
  using T = typename Elem<TYPE>::T;
  float v[TYPE == kDenseF32 ? 8 : 1];
  s16x8 h;

  __device__ void set(const T* x) {
    if constexpr (TYPE == kDenseF32) {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = x[e];
    } else {
      __builtin_memcpy(&h, x, 16);
    }
  }

  // elements at .. at + 7 of a row of n at any alignment; zeros behind it
  __device__ void load(const T* row, int at, int n) {
    T x[8];
    if (at + 8 <= n) {
      __builtin_memcpy(x, row + at, sizeof(x));
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = at + e < n ? row[at + e] : T(0.0f);
    }
    set(x);
  }

  __device__ void load(const int8_t* row, int at, int n) {
    int8_t b[8];
    if (at + 8 <= n) {
      __builtin_memcpy(b, row + at, 8);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] = at + e < n ? row[at + e] : int8_t(0);
    }
    T x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = T(static_cast<float>(b[e]));   // exact in every type
    set(x);
  }
};

template <int TYPE>
__device__ inline f32x4 product(const Piece<TYPE>& w, const Piece<TYPE>& x, f32x4 c) {
  if constexpr (TYPE == kDenseF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[e], x.v[e], c, 0, 0, 0);
    return c;
  } else {
    return mfma16<TYPE>(w.h, x.h, c);
  }
}

constexpr int kUses = 512;   // that a workgroup looks at at a time

// The uses of one expert among up to kUses of them, `first` .. `first + count - 1`: a wavefront lists them in LDS of its own,
// in order, and has their number.
struct Uses {
  int id[kUses / 64];   // the experts of a lane's uses

  __device__ void read(const Moe& a, int64_t first, int count, int lane) {
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) id[n] = n * 64 + lane < count ? a.chosen[first + n * 64 + lane] : -1;
  }

  __device__ int list(int expert, uint16_t* to, int lane) const {
    int have = 0;
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      const uint64_t mask = __ballot(id[n] == expert);
      if (id[n] == expert) to[have + __popcll(mask & ((uint64_t(1) << lane) - 1))] = static_cast<uint16_t>(n * 64 + lane);
      have += __popcll(mask);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    return have;
  }

  // the least expert above `last`, or kMostExperts
  __device__ int next(int last) const {
    int least = kMostExperts;
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n)
      if (id[n] > last) least = min(least, id[n]);
    for (int step = 32; step > 0; step >>= 1) least = min(least, __shfl_xor(least, step));
    return __builtin_amdgcn_readfirstlane(least);
  }
};

// act(x Wg^T) * (x Wu^T) of an expert's uses: 16 columns a workgroup, whose eight wavefronts take every eighth step each.
template <int TYPE, bool EIGHT>
__global__ __launch_bounds__(512) void moe_up(Moe a) {
  using T = typename Elem<TYPE>::T;
  using W = std::conditional_t<EIGHT, int8_t, T>;
  using P = Piece<TYPE>;
  __shared__ uint16_t lists[8][kUses];
  __shared__ float sums[8][2][16][17];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int expert = blockIdx.y, j0 = blockIdx.x * 16;
  const int64_t uses = int64_t(a.m) * a.top_k;
  const int64_t row = min(j0 + c, a.f - 1);
  const W* const wg = static_cast<const W*>(a.w[0]) + expert * a.stride[0] + row * a.ldw[0];
  const W* const wu = static_cast<const W*>(a.w[1]) + expert * a.stride[1] + row * a.ldw[1];
  for (int64_t first = 0; first < uses; first += kUses) {
    Uses u;
    u.read(a, first, static_cast<int>(min(uses - first, int64_t(kUses))), lane);
    const int have = u.list(expert, lists[wave], lane);
    for (int at = 0; at < have; at += 16) {
      const int64_t use = first + lists[wave][min(at + c, have - 1)];
      const T* const x = static_cast<const T*>(a.x) + use / a.top_k * a.ldx;
      f32x4 g = {}, v = {};
      for (int r0 = wave * 32; r0 < a.d; r0 += 8 * 32) {
        P pg, pu, px;
        pg.load(wg, r0 + 8 * q, a.d);
        pu.load(wu, r0 + 8 * q, a.d);
        px.load(x, r0 + 8 * q, a.d);
        g = product<TYPE>(pg, px, g);
        v = product<TYPE>(pu, px, v);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) sums[wave][0][c][4 * q + e] = g[e], sums[wave][1][c][4 * q + e] = v[e];
      __syncthreads();
      if (threadIdx.x < 32) {
        const int r = threadIdx.x >> 1, half = threadIdx.x & 1, j = j0 + half * 8;
        float s[2][8] = {};
        for (int w = 0; w < 8; ++w)
          for (int mat = 0; mat < 2; ++mat)
            for (int e = 0; e < 8; ++e) s[mat][e] += sums[w][mat][r][half * 8 + e];
        if (at + r < have && j < a.f) {
          const int n = min(8, a.f - j);
          if constexpr (EIGHT) {
            for (int mat = 0; mat < 2; ++mat)
              for (int e = 0; e < 8; ++e) s[mat][e] *= a.scale[mat][int64_t(expert) * a.f + j + min(e, n - 1)];
          }
          act8<TYPE>(s[0], a.act);
          for (int e = 0; e < 8; ++e) s[0][e] *= s[1][e];
          store8<TYPE>(static_cast<T*>(a.h) + (first + lists[wave][at + r]) * a.ldh + j, n, s[0]);
        }
      }
      __syncthreads();
    }
  }
}

constexpr int kDownRows = 64;   // rows of x that a workgroup of the down projection has at a time

// y = sum of a row's experts' h Wd^T times their shares: 16 columns a workgroup.
template <int TYPE, bool EIGHT>
__global__ __launch_bounds__(512) void moe_down(Moe a) {
  using T = typename Elem<TYPE>::T;
  using W = std::conditional_t<EIGHT, int8_t, T>;
  using P = Piece<TYPE>;
  __shared__ uint16_t lists[8][kUses];
  __shared__ float sums[8][kDownRows][16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int j0 = blockIdx.x * 16;
  const int rows_each = min(kDownRows, kUses / a.top_k), first_row = blockIdx.y * rows_each;
  const int rows = min(rows_each, a.m - first_row);
  const int64_t first = int64_t(first_row) * a.top_k;
  const int64_t row = min(j0 + c, a.d - 1);
  for (int at = lane; at < rows * 16; at += 64) sums[wave][at >> 4][at & 15] = 0.0f;
  Uses u;
  u.read(a, first, rows * a.top_k, lane);
  for (int expert = u.next(-1); expert < kMostExperts; expert = u.next(expert)) {
    const int have = u.list(expert, lists[wave], lane);
    const W* const w = static_cast<const W*>(a.w[2]) + expert * a.stride[2] + row * a.ldw[2];
    for (int at = 0; at < have; at += 16) {
      const int use = lists[wave][min(at + c, have - 1)];
      const T* const h = static_cast<const T*>(a.h) + (first + use) * a.ldh;
      f32x4 v = {};
      for (int r0 = wave * 32; r0 < a.f; r0 += 8 * 32) {
        P pw, ph;
        pw.load(w, r0 + 8 * q, a.f);
        ph.load(h, r0 + 8 * q, a.f);
        v = product<TYPE>(pw, ph, v);
      }
      if (at + c < have) {
        const float share = a.share[first + use];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float s = v[e] * share;
          if constexpr (EIGHT) s *= a.scale[2][int64_t(expert) * a.d + min(j0 + 4 * q + e, a.d - 1)];
          sums[wave][use / a.top_k][4 * q + e] += s;
        }
      }
    }
  }
  __syncthreads();
  for (int at = threadIdx.x; at < rows * 2; at += 512) {
    const int r = at >> 1, half = at & 1, j = j0 + half * 8;
    if (j >= a.d) continue;
    float s[8] = {};
    for (int w = 0; w < 8; ++w)
      for (int e = 0; e < 8; ++e) s[e] += sums[w][r][half * 8 + e];
    store8<TYPE>(static_cast<T*>(a.y) + (first_row + r) * a.ldy + j, min(8, a.d - j), s);
  }
}

template <int TYPE, bool EIGHT>
int launch(const Moe& a, hipStream_t s) {
  moe_route<TYPE><<<static_cast<uint32_t>(a.m), 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0) return rc;
  moe_up<TYPE, EIGHT><<<dim3((a.f + 15) / 16, a.experts), 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0) return rc;
  const int rows = std::min(kDownRows, kUses / a.top_k);
  moe_down<TYPE, EIGHT><<<dim3((a.d + 15) / 16, (a.m + rows - 1) / rows), 512, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE>
int launch_type(const Moe& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  return a.scale[0] ? launch<TYPE, true>(a, s) : launch<TYPE, false>(a, s);
}

}  // namespace

#if EMBX_HAS_MPART(0)
int moe_launch_f32(const Moe& a, void* stream) { return launch_type<kDenseF32>(a, stream); }
#endif
#if EMBX_HAS_MPART(1)
int moe_launch_f16(const Moe& a, void* stream) { return launch_type<kDenseF16>(a, stream); }
#endif
#if EMBX_HAS_MPART(2)
int moe_launch_bf16(const Moe& a, void* stream) { return launch_type<kDenseBF16>(a, stream); }
#endif

}  // namespace embx
