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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- router

// f64 to whole numbers of the same order; NaN above everything, both zeros alike
__device__ inline uint64_t order_of(double v) {
  if (v != v) return ~uint64_t(0);
  const uint64_t b = static_cast<uint64_t>(__double_as_longlong(v + 0.0));
  return b >> 63 ? ~b : b | uint64_t(1) << 63;
}

// A row's 16 bytes at element `at` of n: eight elements, or 16 of 8 bits.  Where rows start at multiples of 16 bytes (WHOLE)
// the last ones are read whole; what lies behind the row's end counts as zeros.
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

  __device__ float get(int e) const {
    if constexpr (TYPE == kDenseF32) return v[e];
    else if constexpr (TYPE == kDenseBF16) return __uint_as_float(uint32_t(static_cast<uint16_t>(h[e])) << 16);
    else return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<short>(h[e])));
  }

  // FULL: all of it is inside
  template <bool WHOLE, bool FULL>
  __device__ void load(const T* row, int at, int n) {
    T x[8];
    if constexpr (FULL) {
      if constexpr (WHOLE) __builtin_memcpy(x, __builtin_assume_aligned(row + at, 16), sizeof(x));
      else __builtin_memcpy(x, row + at, sizeof(x));
    } else if constexpr (WHOLE) {
      constexpr int kPer = 16 / sizeof(T);   // (f32: two chunks, of which the second may be outside)
      const int last = (n - 1) / kPer * kPer;
#pragma unroll
      for (int c = 0; c < 8; c += kPer) __builtin_memcpy(x + c, __builtin_assume_aligned(row + min(at + c, last), 16), 16);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = at + e < n ? x[e] : T(0.0f);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = row[min(at + e, n - 1)];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = at + e < n ? x[e] : T(0.0f);
    }
    set(x);
  }
};

// The same of an expert's matrix, whose elements may have 8 bits (EIGHT): whole numbers, exact in every type.
template <int TYPE, bool EIGHT>
struct Weights {
  using W = typename Elem<TYPE>::T;
  static constexpr int kPieces = 1, kPer = 8;
  Piece<TYPE> p;

  template <bool WHOLE, bool FULL>
  __device__ void load(const W* row, int at, int n) { p.template load<WHOLE, FULL>(row, at, n); }

  __device__ const Piece<TYPE>& piece(int) const { return p; }
};

template <int TYPE>
struct Weights<TYPE, true> {
  using W = int8_t;
  static constexpr int kPieces = 2, kPer = 16;
  u32x4 b;

  template <bool WHOLE, bool FULL>
  __device__ void load(const W* row, int at, int n) {
    if constexpr (FULL && !WHOLE) {
      __builtin_memcpy(&b, row + at, 16);
    } else if constexpr (WHOLE) {
      b = *reinterpret_cast<const u32x4*>(row + (FULL ? at : min(at, (n - 1) / 16 * 16)));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        b[e] = 0;
#pragma unroll
        for (int x = 0; x < 4; ++x) b[e] |= uint32_t(static_cast<uint8_t>(row[min(at + 4 * e + x, n - 1)])) << 8 * x;
      }
    }
    if constexpr (!FULL) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int left = n - at - 4 * e;   // bytes of this word that are inside
        b[e] = left >= 4 ? b[e] : left <= 0 ? 0 : b[e] & ((1u << 8 * left) - 1);
      }
    }
  }

  __device__ Piece<TYPE> piece(int i) const {
    Piece<TYPE> out;
    u32x4 pairs;
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint32_t word = b[2 * i + e / 4];
      const float lo = static_cast<float>(static_cast<int8_t>(word >> 8 * (e & 3)));
      const float hi = static_cast<float>(static_cast<int8_t>(word >> 8 * (e & 3) + 8));
      if constexpr (TYPE == kDenseF32) out.v[e] = lo, out.v[e + 1] = hi;
      else if constexpr (TYPE == kDenseBF16) pairs[e / 2] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);
      else pairs[e / 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
    }
    if constexpr (TYPE != kDenseF32) out.h = __builtin_bit_cast(s16x8, pairs);
    return out;
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

// A workgroup takes a row: a wavefront four experts' logits at a time, summed in 64 bits, then the first one the choice.
template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(512) void moe_route(Moe a) {
  using T = typename Elem<TYPE>::T;
  __shared__ double logit[kMostExperts];
  __shared__ uint64_t key[kMostExperts];
  constexpr int kMany = 4;
  const int64_t i = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const T* const x = static_cast<const T*>(a.x) + i * a.ldx;
  for (int first = wave; first < a.experts; first += 8 * kMany) {
    const T* r[kMany];
    double sum[kMany] = {};
#pragma unroll
    for (int n = 0; n < kMany; ++n) r[n] = static_cast<const T*>(a.router) + int64_t(min(first + n * 8, a.experts - 1)) * a.ldr;
    auto add = [&](int j, auto full) {
      constexpr bool kFull = decltype(full)::value;
      Piece<TYPE> px, pr[kMany];
      px.template load<WHOLE, kFull>(x, j, a.d);
#pragma unroll
      for (int n = 0; n < kMany; ++n) pr[n].template load<WHOLE, kFull>(r[n], j, a.d);
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int n = 0; n < kMany; ++n) sum[n] = fma(double(px.get(e)), double(pr[n].get(e)), sum[n]);
    };
    int j = lane * 8;
    for (; j + 8 <= a.d; j += 512) add(j, std::true_type());
    if (j < a.d) add(j, std::false_type());
#pragma unroll
    for (int n = 0; n < kMany; ++n) {
      for (int step = 32; step > 0; step >>= 1) sum[n] += __shfl_xor(sum[n], step);
      if (lane == 0 && first + n * 8 < a.experts) logit[first + n * 8] = sum[n], key[first + n * 8] = order_of(sum[n]);
    }
  }
  __syncthreads();
  if (wave != 0) return;
  int mine = 0;          // lane p: the expert in place p
  double best_logit = 0.0;
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
    if (place == 0) best_logit = logit[at];
    if (lane == place) mine = at;
    if (lane == 0) key[at] = 0;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  float total = 0.0f, e = 0.0f;
  if (lane < a.top_k) e = expf(static_cast<float>(logit[mine] - best_logit));
  if (a.renormalize) {
    total = e;
  } else {
    for (int n = lane; n < a.experts; n += 64) total += expf(static_cast<float>(logit[n] - best_logit));
  }
  for (int step = 32; step > 0; step >>= 1) total += __shfl_xor(total, step);
  if (lane < a.top_k) {
    a.chosen[i * a.top_k + lane] = mine;
    a.share[i * a.top_k + lane] = e / total;
  }
}

// ---------------------------------------------------------------- products
//
// A matrix instruction multiplies 16 rows of weights by 16 rows of x.  With S segments, its 16 are 16 / S rows and, of each,
// S consecutive pieces of the reduction: sums whose pieces differ mean nothing, the others are added up at the end.  So a
// workgroup can have few rows of weights, and there are enough of them where x has few rows; a row's 256 bytes are read at once.

constexpr int kWaves = 8;

// acc += the reduction from `begin` to `end` of a lane's R rows of weights by FR rows of x (in PARTS parts, added up), of
// which each wavefront takes every eighth step.
template <int TYPE, bool EIGHT, bool WHOLE, int S, int R, int FR, int PARTS>
__device__ inline void accumulate(const typename Weights<TYPE, EIGHT>::W* const (&w)[R], const typename Elem<TYPE>::T* const (&x)[FR],
                                  int64_t part, int begin, int end, int wave, int lane, f32x4 (&acc)[R][FR]) {
  using Ws = Weights<TYPE, EIGHT>;
  constexpr int kSpan = 4 * Ws::kPer, kStep = kSpan * S;
  constexpr int kGo = S == 1 && TYPE != kDenseF32 && FR * PARTS < 4 ? 2 : 1;   // steps at a time: 128 bytes of a row
  const int own = (lane & (S - 1)) * kSpan + (lane >> 4) * Ws::kPer;
  auto go = [&](int r0, auto full) {
    constexpr bool kFull = decltype(full)::value;
    Ws pw[kGo][R];
    Piece<TYPE> px[kGo][FR][PARTS][Ws::kPieces];
#pragma unroll
    for (int g = 0; g < kGo; ++g)
#pragma unroll
      for (int r = 0; r < R; ++r) pw[g][r].template load<WHOLE, kFull>(w[r], r0 + g * kStep + own, end);
#pragma unroll
    for (int g = 0; g < kGo; ++g)
#pragma unroll
      for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int i = 0; i < Ws::kPieces; ++i)
            px[g][f][p][i].template load<WHOLE, kFull>(x[f] + p * part, r0 + g * kStep + own + 8 * i, end);
#pragma unroll
    for (int g = 0; g < kGo; ++g)
#pragma unroll
      for (int i = 0; i < Ws::kPieces; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const Piece<TYPE> one = pw[g][r].piece(i);
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p)
#pragma unroll
            for (int f = 0; f < FR; ++f) acc[r][f] = product<TYPE>(one, px[g][f][p][i], acc[r][f]);
        }
  };
  int r0 = begin + wave * kStep * kGo;
  constexpr int kUnroll = FR * PARTS * Ws::kPieces < 8 ? 2 : 1;
#pragma unroll kUnroll
  for (; r0 + kStep * kGo <= end; r0 += kWaves * kStep * kGo) go(r0, std::true_type());
  if (r0 < end) go(r0, std::false_type());
}

// With segments: a lane's own sum of row lane / 16 and x's row (lane % 16) / 4, in all four lanes that share them.
__device__ inline float segments(f32x4 v, int lane) {
  const int s = lane & 3;
  float sum = s == 0 ? v[0] : s == 1 ? v[1] : s == 2 ? v[2] : v[3];
  sum += __shfl_xor(sum, 1);
  return sum + __shfl_xor(sum, 2);
}

constexpr int kUses = 512;   // that a workgroup looks at at a time

// The uses of one expert among up to kUses of them, `first` .. `first + count - 1`: a wavefront lists them in LDS of its own,
// in order, and has their number.
struct Uses {
  int id[kUses / 64];   // the experts of a lane's uses

  __device__ void read(const Moe& a, int64_t first, int count, int lane) {
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      id[n] = -1;
      if (n * 64 < count && n * 64 + lane < count) id[n] = a.chosen[first + n * 64 + lane];
    }
  }

  __device__ int list(int expert, uint16_t* to, int count, int lane) const {
    int have = 0;
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      if (n * 64 >= count) break;
      const uint64_t mask = __ballot(id[n] == expert);
      if (id[n] == expert) to[have + __popcll(mask & ((uint64_t(1) << lane) - 1))] = static_cast<uint16_t>(n * 64 + lane);
      have += __popcll(mask);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    return have;
  }

  // the least expert above `last`, or kMostExperts
  __device__ int next(int last, int count) const {
    int least = kMostExperts;
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      if (n * 64 >= count) break;
      if (id[n] > last) least = min(least, id[n]);
    }
    for (int step = 32; step > 0; step >>= 1) least = min(least, __shfl_xor(least, step));
    return __builtin_amdgcn_readfirstlane(least);
  }
};

// act(x Wg^T) * (x Wu^T) of an expert's uses: 16 / S columns a workgroup, whose eight wavefronts share the reduction.  The
// result is stored as two values of the type, the rounded one and the rest, so that the product with Wd has it in nearly 32
// bits: one part alone would make results 1.4 times as far from exact ones as their own rounding makes them.
template <int TYPE, bool EIGHT, bool WHOLE, int S, int FR>
__global__ __launch_bounds__(512) void moe_up(Moe a) {
  using T = typename Elem<TYPE>::T;
  using W = typename Weights<TYPE, EIGHT>::W;
  constexpr int kRows = 16 / S, kTokens = 16 / S * FR;
  __shared__ uint16_t lists[kWaves][kUses];
  __shared__ float sums[kWaves][2][kTokens][kRows + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int j0 = blockIdx.x * kRows;
  const int64_t uses = int64_t(a.m) * a.top_k;
  int expert = blockIdx.y;
  if (uses < a.experts) {   // a workgroup for each use, of which the first one of an expert does the work
    const int use = expert;
    expert = __builtin_amdgcn_readfirstlane(a.chosen[use]);
    for (int at = 0; at < use; at += 64)
      if (__any(at + lane < use && a.chosen[min(at + lane, use)] == expert)) return;
  }
  const int64_t row = min(j0 + c / S, a.f - 1);
  const W* const w[2] = {static_cast<const W*>(a.w[0]) + expert * a.stride[0] + row * a.ldw[0],
                         static_cast<const W*>(a.w[1]) + expert * a.stride[1] + row * a.ldw[1]};
  for (int64_t first = 0; first < uses; first += kUses) {
    const int count = static_cast<int>(min(uses - first, int64_t(kUses)));
    Uses u;
    u.read(a, first, count, lane);
    const int have = u.list(expert, lists[wave], count, lane);
    for (int at = 0; at < have; at += kTokens) {
      const T* x[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f)
        x[f] = static_cast<const T*>(a.x) + (first + lists[wave][min(at + f * kRows + c / S, have - 1)]) / a.top_k * a.ldx;
      f32x4 acc[2][FR] = {};
      accumulate<TYPE, EIGHT, WHOLE, S, 2, FR, 1>(w, x, 0, 0, a.d, wave, lane, acc);
#pragma unroll
      for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int mat = 0; mat < 2; ++mat) {
          if constexpr (S == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wave][mat][f * 16 + c][4 * q + e] = acc[mat][f][e];
          } else {
            const float s = segments(acc[mat][f], lane);
            if ((c & 3) == 0) sums[wave][mat][f * 4 + c / 4][q] = s;
          }
        }
      __syncthreads();
      for (int t = threadIdx.x; t < kTokens * kRows; t += 512) {
        const int r = t / kRows, j = t % kRows;
        if (at + r >= have || j0 + j >= a.f) continue;
        float g[8] = {}, v = 0.0f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n) g[0] += sums[n][0][r][j], v += sums[n][1][r][j];
        if constexpr (EIGHT) {
          g[0] *= a.scale[0][int64_t(expert) * a.f + j0 + j];
          v *= a.scale[1][int64_t(expert) * a.f + j0 + j];
        }
        act8<TYPE>(g, a.act);
        v *= g[0];
        T* const h = static_cast<T*>(a.h) + (first + lists[wave][at + r]) * a.ldh + j0 + j;
        *h = T(v);
        if constexpr (TYPE != kDenseF32) {
          const float rest = v - float(T(v));
          h[uses * a.ldh] = T(fabsf(rest) < __builtin_inff() ? rest : 0.0f);   // (of an infinity there is none)
        }
      }
      __syncthreads();
    }
  }
}

constexpr int kDownRows = 64;   // rows of x that a workgroup of the down projection has at a time

// y = sum of a row's experts' h Wd^T times their shares: FI * 16 / S columns a workgroup, and one of a.splits parts of the
// reduction.  Each wavefront adds up sums of its own, over the experts in order.
template <int TYPE, bool EIGHT, bool WHOLE, int S, int FI, int FR>
__global__ __launch_bounds__(512) void moe_down(Moe a) {
  using T = typename Elem<TYPE>::T;
  using W = typename Weights<TYPE, EIGHT>::W;
  constexpr int kParts = TYPE == kDenseF32 ? 1 : 2;
  constexpr int kRows = 16 / S, kCols = kRows * FI, kTokens = kRows * FR;
  __shared__ uint16_t lists[kWaves][kUses];
  __shared__ float sums[kWaves][kDownRows][kCols];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int j0 = blockIdx.x * kCols;
  const int rows_each = min(kDownRows, kUses / a.top_k), first_row = blockIdx.y * rows_each;
  const int rows = min(rows_each, a.m - first_row), count = rows * a.top_k;
  const int64_t first = int64_t(first_row) * a.top_k, part = int64_t(a.m) * a.top_k * a.ldh;
  const int begin = static_cast<int>(int64_t(a.split_step) * blockIdx.z), end = min(a.f, begin + a.split_step);
  for (int at = lane; at < rows * kCols; at += 64) sums[wave][at / kCols][at % kCols] = 0.0f;
  Uses u;
  u.read(a, first, count, lane);
  for (int expert = u.next(-1, count); expert < kMostExperts; expert = u.next(expert, count)) {
    const int have = u.list(expert, lists[wave], count, lane);
    const W* w[FI];
#pragma unroll
    for (int i = 0; i < FI; ++i)
      w[i] = static_cast<const W*>(a.w[2]) + expert * a.stride[2] + int64_t(min(j0 + i * kRows + c / S, a.d - 1)) * a.ldw[2];
    for (int at = 0; at < have; at += kTokens) {
      const T* h[FR];
      int use[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        use[f] = lists[wave][min(at + f * kRows + c / S, have - 1)];
        h[f] = static_cast<const T*>(a.h) + (first + use[f]) * a.ldh;
      }
      f32x4 acc[FI][FR] = {};
      accumulate<TYPE, EIGHT, WHOLE, S, FI, FR, kParts>(w, h, part, begin, end, wave, lane, acc);
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        const bool in = at + f * kRows + c / S < have;
        const float share = a.share[first + use[f]];
        float* const mine = sums[wave][use[f] / a.top_k];
#pragma unroll
        for (int i = 0; i < FI; ++i) {
          auto add = [&](int j, float s) {
            s *= share;
            if constexpr (EIGHT) s *= a.scale[2][int64_t(expert) * a.d + min(j0 + j, a.d - 1)];
            if (in) mine[j] += s;
          };
          if constexpr (S == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e) add(i * 16 + 4 * q + e, acc[i][f][e]);
          } else {
            const float s = segments(acc[i][f], lane);
            if ((c & 3) == 0) add(i * 4 + q, s);
          }
        }
      }
    }
  }
  __syncthreads();
  for (int at = threadIdx.x; at < rows * kCols; at += 512) {
    const int r = at / kCols, j = j0 + at % kCols;
    if (j >= a.d) continue;
    float s = 0.0f;
#pragma unroll
    for (int n = 0; n < kWaves; ++n) s += sums[n][r][at % kCols];
    if (a.splits > 1) a.partial[(int64_t(blockIdx.z) * a.m + first_row + r) * a.d + j] = s;
    else static_cast<T*>(a.y)[(first_row + r) * a.ldy + j] = T(s);
  }
}

// the parts of a split reduction, added up in order
template <int TYPE>
__global__ __launch_bounds__(256) void moe_join(Moe a) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, all = int64_t(a.m) * a.d;
  if (at >= all) return;
  float s = 0.0f;
  for (int n = 0; n < a.splits; ++n) s += a.partial[n * all + at];
  static_cast<typename Elem<TYPE>::T*>(a.y)[at / a.d * a.ldy + at % a.d] = typename Elem<TYPE>::T(s);
}

template <int TYPE, bool EIGHT, bool WHOLE, int S, int FI, int FR>
int products(const Moe& a, hipStream_t s) {
  constexpr int kRows = 16 / S;
  const int64_t uses = int64_t(a.m) * a.top_k;
  moe_up<TYPE, EIGHT, WHOLE, S, FR><<<dim3((a.f + kRows - 1) / kRows, static_cast<uint32_t>(std::min<int64_t>(uses, a.experts))), 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0) return rc;
  const int rows = std::min(kDownRows, kUses / a.top_k), cols = kRows * FI;
  moe_down<TYPE, EIGHT, WHOLE, S, FI, FR><<<dim3((a.d + cols - 1) / cols, (a.m + rows - 1) / rows, a.splits), 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0 || a.splits == 1) return rc;
  moe_join<TYPE><<<static_cast<uint32_t>((int64_t(a.m) * a.d + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT, bool WHOLE>
int launch(const Moe& a, hipStream_t s) {
  moe_route<TYPE, WHOLE><<<static_cast<uint32_t>(a.m), 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0) return rc;
  switch (a.variant) {
    case kMoeFew: return products<TYPE, EIGHT, WHOLE, 4, 1, 1>(a, s);
    case kMoeSome: return products<TYPE, EIGHT, WHOLE, 4, 1, 2>(a, s);
    case kMoeMore: return products<TYPE, EIGHT, WHOLE, 1, 2, 1>(a, s);
    default: return products<TYPE, EIGHT, WHOLE, 1, 2, 4>(a, s);
  }
}

template <int TYPE>
int launch_type(const Moe& a, void* stream) {
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if (a.scale[0]) return a.whole ? launch<TYPE, true, true>(a, s) : launch<TYPE, true, false>(a, s);
  return a.whole ? launch<TYPE, false, true>(a, s) : launch<TYPE, false, false>(a, s);
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
