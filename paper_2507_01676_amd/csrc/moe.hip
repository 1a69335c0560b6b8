// A layer of experts for few rows on gfx950 (MI355X).  See include/embx_serving.h for the formulas.
//
// Two launches with few rows and experts, the gate and up projections of each row's experts with the activation between them
// and the down projection, which adds up a row's experts; up to three more with more: the router's logits, which experts a
// row takes and their shares, and a sum over the workgroups that shared the down projection.  Rows and their experts are pairs
// ("uses"), number row * top_k + place; a workgroup finds the uses of an expert by itself, so nothing is sorted or counted in
// memory.
//
// What bounds it is reading the weights of the experts that are used, once: 64 rows of bf16, 4 of 32 experts of 5632 x 2048, 426
// us a call, 2.2 GB at 5.2 TB/s (the up projections 268 us, 5.5 TB/s; down 143).  With few rows a launch is not long enough to
// get there (about 5 us each, of which the loads' and the routing's latency is most): one query, two of eight of 2816 x 1024,
// 16.2 us, 35 MB; five with 8-bit weights 31.3.
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

// Consecutive elements of SIZE bytes of a row, WORDS * 4 bytes in all.
template <int SIZE, int WORDS>
struct Chunk {
  u32x4 v[WORDS / 4];
  static constexpr int kPer = WORDS * 4 / SIZE;

  template <bool WHOLE>
  __device__ void load(const char* p) {
#pragma unroll
    for (int h = 0; h < WORDS / 4; ++h) {
      if constexpr (WHOLE) v[h] = *reinterpret_cast<const u32x4*>(p + 16 * h);
      else __builtin_memcpy(&v[h], p + 16 * h, 16);
    }
  }

  // keeps `left` elements, zeros behind them
  __device__ void keep(int left) {
#pragma unroll
    for (int h = 0; h < WORDS / 4; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int bytes = left * SIZE - (h * 4 + i) * 4;
        v[h][i] = bytes >= 4 ? v[h][i] : bytes <= 0 ? 0 : v[h][i] & ((1u << 8 * bytes) - 1);
      }
  }
};

// A chunk as it was loaded.  Where rows of less than 32 bits start anywhere, that is the words that it lies in, which are shifted
// when they are needed: 16-byte loads at odd addresses take twice as long.
template <int SIZE, int WORDS, bool WHOLE>
struct Loaded : Chunk<SIZE, WORDS> {
  static constexpr bool kShifted = !WHOLE && SIZE < 4;
  uint32_t more[kShifted ? 1 : 0];

  // bytes behind a word's start
  __device__ static uint32_t shift_of(const char* p) { return kShifted ? static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 3 : 0; }

  __device__ void load_at(const char* p) {
    if constexpr (kShifted) {
      const uint32_t shift = shift_of(p);
      const char* const a = p - shift;
      __builtin_memcpy(&this->v[0], __builtin_assume_aligned(a, 4), 16);
      more[0] = *reinterpret_cast<const uint32_t*>(a + (shift ? 16 : 0));   // (no word without a byte of the chunk)
    } else {
      this->template load<WHOLE>(p);
    }
  }

  // Elements at .. of a row of n, of which some may be behind its end and are something else.  Nothing is read without one of
  // the row's bytes in the same 16, or word.
  __device__ void load_end(const char* row, int at, int n) {
    constexpr int kPer16 = 16 / SIZE;
    if constexpr (kShifted) {
      const int first = min(at, n - 1);
      const char* const p = row + int64_t(first) * SIZE;
      const uint32_t shift = shift_of(p), last = (shift + min((n - first) * SIZE, 20) - 1) / 4 * 4;
#pragma unroll
      for (uint32_t i = 0; i < 4; ++i) this->v[0][i] = *reinterpret_cast<const uint32_t*>(p - shift + min(4 * i, last));
      more[0] = *reinterpret_cast<const uint32_t*>(p - shift + min(16u, last));
    } else if constexpr (WHOLE) {
#pragma unroll
      for (int h = 0; h < WORDS / 4; ++h)
        this->v[h] = *reinterpret_cast<const u32x4*>(row + int64_t(min(at + h * kPer16, (n - 1) / kPer16 * kPer16)) * SIZE);
    } else {
#pragma unroll
      for (int h = 0; h < WORDS / 4; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) this->v[h][i] = reinterpret_cast<const uint32_t*>(row)[min(at + h * 4 + i, n - 1)];
    }
  }

  __device__ Chunk<SIZE, WORDS> shifted(uint32_t shift) const {
    Chunk<SIZE, WORDS> out = *this;
    if constexpr (kShifted) {
#pragma unroll
      for (int i = 0; i < 4; ++i) out.v[0][i] = __builtin_amdgcn_alignbyte(i < 3 ? this->v[0][i + 1] : more[0], this->v[0][i], shift);
    }
    return out;
  }
};

template <int TYPE>
struct Piece : Chunk<TYPE == kDenseF32 ? 4 : 2, TYPE == kDenseF32 ? 8 : 4> {   // eight elements
  __device__ float get(int e) const {
    if constexpr (TYPE == kDenseF32) return __uint_as_float(this->v[e / 4][e % 4]);
    const uint32_t word = this->v[0][e / 2 % 4];
    if constexpr (TYPE == kDenseBF16) return __uint_as_float(e % 2 ? word & 0xffff0000u : word << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(e % 2 ? word >> 16 : word)));
  }
};

// The same of an expert's matrix, whose elements may have 8 bits (EIGHT): 16 whole numbers, exact in every type.
template <int TYPE, bool EIGHT>
struct Weights : Piece<TYPE> {
  static constexpr int kSize = TYPE == kDenseF32 ? 4 : 2, kWords = TYPE == kDenseF32 ? 8 : 4, kPieces = 1;
  __device__ const Piece<TYPE>& piece(int) const { return *this; }
};

template <int TYPE>
struct Weights<TYPE, true> : Chunk<1, 4> {
  static constexpr int kSize = 1, kWords = 4, kPieces = 2;

  __device__ Piece<TYPE> piece(int i) const {
    Piece<TYPE> out;
    uint32_t words[2] = {this->v[0][2 * i], this->v[0][2 * i + 1]};
    // (keeps the compiler from taking the bytes apart where they are loaded, a register each)
    asm("" : "+v"(words[0]), "+v"(words[1]));
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const uint32_t word = words[e / 4];
      const float lo = static_cast<float>(static_cast<int8_t>(word >> 8 * (e & 3)));
      const float hi = static_cast<float>(static_cast<int8_t>(word >> (8 * (e & 3) + 8)));
      if constexpr (TYPE == kDenseF32) {
        out.v[e / 4][e % 4] = __float_as_uint(lo), out.v[e / 4][e % 4 + 1] = __float_as_uint(hi);
      } else if constexpr (TYPE == kDenseBF16) {
        out.v[0][e / 2] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302);   // (the rest is zeros)
      } else {
        out.v[0][e / 2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
      }
    }
    return out;
  }
};

// The largest magnitude of eight values and `most`; NaN is passed over.
__device__ inline float largest(const Chunk<4, 8>& x, float most) {
#pragma unroll
  for (int e = 0; e < 8; e += 2) asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(most) : "v"(x.v[e / 4][e % 4]), "v"(x.v[e / 4][e % 4 + 1]));
  return most;
}

// f32 values are three bf16 ones that add up to them, 8 of their 24 bits each: this takes the first one off.  (FIRST: an
// infinity's rest is that of the largest number, so that its product is no NaN.)
template <bool FIRST>
__device__ inline Piece<kDenseBF16> third(Piece<kDenseF32>* x) {
  Piece<kDenseBF16> out;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    float v[2] = {x->get(e), x->get(e + 1)};
    out.v[0][e / 2] = __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      if constexpr (FIRST) v[i] = __builtin_amdgcn_fmed3f(v[i], -0x1.fffffep127f, 0x1.fffffep127f);
      v[i] -= __uint_as_float(__float_as_uint(v[i]) & 0xffff0000u);
      x->v[e / 4][e % 4 + i] = __float_as_uint(v[i]);
    }
  }
  return out;
}

// f32 values times a power of two as two f16 ones, the rounded and the rest.  (An infinity's is a number.)
__device__ inline void two_halves(const Piece<kDenseF32>& x, float scale, Piece<kDenseF16>* rounded, Piece<kDenseF16>* left) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const float v[2] = {x.get(e) * scale, x.get(e + 1) * scale};
    const f16x2 near = {static_cast<_Float16>(v[0]), static_cast<_Float16>(v[1])};
    const f16x2 rest = {static_cast<_Float16>(fmaf(static_cast<float>(near[0]), -1.0f, v[0])),
                        static_cast<_Float16>(fmaf(static_cast<float>(near[1]), -1.0f, v[1]))};
    rounded->v[0][e / 2] = __builtin_bit_cast(uint32_t, near);
    left->v[0][e / 2] = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(rest, f16x2{65504.0f, 65504.0f}));
  }
}

template <int TYPE>
__device__ inline f32x4 product(const Piece<TYPE>& w, const Piece<TYPE>& x, f32x4 c) {
  if constexpr (TYPE == kDenseF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w.v[e / 4][e % 4]), __uint_as_float(x.v[e / 4][e % 4]), c, 0, 0, 0);
    return c;
  } else {
    return mfma16<TYPE>(__builtin_bit_cast(s16x8, w.v[0]), __builtin_bit_cast(s16x8, x.v[0]), c);
  }
}

// What the router works out of some rows of x, in LDS: up to DOTS logits.
template <int DOTS>
struct Routing {
  double logit[DOTS];
  uint64_t key[DOTS];
  int chosen[DOTS];    // [rows][top_k], as shares
  float share[DOTS];
};

// The logits of x's rows from first_row on, numbers row * experts + expert, MANY at a time in a wavefront, summed in 64 bits: those
// from `from` on, every eighth, which put(number, logit) takes.
template <int TYPE, bool WHOLE, int MANY, class PUT>
__device__ inline void logits(const Moe& a, int first_row, int from, int dots, int lane, PUT put) {
  using T = typename Elem<TYPE>::T;
  for (int first = from; first < dots; first += 8 * MANY) {
    const T *r[MANY], *x[MANY];
    double sum[MANY] = {};
#pragma unroll
    for (int n = 0; n < MANY; ++n) {
      const int dot = min(first + n * 8, dots - 1), row = dot / a.experts;
      r[n] = static_cast<const T*>(a.router) + int64_t(dot - row * a.experts) * a.ldr;
      x[n] = static_cast<const T*>(a.x) + int64_t(first_row + row) * a.ldx;
    }
    auto add = [&](int j, auto full) {
      Piece<TYPE> px[MANY], pr[MANY];
      auto load = [&](Piece<TYPE>& p, const T* row) {
        const char* const bytes = reinterpret_cast<const char*>(row);
        if constexpr (decltype(full)::value) {
          p.template load<WHOLE>(bytes + int64_t(j) * sizeof(T));
        } else {
          Loaded<sizeof(T), TYPE == kDenseF32 ? 8 : 4, WHOLE> end;
          end.load_end(bytes, j, a.d);
          static_cast<Chunk<sizeof(T), TYPE == kDenseF32 ? 8 : 4>&>(p) = end.shifted(end.shift_of(bytes));
          p.keep(a.d - j);
        }
      };
#pragma unroll
      for (int n = 0; n < MANY; ++n) load(pr[n], r[n]), load(px[n], x[n]);
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int n = 0; n < MANY; ++n) sum[n] = fma(double(px[n].get(e)), double(pr[n].get(e)), sum[n]);
    };
    int j = lane * 8;
#pragma unroll (MANY == 1 ? 4 : 2)
    for (; j + 8 <= a.d; j += 512) add(j, std::true_type());
    if (j < a.d) add(j, std::false_type());
#pragma unroll
    for (int n = 0; n < MANY; ++n)
      for (int step = 32; step > 0; step >>= 1) sum[n] += __shfl_xor(sum[n], step);
#pragma unroll
    for (int n = 0; n < MANY; ++n)
      if (lane == n && first + n * 8 < dots) put(first + n * 8, sum[n]);
  }
}

// The experts of some rows and their shares; a workgroup of 512.
template <int TYPE, bool WHOLE, int DOTS>
__device__ inline void route(const Moe& a, int first_row, int rows, Routing<DOTS>& out) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), dots = rows * a.experts;
  auto put = [&](int dot, double logit) { out.logit[dot] = logit, out.key[dot] = order_of(logit); };
  if (a.logits)
    for (int dot = threadIdx.x; dot < dots; dot += 512) put(dot, a.logits[int64_t(first_row) * a.experts + dot]);
  else if (dots <= 8) logits<TYPE, WHOLE, 1>(a, first_row, wave, dots, lane, put);
  else if (DOTS == kPicked || dots <= 16) logits<TYPE, WHOLE, 2>(a, first_row, wave, dots, lane, put);
  else logits<TYPE, WHOLE, 4>(a, first_row, wave, dots, lane, put);
  __syncthreads();
  // an expert's place: how many come before it
  for (int dot = threadIdx.x; dot < dots; dot += 512) {
    const int row = dot / a.experts, e = dot - row * a.experts;
    const uint64_t mine = out.key[dot];
    int place = 0;
#pragma unroll 8
    for (int other = 0; other < a.experts; ++other) {
      const uint64_t its = out.key[row * a.experts + other];
      place += its > mine || (its == mine && other < e);
    }
    if (place < a.top_k) out.chosen[row * a.top_k + place] = e;
  }
  __syncthreads();
  for (int row = wave; row < rows; row += 8) {
    const double* const l = out.logit + row * a.experts;
    const int* const chosen = out.chosen + row * a.top_k;
    const double most = l[chosen[0]];
    const float e = lane < a.top_k ? expf(static_cast<float>(l[chosen[min(lane, a.top_k - 1)]] - most)) : 0.0f;
    float total = e;
    if (!a.renormalize) {
      total = 0.0f;
      for (int n = lane; n < a.experts; n += 64) total += expf(static_cast<float>(l[n] - most));
    }
    for (int step = 32; step > 0; step >>= 1) total += __shfl_xor(total, step);
    if (lane < a.top_k) out.share[row * a.top_k + lane] = e / total;
  }
}

// what route() has found, to memory; by the wavefronts that have found it
template <int DOTS>
__device__ inline void store(const Moe& a, int first_row, int rows, const Routing<DOTS>& r) {
  const int lane = threadIdx.x & 63;
  for (int row = threadIdx.x >> 6; row < rows; row += 8)
    if (lane < a.top_k) {
      const int64_t to = int64_t(first_row + row) * a.top_k + lane;
      a.chosen[to] = r.chosen[row * a.top_k + lane];
      a.share[to] = r.share[row * a.top_k + lane];
    }
}

// Eight logits a workgroup: one workgroup that reads the rows of 256 experts of 4096 took 70 us of the 125 of one query.
template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(512) void moe_logits(Moe a) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), first = blockIdx.x * 8;
  logits<TYPE, WHOLE, 1>(a, blockIdx.y, first + wave, min(a.experts, first + 8), lane,
                         [&](int e, double logit) { a.logits[int64_t(blockIdx.y) * a.experts + e] = logit; });
}

// a workgroup a row
template <int TYPE, bool WHOLE>
__global__ __launch_bounds__(512) void moe_route(Moe a) {
  __shared__ Routing<kMostExperts> r;
  route<TYPE, WHOLE>(a, blockIdx.x, 1, r);
  store(a, blockIdx.x, 1, r);
}

// ---------------------------------------------------------------- products
//
// A matrix instruction multiplies 16 rows of weights by 16 rows of x.  With S segments, its 16 are 16 / S rows and, of each,
// S consecutive pieces of the reduction: sums whose pieces differ mean nothing, the others are added up at the end.  So a
// workgroup can have few rows of weights, and there are enough of them where x has few rows; a row's 256 bytes are read at once.

constexpr int kWaves = 8;

// What a wavefront multiplies at a time: of R * 16 / S rows of weights by FR * 16 / S rows of x, or (HANDED) of what moe_up
// handed on, kAll of the reduction.  It is loaded while the one before it is multiplied.
//
// What is handed on is f32, and multiplied as it is.  Weights of bf16 or 8 bits multiply it as three bf16 values, which have its
// range and all of its bits.  Those of f16 multiply two f16 values of it times a power of two, which a lane keeps for its row's
// sums: the largest of the row so far is below 2^16 with it.  A larger one makes it smaller, and the sums with it.  So it has 23
// bits, or 2^-36 of the row's largest, whatever its range.
template <int TYPE, bool EIGHT, bool WHOLE, bool WHOLE_X, int S, int R, int FR, bool HANDED>
struct Step {
  static constexpr bool kThirds = HANDED && (TYPE == kDenseBF16 || (TYPE == kDenseF16 && EIGHT));
  static constexpr bool kScaled = HANDED && TYPE == kDenseF16 && !EIGHT;
  static constexpr int kType = kThirds ? kDenseBF16 : TYPE;   // of the products
  using Ws = Weights<kType, EIGHT>;
  static constexpr int kSizeX = HANDED || TYPE == kDenseF32 ? 4 : 2;
  using X = Piece<kSizeX == 4 ? kDenseF32 : TYPE>;
  static constexpr int kSpan = 4 * Ws::kPer, kStep = kSpan * S;
  static constexpr int kGo = S == 1 && TYPE != kDenseF32 && FR * (HANDED ? 2 : 1) < 4 ? 2 : 1;   // 128 bytes of a row, or 64
  static constexpr int kAll = kStep * kGo;
  static_assert(!HANDED || WHOLE_X);
  Loaded<Ws::kSize, Ws::kWords, WHOLE> w[kGo][R];
  Loaded<kSizeX, kSizeX * 2, WHOLE_X> x[kGo][FR][Ws::kPieces];
  // a lane's first element of a step
  __device__ static int own(int lane) { return (lane & (S - 1)) * kSpan + (lane >> 4) * Ws::kPer; }

  // the power of two that a lane's sums are times, by its exponent
  struct Power {
    int at[kScaled ? FR : 1];
    __device__ Power() { reset(); }
    __device__ void reset() {
#pragma unroll
      for (int f = 0; f < (kScaled ? FR : 1); ++f) at[f] = 126;
    }
    __device__ f32x4 undo(f32x4 sums, int f) const {
      if constexpr (kScaled) {
        const float back = __uint_as_float(static_cast<uint32_t>(127 - at[f]) << 23);
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[e] *= back;
      }
      return sums;
    }
  };

  // A whole step of weights from r0 on: `base` the first row of 16 / S, `row` bytes to the lane's own row and element.
  __device__ void load_w(const char* const (&base)[R], const uint32_t (&row)[R], int r0) {
#pragma unroll
    for (int g = 0; g < kGo; ++g)
#pragma unroll
      for (int r = 0; r < R; ++r) w[g][r].load_at(base[r] + int64_t(r0 + g * kStep) * Ws::kSize + row[r]);
  }

  // and of x's rows: p, at the lane's own element
  __device__ void load_x(const char* const (&p)[FR], int r0) {
#pragma unroll
    for (int g = 0; g < kGo; ++g)
#pragma unroll
      for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int i = 0; i < Ws::kPieces; ++i) x[g][f][i].load_at(p[f] + int64_t(r0 + g * kStep + 8 * i) * kSizeX);
  }

  // with the pointers that it was loaded from, as far as they lie behind words' starts
  __device__ void multiply(const char* const (&base)[R], const uint32_t (&row)[R], const char* const (&p)[FR], f32x4 (&acc)[R][FR],
                           Power& power) const {
    fit<kGo>(acc, power);
#pragma unroll
    for (int g = 0; g < kGo; ++g) products<false>(g, base, row, p, 0, acc, power);
  }

  // The last step, of which only what is below `end` is there; not loaded ahead.
  __device__ void rest(const char* const (&base)[R], const uint32_t (&row)[R], const char* const (&p)[FR], int r0, int end, int lane,
                       f32x4 (&acc)[R][FR], Power& power) {
    auto load = [&](int g, int at) {
#pragma unroll
      for (int r = 0; r < R; ++r) w[g][r].load_end(base[r] + row[r] - own(lane) * Ws::kSize, at, end);
#pragma unroll
      for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int i = 0; i < Ws::kPieces; ++i) {
          x[g][f][i].load_end(p[f] - own(lane) * kSizeX, at + 8 * i, end);
          if constexpr (WHOLE_X) x[g][f][i].keep(end - at - 8 * i);
        }
    };
    if constexpr (WHOLE) {   // (one at a time, in place: fewer registers)
      for (; r0 < end; r0 += kStep) {
        const int left = end - r0 - own(lane);
        load(0, r0 + own(lane));
#pragma unroll
        for (int r = 0; r < R; ++r) w[0][r].keep(left);
        fit<1>(acc, power);
        products<false>(0, base, row, p, 0, acc, power);
      }
    } else {
#pragma unroll
      for (int g = 0; g < kGo; ++g) load(g, r0 + g * kStep + own(lane));
      fit<kGo>(acc, power);
#pragma unroll
      for (int g = 0; g < kGo; ++g) products<true>(g, base, row, p, end - r0 - g * kStep - own(lane), acc, power);
    }
  }

  // Brings sums and their power down to what the step's first GO are about to take.
  template <int GO>
  __device__ void fit(f32x4 (&acc)[R][FR], Power& power) const {
    if constexpr (kScaled) {
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        float most = 0.0f;
#pragma unroll
        for (int g = 0; g < GO; ++g)
#pragma unroll
          for (int i = 0; i < Ws::kPieces; ++i) most = largest(x[g][f][i], most);
        if (!__any(__builtin_amdgcn_ldexpf(most, power.at[f]) > 61440.0f)) continue;   // (what rounds to a number of f16)
        // the four lanes that hold a row's step
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        // to 2^12 and more, so that the next ones hardly ever bring it down again
        const int to = min(power.at[f], 12 + 127 - static_cast<int>(min(__float_as_uint(most) >> 23, 254u)));
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[r][f][e] = __builtin_amdgcn_ldexpf(acc[r][f][e], to - power.at[f]);
        power.at[f] = to;
      }
    }
  }

  // END: only `left` of the reduction from the lane's first element on are there
  template <bool END>
  __device__ void products(int g, const char* const (&base)[R], const uint32_t (&row)[R], const char* const (&p)[FR], int left,
                           f32x4 (&acc)[R][FR], const Power& power) const {
#pragma unroll
    for (int i = 0; i < Ws::kPieces; ++i) {
      X xs[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f) {
        static_cast<Chunk<kSizeX, kSizeX * 2>&>(xs[f]) = x[g][f][i].shifted(x[g][f][i].shift_of(p[f]));
        if constexpr (END && !WHOLE_X) xs[f].keep(left - 8 * i);
      }
      Piece<kType> ws[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        Ws all;
        static_cast<Chunk<Ws::kSize, Ws::kWords>&>(all) = w[g][r].shifted(w[g][r].shift_of(base[r] + row[r]));   // (steps are whole words)
        if constexpr (END) all.keep(left);
        ws[r] = all.piece(i);
      }
      auto add = [&](const Piece<kType>(&part)[FR]) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int f = 0; f < FR; ++f) acc[r][f] = product<kType>(ws[r], part[f], acc[r][f]);
      };
      if constexpr (kThirds) {
        Piece<kType> part[FR];
#pragma unroll
        for (int n = 0; n < 3; ++n) {   // (one after another: fewer registers)
#pragma unroll
          for (int f = 0; f < FR; ++f) part[f] = n == 0 ? third<true>(&xs[f]) : third<false>(&xs[f]);
          add(part);
          if constexpr (S == 1) __builtin_amdgcn_sched_barrier(0);
        }
      } else if constexpr (kScaled) {
        Piece<kType> rounded[FR], rest[FR];
#pragma unroll
        for (int f = 0; f < FR; ++f) two_halves(xs[f], __builtin_amdgcn_ldexpf(1.0f, power.at[f]), &rounded[f], &rest[f]);
        add(rest);
        add(rounded);
      } else {
        add(xs);
      }
    }
  }
};

// With segments: a lane's own sum of row lane / 16 and x's row (lane % 16) / 4, in all four lanes that share them.
__device__ inline float segments(f32x4 v, int lane) {
  const int s = lane & 3;
  float sum = s == 0 ? v[0] : s == 1 ? v[1] : s == 2 ? v[2] : v[3];
  sum += __shfl_xor(sum, 1);
  return sum + __shfl_xor(sum, 2);
}

// Wavefronts of a SIMD, by the registers that two steps take, of which each has so many fragments of x: without a stack.
template <int TYPE, bool EIGHT, bool WHOLE>
constexpr int waves_of(int fragments) {
  return fragments * (EIGHT ? 2 : 1) * (TYPE == kDenseF32 ? 2 : 1) + (WHOLE ? 0 : EIGHT ? 2 : 4) <= (TYPE == kDenseF32 || EIGHT ? 3 : 4) ? 4 : 2;
}

// Uses of an expert that a workgroup lists before it multiplies, as many as leave room for two workgroups a CU: its weights come
// from memory once for them, and from a cache for each further 16 to 64 (as many as are multiplied at a time).
constexpr int kListed = kUses + 192;

// The uses of one expert among up to kUses of them, `first` .. `first + count - 1`: a wavefront lists them in LDS of its own,
// in order, and has their number.
struct Uses {
  int id[kUses / 64];   // the experts of a lane's uses

  template <class T>
  __device__ void read(const T* chosen, int count, int lane) {
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      id[n] = -1;
      if (n * 64 < count && n * 64 + lane < count) id[n] = chosen[n * 64 + lane];
    }
  }

  __device__ bool any(int expert) const {
    bool is = false;
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) is |= id[n] == expert;
    return __any(is);
  }

  // behind the `have` that are listed, with `before` added
  __device__ int list(int expert, uint16_t* to, int have, int before, int count, int lane) const {
#pragma unroll
    for (int n = 0; n < kUses / 64; ++n) {
      if (n * 64 >= count) break;
      const uint64_t mask = __ballot(id[n] == expert);
      if (id[n] == expert) to[have + __popcll(mask & ((uint64_t(1) << lane) - 1))] = static_cast<uint16_t>(before + n * 64 + lane);
      have += __popcll(mask);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    return have;
  }
};

// act(x Wg^T) * (x Wu^T) of an expert's uses: 16 / S columns of each of which some wavefronts share the reduction.  The
// result is handed on in f32: rounded to a type of 16 bits it would make results 1.4 times as far from exact ones as their own
// rounding makes them, and f16 has neither its range nor, below 2^-14, its bits.
// ROUTE: every workgroup routes by itself (kFused, kPicked logits at most), and the first one stores it, instead of a launch
// before this one.
// Every wavefront loads the next 128 bytes of its rows of both matrices, or 256 where 4 rows are all, while it multiplies those
// before: whole lines, and enough under way with the CU's other wavefronts.  64 bytes at a time instead took 64 rows, 4 of 32 of
// 5632 x 2048 from 433 us to 517.  (With 64 rows of x at a time, which come from 26 uses an expert on, it is 64 bytes, and so it
// is in moe_down_each with 32: registers hold no more.)
template <int TYPE, bool EIGHT, bool WHOLE, int S, int FR, bool ROUTE>
__global__ __launch_bounds__(512, (waves_of<TYPE, EIGHT, WHOLE>(FR))) void moe_up(Moe a) {
  constexpr int kRows = 16 / S, kTokens = 16 / S * FR;
  __shared__ uint16_t lists[kWaves][kListed];
  __shared__ float sums[kWaves][2][kTokens][kRows + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int sharing = a.up_waves, groups = kWaves / sharing;   // wavefronts that share a reduction; 16 / S columns each
  const int j0 = (blockIdx.x * groups + wave / sharing) * kRows;
  const int64_t uses = int64_t(a.m) * a.top_k;
  __shared__ Routing<ROUTE ? kPicked : 1> r;
  const int32_t* chosen = a.chosen;
  if constexpr (ROUTE) {
    route<TYPE, WHOLE>(a, 0, a.m, r);
    if (blockIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) store(a, 0, a.m, r);
    chosen = r.chosen;
  }
  int expert = blockIdx.y;
  if (uses < a.experts) {   // a workgroup for each use, of which the first one of an expert does the work
    const int use = expert;
    expert = __builtin_amdgcn_readfirstlane(chosen[use]);
    for (int at = 0; at < use; at += 64)
      if (__any(at + lane < use && chosen[min(at + lane, use)] == expert)) return;
  }
  using P = Step<TYPE, EIGHT, WHOLE, WHOLE, S, 2, FR, false>;
  // (16 rows of at most 2^25 elements of a row's stride: 32 bits)
  const int row0 = min(j0, a.f - 1), lane_row = min(j0 + c / S, a.f - 1) - row0;
  const char* base[2];
  uint32_t row[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    base[n] = static_cast<const char*>(a.w[n]) + (expert * a.stride[n] + row0 * a.ldw[n]) * P::Ws::kSize;
    row[n] = (static_cast<uint32_t>(lane_row) * static_cast<uint32_t>(a.ldw[n]) + P::own(lane)) * P::Ws::kSize;
  }
  const int begin = wave % sharing * P::kAll, every = sharing * P::kAll;
  for (int64_t first = 0, next = 0; first < uses; first = next) {
    P one, two;
    int have = 0;   // uses, which the workgroups along z share
    do {
      const int count = static_cast<int>(min(uses - next, int64_t(kUses)));
      Uses u;
      u.read(chosen + next, count, lane);
      if (u.any(expert)) {
        if (have == 0 && begin + P::kAll <= a.d) one.load_w(base, row, begin);   // before they are listed
        have = u.list(expert, lists[wave], have, static_cast<int>(next - first), count, lane);
      }
      next += count;
    } while (next < uses && have <= kListed - kUses && next - first <= 65536 - kUses);
    if (have == 0) continue;
    for (int at = blockIdx.z * kTokens; at < have; at += gridDim.z * kTokens) {
      const char* x[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f)
        x[f] = static_cast<const char*>(a.x) +
               ((first + lists[wave][min(at + f * kRows + c / S, have - 1)]) / a.top_k * a.ldx + P::own(lane)) * P::kSizeX;
      f32x4 acc[2][FR] = {};
      typename P::Power power;
      int r0 = begin;
      if (begin + P::kAll <= a.d) {
        if (at != static_cast<int>(blockIdx.z) * kTokens) one.load_w(base, row, begin);
        one.load_x(x, begin);
        auto go = [&](const P& now, P& next) {   // whether there is a next one
          r0 += every;
          const bool more = r0 + P::kAll <= a.d;
          if (more) next.load_w(base, row, r0), next.load_x(x, r0);
          now.multiply(base, row, x, acc, power);
          return more;
        };
        while (go(one, two) && go(two, one)) {}
      }
      if (r0 < a.d) one.rest(base, row, x, r0, a.d, lane, acc, power);
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
      for (int t = threadIdx.x; t < kTokens * kRows * groups; t += 512) {
        const int r = t / (kRows * groups), group = t / kRows % groups, column = t % kRows;
        const int j = (blockIdx.x * groups + group) * kRows + column;
        if (at + r >= have || j >= a.f) continue;
        float g = 0.0f, v = 0.0f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n) {
          const int from = group * sharing + min(n, sharing - 1);
          g += n < sharing ? sums[from][0][r][column] : 0.0f, v += n < sharing ? sums[from][1][r][column] : 0.0f;
        }
        if constexpr (EIGHT) {
          g *= a.scale[0][int64_t(expert) * a.f + j];
          v *= a.scale[1][int64_t(expert) * a.f + j];
        }
        v *= act_f(g, a.act);
        // (a NaN whose upper half says so)
        a.h[(first + lists[wave][at + r]) * a.ldh + j] = v == v ? v : __uint_as_float(0x7fc00000u);
      }
      __syncthreads();
    }
  }
}

// y = sum of a row's experts' h Wd^T times their shares: FI * 16 / S columns of a.down_rows rows.  That is items, an expert and
// a.chunk of the reduction, which the wavefronts of a.splits workgroups take in turn; each adds up sums of its own, so that no
// expert waits for another.  Neighbouring items go to neighbouring workgroups: experts have unlike numbers of rows (five rows,
// 2 of 8 of 2816 x 1024, 8-bit weights 31.3 us a call, 32.7 with eight items in a row to a workgroup; 128 rows 75.8 and 78.8).
template <int TYPE, bool EIGHT, bool WHOLE, int S, int FI, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 16 ? 4 : (waves_of<TYPE, EIGHT, WHOLE>(TYPE == kDenseF32 ? 1 : 2))) void moe_down(Moe a) {
  using T = typename Elem<TYPE>::T;
  constexpr int FR = 1, kRows = 16 / S, kCols = kRows * FI, kTokens = kRows * FR;
  __shared__ uint16_t lists[WAVES][2][kDownRows], used[kUses], ids[kUses];   // (a row uses an expert once)
  __shared__ uint32_t mask[kMostExperts / 32];
  __shared__ float sums[WAVES][kDownRows][kCols];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), q = lane >> 4, c = lane & 15;
  const int j0 = blockIdx.x * kCols;
  const int first_row = blockIdx.y * a.down_rows, rows = min(a.down_rows, a.m - first_row), count = rows * a.top_k;
  const int64_t first = int64_t(first_row) * a.top_k;
  int32_t id = -1;   // (wavefronts from kUses / 64 on have none)
  if (tid < count) ids[tid] = static_cast<uint16_t>(id = a.chosen[first + tid]);
  if (tid < kMostExperts / 32) mask[tid] = 0;
  for (int at = lane; at < rows * kCols; at += 64) sums[wave][at / kCols][at % kCols] = 0.0f;
  __syncthreads();
  // the experts that are used, in order
  if (id >= 0) atomicOr(&mask[id >> 5], 1u << (id & 31));
  __syncthreads();
  for (int e = tid; e < a.experts; e += 64 * WAVES) {
    if (!(mask[e >> 5] >> (e & 31) & 1)) continue;
    int at = __popc(mask[e >> 5] & ((1u << (e & 31)) - 1));
    for (int n = 0; n < e >> 5; ++n) at += __popc(mask[n]);
    used[at] = static_cast<uint16_t>(e);
  }
  int total = 0;
  for (int n = 0; n < (a.experts + 31) / 32; ++n) total += __popc(mask[n]);
  __syncthreads();
  const int chunks = (a.f + a.chunk - 1) / a.chunk;
  using P = Step<TYPE, EIGHT, WHOLE, true, S, FI, FR, true>;   // (rows of h start at multiples of 16 bytes)
  // Where a wavefront is: an item, its expert's uses from `at` on, and r0 of its reduction.
  struct Place {
    int item, expert, to, have, at, r0, which;
    const char* w[FI];
    uint32_t row[FI];
    const char* h[FR];
    int use[FR];
  };
  auto begin_item = [&](Place& p) {
    p.expert = __builtin_amdgcn_readfirstlane(used[p.item / chunks]);
    p.which ^= 1;
    Uses u;   // (held, its registers would be those of the loads)
    u.read(ids, count, lane);
    p.have = u.list(p.expert, lists[wave][p.which], 0, 0, count, lane);
#pragma unroll
    for (int i = 0; i < FI; ++i) {
      const int row0 = min(j0 + i * kRows, a.d - 1);
      p.w[i] = static_cast<const char*>(a.w[2]) + (p.expert * a.stride[2] + row0 * a.ldw[2]) * P::Ws::kSize;
      p.row[i] = (static_cast<uint32_t>(min(j0 + i * kRows + c / S, a.d - 1) - row0) * static_cast<uint32_t>(a.ldw[2]) + P::own(lane)) *
                 P::Ws::kSize;
    }
    p.at = 0;
  };
  auto begin_rows = [&](Place& p) {
    p.r0 = p.item % chunks * a.chunk, p.to = min(a.f, p.r0 + a.chunk);
#pragma unroll
    for (int f = 0; f < FR; ++f) {
      p.use[f] = lists[wave][p.which][min(p.at + f * kRows + c / S, p.have - 1)];
      p.h[f] = reinterpret_cast<const char*>(a.h + (first + p.use[f]) * a.ldh + P::own(lane));
    }
  };
  auto load = [&](P& s, const Place& p) {
    if (p.r0 + P::kAll <= p.to) s.load_w(p.w, p.row, p.r0), s.load_x(p.h, p.r0);
  };
  f32x4 acc[FI][FR] = {};
  typename P::Power power;
  auto finish = [&](const Place& p) {
#pragma unroll
    for (int f = 0; f < FR; ++f) {
      const bool in = p.at + f * kRows + c / S < p.have;
      const float share = a.share[first + p.use[f]];
      float* const mine = sums[wave][p.use[f] / a.top_k];
#pragma unroll
      for (int i = 0; i < FI; ++i) {
        const f32x4 whole = power.undo(acc[i][f], f);
        auto add = [&](int j, float s) {
          s *= share;
          if constexpr (EIGHT) s *= a.scale[2][int64_t(p.expert) * a.d + min(j0 + j, a.d - 1)];
          if (in) mine[j] += s;
        };
        if constexpr (S == 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e) add(i * 16 + 4 * q + e, whole[e]);
        } else {
          const float s = segments(whole, lane);
          if ((c & 3) == 0) add(i * 4 + q, s);
        }
        acc[i][f] = f32x4{};
      }
    }
    power.reset();
  };
  const int items = total * chunks;
  P one, two;
  Place now = {wave * static_cast<int>(gridDim.z) + static_cast<int>(blockIdx.z)}, then;
  bool more = now.item < items;
  if (more) begin_item(now), begin_rows(now), load(one, now);
  auto go = [&](P& s, P& other) {
    then = now;
    if (now.r0 + P::kAll <= now.to) then.r0 += P::kAll;
    const bool last = then.r0 + P::kAll > then.to;
    const int left = then.r0;   // where whole steps end
    if (last) {
      then.at += kTokens;
      if (then.at >= then.have) {
        then.item += static_cast<int>(gridDim.z) * WAVES;
        more = then.item < items;
        if (more) begin_item(then);
      }
      if (more) begin_rows(then);
    }
    if (more && then.r0 + P::kAll <= then.to && left > now.r0) {   // (a block of its own waits for what it multiplies, and no more)
      other.load_w(then.w, then.row, then.r0), other.load_x(then.h, then.r0);
      s.multiply(now.w, now.row, now.h, acc, power);
      asm volatile("");
    } else {
      if (more) load(other, then);
      if (left > now.r0) s.multiply(now.w, now.row, now.h, acc, power);
    }
    if (last) {
      if (left < now.to) s.rest(now.w, now.row, now.h, left, now.to, lane, acc, power);
      finish(now);
    }
    now = then;
  };
  while (more) {
    go(one, two);
    if (!more) break;
    go(two, one);
  }
  __syncthreads();
  for (int at = threadIdx.x; at < rows * kCols; at += 64 * WAVES) {
    const int r = at / kCols, j = j0 + at % kCols;
    if (j >= a.d) continue;
    float s = 0.0f;
#pragma unroll
    for (int n = 0; n < WAVES; ++n) s += sums[n][r][at % kCols];
    if (a.splits > 1) a.partial[(int64_t(blockIdx.z) * a.m + first_row + r) * a.d + j] = s;
    else static_cast<T*>(a.y)[(first_row + r) * a.ldy + j] = T(s);
  }
}

// The same for many rows: the uses of one expert and 32 columns for some wavefronts, as in moe_up, so that its weights come from
// memory once, and not once for every a.down_rows rows: 200 rows, 4 of 64 of 704 x 4096 302 us a call, by rows 445.  Results go to
// memory in f32, a row for each use, without their shares.
template <int TYPE, bool WHOLE, int FR>
__global__ __launch_bounds__(512, (waves_of<TYPE, false, WHOLE>(TYPE == kDenseF32 ? FR : 2 * FR))) void moe_down_each(Moe a) {
  constexpr int kTokens = 16 * FR, kCols = 32;
  __shared__ uint16_t lists[kWaves][kListed];
  __shared__ float sums[kWaves][kTokens][kCols + 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const int sharing = a.down_waves, groups = kWaves / sharing, expert = blockIdx.y;
  const int j0 = (blockIdx.x * groups + wave / sharing) * kCols;
  const int64_t uses = int64_t(a.m) * a.top_k;
  using P = Step<TYPE, false, WHOLE, true, 1, 2, FR, true>;
  const char* base[2];
  uint32_t row[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int row0 = min(j0 + n * 16, a.d - 1), lane_row = min(j0 + n * 16 + c, a.d - 1) - row0;
    base[n] = static_cast<const char*>(a.w[2]) + (expert * a.stride[2] + row0 * a.ldw[2]) * P::Ws::kSize;
    row[n] = (static_cast<uint32_t>(lane_row) * static_cast<uint32_t>(a.ldw[2]) + P::own(lane)) * P::Ws::kSize;
  }
  const int begin = wave % sharing * P::kAll, every = sharing * P::kAll;
  for (int64_t first = 0, next = 0; first < uses; first = next) {
    P one, two;
    int have = 0;   // uses, which the workgroups along z share
    do {
      const int count = static_cast<int>(min(uses - next, int64_t(kUses)));
      Uses u;
      u.read(a.chosen + next, count, lane);
      if (u.any(expert)) {
        if (have == 0 && begin + P::kAll <= a.f) one.load_w(base, row, begin);   // before they are listed
        have = u.list(expert, lists[wave], have, static_cast<int>(next - first), count, lane);
      }
      next += count;
    } while (next < uses && have <= kListed - kUses && next - first <= 65536 - kUses);
    if (have == 0) continue;
    for (int at = blockIdx.z * kTokens; at < have; at += gridDim.z * kTokens) {
      const char* h[FR];
#pragma unroll
      for (int f = 0; f < FR; ++f)
        h[f] = reinterpret_cast<const char*>(a.h + (first + lists[wave][min(at + f * 16 + c, have - 1)]) * a.ldh + P::own(lane));
      f32x4 acc[2][FR] = {};
      typename P::Power power;
      int r0 = begin;
      if (begin + P::kAll <= a.f) {
        if (at != static_cast<int>(blockIdx.z) * kTokens) one.load_w(base, row, begin);
        one.load_x(h, begin);
        auto go = [&](const P& now, P& next) {   // whether there is a next one
          r0 += every;
          const bool more = r0 + P::kAll <= a.f;
          if (more) next.load_w(base, row, r0), next.load_x(h, r0);
          now.multiply(base, row, h, acc, power);
          return more;
        };
        while (go(one, two) && go(two, one)) {}
      }
      if (r0 < a.f) one.rest(base, row, h, r0, a.f, lane, acc, power);
#pragma unroll
      for (int f = 0; f < FR; ++f)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 whole = power.undo(acc[i][f], f);
#pragma unroll
          for (int e = 0; e < 4; ++e) sums[wave][f * 16 + c][i * 16 + 4 * q + e] = whole[e];
        }
      __syncthreads();
      for (int t = threadIdx.x; t < kTokens * kCols * groups; t += 512) {
        const int r = t / (kCols * groups), group = t / kCols % groups, column = t % kCols;
        const int j = (blockIdx.x * groups + group) * kCols + column;
        if (at + r >= have || j >= a.d) continue;
        float v = 0.0f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n) v += n < sharing ? sums[group * sharing + min(n, sharing - 1)][r][column] : 0.0f;
        a.partial[(first + lists[wave][at + r]) * a.d + j] = v;
      }
      __syncthreads();
    }
  }
}

// and the sums over a row's experts
template <int TYPE>
__global__ __launch_bounds__(256) void moe_join_uses(Moe a) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t row = at / a.d, j = at % a.d;
  if (row >= a.m) return;
  float s = 0.0f;
  for (int64_t use = row * a.top_k; use < (row + 1) * a.top_k; ++use) s += a.share[use] * a.partial[use * a.d + j];
  static_cast<typename Elem<TYPE>::T*>(a.y)[row * a.ldy + j] = typename Elem<TYPE>::T(s);
}

// the parts of workgroups that shared a down projection, added up in order.  (About 3 us a call.  The last workgroup to arrive can
// do it, but has to write its CUs' caches back first and the others' parts may not be in its own: five rows, 2 of 8 of
// 2816 x 1024 with 8-bit weights 66 us so, 32 with this launch.)
template <int TYPE>
__global__ __launch_bounds__(256) void moe_join(Moe a) {
  const int64_t at = int64_t(blockIdx.x) * 256 + threadIdx.x, all = int64_t(a.m) * a.d;
  if (at >= all) return;
  float s = 0.0f;
  for (int n = 0; n < a.splits; ++n) s += a.partial[n * all + at];
  static_cast<typename Elem<TYPE>::T*>(a.y)[at / a.d * a.ldy + at % a.d] = typename Elem<TYPE>::T(s);
}

template <int TYPE, bool EIGHT, bool WHOLE, int S, int FR>
int up(const Moe& a, hipStream_t s) {
  const int columns = 16 / S * (kWaves / a.up_waves);
  const int64_t experts = std::min<int64_t>(int64_t(a.m) * a.top_k, a.experts);
  const dim3 grid((a.f + columns - 1) / columns, static_cast<uint32_t>(experts), a.up_parts);
  if (a.logits) {
    moe_logits<TYPE, WHOLE><<<dim3((a.experts + 7) / 8, static_cast<uint32_t>(a.m)), 512, 0, s>>>(a);
    if (const int rc = hipGetLastError(); rc != 0) return rc;
  }
  if (a.fused && FR == 1) {
    moe_up<TYPE, EIGHT, WHOLE, S, 1, true><<<grid, 512, 0, s>>>(a);
  } else {
    moe_route<TYPE, WHOLE><<<static_cast<uint32_t>(a.m), 512, 0, s>>>(a);
    if (const int rc = hipGetLastError(); rc != 0) return rc;
    moe_up<TYPE, EIGHT, WHOLE, S, FR, false><<<grid, 512, 0, s>>>(a);
  }
  return hipGetLastError();
}

template <int TYPE, bool EIGHT, bool WHOLE, int S, int FI, int WAVES>
int down(const Moe& a, hipStream_t s) {
  const int columns = 16 / S * FI;
  const dim3 grid((a.d + columns - 1) / columns, (a.m + a.down_rows - 1) / a.down_rows, a.splits);
  moe_down<TYPE, EIGHT, WHOLE, S, FI, WAVES><<<grid, 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE, bool WHOLE>
int down_each(const Moe& a, hipStream_t s) {
  const int columns = 32 * (kWaves / a.down_waves);
  const dim3 grid((a.d + columns - 1) / columns, a.experts, a.down_parts);
  if (TYPE == kDenseF32 || a.down_blocks == 1) moe_down_each<TYPE, WHOLE, 1><<<grid, 512, 0, s>>>(a);
  else moe_down_each<TYPE, WHOLE, TYPE == kDenseF32 ? 1 : 2><<<grid, 512, 0, s>>>(a);
  if (const int rc = hipGetLastError(); rc != 0) return rc;
  moe_join_uses<TYPE><<<static_cast<uint32_t>((int64_t(a.m) * a.d + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
}

template <int TYPE, bool EIGHT, bool WHOLE>
int launch(const Moe& a, hipStream_t s) {
  int rc;
  switch (a.up_variant) {
    case kMoeFew: rc = up<TYPE, EIGHT, WHOLE, 4, 1>(a, s); break;
    case kMoeMore: rc = up<TYPE, EIGHT, WHOLE, 1, 1>(a, s); break;
    default:
      if (a.up_blocks == 2) {
        rc = up<TYPE, EIGHT, WHOLE, 1, 2>(a, s);
        break;
      }
      if constexpr (!EIGHT && TYPE != kDenseF32) rc = up<TYPE, EIGHT, WHOLE, 1, 4>(a, s);   // (the others have no registers for it)
      else rc = hipErrorInvalidValue;
  }
  if (rc != 0) return rc;
  if constexpr (!EIGHT)
    if (a.down_variant == kMoeMany) return down_each<TYPE, WHOLE>(a, s);
  if (a.down_variant != kMoeFew) rc = down<TYPE, EIGHT, WHOLE, 1, 2, 8>(a, s);
  else if (a.down_waves == 16) rc = down<TYPE, EIGHT, WHOLE, 4, 1, 16>(a, s);
  else rc = down<TYPE, EIGHT, WHOLE, 4, 1, 8>(a, s);
  if (rc != 0 || a.splits == 1) return rc;
  moe_join<TYPE><<<static_cast<uint32_t>((int64_t(a.m) * a.d + 255) / 256), 256, 0, s>>>(a);
  return hipGetLastError();
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
