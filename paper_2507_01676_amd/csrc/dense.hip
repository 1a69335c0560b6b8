// Dense layers for gfx950 (MI355X): the matrix products of fully connected layers and gated
// feed-forward blocks, forward and backward.  See include/embx_dense.h for the formulas.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "../../include/embx_dense.h"
#include "dense.hpp"
#include "dense_device.hpp"
#include "quantize_device.hpp"

#ifndef EMBX_DPART
#define EMBX_DPART -1
#endif
#define EMBX_HAS_DPART(p) (EMBX_DPART < 0 || EMBX_DPART == (p))

namespace embx {
namespace {

// ---------------------------------------------------------------- tiles
//
// A workgroup computes BM x BN sums (kGated: BN / 2 columns of each projection) in WI x WJ
// wavefronts.  Each step takes 128 bytes of the reduction (BK elements) of both operands from LDS, while
// later steps are on their way there.  A tile of 16-bit elements lies in LDS as in memory: rows of BK elements
// (operand along the reduction) or BK rows of BM or BN elements (reduction-major), with the
// 16-byte chunks of a row permuted so that what a wavefront reads at once lies in different
// banks (counted: no conflicts; half the step, rows of 64 bytes, had them in 49% of the LDS cycles).  Chunks go from
// memory to LDS without registers, so their order within a wavefront's
// 1 KB is fixed in LDS, and the permutation is applied to the address each lane loads from.
constexpr int kOutOfRange = static_cast<int>(0x80000000u);   // past every descriptor: reads zeros

#define LDS_PTR(T) __attribute__((address_space(3))) T*

// elements from an operand's start to a column of its first row: see kPanel
__device__ inline int64_t column_at(int column, int64_t panel) {
  return int64_t(column >> kPanelLog) * panel + (column & (int(kPanel) - 1));
}

__device__ inline uint32_t lds_address(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((LDS_PTR(const void))p));
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

__device__ inline i32x4 descriptor(const void* base) {
  const uint64_t p = reinterpret_cast<uint64_t>(base);
  i32x4 r;
  r[0] = __builtin_amdgcn_readfirstlane(static_cast<int>(p));
  r[1] = __builtin_amdgcn_readfirstlane(static_cast<int>(p >> 32) & 0xffff);
  r[2] = 0x7fffffff;
  r[3] = 0x00027000;
  return r;
}

// 16 bytes a lane from descriptor + voffset to LDS at lds + 16 * lane.  The wait for it is
// written out where the tile is needed (stage_done): the compiler, told of the write, would
// wait at the next LDS read of any kind.  (It is told of m0, which it reserves for instructions like this one, and warns
// that it will not save it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ inline void load_to_lds(i32x4 rsrc, int voffset, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(voffset), "s"(rsrc) : "memory", "m0");
}
#pragma clang diagnostic pop

// Waits until all but this wavefront's last LOADS loads are in LDS and every LDS read of it is done,
// then for the other wavefronts.
template <int LOADS>
__device__ inline void stage_done() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LOADS) : "memory");
}

__device__ f32x4 buffer_load_f32x4(i32x4 rsrc, int voffset, int soffset, int aux) __asm("llvm.amdgcn.raw.buffer.load.v4f32");

// One operand's tile of ROWS results (rows of x or dz, columns of the result) by BK elements of SIZE bytes of the reduction.
// RM: reduction-major in memory (16-bit elements).
template <int ROWS, bool RM, int WAVES, int SIZE = 2>
struct Tile {
  static constexpr int BK = 128 / SIZE, kPer = 16 / SIZE;     // kPer: elements of a chunk
  static_assert(!RM || SIZE == 2);
  static constexpr int kBytes = ROWS * 128;
  static constexpr int kLoads = kBytes / 1024 / WAVES;        // 1 KB pieces a wavefront loads
  static constexpr int kRowBytes = RM ? ROWS * 2 : 128;
  static constexpr int kChunks = kRowBytes / 16;
  static constexpr int kRowsPerLoad = 1024 / kRowBytes;
  static_assert(kBytes % (1024 * WAVES) == 0, "every wavefront loads alike");

  // the permutation of a row's chunks
  __device__ static int swizzle(int row) {
    if (RM) return (kChunks >= 16 ? (row & 3) | ((row >> 1) & 4) : row & 3) << 1;
    return (row >> 1) & 7;
  }

  // row and chunk in memory that this lane loads with piece n
  __device__ static int load_row(int n, int wave, int lane) { return (n * WAVES + wave) * kRowsPerLoad + lane / kChunks; }
  __device__ static int load_chunk(int row, int lane) { return (lane % kChunks) ^ swizzle(row); }

  int voff[kLoads];

  // rows: valid rows (RM: valid columns, whole chunks) from the tile's origin on
  __device__ void init(int wave, int lane, int64_t ld, int rows) {
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const int row = load_row(n, wave, lane), chunk = load_chunk(row, lane);
      const bool in = RM ? chunk * kPer < rows : row < rows;
      voff[n] = in ? static_cast<int>(row * ld * SIZE) + chunk * 16 : kOutOfRange;
    }
  }

  // valid: how many of this step's BK are inside
  __device__ void load(i32x4 rsrc, uint32_t lds, int wave, int lane, int valid, int n) const {
    int v = voff[n];
    if (valid < BK) {
      const int row = load_row(n, wave, lane), chunk = load_chunk(row, lane);
      v = (RM ? row < valid : chunk * kPer < valid) ? v : kOutOfRange;
    }
    load_to_lds(rsrc, v, lds + (n * WAVES + wave) * 1024);
  }

  // fragment of 16 results (from `first` on, a multiple of 16) by half of the step (half ks): lane: result
  // lane % 16, chunk lane / 16 of the half
  __device__ static s16x8 fragment(const char* tile, int first, int ks, int lane) {
    const int q = lane >> 4, c = lane & 15;
    if constexpr (RM) {
      const int r = ks * 32 + 8 * q + (c >> 2);
      const int unit = (first >> 4) ^ (swizzle(r) >> 1);     // (r + 4 has the same permutation)
      const char* p = tile + r * kRowBytes + unit * 32 + (c & 3) * 8;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(p + 4 * kRowBytes));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = first + c;
      return *reinterpret_cast<const s16x8*>(tile + row * kRowBytes + (((ks * 4 + q) ^ swizzle(row)) << 4));
    }
  }
};

// f32 products.  The matrix cores multiply f32 at a sixteenth of their bf16 rate.  So each f32 value, times 2^24, is taken as
// a sum of three bf16 values (the value rounded, the rest rounded, the rest of that: 24 bits in all, exact for every normal
// value: the last bit, 2^-149 at least, is 2^-125 at least then, and no part is too small for a normal bf16), and a product
// as the six of their nine products that count; the other three come to 2^-23 of it at most.  Small ones are added first,
// and the finished sum is multiplied by 2^-48.  Six bf16 products for each f32 one are 2.7 times less
// work than f32 products, at f32's accuracy.  Values or sums too large for this (2^104 or 2^80, about), infinities and NaN
// turn the sums that they reach into infinities or NaN, and a tile with sums that are not finite is computed again with f32
// products (tile_by_f32).  The first factor costs 1% (4096^3 610 us when it was added, without it 606).
struct Parts { s16x8 p[3]; };   // high to low

constexpr float kScale = 0x1p24f;

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ inline uint32_t round2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

__device__ inline Parts split3(const float* v) {
  u32x4 part[3];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = v[2 * e] * kScale, b = v[2 * e + 1] * kScale;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      part[p][e] = round2(a, b);
      a -= __uint_as_float(part[p][e] << 16), b -= __uint_as_float(part[p][e] & 0xffff0000u);
    }
  }
  return {{__builtin_bit_cast(s16x8, part[0]), __builtin_bit_cast(s16x8, part[1]), __builtin_bit_cast(s16x8, part[2])}};
}

// The parts of a tile of f32 (ROWS results by 32 of the reduction) in LDS: a tile of bf16 for each.  Taken apart once for
// the workgroup, not at each wavefront's fragments: the matrix cores and the other vector instructions of a SIMD overlap
// by half at most (8 matrix instructions take 160 cycles, 32 others 173, all of them from two wavefronts 249), so every
// instruction of the latter counts.  4096 x 4096 x 4096: 595 us; with the parts taken at the fragments
// 46 more.
template <int ROWS, bool RM, int WAVES>
struct PartTile {
  static constexpr int kBytes = ROWS * 64;                     // of a part
  static constexpr int kRowBytes = RM ? ROWS * 2 : 64, kChunks = kRowBytes / 16;   // chunks of eight values
  static constexpr int kPieces = (ROWS * 4 + 64 * WAVES - 1) / (64 * WAVES);   // of a thread

  __device__ static int swizzle(int row) {
    if (RM) return (kChunks >= 16 ? (row & 3) | ((row >> 1) & 4) : row & 3) << 1;
    return -(row >> 2) & 3;
  }

  // A thread's pieces of eight values: loaded from memory (what lies outside is read as zeros), then taken apart and
  // written to the parts, `plane` bytes apart.
  int voff[kPieces][2];
  f32x4 held[kPieces][2];

  __device__ static bool mine(int at) { return ROWS * 4 >= 64 * WAVES || at < ROWS * 4; }

  // rows: valid rows (RM: valid columns, whole chunks) from the tile's origin on
  __device__ void init(int tid, int64_t ld, int rows) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int at = n * 64 * WAVES + tid, row = at / kChunks, first = at % kChunks * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        voff[n][h] = mine(at) && (RM ? first + 4 * h < rows : row < rows) ? static_cast<int>(row * ld * 4) + (first + 4 * h) * 4
                                                                          : kOutOfRange;
    }
  }

  // valid: how many of this step's 32 are inside
  __device__ void load(i32x4 rsrc, int tid, int valid) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int at = n * 64 * WAVES + tid, row = at / kChunks, first = at % kChunks * 8;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int v = voff[n][h];
        if (valid < 32) v = (RM ? row < valid : first + 4 * h < valid) ? v : kOutOfRange;
        held[n][h] = buffer_load_f32x4(rsrc, v, 0, 0);
      }
    }
  }

  __device__ void take_apart(char* to, int plane, int tid) const {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int at = n * 64 * WAVES + tid, row = at / kChunks, chunk = at % kChunks;
      if (!mine(at)) break;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = held[n][e / 4][e % 4];
      const Parts parts = split3(v);
      char* p = to + row * kRowBytes + ((chunk ^ swizzle(row)) << 4);
#pragma unroll
      for (int part = 0; part < 3; ++part) *reinterpret_cast<s16x8*>(p + part * plane) = parts.p[part];
    }
  }

  // as Tile::fragment
  __device__ static s16x8 fragment(const char* tile, int first, int lane) {
    const int q = lane >> 4, c = lane & 15;
    if constexpr (RM) {
      const int r = 8 * q + (c >> 2);
      const char* p = tile + r * kRowBytes + (((first >> 4) ^ (swizzle(r) >> 1)) << 5) + (c & 3) * 8;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))p);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s16x4))(p + 4 * kRowBytes));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const int row = first + c;
      return *reinterpret_cast<const s16x8*>(tile + row * kRowBytes + ((q ^ swizzle(row)) << 4));
    }
  }
};

// c[fi][fj] += the products of FI by FJ fragments
template <int FI, int FJ>
__device__ inline void products6(const Parts* a, const Parts* b, f32x4 (*c)[FJ]) {
  constexpr int kA[6] = {2, 0, 1, 1, 0, 0}, kB[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
  for (int n = 0; n < 6; ++n)
#pragma unroll
    for (int fi = 0; fi < FI; ++fi)
#pragma unroll
      for (int fj = 0; fj < FJ; ++fj) c[fi][fj] = mfma16<kDenseBF16>(b[fj].p[kB[n]], a[fi].p[kA[n]], c[fi][fj]);
}

// Which tile a workgroup computes.  Workgroups go round-robin over the 8 XCDs, each with an L2 of its
// own: XCD x takes the x-th eighth of the tiles, in bands of kBand tile rows walked column by column,
// so that the tiles in flight on one XCD share few rows of A and of B.
constexpr int kBand = 4;

__device__ inline void tile_of(uint32_t id, uint32_t tiles_i, uint32_t tiles_j, int* ti, int* tj) {
  const uint32_t tiles = tiles_i * tiles_j;
  const uint32_t per = tiles / kXcds, more = tiles % kXcds;
  const uint32_t x = id % kXcds, at = id / kXcds;
  const uint32_t t = x * per + min(x, more) + at;
  const uint32_t band = t / (kBand * tiles_j), in = t % (kBand * tiles_j);
  const uint32_t rows = min(static_cast<uint32_t>(kBand), tiles_i - band * kBand);
  *ti = band * kBand + in % rows;
  *tj = in / rows;
}

// Turns sums into results: eight consecutive columns, from j on, of a lane's rows, which are `step` rows apart.  What does
// not change from row to row is worked out once: of products with short sums the epilogue's instructions are a good part.
template <int TYPE, int KIND>
struct Finish {
  using T = typename Elem<TYPE>::T;
  static constexpr bool kFwd = KIND == kForward || KIND == kGated;
  static constexpr int kMats = KIND == kGated ? 2 : 1;
  T* y;
  T* z[kMats];
  const T* r;
  int64_t y_step, z_step[kMats], r_step;
  float bias[kMats][8];
  int n, act;
  bool has_z[kMats], has_r, has_bias;

  __device__ Finish(const DenseGemm& g, int part, int64_t i, int j, int step) : n(min(8, g.nj - j)), act(g.act) {
    const int at = kFwd ? 0 : part;
    y = static_cast<T*>(g.c[at]) + i * g.ldc[at] + j;
    y_step = step * g.ldc[at];
    if constexpr (kFwd) {
      has_bias = g.bias[0] || (kMats == 2 && g.bias[1]);
#pragma unroll
      for (int m = 0; m < kMats; ++m) {
        has_z[m] = g.z[m];
        z[m] = static_cast<T*>(g.z[m]) + i * g.ldz[m] + j;
        z_step[m] = step * g.ldz[m];
#pragma unroll
        for (int e = 0; e < 8; ++e) bias[m][e] = 0.0f;
        if (g.bias[m] && n > 0) load8<TYPE>(static_cast<const T*>(g.bias[m]) + j, n, bias[m]);
      }
      has_r = KIND == kForward && g.res;
      r = static_cast<const T*>(g.res) + i * g.ldr + j;
      r_step = step * g.ldr;
    }
  }

  __device__ void next() {
    y += y_step;
    if constexpr (kFwd) {
#pragma unroll
      for (int m = 0; m < kMats; ++m) z[m] += z_step[m];
      r += r_step;
    }
  }

  // of a row that is inside (n >= 1)
  __device__ void put(float* s0, float* s1) const {
    if constexpr (kFwd) {
      if (has_bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s0[e] += bias[0][e];
      }
      if (has_z[0]) store8<TYPE>(z[0], n, s0);
      act8<TYPE>(s0, act);
      if constexpr (KIND == kGated) {
        if (has_bias) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s1[e] += bias[1][e];
        }
        if (has_z[1]) store8<TYPE>(z[1], n, s1);
#pragma unroll
        for (int e = 0; e < 8; ++e) s0[e] *= s1[e];
      } else if (has_r) {
        float b[8];
        load8<TYPE>(r, n, b);
#pragma unroll
        for (int e = 0; e < 8; ++e) s0[e] += b[e];
      }
    }
    store8<TYPE>(y, n, s0);
  }
};

// The same for products of 8-bit integers: y = act(s_i t_j sum + b_j) + r, whose bias, residual and result have a type of
// their own.  Sums become f32 here (2^-24 of themselves at most, as the products with both scales).
template <>
struct Finish<kDenseI8, kForward> {
  const DenseGemm& g;
  int64_t i;
  int j, n, step;
  float scale[8], bias[8];

  __device__ Finish(const DenseGemm& g_, int, int64_t i_, int j_, int step_) : g(g_), i(i_), j(j_), n(min(8, g_.nj - j_)), step(step_) {
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = 0.0f, scale[e] = n > 0 ? g.scale_b[j + min(e, n - 1)] : 0.0f;
    if (g.bias[0] && n > 0) load(static_cast<const char*>(g.bias[0]), j, bias);
  }

  __device__ void load(const char* p, int64_t at, float* v) const {
    switch (g.result) {
      case kDenseF32: load8<kDenseF32>(p + at * 4, n, v); break;
      case kDenseF16: load8<kDenseF16>(p + at * 2, n, v); break;
      default: load8<kDenseBF16>(p + at * 2, n, v); break;
    }
  }

  // What a row needs from memory, asked for before the rows before it are finished: the `which`-th from here on.
  struct Held {
    float row, lo[4], hi[4];   // (of a residual of 16 bits: lo)
  };

  __device__ Held ask(int which) const {
    Held h = ask_residual(which);
    h.row = g.scale_a[min(i + which * step, int64_t(g.ni) - 1)];
    return h;
  }

  __device__ Held ask_residual(int which = 0) const {
    Held h = {};
    const int64_t at = min(i + which * step, int64_t(g.ni) - 1);
    if (g.res && n == 8) {
      const char* const p = static_cast<const char*>(g.res) + (at * g.ldr + j) * (g.result == kDenseF32 ? 4 : 2);
      __builtin_memcpy(h.lo, p, 16);
      if (g.result == kDenseF32) __builtin_memcpy(h.hi, p + 16, 16);
    }
    return h;
  }

  __device__ void put(float* s, const Held& h, int which) const {
    const int64_t row = i + which * step;
    // (a sum, below 2^31, times a row's scale is no infinity on the way if that is below 2^96; if not, a sum times a column's scale
    // is none, or the result is one.  Asked of a wavefront's rows at once: one by one 2048 x 4096 x 256 took 15.9 us, so 15.6)
    const bool large = !(fabsf(h.row) < 0x1p96f);
    if (__any(large)) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float sum = static_cast<float>(__float_as_int(s[e]));
        s[e] = sum * (large ? scale[e] : h.row) * (large ? h.row : scale[e]) + bias[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] = static_cast<float>(__float_as_int(s[e])) * h.row * scale[e] + bias[e];
    }
    if (g.result == kDenseF32) act8<kDenseF32>(s, g.act);
    else act8<kDenseBF16>(s, g.act);
    if (g.res) {
      float b[8];
      if (n < 8) {
        load(static_cast<const char*>(g.res), row * g.ldr + j, b);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t pair = __float_as_uint(h.lo[e / 2]);
          b[e] = g.result == kDenseF32   ? (e < 4 ? h.lo[e % 4] : h.hi[e % 4])
                 : g.result == kDenseF16 ? static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(e % 2 ? pair >> 16 : pair)))
                                         : __uint_as_float(e % 2 ? pair & 0xffff0000u : pair << 16);
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s[e] += b[e];
    }
    char* const y = static_cast<char*>(g.c[0]);
    const int64_t at = row * g.ldc[0] + j;
    switch (g.result) {
      case kDenseF32: store8<kDenseF32>(y + at * 4, n, s); break;
      case kDenseF16: store8<kDenseF16>(y + at * 2, n, s); break;
      default: store8<kDenseBF16>(y + at * 2, n, s); break;
    }
  }

  __device__ void put(float* s, float*) const { put(s, ask(0), 0); }
};

// Stores a wavefront's sums, from row i0 and column j0 on, through LDS of its own: 64 rows of FJ * 16 sums at a time, so
// that a lane has eight consecutive columns and the activation's code is there once.  Lane (q, c) holds row c and
// columns 4 q .. + 3 of each fragment.  The 16-byte chunks of a row in LDS are permuted by the row.
template <int FJ>
constexpr int kSumsLds = 64 * FJ * 64;   // (half of it with two fragments of rows)

// Of 8-bit integers: what a lane's first four rows need from memory, which can be asked for before the sums are there.  (One
// row after another, each waits for memory; and four after four, asked for while those before are finished: 16384 x 8192 x 512
// with a bf16 residual 245 us, so 224, without one 164 and 154.)
template <int TYPE, int KIND, int FJ>
struct Asked {};
template <int FJ>
struct Asked<kDenseI8, kForward, FJ> {
  static constexpr int kTogether = 4, kLanes = FJ * 2, kRows = 64 / kLanes;
  using F = Finish<kDenseI8, kForward>;
  F out;
  typename F::Held held[kTogether];

  // of a wavefront's sums from row i0 and column j0 on
  __device__ Asked(const DenseGemm& g, int lane, int64_t i0, int j0)
      : out(g, 0, i0 + lane / kLanes, min(j0 + lane % kLanes * 8, g.nj - 1), kRows) {
    ask();
  }

  __device__ void ask(int first = 0) {
#pragma unroll
    for (int x = 0; x < kTogether; ++x) held[x] = out.ask(first + x);
  }
};

template <int TYPE, int KIND, int FI, int FJ>
__device__ inline void store_sums(const DenseGemm& g, Sums<TYPE> (&acc)[FI][FJ], char* own, int lane, int64_t i0, int j0, int part,
                                  int split, const Asked<TYPE, KIND, FJ>* asked = nullptr) {
  constexpr bool kGate = KIND == kGated;
  constexpr int kRowBytes = FJ * 64, kMask = FJ * 4 - 1, kUp = FJ * 2;   // kUp: first chunk of the up projection
  constexpr int kPass = FI < 4 ? FI : 4;   // fragments of rows at a time
  const int q = lane >> 4, c = lane & 15;
  constexpr bool kAsk = TYPE == kDenseI8 && FI > 2;   // (of two fragments of rows the caller has asked for all)
  auto four = [&] {                                   // (while the sums pass through LDS)
    if constexpr (kAsk) return Asked<TYPE, KIND, FJ>(g, lane, i0, j0);
    else return 0;
  }();
#pragma unroll
  for (int h = 0; h < FI / kPass; ++h) {
#pragma unroll
    for (int fi = 0; fi < kPass; ++fi)
#pragma unroll
      for (int fj = 0; fj < FJ; ++fj)
        *reinterpret_cast<Sums<TYPE>*>(own + (fi * 16 + c) * kRowBytes + (((fj * 4 + q) ^ (c & kMask)) << 4)) = acc[h * kPass + fi][fj];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    constexpr int kLanes = kGate ? FJ : FJ * 2, kRows = 64 / kLanes;   // lanes of a row, rows at a time
    const int e = lane % kLanes * 2, j = j0 + e * 4;                   // the row's first chunk of this lane
    const int64_t first = i0 + h * 64 + lane / kLanes;
    auto sums = [&](int row, float* s0, float* s1) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(own + row * kRowBytes + (((e + x) ^ (row & kMask)) << 4));
        s0[4 * x] = v[0], s0[4 * x + 1] = v[1], s0[4 * x + 2] = v[2], s0[4 * x + 3] = v[3];
        if constexpr (kGate) {
          const f32x4 w = *reinterpret_cast<const f32x4*>(own + row * kRowBytes + (((kUp + e + x) ^ (row & kMask)) << 4));
          s1[4 * x] = w[0], s1[4 * x + 1] = w[1], s1[4 * x + 2] = w[2], s1[4 * x + 3] = w[3];
        }
      }
    };
    if (j < g.nj) {
      float s0[8], s1[8];
      if (g.slots > 1) {
        // partial sums: rows padded to whole eights
        const int64_t ld = (g.nj + 7) / 8 * 8, slice = int64_t(g.ni) * ld;
        float* p = g.partial + (int64_t(kGate ? 0 : part) * g.slots + g.first + split) * slice + first * ld + j;
#pragma unroll 1
        for (int row0 = 0; row0 < kPass * 16; row0 += kRows, p += kRows * ld) {
          if (first + row0 >= g.ni) break;
          sums(row0 + lane / kLanes, s0, s1);
          reinterpret_cast<f32x4*>(p)[0] = f32x4{s0[0], s0[1], s0[2], s0[3]};
          reinterpret_cast<f32x4*>(p)[1] = f32x4{s0[4], s0[5], s0[6], s0[7]};
          if constexpr (kGate) {
            float* u = p + g.slots * slice;
            reinterpret_cast<f32x4*>(u)[0] = f32x4{s1[0], s1[1], s1[2], s1[3]};
            reinterpret_cast<f32x4*>(u)[1] = f32x4{s1[4], s1[5], s1[6], s1[7]};
          }
        }
      } else if constexpr (TYPE == kDenseI8) {
        using A = Asked<TYPE, KIND, FJ>;
        static_assert(kPass * 16 % (A::kTogether * kRows) == 0 && A::kRows == kRows);
        auto put = [&](const typename A::F& out, const typename A::F::Held* held, int row0) {
#pragma unroll
          for (int x = 0; x < A::kTogether; ++x) {
            if (first + row0 + x * kRows >= g.ni) break;
            sums(row0 + x * kRows + lane / kLanes, s0, s1);
            out.put(s0, held[x], x);
          }
        };
        if constexpr (!kAsk) {
          static_assert(kPass * 16 == A::kTogether * kRows);
          if (first < g.ni) put(asked->out, asked->held, 0);
        } else {
#pragma unroll 1
          for (int row0 = 0; row0 < kPass * 16; row0 += A::kTogether * kRows) {
            if (first + row0 >= g.ni) break;
            typename A::F::Held now[A::kTogether];
#pragma unroll
            for (int x = 0; x < A::kTogether; ++x) now[x] = four.held[x];
            if (h + 1 < FI / kPass || row0 + A::kTogether * kRows < kPass * 16) four.ask(A::kTogether);   // the next four
            put(four.out, now, row0);
            four.out.i += A::kTogether * kRows;
          }
        }
      } else {
        Finish<TYPE, KIND> out(g, part, first, j, kRows);
#pragma unroll 1
        for (int row0 = 0; row0 < kPass * 16; row0 += kRows, out.next()) {
          if (first + row0 >= g.ni) break;
          sums(row0 + lane / kLanes, s0, s1);
          out.put(s0, s1);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
}

// A tile of BM x BN with f32 products: right for every value, and slow.  In line, as a call that is hardly ever made gives
// the kernel a stack, and that alone cost 5 to 8 us a launch (f32 4096 x 512 x 1664 50.4 us, so 44.7).
template <int KIND, int BM, int BN, int WJ, int WAVES, int FI, int FJ>
__device__ __forceinline__ void tile_by_f32(const DenseGemm& g, char* lds, int i0, int j0, int wi, int wj, int begin, int end,
                                         int per_part, int wpart, int split) {
  constexpr bool kGate = KIND == kGated, kRm = KIND == kInputGrad || KIND == kWeightGrad;
  constexpr int BK = 32, kRow = BK + 1, kCols = kGate ? BN / 2 : BN, kThreads = 64 * WAVES;
  f32x4 acc[FI][FJ] = {};
  float* sa = reinterpret_cast<float*>(lds);
  float* sb = sa + BM * kRow;
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  for (int step = begin; step < end; ++step) {
    const int part = KIND == kInputGrad && step >= per_part ? 1 : 0;
    const int r0 = (step - part * per_part) * BK;
    const float* a = static_cast<const float*>(g.a[KIND == kWeightGrad ? wpart : part]) +
                     (KIND == kWeightGrad ? r0 * g.lda + column_at(i0, g.panel_a) : i0 * g.lda + r0);
    __syncthreads();
    for (int e = tid; e < BM * BK; e += kThreads) {
      const int i = KIND == kWeightGrad ? e % BM : e / BK, r = KIND == kWeightGrad ? e / BM : e % BK;
      const int64_t at = KIND == kWeightGrad ? r * g.lda + i : i * g.lda + r;
      sa[i * kRow + r] = r0 + r < g.nr && i0 + i < g.ni ? a[at] : 0.0f;
    }
    for (int e = tid; e < BN * BK; e += kThreads) {
      const int row = kRm ? e % BN : e / BK, r = kRm ? e / BN : e % BK;
      const int mat = kGate ? row / kCols : part, j = kGate ? row % kCols : row;
      const float* b = static_cast<const float*>(g.b[mat]) +
                       (kRm ? r0 * g.ldb[mat] + column_at(j0, g.panel_b[mat]) : j0 * g.ldb[mat] + r0);
      const int64_t at = kRm ? r * g.ldb[mat] + j : j * g.ldb[mat] + r;
      sb[row * kRow + r] = r0 + r < g.nr && j0 + j < g.nj ? b[at] : 0.0f;
    }
    __syncthreads();
    for (int s = 0; s < BK; s += 4) {
#pragma unroll
      for (int fi = 0; fi < FI; ++fi)
#pragma unroll
        for (int fj = 0; fj < FJ; ++fj) {
          const int row = kGate ? (fj / (FJ / 2)) * kCols + wj + (fj % (FJ / 2)) * 16 + c : wj + fj * 16 + c;
          acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x4f32(sb[row * kRow + s + q], sa[(wi + fi * 16 + c) * kRow + s + q],
                                                             acc[fi][fj], 0, 0, 0);
        }
    }
  }
  __syncthreads();
  store_sums<kDenseF32, KIND, FI, FJ>(g, acc, lds + (tid >> 6) * kSumsLds<FJ>, lane, int64_t(i0) + wi, j0 + wj, wpart, split);
}

// bytes of LDS of a tile: the steps under way, or what the epilogue takes
template <int TYPE, int BM, int BN, int WJ, int WAVES>
constexpr int kTileLds = [] {   // (of each half)
  const int steps = TYPE == kDenseF32 ? (BM + BN) * 64 * 3 * 2     // three bf16 parts of two steps
                                      : ((WAVES == 8 ? 3 : 2) * BM + 2 * BN) * 128;
  const int sums = WAVES * kSumsLds<BN / WJ / 16>;
  return steps > sums ? steps : sums;
}();

// One tile of a product: `tile` of its tiles, `split` of its splits, `wpart` of kWeightGrad's two results.  Three main
// loops:
//   16 bits, 128 x 128, four wavefronts of 64 x 64, two workgroups a CU: for products that do not fill the GPU with larger
//     ones; a tile's operands pass through L2 twice as often as those of 256 x 256 (bf16 8192^3: 1004 us, 1.1 PFLOP/s)
//     where there is no second tile for a CU (HALVES = 2), eight wavefronts of one workgroup: each four take half of the
//     steps, as two workgroups would, and then half of the rows of the sum (bf16 4096 x 1024 x 1024 14.2 us a call, with
//     four wavefronts 16.9)
//   16 bits, 256 x 256, eight wavefronts of 128 x 64 in turns, one workgroup a CU (its 160 KB of LDS, and 128 + 96 of the
//     registers): bf16 8192^3 765 us, 1.44 PFLOP/s, where one library product reaches 1.42 to 1.61; 65536 x 1024 x 12800
//     1255 us, 1.37.  Bound by the matrix cores at the clock that they leave (about 1.75 GHz), less some 7 us a tile for its
//     first loads and its results, which nothing hides (one workgroup a CU that goes on to the next tile was slower: its
//     loads wait for the stores before them)
//   f32, 256 x 128 or 128 x 128, eight wavefronts, one workgroup a CU: see PartTile; 4096^3 595 us, 231 TFLOP/s (f32
//     products on the matrix cores reach 153 in a library)
template <int TYPE, int KIND, int BM, int BN, int WI, int WJ, int HALVES>
__device__ __forceinline__ void tile_product(const DenseGemm& g, char* all, uint32_t tile, int split, int wpart) {
  constexpr bool kGate = KIND == kGated;
  constexpr bool kRmA = KIND == kWeightGrad, kRmB = KIND == kWeightGrad || KIND == kInputGrad;
  constexpr int kWaves = WI * WJ;
  constexpr bool kF32 = TYPE == kDenseF32;
  constexpr bool kTurns = kWaves == 8 && !kF32;                   // see the main loop
  constexpr int kSlotsA = kF32 ? 1 : kTurns ? 3 : 2, kSlotsB = kF32 ? 1 : 2;   // tiles of steps in LDS
  constexpr int kCols = kGate ? BN / 2 : BN;               // result columns of a tile
  constexpr int kWI = BM / WI, kWJ = kCols / WJ;           // results of a wavefront
  constexpr int kFI = kWI / 16, kFJ = BN / WJ / 16;        // its fragments
  constexpr int kSize = TYPE == kDenseI8 ? 1 : 2;          // of elements that go to LDS as they are
  using TileA = Tile<BM, kRmA, kWaves, kSize>;             // (not f32)
  using TileB = Tile<BN, kRmB, kWaves, kSize>;
  using TileH = Tile<kCols, kRmB, kWaves, kSize>;          // one projection's half of B
  constexpr int BK = kF32 ? 32 : TileA::BK;
  static_assert(kF32 || kSlotsA * TileA::kBytes + kSlotsB * TileB::kBytes <= kTileLds<TYPE, BM, BN, WJ, kWaves>);

  static_assert(HALVES == 1 || (!kF32 && !kTurns && kFI == 4));
  const int half = HALVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * kWaves));
  char* const lds = all + half * kTileLds<TYPE, BM, BN, WJ, kWaves>;
  const int tid = threadIdx.x - half * 64 * kWaves, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int ti, tj;
  tile_of(tile, (g.ni + BM - 1) / BM, (g.nj + kCols - 1) / kCols, &ti, &tj);
  const int i0 = ti * BM, j0 = tj * kCols;
  const int per_part = (g.nr + BK - 1) / BK;
  const int steps = per_part * (KIND == kInputGrad ? g.parts : 1);
  int begin = static_cast<int>(int64_t(steps) * split / g.splits);
  int end = static_cast<int>(int64_t(steps) * (split + 1) / g.splits);
  const int trips = (end - begin + HALVES - 1) / HALVES;   // of both halves alike: a step past the end is zeros
  if constexpr (HALVES == 2) {
    if (half == 0) end = min(end, begin + trips);
    else begin = min(end, begin + trips);
  }

  TileA ta;
  ta.init(wave, lane, g.lda, g.ni - i0);
  // kGated: two halves with the rows of each projection; kInputGrad: strides may differ by part
  TileB tb;
  TileH th[2];
  if constexpr (kGate) {
    th[0].init(wave, lane, g.ldb[0], g.nj - j0);
    th[1].init(wave, lane, g.ldb[1], g.nj - j0);
  } else {
    tb.init(wave, lane, g.ldb[0], g.nj - j0);
  }
  int tb_part = 0;

  const uint32_t lds0 = lds_address(lds);
  constexpr int kIssues = TileA::kLoads + TileB::kLoads;
  // LDS: kSlotsA tiles of A, then kSlotsB tiles of B.  set_a, set_b: the step that issue_a, issue_b load
  // next and where to; steps past the last are loaded too, as zeros, so that the count of loads under
  // way is always the same.
  constexpr int kAreaB = kSlotsA * TileA::kBytes;
  struct Next { i32x4 a, b0, b1; int valid_a, valid_b; uint32_t at_a, at_b; } next;
  auto set_a = [&](int step, int slot) {
    const int part = KIND == kInputGrad && step >= per_part && g.parts > 1 ? 1 : 0;
    const int r0 = (step - part * per_part) * BK;
    next.valid_a = step < end ? g.nr - r0 : 0;
    const char* a = static_cast<const char*>(g.a[KIND == kWeightGrad ? wpart : part]);
    next.a = descriptor(a + (kRmA ? int64_t(r0) * g.lda + column_at(i0, g.panel_a) : int64_t(i0) * g.lda + r0) * kSize);
    next.at_a = lds0 + slot * TileA::kBytes;
  };
  auto set_b = [&](int step, int slot) {
    const int part = KIND == kInputGrad && step >= per_part && g.parts > 1 ? 1 : 0;
    const int r0 = (step - part * per_part) * BK;
    next.valid_b = step < end ? g.nr - r0 : 0;
    const char* b = static_cast<const char*>(g.b[part]);
    const int64_t at = kRmB ? int64_t(r0) * g.ldb[part] + column_at(j0, g.panel_b[part]) : int64_t(j0) * g.ldb[part] + r0;
    next.b0 = descriptor(b + at * kSize);
    if constexpr (kGate) next.b1 = descriptor(static_cast<const char*>(g.b[1]) + (int64_t(j0) * g.ldb[1] + r0) * kSize);
    if constexpr (KIND == kInputGrad) {
      if (part != tb_part) {
        tb.init(wave, lane, g.ldb[part], g.nj - j0);
        tb_part = part;
      }
    }
    next.at_b = lds0 + kAreaB + slot * TileB::kBytes;
  };
  auto issue_a = [&](int n) { ta.load(next.a, next.at_a, wave, lane, next.valid_a, n); };
  auto issue_b = [&](int n) {
    if constexpr (kGate) {
      if (n < TileH::kLoads) th[0].load(next.b0, next.at_b, wave, lane, next.valid_b, n);
      else th[1].load(next.b1, next.at_b + TileH::kBytes, wave, lane, next.valid_b, n - TileH::kLoads);
    } else {
      tb.load(next.b0, next.at_b, wave, lane, next.valid_b, n);
    }
  };
  auto issue = [&](int n) {   // B first: stage_done<kLoads of A> leaves A's under way
    if (n < TileB::kLoads) issue_b(n);
    else issue_a(n - TileB::kLoads);
  };

  const int wi = (wave / WJ) * kWI, wj = (wave % WJ) * kWJ;
  // (asked for here, as a CU's one workgroup has nothing else to hide it: 4096 x 1024 x 1024 with a residual)
  const auto asked = [&] {
    if constexpr (TYPE == kDenseI8 && HALVES == 2) return Asked<TYPE, KIND, kFJ>(g, lane, int64_t(i0) + wi + half * 32, j0 + wj);
    else return 0;
  }();
  Sums<TYPE> acc[kFI][kFJ] = {};
  // fragments of a half step (not f32)
  auto fragments_a = [&](const char* sa, int ks, s16x8* f) {
#pragma unroll
    for (int n = 0; n < kFI; ++n) f[n] = TileA::fragment(sa, wi + n * 16, ks, lane);
  };
  auto fragments_b = [&](const char* sb, int ks, s16x8* f) {
#pragma unroll
    for (int n = 0; n < kFJ; ++n) {
      if constexpr (kGate)
        f[n] = TileH::fragment(sb + (n >= kFJ / 2) * TileH::kBytes, wj + (n % (kFJ / 2)) * 16, ks, lane);
      else
        f[n] = TileB::fragment(sb, wj + n * 16, ks, lane);
    }
  };
  int at_a = 0, at_b = 0;   // slots of the step that is multiplied
  if constexpr (kF32) {
    // The parts of two steps lie in LDS: while one is multiplied, the next, whose values are in registers, is taken apart,
    // and the one after it is loaded.
    using PartA = PartTile<BM, kRmA, kWaves>;
    using PartB = PartTile<kGate ? kCols : BN, kRmB, kWaves>;
    constexpr int kMats = kGate ? 2 : 1, kPlane = PartA::kBytes + kMats * PartB::kBytes;
    PartA va;
    PartB vb[kMats];
    va.init(tid, g.lda, g.ni - i0);
#pragma unroll
    for (int m = 0; m < kMats; ++m) vb[m].init(tid, g.ldb[m], g.nj - j0);
    auto fetch = [&](int step) {
      const int part = KIND == kInputGrad && step >= per_part && g.parts > 1 ? 1 : 0;
      const int r0 = (step - part * per_part) * BK, valid = step < end ? g.nr - r0 : 0;
      const float* a = static_cast<const float*>(g.a[KIND == kWeightGrad ? wpart : part]);
      va.load(descriptor(a + (kRmA ? int64_t(r0) * g.lda + column_at(i0, g.panel_a) : int64_t(i0) * g.lda + r0)), tid, valid);
      if constexpr (KIND == kInputGrad) {
        if (part != tb_part) {
          vb[0].init(tid, g.ldb[part], g.nj - j0);
          tb_part = part;
        }
      }
#pragma unroll
      for (int m = 0; m < kMats; ++m) {
        const int mat = kGate ? m : part;
        const float* b = static_cast<const float*>(g.b[mat]);
        const int64_t at = kRmB ? int64_t(r0) * g.ldb[mat] + column_at(j0, g.panel_b[mat]) : int64_t(j0) * g.ldb[mat] + r0;
        vb[m].load(descriptor(b + at), tid, valid);
      }
    };
    auto take_apart = [&](int slot) {
      char* to = lds + slot * 3 * kPlane;
      va.take_apart(to, kPlane, tid);
#pragma unroll
      for (int m = 0; m < kMats; ++m) vb[m].take_apart(to + PartA::kBytes + m * PartB::kBytes, kPlane, tid);
    };
    fetch(begin);
    take_apart(0);
    fetch(begin + 1);
    int slot = 0;
    for (int step = begin; step < end; ++step) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // (loads stay under way)
      const char* parts = lds + slot * 3 * kPlane;
      slot ^= 1;
      Parts fa[kFI], fb[kFJ];
#pragma unroll
      for (int p = 2; p >= 0; --p) {
        const char* pa = parts + p * kPlane;
        const char* pb = pa + PartA::kBytes;
#pragma unroll
        for (int n = 0; n < kFI; ++n) fa[n].p[p] = PartA::fragment(pa, wi + n * 16, lane);
#pragma unroll
        for (int n = 0; n < kFJ; ++n) {
          if constexpr (kGate) fb[n].p[p] = PartB::fragment(pb + (n >= kFJ / 2) * PartB::kBytes, wj + (n % (kFJ / 2)) * 16, lane);
          else fb[n].p[p] = PartB::fragment(pb, wj + n * 16, lane);
        }
      }
      take_apart(slot);
      fetch(step + 2);
      products6<kFI, kFJ>(fa, fb, acc);
    }
  } else if constexpr (!kTurns) {
    // One step is on its way while another is multiplied.  Two workgroups share a CU, so that one reads while the other
    // multiplies.
    set_a(begin, 0);
    set_b(begin, 0);
#pragma unroll
    for (int n = 0; n < kIssues; ++n) issue(n);
    for (int step = begin, left = trips; left > 0; ++step, --left) {
      stage_done<0>();
      const char* sa = lds + at_a * TileA::kBytes;
      const char* sb = lds + kAreaB + at_a * TileB::kBytes;
      at_a ^= 1;
      set_a(step + 1, at_a);
      set_b(step + 1, at_a);
#pragma unroll
      for (int n = 0; n < kIssues; ++n) issue(n);
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        s16x8 fa[kFI], fb[kFJ];
        fragments_b(sb, ks, fb);
        fragments_a(sa, ks, fa);
#pragma unroll
        for (int fi = 0; fi < kFI; ++fi)
#pragma unroll
          for (int fj = 0; fj < kFJ; ++fj) acc[fi][fj] = mfma16<TYPE>(fb[fj], fa[fi], acc[fi][fj]);
      }
    }
  } else {
    // The two wavefronts of a SIMD take turns: while one multiplies a step, the other reads its fragments of a
    // step into registers (wavefronts 0-3 are one to a SIMD, and so are 4-7, which run a turn behind).  B has two
    // slots, A three: a step of A, whose rows come from memory, is asked for four turns before it is read, one of
    // B, which other tiles share in L2, two.  A slot is loaded again after the turn in which the late wavefronts
    // have read it.
    constexpr int kUnderWay = TileA::kLoads;
    const bool late = wave >= 4;
    auto after = [](int slot) { return slot == 2 ? 0 : slot + 1; };
    set_a(begin, 0);
    set_b(begin, 0);
#pragma unroll
    for (int n = 0; n < kIssues; ++n) issue(n);
    set_a(begin + 1, 1);
#pragma unroll
    for (int n = 0; n < TileA::kLoads; ++n) issue_a(n);
    stage_done<kUnderWay>();
    s16x8 fa[2][kFI], fb[2][kFJ];
    auto read = [&]() {
      const char* sa = lds + at_a * TileA::kBytes;
      const char* sb = lds + kAreaB + at_b * TileB::kBytes;
#pragma unroll
      for (int ks = 0; ks < 2; ++ks) {
        fragments_b(sb, ks, fb[ks]);
        fragments_a(sa, ks, fa[ks]);
      }
    };
    auto multiply = [&](int ks, int fi) {
#pragma unroll
      for (int fj = 0; fj < kFJ; ++fj) acc[fi][fj] = mfma16<TYPE>(fb[ks][fj], fa[ks][fi], acc[fi][fj]);
    };
    if (!late) {
      for (int step = begin; step < end; ++step) {
        read();
        set_b(step + 1, at_b ^ 1);
        set_a(step + 2, after(after(at_a)));
        at_b ^= 1;
        at_a = after(at_a);
#pragma unroll
        for (int n = 0; n < kIssues; ++n) issue(n);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int fi = 0; fi < kFI; ++fi) multiply(ks, fi);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        stage_done<kUnderWay>();
      }
      asm volatile("s_barrier" ::: "memory");
    } else {
      set_b(begin + 1, 1);
      set_a(begin + 2, 2);
#pragma unroll
      for (int n = 0; n < kIssues; ++n) issue(n);
      asm volatile("s_barrier" ::: "memory");
      for (int step = begin; step < end; ++step) {
        read();
        set_b(step + 2, at_b);
        set_a(step + 3, at_a);
        at_b ^= 1;
        at_a = after(at_a);
        __builtin_amdgcn_sched_barrier(0);
        stage_done<kUnderWay>();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
          for (int fi = 0; fi < kFI; ++fi) {
            multiply(ks, fi);
            if (ks * kFI + fi < kIssues) issue(ks * kFI + fi);
            __builtin_amdgcn_sched_barrier(0);
          }
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
      }
    }
  }

  stage_done<0>();
  if constexpr (kF32) {
    uint32_t largest = 0;
#pragma unroll
    for (int fi = 0; fi < kFI; ++fi)
#pragma unroll
      for (int fj = 0; fj < kFJ; ++fj)
#pragma unroll
        for (int e = 0; e < 4; ++e) largest = max(largest, __float_as_uint(acc[fi][fj][e]) << 1);
    int* redo = reinterpret_cast<int*>(lds);
    if (tid == 0) *redo = 0;
    __syncthreads();
    if (largest >= 0xff000000u) *redo = 1;   // an infinity or NaN
    __syncthreads();
    const int again = __builtin_amdgcn_readfirstlane(*redo);
    __syncthreads();
    if (again) {
      tile_by_f32<KIND, BM, BN, WJ, kWaves, kFI, kFJ>(g, lds, i0, j0, wi, wj, begin, end, per_part, wpart, split);
      return;
    }
  }
  if constexpr (kF32) {
#pragma unroll
    for (int fi = 0; fi < kFI; ++fi)
#pragma unroll
      for (int fj = 0; fj < kFJ; ++fj) acc[fi][fj] *= 1.0f / (kScale * kScale);
  }
  if constexpr (HALVES == 2) {
    // the first half gives its lower rows away, the second its upper ones
    char* const pass = all + wave * 2 * kFJ * 1024 + lane * 16;
    constexpr int kGiven = kWaves * 2 * kFJ * 1024;   // bytes that a half gives
    auto give = [&](int from) {
#pragma unroll
      for (int fi = 0; fi < 2; ++fi)
#pragma unroll
        for (int fj = 0; fj < kFJ; ++fj)
          *reinterpret_cast<Sums<TYPE>*>(pass + half * kGiven + (fi * kFJ + fj) * 1024) = acc[from + fi][fj];
    };
    if (half == 0) give(2);
    else give(0);
    __syncthreads();
    Sums<TYPE> sum[2][kFJ];
    auto take = [&](int at) {
#pragma unroll
      for (int fi = 0; fi < 2; ++fi)
#pragma unroll
        for (int fj = 0; fj < kFJ; ++fj)
          sum[fi][fj] = acc[at + fi][fj] + *reinterpret_cast<const Sums<TYPE>*>(pass + (half ^ 1) * kGiven + (fi * kFJ + fj) * 1024);
    };
    if (half == 0) take(0);
    else take(2);
    char* const own = all + 2 * kGiven + (half * kWaves + wave) * (kSumsLds<kFJ> / 2);
    static_assert(2 * kGiven + kWaves * kSumsLds<kFJ> <= HALVES * kTileLds<TYPE, BM, BN, WJ, kWaves>);
    if constexpr (TYPE == kDenseI8)
      store_sums<TYPE, KIND, 2, kFJ>(g, sum, own, lane, int64_t(i0) + wi + half * 32, j0 + wj, wpart, split, &asked);
    else
      store_sums<TYPE, KIND, 2, kFJ>(g, sum, own, lane, int64_t(i0) + wi + half * 32, j0 + wj, wpart, split);
  } else {
    store_sums<TYPE, KIND, kFI, kFJ>(g, acc, lds + wave * kSumsLds<kFJ>, lane, int64_t(i0) + wi, j0 + wj, wpart, split);
  }
}

template <int TYPE, int KIND, int BM, int BN, int WI, int WJ, int PER_CU, int HALVES>
__global__ __launch_bounds__(64 * WI * WJ * HALVES, WI * WJ * HALVES * PER_CU / 4) void dense_tile(DenseGemm g) {
  __shared__ __align__(1024) char lds[HALVES * kTileLds<TYPE, BM, BN, WJ, WI * WJ>];
  tile_product<TYPE, KIND, BM, BN, WI, WJ, HALVES>(g, lds, blockIdx.x, blockIdx.y, 0);
}

// Both products of a backward pass in one launch: the weights' gradient first, whose tiles are few and long, then the
// input's, whose many short ones fill the CUs that are left (either may be absent).  With this
// launch and the last one instead of a launch for each, a call took 250 us instead of 265 (f16 16384 x 1024 x 3328), 272
// instead of 315 (gated, bf16 8192 x 4096 x 1024) and 43 instead of 55 (gated, f16 777 x 1365 x 1001).
template <int TYPE, int BM, int BN, int WI, int WJ, int PER_CU, int HALVES>
__global__ __launch_bounds__(64 * WI * WJ * HALVES, WI * WJ * HALVES * PER_CU / 4) void dense_grads(DenseGemm w, DenseGemm x,
                                                                                                  uint32_t w_groups) {
  __shared__ __align__(1024) char lds[HALVES * kTileLds<TYPE, BM, BN, WJ, WI * WJ>];
  uint32_t id = blockIdx.x;
  if (id < w_groups) {
    const uint32_t tiles = (w.ni + BM - 1) / BM * ((w.nj + BN - 1) / BN), rest = id / tiles;
    if (rest >= uint32_t(w.splits * w.parts)) return;   // (w_groups is a multiple of the XCDs)
    tile_product<TYPE, kWeightGrad, BM, BN, WI, WJ, HALVES>(w, lds, id % tiles, rest % w.splits, rest / w.splits);
  } else {
    id -= w_groups;
    const uint32_t tiles = (x.ni + BM - 1) / BM * ((x.nj + BN - 1) / BN);
    tile_product<TYPE, kInputGrad, BM, BN, WI, WJ, HALVES>(x, lds, id % tiles, id / tiles, 0);
  }
}

// of sums as they are held (8-bit integers': whole numbers' bits)
template <int TYPE>
__device__ inline float plus(float a, float b) {
  return TYPE == kDenseI8 ? __int_as_float(__float_as_int(a) + __float_as_int(b)) : a + b;
}

// Eight columns of a result whose reduction was split: the splits' sums are added in order.
template <int TYPE, int KIND>
__device__ inline void join8(const DenseGemm& g, int64_t at, int part) {
  const int groups = (g.nj + 7) / 8;
  if (at >= int64_t(groups) * g.ni) return;
  const int64_t i = at / groups, slice = int64_t(g.ni) * groups * 8;
  const int j = static_cast<int>(at % groups) * 8;
  float s[2][8];
#pragma unroll
  for (int mat = 0; mat < (KIND == kGated ? 2 : 1); ++mat) {
    const float* p = g.partial + int64_t(KIND == kGated ? mat : part) * g.slots * slice + at * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[mat][e] = 0.0f;
    int split = 0;
    auto add = [&](auto count) {   // that many splits' loads at a time
      constexpr int N = decltype(count)::value;
      f32x4 lo[N], hi[N];
#pragma unroll
      for (int n = 0; n < N; ++n, p += slice) {
        lo[n] = reinterpret_cast<const f32x4*>(p)[0];
        hi[n] = reinterpret_cast<const f32x4*>(p)[1];
      }
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[mat][e] = plus<TYPE>(s[mat][e], lo[n][e]);
          s[mat][4 + e] = plus<TYPE>(s[mat][4 + e], hi[n][e]);
        }
      split += N;
    };
    while (g.slots - split >= 8) add(std::integral_constant<int, 8>{});
    if (g.slots - split >= 4) add(std::integral_constant<int, 4>{});
    if (g.slots - split >= 2) add(std::integral_constant<int, 2>{});
    if (g.slots - split >= 1) add(std::integral_constant<int, 1>{});
  }
  Finish<TYPE, KIND>(g, part, i, j, 0).put(s[0], s[1]);
}

template <int TYPE, int KIND>
__global__ __launch_bounds__(256) void dense_join(DenseGemm g) {
  join8<TYPE, KIND>(g, int64_t(blockIdx.x) * 256 + threadIdx.x, 0);
}

// The last launch of a backward pass, as far as there is something left: the column sums from those of the blocks of
// rows (32 columns a workgroup, eight threads a column), then the joins of both products.  No two of them depend on
// each other.
template <int TYPE>
__global__ __launch_bounds__(256) void dense_tail(DenseGemm w, DenseGemm x, DenseColsum c, DenseTail t) {
  using T = typename Elem<TYPE>::T;
  uint32_t id = blockIdx.x;
  if (id < t.colsum_groups) {
    __shared__ float sums[8][32];
    const uint32_t per = (c.n + 31) / 32;
    const int mat = id / per, column = threadIdx.x & 31, y = threadIdx.x >> 5, j = id % per * 32 + column;
    const float* p = c.partial[mat];
    if (!p) return;
    float sum = 0.0f;
    if (j < c.n) {
      for (int first = y; first < c.blocks; first += 16 * 8) {
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = p[int64_t(min(first + e * 8, c.blocks - 1)) * c.n + j];
#pragma unroll
        for (int e = 0; e < 16; ++e) sum += first + e * 8 < c.blocks ? v[e] : 0.0f;
      }
    }
    sums[y][column] = sum;
    __syncthreads();
    if (y == 0 && j < c.n) {
#pragma unroll
      for (int r = 1; r < 8; ++r) sum += sums[r][column];
      static_cast<T*>(c.out[mat])[j] = T(sum);
    }
    return;
  }
  id -= t.colsum_groups;
  if (id < t.w_groups * w.parts) {
    join8<TYPE, kWeightGrad>(w, int64_t(id % t.w_groups) * 256 + threadIdx.x, id / t.w_groups);
    return;
  }
  id -= t.w_groups * w.parts;
  join8<TYPE, kInputGrad>(x, int64_t(id) * 256 + threadIdx.x, 0);
}

// ---------------------------------------------------------------- few rows, or a short reduction
//
// Forward products that tiles suit badly, in one launch and without copies, at any alignment: where both operands' rows
// start at multiples of 16 bytes and hold whole chunks of 16 (WHOLE), a wavefront loads its fragments straight into
// registers, 16 rows of 64 bytes an instruction; else it loads consecutive elements and turns them in LDS.
template <int TYPE>
struct Loader {
  using T = typename Elem<TYPE>::T;
  float v[TYPE == kDenseF32 ? 8 : 1];   // f32 values
  s16x8 h;                              // or 16-bit ones

  __device__ void read(const T* p) {   // whole, aligned
    if constexpr (TYPE == kDenseF32) __builtin_memcpy(v, __builtin_assume_aligned(p, 16), 32);
    else h = *reinterpret_cast<const s16x8*>(p);
  }

  // elements at .. at + 7 of a row whose chunks of 16 bytes are whole; those from n on are zeros
  __device__ void load(const T* row, int at, int n) {
    if constexpr (TYPE == kDenseF32) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(row + min(at + 4 * h, n - 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] = at + 4 * h < n ? x[e] : 0.0f;
      }
    } else {
      h = *reinterpret_cast<const s16x8*>(row + min(at, n - 8));
      if (at >= n) h = s16x8{};
    }
  }
};

template <int TYPE>
__device__ inline f32x4 multiply(const Loader<TYPE>& w, const Loader<TYPE>& x, f32x4 c) {
  if constexpr (TYPE == kDenseF32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[e], x.v[e], c, 0, 0, 0);
    return c;
  } else {
    return mfma16<TYPE>(w.h, x.h, c);
  }
}

// Few rows, few columns, or few of both: the longer operand is read once, and latency counts.  Eight wavefronts share FR *
// 16 rows by 16 columns and take every eighth step of 32 each; their sums are added in order in LDS.  bf16, 1 x 512 x 1664:
// 4.3 us of GPU time, a launch and two rounds of loads; gated 19 x 2816 x 1024: 5.8 us for 11.7 MB; f16 65536 x 1 x 1024:
// 134 MB in 21 us, 6.3 TB/s.
template <int TYPE, int KIND, int FR, bool WHOLE>
__global__ __launch_bounds__(512) void dense_rows(DenseGemm g) {
  using T = typename Elem<TYPE>::T;
  using L = Loader<TYPE>;
  constexpr int kMats = KIND == kGated ? 2 : 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const uint32_t across = (g.nj + 15) / 16, down = (g.ni + FR * 16 - 1) / (FR * 16);
  uint32_t i = blockIdx.x / across, j_ = blockIdx.x % across;
  if (down >= kXcds) {   // rows of x stay with one XCD's L2
    j_ = blockIdx.x / kXcds % across, i = blockIdx.x / (kXcds * across) * kXcds + blockIdx.x % kXcds;
    if (i >= down) return;
  }
  const int i0 = i * FR * 16, j0 = j_ * 16;
  f32x4 acc[FR][kMats] = {};
  auto products = [&](const L* x, const L* w) {
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
      for (int m = 0; m < kMats; ++m) acc[f][m] = multiply<TYPE>(w[m], x[f], acc[f][m]);
  };
  if constexpr (WHOLE) {
    const T* rows[FR];
    const T* weights[kMats];
#pragma unroll
    for (int f = 0; f < FR; ++f) rows[f] = static_cast<const T*>(g.a[0]) + min(i0 + f * 16 + c, g.ni - 1) * g.lda;
#pragma unroll
    for (int m = 0; m < kMats; ++m) weights[m] = static_cast<const T*>(g.b[m]) + min(j0 + c, g.nj - 1) * g.ldb[m];
#pragma unroll 4
    for (int r0 = wave * 32; r0 < g.nr; r0 += 8 * 32) {
      L x[FR], w[kMats];
#pragma unroll
      for (int m = 0; m < kMats; ++m) w[m].load(weights[m], r0 + 8 * q, g.nr);
#pragma unroll
      for (int f = 0; f < FR; ++f) x[f].load(rows[f], r0 + 8 * q, g.nr);
      products(x, w);
    }
  } else {
    // A load reads consecutive elements, 32 of each of two rows, and LDS of the wavefront's own turns sixteen rows into a
    // fragment; the next step's loads are under way meanwhile.  (One load for each lane's own row and place takes 64
    // accesses of the cache: f16 32 x 512 x 1001 12.2 us a call, so 5.7.)  A wavefront's LDS instructions run in order, so
    // it waits for none of them.
    constexpr int kRow = 32 + 16 / int(sizeof(T));
    __shared__ __align__(16) T turned[8][2][16 * kRow];
    const int column = lane & 31, row = lane >> 5;
    T held[FR + kMats][8];
    auto ask = [&](T* h, const void* from, int64_t ld, int first, int count, int at) {
      const T* const p = static_cast<const T*>(from);
      if (ld < (1 << 24) && first + 16 <= count) {
        const uint32_t mine = static_cast<uint32_t>(row) * static_cast<uint32_t>(ld) + at;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = p[(first + e * 2) * ld + mine];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = p[min(first + e * 2 + row, count - 1) * ld + at];
      }
    };
    auto fetch = [&](int r0) {
      const int at = min(r0 + column, g.nr - 1);
#pragma unroll
      for (int m = 0; m < kMats; ++m) ask(held[FR + m], g.b[m], g.ldb[m], j0, g.nj, at);
#pragma unroll
      for (int f = 0; f < FR; ++f) ask(held[f], g.a[0], g.lda, i0 + f * 16, g.ni, at);
    };
    int r0 = wave * 32;
    if (r0 < g.nr) fetch(r0);
    for (; r0 < g.nr; r0 += 8 * 32) {
      L v[FR + kMats];
#pragma unroll
      for (int f = 0; f < FR + kMats; ++f) {
        T* const own = turned[wave][f & 1];
#pragma unroll
        for (int e = 0; e < 8; ++e) own[(e * 2 + row) * kRow + column] = r0 + column < g.nr ? held[f][e] : T(0.0f);
        v[f].read(own + c * kRow + 8 * q);
      }
      if (r0 + 8 * 32 < g.nr) fetch(r0 + 8 * 32);
      products(v, v + FR);
    }
  }
  __shared__ float sums[8][FR][kMats][16][16];   // [wavefront][..][..][row][column]
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int m = 0; m < kMats; ++m) *reinterpret_cast<f32x4*>(&sums[wave][f][m][c][4 * q]) = acc[f][m];
  __syncthreads();
  const int t = threadIdx.x, row = t >> 1, j = j0 + (t & 1) * 8;
  if (row >= FR * 16 || i0 + row >= g.ni || j >= g.nj) return;
  float s[2][8] = {};
#pragma unroll
  for (int w = 0; w < 8; ++w)
#pragma unroll
    for (int m = 0; m < kMats; ++m)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[m][e] += sums[w][row >> 4][m][row & 15][(t & 1) * 8 + e];
  Finish<TYPE, KIND>(g, 0, i0 + row, j, 0).put(s[0], s[1]);
}

// The same for 8-bit integers: of few rows, bound by reading the weights.  A wavefront takes 128 bytes of every eighth step of
// 1024, and asks for the weights of eight loads at a time, the next eight while it multiplies.  x is 8-bit rows in memory
// (XT kDenseI8), or a few rows of the result's type (g.m of 8 at most) that each workgroup quantizes by itself, while its
// weights are on their way, instead of a launch before this one.
constexpr int kQuantizedLds = 16640;   // up to 16384 elements

// Sixteen bytes of a row, at a multiple of ALIGN bytes: 16, 4 or 1.  At odd addresses, the words that they lie in, shifted when
// they are needed (16-byte loads there take twice as long: 4 x 2100 x 11991 25.7 us, so 18.3; at multiples of 4 13.4, so 18.5).
// Where rows do not start at multiples of 16, `left` bytes can be read from p on, at least one: to the end of the matrix.  No
// word without one of them is read.
template <int ALIGN>
struct Eights {
  i32x4 v;
  int more[ALIGN == 1 ? 1 : 0];

  __device__ static Eights load(const int8_t* p, int64_t left) {
    Eights e;
    if constexpr (ALIGN == 16) {
      e.v = *reinterpret_cast<const i32x4*>(p);
    } else {
      const uintptr_t shift = ALIGN == 1 ? reinterpret_cast<uintptr_t>(p) & 3 : 0;
      const int8_t* const a = p - shift;
      const int64_t last = left >= 16 ? 16 : (shift + left - 1) / 4 * 4;
      if (left >= 16) {
        __builtin_memcpy(&e.v, __builtin_assume_aligned(a, 4), 16);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) e.v[i] = *reinterpret_cast<const int*>(a + min(int64_t(4 * i), last));
      }
      if constexpr (ALIGN == 1) e.more[0] = *reinterpret_cast<const int*>(a + (shift ? min(int64_t(16), last) : 0));
    }
    return e;
  }

  // row: any address as far from a multiple of 4 as p was
  __device__ s16x8 get(const int8_t* row) const {
    i32x4 out = v;
    if constexpr (ALIGN == 1) {
      const uint32_t shift = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row)) & 3;
#pragma unroll
      for (int i = 0; i < 4; ++i) out[i] = __builtin_amdgcn_alignbyte(i < 3 ? v[i + 1] : more[0], v[i], shift);
    }
    return __builtin_bit_cast(s16x8, out);
  }
};

template <int XT, int FR, int FJ, int ALIGN>
__global__ __launch_bounds__(512, (FR > 1 && ALIGN < 16 ? 2 : 4)) void dense_rows_i8(DenseGemm g) {
  constexpr bool kQuantize = XT != kDenseI8;
  constexpr int kRounds = 4 / FJ;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, c = lane & 15;
  const uint32_t across = (g.nj + FJ * 16 - 1) / (FJ * 16), down = (g.ni + FR * 16 - 1) / (FR * 16);
  uint32_t i = blockIdx.x / across, j_ = blockIdx.x % across;
  if (down >= kXcds) {   // rows of x stay with one XCD's L2
    j_ = blockIdx.x / kXcds % across, i = blockIdx.x / (kXcds * across) * kXcds + blockIdx.x % kXcds;
    if (i >= down) return;
  }
  const int i0 = i * FR * 16, j0 = j_ * FJ * 16;
  const int8_t* weights[FJ];
#pragma unroll
  for (int f = 0; f < FJ; ++f) weights[f] = static_cast<const int8_t*>(g.b[0]) + min(j0 + f * 16 + c, g.nj - 1) * g.ldb[0];
  const int last = (g.nr - 1) / 16 * 16;   // the last chunk of a row; what lies behind the row's end meets zeros of x
  using Raw = Eights<ALIGN>;
  // (rows at any alignment are read up to the end of the matrix, `after` bytes behind the row's)
  auto chunk = [&](const int8_t* row, int at, int64_t after) {
    at = min(at, last);
    return Raw::load(row + at, g.nr - at + after);
  };
  int64_t after_w[FJ];
#pragma unroll
  for (int f = 0; f < FJ; ++f) after_w[f] = (g.nj - 1 - min(j0 + f * 16 + c, g.nj - 1)) * g.ldb[0];
  Raw w[2][kRounds][2][FJ];
  auto ask = [&](Raw (*to)[2][FJ], int r0) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int f = 0; f < FJ; ++f)
          to[r][h][f] = chunk(weights[f], r0 + r * 1024 + h * 64 + q * 16, after_w[f]);
  };
  ask(w[0], wave * 128);
  __shared__ __align__(16) int8_t quantized[kQuantize ? kQuantizedLds : 16];
  __shared__ float row_scale[8];
  const int row_bytes = (g.nr + 127) / 128 * 128 + 16;   // of a row in LDS: 16 rows' chunks lie in different banks
  if constexpr (kQuantize) {
    using T = typename Elem<XT>::T;
    __shared__ uint32_t most[8];
    // wavefronts of a row: all of its elements are in their registers
    const int each = g.ni == 1 ? 8 : g.ni == 2 ? 4 : g.ni <= 4 ? 2 : 1, row = wave / each, first = (wave % each) * 64 + lane;
    const bool mine = row < g.ni;
    const T* const x = static_cast<const T*>(g.a[0]) + min(row, g.ni - 1) * g.lda;
    float v[4][8];
    uint32_t largest = 0;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int at = (first + n * each * 64) * 8;
      if (n * each * 512 < g.nr) load8<XT>(x + min(at, g.nr - 1), min(8, max(1, g.nr - at)), v[n]);
    }
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int at = (first + n * each * 64) * 8;
      if (n * each * 512 >= row_bytes) break;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (at + e >= g.nr) v[n][e] = 0.0f;
        largest = max(largest, __float_as_uint(v[n][e]) & 0x7fffffffu);
      }
    }
    for (int step = 32; step > 0; step >>= 1) largest = max(largest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(largest), step)));
    if (lane == 0) most[wave] = largest;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 8; ++n) largest = max(largest, most[row * each + (n & (each - 1))]);
    const Scale s = Scale::of(__uint_as_float(largest));
    if (mine && first == 0) row_scale[row] = s.stored();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int at = (first + n * each * 64) * 8;
      if (n * each * 512 >= row_bytes) break;
      uint32_t out[2];
      quantize8(s, v[n], out);
      if (mine && at < row_bytes - 16) *reinterpret_cast<uint2*>(quantized + row * row_bytes + at) = uint2{out[0], out[1]};
    }
    __syncthreads();
  }
  const int8_t* rows[FR];
  int64_t after_x[FR];
#pragma unroll
  for (int f = 0; f < FR; ++f) {
    const int row = min(i0 + f * 16 + c, g.ni - 1);
    rows[f] = kQuantize ? quantized + row * row_bytes : static_cast<const int8_t*>(g.a[0]) + row * g.lda;
    after_x[f] = (g.ni - 1 - row) * g.lda;
  }
  i32x4 acc[FR][FJ] = {};
  auto multiply = [&](const Raw (*with)[2][FJ], int r0) {
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
      if (r0 + r * 1024 >= g.nr) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int at = r0 + r * 1024 + h * 64 + q * 16;
        s16x8 wide[FJ];
#pragma unroll
        for (int j = 0; j < FJ; ++j) wide[j] = with[r][h][j].get(weights[j]);
#pragma unroll
        for (int f = 0; f < FR; ++f) {
          s16x8 x;
          if constexpr (kQuantize) {
            x = *reinterpret_cast<const s16x8*>(rows[f] + at);
          } else {
            x = chunk(rows[f], at, after_x[f]).get(rows[f]);
            if (at + 16 > g.nr) x = keep16(x, g.nr - at);
          }
#pragma unroll
          for (int j = 0; j < FJ; ++j) acc[f][j] = mfma16<kDenseI8>(wide[j], x, acc[f][j]);
        }
      }
    }
  };
  for (int r0 = wave * 128; r0 < g.nr; r0 += 2 * kRounds * 1024) {
    if (r0 + kRounds * 1024 < g.nr) ask(w[1], r0 + kRounds * 1024);
    multiply(w[0], r0);
    if (r0 + kRounds * 1024 >= g.nr) break;
    if (r0 + 2 * kRounds * 1024 < g.nr) ask(w[0], r0 + 2 * kRounds * 1024);
    multiply(w[1], r0 + kRounds * 1024);
  }
  __shared__ int sums[8][FR * 16][FJ * 16];   // [wavefront][row][column]
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int j = 0; j < FJ; ++j) *reinterpret_cast<i32x4*>(&sums[wave][f * 16 + c][j * 16 + 4 * q]) = acc[f][j];
  constexpr int kEights = FJ * 2;   // of a row
  const int row = threadIdx.x / kEights, column = threadIdx.x % kEights * 8, j = j0 + column;
  const bool in = row < FR * 16 && i0 + row < g.ni && j < g.nj;
  Finish<kDenseI8, kForward> out(g, 0, min(i0 + row, g.ni - 1), min(j, g.nj - 1), 0);
  typename Finish<kDenseI8, kForward>::Held held = {};
  if (in) {
    if constexpr (kQuantize) held = out.ask_residual(), held.row = row_scale[row];
    else held = out.ask(0);
  }
  __syncthreads();
  if (!in) return;
  float s[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    int sum = 0;
#pragma unroll
    for (int n = 0; n < 8; ++n) sum += sums[n][row][column + e];
    s[e] = __int_as_float(sum);
  }
  out.put(s, held, 0);
}

// A reduction of at most KS * 32: writing the results is all.  Four wavefronts, each with the weights of FC * 16 columns in
// registers, walk rows of x by chunks of 64, which pass through LDS: loaded once for all columns of the workgroup, as
// 16-byte chunks (WHOLE) or consecutive elements, while the chunk before is multiplied.  Where there are fewer columns
// than the four hold, several take the same columns and other rows of the chunk.  Results leave through LDS, in whole
// 128-byte lines.  bf16, 65536 x 512 x 64: 75 MB in 20.9 us a call, 3.6 TB/s (at first, without LDS on the way in,
// 28.5, and with results stored from the fragments' lanes 26.3); the stores and the epilogue's instructions bound it.
template <int TYPE, int KIND, int FC, int KS, bool WHOLE>
__global__ __launch_bounds__(256) void dense_short(DenseGemm g) {
  using T = typename Elem<TYPE>::T;
  using L = Loader<TYPE>;
  constexpr int kMats = KIND == kGated ? 2 : 1;
  constexpr int kRow = KS * 32 + 16 / int(sizeof(T));   // of LDS: 16 rows' chunks lie in different banks
  __shared__ __align__(16) T tile[2][64 * kRow];
  __shared__ __align__(16) char sums[4][4096];          // 16 rows of 64 sums of each wavefront, as in store_sums
  static_assert(FC * kMats == 4);
  const int tid = threadIdx.x, lane = tid & 63, q = lane >> 4, c = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int waves_j = g.short_waves, waves_i = 4 / waves_j;        // 1, 2 or 4
  const int across = (g.nj + waves_j * FC * 16 - 1) / (waves_j * FC * 16), chunks = (g.ni + 63) / 64;
  const int j0 = (blockIdx.x % across * waves_j + wave % waves_j) * FC * 16;
  const int first = blockIdx.x / across * g.row_chunks, end = min(chunks, first + g.row_chunks);
  L w[kMats][FC][KS];
  // the epilogue's lanes: eight consecutive columns of a row
  constexpr int kLanes = KIND == kGated ? 4 : 8;
  const int e0 = lane % kLanes * 2, j = j0 + e0 * 4;
  if constexpr (WHOLE) {
#pragma unroll
    for (int m = 0; m < kMats; ++m)
#pragma unroll
      for (int n = 0; n < FC; ++n) {
        const int column = min(j0 + n * 16 + c, g.nj - 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) w[m][n][k].load(static_cast<const T*>(g.b[m]) + column * g.ldb[m], k * 32 + 8 * q, g.nr);
      }
  } else {
    // Sixteen rows at a time through LDS of the wavefront's own, so that a load reads consecutive elements: one for each
    // lane's own row and place is 64 accesses of the cache (f16 65536 x 512 x 13 in all 9.5 M instead of 2 M, 21.9 us a
    // call, so 2.6 M and 21.1; 16384 x 512 x 61 15.5 and 12.0).
    constexpr int kSide = 2 / KS, kLoads = 16 / kSide;   // rows of a load
    T* const own = &tile[0][0] + wave * 32 * kRow;
    const int column = lane % (KS * 32), row = lane / (KS * 32);
#pragma unroll
    for (int m = 0; m < kMats; ++m) {
      const T* const from = static_cast<const T*>(g.b[m]) + min(column, g.nr - 1);
      T held[FC][kLoads];
#pragma unroll
      for (int n = 0; n < FC; ++n)
#pragma unroll
        for (int e = 0; e < kLoads; ++e) held[n][e] = from[min(j0 + n * 16 + e * kSide + row, g.nj - 1) * g.ldb[m]];
#pragma unroll
      for (int n = 0; n < FC; ++n) {
#pragma unroll
        for (int e = 0; e < kLoads; ++e) own[(e * kSide + row) * kRow + column] = column < g.nr ? held[n][e] : T(0.0f);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int k = 0; k < KS; ++k) w[m][n][k].read(own + c * kRow + k * 32 + 8 * q);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    __syncthreads();
  }
  // a chunk of x: pieces of kPer elements, the same columns of different rows for a thread
  constexpr int kPer = WHOLE ? 16 / sizeof(T) : 1;
  constexpr int kWide = KS * 32 / kPer, kDown = 256 / kWide, kPieces = 64 / kDown;
  typedef T Piece __attribute__((ext_vector_type(kPer)));
  Piece held[kPieces];
  const int at = tid % kWide * kPer, down = tid / kWide;
  const bool inside = at < g.nr;
  const T* const x = static_cast<const T*>(g.a[0]) + (inside ? at : 0);
  auto fetch = [&](int chunk) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n) {
      const int64_t i = min(int64_t(chunk) * 64 + n * kDown + down, int64_t(g.ni) - 1);
      held[n] = *reinterpret_cast<const Piece*>(x + i * g.lda);
    }
  };
  auto put = [&](int slot) {
#pragma unroll
    for (int n = 0; n < kPieces; ++n)
      *reinterpret_cast<Piece*>(&tile[slot][(n * kDown + down) * kRow + at]) = inside ? held[n] : Piece(T(0.0f));
  };
  if (first >= end) return;
  constexpr int kDownRows = 64 / kLanes;   // rows that the epilogue takes at a time
  Finish<TYPE, KIND> out(g, 0, int64_t(first) * 64 + wave / waves_j * 16 + lane / kLanes, j, kDownRows);
  fetch(first);
  put(0);
  for (int chunk = first; chunk < end; ++chunk) {
    const int slot = (chunk - first) & 1;
    __syncthreads();
    if (chunk + 1 < end) fetch(chunk + 1);
#pragma unroll 1
    for (int block = wave / waves_j; block < 4; block += waves_i) {
      f32x4 acc[kMats][FC] = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        L v;
        v.read(&tile[slot][(block * 16 + c) * kRow + k * 32 + 8 * q]);
#pragma unroll
        for (int m = 0; m < kMats; ++m)
#pragma unroll
          for (int n = 0; n < FC; ++n) acc[m][n] = multiply<TYPE>(w[m][n][k], v, acc[m][n]);
      }
      char* own = sums[wave];
#pragma unroll
      for (int m = 0; m < kMats; ++m)
#pragma unroll
        for (int n = 0; n < FC; ++n)
          *reinterpret_cast<f32x4*>(own + c * 256 + ((((m * FC + n) * 4 + q) ^ c) << 4)) = acc[m][n];
#pragma unroll
      for (int row0 = 0; row0 < 16; row0 += kDownRows, out.next()) {
        const int row = row0 + lane / kLanes;
        const int64_t i = int64_t(chunk) * 64 + block * 16 + row;
        float s[2][8];
#pragma unroll
        for (int m = 0; m < kMats; ++m)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(own + row * 256 + (((m * FC * 4 + e0 + h) ^ row) << 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) s[m][4 * h + e] = v[e];
          }
        if (i < g.ni && j < g.nj) out.put(s[0], s[1]);
      }
      for (int skip = (waves_i - 1) * 16; skip > 0; skip -= kDownRows) out.next();   // the other wavefronts' blocks
    }
    if (chunk + 1 < end) put(slot ^ 1);
  }
}

// ---------------------------------------------------------------- elementwise parts of the gradients

template <class E>
__global__ __launch_bounds__(256) void dense_pack(DensePack p) {
  if constexpr (sizeof(E) == 1) pack_eights(p, blockIdx.x / p.groups, blockIdx.x % p.groups);
  else pack_rows<E>(p, blockIdx.x / p.groups, blockIdx.x % p.groups);
}

// dz (or dg and du), and the sums of their columns over a block of rows.  A thread has eight columns and every
// lanes_y-th row of its block: 256 threads are lanes_x eights of columns by lanes_y rows.  One pass over the data.
// Where all rows start at multiples of 16 bytes and hold whole eights (WHOLE), a thread's columns are consecutive and
// read and written 16 bytes at a time (8192 x 4096 gated: 335 MB in 60 us, 5.6 TB/s); else they are lanes_x apart, and a
// wavefront reads consecutive elements.  The column sums are of the 32-bit values, not of the rounded ones.  dz is rounded
// to the type, as the matrix cores take one type for both operands: the results are then 1.41 times as far from exact ones
// (bf16, gated 8192 x 4096 x 1024: 0.00234 of their norm, so 0.00166).  Two parts of dz would keep its bits and double the
// products, 210 of that call's 270 us; a slope formed in the tiles would be rounded there all the same.
template <int TYPE, bool GATED, bool WHOLE>
__global__ __launch_bounds__(256) void dense_slope(DenseSlope s) {
  using T = typename Elem<TYPE>::T;
  constexpr int kMats = GATED ? 2 : 1;
  __shared__ float sums[256][kMats * 8 + 1];
  const int lanes_x = 1 << s.log_x, x = threadIdx.x & (lanes_x - 1), y = threadIdx.x >> s.log_x;
  const int lanes_y = 256 >> s.log_x;
  const int n8 = (s.n + 7) / 8 * 8, across = (n8 / 8 + lanes_x - 1) >> s.log_x;
  const int block = blockIdx.x / across, j0 = (blockIdx.x % across) * lanes_x * 8;
  if (block >= s.row_blocks) {
    const uint32_t id = blockIdx.x - static_cast<uint32_t>(s.row_blocks) * across;
    pack_rows<std::conditional_t<TYPE == kDenseF32, uint32_t, uint16_t>>(s.pack, id / s.pack.groups, id % s.pack.groups);
    return;
  }
  const int j = j0 + (WHOLE ? x * 8 : x);
  const int rows = (s.m + s.row_blocks - 1) / s.row_blocks;
  const int64_t first = int64_t(block) * rows, end = min(int64_t(s.m), first + rows);
  float sum[kMats][8] = {};
  auto load = [&](const void* base, int64_t row, float* v) {
    const T* p = static_cast<const T*>(base) + row + j;
    if constexpr (WHOLE) {
      load8<TYPE>(p, 8, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = float(p[min(e * lanes_x, s.n - 1 - j)]);   // no branches between loads
    }
  };
  const int64_t dz_at = column_at(j, s.dz_panel);   // (a workgroup's columns are in one panel)
  auto store = [&](void* base, int64_t row, const float* v) {   // rows of dz are padded to whole eights, with zeros
    T* p = static_cast<T*>(base) + row + dz_at;
    if constexpr (WHOLE) {
      store8<TYPE>(p, 8, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (j + e * lanes_x < n8) p[e * lanes_x] = T(v[e]);
    }
  };
  if (j < n8) {
#pragma unroll(WHOLE ? 2 : 1)
    for (int64_t i = first + y; i < end; i += lanes_y) {
      float dy[8], z[8], u[8], d0[8], d1[8];
      load(s.dy, i * s.lddy, dy);
      if (s.z[0]) {
        load(s.z[0], i * s.ldz[0], z);
        if constexpr (GATED) load(s.z[1], i * s.ldz[1], u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float value;
          if constexpr (GATED) {
            d0[e] = slope_f<TYPE>(dy[e] * u[e], z[e], s.act, &value);
            d1[e] = dy[e] * value;
          } else {
            d0[e] = slope_f<TYPE>(dy[e], z[e], s.act, &value);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) d0[e] = dy[e];
      }
      if constexpr (!WHOLE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (j + e * lanes_x < s.n) continue;
          d0[e] = 0.0f;
          if constexpr (GATED) d1[e] = 0.0f;
        }
      }
      if (s.dz[0]) store(s.dz[0], i * s.lddz, d0);
      if constexpr (GATED)
        if (s.dz[1]) store(s.dz[1], i * s.lddz, d1);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum[0][e] += d0[e];
        if constexpr (GATED) sum[1][e] += d1[e];
      }
    }
  }
  if (!s.colsum[0] && !s.colsum[1] && !s.total[0] && !s.total[1]) return;
#pragma unroll
  for (int e = 0; e < kMats * 8; ++e) sums[threadIdx.x][e] = sum[e / 8][e % 8];
  __syncthreads();
  // the rows' sums are added in order, a column a thread
  for (int c = threadIdx.x; c < lanes_x * 8 * kMats; c += 256) {
    const int mat = c / (lanes_x * 8), column = c % (lanes_x * 8);
    const int thread = WHOLE ? column / 8 : column % lanes_x, e = WHOLE ? column % 8 : column / lanes_x;
    float total = 0.0f;
    for (int r = 0; r < lanes_y; ++r) total += sums[r * lanes_x + thread][mat * 8 + e];
    const int at = j0 + column;
    if (at >= s.n) continue;
    if (s.colsum[mat]) s.colsum[mat][int64_t(block) * s.n + at] = total;
    if (s.total[mat]) static_cast<T*>(s.total[mat])[at] = T(total);
  }
}

template <int TYPE, int KIND, int BM, int BN, int WI, int WJ, int PER_CU, int HALVES = 1>
int tile_launch(const DenseGemm& g, hipStream_t stream) {
  const int cols = KIND == kGated ? BN / 2 : BN;
  const int64_t tiles = int64_t((g.ni + BM - 1) / BM) * ((g.nj + cols - 1) / cols);
  const dim3 grid(static_cast<uint32_t>(tiles), g.splits);
  dense_tile<TYPE, KIND, BM, BN, WI, WJ, PER_CU, HALVES><<<grid, 64 * WI * WJ * HALVES, 0, stream>>>(g);
  if (const int rc = hipGetLastError(); rc != 0 || g.slots == 1 || g.first + g.splits < g.slots) return rc;
  const int64_t threads = int64_t((g.nj + 7) / 8) * g.ni;
  dense_join<TYPE, KIND><<<static_cast<uint32_t>((threads + 255) / 256), 256, 0, stream>>>(g);
  return hipGetLastError();
}

template <int TYPE, int BM, int BN, int WI, int WJ, int PER_CU, int HALVES = 1>
int grads_launch(const DenseGemm& w, const DenseGemm& x, hipStream_t stream) {
  auto tiles = [](const DenseGemm& g) { return int64_t((g.ni + BM - 1) / BM) * ((g.nj + BN - 1) / BN) * g.splits; };
  const int64_t w_groups = w.parts ? (tiles(w) * w.parts + kXcds - 1) / kXcds * kXcds : 0, x_groups = x.parts ? tiles(x) : 0;
  if (w_groups + x_groups == 0) return 0;
  const uint32_t grid = static_cast<uint32_t>(w_groups + x_groups);
  dense_grads<TYPE, BM, BN, WI, WJ, PER_CU, HALVES><<<grid, 64 * WI * WJ * HALVES, 0, stream>>>(w, x,
                                                                                               static_cast<uint32_t>(w_groups));
  return hipGetLastError();
}

template <int TYPE>
int products_launch(const DenseGemm& w, const DenseGemm& x, int variant, hipStream_t stream) {
  if constexpr (TYPE == kDenseF32) {
    if (variant == kTile256) return grads_launch<TYPE, 256, 128, 4, 2, 1>(w, x, stream);
    return grads_launch<TYPE, 128, 128, 2, 4, 1>(w, x, stream);
  } else if (variant == kTile256) return grads_launch<TYPE, 256, 256, 2, 4, 1>(w, x, stream);
  else if (variant == kTile128Halves) return grads_launch<TYPE, 128, 128, 2, 2, 1, 2>(w, x, stream);
  else return grads_launch<TYPE, 128, 128, 2, 2, 2>(w, x, stream);
}

template <int TYPE>
int tail_launch(const DenseGemm& w, const DenseGemm& x, const DenseColsum& c, hipStream_t stream) {
  auto joins = [](const DenseGemm& g) {
    return g.parts && g.slots > 1 ? static_cast<uint32_t>((int64_t((g.nj + 7) / 8) * g.ni + 255) / 256) : 0u;
  };
  const DenseTail t = {c.partial[0] || c.partial[1] ? uint32_t(c.n + 31) / 32 * 2 : 0u, joins(w)};
  const uint32_t groups = t.colsum_groups + t.w_groups * w.parts + joins(x);
  if (groups == 0) return 0;
  dense_tail<TYPE><<<groups, 256, 0, stream>>>(w, x, c, t);
  return hipGetLastError();
}

template <int FR, int ALIGN>
int rows_i8_launch(const DenseGemm& g, uint32_t grid, uint32_t down, hipStream_t stream) {
  const uint32_t wide = (g.nj + 31) / 32;
  if (FR > 1 || !g.quantize) {
    // (32 columns read x half as often, and may be one round of workgroups instead of two: 19 x 8192 x 4096 11.8 us, with 16
    // 13.5; 16 x 5120 x 1024 4.8 and 7.6; but 1 x 8192 x 8192 20.7 and 16.0)
    if (g.row_columns == 2) dense_rows_i8<kDenseI8, FR, 2, ALIGN><<<wide * down, 512, 0, stream>>>(g);
    else dense_rows_i8<kDenseI8, FR, 1, ALIGN><<<grid, 512, 0, stream>>>(g);
  } else if (g.result == kDenseF32) {
    dense_rows_i8<kDenseF32, 1, 1, ALIGN><<<grid, 512, 0, stream>>>(g);
  } else if (g.result == kDenseF16) {
    dense_rows_i8<kDenseF16, 1, 1, ALIGN><<<grid, 512, 0, stream>>>(g);
  } else {
    dense_rows_i8<kDenseBF16, 1, 1, ALIGN><<<grid, 512, 0, stream>>>(g);
  }
  return hipGetLastError();
}

template <int TYPE, int KIND, int FR>
int rows_launch(const DenseGemm& g, hipStream_t stream) {
  const uint32_t across = (g.nj + 15) / 16, down = (g.ni + FR * 16 - 1) / (FR * 16);
  const uint32_t grid = across * (down >= kXcds ? (down + kXcds - 1) / kXcds * kXcds : down);
  if constexpr (TYPE == kDenseI8) {
    if (g.whole == 16) return rows_i8_launch<FR, 16>(g, grid, down, stream);
    return g.whole == 4 ? rows_i8_launch<FR, 4>(g, grid, down, stream) : rows_i8_launch<FR, 1>(g, grid, down, stream);
  } else if (g.whole) dense_rows<TYPE, KIND, FR, true><<<grid, 512, 0, stream>>>(g);
  else dense_rows<TYPE, KIND, FR, false><<<grid, 512, 0, stream>>>(g);
  return hipGetLastError();
}

template <int TYPE, int KIND, int FC, int KS>
int short_launch(const DenseGemm& given, hipStream_t stream) {
  DenseGemm g = given;
  g.short_waves = g.nj <= FC * 16 ? 1 : g.nj <= FC * 32 ? 2 : 4;
  const int64_t columns = g.short_waves * FC * 16, across = (g.nj + columns - 1) / columns, chunks = (g.ni + 63) / 64;
  // Workgroups, as long as each has a chunk of rows: two a CU, as each loads its weights first (f16 65536 x 64 x 64 7.7 us,
  // with four 9.6; f32 65536 x 512 x 64 48, 51), but four where there is little to load (f16 65536 x 512 x 32 15.7, with two
  // 18.1).
  const int64_t most = KS == 1 && TYPE != kDenseF32 ? 1024 : 512, down = std::min(chunks, std::max<int64_t>(1, most / across));
  g.row_chunks = static_cast<int32_t>((chunks + down - 1) / down);
  const dim3 grid(static_cast<uint32_t>((chunks + g.row_chunks - 1) / g.row_chunks * across));
  if (g.whole) dense_short<TYPE, KIND, FC, KS, true><<<grid, 256, 0, stream>>>(g);
  else dense_short<TYPE, KIND, FC, KS, false><<<grid, 256, 0, stream>>>(g);
  return hipGetLastError();
}

template <int TYPE, int KIND>
int forward_launch(const DenseGemm& g, hipStream_t stream) {
  if (g.variant == kRows) {
    if (g.row_blocks == 1) return rows_launch<TYPE, KIND, 1>(g, stream);
    if (g.row_blocks == 2) return rows_launch<TYPE, KIND, 2>(g, stream);
    return rows_launch<TYPE, KIND, 4>(g, stream);
  }
  if constexpr (TYPE != kDenseI8) {
    if (g.variant == kShort) {
      constexpr int kColumns = KIND == kGated ? 2 : 4;
      if (g.nr <= 32) return short_launch<TYPE, KIND, kColumns, 1>(g, stream);
      return short_launch<TYPE, KIND, kColumns, 2>(g, stream);
    }
  }
  if constexpr (TYPE == kDenseF32) {
    if (g.variant == kTile256) return tile_launch<TYPE, KIND, 256, 128, 4, 2, 1>(g, stream);
    return tile_launch<TYPE, KIND, 128, 128, 2, 4, 1>(g, stream);
  }
  else if (g.variant == kTile256) return tile_launch<TYPE, KIND, 256, 256, 2, 4, 1>(g, stream);
  else if (g.variant == kTile128Halves) return tile_launch<TYPE, KIND, 128, 128, 2, 2, 1, 2>(g, stream);
  else return tile_launch<TYPE, KIND, 128, 128, 2, 2, 2>(g, stream);
}

template <int TYPE>
int slope_launch(const DenseSlope& s, hipStream_t stream) {
  const int eights = (s.n + 7) / 8, x = 1 << s.log_x;
  const uint32_t grid = static_cast<uint32_t>((eights + x - 1) / x) * s.row_blocks + s.pack.count * s.pack.groups;
  if (s.gated && s.whole) dense_slope<TYPE, true, true><<<grid, 256, 0, stream>>>(s);
  else if (s.gated) dense_slope<TYPE, true, false><<<grid, 256, 0, stream>>>(s);
  else if (s.whole) dense_slope<TYPE, false, true><<<grid, 256, 0, stream>>>(s);
  else dense_slope<TYPE, false, false><<<grid, 256, 0, stream>>>(s);
  return hipGetLastError();
}

}  // namespace

#define EMBX_DENSE_TYPE(NAME, TYPE)                                                                             \
  int dense_forward_##NAME(int kind, const DenseGemm& g, void* stream) {                                        \
    const hipStream_t s = static_cast<hipStream_t>(stream);                                                     \
    return kind == kGated ? forward_launch<TYPE, kGated>(g, s) : forward_launch<TYPE, kForward>(g, s);          \
  }                                                                                                             \
  int dense_grads_##NAME(const DenseGemm& w, const DenseGemm& x, int variant, void* stream) {                   \
    return products_launch<TYPE>(w, x, variant, static_cast<hipStream_t>(stream));                              \
  }                                                                                                             \
  int dense_tail_##NAME(const DenseGemm& w, const DenseGemm& x, const DenseColsum& c, void* stream) {           \
    return tail_launch<TYPE>(w, x, c, static_cast<hipStream_t>(stream));                                        \
  }                                                                                                             \
  int dense_slope_##NAME(const DenseSlope& s, void* stream) {                                                   \
    return slope_launch<TYPE>(s, static_cast<hipStream_t>(stream));                                             \
  }

#if EMBX_HAS_DPART(0)
int dense_pack_launch(const DensePack& p, void* stream) {
  const uint32_t grid = p.groups * p.count;
  if (p.esize == 4) dense_pack<uint32_t><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(p);
  else if (p.esize == 1) dense_pack<uint8_t><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(p);
  else dense_pack<uint16_t><<<grid, 256, 0, static_cast<hipStream_t>(stream)>>>(p);
  return hipGetLastError();
}
#endif

#if EMBX_HAS_DPART(0)
EMBX_DENSE_TYPE(f32, kDenseF32)
#endif
#if EMBX_HAS_DPART(1)
EMBX_DENSE_TYPE(f16, kDenseF16)
#endif
#if EMBX_HAS_DPART(2)
EMBX_DENSE_TYPE(bf16, kDenseBF16)
#endif
#if EMBX_HAS_DPART(3)
int dense_forward_i8(const DenseGemm& g, void* stream) { return forward_launch<kDenseI8, kForward>(g, static_cast<hipStream_t>(stream)); }
#endif

}  // namespace embx
