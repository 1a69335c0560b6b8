// C entry points of the dense layers: argument checks, the layout of the workspace and the
// launches.  See include/embx_dense.h for the contract.
#include <algorithm>
#include <cstdint>
#include <cmath>

#include "../../include/embx_dense.h"
#include "dense.hpp"

using namespace embx;

namespace {

constexpr int64_t kMaxSize = int64_t(1) << 30;     // of m, n and k: tile positions stay below 2^31
constexpr int64_t kMaxStride = int64_t(1) << 40;
constexpr size_t kAlign = 256;

size_t esize(int32_t dtype) { return dtype == EMB_DTYPE_F32 ? 4 : 2; }

// sizes, type and activation
emb_status_t check_shape(int64_t m, int64_t n, int64_t k, int32_t dtype, int32_t act) {
  if (m < 0 || n < 1 || k < 1) return EMB_ERR_INVALID_ARGUMENT;
  if (act < EMB_ACT_NONE || act > EMB_ACT_GELU) return EMB_ERR_INVALID_ARGUMENT;
  if (m > kMaxSize || n > kMaxSize || k > kMaxSize) return EMB_ERR_UNSUPPORTED;
  if (dtype != EMB_DTYPE_F32 && dtype != EMB_DTYPE_F16 && dtype != EMB_DTYPE_BF16) return EMB_ERR_UNSUPPORTED;
  return EMB_OK;
}

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// a matrix [rows, cols] that has to be there (unless it has no rows)
emb_status_t check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype) {
  if (rows == 0) return EMB_OK;
  if (!p || misaligned(p, esize(dtype))) return EMB_ERR_INVALID_ARGUMENT;
  if (ld < cols) return EMB_ERR_INVALID_ARGUMENT;
  if (ld > kMaxStride) return EMB_ERR_UNSUPPORTED;
  return EMB_OK;
}

emb_status_t check_optional(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t dtype) {
  return p ? check_matrix(p, ld, rows, cols, dtype) : EMB_OK;
}

emb_status_t check_vector(const void* p, int32_t dtype) {
  return p && misaligned(p, esize(dtype)) ? EMB_ERR_INVALID_ARGUMENT : EMB_OK;
}

#define EMBX_TRY(x)                       \
  do {                                    \
    const emb_status_t s_ = (x);          \
    if (s_ != EMB_OK) return s_;          \
  } while (0)

emb_status_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return EMB_OK;
  return !ws || misaligned(ws, kAlign) || have < need ? EMB_ERR_INVALID_ARGUMENT : EMB_OK;
}

emb_status_t run(int rc) { return rc == 0 ? EMB_OK : EMB_ERR_DEVICE; }

int64_t chunk(int32_t dtype) { return 16 / static_cast<int64_t>(esize(dtype)); }   // elements of 16 bytes

// Whether the products can read a matrix where it lies: rows that start at multiples of 16 bytes and hold whole
// chunks of 16 bytes (and a tile's offsets fit 32 bits).
bool whole(const void* p, int64_t ld, int64_t cols, int32_t dtype) {
  return !misaligned(p, 16) && ld % chunk(dtype) == 0 && cols % chunk(dtype) == 0 &&
         ld * static_cast<int64_t>(esize(dtype)) <= kMostStride;
}

// In how many panels a matrix of the workspace is: one, where a tile with so many of its rows (256 at most) can be addressed.
int32_t panels_of(int64_t rows, int64_t cols, int32_t dtype) {
  const int64_t last = (std::min<int64_t>(rows, 256) - 1) * cols * static_cast<int64_t>(esize(dtype));
  return last > kMostOffset ? static_cast<int32_t>((cols + kPanel - 1) / kPanel) : 1;
}

// the same as whole() for the elementwise passes, of every type
bool whole16(const void* p, int64_t ld, int64_t cols, int32_t dtype) {
  return !misaligned(p, 16) && ld * esize(dtype) % 16 == 0 && cols % 8 == 0;
}

using Choice = DenseChoice;

constexpr int64_t kShortSum = 64;   // the longest reduction that kShort takes

constexpr int kCus = 256;

// Microseconds of a step of 128 bytes of the reduction: where a CU has one workgroup on a GPU that is otherwise idle, and
// where every CU is full (the clock drops, and L2 is shared), with how many; and those in which a tile starts and ends.
// Measured on products of 256 to 8192 rows, with 16-bit types by tiles of 256 x 256 or 128 x 128, the latter whole or in
// halves, which take two steps at a time, with f32 by 256 x 128 or 128 x 128.
struct TileTime { double alone, full; int per_cu; double ends; int at_a_time; };

constexpr int32_t kInt8 = -8;   // "type" of products of 8-bit integers

TileTime tile_time(int32_t dtype, int variant) {
  // (a step of 128 bytes holds twice as many 8-bit integers as of 16; their results take longer, with both scales)
  if (dtype == kInt8)
    return variant == kTile256 ? TileTime{0.95, 1.54, 1, 11.0, 1}
                               : variant == kTile128 ? TileTime{0.60, 1.08, 2, 5.0, 1} : TileTime{0.47, 0.55, 1, 4.3, 2};
  if (dtype == EMB_DTYPE_F32) return variant == kTile256 ? TileTime{2.05, 2.35, 1, 3.0, 1} : TileTime{1.17, 1.30, 1, 3.0, 1};
  return variant == kTile256 ? TileTime{0.97, 1.50, 1, 3.0, 1}
                             : variant == kTile128 ? TileTime{0.62, 1.03, 2, 3.0, 1} : TileTime{0.49, 0.55, 1, 2.6, 2};
}

constexpr int kTiles[] = {kTile256, kTile128, kTile128Halves};

int tile_count(int32_t dtype) { return dtype == EMB_DTYPE_F32 ? 2 : 3; }

// steps of a tile whose reduction is split s ways
double steps_each(const TileTime& t, double steps, int s) { return std::ceil(steps / s / t.at_a_time) * t.at_a_time; }

constexpr double kMostThreads = 4294967295.0;   // of a launch, along an axis of its grid

// whether a launch may have so many workgroups of a tile's kernel
bool launches(int32_t dtype, int variant, double groups) {
  return groups * (dtype != EMB_DTYPE_F32 && variant == kTile128 ? 256 : 512) <= kMostThreads;
}

constexpr double kLaunchUs = 5.0, kCallUs = 2.0;   // of a further launch, and what the first adds to the tiles' times
constexpr double kJoinBytes = 3.0e6;      // a microsecond, of partial sums written and read back
constexpr double kMostPartial = 256 << 20;

int64_t tiles_of(int32_t dtype, int variant, int64_t rows, int64_t columns) {
  const int64_t down = variant == kTile256 ? 256 : 128, across = variant == kTile256 && dtype != EMB_DTYPE_F32 ? 256 : 128;
  return ((rows + down - 1) / down) * ((columns + across - 1) / across);
}

int64_t steps_of(int32_t dtype, int64_t nr) {
  const int64_t step = 128 / static_cast<int64_t>(esize(dtype));
  return (nr + step - 1) / step;
}

// of a step where `groups` workgroups are on the GPU
double step_of(const TileTime& t, double groups) {
  if (t.per_cu == 1) return t.alone + (t.full - t.alone) * std::min(1.0, groups / kCus);
  return groups <= kCus ? t.alone : t.full;
}

// a forward product whose reduction is split s ways
double tile_us(int32_t dtype, int variant, double tiles, double steps, int s, double result_bytes) {
  const TileTime t = tile_time(dtype, variant);
  const double groups = tiles * s, each = steps_each(t, steps, s), slots = kCus * t.per_cu;
  const double whole = std::floor(groups / slots), rest = groups - whole * slots;
  double us = whole * (each * t.full + t.ends);
  if (rest > 0) us += each * (whole > 0 && t.per_cu == 1 ? t.full : step_of(t, rest)) + t.ends;
  if (s > 1) us += kLaunchUs + result_bytes * s / kJoinBytes;
  return us;
}

// The same by workgroups of 16 columns and 16 times `blocks` rows, a step being 32 of the reduction of each of eight
// wavefronts.  Measured on 1 to 65536 rows by 1 to 8192 columns and 256 to 8192 inputs, whole operands and others.
double rows_us(int32_t dtype, int mats, bool whole, int blocks, int64_t ni, int64_t nj, int64_t nr) {
  const double groups = double((nj + 15) / 16) * double((ni + 16 * blocks - 1) / (16 * blocks)), a_cu = groups / kCus;
  // a last step that some of the wavefronts have counts whole where nothing else runs meanwhile, and so does a second group
  // that some of the CUs have, by half
  const double steps = a_cu > 1.0 ? std::max(whole ? 0.6 : 1.0, nr / 256.0) : std::ceil(nr / 256.0);
  const double load = a_cu <= 1.0 ? 1.0 : a_cu <= 2.0 ? (a_cu + 2.0) / 2.0 : a_cu;
  const int at = blocks == 1 ? 0 : blocks == 2 ? 1 : 2;
  static const double k16[] = {0.5, 0.7, 1.05}, kOdd16[] = {0.58, 0.8, 1.3}, kOddFull16[] = {0.58, 0.8, 2.0},
                      k32[] = {0.93, 1.35, 2.45}, kTwo16[] = {1.5, 1.33, 1.2}, kTwo[] = {1.6, 1.6, 1.4};
  const bool f32 = dtype == EMB_DTYPE_F32;
  const double step = (f32 ? k32 : whole ? k16 : a_cu > 1.0 ? kOddFull16 : kOdd16)[at];
  const double two = mats == 1 ? 1.0 : (f32 || !whole ? kTwo : kTwo16)[at];   // a second weight beside each
  const double idle = a_cu <= 0.5 ? 0.75 : 1.0;   // fewer groups than half of the CUs load faster
  return 3.0 + steps * step * two * load * idle;
}

// Microseconds of the kernel of few rows of 8-bit integers, with 16 times `blocks` rows and `columns` columns a workgroup:
// measured on 1 to 256 rows by 512 to 14336 columns and 256 to 8192 inputs, whole operands and others.  A round of a workgroup
// a CU takes so much, and so much for each 1024 of the reduction (a round that some of the CUs have counts whole); and what
// reading the weights adds.
double rows_i8_us(int blocks, int columns, int64_t m, int64_t n, int64_t k, int align) {
  struct Round { double start, step, read; };
  static const Round kRound[3][2] = {{{1.32, 0.65, 0.03}, {0.63, 1.16, 0.23}}, {{1.57, 1.03, 0.27}, {1.18, 1.54, 0.29}},
                                     {{1.91, 1.67, 0.0}, {2.12, 2.42, 0.20}}};
  const Round& r = kRound[blocks == 1 ? 0 : blocks == 2 ? 1 : 2][columns == 1 ? 0 : 1];
  const int64_t groups = ((m + 16 * blocks - 1) / (16 * blocks)) * ((n + 16 * columns - 1) / (16 * columns));
  const double rounds = std::ceil(double(groups) / kCus), steps = std::max(0.25, k / 1024.0);
  const double slower = align == 16 ? 1.0 : align == 4 ? 1.2 : blocks == 1 ? 1.5 : 2.0;
  return 3.0 + rounds * (r.start * std::clamp(steps, 0.5, 1.0) + r.step * steps) * slower + r.read * n * k / 5e6;
}

// The same of the kernel for short reductions: its workgroups (the launch's own arithmetic), each with `rows` chunks of 64
// rows one after another.  A chunk takes 6.6 us in f32 (4 of at most 32 inputs) and 3 (2.2) in 16 bits where a CU has one
// workgroup, and two to four share a CU at 0.85 of each one's time.
double short_us(int32_t dtype, int mats, int64_t ni, int64_t nj, int64_t nr) {
  const int64_t wide = 64 / mats, waves = nj <= wide ? 1 : nj <= 2 * wide ? 2 : 4;
  const int64_t across = (nj + waves * wide - 1) / (waves * wide);
  const int64_t most = nr <= 32 && dtype != EMB_DTYPE_F32 ? 1024 : 512, chunks = std::max<int64_t>(1, (ni + 63) / 64);
  const int64_t down = std::min(chunks, std::max<int64_t>(1, most / across)), rows = (chunks + down - 1) / down;
  const double a_cu = std::ceil(double((chunks + rows - 1) / rows * across) / kCus);
  const double chunk = dtype == EMB_DTYPE_F32 ? (nr <= 32 ? 4.0 : 6.6) : nr <= 32 ? 2.2 : 3.0;
  const double later = std::max<double>(0.0, rows - 2.0) * (dtype == EMB_DTYPE_F32 ? 0.9 : 0.6);   // the loads are ahead by then
  return 3.3 + (std::min<double>(2.0, rows) + later) * chunk * waves / 4.0 * (a_cu > 1.0 ? 0.85 * a_cu : 1.0);
}

// the copies of operands that are not whole
double pack_us(double bytes) { return 3.0 + bytes / 2.1e6; }

// How a forward product is computed.  What the alternatives measured, in us a call (a call takes 4.4 from the host):
//   a reduction of at most 64: the kernel for it, unless another is estimated to be faster (f16 65536 x 512 x 64 20.7, best
//     tile 26.8; x 32 15.9 and 26.7; f32 x 64 49.0 and 53.9; but f32 12247 x 576 x 64 27.4 and 15.2, f16 12.8 and 9.0; f32 408
//     x 256 x 64 9.8, the kernel of few rows 4.7)
//   few rows or columns: the kernel for them, where it is estimated to be faster than tiles (bf16 16 x 512 x 1664 5.3, best
//     tile 9.0; 16 x 4096 x 4096 9.9 and 13.0; f16 2048 x 64 x 1024 5.3 and 9.8, 65536 x 1 x 1024 21.6 and 25.3; but 64 x 8192
//     x 8192 73 and 29.5, 65536 x 32 x 1024 39.7 and 24.6; f32 64 x 4096 x 4096 38.6 and 27.6)
//   tiles of 256 where they fill the GPU (bf16 4096^3 100, tiles of 128 135), of 128 else (2048^3 44 and 27.6), in halves
//     where a CU has one (2048^3 23.1, 4096 x 1024 x 1024 14.1, whole 16.8; 2 x 704 columns, 352 tiles, 13.2 and 9.3), their
//     reductions split where there are few (f32 4096 x 512 x 1664 whole 61, in two 45, in four 54)
// `whole`, `bytes`: whether both operands are, and the size of those that are not; `panels`: launches that tiles take, one
// after another.
Choice choose_forward(int32_t dtype, int kind, int64_t m, int64_t n, int64_t k, bool whole, double bytes, int panels) {
  const int mats = kind == kGated ? 2 : 1;
  const double steps = static_cast<double>(steps_of(dtype, panels > 1 ? kPanel : k)), result_bytes = 4.0 * m * n * mats;
  Choice best = {kTile128, 1, 0}, few = {kRows, 1, 1};
  double least = 0.0, few_us = 0.0;
  for (int i = 0; i < tile_count(dtype); ++i) {
    const int variant = kTiles[i];
    const double tiles = static_cast<double>(tiles_of(dtype, variant, m, n * mats));
    if (i > 0 && !launches(dtype, variant, tiles)) continue;
    for (int s = 1; s <= 128 && (s == 1 || (s * 4 <= steps && result_bytes * s * panels <= kMostPartial)); ++s) {
      const double us = tile_us(dtype, variant, tiles, steps, s, result_bytes);
      if (least == 0.0 || us < 0.98 * least) least = us, best = {variant, s, 0};
    }
  }
  least *= panels;
  // weights that come from memory: f32 tiles ask for them two steps ahead, which reaches 2.2 TB/s
  if (dtype == EMB_DTYPE_F32) least = std::max(least, 4.0 * n * k * mats / 2.2e6);
  least += kCallUs;   // (the other estimates count from the launch)
  if (k <= kShortSum) least += double(esize(dtype)) * m * n / 5.1e6;   // writing the results is not hidden then
  if (!whole) least += pack_us(bytes);
  for (int blocks : {1, 2, 4}) {
    if (blocks > 1 && m <= 8 * blocks) break;
    if (512.0 * ((n + 15) / 16) * ((m + 16 * blocks - 1) / (16 * blocks) + kXcds) > kMostThreads) continue;
    const double us = rows_us(dtype, mats, whole, blocks, m, n, k);
    if (few_us == 0.0 || us < few_us) few_us = us, few.row_blocks = blocks;
  }
  if (few_us == 0.0) few_us = HUGE_VAL;
  if (k <= kShortSum && short_us(dtype, mats, m, n, k) < std::min(1.25 * least, few_us)) return {kShort, 1, 0};
  return few_us <= least ? few : best;
}

// The tile of a backward pass's two products, and how often the reduction of each is split.
struct GradChoice { int32_t variant, w_splits, x_splits; };

// when `slots` workgroups at a time have done w_items of w us each and then x_items of x us each
double both_us(int64_t slots, int64_t w_items, double w, int64_t x_items, double x) {
  const int64_t rounds = w_items / slots, late = w_items % slots;
  double end = rounds * w + (late ? w : 0.0);
  // x's items fill the slots that end early, then all of them
  const double early = rounds * w, gap = late ? w : 0.0;
  const int64_t in_gap = late ? (slots - late) * static_cast<int64_t>(gap / x) : 0;
  if (x_items <= in_gap) return std::max(end, early + x * std::ceil(double(x_items) / std::max<int64_t>(1, slots - late)));
  const int64_t left = x_items - in_gap;
  return std::max(end, early + gap) + x * std::ceil(double(left) / slots);
}

// `panels`: of x's reduction, a launch each.
GradChoice choose_backward(int32_t dtype, int64_t m, int64_t n, int64_t k, int mats, bool want_x, int want_w, bool sums,
                           int panels) {
  static const int kSplits[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128};
  const int64_t w_steps = steps_of(dtype, m), x_steps = steps_of(dtype, panels > 1 ? kPanel : n) * mats;
  const double w_bytes = 4.0 * n * k * want_w, x_bytes = 4.0 * m * k;
  GradChoice best = {kTile128, 1, 1};
  double least = 0.0;
  for (int i = 0; i < tile_count(dtype); ++i) {
    const int variant = kTiles[i];
    const TileTime t = tile_time(dtype, variant);
    const int64_t w_tiles = want_w * tiles_of(dtype, variant, n, k), x_tiles = want_x ? tiles_of(dtype, variant, m, k) : 0;
    if (i > 0 && !launches(dtype, variant, static_cast<double>(w_tiles + x_tiles) + kXcds)) continue;
    for (int sw : kSplits) {
      if (sw > 1 && (!want_w || sw * 4 > w_steps || w_bytes * sw > kMostPartial || w_tiles * sw > 8 * kCus)) break;
      for (int sx : kSplits) {
        if (sx > 1 && (!want_x || sx * 4 > x_steps || x_bytes * sx * panels > kMostPartial || x_tiles * sx > 8 * kCus)) break;
        const int64_t items = w_tiles * sw + x_tiles * sx, slots = items <= kCus ? kCus : kCus * t.per_cu;
        const double step = step_of(t, static_cast<double>(items));
        double us = both_us(slots, w_tiles * sw, steps_each(t, w_steps, sw) * step + t.ends, x_tiles * sx,
                            steps_each(t, x_steps, sx) * step + t.ends);
        if (sw > 1 || sx > 1 || sums) us += kLaunchUs;
        us += ((sw > 1 ? w_bytes * sw : 0.0) + (sx > 1 ? x_bytes * sx : 0.0)) / kJoinBytes;
        if (least == 0.0 || us < 0.98 * least) least = us, best = {variant, sw, sx};
      }
    }
  }
  return best;
}

// bytes of partial sums: rows of whole eights
size_t partial_bytes(int64_t rows, int64_t columns, int results, int splits) {
  return splits > 1 ? size_t(splits) * rows * ((columns + 7) / 8 * 8) * results * 4 : 0;
}

emb_status_t forward(int32_t dtype, int kind, const DenseGemm& g, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_forward_f32(kind, g, stream));
    case EMB_DTYPE_F16: return run(dense_forward_f16(kind, g, stream));
    default: return run(dense_forward_bf16(kind, g, stream));
  }
}

emb_status_t grads(int32_t dtype, const DenseGemm& w, const DenseGemm& x, int variant, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_grads_f32(w, x, variant, stream));
    case EMB_DTYPE_F16: return run(dense_grads_f16(w, x, variant, stream));
    default: return run(dense_grads_bf16(w, x, variant, stream));
  }
}

emb_status_t tail(int32_t dtype, const DenseGemm& w, const DenseGemm& x, const DenseColsum& c, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_tail_f32(w, x, c, stream));
    case EMB_DTYPE_F16: return run(dense_tail_f16(w, x, c, stream));
    default: return run(dense_tail_bf16(w, x, c, stream));
  }
}

emb_status_t slope(int32_t dtype, const DenseSlope& s, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_slope_f32(s, stream));
    case EMB_DTYPE_F16: return run(dense_slope_f16(s, stream));
    default: return run(dense_slope_bf16(s, stream));
  }
}

// Hands out the workspace; with a NULL base it only counts.
struct Arena {
  char* base;
  size_t used = 0;
  template <class P>
  P* take(size_t bytes) {
    char* p = base ? base + used : nullptr;
    used += (bytes + kAlign - 1) / kAlign * kAlign;
    return reinterpret_cast<P*>(p);
  }
};

// A matrix as the products read it: where it lies, or in the workspace.
struct Operand {
  const void* p;
  int64_t ld, panel = kPanel;
  int32_t panels = 1;
};

// A matrix of the workspace whose rows are padded to multiples of `pad` elements; long rows in panels (whose rows are kept
// from starting a power of two apart).
Operand matrix_space(Arena& ar, int64_t rows, int64_t cols, int64_t pad, int32_t panels, int32_t dtype) {
  const int64_t size = static_cast<int64_t>(esize(dtype));
  Operand o = {nullptr, (cols + pad - 1) / pad * pad};
  o.panels = panels;
  if (panels > 1) o.ld = kPanel + 64, o.panel = rows * o.ld;
  o.p = ar.take<void>(static_cast<size_t>(o.panels) * rows * o.ld * size);
  return o;
}

// its panel p
const void* panel_of(const Operand& o, int32_t p, int32_t dtype) {
  return static_cast<const char*>(o.p) + p * o.panel * static_cast<int64_t>(esize(dtype));
}

// Collects the matrices of a call that have to be copied.
struct Packer {
  Arena& ar;
  int32_t dtype;
  DensePack pack = {};
  bool where_they_lie = false;   // nothing is copied
  // panels: of a copy
  Operand use(const void* p, int64_t ld, int64_t rows, int64_t cols, int32_t panels) {
    if (rows == 0 || where_they_lie || whole(p, ld, cols, dtype)) return {p, ld};
    const Operand copy = matrix_space(ar, rows, cols, chunk(dtype), panels, dtype);
    pack.esize = static_cast<int32_t>(esize(dtype));
    const int at = pack.count++;
    pack.src[at] = p, pack.lds[at] = ld;
    pack.dst[at] = const_cast<void*>(copy.p), pack.ldd[at] = copy.ld, pack.panel[at] = copy.panel;
    pack.rows[at] = static_cast<uint32_t>(rows), pack.cols[at] = static_cast<uint32_t>(cols);
    uint32_t wide = 8;
    while (wide < 256 && wide < cols) wide *= 2;
    pack.wide[at] = wide;
    // enough workgroups for the longest matrix, with four rows a thread, at most eight a CU
    pack.groups = std::max<int32_t>(pack.groups, static_cast<int32_t>(std::min<int64_t>(8 * kCus, (rows * wide + 1023) / 1024)));
    return copy;
  }
};

// log2 of the eights of columns that a workgroup of the elementwise pass has side by side: as many as a row has, at
// most 64 (a wavefront reads 1 KB of a row)
int32_t slope_log_x(int64_t n) {
  int32_t l = 0;
  while (l < 6 && (int64_t(8) << l) < n) ++l;
  return l;
}

// Blocks of rows of that pass.  One where each thread has at most four rows: it adds the column sums up by itself, and
// no other launch is needed for them (77 columns of 63 rows: 20.4 us a call against 23.2).  Else as many as there are
// rows for, up to 1024 workgroups (3001 x 77 with one row a thread 29 us a call, with four 35) and 512 blocks, whose sums
// are added up afterwards (16384 x 1024 with 256: 242 us a call, with 512: 234).
int32_t slope_blocks(int64_t m, int64_t n) {
  const int32_t log_x = slope_log_x(n);
  const int64_t across = ((n + 7) / 8 + (1 << log_x) - 1) >> log_x;
  const int64_t rows = 256 >> log_x;
  if (m <= 4 * rows) return 1;
  return static_cast<int32_t>(std::min({int64_t(512), (1024 + across - 1) / across, (m + rows - 1) / rows}));
}

// The workspace of each call: copies of operands, dz, column sums and partial sums of products.
struct Space {
  Choice choice = {kTile128, 1, 0};   // of the forward calls
  Operand x, w[2], dz[2];
  DensePack pack;
  float* colsum[2] = {nullptr, nullptr};
  float* partial = nullptr;                   // of the forward product
  GradChoice grads = {kTile128, 1, 1};        // of the backward calls (x's splits: of a panel)
  float *w_partial = nullptr, *x_partial = nullptr;
  int32_t blocks = 1;         // of rows of column sums
  bool slopes = false;        // dz is computed
};

void forward_partial(Arena& ar, Space& s, int64_t m, int64_t n, int mats) {
  if (s.choice.variant >= kRows) return;
  s.partial = ar.take<float>(partial_bytes(m, n, mats, s.choice.splits * s.x.panels));
}

Space linear_space(Arena& ar, const emb_linear_t& a) {
  Space s;
  Packer pk{ar, a.dtype};
  const bool x = whole(a.x, a.ldx, a.k, a.dtype), w = whole(a.weight, a.ldw, a.k, a.dtype);
  const double bytes = double(esize(a.dtype)) * a.k * ((x ? 0 : a.m) + (w ? 0 : a.n));
  const int32_t panels = panels_of(std::max(a.m, a.n), a.k, a.dtype);   // of both operands alike
  s.choice = choose_forward(a.dtype, kForward, a.m, a.n, a.k, x && w, bytes, panels);
  pk.where_they_lie = s.choice.variant >= kRows;
  s.x = pk.use(a.x, a.ldx, a.m, a.k, panels);
  s.w[0] = pk.use(a.weight, a.ldw, a.n, a.k, panels);
  s.pack = pk.pack;
  forward_partial(ar, s, a.m, a.n, 1);
  return s;
}

Space gated_space(Arena& ar, const emb_gated_t& a) {
  Space s;
  Packer pk{ar, a.dtype};
  const bool x = whole(a.x, a.ldx, a.k, a.dtype);
  const bool w = whole(a.w_gate, a.ld_gate, a.k, a.dtype) && whole(a.w_up, a.ld_up, a.k, a.dtype);
  const double bytes = double(esize(a.dtype)) * a.k * ((x ? 0 : a.m) + (w ? 0 : 2 * a.n));
  const int32_t panels = panels_of(std::max(a.m, a.n), a.k, a.dtype);   // of both operands alike
  s.choice = choose_forward(a.dtype, kGated, a.m, a.n, a.k, x && w, bytes, panels);
  pk.where_they_lie = s.choice.variant >= kRows;
  s.x = pk.use(a.x, a.ldx, a.m, a.k, panels);
  s.w[0] = pk.use(a.w_gate, a.ld_gate, a.n, a.k, panels);
  s.w[1] = pk.use(a.w_up, a.ld_up, a.n, a.k, panels);
  s.pack = pk.pack;
  forward_partial(ar, s, a.m, a.n, 2);
  return s;
}

// a computed dz: rows padded to whole eights
Operand dz_space(Arena& ar, int64_t m, int64_t n, int32_t dtype) {
  return matrix_space(ar, m, n, 8, panels_of(m, n, dtype), dtype);
}

float* colsum_space(Arena& ar, bool wanted, int32_t blocks, int64_t n) {
  return wanted && blocks > 1 ? ar.take<float>(size_t(blocks) * n * 4) : nullptr;
}

void partial_space(Arena& ar, Space& s, int32_t dtype, int64_t m, int64_t n, int64_t k, int mats, bool want_x, int want_w,
                   bool sums) {
  s.grads = choose_backward(dtype, m, n, k, mats, want_x, want_w, sums, s.dz[0].panels);
  s.w_partial = ar.take<float>(partial_bytes(n, k, want_w, s.grads.w_splits));
  s.x_partial = ar.take<float>(partial_bytes(m, k, 1, s.grads.x_splits * s.dz[0].panels));
}

Space linear_grad_space(Arena& ar, const emb_linear_grad_t& a) {
  Space s;
  Packer pk{ar, a.dtype};
  const bool dx = a.dx && a.m > 0;
  s.slopes = a.activation != EMB_ACT_NONE && a.m > 0 && (dx || a.dweight);
  if (s.slopes) s.dz[0] = dz_space(ar, a.m, a.n, a.dtype);
  else if (dx || a.dweight) s.dz[0] = pk.use(a.dy, a.lddy, a.m, a.n, panels_of(a.m, a.n, a.dtype));
  if (dx) s.w[0] = pk.use(a.weight, a.ldw, a.n, a.k, panels_of(a.n, a.k, a.dtype));
  if (a.dweight) s.x = pk.use(a.x, a.ldx, a.m, a.k, panels_of(a.m, a.k, a.dtype));
  s.pack = pk.pack;
  s.blocks = slope_blocks(a.m, a.n);
  s.colsum[0] = colsum_space(ar, a.dbias, s.blocks, a.n);
  partial_space(ar, s, a.dtype, a.m, a.n, a.k, 1, dx, a.dweight ? 1 : 0, a.dbias && s.blocks > 1);
  return s;
}

Space gated_grad_space(Arena& ar, const emb_gated_grad_t& a) {
  Space s;
  Packer pk{ar, a.dtype};
  const bool dx = a.dx && a.m > 0;
  const int weights = (a.dw_gate != nullptr) + (a.dw_up != nullptr);
  s.slopes = a.m > 0 && (dx || weights);
  for (int i = 0; i < 2 && s.slopes; ++i) s.dz[i] = dz_space(ar, a.m, a.n, a.dtype);
  if (dx) {
    s.w[0] = pk.use(a.w_gate, a.ld_gate, a.n, a.k, panels_of(a.n, a.k, a.dtype));
    s.w[1] = pk.use(a.w_up, a.ld_up, a.n, a.k, panels_of(a.n, a.k, a.dtype));
  }
  if (weights) s.x = pk.use(a.x, a.ldx, a.m, a.k, panels_of(a.m, a.k, a.dtype));
  s.pack = pk.pack;
  s.blocks = slope_blocks(a.m, a.n);
  s.colsum[0] = colsum_space(ar, a.db_gate, s.blocks, a.n);
  s.colsum[1] = colsum_space(ar, a.db_up, s.blocks, a.n);
  partial_space(ar, s, a.dtype, a.m, a.n, a.k, 2, dx, weights, (a.db_gate || a.db_up) && s.blocks > 1);
  return s;
}

// A forward product: a launch, or one for each panel of its reduction.
emb_status_t run_forward(int32_t dtype, int kind, DenseGemm& g, const Space& sp, void* stream) {
  const bool tiles = sp.choice.variant < kRows;
  g.a[0] = sp.x.p, g.lda = sp.x.ld, g.panel_a = sp.x.panel;
  for (int i = 0; i < (kind == kGated ? 2 : 1); ++i)
    g.b[i] = sp.w[i].p, g.ldb[i] = sp.w[i].ld, g.panel_b[i] = sp.w[i].panel;
  g.parts = 1, g.variant = sp.choice.variant, g.splits = sp.choice.splits, g.row_blocks = sp.choice.row_blocks;
  g.partial = sp.partial, g.slots = g.splits * sp.x.panels;
  if (!tiles || sp.x.panels == 1) return forward(dtype, kind, g, stream);
  const int32_t nr = g.nr;
  for (int32_t p = 0; p < sp.x.panels; ++p) {
    g.a[0] = panel_of(sp.x, p, dtype);
    for (int i = 0; i < (kind == kGated ? 2 : 1); ++i) g.b[i] = panel_of(sp.w[i], p, dtype);
    g.nr = static_cast<int32_t>(std::min<int64_t>(kPanel, nr - p * kPanel));
    g.first = p * g.splits;
    EMBX_TRY(forward(dtype, kind, g, stream));
  }
  return EMB_OK;
}

// Both products of a backward pass: a launch, or one for each panel of x's reduction; then the joins.
emb_status_t run_backward(int32_t dtype, const DenseGemm& w, DenseGemm& x, const DenseColsum& c, const Space& sp,
                          void* stream) {
  const int32_t variant = sp.grads.variant, panels = x.parts ? sp.dz[0].panels : 1, nr = x.nr;
  const DenseGemm none = {};
  x.slots = x.splits * panels;
  double groups = kXcds;
  if (w.parts) groups += double(w.splits) * w.parts * tiles_of(dtype, variant, w.ni, w.nj);
  if (x.parts) groups += double(x.splits) * tiles_of(dtype, variant, x.ni, x.nj);
  const bool together = launches(dtype, variant, groups);
  for (int i = 0; i < w.parts && !together; ++i) {   // (so many results are not split: there are no partial sums)
    DenseGemm one = w;
    one.parts = 1, one.a[0] = w.a[i], one.c[0] = w.c[i], one.ldc[0] = w.ldc[i];
    EMBX_TRY(grads(dtype, one, none, variant, stream));
  }
  for (int32_t p = 0; p < panels; ++p) {
    if (panels > 1) {
      for (int i = 0; i < x.parts; ++i) {
        x.a[i] = panel_of(sp.dz[i], p, dtype);
        x.b[i] = static_cast<const char*>(sp.w[i].p) + p * kPanel * sp.w[i].ld * static_cast<int64_t>(esize(dtype));
      }
      x.nr = static_cast<int32_t>(std::min<int64_t>(kPanel, nr - p * kPanel));
      x.first = p * x.splits;
    }
    EMBX_TRY(grads(dtype, p == 0 && together ? w : none, x, variant, stream));
  }
  return tail(dtype, w, x, c, stream);
}

emb_status_t run_pack(const DensePack& p, void* stream) {
  return p.count ? run(dense_pack_launch(p, stream)) : EMB_OK;
}

}  // namespace

// Products of 8-bit integers: the same tiles, whose steps hold twice as many of the reduction as of 16-bit elements.
DenseChoice embx::dense_choose_i8(int64_t m, int64_t n, int64_t k, int align, double copied) {
  const double steps = std::ceil(k / 128.0), result_bytes = 4.0 * m * n;
  Choice best = {-1, 1, 0}, few = {kRows, 1, 1};
  double least = HUGE_VAL, few_us = HUGE_VAL;
  for (const int variant : kTiles) {
    const double tiles = static_cast<double>(tiles_of(kInt8, variant, m, n));
    if (!launches(kInt8, variant, tiles)) continue;
    for (int s = 1; s <= 128 && (s == 1 || (s * 4 <= steps && result_bytes * s <= kMostPartial && tiles * s <= 4 * kCus)); ++s) {
      const double us = tile_us(kInt8, variant, tiles, steps, s, result_bytes);
      if (us < 0.98 * least) least = us, best = {variant, s, 0};
    }
  }
  least += kCallUs;
  if (copied > 0) least += 2.0 + copied / 2.2e6;
  if (k <= 128) least += 1.5 + 2.0 * m * n / 5.1e6;   // a tile's first loads and its results are all
  for (const int blocks : {1, 2, 4}) {
    if (blocks > 1 && m <= 8 * blocks) break;
    const int64_t down = (m + 16 * blocks - 1) / (16 * blocks);
    if (512.0 * ((n + 15) / 16) * (down + kXcds) > kMostThreads) continue;
    for (const int columns : {1, 2}) {
      if (columns == 2 && down >= kXcds) continue;
      const double us = rows_i8_us(blocks, columns, m, n, k, align);
      if (us < few_us) few_us = us, few.row_blocks = blocks, few.row_columns = columns;
    }
  }
  return few_us < HUGE_VAL && few_us <= least ? few : best;
}

extern "C" {

emb_status_t emb_linear_workspace(const emb_linear_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  Arena ar{nullptr};
  linear_space(ar, *a);
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_linear(const emb_linear_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->weight, a->ldw, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->bias, a->dtype));
  EMBX_TRY(check_optional(a->residual, a->ldr, a->m, a->n, a->dtype));
  EMBX_TRY(check_matrix(a->y, a->ldy, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->z, a->ldz, a->m, a->n, a->dtype));
  Arena ar{static_cast<char*>(workspace)};
  const Space sp = linear_space(ar, *a);
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  if (a->m == 0) return EMB_OK;
  EMBX_TRY(run_pack(sp.pack, stream));
  DenseGemm g = {};
  g.c[0] = a->y, g.ldc[0] = a->ldy;
  g.z[0] = a->z, g.ldz[0] = a->ldz;
  g.bias[0] = a->bias;
  g.res = a->residual, g.ldr = a->ldr;
  g.ni = a->m, g.nj = a->n, g.nr = a->k;
  g.act = a->activation;
  g.whole = whole(a->x, a->ldx, a->k, a->dtype) && whole(a->weight, a->ldw, a->k, a->dtype);
  return run_forward(a->dtype, kForward, g, sp, stream);
}

emb_status_t emb_linear_backward_workspace(const emb_linear_grad_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  Arena ar{nullptr};
  linear_grad_space(ar, *a);
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_linear_backward(const emb_linear_grad_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  const bool slopes = a->activation != EMB_ACT_NONE;
  EMBX_TRY(check_matrix(a->dy, a->lddy, a->m, a->n, a->dtype));
  if (slopes) EMBX_TRY(check_matrix(a->z, a->ldz, a->m, a->n, a->dtype));
  if (a->dweight) EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  if (a->dx) EMBX_TRY(check_matrix(a->weight, a->ldw, a->n, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dx, a->lddx, a->m, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dweight, a->lddw, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->dbias, a->dtype));
  Arena ar{static_cast<char*>(workspace)};
  const Space sp = linear_grad_space(ar, *a);
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  if (a->dbias || sp.slopes) {
    DenseSlope s = {};
    s.dy = a->dy, s.lddy = a->lddy;
    s.z[0] = slopes ? a->z : nullptr, s.ldz[0] = a->ldz;
    s.dz[0] = sp.slopes ? const_cast<void*>(sp.dz[0].p) : nullptr, s.lddz = sp.dz[0].ld, s.dz_panel = sp.dz[0].panel;
    s.colsum[0] = sp.colsum[0];
    if (sp.blocks == 1) s.total[0] = a->dbias;
    s.m = a->m, s.n = a->n, s.act = a->activation, s.gated = 0, s.row_blocks = sp.blocks;
    s.log_x = slope_log_x(a->n);
    s.whole = whole16(a->dy, a->lddy, a->n, a->dtype) && (!slopes || whole16(a->z, a->ldz, a->n, a->dtype));
    s.pack = sp.pack;
    EMBX_TRY(slope(a->dtype, s, stream));
  } else {
    EMBX_TRY(run_pack(sp.pack, stream));
  }
  DenseGemm w = {}, x = {};
  if (a->dx && a->m > 0) {
    x.a[0] = sp.dz[0].p, x.lda = sp.dz[0].ld, x.panel_a = sp.dz[0].panel;
    x.b[0] = sp.w[0].p, x.ldb[0] = sp.w[0].ld, x.panel_b[0] = sp.w[0].panel;
    x.c[0] = a->dx, x.ldc[0] = a->lddx;
    x.ni = a->m, x.nj = a->k, x.nr = a->n, x.parts = 1;
    x.splits = sp.grads.x_splits, x.partial = sp.x_partial;
  }
  if (a->dweight) {
    w.a[0] = sp.dz[0].p, w.lda = sp.dz[0].ld, w.panel_a = sp.dz[0].panel;
    w.b[0] = sp.x.p, w.ldb[0] = sp.x.ld, w.panel_b[0] = sp.x.panel;
    w.c[0] = a->dweight, w.ldc[0] = a->lddw;
    w.ni = a->n, w.nj = a->k, w.nr = a->m, w.parts = 1;
    w.splits = w.slots = sp.grads.w_splits, w.partial = sp.w_partial;
  }
  const DenseColsum c = {{sp.colsum[0], nullptr}, {a->dbias, nullptr}, sp.blocks, static_cast<int32_t>(a->n)};
  return run_backward(a->dtype, w, x, c, sp, stream);
}

emb_status_t emb_gated_workspace(const emb_gated_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  Arena ar{nullptr};
  gated_space(ar, *a);
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_gated(const emb_gated_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->w_gate, a->ld_gate, a->n, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->w_up, a->ld_up, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->b_gate, a->dtype));
  EMBX_TRY(check_vector(a->b_up, a->dtype));
  EMBX_TRY(check_matrix(a->h, a->ldh, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->g, a->ldg, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->u, a->ldu, a->m, a->n, a->dtype));
  Arena ar{static_cast<char*>(workspace)};
  const Space sp = gated_space(ar, *a);
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  if (a->m == 0) return EMB_OK;
  EMBX_TRY(run_pack(sp.pack, stream));
  DenseGemm g = {};
  g.c[0] = a->h, g.ldc[0] = a->ldh;
  g.z[0] = a->g, g.ldz[0] = a->ldg;
  g.z[1] = a->u, g.ldz[1] = a->ldu;
  g.bias[0] = a->b_gate, g.bias[1] = a->b_up;
  g.ni = a->m, g.nj = a->n, g.nr = a->k;
  g.act = a->activation;
  g.whole = whole(a->x, a->ldx, a->k, a->dtype) && whole(a->w_gate, a->ld_gate, a->k, a->dtype) &&
            whole(a->w_up, a->ld_up, a->k, a->dtype);
  return run_forward(a->dtype, kGated, g, sp, stream);
}

emb_status_t emb_gated_backward_workspace(const emb_gated_grad_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  Arena ar{nullptr};
  gated_grad_space(ar, *a);
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_gated_backward(const emb_gated_grad_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  const bool weights = a->dw_gate || a->dw_up;
  EMBX_TRY(check_matrix(a->dh, a->lddh, a->m, a->n, a->dtype));
  EMBX_TRY(check_matrix(a->g, a->ldg, a->m, a->n, a->dtype));
  EMBX_TRY(check_matrix(a->u, a->ldu, a->m, a->n, a->dtype));
  if (weights) EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  if (a->dx) {
    EMBX_TRY(check_matrix(a->w_gate, a->ld_gate, a->n, a->k, a->dtype));
    EMBX_TRY(check_matrix(a->w_up, a->ld_up, a->n, a->k, a->dtype));
  }
  EMBX_TRY(check_optional(a->dx, a->lddx, a->m, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dw_gate, a->ldd_gate, a->n, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dw_up, a->ldd_up, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->db_gate, a->dtype));
  EMBX_TRY(check_vector(a->db_up, a->dtype));
  Arena ar{static_cast<char*>(workspace)};
  const Space sp = gated_grad_space(ar, *a);
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  const bool sums = a->db_gate || a->db_up;
  if (sums || sp.slopes) {
    DenseSlope s = {};
    s.dy = a->dh, s.lddy = a->lddh;
    s.z[0] = a->g, s.ldz[0] = a->ldg;
    s.z[1] = a->u, s.ldz[1] = a->ldu;
    for (int i = 0; i < 2; ++i) s.dz[i] = sp.slopes ? const_cast<void*>(sp.dz[i].p) : nullptr;
    s.lddz = sp.dz[0].ld, s.dz_panel = sp.dz[0].panel;
    s.colsum[0] = sp.colsum[0], s.colsum[1] = sp.colsum[1];
    if (sp.blocks == 1) s.total[0] = a->db_gate, s.total[1] = a->db_up;
    s.m = a->m, s.n = a->n, s.act = a->activation, s.gated = 1, s.row_blocks = sp.blocks;
    s.log_x = slope_log_x(a->n);
    s.whole = whole16(a->dh, a->lddh, a->n, a->dtype) && whole16(a->g, a->ldg, a->n, a->dtype) &&
              whole16(a->u, a->ldu, a->n, a->dtype);
    s.pack = sp.pack;
    EMBX_TRY(slope(a->dtype, s, stream));
  } else {
    EMBX_TRY(run_pack(sp.pack, stream));
  }
  DenseGemm w = {}, x = {};
  if (a->dx && a->m > 0) {
    for (int i = 0; i < 2; ++i) x.a[i] = sp.dz[i].p, x.b[i] = sp.w[i].p, x.ldb[i] = sp.w[i].ld, x.panel_b[i] = sp.w[i].panel;
    x.lda = sp.dz[0].ld, x.panel_a = sp.dz[0].panel;
    x.c[0] = a->dx, x.ldc[0] = a->lddx;
    x.ni = a->m, x.nj = a->k, x.nr = a->n, x.parts = 2;
    x.splits = sp.grads.x_splits, x.partial = sp.x_partial;
  }
  if (weights) {
    for (int i = 0; i < 2; ++i) {
      void* dw = i == 0 ? a->dw_gate : a->dw_up;
      if (!dw) continue;
      w.a[w.parts] = sp.dz[i].p;
      w.c[w.parts] = dw, w.ldc[w.parts] = i == 0 ? a->ldd_gate : a->ldd_up;
      ++w.parts;
    }
    w.lda = sp.dz[0].ld, w.panel_a = sp.dz[0].panel;
    w.b[0] = w.b[1] = sp.x.p, w.ldb[0] = w.ldb[1] = sp.x.ld, w.panel_b[0] = w.panel_b[1] = sp.x.panel;
    w.ni = a->n, w.nj = a->k, w.nr = a->m;
    w.splits = w.slots = sp.grads.w_splits, w.partial = sp.w_partial;
  }
  const DenseColsum c = {{sp.colsum[0], sp.colsum[1]}, {a->db_gate, a->db_up}, sp.blocks, static_cast<int32_t>(a->n)};
  return run_backward(a->dtype, w, x, c, sp, stream);
}

}  // extern "C"
