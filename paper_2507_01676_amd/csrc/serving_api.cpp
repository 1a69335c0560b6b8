// C entry points of the dense layers' serving forms: argument checks, the layout of the workspace and the launches.  See
// include/embx_serving.h for the contract.
#include <algorithm>
#include <cstdint>

#include "../../include/embx_serving.h"
#include "dense.hpp"
#include "serving.hpp"

using namespace embx;

namespace {

constexpr int64_t kMaxSize = int64_t(1) << 30, kMaxStride = int64_t(1) << 40;
constexpr int64_t kMostInputs = 131071;        // of sums of 8-bit products in 32 bits: 2^14 each
constexpr int64_t kMostRows = 65536, kMostColumns = int64_t(1) << 25;   // moe
// moe: elements, 256 MB (2 of 8 of 1408 x 1024: 32768 rows 6.06 ms, 32769, which go by rows, 6.88; of 264 x 1024 2.13 and 1.88)
constexpr int64_t kMostPartial = 64 << 20;
constexpr size_t kAlign = 256;

#define EMBX_TRY(x)                       \
  do {                                    \
    const emb_status_t s_ = (x);          \
    if (s_ != EMB_OK) return s_;          \
  } while (0)

size_t esize(int32_t dtype) { return dtype == EMB_DTYPE_F32 ? 4 : 2; }

bool misaligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

emb_status_t check_type(int32_t dtype) {
  return dtype == EMB_DTYPE_F32 || dtype == EMB_DTYPE_F16 || dtype == EMB_DTYPE_BF16 ? EMB_OK : EMB_ERR_UNSUPPORTED;
}

emb_status_t check_activation(int32_t act) {
  return act < EMB_ACT_NONE || act > EMB_ACT_GELU ? EMB_ERR_INVALID_ARGUMENT : EMB_OK;
}

// a matrix [rows, cols] of elements of `size` bytes that has to be there (unless it has no rows)
emb_status_t check_matrix(const void* p, int64_t ld, int64_t rows, int64_t cols, size_t size) {
  if (rows == 0) return EMB_OK;
  if (!p || misaligned(p, size) || ld < cols) return EMB_ERR_INVALID_ARGUMENT;
  return ld > kMaxStride ? EMB_ERR_UNSUPPORTED : EMB_OK;
}

emb_status_t check_vector(const void* p, int64_t n, size_t size) {
  return n > 0 && (!p || misaligned(p, size)) ? EMB_ERR_INVALID_ARGUMENT : EMB_OK;
}

emb_status_t check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return EMB_OK;
  return !ws || misaligned(ws, kAlign) || have < need ? EMB_ERR_INVALID_ARGUMENT : EMB_OK;
}

emb_status_t run(int rc) { return rc == 0 ? EMB_OK : EMB_ERR_DEVICE; }

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

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

// Whether the products can read 8-bit rows where they lie, as chunks of 16 bytes (and a tile's offsets fit 32 bits).
bool whole(const void* p, int64_t ld) { return !misaligned(p, 16) && ld % 16 == 0 && ld <= kMostStride; }

// ---------------------------------------------------------------- linear_int8

emb_status_t check_shape(const emb_linear_int8_t& a) {
  if (a.m < 0 || a.n < 1 || a.k < 1) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_activation(a.activation));
  if (a.m > kMaxSize || a.n > kMaxSize || a.k > kMostInputs) return EMB_ERR_UNSUPPORTED;
  return check_type(a.dtype);
}

// x as the products read it: 8-bit rows that end in zeros up to a whole chunk, so that what lies behind the weights' rows
// counts for nothing.
struct Int8Space {
  DenseChoice choice;
  bool inside, quantized, packed_x, packed_w;
  int32_t align;
  const int8_t *x, *w;
  int64_t ldx, ldw;
  const float* scale;
  float* partial;
};

Int8Space int8_space(Arena& ar, const emb_linear_int8_t& a) {
  Int8Space s = {};
  const bool x = a.x_scale && whole(a.x, a.ldx) && a.k % 16 == 0, w = whole(a.weight, a.ldw);
  auto words = [](const void* p, int64_t ld) { return !misaligned(p, 4) && ld % 4 == 0; };
  s.align = w && (x || !a.x_scale) ? 16 : words(a.weight, a.ldw) && (!a.x_scale || words(a.x, a.ldx)) ? 4 : 1;
  s.choice = dense_choose_i8(a.m, a.n, a.k, s.align, double(a.k) * ((a.x_scale && !x ? a.m : 0) + (w ? 0 : a.n)));
  // A few rows that a workgroup's registers hold are quantized by each of the product's workgroups, as long as that is a round
  // of them and little beside the weights (one row of 512 x 1664 6.0 us a call, with a launch for it 7.6, of 4096 x 4096 8.2 and
  // 10.3, four 11.6 and 10.4; of 14336 x 2048 16.0 and 10.9, of 14336 x 8192 30 and 36).
  const int64_t across = (a.n + 15) / 16;
  s.inside = !a.x_scale && s.choice.variant == kRows && s.choice.row_blocks == 1 && a.m <= 8 &&
             a.k * (a.m == 1 ? 1 : a.m == 2 ? 2 : a.m <= 4 ? 4 : 8) <= (a.m <= 2 ? 16384 : 8192) &&
             (across <= 256 || (a.m == 1 && across * 8 <= a.k));
  s.quantized = !a.x_scale && !s.inside;
  const bool rows = s.choice.variant == kRows;   // reads any rows where they lie
  s.packed_x = a.x_scale && !x && !rows;
  s.packed_w = !w && !rows;
  s.x = static_cast<const int8_t*>(a.x), s.ldx = a.ldx, s.scale = a.x_scale;
  s.w = a.weight, s.ldw = a.ldw;
  if (s.quantized || s.packed_x) s.x = ar.take<int8_t>(a.m * up16(a.k)), s.ldx = up16(a.k);
  if (s.quantized) s.scale = ar.take<float>(a.m * 4);
  if (s.packed_w) s.w = ar.take<int8_t>(a.n * up16(a.k)), s.ldw = up16(a.k);
  if (s.choice.splits > 1) s.partial = ar.take<float>(size_t(s.choice.splits) * a.m * ((a.n + 7) / 8 * 8) * 4);
  return s;
}

// a matrix that is copied to rows of whole chunks
void add_copy(DensePack& p, const void* src, int64_t ld, const void* dst, int64_t rows, int64_t cols) {
  const int at = p.count++;
  p.esize = 1;
  p.src[at] = src, p.lds[at] = ld;
  p.dst[at] = const_cast<void*>(dst), p.ldd[at] = up16(cols), p.panel[at] = kPanel;
  p.rows[at] = static_cast<uint32_t>(rows), p.cols[at] = static_cast<uint32_t>(cols);
  uint32_t wide = 1;
  while (wide < 256 && wide * 16 < cols) wide *= 2;
  p.wide[at] = wide;
  p.groups = std::max<int32_t>(p.groups, static_cast<int32_t>(std::min<int64_t>(2048, (rows * wide + 1023) / 1024)));
}

// ---------------------------------------------------------------- moe

emb_status_t check_experts(const emb_experts_t& w, const emb_moe_t& a, int64_t rows, int64_t cols) {
  EMBX_TRY(check_matrix(w.p, w.ld, rows, cols, w.scale ? 1 : esize(a.dtype)));
  EMBX_TRY(check_vector(w.scale, w.scale ? 1 : 0, 4));
  if (w.stride < 0) return EMB_ERR_INVALID_ARGUMENT;
  return w.stride > kMaxStride || w.ld > kMostColumns ? EMB_ERR_UNSUPPORTED : EMB_OK;
}

emb_status_t check_shape(const emb_moe_t& a) {
  if (a.m < 0 || a.f < 1 || a.d < 1 || a.experts < 1 || a.top_k < 1 || a.top_k > a.experts) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_activation(a.activation));
  if (!a.gate.scale != !a.up.scale || !a.gate.scale != !a.down.scale) return EMB_ERR_INVALID_ARGUMENT;
  if (a.m > kMostRows || a.f > kMostColumns || a.d > kMostColumns) return EMB_ERR_UNSUPPORTED;
  if (a.experts > kMostExperts || a.top_k > kMostTopK) return EMB_ERR_UNSUPPORTED;
  return check_type(a.dtype);
}

// Rows that start at multiples of 16 bytes
bool aligned(const void* p, int64_t ld, size_t size) { return !misaligned(p, 16) && ld * static_cast<int64_t>(size) % 16 == 0; }

bool aligned(const emb_experts_t& w, size_t size) {
  return aligned(w.p, w.ld, w.scale ? 1 : size) && aligned(w.p, w.stride, w.scale ? 1 : size);
}

struct MoeSpace {
  float* h;
  int64_t ldh;
  int32_t* chosen;
  float* share;
  float* partial;
  double* logits;
};

MoeSpace moe_space(Arena& ar, const emb_moe_t& a, const MoeChoice& c) {
  const int64_t uses = a.m * a.top_k;
  MoeSpace s = {};
  s.ldh = (a.f + 7) / 8 * 8, s.chosen = a.chosen, s.share = a.share;
  if (c.apart) s.logits = ar.take<double>(a.m * a.experts * 8);
  if (c.down_variant == kMoeMany) s.partial = ar.take<float>(uses * a.d * 4);
  else if (c.splits > 1) s.partial = ar.take<float>(c.splits * a.m * a.d * 4);
  s.h = ar.take<float>(uses * s.ldh * 4);
  if (!s.chosen) s.chosen = ar.take<int32_t>(uses * 4);
  if (!s.share) s.share = ar.take<float>(uses * 4);
  return s;
}

}  // namespace

MoeChoice embx::moe_choose(const emb_moe_t& a) {
  const int64_t uses = a.m * a.top_k;
  MoeChoice s = {};
  const int64_t used = std::min<int64_t>(uses, a.experts);   // experts, at most
  const int64_t step = a.gate.scale ? 64 : 32;               // of the reduction: a matrix instruction, or two
  // The up projections: four rows of x at most go by columns of four to a wavefront (kMoeFew; us a call: one query, one expert
  // of 1024 x 4096 23.3, by 16 columns 28.4; two of eight of 2816 x 1024 16.3 and 16.5, of 5632 x 2048 40.8 and 43; four rows
  // 32.9 and 33.9), unless there are many long rows (one query, 8 of 256 of 1024 x 4096 60.6 and 59.2), or, of f32 and 8-bit
  // weights, more than a few columns (f32, two of eight of 1408 x 1024 19.7 and 18.2, of 1024 x 1024 15.3 and 16.4; 8 bits
  // 13.7 and 13.3).  As many wavefronts share the reduction as make about a workgroup a CU (two of eight of 1408 x 1024 12.9
  // with two, 16.5 with eight; of 512 x 1024 12.1 and 11.2).
  // Others by 16 columns to four wavefronts, and a workgroup has 32, where that leaves workgroups enough (64 rows, 4 of 32
  // experts of 5632 x 2048 441 with eight, 432 with four; f32, one, two of eight of 2112 x 1024 26.0 and 23.8; 19 rows, 3 of 7 of
  // 333 x 1001 35.7 and 40.9) and rows are not long (16 rows, 4 of 32 of 2048 x 4096 252 and 284; 200 rows, 4 of 64 of
  // 704 x 4096 302 and 320), else to eight.  Several times 16 rows of an expert at once where it is expected to have more than
  // 14 (128 rows, 2 of 8 91.6 with 16 at a time, 75.7 with 64; f32, 64 rows, 2 of 8 of 704 x 1024 48.0 and 44.0; but 200 rows, 4
  // of 64 of 704 x 4096 555 and 604), and 64 instead of 32 where it is more than 26 (128 rows, 2 of 8 of 2816 x 1024 72 and 80;
  // but 128 rows, 4 of 32 of 1408 x 2048 178 and 163).
  const int64_t tiles = (a.f + 15) / 16 * used;
  const int64_t size = a.gate.scale ? 1 : static_cast<int64_t>(esize(a.dtype));   // of a weight
  const bool few = size == 2 ? tiles < 352 || a.d * size < 8192 : tiles <= 128;
  s.up_variant = a.m <= 4 && few ? kMoeFew : uses <= 14 * a.experts ? kMoeMore : kMoeMany;
  s.up_waves = s.up_variant != kMoeFew && tiles > 256 && a.d * size < 8192 ? 4 : 8;
  s.up_blocks = size == 2 && uses > 26 * a.experts ? 4 : 2;
  if (s.up_variant == kMoeFew && size == 2)
    while (s.up_waves > 1 && (a.f * s.up_waves + 31) / 32 * used > 256) s.up_waves /= 2;
  const int64_t up_step = s.up_variant == kMoeFew ? step * 4 : step * 2;
  // fewer where d has no step for each, unless that leaves few workgroups (f32, 115 rows, 4 of 4 of 64 x 256, 8-bit weights
  // 30.3 with two, 18.4 with eight; 69 rows, 4 of 35 of 64 x 832 51.6 with one, 30.0 with eight; but 3 rows, 2 of 8 of
  // 256 x 512, which kMoeFew takes, 12.9 with four, 14.9 with eight), and several workgroups an expert for 32 rows each where
  // there are few (the 115 rows: 18.2 with three, 15.2 with four).
  while (s.up_waves > 1 && s.up_waves * up_step > a.d && (tiles >= 256 || s.up_variant == kMoeFew)) s.up_waves /= 2;
  const int64_t up_groups = (a.f * s.up_waves + 127) / 128 * used;
  s.up_parts = static_cast<int32_t>(std::max<int64_t>(1, std::min(256 / up_groups, (uses + used * 32 - 1) / (used * 32))));
  // The routing in every workgroup, without a launch (two of eight of 2816 x 1024: one query 16.3, with one 18.9; two 24.2 and
  // 25.9; but three 28.6 and 27.8).
  s.fused = s.up_variant != kMoeMany && a.m * a.experts <= kFused && a.m * a.experts * a.d <= 65536;
  // Logits in workgroups of their own where one would read the rows of many experts (one query, 8 of 256 of 1024 x 4096 125 us,
  // so 61; 4 of 64 of 704 x 2048 29 and 23.7; 22 rows, 2 of 20 of 1792 x 1088 62.6 and 62.0; but 8 rows, 4 of 16 of 704 x 256 23.0
  // and 24.5), and what is left of the routing in every workgroup of the up projections up to kPicked (those of 256 63 us with
  // a launch for it; f32, two rows, 4 of 64 of 512 x 1024 24.4 and 25.9)
  s.apart = a.m <= 256 && a.experts > 16;
  if (s.apart) s.fused = s.up_variant != kMoeMany && a.m * a.experts <= kPicked;
  // The down projection: 32 columns a workgroup, or 4 (one query, two of eight experts of 2816 x 1024: 17.9 with 4 columns,
  // 19.6 with 32; eight queries 37.8 and 41.7, but five with 8-bit weights 32.9 and 31.8; one, 1024 x 4096 19.8 and 17.9; f32,
  // 8 rows, 4 of 16 of 704 x 256 24.3 and 32).
  s.down_variant = (a.m <= 4 && a.d <= 2048) || (a.m <= 8 && a.d <= (a.down.scale ? 512 : 1024)) ? kMoeFew : kMoeMore;
  // Or, for more rows than that has at a time, an expert's uses together, and the sums over a row's experts in another launch
  // (200 rows, 4 of 64 of 704 x 4096 333 and 445; 1000 rows, 6 of 64 of 704 x 1024 337 and 433; 128 rows, 2 of 8 of
  // 2816 x 1024 71.9 and 75.5), unless the weights are few or of 8 bits (512 rows, 4 of 8 of 256 x 512 37 and 32; 128 rows, 4 of
  // 32 of 704 x 2048 with 8 bits 94 and 82).
  const bool many = a.m > kDownRows && !a.down.scale && a.experts * a.f * a.d * size >= 4 << 20;
  if (many && uses * a.d <= kMostPartial) s.down_variant = kMoeMany;
  const int64_t columns = s.down_variant == kMoeFew ? 4 : 32, across = (a.d + columns - 1) / columns;
  s.down_rows = static_cast<int32_t>(std::min<int64_t>(kDownRows, kUses / a.top_k));
  int64_t groups = across * ((a.m + s.down_rows - 1) / s.down_rows);
  const int64_t down_step = s.down_variant == kMoeFew ? step * 4 : step * 2;
  // Its items, of about two steps at least, are shared by up to about 256 workgroups, five items or more to each (64 rows, 4 of
  // 32 of 5632 x 2048 431 in four parts, 440 in eight; 16 rows, 2 of 8 of 2816 x 1024 47 in two, 42.7 in eight; 23 rows, 2 of
  // 29 of 32 x 165 32.8 in one, 24.6 in five; one row, one of 16 of 1024 x 4096 18.0 in one, 20.0 in two).  With few of those a
  // workgroup has fewer rows, as long as an expert has four of them or so (bf16, 1000 rows, 4 of 4 of 64 x 256 with 64 rows
  // 84, with 16 50; 115 rows, 4 of 8 of 64 x 1024 28 and 20.3; but 128 rows, 2 of 8 of 2816 x 1024 76, with 32 79).
  const int64_t shortest = (a.f + 2 * down_step - 1) / (2 * down_step);   // (parts of two steps)
  s.splits = static_cast<int32_t>(std::max<int64_t>(1, std::min({int64_t(16), used * shortest / 5, 256 / groups})));
  while (groups * s.splits <= 128 && s.down_rows > 8 && a.m > s.down_rows / 2 && s.down_rows * a.top_k >= 4 * used) {
    s.down_rows /= 2;
    groups = across * ((a.m + s.down_rows - 1) / s.down_rows);
  }
  // 16 wavefronts where a CU has one workgroup (one query, two of eight experts of 2816 x 1024: 6.4 us of GPU time, with eight
  // 8.0; but of 5632 x 2048, two workgroups a CU, a call 46.2 and with eight 44.0)
  s.down_waves = s.down_variant == kMoeFew && groups * s.splits <= 256 ? 16 : 8;
  const int64_t waves = s.splits * s.down_waves;
  // (an item a wavefront; where there are more experts than wavefronts, every workgroup has its part of each, since experts
  // have unlike numbers of rows: 64 rows, 4 of 32 of 5632 x 2048 432 us, an item an expert 436.5)
  const int64_t chunks = std::min(shortest, waves > used ? (waves + used - 1) / used : s.splits);
  s.chunk = static_cast<int32_t>(((a.f + chunks - 1) / chunks + down_step - 1) / down_step * down_step);
  if (s.down_variant == kMoeMany) {
    // (eight wavefronts share a reduction, or fewer where that leaves workgroups and steps enough: the 200 rows 493 with eight,
    // 478 with two; 256 rows, 2 of 16 of 1408 x 2048 128 and 130.  16 rows at a time, or 32 where there are as many: the 200
    // rows 478 with 16, 501 with 32; 100 rows, 2 of 9 of 1111 x 777 48.6 and 44.4)
    auto workgroups = [&](int64_t sharing) { return (a.d * sharing + 255) / 256 * a.experts; };
    s.down_waves = 8;
    auto fewer = [&] { return s.down_waves * 64 > a.f || (s.down_waves > 2 && workgroups(s.down_waves / 2) >= 512); };
    while (s.down_waves > 1 && fewer()) s.down_waves /= 2;
    s.down_blocks = uses > 14 * a.experts && a.dtype != EMB_DTYPE_F32 ? 2 : 1;
    const int64_t tile = 16 * s.down_blocks, tiles_each = (uses / a.experts + 16 + tile - 1) / tile;
    s.down_parts = static_cast<int32_t>(std::max<int64_t>(1, std::min(512 / workgroups(s.down_waves), tiles_each)));
    s.splits = 1;
  }
  return s;
}

extern "C" {

emb_status_t emb_quantize(const emb_quantize_t* a, void* stream) {
  if (!a || a->m < 0 || a->k < 1) return EMB_ERR_INVALID_ARGUMENT;
  if (a->m > kMaxSize || a->k > kMaxSize) return EMB_ERR_UNSUPPORTED;
  EMBX_TRY(check_type(a->dtype));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, esize(a->dtype)));
  EMBX_TRY(check_matrix(a->q, a->ldq, a->m, a->k, 1));
  EMBX_TRY(check_vector(a->scale, a->m, 4));
  if (a->m == 0) return EMB_OK;
  return run(quantize_launch(a->dtype, {a->x, a->q, a->scale, a->ldx, a->ldq, a->m, static_cast<int32_t>(a->k),
                                        static_cast<int32_t>(a->k), {}, 0}, stream));
}

emb_status_t emb_linear_int8_workspace(const emb_linear_int8_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(*a));
  Arena ar{nullptr};
  if (a->m > 0 && int8_space(ar, *a).choice.variant < 0) return EMB_ERR_UNSUPPORTED;
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_linear_int8(const emb_linear_int8_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(*a));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->x_scale ? 1 : esize(a->dtype)));
  EMBX_TRY(check_vector(a->x_scale, a->x_scale ? 1 : 0, 4));
  EMBX_TRY(check_matrix(a->weight, a->ldw, a->n, a->k, 1));
  EMBX_TRY(check_vector(a->w_scale, a->n, 4));
  EMBX_TRY(check_vector(a->bias, a->bias ? 1 : 0, esize(a->dtype)));
  if (a->residual) EMBX_TRY(check_matrix(a->residual, a->ldr, a->m, a->n, esize(a->dtype)));
  EMBX_TRY(check_matrix(a->y, a->ldy, a->m, a->n, esize(a->dtype)));
  if (a->m == 0) return EMB_OK;
  Arena ar{static_cast<char*>(workspace)};
  const Int8Space s = int8_space(ar, *a);
  if (s.choice.variant < 0) return EMB_ERR_UNSUPPORTED;
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  DensePack pack = {};
  if (s.packed_x) add_copy(pack, a->x, a->ldx, s.x, a->m, a->k);
  if (s.packed_w) add_copy(pack, a->weight, a->ldw, s.w, a->n, a->k);
  if (s.quantized)
    EMBX_TRY(run(quantize_launch(a->dtype, {a->x, const_cast<int8_t*>(s.x), const_cast<float*>(s.scale), a->ldx, s.ldx, a->m,
                                            static_cast<int32_t>(a->k), static_cast<int32_t>(s.ldx), pack, 0}, stream)));
  else if (pack.count)
    EMBX_TRY(run(dense_pack_launch(pack, stream)));
  DenseGemm g = {};
  g.a[0] = s.x, g.lda = s.ldx, g.panel_a = kPanel;
  g.b[0] = s.w, g.ldb[0] = s.ldw, g.panel_b[0] = kPanel;
  g.c[0] = a->y, g.ldc[0] = a->ldy;
  g.bias[0] = a->bias;
  g.res = a->residual, g.ldr = a->ldr;
  g.quantize = s.inside;
  g.scale_a = s.scale, g.scale_b = a->w_scale;
  g.result = a->dtype == EMB_DTYPE_F32 ? kDenseF32 : a->dtype == EMB_DTYPE_F16 ? kDenseF16 : kDenseBF16;
  g.ni = static_cast<int32_t>(a->m), g.nj = static_cast<int32_t>(a->n), g.nr = static_cast<int32_t>(a->k);
  g.act = a->activation, g.parts = 1, g.whole = s.align;
  g.variant = s.choice.variant, g.splits = g.slots = s.choice.splits, g.row_blocks = s.choice.row_blocks;
  g.row_columns = s.choice.row_columns;
  g.partial = s.partial;
  return run(dense_forward_i8(g, stream));
}

emb_status_t emb_moe_workspace(const emb_moe_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(*a));
  Arena ar{nullptr};
  if (a->m > 0) moe_space(ar, *a, moe_choose(*a));
  *bytes = ar.used;
  return EMB_OK;
}

emb_status_t emb_moe(const emb_moe_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(*a));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->d, esize(a->dtype)));
  EMBX_TRY(check_matrix(a->router, a->ldr, a->experts, a->d, esize(a->dtype)));
  EMBX_TRY(check_experts(a->gate, *a, a->f, a->d));
  EMBX_TRY(check_experts(a->up, *a, a->f, a->d));
  EMBX_TRY(check_experts(a->down, *a, a->d, a->f));
  EMBX_TRY(check_matrix(a->y, a->ldy, a->m, a->d, esize(a->dtype)));
  EMBX_TRY(check_vector(a->chosen, a->chosen ? 1 : 0, 4));
  EMBX_TRY(check_vector(a->share, a->share ? 1 : 0, 4));
  if (a->m == 0) return EMB_OK;
  Arena ar{static_cast<char*>(workspace)};
  const MoeChoice c = moe_choose(*a);
  const MoeSpace s = moe_space(ar, *a, c);
  EMBX_TRY(check_workspace(workspace, workspace_bytes, ar.used));
  Moe g = {};
  static_cast<MoeChoice&>(g) = c;
  g.x = a->x, g.ldx = a->ldx, g.router = a->router, g.ldr = a->ldr;
  int i = 0;
  for (const emb_experts_t* w : {&a->gate, &a->up, &a->down}) {
    g.w[i] = w->p, g.ldw[i] = w->ld, g.stride[i] = w->stride, g.scale[i] = w->scale;
    ++i;
  }
  g.h = s.h, g.ldh = s.ldh, g.chosen = s.chosen, g.share = s.share;
  g.partial = s.partial, g.logits = s.logits;
  const size_t size = esize(a->dtype);
  g.whole = aligned(a->x, a->ldx, size) && aligned(a->router, a->ldr, size) && aligned(a->gate, size) && aligned(a->up, size) &&
            aligned(a->down, size);
  g.y = a->y, g.ldy = a->ldy;
  g.m = static_cast<int32_t>(a->m), g.f = static_cast<int32_t>(a->f), g.d = static_cast<int32_t>(a->d);
  g.experts = a->experts, g.top_k = a->top_k, g.act = a->activation, g.renormalize = a->renormalize != 0;
  switch (a->dtype) {
    case EMB_DTYPE_F32: return run(moe_launch_f32(g, stream));
    case EMB_DTYPE_F16: return run(moe_launch_f16(g, stream));
    default: return run(moe_launch_bf16(g, stream));
  }
}

}  // extern "C"
