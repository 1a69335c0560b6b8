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

// (a tile's offsets, 256 rows at most, are 32-bit)
bool whole(const void* p, int64_t ld) { return !misaligned(p, 16) && ld % 8 == 0 && ld <= (int64_t(1) << 22); }

// Whether rows of every operand and result start at multiples of 16 bytes and hold whole chunks of
// eight elements (16-bit types).
bool aligned16(int kind, const DenseGemm& g) {
  const int parts = g.parts;
  bool ok = g.nj % 8 == 0;
  for (int p = 0; p < (kind == kGated ? 1 : parts); ++p) ok = ok && whole(g.a[p], g.lda);
  for (int p = 0; p < (kind == kGated ? 2 : parts); ++p) ok = ok && whole(g.b[p], g.ldb[p]);
  // along the reduction: whole chunks of it; reduction-major: whole chunks of results
  if (kind != kWeightGrad) ok = ok && g.nr % 8 == 0;
  if (kind == kWeightGrad) ok = ok && g.ni % 8 == 0;
  return ok;
}

bool aligned_results(int kind, const DenseGemm& g) {
  bool ok = g.nj % 8 == 0;
  for (int p = 0; p < (kind == kWeightGrad ? g.parts : 1); ++p) ok = ok && whole(g.c[p], g.ldc[p]);
  for (int p = 0; p < 2; ++p) {
    if (g.z[p]) ok = ok && whole(g.z[p], g.ldz[p]);
    if (g.bias[p]) ok = ok && !misaligned(g.bias[p], 16);
  }
  if (g.res) ok = ok && whole(g.res, g.ldr);
  return ok;
}

// Which tile a product takes and over how many workgroups its reduction is split.
struct Choice { int32_t variant, splits; };

constexpr int kCus = 256;
constexpr int kStep = 64;   // of the reduction

// Microseconds of a product by tiles of 256 x 256 or 128 x 128 over `steps` steps, split s ways.  Measured on bf16
// products of 256 to 8192 rows: a step of the large tile takes 0.97 us on a GPU that is otherwise idle and 1.50 us
// with a workgroup on every CU (the clock drops, and L2 is shared); one of the small tile 0.62 us alone on its CU, 1.03
// us where two share it.  A round starts and ends in 3 us.  Split products write their sums and read them back.
double tile_us(int variant, double tiles, int steps, int s, double result_bytes) {
  const double groups = tiles * s, each = (steps + s - 1) / s;
  double us;
  if (variant == kTile256) {
    const double rounds = std::ceil(groups / kCus);
    us = rounds * (each * (0.97 + 0.53 * std::min(1.0, groups / kCus)) + 3.0);
  } else {
    const double whole = std::floor(groups / (2 * kCus)), rest = groups - whole * 2 * kCus;
    us = whole * (each * 1.03 + 3.0);
    if (rest > 0) us += each * (rest <= kCus ? 0.62 + 0.1 * rest / kCus : 1.03) + 3.0;
  }
  if (s > 1) us += 3.0 + result_bytes * s / 2.0e6;
  return us;
}

Choice choose(int kind, int64_t ni, int64_t nj, int64_t nr, int parts, bool large_tiles) {
  const int64_t steps = (nr + kStep - 1) / kStep * (kind == kInputGrad ? parts : 1);
  const int results = kind == kWeightGrad ? parts : kind == kGated ? 2 : 1;
  const double result_bytes = 4.0 * ni * nj * results;
  Choice best = {kTile128, 1};
  double least = 0.0;
  for (int variant = kTile256; variant >= kTile128; --variant) {
    if (variant == kTile256 && !large_tiles) continue;
    const int64_t side = variant == kTile256 ? 256 : 128;
    const double tiles = double((ni + side - 1) / side) * ((nj * (kind == kGated ? 2 : 1) + side - 1) / side) *
                         (kind == kWeightGrad ? parts : 1);
    for (int s = 1; s <= 128 && (s == 1 || (s * 4 <= steps && result_bytes * s <= (256 << 20))); ++s) {
      const double us = tile_us(variant, tiles, static_cast<int>(std::min<int64_t>(steps, 1 << 30)), s, result_bytes);
      if (least == 0.0 || us < 0.98 * least) least = us, best = {variant, s};
    }
  }
  return best;
}

// Bytes of partial sums of a product, whatever its operands' alignment.
size_t partial_bytes(int32_t dtype, int kind, int64_t ni, int64_t nj, int64_t nr, int parts) {
  if (dtype == EMB_DTYPE_F32) return 0;
  const int results = kind == kWeightGrad ? parts : kind == kGated ? 2 : 1;
  size_t most = 0;
  for (bool large : {false, true}) {
    const int s = choose(kind, ni, nj, nr, parts, large).splits;
    if (s > 1) most = std::max(most, size_t(s) * ni * nj * results * 4);
  }
  return most;
}

emb_status_t gemm(int32_t dtype, int kind, const DenseGemm& given, float* partial, void* stream) {
  DenseGemm g = given;
  g.splits = 1;
  g.partial = partial;
  if (dtype != EMB_DTYPE_F32) {
    g.aligned = aligned16(kind, g);
    g.vec = aligned_results(kind, g);
    const Choice c = choose(kind, g.ni, g.nj, g.nr, g.parts, g.aligned);
    g.variant = c.variant, g.splits = c.splits;
  }
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_gemm_f32(kind, g, stream));
    case EMB_DTYPE_F16: return run(dense_gemm_f16(kind, g, stream));
    default: return run(dense_gemm_bf16(kind, g, stream));
  }
}

emb_status_t slope(int32_t dtype, const DenseSlope& s, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_slope_f32(s, stream));
    case EMB_DTYPE_F16: return run(dense_slope_f16(s, stream));
    default: return run(dense_slope_bf16(s, stream));
  }
}

emb_status_t colsum(int32_t dtype, const float* p, int32_t blocks, int64_t n, void* out, void* stream) {
  switch (dtype) {
    case EMB_DTYPE_F32: return run(dense_colsum_f32(p, blocks, n, out, stream));
    case EMB_DTYPE_F16: return run(dense_colsum_f16(p, blocks, n, out, stream));
    default: return run(dense_colsum_bf16(p, blocks, n, out, stream));
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

// blocks of rows of the column sums
int32_t slope_blocks(int64_t m) { return static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(256, m / 16))); }

struct GradSpace {
  void* dz[2] = {nullptr, nullptr};
  float* colsum[2] = {nullptr, nullptr};
  float* partial = nullptr;   // of one product after the other
  int64_t lddz = 0;
  int32_t blocks = 1;
};

// dz of `mats` results, and partial column sums, as wanted
GradSpace grad_space(Arena& ar, int64_t m, int64_t n, int32_t dtype, int mats, bool dz, const bool* sums) {
  GradSpace g;
  g.lddz = (n + 63) / 64 * 64;
  g.blocks = slope_blocks(m);
  for (int i = 0; i < mats; ++i)
    if (dz) g.dz[i] = ar.take<void>(m * g.lddz * esize(dtype));
  for (int i = 0; i < mats; ++i)
    if (sums[i]) g.colsum[i] = ar.take<float>(size_t(g.blocks) * n * 4);
  return g;
}

GradSpace linear_grad_space(Arena& ar, const emb_linear_grad_t& a) {
  const bool sums[2] = {a.dbias != nullptr, false};
  GradSpace g = grad_space(ar, a.m, a.n, a.dtype, 1, a.activation != EMB_ACT_NONE && (a.dx || a.dweight), sums);
  g.partial = ar.take<float>(std::max(a.dx ? partial_bytes(a.dtype, kInputGrad, a.m, a.k, a.n, 1) : 0,
                                      a.dweight ? partial_bytes(a.dtype, kWeightGrad, a.n, a.k, a.m, 1) : 0));
  return g;
}

GradSpace gated_grad_space(Arena& ar, const emb_gated_grad_t& a) {
  const bool sums[2] = {a.db_gate != nullptr, a.db_up != nullptr};
  GradSpace g = grad_space(ar, a.m, a.n, a.dtype, 2, a.dx || a.dw_gate || a.dw_up, sums);
  const int weights = (a.dw_gate != nullptr) + (a.dw_up != nullptr);
  g.partial = ar.take<float>(std::max(a.dx ? partial_bytes(a.dtype, kInputGrad, a.m, a.k, a.n, 2) : 0,
                                      weights ? partial_bytes(a.dtype, kWeightGrad, a.n, a.k, a.m, weights) : 0));
  return g;
}

}  // namespace

extern "C" {

emb_status_t emb_linear_workspace(const emb_linear_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  *bytes = partial_bytes(a->dtype, kForward, a->m, a->n, a->k, 1);
  return EMB_OK;
}

emb_status_t emb_linear(const emb_linear_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  EMBX_TRY(emb_linear_workspace(a, &need));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->weight, a->ldw, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->bias, a->dtype));
  EMBX_TRY(check_optional(a->residual, a->ldr, a->m, a->n, a->dtype));
  EMBX_TRY(check_matrix(a->y, a->ldy, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->z, a->ldz, a->m, a->n, a->dtype));
  EMBX_TRY(check_workspace(workspace, workspace_bytes, need));
  if (a->m == 0) return EMB_OK;
  DenseGemm g = {};
  g.a[0] = a->x, g.lda = a->ldx;
  g.b[0] = a->weight, g.ldb[0] = a->ldw;
  g.c[0] = a->y, g.ldc[0] = a->ldy;
  g.z[0] = a->z, g.ldz[0] = a->ldz;
  g.bias[0] = a->bias;
  g.res = a->residual, g.ldr = a->ldr;
  g.ni = a->m, g.nj = a->n, g.nr = a->k;
  g.parts = 1, g.splits = 1, g.act = a->activation;
  return gemm(a->dtype, kForward, g, static_cast<float*>(workspace), stream);
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
  size_t need = 0;
  EMBX_TRY(emb_linear_backward_workspace(a, &need));
  const bool slopes = a->activation != EMB_ACT_NONE;
  EMBX_TRY(check_matrix(a->dy, a->lddy, a->m, a->n, a->dtype));
  if (slopes) EMBX_TRY(check_matrix(a->z, a->ldz, a->m, a->n, a->dtype));
  if (a->dweight) EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  if (a->dx) EMBX_TRY(check_matrix(a->weight, a->ldw, a->n, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dx, a->lddx, a->m, a->k, a->dtype));
  EMBX_TRY(check_optional(a->dweight, a->lddw, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->dbias, a->dtype));
  EMBX_TRY(check_workspace(workspace, workspace_bytes, need));
  Arena ar{static_cast<char*>(workspace)};
  const GradSpace sp = linear_grad_space(ar, *a);
  const bool dz = sp.dz[0] != nullptr;
  if (a->dbias || (dz && a->m > 0)) {
    DenseSlope s = {};
    s.dy = a->dy, s.lddy = a->lddy;
    s.z[0] = slopes ? a->z : nullptr, s.ldz[0] = a->ldz;
    s.dz[0] = sp.dz[0], s.lddz = sp.lddz;
    s.colsum[0] = sp.colsum[0];
    s.m = a->m, s.n = a->n, s.act = a->activation, s.gated = 0, s.row_blocks = sp.blocks;
    EMBX_TRY(slope(a->dtype, s, stream));
    if (a->dbias) EMBX_TRY(colsum(a->dtype, sp.colsum[0], sp.blocks, a->n, a->dbias, stream));
  }
  DenseGemm g = {};
  g.a[0] = dz ? sp.dz[0] : a->dy, g.lda = dz ? sp.lddz : a->lddy;
  g.parts = 1, g.splits = 1;
  if (a->dx && a->m > 0) {
    g.b[0] = a->weight, g.ldb[0] = a->ldw;
    g.c[0] = a->dx, g.ldc[0] = a->lddx;
    g.ni = a->m, g.nj = a->k, g.nr = a->n;
    EMBX_TRY(gemm(a->dtype, kInputGrad, g, sp.partial, stream));
  }
  if (a->dweight) {
    g.b[0] = a->x, g.ldb[0] = a->ldx;
    g.c[0] = a->dweight, g.ldc[0] = a->lddw;
    g.ni = a->n, g.nj = a->k, g.nr = a->m;
    EMBX_TRY(gemm(a->dtype, kWeightGrad, g, sp.partial, stream));
  }
  return EMB_OK;
}

emb_status_t emb_gated_workspace(const emb_gated_t* a, size_t* bytes) {
  if (!a || !bytes) return EMB_ERR_INVALID_ARGUMENT;
  EMBX_TRY(check_shape(a->m, a->n, a->k, a->dtype, a->activation));
  *bytes = partial_bytes(a->dtype, kGated, a->m, a->n, a->k, 1);
  return EMB_OK;
}

emb_status_t emb_gated(const emb_gated_t* a, void* workspace, size_t workspace_bytes, void* stream) {
  size_t need = 0;
  EMBX_TRY(emb_gated_workspace(a, &need));
  EMBX_TRY(check_matrix(a->x, a->ldx, a->m, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->w_gate, a->ld_gate, a->n, a->k, a->dtype));
  EMBX_TRY(check_matrix(a->w_up, a->ld_up, a->n, a->k, a->dtype));
  EMBX_TRY(check_vector(a->b_gate, a->dtype));
  EMBX_TRY(check_vector(a->b_up, a->dtype));
  EMBX_TRY(check_matrix(a->h, a->ldh, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->g, a->ldg, a->m, a->n, a->dtype));
  EMBX_TRY(check_optional(a->u, a->ldu, a->m, a->n, a->dtype));
  EMBX_TRY(check_workspace(workspace, workspace_bytes, need));
  if (a->m == 0) return EMB_OK;
  DenseGemm g = {};
  g.a[0] = a->x, g.lda = a->ldx;
  g.b[0] = a->w_gate, g.ldb[0] = a->ld_gate;
  g.b[1] = a->w_up, g.ldb[1] = a->ld_up;
  g.c[0] = a->h, g.ldc[0] = a->ldh;
  g.z[0] = a->g, g.ldz[0] = a->ldg;
  g.z[1] = a->u, g.ldz[1] = a->ldu;
  g.bias[0] = a->b_gate, g.bias[1] = a->b_up;
  g.ni = a->m, g.nj = a->n, g.nr = a->k;
  g.parts = 1, g.splits = 1, g.act = a->activation;
  return gemm(a->dtype, kGated, g, static_cast<float*>(workspace), stream);
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
  size_t need = 0;
  EMBX_TRY(emb_gated_backward_workspace(a, &need));
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
  EMBX_TRY(check_workspace(workspace, workspace_bytes, need));
  Arena ar{static_cast<char*>(workspace)};
  const GradSpace sp = gated_grad_space(ar, *a);
  const bool sums = a->db_gate || a->db_up;
  if (sums || (sp.dz[0] && a->m > 0)) {
    DenseSlope s = {};
    s.dy = a->dh, s.lddy = a->lddh;
    s.z[0] = a->g, s.ldz[0] = a->ldg;
    s.z[1] = a->u, s.ldz[1] = a->ldu;
    s.dz[0] = sp.dz[0], s.dz[1] = sp.dz[1], s.lddz = sp.lddz;
    s.colsum[0] = sp.colsum[0], s.colsum[1] = sp.colsum[1];
    s.m = a->m, s.n = a->n, s.act = a->activation, s.gated = 1, s.row_blocks = sp.blocks;
    EMBX_TRY(slope(a->dtype, s, stream));
    if (a->db_gate) EMBX_TRY(colsum(a->dtype, sp.colsum[0], sp.blocks, a->n, a->db_gate, stream));
    if (a->db_up) EMBX_TRY(colsum(a->dtype, sp.colsum[1], sp.blocks, a->n, a->db_up, stream));
  }
  DenseGemm g = {};
  g.lda = sp.lddz;
  g.splits = 1;
  if (a->dx && a->m > 0) {
    g.a[0] = sp.dz[0], g.a[1] = sp.dz[1];
    g.b[0] = a->w_gate, g.ldb[0] = a->ld_gate;
    g.b[1] = a->w_up, g.ldb[1] = a->ld_up;
    g.c[0] = a->dx, g.ldc[0] = a->lddx;
    g.ni = a->m, g.nj = a->k, g.nr = a->n, g.parts = 2;
    EMBX_TRY(gemm(a->dtype, kInputGrad, g, sp.partial, stream));
  }
  if (weights) {
    g.parts = 0;
    for (int i = 0; i < 2; ++i) {
      void* dw = i == 0 ? a->dw_gate : a->dw_up;
      if (!dw) continue;
      g.a[g.parts] = sp.dz[i];
      g.c[g.parts] = dw, g.ldc[g.parts] = i == 0 ? a->ldd_gate : a->ldd_up;
      ++g.parts;
    }
    g.b[0] = g.b[1] = a->x, g.ldb[0] = g.ldb[1] = a->ldx;
    g.ni = a->n, g.nj = a->k, g.nr = a->m;
    EMBX_TRY(gemm(a->dtype, kWeightGrad, g, sp.partial, stream));
  }
  return EMB_OK;
}

}  // extern "C"
