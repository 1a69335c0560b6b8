// What the dense layers' entry points (dense_api.cpp) and kernels (dense.hip) share.
#ifndef EMBX_DENSE_HPP
#define EMBX_DENSE_HPP

#include <cstddef>
#include <cstdint>

namespace embx {

enum DenseType { kDenseF32 = 0, kDenseF16 = 1, kDenseBF16 = 2 };

// The three products of a layer.  A matrix is "reduction-major" (R) where consecutive
// elements in memory step along the outputs, and "along the reduction" (K) otherwise.
enum DenseKind {
  kForward = 0,      // C[i][j] = sum_r A[i][r] B[j][r]   A = x, B = W        (K, K)
  kGated = 1,        // the same with two B's, joined by the gate
  kInputGrad = 2,    // C[i][j] = sum_r A[i][r] B[r][j]   A = dz, B = W       (K, R)
  kWeightGrad = 3    // C[i][j] = sum_r A[r][i] B[r][j]   A = dz, B = x       (R, R)
};

enum DenseVariant { kTile128 = 0, kTile256 = 1, kTile128Halves = 2, kRows = 3, kShort = 4 };

// Offsets within a tile of an operand have 32 bits: rows further apart than kMostStride bytes are copied first.  Where the
// rows of a copy, or of dz, are so long that a tile's would still reach too far, it is in panels of kPanel columns, each a
// matrix of its own; a product whose reduction runs along such rows takes a launch for each panel, which leave partial
// sums.  Columns of a matrix that is not in panels lie as if panels were kPanel elements apart.
constexpr int kPanelLog = 19;
constexpr int64_t kPanel = int64_t(1) << kPanelLog;
constexpr int64_t kMostStride = int64_t(1) << 23;   // 256 rows, and 256 elements of the last, stay below 2^31 bytes
constexpr int64_t kMostOffset = (int64_t(1) << 31) - (1 << 20);   // bytes to a tile's last row

constexpr int kXcds = 8;

// One matrix product.  Arrays of two: kGated's two weights and results; kInputGrad's two
// products summed into one result (parts = 2); kWeightGrad's two results (parts = 2).
struct DenseGemm {
  const void* a[2];
  const void* b[2];
  void* c[2];
  void* z[2];              // forward kinds: sums before the activation, or NULL
  const void* bias[2];     // forward kinds, or NULL
  const void* res;         // kForward, or NULL
  float* partial;          // [parts of the result][slots][ni][nj], with slots > 1
  int64_t lda, ldb[2], ldc[2], ldz[2], ldr;
  int32_t ni, nj, nr;      // C is [ni][nj], the sum over nr (in each part)
  int32_t parts, splits, act;   // parts = 0: no product
  int32_t variant;         // DenseVariant
  int32_t row_blocks;      // kRows: 16 rows each, of a workgroup: 1, 2 or 4
  int32_t row_chunks, short_waves;   // kShort: chunks of 64 rows of a workgroup, its wavefronts along columns
  int32_t whole;           // kRows, kShort: operands' rows start at multiples of 16 bytes and hold whole chunks
  int32_t slots, first;    // tiles: partial sums, the splits of all launches, and the first one of this
  int64_t panel_a, panel_b[2];   // tiles: elements from a panel of columns to the next
};

// matrices copied to rows of whole 16-byte chunks, in panels
struct DensePack {
  const void* src[3];
  void* dst[3];
  int64_t lds[3], ldd[3], panel[3];
  uint32_t rows[3], cols[3], wide[3];
  int32_t count, groups, esize;
};

// dz = dy * act'(z), or dg, du; and column sums of them
struct DenseSlope {
  const void* dy;
  const void* z[2];        // z, or g and u; NULL z[0]: dz = dy (only column sums)
  void* dz[2];             // NULL: not written
  float* colsum[2];        // [row blocks][n], or NULL: not wanted, or
  void* total[2];          // [n], with one block of rows: the finished sums; or NULL
  int64_t lddy, ldz[2], lddz, dz_panel;
  int32_t m, n, act, gated, row_blocks;
  int32_t log_x;           // log2 of the eights of columns of a workgroup
  int32_t whole;           // rows of all operands start at multiples of 16 bytes and hold whole eights
  DensePack pack;          // matrices that the same launch copies
};

// workgroups of the last launch of a backward pass: of the column sums, and of the join of one of w's results
struct DenseTail {
  uint32_t colsum_groups, w_groups;
};

// column sums from those of blocks of rows
struct DenseColsum {
  const float* partial[2];   // [blocks][n], or NULL
  void* out[2];
  int32_t blocks, n;
};

int dense_pack_launch(const DensePack& p, void* stream);

// launches of the kernels of one type (dense.hip is compiled once per type); 0 or a hipError_t
#define EMBX_DENSE_DECLARE(NAME)                                                        \
  int dense_forward_##NAME(int kind, const DenseGemm& g, void* stream);                 \
  int dense_grads_##NAME(const DenseGemm& w, const DenseGemm& x, int variant, void* stream); \
  int dense_tail_##NAME(const DenseGemm& w, const DenseGemm& x, const DenseColsum& c, void* stream); \
  int dense_slope_##NAME(const DenseSlope& s, void* stream);
EMBX_DENSE_DECLARE(f32)
EMBX_DENSE_DECLARE(f16)
EMBX_DENSE_DECLARE(bf16)
#undef EMBX_DENSE_DECLARE

}  // namespace embx
#endif
