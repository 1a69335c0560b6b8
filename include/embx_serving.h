/*
 * embx_serving -- the dense layers' serving forms (embx_dense.h), on one AMD Instinct MI355X
 * (gfx950): layers whose operands are 8-bit integers with a scale for each row, and a layer
 * of experts of which every row of x takes a few.
 *
 *   quantize      s_i = max_k |x_ik| / 127, at least 2^-126;  q_ik = x_ik / s_i, rounded half
 *                 to even: whole numbers from -127 to 127
 *   linear_int8   y = act(xs_i ws_j sum_k xq_ik wq_jk + b_j) + r_ij
 *   moe           l = x R^T;  each row takes the top_k experts e of the largest l_e (ties: the
 *                 lowest e), with shares c_e = exp(l_e) / sum of exp(l), over the experts taken
 *                 (renormalize) or over all;
 *                 y = sum_e c_e (act(x Wg_e^T) * (x Wu_e^T)) Wd_e^T
 *
 * Matrices are row-major with a row stride (ld..) in elements, at least the row's length;
 * vectors are contiguous.  Types are emb_dtype_t's; 8-bit integers are signed.
 *
 * quantize: the scale is rounded to f32, and q is exact for that scale.  A row of zeros has
 * scale 2^-126.  A row with an infinity or NaN has scale NaN and zeros, so that what is
 * computed from it is NaN and not a number that looks right.
 *
 * linear_int8: sums of the products are exact; the scales (in an order in which no infinity
 * comes between), bias, activation and residual are applied in f32, and the result is rounded
 * once.  x is 8-bit integers with their scales
 * (x_scale), or, without x_scale, a matrix of the call's type whose rows the call quantizes
 * first, as emb_quantize does.  A scale may be any f32 value, NaN among them.
 *
 * moe: logits are summed in 64 bits, so which experts a row takes does not depend on the order
 * of the sums; NaN counts as the largest logit, and makes the row's shares and results NaN,
 * as does an infinite one that is the largest.  Sums are held in f32, and so are shares.
 * act(..) * (..) is f32 with every type, and goes into the product with Wd as it is, but for
 * 2^-23 of it, or 2^-36 of the largest of its row, where Wd is f16; the result is rounded once.
 * (An infinite element of Wd gives an infinity or NaN.)  The experts' matrices have the call's
 * type, or are 8-bit integers with a scale for each of their rows (all three or none).  A row's result
 * comes from that row and its experts only; in which order its sums are added up, and so
 * their last bits in f32, is up to the whole call.  It is made for few rows, where the layer
 * is bound by reading the experts' matrices; any number is right.
 *
 * Calls take plain device pointers of the current HIP device, aligned to their element; the
 * structs are host memory, read during the call.  No call allocates or synchronizes; each
 * enqueues its kernels on `stream` (a hipStream_t as void*, NULL = null stream) and returns.
 * A call's outputs and workspace must not overlap its inputs, except that linear_int8's y may
 * be the residual itself (same pointer and row stride).  Calls that share a workspace must
 * not overlap in time.  Nothing is kept between calls, and equal calls give equal bits.
 * The aligned 16 bytes, or 4, that hold a row's start or end may be read whole, and of 8-bit
 * matrices what lies between two rows; what that holds does not matter.
 *
 * Errors (emb_status_t of embx.h): EMB_ERR_INVALID_ARGUMENT for a NULL or misaligned pointer,
 * a size below its least (m >= 0, the others >= 1), a row stride below its row, top_k above
 * experts, an unknown activation, scales of some of the experts' matrices only, or a workspace
 * that is NULL or too small; EMB_ERR_UNSUPPORTED for an unknown type, m or n above 2^30,
 * a stride above 2^40, linear_int8's k above 131071 (its sums have to fit 32 bits) and
 * quantize's above 2^30, experts above 1024, top_k above 32, moe's m above 65536, its f, d or
 * experts' row strides above 2^25, or a product too large for a launch; EMB_ERR_DEVICE if a
 * launch fails.  With m == 0 calls do nothing.
 */
#ifndef EMBX_SERVING_H
#define EMBX_SERVING_H

#include <stddef.h>
#include <stdint.h>

#include "embx.h"
#include "embx_dense.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int64_t m, k;
  int32_t dtype;                     /* emb_dtype_t of x */
  const void* x; int64_t ldx;        /* [m, k] */
  int8_t* q; int64_t ldq;            /* [m, k] */
  float* scale;                      /* [m] */
} emb_quantize_t;

typedef struct {
  int64_t m, n, k;
  int32_t dtype;                     /* emb_dtype_t of bias, residual, y, and of x without x_scale */
  int32_t activation;                /* emb_activation_t */
  const void* x; int64_t ldx;        /* [m, k]: int8_t with x_scale, else of the call's type */
  const float* x_scale;              /* [m], or NULL */
  const int8_t* weight; int64_t ldw; /* [n, k] */
  const float* w_scale;              /* [n] */
  const void* bias;                  /* [n], or NULL */
  const void* residual; int64_t ldr; /* [m, n], or NULL */
  void* y; int64_t ldy;              /* [m, n] */
} emb_linear_int8_t;

/* matrices of all experts: [experts][rows][cols], `stride` elements from one expert's to the next's */
typedef struct {
  const void* p; int64_t ld, stride;
  const float* scale;                /* [experts][rows]: p holds int8_t; or NULL: the call's type */
} emb_experts_t;

typedef struct {
  int64_t m, f, d;
  int32_t experts, top_k;
  int32_t dtype;                     /* emb_dtype_t */
  int32_t activation;                /* emb_activation_t */
  int32_t renormalize;               /* shares of a row's experts add up to one */
  const void* x; int64_t ldx;        /* [m, d] */
  const void* router; int64_t ldr;   /* [experts, d] */
  emb_experts_t gate, up;            /* [experts][f][d] */
  emb_experts_t down;                /* [experts][d][f] */
  void* y; int64_t ldy;              /* [m, d] */
  int32_t* chosen;                   /* [m, top_k]: the experts taken, the largest first; or NULL */
  float* share;                      /* [m, top_k]: their shares; or NULL */
} emb_moe_t;

/* Device bytes of workspace that a call with this struct needs (0: none); from its sizes and
 * types, which optional pointers are NULL, and the alignment of pointers and row strides
 * modulo 16 bytes.  256-byte aligned; its contents mean nothing before or after. */
emb_status_t emb_linear_int8_workspace(const emb_linear_int8_t* a, size_t* bytes);
emb_status_t emb_moe_workspace(const emb_moe_t* a, size_t* bytes);

emb_status_t emb_quantize(const emb_quantize_t* a, void* stream);
emb_status_t emb_linear_int8(const emb_linear_int8_t* a, void* workspace, size_t workspace_bytes, void* stream);
emb_status_t emb_moe(const emb_moe_t* a, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EMBX_SERVING_H */
