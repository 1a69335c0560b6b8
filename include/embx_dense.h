/*
 * embx_dense -- the dense layers behind the pooled rows: a fully connected layer (matrix
 * product with bias, activation and residual in its epilogue) and a gated feed-forward
 * block (both projections, the activation and the product in one kernel), each with its
 * backward pass, on one AMD Instinct MI355X (gfx950).
 *
 *   linear            z = x W^T + b;  y = act(z) + r
 *   linear backward   dz = dy * act'(z);  dx = dz W;  dW = dz^T x;  db = column sums of dz
 *   gated             g = x Wg^T + bg;  u = x Wu^T + bu;  h = act(g) * u
 *   gated backward    dg = dh * u * act'(g);  du = dh * act(g);  dx = dg Wg + du Wu;
 *                     dWg = dg^T x;  dWu = du^T x;  dbg, dbu = column sums of dg, du
 *
 * (The residual's gradient is dy itself.)  x is [m, k], W [n, k], y, z, r, dy, g, u, h and
 * dh [m, n]; all matrices are row-major with a row stride (ld..) in elements, at least the
 * row's length; vectors are contiguous.  Every operand of a call has the call's type.  Sums
 * are held in fp32 whatever the type; each result is rounded once, to the call's type,
 * except that dz, dg and du are rounded to it before the products that read them, as the
 * matrix cores take them: 16-bit gradients are then 1.4 times as far from the exact ones as
 * their own rounding makes them (more for a few values), and in fp16 a dz beyond 65504 is an
 * infinity and one below 2^-14 loses bits.  Where that matters, give the call's operands in
 * fp32, whose dz is not rounded.  Biases' gradients are summed from the values before
 * rounding, and without an activation, or with relu, dz is exact.  Large products of fp32 operands go through
 * the matrix cores as three bf16 parts of each value, which hold all 24 bits of every normal
 * number: a product is off by less than 2^-22 of itself.  Where sums leave the range of that
 * (beyond 2^80, about), or operands are infinite or NaN, the products are formed in fp32
 * instead: the same results, five times slower for the tile of up to 256 rows and columns
 * that has them.
 * Results do not depend on timing: equal calls give equal bits.
 *
 * Calls take plain device pointers of the current HIP device, aligned to their element
 * (rows that start at multiples of 16 bytes are read fastest); the structs themselves are
 * host memory, read during the call.  No call allocates or synchronizes; each enqueues its
 * kernels on `stream` (a hipStream_t as void*, NULL = null stream) and returns.  A call's
 * outputs and workspace must not overlap its inputs, except that y may be the residual
 * itself (same pointer and row stride).  Calls that share a workspace must not overlap in
 * time.  Nothing is kept between calls.
 *
 * Errors (emb_status_t of embx.h): EMB_ERR_INVALID_ARGUMENT for a NULL or misaligned
 * pointer, a size below its least (m >= 0, n >= 1, k >= 1), a row stride below its row, an
 * unknown activation or a workspace that is NULL or too small; EMB_ERR_UNSUPPORTED for an
 * unknown type, m, n or k above 2^30 or a row stride above 2^40; EMB_ERR_DEVICE if a launch
 * fails.  With m == 0 the forward calls do nothing and the backward calls write zeros to
 * the gradients of weights and biases; pointers to matrices of no rows may then be NULL.
 */
#ifndef EMBX_DENSE_H
#define EMBX_DENSE_H

#include <stddef.h>
#include <stdint.h>

#include "embx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations.  gelu is z times the normal distribution function (by erf, no tanh form).
 * relu passes NaN on, and its slope at 0 is 0.  The gradient is taken at the z (or g) that
 * is given, thus at the rounded one that the forward call has saved. */
typedef enum {
  EMB_ACT_NONE = 0,
  EMB_ACT_RELU = 1,
  EMB_ACT_SIGMOID = 2,
  EMB_ACT_SILU = 3,
  EMB_ACT_GELU = 4
} emb_activation_t;

typedef struct {
  int64_t m, n, k;
  int32_t dtype;                     /* emb_dtype_t */
  int32_t activation;                /* emb_activation_t */
  const void* x; int64_t ldx;        /* [m, k] */
  const void* weight; int64_t ldw;   /* [n, k] */
  const void* bias;                  /* [n], or NULL */
  const void* residual; int64_t ldr; /* [m, n], or NULL */
  void* y; int64_t ldy;              /* [m, n] */
  void* z; int64_t ldz;              /* [m, n]: the sums before the activation, or NULL */
} emb_linear_t;

typedef struct {
  int64_t m, n, k;
  int32_t dtype, activation;
  const void* dy; int64_t lddy;      /* [m, n] */
  const void* x; int64_t ldx;        /* [m, k] */
  const void* weight; int64_t ldw;   /* [n, k] */
  const void* z; int64_t ldz;        /* [m, n] as emb_linear has saved it; not read with EMB_ACT_NONE */
  void* dx; int64_t lddx;            /* [m, k], or NULL: not wanted */
  void* dweight; int64_t lddw;       /* [n, k], or NULL */
  void* dbias;                       /* [n], or NULL */
} emb_linear_grad_t;

typedef struct {
  int64_t m, n, k;
  int32_t dtype, activation;
  const void* x; int64_t ldx;           /* [m, k] */
  const void* w_gate; int64_t ld_gate;  /* [n, k] */
  const void* w_up; int64_t ld_up;      /* [n, k] */
  const void* b_gate;                   /* [n], or NULL */
  const void* b_up;                     /* [n], or NULL */
  void* h; int64_t ldh;                 /* [m, n] */
  void* g; int64_t ldg;                 /* [m, n]: kept for the backward call, or NULL */
  void* u; int64_t ldu;                 /* [m, n], or NULL */
} emb_gated_t;

typedef struct {
  int64_t m, n, k;
  int32_t dtype, activation;
  const void* dh; int64_t lddh;         /* [m, n] */
  const void* x; int64_t ldx;           /* [m, k] */
  const void* w_gate; int64_t ld_gate;  /* [n, k] */
  const void* w_up; int64_t ld_up;      /* [n, k] */
  const void* g; int64_t ldg;           /* [m, n] as emb_gated has kept them */
  const void* u; int64_t ldu;           /* [m, n] */
  void* dx; int64_t lddx;               /* [m, k], or NULL: not wanted */
  void* dw_gate; int64_t ldd_gate;      /* [n, k], or NULL */
  void* dw_up; int64_t ldd_up;          /* [n, k], or NULL */
  void* db_gate;                        /* [n], or NULL */
  void* db_up;                          /* [n], or NULL */
} emb_gated_grad_t;

/* Device bytes of workspace that a call with this struct needs (0: none).  They follow from
 * its sizes, types and wanted gradients and from the alignment of its pointers and row
 * strides modulo 16 bytes; nothing is read through a pointer, and no device is touched.  The
 * workspace holds partial sums of a product whose long axis is split over the GPU, dz (dg,
 * du), and copies of matrices whose rows do not start at multiples of 16 bytes, do not hold
 * whole multiples of 16 bytes or start more than 2^23 bytes apart.  256-byte aligned; its
 * contents mean nothing before or after. */
emb_status_t emb_linear_workspace(const emb_linear_t* a, size_t* bytes);
emb_status_t emb_linear_backward_workspace(const emb_linear_grad_t* a, size_t* bytes);
emb_status_t emb_gated_workspace(const emb_gated_t* a, size_t* bytes);
emb_status_t emb_gated_backward_workspace(const emb_gated_grad_t* a, size_t* bytes);

emb_status_t emb_linear(const emb_linear_t* a, void* workspace, size_t workspace_bytes, void* stream);
emb_status_t emb_linear_backward(const emb_linear_grad_t* a, void* workspace, size_t workspace_bytes, void* stream);
emb_status_t emb_gated(const emb_gated_t* a, void* workspace, size_t workspace_bytes, void* stream);
emb_status_t emb_gated_backward(const emb_gated_grad_t* a, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* EMBX_DENSE_H */
