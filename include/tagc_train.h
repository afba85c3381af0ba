/*
 * libtagc -- the two ends of a data-parallel step that the exchange (tagc.h) lies between, for
 * AMD MI355X (gfx950): the linear layers whose weight gradients fill a bucket, and the
 * optimizer that takes the summed gradient.
 *
 *   tagc_linear_forward     y = act(x w^T + b) + r
 *   tagc_linear_backward    dx, and dw and db written into (or added to) the bucket's gradient
 *   tagc_grad_norm          2-norm over all gradients, clip factor, step count, on the device
 *   tagc_adamw_step         AdamW over many tensors in one launch, moments in 32 bits or in 8
 *   tagc_adamw_unpack       what 8-bit moments stand for
 *
 * The conventions are those of tagc.h: error codes, caller-owned device memory, nothing
 * allocated, nothing synchronised, all work enqueued in order on `stream`, argument errors
 * reported before anything is enqueued.  Every entry point but tagc_optim_upload may be
 * captured in a HIP graph.
 */
#ifndef TAGC_TRAIN_H
#define TAGC_TRAIN_H

#include <stdint.h>

#include "tagc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ optimizer */

#define TAGC_MOMENT_BLOCK 256u /* neighbours of a tensor whose 8-bit moments share a base */
#define TAGC_MAX_GROUPS 16u

/*
 * One tensor (all pointers dev, each aligned to its element).  A tensor with length 0 needs none.
 * What is written (param, m, v, bases, copy) must share no element with anything else of the plan, but for the
 * tensor's own gradient where that lies in the same place with the same bytes to an element.
 * Gradients may be what a layer's backward pass left (a segment of the flat gradient), or the
 * decoder's dense output from the segment's c-offset on (TAGC_F32).
 */
typedef struct tagc_tensor {
    void *param;       /* [length] param_type, updated in place; NULL in a plan that is only
                          asked for the norm (then in all tensors)                        */
    const void *grad;  /* [length] grad_type                                            */
    void *m, *v;       /* [length] first and second moment: float32, or 8-bit codes     */
    uint32_t *bases;   /* [ceil(length / TAGC_MOMENT_BLOCK)] 8-bit moments only: per block the
                          base of m in the low 16 bits, that of v in the high 16        */
    void *copy;        /* [length] bfloat16 copy of the updated parameter, or NULL      */
    uint64_t length;   /* < 2^34                                                        */
    uint32_t param_type, grad_type; /* TAGC_F32 | TAGC_BF16                             */
    uint32_t group;    /* which of tagc_adamw_step's groups, < TAGC_MAX_GROUPS          */
    uint32_t reserved; /* must be 0                                                     */
} tagc_tensor;

typedef struct tagc_optim_config {
    double beta1, beta2; /* in [0, 1)                                                   */
    double eps;          /* >= 0                                                        */
    double grad_scale;   /* the gradients times this are what is meant (1 / ranks for a
                            mean); finite, > 0                                          */
    double max_norm;     /* the scaled gradients are clipped to this norm; 0 = never    */
    uint64_t seed;       /* of the 8-bit moments' rounding                              */
    uint32_t moment_bits; /* 32 or 8                                                    */
    uint32_t reserved;   /* must be 0                                                   */
} tagc_optim_config;

/* What a group's tensors share, given anew with every step. */
typedef struct tagc_group {
    double lr, weight_decay;
} tagc_group;

/*
 * Device state of an optimizer (dev, 64 bytes, 16-byte aligned, caller-owned).  Before the first step
 * the caller writes zeros and lr_scale = 1 (and `step` = steps done, to carry on); afterwards
 * tagc_grad_norm writes all but lr_scale.
 */
typedef struct tagc_optim_control {
    uint32_t step;        /* steps begun, this one included                             */
    uint32_t skipped;     /* calls of tagc_grad_norm that found a norm that is not finite */
    uint32_t apply;       /* 1: the last call's norm was finite                         */
    float norm;           /* 2-norm of grad_scale * all gradients                       */
    float factor;         /* grad_scale, times max_norm / norm where that clips         */
    float lr_scale;       /* read by tagc_adamw_step: a schedule that a captured graph
                             can follow                                                 */
    uint32_t reserved[2];
    double bias1, bias2;  /* 1 / (1 - beta1^step), 1 / sqrt(1 - beta2^step)             */
    uint32_t reserved2[4];
} tagc_optim_control;

typedef struct tagc_optim_sizes {
    uint64_t table_bytes;
    uint64_t n_elems;     /* sum of the lengths                                         */
    uint64_t n_blocks;    /* sum of the tensors' blocks of TAGC_MOMENT_BLOCK            */
    uint64_t n_chunks;    /* pieces of tensors that a workgroup takes                   */
} tagc_optim_sizes;

typedef struct tagc_optim_s tagc_optim_t; /* opaque, host memory, immutable */

/*
 * Builds the host-side plan of an optimizer over `tensors` (host, copied).  Errors: TAGC_EINVAL
 * (null or misaligned pointers, unknown type, group, bits, a value out of its range, bases
 * missing or given with 32-bit moments), TAGC_ESIZE (a tensor of 2^34 elements or more, 2^24 chunks of 4096
 * elements or more, 2^23 with 8-bit moments), TAGC_ENOMEM.  *out is owned by the caller: tagc_optim_destroy.
 */
int tagc_optim_plan(const tagc_optim_config *config, const tagc_tensor *tensors, uint32_t n_tensors,
                    tagc_optim_t **out);
void tagc_optim_destroy(tagc_optim_t *plan);
int tagc_optim_plan_sizes(const tagc_optim_t *plan, tagc_optim_sizes *out);

/* Copies the plan's table of tensors into `table_dev` (table_bytes, 16-byte aligned) and clears
 * the device state behind it.  The plan must outlive the copy; the table holds the tensors' addresses, so
 * tensors that move need a plan and an upload of their own. */
int tagc_optim_upload(const tagc_optim_t *plan, void *table_dev, void *stream);

/*
 * Begins a step: norm = grad_scale * sqrt(sum of all gradients' squares), added up in float64 in an order
 * that depends on nothing but the plan and the number of compute units; factor = grad_scale * min(1,
 * max_norm / norm).  A finite norm sets apply and advances step; any other leaves step, sets
 * apply = 0 (the tagc_adamw_step that follows then changes nothing) and counts in skipped.
 * Calls that share a table must not overlap in time.
 */
int tagc_grad_norm(const tagc_optim_t *plan, void *table_dev, tagc_optim_control *control,
                   void *stream);

/*
 * One AdamW step of all tensors, in float32 (t the step, b1, b2 the betas):
 *   g = factor * grad;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
 *   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
 * (with eps = 0 where v is 0, too, that is m / 0: gradients under 1e-22 have squares that float32 does not hold).
 * param and copy are rounded to nearest, ties to even, where they are bfloat16.
 * step > 0: that is t, factor is grad_scale, control is not looked at (may be NULL).
 * step = 0: t, factor, lr_scale and whether to do anything come from control.
 *
 * 8-bit moments are rounded after they have been used.  In a block with base B a code c > 0 stands
 * for the float32 with the bits (B + c) << 20 (three bits behind the leading one), c = 0 for 0;
 * m has 7 bits of code and the sign above them, v 8.  With q = (bits(|x|) + 16 u) >> 20, u
 * 16 random bits, B is the block's largest q less the largest code, or 0, and c = q - B where that
 * is positive: unbiased rounding, as a second moment that moves by a thousandth a step needs to move
 * at all.  Below, v > 0 keeps code 1 (the update divides by its root), and m gets code 1 where
 * u / 2^16 times what code 1 stands for is under |m|.  (A sum that is finite stays finite.)
 * u comes from mix32(seed, t, the tensor's number, the element's number / 4), turned
 * right by 8 bits per element of the four: low 16 bits for m, high 16 for v.
 * A block of zeros with base 0 is where a training run starts.
 *
 * groups: host array, copied before the call returns.
 */
int tagc_adamw_step(const tagc_optim_t *plan, const void *table_dev, const tagc_group *groups,
                    uint32_t n_groups, uint32_t step, const tagc_optim_control *control, void *stream);

/* What 8-bit moments stand for, exactly, as bfloat16: all tensors one behind the other in `m_out` and
 * `v_out` (dev, n_elems each, 2-byte aligned).  TAGC_EUNSUPPORTED for 32-bit moments. */
int tagc_adamw_unpack(const tagc_optim_t *plan, const void *table_dev, void *m_out, void *v_out,
                      void *stream);

/* ------------------------------------------------------------------ linear layers */

enum { TAGC_ACT_NONE = 0, TAGC_ACT_RELU = 1, TAGC_ACT_GELU = 2 /* with erf */,
       TAGC_ACT_GELU_TANH = 3, TAGC_ACT_SILU = 4 };

/*
 * A linear layer, all operands of one type (TAGC_F32 | TAGC_BF16), rows contiguous, `ld*` the
 * elements from one row to the next (>= the row's length).  Pointers are dev, aligned to their
 * element; speed is best where they and the strides are multiples of 16 bytes.
 */
typedef struct tagc_linear {
    uint64_t rows, in, out;         /* tokens, features in and out; each < 2^22 (float32:
                                       2^20), the three matrices together < 2^36 elements */
    uint32_t dtype, activation;     /* TAGC_F32 | TAGC_BF16; TAGC_ACT_*                   */
    const void *x; uint64_t ldx;    /* [rows, in]                                         */
    const void *w; uint64_t ldw;    /* [out, in]                                          */
    const void *bias;               /* [out] or NULL                                      */
    const void *residual; uint64_t ldr; /* [rows, out] or NULL                            */
    void *y; uint64_t ldy;          /* [rows, out]; may be the residual itself, and must
                                       share no element with another operand              */
    void *pre; uint64_t ldp;        /* [rows, out] or NULL: x w^T + bias, for the backward pass; shares
                                       none either (y only where both are the same numbers) */
} tagc_linear;

/* Of dx, dw and db none may share an element with another one or with an operand that is read, but for
 * dy and pre where there is an activation, and for float32 operands. */
typedef struct tagc_linear_grad {
    uint64_t rows, in, out;
    uint32_t dtype, activation;
    const void *x; uint64_t ldx;    /* [rows, in]; not read if dw is NULL                 */
    const void *w; uint64_t ldw;    /* [out, in]; not read if dx is NULL                  */
    const void *pre; uint64_t ldp;  /* [rows, out] as forward left it; NULL without an activation */
    const void *dy; uint64_t lddy;  /* [rows, out]                                        */
    void *dx; uint64_t lddx;        /* [rows, in] or NULL                                 */
    void *dw; uint64_t lddw;        /* [out, in] or NULL: a place in the bucket's gradient */
    void *db;                       /* [out] or NULL                                      */
    uint32_t accumulate;            /* 1: dw and db are added to what is there            */
    uint32_t reserved;              /* must be 0                                          */
} tagc_linear_grad;

/* Bytes of workspace (dev, 256-byte aligned, contents do not matter) that the calls need. */
int tagc_linear_forward_workspace(const tagc_linear *l, uint64_t *bytes);
int tagc_linear_backward_workspace(const tagc_linear_grad *l, uint64_t *bytes);

/*
 * z = x w^T + bias with float32 sums; pre = z; y = act(z) + residual, each rounded once.  bfloat16
 * products are exact.  float32 operands are taken as three bfloat16 numbers each, of which six products are
 * added: what is left out is at most 2^-22 of a product and mostly 2^-24, of either sign, like a
 * rounding; an infinity in x or w makes the sums it enters NaN, and operands under some 2^-100 lose their last bits.
 */
int tagc_linear_forward(const tagc_linear *l, void *workspace, void *stream);

/*
 * dz = dy act'(pre); dx = dz w; dw (+)= dz^T x; db (+)= the sum of dz over the rows.  With an
 * activation dz is rounded to the operands' type before the two products (not for db).  The residual's
 * gradient is dy.
 */
int tagc_linear_backward(const tagc_linear_grad *l, void *workspace, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* TAGC_TRAIN_H */
