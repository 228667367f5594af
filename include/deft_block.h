/*
 * deft_block.h - C ABI of the operators of a layer's feed-forward block, for AMD MI355X (gfx950):
 * the gated feed-forward block with its gradient, and activation checkpoints in 8 bits.
 *
 * Between a model's two ends (deft_ends.h) these make most of what a training step computes and
 * most of the gradient buckets that a schedule has to place: the gradients of the three matrices
 * are final one after the other while the backward pass goes on, and an event can be recorded as
 * each is.  What a layer keeps from the forward to the backward pass bounds the batch: it can be
 * kept in 8 bits, or only the layer's input is, and the rest computed again.
 *
 * As in deft_ends.h, all array arguments are DEVICE pointers owned by the caller, never retained;
 * the library never prints, throws or aborts; every failure is a return code.  A handle owns its
 * scratch memory and serves one call at a time (not thread-safe; one handle per stream).  Calls
 * enqueue kernels on `stream` and return without waiting; they allocate nothing, set nothing with
 * a memset node and read no device data on the host, so they may be recorded into a HIP graph
 * (ffn_grad without events).  Rows are `stride` ELEMENTS apart (at least as many as a row has);
 * pointers need no more than their element's own alignment, though rows whose starts are multiples
 * of 16 bytes are quicker.  Arrays may pass 2^31 elements.  Outputs overlap neither inputs
 * nor each other.
 *
 * Sums are held in 32 bits, each in one fixed order (results do not change from call to call), and
 * outputs are rounded once to the handle's type.  In 16-bit types of more than 64 rows what one
 * product leaves to the next (the hidden activations, and the derivatives by the two projections) is
 * rounded to the type in between, as the matrix instructions take it, so that an output's error is
 * about sqrt 2 of its own rounding's.  In 32 bits, and of fewer rows, it is not, but in y of 9 to 16 rows
 * and, unless hidden and inner are multiples of 64 and all rows of x and the matrices start at multiples
 * of 16 bytes and at most 2^22 elements apart, of up to 64 rows (hidden x inner up to 2^21) or 32 (up to
 * 6 x 2^20).
 * Hidden activations beyond the type's range are infinite there, of few rows too.
 *
 * Rows that stand for nothing (the padding of a batch) are rows of zeros, as deft_embed gives them
 * for a token of -1: they add nothing to any gradient.
 */
#ifndef DEFT_BLOCK_H
#define DEFT_BLOCK_H

#include <stdint.h>

#include "deft_ends.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct deft_block deft_block_t; /* opaque */

/* operators that a handle serves; they size its scratch memory (checkpoint and restore need none; ffn alone of up to 16
 * rows, or 32 of max_hidden x max_inner up to 2^21, or 64 in 32 bits, none for operands and parts of sums) */
#define DEFT_BLOCK_FFN 1u
#define DEFT_BLOCK_FFN_GRAD 2u
#define DEFT_BLOCK_CHECKPOINT 4u
#define DEFT_BLOCK_RESTORE 8u

typedef struct {
    int32_t device;     /* HIP device ordinal                                                  */
    int32_t dtype;      /* DEFT_F32, DEFT_F16 or DEFT_BF16                                     */
    uint32_t operators; /* DEFT_BLOCK_*, at least one                                          */
    int32_t max_rows;   /* tokens per call (1 .. 2^20)                                         */
    int32_t max_hidden; /* 1 .. 16384 (a checkpoint's width: up to max_hidden or max_inner)    */
    int32_t max_inner;  /* 1 .. 65536; 0 where neither DEFT_BLOCK_FFN nor _FFN_GRAD is served  */
} deft_block_config_t;

/* Checks the limits and the device and allocates the scratch memory.
 * Errors: INVALID_ARG (NULL, unknown type or operator, a limit below 1 that an operator needs),
 * LIMIT (beyond the ranges above), OOM, DEVICE.  *out is NULL on error. */
deft_status_t deft_block_create(const deft_block_config_t *cfg, deft_block_t **out);

/* Frees the scratch memory and the handle.  NULL is a no-op. */
void deft_block_destroy(deft_block_t *h);

typedef struct {
    int64_t scratch_bytes; /* device memory that the handle holds                              */
    int32_t compute_units;
} deft_block_info_t;

deft_status_t deft_block_get_info(const deft_block_t *h, deft_block_info_t *info);

/*
 * A checkpoint holds a row in groups of 32 elements (the last one may be shorter).  Of each group:
 *   s = the smallest number of 8 significant bits, at least 2^-126, with 127 s >= max |x|,
 *   codes = the whole number nearest to x / s, ties to the even one (-127 .. 127),
 * and it stands for codes * s: off by at most s / 2, which is at most (1 + 2^-7) max |x| / 254, in
 * 8.5 bits an element.  An element that is not finite has code -128, takes no part in the largest
 * and comes back as NaN, as all of a group does whose scale is NaN (deft_ffn writes such ones).  Scales are the
 * upper halves of 32-bit floats (bfloat16).  What lies beyond the type's largest number comes back as that.
 */
#define DEFT_CHECKPOINT_GROUP 32

typedef struct {
    void *codes;           /* int8 [n_rows][width]                                             */
    int64_t codes_stride;
    void *scales;          /* bfloat16 [n_rows][(width + 31) / 32]                             */
    int64_t scales_stride;
} deft_checkpoint_t;

/* deft_checkpoint: writes the checkpoint of x. */
typedef struct {
    int32_t n_rows;
    int32_t width;
    const void *x;         /* [n_rows][width]                                                  */
    int64_t x_stride;
    deft_checkpoint_t out;
    void *stream;          /* hipStream_t; NULL = the default stream                           */
} deft_checkpoint_call_t;

deft_status_t deft_checkpoint(deft_block_t *h, const deft_checkpoint_call_t *a);

/* deft_restore: out = what the checkpoint stands for, rounded once to the handle's type. */
typedef struct {
    int32_t n_rows;
    int32_t width;
    deft_checkpoint_t from;
    void *out;             /* [n_rows][width]                                                  */
    int64_t out_stride;
    void *stream;
} deft_restore_call_t;

deft_status_t deft_restore(deft_block_t *h, const deft_restore_call_t *a);

/* act(a): a / (1 + exp(-a));  a (1 + erf(a / sqrt 2)) / 2;
 * a (1 + tanh(sqrt(2 / pi) (a + 0.044715 a^3))) / 2;  max(a, 0) with derivative 0 at 0 */
enum { DEFT_SILU = 0, DEFT_GELU = 1, DEFT_GELU_TANH = 2, DEFT_RELU = 3 };

/* what is kept of the two projections between the passes: nothing, themselves in as many bits as the
 * handle's type has, or their checkpoints */
enum { DEFT_SAVE_NONE = 0, DEFT_SAVE_FULL = 1, DEFT_SAVE_PACKED = 2 };

/* of width `inner`.  FULL: in 32 bits `codes` are the numbers themselves (float) and there are no
 * scales; in 16-bit types they are checkpoints whose codes are int16 (-32767 .. 32767), in 16.5 bits an
 * element off by at most (1 + 2^-7) / 65534 of the group's largest: as good as the sums in 32 bits for what
 * is rounded to the type afterwards.  A sum within its own error of the middle between two codes may get
 * either; with relu, whose derivative changes there, a positive sum of the gate gets 1 at least (and may be
 * off by the step).  A group with a sum that is not finite has NaN as its scale, and comes back as NaN. */
typedef struct {
    int32_t kind;          /* DEFT_SAVE_*                                                      */
    deft_checkpoint_t gate, up;
} deft_saved_t;

/*
 * deft_ffn, with the matrices stored as [outputs][inputs]:
 *   gate = x w_gate^T,  up = x w_up^T,  y = (act(gate) * up) w_down^T,
 * and gate and up kept as `save` says, from their sums in 32 bits.
 * A row of y depends on its own row of x alone.  Where that or a matrix holds infinities or NaN, so does what is made of them (NaN
 * possibly in the place of an infinity).
 */
typedef struct {
    int32_t n_rows;
    int32_t hidden;
    int32_t inner;
    int32_t activation;    /* DEFT_SILU ..                                                     */
    const void *x;         /* [n_rows][hidden]                                                 */
    int64_t x_stride;
    const void *w_gate;    /* [inner][hidden]                                                  */
    int64_t w_gate_stride;
    const void *w_up;      /* [inner][hidden]                                                  */
    int64_t w_up_stride;
    const void *w_down;    /* [hidden][inner]                                                  */
    int64_t w_down_stride;
    void *y;               /* [n_rows][hidden]                                                 */
    int64_t y_stride;
    deft_saved_t save;     /* written                                                          */
    void *stream;
} deft_ffn_t;

deft_status_t deft_ffn(deft_block_t *h, const deft_ffn_t *a);

/*
 * deft_ffn_grad: with gate and up as `saved` has them (computed again from x where its kind is NONE),
 *   d = grad_y w_down,  d_gate = d * up * act'(gate),  d_up = d * act(gate):
 *   grad_down = grad_y^T (act(gate) * up),  grad_gate = d_gate^T x,  grad_up = d_up^T x,
 *   grad_x = d_gate w_gate + d_up w_up.
 * accumulate = 1 adds the three matrices' gradients to what is there (an earlier iteration whose update is
 * delayed).  Each of the four gradients may be NULL, not all.  Where `x` is NULL, packed_x is its
 * checkpoint.  events (a HOST array of two hipEvent_t, or NULL) are recorded on the stream: the first once
 * grad_down is written, the second once grad_gate and grad_up are; grad_x comes last.  Such a call must
 * not be captured.
 * Where rows of x or grad_y hold infinities or NaN, so do their rows of grad_x and the matrices' gradients (NaN
 * possibly in the place of an infinity); other rows of grad_x do not.
 * In 16-bit floats d_gate and d_up are held times a power of two that brings grad_y's largest magnitude to
 * 1 .. 2: elements below 2^-14 of that lose bits, one more than 2^15 times it is infinite.
 */
typedef struct {
    int32_t n_rows;
    int32_t hidden;
    int32_t inner;
    int32_t activation;
    int32_t accumulate;    /* 0 or 1                                                           */
    const void *grad_y;    /* [n_rows][hidden]                                                 */
    int64_t grad_y_stride;
    const void *x;         /* [n_rows][hidden], or NULL                                        */
    int64_t x_stride;
    deft_checkpoint_t packed_x; /* where x is NULL                                             */
    const void *w_gate;    /* as in deft_ffn                                                   */
    int64_t w_gate_stride;
    const void *w_up;
    int64_t w_up_stride;
    const void *w_down;
    int64_t w_down_stride;
    deft_saved_t saved;    /* as deft_ffn wrote it                                             */
    void *grad_x;          /* [n_rows][hidden] or NULL                                         */
    int64_t grad_x_stride;
    void *grad_gate;       /* [inner][hidden] or NULL                                          */
    int64_t grad_gate_stride;
    void *grad_up;         /* [inner][hidden] or NULL                                          */
    int64_t grad_up_stride;
    void *grad_down;       /* [hidden][inner] or NULL                                          */
    int64_t grad_down_stride;
    void **events;         /* HOST array of 2 hipEvent_t, or NULL                              */
    void *stream;
} deft_ffn_grad_t;

deft_status_t deft_ffn_grad(deft_block_t *h, const deft_ffn_grad_t *a);

#ifdef __cplusplus
}
#endif

#endif /* DEFT_BLOCK_H */
