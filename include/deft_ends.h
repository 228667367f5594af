/*
 * deft_ends.h - C ABI of the operators at the two ends of a language model, for AMD MI355X
 * (gfx950): the token embedding, the head with its softmax cross entropy, and distillation from a
 * teacher's top logits.
 *
 * These are the first and the last thing that a training step computes, and the table that they
 * share is the largest gradient bucket that a schedule has to place: its gradient begins with
 * the loss (deft_head_grad writes it, a piece of the vocabulary after the other) and is complete
 * once the embedding has merged its part into it (deft_embed_grad with `accumulate`).
 *
 * As in deft_knapsack.h, all array arguments are DEVICE pointers owned by the caller, never
 * retained; integers are int32 unless stated; the library never prints, throws or aborts; every
 * failure is a return code, or a status of the row where the data is at fault.  A handle owns its
 * scratch memory and serves one call at a time (not thread-safe; one handle per stream).  Calls
 * enqueue kernels on `stream` and return without waiting; they allocate nothing, set nothing with
 * a memset node and read no device data on the host, so they may be recorded into a HIP graph.
 *
 * Rows are `stride` ELEMENTS apart (at least as many as a row has); pointers need no more than
 * their element's own alignment, though rows whose starts are multiples of 16 bytes are quicker.
 * Arrays may pass 2^31 elements.  Sums, softmax statistics and norms are held in 32 bits, each
 * gradient is summed in one fixed order (results do not change from call to call), and outputs
 * are rounded once to the handle's type, except where two calls add into one array.
 *
 * -1 stands for nothing: an empty slot among the tokens, a position without a label, an entry that
 * the teacher did not keep.  What such a row gives is zero, whatever its other inputs hold, NaN
 * and infinities included.
 */
#ifndef DEFT_ENDS_H
#define DEFT_ENDS_H

#include <stdint.h>

#include "deft_knapsack.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct deft_ends deft_ends_t; /* opaque */

/* type of tables, hidden states, logits and their gradients */
enum { DEFT_F32 = 0, DEFT_F16 = 1, DEFT_BF16 = 2 };

/* operators that a handle serves; they size its scratch memory */
#define DEFT_ENDS_EMBED 1u
#define DEFT_ENDS_EMBED_GRAD 2u
#define DEFT_ENDS_HEAD_LOSS 4u
#define DEFT_ENDS_HEAD_GRAD 8u
#define DEFT_ENDS_DISTILL 16u

typedef struct {
    int32_t device;     /* HIP device ordinal                                                  */
    int32_t dtype;      /* DEFT_F32, DEFT_F16 or DEFT_BF16                                     */
    uint32_t operators; /* DEFT_ENDS_*, at least one                                           */
    int32_t max_rows;   /* tokens or positions per call (1 .. 2^20)                            */
    int32_t max_vocab;  /* 1 .. 2^21                                                           */
    int32_t max_hidden; /* 1 .. 16384; 0 where only DEFT_ENDS_DISTILL is served                */
    int32_t max_top_k;  /* 1 .. 1024 with DEFT_ENDS_DISTILL; 0 otherwise                       */
} deft_ends_config_t;

/* Checks the limits and the device and allocates the scratch memory.
 * Errors: INVALID_ARG (NULL, unknown type or operator, a limit below 1 that an operator needs),
 * LIMIT (beyond the ranges above), OOM, DEVICE.  *out is NULL on error. */
deft_status_t deft_ends_create(const deft_ends_config_t *cfg, deft_ends_t **out);

/* Frees the scratch memory and the handle.  NULL is a no-op. */
void deft_ends_destroy(deft_ends_t *h);

typedef struct {
    int64_t scratch_bytes; /* device memory that the handle holds                              */
    int32_t vocab_piece;   /* rows of the vocabulary that deft_head_grad takes at a time        */
    int32_t compute_units;
} deft_ends_info_t;

deft_status_t deft_ends_get_info(const deft_ends_t *h, deft_ends_info_t *info);

/*
 * deft_embed: out[n] = scale * table[tokens[n]].
 * A token of -1 gives a row of zeros; one outside 0 .. vocab-1 too, and status INVALID_ARG.
 */
typedef struct {
    int32_t n_rows;
    int32_t vocab;
    int32_t hidden;
    float scale;
    const int32_t *tokens; /* [n_rows]                                                         */
    const void *table;     /* [vocab][hidden]                                                  */
    int64_t table_stride;
    void *out;             /* [n_rows][hidden]                                                 */
    int64_t out_stride;
    int32_t *status;       /* [n_rows], may be NULL                                            */
    void *stream;          /* hipStream_t; NULL = the default stream                           */
} deft_embed_t;

deft_status_t deft_embed(deft_ends_t *h, const deft_embed_t *e);

/*
 * deft_embed_grad: grad_table[v] = scale * sum of grad_out[n] over the n with tokens[n] == v,
 * summed in the order of n.  accumulate = 0 writes every row of the table (zeros where no token
 * points); 1 adds to what is there and leaves the other rows alone: the gradient of the head that
 * shares the table, or of an earlier iteration whose update is delayed.  Tokens of -1 and tokens
 * outside the vocabulary add nothing.
 */
typedef struct {
    int32_t n_rows;
    int32_t vocab;
    int32_t hidden;
    float scale;
    int32_t accumulate;     /* 0 or 1                                                          */
    const int32_t *tokens;  /* [n_rows]                                                        */
    const void *grad_out;   /* [n_rows][hidden]                                                */
    int64_t grad_out_stride;
    void *grad_table;       /* [vocab][hidden]                                                 */
    int64_t grad_table_stride;
    void *stream;
} deft_embed_grad_t;

deft_status_t deft_embed_grad(deft_ends_t *h, const deft_embed_grad_t *e);

/*
 * deft_head_loss: z[n][v] = logit_scale * <hidden[n], weight[v]> over the whole vocabulary, never
 * kept;  lse[n] = log sum_v exp(z[n][v]),  loss[n] = lse[n] - z[n][labels[n]].
 * A label of -1 gives loss and lse 0; one outside 0 .. vocab-1 too, and status INVALID_ARG.
 * Where hidden states or weights are infinite, 32-bit logits of more than 64 positions may be NaN in
 * the place of an infinity (an operand is multiplied in three parts, zeros among them); so may the
 * gradients.
 */
typedef struct {
    int32_t n_rows;
    int32_t vocab;
    int32_t hidden;
    float logit_scale;
    const void *hidden_states; /* [n_rows][hidden]                                             */
    int64_t hidden_stride;
    const void *weight;        /* [vocab][hidden]                                              */
    int64_t weight_stride;
    const int32_t *labels;     /* [n_rows]                                                     */
    float *loss;               /* [n_rows]                                                     */
    float *lse;                /* [n_rows]                                                     */
    int32_t *status;           /* [n_rows], may be NULL                                        */
    void *stream;
} deft_head_loss_t;

deft_status_t deft_head_loss(deft_ends_t *h, const deft_head_loss_t *a);

/*
 * deft_head_grad: with d[n][v] = row_grad[n] * (exp(z[n][v] - lse[n]) - [v == labels[n]]),
 *   grad_hidden[n] = logit_scale * sum_v d[n][v] weight[v]
 *   grad_weight[v] = logit_scale * sum_n d[n][v] hidden[n]     (added to what is there where
 *                                                               accumulate is 1)
 * lse is what deft_head_loss gave for the same inputs.  The logits are computed again, a piece of
 * the vocabulary at a time; the rows of grad_weight are final piece by piece, in order: where
 * piece_events is given, its element i (a hipEvent_t) is recorded on the stream once the rows
 * below (i + 1) * vocab_piece are written (deft_ends_get_info), so that the communication of a
 * bucket can begin while the next one is computed (elements past the last piece: once all are; of a
 * table that other calls add into afterwards, a bucket is ready once they have).  Such a call must not
 * be captured.
 * Rows without a valid label have a zero row in grad_hidden and no part in grad_weight.
 * Either gradient may be NULL, not both.
 * In 16-bit types d is rounded to the type before the two products, as their matrix instructions
 * take it (scaled so that a row of the largest row_grad fills the range up to a power of two, and
 * 16-bit floats into their range), so that grad_weight is off by somewhat more than its own rounding
 * (a tenth to a seventh more, in the norm); in 32 bits it is not.  In 16-bit floats a position whose
 * row_grad is 2^-r of the largest has errors of its own beside, where values pass below the type's
 * range: row_grad 2^(s - 38) in an element of d, and in grad_weight d 2^(t - 25) for each of its
 * hidden states' elements, with s = r - 4, from 0 to 12, and t = r - s.
 */
typedef struct {
    int32_t n_rows;
    int32_t vocab;
    int32_t hidden;
    float logit_scale;
    int32_t accumulate;        /* 0 or 1                                                       */
    int32_t n_piece_events;    /* elements of piece_events                                     */
    const void *hidden_states; /* [n_rows][hidden]                                             */
    int64_t hidden_stride;
    const void *weight;        /* [vocab][hidden]                                              */
    int64_t weight_stride;
    const int32_t *labels;     /* [n_rows]                                                     */
    const float *lse;          /* [n_rows]                                                     */
    const float *row_grad;     /* [n_rows]                                                     */
    void *grad_hidden;         /* [n_rows][hidden] or NULL                                     */
    int64_t grad_hidden_stride;
    void *grad_weight;         /* [vocab][hidden] or NULL                                      */
    int64_t grad_weight_stride;
    void **piece_events;       /* HOST array of hipEvent_t, or NULL                            */
    void *stream;
} deft_head_grad_t;

deft_status_t deft_head_grad(deft_ends_t *h, const deft_head_grad_t *a);

/*
 * deft_distill: the student's logits against the logits that a teacher kept for each row.
 *   p = softmax(teacher_logit / temperature) over the row's entries with teacher_index >= 0,
 *   q = softmax(logits / temperature) over the vocabulary,
 *   loss[n]        = temperature^2 * sum_k p_k (log p_k - log q[index_k])
 *   grad_logits[n] = row_grad[n] * temperature * (q - p at its indices)
 * grad_logits may be the logits themselves, with the same stride; NULL computes the loss alone.
 * Entries of a row may be fewer than top_k (the others -1, anywhere) and in any order; an index
 * that occurs twice is two terms of the loss and counts with the sum of its p in the gradient.  A row
 * without any entry gives zeros.  An index outside -1 .. vocab-1, or a row whose kept entries (or whose logits) are all -infinity, has
 * no such softmax: zeros, and status INVALID_ARG.
 */
typedef struct {
    int32_t n_rows;
    int32_t vocab;
    int32_t top_k;
    float temperature;            /* > 0, finite                                               */
    const void *logits;           /* [n_rows][vocab]                                           */
    int64_t logits_stride;
    const int32_t *teacher_index; /* [n_rows][top_k]                                           */
    const float *teacher_logit;   /* [n_rows][top_k]                                           */
    const float *row_grad;        /* [n_rows]; NULL where grad_logits is                       */
    float *loss;                  /* [n_rows]                                                  */
    void *grad_logits;            /* [n_rows][vocab] or NULL                                   */
    int64_t grad_stride;
    int32_t *status;              /* [n_rows], may be NULL                                     */
    void *stream;
} deft_distill_t;

deft_status_t deft_distill(deft_ends_t *h, const deft_distill_t *a);

#ifdef __cplusplus
}
#endif

#endif /* DEFT_ENDS_H */
