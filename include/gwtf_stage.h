/*
 * gwtf_stage.h -- C ABI of the operators on a routed microbatch, on AMD
 * Instinct MI355X (gfx950), in the same library as gwtf_mcf.h.
 *
 * gwtf_mcf.h says which machine carries which microbatch; these calls work on
 * the microbatch itself where its route begins, changes machines and ends
 * (paper Sec. II and III: the first and the last stage sit on the data node,
 * relay nodes hold the stages between them; Sec. V-D: the microbatch of a
 * crashed relay is sent to another one, which repeats the stage):
 *
 *   gwtf_stage_embed, _embed_grad      data node, first stage: tokens to rows
 *                                      of the embedding table, and the
 *                                      table's gradient by sorted tokens
 *   gwtf_stage_norm, _norm_grad        hand-off: residual added, RMS norm,
 *                                      8-bit values with scales (a quarter of
 *                                      the 32-bit bytes of Eq. 1's size term)
 *   gwtf_stage_dropout                 dropout that any machine repeats
 *                                      exactly from the row's identity; its
 *                                      own gradient
 *   gwtf_stage_logprob, _logprob_grad  data node, last stage: log
 *                                      probabilities of given tokens, entropy,
 *                                      the most likely tokens, and the
 *                                      gradient
 *
 * A matrix is row-major: a device pointer, the distance between its rows in
 * elements (its columns are adjacent; the distance is at least the width,
 * except that with one row it is not looked at) and its element type.  Rows
 * need no more alignment than their element type.  A row may be a token of
 * any microbatch.  Outputs must not overlap inputs or each other, except
 * where a call says so.
 *
 * As in gwtf_mcf.h: pointers are DEVICE pointers on the handle's GPU, owned
 * by the caller; work is enqueued on the handle's HIP stream and calls return
 * after enqueueing; argument errors give GWTF_ERR_INVALID_ARG with nothing
 * enqueued; a handle serves one stream and is not thread-safe.  No call
 * allocates or synchronises, so all may be captured into a HIP graph (one
 * graph, or eager calls, at a time: they share the handle's workspace).
 * Results are deterministic: the same inputs give the same bits, on every
 * call with the same shapes (of log probabilities, with rows that also lie the
 * same way to 16-byte boundaries).  Sums, statistics and gradients are held in 32
 * bits and rounded once to the output's type.
 */
#ifndef GWTF_STAGE_H
#define GWTF_STAGE_H

#include "gwtf_mcf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gwtf_stage gwtf_stage_t; /* opaque; owns its device workspace */

/* Element types. */
enum {
    GWTF_TYPE_F32 = 0,
    GWTF_TYPE_F16 = 1,
    GWTF_TYPE_BF16 = 2
};

/* Integer types of tokens. */
enum {
    GWTF_TOKEN_I32 = 0,
    GWTF_TOKEN_I64 = 1
};

/* Form of gwtf_stage_norm's output. */
enum {
    GWTF_NORM_PLAIN = 0,    /* values in x's type */
    GWTF_NORM_F8_ROW = 1,   /* 8-bit values (OCP e4m3), one scale a row */
    GWTF_NORM_F8_BLOCK = 2  /* 8-bit values (OCP e4m3), one scale for each GWTF_NORM_BLOCK columns of a row */
};

#define GWTF_NORM_BLOCK 128
#define GWTF_STAGE_MAX_HIDDEN 16384 /* widest row of the norm */
#define GWTF_STAGE_MAX_TOP 64       /* most alternatives of gwtf_stage_logprob */

typedef struct {
    int64_t max_tokens; /* most rows a call may pass, 1 .. 2^31 - 1 */
    int64_t max_hidden; /* widest row of an embedding, norm or dropout call, 1 .. 2^20 */
    int64_t max_vocab;  /* largest vocabulary, 1 .. 2^31 - 1 */
    int32_t device;     /* HIP device ordinal the handle works on */
} gwtf_stage_shape_t;

/* Creates a handle on shape->device that enqueues on `hip_stream` (a
 * hipStream_t; NULL = the device's null stream) and allocates its workspace:
 * 16 bytes a token; for the embedding's gradient 16.8 MB and 8 bytes a column
 * (where that is less, 8 bytes a column and 2 a column and token), and a bit for
 * each row of the table, 0.6 MB at most; for the norm's 2048 bytes a column, 34
 * MB at most; and 1.1 MB for gwtf_stage_logprob.  *out receives the handle, or NULL on failure. */
gwtf_status_t gwtf_stage_create(const gwtf_stage_shape_t *shape, void *hip_stream, gwtf_stage_t **out);

/* Frees the handle and its workspace after draining its stream; NULL-safe. */
void gwtf_stage_destroy(gwtf_stage_t *h);

/* Text of the last error on this handle ("" if none); a NULL handle gives the
 * last error of a gwtf_stage_create, or of a call with a NULL handle, on the
 * calling thread. */
const char *gwtf_stage_last_error(const gwtf_stage_t *h);

/* ---- Embedding ----
 *
 * out[i][:] = scale * table[tokens[i]][:], in 32 bits, rounded to `type`.  A
 * token outside [0, vocab) (padding) gives a row of zeros. */
typedef struct {
    int64_t num_tokens, hidden, vocab; /* N >= 0, H >= 1, V >= 1 */
    int32_t type, token_type;          /* GWTF_TYPE_* of table and out, GWTF_TOKEN_* */
    float scale;
    const void *tokens;                /* [N] */
    const void *table;                 /* [V][H] */
    int64_t table_stride;
    void *out;                         /* [N][H] */
    int64_t out_stride;
} gwtf_stage_embed_t;
gwtf_status_t gwtf_stage_embed(gwtf_stage_t *h, const gwtf_stage_embed_t *a);

/* grad[v][:] = scale * sum of dout[i][:] over the i with tokens[i] == v, in
 * ascending order of i within pieces whose sums are then added in order.
 * With accumulate == 0 all of grad is written (zeros where no token is v);
 * otherwise the sum is added to grad and rows of absent tokens are neither
 * read nor written.  Tokens outside [0, vocab) take no part. */
typedef struct {
    int64_t num_tokens, hidden, vocab; /* N >= 0, H >= 1, V >= 1 */
    int32_t type, grad_type;           /* GWTF_TYPE_* of dout; of grad: that type or GWTF_TYPE_F32 */
    int32_t token_type, accumulate;
    float scale;
    const void *tokens;                /* [N] */
    const void *dout;                  /* [N][H] */
    int64_t dout_stride;
    void *grad;                        /* [V][H] */
    int64_t grad_stride;
} gwtf_stage_embed_grad_t;
gwtf_status_t gwtf_stage_embed_grad(gwtf_stage_t *h, const gwtf_stage_embed_grad_t *a);

/* ---- Dropout ----
 *
 * out[i][c] = residual[i][c] + (u >= t ? x[i][c] * 65536 / (65536 - t) : 0)
 * with t = p rounded to a multiple of 2^-16, times 65536 (p < 1 after the
 * rounding), and u 16 bits of Philox4x32-10 with key (low, high half of
 * `seed`) and counter (c / 8, site, low, high half of rows[i]): word
 * (c % 8) / 2, its low half for even c.  The mask depends on the seed, the
 * site (a number of the caller's, one for each place of the model) and the
 * row's identity alone, not on the row's place in the call or the machine, and
 * is never stored; a dropped NaN or infinity gives 0.  The gradient is the same call
 * on the gradient of out, without residual.  out may be x or residual
 * itself (same pointer and stride). */
typedef struct {
    int64_t num_tokens, hidden; /* N >= 0, H >= 1 */
    int32_t type;               /* GWTF_TYPE_* of x, residual and out */
    uint32_t site;
    uint64_t seed;
    double p;                   /* probability of a zero, 0 <= p < 1 */
    const int64_t *rows;        /* [N] identities of the rows; NULL = 0, 1, 2, .. */
    const void *x;              /* [N][H] */
    int64_t x_stride;
    const void *residual;       /* [N][H] or NULL = 0 */
    int64_t residual_stride;
    void *out;                  /* [N][H] */
    int64_t out_stride;
} gwtf_stage_dropout_t;
gwtf_status_t gwtf_stage_dropout(gwtf_stage_t *h, const gwtf_stage_dropout_t *a);

/* ---- Hand-off: residual, RMS norm, 8 bits ----
 *
 * h = x + residual; rstd = 1 / sqrt(mean(h^2) + eps); y = h * rstd * weight,
 * from the 32-bit sum h (h_out receives it rounded), also where h^2 leaves the
 * range of 32 bits and rstd does not.  With an 8-bit form each row, or each
 * GWTF_NORM_BLOCK columns of a row (the last block may be shorter), has a
 * 32-bit scale s = max(max |y| / 448, 2^-126), and y / s, rounded to 32 bits, to
 * the nearest e4m3 value, the even one of two that are as near: y is about
 * q * s.  A NaN or infinity among the y of a scale makes the scale and all of
 * its values NaN. */
typedef struct {
    int64_t num_tokens, hidden; /* N >= 0, 1 <= H <= GWTF_STAGE_MAX_HIDDEN */
    int32_t type;               /* GWTF_TYPE_* of x, residual, weight, h_out and a plain y */
    int32_t form;               /* GWTF_NORM_* */
    float eps;                  /* >= 0 */
    const void *x;              /* [N][H] */
    int64_t x_stride;
    const void *residual;       /* [N][H] or NULL = 0 */
    int64_t residual_stride;
    const void *weight;         /* [H] */
    void *y;                    /* [N][H], one byte each with an 8-bit form */
    int64_t y_stride;
    void *h_out;                /* [N][H], or NULL; may be x or residual itself */
    int64_t h_stride;
    float *scales;              /* [N] or [N][ceil(H / 128)]; NULL iff form is plain */
    float *rstd;                /* [N] or NULL */
} gwtf_stage_norm_t;
gwtf_status_t gwtf_stage_norm(gwtf_stage_t *h, const gwtf_stage_norm_t *a);

/* Gradient of the norm, given the gradient dy of y (of the values that 8 bits
 * stand for), h and rstd of the forward call, and dh, what reaches h
 * by the residual path: with xhat = h * rstd and c = mean(dy * weight * xhat),
 *   dx = dh + rstd * (dy * weight - xhat * c)   (the residual's gradient too)
 *   dweight = sum over the rows of dy * xhat
 * dx may be dy or dh itself (same pointer and stride). */
typedef struct {
    int64_t num_tokens, hidden; /* N >= 0, 1 <= H <= GWTF_STAGE_MAX_HIDDEN */
    int32_t type;               /* GWTF_TYPE_* of dy, h, dh, weight and dx */
    const void *dy;             /* [N][H] */
    int64_t dy_stride;
    const void *h;              /* [N][H] */
    int64_t h_stride;
    const void *dh;             /* [N][H] or NULL = 0 */
    int64_t dh_stride;
    const void *weight;         /* [H] */
    const float *rstd;          /* [N] */
    void *dx;                   /* [N][H] */
    int64_t dx_stride;
    float *dweight;             /* [H], or NULL */
} gwtf_stage_norm_grad_t;
gwtf_status_t gwtf_stage_norm_grad(gwtf_stage_t *h, const gwtf_stage_norm_grad_t *a);

/* ---- Log probabilities ----
 *
 * Per row of logits x: lse = ln sum exp(x); logp = x[target] - lse; entropy =
 * -sum p ln p with p = exp(x - lse); and the `top` largest x, largest first,
 * equal ones by ascending index: top_ids and their log probabilities top_logp.
 * Rounding puts no log probability above 0 and no entropy below.
 * A target outside [0, vocab) gives logp 0.  An entry of -infinity is masked: p = 0,
 * log probability -infinity; a row of nothing else gives lse = -infinity,
 * entropy 0 and alternatives 0, 1, 2, .. .  A NaN or +infinity makes lse,
 * entropy and the row's log probabilities NaN; a NaN is no alternative, and
 * alternatives that are missing for that have index -1.  Finite logits may have
 * any value, masks of -1e30 or the type's lowest value among them: where a row's
 * largest logit is beyond 9e4 in magnitude, so that lse in 32 bits does not
 * resolve a probability, log probabilities come from differences to it. */
typedef struct {
    int64_t num_tokens, vocab;  /* N >= 0, V >= 1 */
    int32_t type, token_type;   /* GWTF_TYPE_* of logits, GWTF_TOKEN_* of targets */
    int32_t top;                /* 0 <= top <= min(V, GWTF_STAGE_MAX_TOP) */
    const void *logits;         /* [N][V] */
    int64_t logits_stride;
    const void *targets;        /* [N], or NULL iff logp is NULL */
    float *logp, *entropy, *lse; /* [N], each may be NULL */
    float *top_logp;            /* [N][top], NULL iff top == 0 */
    int32_t *top_ids;           /* [N][top], NULL iff top == 0 */
} gwtf_stage_logprob_t;
gwtf_status_t gwtf_stage_logprob(gwtf_stage_t *h, const gwtf_stage_logprob_t *a);

/* Gradient of logp and entropy:
 *   dlogits[j] = dlogp * ([j == target] - p_j) - dentropy * p_j * (ln p_j + entropy)
 * from lse and entropy of the forward call.  dlogp counts as 0 where the
 * target is outside [0, vocab); a row whose lse is -infinity gets zeros.  p is
 * exp(logits - lse), no better than the 32 bits of lse: a row whose largest
 * logit is of the order of 1e5 or more is best shifted before both calls.
 * dlogits may be logits itself (same pointer and stride). */
typedef struct {
    int64_t num_tokens, vocab;  /* N >= 0, V >= 1 */
    int32_t type, token_type;   /* GWTF_TYPE_* of logits and dlogits, GWTF_TOKEN_* of targets */
    const void *logits;         /* [N][V] */
    int64_t logits_stride;
    const void *targets;        /* [N], or NULL iff dlogp is NULL */
    const float *lse;           /* [N] */
    const float *entropy;       /* [N], or NULL iff dentropy is NULL */
    const float *dlogp;         /* [N] or NULL = 0 */
    const float *dentropy;      /* [N] or NULL = 0 */
    void *dlogits;              /* [N][V] */
    int64_t dlogits_stride;
} gwtf_stage_logprob_grad_t;
gwtf_status_t gwtf_stage_logprob_grad(gwtf_stage_t *h, const gwtf_stage_logprob_grad_t *a);

#ifdef __cplusplus
}
#endif
#endif /* GWTF_STAGE_H */
