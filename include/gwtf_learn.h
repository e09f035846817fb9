/*
 * gwtf_learn.h -- C ABI of the operators that close a training step, on AMD
 * Instinct MI355X (gfx950), in the same library as gwtf_mcf.h and
 * gwtf_stage.h.
 *
 * gwtf_stage.h takes a routed microbatch from its tokens to the gradients;
 * these calls are what a step has before and after that (paper Sec. II and
 * V-E: forward, backward and update phases; the data node holds the first and
 * the last stage):
 *
 *   gwtf_learn_sample      data node, last stage: answers drawn from the
 *                          logits with temperature, top k, top p and min p and
 *                          given random numbers, for gwtf_stage_logprob to
 *                          score and gwtf_stage_logprob_grad to learn from
 *   gwtf_learn_grad_norm   every node, before its update: the norm of all of
 *                          its gradients and the factor that clips them
 *   gwtf_learn_adamw       every node, update phase: an AdamW step over all
 *                          of its parameters, states in 32 bits or in 8
 *
 * Element types are GWTF_TYPE_* of gwtf_stage.h.  As there: pointers are
 * DEVICE pointers on the handle's GPU, owned by the caller; work is enqueued on
 * the handle's HIP stream and calls return after enqueueing; argument errors
 * give GWTF_ERR_INVALID_ARG with nothing enqueued; a handle serves one stream
 * and is not thread-safe.  Of the calls only those that create or destroy
 * allocate or synchronise, so the others may be captured into a HIP graph (one
 * graph, or eager calls, at a time: they share the handle's workspace).  Arrays need no more alignment than their element type.
 * Outputs must not overlap inputs or each other, except where a call says so.
 * Results are deterministic: the same inputs give the same bits on every call.
 */
#ifndef GWTF_LEARN_H
#define GWTF_LEARN_H

#include "gwtf_stage.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct gwtf_learn gwtf_learn_t;           /* opaque; owns its device workspace */
typedef struct gwtf_learn_list gwtf_learn_list_t; /* opaque; a node's parameters, owns a table of them on the device */

/* Types of given random numbers. */
enum {
    GWTF_UNIFORM_F32 = 0,
    GWTF_UNIFORM_F64 = 1
};

/* Forms of the states of gwtf_learn_adamw. */
enum {
    GWTF_STATE_F32 = 0, /* m and v in 32 bits */
    GWTF_STATE_F8 = 1,  /* m in OCP e4m3, v in OCP e5m2, a scale for each GWTF_STATE_BLOCK values */
    GWTF_STATE_NONE = 2 /* gradients alone, for gwtf_learn_grad_norm */
};

#define GWTF_STATE_BLOCK 128

/* Creates a handle on `device` that enqueues on `hip_stream` (a hipStream_t;
 * NULL = the device's null stream) and allocates its workspace, 2.2 MB.  *out
 * receives the handle, or NULL on failure. */
gwtf_status_t gwtf_learn_create(int32_t device, void *hip_stream, gwtf_learn_t **out);

/* Frees the handle and its workspace after draining its stream; NULL-safe. */
void gwtf_learn_destroy(gwtf_learn_t *h);

/* Text of the last error on this handle ("" if none); a NULL handle gives the
 * last error of a gwtf_learn_create, or of a call with a NULL handle, on the
 * calling thread. */
const char *gwtf_learn_last_error(const gwtf_learn_t *h);

/* ---- Answers drawn from logits ----
 *
 * Per row of logits x, with temperature T, top_k k, top_p p, min_p q and the
 * row's random number u: w_j = exp((x_j - max x) / T), and the tokens in the
 * order of descending x, equal ones by ascending index.  A token stays
 * that is
 *   among the first K, K = min(k, number of x above -infinity); k <= 0: no bound,
 *   among the first n, the least n whose sum of w is p times that of the first
 *     K or more; p >= 1: no bound,
 *   and has w >= q.
 * The first token always stays; T = 0 leaves it alone.  Of those that stay,
 * by ascending index, the token drawn is the first whose sum of w, its own
 * and of those before it, is above u times that of all:
 *   ids = its index, logp = ln of its share of the sum, kept = how many stay.
 * Sums, w and their products with u and p are held in 64 bits, so that a draw is
 * that of exact arithmetic unless u falls within some 1e-13 of a border, p
 * within some 1e-11 (V 2^-61 where that is more), or q, below 1, within 1e-13 of itself of
 * a w; a w below 2^-600 may count as 0.  logp is rounded once from 64
 * bits, but where nothing is filtered (the numbers top_k <= 0, top_p >= 1, min_p 0)
 * it comes from a sum that is off by 2^-24 (2 ln 2 (log2 V + 2) + 12) of itself at most.
 * u counts as within [0, 1)
 * (a NaN as 0).  An entry of -infinity is masked; a row of nothing else gives
 * ids -1, logp -infinity, kept 0.  A row with a NaN or +infinity, and one
 * whose settings are out of range (below), gives ids -1, logp NaN, kept 0.
 *
 * A setting is the same number for all rows, which the call refuses out of
 * range, or one for each row. */
typedef struct {
    int64_t num_tokens, vocab;  /* N >= 0, 1 <= V < 2^31 */
    int32_t type, uniform_type; /* GWTF_TYPE_* of logits, GWTF_UNIFORM_* of u */
    int32_t top_k;
    double temperature;         /* finite, >= 0 */
    double top_p;               /* >= 0 */
    double min_p;               /* within [0, 1] */
    const float *temperatures;  /* [N], or NULL = temperature */
    const int32_t *top_ks;      /* [N], or NULL = top_k */
    const float *top_ps;        /* [N], or NULL = top_p */
    const float *min_ps;        /* [N], or NULL = min_p */
    const void *logits;         /* [N][V], rows any distance apart */
    int64_t logits_stride;
    const void *u;              /* [N] */
    int32_t *ids;               /* [N] */
    float *logp;                /* [N] or NULL */
    int32_t *kept;              /* [N] or NULL */
} gwtf_learn_sample_t;
gwtf_status_t gwtf_learn_sample(gwtf_learn_t *h, const gwtf_learn_sample_t *a);

/* ---- Parameters ----
 *
 * A tensor of a node's parameters: `size` adjacent values. */
typedef struct {
    int64_t size;               /* 0 <= size < 2^35 */
    int32_t type, grad_type;    /* GWTF_TYPE_* of param; of grad: that type or GWTF_TYPE_F32 */
    const void *grad;           /* [size] */
    void *param;                /* [size] */
    float *master;              /* [size], the parameters in 32 bits, or NULL */
    void *m, *v;                /* [size], in the form of the list */
    float *m_scale, *v_scale;   /* [ceil(size / GWTF_STATE_BLOCK)]; with GWTF_STATE_F8 only */
    float weight_decay;         /* finite */
    uint32_t site;              /* number of the tensor; with GWTF_STATE_F8 only */
} gwtf_learn_tensor_t;

/* Makes a list of tensors, a HOST array, on the handle's GPU: a table of where
 * they lie, 80 bytes a tensor and 4 for each 2048 of its values, which the calls
 * that are given the list read.  All arrays have to stay where they are as long
 * as the list is in use, and none that a step writes may overlap another.  With
 * GWTF_STATE_NONE of a tensor size, grad_type and grad count alone.  At most 2^42
 * values in all.  Lists are made and destroyed outside of stream captures. */
gwtf_status_t gwtf_learn_list_create(gwtf_learn_t *h, int64_t num_tensors, const gwtf_learn_tensor_t *tensors, int32_t form,
                                     gwtf_learn_list_t **out);

/* Frees the list, after the work of its device that may read it; NULL-safe. */
void gwtf_learn_list_destroy(gwtf_learn_list_t *list);

/* norm = scale * sqrt(sum of the squares of all gradients) and
 * factor = scale * min(1, max_norm / norm), NaN where norm is not a finite
 * number of 32 bits: what the gradients are to be multiplied with, for gwtf_learn_adamw.
 * Sums are held in 64 bits.  The list may have any form. */
typedef struct {
    const gwtf_learn_list_t *list;
    double max_norm; /* >= 0; +infinity: no bound */
    double scale;    /* finite in 32 bits, >= 0 */
    float *norm;     /* [1], or NULL */
    float *factor;   /* [1], or NULL */
} gwtf_learn_grad_norm_t;
gwtf_status_t gwtf_learn_grad_norm(gwtf_learn_t *h, const gwtf_learn_grad_norm_t *a);

/* One step of AdamW on every tensor, in place, in 32 bits:
 *   g = factor * grad
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
 *   p = p - lr (m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps) + weight_decay p)
 * where p is master, rounded to param too, or param itself where master is
 * NULL, and a denominator below 2^-126 counts as 2^-126 (with eps 0, values whose
 * gradients have all been 0 stay).  With a factor, or a rate at lr_at, that is not a
 * finite number, or a step number below 1 at step_at, nothing is written.
 *
 * GWTF_STATE_F8: m and v are values times the scale of their block, a power of
 * two that puts the block's largest magnitude into (224, 448] of m, (28672, 57344]
 * of v (2^-126 at least).  The step takes the new m and v as they are;
 * what is kept of them is one of the two 8-bit values around, the upper one with
 * the probability of the remainder, so that an average which moves by less
 * than half a step of 8 bits moves at all: with r = 16 bits of Philox4x32-10
 * under the key (low, high half of `seed`) and the counter (i / 8, site, low, high
 * half of step), word (i % 8) / 2, its low half for even i, for value i of a
 * tensor, the magnitude in steps of 8 bits plus (r + 0.5) 2^-16 (rounded to 32 bits
 * where the magnitude is below the code's smallest normal number) is cut down to a
 * whole number.  A v above 0 is kept above 0, so that m / sqrt(v) stays bounded.
 * A NaN or infinity among a block's new values makes its scale NaN. */
typedef struct {
    const gwtf_learn_list_t *list; /* of GWTF_STATE_F32 or GWTF_STATE_F8 */
    int64_t step;                  /* >= 1, number of this step */
    const int64_t *step_at;        /* [1], to be read in its place, or NULL */
    double lr;                     /* finite in 32 bits */
    const float *lr_at;            /* [1], to be read in its place, or NULL */
    double beta1, beta2;           /* within [0, 1), in 32 bits too */
    double eps;                    /* finite in 32 bits, >= 0 */
    uint64_t seed;                 /* with GWTF_STATE_F8 only */
    const float *factor;           /* [1], or NULL = 1 */
} gwtf_learn_adamw_t;
gwtf_status_t gwtf_learn_adamw(gwtf_learn_t *h, const gwtf_learn_adamw_t *a);

#ifdef __cplusplus
}
#endif
#endif /* GWTF_LEARN_H */
