/*
 * tns_train -- operators of a training step on sampled neighbourhoods, on one AMD MI355X (gfx950):
 *   - a gated linear recurrence over ragged lists of events (the dense result of tns_run, or whole
 *     histories of nodes), its gradients, and its step for one event per node;
 *   - the paired log-ratio loss of true links against sampled ones, with its gradients;
 *   - AdamW over all tensors of a model in one launch, its states in 32 or in 8 bits.
 *
 * Plain C ABI with the conventions of include/tns.h.  All pointers are DEVICE unless marked HOST; buffers
 * are the caller's and are not kept after the queued work is done (tns_adamw keeps the addresses it was
 * created with).  Calls enqueue work on the given stream of the calling thread's current device (tns_adamw:
 * of its own device) and never block, allocate or free, creating and destroying an optimizer excepted.
 * They may be captured into a graph.  Functions return 0 (TNS_OK) or a negative tns_status; details via
 * tns_last_error().  Results do not depend on timing: the same inputs give the same bits.
 */
#ifndef TNS_TRAIN_H
#define TNS_TRAIN_H

#include "tns.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Type of the values called T below; sums, states and statistics are fp32 whatever it is. */
enum { TNS_F32 = 0, TNS_BF16 = 1 };

/* ---- gated linear recurrence ------------------------------------------------------------------------
 *
 * List s holds the rows d_rowptr[s] .. d_rowptr[s+1]-1.  Walked from its oldest event to its newest, for
 * every channel on its own:
 *     z = sigmoid(u),  f = (1 - z) exp(-decay * gap),  h = f h_before + z x
 * h_before of a list's first event is h0 (zero without d_h0); gap = max(t - t_before, 0), where t_before of
 * the first event is t0 (without d_t0 that gap is 0).  A gap that is not a number counts as 0, an
 * infinite one as the largest fp32 value.  Without d_ts and d_decay f = 1 - z.
 * Relative errors: of z and 1 - z (1.5 |u| + 6) 2^-24 at most where they are normal numbers, of exp(-decay * gap)
 * (2.5 decay gap + 3) 2^-24.
 * A state that is not finite stays so over the rest of its list, where an infinite one may become NaN.
 *
 *   S, d_rowptr[S+1]  lists; d_rowptr[0] = 0, non-decreasing, as tns_run writes it.  S < 2^31
 *   rows              rows that the arrays have room for, at least d_rowptr[S]; rows from d_rowptr[S] on are
 *                     neither read nor, without TNS_ZERO_BEYOND, written.  rows < 2^40
 *   dim, dtype        channels per row, 1 .. 2^16; TNS_F32 | TNS_BF16
 *   flags             TNS_NEWEST_FIRST: a list's first row is its newest event (tns_run's order under the
 *                     recent policy); otherwise its oldest.  TNS_ZERO_BEYOND: the rows from d_rowptr[S] on of d_h, d_du
 *                     and d_dx are written as zeros, so that they can be summed over without reading d_rowptr[S] back
 *   d_u, d_x          T [rows, dim], ld_u / ld_x elements from one row to the next (>= dim); aligned to T
 *   d_ts [rows], d_decay [dim]   both or neither; decay >= 0 (with a negative one the state grows, and what rows do
 *                     to a state, multiplied up over a long list, may overflow)
 *   d_h0 [S, dim], d_t0 [S]      may be NULL; d_t0 needs d_ts
 */
enum { TNS_NEWEST_FIRST = 1, TNS_ZERO_BEYOND = 4 };
typedef struct {
    int64_t S, rows;
    int32_t dim, dtype, flags, reserved; /* reserved: 0 */
    const int64_t *d_rowptr;
    const void *d_u, *d_x;
    int64_t ld_u, ld_x;
    const float *d_ts, *d_decay, *d_h0, *d_t0;
} tns_recur;

/* Bytes of workspace of tns_recur_run and tns_recur_grad and of the states that the first saves for the second.  Any may be NULL.
   Depends on S, rows, dim and dtype alone; the pointers are not looked at. */
TNS_API int tns_recur_workspace(const tns_recur *r, size_t *run_bytes, size_t *grad_bytes, size_t *saved_bytes);

/*
 * States.
 *   d_h         T [rows, dim] with ld_h, the state after every event; may be NULL
 *   d_h_last    [S, dim], the state after a list's newest event (a list without events: h0, or zero); may be NULL
 *   d_saved     saved_bytes, 256-byte aligned, for tns_recur_grad; may be NULL
 *   d_workspace run_bytes, 256-byte aligned
 */
TNS_API int tns_recur_run(const tns_recur *r, void *d_h, int64_t ld_h, float *d_h_last, void *d_saved, void *d_workspace,
                          size_t workspace_bytes, void *hip_stream);

/*
 * Gradients of a scalar, given its gradient by the states (d_dh) and by the last states (d_dh_last); either may be NULL (zero).
 *   r, d_saved  as given to, and written by, tns_recur_run
 *   d_du, d_dx  T [rows, dim] with ld_du / ld_dx, gradients by u and x
 *   d_ddecay    [dim], may be NULL; summed over all rows in a fixed order
 *   d_dh0       [S, dim], may be NULL
 */
TNS_API int tns_recur_grad(const tns_recur *r, const void *d_saved, const void *d_dh, int64_t ld_dh, const float *d_dh_last,
                           void *d_du, int64_t ld_du, void *d_dx, int64_t ld_dx, float *d_ddecay, float *d_dh0,
                           void *d_workspace, size_t workspace_bytes, void *hip_stream);

/*
 * One event for each of B nodes: h = f state[id] + z x, written to state[id] and, as T, to d_out.
 *   d_ids[B]           rows of the state table; ids outside [0, num_ids) hold no state: their rows of d_out are zero.
 *                      The other ids have to be distinct (otherwise one of their events wins, in part or as a whole)
 *   d_u, d_x, d_out    T [B, dim]; d_out may be NULL
 *   d_ts[B], d_decay[dim], d_state_ts[num_ids]   all or none; state_ts[id] becomes ts
 *   d_state            [num_ids, dim]
 */
TNS_API int tns_recur_step(int64_t B, int64_t num_ids, int32_t dim, int32_t dtype, const int32_t *d_ids, const void *d_u, int64_t ld_u,
                           const void *d_x, int64_t ld_x, const float *d_ts, const float *d_decay, float *d_state, float *d_state_ts,
                           void *d_out, int64_t ld_out, void *hip_stream);

/* ---- paired log-ratio loss --------------------------------------------------------------------------
 *
 * The log ratio of a true link (anchor, pos) to a sampled one (anchor, neg) is the difference of their
 * scores, the scalar products of their embeddings; with ref it is taken relative to a frozen model's:
 *     m = beta * (anchor . pos - anchor . neg_k - ref)
 *     loss = scale * sum weight * ((1 - smoothing) softplus(-m) + smoothing softplus(m))
 * A term whose factor is 0 is left out: without smoothing a pair of margin +infinity (ref = -infinity: the frozen model rules the
 * link out) adds nothing to the loss, as its gradients are 0.
 *
 *   B, K         events and sampled links of each; B * K < 2^40, dim 1 .. 2^16
 *   d_anchor, d_pos   T [B, dim] with ld; d_neg T [B, K, dim], dense
 *   d_ref, d_weight   [B, K], may be NULL (0 and 1).  A pair of weight 0 is not read, whatever lies there: its
 *                margin and its gradients are 0, and an event all of whose weights are 0 has zero gradients
 *   d_loss [1]
 *   d_margin [B, K]   m; may be NULL
 *   d_danchor, d_dpos, d_dneg   T, dense, gradients of the loss; all or none
 *   d_workspace  tns_pair_loss_workspace() bytes, 256-byte aligned
 */
typedef struct {
    int64_t B, K;
    int32_t dim, dtype;
    const void *d_anchor, *d_pos, *d_neg;
    int64_t ld_anchor, ld_pos;
    const float *d_ref, *d_weight;
    double beta, smoothing, scale; /* 0 <= smoothing <= 1 */
} tns_pairs;
TNS_API int tns_pair_loss_workspace(int64_t B, int64_t K, int32_t dim, size_t *bytes);
TNS_API int tns_pair_loss(const tns_pairs *p, float *d_loss, float *d_margin, void *d_danchor, void *d_dpos, void *d_dneg,
                          void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- AdamW ------------------------------------------------------------------------------------------
 *
 * One step over all tensors.  m, v, codes and scales are rounded to fp32 operation by operation and so have the same bits wherever
 * they are computed; a weight's change is a product with an approximate reciprocal, right to 8 parts in 2^24:
 *     g = grad * *d_grad_scale,  m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) (g g)
 *     param = param (1 - lr weight_decay) - (lr / (1 - beta1^t)) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 *
 * State of 8 bits: m and r = sqrt(v) as OCP e4m3 codes with an fp32 scale for every 256 weights of a tensor,
 * the largest magnitude over 448; m = code * scale, v = (code * scale)^2.  A new m or r is rounded to one
 * of the two codes around it at random so that it is right on average (an average that moves by a tenth of
 * a percent a step would otherwise stay on its code for ever).  v is not: a square is larger by the rounding's
 * variance, which adds up over the steps that v averages.  With beta2 = 0.999 and normal gradients v is some 5 % high
 * on average after thousands of steps (r 1 %), 0.7 to 1.6 times its value for a single weight over thousands
 * of steps, 0.25 to 3 times at a single step.  Only normal codes are written: an m below 2^-6 of a scale becomes 0, an r
 * below that is raised to it, so that no step is divided by a zero the state cannot express; where all 256
 * are below 2^-100 the codes and the scale are 0.  The sixteen random bits of weight i, the same for m and r, are
 * those numbered 16 (i mod 4) of mix(key + G (i / 4 + 1)), key = mix(seed + G t), with the mixing function mix and
 * the increment G of splitmix64; i counts from a tensor's first weight on and tensors follow each other, each
 * rounded up to 256.
 * States that are not finite poison their 256 weights, as they would poison single ones in 32 bits.
 */
typedef struct {
    int64_t n;                 /* weights, 0 .. 2^36; fewer than 2^36 in all tensors, each rounded up to 4096 */
    float *d_param;            /* fp32                                                                     */
    void *d_copy;              /* bf16 [n], may be NULL: receives the new weights, rounded to nearest       */
    const void *d_grad;        /* of the configuration's grad_dtype                                         */
    void *d_m, *d_v;           /* fp32 [n], or e4m3 codes [n] (d_v: of sqrt(v))                              */
    float *d_m_scale, *d_v_scale; /* 8 bits: [(n + 255) / 256]                                               */
    double weight_decay;
} tns_adamw_tensor;
typedef struct {
    double beta1, beta2, eps;  /* 0 <= beta < 1, eps >= 0                                                    */
    uint64_t seed;
    int32_t state_bits;        /* 8 | 32                                                                    */
    int32_t grad_dtype;        /* TNS_F32 | TNS_BF16                                                        */
    int32_t device, reserved;
} tns_adamw_config;
typedef struct tns_adamw tns_adamw;

/* `tensors` (HOST, count entries) is copied; the buffers they name have to stay where they are.  Buffers of one optimizer must not overlap. */
TNS_API int tns_adamw_create(const tns_adamw_config *cfg, int32_t count, const tns_adamw_tensor *tensors, tns_adamw **out);
/* Step t >= 1.  A captured step keeps its lr and t.  d_grad_scale [1] may be NULL (1); where it is 0 or not finite nothing is changed: the step is left out. */
TNS_API int tns_adamw_step(tns_adamw *opt, double lr, int64_t t, const float *d_grad_scale, void *hip_stream);
/* Waits for the device; opt may be NULL. */
TNS_API int tns_adamw_destroy(tns_adamw *opt);

#ifdef __cplusplus
}
#endif
#endif /* TNS_TRAIN_H */
