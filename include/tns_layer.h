/*
 * tns_layer -- operators of an attention layer over sampled neighbourhoods, on one AMD MI355X (gfx950):
 *   - attention of targets over ragged lists of events (the dense result of tns_run, or whole histories), with a learned
 *     bias by buckets of the events' age or place, and its gradients;
 *   - what stands between two such layers: norm of the branch, its gate and scale, the sum with the residual and the norm
 *     before the next branch, in one pass, and its gradients;
 *   - the loss of a student's scores of all candidates against a teacher's highest ones, with its gradient.
 *
 * Plain C ABI with the conventions of include/tns_train.h (types T, status codes, streams, workspaces; the same inputs give the same
 * bits).  Output and workspace buffers must not overlap each other or inputs.  Two calls that may run at once, captured ones among them,
 * need workspaces of their own.
 */
#ifndef TNS_LAYER_H
#define TNS_LAYER_H

#include "tns_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- attention over event lists -----------------------------------------------------------------------
 *
 * List s holds the rows d_rowptr[s] .. d_rowptr[s+1]-1, one event each; target s has one query per head.  Head h reads the keys and
 * values of head h / (heads / kv_heads).  For every event i of the list and every head:
 *     age    = max(t - ts, 0) in fp32 (a difference that is not a number counts as 0, an infinite one as the largest fp32 value);
 *              without d_ts: the number of events of the list that are newer
 *     bucket = number of edges <= age
 *     score  = scale * q . k + table[bucket][h]
 *     out    = sum p v, p = softmax of the scores over the list
 * An event is left out, whatever its rows of k and v hold, where its mask is 0, its index is outside [0, num), or, head by head, its
 * table entry is -infinity (a finite one, however low, leaves nothing out).  Where no event is left out is zero, and its gradients are.
 * Scores are rounded to fp32: beside a table entry of 1e9, say, what q . k says below 64 is lost.
 *
 *   S, d_rowptr[S+1]  lists, as in tns_recur.  S < 2^31
 *   rows              rows that the events' arrays have room for, at least d_rowptr[S]; rows from d_rowptr[S] on do not count,
 *                     whatever they hold.  < 2^40 (calls of more than 2^34 rows times 256 channels of all heads are refused)
 *   num               rows of k and v with d_index, < 2^31 (without: k and v have `rows` rows, and num is 0)
 *   heads, kv_heads   heads of q; of k and v.  kv_heads divides heads, heads / kv_heads <= 8, heads <= 1024
 *   head_dim          1 .. 256
 *   buckets           0: no bias (no edges, no table); otherwise 1 .. 256, and buckets * heads <= 2048
 *   flags             TNS_NEWEST_FIRST: a list's first row is its newest event (of account without d_ts only).  TNS_ZERO_BEYOND: the
 *                     rows from d_rowptr[S] on of d_dk and d_dv are written as zeros; otherwise they are not written
 *   d_q               T [S, heads, head_dim], ld_q elements from one target to the next (>= heads * head_dim); aligned to T
 *   d_k, d_v          T [rows or num, kv_heads, head_dim], ld_k / ld_v from one row to the next, < 2^22
 *   d_index[rows]     row of k and v that holds the event's; may be NULL (row i holds event i's)
 *   d_mask[rows]      bytes, 0: the event is left out; may be NULL
 *   d_t[S], d_ts[rows]   times of the targets and of the events; both or neither
 *   d_edges[buckets-1]   non-decreasing; may be NULL with one bucket
 *   d_table           [buckets, heads]
 */
typedef struct {
    int64_t S, rows, num;
    int32_t heads, kv_heads, head_dim, dtype, buckets, flags;
    const int64_t *d_rowptr;
    const void *d_q, *d_k, *d_v;
    int64_t ld_q, ld_k, ld_v;
    const int32_t *d_index;
    const uint8_t *d_mask;
    const float *d_t, *d_ts, *d_edges, *d_table;
    double scale;
} tns_attend;

/* Bytes of workspace of tns_attend_run and tns_attend_grad, and of what the first saves for the second.  Any may be NULL.  Depends on S,
   rows, heads, kv_heads, head_dim, dtype and buckets alone; the pointers are not looked at. */
TNS_API int tns_attend_workspace(const tns_attend *a, size_t *run_bytes, size_t *grad_bytes, size_t *saved_bytes);

/*
 *   d_out       T [S, heads, head_dim], dense
 *   d_saved     saved_bytes, 256-byte aligned, for tns_attend_grad; may be NULL
 *   d_workspace run_bytes, 256-byte aligned
 */
TNS_API int tns_attend_run(const tns_attend *a, void *d_out, void *d_saved, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Gradients of a scalar, given its gradient by the outputs.  Refuses d_index: the gradient by a shared row is a sum over its events.
 *   a, d_saved  as given to, and written by, tns_attend_run
 *   d_dout      T [S, heads, head_dim], dense
 *   d_dq        T [S, heads, head_dim], dense
 *   d_dk, d_dv  T [rows, kv_heads, head_dim], dense; rows of events that are left out are zero
 *   d_dtable    [buckets, heads]; NULL without buckets; summed in a fixed order
 */
TNS_API int tns_attend_grad(const tns_attend *a, const void *d_saved, const void *d_dout, void *d_dq, void *d_dk, void *d_dv, float *d_dtable,
                            void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- between two layers --------------------------------------------------------------------------------
 *
 * For every row, channel by channel:
 *     out  = x + scale * sigmoid(gate) * post * norm(branch)
 *     next = pre * norm(out)                     (of out before it is rounded to T)
 * norm(v) = v / sqrt(mean(v^2) + eps), with TNS_CENTER of v - mean(v).  Without d_post the branch is taken as it is, without d_gate and
 * d_scale these factors are 1.  Squares are summed in fp32: they hold for values up to 1e17, and without eps from 1e-17 on.
 *
 *   rows < 2^40, dim 1 .. 8192
 *   d_x, d_branch, d_gate   T [rows, dim] with ld; d_gate may be NULL
 *   d_scale, d_post, d_pre  [dim], may be NULL; without d_pre there is no next
 *   eps                     >= 0 (with 0 a row without spread is 0 / 0)
 */
enum { TNS_CENTER = 1 };
typedef struct {
    int64_t rows;
    int32_t dim, dtype, flags, reserved; /* reserved: 0 */
    const void *d_x, *d_branch, *d_gate;
    int64_t ld_x, ld_branch, ld_gate;
    const float *d_scale, *d_post, *d_pre;
    double eps;
} tns_block;

/* d_out, d_next: T [rows, dim], dense; d_next NULL exactly where d_pre is */
TNS_API int tns_block_run(const tns_block *b, void *d_out, void *d_next, void *hip_stream);

/*
 * Gradients of a scalar, given those by out (d_dout) and next (d_dnext); either may be NULL (zero), d_dnext has to be without d_pre.
 *   d_dx, d_dbranch, d_dgate    T [rows, dim], dense; d_dgate NULL exactly where d_gate is
 *   d_dscale, d_dpost, d_dpre   [dim], each may be NULL, and has to be where the weight is; summed over the rows in a fixed order
 */
TNS_API int tns_block_workspace(int64_t rows, int32_t dim, size_t *grad_bytes);
TNS_API int tns_block_grad(const tns_block *b, const void *d_dout, int64_t ld_dout, const void *d_dnext, int64_t ld_dnext, void *d_dx, void *d_dbranch, void *d_dgate,
                           float *d_dscale, float *d_dpost, float *d_dpre, void *d_workspace, size_t workspace_bytes, void *hip_stream);

/* ---- distillation from a teacher's highest scores --------------------------------------------------------
 *
 * The student scores V candidates of a row, q = softmax(logits / temperature); of the teacher the K highest scores and their candidates
 * are known.  Without d_lse  p = softmax over them of teacher / temperature, and
 *     loss = weight * sum_k p_k (log p_k - log q[id_k])
 * With d_lse, the logarithm of the sum over all the teacher's candidates of exp(score / temperature), p_k = exp(teacher_k / temperature - lse),
 * and the mass of the others, rest = max(1 - sum p, 0), is compared as a whole:
 *     loss = weight * (sum_k p_k (log p_k - log q[id_k]) + rest (log rest - log(sum of q over the candidates that no id names)))
 * An id outside [0, V) and a teacher's score of -infinity have p = 0 (the latter's id is named all the same); terms of p = 0 and rest = 0
 * are 0; a loss is infinite where p (rest) is above 0 and the student's q (of all others) is 0.  A candidate named twice has two terms.
 * Without d_lse a row without any p > 0 has loss 0 and gradient 0.
 * A row of weight 0 is not read, whatever lies there: its loss and gradient are 0.
 *
 *   B, V, K         rows, candidates, ids of a row: B, V < 2^31, V >= 1, 0 <= K <= 1024
 *   d_logits        T [B, V] with ld (>= V)
 *   d_ids, d_teacher   [B, K]
 *   d_lse, d_weight    [B], may be NULL (weight 1)
 *   temperature     > 0
 *   d_loss [1]      scale * sum of the rows' losses
 *   d_rows [B]      weight * loss of each row; may be NULL
 *   d_dlogits       T [B, V], dense, gradient of *d_loss; may be NULL
 *   d_workspace     tns_distill_workspace() bytes, 256-byte aligned
 */
typedef struct {
    int64_t B, V;
    int32_t K, dtype;
    const void *d_logits;
    int64_t ld_logits;
    const int32_t *d_ids;
    const float *d_teacher, *d_lse, *d_weight;
    double temperature, scale;
} tns_distill_desc;
TNS_API int tns_distill_workspace(int64_t B, int64_t V, int32_t K, size_t *bytes);
TNS_API int tns_distill(const tns_distill_desc *d, float *d_loss, float *d_rows, void *d_dlogits, void *d_workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* TNS_LAYER_H */
