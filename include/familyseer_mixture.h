/*
 * familyseer_mixture.h -- C ABI: mixtures of family models.
 *
 * The tuner keeps a cost model per subgraph family and finds a subgraph's family by static analysis
 * (Section 4.1; find_family in Algorithm 1).  Candidates of a subgraph that no family owns yet have no
 * such model.  A learned router then chooses, for every statement row (here: a token), the k family
 * models (here: experts) that score it, and how much each has to say.  The calls are the operators of
 * such a router, forwards and backwards:
 *
 *   fs_embed               tokens, or bags of tokens such as the leaves that a row reaches in an
 *                          ensemble (leaf_idx of fs_score_families), to scaled sums of learned vectors
 *   fs_route               logits to the k chosen experts of every token and their weights
 *   fs_expert_plan         the choices, grouped by expert: which slot each takes
 *   fs_expert_gather       tokens' rows into the experts' slots
 *   fs_expert_combine      the slots' results back to the tokens, weighted
 *   fs_..._backward        the gradients
 *
 * Conventions are those of familyseer.h: FS_OK or a negative code with fs_last_error(); every argument
 * error is found on the host before anything is enqueued; HOST / DEVICE says which memory a pointer
 * means; work is enqueued on `stream` and the call returns without waiting.  Three things differ.
 * The calls neither allocate nor use the library's scratch: where one needs working memory, the
 * caller hands it in (..._workspace_bytes says how much), and it is free again when the call's work
 * has finished; calls on different streams therefore never disturb each other, and every call can be recorded
 * into a HIP graph at any time.  Results are the same, bit for bit, from run to run: nothing is added up by atomics.
 * And matrices have a row stride, counted in elements, so that a part of a wider matrix can be
 * handed in; a row's elements are adjacent.  Pointers are aligned to the size of an element, workspaces to 256 bytes.
 * Outputs must not overlap inputs, workspaces or each other.
 *
 * fs_profile_begin counts these calls among the kernel classes of familyseer.h: routing as FS_KERNEL_TOPK, the exchange and
 * lookups as FS_KERNEL_PACK, gradients as FS_KERNEL_TRAIN_OTHER.
 *
 * Sums, softmax statistics and gradients are held in fp32 or wider and rounded once (to nearest, ties to
 * even) where the output has fewer bits.
 */
#ifndef FAMILYSEER_MIXTURE_H
#define FAMILYSEER_MIXTURE_H

#include "familyseer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of a matrix. */
enum { FS_F32 = 0, FS_BF16 = 1, FS_F16 = 2 };
/* Types of token ids. */
enum {
    FS_ID_I32 = 0,
    FS_ID_I64 = 1,
    FS_ID_U16 = 2   /* leaf_idx of fs_score_families; 0 to 65535, so that a -1 of 16 bits is 65535 */
};
/* Scores of an expert, from its logit. */
enum {
    FS_SCORE_SOFTMAX = 0,  /* exp(l_e) / sum over the token's experts */
    FS_SCORE_SIGMOID = 1   /* 1 / (1 + exp(-l_e))                     */
};

#define FS_MAX_EXPERTS 1024
#define FS_MAX_CHOICES 16      /* experts of a token                                             */
#define FS_MAX_WIDTH 1048576   /* elements of a row that travels or is looked up                 */

/* ---- routing ------------------------------------------------------------------------------ */

typedef struct fs_route_params {
    int32_t n_experts;   /* 1 .. FS_MAX_EXPERTS                                                    */
    int32_t k;           /* 1 .. FS_MAX_CHOICES, <= n_experts                                      */
    int32_t score;       /* FS_SCORE_SOFTMAX or FS_SCORE_SIGMOID                                   */
    int32_t renormalise; /* 1: a token's weights are divided by their sum; 0: they are the scores  */
    int32_t n_groups;    /* 1: every expert may be chosen; else n_experts is a multiple of it:
                            groups of consecutive experts                                          */
    int32_t top_groups;  /* 1 .. n_groups: experts are chosen from so many groups                  */
    int32_t group_best;  /* 1 or 2: a group ranks by the sum of its so many best keys (scores, where
                            there is no bias); by what it has, if fewer are eligible               */
    float scale;         /* factor on all weights, finite                                          */
} fs_route_params;

/*
 * For every token the k eligible experts with the largest keys, by (key descending, expert ascending), and
 * their weights.  An expert's key is its logit, or, with a bias, score + bias: the bias balances how often
 * experts are chosen and does not enter the weights.  Keys and groups' sums are compared as in 64-bit
 * arithmetic.  Not eligible (masked) are experts whose logit is -infinity or NaN, or whose key is; a logit of +infinity
 * counts as the largest float.  Masked experts have the score 0.  Groups rank by (sum descending, group ascending);
 * a group without an eligible expert is never taken.
 * Where fewer than k experts are to be had, the remaining entries are expert -1 with the weight 0.
 */
int fs_route(const fs_route_params *params /* HOST */, int64_t n_tokens, const void *logits /* DEVICE */,
             int32_t logit_type, int64_t logit_stride, const float *bias /* DEVICE, n_experts, or NULL */,
             int32_t *expert /* DEVICE out, n_tokens*k */, float *weight /* DEVICE out, n_tokens*k */, void *stream);

/*
 * The logits' gradient: d_logits[t][e] = sum over j of d_weight[t][j] * d weight[t][j] / d logits[t][e] for the
 * choice `expert` that fs_route made of the same logits; the choice itself has no gradient, and a masked expert's is 0.
 * Entries of `expert` outside [0, n_experts) are skipped, whatever d_weight holds there.
 */
int fs_route_backward(const fs_route_params *params /* HOST */, int64_t n_tokens, const void *logits /* DEVICE */,
                      int32_t logit_type, int64_t logit_stride, const int32_t *expert /* DEVICE */,
                      const float *d_weight /* DEVICE, n_tokens*k */, void *d_logits /* DEVICE out, of logit_type */,
                      int64_t d_logit_stride, void *stream);

/* ---- the exchange between tokens and experts ------------------------------------------------- */

/*
 * Groups n_tokens*k choices by expert.  Expert e gets the slots [first[e], first[e+1]); order[s] is the choice in slot
 * s, as token*k + j, ascending within an expert; place[token*k + j] is that choice's slot.  Choices outside
 * [0, n_experts) get no slot: their place is -1, and order is -1 from first[n_experts] on.
 * n_tokens*k < 2^31.
 */
size_t fs_expert_plan_workspace_bytes(int64_t n_tokens, int32_t k, int32_t n_experts);
int fs_expert_plan(int64_t n_tokens, int32_t k, int32_t n_experts, const int32_t *expert /* DEVICE */,
                   int32_t *first /* DEVICE out, n_experts+1 */, int32_t *order /* DEVICE out, n_tokens*k */,
                   int32_t *place /* DEVICE out, n_tokens*k */, void *work /* DEVICE */, size_t work_bytes, void *stream);

/* xs[place[t*k + j]] = x[t]; the slots from first[n_experts] on are filled with 0.  x: n_tokens rows, xs: n_tokens*k. */
int fs_expert_gather(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *x /* DEVICE */, int32_t type,
                     int64_t x_stride, const int32_t *first, const int32_t *place, void *xs /* DEVICE out */,
                     int64_t xs_stride, void *stream);

/*
 * out[t] = sum over j ascending of weight[t*k + j] * y[place[t*k + j]], from 0; without weights (NULL) every weight is 1,
 * which is the gradient of fs_expert_gather.  Choices without a slot add nothing, whatever y and weight hold.
 */
int fs_expert_combine(int64_t n_tokens, int32_t k, int32_t width, const void *y /* DEVICE */, int32_t type, int64_t y_stride,
                      const int32_t *place, const float *weight /* DEVICE or NULL */, void *out /* DEVICE out */,
                      int64_t out_stride, void *stream);

/*
 * Gradients of a weighted fs_expert_combine: d_y[place] = weight * d_out[t], 0 in the slots from first[n_experts] on, and
 * d_weight[t*k + j] = the product of d_out[t] with y[place], 0 without a slot.
 */
int fs_expert_combine_backward(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *d_out /* DEVICE */,
                               int32_t type, int64_t d_out_stride, const void *y /* DEVICE, of the same type */, int64_t y_stride,
                               const int32_t *first, const int32_t *place, const float *weight /* DEVICE */,
                               void *d_y /* DEVICE out, of the same type */, int64_t d_y_stride,
                               float *d_weight /* DEVICE out, n_tokens*k */, void *stream);

/* ---- embedding ----------------------------------------------------------------------------- */

/*
 * out[r] = scale * sum over c of table[col_base[c] + ids[r*n_cols + c]], c < n_cols, in an order that depends on the
 * sizes alone: at most 256 terms after each other in fp32, such sums in 64 bits.  One column is the plain lookup; without col_base its entries count as 0.  Leaves of an ensemble: FS_ID_U16 ids with
 * col_base = the tree_off of fs_model_create, n_cols = n_trees.  Ids whose row, col_base + id, is outside
 * [0, n_vocab) add nothing (for padding: -1 without col_base, or any id past the table; 16-bit ids have no -1).  out_type is the table's type or FS_F32.
 * n_rows*n_cols < 2^31.
 */
int fs_embed(int32_t n_vocab, int32_t width, const void *table /* DEVICE */, int32_t table_type, int64_t table_stride,
             int64_t n_rows, int32_t n_cols, const void *ids /* DEVICE, n_rows*n_cols */, int32_t id_type,
             const int32_t *col_base /* DEVICE, n_cols, or NULL */, float scale, void *out /* DEVICE out */, int32_t out_type,
             int64_t out_stride, void *stream);

/*
 * The table's gradient: d_table[v] = scale * sum of d_out[r] over the (r, c) whose row is v, in an order that depends on
 * the ids alone; rows that no id names get 0.  accumulate = 1: it is added to what d_table holds.  d_table_type is d_out's
 * type or FS_F32.
 */
size_t fs_embed_backward_workspace_bytes(int32_t n_vocab, int32_t width, int32_t d_out_type, int64_t n_rows, int32_t n_cols);
int fs_embed_backward(int32_t n_vocab, int32_t width, const void *d_out /* DEVICE */, int32_t d_out_type, int64_t d_out_stride,
                      int64_t n_rows, int32_t n_cols, const void *ids /* DEVICE */, int32_t id_type,
                      const int32_t *col_base /* DEVICE or NULL */, float scale, int32_t accumulate, void *d_table /* DEVICE out */,
                      int32_t d_table_type, int64_t d_table_stride, void *work /* DEVICE */, size_t work_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FAMILYSEER_MIXTURE_H */
