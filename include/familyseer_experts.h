/*
 * familyseer_experts.h -- C ABI: networks as the experts of a mixture.
 *
 * familyseer_mixture.h shares rows (tokens) out over experts and brings their results back.  Where an expert is a
 * small network instead of a tree ensemble, the rows in its slots meet its weights in a matrix product.  The calls
 * here are those products, forwards and backwards, the same in 8-bit integers, and the loss that a model which
 * answers with logits -- a router, or a wider one -- learns from when of its teacher only the largest logits are kept:
 *
 *   fs_expert_matmul            rows in slots times their expert's weights; also the rows' gradient
 *   fs_expert_matmul_backward   the weights' gradient
 *   fs_quantize_rows            rows in 8-bit integers, a scale each: weights once, or rows that are in place
 *   fs_expert_gather_i8         tokens' rows in 8-bit integers in the experts' slots (fs_expert_gather and the former)
 *   fs_expert_matmul_i8         their products with 8-bit weights
 *   fs_distill                  divergence from a teacher's largest logits, and
 *   fs_distill_backward         its gradient
 *
 * Conventions are those of familyseer_mixture.h: no allocation and no scratch of the library's, working memory from
 * the caller (aligned to 256 bytes), the same results bit for bit from run to run, any call may be recorded into a HIP graph, matrices
 * have row strides in elements, pointers are aligned to their elements, outputs must not overlap anything else.
 * Where pointers and strides are multiples of 16 bytes the products load faster.
 *
 * fs_profile_begin counts the products of rows as FS_KERNEL_PACK, gradients of weights and distillation as FS_KERNEL_TRAIN_OTHER.
 */
#ifndef FAMILYSEER_EXPERTS_H
#define FAMILYSEER_EXPERTS_H

#include "familyseer_mixture.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- products by expert ---------------------------------------------------------------------- */

/*
 * The slots [first[e], first[e+1]) are expert e's, as fs_expert_plan leaves them; from first[n_experts] on nobody's.
 * Bounds are taken as max(0, min(n_slots, .)), so that no list of them leads outside the matrices; of bounds that descend
 * anywhere the results are not defined (those of fs_expert_matmul_backward too).
 *
 * Weights: turned = 0: expert e's are out_width rows of in_width elements, row o at w + e * w_step + o * w_stride, and
 *   y[s][o] = sum over i of x[s][i] * w[e][o][i];
 * turned = 1: they are in_width rows of out_width elements, and
 *   y[s][o] = sum over i of x[s][i] * w[e][i][o],
 * which, of the same weights, is the rows' gradient from the results': d_x = fs_expert_matmul(d_y, turned = 1) where x went
 * through turned = 0, and the other way round.  Nobody's slots get 0, whatever x holds there.  Products are added in fp32; of
 * fp32 inputs too each is a product of whole fp32 numbers.  y_type is the type of x and w, or FS_F32.
 * n_slots < 2^31; w_step may be 0 (one matrix for all experts).
 */
int fs_expert_matmul(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const void *x /* DEVICE */,
                     int32_t type, int64_t x_stride, const int32_t *first /* DEVICE, n_experts+1 */, const void *w /* DEVICE */,
                     int64_t w_stride, int64_t w_step, int32_t turned, void *y /* DEVICE out */, int32_t y_type, int64_t y_stride,
                     void *stream);

/*
 * The weights' gradient: d_w[e][o][i] = sum over e's slots s of d_y[s][o] * x[s][i], 0 for an expert without slots;
 * accumulate = 1: it is added to what d_w holds.  d_y has out_width columns, x in_width; for weights that were used
 * turned, x and d_y change places.  d_w_type is the type of d_y and x, or FS_F32; d_w_step: at least
 * out_width * d_w_stride.  Long lists of slots are split, and partial sums meet in the working memory.
 */
size_t fs_expert_matmul_backward_workspace_bytes(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, int32_t type);
int fs_expert_matmul_backward(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const void *d_y /* DEVICE */,
                              int32_t type, int64_t d_y_stride, const void *x /* DEVICE */, int64_t x_stride,
                              const int32_t *first /* DEVICE */, int32_t accumulate, void *d_w /* DEVICE out */, int32_t d_w_type,
                              int64_t d_w_stride, int64_t d_w_step, void *work /* DEVICE */, size_t work_bytes, void *stream);

/* ---- products in 8-bit integers -------------------------------------------------------------- */

#define FS_MAX_I8_WIDTH 131072   /* of a sum: 2^17 products of at most 127 * 127 stay below 2^31 */

/*
 * q[r][c] = x[r][c] / scale[r] to the nearest integer, ties to even, of the exact quotient; scale[r] = the largest |x[r][.]|
 * divided by 127 and rounded to fp32, at least 2^-126.  |q| is at most 127.  A row that holds an infinity or NaN has the scale
 * NaN, and its q are 0, so that every product with it is NaN.  Rows of q: q_stride bytes apart.
 */
int fs_quantize_rows(int64_t n_rows, int32_t width, const void *x /* DEVICE */, int32_t type, int64_t x_stride,
                     int8_t *q /* DEVICE out */, int64_t q_stride, float *scale /* DEVICE out, n_rows */, void *stream);

/* The same of token t's row, in each of the slots place[t*k + j]; nobody's slots get 0 and the scale 0. */
int fs_expert_gather_i8(int64_t n_tokens, int32_t k, int32_t n_experts, int32_t width, const void *x /* DEVICE */, int32_t type,
                        int64_t x_stride, const int32_t *first, const int32_t *place, int8_t *q /* DEVICE out, n_tokens*k rows */,
                        int64_t q_stride, float *scale /* DEVICE out, n_tokens*k */, void *stream);

/*
 * y[s][o] = (sum over i of q[s][i] * w[e][o][i]) * scale[s] * w_scale[e*out_width + o], the sum exact (for q and w of -127 to 127;
 * in_width <= FS_MAX_I8_WIDTH), then multiplied in fp32 in this order; nobody's slots get 0.  Strides and w_step in bytes.
 */
int fs_expert_matmul_i8(int64_t n_slots, int32_t n_experts, int32_t in_width, int32_t out_width, const int8_t *q /* DEVICE */,
                        int64_t q_stride, const float *scale /* DEVICE, n_slots */, const int32_t *first /* DEVICE */,
                        const int8_t *w /* DEVICE */, int64_t w_stride, int64_t w_step, const float *w_scale /* DEVICE, n_experts*out_width */,
                        void *y /* DEVICE out */, int32_t y_type, int64_t y_stride, void *stream);

/* ---- distillation from a teacher's largest logits ---------------------------------------------- */

#define FS_MAX_CLASSES 1048576
#define FS_MAX_LISTED 1024       /* of a token's classes */

typedef struct fs_distill_params {
    int32_t n_classes;   /* 1 .. FS_MAX_CLASSES                                  */
    int32_t k;           /* 1 .. FS_MAX_LISTED: entries of a token's list        */
    float temperature;   /* >= 2^-126, finite: all logits are divided by it      */
    float scale;         /* factor on the loss, finite (often temperature^2)     */
} fs_distill_params;

/*
 * A token's student gives logits over n_classes; a logit of -infinity or NaN is a class that it may not take (its
 * probability is 0), one of +infinity counts as the largest float.  Its teacher gives k entries: classes (FS_ID_I32 or
 * FS_ID_I64, in any order) and their logits.  An entry counts where its class is in [0, n_classes), the student may take the class, and the
 * teacher's logit is not -infinity or NaN (+infinity: the largest float); entries that do not count are as if they were not there.
 * With p_c = exp(student_c / T) / sum over c' of exp(student_c' / T), T the temperature:
 *
 * total = NULL: q_j = exp(teacher_j / T) / sum over entries of the same, and
 *     loss = scale * sum over entries of q_j * (log q_j - log p_class(j)).
 * total: log of the sum of exp(logit / T) over ALL of the teacher's classes, a number a token.  q_j = exp(teacher_j / T - total),
 * 1 at most, and all classes without an entry are one class more, the rest, with q_rest = max(0, 1 - sum of q_j) and p_rest = the sum
 * of their p:
 *     loss = scale * (sum over entries of q_j * (log q_j - log p_class(j)) + q_rest * (log q_rest - log p_rest)).
 * A token whose student may take no class without an entry has no rest, and is treated as without a total; so is one whose total is not finite.
 *
 * A class should be named once; named more often, each entry counts by itself, and the class is listed.  A token
 * without entries has the loss 0 and no gradient.
 */
size_t fs_distill_workspace_bytes(const fs_distill_params *params /* HOST */, int64_t n_tokens, int32_t logit_type);
int fs_distill(const fs_distill_params *params /* HOST */, int64_t n_tokens, const void *logits /* DEVICE */, int32_t logit_type,
               int64_t logit_stride, const void *ids /* DEVICE, n_tokens*k */, int32_t id_type, const void *teacher /* DEVICE, n_tokens*k */,
               int32_t teacher_type, const float *total /* DEVICE, n_tokens, or NULL */, float *loss /* DEVICE out, n_tokens */,
               void *work /* DEVICE */, size_t work_bytes, void *stream);

/*
 * d_logits[t][c] = d_loss[t] * d loss[t] / d logits[t][c], 0 for classes that the student may not take; and, where
 * `loss` is not NULL, the losses too: a training step that knows d_loss before needs no fs_distill.
 * The teacher has no gradient.
 */
int fs_distill_backward(const fs_distill_params *params /* HOST */, int64_t n_tokens, const void *logits /* DEVICE */,
                        int32_t logit_type, int64_t logit_stride, const void *ids /* DEVICE */, int32_t id_type,
                        const void *teacher /* DEVICE */, int32_t teacher_type, const float *total /* DEVICE or NULL */,
                        const float *d_loss /* DEVICE, n_tokens */, float *loss /* DEVICE out, n_tokens, or NULL */,
                        void *d_logits /* DEVICE out, of logit_type */, int64_t d_logit_stride, void *work /* DEVICE */,
                        size_t work_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* FAMILYSEER_EXPERTS_H */
