/*
 * agft_diff.h -- C ABI of differential attention over a serving node's paged
 * cache (agft_kv.h), on AMD Instinct MI355X (gfx950).
 *
 * The cache's heads go in pairs: heads 2 p and 2 p + 1 hold the keys of pair p's
 * two maps, and their values, side by side, are the 2 dim numbers that both maps
 * weigh.  For every token of the window and each g < group, with query heads
 * group (2 p + a) + g, a = 0, 1, as agft_kv_attend has them (so the two that make
 * one output lie group heads apart; a projection that puts them side by side has its
 * rows in another order when group > 1, and no strides of q can tell):
 *
 *   A_a = softmax(scale q_a K_{2p+a}^T)          over the request's tokens up to this one
 *   y   = A_0 V - lambda A_1 V,                  V = [V_{2p} V_{2p+1}]
 *   out = gain y                                 without a weight
 *   out = gain weight y / sqrt(mean(y^2) + eps)  with one: 2 dim numbers, one for all heads
 *
 * lambda is a number per pair and g, or per token, pair and g: what a layer's
 * learned vectors or projection give.
 *
 * It stands in a window where agft_kv_attend does, after agft_kv_append, and
 * follows its rules: tokens that were not granted get out 0 and log sums -infinity,
 * rows past the window's tokens are left alone, max_new bounds a request's new
 * tokens (rows that only a saved launch would have made are NaN), calls that share
 * a step or a workspace run one after another.  There is no backward pass: the
 * cache holds codes.
 *
 * Products and sums are kept in fp32, the sums of the probabilities and of y^2
 * too; probabilities meet the values in fp16, with the eleven bits and the range
 * that agft_kv_attend gives them, relative to the larger of a page's two value
 * scales.  Where outputs are fp16 and a request brings few rows (tokens x group up
 * to 16, or to 64 while such requests are little work), what that rounding leaves of
 * each probability is summed as well: the error is that of 32-bit probabilities.  In
 * tiles of more rows it is not: fp16 outputs are off by 1.2 to 1.4 times as much there,
 * bf16 ones by 1.01 times.  The other head's values of that page keep all their bits while
 * its scale lies within 2^22 (e4m3) or 2^29 (int8) of the larger.  Beyond, e4m3 values
 * lose them by and by, from the smallest codes on, until 2^41 leaves none; int8 ones
 * count for nothing.
 */
#ifndef AGFT_DIFF_H
#define AGFT_DIFF_H

#include "agft_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct agft_diff_args {
    const float *lambda;               /* device, fp32 */
    int64_t lambda_token, lambda_head; /* strides in numbers, >= 0; token 0: the same for all tokens; heads: p * group + g */
    const float *weight;               /* device, fp32 [2 dim], 16-byte aligned, or NULL */
    float eps;                         /* >= 0, of a weight */
    float gain;
} agft_diff_args;

/* workspace of agft_diff_attend, whatever it holds; 0 where that is refused */
size_t agft_diff_attend_bytes(const agft_kv_config *cfg, int32_t max_tokens);

/*
 * q: [tokens][heads * group][dim], out: [tokens][heads / 2 * group][2 * dim], bf16
 * or fp16, equal types.  d_lse: fp32 [max_tokens][heads * group], both maps' natural
 * logarithms of their sums, or NULL.  An odd number of heads is AGFT_E_INVAL, dim
 * 256 AGFT_E_UNSUPPORTED.
 */
int agft_diff_attend(const agft_kv_config *cfg, const void *d_cache, size_t cache_bytes, const void *d_tables,
                     size_t tables_bytes, void *d_step, size_t step_bytes, int32_t max_tokens, int32_t max_new,
                     const agft_kv_dense *q, const agft_diff_args *diff, const agft_kv_dense *out, float *d_lse,
                     float scale, void *d_work, size_t work_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* AGFT_DIFF_H */
