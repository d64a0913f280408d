/*
 * cbinfer_tokens.h -- C ABI of the token operators: what follows the per-frame network when its
 * answers are turned into tokens and decisions, one token per stream and frame.
 *
 *   cbinfer_log_probs          scores of classes -> log probability of given labels, entropy, alternatives
 *   cbinfer_linear_attention   linear attention with a decay for each head, state per stream
 *   cbinfer_quantised_product  few tokens times a matrix of 4-bit weights with group scales
 *   cbinfer_gated_norm         norm behind a block, gate, residual scale, norm in front of the next
 *
 * Conventions: those of cbinfer.h (plain pointers and sizes, CBINFER_* codes, cbinfer_last_error,
 * CBINFER_F32 / CBINFER_BF16), and
 *   - Every pointer below is DEVICE memory of the current device unless it says HOST; it must be aligned to its
 *     element.  `stream` is the hipStream_t that the call's work is enqueued on (NULL = default stream).
 *   - Calls are asynchronous, allocate nothing and keep nothing: what they need beyond inputs and
 *     outputs is the workspace that the caller passes (256-byte aligned, of the size that the function beside
 *     the call returns, its contents of no matter before and after).  Two calls that may run at the same time need two.
 *   - Strides are in elements.  Outputs must not overlap themselves, nor inputs except where a call says so.
 *   - Sums, softmax statistics, states and norms are float32 at least whatever the type of the
 *     tensors; values are rounded to bfloat16 once, when they are stored.
 */
#ifndef CBINFER_TOKENS_H
#define CBINFER_TOKENS_H

#include "cbinfer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- log probabilities ----------------------------------------------------------------------
 * scores x[o][c][i]: a position (o, i) has `classes` scores, at any strides.  [rows][classes]: inner 1;
 * the network's output [streams][classes][H][W]: inner H*W.  With m = max_c x, s = sum_c exp(x_c - m):
 *   log probability of class c   x_c - m - log s
 *   entropy                      log s - sum_c exp(x_c - m) (x_c - m) / s, in nats
 *   alternatives                 the `top` classes of the largest scores, largest first, the lowest class first
 *                                among equals, and their log probabilities
 * A score of -inf is a class of probability 0; where all are, log probabilities are -inf and the entropy is 0.
 * Where a score is NaN or +inf, log probabilities and entropy are NaN, and the alternatives are ordered with NaN
 * in front of every number.  A label < 0 is a position that is not scored: 0.  A label >= classes: NaN. */
typedef struct {
    int32_t dtype;                                      /* of the scores */
    int32_t label_bytes;                                /* 4 or 8: int32 or int64 labels */
    int32_t top;                                        /* 0 .. 64, at most `classes` */
    int32_t reserved;                                   /* 0 */
    int64_t outer, classes, inner;                      /* 1 <= classes < 2^31; outer * inner < 2^31 */
    int64_t outer_stride, class_stride, inner_stride;
    const void *scores;
    const void *labels;                                 /* [outer][inner], or NULL */
    float *label;                                       /* [outer][inner], or NULL; not without labels */
    float *entropy;                                     /* [outer][inner], or NULL */
    float *top_values;                                  /* [outer][top][inner] (top > 0) */
    int32_t *top_index;                                 /* [outer][top][inner] (top > 0) */
    void *workspace;
    size_t workspace_bytes;
} cbinfer_log_probs_args;

/* 0 also if the arguments are invalid.  Looks at sizes, strides and types only. */
size_t cbinfer_log_probs_workspace_bytes(const cbinfer_log_probs_args *a);
int cbinfer_log_probs(const cbinfer_log_probs_args *a, void *stream);

/* ---- linear attention with a decay for each head ----------------------------------------------
 * Per stream and head, with a state S [key_size][value_size] and a decay g of the head:
 *   S_t = g S_(t-1) + k_t (x) v_t        o_t = scale * q_t S_t
 * for the tokens t = 0 .. length-1 of the stream, S_(-1) being the state as the call finds it; S of the last token is
 * left in its place.  Head h reads the keys and values of head h / (heads / kv_heads).  q [streams][tokens][heads][key_size],
 * k [streams][tokens][kv_heads][key_size], v [streams][tokens][kv_heads][value_size], o like q with value_size:
 * strides of the first three axes are given, the last axis is contiguous.  A stream of length 0 keeps its state; o is 0
 * from a stream's length on, where q, k and v are not read.  A value that is not finite makes its column of S infinite or NaN,
 * a key its row, and the outputs that follow; earlier outputs stay as they are. */
typedef struct {
    int32_t dtype;                                      /* of q, k, v, o */
    int32_t streams, tokens, heads, kv_heads;           /* each >= 0; heads a multiple of kv_heads */
    int32_t key_size, value_size;                       /* 1 .. 256 */
    float scale;
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3]; /* stream, token, head */
    const void *q, *k, *v;
    void *o;
    float *state;                                       /* [streams][heads][key_size][value_size] */
    const float *decay;                                 /* [heads], each in 0 .. 1 */
    const int32_t *lengths;                             /* [streams], taken as 0 .. tokens; or NULL: all tokens */
    void *workspace;
    size_t workspace_bytes;
} cbinfer_linear_attention_args;

size_t cbinfer_linear_attention_workspace_bytes(const cbinfer_linear_attention_args *a);
int cbinfer_linear_attention(const cbinfer_linear_attention_args *a, void *stream);

/* ---- products with 4-bit weights ----------------------------------------------------------------
 * w[n][k] = scale[n][k / group] * value(code[n][k]), value of the codes 0 .. 7: 0, 0.5, 1, 1.5, 2, 3, 4, 6, of
 * 8 .. 15 the same negative (sign, two bits of exponent, one of mantissa: the 4-bit float that this GPU converts in
 * hardware).  A group is 32, 64 or 128 weights along a row, the last of a row may be shorter.  scales are bfloat16.
 *   y[m][n] = bias[n] + sum_k x[m][k] w[n][k]
 * A group's products are added up in float32 before its scale is applied: where they pass 3.4e38 the result is not finite
 * even if the scaled sum would be. */

/* weights [rows][cols] float32 or bfloat16, finite, -> codes [rows][cols], one byte each, and scales
 * [rows][ceil(cols / group)]: the scale is a sixth of the largest magnitude of the group, rounded to bfloat16, and
 * each weight takes the code whose value is nearest (of two as near, the one of even code). */
int cbinfer_quantise_weights(const void *weights, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, int32_t group,
                             uint8_t *codes, uint16_t *scales, void *stream);

/* Codes (their lower four bits) and scales in the order in which the product reads them.  `packed` is 256-byte aligned, of
 * cbinfer_packed_weights_bytes() bytes (0: the sizes are invalid). */
size_t cbinfer_packed_weights_bytes(int64_t rows, int64_t cols, int32_t group);
int cbinfer_pack_weights(const uint8_t *codes, const uint16_t *scales, int64_t rows, int64_t cols, int32_t group, void *packed,
                         void *stream);

typedef struct {
    int32_t dtype;                                      /* of x and y */
    int32_t group;
    int64_t tokens, rows, cols;                         /* x [tokens][cols], y [tokens][rows]; 0 .. 2^19, 1 .. 2^26, 1 .. 2^25 */
    int64_t x_stride, y_stride;                         /* from token to token */
    const void *x;
    const void *packed;
    const float *bias;                                  /* [rows], or NULL */
    void *y;
    void *workspace;
    size_t workspace_bytes;
} cbinfer_quantised_product_args;

size_t cbinfer_quantised_product_workspace_bytes(const cbinfer_quantised_product_args *a);
int cbinfer_quantised_product(const cbinfer_quantised_product_args *a, void *stream);

/* ---- norms around a block, with its gate and residual scale ---------------------------------------
 * Per row of `size` values, in this order, each part left out where its pointer is NULL (or its kind 0):
 *   u = x / sqrt(mean of x^2 over its group + eps) * weight      (groups of `group` values; 0: the whole row)
 *   u = u * gate / (1 + exp(-gate))                               (CBINFER_GATE_SILU; _SIGMOID: u / (1 + exp(-gate)))
 *   h = residual + scale * channel_scale * u
 *   y = h / sqrt(mean of h^2 over the row + eps) * next_weight
 * Everything between x and the two outputs stays in float32, y is formed from h before its rounding.
 * h may be the same memory as residual, and h or y the same as x or gate (same rows, same strides). */
enum { CBINFER_GATE_NONE = 0, CBINFER_GATE_SILU = 1, CBINFER_GATE_SIGMOID = 2 };
typedef struct {
    int32_t dtype;                                      /* of x, gate and y */
    int32_t sum_dtype;                                  /* of residual and h: CBINFER_F32, or dtype */
    int32_t gate_kind;
    int32_t group;                                      /* 0, or a divisor of size; only with weight */
    int64_t rows, size;                                 /* size 1 .. 16384 */
    int64_t x_stride, gate_stride, residual_stride, h_stride, y_stride; /* from row to row */
    float scale, eps;
    const void *x;
    const float *weight;                                /* [size] */
    const void *gate;
    const void *residual;
    const float *channel_scale;                         /* [size] */
    void *h;
    const float *next_weight;                           /* [size]; together with y */
    void *y;
} cbinfer_gated_norm_args;

int cbinfer_gated_norm(const cbinfer_gated_norm_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CBINFER_TOKENS_H */
