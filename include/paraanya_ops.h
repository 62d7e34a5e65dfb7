/*
 * paraanya_ops.h — operators of a text-conditioned noise network (MI355X, gfx950).
 *
 * The sampler of paraanya.h evaluates a noise network that sees no prompt. These entry points
 * are what a conditioned network needs beside it: layer norm, cross attention to the states of
 * a prompt encoder, a shared projection with the low-rank adapters of many requests, group norm with
 * an activation, a gated feed-forward block, and a projection in 8-bit integers.
 *
 * Conventions (those of paraanya.h, and)
 *   - Every call is stateless: it checks its arguments (nothing is enqueued when it fails),
 *     enqueues its kernels on `stream` (a hipStream_t, NULL = the null stream) and returns
 *     without waiting. It allocates nothing; a call that needs scratch memory takes a
 *     `workspace` (device, 256-byte aligned) of at least the size that its
 *     *_workspace function reports for the same sizes. The workspace needs no initialisation
 *     and holds nothing between calls; two calls that may overlap need two.
 *   - Calls are safe to capture into a HIP graph (no host memory is read after the return, no
 *     synchronisation).
 *   - Results are the same bit for bit whenever a call is repeated on one device (no atomics).
 *   - Strides count elements. Pointers need the alignment of their element type only; 16-byte
 *     alignment of rows is faster.
 *   - Sums, softmax statistics and products are accumulated in fp32 whatever the element type.
 *     What is rounded to the element type on the way, as the operand of a second product, is said
 *     at each operator.
 */
#ifndef PARAANYA_OPS_H
#define PARAANYA_OPS_H

#include <stddef.h>

#include "paraanya.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PA_F32  0
#define PA_BF16 1
#define PA_F16  2

/* ------------------------------------------------------------------ layer norm
 * y = (x - mean) rstd * weight + bias over the cols elements of each row, with the row's mean,
 * v = mean (x - mean)^2 and rstd = 1 / sqrt(v + eps). */
typedef struct {
    int64_t rows;          /* >= 0 */
    int64_t cols;          /* 1 .. PA_NORM_MAX_COLS */
    int32_t dtype;         /* x, y, dy, dx: PA_F32, PA_BF16 or PA_F16 */
    int32_t param_dtype;   /* weight, bias, dweight, dbias: dtype or PA_F32 */
    double  eps;           /* >= 0, finite */
    int64_t x_stride;      /* elements from a row of x to the next, >= cols */
    int64_t y_stride;      /* of y (forward) or dy (backward) */
    int64_t dx_stride;     /* of dx (backward; ignored by the forward) */
} pa_norm_t;

#define PA_NORM_MAX_COLS (1 << 20)

/* weight and bias may be NULL (1 and 0). mean and rstd (fp32, rows) are written for the
 * backward pass; both may be NULL. y may be x (same stride). */
PA_API int paraanya_layer_norm(const pa_norm_t* p, const void* x, const void* weight, const void* bias,
                               void* y, float* mean, float* rstd, void* stream);

/* Gradients of the same norm from dy, the forward's x, mean and rstd: with g = dy weight,
 * xh = (x - mean) rstd: dx = rstd (g - mean(g) - xh mean(g xh)), dweight = sum over rows of
 * dy xh, dbias = sum over rows of dy. Any of dx, dweight, dbias may be NULL (not computed).
 * dx may be dy or x (same stride). rows = 0 writes zeros to dweight and dbias. */
PA_API int paraanya_layer_norm_backward(const pa_norm_t* p, const void* dy, const void* x, const float* mean,
                                        const float* rstd, const void* weight, void* dx, void* dweight,
                                        void* dbias, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_layer_norm_backward_workspace(const pa_norm_t* p, size_t* bytes);

/* ------------------------------------------------------------------ cross attention
 * o = softmax(scale q k^T + bias) v per sample and query head, where k and v are the projected
 * states of an encoder with a length of its own. q_heads / kv_heads query heads share a key and
 * value head (query head h reads kv head h / (q_heads / kv_heads)).
 *
 * Which keys a sample's queries see: keys below kv_lens[b] (all kv_len without it; values are
 * clamped to [0, kv_len]) that the key mask admits. PA_MASK_BOOL: one byte per key, nonzero =
 * visible. PA_MASK_ADD: fp32 per key, added to the scaled score; -inf = not visible (the type's
 * lowest value is a finite bias: a row that has nothing else averages those keys).
 * What an invisible key's k and v hold, infinities and NaN included, has no effect. A row that
 * sees no key gives o = 0 and zero gradients.
 *
 * Roundings to the element type beside those of the results: the weights (relative to the row's
 * largest) for their product with v, P for dv, and dS = P (do v^T - delta) for dq and dk. In fp16, P
 * and dS are scaled by powers of two, so that weights and gradients below its normal numbers, or
 * beyond its range, keep their digits. delta is formed in fp32 up to kv_len = 256, from the rounded o
 * above. Errors, root mean square over the result's own: o 1.1 to 1.4 times that of its rounding
 * alone, gradients 1.3 to 1.65 times. */
#define PA_MASK_NONE 0
#define PA_MASK_BOOL 1
#define PA_MASK_ADD  2

typedef struct {
    int64_t batch;               /* 0 .. 65535 */
    int64_t q_len;               /* 0 .. 2^30 */
    int64_t kv_len;              /* 0 .. 2^30 */
    int32_t q_heads, kv_heads;   /* 1 .. 65535, q_heads a multiple of kv_heads; q_len * q_heads <= 2^30 */
    int32_t head_dim;            /* 1 .. 128 */
    int32_t dtype;               /* PA_BF16 or PA_F16 */
    double  scale;               /* finite */
    /* Strides of batch, token and head; a head's elements are consecutive. A stride of 0 in
     * q, k or v (not in an output) repeats what it points to. */
    int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
    const int32_t* kv_lens;      /* device, batch; NULL = all kv_len */
    const void* mask;            /* device, batch x kv_len; NULL with PA_MASK_NONE */
    int32_t mask_kind;
    int32_t pad;
    int64_t mask_stride;         /* elements from a sample's mask row to the next (0 = shared) */
} pa_cross_t;

/* stats (fp32, [batch][q_heads][q_len][2]; may be NULL) receives for each row a score m near its
 * largest (at most log(256) below it) and log(sum of exp(score - m)), for a row that sees no key
 * (-inf, -inf): the log-sum-exp in two parts, so that scores at the type's lowest value keep their
 * weights in the backward pass. */
PA_API int paraanya_cross_attention(const pa_cross_t* p, const void* q, const void* k, const void* v, void* o,
                                    float* stats, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_cross_attention_workspace(const pa_cross_t* p, size_t* bytes);

/* Gradients from the forward's inputs, o (o_stride) and stats. do has the strides do_stride;
 * dq, dk, dv have their own. Any of dq, dk, dv may be NULL (dk and dv only together). */
typedef struct {
    int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} pa_cross_grad_t;

PA_API int paraanya_cross_attention_backward(const pa_cross_t* p, const pa_cross_grad_t* g, const void* d_o,
                                             const void* q, const void* k, const void* v, const void* o,
                                             const float* stats, void* dq, void* dk, void* dv, void* workspace,
                                             size_t workspace_bytes, void* stream);
PA_API int paraanya_cross_attention_backward_workspace(const pa_cross_t* p, size_t* bytes);

/* ------------------------------------------------------------------ projection with adapters
 * y = x W^T + bias + s_a (x A_a^T) B_a^T for the rows of many requests at once: request i is rows
 * offsets[i] .. offsets[i + 1] - 1 and uses adapter a = ids[i] (a < 0 or >= adapters: none). Rows
 * before offsets[0] and from offsets[requests] on have no adapter. Offsets must not decrease; they
 * are clamped to [0, rows]. Inference only: no gradients. What a request's adapter or rows hold,
 * infinities and NaN included, has no effect on the rows of others. */
#define PA_LORA_MAX_RANK 128

typedef struct {
    int64_t rows;                /* x and y, 0 .. 2^30 */
    int32_t in_features;         /* K: 1 .. 2^20 */
    int32_t out_features;        /* N: 1 .. 2^20 */
    int32_t rank;                /* R: 1 .. PA_LORA_MAX_RANK, of the stored adapters */
    int32_t adapters;            /* stored adapters, >= 0 */
    int32_t requests;            /* 0 .. 65535 */
    int32_t dtype;               /* PA_BF16 or PA_F16: x, W, bias, A, B and y */
    int64_t x_stride, w_stride, y_stride;   /* row strides: >= K, >= K, >= N */
    const int32_t* offsets;      /* device, requests + 1 */
    const int32_t* ids;          /* device, requests */
    const float* scales;         /* device, adapters; NULL = 1 */
} pa_lora_t;

/* weight [N][K] (w_stride), bias [N] or NULL, a [adapters][R][K], b [adapters][N][R] (both dense).
 * The row's x A^T is scaled, then rounded to the element type for its product with B. */
PA_API int paraanya_lora_linear(const pa_lora_t* p, const void* x, const void* weight, const void* bias,
                                const void* a, const void* b, void* y, void* workspace,
                                size_t workspace_bytes, void* stream);
PA_API int paraanya_lora_linear_workspace(const pa_lora_t* p, size_t* bytes);

/* ------------------------------------------------------------------ group norm
 * y = act((x - mean) rstd * weight + bias) over a channels-last tensor [batch][pixels][channels]: mean
 * and v = mean (x - mean)^2 are those of a sample's group (channels / groups consecutive channels, all
 * pixels), rstd = 1 / sqrt(v + eps). In fp32 throughout: a group's sum of (x - mean)^2 has to stay below 2^128. */
#define PA_ACT_NONE 0
#define PA_ACT_SILU 1          /* z / (1 + e^-z) */
#define PA_ACT_GELU 2          /* z Phi(z), the normal distribution's */

#define PA_GROUP_MAX_CHANNELS 4096      /* of one group */

typedef struct {
    int64_t batch;             /* 0 .. 65535 */
    int64_t pixels;            /* 0 .. 2^30 */
    int32_t channels;          /* 1 .. 2^20, a multiple of groups */
    int32_t groups;            /* >= 1 */
    int32_t dtype;             /* x, y, dy, dx: PA_F32, PA_BF16 or PA_F16 */
    int32_t param_dtype;       /* weight, bias, dweight, dbias: dtype or PA_F32 */
    int32_t activation;        /* PA_ACT_* */
    int32_t pad;
    double  eps;               /* >= 0, finite */
    /* Strides of batch and pixel; a pixel's channels are consecutive. Of inputs a batch stride of 0 repeats a
     * sample. y_stride: of y (forward) or dy (backward). */
    int64_t x_stride[2], y_stride[2], dx_stride[2];
} pa_group_norm_t;

/* weight and bias may be NULL (1 and 0). mean and rstd (fp32, [batch][groups]) are written for the backward
 * pass; both may be NULL. y may be x (same strides). */
PA_API int paraanya_group_norm(const pa_group_norm_t* p, const void* x, const void* weight, const void* bias, void* y,
                               float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_group_norm_workspace(const pa_group_norm_t* p, size_t* bytes);

/* Gradients from dy, the forward's x, weight, bias, mean and rstd: with z the activation's argument,
 * dz = dy act'(z), g = dz weight, xh = (x - mean) rstd: dx = rstd (g - mean(g) - xh mean(g xh)),
 * dweight = sum of dz xh, dbias = sum of dz over samples and pixels. Any of dx, dweight, dbias may be NULL (not
 * computed). dx may be dy or x (same strides). No samples or pixels: zeros in dweight and dbias. */
PA_API int paraanya_group_norm_backward(const pa_group_norm_t* p, const void* dy, const void* x, const void* weight,
                                        const void* bias, const float* mean, const float* rstd, void* dx, void* dweight,
                                        void* dbias, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_group_norm_backward_workspace(const pa_group_norm_t* p, size_t* bytes);

/* ------------------------------------------------------------------ gated feed-forward block
 * h = act(x G^T + bg) * (x U^T + bu), y = h D^T + bd: both projections, the activation and the product in one
 * kernel, the projection back in a second. h is rounded to the element type as the second product's operand; so are
 * the gradients by the two projections g and u as operands of those of x and of the weights (in fp16 multiplied by a power
 * of two that brings the largest |dy| to 1/16 .. 1/8, so that small gradients keep their digits; they may be 2^19 times as
 * large as dy). u act'(g) and act(g), by which dh gives them, are kept in 24 bits, with fp32's range. An error is so
 * 1.4 times that of rounding the result alone, of y and of every gradient. In fp16 an h beyond 65504 is infinite. */
typedef struct {
    int64_t rows;                /* 0 .. 2^30; a matrix has at most 2^34 elements and 2^23 tiles of 64 x 64 */
    int32_t in_features;         /* K: 1 .. 2^20 */
    int32_t hidden_features;     /* H: 1 .. 2^20 */
    int32_t out_features;        /* N: 1 .. 2^20 */
    int32_t dtype;               /* PA_BF16 or PA_F16, of all tensors */
    int32_t activation;          /* PA_ACT_* */
    int32_t alignment;           /* bytes that all pointers to x, the weights and dy are multiples of: 2 .. 16. Rows are
                                    read in place where it is 16 and strides and lengths are multiples of 8, and copied
                                    into the workspace otherwise (beyond 32 rows). */
    int64_t x_stride;            /* row strides: >= K */
    int64_t gate_stride, up_stride;         /* >= K */
    int64_t down_stride;         /* >= H */
    int64_t y_stride;            /* of y (forward) or dy (backward), >= N */
} pa_feed_t;

/* gate and up [H][K], down [N][H]; biases [H], [H] and [N] or NULL. saved: what the backward pass needs (256-byte
 * aligned, of the size that paraanya_feed_forward_saved reports; the caller keeps it), or NULL. Nothing that is written,
 * here or by the backward pass, may overlap an input. */
PA_API int paraanya_feed_forward(const pa_feed_t* p, const void* x, const void* gate, const void* gate_bias, const void* up,
                                 const void* up_bias, const void* down, const void* down_bias, void* y, void* saved,
                                 size_t saved_bytes, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_feed_forward_saved(const pa_feed_t* p, size_t* bytes);
PA_API int paraanya_feed_forward_workspace(const pa_feed_t* p, int with_saved, size_t* bytes);

/* Gradients, dense, of the element type: dx [rows][K], dgate and dup [H][K], ddown [N][H], dgate_bias and dup_bias
 * [H], ddown_bias [N]. Any may be NULL (not computed); a bias's gradient comes with its weight's. No rows: zeros
 * in the weights' and biases' gradients. */
typedef struct {
    void *dx, *dgate, *dup, *ddown, *dgate_bias, *dup_bias, *ddown_bias;
} pa_feed_grad_t;

PA_API int paraanya_feed_forward_backward(const pa_feed_t* p, const pa_feed_grad_t* g, const void* dy, const void* x,
                                          const void* gate, const void* up, const void* down, const void* saved,
                                          size_t saved_bytes, void* workspace, size_t workspace_bytes, void* stream);
PA_API int paraanya_feed_forward_backward_workspace(const pa_feed_t* p, size_t* bytes);

/* ------------------------------------------------------------------ projection in 8-bit integers
 * Rows to 8 bits: scale[i] = max |x[i]| / 127 in fp32, q = x / scale rounded to the nearest (even) integer. A row of
 * zeros has scale 0 and q 0; one that holds an infinity or a NaN has scale NaN and q 0, so that its results are NaN.
 * q's rows are q_stride bytes apart; bytes from cols up to the next multiple of 16 are written as zeros. */
typedef struct {
    int64_t rows;                /* 0 .. 2^40 */
    int64_t cols;                /* 1 .. 2^20 */
    int32_t dtype;               /* of x: PA_F32, PA_BF16 or PA_F16 */
    int32_t pad;
    int64_t x_stride;            /* >= cols */
    int64_t q_stride;            /* bytes, a multiple of 16, >= cols; q 16-byte aligned */
} pa_quantize_t;

PA_API int paraanya_quantize_rows(const pa_quantize_t* p, const void* x, int8_t* q, float* scale, void* stream);

/* y = (xq wq^T) x_scale w_scale + bias: 8-bit products summed in 32-bit integers (exact), then one fp32 product with the
 * row's scale, one with the channel's, and the bias added. xq [rows][K], wq [N][K] with rows of any
 * multiple of 16 bytes at 16-byte addresses; bytes past K up to the next multiple of 16 are read and have no effect.
 * Neither this nor paraanya_quantize_rows writes into an input. */
typedef struct {
    int64_t rows;                /* 0 .. 2^30 */
    int32_t in_features;         /* K: 1 .. PA_INT8_MAX_IN */
    int32_t out_features;        /* N: 1 .. 2^20 */
    int32_t dtype;               /* of y and bias: PA_BF16 or PA_F16 */
    int32_t pad;
    int64_t x_stride, w_stride;  /* bytes, multiples of 16, >= K */
    int64_t y_stride;            /* >= N */
} pa_int8_linear_t;

#define PA_INT8_MAX_IN ((1 << 17) - 1)   /* so many products of at most 128 x 128 stay within 32 bits */

PA_API int paraanya_int8_linear(const pa_int8_linear_t* p, const int8_t* xq, const float* x_scale, const int8_t* wq,
                                const float* w_scale, const void* bias, void* y, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PARAANYA_OPS_H */
