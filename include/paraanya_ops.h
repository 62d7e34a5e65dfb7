/*
 * paraanya_ops.h — operators of a text-conditioned noise network (MI355X, gfx950).
 *
 * The sampler of paraanya.h evaluates a noise network that sees no prompt. These entry points
 * are what a conditioned network needs beside it: layer norm, cross attention to the states of
 * a prompt encoder, and a shared projection with the low-rank adapters of many requests.
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

#ifdef __cplusplus
}
#endif
#endif /* PARAANYA_OPS_H */
