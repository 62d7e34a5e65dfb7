// Host side of the group norm, the feed-forward block and the 8-bit projection declared in
// include/paraanya_ops.h: argument checks (before any HIP call), workspace layout, launches. Stateless; nothing
// is allocated.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>

#include "pa_ops_host.h"

using namespace pa;

namespace {

constexpr int64_t kMaxBlocks = 1 << 23;       // a grid holds fewer than 2^32 threads
// Row strides below this leave every offset within a tile of 256 rows of 16 bits to 31 bits.
constexpr int64_t kBufferStride = 1 << 22;

bool known_activation(int a) { return a == PA_ACT_NONE || a == PA_ACT_SILU || a == PA_ACT_GELU; }

// ------------------------------------------------------------------ group norm
int check_group_stride(const pa_group_norm_t* p, const int64_t s[2], const char* what, bool output) {
    if (s[0] < 0 || s[0] > (1ll << 40) || s[1] < 0 || s[1] > (1ll << 40)) return fail(PA_ERR_INVALID_ARG, "group norm: stride of %s out of range", what);
    if (p->pixels > 1 && s[1] < p->channels) return fail(PA_ERR_INVALID_ARG, "group norm: pixel stride of %s must be at least channels", what);
    // Samples one after the other, or side by side in every pixel.
    if (output && p->batch > 1 && p->pixels > 0) {
        const bool after = s[0] >= (p->pixels - 1) * s[1] + p->channels;
        const bool beside = s[0] >= p->channels && (p->pixels == 1 || s[1] >= (p->batch - 1) * s[0] + p->channels);
        if (!after && !beside) return fail(PA_ERR_INVALID_ARG, "group norm: %s overlaps itself", what);
    }
    return PA_OK;
}

int check_group(const pa_group_norm_t* p, bool backward) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "group norm: p is NULL");
    if (p->batch < 0 || p->batch > 65535) return fail(PA_ERR_INVALID_ARG, "group norm: batch must lie in [0, 65535]");
    if (p->pixels < 0 || p->pixels > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "group norm: pixels must lie in [0, 2^30]");
    if (p->channels < 1 || p->channels > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "group norm: channels must lie in [1, 2^20]");
    if (p->groups < 1 || p->channels % p->groups != 0) return fail(PA_ERR_INVALID_ARG, "group norm: channels must be a multiple of groups");
    if (p->channels / p->groups > PA_GROUP_MAX_CHANNELS)
        return fail(PA_ERR_UNSUPPORTED, "group norm: more than %d channels in a group are not built", PA_GROUP_MAX_CHANNELS);
    if (p->dtype != PA_F32 && p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "group norm: unknown dtype %d", p->dtype);
    if (p->param_dtype != p->dtype && p->param_dtype != PA_F32)
        return fail(PA_ERR_INVALID_ARG, "group norm: param_dtype must be dtype or PA_F32");
    if (!known_activation(p->activation)) return fail(PA_ERR_INVALID_ARG, "group norm: unknown activation %d", p->activation);
    if (!(p->eps >= 0.0) || !(p->eps <= 1e30)) return fail(PA_ERR_INVALID_ARG, "group norm: eps must be finite and not negative");
    if (int rc = check_group_stride(p, p->x_stride, "x", false)) return rc;
    return check_group_stride(p, p->y_stride, backward ? "dy" : "y", !backward);
}

int group_align(const pa_group_norm_t* p, const void* const* data, int n, const void* const* par, int np) {
    for (int i = 0; i < n; ++i)
        if (misaligned(data[i], element_size(p->dtype))) return fail(PA_ERR_INVALID_ARG, "group norm: a pointer is not aligned to its element");
    for (int i = 0; i < np; ++i)
        if (misaligned(par[i], element_size(p->param_dtype))) return fail(PA_ERR_INVALID_ARG, "group norm: a pointer is not aligned to its element");
    return PA_OK;
}

GroupDev group_dev(const pa_group_norm_t* p, bool backward) {
    GroupDev d{};
    d.batch = (int)p->batch;
    d.pixels = (int)p->pixels;
    d.channels = p->channels;
    d.groups = p->groups;
    d.param_dtype = p->param_dtype;
    d.act = p->activation;
    d.eps = (float)p->eps;
    for (int i = 0; i < 2; ++i) {
        d.xs[i] = p->x_stride[i];
        d.ys[i] = p->y_stride[i];
        d.dxs[i] = p->dx_stride[i];
    }
    group_plan(d, p->dtype, backward);
    return d;
}

size_t group_layout(GroupDev& d, bool backward, void* ws) {
    Parts w(ws);
    if (!backward) {
        if (!d.whole) d.part = static_cast<float*>(w.take((size_t)d.batch * d.groups * d.chunks * 2 * sizeof(float)));
    } else {
        if (!d.whole) d.part = static_cast<float*>(w.take((size_t)d.batch * d.chunks * 2 * d.channels * sizeof(float)));
        d.sums = static_cast<float*>(w.take((size_t)d.batch * 2 * d.channels * sizeof(float)));
        d.means = static_cast<float*>(w.take((size_t)d.batch * d.groups * 2 * sizeof(float)));
    }
    return w.used;
}

// ------------------------------------------------------------------ feed-forward block
int check_feed(const pa_feed_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "feed forward: p is NULL");
    if (p->rows < 0 || p->rows > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "feed forward: rows must lie in [0, 2^30]");
    if (p->in_features < 1 || p->in_features > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "feed forward: in_features must lie in [1, 2^20]");
    if (p->hidden_features < 1 || p->hidden_features > (1 << 20))
        return fail(PA_ERR_INVALID_ARG, "feed forward: hidden_features must lie in [1, 2^20]");
    if (p->out_features < 1 || p->out_features > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "feed forward: out_features must lie in [1, 2^20]");
    if (p->dtype == PA_F32) return fail(PA_ERR_UNSUPPORTED, "feed forward: fp32 is not built (PA_BF16 or PA_F16)");
    if (p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "feed forward: unknown dtype %d", p->dtype);
    if (!known_activation(p->activation)) return fail(PA_ERR_INVALID_ARG, "feed forward: unknown activation %d", p->activation);
    if (p->alignment != 2 && p->alignment != 4 && p->alignment != 8 && p->alignment != 16)
        return fail(PA_ERR_INVALID_ARG, "feed forward: alignment must be 2, 4, 8 or 16");
    if (p->x_stride < p->in_features || p->gate_stride < p->in_features || p->up_stride < p->in_features ||
        p->down_stride < p->hidden_features || p->y_stride < p->out_features)
        return fail(PA_ERR_INVALID_ARG, "feed forward: row strides must be at least the row's length");
    // Tiles of 64 x 64 of every product fit a grid.
    const int64_t most = 1ll << 34;
    const int64_t wide = p->in_features > p->hidden_features ? (p->in_features > p->out_features ? p->in_features : p->out_features)
                                                             : (p->hidden_features > p->out_features ? p->hidden_features : p->out_features);
    if (p->rows * wide > most || (int64_t)p->hidden_features * (p->in_features > p->out_features ? p->in_features : p->out_features) > most)
        return fail(PA_ERR_UNSUPPORTED, "feed forward: more than 2^34 elements in a matrix");
    if ((p->rows + 63) / 64 * ((wide + 63) / 64) > kMaxBlocks)
        return fail(PA_ERR_UNSUPPORTED, "feed forward: more than 2^23 tiles of 64 x 64 elements in a matrix");
    return PA_OK;
}

int feed_align(const pa_feed_t* p, const void* const* given, int n, const void* const* others, int m) {
    for (int i = 0; i < n; ++i)
        if (misaligned(given[i], p->alignment)) return fail(PA_ERR_INVALID_ARG, "feed forward: a pointer is not aligned to %d bytes", p->alignment);
    for (int i = 0; i < m; ++i)
        if (misaligned(others[i], 2)) return fail(PA_ERR_INVALID_ARG, "feed forward: a pointer is not aligned to its element");
    return PA_OK;
}

int pad8(int n) { return (n + 7) / 8 * 8; }

FeedDev feed_dev(const pa_feed_t* p) {
    FeedDev d{};
    d.rows = (int)p->rows;
    d.in = p->in_features;
    d.hidden = p->hidden_features;
    d.out = p->out_features;
    d.in_pad = pad8(d.in);
    d.hidden_pad = pad8(d.hidden);
    d.out_pad = pad8(d.out);
    d.x_stride = p->x_stride;
    d.gate_stride = p->gate_stride;
    d.up_stride = p->up_stride;
    d.down_stride = p->down_stride;
    d.y_stride = p->y_stride;
    return d;
}

size_t feed_saved(const pa_feed_t* p) { return 4 * round256((size_t)p->rows * pad8(p->hidden_features) * 2); }

void feed_saved_parts(FeedDev& d, void* saved) {
    Parts w(saved);
    const size_t n = (size_t)d.rows * d.hidden_pad * 2;
    d.by_z = static_cast<uint16_t*>(w.take(n));
    d.by_u = static_cast<uint16_t*>(w.take(n));
    d.last = static_cast<uint16_t*>(w.take(n));
    d.h = w.take(n);
}

// Whether rows of `n` elements, `stride` apart, are read in place by the tiles.
bool in_place(const pa_feed_t* p, int n, int64_t stride) {
    return p->alignment == 16 && n % 8 == 0 && stride % 8 == 0 && stride < kBufferStride;
}

// Gate and up are one operand: both are read in place, with one stride, or both copied.
size_t feed_layout(const pa_feed_t* p, FeedDev& d, bool backward, bool with_saved, void* ws) {
    Parts w(ws);
    const size_t hidden = (size_t)d.rows * d.hidden_pad * 2;
    if (!backward && !with_saved) d.h = w.take(hidden);
    if (backward) {
        d.dz = w.take(hidden);
        d.du = w.take(hidden);
        if (p->dtype == PA_F16) d.largest = static_cast<float*>(w.take(kLargest * sizeof(float)));
    }
    if (backward || !feed_few(p->rows)) {
        if (!in_place(p, d.in, d.x_stride)) d.x_pad = w.take((size_t)d.rows * d.in_pad * 2);
        if (!in_place(p, d.in, d.gate_stride) || d.gate_stride != d.up_stride) {
            d.gate_pad = w.take((size_t)d.hidden * d.in_pad * 2);
            d.up_pad = w.take((size_t)d.hidden * d.in_pad * 2);
        }
        if (!in_place(p, d.hidden, d.down_stride)) d.down_pad = w.take((size_t)d.out * d.hidden_pad * 2);
        if (backward && !in_place(p, d.out, d.y_stride)) d.dy_pad = w.take((size_t)d.rows * d.out_pad * 2);
    }
    if (const size_t n = feed_plan(d, backward)) d.part = static_cast<float*>(w.take(n));
    return w.used;
}

// ------------------------------------------------------------------ 8-bit integers
int check_quantize(const pa_quantize_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "quantize rows: p is NULL");
    if (p->rows < 0 || p->rows > (1ll << 40)) return fail(PA_ERR_INVALID_ARG, "quantize rows: rows must lie in [0, 2^40]");
    if (p->cols < 1 || p->cols > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "quantize rows: cols must lie in [1, 2^20]");
    if (p->dtype != PA_F32 && p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "quantize rows: unknown dtype %d", p->dtype);
    if (p->x_stride < p->cols || p->q_stride < p->cols) return fail(PA_ERR_INVALID_ARG, "quantize rows: row strides must be at least cols");
    if (p->q_stride % 16 != 0) return fail(PA_ERR_INVALID_ARG, "quantize rows: q_stride must be a multiple of 16");
    return PA_OK;
}

int check_int8(const pa_int8_linear_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "int8 linear: p is NULL");
    if (p->rows < 0 || p->rows > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "int8 linear: rows must lie in [0, 2^30]");
    if (p->in_features < 1) return fail(PA_ERR_INVALID_ARG, "int8 linear: in_features must be positive");
    if (p->in_features > PA_INT8_MAX_IN) return fail(PA_ERR_UNSUPPORTED, "int8 linear: in_features above %d is not built", PA_INT8_MAX_IN);
    if (p->out_features < 1 || p->out_features > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "int8 linear: out_features must lie in [1, 2^20]");
    if (p->dtype == PA_F32) return fail(PA_ERR_UNSUPPORTED, "int8 linear: fp32 is not built (PA_BF16 or PA_F16)");
    if (p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "int8 linear: unknown dtype %d", p->dtype);
    if (p->x_stride < p->in_features || p->w_stride < p->in_features || p->y_stride < p->out_features)
        return fail(PA_ERR_INVALID_ARG, "int8 linear: row strides must be at least the row's length");
    if (p->x_stride % 16 != 0 || p->w_stride % 16 != 0) return fail(PA_ERR_INVALID_ARG, "int8 linear: strides of 8-bit rows must be multiples of 16");
    if (p->x_stride > kBufferStride || p->w_stride > kBufferStride)
        return fail(PA_ERR_UNSUPPORTED, "int8 linear: strides of 8-bit rows above 2^22 are not built");
    if ((p->rows + 63) / 64 * ((p->out_features + 63) / 64) > kMaxBlocks)
        return fail(PA_ERR_UNSUPPORTED, "int8 linear: more than 2^35 outputs in a call");
    return PA_OK;
}

}  // namespace

extern "C" {

int paraanya_group_norm_workspace(const pa_group_norm_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_group(p, false)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "group norm: bytes is NULL");
        GroupDev d = group_dev(p, false);
        *bytes = group_layout(d, false, nullptr);
        return PA_OK;
    });
}

int paraanya_group_norm(const pa_group_norm_t* p, const void* x, const void* weight, const void* bias, void* y, float* mean,
                        float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_group(p, false)) return rc;
        if (p->batch == 0 || p->pixels == 0) return PA_OK;
        if (!x || !y) return fail(PA_ERR_INVALID_ARG, "group norm: x or y is NULL");
        const void* data[] = {x, y};
        const void* par[] = {weight, bias};
        if (int rc = group_align(p, data, 2, par, 2)) return rc;
        if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(PA_ERR_INVALID_ARG, "group norm: a pointer is not aligned to its element");
        GroupDev d = group_dev(p, false);
        if (int rc = check_workspace(workspace, workspace_bytes, group_layout(d, false, workspace))) return rc;
        d.x = x;
        d.w = weight;
        d.b = bias;
        d.y = y;
        d.mean = mean;
        d.rstd = rstd;
        return launched(group_forward(d, p->dtype, static_cast<hipStream_t>(stream)), "group norm launch");
    });
}

int paraanya_group_norm_backward_workspace(const pa_group_norm_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_group(p, true)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "group norm: bytes is NULL");
        GroupDev d = group_dev(p, true);
        *bytes = group_layout(d, true, nullptr);
        return PA_OK;
    });
}

int paraanya_group_norm_backward(const pa_group_norm_t* p, const void* dy, const void* x, const void* weight, const void* bias,
                                 const float* mean, const float* rstd, void* dx, void* dweight, void* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_group(p, true)) return rc;
        if (dx) {
            if (int rc = check_group_stride(p, p->dx_stride, "dx", true)) return rc;
        }
        if (p->batch > 0 && p->pixels > 0 && (!dy || !x || !mean || !rstd))
            return fail(PA_ERR_INVALID_ARG, "group norm: dy, x, mean or rstd is NULL");
        const void* data[] = {dy, x, dx};
        const void* par[] = {weight, bias, dweight, dbias};
        if (int rc = group_align(p, data, 3, par, 4)) return rc;
        if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(PA_ERR_INVALID_ARG, "group norm: a pointer is not aligned to its element");
        if (!dx && !dweight && !dbias) return PA_OK;
        GroupDev d = group_dev(p, true);
        if (int rc = check_workspace(workspace, workspace_bytes, group_layout(d, true, workspace))) return rc;
        d.dy = dy;
        d.x = x;
        d.w = weight;
        d.b = bias;
        d.mean = const_cast<float*>(mean);
        d.rstd = const_cast<float*>(rstd);
        d.dx = dx;
        d.dw = dweight;
        d.db = dbias;
        return launched(group_backward(d, p->dtype, static_cast<hipStream_t>(stream)), "group norm backward launch");
    });
}

int paraanya_feed_forward_saved(const pa_feed_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_feed(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "feed forward: bytes is NULL");
        *bytes = feed_saved(p);
        return PA_OK;
    });
}

int paraanya_feed_forward_workspace(const pa_feed_t* p, int with_saved, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_feed(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "feed forward: bytes is NULL");
        FeedDev d = feed_dev(p);
        *bytes = feed_layout(p, d, false, with_saved != 0, nullptr);
        return PA_OK;
    });
}

int paraanya_feed_forward(const pa_feed_t* p, const void* x, const void* gate, const void* gate_bias, const void* up,
                          const void* up_bias, const void* down, const void* down_bias, void* y, void* saved, size_t saved_bytes,
                          void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_feed(p)) return rc;
        if (p->rows == 0) return PA_OK;
        if (!x || !gate || !up || !down || !y) return fail(PA_ERR_INVALID_ARG, "feed forward: x, gate, up, down or y is NULL");
        const void* given[] = {x, gate, up, down};
        const void* others[] = {gate_bias, up_bias, down_bias, y};
        if (int rc = feed_align(p, given, 4, others, 4)) return rc;
        if (saved) {
            if (int rc = check_workspace(saved, saved_bytes, feed_saved(p), "saved")) return rc;
        }
        FeedDev d = feed_dev(p);
        if (int rc = check_workspace(workspace, workspace_bytes, feed_layout(p, d, false, saved != nullptr, workspace))) return rc;
        if (saved) feed_saved_parts(d, saved);
        d.x = x;
        d.gate = gate;
        d.up = up;
        d.down = down;
        d.gate_bias = gate_bias;
        d.up_bias = up_bias;
        d.down_bias = down_bias;
        d.y = y;
        return launched(feed_forward(d, p->dtype, p->activation, static_cast<hipStream_t>(stream)), "feed forward launch");
    });
}

int paraanya_feed_forward_backward_workspace(const pa_feed_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_feed(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "feed forward: bytes is NULL");
        FeedDev d = feed_dev(p);
        *bytes = feed_layout(p, d, true, true, nullptr);
        return PA_OK;
    });
}

int paraanya_feed_forward_backward(const pa_feed_t* p, const pa_feed_grad_t* g, const void* dy, const void* x, const void* gate,
                                   const void* up, const void* down, const void* saved, size_t saved_bytes, void* workspace,
                                   size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_feed(p)) return rc;
        if (!g) return fail(PA_ERR_INVALID_ARG, "feed forward: g is NULL");
        if ((g->dgate_bias && !g->dgate) || (g->dup_bias && !g->dup) || (g->ddown_bias && !g->ddown))
            return fail(PA_ERR_INVALID_ARG, "feed forward: a bias's gradient comes with its weight's");
        const void* given[] = {x, gate, up, down, dy};
        const void* others[] = {g->dx, g->dgate, g->dup, g->ddown, g->dgate_bias, g->dup_bias, g->ddown_bias};
        if (p->rows > 0 && (!dy || !x || !gate || !up || !down))
            return fail(PA_ERR_INVALID_ARG, "feed forward: dy, x, gate, up or down is NULL");
        if (int rc = feed_align(p, given, 5, others, 7)) return rc;
        if (!g->dx && !g->dgate && !g->dup && !g->ddown) return PA_OK;
        if (int rc = check_workspace(saved, saved_bytes, feed_saved(p), "saved")) return rc;
        FeedDev d = feed_dev(p);
        if (int rc = check_workspace(workspace, workspace_bytes, feed_layout(p, d, true, true, workspace))) return rc;
        feed_saved_parts(d, const_cast<void*>(saved));
        d.x = x;
        d.gate = gate;
        d.up = up;
        d.down = down;
        d.dy = dy;
        d.dx = g->dx;
        d.dgate = g->dgate;
        d.dup = g->dup;
        d.ddown = g->ddown;
        d.dgate_bias = g->dgate_bias;
        d.dup_bias = g->dup_bias;
        d.ddown_bias = g->ddown_bias;
        return launched(feed_backward(d, p->dtype, static_cast<hipStream_t>(stream)), "feed forward backward launch");
    });
}

int paraanya_quantize_rows(const pa_quantize_t* p, const void* x, int8_t* q, float* scale, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_quantize(p)) return rc;
        if (p->rows == 0) return PA_OK;
        if (!x || !q || !scale) return fail(PA_ERR_INVALID_ARG, "quantize rows: x, q or scale is NULL");
        if (misaligned(x, element_size(p->dtype)) || misaligned(scale, 4))
            return fail(PA_ERR_INVALID_ARG, "quantize rows: a pointer is not aligned to its element");
        if (misaligned(q, 16)) return fail(PA_ERR_INVALID_ARG, "quantize rows: q must be 16-byte aligned");
        QuantizeDev d{};
        d.x = x;
        d.q = q;
        d.scale = scale;
        d.rows = p->rows;
        d.x_stride = p->x_stride;
        d.q_stride = p->q_stride;
        d.cols = (int)p->cols;
        return launched(quantize_rows(d, p->dtype, static_cast<hipStream_t>(stream)), "quantize rows launch");
    });
}

int paraanya_int8_linear(const pa_int8_linear_t* p, const int8_t* xq, const float* x_scale, const int8_t* wq, const float* w_scale,
                         const void* bias, void* y, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_int8(p)) return rc;
        if (p->rows == 0) return PA_OK;
        if (!xq || !x_scale || !wq || !w_scale || !y) return fail(PA_ERR_INVALID_ARG, "int8 linear: xq, wq, a scale or y is NULL");
        if (misaligned(xq, 16) || misaligned(wq, 16)) return fail(PA_ERR_INVALID_ARG, "int8 linear: xq and wq must be 16-byte aligned");
        if (misaligned(x_scale, 4) || misaligned(w_scale, 4) || misaligned(bias, 2) || misaligned(y, 2))
            return fail(PA_ERR_INVALID_ARG, "int8 linear: a pointer is not aligned to its element");
        Int8Dev d{};
        d.x = xq;
        d.w = wq;
        d.x_scale = x_scale;
        d.w_scale = w_scale;
        d.bias = bias;
        d.y = y;
        d.rows = (int)p->rows;
        d.in = p->in_features;
        d.out = p->out_features;
        d.x_stride = p->x_stride;
        d.w_stride = p->w_stride;
        d.y_stride = p->y_stride;
        return launched(int8_linear(d, p->dtype, static_cast<hipStream_t>(stream)), "int8 linear launch");
    });
}

}  // extern "C"
