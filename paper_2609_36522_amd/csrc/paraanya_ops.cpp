// Host side of the operators declared in include/paraanya_ops.h: argument checks (before any HIP
// call), workspace layout, launches. Stateless; nothing is allocated.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>

#include "pa_ops_host.h"

using namespace pa;

namespace {

constexpr int64_t kMaxBlocks = 1 << 23;       // a grid holds fewer than 2^32 threads

// ------------------------------------------------------------------ layer norm
int check_norm(const pa_norm_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "layer norm: p is NULL");
    if (p->rows < 0 || p->rows > (1ll << 40)) return fail(PA_ERR_INVALID_ARG, "layer norm: rows must lie in [0, 2^40]");
    if (p->cols < 1 || p->cols > PA_NORM_MAX_COLS) return fail(PA_ERR_INVALID_ARG, "layer norm: cols must lie in [1, %d]", PA_NORM_MAX_COLS);
    if (p->dtype != PA_F32 && p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "layer norm: unknown dtype %d", p->dtype);
    if (p->param_dtype != p->dtype && p->param_dtype != PA_F32)
        return fail(PA_ERR_INVALID_ARG, "layer norm: param_dtype must be dtype or PA_F32");
    if (!(p->eps >= 0.0) || !(p->eps <= 1e30)) return fail(PA_ERR_INVALID_ARG, "layer norm: eps must be finite and not negative");
    if (p->x_stride < p->cols || p->y_stride < p->cols) return fail(PA_ERR_INVALID_ARG, "layer norm: row strides must be at least cols");
    return PA_OK;
}

int norm_align(const pa_norm_t* p, const void* const* data, int n, const void* const* par, int np) {
    for (int i = 0; i < n; ++i)
        if (misaligned(data[i], element_size(p->dtype))) return fail(PA_ERR_INVALID_ARG, "layer norm: a pointer is not aligned to its element");
    for (int i = 0; i < np; ++i)
        if (misaligned(par[i], element_size(p->param_dtype))) return fail(PA_ERR_INVALID_ARG, "layer norm: a pointer is not aligned to its element");
    return PA_OK;
}

size_t norm_workspace(const pa_norm_t* p) {
    return round256((size_t)pa::norm_backward_blocks(p->rows, p->cols) * 2 * p->cols * sizeof(float));
}

// ------------------------------------------------------------------ cross attention
int check_stride(const int64_t s[3], const char* what) {
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || s[i] > (1ll << 40)) return fail(PA_ERR_INVALID_ARG, "cross attention: stride %d of %s out of range", i, what);
    return PA_OK;
}

// Outputs: distinct elements at distinct addresses need strides that are not 0 (one without elements may have any).
int check_out_stride(const int64_t s[3], int64_t b, int64_t l, int64_t h, int dim, const char* what) {
    if (int rc = check_stride(s, what)) return rc;
    if (b == 0 || l == 0) return PA_OK;
    if ((b > 1 && s[0] == 0) || (l > 1 && s[1] < dim) || (h > 1 && s[2] < dim))
        return fail(PA_ERR_INVALID_ARG, "cross attention: %s overlaps itself", what);
    return PA_OK;
}

int check_cross(const pa_cross_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "cross attention: p is NULL");
    if (p->batch < 0 || p->batch > 65535) return fail(PA_ERR_INVALID_ARG, "cross attention: batch must lie in [0, 65535]");
    if (p->q_len < 0 || p->q_len > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "cross attention: q_len must lie in [0, 2^30]");
    if (p->kv_len < 0 || p->kv_len > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "cross attention: kv_len must lie in [0, 2^30]");
    if (p->q_heads < 1 || p->q_heads > 65535 || p->kv_heads < 1 || p->q_heads % p->kv_heads != 0)
        return fail(PA_ERR_INVALID_ARG, "cross attention: q_heads must be a multiple of kv_heads");
    if (p->q_len * p->q_heads > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "cross attention: q_len * q_heads exceeds 2^30");
    if (p->head_dim < 1) return fail(PA_ERR_INVALID_ARG, "cross attention: head_dim must be positive");
    if (p->head_dim > 128) return fail(PA_ERR_UNSUPPORTED, "cross attention: head_dim above 128 is not built");
    if (p->dtype == PA_F32) return fail(PA_ERR_UNSUPPORTED, "cross attention: fp32 is not built (PA_BF16 or PA_F16)");
    if (p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "cross attention: unknown dtype %d", p->dtype);
    if (!(fabs(p->scale) <= 1e30)) return fail(PA_ERR_INVALID_ARG, "cross attention: scale must be finite");
    if (p->mask_kind != PA_MASK_NONE && p->mask_kind != PA_MASK_BOOL && p->mask_kind != PA_MASK_ADD)
        return fail(PA_ERR_INVALID_ARG, "cross attention: unknown mask_kind %d", p->mask_kind);
    if ((p->mask_kind != PA_MASK_NONE) != (p->mask != nullptr) && p->batch * p->kv_len > 0)
        return fail(PA_ERR_INVALID_ARG, "cross attention: mask and mask_kind disagree");
    if (p->mask_kind == PA_MASK_ADD && misaligned(p->mask, 4)) return fail(PA_ERR_INVALID_ARG, "cross attention: mask is not aligned to its element");
    if (p->mask_stride < 0) return fail(PA_ERR_INVALID_ARG, "cross attention: mask_stride must not be negative");
    if (misaligned(p->kv_lens, 4)) return fail(PA_ERR_INVALID_ARG, "cross attention: kv_lens is not aligned to its element");
    if (int rc = check_stride(p->q_stride, "q")) return rc;
    if (int rc = check_stride(p->k_stride, "k")) return rc;
    if (int rc = check_stride(p->v_stride, "v")) return rc;
    if (int rc = check_out_stride(p->o_stride, p->batch, p->q_len, p->q_heads, p->head_dim, "o")) return rc;
    // Blocks of 32 rows or keys, and threads of the passes over them, fit a grid.
    const int64_t rows = p->batch * p->q_len * p->q_heads, keys = p->batch * p->kv_len * p->kv_heads;
    if (rows > (1ll << 27) || keys > (1ll << 30) || p->batch * p->kv_heads > kMaxBlocks)
        return fail(PA_ERR_UNSUPPORTED, "cross attention: more than 2^27 rows or 2^30 keys in a call");
    return PA_OK;
}

pa::CrossDev cross_dev(const pa_cross_t* p, bool backward) {
    pa::CrossDev d{};
    d.kv_lens = p->kv_lens;
    d.mask = p->mask;
    d.mask_kind = p->mask_kind;
    d.mask_stride = p->mask_stride;
    d.batch = (int)p->batch;
    d.q_heads = p->q_heads;
    d.kv_heads = p->kv_heads;
    d.group = p->q_heads / p->kv_heads;
    d.q_len = (int)p->q_len;
    d.kv_len = (int)p->kv_len;
    d.dim = p->head_dim;
    d.rows = (int)(p->q_len * d.group);
    d.scale = (float)p->scale;
    for (int i = 0; i < 3; ++i) {
        d.qs[i] = p->q_stride[i];
        d.ks[i] = p->k_stride[i];
        d.vs[i] = p->v_stride[i];
        d.os[i] = p->o_stride[i];
    }
    pa::cross_plan(d, backward);
    return d;
}

// The workspace's parts; returns its size (all that is wanted of a workspace that is not there).
size_t cross_layout(pa::CrossDev& d, bool backward, void* ws) {
    size_t used = 0;
    auto take = [&](size_t floats) {
        float* p = ws ? reinterpret_cast<float*>(static_cast<char*>(ws) + used) : nullptr;
        used += round256(floats * sizeof(float));
        return p;
    };
    const size_t keys = (size_t)d.batch * d.kv_heads * d.kv_len;
    if (d.whole < d.tiles) {
        const size_t parts = (size_t)(d.tiles - d.whole) * d.splits * d.tile_rows;
        d.part = take(parts * d.dim);
        if (!backward) d.part_stats = take(parts * 2);
    }
    if (backward) {
        d.row_stats = take((size_t)d.batch * d.q_heads * ((d.q_len + 31) / 32) * 96);
        if (d.row_splits > 1) {
            d.part_dk = take((size_t)d.row_splits * keys * d.dim);
            d.part_dv = take((size_t)d.row_splits * keys * d.dim);
        }
    }
    return used;
}

// ------------------------------------------------------------------ projection with adapters
int check_lora(const pa_lora_t* p) {
    if (!p) return fail(PA_ERR_INVALID_ARG, "lora linear: p is NULL");
    if (p->rows < 0 || p->rows > (1 << 30)) return fail(PA_ERR_INVALID_ARG, "lora linear: rows must lie in [0, 2^30]");
    if (p->in_features < 1 || p->in_features > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "lora linear: in_features must lie in [1, 2^20]");
    if (p->out_features < 1 || p->out_features > (1 << 20)) return fail(PA_ERR_INVALID_ARG, "lora linear: out_features must lie in [1, 2^20]");
    if (p->rank < 1) return fail(PA_ERR_INVALID_ARG, "lora linear: rank must be positive");
    if (p->rank > PA_LORA_MAX_RANK) return fail(PA_ERR_UNSUPPORTED, "lora linear: rank above %d is not built", PA_LORA_MAX_RANK);
    if (p->adapters < 0) return fail(PA_ERR_INVALID_ARG, "lora linear: adapters must not be negative");
    if (p->requests < 0 || p->requests > 65535) return fail(PA_ERR_INVALID_ARG, "lora linear: requests must lie in [0, 65535]");
    if (p->dtype == PA_F32) return fail(PA_ERR_UNSUPPORTED, "lora linear: fp32 is not built (PA_BF16 or PA_F16)");
    if (p->dtype != PA_BF16 && p->dtype != PA_F16) return fail(PA_ERR_INVALID_ARG, "lora linear: unknown dtype %d", p->dtype);
    if (p->x_stride < p->in_features || p->w_stride < p->in_features || p->y_stride < p->out_features)
        return fail(PA_ERR_INVALID_ARG, "lora linear: row strides must be at least the row's length");
    if (p->requests > 0 && p->adapters > 0 && (!p->offsets || !p->ids)) return fail(PA_ERR_INVALID_ARG, "lora linear: offsets or ids is NULL");
    if (misaligned(p->offsets, 4) || misaligned(p->ids, 4) || misaligned(p->scales, 4))
        return fail(PA_ERR_INVALID_ARG, "lora linear: a pointer is not aligned to its element");
    if ((p->rows + 31) / 32 * ((p->out_features + 31) / 32) > kMaxBlocks * 4)
        return fail(PA_ERR_UNSUPPORTED, "lora linear: more than 2^35 outputs in a call");
    return PA_OK;
}

size_t lora_workspace(const pa_lora_t* p) {
    if (p->requests == 0 || p->adapters == 0) return 0;
    return round256((size_t)p->rows * ((p->rank + 15) / 16 * 16) * 2);
}

}  // namespace

extern "C" {

int paraanya_layer_norm(const pa_norm_t* p, const void* x, const void* weight, const void* bias, void* y, float* mean,
                        float* rstd, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_norm(p)) return rc;
        if (p->rows == 0) return PA_OK;
        if (!x || !y) return fail(PA_ERR_INVALID_ARG, "layer norm: x or y is NULL");
        const void* data[] = {x, y};
        const void* par[] = {weight, bias};
        if (int rc = norm_align(p, data, 2, par, 2)) return rc;
        if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(PA_ERR_INVALID_ARG, "layer norm: a pointer is not aligned to its element");
        pa::NormDev d{};
        d.x = x;
        d.w = weight;
        d.b = bias;
        d.y = y;
        d.mean = mean;
        d.rstd = rstd;
        d.rows = p->rows;
        d.cols = (int)p->cols;
        d.x_stride = p->x_stride;
        d.y_stride = p->y_stride;
        d.eps = (float)p->eps;
        return launched(pa::norm_forward(d, p->dtype, p->param_dtype, static_cast<hipStream_t>(stream)), "layer norm launch");
    });
}

int paraanya_layer_norm_backward_workspace(const pa_norm_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_norm(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "layer norm: bytes is NULL");
        *bytes = norm_workspace(p);
        return PA_OK;
    });
}

int paraanya_layer_norm_backward(const pa_norm_t* p, const void* dy, const void* x, const float* mean, const float* rstd,
                                 const void* weight, void* dx, void* dweight, void* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_norm(p)) return rc;
        if (p->rows > 0 && (!dy || !x || !mean || !rstd)) return fail(PA_ERR_INVALID_ARG, "layer norm: dy, x, mean or rstd is NULL");
        if (dx && p->dx_stride < p->cols) return fail(PA_ERR_INVALID_ARG, "layer norm: row strides must be at least cols");
        const void* data[] = {dy, x, dx};
        const void* par[] = {weight, dweight, dbias};
        if (int rc = norm_align(p, data, 3, par, 3)) return rc;
        if (misaligned(mean, 4) || misaligned(rstd, 4)) return fail(PA_ERR_INVALID_ARG, "layer norm: a pointer is not aligned to its element");
        if (!dx && !dweight && !dbias) return PA_OK;
        const bool sums = dweight || dbias;
        if (int rc = check_workspace(workspace, workspace_bytes, sums ? norm_workspace(p) : 0)) return rc;
        pa::NormDev d{};
        d.dy = dy;
        d.x = x;
        d.w = weight;
        d.dx = dx;
        d.dw = dweight;
        d.db = dbias;
        d.mean = const_cast<float*>(mean);
        d.rstd = const_cast<float*>(rstd);
        d.part = sums ? static_cast<float*>(workspace) : nullptr;
        d.rows = p->rows;
        d.cols = (int)p->cols;
        d.x_stride = p->x_stride;
        d.y_stride = p->y_stride;
        d.dx_stride = p->dx_stride;
        d.blocks = pa::norm_backward_blocks(p->rows, p->cols);
        return launched(pa::norm_backward(d, p->dtype, p->param_dtype, static_cast<hipStream_t>(stream)), "layer norm backward launch");
    });
}

int paraanya_cross_attention_workspace(const pa_cross_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_cross(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "cross attention: bytes is NULL");
        pa::CrossDev d = cross_dev(p, false);
        *bytes = cross_layout(d, false, nullptr);
        return PA_OK;
    });
}

int paraanya_cross_attention(const pa_cross_t* p, const void* q, const void* k, const void* v, void* o, float* stats,
                             void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_cross(p)) return rc;
        if (p->batch == 0 || p->q_len == 0) return PA_OK;
        if (!q || !o || (p->kv_len > 0 && (!k || !v))) return fail(PA_ERR_INVALID_ARG, "cross attention: q, k, v or o is NULL");
        if (misaligned(q, 2) || misaligned(k, 2) || misaligned(v, 2) || misaligned(o, 2) || misaligned(stats, 4))
            return fail(PA_ERR_INVALID_ARG, "cross attention: a pointer is not aligned to its element");
        pa::CrossDev d = cross_dev(p, false);
        if (int rc = check_workspace(workspace, workspace_bytes, cross_layout(d, false, workspace))) return rc;
        d.q = q;
        d.k = k;
        d.v = v;
        d.o = o;
        d.stats = stats;
        return launched(pa::cross_forward(d, p->dtype, static_cast<hipStream_t>(stream)), "cross attention launch");
    });
}

int paraanya_cross_attention_backward_workspace(const pa_cross_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_cross(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "cross attention: bytes is NULL");
        pa::CrossDev d = cross_dev(p, true);
        *bytes = cross_layout(d, true, nullptr);
        return PA_OK;
    });
}

int paraanya_cross_attention_backward(const pa_cross_t* p, const pa_cross_grad_t* g, const void* d_o, const void* q, const void* k,
                                      const void* v, const void* o, const float* stats, void* dq, void* dk, void* dv,
                                      void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_cross(p)) return rc;
        if (!g) return fail(PA_ERR_INVALID_ARG, "cross attention: g is NULL");
        if ((dk == nullptr) != (dv == nullptr)) return fail(PA_ERR_INVALID_ARG, "cross attention: dk and dv are given together or not at all");
        if (int rc = check_stride(g->do_stride, "do")) return rc;
        if (dq) {
            if (int rc = check_out_stride(g->dq_stride, p->batch, p->q_len, p->q_heads, p->head_dim, "dq")) return rc;
        }
        if (dk) {
            if (int rc = check_out_stride(g->dk_stride, p->batch, p->kv_len, p->kv_heads, p->head_dim, "dk")) return rc;
            if (int rc = check_out_stride(g->dv_stride, p->batch, p->kv_len, p->kv_heads, p->head_dim, "dv")) return rc;
        }
        if (p->batch == 0 || (!dq && !dk)) return PA_OK;
        if (p->q_len > 0 && (!q || !d_o || !o || !stats)) return fail(PA_ERR_INVALID_ARG, "cross attention: do, q, o or stats is NULL");
        if (p->kv_len > 0 && (!k || !v)) return fail(PA_ERR_INVALID_ARG, "cross attention: k or v is NULL");
        if (misaligned(q, 2) || misaligned(k, 2) || misaligned(v, 2) || misaligned(o, 2) || misaligned(d_o, 2) ||
            misaligned(dq, 2) || misaligned(dk, 2) || misaligned(dv, 2) || misaligned(stats, 4))
            return fail(PA_ERR_INVALID_ARG, "cross attention: a pointer is not aligned to its element");
        pa::CrossDev d = cross_dev(p, true);
        if (int rc = check_workspace(workspace, workspace_bytes, cross_layout(d, true, workspace))) return rc;
        d.q = q;
        d.k = k;
        d.v = v;
        d.o = const_cast<void*>(o);
        d.d_o = d_o;
        d.stats = const_cast<float*>(stats);
        d.dq = dq;
        d.dk = dk;
        d.dv = dv;
        for (int i = 0; i < 3; ++i) {
            d.dos[i] = g->do_stride[i];
            d.dqs[i] = g->dq_stride[i];
            d.dks[i] = g->dk_stride[i];
            d.dvs[i] = g->dv_stride[i];
        }
        return launched(pa::cross_backward(d, p->dtype, static_cast<hipStream_t>(stream)), "cross attention backward launch");
    });
}

int paraanya_lora_linear_workspace(const pa_lora_t* p, size_t* bytes) {
    return guarded([&]() -> int {
        if (int rc = check_lora(p)) return rc;
        if (!bytes) return fail(PA_ERR_INVALID_ARG, "lora linear: bytes is NULL");
        *bytes = lora_workspace(p);
        return PA_OK;
    });
}

int paraanya_lora_linear(const pa_lora_t* p, const void* x, const void* weight, const void* bias, const void* a, const void* b,
                         void* y, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&]() -> int {
        if (int rc = check_lora(p)) return rc;
        if (p->rows == 0) return PA_OK;
        const bool adapted = p->requests > 0 && p->adapters > 0;
        if (!x || !weight || !y || (adapted && (!a || !b))) return fail(PA_ERR_INVALID_ARG, "lora linear: x, weight, a, b or y is NULL");
        if (misaligned(x, 2) || misaligned(weight, 2) || misaligned(bias, 2) || misaligned(a, 2) || misaligned(b, 2) || misaligned(y, 2))
            return fail(PA_ERR_INVALID_ARG, "lora linear: a pointer is not aligned to its element");
        if (int rc = check_workspace(workspace, workspace_bytes, lora_workspace(p))) return rc;
        pa::LoraDev d{};
        d.x = x;
        d.w = weight;
        d.bias = bias;
        d.a = a;
        d.b = b;
        d.y = y;
        d.t = workspace;
        d.offsets = p->offsets;
        d.ids = p->ids;
        d.scales = p->scales;
        d.rows = (int)p->rows;
        d.in = p->in_features;
        d.out = p->out_features;
        d.rank = p->rank;
        d.rank_pad = (p->rank + 15) / 16 * 16;
        d.adapters = adapted ? p->adapters : 0;
        d.requests = adapted ? p->requests : 0;
        d.x_stride = p->x_stride;
        d.w_stride = p->w_stride;
        d.y_stride = p->y_stride;
        return launched(pa::lora_linear(d, p->dtype, static_cast<hipStream_t>(stream)), "lora linear launch");
    });
}

}  // extern "C"
