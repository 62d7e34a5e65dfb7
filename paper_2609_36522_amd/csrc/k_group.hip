// Group norm with an activation over channels-last tensors, forward and backward, for gfx950.
//
// A block takes a run of pixels (a chunk) of one sample and all or a slab of its channels: whole groups, so that
// memory is read in the order in which it lies. A thread owns 8 consecutive channels of every PP-th pixel; what
// belongs to a channel (weight, bias, its group's statistics) stays in its registers.
//
// Statistics: a chunk's values stay in registers, so that its groups' means and then the sums of squared
// differences from them are two passes over registers (no cancellation between a sum of squares and a squared
// sum). Chunks are joined by their means' distances from the group's. A slab whose pixels fit one block's registers
// is done in one launch; otherwise the chunks' statistics go to `part`, and a second launch joins them and
// normalizes.
//
// Backward: dx needs two sums over the group (g = dz w; g and g xh), which are sums over its channels of
// w times the channel's sums of dz and dz xh over pixels; those are dbias and dweight of the sample. So one pass
// over x and dy gives all sums, a small launch joins them, and a second pass writes dx.
#include "pa_act.h"
#include "pa_ops_device.h"

namespace pa {

namespace {

constexpr int kBlock = 512, kWaves = kBlock / 64;
constexpr int kMaxGroups = 512;          // groups of a slab
constexpr int kMaxSlab = kBlock * 8;     // channels of a slab

// Pixels that a thread's registers hold: 64 (16 bits) or 32 registers of x.
template <class T> constexpr int kHeld = sizeof(T) == 2 ? 16 : 8;
int held(int dtype) { return dtype == PA_F32 ? 8 : 16; }

// The block's place: its sample, channels c0 .. c0 + n - 1 and pixels p0 .. p1 - 1; the thread's piece of 8 channels
// and its first pixel (pixels beyond the last one where the thread has none).
struct Place {
    int b, c0, n, pieces, lanes, c, lane, p0, p1, own;
    __device__ __forceinline__ explicit Place(const GroupDev& d) {
        b = blockIdx.z;
        c0 = blockIdx.y * d.slab;
        n = d.channels - c0 < d.slab ? d.channels - c0 : d.slab;
        pieces = (n + 7) / 8;
        lanes = kBlock / pieces;             // threads of a piece
        lane = (int)threadIdx.x / pieces;
        c = ((int)threadIdx.x - lane * pieces) * 8;
        p0 = (int)blockIdx.x * d.chunk;
        p1 = d.pixels - p0 < d.chunk ? d.pixels : p0 + d.chunk;
        own = lane < lanes ? 1 : 0;
    }
};

// Row `p` of a tensor at this block's channels.
template <class T>
__device__ __forceinline__ const T* row_at(const void* x, const int64_t (&s)[2], const Place& q, int p) {
    return static_cast<const T*>(x) + q.b * s[0] + p * s[1] + q.c0;
}

// A channel's sums over the threads of its piece, then over the channels of each group, in a fixed order:
// v[8] of every thread -> group[g]. `lds` holds kBlock * 8 floats and kBlock + kMaxSlab after them.
__device__ __forceinline__ void channel_sums(const Place& q, const float (&v)[8], float* lds, float* channel) {
    // [lane][channel]
    const int width = q.pieces * 8;
    if (q.own) {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[q.lane * width + q.c + i] = v[i];
    }
    __syncthreads();
    // Where there are more threads than channels, several take a channel's lanes in turn.
    const int turns = width < kBlock ? kBlock / width : 1;
    for (int i = threadIdx.x; i < width * turns; i += kBlock) {
        const int t = i / width, c = i - t * width;
        float s = 0.0f;
        for (int l = t; l < q.lanes; l += turns) s += lds[l * width + c];
        channel[i] = s;
    }
    __syncthreads();
    if (turns > 1) {
        for (int c = threadIdx.x; c < width; c += kBlock) {      // at most one a thread
            float s = 0.0f;
            for (int t = 0; t < turns; ++t) s += channel[t * width + c];
            lds[c] = s;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < width; c += kBlock) channel[c] = lds[c];
        __syncthreads();
    }
}

// Sums over each group's channels: a wave a group.
__device__ __forceinline__ void group_sums(const Place& q, int width, const float* channel, float* group) {
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, groups = q.n / width;
    for (int g = w; g < groups; g += kWaves) {
        float s = 0.0f;
        for (int c = lane; c < width; c += 64) s += channel[g * width + c];
        s = wave_sum_f32(s);
        if (lane == 0) group[g] = s;
    }
    __syncthreads();
}

struct Shared {
    float lanes[kBlock * 8];
    float channel[kMaxSlab];
    float group[2][kMaxGroups];
};

// Means and sums of squared differences of the slab's groups over pixels a .. b - 1 (which the registers hold), in
// s.group[0] and [1].
template <class T>
__device__ __forceinline__ void statistics(const GroupDev& d, const Place& q, const Pack8<T> (&x)[kHeld<T>], int a, int b, Shared& s) {
    float v[8] = {};
#pragma unroll
    for (int k = 0; k < kHeld<T>; ++k) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += (float)x[k].v[i];        // zeros where there is no pixel or channel
    }
    channel_sums(q, v, s.lanes, s.channel);
    group_sums(q, d.width, s.channel, s.group[0]);
    const float n = (float)(b - a) * (float)d.width;
    for (int g = threadIdx.x; g < q.n / d.width; g += kBlock) s.group[0][g] /= n;
    __syncthreads();
    float mean[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        mean[i] = q.own && q.c + i < q.n ? s.group[0][(q.c + i) / d.width] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < kHeld<T>; ++k) {
        const bool in = q.own && a + q.lane + k * q.lanes < b;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = (float)x[k].v[i] - mean[i];
            v[i] += in && q.c + i < q.n ? e * e : 0.0f;
        }
    }
    channel_sums(q, v, s.lanes, s.channel);
    group_sums(q, d.width, s.channel, s.group[1]);
}

template <class T>
__device__ __forceinline__ void hold(const GroupDev& d, const Place& q, int a, int b, Pack8<T> (&x)[kHeld<T>]) {
#pragma unroll
    for (int k = 0; k < kHeld<T>; ++k) {
        const int p = a + q.lane + k * q.lanes;
        x[k] = load8(row_at<T>(d.x, d.xs, q, q.own && p < b ? p : a), q.c, q.n, q.own && p < b);
    }
}

template <class W>
__device__ __forceinline__ void parameters(const void* p, const Place& q, float otherwise, float (&v)[8]) {
    Pack8<W> r;
    if (p) r = load8(static_cast<const W*>(p) + q.c0, q.c, q.n, q.own);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p ? (float)r.v[i] : otherwise;
}

// act((x - mean) rstd w + b) of one piece.
template <class T, int ACT>
__device__ __forceinline__ Pack8<T> normalized(const Pack8<T>& x, const float (&mean)[8], const float (&a)[8], const float (&b)[8]) {
    Pack8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (T)activate<ACT>(fmaf((float)x.v[i] - mean[i], a[i], b[i]));
    return o;
}

// A slab's pixels in one block's registers: statistics and result in one launch.
template <class T, class W, int ACT>
__global__ __launch_bounds__(kBlock) void k_group_whole(GroupDev d) {
    __shared__ Shared s;
    const Place q(d);
    Pack8<T> x[kHeld<T>];
    hold<T>(d, q, q.p0, q.p1, x);
    float a[8], b[8], mean[8];
    parameters<W>(d.w, q, 1.0f, a);
    parameters<W>(d.b, q, 0.0f, b);
    statistics<T>(d, q, x, q.p0, q.p1, s);
    const float n = (float)(q.p1 - q.p0) * (float)d.width;
    for (int g = threadIdx.x; g < q.n / d.width; g += kBlock) {
        const float rstd = 1.0f / sqrtf(s.group[1][g] / n + d.eps);
        const int64_t at = (int64_t)q.b * d.groups + q.c0 / d.width + g;
        if (d.mean) d.mean[at] = s.group[0][g];
        if (d.rstd) d.rstd[at] = rstd;
        s.group[1][g] = rstd;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int g = q.own && q.c + i < q.n ? (q.c + i) / d.width : 0;
        mean[i] = s.group[0][g];
        a[i] *= s.group[1][g];
    }
#pragma unroll
    for (int k = 0; k < kHeld<T>; ++k) {
        const int p = q.p0 + q.lane + k * q.lanes;
        if (q.own && p < q.p1)
            store8(const_cast<T*>(row_at<T>(d.y, d.ys, q, p)) + q.c, normalized<T, ACT>(x[k], mean, a, b), q.n - q.c);
    }
}

// Statistics of a chunk, one run of pixels that the registers hold after the other.
template <class T>
__global__ __launch_bounds__(kBlock) void k_group_stats(GroupDev d) {
    __shared__ Shared s;
    __shared__ float run[2][kMaxGroups];
    const Place q(d);
    const int step = q.lanes * kHeld<T>;
    for (int a = q.p0; a < q.p1; a += step) {
        const int b = q.p1 - a < step ? q.p1 : a + step;
        Pack8<T> x[kHeld<T>];
        hold<T>(d, q, a, b, x);
        statistics<T>(d, q, x, a, b, s);
        const float n0 = (float)(a - q.p0) * (float)d.width, n1 = (float)(b - a) * (float)d.width;
        for (int g = threadIdx.x; g < q.n / d.width; g += kBlock) {
            float m = s.group[0][g], m2 = s.group[1][g];
            if (a > q.p0) {
                const float e = m - run[0][g];
                m = run[0][g] + e * (n1 / (n0 + n1));
                m2 = run[1][g] + m2 + e * e * (n0 * n1 / (n0 + n1));
            }
            run[0][g] = m;
            run[1][g] = m2;
        }
        __syncthreads();
    }
    for (int g = threadIdx.x; g < q.n / d.width; g += kBlock) {
        float* out = d.part + (((int64_t)q.b * d.groups + q.c0 / d.width + g) * d.chunks + blockIdx.x) * 2;
        out[0] = run[0][g];
        out[1] = run[1][g];
    }
}

// Joins the chunks' statistics (every block for its own groups, a wave a group) and writes the chunk's results.
template <class T, class W, int ACT>
__global__ __launch_bounds__(kBlock) void k_group_apply(GroupDev d) {
    __shared__ float group[2][kMaxGroups];
    const Place q(d);
    float a[8], b[8], mean[8];
    parameters<W>(d.w, q, 1.0f, a);
    parameters<W>(d.b, q, 0.0f, b);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const float total = (float)d.pixels * (float)d.width, each = (float)d.chunk * (float)d.width;
    const float rest = total - each * (float)(d.chunks - 1);
    for (int g = wave; g < q.n / d.width; g += kWaves) {
        const int64_t at = (int64_t)q.b * d.groups + q.c0 / d.width + g;
        const float* in = d.part + at * d.chunks * 2;
        float m = 0.0f, m2 = 0.0f;
        for (int k = lane; k < d.chunks; k += 64) m += in[2 * k] * ((k + 1 < d.chunks ? each : rest) / total);
        m = wave_sum_f32(m);
        for (int k = lane; k < d.chunks; k += 64) {
            const float e = in[2 * k] - m;
            m2 += in[2 * k + 1] + e * e * (k + 1 < d.chunks ? each : rest);
        }
        m2 = wave_sum_f32(m2);
        if (lane == 0) {
            const float rstd = 1.0f / sqrtf(m2 / total + d.eps);
            group[0][g] = m;
            group[1][g] = rstd;
            if (blockIdx.x == 0) {
                if (d.mean) d.mean[at] = m;
                if (d.rstd) d.rstd[at] = rstd;
            }
        }
    }
    __syncthreads();
    if (!q.own) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int g = q.c + i < q.n ? (q.c + i) / d.width : 0;
        mean[i] = group[0][g];
        a[i] *= group[1][g];
    }
    for (int p = q.p0 + q.lane; p < q.p1; p += 4 * q.lanes) {
        Pack8<T> x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            x[k] = load8(row_at<T>(d.x, d.xs, q, p + k * q.lanes < q.p1 ? p + k * q.lanes : p), q.c, q.n);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (p + k * q.lanes < q.p1)
                store8(const_cast<T*>(row_at<T>(d.y, d.ys, q, p + k * q.lanes)) + q.c, normalized<T, ACT>(x[k], mean, a, b), q.n - q.c);
    }
}

// ------------------------------------------------------------------ backward
struct Channels {                    // of the thread's 8: group mean, rstd, weight, bias
    float mean[8], rstd[8], w[8], b[8];
};

template <class W>
__device__ __forceinline__ Channels channels(const GroupDev& d, const Place& q) {
    Channels k;
    parameters<W>(d.w, q, 1.0f, k.w);
    parameters<W>(d.b, q, 0.0f, k.b);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t at = (int64_t)q.b * d.groups + (q.c0 + (q.own && q.c + i < q.n ? q.c + i : 0)) / d.width;
        k.mean[i] = d.mean[at];
        k.rstd[i] = d.rstd[at];
    }
    return k;
}

// {xh, dz} of element i.
template <int ACT>
__device__ __forceinline__ float2 through(const Channels& k, float x, float dy, int i) {
    const float xh = (x - k.mean[i]) * k.rstd[i];
    return make_float2(xh, ACT == PA_ACT_NONE ? dy : dy * activate_grad<ACT>(fmaf(xh, k.w[i], k.b[i])).y);
}

// Sums over a chunk's pixels of dz xh and dz for each channel.
template <class T, class W, int ACT>
__global__ __launch_bounds__(kBlock) void k_group_sums(GroupDev d) {
    __shared__ float lanes[kBlock * 8];
    __shared__ float channel[kMaxSlab];
    const Place q(d);
    const Channels ch = channels<W>(d, q);
    float sw[8] = {}, sb[8] = {};
    if (q.own) {
        for (int p = q.p0 + q.lane; p < q.p1; p += 2 * q.lanes) {
            Pack8<T> x[2], dy[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const bool in = p + k * q.lanes < q.p1;
                x[k] = load8(row_at<T>(d.x, d.xs, q, in ? p + k * q.lanes : p), q.c, q.n);
                dy[k] = load8(row_at<T>(d.dy, d.ys, q, in ? p + k * q.lanes : p), q.c, q.n);
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if (p + k * q.lanes >= q.p1) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 t = through<ACT>(ch, (float)x[k].v[i], (float)dy[k].v[i], i);
                    sw[i] += t.y * t.x;
                    sb[i] += t.y;
                }
            }
        }
    }
    float* out = d.part + ((int64_t)q.b * d.chunks + blockIdx.x) * 2 * d.channels + q.c0;
    channel_sums(q, sw, lanes, channel);
    for (int c = threadIdx.x; c < q.n; c += kBlock) out[c] = channel[c];
    __syncthreads();
    channel_sums(q, sb, lanes, channel);
    for (int c = threadIdx.x; c < q.n; c += kBlock) out[d.channels + c] = channel[c];
}

// A sample's group: the channels' sums over the chunks, and from them the means over the group of g xh and g.
template <class W>
__global__ __launch_bounds__(256) void k_group_join(GroupDev d) {
    __shared__ float sum[2][256], red[2][4];
    const int g = blockIdx.x, b = blockIdx.y, L = d.width;
    // Threads of a channel: the chunks in turn.
    const int turns = L < 256 ? 256 / L : 1, t = (int)threadIdx.x / L, span = L < 256 ? L : 256;
    float m[2] = {};
    for (int c0 = 0; c0 < L; c0 += span) {
        const int c = c0 + (L < 256 ? (int)threadIdx.x - t * L : (int)threadIdx.x), ch = g * L + c;
        float v[2] = {};
        const bool own = c < L && (L >= 256 || t < turns);
        if (own)
            for (int k = L < 256 ? t : 0; k < d.chunks; k += turns) {
                const float* in = d.part + ((int64_t)b * d.chunks + k) * 2 * d.channels + ch;
                v[0] += in[0];
                v[1] += in[d.channels];
            }
        sum[0][threadIdx.x] = v[0];
        sum[1][threadIdx.x] = v[1];
        __syncthreads();
        if (own && (L >= 256 || t == 0)) {
            for (int k = 1; k < turns; ++k) {
                v[0] += sum[0][threadIdx.x + k * L];
                v[1] += sum[1][threadIdx.x + k * L];
            }
            float* out = d.sums + (int64_t)b * 2 * d.channels + ch;
            out[0] = v[0];
            out[d.channels] = v[1];
            const float w = d.w ? (float)static_cast<const W*>(d.w)[ch] : 1.0f;
            m[0] += v[1] * w;
            m[1] += v[0] * w;
        }
        __syncthreads();
    }
    for (int i = 0; i < 2; ++i) {
        const float s = wave_sum_f32(m[i]);
        if ((threadIdx.x & 63) == 0) red[i][threadIdx.x >> 6] = s;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        const float* r = red[threadIdx.x];
        d.means[((int64_t)b * d.groups + g) * 2 + threadIdx.x] = ((r[0] + r[1]) + (r[2] + r[3])) / ((float)d.pixels * (float)L);
    }
}

template <class T, class W, int ACT>
__global__ __launch_bounds__(kBlock) void k_group_dx(GroupDev d) {
    const Place q(d);
    if (!q.own) return;
    Channels ch = channels<W>(d, q);
    float m1[8], m2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t at = (int64_t)q.b * d.groups + (q.c0 + (q.c + i < q.n ? q.c + i : 0)) / d.width;
        m1[i] = d.means[2 * at];
        m2[i] = d.means[2 * at + 1];
    }
    for (int p = q.p0 + q.lane; p < q.p1; p += 2 * q.lanes) {
        Pack8<T> x[2], dy[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const bool in = p + k * q.lanes < q.p1;
            x[k] = load8(row_at<T>(d.x, d.xs, q, in ? p + k * q.lanes : p), q.c, q.n);
            dy[k] = load8(row_at<T>(d.dy, d.ys, q, in ? p + k * q.lanes : p), q.c, q.n);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (p + k * q.lanes >= q.p1) continue;
            Pack8<T> o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 t = through<ACT>(ch, (float)x[k].v[i], (float)dy[k].v[i], i);
                o.v[i] = (T)(ch.rstd[i] * (t.y * ch.w[i] - m1[i] - t.x * m2[i]));
            }
            store8(const_cast<T*>(row_at<T>(d.dx, d.dxs, q, p + k * q.lanes)) + q.c, o, q.n - q.c);
        }
    }
}

// dweight (blockIdx.y 0) and dbias from the samples' sums, in order.
template <class W>
__global__ __launch_bounds__(256) void k_group_params(GroupDev d) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    W* out = static_cast<W*>(blockIdx.y ? d.db : d.dw);
    if (!out || c >= d.channels) return;
    float s = 0.0f;
#pragma unroll 8
    for (int b = 0; b < d.batch; ++b) s += d.sums[((int64_t)b * 2 + blockIdx.y) * d.channels + c];
    out[c] = (W)s;
}

template <class F>
hipError_t dispatch(int dtype, int param_dtype, int act, F f) {
    auto with_act = [&](auto t, auto w) {
        if (act == PA_ACT_SILU) return f(t, w, std::integral_constant<int, PA_ACT_SILU>{});
        if (act == PA_ACT_GELU) return f(t, w, std::integral_constant<int, PA_ACT_GELU>{});
        return f(t, w, std::integral_constant<int, PA_ACT_NONE>{});
    };
    const bool pf = param_dtype == PA_F32;
    if (dtype == PA_F32) return with_act((float)0, (float)0);
    if (dtype == PA_BF16) return pf ? with_act((__bf16)0, (float)0) : with_act((__bf16)0, (__bf16)0);
    return pf ? with_act((_Float16)0, (float)0) : with_act((_Float16)0, (_Float16)0);
}

}  // namespace

// Slabs of whole groups and of whole pieces of 8 channels. The smallest such slab (with at least 32 channels, so that a
// pixel's piece of it is no smaller than a cache line's sector) if a block's registers hold its pixels, and if the
// tensor is small enough to be bound by latency or there are slabs for every CU; otherwise as many groups
// as a block can take, in chunks of pixels.
void group_plan(GroupDev& d, int dtype, bool backward) {
    d.width = d.channels / d.groups;
    int unit = 1;                                   // groups whose channels make whole pieces
    while (unit < 8 && d.width * unit % 8 != 0) unit *= 2;
    const int most = kMaxSlab / d.width < kMaxGroups ? kMaxSlab / d.width : kMaxGroups;
    auto slab = [&](int groups) {
        if (groups > d.groups) groups = d.groups;
        if (groups > most) groups = most >= unit ? most / unit * unit : most;
        d.slab = groups * d.width;
        d.slabs = (d.channels + d.slab - 1) / d.slab;
    };
    const int small = (32 + d.width * unit - 1) / (d.width * unit) * unit;
    slab(small);
    const int64_t fits = (int64_t)(kBlock / ((d.slab + 7) / 8)) * held(dtype);
    const int64_t bytes = (int64_t)d.batch * d.pixels * d.channels * (dtype == PA_F32 ? 4 : 2);
    if (!backward && d.pixels <= fits && (bytes <= (4 << 20) || (int64_t)d.batch * d.slabs >= 256)) {
        d.chunk = d.pixels > 0 ? d.pixels : 1;
        d.chunks = 1;
        return;
    }
    slab(d.groups);
    // What the registers hold at a time, fewer where that gives too few blocks, and more beyond 256 chunks a sample.
    const int lanes = kBlock / ((d.slab + 7) / 8);
    const int64_t per = (int64_t)d.batch * d.slabs;
    int64_t chunk = (int64_t)lanes * (backward ? 8 : held(dtype));
    while (chunk > lanes * 2 && (d.pixels + chunk - 1) / chunk * per < 512) chunk /= 2;
    if ((d.pixels + chunk - 1) / chunk > 256) chunk = (d.pixels + 255) / 256;
    d.chunk = (int)(chunk < 1 ? 1 : chunk);
    d.chunks = d.pixels > 0 ? (d.pixels + d.chunk - 1) / d.chunk : 1;
}

hipError_t group_forward(const GroupDev& d, int dtype, int param_dtype, int act, hipStream_t st) {
    return dispatch(dtype, param_dtype, act, [&](auto t, auto w, auto a) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int ACT = decltype(a)::value;
        const dim3 grid((unsigned)d.chunks, (unsigned)d.slabs, (unsigned)d.batch);
        if (!d.part) {
            k_group_whole<T, W, ACT><<<grid, kBlock, 0, st>>>(d);
            return hipGetLastError();
        }
        k_group_stats<T><<<grid, kBlock, 0, st>>>(d);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        k_group_apply<T, W, ACT><<<grid, kBlock, 0, st>>>(d);
        return hipGetLastError();
    });
}

hipError_t group_backward(const GroupDev& d, int dtype, int param_dtype, int act, hipStream_t st) {
    return dispatch(dtype, param_dtype, act, [&](auto t, auto w, auto a) {
        typedef decltype(t) T;
        typedef decltype(w) W;
        constexpr int ACT = decltype(a)::value;
        const dim3 grid((unsigned)d.chunks, (unsigned)d.slabs, (unsigned)d.batch);
        if (d.pixels > 0 && d.batch > 0) {
            k_group_sums<T, W, ACT><<<grid, kBlock, 0, st>>>(d);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            k_group_join<W><<<dim3((unsigned)d.groups, (unsigned)d.batch), 256, 0, st>>>(d);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            if (d.dx) {
                k_group_dx<T, W, ACT><<<grid, kBlock, 0, st>>>(d);
                e = hipGetLastError();
                if (e != hipSuccess) return e;
            }
        }
        if (d.dw || d.db) {
            GroupDev c = d;
            if (d.pixels == 0) c.batch = 0;
            k_group_params<W><<<dim3((unsigned)((d.channels + 255) / 256), 2), 256, 0, st>>>(c);
        }
        return hipGetLastError();
    });
}

}  // namespace pa
