// Group norm with an activation over channels-last tensors, forward and backward, for gfx950.
//
// A block takes a run of pixels (a chunk) of one sample and all or a slab of its channels: whole groups, so that
// memory is read in the order in which it lies. A thread owns 8 consecutive channels of every `lanes`-th pixel; what
// belongs to a channel (weight, bias, its group's statistics) stays in its registers.
//
// Statistics: a thread takes a batch of pixels at a time, whose mean and sum of squared differences from it are two
// passes over registers, and joins them to what it has by the distance of the means; so do threads and then
// chunks (no cancellation between a sum of squares and a squared sum anywhere). A slab whose pixels fit one
// block's registers is done in one launch; otherwise the chunks' statistics go to `part`, and a second launch joins
// them and normalizes.
//
// Backward: dx needs two sums over the group (g = dz w; g and g xh), which are sums over its channels of
// w times the channel's sums of dz and dz xh over pixels; those are dbias and dweight of the sample. So one pass
// over x and dy gives all sums, a small launch joins them, and a second pass writes dx (and joins the samples'
// sums). Slabs that fit registers take one launch, and one for the samples' sums.
#include <type_traits>

#include "pa_act.h"
#include "pa_mma.h"

namespace pa {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 512, kWaves = kBlock / 64;
constexpr int kMaxGroups = 512;          // groups of a slab
constexpr int kMaxSlab = kBlock * 8;     // channels of a slab
constexpr int kBatch = 4;                // pixels that a thread takes at a time
constexpr int kHeld = 8;                 // pixels that it holds in the one-launch kernels,
constexpr int kHeldBatch = 7;            // or 2 or 6 (fp32: 3) batches of this
template <class T> constexpr int kHeldMost = sizeof(T) == 2 ? 42 : 21;      // 168 of a thread's 256 registers: one block a CU
// Blocks of r pixels a thread, r > kHeld, that share a CU.
template <class T>
__device__ __host__ constexpr int held_blocks(int r) { return sizeof(T) == 2 && r <= 2 * kHeldBatch ? 2 : 1; }

// a / b of whole numbers below 2^20 by b's reciprocal in fp32: (a + 1/2) / b is at least 1 / (2 b) from a whole number,
// relative to itself 2^-21, and the product's two roundings are 2^-23.
__device__ __forceinline__ int divided(int a, float inverse) { return (int)(((float)a + 0.5f) * inverse); }

// The block's place: its sample, channels c0 .. c0 + n - 1 and pixels p0 .. p1 - 1; the thread's piece of 8 channels
// (at c), the slab's group of the first of them and its place in the group, and the first of the thread's pixels.
struct Place {
    int b, c0, n, pieces, lanes, c, lane, p0, p1, groups, first, inside;
    bool own;                            // whether the thread has a piece
    __device__ __forceinline__ Place(const GroupDev& d, int chunk, int size, int slab, int sample) : b(sample) {
        c0 = slab * d.slab;
        const bool last = d.channels - c0 < d.slab;
        n = last ? d.channels - c0 : d.slab;
        groups = divided(n, d.per_width);
        pieces = (n + 7) / 8;
        const float per_pieces = 1.0f / (float)pieces;
        lanes = divided(kBlock, per_pieces);      // threads of a piece
        lane = divided((int)threadIdx.x, per_pieces);
        c = ((int)threadIdx.x - lane * pieces) * 8;
        first = divided(c, d.per_width);
        inside = c - first * d.width;
        p0 = chunk * size;
        p1 = d.pixels - p0 < size ? d.pixels : p0 + size;
        own = lane < lanes;
    }
    // f(i, group within the slab) of the thread's 8 channels; those past the slab count as the last group's.
    template <class F>
    __device__ __forceinline__ void each_group(const GroupDev& d, F f) const {
        int g = first, r = inside;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            f(i, g < groups ? g : groups - 1);
            if (++r == d.width) {
                r = 0;
                ++g;
            }
        }
    }
};

template <class T>
__device__ __forceinline__ T* row_at(const void* x, const int64_t (&s)[2], const Place& q, int p) {
    return const_cast<T*>(static_cast<const T*>(x)) + q.b * s[0] + p * s[1] + q.c0;
}

// Index of the slab's first group among all samples'.
__device__ __forceinline__ int64_t group_at(const GroupDev& d, const Place& q) { return (int64_t)q.b * d.groups + divided(q.c0, d.per_width); }

// The thread's piece of an existing pixel: fetch starts the load (slabs of whole pieces, of 8 or more channels, or
// smaller ones), mend puts a piece that holds the slab's end into place.
template <class T, int WIDTH>
__device__ __forceinline__ Pack8<T> fetch(const T* row, const Place& q) {
    if constexpr (WIDTH == kWhole) return *reinterpret_cast<const Pack8<T>*>(row + q.c);
    if constexpr (WIDTH == kRagged) return load8_raw(row, q.c, q.n);
    return load8(row, q.c, q.n);
}
template <class T, int WIDTH>
__device__ __forceinline__ Pack8<T> mend(const Pack8<T>& r, const Place& q) {
    if constexpr (WIDTH == kRagged) return fix8(r, q.c, q.n);
    return r;
}

// Stores a piece at channel c of a row.
template <class T, int WIDTH>
__device__ __forceinline__ void put(T* row, const Pack8<T>& v, const Place& q) {
    if constexpr (WIDTH == kWhole) *reinterpret_cast<Pack8<T>*>(row + q.c) = v;
    else store8(row + q.c, v, q.n - q.c);
}

// R pixels of the thread from `p` on, `lanes` apart; beyond the chunk's last one, which stands in for them, nothing is
// counted by the callers.
template <class T, int WIDTH, int R>
__device__ __forceinline__ void fetch_pixels(const void* x, const int64_t (&s)[2], const Place& q, int p, Pack8<T> (&out)[R]) {
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int at = p + k * q.lanes;
        out[k] = fetch<T, WIDTH>(row_at<T>(x, s, q, at < q.p1 ? at : q.p1 - 1), q);
    }
}

// Eight of a parameter's values as they lie in memory, so that their load can be in flight, and as numbers.
struct Raw {
    uint4 lo, hi;
};
template <int WIDTH>
__device__ __forceinline__ Raw load_parameters(const GroupDev& d, const void* p, const Place& q) {
    Raw r{};
    if (!p) return r;
    if (d.param_dtype == PA_F32) return __builtin_bit_cast(Raw, fetch<float, WIDTH>(static_cast<const float*>(p) + q.c0, q));
    r.lo = __builtin_bit_cast(uint4, fetch<__bf16, WIDTH>(static_cast<const __bf16*>(p) + q.c0, q));
    return r;
}
template <int WIDTH>
__device__ __forceinline__ void numbers(const GroupDev& d, const void* p, const Raw& r, const Place& q, float otherwise, float (&v)[8]) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = otherwise;
    } else if (d.param_dtype == PA_F32) {
        const Pack8<float> t = mend<float, WIDTH>(__builtin_bit_cast(Pack8<float>, r), q);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = t.v[i];
    } else {
        const Pack8<__bf16> t = mend<__bf16, WIDTH>(__builtin_bit_cast(Pack8<__bf16>, r.lo), q);
        const Pack8<_Float16> h = __builtin_bit_cast(Pack8<_Float16>, t);
        const bool bf = d.param_dtype == PA_BF16;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = bf ? (float)t.v[i] : (float)h.v[i];
    }
}

// The activation is the same for all: one branch for 8 values. EXACT: of results in fp32.
template <bool EXACT>
__device__ __forceinline__ void activate8(int act, float (&v)[8]) {
    if (act == PA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate<PA_ACT_SILU>(v[i]);
    } else if (act == PA_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate<PA_ACT_GELU, EXACT>(v[i]);
    }
}
template <bool EXACT>
__device__ __forceinline__ void slope8(int act, float (&v)[8]) {       // its derivative
    if (act == PA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate_grad<PA_ACT_SILU>(v[i]).y;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = activate_grad<PA_ACT_GELU, EXACT>(v[i]).y;
    }
}

// Sums over the threads and channels of each group of the slab, a wave a group, in a fixed order. `lds`: kBlock * 8
// floats, free before and after.
__device__ __forceinline__ void group_sums(const GroupDev& d, const Place& q, const float (&v)[8], float* lds, float* group) {
    const int width = q.pieces * 8, L = d.width;
    if (q.own) {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[q.lane * width + q.c + i] = v[i];
    }
    __syncthreads();
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int total = q.lanes * L;               // at most 4096: value k is channel k % L of lane k / L
    for (int g = w; g < q.groups; g += kWaves) {
        float s = 0.0f;
        for (int k0 = lane; k0 < total; k0 += 256) {
            float t[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + 64 * j < total ? k0 + 64 * j : k0;
                t[j] = lds[k + divided(k, d.per_width) * (width - L) + g * L];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) s += k0 + 64 * j < total ? t[j] : 0.0f;
        }
        s = wave_sum_f32(s);
        if (lane == 0) group[g] = s;
    }
    __syncthreads();
}

// Sum over 16 lanes, in each of them.
__device__ __forceinline__ float sum16(float v) {
    v += dpp_f32<0xB1>(v);
    v += dpp_f32<0x4E>(v);
    v += dpp_f32<0x141>(v);
    v += dpp_f32<0x140>(v);
    return v;
}

// A thread's pixels so far: their number, and each channel's mean and sum of squared differences.
struct Running {
    float n = 0.0f, mean[8] = {}, m2[8] = {};
    template <class T, int R>
    __device__ __forceinline__ void add(const Pack8<T> (&x)[R], int count) {       // the first `count` of them
        if (count <= 0) return;
        const float k = (float)(count < R ? count : R), total = n + k, part = k / total, both = n * part;
        const float inv = 1.0f / k;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // Relative to the first of them: equal values have exactly their mean.
            const float x0 = (float)x[0].v[i];
            float s = 0.0f;
#pragma unroll
            for (int r = 1; r < R; ++r) s += r < count ? (float)x[r].v[i] - x0 : 0.0f;
            const float m = fmaf(s, inv, x0), e = m - mean[i];
            float q = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float t = (float)x[r].v[i] - m;
                q += r < count ? t * t : 0.0f;
            }
            mean[i] = fmaf(e, part, mean[i]);
            m2[i] += fmaf(e * both, e, q);          // (e * e alone overflows from 2^64 on, also where there is nothing to join it to)
        }
        n = total;
    }
};

// Pixels of the thread from p to p1.
__device__ __forceinline__ int pixels_left(const Place& q, int p) {
    return q.own && p < q.p1 ? (q.p1 - p + q.lanes - 1) / q.lanes : 0;
}

// Of the slab's groups: a value of each, relative to which means are joined, the sum of differences from it, and the sum of
// squared differences from the mean.
struct Groups {
    float first[kMaxGroups], sum[kMaxGroups], m2[kMaxGroups];
};

// The groups' statistics over the chunk from every thread's; the mean is first + sum / (values).
__device__ __forceinline__ void statistics(const GroupDev& d, const Place& q, const Running& r, float* lds, Groups& out) {
    float v[8];
    if (q.own && q.lane == 0) {
        int at = q.inside;
        q.each_group(d, [&](int i, int g) {
            if (at == 0 && q.c + i < q.n) out.first[g] = r.mean[i];
            at = at + 1 == d.width ? 0 : at + 1;
        });
    }
    __syncthreads();
    q.each_group(d, [&](int i, int g) { v[i] = r.n * (r.mean[i] - out.first[g]); });
    group_sums(d, q, v, lds, out.sum);
    const float inv = 1.0f / ((float)(q.p1 - q.p0) * (float)d.width);
    q.each_group(d, [&](int i, int g) {
        const float e = r.mean[i] - fmaf(out.sum[g], inv, out.first[g]);
        v[i] = fmaf(e * r.n, e, r.m2[i]);           // likewise of a thread without pixels
    });
    group_sums(d, q, v, lds, out.m2);
}

// act((x - mean) rstd w + b) of one piece (a = rstd w).
template <class T>
__device__ __forceinline__ Pack8<T> normalized(const Pack8<T>& x, const float (&mean)[8], const float (&a)[8], const float (&b)[8], int act) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = fmaf((float)x.v[i] - mean[i], a[i], b[i]);
    activate8<sizeof(T) == 4>(act, v);
    Pack8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (T)v[i];
    return o;
}

// The same bits, as far as the compiler knows others: a pixel's 16-bit values stay so between two uses instead of as 32-bit
// numbers, in twice the registers.
template <class T>
__device__ __forceinline__ void keep_packed(Pack8<T>& p) {
    if constexpr (sizeof(T) == 2) {
        i32x4 v = __builtin_bit_cast(i32x4, p);
        asm volatile("" : "+v"(v));
        p = __builtin_bit_cast(Pack8<T>, v);
    }
}

// A slab's pixels in one block's registers, up to R a thread: statistics and result in one launch, x read once. The slabs of
// a sample are neighbours on an XCD, so that the lines that two of them share are fetched once. Bound by its phases, one
// after the other where a CU has one block: the loads, then vector instructions (20 a value, silu's included: 27 us) that only
// the stores overlap. 32x4096x320 in bf16: 45 us, 3.7 TB/s; in two launches 23 + 29.
template <class T, int WIDTH, int R>
__global__ __launch_bounds__(kBlock, (R <= kHeld ? 4 : held_blocks<T>(R) * 2)) void k_group_whole(GroupDev d) {
    __shared__ float lds[kBlock * 8], group[2][kMaxGroups];
    __shared__ Groups s;
    constexpr int N = R % kHeldBatch == 0 ? kHeldBatch : R;          // in batches, of which those that no thread has are left out
    const int id = xcd_order(blockIdx.x, gridDim.x), sample = id / d.slabs;
    const Place q(d, 0, d.pixels, id - sample * d.slabs, sample);
    const int every = divided(d.pixels, 1.0f / (float)q.lanes), any = every + (every * q.lanes < d.pixels);      // a thread's pixels: at least, at most
    Pack8<T> x[R / N][N];
#pragma unroll
    for (int k = 0; k < R / N; ++k) {
        if (k * N < any) fetch_pixels<T, WIDTH>(d.x, d.xs, q, q.lane + k * N * q.lanes, x[k]);
        __builtin_amdgcn_sched_barrier(0);               // (addresses and numbers of one batch in registers at a time, here and below)
    }
    float a[8], b[8], mean[8];
    const Raw rw = load_parameters<WIDTH>(d, d.w, q), rb = load_parameters<WIDTH>(d, d.b, q);
    const int count = pixels_left(q, q.lane);
    Running r;
#pragma unroll
    for (int k = 0; k < R / N; ++k) {
        if (k * N >= any) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) x[k][i] = mend<T, WIDTH>(x[k][i], q);
        if ((k + 1) * N <= every) r.add(x[k], N);
        else r.add(x[k], count - k * N);
#pragma unroll
        for (int i = 0; i < N; ++i) keep_packed(x[k][i]);
        __builtin_amdgcn_sched_barrier(0);
    }
    if (!q.own) r = Running();
    statistics(d, q, r, lds, s);
    const float n = (float)d.pixels * (float)d.width;
    for (int g = threadIdx.x; g < q.groups; g += kBlock) {
        const float m = fmaf(s.sum[g], 1.0f / n, s.first[g]), rstd = 1.0f / sqrtf(s.m2[g] / n + d.eps);
        const int64_t at = group_at(d, q) + g;
        if (d.mean) d.mean[at] = m;
        if (d.rstd) d.rstd[at] = rstd;
        group[0][g] = m;
        group[1][g] = rstd;
    }
    __syncthreads();
    numbers<WIDTH>(d, d.w, rw, q, 1.0f, a);
    numbers<WIDTH>(d, d.b, rb, q, 0.0f, b);
    q.each_group(d, [&](int i, int g) {
        mean[i] = group[0][g];
        a[i] *= group[1][g];
    });
    if (!q.own) return;
    T* row = row_at<T>(d.y, d.ys, q, q.lane);
    const int64_t step = q.lanes * d.ys[1];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        if (k < every || k < count) put<T, WIDTH>(row, normalized(x[k / N][k % N], mean, a, b, d.act), q);
        row += step;
        if (k % 2) __builtin_amdgcn_sched_barrier(0);
    }
}

// Statistics of a chunk. The next batch is on its way while one is worked on. Bound by the loads' latency and rate: 8x4096x640
// in bf16 16 to 17 us, 2.5 TB/s.
template <class T, int WIDTH>
__global__ __launch_bounds__(kBlock, 4) void k_group_stats(GroupDev d) {
    __shared__ float lds[kBlock * 8];
    __shared__ Groups s;
    const Place q(d, blockIdx.x, d.chunk, blockIdx.y, d.sample0 + blockIdx.z);
    Running r;
    Pack8<T> x[kBatch], next[kBatch];
    int p = q.p0 + q.lane, left = pixels_left(q, p);
    fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, next);
    while (left > 0) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) x[k] = mend<T, WIDTH>(next[k], q);
        p += kBatch * q.lanes;
        if (left > kBatch) fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, next);
        r.add(x, left);
        left -= kBatch;
    }
    statistics(d, q, r, lds, s);
    const float n = (float)(q.p1 - q.p0) * (float)d.width;
    for (int g = threadIdx.x; g < q.groups; g += kBlock) {
        float* out = d.part + ((group_at(d, q) + g) * d.chunks + blockIdx.x) * 2;
        out[0] = fmaf(s.sum[g], 1.0f / n, s.first[g]);
        out[1] = s.m2[g];
    }
}

// Joins the chunks' statistics (every block for its own groups, 16 lanes a group) and writes the results of d.spread
// pixels. 8x4096x640 in bf16 17 us for 84 MB, 4.9 TB/s: the copy rate.
template <class T, int WIDTH>
__global__ __launch_bounds__(kBlock, 4) void k_group_apply(GroupDev d) {
    __shared__ float group[2][kMaxGroups];
    const Place q(d, blockIdx.x, d.spread, blockIdx.y, d.sample0 + blockIdx.z);
    Pack8<T> next[kBatch];
    int p = q.p0 + q.lane, left = pixels_left(q, p);
    fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, next);
    float a[8], b[8], mean[8];
    const Raw rw = load_parameters<WIDTH>(d, d.w, q), rb = load_parameters<WIDTH>(d, d.b, q);
    const int sub = threadIdx.x & 15;
    const float total = (float)d.pixels * (float)d.width, each = (float)d.chunk * (float)d.width;
    const float rest = (float)(d.pixels - (d.chunks - 1) * d.chunk) * (float)d.width;
    for (int g0 = 0; g0 < q.groups; g0 += kBlock / 16) {
        const int g = g0 + ((int)threadIdx.x >> 4);
        const int64_t at = group_at(d, q) + (g < q.groups ? g : 0);
        const float2* in = reinterpret_cast<const float2*>(d.part) + at * d.chunks;
        const float first = in[0].x;
        float m = 0.0f, m2 = 0.0f;
#pragma unroll 4
        for (int k = sub; k < d.chunks; k += 16) m += (in[k].x - first) * (k + 1 < d.chunks ? each : rest);
        m = first + sum16(m) / total;
#pragma unroll 4
        for (int k = sub; k < d.chunks; k += 16) {
            const float2 v = in[k];
            const float e = v.x - m;
            m2 += v.y + e * e * (k + 1 < d.chunks ? each : rest);
        }
        m2 = sum16(m2);
        if (sub == 0 && g < q.groups) {
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
    numbers<WIDTH>(d, d.w, rw, q, 1.0f, a);
    numbers<WIDTH>(d, d.b, rb, q, 0.0f, b);
    q.each_group(d, [&](int i, int g) {
        mean[i] = group[0][g];
        a[i] *= group[1][g];
    });
    while (left > 0) {
        Pack8<T> x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) x[k] = mend<T, WIDTH>(next[k], q);
        if (left > kBatch) fetch_pixels<T, WIDTH>(d.x, d.xs, q, p + kBatch * q.lanes, next);
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (k < left) put<T, WIDTH>(row_at<T>(d.y, d.ys, q, p + k * q.lanes), normalized(x[k], mean, a, b, d.act), q);
        p += kBatch * q.lanes;
        left -= kBatch;
    }
}

// ------------------------------------------------------------------ backward
struct Channels {                    // of the thread's 8: group mean, rstd, weight, bias
    float mean[8], rstd[8], w[8], b[8];
};

template <int WIDTH>
__device__ __forceinline__ Channels channels(const GroupDev& d, const Place& q) {
    Channels k;
    const Raw rw = load_parameters<WIDTH>(d, d.w, q), rb = load_parameters<WIDTH>(d, d.b, q);
    const int64_t at = group_at(d, q);
    q.each_group(d, [&](int i, int g) {
        k.mean[i] = d.mean[at + g];
        k.rstd[i] = d.rstd[at + g];
    });
    numbers<WIDTH>(d, d.w, rw, q, 1.0f, k.w);
    numbers<WIDTH>(d, d.b, rb, q, 0.0f, k.b);
    return k;
}

// xh and dz of one piece.
template <class T>
__device__ __forceinline__ void through(const Channels& k, const Pack8<T>& x, const Pack8<T>& dy, int act, float (&xh)[8], float (&dz)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        xh[i] = ((float)x.v[i] - k.mean[i]) * k.rstd[i];
        dz[i] = (float)dy.v[i];
    }
    if (act == PA_ACT_NONE) return;
    float s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = fmaf(xh[i], k.w[i], k.b[i]);
    slope8<sizeof(T) == 4>(act, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) dz[i] *= s[i];
}

// Sums over the block's threads for each channel, in a fixed order: of u into out, of v `channels` after it.
// `lds`: kBlock * 16 floats.
__device__ __forceinline__ void channel_sums(const Place& q, const float (&u)[8], const float (&v)[8], float* lds, float* out, int channels) {
    const int width = q.pieces * 8;
    float* second = lds + kBlock * 8;
    if (q.own) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lds[q.lane * width + q.c + i] = u[i];
            second[q.lane * width + q.c + i] = v[i];
        }
    }
    __syncthreads();
    // Where there are twice as many threads as channels, or more, several take a channel's lanes in turn.
    const float per = 1.0f / (float)width;
    const int turns = width < kBlock ? divided(kBlock, per) : 1;
    if (turns > 1) {
        const int t = divided((int)threadIdx.x, per), c = (int)threadIdx.x - t * width;
        float a = 0.0f, b = 0.0f;
        if (t < turns)
            for (int l = t; l < q.lanes; l += turns) {
                a += lds[l * width + c];
                b += second[l * width + c];
            }
        __syncthreads();
        if (t < turns) {
            lds[t * width + c] = a;
            second[t * width + c] = b;
        }
        __syncthreads();
    }
    const int rows = turns > 1 ? turns : q.lanes;
    for (int c = threadIdx.x; c < q.n; c += kBlock) {
        float a = 0.0f, b = 0.0f;
        for (int l = 0; l < rows; ++l) {
            a += lds[l * width + c];
            b += second[l * width + c];
        }
        out[c] = a;
        out[channels + c] = b;
    }
}

// Sums over a chunk's pixels of dz xh and dz for each channel. 8x4096x640 in bf16 20 us, 84 MB at 4.2 TB/s.
template <class T, int WIDTH>
__global__ __launch_bounds__(kBlock, 4) void k_group_sums(GroupDev d) {
    __shared__ float lds[kBlock * 16];
    const Place q(d, blockIdx.x, d.chunk, blockIdx.y, d.sample0 + blockIdx.z);
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    Pack8<T> nx[R], ny[R];
    int p = q.p0 + q.lane, left = pixels_left(q, p);
    fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, nx);
    fetch_pixels<T, WIDTH>(d.dy, d.ys, q, p, ny);
    const Channels ch = channels<WIDTH>(d, q);
    float sw[8] = {}, sb[8] = {};
    while (left > 0) {
        Pack8<T> x[R], y[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            x[k] = mend<T, WIDTH>(nx[k], q);
            y[k] = mend<T, WIDTH>(ny[k], q);
        }
        p += R * q.lanes;
        if (left > R) {
            fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, nx);
            fetch_pixels<T, WIDTH>(d.dy, d.ys, q, p, ny);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k >= left) break;
            float xh[8], dz[8];
            through(ch, x[k], y[k], d.act, xh, dz);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sw[i] = fmaf(dz[i], xh[i], sw[i]);
                sb[i] += dz[i];
            }
        }
        left -= R;
    }
    channel_sums(q, sw, sb, lds, d.part + ((int64_t)q.b * d.chunks + blockIdx.x) * 2 * d.channels + q.c0, d.channels);
}

// A sample's group: the channels' sums over the chunks, and from them the means over the group of g and g xh.
__global__ __launch_bounds__(256) void k_group_join(GroupDev d) {
    __shared__ float sum[2][256], red[2][4];
    const int g = blockIdx.x, b = d.sample0 + blockIdx.y, L = d.width;
    // Threads of a channel: the chunks in turn.
    const int turns = L < 256 ? 256 / L : 1, t = (int)threadIdx.x / L, span = L < 256 ? L : 256;
    float m[2] = {};
    for (int c0 = 0; c0 < L; c0 += span) {
        const int c = c0 + (L < 256 ? (int)threadIdx.x - t * L : (int)threadIdx.x), ch = g * L + c;
        float v[2] = {};
        const bool own = c < L && (L >= 256 || t < turns);
        if (own) {
#pragma unroll 8
            for (int k = L < 256 ? t : 0; k < d.chunks; k += turns) {
                const float* in = d.part + ((int64_t)b * d.chunks + k) * 2 * d.channels + ch;
                v[0] += in[0];
                v[1] += in[d.channels];
            }
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
            float w = 1.0f;
            if (d.w)
                w = d.param_dtype == PA_F32 ? static_cast<const float*>(d.w)[ch]
                    : d.param_dtype == PA_BF16 ? (float)static_cast<const __bf16*>(d.w)[ch] : (float)static_cast<const _Float16*>(d.w)[ch];
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

// dweight and dbias from the samples' sums, in order; `block` of 512 of the 2 x channels values.
__device__ __forceinline__ void join_samples(const GroupDev& d, int block) {
    const int64_t i = (int64_t)block * kBlock + threadIdx.x;
    if (i >= 2 * (int64_t)d.channels) return;
    const bool second = i >= d.channels;
    void* out = second ? d.db : d.dw;
    if (!out) return;
    const int c = (int)(second ? i - d.channels : i);
    float s = 0.0f;
#pragma unroll 8
    for (int b = 0; b < d.batch; ++b) s += d.sums[(int64_t)b * 2 * d.channels + i];
    if (d.param_dtype == PA_F32) static_cast<float*>(out)[c] = s;
    else if (d.param_dtype == PA_BF16) static_cast<__bf16*>(out)[c] = (__bf16)s;
    else static_cast<_Float16*>(out)[c] = (_Float16)s;
}

__global__ __launch_bounds__(kBlock) void k_group_params(GroupDev d) { join_samples(d, blockIdx.x); }

// dx of one piece from the means over its channels' groups.
template <class T>
__device__ __forceinline__ Pack8<T> gradient(const Channels& ch, const Pack8<T>& x, const Pack8<T>& dy, const float (&m1)[8], const float (&m2)[8], int act) {
    float xh[8], dz[8];
    through(ch, x, dy, act, xh, dz);
    Pack8<T> o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o.v[i] = (T)(ch.rstd[i] * (dz[i] * ch.w[i] - m1[i] - xh[i] * m2[i]));
    return o;
}

// dx of a chunk (`spreads` of them a sample and slab); the launch's last blocks join the samples' sums (there are `blocks` in
// front of them). Bound by memory:
// 8x4096x640 in bf16 27 to 28 us, 126 MB at 4.5 TB/s.
template <class T, int WIDTH>
__global__ __launch_bounds__(kBlock, 4) void k_group_dx(GroupDev d, unsigned blocks, int spreads) {
    if (blockIdx.x >= blocks) {
        join_samples(d, (int)(blockIdx.x - blocks));
        return;
    }
    const int chunk = (int)(blockIdx.x % spreads), rest = (int)(blockIdx.x / spreads);
    const Place q(d, chunk, d.spread, rest % d.slabs, d.sample0 + rest / d.slabs);
    constexpr int R = sizeof(T) == 2 ? 2 : 1;
    Pack8<T> nx[R], ny[R];
    int p = q.p0 + q.lane, left = pixels_left(q, p);
    fetch_pixels<T, WIDTH>(d.x, d.xs, q, p, nx);
    fetch_pixels<T, WIDTH>(d.dy, d.ys, q, p, ny);
    const Channels ch = channels<WIDTH>(d, q);
    float m1[8], m2[8];
    const float2* means = reinterpret_cast<const float2*>(d.means) + group_at(d, q);
    q.each_group(d, [&](int i, int g) {
        const float2 v = means[g];
        m1[i] = v.x;
        m2[i] = v.y;
    });
    while (left > 0) {
        Pack8<T> x[R], y[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            x[k] = mend<T, WIDTH>(nx[k], q);
            y[k] = mend<T, WIDTH>(ny[k], q);
        }
        if (left > R) {
            fetch_pixels<T, WIDTH>(d.x, d.xs, q, p + R * q.lanes, nx);
            fetch_pixels<T, WIDTH>(d.dy, d.ys, q, p + R * q.lanes, ny);
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k < left) put<T, WIDTH>(row_at<T>(d.dx, d.dxs, q, p + k * q.lanes), gradient(ch, x[k], y[k], m1, m2, d.act), q);
            __builtin_amdgcn_sched_barrier(0);           // one pixel's numbers in registers at a time
        }
        p += R * q.lanes;
        left -= R;
    }
}

// A slab's pixels of x and dy in one block's registers, R a thread: sums and dx in one launch.
template <class T, int WIDTH, int R>
__global__ __launch_bounds__(kBlock) void k_group_bwd_whole(GroupDev d) {
    __shared__ float lds[kBlock * 16], group[2][kMaxGroups];
    const Place q(d, 0, d.pixels, blockIdx.x, blockIdx.y);
    Pack8<T> x[R], y[R];
    fetch_pixels<T, WIDTH>(d.x, d.xs, q, q.lane, x);
    fetch_pixels<T, WIDTH>(d.dy, d.ys, q, q.lane, y);
    const Channels ch = channels<WIDTH>(d, q);
    const int count = pixels_left(q, q.lane);
    float sw[8] = {}, sb[8] = {}, v[8];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        x[k] = mend<T, WIDTH>(x[k], q);
        y[k] = mend<T, WIDTH>(y[k], q);
        if (k < count) {
            float xh[8], dz[8];
            through(ch, x[k], y[k], d.act, xh, dz);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sw[i] = fmaf(dz[i], xh[i], sw[i]);
                sb[i] += dz[i];
            }
        }
    }
    if (d.dx) {
        const float inv = 1.0f / ((float)d.pixels * (float)d.width);
        float m1[8], m2[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sb[i] * ch.w[i];
        group_sums(d, q, v, lds, group[0]);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = sw[i] * ch.w[i];
        group_sums(d, q, v, lds, group[1]);
        q.each_group(d, [&](int i, int g) {
            m1[i] = group[0][g] * inv;
            m2[i] = group[1][g] * inv;
        });
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < count) put<T, WIDTH>(row_at<T>(d.dx, d.dxs, q, q.lane + k * q.lanes), gradient(ch, x[k], y[k], m1, m2, d.act), q);
    }
    if (d.dw || d.db) channel_sums(q, sw, sb, lds, d.sums + (int64_t)q.b * 2 * d.channels + q.c0, d.channels);
}

// ------------------------------------------------------------------ launches
int64_t parts_of(int64_t n, int64_t size) { return (n + size - 1) / size; }

// A launch of so many blocks lasts a millisecond and more: beyond (long batches of many narrow groups) it goes in ranges of the
// samples, so that no grid comes near 2^32 threads. launch(d, samples) for each range, which begins at d.sample0.
constexpr int64_t kMaxBlocks = 1 << 20;
template <class F>
hipError_t in_ranges(GroupDev d, int64_t blocks_a_sample, F launch) {
    const int64_t most = blocks_a_sample < kMaxBlocks ? kMaxBlocks / blocks_a_sample : 1;
    for (int64_t b = 0; b < d.batch; b += most) {
        d.sample0 = (int)b;
        launch(d, (unsigned)(d.batch - b < most ? d.batch - b : most));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <class F>
hipError_t dispatch(int dtype, const GroupDev& d, F f) {
    auto width = [&](auto t) {
        const int last = d.channels - (d.slabs - 1) * d.slab;
        if (d.slab % 8 == 0 && last % 8 == 0) return f(t, std::integral_constant<int, kWhole>{});
        if (d.slab >= 8 && last >= 8) return f(t, std::integral_constant<int, kRagged>{});
        return f(t, std::integral_constant<int, kTiny>{});
    };
    if (dtype == PA_F32) return width((float)0);
    return dtype == PA_BF16 ? width((__bf16)0) : width((_Float16)0);
}

// A thread's pixels of a slab of one block.
int64_t held(const GroupDev& d) { return parts_of(d.pixels, kBlock / ((d.slab + 7) / 8)); }

}  // namespace

// Slabs of whole groups and of whole pieces of 8 channels. The smallest such slab (with at least 32 channels, so that a
// pixel's piece of it is no smaller than a cache line's sector) if a block's registers hold its pixels in one launch; else as
// many groups as a block can take, in chunks of pixels.
//
// One launch or two, us of a bf16 call: 1024 pixels of 640 channels (11 a thread), 16 to 1280 slabs: 15 and 20 (16), 19 and 24
// (256), 28 and 33 (512), 54 and 54 (1024), 65 and 81 (1280). 4096 pixels of 320 channels (41 a thread, one block a CU): 43
// and 35 (128 slabs), 44 and 48 (160), 49 and 56 (256), 82 and 76 (288), 86 and 95 (352), 106 and 111 (512): a block a CU
// pays where two thirds of the CUs and more have one.
//
// The backward pass holds x and dy: up to 4 pixels of both, or up to 8 where half of the CUs and more have a block. us in one pass
// and in three launches, 320 channels in slabs of 40: 100 pixels (1 a thread) 8.6 and 12.7 (8 slabs), 9.5 and 13.7 (128), 14.9
// and 15.1 (320); 400 pixels (4 a thread) 12.4 and 12.9 (8), 15.1 and 14.0 (64), 16.8 and 18.9 (128), 19.0 and 20.9 (192); 800
// pixels (8 a thread) 16.8 and 13.4 (8), 21.4 and 19.1 (64), 24.3 and 23.4 (128), 27.4 and 31.6 (192); the last in fp32 16.9 and
// 15.0 (8), 21.2 and 23.4 (64), 24.2 and 27.8 (128), 28.8 and 39.7 (192).
void group_plan(GroupDev& d, int dtype, bool backward) {
    d.width = d.channels / d.groups;
    d.per_width = 1.0f / (float)d.width;
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
    const int64_t n = held(d), blocks = (int64_t)d.batch * d.slabs;
    bool whole = n <= kHeld;
    if (backward) {
        whole = n <= kHeld / 2 || (whole && blocks >= 128);
    } else if (!whole && d.slab % 8 == 0 && d.channels % 8 == 0 && n <= (dtype == PA_F32 ? kHeldMost<float> : kHeldMost<__bf16>)) {
        whole = n <= 2 * kHeldBatch || 3 * blocks >= 2 * 256 * parts_of(blocks, 256);
    }
    if (whole && blocks < (1 << 23)) {
        d.chunk = d.pixels > 0 ? d.pixels : 1;
        d.chunks = 1;
        d.whole = 1;
        return;
    }
    slab(d.groups);
    // 512 blocks, two for each CU, as its registers allow, but chunks of two pixels a thread at least (four where
    // they come in batches of four: 4x1024x640 statistics 10.6 and 8.2 us), and at most 256 of them a sample. us with 512,
    // 768, 1024 and 2048 blocks, 32x4096x320: statistics 23, 24, 25, 35, results 33, 33, 34,
    // 38; 8x4096x640: sums of the backward pass 21, 22, 22, dx 34, 39, 37, 41.
    const int lanes = kBlock / ((d.slab + 7) / 8);
    const int64_t per = (int64_t)d.batch * d.slabs, want = (512 + per - 1) / (per > 0 ? per : 1);
    int64_t chunk = (d.pixels + want - 1) / want;
    if (chunk < lanes * (backward ? 2 : 4)) chunk = lanes * (backward ? 2 : 4);
    if ((d.pixels + chunk - 1) / chunk > 256) chunk = (d.pixels + 255) / 256;
    d.chunk = (int)(chunk < 1 ? 1 : chunk);
    d.chunks = d.pixels > 0 ? (int)parts_of(d.pixels, d.chunk) : 1;
    int64_t spread = (d.pixels + want - 1) / want;
    if (spread < lanes * 2) spread = lanes * 2;
    d.spread = (int)spread;
    d.whole = 0;
}

hipError_t group_forward(const GroupDev& d, int dtype, hipStream_t st) {
    return dispatch(dtype, d, [&](auto t, auto wd) {
        typedef decltype(t) T;
        constexpr int WIDTH = decltype(wd)::value;
        if (d.whole) {
            const unsigned blocks = (unsigned)((int64_t)d.slabs * d.batch);
            const int64_t n = held(d);
            if (n <= 2) k_group_whole<T, WIDTH, 2><<<blocks, kBlock, 0, st>>>(d);
            else if (n <= kHeld) k_group_whole<T, WIDTH, kHeld><<<blocks, kBlock, 0, st>>>(d);
            else if constexpr (WIDTH == kWhole) {
                if (n <= 2 * kHeldBatch) k_group_whole<T, WIDTH, 2 * kHeldBatch><<<blocks, kBlock, 0, st>>>(d);
                else k_group_whole<T, WIDTH, kHeldMost<T>><<<blocks, kBlock, 0, st>>>(d);
            }
            return hipGetLastError();
        }
        const unsigned chunks = (unsigned)d.chunks, spreads = (unsigned)parts_of(d.pixels, d.spread), slabs = (unsigned)d.slabs;
        const hipError_t e = in_ranges(d, (int64_t)chunks * slabs, [&](const GroupDev& c, unsigned n) {
            k_group_stats<T, WIDTH><<<dim3(chunks, slabs, n), kBlock, 0, st>>>(c);
        });
        if (e != hipSuccess) return e;
        return in_ranges(d, (int64_t)spreads * slabs, [&](const GroupDev& c, unsigned n) {
            k_group_apply<T, WIDTH><<<dim3(spreads, slabs, n), kBlock, 0, st>>>(c);
        });
    });
}

hipError_t group_backward(const GroupDev& d, int dtype, hipStream_t st) {
    return dispatch(dtype, d, [&](auto t, auto wd) {
        typedef decltype(t) T;
        constexpr int WIDTH = decltype(wd)::value;
        const unsigned params = d.dw || d.db ? (unsigned)((2 * (int64_t)d.channels + kBlock - 1) / kBlock) : 0;
        const bool any = d.batch > 0 && d.pixels > 0;
        if (any && !d.whole) {
            const unsigned chunks = (unsigned)d.chunks, slabs = (unsigned)d.slabs, groups = (unsigned)d.groups;
            hipError_t e = in_ranges(d, (int64_t)chunks * slabs, [&](const GroupDev& c, unsigned n) {
                k_group_sums<T, WIDTH><<<dim3(chunks, slabs, n), kBlock, 0, st>>>(c);
            });
            if (e != hipSuccess) return e;
            e = in_ranges(d, groups, [&](const GroupDev& c, unsigned n) { k_group_join<<<dim3(groups, n), 256, 0, st>>>(c); });
            if (e != hipSuccess) return e;
            const unsigned spreads = (unsigned)parts_of(d.pixels, d.spread);
            if (d.dx) {
                unsigned with = params;              // the first range's launch joins the samples' sums too
                return in_ranges(d, (int64_t)spreads * slabs, [&](const GroupDev& c, unsigned n) {
                    const unsigned blocks = spreads * slabs * n;
                    k_group_dx<T, WIDTH><<<blocks + with, kBlock, 0, st>>>(c, blocks, (int)spreads);
                    with = 0;
                });
            }
        } else if (any) {
            const dim3 grid((unsigned)d.slabs, (unsigned)d.batch);
            if (held(d) <= 2) k_group_bwd_whole<T, WIDTH, 2><<<grid, kBlock, 0, st>>>(d);
            else k_group_bwd_whole<T, WIDTH, kHeld><<<grid, kBlock, 0, st>>>(d);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (params) {
            GroupDev c = d;
            if (!any) c.batch = 0;
            k_group_params<<<params, kBlock, 0, st>>>(c);
        }
        return hipGetLastError();
    });
}

}  // namespace pa
