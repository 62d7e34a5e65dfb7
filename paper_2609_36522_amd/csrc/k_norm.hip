// Layer norm, forward and backward, for gfx950.
//
// Forward, y = (x - mean) rstd w + b: a row lives in the registers of one wave or, from 8 columns to
// 8192, of one block of four waves, so x is read once and the mean and the sum of squared differences
// from it are two passes over registers (no cancellation between a sum of squares and a squared sum).
// Rows too long for that are read three times by one block, from L2 after the first.
//
// Backward: dx needs two sums over the row (g = dy w; g and g xh), dweight and dbias one sum over
// all rows for each column. A block walks over rows and keeps its columns' two running sums in
// registers, so dy and x are read once; the blocks' sums go to `part` and a second kernel adds
// them in a fixed order. Both passes are bound by memory traffic: at 32768x1024 in 16 bits 28 to 33 us
// forward (4.1 to 4.8 TB/s), 39 us backward (5.1 TB/s, part of x and dy still in the last-level
// cache) and 4.6 us for the sums' join. Rows at odd addresses take 4-byte or 2-byte pieces of the same
// lines: 5003x1333 in 32 bits 15 us forward, 20.7 backward.
#include "pa_ops_device.h"

namespace pa {

namespace {

constexpr int kThreads = 256;
constexpr int64_t kLaunchRows = 1 << 23;

// Sum over the WPR waves that share a row. `lds` holds 4 floats per call; the caller alternates
// two of them so that one barrier per sum is enough.
template <int WPR>
__device__ __forceinline__ float row_sum(float v, float* lds) {
    v = wave_sum_f32(v);
    if constexpr (WPR == 1) return v;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[w] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// A thread's chunk of 8 columns from `col`, once loaded. Only the chunks at the row's end (the same for all
// threads) need fixing.
template <class T>
__device__ __forceinline__ Pack8<T> ready(const Pack8<T>& r, int col, int N, bool last) {
    return last ? fix8(r, col, N) : r;
}

// CH chunks of 8 columns per thread, WPR (1 or 4) waves per row.
template <class T, class W, int WPR, int CH>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(NormDev d) {
    constexpr int TPR = 64 * WPR, RPB = 4 / WPR;
    __shared__ float red[2][4];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= d.rows) return;               // whole waves (WPR = 1) or none (one row per block)
    const int N = d.cols;
    const T* x = static_cast<const T*>(d.x) + row * d.x_stride;
    T* y = static_cast<T*>(d.y) + row * d.y_stride;
    const W* w = static_cast<const W*>(d.w);
    const W* b = static_cast<const W*>(d.b);
    Pack8<T> raw[CH];
    Pack8<W> pw[CH], pb[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) raw[c] = load8_raw(x, (c * TPR + t) * 8, N);
    if (w) {
#pragma unroll
        for (int c = 0; c < CH; ++c) pw[c] = load8_raw(w, (c * TPR + t) * 8, N);
    }
    if (b) {
#pragma unroll
        for (int c = 0; c < CH; ++c) pb[c] = load8_raw(b, (c * TPR + t) * 8, N);
    }
    float v[CH][8];
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * 8;
        const Pack8<T> p = ready(raw[c], col, N, (c + 1) * TPR * 8 > N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[c][i] = (float)p.v[i];
            s += v[c][i];
        }
    }
    const float n_f = (float)N;
    const float mean = row_sum<WPR>(s, red[0]) / n_f;
    float q = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = v[c][i] - mean;
            q += col + i < N ? e * e : 0.0f;
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<WPR>(q, red[1]) / n_f + d.eps);
    if (t == 0) {
        if (d.mean) d.mean[row] = mean;
        if (d.rstd) d.rstd[row] = rstd;
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int col = (c * TPR + t) * 8;
        if (w) pw[c] = ready(pw[c], col, N, (c + 1) * TPR * 8 > N);
        if (b) pb[c] = ready(pb[c], col, N, (c + 1) * TPR * 8 > N);
        Pack8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float r = (v[c][i] - mean) * rstd;
            if (w) r *= (float)pw[c].v[i];
            if (b) r += (float)pb[c].v[i];
            o.v[i] = (T)r;
        }
        store8(y + col, o, N - col);
    }
}

// Rows of any length: three passes over the row by one block.
template <class T, class W>
__global__ __launch_bounds__(kThreads) void k_norm_fwd_long(NormDev d) {
    __shared__ float red[2][4];
    const int64_t row = blockIdx.x;
    const int N = d.cols;
    const T* x = static_cast<const T*>(d.x) + row * d.x_stride;
    T* y = static_cast<T*>(d.y) + row * d.y_stride;
    const W* w = static_cast<const W*>(d.w);
    const W* b = static_cast<const W*>(d.b);
    const float n_f = (float)N;
    float s = 0.0f;
    for (int col = threadIdx.x * 8; col < N; col += kThreads * 8) {
        const Pack8<T> p = load8(x, col, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += (float)p.v[i];
    }
    const float mean = row_sum<4>(s, red[0]) / n_f;
    float q = 0.0f;
    for (int col = threadIdx.x * 8; col < N; col += kThreads * 8) {
        const Pack8<T> p = load8(x, col, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float e = (float)p.v[i] - mean;
            q += col + i < N ? e * e : 0.0f;
        }
    }
    const float rstd = 1.0f / sqrtf(row_sum<4>(q, red[1]) / n_f + d.eps);
    if (threadIdx.x == 0) {
        if (d.mean) d.mean[row] = mean;
        if (d.rstd) d.rstd[row] = rstd;
    }
    for (int col = threadIdx.x * 8; col < N; col += kThreads * 8) {
        const int n = N - col;
        const Pack8<T> p = load8(x, col, N);
        Pack8<W> pw, pb;
        if (w) pw = load8(w, col, N);
        if (b) pb = load8(b, col, N);
        Pack8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float r = ((float)p.v[i] - mean) * rstd;
            if (w) r *= (float)pw.v[i];
            if (b) r += (float)pb.v[i];
            o.v[i] = (T)r;
        }
        store8(y + col, o, n);
    }
}

// Backward, dx = rstd (g - mean(g) - xh mean(g xh)), for rows that fit the registers of
// WPR waves: dx of the block's rows (every gridDim.x-th group), and the block's sums of dy xh and dy into part[blockIdx.x].
template <class T, class W, int WPR, int CH>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(NormDev d) {
    constexpr int TPR = 64 * WPR, RPB = 4 / WPR;
    __shared__ float red[2][2][4];
    // Sums of the block's four waves (WPR = 1), 64 columns of 8 at a time.
    __shared__ float fold[WPR == 1 ? 4 * 512 : 1];
    const int t = threadIdx.x % TPR, g = threadIdx.x / TPR;
    const int N = d.cols;
    const W* w = static_cast<const W*>(d.w);
    float aw[CH][8] = {}, ab[CH][8] = {};
    const float n_f = (float)N;
    Pack8<W> pw[CH];
    if (w) {
#pragma unroll
        for (int c = 0; c < CH; ++c) pw[c] = load8_raw(w, (c * TPR + t) * 8, N);
#pragma unroll
        for (int c = 0; c < CH; ++c) pw[c] = ready(pw[c], (c * TPR + t) * 8, N, (c + 1) * TPR * 8 > N);
    }
    // The next row is on its way while a row is worked on.
    Pack8<T> nx[CH], nd[CH];
    float n_mean = 0.0f, n_rstd = 0.0f;
    auto load = [&](int64_t row) {
        const T* x = static_cast<const T*>(d.x) + row * d.x_stride;
        const T* dy = static_cast<const T*>(d.dy) + row * d.y_stride;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            nx[c] = load8_raw(x, (c * TPR + t) * 8, N);
            nd[c] = load8_raw(dy, (c * TPR + t) * 8, N);
        }
        n_mean = d.mean[row];
        n_rstd = d.rstd[row];
    };
    const int64_t step = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + g;
    if (row < d.rows) load(row);
    for (int turn = 0; row < d.rows; row += step, turn ^= 1) {
        const float mean = n_mean, rstd = n_rstd;
        Pack8<T> px[CH], pd[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            px[c] = ready(nx[c], (c * TPR + t) * 8, N, (c + 1) * TPR * 8 > N);
            pd[c] = ready(nd[c], (c * TPR + t) * 8, N, (c + 1) * TPR * 8 > N);
        }
        load(row + step < d.rows ? row + step : row);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float dyi = (float)pd[c].v[i];          // 0 past the row
                const float xh = ((float)px[c].v[i] - mean) * rstd;
                const float gi = w ? dyi * (float)pw[c].v[i] : dyi;
                s1 += gi;
                s2 += gi * xh;
                aw[c][i] += dyi * xh;
                ab[c][i] += dyi;
            }
        }
        if (!d.dx) continue;
        s1 = row_sum<WPR>(s1, red[turn][0]) / n_f;
        s2 = row_sum<WPR>(s2, red[turn][1]) / n_f;
        T* dx = static_cast<T*>(d.dx) + row * d.dx_stride;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * 8;
            Pack8<T> o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float dyi = (float)pd[c].v[i];
                const float xh = ((float)px[c].v[i] - mean) * rstd;
                const float gi = w ? dyi * (float)pw[c].v[i] : dyi;
                o.v[i] = (T)(rstd * (gi - s1 - xh * s2));
            }
            store8(dx + col, o, N - col);
        }
    }
    if (!d.part) return;
    float* out = d.part + (int64_t)blockIdx.x * 2 * N;
    if constexpr (WPR == 1) {
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) fold[g * 512 + i * 64 + t] = which ? ab[c][i] : aw[c][i];
                __syncthreads();
                for (int k = threadIdx.x; k < 512; k += kThreads) {
                    const int col = c * 512 + (k & 63) * 8 + (k >> 6);
                    if (col < N)
                        out[(int64_t)which * N + col] = (fold[k] + fold[512 + k]) + (fold[1024 + k] + fold[1536 + k]);
                }
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (col + i < N) {
                    out[col + i] = aw[c][i];
                    out[(int64_t)N + col + i] = ab[c][i];
                }
            }
        }
    }
}

// dx of rows of any length: two passes over the row by one block.
template <class T, class W>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_long_dx(NormDev d) {
    __shared__ float red[2][4];
    const int64_t row = blockIdx.x;
    const int N = d.cols;
    const T* x = static_cast<const T*>(d.x) + row * d.x_stride;
    const T* dy = static_cast<const T*>(d.dy) + row * d.y_stride;
    T* dx = static_cast<T*>(d.dx) + row * d.dx_stride;
    const W* w = static_cast<const W*>(d.w);
    const float mean = d.mean[row], rstd = d.rstd[row], n_f = (float)N;
    float s1 = 0.0f, s2 = 0.0f;
    for (int col = threadIdx.x * 8; col < N; col += kThreads * 8) {
        const Pack8<T> px = load8(x, col, N), pd = load8(dy, col, N);
        Pack8<W> pw;
        if (w) pw = load8(w, col, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float gi = (float)pd.v[i] * (w ? (float)pw.v[i] : 1.0f);
            s1 += gi;
            s2 += gi * (((float)px.v[i] - mean) * rstd);
        }
    }
    s1 = row_sum<4>(s1, red[0]) / n_f;
    s2 = row_sum<4>(s2, red[1]) / n_f;
    for (int col = threadIdx.x * 8; col < N; col += kThreads * 8) {
        const int n = N - col;
        const Pack8<T> px = load8(x, col, N), pd = load8(dy, col, N);
        Pack8<W> pw;
        if (w) pw = load8(w, col, N);
        Pack8<T> o;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float gi = (float)pd.v[i] * (w ? (float)pw.v[i] : 1.0f);
            o.v[i] = (T)(rstd * (gi - s1 - ((float)px.v[i] - mean) * rstd * s2));
        }
        store8(dx + col, o, n);
    }
}

// Partial sums of dweight and dbias for rows of any length: 2048 columns per blockIdx.y, every
// gridDim.x-th row.
template <class T, class W>
__global__ __launch_bounds__(kThreads) void k_norm_bwd_long_dw(NormDev d) {
    const int N = d.cols, col = ((int)blockIdx.y * kThreads + threadIdx.x) * 8, n = N - col;
    if (n <= 0) return;
    float aw[8] = {}, ab[8] = {};
    for (int64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const float mean = d.mean[row], rstd = d.rstd[row];
        const Pack8<T> px = load8(static_cast<const T*>(d.x) + row * d.x_stride, col, N);
        const Pack8<T> pd = load8(static_cast<const T*>(d.dy) + row * d.y_stride, col, N);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float dyi = (float)pd.v[i];
            aw[i] += dyi * (((float)px.v[i] - mean) * rstd);
            ab[i] += dyi;
        }
    }
    float* out = d.part + (int64_t)blockIdx.x * 2 * N + col;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i < n) {
            out[i] = aw[i];
            out[(int64_t)N + i] = ab[i];
        }
    }
}

// dweight and dbias from the blocks' partial sums: 16 columns per block, 16 rows of `part` side
// by side, added in a fixed order. blockIdx.y: 0 dweight, 1 dbias.
template <class W>
__global__ __launch_bounds__(kThreads) void k_norm_fold(NormDev d) {
    __shared__ float s[16][17];
    const int N = d.cols, c = threadIdx.x & 15, r = threadIdx.x >> 4;
    const int col = blockIdx.x * 16 + c;
    W* out = static_cast<W*>(blockIdx.y ? d.db : d.dw);
    if (!out) return;                        // the whole block
    float a = 0.0f;
    if (col < N)
#pragma unroll 8
        for (int k = r; k < d.blocks; k += 16) a += d.part[((int64_t)k * 2 + blockIdx.y) * N + col];
    s[r][c] = a;
    __syncthreads();
    if (r == 0 && col < N) {
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < 16; ++k) sum += s[k][c];
        out[col] = (W)sum;
    }
}

// A wave per row while its registers hold it (no barrier, four rows a block in flight), a block per row
// beyond. 16384x2048: fp32 52 us a wave, 41 a block; bf16 30 a wave, 34 a block.
template <class T, class W>
hipError_t fwd(const NormDev& d, hipStream_t st) {
    const int64_t N = d.cols;
    const unsigned wave_rows = (unsigned)((d.rows + 3) / 4), block_rows = (unsigned)d.rows;
    if (N < 8)          k_norm_fwd_long<T, W><<<block_rows, kThreads, 0, st>>>(d);
    else if (N <= 512)  k_norm_fwd<T, W, 1, 1><<<wave_rows, kThreads, 0, st>>>(d);
    else if (N <= 1024) k_norm_fwd<T, W, 1, 2><<<wave_rows, kThreads, 0, st>>>(d);
    else if (N <= 2048 && sizeof(T) == 2) k_norm_fwd<T, W, 1, 4><<<wave_rows, kThreads, 0, st>>>(d);
    else if (N <= 2048) k_norm_fwd<T, W, 4, 1><<<block_rows, kThreads, 0, st>>>(d);
    else if (N <= 4096) k_norm_fwd<T, W, 4, 2><<<block_rows, kThreads, 0, st>>>(d);
    else if (N <= 8192) k_norm_fwd<T, W, 4, 4><<<block_rows, kThreads, 0, st>>>(d);
    else                k_norm_fwd_long<T, W><<<block_rows, kThreads, 0, st>>>(d);
    return hipGetLastError();
}

// The backward pass holds two rows, the next two and two sums per column, so a row takes a block from
// 1025 columns on: bf16 16384x2048 55 us a wave, 50 a block; fp32 5003x1333 32 and 26.
template <class T, class W>
hipError_t bwd(const NormDev& d, hipStream_t st) {
    const int64_t N = d.cols;
    const unsigned nb = (unsigned)d.blocks;
    if (d.rows > 0) {
        if (N >= 8 && N <= 512) k_norm_bwd<T, W, 1, 1><<<nb, kThreads, 0, st>>>(d);
        else if (N >= 8 && N <= 1024) k_norm_bwd<T, W, 1, 2><<<nb, kThreads, 0, st>>>(d);
        else if (N >= 8 && N <= 2048) k_norm_bwd<T, W, 4, 1><<<nb, kThreads, 0, st>>>(d);
        else if (N >= 8 && N <= 4096) k_norm_bwd<T, W, 4, 2><<<nb, kThreads, 0, st>>>(d);
        else if (N >= 8 && N <= 8192) k_norm_bwd<T, W, 4, 4><<<nb, kThreads, 0, st>>>(d);
        else {
            // dx may overwrite dy: the sums over dy come first.
            if (d.part) k_norm_bwd_long_dw<T, W><<<dim3(nb, (unsigned)((N + 2047) / 2048)), kThreads, 0, st>>>(d);
            for (int64_t r0 = 0; d.dx && r0 < d.rows; r0 += kLaunchRows) {
                NormDev c = d;
                c.rows = d.rows - r0 < kLaunchRows ? d.rows - r0 : kLaunchRows;
                c.x = static_cast<const T*>(d.x) + r0 * d.x_stride;
                c.dy = static_cast<const T*>(d.dy) + r0 * d.y_stride;
                c.dx = static_cast<T*>(d.dx) + r0 * d.dx_stride;
                c.mean += r0;
                c.rstd += r0;
                k_norm_bwd_long_dx<T, W><<<(unsigned)c.rows, kThreads, 0, st>>>(c);
            }
        }
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.dw || d.db) k_norm_fold<W><<<dim3((unsigned)((N + 15) / 16), 2), kThreads, 0, st>>>(d);
    return hipGetLastError();
}

template <class F>
hipError_t dispatch(int dtype, int param_dtype, F f) {
    const bool pf = param_dtype == PA_F32;
    if (dtype == PA_F32) return f((float)0, (float)0);
    if (dtype == PA_BF16) return pf ? f((__bf16)0, (float)0) : f((__bf16)0, (__bf16)0);
    return pf ? f((_Float16)0, (float)0) : f((_Float16)0, (_Float16)0);
}

}  // namespace

// Launches of one block per row take at most 2^23 rows (a grid holds fewer than 2^32 threads).
hipError_t norm_forward(const NormDev& d, int dtype, int param_dtype, hipStream_t st) {
    return dispatch(dtype, param_dtype, [&](auto t, auto w) {
        for (int64_t r0 = 0; r0 < d.rows; r0 += kLaunchRows) {
            NormDev c = d;
            c.rows = d.rows - r0 < kLaunchRows ? d.rows - r0 : kLaunchRows;
            c.x = static_cast<const decltype(t)*>(d.x) + r0 * d.x_stride;
            c.y = static_cast<decltype(t)*>(d.y) + r0 * d.y_stride;
            c.mean = d.mean ? d.mean + r0 : nullptr;
            c.rstd = d.rstd ? d.rstd + r0 : nullptr;
            const hipError_t e = fwd<decltype(t), decltype(w)>(c, st);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    });
}

// Blocks of the backward pass: two for each of the 256 CUs, as the registers allow, and no more than
// there are groups of rows. More blocks cost more partial sums to write and join (512 rows of 4096 in 16 bits: 12.6 MB
// of data, 16.8 MB of sums). us with 512, 256 and 128 blocks: 32768x1024 40, 41, 71; 8192x1024 18, 17, 23; 5003x1333
// 24, 27, 44; but 2048x4096 30, 24, 29 and 512x4096 28, 20, 16 (all in 16 bits).
int norm_backward_blocks(int64_t rows, int64_t cols) {
    const int64_t groups = cols <= 1024 ? (rows + 3) / 4 : rows;
    const int64_t most = 512;
    return (int)(groups < most ? groups : most);
}

hipError_t norm_backward(const NormDev& d, int dtype, int param_dtype, hipStream_t st) {
    return dispatch(dtype, param_dtype, [&](auto t, auto w) { return bwd<decltype(t), decltype(w)>(d, st); });
}

}  // namespace pa
