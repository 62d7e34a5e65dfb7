// Projection with the low-rank adapters of many requests, for gfx950: y = x W^T + bias + t B_a^T with
// t = s_a (x A_a^T), a the adapter of the row's request.
//
// Two launches. k_lora_down computes t for the rows that have an adapter: a block takes 32 rows of
// one request, so it reads one adapter's A. The projection kernel computes x W^T and goes on
// accumulating: t is `rank` more columns of x and B_a as many more columns of W, a reduction that a
// tile repeats for each request that has rows in it, with the other requests' rows of t taken as
// zero. So the adapters cost their own products and no pass over y.
//
// t is rounded to the element type for the second product, as its operand has to be.
//
// The products are transposed (a lane owns a row of x, its registers hold output features), so that
// a lane stores consecutive features.
#include "pa_mma.h"

namespace pa {

namespace {

constexpr int kThreads = 256;

// Rows of request i, clamped to the matrix.
__device__ __forceinline__ int offset_at(const LoraDev& d, int i) {
    const int o = d.offsets[i];
    return o < 0 ? 0 : o > d.rows ? d.rows : o;
}

__device__ __forceinline__ int adapter_of(const LoraDev& d, int i) {
    const int a = d.ids[i];
    return a >= 0 && a < d.adapters ? a : -1;
}

// First request whose end lies beyond `row` (d.requests if none).
__device__ __forceinline__ int request_from(const LoraDev& d, int row) {
    int lo = 0, hi = d.requests;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (offset_at(d, mid + 1) > row) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// t of 32 rows of one request: block (c, i) takes rows 32 c .. of request i. Four waves take every
// fourth 64-column part of the reduction; NR 32-row tiles of A.
template <class T, int NR>
__global__ __launch_bounds__(kThreads) void k_lora_down(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    __shared__ float part[4][NR * 32][33];
    const int i = blockIdx.y, ad = adapter_of(d, i);
    if (ad < 0) return;
    const int beg = offset_at(d, i), end = offset_at(d, i + 1);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in;
    for (int r0 = beg + blockIdx.x * 32; r0 < end; r0 += gridDim.x * 32) {
        const int row = r0 + (lane & 31);
        const bool valid = row < end;
        const T* x = static_cast<const T*>(d.x) + (int64_t)(valid ? row : r0) * d.x_stride;
        const T* a = static_cast<const T*>(d.a) + (int64_t)ad * d.rank * K;
        f32x16 acc[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) acc[n] = f32x16{};
        for (int k0 = w * 64; k0 < K; k0 += 256) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const int k = k0 + ks * 16 + half * 8;
                const v8 xv = __builtin_bit_cast(v8, load8(x, k, K, valid));
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int r = n * 32 + (lane & 31);
                    const v8 av = __builtin_bit_cast(v8, load8(a + (int64_t)r * K, k, K, r < d.rank));
                    acc[n] = mma(av, xv, acc[n]);
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) part[w][n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][lane & 31] = acc[n][r];
        __syncthreads();
        const float s = d.scales ? d.scales[ad] : 1.0f;
        // Thread: row threadIdx / 8, ranks threadIdx % 8 + 8 j.
        const int tr = threadIdx.x >> 3;
        if (r0 + tr < end) {
            T* t = static_cast<T*>(d.t) + (int64_t)(r0 + tr) * d.rank_pad;
            for (int r = threadIdx.x & 7; r < d.rank_pad; r += 8)
                t[r] = (T)(((part[0][r][tr] + part[1][r][tr]) + (part[2][r][tr] + part[3][r][tr])) * s);
        }
    }
}

// The adapters' part of NM x NX 32 x 32 tiles: features f0 + 32 i + .., rows r0 + 32 j + ...
template <class T, int NM, int NX>
__device__ __forceinline__ void add_adapters(const LoraDev& d, int f0, int r0, int lane, f32x16 (&acc)[NM][NX]) {
    typedef typename Vec<T>::v8 v8;
    const int half = lane >> 5, r1 = r0 + 32 * NX < d.rows ? r0 + 32 * NX : d.rows;
    for (int i = request_from(d, r0); i < d.requests; ++i) {
        const int beg = offset_at(d, i), end = offset_at(d, i + 1);
        if (beg >= r1) break;
        const int ad = adapter_of(d, i);
        if (ad < 0 || beg >= end) continue;
        const T* b = static_cast<const T*>(d.b) + (int64_t)ad * d.out * d.rank;
        for (int k0 = 0; k0 < d.rank; k0 += 16) {
            const int k = k0 + half * 8;
            v8 tv[NX];
#pragma unroll
            for (int j = 0; j < NX; ++j) {
                const int row = r0 + j * 32 + (lane & 31);
                const bool mine = row >= beg && row < end;
                tv[j] = __builtin_bit_cast(v8, load8(static_cast<const T*>(d.t) + (int64_t)row * d.rank_pad, k, d.rank_pad, mine));
            }
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int f = f0 + m * 32 + (lane & 31);
                const v8 bv = __builtin_bit_cast(v8, load8(b + (int64_t)f * d.rank, k, d.rank, f < d.out));
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[m][j] = mma(bv, tv[j], acc[m][j]);
            }
        }
    }
}

// Adds the bias and stores NM x NX tiles.
template <class T, int NM, int NX>
__device__ __forceinline__ void finish(const LoraDev& d, int f0, int r0, int lane, f32x16 (&acc)[NM][NX]) {
    const int half = lane >> 5;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
        if (d.bias) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int f = f0 + m * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                const float bv = f < d.out ? (float)static_cast<const T*>(d.bias)[f] : 0.0f;
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[m][j][r] += bv;
            }
        }
#pragma unroll
        for (int j = 0; j < NX; ++j) {
            const int row = r0 + j * 32 + (lane & 31);
            T* y = static_cast<T*>(d.y) + (int64_t)row * d.y_stride;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const Pack8<T> p = gather8<T>(acc[m][j], q, 1.0f);
                const int f = f0 + m * 32 + q * 16 + half * 8;
                if (row < d.rows) store8(y + f, p, d.out - f);
            }
        }
    }
}

// 128 features x 128 rows per block, four waves of 64 x 64; the reduction goes through LDS in
// parts of 64 columns, the next part's loads in flight during the products of the current one.
template <class T>
__global__ __launch_bounds__(kThreads, 2) void k_lora_tile(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    constexpr int BK = 64, TILE = 128, PIECES = TILE * (BK / 8) / kThreads;
    __shared__ __align__(16) T tiles[2 * TILE * BK];
    T* wt = tiles;
    T* xt = tiles + TILE * BK;
    const int f_tiles = (d.out + TILE - 1) / TILE;
    const int id = xcd_order(blockIdx.x, gridDim.x);
    const int f0 = (id % f_tiles) * TILE, r0 = (id / f_tiles) * TILE;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in;
    Pack8<T> pw[PIECES], px[PIECES];
    auto load = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = threadIdx.x + i * kThreads, row = c >> 3, k = k0 + (c & 7) * 8;
            pw[i] = load8(static_cast<const T*>(d.w) + (int64_t)(f0 + row) * d.w_stride, k, K, f0 + row < d.out);
            px[i] = load8(static_cast<const T*>(d.x) + (int64_t)(r0 + row) * d.x_stride, k, K, r0 + row < d.rows);
        }
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[m][j] = f32x16{};
    const int fw = (w & 1) * 64, rw = (w >> 1) * 64;
    load(0);
    for (int k0 = 0; k0 < K; k0 += BK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int c = threadIdx.x + i * kThreads, at = piece_at<BK>(c >> 3, c & 7);
            *reinterpret_cast<uint4*>(wt + at) = __builtin_bit_cast(uint4, pw[i]);
            *reinterpret_cast<uint4*>(xt + at) = __builtin_bit_cast(uint4, px[i]);
        }
        __syncthreads();
        if (k0 + BK < K) load(k0 + BK);
#pragma unroll
        for (int ks = 0; ks < BK / 16; ++ks) {
            v8 a[2], b[2];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                a[m] = read_rows<T, BK>(wt, fw + m * 32 + (lane & 31), ks, half);
                b[m] = read_rows<T, BK>(xt, rw + m * 32 + (lane & 31), ks, half);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[m][j] = mma(a[m], b[j], acc[m][j]);
        }
    }
    if (d.adapters > 0) add_adapters<T, 2, 2>(d, f0 + fw, r0 + rw, lane, acc);
    finish<T, 2, 2>(d, f0 + fw, r0 + rw, lane, acc);
}

// Few rows: 32 features x 32 rows per block; W is read once, straight into operand registers, the
// four waves take every fourth 64-column part of the reduction and every fourth ... of it is joined
// through LDS.
template <class T>
__global__ __launch_bounds__(kThreads) void k_lora_rows(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    __shared__ float part[3][16][64];
    const int f0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in, f = f0 + (lane & 31), row = r0 + (lane & 31);
    const T* wp = static_cast<const T*>(d.w) + (int64_t)(f < d.out ? f : 0) * d.w_stride;
    const T* xp = static_cast<const T*>(d.x) + (int64_t)(row < d.rows ? row : 0) * d.x_stride;
    f32x16 acc[1][1] = {{f32x16{}}};
    for (int k0 = w * 64; k0 < K; k0 += 256) {
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int k = k0 + ks * 16 + half * 8;
            const v8 wv = __builtin_bit_cast(v8, load8(wp, k, K, f < d.out));
            const v8 xv = __builtin_bit_cast(v8, load8(xp, k, K, row < d.rows));
            acc[0][0] = mma(wv, xv, acc[0][0]);
        }
    }
    if (w > 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) part[w - 1][r][lane] = acc[0][0][r];
    }
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] = (acc[0][0][r] + part[0][r][lane]) + (part[1][r][lane] + part[2][r][lane]);
    if (d.adapters > 0) add_adapters<T, 1, 1>(d, f0, r0, lane, acc);
    finish<T, 1, 1>(d, f0, r0, lane, acc);
}

template <class T>
hipError_t run(const LoraDev& d, hipStream_t st) {
    if (d.adapters > 0 && d.requests > 0) {
        // Blocks per request: its share of the rows, so that a launch has about rows / 32 of them.
        const int per = d.rows / 32 / d.requests + 1;
        const dim3 grid((unsigned)(per < 4096 ? per : 4096), (unsigned)d.requests);
        if (d.rank <= 32)      k_lora_down<T, 1><<<grid, kThreads, 0, st>>>(d);
        else if (d.rank <= 64) k_lora_down<T, 2><<<grid, kThreads, 0, st>>>(d);
        else                   k_lora_down<T, 4><<<grid, kThreads, 0, st>>>(d);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.rows <= 64) k_lora_rows<T><<<dim3((unsigned)((d.out + 31) / 32), (unsigned)((d.rows + 31) / 32)), kThreads, 0, st>>>(d);
    else k_lora_tile<T><<<(unsigned)(((int64_t)d.out + 127) / 128 * ((d.rows + 127) / 128)), kThreads, 0, st>>>(d);
    return hipGetLastError();
}

}  // namespace

hipError_t lora_linear(const LoraDev& d, int dtype, hipStream_t st) {
    return dtype == PA_BF16 ? run<__bf16>(d, st) : run<_Float16>(d, st);
}

}  // namespace pa
