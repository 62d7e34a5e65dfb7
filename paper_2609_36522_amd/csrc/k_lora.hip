// Projection with the low-rank adapters of many requests, for gfx950: y = x W^T + bias + t B_a^T with
// t = s_a (x A_a^T), a the adapter of the row's request.
//
// Two launches. The first computes t for the rows that have an adapter: a block takes rows of one
// request, so it reads one adapter's A. The projection computes x W^T and goes on accumulating: t is
// `rank` more columns of x and B_a as many more columns of W, a reduction that a tile repeats for each
// request that has rows in it, with the other requests' rows of t taken as zero. So the adapters cost
// their own products and no pass over y.
//
// t is rounded to the element type for the second product, as its operand has to be.
//
// The products are transposed (a lane owns a row of x, its registers hold output features), so that
// a lane stores consecutive features.
#include <type_traits>

#include "pa_mma.h"

namespace pa {

namespace {

// Row strides below this leave every offset within a tile of 256 rows to 32 bits.
constexpr int64_t kBufferStride = 1 << 22;
constexpr int kCUs = 256;

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

// Eight elements at .. of a row of len; without RAGGED len is a multiple of 8, with it the operand is
// whole after `fixed`.
template <class T, bool RAGGED>
__device__ __forceinline__ typename Vec<T>::v8 operand(const T* row, int at, int len, bool valid) {
    if constexpr (RAGGED) {
        return __builtin_bit_cast(typename Vec<T>::v8, load8_raw(row, at, len, valid));
    } else {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (valid && at < len) r = __builtin_bit_cast(uint4, *reinterpret_cast<const Pack8<T>*>(row + at));
        return __builtin_bit_cast(typename Vec<T>::v8, r);
    }
}

template <class T, bool RAGGED>
__device__ __forceinline__ typename Vec<T>::v8 fixed(typename Vec<T>::v8 r, int at, int len) {
    if constexpr (RAGGED) return __builtin_bit_cast(typename Vec<T>::v8, fix8(__builtin_bit_cast(Pack8<T>, r), at, len));
    return r;
}

// ROWS rows x 64 columns of a matrix on their way to LDS, THREADS threads. Without RAGGED by loads that
// write LDS themselves (a wave's lanes fill consecutive 16-byte slots, so the permutation of a row's
// pieces is in the addresses that they read; what does not exist has an offset out of the buffer's range,
// which reads as zero), otherwise through registers.
template <class T, int ROWS, int THREADS, bool RAGGED>
struct Stage {
    static constexpr int kPieces = ROWS * 8 / THREADS, kStep = THREADS / 8;
    uint4 r[RAGGED ? kPieces : 1];
    uint32_t off[RAGGED ? 1 : kPieces];
    int piece, row, left;

    __device__ __forceinline__ Stage(int64_t stride, int rows) {
        row = (int)threadIdx.x >> 3;
        piece = (int)threadIdx.x & 7;
        if constexpr (!RAGGED) {
            piece = (piece_at<64>(row, piece) - row * 64) >> 3;     // the same for every kStep (16 or more) rows
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                off[i] = row + i * kStep < rows ? (uint32_t)((row + i * kStep) * (int)stride + piece * 8) * 2 : kNowhere;
        }
    }
    // The 64 columns at `base` (rows of it exist), `cols` of them left in the row.
    __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int cols, T* tile) {
        if constexpr (RAGGED) {
            left = cols;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                r[i] = __builtin_bit_cast(uint4, load8_raw(base + (row + i * kStep) * stride, piece * 8, cols, row + i * kStep < rows));
        } else {
            const __amdgpu_buffer_rsrc_t from = buffer_at(base);
            const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            const bool in = piece * 8 < cols;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                load_lds(from, tile + (w * 64 + i * THREADS) * 8, in ? off[i] : kNowhere, 0);
        }
    }
    // The tile is in LDS once every thread has called this and a barrier has passed.
    __device__ __forceinline__ void arrive(T* tile) const {
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                *reinterpret_cast<uint4*>(tile + piece_at<64>(row + i * kStep, piece)) =
                    __builtin_bit_cast(uint4, fix8(__builtin_bit_cast(Pack8<T>, r[i]), piece * 8, left));
        } else {
            wait_loads();
        }
    }
};

// t of 64 rows of one request: block (c, i) takes rows 64 c .. of request i, all of them if the grid is
// smaller. Of the four waves two take 32 rows each, over half of the reduction; NR 32-row tiles of A.
template <class T, int NR, bool RAGGED>
__global__ __launch_bounds__(256) void k_lora_down(LoraDev d) {
    constexpr int ROWS = 64;
    __shared__ __align__(16) T tiles[2][(ROWS + NR * 32) * 64];
    __shared__ float part[NR * 32][ROWS + 1];
    const int i = blockIdx.y, ad = adapter_of(d, i);
    if (ad < 0) return;
    const int beg = offset_at(d, i), end = offset_at(d, i + 1);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6, rw = w & 1, kw = w >> 1;
    const int K = d.in;
    const T* a = static_cast<const T*>(d.a) + (int64_t)ad * d.rank * K;
    const float s = d.scales ? d.scales[ad] : 1.0f;
    for (int r0 = beg + blockIdx.x * ROWS; r0 < end; r0 += gridDim.x * ROWS) {
        const T* x = static_cast<const T*>(d.x) + (int64_t)r0 * d.x_stride;
        Stage<T, ROWS, 256, RAGGED> sx(d.x_stride, end - r0);
        Stage<T, NR * 32, 256, RAGGED> sa(K, d.rank);
        f32x16 acc[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) acc[n] = f32x16{};
        auto load = [&](int k0, int p) {
            sx.load(x + k0, d.x_stride, end - r0, K - k0, tiles[p]);
            sa.load(a + k0, K, d.rank, K - k0, tiles[p] + ROWS * 64);
        };
        auto arrive = [&](int p) {
            sx.arrive(tiles[p]);
            sa.arrive(tiles[p] + ROWS * 64);
        };
        load(0, 0);
        arrive(0);
        __syncthreads();
        int p = 0;
        for (int k0 = 0; k0 < K; k0 += 64, p ^= 1) {
            if (k0 + 64 < K) load(k0 + 64, p ^ 1);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const auto xv = read_rows<T, 64>(tiles[p], rw * 32 + (lane & 31), kw * 2 + ks, half);
#pragma unroll
                for (int n = 0; n < NR; ++n)
                    acc[n] = mma(read_rows<T, 64>(tiles[p] + ROWS * 64, n * 32 + (lane & 31), kw * 2 + ks, half), xv, acc[n]);
            }
            if (k0 + 64 < K) arrive(p ^ 1);
            __syncthreads();
        }
        if (kw == 1) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) part[n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][rw * 32 + (lane & 31)] = acc[n][r];
        }
        __syncthreads();
        if (kw == 0) {
            const int row = r0 + rw * 32 + (lane & 31);
            T* t = static_cast<T*>(d.t) + (int64_t)row * d.rank_pad;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][r] += part[n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][rw * 32 + (lane & 31)];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const Pack8<T> o = gather8<T>(acc[n], q, s);
                    const int r = n * 32 + q * 16 + half * 8;
                    if (row < end && r < d.rank_pad) *reinterpret_cast<Pack8<T>*>(t + r) = o;
                }
            }
        }
        __syncthreads();
    }
}

// The same for requests of few rows: 32 rows a block, 16 / NR waves that take parts of 64 columns in
// turn, every operand straight from memory, so that one token's reduction is in flight all at once.
template <class T, int NR, bool RAGGED>
__global__ __launch_bounds__(1024 / NR) void k_lora_down_few(LoraDev d) {
    constexpr int WAVES = 16 / NR;
    __shared__ float part[WAVES][NR * 32][33];
    const int i = blockIdx.y, ad = adapter_of(d, i);
    if (ad < 0) return;
    const int beg = offset_at(d, i), end = offset_at(d, i + 1);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in;
    const T* a = static_cast<const T*>(d.a) + (int64_t)ad * d.rank * K;
    const float s = d.scales ? d.scales[ad] : 1.0f;
    for (int r0 = beg + blockIdx.x * 32; r0 < end; r0 += gridDim.x * 32) {
        const int row = r0 + (lane & 31);
        const T* x = static_cast<const T*>(d.x) + (int64_t)(row < end ? row : r0) * d.x_stride;
        f32x16 acc[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) acc[n] = f32x16{};
        for (int k0 = w * 64; k0 < K; k0 += WAVES * 64) {
            typename Vec<T>::v8 xv[4], av[4][NR];
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                const int k = k0 + ks * 16 + half * 8;
                xv[ks] = operand<T, RAGGED>(x, k, K, row < end);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int r = n * 32 + (lane & 31);
                    av[ks][n] = operand<T, RAGGED>(a + (int64_t)(r < d.rank ? r : 0) * K, k, K, r < d.rank);
                }
            }
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int k = k0 + ks * 16 + half * 8;
                    acc[n] = mma(fixed<T, RAGGED>(av[ks][n], k, K), fixed<T, RAGGED>(xv[ks], k, K), acc[n]);
                }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) part[w][n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][lane & 31] = acc[n][r];
        __syncthreads();
        for (int e = threadIdx.x; e < 32 * d.rank_pad; e += WAVES * 64) {
            const int tr = e / d.rank_pad, r = e - tr * d.rank_pad;
            if (r0 + tr >= end) continue;
            float v = 0.0f;
#pragma unroll
            for (int j = 0; j < WAVES; ++j) v += part[j][r][tr];
            static_cast<T*>(d.t)[(int64_t)(r0 + tr) * d.rank_pad + r] = (T)(v * s);
        }
    }
}

// The adapters' part of NM x NX 32 x 32 tiles: features f0 + 32 i + .., rows r0 + 32 j + ..; every
// `step`-th request from the `first`-th of those that have rows here.
template <class T, int NM, int NX, bool RAGGED>
__device__ __forceinline__ void add_adapters(const LoraDev& d, int f0, int r0, int lane, f32x16 (&acc)[NM][NX], int first = 0, int step = 1) {
    typedef typename Vec<T>::v8 v8;
    const int half = lane >> 5, r1 = r0 + 32 * NX < d.rows ? r0 + 32 * NX : d.rows;
    for (int i = request_from(d, r0) + first; i < d.requests; i += step) {
        const int beg = offset_at(d, i), end = offset_at(d, i + 1);
        if (beg >= r1) break;
        const int ad = adapter_of(d, i);
        if (ad < 0 || beg >= end) continue;
        const T* b = static_cast<const T*>(d.b) + (int64_t)ad * d.out * d.rank;
        for (int k0 = 0; k0 < d.rank; k0 += 16) {
            const int k = k0 + half * 8;
            v8 tv[NX], bv[NM];
#pragma unroll
            for (int j = 0; j < NX; ++j) {
                const int row = r0 + j * 32 + (lane & 31);
                tv[j] = operand<T, false>(static_cast<const T*>(d.t) + (int64_t)row * d.rank_pad, k, d.rank_pad, row >= beg && row < end);
            }
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                const int f = f0 + m * 32 + (lane & 31);
                bv[m] = operand<T, RAGGED>(b + (int64_t)f * d.rank, k, d.rank, f < d.out);
            }
#pragma unroll
            for (int m = 0; m < NM; ++m)
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[m][j] = mma(fixed<T, RAGGED>(bv[m], k, d.rank), tv[j], acc[m][j]);
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

// WF x WR waves of NM x NX tiles of 32 x 32 (features x rows) per block. The reduction goes through LDS in
// parts of 64 columns, double buffered: the next part's loads are in flight during the products of the
// current one.
template <class T, int WF, int WR, int NM, int NX, bool RAGGED>
__global__ __launch_bounds__(64 * WF * WR, 2) void k_lora_tile(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    constexpr int TF = WF * NM * 32, TR = WR * NX * 32, THREADS = 64 * WF * WR;
    __shared__ __align__(16) T tiles[2][(TF + TR) * 64];
    const int f_tiles = (d.out + TF - 1) / TF;
    const int id = xcd_order(blockIdx.x, gridDim.x);
    const int f0 = (id % f_tiles) * TF, r0 = (id / f_tiles) * TR;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in;
    const T* wp = static_cast<const T*>(d.w) + (int64_t)f0 * d.w_stride;
    const T* xp = static_cast<const T*>(d.x) + (int64_t)r0 * d.x_stride;
    Stage<T, TF, THREADS, RAGGED> sw(d.w_stride, d.out - f0);
    Stage<T, TR, THREADS, RAGGED> sx(d.x_stride, d.rows - r0);
    auto load = [&](int k0, int p) {
        sw.load(wp + k0, d.w_stride, d.out - f0, K - k0, tiles[p]);
        sx.load(xp + k0, d.x_stride, d.rows - r0, K - k0, tiles[p] + TF * 64);
    };
    auto arrive = [&](int p) {
        sw.arrive(tiles[p]);
        sx.arrive(tiles[p] + TF * 64);
    };
    f32x16 acc[NM][NX];
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int j = 0; j < NX; ++j) acc[m][j] = f32x16{};
    const int fw = (w % WF) * NM * 32, rw = (w / WF) * NX * 32;
    load(0, 0);
    arrive(0);
    __syncthreads();
    int p = 0;
    for (int k0 = 0; k0 < K; k0 += 64, p ^= 1) {
        if (k0 + 64 < K) load(k0 + 64, p ^ 1);
        const T* wt = tiles[p];
        const T* xt = tiles[p] + TF * 64;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            v8 a[NM], b[NX];
#pragma unroll
            for (int m = 0; m < NM; ++m) a[m] = read_rows<T, 64>(wt, fw + m * 32 + (lane & 31), ks, half);
#pragma unroll
            for (int j = 0; j < NX; ++j) b[j] = read_rows<T, 64>(xt, rw + j * 32 + (lane & 31), ks, half);
#pragma unroll
            for (int m = 0; m < NM; ++m)
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[m][j] = mma(a[m], b[j], acc[m][j]);
        }
        if (k0 + 64 < K) arrive(p ^ 1);
        __syncthreads();
    }
    if (d.adapters > 0) add_adapters<T, NM, NX, RAGGED>(d, f0 + fw, r0 + rw, lane, acc);
    finish<T, NM, NX>(d, f0 + fw, r0 + rw, lane, acc);
}

// Few rows: 32 features x 32 rows per block. W is read once, straight into operand registers; 16 waves
// take parts of 64 columns in turn, and the requests' adapters in turn, and are joined through LDS.
template <class T, bool RAGGED>
__global__ __launch_bounds__(1024) void k_lora_rows(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    __shared__ float part[16][16][64];
    const int f0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in, f = f0 + (lane & 31), row = r0 + (lane & 31);
    const T* wp = static_cast<const T*>(d.w) + (int64_t)(f < d.out ? f : 0) * d.w_stride;
    const T* xp = static_cast<const T*>(d.x) + (int64_t)(row < d.rows ? row : 0) * d.x_stride;
    f32x16 acc[1][1] = {{f32x16{}}};
    for (int k0 = w * 64; k0 < K; k0 += 1024) {
        v8 wv[4], xv[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int k = k0 + ks * 16 + half * 8;
            wv[ks] = operand<T, RAGGED>(wp, k, K, f < d.out);
            xv[ks] = operand<T, RAGGED>(xp, k, K, row < d.rows);
        }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int k = k0 + ks * 16 + half * 8;
            acc[0][0] = mma(fixed<T, RAGGED>(wv[ks], k, K), fixed<T, RAGGED>(xv[ks], k, K), acc[0][0]);
        }
    }
    if (d.adapters > 0) add_adapters<T, 1, 1, RAGGED>(d, f0, r0, lane, acc, w, 16);
#pragma unroll
    for (int r = 0; r < 16; ++r) part[w][r][lane] = acc[0][0][r];
    __syncthreads();
    // Wave w sums register w of the accumulators, in a fixed order; wave 0 stores.
    float v = 0.0f;
#pragma unroll
    for (int j = 0; j < 16; ++j) v += part[j][w][lane];
    __syncthreads();
    part[0][w][lane] = v;
    __syncthreads();
    if (w > 0) return;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] = part[0][r][lane];
    finish<T, 1, 1>(d, f0, r0, lane, acc);
}

template <class T, int NR, bool RAGGED>
void down(const LoraDev& d, hipStream_t st) {
    // Blocks per request: its share of the rows, so that the launch has about rows / 64 (or 32) of them.
    // Requests of fewer than 64 rows on average are latency bound.
    const bool few = d.rows < 64 * d.requests;
    const int per = d.rows / (few ? 32 : 64) / d.requests + 1;
    const dim3 grid((unsigned)(per < 4096 ? per : 4096), (unsigned)d.requests);
    if (few) k_lora_down_few<T, NR, RAGGED><<<grid, 1024 / NR, 0, st>>>(d);
    else k_lora_down<T, NR, RAGGED><<<grid, 256, 0, st>>>(d);
}

int64_t tiles_of(const LoraDev& d, int t) { return (int64_t)((d.out + t - 1) / t) * ((d.rows + t - 1) / t); }

// The largest tile that still gives every CU a block; few rows read W straight from memory.
template <class T, bool RAGGED>
hipError_t run(const LoraDev& d, hipStream_t st) {
    if (d.adapters > 0) {
        if (d.rank <= 32)      down<T, 1, RAGGED>(d, st);
        else if (d.rank <= 64) down<T, 2, RAGGED>(d, st);
        else                   down<T, 4, RAGGED>(d, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.rows <= 64)
        k_lora_rows<T, RAGGED><<<dim3((unsigned)((d.out + 31) / 32), (unsigned)((d.rows + 31) / 32)), 1024, 0, st>>>(d);
    else if (!RAGGED && tiles_of(d, 256) >= kCUs)
        k_lora_tile<T, 2, 4, 4, 2, false><<<(unsigned)tiles_of(d, 256), 512, 0, st>>>(d);
    else if (tiles_of(d, 128) >= kCUs)
        k_lora_tile<T, 2, 2, 2, 2, RAGGED><<<(unsigned)tiles_of(d, 128), 256, 0, st>>>(d);
    else
        k_lora_tile<T, 2, 2, 1, 1, RAGGED><<<(unsigned)tiles_of(d, 64), 256, 0, st>>>(d);
    return hipGetLastError();
}

}  // namespace

hipError_t lora_linear(const LoraDev& d, int dtype, hipStream_t st) {
    const bool ragged = d.in % 8 != 0 || d.rank % 8 != 0 || d.x_stride >= kBufferStride || d.w_stride >= kBufferStride;
    if (dtype == PA_BF16) return ragged ? run<__bf16, true>(d, st) : run<__bf16, false>(d, st);
    return ragged ? run<_Float16, true>(d, st) : run<_Float16, false>(d, st);
}

}  // namespace pa
