// Projection with the low-rank adapters of many requests, for gfx950: y = x W^T + bias + t B_a^T with
// t = s_a (x A_a^T), a the adapter of the row's request.
//
// Two launches. The first computes t for the rows that have an adapter: a block takes rows of one
// request, so it reads one adapter's A. The projection computes x W^T and goes on accumulating: t is
// `rank` more columns of x and B_a as many more columns of W, a reduction that a tile repeats for each
// request that has rows in it, with the other requests' rows of t taken as zero. So the adapters cost
// their own products and no pass over y.
//
// t is rounded to the element type for the second product, as its operand has to be. Its columns past the
// rank (up to a multiple of 16) are stored as zeros: an infinity in x times the zeros in the place of A's
// missing rows is a NaN.
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

// A width of its own for the tiles: rows of an even number of elements (at least 8) at even addresses and
// strides, which are read as whole ones are but for the piece that holds the row's end (32768x2044x2048:
// 492 us as ragged rows, 289 so). It and kWhole are for ranks of a multiple of 8. Rows of an odd length, stride or
// address are taken as ragged ones; loads that write LDS serve them too (cross attention's do) and are not used
// here: 32768x2045x2048, rank 64, 533 us as ragged rows, 350 as even ones would be.
constexpr int kEven = 3;
constexpr bool direct(int width) { return width == kWhole || width == kEven; }

// Rows of request i, clamped to the matrix.
__device__ __forceinline__ int offset_at(const LoraDev& d, int i) {
    const int o = d.offsets[i];
    return o < 0 ? 0 : o > d.rows ? d.rows : o;
}

__device__ __forceinline__ int adapter_of(const LoraDev& d, int i) {
    const int a = d.ids[i];
    return a >= 0 && a < d.adapters ? a : -1;
}

// First request whose end lies beyond `row` (d.requests if none): a wave looks at 64 requests at a time.
__device__ __forceinline__ int request_from(const LoraDev& d, int row) {
    const int lane = threadIdx.x & 63;
    for (int i = 0; i < d.requests; i += 64) {
        const unsigned long long beyond = __ballot(i + lane < d.requests && offset_at(d, i + lane + 1) > row);
        if (beyond) return i + __builtin_ctzll(beyond);
    }
    return d.requests;
}

// ROWS rows x 64 columns of a matrix on their way to LDS, THREADS threads. kWhole and kEven by loads that write
// LDS themselves (a wave's lanes fill consecutive 16-byte slots, so the permutation of a row's pieces is in
// the addresses that they read; what does not exist has an offset out of the buffer's range, which reads
// as zero), otherwise through registers. A piece that holds a row's end is read as the row's last eight
// elements and moved into place once it is there.
template <class T, int ROWS, int THREADS, int WIDTH>
struct Stage {
    static constexpr int kPieces = ROWS * 8 / THREADS, kStep = THREADS / 8;
    uint4 r[2][direct(WIDTH) ? 1 : kPieces];         // two sets of registers: parts of two loads in flight
    uint32_t off[direct(WIDTH) ? kPieces : 1];
    int piece, row, rows, at[2], len;

    // The matrix's row 0 of this tile exists, and rows - 1 more; rows are n long.
    __device__ __forceinline__ Stage(int64_t stride, int rows_, int n) : rows(rows_), at{0, 0}, len(n) {
        row = (int)threadIdx.x >> 3;
        piece = (int)threadIdx.x & 7;
        if constexpr (direct(WIDTH)) {
            piece = (piece_at<64>(row, piece) - row * 64) >> 3;     // the same for every kStep (16 or more) rows
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                off[i] = row + i * kStep < rows ? (uint32_t)((row + i * kStep) * (int)stride + piece * 8) * 2 : kNowhere;
        }
    }
    // Columns k0 .. of the rows at `base`.
    template <int SET = 0>
    __device__ __forceinline__ void load(const T* base, int64_t stride, int k0, T* tile) {
        if constexpr (direct(WIDTH)) {
            const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            const bool in = k0 + piece * 8 < len;
            if (WIDTH == kEven && k0 + 64 > len) {                  // the rows' last columns
                at[0] = k0 + piece * 8;
                const uint32_t col = (at[0] + 8 <= len ? k0 : len - 8 - piece * 8) * 2;
                const __amdgpu_buffer_rsrc_t from = buffer_at(base);
#pragma unroll
                for (int i = 0; i < kPieces; ++i)
                    load_lds(from, tile + (w * 64 + i * THREADS) * 8, in && off[i] != kNowhere ? off[i] + col : kNowhere, 0);
            } else {
                const __amdgpu_buffer_rsrc_t from = buffer_at(base + k0);
#pragma unroll
                for (int i = 0; i < kPieces; ++i) load_lds(from, tile + (w * 64 + i * THREADS) * 8, in ? off[i] : kNowhere, 0);
            }
        } else {
            at[SET] = k0 + piece * 8;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const bool valid = row + i * kStep < rows;
                const T* p = base + (valid ? row + i * kStep : 0) * stride;
                r[SET][i] = WIDTH == kRagged ? __builtin_bit_cast(uint4, load8_raw(p, at[SET], len))
                                             : __builtin_bit_cast(uint4, load8(p, at[SET], len, valid));
            }
        }
    }
    // Registers into LDS; direct loads (which the caller has waited for) are in place but for the rows' last
    // columns, which the last part's threads move.
    template <int SET = 0>
    __device__ __forceinline__ void arrive(T* tile, bool last) {
        if constexpr (WIDTH == kEven) {
            if (last && at[0] < len && at[0] + 8 > len) {
#pragma unroll
                for (int i = 0; i < kPieces; ++i) {
                    uint4* slot = reinterpret_cast<uint4*>(tile + (threadIdx.x + i * THREADS) * 8);
                    *slot = __builtin_bit_cast(uint4, shift8(__builtin_bit_cast(Pack8<T>, *slot), at[0] + 8 - len));
                }
            }
        } else if constexpr (WIDTH != kWhole) {
            const bool whole = at[SET] - piece * 8 + 64 <= len && rows >= ROWS; // nothing to fix (the same in all lanes)
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if (WIDTH == kRagged && !whole)
                    r[SET][i] = __builtin_bit_cast(uint4, fix8(__builtin_bit_cast(Pack8<T>, r[SET][i]), at[SET], len, row + i * kStep < rows));
                *reinterpret_cast<uint4*>(tile + piece_at<64>(row + i * kStep, piece)) = r[SET][i];
            }
        }
    }
};

// t of 64 rows of one request: block (c, i) takes rows 64 c .. of request i, all of them if the grid is
// smaller. Of the four waves two take 32 rows each, over half of the reduction; NR 32-row tiles of A. Bound by
// the reading of x: three parts of 64 columns are on their way during the products of the current one.
// 32768x2048, rank 64: 32 to 52 us (134 MB, 2.6 to 4.2 TB/s, by what the last-level cache holds of x).
template <class T, int NR, int WIDTH>
__global__ __launch_bounds__(256) void k_lora_down(LoraDev d) {
    constexpr int ROWS = 64, STAGES = direct(WIDTH) ? 4 : 2, PART = (ROWS + NR * 32) * 64, LOADS = (ROWS + NR * 32) * 8 / 256;
    static_assert(STAGES * PART * 2 >= NR * 32 * (ROWS + 1) * 4, "the halves of the reduction are joined in the tiles' memory");
    __shared__ __align__(16) T tiles[STAGES * PART];
    float (*join)[ROWS + 1] = reinterpret_cast<float (*)[ROWS + 1]>(tiles);
    const int i = blockIdx.y, ad = adapter_of(d, i);
    if (ad < 0) return;
    const int beg = offset_at(d, i), end = offset_at(d, i + 1);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6, rw = w & 1, kw = w >> 1;
    const int K = d.in, parts = (K + 63) / 64;
    const T* a = static_cast<const T*>(d.a) + (int64_t)ad * d.rank * K;
    const float s = d.scales ? d.scales[ad] : 1.0f;
    for (int r0 = beg + blockIdx.x * ROWS; r0 < end; r0 += gridDim.x * ROWS) {
        const T* x = static_cast<const T*>(d.x) + (int64_t)r0 * d.x_stride;
        Stage<T, ROWS, 256, WIDTH> sx(d.x_stride, end - r0, K);
        Stage<T, NR * 32, 256, WIDTH> sa(K, d.rank, K);
        f32x16 acc[NR];
#pragma unroll
        for (int n = 0; n < NR; ++n) acc[n] = f32x16{};
        auto load = [&](int part, int p) {
            sx.load(x, d.x_stride, part * 64, tiles + p * PART);
            sa.load(a, K, part * 64, tiles + p * PART + ROWS * 64);
        };
        auto arrive = [&](int part, int p) {
            sx.arrive(tiles + p * PART, part == parts - 1);
            sa.arrive(tiles + p * PART + ROWS * 64, part == parts - 1);
        };
#pragma unroll
        for (int n = 0; n < STAGES - 1; ++n)
            if (n < parts) load(n, n);
        if (parts >= STAGES - 1) wait_loads<(STAGES - 2) * LOADS>();
        else wait_loads();
        arrive(0, 0);
        lds_barrier();
        for (int n = 0; n < parts; ++n) {
            const T* xt = tiles + n % STAGES * PART;
            const T* at = xt + ROWS * 64;
            const int q = (n + STAGES - 1) % STAGES;
            if (n + STAGES - 1 < parts) load(n + STAGES - 1, q);
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                const auto xv = read_rows<T, 64>(xt, rw * 32 + (lane & 31), kw * 2 + ks, half);
#pragma unroll
                for (int m = 0; m < NR; ++m)
                    acc[m] = mma(read_rows<T, 64>(at, m * 32 + (lane & 31), kw * 2 + ks, half), xv, acc[m]);
            }
            if (n + 1 < parts) {
                if (n + STAGES - 1 < parts) wait_loads<(STAGES - 2) * LOADS>();      // the next part is there
                else wait_loads();
                arrive(n + 1, (n + 1) % STAGES);
            }
            lds_barrier();
        }
        if (kw == 1) {
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) join[n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][rw * 32 + (lane & 31)] = acc[n][r];
        }
        __syncthreads();
        if (kw == 0) {
            const int row = r0 + rw * 32 + (lane & 31);
            T* t = static_cast<T*>(d.t) + (int64_t)row * d.rank_pad;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][r] += join[n * 32 + 8 * (r >> 2) + 4 * half + (r & 3)][rw * 32 + (lane & 31)];
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    Pack8<T> o = gather8<T>(acc[n], q, s);
                    const int r = n * 32 + q * 16 + half * 8;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (r + e >= d.rank) o.v[e] = (T)0.0f;
                    if (row < end && r < d.rank_pad) *reinterpret_cast<Pack8<T>*>(t + r) = o;
                }
            }
        }
        __syncthreads();
    }
}

// The same for requests of few rows: 32 rows a block, 16 / NR waves that take parts of 64 columns in
// turn, every operand straight from memory, so that one token's reduction is in flight all at once: 5 us for
// eight rows of 1024, of which a launch and a chain of two loads are most.
template <class T, int NR, int WIDTH>
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
                xv[ks] = operand<T, WIDTH>(x, k, K, row < end);
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int r = n * 32 + (lane & 31);
                    av[ks][n] = operand<T, WIDTH>(a + (int64_t)(r < d.rank ? r : 0) * K, k, K, r < d.rank);
                }
            }
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int n = 0; n < NR; ++n) {
                    const int k = k0 + ks * 16 + half * 8;
                    acc[n] = mma(fixed<T, WIDTH>(av[ks][n], k, K, n * 32 + (lane & 31) < d.rank), fixed<T, WIDTH>(xv[ks], k, K, row < end), acc[n]);
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
            static_cast<T*>(d.t)[(int64_t)(r0 + tr) * d.rank_pad + r] = (T)(r < d.rank ? v * s : 0.0f);
        }
    }
}

// The adapters' part of NM x NX 32 x 32 tiles: features f0 + 32 i + .., rows r0 + 32 j + ..; every
// `step`-th request from `first`, the first that has rows at r0 or after. Where a request has all of the
// tiles' rows its product goes on in their accumulators. Otherwise 32 rows that it has a part of are carried on
// in a copy, of which the lanes of its rows (a lane owns a row) are taken: zeros in t for the others would not
// do, as 0 times an infinity or a NaN in B is a NaN. It costs up to 3% where requests are long, and a tenth
// where each row is one (256 rows of 1024x1024, rank 16: 28 us with zeros in t, 31 so; sums of their own, added
// by the request's lanes, 30, but 342 in place of 334 for 32768x2048x2048, rank 64).
template <class T, int NM, int NX, int WIDTH>
__device__ __forceinline__ void add_adapters(const LoraDev& d, int f0, int r0, int lane, f32x16 (&acc)[NM][NX], int first, int step = 1) {
    typedef typename Vec<T>::v8 v8;
    const int half = lane >> 5, r1 = r0 + 32 * NX < d.rows ? r0 + 32 * NX : d.rows;
    for (int i = first; i < d.requests; i += step) {
        const int beg = offset_at(d, i), end = offset_at(d, i + 1);
        if (beg >= r1) break;
        const int ad = adapter_of(d, i);
        if (ad < 0 || beg >= end) continue;
        const T* b = static_cast<const T*>(d.b) + (int64_t)ad * d.out * d.rank;
        auto t_at = [&](int j, int k) {
            const int row = r0 + j * 32 + (lane & 31);
            return operand<T, kWhole>(static_cast<const T*>(d.t) + (int64_t)row * d.rank_pad, k, d.rank_pad, row >= beg && row < end);
        };
        auto b_at = [&](int m, int k) {
            const int f = f0 + m * 32 + (lane & 31);
            return operand<T, direct(WIDTH) ? kWhole : kTiny>(b + (int64_t)f * d.rank, k, d.rank, f < d.out);
        };
        if (beg <= r0 && end >= r1) {
            for (int k0 = 0; k0 < d.rank; k0 += 16) {
                const int k = k0 + half * 8;
                v8 tv[NX], bv[NM];
#pragma unroll
                for (int j = 0; j < NX; ++j) tv[j] = t_at(j, k);
#pragma unroll
                for (int m = 0; m < NM; ++m) bv[m] = b_at(m, k);
#pragma unroll
                for (int m = 0; m < NM; ++m)
#pragma unroll
                    for (int j = 0; j < NX; ++j) acc[m][j] = mma(bv[m], tv[j], acc[m][j]);
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < NX; ++j) {
            const int row = r0 + j * 32 + (lane & 31);
            if (beg >= r0 + j * 32 + 32 || end <= r0 + j * 32) continue;     // the same in all lanes
            f32x16 sum[NM];
#pragma unroll
            for (int m = 0; m < NM; ++m) sum[m] = acc[m][j];
            for (int k0 = 0; k0 < d.rank; k0 += 16) {
                const int k = k0 + half * 8;
                const v8 tv = t_at(j, k);
                v8 bv[NM];
#pragma unroll
                for (int m = 0; m < NM; ++m) bv[m] = b_at(m, k);
#pragma unroll
                for (int m = 0; m < NM; ++m) sum[m] = mma(bv[m], tv, sum[m]);
            }
            const bool own = row >= beg && row < end;
#pragma unroll
            for (int m = 0; m < NM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[m][j][r] = own ? sum[m][r] : acc[m][j][r];
        }
    }
}

// Accumulators that start from the bias.
template <class T, int NM, int NX>
__device__ __forceinline__ void start(const LoraDev& d, int f0, int lane, f32x16 (&acc)[NM][NX]) {
    const int half = lane >> 5;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int f = f0 + m * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
            const float v = d.bias ? (float)static_cast<const T*>(d.bias)[f < d.out ? f : 0] : 0.0f;
#pragma unroll
            for (int j = 0; j < NX; ++j) acc[m][j][r] = v;
        }
}

// Stores NM x NX tiles.
template <class T, int NM, int NX>
__device__ __forceinline__ void finish(const LoraDev& d, int f0, int r0, int lane, f32x16 (&acc)[NM][NX]) {
    const int half = lane >> 5;
#pragma unroll
    for (int m = 0; m < NM; ++m) {
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
// parts of 64 columns, of which STAGES - 1 are on their way during the products of the current one. Bound by the
// matrix units and the LDS reads that feed them: 32768x2048x2048, rank 64, 289 to 298 us (950 to 920 TFLOP/s,
// 1415 for a large library product).
template <class T, int WF, int WR, int NM, int NX, int STAGES, int WIDTH>
__global__ __launch_bounds__(64 * WF * WR, 2) void k_lora_tile(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    constexpr int TF = WF * NM * 32, TR = WR * NX * 32, THREADS = 64 * WF * WR;
    static_assert(direct(WIDTH) || STAGES == 2, "registers hold one part");
    __shared__ __align__(16) T tiles[STAGES][(TF + TR) * 64];
    const int f_tiles = (d.out + TF - 1) / TF;
    const int id = xcd_order(blockIdx.x, gridDim.x);
    const int f0 = (id % f_tiles) * TF, r0 = (id / f_tiles) * TR;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in, parts = (K + 63) / 64;
    const T* wp = static_cast<const T*>(d.w) + (int64_t)f0 * d.w_stride;
    const T* xp = static_cast<const T*>(d.x) + (int64_t)r0 * d.x_stride;
    Stage<T, TF, THREADS, WIDTH> sw(d.w_stride, d.out - f0, K);
    Stage<T, TR, THREADS, WIDTH> sx(d.x_stride, d.rows - r0, K);
    constexpr int LOADS = (TF + TR) * 8 / THREADS;       // a thread's loads of one part
    auto load = [&](int i, int p) {
        sw.load(wp, d.w_stride, i * 64, tiles[p]);
        sx.load(xp, d.x_stride, i * 64, tiles[p] + TF * 64);
    };
    auto arrive = [&](int i, int p) {
        sw.arrive(tiles[p], i == parts - 1);
        sx.arrive(tiles[p] + TF * 64, i == parts - 1);
    };
    f32x16 acc[NM][NX];
    const int fw = (w % WF) * NM * 32, rw = (w / WF) * NX * 32;
    auto multiply = [&](int p) {
        const T* wt = tiles[p];
        const T* xt = tiles[p] + TF * 64;
        // The operands of the next 16 columns are read while those of the current ones are multiplied.
        v8 a[2][NM], b[2][NX];
        auto read = [&](int ks) {
#pragma unroll
            for (int m = 0; m < NM; ++m) a[ks & 1][m] = read_rows<T, 64>(wt, fw + m * 32 + (lane & 31), ks, half);
#pragma unroll
            for (int j = 0; j < NX; ++j) b[ks & 1][j] = read_rows<T, 64>(xt, rw + j * 32 + (lane & 31), ks, half);
        };
        read(0);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            if (ks < 3) read(ks + 1);
#pragma unroll
            for (int m = 0; m < NM; ++m)
#pragma unroll
                for (int j = 0; j < NX; ++j) acc[m][j] = mma(a[ks & 1][m], b[ks & 1][j], acc[m][j]);
            if (ks < 3) {
#pragma unroll
                for (int g = 0; g < NM + NX; ++g) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);                      // one LDS read
                    __builtin_amdgcn_sched_group_barrier(0x008, NM * NX / (NM + NX), 0);     // some products
                }
            }
        }
    };
    int first = 0;
    if constexpr (direct(WIDTH)) {
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (i < parts) load(i, i);
        start<T, NM, NX>(d, f0 + fw, lane, acc);
        if (d.adapters > 0) first = request_from(d, r0 + rw);
        if (parts >= STAGES - 1) wait_loads<(STAGES - 2) * LOADS>();
        else wait_loads();
        arrive(0, 0);
        lds_barrier();
        int p = 0;
        for (int i = 0; i < parts; ++i) {
            int q = p + STAGES - 1;
            if (q >= STAGES) q -= STAGES;
            if (i + STAGES - 1 < parts) load(i + STAGES - 1, q);
            multiply(p);
            if (i + 1 < parts) {
                if (i + STAGES - 1 < parts) wait_loads<(STAGES - 2) * LOADS>();      // the next part is there
                else wait_loads();
                arrive(i + 1, p + 1 == STAGES ? 0 : p + 1);
            }
            lds_barrier();
            if (++p == STAGES) p = 0;
        }
    } else {
        // Registers: part i + 2 is on its way in one set while part i + 1 waits in the other.
        sw.template load<0>(wp, d.w_stride, 0, nullptr);
        sx.template load<0>(xp, d.x_stride, 0, nullptr);
        if (parts > 1) {
            sw.template load<1>(wp, d.w_stride, 64, nullptr);
            sx.template load<1>(xp, d.x_stride, 64, nullptr);
        }
        start<T, NM, NX>(d, f0 + fw, lane, acc);
        if (d.adapters > 0) first = request_from(d, r0 + rw);
        sw.template arrive<0>(tiles[0], parts == 1);
        sx.template arrive<0>(tiles[0] + TF * 64, parts == 1);
        __syncthreads();
        auto step = [&](int i, auto set) {
            constexpr int A = decltype(set)::value, B = 1 - A;
            if (i + 2 < parts) {
                sw.template load<A>(wp, d.w_stride, (i + 2) * 64, nullptr);
                sx.template load<A>(xp, d.x_stride, (i + 2) * 64, nullptr);
            }
            multiply(A);
            if (i + 1 < parts) {
                sw.template arrive<B>(tiles[B], i + 1 == parts - 1);
                sx.template arrive<B>(tiles[B] + TF * 64, i + 1 == parts - 1);
            }
            lds_barrier();
        };
        for (int i = 0; i < parts; i += 2) {
            step(i, std::integral_constant<int, 0>{});
            if (i + 1 < parts) step(i + 1, std::integral_constant<int, 1>{});
        }
    }
    if (d.adapters > 0) add_adapters<T, NM, NX, WIDTH>(d, f0 + fw, r0 + rw, lane, acc, first);
    finish<T, NM, NX>(d, f0 + fw, r0 + rw, lane, acc);
}

// Few rows: 32 features x 32 rows per block. W is read once, straight into operand registers; 16 waves
// take parts of 64 columns in turn, and the requests' adapters in turn, and are joined through LDS. Bound by
// latency: eight rows of 1024x1024 7 us (2.1 MB).
template <class T, int WIDTH>
__global__ __launch_bounds__(1024) void k_lora_rows(LoraDev d) {
    typedef typename Vec<T>::v8 v8;
    __shared__ float part[16][16][64];
    const int f0 = blockIdx.x * 32, r0 = blockIdx.y * 32;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int K = d.in, f = f0 + (lane & 31), row = r0 + (lane & 31);
    const T* wp = static_cast<const T*>(d.w) + (int64_t)(f < d.out ? f : 0) * d.w_stride;
    const T* xp = static_cast<const T*>(d.x) + (int64_t)(row < d.rows ? row : 0) * d.x_stride;
    const int first = d.adapters > 0 ? request_from(d, r0) : 0;
    f32x16 acc[1][1] = {{f32x16{}}};
    if (w == 0) start<T, 1, 1>(d, f0, lane, acc);
    for (int k0 = w * 64; k0 < K; k0 += 1024) {
        v8 wv[4], xv[4];
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int k = k0 + ks * 16 + half * 8;
            wv[ks] = operand<T, WIDTH>(wp, k, K, f < d.out);
            xv[ks] = operand<T, WIDTH>(xp, k, K, row < d.rows);
        }
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int k = k0 + ks * 16 + half * 8;
            acc[0][0] = mma(fixed<T, WIDTH>(wv[ks], k, K, f < d.out), fixed<T, WIDTH>(xv[ks], k, K, row < d.rows), acc[0][0]);
        }
    }
    if (d.adapters > 0) add_adapters<T, 1, 1, WIDTH>(d, f0, r0, lane, acc, first + w, 16);
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

// The kernels that read operands straight from memory take even rows as ragged ones.
constexpr int in_place(int width) { return width == kEven ? kRagged : width; }

template <class T, int NR, int WIDTH>
void down(const LoraDev& d, hipStream_t st) {
    // Blocks per request: its share of the rows, so that the launch has about rows / 64 (or 32) of them.
    // Where those of 64 rows are fewer than the CUs, or requests shorter, latency counts (1999 rows: 42 us in
    // blocks of 64 rows, 14 in blocks of 32; 8192: 11.8 and 11.6; 32768: 32 and 77). A request far above the average
    // keeps its share of the blocks: 48 requests, one with 8098 of 8192 rows, take 216 us in place of 36.
    const bool few = d.rows < 64 * kCUs || d.rows < 64 * d.requests;
    const int per = d.rows / (few ? 32 : 64) / d.requests + 1;
    const dim3 grid((unsigned)(per < 4096 ? per : 4096), (unsigned)d.requests);
    if (few) k_lora_down_few<T, NR, in_place(WIDTH)><<<grid, 1024 / NR, 0, st>>>(d);
    else k_lora_down<T, NR, WIDTH><<<grid, 256, 0, st>>>(d);
}

int64_t tiles_of(const LoraDev& d, int f, int r) { return (int64_t)((d.out + f - 1) / f) * ((d.rows + r - 1) / r); }

// 256 x 256 tiles (features x rows) where they give every CU a block; 64 x 64 ones where they are few enough
// for one round of two blocks a CU, or, loaded through registers (where 128 x 128 ones keep too few loads
// in flight), as long as 128 x 128 ones would not give every CU a block; 128 x 128 ones otherwise. Up to
// 64 rows W is read straight from memory. Both sides of each rule, with the adapters' first product, in us (taken
// before the requests of a tile were kept apart, which costs 0 to 1 us on these sizes):
//   32768x2048x2048, rank 64: 256 x 256 tiles 320, 128 x 128 ones 362
//   8192x1024x1024, rank 16:  128 x 128 tiles 33.3, 256 x 128 ones of eight waves (not built) 34.4
//   2048x1024x1024, rank 16:  64 x 64 tiles (512) 17.4, 128 x 128 ones 21.5
//   1999x1024x1347, rank 24:  128 x 128 tiles 25.4, 64 x 64 ones (704) 30.1
//   1999x1101x1347, rank 24:  64 x 64 tiles 44, 128 x 128 ones (176) 54; 8192x1101x1024: 75 and 56
//   8x1024x1024, rank 16, in a graph:  straight from memory 9.5, 64 x 64 tiles 15.2; 64 rows: 10.6 and 14.4
template <class T, int WIDTH>
hipError_t run(const LoraDev& d, hipStream_t st) {
    if (d.adapters > 0) {
        if (d.rank <= 32)      down<T, 1, WIDTH>(d, st);
        else if (d.rank <= 64) down<T, 2, WIDTH>(d, st);
        else                   down<T, 4, WIDTH>(d, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.rows <= 64) {
        k_lora_rows<T, in_place(WIDTH)><<<dim3((unsigned)((d.out + 31) / 32), (unsigned)((d.rows + 31) / 32)), 1024, 0, st>>>(d);
        return hipGetLastError();
    }
    if constexpr (direct(WIDTH)) {
        if (tiles_of(d, 256, 256) >= kCUs) {
            k_lora_tile<T, 2, 4, 4, 2, 2, WIDTH><<<(unsigned)tiles_of(d, 256, 256), 512, 0, st>>>(d);
            return hipGetLastError();
        }
    }
    if (direct(WIDTH) ? tiles_of(d, 64, 64) > 2 * kCUs : tiles_of(d, 128, 128) >= kCUs)
        k_lora_tile<T, 2, 2, 2, 2, 2, WIDTH><<<(unsigned)tiles_of(d, 128, 128), 256, 0, st>>>(d);
    else
        k_lora_tile<T, 2, 2, 1, 1, direct(WIDTH) ? 4 : 2, WIDTH><<<(unsigned)tiles_of(d, 64, 64), 256, 0, st>>>(d);
    return hipGetLastError();
}

}  // namespace

hipError_t lora_linear(const LoraDev& d, int dtype, hipStream_t st) {
    const int64_t odd = (int64_t)d.in | d.x_stride | d.w_stride;
    const uintptr_t at = reinterpret_cast<uintptr_t>(d.x) | reinterpret_cast<uintptr_t>(d.w) | reinterpret_cast<uintptr_t>(d.a);
    const bool near = d.x_stride < kBufferStride && d.w_stride < kBufferStride && at % 4 == 0 && odd % 2 == 0 && d.rank % 8 == 0;
    auto typed = [&](auto t) {
        typedef decltype(t) T;
        if (d.in < 8) return run<T, kTiny>(d, st);
        return !near ? run<T, kRagged>(d, st) : d.in % 8 != 0 ? run<T, kEven>(d, st) : run<T, kWhole>(d, st);
    };
    return dtype == PA_BF16 ? typed((__bf16)0) : typed((_Float16)0);
}

}  // namespace pa
