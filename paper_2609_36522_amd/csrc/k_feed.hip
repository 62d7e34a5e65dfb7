// A gated feed-forward block, forward and backward, for gfx950: h = act(x G^T + bg) (x U^T + bu),
// y = h D^T + bd.
//
// Forward, two launches. A block of the first takes as many features of G as of U, so that a wave has both
// projections of a value in the same lane, and stores h (and, for the backward pass, by what dh gives the gradients by the
// projections). Backward: dh = dy D with these factors in its epilogue (dz by the gate's projection, du by the other's);
// dx = dz G + du U as one reduction over both; the weights' gradients dz^T x, du^T x and dy^T h, reductions
// over the rows, in one launch, which also sums dz, du and dy over the rows (the biases' gradients) from the
// operands that pass by.
#include <type_traits>

#include "pa_act.h"
#include "pa_gemm.h"

namespace pa {

namespace {

template <class T> constexpr bool kScaled = std::is_same_v<T, _Float16>;

// fp16: the power of two that brings the largest |dy| to 1/16 .. 1/8 (1 where that is zero or no finite number): dz and du
// may grow to 2^19 times dy before they overflow, and lose digits (2^-25 of absolute error) only below 2^-10 of it.
template <class T>
__device__ __forceinline__ float gradient_scale(const float* largest) {
    if constexpr (!kScaled<T>) return 1.0f;
    const f32x4 v = *reinterpret_cast<const f32x4*>(largest + (threadIdx.x & 63) * 4);
    float m = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
    const int e = (int)(__builtin_bit_cast(uint32_t, m) >> 23);
    return e == 0 || e == 255 ? 1.0f : __builtin_bit_cast(float, (uint32_t)(250 - e) << 23);
}

// Partial maxima of |dy|; a NaN among them stays out (it is in every gradient anyway).
template <class T>
__global__ __launch_bounds__(256) void k_feed_largest(FeedDev d) {
    __shared__ float red[4];
    float m = 0.0f;
    const int pieces = (d.out + 7) / 8;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)d.rows * pieces; i += 256 * kLargest) {
        const int64_t row = i / pieces;
        const Pack8<T> p = load8(static_cast<const T*>(d.dy) + row * d.y_stride, (int)(i - row * pieces) * 8, d.out);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf((float)p.v[e]));
    }
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) m = fmaxf(m, __shfl_xor(m, i));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) d.largest[blockIdx.x] = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
}

// Copies of matrices in whole pieces of 16 bytes, zeros past a row's end, so that tiles are loaded straight into LDS. Bound by
// memory: x and the weights of 1999x1100x2731 in fp16 (22 MB), each way, 10 us.
struct CopyDev {
    const void* from[5];
    void* to[5];
    int64_t stride[5], first[6];     // first: block of a matrix's first pieces
    int rows[5], cols[5];
};

template <class T>
__global__ __launch_bounds__(256) void k_feed_copy(CopyDev d, int64_t block0) {
    const int64_t block = block0 + blockIdx.x;
    int i = 0;
    while (block >= d.first[i + 1]) ++i;
    const int pieces = (d.cols[i] + 7) / 8;
    const int64_t at = (block - d.first[i]) * 256 + threadIdx.x, row = at / pieces;
    if (row >= d.rows[i]) return;
    reinterpret_cast<Pack8<T>*>(d.to[i])[at] =
        load8(static_cast<const T*>(d.from[i]) + row * d.stride[i], (int)(at - row * pieces) * 8, d.cols[i]);
}

// Eight values from accumulator registers, zeros from feature `n` on, stored where the row exists.
template <class T>
__device__ __forceinline__ void store_padded(T* at, Pack8<T> p, int n) {
    if (n < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= n) p.v[e] = (T)0.0f;
    }
    *reinterpret_cast<Pack8<T>*>(at) = p;
}

// The factors kept for the backward pass are numbers of 24 bits, the upper three bytes of fp32's four (cut: 2^-15 at most), so
// that a gradient is rounded to the element type where it is an operand and where it is a result, and nowhere else. (With factors
// of the element type the gradients were off by 1.73 times the rounding of a result, so by 1.41; and fp16's range ended theirs.)
// Their upper halves are matrices of their own; a third one has the last byte of both.
__device__ __forceinline__ uint32_t bits(float v) { return __builtin_bit_cast(uint32_t, v); }
__device__ __forceinline__ uint32_t last_bytes(float z, float u) { return (bits(z) >> 8 & 0xffu) | (bits(u) & 0xff00u); }
__device__ __forceinline__ float by_z_of(uint32_t upper, uint32_t last) { return __builtin_bit_cast(float, upper << 16 | (last & 0xffu) << 8); }
__device__ __forceinline__ float by_u_of(uint32_t upper, uint32_t last) { return __builtin_bit_cast(float, upper << 16 | (last & 0xff00u)); }

// Words of 16 bits, word(i) of accumulator register 8 j + i, to the places of gather8.
template <class F>
__device__ __forceinline__ uint4 gather_words(F word) {
    uint32_t w[2][2];
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int p = 0; p < 2; ++p) w[q][p] = word(4 * q + 2 * p) | word(4 * q + 2 * p + 1) << 16;
    return rows8(w);
}

template <class X>
__device__ __forceinline__ void clear(typename X::acc_t (&acc)[X::NM][X::NX], float (&sums)[X::NX]) {
#pragma unroll
    for (int m = 0; m < X::NM; ++m)
#pragma unroll
        for (int j = 0; j < X::NX; ++j) acc[m][j] = typename X::acc_t{};
#pragma unroll
    for (int j = 0; j < X::NX; ++j) sums[j] = 0.0f;
}

// Adds a value for each feature to tiles m0 .. m0 + N - 1.
template <int N, int NM, int NX>
__device__ __forceinline__ void add(const float* per_feature, int half, f32x16 (&acc)[NM][NX], int m0) {
#pragma unroll
    for (int m = 0; m < N; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const f32x4 v = PerFeature<N>::at(per_feature, m, q, half);
#pragma unroll
            for (int j = 0; j < NX; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m0 + m][j][4 * q + i] += v[i];
        }
}

// ------------------------------------------------------------------ forward
// Both projections of a tile of rows, which read x once for the two; the activation and the product are formed in the
// registers that hold them. Bound by the matrix units (the clock falls to 1.64 GHz under them, 77% busy) at long
// reductions, by what follows the products at short ones: 32768x2048x8192 1720 us (1280 TFLOP/s; the library's product of this
// size alone 1555), 8192x1024x4096 126 to 141 (1090 to 970), 156 to 174 where the factors of the backward pass are formed and kept.
template <class X, int ACT>
__global__ __launch_bounds__(X::THREADS, X::WAVES) void k_feed_gate(FeedDev d, GemmJob job) {
    typedef typename X::T T;
    __shared__ __align__(16) char lds[X::BYTES];
    f32x16 acc[X::NM][X::NX];
    float sums[X::NX];
    clear<X>(acc, sums);
    int f, r;
    tile_of(job, xcd_order(blockIdx.x, gridDim.x), f, r);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    constexpr int HM = X::NM / 2;
    const int f0 = f * X::OUT + (w % X::WF) * HM * 32, r0 = r * X::TR + (w / X::WF) * X::NX * 32;
    const PerFeature<HM> bg(static_cast<const T*>(d.gate_bias), f0, d.hidden, lane), bu(static_cast<const T*>(d.up_bias), f0, d.hidden, lane);
    X::run(job, f * X::OUT, r * X::TR, 0, (job.len + X::PART - 1) / X::PART, lds, acc, sums);
    char* own = lds + w * HM * 2048;
    if (d.gate_bias || d.up_bias) {
        float* per = reinterpret_cast<float*>(lds + X::THREADS / 64 * HM * 2048 + w * 512);
        bg.put(per, lane);
        bu.put(per + 64, lane);
        add<HM>(per, half, acc, 0);
        add<HM>(per + 64, half, acc, HM);
    }
#pragma unroll
    for (int j = 0; j < X::NX; ++j) {
        auto store = [&](void* to, auto value) {
            through_lds<uint16_t, HM>(own, lane, value, [&](int row, int at, const Pack8<uint16_t>& v) {
                if (r0 + j * 32 + row < d.rows && f0 + at < d.hidden_pad)
                    store_padded(static_cast<uint16_t*>(to) + (int64_t)(r0 + j * 32 + row) * d.hidden_pad + f0 + at, v, d.hidden - f0 - at);
            });
        };
        if (d.by_z) {
            uint4 by_z[HM][2], last[HM][2];
#pragma unroll
            for (int m = 0; m < HM; ++m) {
                f32x16 v;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 a = activate_grad<ACT>(acc[m][j][i]);
                    v[i] = a.y * acc[m + HM][j][i];
                    acc[m][j][i] = a.x;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    by_z[m][q] = gather_words([&](int i) { return bits(v[8 * q + i]) >> 16; });
                    last[m][q] = gather_words([&](int i) { return last_bytes(v[8 * q + i], acc[m][j][8 * q + i]); });
                }
            }
            store(d.by_z, [&](int m, int q) { return by_z[m][q]; });
            store(d.last, [&](int m, int q) { return last[m][q]; });
            store(d.by_u, [&](int m, int q) { return gather_words([&](int i) { return bits(acc[m][j][8 * q + i]) >> 16; }); });
        } else {
#pragma unroll
            for (int m = 0; m < HM; ++m)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[m][j][i] = activate<ACT>(acc[m][j][i]);
        }
#pragma unroll
        for (int m = 0; m < HM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][j][i] *= acc[m + HM][j][i];
        store(d.h, [&](int m, int q) { return gather8<T>(acc[m][j], q, 1.0f); });
    }
}

// out = R F^T + bias, or its partial sums over ranges of the reduction: [split][rows][feature_pad] in `part`: the projection
// back, and dx. Bound as k_feed_gate is: 32768x8192 to 2048 900 us (1220 TFLOP/s), 8192x4096 to 1024 66 (1040; the library 60),
// dx of 8192x1024x4096, over both projections, 127 to 144 (the library's product of this size 144).
struct PlainDev {
    const void* bias;
    void* out;
    int64_t out_stride;
    float* part;
    const float* largest;            // not null: divided by its scale
    int splits, feature_pad;
};

template <class X>
__global__ __launch_bounds__(X::THREADS, X::WAVES) void k_feed_plain(PlainDev d, GemmJob job) {
    typedef typename X::T T;
    __shared__ __align__(16) char lds[X::BYTES];
    f32x16 acc[X::NM][X::NX];
    float sums[X::NX];
    clear<X>(acc, sums);
    const int tiles = job.f_tiles * job.r_tiles, id = xcd_order(blockIdx.x, gridDim.x), split = id / tiles;
    int f, r;
    tile_of(job, id - split * tiles, f, r);
    const int parts = (job.len + X::PART - 1) / X::PART * (job.f[1] ? 2 : 1);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int f0 = f * X::TF + (w % X::WF) * X::NM * 32, r0 = r * X::TR + (w / X::WF) * X::NX * 32;
    const PerFeature<X::NM> bias(static_cast<const T*>(d.bias), f0, job.features, lane);
    X::run(job, f * X::TF, r * X::TR, (int)((int64_t)parts * split / d.splits), (int)((int64_t)parts * (split + 1) / d.splits), lds, acc, sums);
    if (d.splits == 1) {
        const float s = d.largest ? 1.0f / gradient_scale<T>(d.largest) : 1.0f;
        if (d.bias) {
            float* per = reinterpret_cast<float*>(lds + X::THREADS / 64 * X::NM * 2048 + w * 512);
            bias.put(per, lane);
            add<X::NM>(per, half, acc, 0);
        }
#pragma unroll
        for (int j = 0; j < X::NX; ++j)
            through_lds<T, X::NM>(lds + w * X::NM * 2048, lane, [&](int m, int q) { return gather8<T>(acc[m][j], q, s); },
                                  [&](int row, int at, const Pack8<T>& v) {
                                      if (r0 + j * 32 + row < job.rows)
                                          store8(static_cast<T*>(d.out) + (int64_t)(r0 + j * 32 + row) * d.out_stride + f0 + at, v, job.features - f0 - at);
                                  });
    } else {
#pragma unroll
        for (int m = 0; m < X::NM; ++m)
#pragma unroll
            for (int j = 0; j < X::NX; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int at = f0 + m * 32 + q * 8 + half * 4, row = r0 + j * 32 + (lane & 31);
                    const f32x4 v = {acc[m][j][4 * q], acc[m][j][4 * q + 1], acc[m][j][4 * q + 2], acc[m][j][4 * q + 3]};
                    if (row < job.rows && at < d.feature_pad)
                        *reinterpret_cast<f32x4*>(d.part + ((int64_t)split * job.rows + row) * d.feature_pad + at) = v;
                }
    }
}

// Partial sums joined in order, eight features a thread.
template <class T>
__global__ __launch_bounds__(256) void k_feed_join(PlainDev d, int rows, int features) {
    const int pieces = d.feature_pad / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / pieces;
    const int at = (int)(i - row * pieces) * 8;
    if (row >= rows) return;
    float v[8] = {};
#pragma unroll 4
    for (int s = 0; s < d.splits; ++s) {
        const float* p = d.part + ((int64_t)s * rows + row) * d.feature_pad + at;
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] += a[e];
            v[4 + e] += b[e];
        }
    }
    const float s = d.largest ? 1.0f / gradient_scale<T>(d.largest) : 1.0f;
    Pack8<T> o;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        o.v[e] = (T)(v[e] * s + (d.bias && at + e < features ? (float)static_cast<const T*>(d.bias)[at + e] : 0.0f));
    store8(static_cast<T*>(d.out) + row * d.out_stride + at, o, features - at);
}

// ------------------------------------------------------------------ few rows
// 16 features a block, up to 16 NR rows: the weights are read once, straight into operand registers; 16
// waves take pieces of 32 U elements of the reduction in turn and are joined through LDS in a fixed order. Bound by the
// latency of a launch and one round of loads: one row of 1024x4096 5.3 to 5.8 us for 16.8 MB and 5.1 to 5.7 for 8.4 MB.
template <class T, int U, int NR, int NW, int WIDTH>
__device__ __forceinline__ void few_rows(const T* const (&wp)[NW], bool f_valid, const T* x, int64_t x_stride, int rows, int len,
                                         float (*part)[NW][NR][4][64], f32x4 (&out)[NW]) {
    typedef typename Vec<T>::v8 v8;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    f32x4 acc[NW][NR];
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int j = 0; j < NR; ++j) acc[n][j] = f32x4{};
    for (int k0 = w * 32 * U; k0 < len; k0 += 16 * 32 * U) {
        v8 wv[NW][U], xv[NR][U];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int k = k0 + s * 32 + (lane >> 4) * 8;
#pragma unroll
            for (int n = 0; n < NW; ++n) wv[n][s] = operand<T, WIDTH>(wp[n], k, len, f_valid);
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const int row = j * 16 + (lane & 15);
                xv[j][s] = operand<T, WIDTH>(x + (row < rows ? row : 0) * x_stride, k, len, row < rows);
            }
        }
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int k = k0 + s * 32 + (lane >> 4) * 8;
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const v8 b = fixed<T, WIDTH>(xv[j][s], k, len, j * 16 + (lane & 15) < rows);
#pragma unroll
                for (int n = 0; n < NW; ++n) acc[n][j] = mma16(fixed<T, WIDTH>(wv[n][s], k, len, f_valid), b, acc[n][j]);
            }
        }
    }
#pragma unroll
    for (int n = 0; n < NW; ++n)
#pragma unroll
        for (int j = 0; j < NR; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[w][n][j][r][lane] = acc[n][j][r];
    __syncthreads();
    // Wave w < 4 NR sums register w % 4 of row group w / 4.
#pragma unroll
    for (int n = 0; n < NW; ++n) out[n] = f32x4{};
    if (w < 4 * NR) {
#pragma unroll
        for (int n = 0; n < NW; ++n) {
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < 16; ++i) v += part[i][n][w >> 2][w & 3][lane];
            out[n][0] = v;
        }
    }
}

template <class T, int ACT, int NR, int WIDTH>
__global__ __launch_bounds__(1024) void k_feed_few_gate(FeedDev d) {
    __shared__ float part[16][2][NR][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, f0 = blockIdx.x * 16, f = f0 + (lane & 15);
    const bool valid = f < d.hidden;
    const T* const wp[2] = {static_cast<const T*>(d.gate) + (valid ? f : 0) * d.gate_stride, static_cast<const T*>(d.up) + (valid ? f : 0) * d.up_stride};
    f32x4 v[2];
    few_rows<T, 2, NR, 2, WIDTH>(wp, valid, static_cast<const T*>(d.x), d.x_stride, d.rows, d.in, part, v);
    const int row = (w >> 2) * 16 + (lane & 15), o = f0 + 4 * (lane >> 4) + (w & 3);
    if (w >= 4 * NR || row >= d.rows || o >= d.hidden_pad) return;
    const bool in = o < d.hidden;
    const float g = v[0][0] + (in && d.gate_bias ? (float)static_cast<const T*>(d.gate_bias)[o] : 0.0f);
    const float u = v[1][0] + (in && d.up_bias ? (float)static_cast<const T*>(d.up_bias)[o] : 0.0f);
    const int64_t to = (int64_t)row * d.hidden_pad + o;
    const float2 a = activate_grad<ACT>(g);
    static_cast<T*>(d.h)[to] = (T)(in ? a.x * u : 0.0f);
    if (d.by_z) {
        const float z = in ? a.y * u : 0.0f, value = in ? a.x : 0.0f;
        d.by_z[to] = (uint16_t)(bits(z) >> 16);
        d.by_u[to] = (uint16_t)(bits(value) >> 16);
        d.last[to] = (uint16_t)last_bytes(z, value);
    }
}

// FEATURES (16 or 8) a block: 8 leave half of the matrix unit's rows empty and take half of the weights a block.
template <class T, int NR, int WIDTH, int FEATURES>
__global__ __launch_bounds__(1024) void k_feed_few_down(FeedDev d) {
    __shared__ float part[16][1][NR][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, f0 = blockIdx.x * FEATURES, f = f0 + (lane & 15);
    const bool valid = f < d.out && (lane & 15) < FEATURES;
    const T* const wp[1] = {static_cast<const T*>(d.down) + (valid ? f : f0) * d.down_stride};
    f32x4 v[1];
    few_rows<T, NR == 1 ? 8 : 4, NR, 1, WIDTH>(wp, valid, static_cast<const T*>(d.h), d.hidden_pad, d.rows, d.hidden, part, v);
    const int row = (w >> 2) * 16 + (lane & 15), in = 4 * (lane >> 4) + (w & 3), o = f0 + in;
    if (w >= 4 * NR || row >= d.rows || in >= FEATURES || o >= d.out) return;
    static_cast<T*>(d.y)[(int64_t)row * d.y_stride + o] = (T)(v[0][0] + (d.down_bias ? (float)static_cast<const T*>(d.down_bias)[o] : 0.0f));
}

// ------------------------------------------------------------------ backward
// dh = dy D, then dz = dh (u act'(g)) and du = dh act(g) by the factors that the forward pass kept. (With g and u kept in their
// place the activation took 28 us more here.) Bound by what follows the products, which reads and writes as much as it:
// 8192x1024x4096 120 to 131 us, of which the product alone is 73 and 336 MB at the copy rate are 69. With factors of 16 bits, 67 MB
// less, 103 to 108.
template <class X>
__global__ __launch_bounds__(X::THREADS, X::WAVES) void k_feed_grad(FeedDev d, GemmJob job) {
    typedef typename X::T T;
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    __shared__ __align__(16) char lds[X::BYTES];
    f32x16 acc[X::NM][X::NX];
    float sums[X::NX];
    clear<X>(acc, sums);
    int f, r;
    tile_of(job, xcd_order(blockIdx.x, gridDim.x), f, r);
    const float scale = gradient_scale<T>(d.largest);
    X::run(job, f * X::TF, r * X::TR, 0, (job.len + X::PART - 1) / X::PART, lds, acc, sums);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int f0 = f * X::TF + (w % X::WF) * X::NM * 32, r0 = r * X::TR + (w / X::WF) * X::NX * 32;
    constexpr int CM = X::NM < 2 ? 1 : 2, P = CM * 4;        // 64 features at a time: 128 bytes of a row
    char* own = lds + w * CM * 2048;
#pragma unroll
    for (int j = 0; j < X::NX; ++j) {
#pragma unroll
        for (int c = 0; c < X::NM; c += CM) {
            // Both factors, in the order in which they lie, then through LDS to the lanes that hold their places.
            const int fc = f0 + c * 32;
            uint4 by[3][P / 2];
#pragma unroll
            for (int i = 0; i < P / 2; ++i) {
                const int at = i * 64 + lane, row = r0 + j * 32 + at / P, col = fc + at % P * 8;
                by[0][i] = by[1][i] = by[2][i] = make_uint4(0, 0, 0, 0);
                if (row < d.rows && col < d.hidden_pad) {
                    const int64_t from = (int64_t)row * d.hidden_pad + col;
                    by[0][i] = *reinterpret_cast<const uint4*>(d.by_z + from);
                    by[1][i] = *reinterpret_cast<const uint4*>(d.by_u + from);
                    by[2][i] = *reinterpret_cast<const uint4*>(d.last + from);
                }
            }
            u16x4 last[CM][4];
            from_lds<CM>(own, lane, by[2], last);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                u16x4 p[CM][4];
                from_lds<CM>(own, lane, by[n], p);
                f32x16 v[CM];
#pragma unroll
                for (int m = 0; m < CM; ++m)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t upper = p[m][i >> 2][i & 3], low = last[m][i >> 2][i & 3];
                        v[m][i] = acc[c + m][j][i] * scale * (n ? by_u_of(upper, low) : by_z_of(upper, low));
                    }
                T* to = static_cast<T*>(n ? d.du : d.dz);
                through_lds<T, CM>(own, lane, [&](int m, int q) { return gather8<T>(v[m], q, 1.0f); }, [&](int row, int at, const Pack8<T>& o) {
                    if (r0 + j * 32 + row < d.rows && fc + at < d.hidden_pad)
                        store_padded(to + (int64_t)(r0 + j * 32 + row) * d.hidden_pad + fc + at, o, d.hidden - fc - at);
                });
            }
        }
    }
}

// The weights' gradients, up to three products in one launch (alone none fills the CUs); a split takes a range of the rows.
// Bound by the matrix units on the 192 CUs that have one of its tiles: 8192x1024x4096 203 to 255 us, 206 GFLOP.
struct WeightsDev {
    GemmJob job[3];
    void *out[3], *bias[3];          // [rows][features], [rows] (sums over the reduction of R; may be null)
    const float* largest[3];
    int64_t part[3];                 // splits > 1: offset of the job's partial sums, [split][rows][feature_pad + 1 piece for the bias]
    int first[4];
    int jobs, splits;
    float* parts;
};

__device__ __host__ __forceinline__ int padded(int n) { return (n + 7) / 8 * 8; }

template <class X>
__global__ __launch_bounds__(X::THREADS, X::WAVES) void k_feed_weights(WeightsDev d) {
    typedef typename X::T T;
    __shared__ __align__(16) char lds[X::BYTES];
    f32x16 acc[X::NM][X::NX];
    float sums[X::NX];
    clear<X>(acc, sums);
    const int total = d.first[d.jobs], id = xcd_order(blockIdx.x, gridDim.x), split = id / total, tile = id - split * total;
    int n = 0;
    while (n + 1 < d.jobs && tile >= d.first[n + 1]) ++n;
    const GemmJob& job = d.job[n];
    int f, r;
    tile_of(job, tile - d.first[n], f, r);
    const int parts = (job.len + X::PART - 1) / X::PART;
    X::run(job, f * X::TF, r * X::TR, (int)((int64_t)parts * split / d.splits), (int)((int64_t)parts * (split + 1) / d.splits), lds, acc, sums);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int f0 = f * X::TF + (w % X::WF) * X::NM * 32, r0 = r * X::TR + (w / X::WF) * X::NX * 32;
    const bool has_sums = d.bias[n] && f == 0 && w % X::WF == 0;
    if (d.splits == 1) {
        const float s = d.largest[n] ? 1.0f / gradient_scale<T>(d.largest[n]) : 1.0f;
#pragma unroll
        for (int j = 0; j < X::NX; ++j) {
            const int own = r0 + j * 32 + (lane & 31);
            const float sum = sums[j] + __shfl_xor(sums[j], 32);
            if (has_sums && half == 0 && own < job.rows) static_cast<T*>(d.bias[n])[own] = (T)(sum * s);
            through_lds<T, X::NM>(lds + w * X::NM * 2048, lane, [&](int m, int q) { return gather8<T>(acc[m][j], q, s); },
                                  [&](int row, int at, const Pack8<T>& v) {
                                      if (r0 + j * 32 + row < job.rows)
                                          store8(static_cast<T*>(d.out[n]) + (int64_t)(r0 + j * 32 + row) * job.features + f0 + at, v,
                                                 job.features - f0 - at);
                                  });
        }
    } else {
        const int pad = padded(job.features) + 8;
        float* out = d.parts + d.part[n] + (int64_t)split * job.rows * pad;
#pragma unroll
        for (int j = 0; j < X::NX; ++j) {
            const int row = r0 + j * 32 + (lane & 31);
            const float sum = sums[j] + __shfl_xor(sums[j], 32);
            if (has_sums && half == 0 && row < job.rows) out[(int64_t)row * pad + pad - 8] = sum;
#pragma unroll
            for (int m = 0; m < X::NM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int at = f0 + m * 32 + q * 8 + half * 4;
                    const f32x4 v = {acc[m][j][4 * q], acc[m][j][4 * q + 1], acc[m][j][4 * q + 2], acc[m][j][4 * q + 3]};
                    if (row < job.rows && at < pad - 8) *reinterpret_cast<f32x4*>(out + (int64_t)row * pad + at) = v;
                }
        }
    }
}

// Their partial sums joined in order, eight features a thread; a row's last piece holds its bias's.
template <class T>
__global__ __launch_bounds__(256) void k_feed_weights_join(WeightsDev d) {
    const int n = blockIdx.y;
    const int rows = d.job[n].rows, features = d.job[n].features, pad = padded(features) + 8, pieces = pad / 8;
    const float s = d.largest[n] ? 1.0f / gradient_scale<T>(d.largest[n]) : 1.0f;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < (int64_t)rows * pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / pieces;
        const int at = (int)(i - row * pieces) * 8;
        if (at == pad - 8) {
            if (!d.bias[n]) continue;
            float v = 0.0f;
            for (int k = 0; k < d.splits; ++k) v += d.parts[d.part[n] + ((int64_t)k * rows + row) * pad + at];
            static_cast<T*>(d.bias[n])[row] = (T)(v * s);
            continue;
        }
        float v[8] = {};
#pragma unroll 4
        for (int k = 0; k < d.splits; ++k) {
            const float* p = d.parts + d.part[n] + ((int64_t)k * rows + row) * pad + at;
            const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] += a[e];
                v[4 + e] += b[e];
            }
        }
        Pack8<T> o;
#pragma unroll
        for (int e = 0; e < 8; ++e) o.v[e] = (T)(v[e] * s);
        store8(static_cast<T*>(d.out[n]) + row * features + at, o, features - at);
    }
}

// No rows: the gradients of weights and biases are zero.
template <class T>
__global__ __launch_bounds__(256) void k_feed_zero(T* p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (T)0.0f;
}

// ------------------------------------------------------------------ launches
int64_t up_to(int64_t n, int64_t d) { return (n + d - 1) / d; }

#define FEED_TRY(call)                      \
    do {                                    \
        const hipError_t e_ = (call);       \
        if (e_ != hipSuccess) return e_;    \
    } while (0)

// What a product's partial sums cost to write, read and join, in us (two of 1999x1100: 7.5).
float join_time(int splits, int64_t values) { return splits < 2 ? 0.0f : 3.0f + (float)values * (float)(8 * splits + 2) / 9.0e6f; }

// The tiles that are expected to take the least time for jobs of features x rows, in `splits` ranges of the reduction each.
struct Choice {
    int kind;
    float time;
};
Choice choose(int cols, bool gated, int jobs, const int* features, const int* rows, int parts, int splits, const float* more = nullptr) {
    Choice best{kSmall, 0.0f};
    for (int k = 0; k < kTileKinds; ++k) {
        // Gated: half of a tile's features are the output's; the smallest has 64 x 128 places, and eight waves need 64 features each.
        if (gated && k == kTall) continue;
        const int f = kTileCost[k].f / (gated ? 2 : 1), r = gated && k == kSmall ? 128 : kTileCost[k].r;
        int64_t tiles = 0;
        for (int n = 0; n < jobs; ++n) tiles += up_to(features[n], f) * up_to(rows[n], r);
        float t = tile_time(k, cols, tiles * splits, (float)((parts + splits - 1) / splits), more ? more[k] : 0.0f);
        if (gated && k == kSmall) t *= 1.7f;
        if (k == 0 || t < best.time) best = {k, t};
    }
    return best;
}

// The number of ranges that makes up for its join, at most 8.
int choose_splits(int cols, int jobs, const int* features, const int* rows, int parts) {
    int best = 1;
    float least = choose(cols, false, jobs, features, rows, parts, 1).time;
    int64_t values = 0;
    for (int n = 0; n < jobs; ++n) values += (int64_t)rows[n] * padded(features[n]);
    for (int s = 2; s <= 8 && 4 * s <= parts; ++s) {
        const float t = choose(cols, false, jobs, features, rows, parts, s).time + join_time(s, values);
        if (t < least) {
            least = t;
            best = s;
        }
    }
    return best;
}

int parts_of(int len) { return (len + 63) / 64; }

template <class X>
void tiled(GemmJob& job) {
    job.f_tiles = (int)up_to(job.features, X::OUT);
    job.r_tiles = (int)up_to(job.rows, X::TR);
}

template <class T, int ACT>
hipError_t gate(const FeedDev& d, GemmJob job, hipStream_t st) {
    return with_tile<T, false, false, true, false>(choose(0, true, 1, &job.features, &job.rows, parts_of(job.len), 1).kind, [&](auto x) {
        typedef decltype(x) X;
        tiled<X>(job);
        k_feed_gate<X, ACT><<<(unsigned)((int64_t)job.f_tiles * job.r_tiles), X::THREADS, 0, st>>>(d, job);
        return hipGetLastError();
    });
}

template <class T, bool FCOL>
hipError_t plain(PlainDev p, GemmJob job, hipStream_t st) {
    const int parts = parts_of(job.len) * (job.f[1] ? 2 : 1);
    p.feature_pad = padded(job.features);
    FEED_TRY((with_tile<T, FCOL, false, false, false>(choose(FCOL, false, 1, &job.features, &job.rows, parts, p.splits).kind, [&](auto x) {
        typedef decltype(x) X;
        tiled<X>(job);
        k_feed_plain<X><<<(unsigned)((int64_t)job.f_tiles * job.r_tiles * p.splits), X::THREADS, 0, st>>>(p, job);
        return hipGetLastError();
    })));
    if (p.splits > 1) {
        k_feed_join<T><<<(unsigned)up_to((int64_t)job.rows * (p.feature_pad / 8), 256), 256, 0, st>>>(p, job.rows, job.features);
        return hipGetLastError();
    }
    return hipSuccess;
}

template <class T>
hipError_t grad(const FeedDev& d, GemmJob job, hipStream_t st) {
    // What follows the products reads three matrices besides and writes two. us with 256 x 256, 256 x 128, 128 x 192, 128 x 128 (two
    // stages), the same (three) and 64 x 64 tiles, and what the rule takes:
    //   8192x1024x4096 131 127 128 131 155 183, 131        2048x1024x4096        41 34 35 31 39 46, 34
    //   4096x1024x4096  59  62  68  65  74  88,  60        1999x1100x2731, fp16  43 29 32 31 40 42, 31
    constexpr float kMore[kTileKinds] = {20.0f, 12.0f, 10.0f, 7.0f, 7.0f, 3.0f};
    return with_tile<T, true, false, false, false>(choose(1, false, 1, &job.features, &job.rows, parts_of(job.len), 1, kMore).kind, [&](auto x) {
        typedef decltype(x) X;
        tiled<X>(job);
        k_feed_grad<X><<<(unsigned)((int64_t)job.f_tiles * job.r_tiles), X::THREADS, 0, st>>>(d, job);
        return hipGetLastError();
    });
}

template <class T>
hipError_t weights(WeightsDev w, hipStream_t st) {
    int features[3], rows[3];
    int64_t at = 0;
    for (int n = 0; n < w.jobs; ++n) {
        features[n] = w.job[n].features;
        rows[n] = w.job[n].rows;
        w.part[n] = at;
        at += (int64_t)w.splits * rows[n] * (padded(features[n]) + 8);
    }
    FEED_TRY((with_tile<T, true, true, false, true>(choose(2, false, w.jobs, features, rows, parts_of(w.job[0].len), w.splits).kind, [&](auto x) {
        typedef decltype(x) X;
        w.first[0] = 0;
        for (int n = 0; n < w.jobs; ++n) {
            tiled<X>(w.job[n]);
            w.first[n + 1] = w.first[n] + w.job[n].f_tiles * w.job[n].r_tiles;
        }
        k_feed_weights<X><<<(unsigned)(w.first[w.jobs] * w.splits), X::THREADS, 0, st>>>(w);
        return hipGetLastError();
    })));
    if (w.splits > 1) {
        k_feed_weights_join<T><<<dim3(1024, (unsigned)w.jobs), 256, 0, st>>>(w);
        return hipGetLastError();
    }
    return hipSuccess;
}

// Copies of what cannot be read in whole pieces; `use` becomes the copy with its stride.
struct Copies {
    CopyDev d{};
    int n = 0;
    const void* use(const void* from, void* pad, int64_t rows, int cols, int64_t& stride) {
        if (!pad) return from;
        d.from[n] = from;
        d.to[n] = pad;
        d.stride[n] = stride;
        d.rows[n] = (int)rows;
        d.cols[n] = cols;
        d.first[n + 1] = d.first[n] + up_to(rows * (padded(cols) / 8), 256);
        ++n;
        stride = padded(cols);
        return pad;
    }
    template <class T>
    hipError_t run(hipStream_t st) const {
        constexpr int64_t most = 1 << 23;            // a grid holds fewer than 2^32 threads
        for (int64_t b = 0; n > 0 && b < d.first[n]; b += most) {
            k_feed_copy<T><<<(unsigned)(d.first[n] - b < most ? d.first[n] - b : most), 256, 0, st>>>(d, b);
            FEED_TRY(hipGetLastError());
        }
        return hipSuccess;
    }
};

template <class T, int ACT, int WIDTH>
hipError_t forward_few(const FeedDev& d, hipStream_t st) {
    const unsigned hb = (unsigned)(d.hidden_pad + 15) / 16, ob = (unsigned)(d.out + 15) / 16;
    const bool thin = ob < kCUs / 2;         // fewer blocks than half of the CUs: 1x4096 to 1024 7.1 us in blocks of 16, 5.8 of 8
    auto go = [&](auto nr) {
        constexpr int NR = decltype(nr)::value;
        k_feed_few_gate<T, ACT, NR, WIDTH><<<hb, 1024, 0, st>>>(d);
        FEED_TRY(hipGetLastError());
        if (thin) k_feed_few_down<T, NR, WIDTH, 8><<<(unsigned)(d.out + 7) / 8, 1024, 0, st>>>(d);
        else k_feed_few_down<T, NR, WIDTH, 16><<<ob, 1024, 0, st>>>(d);
        return hipGetLastError();
    };
    if (d.rows <= 16) return go(std::integral_constant<int, 1>{});
    return go(std::integral_constant<int, 2>{});
}

template <class T, int ACT>
hipError_t forward(const FeedDev& d, hipStream_t st) {
    if (feed_few(d.rows)) {
        const int64_t odd = (int64_t)d.in | d.hidden | d.x_stride | d.gate_stride | d.up_stride | d.down_stride;
        const uintptr_t at = reinterpret_cast<uintptr_t>(d.x) | reinterpret_cast<uintptr_t>(d.gate) | reinterpret_cast<uintptr_t>(d.up) |
                             reinterpret_cast<uintptr_t>(d.down);
        if (d.in < 8 || d.hidden < 8) return forward_few<T, ACT, kTiny>(d, st);
        return odd % 8 == 0 && at % 16 == 0 ? forward_few<T, ACT, kWhole>(d, st) : forward_few<T, ACT, kRagged>(d, st);
    }
    Copies c;
    int64_t xs = d.x_stride, gs = d.gate_stride, us = d.up_stride, ds = d.down_stride;
    const void* x = c.use(d.x, d.x_pad, d.rows, d.in, xs);
    const void* g = c.use(d.gate, d.gate_pad, d.hidden, d.in, gs);
    const void* u = c.use(d.up, d.up_pad, d.hidden, d.in, us);
    const void* dn = c.use(d.down, d.down_pad, d.out, d.hidden, ds);
    FEED_TRY(c.run<T>(st));
    FEED_TRY((gate<T, ACT>(d, GemmJob{{g, u}, {x, nullptr}, gs, xs, d.hidden, d.rows, d.in, 0, 0}, st)));
    const PlainDev p{d.down_bias, d.y, d.y_stride, d.part, nullptr, d.down_splits, 0};
    return plain<T, false>(p, GemmJob{{dn, nullptr}, {d.h, nullptr}, ds, d.hidden_pad, d.out, d.rows, d.hidden, 0, 0}, st);
}

template <class T>
hipError_t zero(void* p, int64_t n, hipStream_t st) {
    if (!p) return hipSuccess;
    const int64_t blocks = up_to(n, 1024);
    k_feed_zero<T><<<(unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(static_cast<T*>(p), n);
    return hipGetLastError();
}

template <class T>
hipError_t backward(const FeedDev& d, hipStream_t st) {
    if (d.rows == 0) {
        const int64_t HK = (int64_t)d.hidden * d.in, NH = (int64_t)d.out * d.hidden;
        FEED_TRY(zero<T>(d.dgate, HK, st));
        FEED_TRY(zero<T>(d.dup, HK, st));
        FEED_TRY(zero<T>(d.ddown, NH, st));
        FEED_TRY(zero<T>(d.dgate_bias, d.hidden, st));
        FEED_TRY(zero<T>(d.dup_bias, d.hidden, st));
        return zero<T>(d.ddown_bias, d.out, st);
    }
    Copies c;
    int64_t xs = d.x_stride, gs = d.gate_stride, us = d.up_stride, ds = d.down_stride, ys = d.y_stride;
    const void* x = c.use(d.x, d.x_pad, d.rows, d.in, xs);
    const void* g = c.use(d.gate, d.gate_pad, d.hidden, d.in, gs);
    const void* u = c.use(d.up, d.up_pad, d.hidden, d.in, us);
    const void* dn = c.use(d.down, d.down_pad, d.out, d.hidden, ds);
    const void* dy = c.use(d.dy, d.dy_pad, d.rows, d.out, ys);
    FEED_TRY(c.run<T>(st));
    const bool through = d.dx || d.dgate || d.dup;
    if (through) {
        if (kScaled<T>) {
            k_feed_largest<T><<<kLargest, 256, 0, st>>>(d);
            FEED_TRY(hipGetLastError());
        }
        FEED_TRY((grad<T>(d, GemmJob{{dn, nullptr}, {dy, nullptr}, ds, ys, d.hidden, d.rows, d.out, 0, 0}, st)));
    }
    const float* largest = kScaled<T> ? d.largest : nullptr;
    if (d.dx) {
        const PlainDev p{nullptr, d.dx, d.in, d.part, largest, d.dx_splits, 0};
        FEED_TRY((plain<T, true>(p, GemmJob{{g, u}, {d.dz, d.du}, gs, d.hidden_pad, d.in, d.rows, d.hidden, 0, 0}, st)));
    }
    WeightsDev w{};
    auto add = [&](const void* f, int64_t fs, const void* r, int64_t rs, int rows, int features, void* out, void* bias, const float* l) {
        if (!out) return;
        w.job[w.jobs] = GemmJob{{f, nullptr}, {r, nullptr}, fs, rs, features, rows, d.rows, 0, 0};
        w.out[w.jobs] = out;
        w.bias[w.jobs] = bias;
        w.largest[w.jobs++] = l;
    };
    add(x, xs, d.dz, d.hidden_pad, d.hidden, d.in, d.dgate, d.dgate_bias, largest);
    add(x, xs, d.du, d.hidden_pad, d.hidden, d.in, d.dup, d.dup_bias, largest);
    add(d.h, d.hidden_pad, dy, ys, d.out, d.hidden, d.ddown, d.ddown_bias, nullptr);
    if (w.jobs == 0) return hipSuccess;
    w.splits = d.weight_splits;
    w.parts = d.part;
    return weights<T>(w, st);
}

template <class F>
hipError_t dispatch(int dtype, int act, F f) {
    auto typed = [&](auto t) {
        if (act == PA_ACT_SILU) return f(t, std::integral_constant<int, PA_ACT_SILU>{});
        if (act == PA_ACT_GELU) return f(t, std::integral_constant<int, PA_ACT_GELU>{});
        return f(t, std::integral_constant<int, PA_ACT_NONE>{});
    };
    return dtype == PA_BF16 ? typed((__bf16)0) : typed((_Float16)0);
}

}  // namespace

// us for 17, 32 and 64 rows of 1024x4096, the weights read once straight from memory and in tiles: 17.2 and 21.5, 21.0 and
// 20.9, 29.8 and 21.6; of 783x2539, where tiles need copies: 22.6 and 28.8 for 24, 34 and 29 for 64.
bool feed_few(int64_t rows) { return rows <= 32; }

size_t feed_plan(FeedDev& d, bool backward) {
    d.down_splits = d.dx_splits = d.weight_splits = 1;
    if (d.rows == 0 || (!backward && feed_few(d.rows))) return 0;
    if (!backward) {
        d.down_splits = choose_splits(0, 1, &d.out, &d.rows, parts_of(d.hidden));
        return d.down_splits > 1 ? (size_t)d.down_splits * d.rows * padded(d.out) * sizeof(float) : 0;
    }
    d.dx_splits = choose_splits(1, 1, &d.in, &d.rows, 2 * parts_of(d.hidden));
    const int features[3] = {d.in, d.in, d.hidden}, rows[3] = {d.hidden, d.hidden, d.out};
    d.weight_splits = choose_splits(2, 3, features, rows, parts_of(d.rows));
    size_t dx = 0, weights = 0;
    if (d.dx_splits > 1) dx = (size_t)d.dx_splits * d.rows * padded(d.in);
    if (d.weight_splits > 1)
        for (int n = 0; n < 3; ++n) weights += (size_t)d.weight_splits * rows[n] * (padded(features[n]) + 8);
    return (dx > weights ? dx : weights) * sizeof(float);
}

hipError_t feed_forward(const FeedDev& d, int dtype, int act, hipStream_t st) {
    return dispatch(dtype, act, [&](auto t, auto a) { return forward<decltype(t), decltype(a)::value>(d, st); });
}

hipError_t feed_backward(const FeedDev& d, int dtype, hipStream_t st) {
    return dtype == PA_BF16 ? backward<__bf16>(d, st) : backward<_Float16>(d, st);
}

}  // namespace pa
