// Projection in 8-bit integers, for gfx950: rows to 8 bits with a scale each, and
// y = (xq wq^T) x_scale w_scale + bias with the product in 32-bit integers (v_mfma_i32_32x32x32_i8, twice the
// 16-bit rate).
#include <type_traits>

#include "pa_gemm.h"

namespace pa {

namespace {

// ------------------------------------------------------------------ rows to 8 bits
// A row's magnitudes are compared as their bit patterns, in which NaN is larger than infinity and that than any
// number.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#pragma unroll
    for (int i = 32; i >= 1; i >>= 1) {
        const uint32_t o = __shfl_xor((int)v, i);
        v = o > v ? o : v;
    }
    return v;
}

template <int WPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* lds) {
    v = wave_max_u32(v);
    if constexpr (WPR == 1) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    const uint32_t a = lds[0] > lds[1] ? lds[0] : lds[1], b = lds[2] > lds[3] ? lds[2] : lds[3];
    return a > b ? a : b;
}

template <class T>
__device__ __forceinline__ uint32_t largest8(const Pack8<T>& p, uint32_t m) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __builtin_bit_cast(uint32_t, (float)p.v[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

__device__ __forceinline__ float scale_of(uint32_t m) {
    return m >= 0x7f800000u ? __builtin_nanf("") : __builtin_bit_cast(float, m) / 127.0f;
}

// How a row is divided by its scale: q is the nearest integer to fp32's quotient, which is rounded once. The product with
// the reciprocal is off by at most 127 x 3 2^-24 and the quotient itself by 127 x 2^-24, together 3.1e-5, so that both round to the
// same integer unless the product is within 2^-14 of the middle of two (one product in 8000): only then is there a division.
// Scales whose reciprocal is not a normal number are divided by. 32768x2048 in bf16: 64 us with divisions only, 45 so.
struct Divisor {
    float scale, inverse;
    bool good, fast;
    __device__ __forceinline__ explicit Divisor(float s) : scale(s), inverse(1.0f / s), good(s > 0.0f), fast(s > 0x1p-120f && s < 0x1p120f) {}
};

template <class T>
__device__ __forceinline__ uint2 quantize8(const Pack8<T>& p, const Divisor& d) {
    float r[8], far = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = (float)p.v[i] * d.inverse;
        r[i] = rintf(t);
        far = fmaxf(far, fabsf(t - r[i]));               // at most 1/2
    }
    if (!d.fast || far > 0.5f - 0x1p-14f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = rintf((float)p.v[i] / d.scale);
    }
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        r[i] = fminf(fmaxf(r[i], -127.0f), 127.0f);
        w[i >> 2] |= ((uint32_t)(int)r[i] & 255u) << (8 * (i & 3));
    }
    return d.good ? make_uint2(w[0], w[1]) : make_uint2(0, 0);    // scale 0 or NaN: all zero
}

// Bound by memory: 32768x2048 in bf16 45 us, 201 MB at 4.5 TB/s.
// WPR (1 or 4) waves per row, CH pieces of 8 columns per thread; CH = 0: rows of any length, read twice.
template <class T, int WPR, int CH>
__global__ __launch_bounds__(256) void k_quantize(QuantizeDev d, int64_t row0) {
    constexpr int TPR = 64 * WPR, RPB = 4 / WPR;
    __shared__ uint32_t red[4];
    const int t = threadIdx.x % TPR;
    const int64_t row = row0 + (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= d.rows) return;               // whole waves (WPR = 1) or none
    const int N = d.cols, end = (N + 15) / 16 * 16;
    const T* x = static_cast<const T*>(d.x) + row * d.x_stride;
    int8_t* q = d.q + row * d.q_stride;
    uint32_t m = 0;
    if constexpr (CH > 0) {
        Pack8<T> p[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) p[c] = load8_raw(x, (c * TPR + t) * 8, N);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            p[c] = fix8(p[c], (c * TPR + t) * 8, N);
            m = largest8(p[c], m);
        }
        const Divisor s(scale_of(row_max<WPR>(m, red)));
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = (c * TPR + t) * 8;
            if (col < end) *reinterpret_cast<uint2*>(q + col) = quantize8(p[c], s);
        }
        if (t == 0) d.scale[row] = s.scale;
    } else {
        for (int col = t * 8; col < N; col += TPR * 8) m = largest8(load8(x, col, N), m);
        const Divisor s(scale_of(row_max<WPR>(m, red)));
        for (int col = t * 8; col < end; col += TPR * 8) *reinterpret_cast<uint2*>(q + col) = quantize8(load8(x, col, N), s);
        if (t == 0) d.scale[row] = s.scale;
    }
}

// ------------------------------------------------------------------ products
// v x_scale w_scale + bias.
template <class T>
__device__ __forceinline__ float scaled(const Int8Dev& d, int v, float xs, int f) {
    float r = (float)v * xs * d.w_scale[f];
    if (d.bias) r += (float)static_cast<const T*>(d.bias)[f];
    return r;
}

// Bound by the matrix units (busy 54% of the time) and, where a tile's reduction is as short as 16 parts, by the results that
// follow it: 32768x2048x8192 557 to 600 us, 1.8 to 2.0 P operations/s.
template <class X, class T>
__global__ __launch_bounds__(X::THREADS, X::WAVES) void k_int8_tile(Int8Dev d, GemmJob job) {
    __shared__ __align__(16) char lds[X::BYTES];
    i32x16 acc[X::NM][X::NX];
    float none[X::NX];
#pragma unroll
    for (int m = 0; m < X::NM; ++m)
#pragma unroll
        for (int j = 0; j < X::NX; ++j) acc[m][j] = i32x16{};
    int f, r;
    tile_of(job, xcd_order(blockIdx.x, gridDim.x), f, r);
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int f0 = f * X::TF + (w % X::WF) * X::NM * 32, r0 = r * X::TR + (w / X::WF) * X::NX * 32;
    const PerFeature<X::NM> scales(d.w_scale, f0, d.out, lane), biases(static_cast<const T*>(d.bias), f0, d.out, lane);
    float xs[X::NX];
#pragma unroll
    for (int j = 0; j < X::NX; ++j) {
        const int row = r0 + j * 32 + (lane & 31);
        xs[j] = row < d.rows ? d.x_scale[row] : 0.0f;
    }
    X::run(job, f * X::TF, r * X::TR, 0, (job.len + X::PART - 1) / X::PART, lds, acc, none);
    constexpr int CM = X::NM < 2 ? 1 : 2;                    // 64 features at a time: 128 bytes of a row
    float* per = reinterpret_cast<float*>(lds + X::THREADS / 64 * CM * 2048 + w * 1024);
    scales.put(per, lane);
    biases.put(per + 128, lane);
#pragma unroll
    for (int c = 0; c < X::NM; c += CM) {
        const int fc = f0 + c * 32;
#pragma unroll
        for (int j = 0; j < X::NX; ++j) {
            f32x16 v[CM];
#pragma unroll
            for (int m = 0; m < CM; ++m)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 s = PerFeature<X::NM>::at(per, c + m, q, half), b = PerFeature<X::NM>::at(per + 128, c + m, q, half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[m][4 * q + i] = (float)acc[c + m][j][4 * q + i] * xs[j] * s[i] + b[i];
                }
            through_lds<T, CM>(lds + w * CM * 2048, lane, [&](int m, int q) { return gather8<T>(v[m], q, 1.0f); },
                               [&](int row, int at, const Pack8<T>& p) {
                                   if (r0 + j * 32 + row < d.rows)
                                       store8(static_cast<T*>(d.y) + (int64_t)(r0 + j * 32 + row) * d.y_stride + fc + at, p, d.out - fc - at);
                               });
        }
    }
}

// Few rows: 16 features x 16 NR rows a block, the weights read once, straight into operand registers; 16 waves
// take pieces of 64 U bytes in turn and are joined through LDS. Bound by latency: 8x1024x4096 3.5 us.
template <class T, int U, int NR>
__global__ __launch_bounds__(1024) void k_int8_few(Int8Dev d) {
    __shared__ int part[16][NR][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, f0 = blockIdx.x * 16, f = f0 + (lane & 15);
    const int8_t* wp = d.w + (int64_t)(f < d.out ? f : 0) * d.w_stride;
    i32x4 acc[NR];
#pragma unroll
    for (int j = 0; j < NR; ++j) acc[j] = i32x4{};
    for (int k0 = w * 64 * U; k0 < d.in; k0 += 16 * 64 * U) {
        i32x4 wv[U], xv[NR][U];
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int k = k0 + s * 64 + (lane >> 4) * 16;
            wv[s] = i32x4{};
            if (k < d.in) wv[s] = *reinterpret_cast<const i32x4*>(wp + k);
#pragma unroll
            for (int j = 0; j < NR; ++j) {
                const int row = j * 16 + (lane & 15);
                xv[j][s] = i32x4{};
                if (k < d.in && row < d.rows) xv[j][s] = *reinterpret_cast<const i32x4*>(d.x + row * d.x_stride + k);
            }
        }
#pragma unroll
        for (int s = 0; s < U; ++s) {
            const int n = d.in - (k0 + s * 64 + (lane >> 4) * 16);       // bytes of the piece that exist
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int left = n - 4 * i;
                const uint32_t keep = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1;
                wv[s][i] &= (int)keep;
            }
#pragma unroll
            for (int j = 0; j < NR; ++j) acc[j] = mma16(wv[s], xv[j][s], acc[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < NR; ++j)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[w][j][r][lane] = acc[j][r];
    __syncthreads();
    const int row = (w >> 2) * 16 + (lane & 15), o = f0 + 4 * (lane >> 4) + (w & 3);
    if (w >= 4 * NR || row >= d.rows || o >= d.out) return;
    int v = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += part[i][w >> 2][w & 3][lane];
    static_cast<T*>(d.y)[(int64_t)row * d.y_stride + o] = (T)scaled<T>(d, v, d.x_scale[row], o);
}

template <class T>
hipError_t linear(const Int8Dev& d, hipStream_t st) {
    // The weights read straight from memory, or tiles: up to 64 rows where a CU has at most one block of 16 features, up to 16
    // where it has more. us of both for 17, 32, 48 and 64 rows: 1024x4096 3.6, 4.0, 4.6, 5.2 and 5.0 to 5.2; 4096x1024 6.7, 8.0,
    // 9.6, 12.2 and 11.6 to 11.8; 2048x4096 5.3, 5.9, 7.0, 7.9 and 7.8 to 8.0; 2048x6144 7.2, 8.7, 11.9, 13.8 and 7.9 to 8.2 (16
    // rows 6.8 and 7.8); 8192x8192 20.8, 27.4, 36.6, 44.6 and 21.8 to 23.1 (16 rows 19.0 and 21.6).
    if (d.rows <= (d.out <= 16 * kCUs ? 64 : 16)) {
        const unsigned blocks = (unsigned)((d.out + 15) / 16);
        if (d.rows <= 16)      k_int8_few<T, 2, 1><<<blocks, 1024, 0, st>>>(d);
        else if (d.rows <= 32) k_int8_few<T, 2, 2><<<blocks, 1024, 0, st>>>(d);
        else                   k_int8_few<T, 2, 4><<<blocks, 1024, 0, st>>>(d);
        return hipGetLastError();
    }
    GemmJob job{{d.w, nullptr}, {d.x, nullptr}, d.w_stride, d.x_stride, d.out, d.rows, d.in, 0, 0};
    // Twice the elements a part at twice the rate: the same rule in parts. us with 256 x 256, 256 x 128, 128 x 192, 128 x 128 (two
    // stages), the same (three) and 64 x 64 tiles, and what the rule takes:
    //   32768x2048x8192 574 668 612 677 782 1055, 573       8192x4096x1024   47  39  45  41  47  65,  40
    //   8192x1024x4096   52  64  56  61  70   81,  52       9216x8192x1024   96 111  85 120 113 141,  85
    //   1999x1100x1347   23  15  16  14  12   14,  12       1000x2048x2048   27  17  18  16  13  11,  11
    int kind = 0;
    float least = 0.0f;
    for (int k = 0; k < kTileKinds; ++k) {
        const int64_t tiles = (int64_t)((d.out + kTileCost[k].f - 1) / kTileCost[k].f) * ((d.rows + (int64_t)kTileCost[k].r - 1) / kTileCost[k].r);
        const float t = tile_time(k, 0, tiles, (float)((d.in + 127) / 128));
        if (k == 0 || t < least) {
            least = t;
            kind = k;
        }
    }
    return with_tile<int8_t, false, false, false, false>(kind, [&](auto x) {
        typedef decltype(x) X;
        job.f_tiles = (job.features + X::TF - 1) / X::TF;
        job.r_tiles = (int)(((int64_t)job.rows + X::TR - 1) / X::TR);
        k_int8_tile<X, T><<<(unsigned)((int64_t)job.f_tiles * job.r_tiles), X::THREADS, 0, st>>>(d, job);
        return hipGetLastError();
    });
}

template <class T>
hipError_t quantize(const QuantizeDev& d, hipStream_t st) {
    for (int64_t r0 = 0; r0 < d.rows; r0 += 1 << 23) {
        const int64_t n = d.rows - r0 < 1 << 23 ? d.rows - r0 : 1 << 23;
        const unsigned waves = (unsigned)((n + 3) / 4), blocks = (unsigned)n;
        QuantizeDev c = d;
        c.rows = r0 + n;
        // A wave per row while its registers hold it, a block beyond.
        if (d.cols < 8)          k_quantize<T, 4, 0><<<blocks, 256, 0, st>>>(c, r0);
        else if (d.cols <= 512)  k_quantize<T, 1, 1><<<waves, 256, 0, st>>>(c, r0);
        else if (d.cols <= 1024) k_quantize<T, 1, 2><<<waves, 256, 0, st>>>(c, r0);
        else if (d.cols <= 2048) k_quantize<T, 1, 4><<<waves, 256, 0, st>>>(c, r0);
        else if (d.cols <= 4096) k_quantize<T, 4, 2><<<blocks, 256, 0, st>>>(c, r0);
        else if (d.cols <= 8192) k_quantize<T, 4, 4><<<blocks, 256, 0, st>>>(c, r0);
        else                     k_quantize<T, 4, 0><<<blocks, 256, 0, st>>>(c, r0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t int8_linear(const Int8Dev& d, int dtype, hipStream_t st) {
    return dtype == PA_BF16 ? linear<__bf16>(d, st) : linear<_Float16>(d, st);
}

hipError_t quantize_rows(const QuantizeDev& d, int dtype, hipStream_t st) {
    if (dtype == PA_F32) return quantize<float>(d, st);
    return dtype == PA_BF16 ? quantize<__bf16>(d, st) : quantize<_Float16>(d, st);
}

}  // namespace pa
