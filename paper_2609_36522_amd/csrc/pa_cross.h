// Cross attention kernels: what the forward and the backward pass share.
//
// Rows. The query heads that share a key/value head are rows of one matrix: row = token * group +
// head in the group, so a shared head's keys and values are read once for all of them, and a
// single token of a model with shared heads already fills several rows.
//
// Products. All use v_mfma_f32_32x32x16 (layouts: pa_mma.h). Scores are computed transposed
// (S^T = K Q^T: a lane owns a query row, its registers hold keys), so the softmax's maximum and
// sum are a lane's own plus one exchange with lane l xor 32, and
// the accumulator, rounded to 16 bits, is already the B operand of the next product over keys
// (O^T = V^T P^T): its slots 8t .. 8t + 7 are keys 16t + 4 (l/32) + {0..3, 8..11}, an order that the
// A operand (V^T) follows, read from the row-major tile with transposing LDS loads
// (read_cols).
// dk and dv come the other way round (S = Q K^T: a lane owns a key, registers hold rows).
//
// Softmax. One pass over the keys with a running maximum and sum in fp32; the accumulator is
// rescaled only in steps where some row's maximum grew. P and dS are rounded to the element type for
// their products (the accumulation stays fp32): their rounding errors are independent, so a sum
// over keys keeps the relative error of one rounding, the size of the output's own. In fp16 that holds for
// normal numbers only, so dS, and P where it is dv's operand, are brought into their range by powers of two
// (k_cross_bwd.hip); the forward pass's weights are relative to the row's largest score.
#pragma once

#include <math.h>

#include <type_traits>

#include "pa_mma.h"

namespace pa {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

// Strides below this many elements leave every offset within a tile of 128 rows to 32 bits.
constexpr int64_t kBufferStride = 1 << 23;

__device__ __forceinline__ int sample_keys(const CrossDev& d, int b) {
    if (!d.kv_lens) return d.kv_len;
    const int n = d.kv_lens[b];
    return n < 0 ? 0 : n > d.kv_len ? d.kv_len : n;
}

// The keys' mask. A value is kept as it lies in memory until it is needed, so that its load can be in
// flight; without a mask (a kernel for masks also takes scales that are not positive) one visible byte
// stands for all keys.
constexpr int kNoMask = 0, kBytes = 1, kBiases = 2;

__device__ const uint8_t kVisible = 1;

template <int MASK>
__device__ __forceinline__ uint32_t mask_load(const CrossDev& d, int b, int key) {
    if constexpr (MASK == kBiases) return static_cast<const uint32_t*>(d.mask)[b * d.mask_stride + key];
    const uint8_t* p = d.mask ? static_cast<const uint8_t*>(d.mask) + b * d.mask_stride : &kVisible;
    return p[d.mask ? key : 0];
}
// The additive bias of the key: -inf if it is not visible.
template <int MASK>
__device__ __forceinline__ float mask_bias(uint32_t v) {
    return MASK == kBiases ? __builtin_bit_cast(float, v) : v ? 0.0f : -INFINITY;
}

// A tile of ROWS rows, `stride` elements apart, on its way from memory to LDS.
// WIDTH kWhole (head_dim a multiple of 8, strides below kBufferStride): buffer loads, whose offset in the
//   tile is a thread's own for all tiles; pieces and rows that do not exist get an offset out of the
//   buffer's range, which reads as zero. With DIRECT they write LDS themselves: a wave's 64 lanes fill
//   consecutive 16-byte slots, so the permutation of a row's pieces is in the addresses that they read.
//   Without it they go through registers, where the values can be changed.
// Otherwise: any stride, any head width.
template <class T, int DP, int ROWS, int WIDTH, bool DIRECT>
struct Stage {
    static constexpr int kPieces = ROWS * (DP / 8) / kThreads, kPerRow = DP / 8, kStep = kThreads / kPerRow;
    uint4 r[DIRECT ? 1 : kPieces];
    uint32_t off;
    int rows;

    __device__ __forceinline__ static int row(int i) { return (int)threadIdx.x / kPerRow + i * kStep; }
    // The thread's piece of its rows. The permutation repeats every 16 rows, and kStep is 16 or 32.
    __device__ __forceinline__ static int piece() {
        const int p = (int)threadIdx.x % kPerRow;
        return DIRECT ? (piece_at<DP>(row(0), p) - row(0) * DP) >> 3 : p;
    }

    __device__ __forceinline__ Stage(int dim, int64_t stride)
        : off(piece() * 8 < dim ? (uint32_t)(row(0) * (int)stride + piece() * 8) * 2 : kNowhere) {}

    // Starts the tile at `base`, of which n (at least 1) rows exist, on its way.
    __device__ __forceinline__ void load(const T* base, int64_t stride, int n, int dim, T* tile) {
        rows = n;
        if constexpr (WIDTH != kWhole) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const T* p = base + (row(i) < rows ? row(i) : 0) * stride;
                r[i] = WIDTH == kRagged ? __builtin_bit_cast(uint4, load8_raw(p, piece() * 8, dim))
                                        : __builtin_bit_cast(uint4, load8(p, piece() * 8, dim, row(i) < rows));
            }
        } else {
            const __amdgpu_buffer_rsrc_t from = buffer_at(base);
            const int step = kStep * (int)stride * 2;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const uint32_t at = row(i) < rows ? off : kNowhere;
                if constexpr (DIRECT) {
                    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
                    load_lds(from, tile + (w * 64 + i * kThreads) * 8, at, i * step);
                } else {
                    r[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(from, at, i * step, 0));
                }
            }
        }
    }
    // Element offset in the tile of what the thread's i-th DIRECT load fills.
    __device__ __forceinline__ static int slot(int i) { return ((int)threadIdx.x + i * kThreads) * 8; }

    // Registers into LDS (DIRECT: nothing to do, the caller waits for the loads).
    __device__ __forceinline__ void arrive(T* tile, int dim) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                if constexpr (WIDTH == kRagged)
                    r[i] = __builtin_bit_cast(uint4, fix8(__builtin_bit_cast(Pack8<T>, r[i]), piece() * 8, dim, row(i) < rows));
                *reinterpret_cast<uint4*>(tile + piece_at<DP>(row(i), piece())) = r[i];
            }
        }
    }
};

// Keys and values of a tile of KEYS keys below kend; with a mask zeros where a key is not visible (0 weight
// times an infinity or a NaN would not be 0), and the keys' biases.
template <class T, int DP, int KEYS, int MASK, int WIDTH, bool DIRECT>
struct KvStage {
    typedef Stage<T, DP, KEYS, WIDTH, DIRECT> S;
    static constexpr int kLoads = 2 * S::kPieces;       // of a thread for one tile (masks not counted)
    S k, v;
    uint32_t bias, seen[MASK ? S::kPieces : 1];
    int left;

    __device__ __forceinline__ KvStage(const CrossDev& d) : k(d.dim, d.ks[1]), v(d.dim, d.vs[1]) {}

    __device__ __forceinline__ void load(const CrossDev& d, const T* kb, const T* vb, int k0, int kend, T* kt, T* vt) {
        k.load(kb + k0 * d.ks[1], d.ks[1], kend - k0, d.dim, kt);
        v.load(vb + k0 * d.vs[1], d.vs[1], kend - k0, d.dim, vt);
    }
    __device__ __forceinline__ void load_mask(const CrossDev& d, int b, int k0, int kend) {
        if constexpr (MASK != kNoMask) {
            left = kend - k0;
            const int i0 = (int)threadIdx.x % KEYS;
            bias = mask_load<MASK>(d, b, k0 + (i0 < left ? i0 : 0));
#pragma unroll
            for (int i = 0; i < S::kPieces; ++i) seen[i] = mask_load<MASK>(d, b, k0 + (S::row(i) < left ? S::row(i) : 0));
        }
    }
    // The tile is in LDS once every thread has called this (DIRECT: after waiting for its loads) and a
    // barrier has passed.
    __device__ __forceinline__ void arrive(T* kt, T* vt, float* bt, int dim) {
        if constexpr (MASK != kNoMask) {
            if ((int)threadIdx.x < KEYS) bt[threadIdx.x] = (int)threadIdx.x < left ? mask_bias<MASK>(bias) : -INFINITY;
#pragma unroll
            for (int i = 0; i < S::kPieces; ++i) {
                if (mask_bias<MASK>(seen[i]) != -INFINITY) continue;
                if constexpr (DIRECT) {
                    *reinterpret_cast<uint4*>(kt + S::slot(i)) = make_uint4(0, 0, 0, 0);
                    *reinterpret_cast<uint4*>(vt + S::slot(i)) = make_uint4(0, 0, 0, 0);
                } else {
                    k.r[i] = v.r[i] = make_uint4(0, 0, 0, 0);
                }
            }
        }
        k.arrive(kt, dim);
        v.arrive(vt, dim);
    }
};

// B operands of one row for all reduction steps: elements 16 ks + 8 half .. of the row at p (which exists
// also where it is not valid).
template <class T, int KS, int WIDTH>
__device__ __forceinline__ void load_row(typename Vec<T>::v8 (&out)[KS], const T* p, int dim, int half, bool valid) {
    typedef typename Vec<T>::v8 v8;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        const int at = ks * 16 + half * 8;
        if constexpr (WIDTH == kRagged) {
            out[ks] = __builtin_bit_cast(v8, load8_raw(p, at, dim));
        } else if constexpr (WIDTH == kTiny) {
            out[ks] = __builtin_bit_cast(v8, load8(p, at, dim, valid));
        } else {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (valid && at < dim) r = __builtin_bit_cast(uint4, *reinterpret_cast<const Pack8<T>*>(p + at));
            out[ks] = __builtin_bit_cast(v8, r);
        }
    }
    if constexpr (WIDTH == kRagged) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            out[ks] = __builtin_bit_cast(v8, fix8(__builtin_bit_cast(Pack8<T>, out[ks]), ks * 16 + half * 8, dim, valid));
    }
}

// Stores a transposed accumulator (lane = row of the output) times f to the row at `out`.
template <class T, int DB, int WIDTH>
__device__ __forceinline__ void store_row(T* out, int dim, const f32x16* acc, float f, int half, bool valid) {
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const Pack8<T> p = gather8<T>(acc[db], j, f);   // every lane takes part in the exchange
            const int c = db * 32 + j * 16 + half * 8;
            if constexpr (WIDTH != kWhole) {
                if (valid) store8(out + c, p, dim - c);
            } else {
                if (valid && c < dim) *reinterpret_cast<Pack8<T>*>(out + c) = p;
            }
        }
    }
}

// The same in fp32 without the exchange.
template <int DB>
__device__ __forceinline__ void store_row_f32(float* out, int dim, const f32x16* acc, int half) {
#pragma unroll
    for (int db = 0; db < DB; ++db) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = db * 32 + q * 8 + half * 4;
            struct __attribute__((packed, aligned(4))) Quad { float v[4]; };
            if (c + 4 <= dim) {
                *reinterpret_cast<Quad*>(out + c) = {{acc[db][4 * q], acc[db][4 * q + 1], acc[db][4 * q + 2], acc[db][4 * q + 3]}};
            } else {
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (c + i < dim) out[c + i] = acc[db][4 * q + i];
            }
        }
    }
}

struct RowAt {
    int token, head;
};
__device__ __forceinline__ RowAt row_at(const CrossDev& d, int hk, int row) {
    const int token = row / d.group;
    return {token, hk * d.group + (row - token * d.group)};
}
__device__ __forceinline__ int64_t stat_at(const CrossDev& d, int b, RowAt r) {
    return ((int64_t)b * d.q_heads + r.head) * d.q_len + r.token;
}

// A block's part of the forward pass or of dq: the first `whole` blocks take a row tile over all keys,
// the others a key range of a row tile each.
struct Work {
    int tile, split, part;           // row tile among those of its kv head, key range, index of the partial result (or -1)
    int b, hk, bh;
};
__device__ __forceinline__ Work work_at(const CrossDev& d) {
    Work w;
    const int row_tiles = (d.rows + d.tile_rows - 1) / d.tile_rows;
    int t;
    if ((int)blockIdx.x < d.whole) {
        t = xcd_order(blockIdx.x, d.whole);
        w.split = 0;
        w.part = -1;
    } else {
        w.part = xcd_order(blockIdx.x - d.whole, gridDim.x - d.whole);
        t = d.whole + w.part / d.splits;
        w.split = w.part % d.splits;
    }
    w.bh = t / row_tiles;
    w.tile = t - w.bh * row_tiles;
    w.b = w.bh / d.kv_heads;
    w.hk = w.bh - w.b * d.kv_heads;
    return w;
}

// Four consecutive columns from c of the n partial results at p, `step` floats apart, times weight(k), summed
// in order.
template <class F>
__device__ __forceinline__ float4 sum_parts(const float* p, int64_t step, int n, int c, int dim, F weight_of) {
    struct __attribute__((packed, aligned(4))) Quad { float v[4]; };
    const int at = c + 4 <= dim ? c : dim - 4;               // a row's last columns, moved into place below
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (dim >= 4) {
#pragma unroll 4
        for (int k = 0; k < n; ++k) {
            const Quad q = *reinterpret_cast<const Quad*>(p + k * step + at);
            const float f = weight_of(k);
            s.x = fmaf(f, q.v[0], s.x), s.y = fmaf(f, q.v[1], s.y), s.z = fmaf(f, q.v[2], s.z), s.w = fmaf(f, q.v[3], s.w);
        }
        for (int m = at; m < c; ++m) s.x = s.y, s.y = s.z, s.z = s.w;
    } else {
        for (int k = 0; k < n; ++k) {
            const float f = weight_of(k);
            s.x = fmaf(f, p[k * step], s.x);
            if (dim > 1) s.y = fmaf(f, p[k * step + 1], s.y);
            if (dim > 2) s.z = fmaf(f, p[k * step + 2], s.z);
        }
    }
    return s;
}
template <class T>
__device__ __forceinline__ void store_quad(T* out, float4 s, float f, int c, int dim) {
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (c + e < dim) out[c + e] = (T)(v[e] * f);
}

// With a mask, or a scale that is not positive (the largest scaled score is then not the scaled
// largest product), scores are formed before the maximum is taken.
inline int mask_of(const CrossDev& d) {
    return d.mask_kind == PA_MASK_ADD ? kBiases : d.mask_kind == PA_MASK_BOOL || !(d.scale > 0.0f) ? kBytes : kNoMask;
}

inline int width_of(const CrossDev& d) {
    if (d.dim < 8) return kTiny;
    for (const int64_t* p : {d.qs, d.ks, d.vs, d.os, d.dos, d.dqs, d.dks, d.dvs})
        if (p[1] >= kBufferStride) return kRagged;
    return d.dim % 8 != 0 ? kRagged : kWhole;
}

inline unsigned blocks_for(int64_t n, int each) { return (unsigned)((n + each - 1) / each); }

// Calls f(type, reduction steps of 16 over the head, mask, width): head widths are padded to 64, 80, 96 or
// 128, ragged ones to 64 or 128.
template <class F>
hipError_t dispatch(const CrossDev& d, int dtype, F f) {
    const int mask = mask_of(d);
    const int width = width_of(d);
    auto with = [&](auto t, auto ks, auto wd) {
        if (mask == kNoMask) return f(t, ks, std::integral_constant<int, kNoMask>{}, wd);
        if (mask == kBytes) return f(t, ks, std::integral_constant<int, kBytes>{}, wd);
        return f(t, ks, std::integral_constant<int, kBiases>{}, wd);
    };
    auto typed = [&](auto t) {
        const std::integral_constant<int, 4> k4;
        const std::integral_constant<int, 8> k8;
        const std::integral_constant<int, kWhole> whole;
        const std::integral_constant<int, kRagged> rag;
        if (width == kTiny) return with(t, k4, std::integral_constant<int, kTiny>{});
        if (width == kRagged) return d.dim > 64 ? with(t, k8, rag) : with(t, k4, rag);
        if (d.dim <= 64) return with(t, k4, whole);
        if (d.dim <= 80) return with(t, std::integral_constant<int, 5>{}, whole);
        return d.dim <= 96 ? with(t, std::integral_constant<int, 6>{}, whole) : with(t, k8, whole);
    };
    return dtype == PA_BF16 ? typed((__bf16)0) : typed((_Float16)0);
}

}  // namespace

}  // namespace pa
