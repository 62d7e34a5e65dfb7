// Matrix-core operands of the operators' kernels (v_mfma_f32_32x32x16, bf16 or fp16): lane l
// supplies row l%32 of A, column l%32 of B and reduction slots 8 (l/32) .. + 7; accumulator register
// r of lane l holds row 8 (r/4) + 4 (l/32) + r%4, column l%32.
#pragma once

#include "pa_ops_device.h"

namespace pa {

template <class T> struct Vec;
template <> struct Vec<__bf16> { typedef bf16x8 v8; };
template <> struct Vec<_Float16> { typedef f16x8 v8; };

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Element offset of 16-byte piece `piece` of row `row` in an LDS tile of DP (64 or 128) columns.
// The pieces of a row are permuted by the row, so that 16 rows read at one column and four rows
// read over 64 bytes both spread over all banks.
template <int DP>
__device__ __forceinline__ int piece_at(int row, int piece) {
    const int f = DP == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return row * DP + ((piece ^ f) << 3);
}

// A or B operand whose row (column) is tile row `row`, reduction over the columns 16 ks ..
template <class T, int DP>
__device__ __forceinline__ typename Vec<T>::v8 read_rows(const T* tile, int row, int ks, int half) {
    return *reinterpret_cast<const typename Vec<T>::v8*>(tile + piece_at<DP>(row, 2 * ks + half));
}

// A operand whose row is tile column 32 db + lane % 32, reduction over the tile rows
// row0 + 4 half + {0..3, 8..11} (the slots of an accumulator's registers). A transposing LDS load
// gives lane i of 16 the i-th of the 16 elements that four lanes each point at in four rows.
template <class T, int DP>
__device__ __forceinline__ typename Vec<T>::v8 read_cols(const T* tile, int row0, int db, int lane) {
    const int half = lane >> 5, r = row0 + 4 * half + ((lane & 15) >> 2);
    const int piece = db * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), e = (lane & 1) * 4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + piece_at<DP>(r, piece) + e));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + piece_at<DP>(r + 8, piece) + e));
    const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(typename Vec<T>::v8, v);
}

// Eight elements at .. of an existing row of len, whole after `fixed`.
template <class T, int WIDTH>
__device__ __forceinline__ typename Vec<T>::v8 operand(const T* row, int at, int len, bool valid) {
    typedef typename Vec<T>::v8 v8;
    if constexpr (WIDTH == kRagged) return __builtin_bit_cast(v8, load8_raw(row, at, len));
    if constexpr (WIDTH == kTiny) return __builtin_bit_cast(v8, load8(row, at, len, valid));
    uint4 r = make_uint4(0, 0, 0, 0);
    if (valid && at < len) r = __builtin_bit_cast(uint4, *reinterpret_cast<const Pack8<T>*>(row + at));
    return __builtin_bit_cast(v8, r);
}
template <class T, int WIDTH>
__device__ __forceinline__ typename Vec<T>::v8 fixed(typename Vec<T>::v8 r, int at, int len, bool valid) {
    if constexpr (WIDTH == kRagged) return __builtin_bit_cast(typename Vec<T>::v8, fix8(__builtin_bit_cast(Pack8<T>, r), at, len, valid));
    return r;
}

// Registers 8t .. 8t + 7 of an accumulator in the element type: a B operand.
template <class T>
__device__ __forceinline__ typename Vec<T>::v8 pack(const f32x16& s, int t) {
    typename Vec<T>::v8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (T)s[8 * t + i];
    return r;
}

// Eight consecutive elements per lane from registers 8j .. 8j + 7 (rows 16 j + 4 half + {0..3, 8..11}):
// lanes below 32 receive rows 16 j .. + 7, the others 16 j + 8 .. + 15. w: the registers' 16-bit values in pairs.
__device__ __forceinline__ uint4 rows8(const uint32_t (&w)[2][2]) {
    const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
    return make_uint4(x[0], y[0], x[1], y[1]);
}
template <class T>
__device__ __forceinline__ Pack8<T> gather8(const f32x16& a, int j, float f) {
    typedef T t2 __attribute__((ext_vector_type(2)));
    uint32_t w[2][2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const t2 e = {(T)(a[8 * j + 4 * q + 2 * p] * f), (T)(a[8 * j + 4 * q + 2 * p + 1] * f)};
            w[q][p] = __builtin_bit_cast(uint32_t, e);
        }
    }
    return __builtin_bit_cast(Pack8<T>, rows8(w));
}

// Blocks are dealt to the 8 XCDs in turn: gives each XCD a contiguous range of work, so that
// blocks that read the same operands share an L2.
__device__ __forceinline__ int xcd_order(int id, int total) {
    const int x = id & 7, per = total >> 3, rem = total & 7;
    return x * per + (x < rem ? x : rem) + (id >> 3);
}

}  // namespace pa
