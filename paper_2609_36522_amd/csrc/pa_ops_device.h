// Device helpers shared by the operators' kernels (wave64, gfx950).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "pa_ops.h"

namespace pa {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Eight elements at an address that is aligned to one of them: a single 16-byte access (two for
// fp32), which the hardware serves at any alignment.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Pack8 {
    T v[8];
};

// r moved down by n elements (0 .. 7), zeros behind.
template <class T>
__device__ __forceinline__ Pack8<T> shift8(Pack8<T> r, int n) {
    if constexpr (sizeof(T) == 2) {
        typedef unsigned long long u64;
        struct Two { u64 lo, hi; };
        Two t = __builtin_bit_cast(Two, r);
        if (n & 4) t = {t.hi, 0};
        const int b = (n & 3) * 16;
        t.lo = (t.lo >> b) | ((t.hi << 1) << (63 - b));
        t.hi >>= b;
        return __builtin_bit_cast(Pack8<T>, t);
    } else {
#pragma unroll
        for (int k = 4; k >= 1; k >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (n & k) r.v[i] = i + k < 8 ? r.v[i + k < 8 ? i + k : 7] : (T)0.0f;
        return r;
    }
}

// Elements at .. at + 7 of a row of len elements, zeros past its end and in an invalid row. No element
// outside the row is touched: a piece that reaches past the end is read as the row's last eight elements
// and moved down. Two halves, so that several loads can be in flight: load8_raw starts the load (without
// a branch; `row` has to exist even where the result is to be zero), fix8 waits for it. Both need
// len >= 8; load8 takes any length. len is the same in all lanes.
template <class T>
__device__ __forceinline__ Pack8<T> load8_raw(const T* row, int at, int len) {
    return *reinterpret_cast<const Pack8<T>*>(row + (at + 8 <= len ? at : len - 8));
}

template <class T>
__device__ __forceinline__ Pack8<T> fix8(Pack8<T> r, int at, int len, bool valid = true) {
    const int n = valid ? len - at : 0;
    if (len & 7) r = shift8(r, n > 0 && n < 8 ? 8 - n : 0);
    struct Words {
        uint32_t w[2 * sizeof(T)];
    };
    Words q = __builtin_bit_cast(Words, r);
#pragma unroll
    for (int i = 0; i < (int)(2 * sizeof(T)); ++i) q.w[i] = n > 0 ? q.w[i] : 0;
    return __builtin_bit_cast(Pack8<T>, q);
}

template <class T>
__device__ __forceinline__ Pack8<T> load8(const T* row, int at, int len, bool valid = true) {
    Pack8<T> r;
    const int n = valid ? len - at : 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = (T)0.0f;
    if (len >= 8) {
        if (n > 0) r = load8_raw(row, at, len);
        if (len & 7) r = shift8(r, n > 0 && n < 8 ? 8 - n : 0);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < n) r.v[i] = row[at + i];
    }
    return r;
}

// How the rows of a kernel's operands are read: rows of a multiple of 8 elements, of any 8 or more, or
// shorter ones.
constexpr int kWhole = 0, kRagged = 1, kTiny = 2;

template <class T>
__device__ __forceinline__ void store8(T* p, const Pack8<T>& r, int n) {
    if (n >= 8) {
        *reinterpret_cast<Pack8<T>*>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = r.v[i];
    }
}

// Buffer loads take 32-bit offsets from a base; one at kNowhere is out of the buffer's range and reads as
// zero.
constexpr uint32_t kBufferBytes = 0x7fffffff, kNowhere = 0x80000000;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void* p) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, kBufferBytes, 0x00020000);
}

// 16 bytes per lane, at `off` + `base_off` of the buffer, into consecutive 16-byte slots of LDS (lds: the
// wave's first). In LDS once wait_loads has returned.
__device__ __forceinline__ void load_lds(__amdgpu_buffer_rsrc_t from, void* lds, uint32_t off, int base_off) {
    typedef __attribute__((address_space(3))) void lds_void;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)lds, 16, off, base_off, 0, 0);
}

// Waits until at most N of the wave's loads are in flight (they complete in order).
template <int N = 0>
__device__ __forceinline__ void wait_loads() {
    static_assert(N < 64);
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4 << 14));
}

// A barrier for data in LDS: the wave's own LDS accesses are done, its loads (those that write LDS included:
// see wait_loads) stay in flight, where __syncthreads waits for them all.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Sum over the wave, in every lane: exchanges within 2, 4, 8 and 16 lanes (DPP), then of 16- and 32-lane
// halves. The order is fixed.
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float wave_sum_f32(float v) {
    v += dpp_f32<0xB1>(v);        // quad_perm [1, 0, 3, 2]
    v += dpp_f32<0x4E>(v);        // quad_perm [2, 3, 0, 1]
    v += dpp_f32<0x141>(v);       // row_half_mirror
    v += dpp_f32<0x140>(v);       // row_mirror
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    const float h = __builtin_bit_cast(float, (uint32_t)p[0]) + __builtin_bit_cast(float, (uint32_t)p[1]);
    const uint32_t g = __builtin_bit_cast(uint32_t, h);
    const auto q = __builtin_amdgcn_permlane32_swap(g, g, false, false);
    return __builtin_bit_cast(float, (uint32_t)q[0]) + __builtin_bit_cast(float, (uint32_t)q[1]);
}

}  // namespace pa
