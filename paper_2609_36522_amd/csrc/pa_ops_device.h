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

// n of the eight elements at p exist; the others read as zero.
template <class T>
__device__ __forceinline__ Pack8<T> load8(const T* p, int n) {
    Pack8<T> r;
    if (n >= 8) {
        r = *reinterpret_cast<const Pack8<T>*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = i < n ? p[i] : (T)0.0f;
    }
    return r;
}

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

__device__ __forceinline__ float wave_sum_f32(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}

}  // namespace pa
