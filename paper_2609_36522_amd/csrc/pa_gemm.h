// Products on the matrix cores, shared by the feed-forward block and the 8-bit projection:
// out[row][feature] = sum over k of R(row, k) F(feature, k), F and R each stored with k along its rows
// (kRow: [free][k]) or with the free index along them (kCol: [k][free]).
//
// The products are transposed (F is the matrix unit's A operand, R its B operand): a lane owns an output row
// and its registers hold features, so that a lane stores consecutive features.
//
// The reduction goes through LDS in parts of 128 bytes of k (64 elements of 16 bits, 128 of 8; kCol: 64 rows),
// loaded straight into LDS, STAGES - 1 of them on their way during the products of the current one. A kRow
// operand is read with 16-byte loads, a kCol one with transposing loads; both give lane l the reduction slots
// 8 (l / 32) .. + 7 of a step of 16 (8 bits: 16 (l / 32) .. + 15 of 32), so that any two fit together.
//
// Operands are read in whole pieces of 16 bytes: rows of whole pieces at addresses of whole pieces (what
// is not so is laid out first). Pieces that do not exist read as zeros.
#pragma once

#include "pa_mma.h"

namespace pa {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Core;
template <> struct Core<__bf16> { typedef bf16x8 v; typedef f32x16 acc; typedef f32x4 acc4; };
template <> struct Core<_Float16> { typedef f16x8 v; typedef f32x16 acc; typedef f32x4 acc4; };
template <> struct Core<int8_t> { typedef i32x4 v; typedef i32x16 acc; typedef i32x4 acc4; };

__device__ __forceinline__ i32x16 mma(i32x4 a, i32x4 b, i32x16 c) {
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}
// 16 x 16: lane l supplies row l % 16 of A, column l % 16 of B and reduction piece l / 16 of four; its
// accumulator register r holds row 4 (l / 16) + r, column l % 16.
__device__ __forceinline__ f32x4 mma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ i32x4 mma16(i32x4 a, i32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// One product: F and R in one or two segments of `len` reduction elements each (the second follows the
// first; same strides).
struct GemmJob {
    const void *f[2], *r[2];
    int64_t f_stride, r_stride;      // elements
    int features, rows, len;
    int f_tiles, r_tiles;
};

// SIZE rows (kRow) or columns (kCol) of one part on their way to LDS. The permutation of a row's pieces
// (piece_at<64>) is in the addresses that are read: a wave's lanes fill consecutive 16-byte slots.
// A kCol tile is SIZE / 64 tiles of 64 k x 64 columns. UNIT > 0: two matrices, whose rows alternate in
// groups of UNIT.
template <class T, int SIZE, int THREADS, bool COL, int UNIT = 0>
struct Loads {
    static constexpr int kPieces = SIZE * 8 / THREADS, kStep = THREADS / 8, kPer = 16 / sizeof(T);
    static_assert(kPieces * THREADS == SIZE * 8 && (!COL || sizeof(T) == 2));
    static_assert(UNIT == 0 || (!COL && UNIT % kStep == 0 && SIZE % (2 * UNIT) == 0));
    uint32_t off[kPieces];
    int at;                          // kRow: the piece's first k; kCol: the first piece's k

    // `free` rows (columns) exist from the tile's first.
    __device__ __forceinline__ Loads(int64_t stride, int free) {
        const int row = (int)threadIdx.x >> 3, p = (int)threadIdx.x & 7;
        const int piece = (piece_at<64>(row, p) - row * 64) >> 3;       // the same for every 16 rows
        at = COL ? row & 63 : piece * kPer;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            if constexpr (COL) {
                const int slot = (int)threadIdx.x + i * THREADS, k = (slot & 511) >> 3, c = (slot >> 9) * 64 + piece * 8;
                off[i] = c < free ? (uint32_t)(k * (int)stride + c) * 2 : kNowhere;
            } else {
                int r = row + i * kStep;
                if (UNIT) r = r / (2 * UNIT) * UNIT + r % UNIT;
                off[i] = r < free ? (uint32_t)(r * (int)stride) * (uint32_t)sizeof(T) + piece * 16 : kNowhere;
            }
        }
    }
    // The part at `base` (UNIT: and at `other`), of whose k `left` exist.
    __device__ __forceinline__ void load(const T* base, const T* other, int left, void* tile) const {
        constexpr int PART = COL ? 64 : 128 / (int)sizeof(T);
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const __amdgpu_buffer_rsrc_t from = buffer_at(base), from2 = buffer_at(UNIT ? other : base);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int k = COL ? at + (THREADS < 512 ? (i & 1) * 32 : 0) : at;
            const bool second = UNIT && (i * kStep / (UNIT ? UNIT : 1)) % 2;
            load_lds(second ? from2 : from, static_cast<char*>(tile) + (w * 64 + i * THREADS) * 16,
                     left >= PART || k < left ? off[i] : kNowhere, 0);
        }
    }
    // 8 bits: what of the part lies past the row's end (in a piece that holds it) becomes zero.
    __device__ __forceinline__ void trim(int left, void* tile) const {
        const int n = left - at;
        if (n <= 0 || n >= kPer) return;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            char* p = static_cast<char*>(tile) + ((int)threadIdx.x + i * THREADS) * 16;
#pragma unroll
            for (int j = 1; j < 16; ++j)
                if (j >= n) p[j] = 0;
        }
    }
};

// The operand of step ks (of four in a part) for rows (columns) 32 g + lane % 32 of a tile.
template <class T, bool COL>
__device__ __forceinline__ typename Core<T>::v read_operand(const void* tile, int g, int ks, int lane) {
    typedef typename Core<T>::v v;
    const short* t = static_cast<const short*>(tile);
    const int half = lane >> 5;
    if constexpr (!COL) {
        return *reinterpret_cast<const v*>(t + piece_at<64>(g * 32 + (lane & 31), 2 * ks + half));
    } else {
        const int r = 16 * ks + 8 * half + ((lane & 15) >> 2), piece = (g & 1) * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
        const short* s = t + (g >> 1) * 4096 + (lane & 1) * 4;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(s + piece_at<64>(r, piece)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(s + piece_at<64>(r + 4, piece)));
        return __builtin_bit_cast(v, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

// The sum of an operand's eight values and c.
__device__ __forceinline__ float sum8(bf16x8 v, float c) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{v[2 * i], v[2 * i + 1]}, bf16x2{(__bf16)1.0f, (__bf16)1.0f}, c, false);
    return c;
}
__device__ __forceinline__ float sum8(f16x8 v, float c) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_fdot2(f16x2{v[2 * i], v[2 * i + 1]}, f16x2{(_Float16)1.0f, (_Float16)1.0f}, c, false);
    return c;
}

// A block's tile: WF x WR waves, each of NM x NX tiles of 32 x 32 (features x rows).
template <class T_, int WF_, int WR_, int NM_, int NX_, int STAGES_, bool FCOL_, bool RCOL_, bool GATED_ = false, bool SUMS_ = false>
struct Tile {
    typedef T_ T;
    typedef typename Core<T>::v v;
    typedef typename Core<T>::acc acc_t;
    static constexpr int WF = WF_, WR = WR_, NM = NM_, NX = NX_, STAGES = STAGES_, THREADS = 64 * WF * WR;
    static constexpr bool FCOL = FCOL_, RCOL = RCOL_, GATED = GATED_, SUMS = SUMS_;
    static constexpr int TF = WF * NM * 32, TR = WR * NX * 32;
    static constexpr int OUT = GATED ? TF / 2 : TF;                      // features of the output
    static constexpr int UNIT = GATED ? NM * 16 : 0;
    static constexpr int PART = FCOL || RCOL ? 64 : 128 / (int)sizeof(T);
    static_assert(!(FCOL || RCOL) || sizeof(T) == 2);
    static constexpr int BYTES = STAGES * (TF + TR) * 128;
    typedef Loads<T, TF, THREADS, FCOL, UNIT> LF;
    typedef Loads<T, TR, THREADS, RCOL> LR;

    // Accumulates parts `first` .. `last` - 1 of the job's tile at feature f0, row r0 into acc (and, SUMS, the
    // sums over k of the lane's rows of R into sums, of which the other half of the wave has the rest).
    __device__ __forceinline__ static void run(const GemmJob& job, int f0, int r0, int first, int last, char* lds, acc_t (&acc)[NM][NX],
                                               float (&sums)[NX]) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int fg = (w % WF) * NM, rg = (w / WF) * NX;
        const int seg_parts = (job.len + PART - 1) / PART;
        const LF lf(job.f_stride, job.features - f0);
        const LR lr(job.r_stride, job.rows - r0);
        auto left_of = [&](int part) { return job.len - (part >= seg_parts ? part - seg_parts : part) * PART; };
        auto load = [&](int part, int p) {
            const bool second = !GATED && part >= seg_parts;
            const int64_t k0 = (int64_t)(second ? part - seg_parts : part) * PART;
            const int left = job.len - (int)k0;
            const int64_t fo = FCOL ? k0 * job.f_stride + f0 : f0 * job.f_stride + k0;
            const int64_t ro = RCOL ? k0 * job.r_stride + r0 : r0 * job.r_stride + k0;
            char* tile = lds + p * (TF + TR) * 128;
            lf.load(static_cast<const T*>(job.f[second]) + fo, GATED ? static_cast<const T*>(job.f[1]) + fo : nullptr, left, tile);
            lr.load(static_cast<const T*>(job.r[second]) + ro, nullptr, left, tile + TF * 128);
        };
        auto arrive = [&](int part, int p) {
            if constexpr (sizeof(T) == 1) {
                if (left_of(part) < PART) lr.trim(left_of(part), lds + (p * (TF + TR) + TF) * 128);
            }
        };
        auto multiply = [&](int p) {
            const char* ft = lds + p * (TF + TR) * 128;
            const char* rt = ft + TF * 128;
            // The operands of the next step are read while those of the current one are multiplied.
            v a[2][NM], b[2][NX];
            auto read = [&](int ks) {
#pragma unroll
                for (int m = 0; m < NM; ++m) a[ks & 1][m] = read_operand<T, FCOL>(ft, fg + m, ks, lane);
#pragma unroll
                for (int j = 0; j < NX; ++j) b[ks & 1][j] = read_operand<T, RCOL>(rt, rg + j, ks, lane);
            };
            read(0);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                if (ks < 3) read(ks + 1);
                if constexpr (SUMS) {
#pragma unroll
                    for (int j = 0; j < NX; ++j) sums[j] = sum8(b[ks & 1][j], sums[j]);
                }
#pragma unroll
                for (int m = 0; m < NM; ++m)
#pragma unroll
                    for (int j = 0; j < NX; ++j) acc[m][j] = mma(a[ks & 1][m], b[ks & 1][j], acc[m][j]);
                if (ks < 3) {
                    constexpr int READS = NM * (FCOL ? 2 : 1) + NX * (RCOL ? 2 : 1);
                    constexpr int EACH = READS > NM * NX ? (READS + NM * NX - 1) / (NM * NX) : 1;
#pragma unroll
                    for (int g = 0; g < NM * NX; ++g) {
                        __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);     // LDS reads
                        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);        // a product
                    }
                }
            }
        };
        constexpr int LOADS = LF::kPieces + LR::kPieces;      // a thread's loads of one part
        const int parts = last - first;
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (i < parts) load(first + i, i);
        if (parts >= STAGES - 1) wait_loads<(STAGES - 2) * LOADS>();
        else wait_loads();
        if (parts > 0) arrive(first, 0);
        lds_barrier();
        int p = 0;
        for (int i = 0; i < parts; ++i) {
            int q = p + STAGES - 1;
            if (q >= STAGES) q -= STAGES;
            if (i + STAGES - 1 < parts) load(first + i + STAGES - 1, q);
            multiply(p);
            if (i + 1 < parts) {
                if (i + STAGES - 1 < parts) wait_loads<(STAGES - 2) * LOADS>();      // the next part is there
                else wait_loads();
                arrive(first + i + 1, p + 1 == STAGES ? 0 : p + 1);
            }
            lds_barrier();
            if (++p == STAGES) p = 0;
        }
    }
};

// The tile of block `id` of a job: groups of 4 row tiles side by side, features before the next group, so that the
// blocks that run together on an XCD share rows of both operands in its L2.
__device__ __forceinline__ void tile_of(const GemmJob& job, int id, int& f, int& r) {
    const int per = 4 * job.f_tiles, g = id / per, in = id - g * per, rows = job.r_tiles - g * 4 < 4 ? job.r_tiles - g * 4 : 4;
    f = in / rows;
    r = g * 4 + in - f * rows;
}

}  // namespace pa
