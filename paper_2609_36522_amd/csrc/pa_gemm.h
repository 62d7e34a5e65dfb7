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

// load_lds (pa_ops_device.h) without the compiler's own bookkeeping, which takes a transposing LDS load for one that
// may read what any load in flight writes and has it wait for all of them (dz G + du U of 8192x1024x4096: 263 us so,
// 158 without). The waits are this file's: wait_loads and a barrier before a buffer is read. The load has no output
// register; a wait that the compiler places for loads of its own can only become stricter by it.
__device__ __forceinline__ void load_lds_untracked(const void* from, void* lds, uint32_t off) {
    typedef __attribute__((address_space(3))) void lds_void;
    const uint64_t a = reinterpret_cast<uint64_t>(from);
    const i32x4 rsrc = {(int)(uint32_t)a, (int)((uint32_t)(a >> 32) & 0xffffu), (int)kBufferBytes, 0x00020000};
    __builtin_assume(lds != nullptr);
    const uint32_t to = __builtin_amdgcn_readfirstlane((int)(uint32_t)(uintptr_t)(lds_void*)lds);
    asm volatile("s_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"{m0}"(to), "v"(off), "s"(rsrc));
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
template <class T, int SIZE, int THREADS, bool COL, int UNIT = 0, bool UNTRACKED = false>
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
    // The i-th piece of the part at `base` (UNIT: and at `other`), of whose k `left` exist; w: the wave.
    __device__ __forceinline__ void load(const T* base, const T* other, int left, char* tile, int w, int i) const {
        const int k = COL && THREADS < 512 ? at + (i & 1) * 32 : at;
        const bool second = UNIT && (i * kStep / (UNIT ? UNIT : 1)) % 2;
        const uint32_t at_byte = k < left ? off[i] : kNowhere;
        if constexpr (UNTRACKED) load_lds_untracked(second ? other : base, tile + (w * 64 + i * THREADS) * 16, at_byte);
        else load_lds(buffer_at(second ? other : base), tile + (w * 64 + i * THREADS) * 16, at_byte, 0);
    }
    // 8 bits: what of the part lies past the row's end (in a piece that holds it) becomes zero.
    __device__ __forceinline__ void trim(int left, char* tile) const {
        const int n = left - at;
        if (n <= 0 || n >= kPer) return;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            char* p = tile + ((int)threadIdx.x + i * THREADS) * 16;
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
    static constexpr int WAVES = THREADS == 256 && BYTES > 81920 ? 1 : 2;      // of a SIMD: one block of 8 waves or two of 4, if LDS holds two
    typedef Loads<T, TF, THREADS, FCOL, UNIT, FCOL || RCOL> LF;
    typedef Loads<T, TR, THREADS, RCOL, 0, FCOL || RCOL> LR;

    static constexpr int LOADS = LF::kPieces + LR::kPieces;      // a thread's loads of one part
    static constexpr int HALF = (LOADS + 1) / 2;

    // Accumulates parts `first` .. `last` - 1 of the job's tile at feature f0, row r0 into acc (and, SUMS, the
    // sums over k of the lane's rows of R into sums, of which the other half of the wave has the rest). All of the
    // block's reads of LDS are done when it returns.
    //
    // A part is four steps. During a step's products the next step's operands are read, two of them and one load a
    // product, in the order in which they are written here. Before the last step the next part has to be there and
    // all waves be done with this one's buffer: its loads are issued then and in the step after.
    // 32768x2048x8192 in bf16, the times of this loop's forms: loads at the start of a part and a wait at its end
    // 1010 us, the wait before the last step 927, loads and reads between the products 895; without any loads
    // 791, without loads and reads 712 (power); four waves of 128 x 128 902, parts of 32 columns 960.
    __device__ __forceinline__ static void run(const GemmJob& job, int f0, int r0, int first, int last, char* lds, acc_t (&acc)[NM][NX],
                                               float (&sums)[NX]) {
        const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int fg = (w % WF) * NM, rg = (w / WF) * NX;
        const int seg_parts = (job.len + PART - 1) / PART, parts = last - first;
        const LF lf(job.f_stride, job.features - f0);
        const LR lr(job.r_stride, job.rows - r0);
        // Pieces lo .. hi - 1 of a part into buffer p.
        auto load = [&](int part, int p, int lo, int hi) {
            const bool second = !GATED && part >= seg_parts;
            const int64_t k0 = (int64_t)(second ? part - seg_parts : part) * PART;
            const int left = job.len - (int)k0;
            const int64_t fo = FCOL ? k0 * job.f_stride + f0 : f0 * job.f_stride + k0;
            const int64_t ro = RCOL ? k0 * job.r_stride + r0 : r0 * job.r_stride + k0;
            const T* fb = static_cast<const T*>(job.f[second]) + fo;
            const T* fb2 = GATED ? static_cast<const T*>(job.f[1]) + fo : nullptr;
            const T* rb = static_cast<const T*>(job.r[second]) + ro;
            char* tile = lds + p * (TF + TR) * 128;
#pragma unroll
            for (int x = lo; x < hi && x < LOADS; ++x) {
                if (x < LF::kPieces) lf.load(fb, fb2, left, tile, w, x);
                else lr.load(rb, nullptr, left, tile + TF * 128, w, x - LF::kPieces);
            }
        };
        // 8 bits: the end of the reduction, in the thread's own pieces, once they are there.
        auto arrive = [&](int part, int p) {
            if constexpr (sizeof(T) == 1) {
                const int left = job.len - part * PART;
                if (left < PART) lr.trim(left, lds + (p * (TF + TR) + TF) * 128);
            }
        };
        // Operands in the order of their use.
        v a[2][NM], b[2][NX];
        auto read = [&](int p, int ks, int s, int x) {
            const char* ft = lds + p * (TF + TR) * 128;
            const char* rt = ft + TF * 128;
            if (x == 0) a[s][0] = read_operand<T, FCOL>(ft, fg, ks, lane);
            else if (x <= NX) b[s][x - 1] = read_operand<T, RCOL>(rt, rg + x - 1, ks, lane);
            else a[s][x - NX] = read_operand<T, FCOL>(ft, fg + x - NX, ks, lane);
        };
        // A step's products, reads of step ks of buffer p for the next one, pieces lo .. hi - 1 of a part into buffer q.
        constexpr int G = NM * NX, READS = NM + NX, AT_ONCE = READS > 2 * G ? READS : 2;
        auto step = [&](int s, bool next, int p, int ks, int part, int q, int lo, int hi) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (next) {
#pragma unroll
                    for (int x = g * AT_ONCE; x < (g + 1) * AT_ONCE && x < READS; ++x) read(p, ks, s ^ 1, x);
                }
                if (hi > lo) load(part, q, lo + (hi - lo) * g / G, lo + (hi - lo) * (g + 1) / G);
                acc[g / NX][g % NX] = mma(a[s][g / NX], b[s][g % NX], acc[g / NX][g % NX]);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (SUMS) {
#pragma unroll
                for (int j = 0; j < NX; ++j) sums[j] = sum8(b[s][j], sums[j]);
            }
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i)
            if (i < parts) load(first + i, i, 0, LOADS);
        if (parts >= STAGES - 1) wait_loads<(STAGES - 2) * LOADS>();
        else wait_loads();
        if (parts > 0) arrive(first, 0);
        lds_barrier();
        if (parts <= 0) return;
#pragma unroll
        for (int x = 0; x < READS; ++x) read(0, 0, 0, x);
        if (STAGES - 1 < parts) load(first + STAGES - 1, STAGES - 1, 0, HALF);
        int p = 0, q = STAGES - 1, i = 0;            // q: the buffer of part i + STAGES - 1, whose second half is to come
        for (; i + STAGES < parts; ++i) {
            const int n = p + 1 == STAGES ? 0 : p + 1;
            step(0, true, p, 1, first + i + STAGES - 1, q, HALF, LOADS);
            step(1, true, p, 2, 0, 0, 0, 0);
            step(0, true, p, 3, 0, 0, 0, 0);
            wait_loads<(STAGES - 2) * LOADS>();
            arrive(first + i + 1, n);
            lds_barrier();
            __builtin_amdgcn_sched_barrier(0);
            step(1, true, n, 0, first + i + STAGES, p, 0, HALF);
            q = p;
            p = n;
        }
        if (i + STAGES - 1 < parts) load(first + i + STAGES - 1, q, HALF, LOADS);
        for (; i < parts; ++i) {
            const int n = p + 1 == STAGES ? 0 : p + 1;
            step(0, true, p, 1, 0, 0, 0, 0);
            step(1, true, p, 2, 0, 0, 0, 0);
            step(0, true, p, 3, 0, 0, 0, 0);
            wait_loads();
            if (i + 1 < parts) arrive(first + i + 1, n);
            lds_barrier();
            __builtin_amdgcn_sched_barrier(0);
            step(1, i + 1 < parts, n, 0, 0, 0, 0, 0);
            p = n;
        }
    }
};

// Stores of 32 rows x 32 NM features that a wave has in its accumulators: through LDS, so that consecutive lanes store
// consecutive features (straight from the registers every row got 32 bytes at a time, and partly written lines cost a
// quarter of a product of 1024 columns). `lds`: the wave's own NM * 2 KB. value(m, q): eight features (Pack8) from
// 32 m + 16 q + 8 half; put(row, feature, piece): stores a piece of row 0 .. 31 at feature 0, 8 ..
template <int P>
__device__ __forceinline__ int slot_of(int r, int piece) {       // rows of P pieces, whose order is permuted by the row
    return r * P + (piece ^ (r / (16 / (P < 16 ? P : 16)) % P));
}
template <class T, int NM, class F, class S>
__device__ __forceinline__ void through_lds(char* lds, int lane, F value, S put) {
    constexpr int P = NM * 4;
    const int half = lane >> 5, row = lane & 31;
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int q = 0; q < 2; ++q)
            *reinterpret_cast<uint4*>(lds + slot_of<P>(row, m * 4 + q * 2 + half) * 16) = __builtin_bit_cast(uint4, value(m, q));
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < P / 2; ++i) {
        const int at = i * 64 + lane, r = at / P, piece = at % P;
        put(r, piece * 8, __builtin_bit_cast(Pack8<T>, *reinterpret_cast<const uint4*>(lds + slot_of<P>(r, piece) * 16)));
    }
    __builtin_amdgcn_wave_barrier();
}

// A value for each of a wave's 32 NM features (biases, scales): loaded before the products, one a lane, and read from LDS
// after them by the lanes whose registers hold the features. us of the
// whole product with a load for each register from memory after the products, and so: 8 bits 32768x2048x8192 656, 585;
// the gated projections of 8192x1024x4096 143, 127.
template <int NM>
struct PerFeature {
    static constexpr int kEach = (NM * 32 + 63) / 64;
    float v[kEach];
    template <class T>
    __device__ __forceinline__ PerFeature(const T* p, int f0, int n, int lane) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int f = f0 + i * 64 + lane;
            v[i] = p ? (float)p[f < n ? f : n - 1] : 0.0f;
        }
    }
    // lds: the wave's own NM * 128 bytes (256 at least).
    __device__ __forceinline__ void put(float* lds, int lane) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i) lds[i * 64 + lane] = v[i];
        __builtin_amdgcn_wave_barrier();
    }
    // Of the features of accumulator registers 4 q .. + 3 of tile m.
    __device__ __forceinline__ static f32x4 at(const float* lds, int m, int q, int half) {
        return *reinterpret_cast<const f32x4*>(lds + m * 32 + q * 8 + half * 4);
    }
};

// The other way: pieces of 32 rows x 32 NM features, lane after lane in the order in which they lie, to the places of
// accumulator registers: out[m][q] are features 32 m + 8 q + 4 half .. + 3 of row lane % 32.
template <int NM, class V>
__device__ __forceinline__ void from_lds(char* lds, int lane, const uint4 (&in)[NM * 2], V (&out)[NM][4]) {
    constexpr int P = NM * 4;
    const int half = lane >> 5, row = lane & 31;
#pragma unroll
    for (int i = 0; i < P / 2; ++i) *reinterpret_cast<uint4*>(lds + slot_of<P>((i * 64 + lane) / P, (i * 64 + lane) % P) * 16) = in[i];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) out[m][q] = *reinterpret_cast<const V*>(lds + slot_of<P>(row, m * 4 + q) * 16 + half * 8);
    __builtin_amdgcn_wave_barrier();
}

// The tile of block `id` of a job: groups of a few row tiles side by side, features before the next group, so that the
// 32 blocks that run together on an XCD form about a square and share rows of both operands in its L2. us with groups
// of 2, 4, 6, 8 and 16 row tiles: 32768x16384x2048 (64 feature tiles) 1826, 1904, 1800, 1886, 2325; 32768x2048x8192
// (8) 895, 895, 926, 927, 1000.
__device__ __forceinline__ void tile_of(const GemmJob& job, int id, int& f, int& r) {
    const int group = job.f_tiles > 8 ? 6 : job.f_tiles > 4 ? 4 : 8;
    const int per = group * job.f_tiles, g = id / per, in = id - g * per, rows = job.r_tiles - g * group < group ? job.r_tiles - g * group : group;
    f = in / rows;
    r = g * group + in - f * rows;
}

// ------------------------------------------------------------------ which tiles (host)
constexpr int kCUs = 256;

enum { kBig, kTall, kWide, kMid, kDeep, kSmall, kTileKinds };

// What a launch of tiles is expected to take, in us: rounds of as many tiles as the CUs hold at once, each so much a part of
// the reduction and so much besides. Measured in bf16 with one and with two tiles on every CU, for two kRow operands, one
// and no kRow operand. Two blocks on a CU hide each other's waits; a CU's only block has LDS for a third stage, which hides
// the loads'. us with 256 x 256, 256 x 128, 128 x 192, 128 x 128 (two stages), the same (three) and 64 x 64 tiles:
//   8192x1024x4096         91   64   78   67   76  112        2000x1104x2736          64   39   45   37   27   36
//   8192x4096x1024         71   77   75   78   88  120        32768x2048x8192        886  966 1025 1093 1168 1763
//   8192x1024x8192, F kCol 148  127  151  135  146  238       9216x1024x8192, kCol    162  223  164  223  222  283
struct TileCost {
    int f, r, at_once;
    float one[3], all[3], besides;
};
constexpr TileCost kTileCost[kTileKinds] = {
    {256, 256, 1, {1.75f, 1.75f, 1.75f}, {1.75f, 1.75f, 1.75f}, 8.0f},
    {256, 128, 1, {0.84f, 0.90f, 0.94f}, {0.84f, 0.90f, 0.94f}, 9.0f},
    {128, 192, 2, {0.75f, 0.84f, 0.90f}, {1.42f, 1.42f, 1.45f}, 8.0f},
    {128, 128, 2, {0.63f, 0.70f, 0.75f}, {0.97f, 1.02f, 1.05f}, 7.0f},
    {128, 128, 1, {0.48f, 0.51f, 0.59f}, {0.48f, 0.51f, 0.59f}, 7.5f},
    {64, 64, 2, {0.28f, 0.34f, 0.35f}, {0.39f, 0.44f, 0.49f}, 4.0f},
};

// cols: operands that are not kRow (0 .. 2); more: what a round of tiles takes besides on top of that.
inline float tile_time(int kind, int cols, int64_t tiles, float parts, float more = 0.0f) {
    const TileCost& c = kTileCost[kind];
    const int64_t slots = (int64_t)kCUs * c.at_once, rounds = tiles / slots, rest = tiles % slots;
    float t = (float)rounds * (parts * c.all[cols] + c.besides + more);
    if (rest > 0) t += parts * (rest <= kCUs ? c.one[cols] : c.all[cols]) + c.besides + more;
    return t;
}

// f(tile type) for a kind.
template <class T, bool FCOL, bool RCOL, bool GATED, bool SUMS, class F>
auto with_tile(int kind, F f) {
    if (kind == kBig) return f(Tile<T, 2, 4, 4, 2, 2, FCOL, RCOL, GATED, SUMS>{});
    if constexpr (!GATED) {
        if (kind == kTall) return f(Tile<T, 4, 2, 2, 2, 3, FCOL, RCOL, GATED, SUMS>{});
    }
    if (kind == kWide) return f(Tile<T, 2, 2, 2, 3, 2, FCOL, RCOL, GATED, SUMS>{});
    if (kind == kMid) return f(Tile<T, 2, 2, 2, 2, 2, FCOL, RCOL, GATED, SUMS>{});
    if (kind == kDeep) return f(Tile<T, 2, 2, 2, 2, 3, FCOL, RCOL, GATED, SUMS>{});
    if constexpr (GATED) return f(Tile<T, 1, 4, 2, 1, 3, FCOL, RCOL, GATED, SUMS>{});
    else return f(Tile<T, 2, 2, 1, 1, 4, FCOL, RCOL, GATED, SUMS>{});
}

}  // namespace pa
