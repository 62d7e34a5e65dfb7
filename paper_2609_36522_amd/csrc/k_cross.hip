// Cross attention, forward and backward, for gfx950.
//
// Rows. The query heads that share a key/value head are rows of one matrix: row = token * group +
// head in the group, so a shared head's keys and values are read once for all of them, and a
// single token of a model with shared heads already fills several rows.
//
// Products. All use v_mfma_f32_32x32x16 (layouts: pa_mma.h). Scores are computed transposed (S^T = K Q^T: a lane owns a query row, its registers hold
// keys), so the softmax's maximum and sum are a lane's own plus one exchange with lane l xor 32, and
// the accumulator, rounded to 16 bits, is already the B operand of the next product over keys
// (O^T = V^T P^T): its slots 8t .. 8t + 7 are keys 16t + 4 (l/32) + {0..3, 8..11}, an order that the
// A operand (V^T) follows, read from the row-major tile with transposing LDS loads
// (read_cols).
// dk and dv come the other way round (S = Q K^T: a lane owns a key, registers hold rows).
//
// Softmax. One pass over the keys with a running maximum and sum in fp32; the accumulator is
// rescaled only in steps where some row's maximum grew. P and dS are rounded to the element type for
// their products (the accumulation stays fp32): their rounding errors are independent, so a sum
// over keys keeps the relative error of one rounding, the size of the output's own.
#include <math.h>

#include <type_traits>

#include "pa_mma.h"

namespace pa {

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ int sample_keys(const CrossDev& d, int b) {
    if (!d.kv_lens) return d.kv_len;
    const int n = d.kv_lens[b];
    return n < 0 ? 0 : n > d.kv_len ? d.kv_len : n;
}

// Additive bias of a key below the sample's length: 0, the mask's value, or -inf.
__device__ __forceinline__ float key_bias(const CrossDev& d, int b, int key) {
    if (d.mask_kind == PA_MASK_NONE) return 0.0f;
    const int64_t at = b * d.mask_stride + key;
    if (d.mask_kind == PA_MASK_ADD) return static_cast<const float*>(d.mask)[at];
    return static_cast<const uint8_t*>(d.mask)[at] ? 0.0f : -INFINITY;
}

// A tile of ROWS rows on its way from memory to LDS: each thread holds some of its 16-byte pieces.
// Rows lie `stride` elements apart. Without RAGGED (head_dim a multiple of 8, strides below
// kBufferStride) a piece is one buffer load whose offset within the tile fits 32 bits and is the same
// for every tile; pieces and rows that do not exist get an offset out of the buffer's range, which reads
// as zero. RAGGED takes any head_dim and stride.
constexpr int64_t kBufferStride = 1 << 23;
constexpr uint32_t kBufferBytes = 0x7fffffff, kNowhere = 0x80000000;

template <class T, int DP, int ROWS, bool RAGGED>
struct Stage {
    static constexpr int kPieces = ROWS * (DP / 8) / kThreads, kPerRow = DP / 8;
    uint4 r[kPieces];
    uint32_t off;

    __device__ __forceinline__ static int row(int i) { return (int)threadIdx.x / kPerRow + i * (kThreads / kPerRow); }
    __device__ __forceinline__ static int piece() { return (int)threadIdx.x % kPerRow; }

    __device__ __forceinline__ Stage(int dim, int64_t stride)
        : off(piece() * 8 < dim ? (uint32_t)(row(0) * (int)stride + piece() * 8) * 2 : kNowhere) {}

    // rows of the tile at `base` exist.
    __device__ __forceinline__ void load(const T* base, int64_t stride, int rows, int dim) {
        if constexpr (RAGGED) {
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                r[i] = __builtin_bit_cast(uint4, load8(base + row(i) * stride, piece() * 8, dim, row(i) < rows));
        } else {
            const __amdgpu_buffer_rsrc_t src = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, kBufferBytes, 0x00020000);
            const int step = (kThreads / kPerRow) * (int)stride * 2;
#pragma unroll
            for (int i = 0; i < kPieces; ++i)
                r[i] = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(src, row(i) < rows ? off : kNowhere, i * step, 0));
        }
    }
    __device__ __forceinline__ void store(T* tile) const {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) *reinterpret_cast<uint4*>(tile + piece_at<DP>(row(i), piece())) = r[i];
    }
};

// Keys and values of a tile, zeros where a key is not visible (0 weight times an infinity or a NaN
// would not be 0), and with MASKED the keys' biases.
template <class T, int DP, int KEYS, bool MASKED, bool RAGGED>
struct KvStage {
    typedef Stage<T, DP, KEYS, RAGGED> S;
    S k, v;
    float bias, seen[MASKED ? S::kPieces : 1];

    __device__ __forceinline__ KvStage(const CrossDev& d) : k(d.dim, d.ks[1]), v(d.dim, d.vs[1]) {}

    __device__ __forceinline__ void load(const CrossDev& d, const T* kb, const T* vb, int b, int k0, int kend) {
        k.load(kb + k0 * d.ks[1], d.ks[1], kend - k0, d.dim);
        v.load(vb + k0 * d.vs[1], d.vs[1], kend - k0, d.dim);
        if constexpr (MASKED) {
            const int key = k0 + (int)threadIdx.x;
            bias = (int)threadIdx.x < KEYS && key < kend ? key_bias(d, b, key) : -INFINITY;
#pragma unroll
            for (int i = 0; i < S::kPieces; ++i) {
                const int kk = k0 + S::row(i);
                seen[i] = kk < kend ? key_bias(d, b, kk) : 0.0f;
            }
        }
    }
    __device__ __forceinline__ void store(T* kt, T* vt, float* bt) {
        if constexpr (MASKED) {
#pragma unroll
            for (int i = 0; i < S::kPieces; ++i)
                if (seen[i] == -INFINITY) k.r[i] = v.r[i] = make_uint4(0, 0, 0, 0);
            if ((int)threadIdx.x < KEYS) bt[threadIdx.x] = bias;
        }
        k.store(kt);
        v.store(vt);
    }
};

// B operands of one row for all reduction steps: elements 16 ks + 8 half .. of the row at p.
template <class T, int DP, bool RAGGED>
__device__ __forceinline__ void load_row(typename Vec<T>::v8 (&out)[DP / 16], const T* p, int dim, int half, bool valid) {
#pragma unroll
    for (int ks = 0; ks < DP / 16; ++ks) {
        const int at = ks * 16 + half * 8;
        if constexpr (RAGGED) {
            out[ks] = __builtin_bit_cast(typename Vec<T>::v8, load8(p, at, dim, valid));
        } else {
            uint4 r = make_uint4(0, 0, 0, 0);
            if (valid && at < dim) r = __builtin_bit_cast(uint4, *reinterpret_cast<const Pack8<T>*>(p + at));
            out[ks] = __builtin_bit_cast(typename Vec<T>::v8, r);
        }
    }
}

// Stores a transposed accumulator (lane = row of the output) times f to the row at `out`.
template <class T, int DP, bool RAGGED>
__device__ __forceinline__ void store_row(T* out, int dim, const f32x16* acc, float f, int half, bool valid) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const Pack8<T> p = gather8<T>(acc[db], j, f);   // every lane takes part in the exchange
            const int c = db * 32 + j * 16 + half * 8;
            if constexpr (RAGGED) {
                if (valid) store8(out + c, p, dim - c);
            } else {
                if (valid && c < dim) *reinterpret_cast<Pack8<T>*>(out + c) = p;
            }
        }
    }
}

// The same in fp32 without the exchange.
template <int DP>
__device__ __forceinline__ void store_row_f32(float* out, int dim, const f32x16* acc, int half) {
#pragma unroll
    for (int db = 0; db < DP / 32; ++db) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = db * 32 + q * 8 + half * 4;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < dim) out[c + i] = acc[db][4 * q + i];
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

// ------------------------------------------------------------------ forward
// KW = 1: four waves of 32 rows share tiles of 64 keys. KW = 4 (at most 32 rows): the four waves
// take 32 keys each of a 128-key tile for the same rows and are joined at the end.
template <class T, int DP, int KW, bool MASKED, bool RAGGED>
__global__ __launch_bounds__(kThreads, 2) void k_cross_fwd(CrossDev d) {
    constexpr int KEYS = KW == 1 ? 64 : 128, ROWS = KW == 1 ? 128 : 32, NT = KW == 1 ? 2 : 1;
    typedef typename Vec<T>::v8 v8;
    // K tile, V tile; with KW = 4 afterwards the waves' accumulators [4][32][DP] in fp32.
    __shared__ __align__(16) T tiles[2 * KEYS * DP];
    __shared__ float bias[MASKED ? KEYS : 1];
    __shared__ float wave_m[4][32], wave_l[4][32];
    T* kt = tiles;
    T* vt = tiles + KEYS * DP;

    const int row_tiles = (d.rows + ROWS - 1) / ROWS;
    int id = xcd_order(blockIdx.x, gridDim.x);
    const int tile = id % row_tiles;
    id /= row_tiles;
    const int split = id % d.splits, bh = id / d.splits;
    const int b = bh / d.kv_heads, hk = bh - b * d.kv_heads;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + (KW == 1 ? w * 32 : 0) + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);

    const T* qp = static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2];
    v8 q[DP / 16];
    load_row<T, DP, RAGGED>(q, qp, d.dim, half, valid);

    const int klen = sample_keys(d, b);
    const int kbeg = split * d.split_keys;
    const int kend = klen < kbeg + d.split_keys ? klen : kbeg + d.split_keys;
    const T* kb = static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2];
    const T* vb = static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2];

    // Scores in units of 1/f: x f is the exponent of 2. With a mask x is the scaled, biased score.
    const float f = MASKED ? kLog2e : d.scale * kLog2e;
    f32x16 acc[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) acc[i] = f32x16{};
    float m = -INFINITY, l = 0.0f;

    KvStage<T, DP, KEYS, MASKED, RAGGED> st(d);
    if (kbeg < kend) st.load(d, kb, vb, b, kbeg, kend);
    for (int k0 = kbeg; k0 < kend; k0 += KEYS) {
        __syncthreads();
        st.store(kt, vt, bias);
        __syncthreads();
        if (k0 + KEYS < kend) st.load(d, kb, vb, b, k0 + KEYS, kend);
        const int koff = KW == 1 ? 0 : w * 32;
        f32x16 s[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            s[nt] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks)
                s[nt] = mma(read_rows<T, DP>(kt, koff + nt * 32 + (lane & 31), ks, half), q[ks], s[nt]);
        }
        if constexpr (MASKED) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[nt][r] = fmaf(s[nt][r], d.scale, bias[koff + nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3)]);
        } else if (k0 + KEYS > kend) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + koff + nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= kend) s[nt][r] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[nt][r]);
        top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
        const float base = top == -INFINITY ? 0.0f : top;   // nothing seen yet: every weight is 0
        if (__any(top > m)) {
            const float a = __builtin_amdgcn_exp2f((m - base) * f);
            l *= a;
#pragma unroll
            for (int i = 0; i < DP / 32; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= a;
            m = top;
        }
        const float mf = base * f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // With a mask the difference comes first: x may be near the type's lowest value.
                const float p = __builtin_amdgcn_exp2f(MASKED ? (s[nt][r] - base) * f : fmaf(s[nt][r], f, -mf));
                s[nt][r] = p;
                l += p;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const v8 p = pack<T>(s[nt], t);
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
                    acc[db] = mma(read_cols<T, DP>(vt, koff + nt * 32 + t * 16, db, lane), p, acc[db]);
            }
        }
    }
    l += __shfl_xor(l, 32, 64);
    const float m_nat = MASKED || m == -INFINITY ? m : m * d.scale;

    if constexpr (KW == 1) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;      // no key seen: acc is 0
        if (d.splits == 1) {
            T* op = static_cast<T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2];
            store_row<T, DP, RAGGED>(op, d.dim, acc, inv, half, valid);
            if (d.stats && valid && half == 0) {
                float* sp = d.stats + stat_at(d, b, ra) * 2;
                sp[0] = m_nat;
                sp[1] = logf(l);
            }
        } else if (valid) {
            const int64_t at = ((int64_t)split * d.batch * d.kv_heads + bh) * d.rows + row;
            store_row_f32<DP>(d.part + at * d.dim, d.dim, acc, half);
            if (half == 0) {
                d.part_stats[at * 2] = m_nat;
                d.part_stats[at * 2 + 1] = l;
            }
        }
    } else {
        float* wa = reinterpret_cast<float*>(tiles);
        __syncthreads();
#pragma unroll
        for (int db = 0; db < DP / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                wa[(w * DP + db * 32 + 8 * (r >> 2) + 4 * half + (r & 3)) * 32 + (lane & 31)] = acc[db][r];
        if (half == 0) {
            wave_m[w][lane] = m_nat;
            wave_l[w][lane] = l;
        }
        __syncthreads();
        // Thread: row threadIdx % 32, columns threadIdx / 32 + 8 i.
        const int rr = threadIdx.x & 31, orow = tile * ROWS + rr;
        if (orow >= d.rows) return;
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, wave_m[i][rr]);
        const float base = top == -INFINITY ? 0.0f : top;
        float a[4], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = __builtin_amdgcn_exp2f((wave_m[i][rr] - base) * kLog2e);
            sum += a[i] * wave_l[i][rr];
        }
        const RowAt oa = row_at(d, hk, orow);
        const int64_t at = ((int64_t)split * d.batch * d.kv_heads + bh) * d.rows + orow;
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        T* op = static_cast<T*>(d.o) + b * d.os[0] + oa.token * d.os[1] + oa.head * d.os[2];
        for (int c = threadIdx.x >> 5; c < d.dim; c += 8) {
            float o = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) o += a[i] * wa[(i * DP + c) * 32 + rr];
            if (d.splits == 1) op[c] = (T)(o * inv);
            else d.part[at * d.dim + c] = o;
        }
        if (threadIdx.x < 32) {
            if (d.splits > 1) {
                d.part_stats[at * 2] = top;
                d.part_stats[at * 2 + 1] = sum;
            } else if (d.stats) {
                float* sp = d.stats + stat_at(d, b, oa) * 2;
                sp[0] = top;
                sp[1] = logf(sum);
            }
        }
    }
}

// Joins the key ranges' partial outputs: a wave per row.
template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_join(CrossDev d) {
    const int64_t n = (int64_t)d.batch * d.kv_heads * d.rows;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= n) return;
    const int lane = threadIdx.x & 63;
    float top = -INFINITY;
    for (int s = 0; s < d.splits; ++s) top = fmaxf(top, d.part_stats[(s * n + at) * 2]);
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, o0 = 0.0f, o1 = 0.0f;
    for (int s = 0; s < d.splits; ++s) {
        const float a = __builtin_amdgcn_exp2f((d.part_stats[(s * n + at) * 2] - base) * kLog2e);
        sum += a * d.part_stats[(s * n + at) * 2 + 1];
        const float* p = d.part + (s * n + at) * d.dim;
        if (lane < d.dim) o0 += a * p[lane];
        if (lane + 64 < d.dim) o1 += a * p[lane + 64];
    }
    const int bh = (int)(at / d.rows), b = bh / d.kv_heads;
    const RowAt ra = row_at(d, bh - b * d.kv_heads, (int)(at - (int64_t)bh * d.rows));
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* op = static_cast<T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2];
    if (lane < d.dim) op[lane] = (T)(o0 * inv);
    if (lane + 64 < d.dim) op[lane + 64] = (T)(o1 * inv);
    if (d.stats && lane == 0) {
        float* sp = d.stats + stat_at(d, b, ra) * 2;
        sp[0] = top;
        sp[1] = logf(sum);
    }
}

// ------------------------------------------------------------------ backward
// delta = sum of do * o over a head: 16 lanes per row of [batch][q_heads][q_len].
template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_delta(CrossDev d) {
    const int64_t n = (int64_t)d.batch * d.q_heads * d.q_len;
    const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int64_t at = i < n ? i : n - 1;
    const int c = (threadIdx.x & 15) * 8;
    // Tokens outermost, as the tensors usually lie.
    const int h = (int)(at % d.q_heads);
    const int64_t bt = at / d.q_heads, t = bt % d.q_len, b = bt / d.q_len;
    const Pack8<T> po = load8(static_cast<const T*>(d.o) + b * d.os[0] + t * d.os[1] + h * d.os[2], c, d.dim);
    const Pack8<T> pd = load8(static_cast<const T*>(d.d_o) + b * d.dos[0] + t * d.dos[1] + h * d.dos[2], c, d.dim);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (float)po.v[e] * (float)pd.v[e];
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) s += __shfl_xor(s, off, 64);
    if (i < n && (threadIdx.x & 15) == 0) d.delta[(b * d.q_heads + h) * d.q_len + t] = s;
}

// A row's statistics as the backward pass uses them: without a mask hi = log2 of the sum of all
// weights (lo unused), with one the maximum and the logarithm apart. A row that sees no key has
// weights 0 whatever its scores.
template <bool MASKED>
__device__ __forceinline__ void row_stats(const CrossDev& d, int64_t at, float& hi, float& lo) {
    const float m = d.stats[at * 2], ll = d.stats[at * 2 + 1];
    const bool empty = ll == -INFINITY;
    hi = MASKED ? (empty ? 0.0f : m) : (empty ? INFINITY : (m + ll) * kLog2e);
    lo = empty ? INFINITY : ll;
}
template <bool MASKED>
__device__ __forceinline__ float weight(float s, float scale, float f, float bias, float hi, float lo) {
    return __builtin_amdgcn_exp2f(MASKED ? ((fmaf(s, scale, bias) - hi) - lo) * kLog2e : fmaf(s, f, -hi));
}

// dq: the forward pass's tiling; a lane owns a row, K and V tiles pass by.
template <class T, int DP, bool MASKED, bool RAGGED>
__global__ __launch_bounds__(kThreads, 2) void k_cross_dq(CrossDev d) {
    constexpr int KEYS = 64, ROWS = 128;
    typedef typename Vec<T>::v8 v8;
    __shared__ __align__(16) T tiles[2 * KEYS * DP];
    __shared__ float bias[MASKED ? KEYS : 1];
    T* kt = tiles;
    T* vt = tiles + KEYS * DP;

    const int row_tiles = (d.rows + ROWS - 1) / ROWS;
    int id = xcd_order(blockIdx.x, gridDim.x);
    const int tile = id % row_tiles;
    id /= row_tiles;
    const int split = id % d.splits, bh = id / d.splits;
    const int b = bh / d.kv_heads, hk = bh - b * d.kv_heads;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + w * 32 + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);
    const int64_t sat = stat_at(d, b, ra);

    const T* qp = static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2];
    const T* dp = static_cast<const T*>(d.d_o) + b * d.dos[0] + ra.token * d.dos[1] + ra.head * d.dos[2];
    v8 q[DP / 16], g[DP / 16];
    load_row<T, DP, RAGGED>(q, qp, d.dim, half, valid);
    load_row<T, DP, RAGGED>(g, dp, d.dim, half, valid);
    float hi, lo;
    row_stats<MASKED>(d, sat, hi, lo);
    const float delta = d.delta[sat], f = d.scale * kLog2e;

    const int klen = sample_keys(d, b);
    const int kbeg = split * d.split_keys;
    const int kend = klen < kbeg + d.split_keys ? klen : kbeg + d.split_keys;
    const T* kb = static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2];
    const T* vb = static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2];
    f32x16 acc[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) acc[i] = f32x16{};

    KvStage<T, DP, KEYS, MASKED, RAGGED> st(d);
    if (kbeg < kend) st.load(d, kb, vb, b, kbeg, kend);
    for (int k0 = kbeg; k0 < kend; k0 += KEYS) {
        __syncthreads();
        st.store(kt, vt, bias);
        __syncthreads();
        if (k0 + KEYS < kend) st.load(d, kb, vb, b, k0 + KEYS, kend);
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            f32x16 s = f32x16{}, e = f32x16{};
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) {
                s = mma(read_rows<T, DP>(kt, nt * 32 + (lane & 31), ks, half), q[ks], s);
                e = mma(read_rows<T, DP>(vt, nt * 32 + (lane & 31), ks, half), g[ks], e);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int key = nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3);
                float p = weight<MASKED>(s[r], d.scale, f, MASKED ? bias[key] : 0.0f, hi, lo);
                if (!MASKED && k0 + key >= kend) p = 0.0f;
                s[r] = p * (e[r] - delta);
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const v8 ds = pack<T>(s, t);
#pragma unroll
                for (int db = 0; db < DP / 32; ++db)
                    acc[db] = mma(read_cols<T, DP>(kt, nt * 32 + t * 16, db, lane), ds, acc[db]);
            }
        }
    }
    if (d.splits == 1) {
        T* out = static_cast<T*>(d.dq) + b * d.dqs[0] + ra.token * d.dqs[1] + ra.head * d.dqs[2];
        store_row<T, DP, RAGGED>(out, d.dim, acc, d.scale, half, valid);
    } else if (valid) {
        const int64_t at = ((int64_t)split * d.batch * d.kv_heads + bh) * d.rows + row;
        store_row_f32<DP>(d.part + at * d.dim, d.dim, acc, half);
    }
}

// dk, dv: a wave owns 32 keys (K and V in registers), tiles of 32 rows of q and do pass by.
template <class T, int DP, bool MASKED, bool RAGGED>
__global__ __launch_bounds__(kThreads, 1) void k_cross_dkv(CrossDev d) {
    constexpr int KEYS = 128, ROWS = 32;
    typedef typename Vec<T>::v8 v8;
    __shared__ __align__(16) T tiles[2 * ROWS * DP];
    __shared__ __align__(16) float stat[3][ROWS];   // hi, lo, delta
    T* qt = tiles;
    T* gt = tiles + ROWS * DP;

    const int key_tiles = (d.kv_len + KEYS - 1) / KEYS;
    int id = xcd_order(blockIdx.x, gridDim.x);
    const int tile = id % key_tiles;
    id /= key_tiles;
    const int split = id % d.row_splits, bh = id / d.row_splits;
    const int b = bh / d.kv_heads, hk = bh - b * d.kv_heads;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int key = tile * KEYS + w * 32 + (lane & 31);
    const int klen = sample_keys(d, b);
    bool seen = key < klen;
    float bias = 0.0f;
    if (MASKED && seen) {
        bias = key_bias(d, b, key);
        seen = bias != -INFINITY;
    }
    const T* kp = static_cast<const T*>(d.k) + b * d.ks[0] + key * d.ks[1] + hk * d.ks[2];
    const T* vp = static_cast<const T*>(d.v) + b * d.vs[0] + key * d.vs[1] + hk * d.vs[2];
    v8 kr[DP / 16], vr[DP / 16];
    load_row<T, DP, RAGGED>(kr, kp, d.dim, half, seen);
    load_row<T, DP, RAGGED>(vr, vp, d.dim, half, seen);
    f32x16 ak[DP / 32], av[DP / 32];
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) ak[i] = av[i] = f32x16{};
    const float f = d.scale * kLog2e;

    // Tiles of 32 tokens of one query head; the heads of the group one after the other.
    const int head_tiles = (d.q_len + ROWS - 1) / ROWS;
    const int tbeg = split * d.split_tiles;
    int tend = d.group * head_tiles;
    if (tend > tbeg + d.split_tiles) tend = tbeg + d.split_tiles;
    if (tile * KEYS >= klen) tend = tbeg;
    const T* qb = static_cast<const T*>(d.q) + b * d.qs[0] + (int64_t)hk * d.group * d.qs[2];
    const T* gb = static_cast<const T*>(d.d_o) + b * d.dos[0] + (int64_t)hk * d.group * d.dos[2];
    Stage<T, DP, ROWS, RAGGED> sq(d.dim, d.qs[1]), sg(d.dim, d.dos[1]);
    float s_hi = 0.0f, s_lo = 0.0f, s_delta = 0.0f;
    auto load = [&](int t) {
        const int g = t / head_tiles, r0 = (t - g * head_tiles) * ROWS, rows = d.q_len - r0;
        sq.load(qb + g * d.qs[2] + r0 * d.qs[1], d.qs[1], rows, d.dim);
        sg.load(gb + g * d.dos[2] + r0 * d.dos[1], d.dos[1], rows, d.dim);
        if (threadIdx.x < ROWS) {
            if ((int)threadIdx.x < rows) {
                const int64_t at = stat_at(d, b, {r0 + (int)threadIdx.x, hk * d.group + g});
                row_stats<MASKED>(d, at, s_hi, s_lo);
                s_delta = d.delta[at];
            } else {
                s_hi = MASKED ? 0.0f : INFINITY;
                s_lo = INFINITY;
                s_delta = 0.0f;
            }
        }
    };
    if (tbeg < tend) load(tbeg);
    for (int it = tbeg; it < tend; ++it) {
        __syncthreads();
        sq.store(qt);
        sg.store(gt);
        if (threadIdx.x < ROWS) {
            stat[0][threadIdx.x] = s_hi;
            stat[1][threadIdx.x] = s_lo;
            stat[2][threadIdx.x] = s_delta;
        }
        __syncthreads();
        if (it + 1 < tend) load(it + 1);
        f32x16 s = f32x16{}, e = f32x16{};
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks) {
            s = mma(read_rows<T, DP>(qt, lane & 31, ks, half), kr[ks], s);
            e = mma(read_rows<T, DP>(gt, lane & 31, ks, half), vr[ks], e);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int rr = 8 * (r >> 2) + 4 * half + (r & 3);
            float p = weight<MASKED>(s[r], d.scale, f, bias, stat[0][rr], MASKED ? stat[1][rr] : 0.0f);
            if (!seen) p = 0.0f;
            s[r] = p;
            e[r] = seen ? p * (e[r] - stat[2][rr]) : 0.0f;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v8 p = pack<T>(s, t), ds = pack<T>(e, t);
#pragma unroll
            for (int db = 0; db < DP / 32; ++db) {
                av[db] = mma(read_cols<T, DP>(gt, t * 16, db, lane), p, av[db]);
                ak[db] = mma(read_cols<T, DP>(qt, t * 16, db, lane), ds, ak[db]);
            }
        }
    }
    const bool valid = key < d.kv_len;
    if (d.row_splits == 1) {
        T* ok = static_cast<T*>(d.dk) + b * d.dks[0] + key * d.dks[1] + hk * d.dks[2];
        T* ov = static_cast<T*>(d.dv) + b * d.dvs[0] + key * d.dvs[1] + hk * d.dvs[2];
        store_row<T, DP, RAGGED>(ok, d.dim, ak, d.scale, half, valid);
        store_row<T, DP, RAGGED>(ov, d.dim, av, 1.0f, half, valid);
    } else if (valid) {
        const int64_t at = ((int64_t)split * d.batch * d.kv_heads + bh) * d.kv_len + key;
        store_row_f32<DP>(d.part_dk + at * d.dim, d.dim, ak, half);
        store_row_f32<DP>(d.part_dv + at * d.dim, d.dim, av, half);
    }
}

// Sums of the key ranges' dq (KIND 0) or the row ranges' dk, dv (1, 2), in a fixed order.
template <class T, int KIND>
__global__ __launch_bounds__(kThreads) void k_cross_sum(CrossDev d) {
    const int rows = KIND == 0 ? d.rows : d.kv_len, n_part = KIND == 0 ? d.splits : d.row_splits;
    const int64_t n = (int64_t)d.batch * d.kv_heads * rows * d.dim;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= n) return;
    const float* part = KIND == 0 ? d.part : KIND == 1 ? d.part_dk : d.part_dv;
    float s = 0.0f;
    for (int k = 0; k < n_part; ++k) s += part[k * n + i];
    const int c = (int)(i % d.dim);
    const int64_t r = i / d.dim, bh = r / rows, b = bh / d.kv_heads;
    const int hk = (int)(bh - b * d.kv_heads), row = (int)(r - bh * rows);
    if constexpr (KIND == 0) {
        const RowAt a = row_at(d, hk, row);
        static_cast<T*>(d.dq)[b * d.dqs[0] + a.token * d.dqs[1] + a.head * d.dqs[2] + c] = (T)(s * d.scale);
    } else if constexpr (KIND == 1) {
        static_cast<T*>(d.dk)[b * d.dks[0] + row * d.dks[1] + hk * d.dks[2] + c] = (T)(s * d.scale);
    } else {
        static_cast<T*>(d.dv)[b * d.dvs[0] + row * d.dvs[1] + hk * d.dvs[2] + c] = (T)s;
    }
}

// With a mask, or a scale that is not positive (the largest scaled score is then not the scaled
// largest product), scores are formed before the maximum is taken.
bool masked(const CrossDev& d) { return d.mask_kind != PA_MASK_NONE || !(d.scale > 0.0f); }

unsigned blocks_for(int64_t n) { return (unsigned)((n + kThreads - 1) / kThreads); }

template <class T, int DP, bool MASKED, bool RAGGED>
hipError_t forward(const CrossDev& d, hipStream_t st) {
    const int64_t bh = (int64_t)d.batch * d.kv_heads;
    if (d.rows <= 32) k_cross_fwd<T, DP, 4, MASKED, RAGGED><<<(unsigned)(d.splits * bh), kThreads, 0, st>>>(d);
    else k_cross_fwd<T, DP, 1, MASKED, RAGGED><<<(unsigned)((d.rows + 127) / 128 * d.splits * bh), kThreads, 0, st>>>(d);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || d.splits == 1) return e;
    k_cross_join<T><<<(unsigned)((bh * d.rows + 3) / 4), kThreads, 0, st>>>(d);
    return hipGetLastError();
}

template <class T, int DP, bool MASKED, bool RAGGED>
hipError_t backward(const CrossDev& d, hipStream_t st) {
    const int64_t bh = (int64_t)d.batch * d.kv_heads;
    hipError_t e = hipSuccess;
    if (d.rows > 0) {
        k_cross_delta<T><<<(unsigned)((bh * d.rows + 15) / 16), kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (d.dq && d.rows > 0) {
        k_cross_dq<T, DP, MASKED, RAGGED><<<(unsigned)((d.rows + 127) / 128 * d.splits * bh), kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (d.splits > 1) {
            k_cross_sum<T, 0><<<blocks_for(bh * d.rows * d.dim), kThreads, 0, st>>>(d);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    }
    if (d.dk && d.kv_len > 0) {
        k_cross_dkv<T, DP, MASKED, RAGGED><<<(unsigned)((d.kv_len + 127) / 128 * d.row_splits * bh), kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (d.row_splits > 1) {
            k_cross_sum<T, 1><<<blocks_for(bh * d.kv_len * d.dim), kThreads, 0, st>>>(d);
            if ((e = hipGetLastError()) != hipSuccess) return e;
            k_cross_sum<T, 2><<<blocks_for(bh * d.kv_len * d.dim), kThreads, 0, st>>>(d);
            e = hipGetLastError();
        }
    }
    return e;
}

bool ragged(const CrossDev& d) {
    for (const int64_t* p : {d.qs, d.ks, d.vs, d.os, d.dos, d.dqs, d.dks, d.dvs})
        if (p[1] >= kBufferStride) return true;
    return d.dim % 8 != 0;
}

template <class F>
hipError_t dispatch(const CrossDev& d, int dtype, F f) {
    const bool m = masked(d), r = ragged(d);
    auto with = [&](auto t, auto dp) {
        if (m) return r ? f(t, dp, std::true_type{}, std::true_type{}) : f(t, dp, std::true_type{}, std::false_type{});
        return r ? f(t, dp, std::false_type{}, std::true_type{}) : f(t, dp, std::false_type{}, std::false_type{});
    };
    auto wide = [&](auto t) {
        return d.dim > 64 ? with(t, std::integral_constant<int, 128>{}) : with(t, std::integral_constant<int, 64>{});
    };
    return dtype == PA_BF16 ? wide((__bf16)0) : wide((_Float16)0);
}

}  // namespace

// Ranges of the split axis: as many as bring the launch to about two blocks per CU, each of at
// least two tiles.
static void split(int64_t blocks, int64_t length, int tile, int& n, int& each) {
    const int64_t tiles = (length + tile - 1) / tile;
    int64_t want = blocks > 0 ? (512 + blocks - 1) / blocks : 1;
    if (want > tiles / 2) want = tiles / 2;
    if (want < 1) want = 1;
    const int64_t per = (tiles + want - 1) / want;
    each = (int)((per > 0 ? per : 1) * tile);
    n = (int)((tiles + per - 1) / (per > 0 ? per : 1));
    if (n < 1) n = 1;
}

void cross_plan(CrossDev& d, bool backward_pass) {
    const int64_t bh = (int64_t)d.batch * d.kv_heads;
    if (!backward_pass && d.rows <= 32) split(bh, d.kv_len, 128, d.splits, d.split_keys);
    else split((d.rows + 127) / 128 * bh, d.kv_len, 64, d.splits, d.split_keys);
    split((d.kv_len + 127) / 128 * bh, (int64_t)d.group * ((d.q_len + 31) / 32), 1, d.row_splits, d.split_tiles);
}

hipError_t cross_forward(const CrossDev& d, int dtype, hipStream_t st) {
    return dispatch(d, dtype, [&](auto t, auto dp, auto m, auto r) {
        return forward<decltype(t), decltype(dp)::value, decltype(m)::value, decltype(r)::value>(d, st);
    });
}

hipError_t cross_backward(const CrossDev& d, int dtype, hipStream_t st) {
    return dispatch(d, dtype, [&](auto t, auto dp, auto m, auto r) {
        return backward<decltype(t), decltype(dp)::value, decltype(m)::value, decltype(r)::value>(d, st);
    });
}

}  // namespace pa
