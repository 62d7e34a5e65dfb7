// Cross attention, forward, for gfx950 (layout and products: pa_cross.h).
//
// One pass over the keys with a running maximum and sum in fp32. Where the rows are too few to fill the
// machine the keys are split over blocks, whose unnormalised outputs a second kernel joins.
#include "pa_cross.h"

namespace pa {

namespace {

// Scaled scores plus the biases of their 32 keys.
__device__ __forceinline__ void add_bias(f32x16& s, float scale, const float* bias, int half) {
#pragma unroll
    for (int g4 = 0; g4 < 4; ++g4) {
        const float4 bv = *reinterpret_cast<const float4*>(bias + 8 * g4 + 4 * half);
        s[4 * g4] = fmaf(s[4 * g4], scale, bv.x);
        s[4 * g4 + 1] = fmaf(s[4 * g4 + 1], scale, bv.y);
        s[4 * g4 + 2] = fmaf(s[4 * g4 + 2], scale, bv.z);
        s[4 * g4 + 3] = fmaf(s[4 * g4 + 3], scale, bv.w);
    }
}

// Rows fill the block: four waves of 32 rows share stages of 64 keys, double buffered (a stage's loads
// are in flight during the products of the one before).
//
// Few keys: bound by memory (32 x 1024 tokens, 16 heads of 64, up to 77 keys: 34 to 38 us, 139 MB, 3.7 to 4.1
// TB/s). Many: by the products and, on the same waves, the exponentials between them (2 x 2304 tokens, 16
// heads of 128, 4096 keys: 161 us, 960 TFLOP/s, matrix units busy 50% of the time; 64 rows a wave, or two
// groups of waves that take products and exponentials in turn, are slower: 410 and 203 us, not built).
//
// The accumulator is rescaled only when some row's maximum has grown by a factor of more than 2^kSlack in
// weight since the last time, so weights reach 2^kSlack, which the element types hold as exactly as 1.
constexpr float kSlack = 8.0f;

template <class T, int KS, int MASK, int WIDTH>
__global__ __launch_bounds__(kThreads, 2) void k_cross_fwd(CrossDev d) {
    constexpr int DP = KS <= 4 ? 64 : 128, DB = (KS + 1) / 2, KEYS = 64, ROWS = 128, NT = 2;
    typedef typename Vec<T>::v8 v8;
    __shared__ __align__(16) T tiles[2][2][KEYS * DP];      // [stage parity][K, V]
    __shared__ __align__(16) float bias[2][MASK ? KEYS : 4];

    const Work wk = work_at(d);
    const int tile = wk.tile, b = wk.b, hk = wk.hk;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + w * 32 + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);

    const int klen = sample_keys(d, b);
    const int kbeg = wk.split * d.split_keys;
    const int kend = wk.part < 0 || klen < kbeg + d.split_keys ? klen : kbeg + d.split_keys;
    const T* kb = static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2];
    const T* vb = static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2];
    constexpr bool DIRECT = WIDTH == kWhole;
    KvStage<T, DP, KEYS, MASK, WIDTH, DIRECT> st(d);
    if (kbeg < kend) {
        st.load(d, kb, vb, kbeg, kend, tiles[0][0], tiles[0][1]);
        st.load_mask(d, b, kbeg, kend);
    }

    const T* qp = static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2];
    v8 q[KS];
    load_row<T, KS, WIDTH>(q, qp, d.dim, half, valid);

    // Scores in units of 1/f: x f is the exponent of 2. With a mask x is the scaled, biased score.
    const float f = MASK ? kLog2e : d.scale * kLog2e;
    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x16{};
    float m = -INFINITY, l = 0.0f;

    const bool second = kbeg + KEYS < kend;
    if (DIRECT && second) {
        st.load(d, kb, vb, kbeg + KEYS, kend, tiles[1][0], tiles[1][1]);
        wait_loads<decltype(st)::kLoads>();
    } else {
        wait_loads();
    }
    if (kbeg < kend) st.arrive(tiles[0][0], tiles[0][1], bias[0], d.dim);
    if (second) {
        if (!DIRECT) st.load(d, kb, vb, kbeg + KEYS, kend, tiles[1][0], tiles[1][1]);
        st.load_mask(d, b, kbeg + KEYS, kend);
    }
    lds_barrier();
    int p = 0;
    for (int k0 = kbeg; k0 < kend; k0 += KEYS, p ^= 1) {
        const T* kt = tiles[p][0];
        const T* vt = tiles[p][1];
        f32x16 s[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            s[nt] = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) s[nt] = mma(read_rows<T, DP>(kt, nt * 32 + (lane & 31), ks, half), q[ks], s[nt]);
        }
        if constexpr (MASK != kNoMask) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) add_bias(s[nt], d.scale, bias[p] + nt * 32, half);
        } else if (k0 + KEYS > kend) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= kend) s[nt][r] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[nt][r]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        if (__any((top - m) * f > kSlack)) {
            const float n = fmaxf(top, m);
            const float a = __builtin_amdgcn_exp2f((m - (n == -INFINITY ? 0.0f : n)) * f);
            m = n;
            l *= a;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= a;
        }
        const float base = m == -INFINITY ? 0.0f : m;       // nothing seen yet: every weight is 0
        const float mf = base * f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                // With a mask the difference comes first: x may be near the type's lowest value.
                const float e = __builtin_amdgcn_exp2f(MASK ? (s[nt][r] - base) * f : fmaf(s[nt][r], f, -mf));
                s[nt][r] = e;
                l += e;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const v8 e = pack<T>(s[nt], t);
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] = mma(read_cols<T, DP>(vt, nt * 32 + t * 16, db, lane), e, acc[db]);
            }
        }
        if (k0 + KEYS < kend) {
            wait_loads();
            st.arrive(tiles[p ^ 1][0], tiles[p ^ 1][1], bias[p ^ 1], d.dim);
        }
        lds_barrier();
        if (k0 + 2 * KEYS < kend) {          // into the buffer that every wave has left
            st.load(d, kb, vb, k0 + 2 * KEYS, kend, tiles[p][0], tiles[p][1]);
            st.load_mask(d, b, k0 + 2 * KEYS, kend);
        }
    }
    l += __shfl_xor(l, 32, 64);
    const float m_nat = MASK || m == -INFINITY ? m : m * d.scale;
    if (wk.part < 0) {
        T* op = static_cast<T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2];
        store_row<T, DB, WIDTH>(op, d.dim, acc, l == 0.0f ? 0.0f : 1.0f / l, half, valid);   // no key seen: acc is 0
        if (d.stats && valid && half == 0) {
            float* sp = d.stats + stat_at(d, b, ra) * 2;
            sp[0] = m_nat;
            sp[1] = logf(l);
        }
    } else if (valid) {
        const int64_t at = (int64_t)wk.part * ROWS + (row - tile * ROWS);
        store_row_f32<DB>(d.part + at * d.dim, d.dim, acc, half);
        if (half == 0) {
            d.part_stats[at * 2] = m_nat;
            d.part_stats[at * 2 + 1] = l;
        }
    }
}

// At most 32 rows: the four waves take 32 keys each of a 128-key tile for the same rows and are joined at
// the end. Bound by the reading of K and V; two blocks a CU keep 128 KB in flight: 4 samples of
// one token, 32 heads over 8 of 128, 16381 keys 46 to 57 us (4.7 to 5.8 TB/s), the join 4.7.
template <class T, int KS, int MASK, int WIDTH>
__global__ __launch_bounds__(kThreads, 2) void k_cross_few(CrossDev d) {
    constexpr int DP = KS <= 4 ? 64 : 128, DB = (KS + 1) / 2, KEYS = 128, ROWS = 32;
    typedef typename Vec<T>::v8 v8;
    // K tile, V tile; afterwards the waves' accumulators [4][DP][32] in fp32.
    __shared__ __align__(16) T tiles[2 * KEYS * DP];
    __shared__ __align__(16) float bias[MASK ? KEYS : 4];
    __shared__ float wave_m[4][32], wave_l[4][32];
    T* kt = tiles;
    T* vt = tiles + KEYS * DP;

    const Work wk = work_at(d);
    const int tile = wk.tile, b = wk.b, hk = wk.hk;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);

    const T* qp = static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2];
    v8 q[KS];
    load_row<T, KS, WIDTH>(q, qp, d.dim, half, valid);

    const int klen = sample_keys(d, b);
    const int kbeg = wk.split * d.split_keys;
    const int kend = wk.part < 0 || klen < kbeg + d.split_keys ? klen : kbeg + d.split_keys;
    const T* kb = static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2];
    const T* vb = static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2];

    // Scores in units of 1/f: x f is the exponent of 2. With a mask x is the scaled, biased score.
    const float f = MASK ? kLog2e : d.scale * kLog2e;
    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x16{};
    float m = -INFINITY, l = 0.0f;

    KvStage<T, DP, KEYS, MASK, WIDTH, false> st(d);
    if (kbeg < kend) {
        st.load(d, kb, vb, kbeg, kend, kt, vt);
        st.load_mask(d, b, kbeg, kend);
    }
    for (int k0 = kbeg; k0 < kend; k0 += KEYS) {
        __syncthreads();
        st.arrive(kt, vt, bias, d.dim);
        __syncthreads();
        if (k0 + KEYS < kend) {
            st.load(d, kb, vb, k0 + KEYS, kend, kt, vt);
            st.load_mask(d, b, k0 + KEYS, kend);
        }
        const int koff = w * 32;
        f32x16 s = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) s = mma(read_rows<T, DP>(kt, koff + (lane & 31), ks, half), q[ks], s);
        if constexpr (MASK != kNoMask) {
            add_bias(s, d.scale, bias + koff, half);
        } else if (k0 + KEYS > kend) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (k0 + koff + 8 * (r >> 2) + 4 * half + (r & 3) >= kend) s[r] = -INFINITY;
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
        top = fmaxf(fmaxf(top, __shfl_xor(top, 32, 64)), m);
        const float base = top == -INFINITY ? 0.0f : top;   // nothing seen yet: every weight is 0
        if (__any(top > m)) {
            const float a = __builtin_amdgcn_exp2f((m - base) * f);
            l *= a;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= a;
            m = top;
        }
        const float mf = base * f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            // With a mask the difference comes first: x may be near the type's lowest value.
            s[r] = __builtin_amdgcn_exp2f(MASK ? (s[r] - base) * f : fmaf(s[r], f, -mf));
            l += s[r];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v8 p = pack<T>(s, t);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mma(read_cols<T, DP>(vt, koff + t * 16, db, lane), p, acc[db]);
        }
    }
    l += __shfl_xor(l, 32, 64);
    const float m_nat = MASK || m == -INFINITY ? m : m * d.scale;

    float* wa = reinterpret_cast<float*>(tiles);
    __syncthreads();
#pragma unroll
    for (int db = 0; db < DB; ++db)
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
    const int64_t at = (int64_t)wk.part * ROWS + rr;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T* op = static_cast<T*>(d.o) + b * d.os[0] + oa.token * d.os[1] + oa.head * d.os[2];
    for (int c = threadIdx.x >> 5; c < d.dim; c += 8) {
        float o = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) o += a[i] * wa[(i * DP + c) * 32 + rr];
        if (wk.part < 0) op[c] = (T)(o * inv);
        else d.part[at * d.dim + c] = o;
    }
    if (threadIdx.x < 32) {
        if (wk.part >= 0) {
            d.part_stats[at * 2] = top;
            d.part_stats[at * 2 + 1] = sum;
        } else if (d.stats) {
            float* sp = d.stats + stat_at(d, b, oa) * 2;
            sp[0] = top;
            sp[1] = logf(sum);
        }
    }
}

// The row of the split row tiles that is i-th among their tile_rows each; false past the last.
__device__ __forceinline__ bool split_row(const CrossDev& d, int64_t i, int& b, RowAt& ra, int64_t& part) {
    const int rt = (int)(i / d.tile_rows), lr = (int)(i - (int64_t)rt * d.tile_rows), t = d.whole + rt;
    const int row_tiles = (d.rows + d.tile_rows - 1) / d.tile_rows, bh = t / row_tiles, row = (t - bh * row_tiles) * d.tile_rows + lr;
    if (t >= d.tiles || row >= d.rows) return false;
    b = bh / d.kv_heads;
    ra = row_at(d, bh - b * d.kv_heads, row);
    part = (int64_t)rt * d.splits * d.tile_rows + lr;        // of the first range; the next are tile_rows apart
    return true;
}

// Joins a few key ranges (at most kFewParts): four columns a thread, which forms the row's weights itself.
constexpr int kFewParts = 8;

template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_join(CrossDev d) {
    const int quads = (d.dim + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, r = i / quads;
    const int c = (int)(i - r * quads) * 4;
    int b;
    RowAt ra;
    int64_t part;
    if (!split_row(d, r, b, ra, part)) return;
    const float* ps = d.part_stats + part * 2;
    const int64_t step = (int64_t)d.tile_rows * 2;
    float m[kFewParts], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kFewParts; ++k) {
        m[k] = k < d.splits ? ps[k * step] : -INFINITY;
        top = fmaxf(top, m[k]);
    }
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int k = 0; k < kFewParts; ++k)
        if (k < d.splits) sum = fmaf(__builtin_amdgcn_exp2f((m[k] - base) * kLog2e), ps[k * step + 1], sum);
    const float4 o = sum_parts(d.part + part * d.dim, (int64_t)d.tile_rows * d.dim, d.splits, c, d.dim,
                               [&](int k) { return __builtin_amdgcn_exp2f((ps[k * step] - base) * kLog2e); });
    store_quad(static_cast<T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2], o, sum == 0.0f ? 0.0f : 1.0f / sum, c, d.dim);
    if (d.stats && c == 0) {
        float* sp = d.stats + stat_at(d, b, ra) * 2;
        sp[0] = top;
        sp[1] = logf(sum);
    }
}

// Joins many: a block per row, its waves take every fourth range.
template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_join_many(CrossDev d) {
    __shared__ float o[4][128];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = threadIdx.x;
    int b;
    RowAt ra;
    int64_t part;
    if (!split_row(d, blockIdx.x, b, ra, part)) return;      // the whole block
    const float* ps = d.part_stats + part * 2;
    const int64_t step = (int64_t)d.tile_rows * 2;
    float top = -INFINITY;
    for (int s = lane; s < d.splits; s += 64) top = fmaxf(top, ps[s * step]);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    for (int s = lane; s < d.splits; s += 64) sum += __builtin_amdgcn_exp2f((ps[s * step] - base) * kLog2e) * ps[s * step + 1];
    sum = wave_sum_f32(sum);
    float o0 = 0.0f, o1 = 0.0f;
    const int c0 = lane < d.dim ? lane : 0, c1 = lane + 64 < d.dim ? lane + 64 : 0;
#pragma unroll 4
    for (int s = w; s < d.splits; s += 4) {
        const float a = __builtin_amdgcn_exp2f((ps[s * step] - base) * kLog2e);
        const float* p = d.part + (part + (int64_t)s * d.tile_rows) * d.dim;
        o0 = fmaf(a, p[c0], o0);
        o1 = fmaf(a, p[c1], o1);
    }
    o[w][lane] = o0;
    o[w][lane + 64] = o1;
    __syncthreads();
    T* op = static_cast<T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2];
    if (c < d.dim) op[c] = (T)(((o[0][c] + o[1][c]) + (o[2][c] + o[3][c])) * (sum == 0.0f ? 0.0f : 1.0f / sum));
    if (d.stats && c == 0) {
        float* sp = d.stats + stat_at(d, b, ra) * 2;
        sp[0] = top;
        sp[1] = logf(sum);
    }
}

template <class T, int KS, int MASK, int WIDTH>
hipError_t forward(const CrossDev& d, hipStream_t st) {
    const unsigned blocks = (unsigned)(d.whole + (d.tiles - d.whole) * d.splits);
    if (d.tile_rows == 32) k_cross_few<T, KS, MASK, WIDTH><<<blocks, kThreads, 0, st>>>(d);
    else k_cross_fwd<T, KS, MASK, WIDTH><<<blocks, kThreads, 0, st>>>(d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || d.whole == d.tiles) return e;
    const int64_t rows = (int64_t)(d.tiles - d.whole) * d.tile_rows;
    if (d.splits > kFewParts) k_cross_join_many<T><<<(unsigned)rows, kThreads, 0, st>>>(d);
    else k_cross_join<T><<<blocks_for(rows * ((d.dim + 3) / 4), kThreads), kThreads, 0, st>>>(d);
    return hipGetLastError();
}

}  // namespace

hipError_t cross_forward(const CrossDev& d, int dtype, hipStream_t st) {
    return dispatch(d, dtype, [&](auto t, auto ks, auto mk, auto wd) {
        return forward<decltype(t), decltype(ks)::value, decltype(mk)::value, decltype(wd)::value>(d, st);
    });
}

}  // namespace pa
