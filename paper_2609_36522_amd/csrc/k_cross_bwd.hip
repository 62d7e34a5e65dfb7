// Cross attention, backward, for gfx950 (layout and products: pa_cross.h).
//
// dq tiles the work as the forward pass does (a block owns rows, keys pass by: three products a tile),
// dk and dv the other way round (a wave owns 32 keys, rows pass by: four products a tile). The scores are
// computed in both; no atomics, so results do not depend on the order of blocks.
#include "pa_cross.h"

namespace pa {

namespace {

// A row's statistics (m, log of the sum) as the backward pass uses them: without a mask hi = log2 of the sum
// of all weights (lo unused), with one the maximum and the log2 of the sum past it apart. A row that sees
// no key has weights 0 whatever its scores.
template <int MASK>
__device__ __forceinline__ void row_stats(float m, float ll, float& hi, float& lo) {
    const bool empty = ll == -INFINITY;
    hi = MASK ? (empty ? 0.0f : m) : (empty ? INFINITY : (m + ll) * kLog2e);
    lo = empty ? INFINITY : ll * kLog2e;
}
template <int MASK>
__device__ __forceinline__ float weight(float s, float scale, float f, float bias, float hi, float lo) {
    return __builtin_amdgcn_exp2f(MASK ? fmaf(fmaf(s, scale, bias) - hi, kLog2e, -lo) : fmaf(s, f, -hi));
}

// dS on its way to 16 bits. Its size follows the incoming gradient and, as weights are about 1 / keys, the number
// of keys: over thousands of them, or with small gradients, it lies below fp16's normal numbers (whose
// rounding is absolute), with large ones beyond its range. So for fp16 each accumulator column (a row's dq, a
// key's dk: a lane and its other half) has a power of two that dS is multiplied by and that is taken out in fp32
// at the end. It follows the largest |dS| seen: where the next one would pass 2^15, it and the accumulators come
// down so that this |dS| lies in [2^9, 2^10), so that rounding stays relative for what is up to 2^23 times smaller
// and accumulators are rescaled when the maximum grew by 2^5, not each time. bf16 has fp32's exponents.
// Error of dq and dk by their norms over 16384 keys (64 wide, 150 rows), for |do| around 1, 1e-2 and 1e-3: 3e-4
// each (dS as it is: 3e-4, 1.1e-3, 1.1e-2). It costs 3% of a training step: 284 and 294 us for the 1541 keys below.
template <class T>
constexpr bool kNarrow = std::is_same<T, _Float16>::value;
template <class T>
constexpr float kFirstPower = kNarrow<T> ? 0x1p100f : 1.0f;      // before a dS has been seen

__device__ __forceinline__ float inverse_power(float f) {       // of a power of two
    return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, f));
}

template <class T, int DB>
__device__ __forceinline__ void fit(f32x16& ds, float& power, f32x16 (&acc)[DB]) {
    if constexpr (kNarrow<T>) {
        float top = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, fabsf(ds[r]));
        const uint32_t u = __builtin_bit_cast(uint32_t, top);
        const auto x = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        top = fmaxf(__builtin_bit_cast(float, (uint32_t)x[0]), __builtin_bit_cast(float, (uint32_t)x[1]));
        const bool past = top * power > 0x1p15f;
        if (__any(past)) {
            // 2^9 / 2^e for top in [2^e, 2^(e + 1)): e is above -86 here.
            const float p = __builtin_bit_cast(float, ((2u * 127 + 9) << 23) - (__builtin_bit_cast(uint32_t, top) & 0x7f800000u));
            const float a = past ? p * inverse_power(power) : 1.0f;
            power = past ? p : power;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][r] *= a;
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) ds[r] *= power;
    }
}

// The accumulators without their power.
template <class T, int DB>
__device__ __forceinline__ void unscale(f32x16 (&acc)[DB], float power) {
    if constexpr (kNarrow<T>) {
        const float f = inverse_power(power);
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][r] *= f;
    }
}

// dk, dv take P itself as an operand, times 2^kLift: a key with little weight has all of its P below fp16's
// normal numbers (keys of weights around 3e-8: dv off by its own size), while P is at most 1 (and a rounding of
// the statistics, for which fp16 leaves two more bits).
template <class T>
constexpr float kLift = kNarrow<T> ? 14.0f : 0.0f;
template <class T>
constexpr float kLifted = kNarrow<T> ? 0x1p14f : 1.0f;

// Where dk, dv find the statistics of 32 tokens of a query head: hi, lo (of lifted weights) and delta, 32 of each.
__device__ __forceinline__ float* tile_stats(const CrossDev& d, int b, RowAt r) {
    const int64_t head = (int64_t)b * d.q_heads + r.head, tiles = (d.q_len + 31) / 32;
    return d.row_stats + (head * tiles + (r.token >> 5)) * 96 + (r.token & 31);
}
template <class T, int MASK>
__device__ __forceinline__ void put_stats(const CrossDev& d, int b, RowAt r, float hi, float lo, float delta) {
    float* out = tile_stats(d, b, r);
    out[0] = MASK ? hi : hi - kLift<T>;
    out[32] = lo - kLift<T>;
    out[64] = delta;
}

// The rows' statistics where dq, which writes them on its way, is not asked for: 16 lanes per row of
// [batch][q_len][q_heads].
template <class T, int MASK>
__global__ __launch_bounds__(kThreads) void k_cross_stats(CrossDev d) {
    const int64_t n = (int64_t)d.batch * d.q_heads * d.q_len;
    const int64_t i = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int64_t at = i < n ? i : n - 1;
    const int c = (threadIdx.x & 15) * 8;
    const int h = (int)(at % d.q_heads);
    const int64_t bt = at / d.q_heads;
    const int t = (int)(bt % d.q_len), b = (int)(bt / d.q_len);
    const Pack8<T> po = load8(static_cast<const T*>(d.o) + b * d.os[0] + t * d.os[1] + h * d.os[2], c, d.dim);
    const Pack8<T> pd = load8(static_cast<const T*>(d.d_o) + b * d.dos[0] + t * d.dos[1] + h * d.dos[2], c, d.dim);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (float)po.v[e] * (float)pd.v[e];
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) s += __shfl_xor(s, off, 64);
    if (i < n && (threadIdx.x & 15) == 0) {
        const int64_t sat = stat_at(d, b, {t, h});
        float hi, lo;
        row_stats<MASK>(d.stats[sat * 2], d.stats[sat * 2 + 1], hi, lo);
        put_stats<T, MASK>(d, b, {t, h}, hi, lo, s);
    }
}

// dq: the forward pass's tiling; a lane owns a row, K and V tiles pass by. Bound by the products and the
// LDS reads that feed them: 2 x 2309 tokens, 16 heads over 4 of 80, 1541 keys in fp16 94 us (matrix
// units busy 32%).
//
// delta, the sum of do * o over the head, equals the sum of P dP over the keys. The first takes the rounded
// o: its error is one of o's rounding, common to the row's keys, which is lost beside dS's own rounding
// where many keys share the weight. Up to kExactKeys keys (EXACT) the second is formed in fp32 by a pass of
// its own over the (few) tiles: the gradients' error at 77 keys is 1.4 instead of 1.6 times the output's
// rounding. The rule goes by kv_len, which the host knows: a sample with few visible keys among more has the
// first form's error (1.5 to 1.65 times over hundreds to thousands of keys).
constexpr int kExactKeys = 256;

template <class T, int KS, int MASK, int WIDTH, bool EXACT>
__global__ __launch_bounds__(kThreads, 2) void k_cross_dq(CrossDev d) {
    constexpr int DP = KS <= 4 ? 64 : 128, DB = (KS + 1) / 2, KEYS = 64, ROWS = 128;
    constexpr bool DIRECT = WIDTH == kWhole;
    typedef typename Vec<T>::v8 v8;
    __shared__ __align__(16) T tiles[2][2][KEYS * DP];
    __shared__ __align__(16) float bias[2][MASK ? KEYS : 4];

    const Work wk = work_at(d);
    const int tile = wk.tile, b = wk.b, hk = wk.hk;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + w * 32 + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);
    const int64_t sat = stat_at(d, b, ra);

    const int klen = sample_keys(d, b);
    const int kbeg = wk.split * d.split_keys;
    const int kend = wk.part < 0 || klen < kbeg + d.split_keys ? klen : kbeg + d.split_keys;
    const T* kb = static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2];
    const T* vb = static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2];
    // Tiles of the key range, once or twice.
    const int n = kend > kbeg ? (kend - kbeg + KEYS - 1) / KEYS : 0, steps = EXACT ? 2 * n : n;
    auto key_at = [&](int i) { return kbeg + (EXACT && i >= n ? i - n : i) * KEYS; };
    KvStage<T, DP, KEYS, MASK, WIDTH, DIRECT> st(d);
    if (steps > 0) {
        st.load(d, kb, vb, kbeg, kend, tiles[0][0], tiles[0][1]);
        st.load_mask(d, b, kbeg, kend);
    }

    v8 q[KS], g[KS];
    load_row<T, KS, WIDTH>(g, static_cast<const T*>(d.d_o) + b * d.dos[0] + ra.token * d.dos[1] + ra.head * d.dos[2], d.dim, half, valid);
    float delta = 0.0f;
    if constexpr (!EXACT) {
        load_row<T, KS, WIDTH>(q, static_cast<const T*>(d.o) + b * d.os[0] + ra.token * d.os[1] + ra.head * d.os[2], d.dim, half, valid);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int i = 0; i < 8; ++i) delta = fmaf((float)g[ks][i], (float)q[ks][i], delta);
        delta += __shfl_xor(delta, 32, 64);
    }
    load_row<T, KS, WIDTH>(q, static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2], d.dim, half, valid);
    float hi, lo;
    row_stats<MASK>(d.stats[sat * 2], d.stats[sat * 2 + 1], hi, lo);
    const float f = d.scale * kLog2e;
    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x16{};
    float power = kFirstPower<T>;

    if (DIRECT && steps > 1) {
        st.load(d, kb, vb, key_at(1), kend, tiles[1][0], tiles[1][1]);
        wait_loads<decltype(st)::kLoads>();
    } else {
        wait_loads();
    }
    if (steps > 0) st.arrive(tiles[0][0], tiles[0][1], bias[0], d.dim);
    if (steps > 1) {
        if (!DIRECT) st.load(d, kb, vb, key_at(1), kend, tiles[1][0], tiles[1][1]);
        st.load_mask(d, b, key_at(1), kend);
    }
    lds_barrier();
    for (int i = 0; i < steps; ++i) {
        const int p = i & 1, k0 = key_at(i);
        const T* kt = tiles[p][0];
        const T* vt = tiles[p][1];
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            if (nt == 1 && k0 + 32 >= kend) break;
            f32x16 s = f32x16{}, e = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = mma(read_rows<T, DP>(kt, nt * 32 + (lane & 31), ks, half), q[ks], s);
                e = mma(read_rows<T, DP>(vt, nt * 32 + (lane & 31), ks, half), g[ks], e);
            }
            if (!MASK && k0 + nt * 32 + 32 > kend) {
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (k0 + nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= kend) s[r] = -INFINITY;
            }
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                float4 bv = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if constexpr (MASK != kNoMask) bv = *reinterpret_cast<const float4*>(&bias[p][nt * 32 + 8 * g4 + 4 * half]);
                const float bs[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 4 * g4 + j;
                    s[r] = weight<MASK>(s[r], d.scale, f, bs[j], hi, lo);
                }
            }
            if (EXACT && i < n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) delta = fmaf(s[r], e[r], delta);
            } else {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] *= e[r] - delta;
                fit<T>(s, power, acc);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const v8 ds = pack<T>(s, t);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
                        acc[db] = mma(read_cols<T, DP>(kt, nt * 32 + t * 16, db, lane), ds, acc[db]);
                }
            }
        }
        if (EXACT && i == n - 1) delta += __shfl_xor(delta, 32, 64);
        if (i + 1 < steps) {
            wait_loads();
            st.arrive(tiles[p ^ 1][0], tiles[p ^ 1][1], bias[p ^ 1], d.dim);
        }
        lds_barrier();
        if (i + 2 < steps) {                 // into the buffer that every wave has left
            st.load(d, kb, vb, key_at(i + 2), kend, tiles[p][0], tiles[p][1]);
            st.load_mask(d, b, key_at(i + 2), kend);
        }
    }
    if (wk.split == 0 && valid && half == 0) put_stats<T, MASK>(d, b, ra, hi, lo, delta);
    unscale<T>(acc, power);
    if (wk.part < 0) {
        T* out = static_cast<T*>(d.dq) + b * d.dqs[0] + ra.token * d.dqs[1] + ra.head * d.dqs[2];
        store_row<T, DB, WIDTH>(out, d.dim, acc, d.scale, half, valid);
    } else if (valid) {
        const int64_t at = (int64_t)wk.part * ROWS + (row - tile * ROWS);
        store_row_f32<DB>(d.part + at * d.dim, d.dim, acc, half);
    }
}

// The same for at most 128 keys and a head width of at most 64: all keys' scores and dP stay in registers
// between the pass that forms delta and the one that uses it: 8 x 1024 tokens, 16 heads of 64, 77 keys 20 us.
constexpr int kShortKeys = 128;

template <class T, int MASK, int WIDTH>
__global__ __launch_bounds__(kThreads, 2) void k_cross_dq_short(CrossDev d) {
    constexpr int KS = 4, DP = 64, DB = 2, KEYS = kShortKeys, ROWS = 128, NT = KEYS / 32;
    constexpr bool DIRECT = WIDTH == kWhole;
    typedef typename Vec<T>::v8 v8;
    __shared__ __align__(16) T tiles[2][KEYS * DP];
    __shared__ __align__(16) float bias[MASK ? KEYS : 4];

    const Work wk = work_at(d);
    const int tile = wk.tile, b = wk.b, hk = wk.hk;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = threadIdx.x >> 6;
    const int row = tile * ROWS + w * 32 + (lane & 31);
    const bool valid = row < d.rows;
    const RowAt ra = row_at(d, hk, valid ? row : 0);
    const int64_t sat = stat_at(d, b, ra);
    const int kend = sample_keys(d, b);
    KvStage<T, DP, KEYS, MASK, WIDTH, DIRECT> st(d);
    if (kend > 0) {
        st.load(d, static_cast<const T*>(d.k) + b * d.ks[0] + hk * d.ks[2], static_cast<const T*>(d.v) + b * d.vs[0] + hk * d.vs[2],
                0, kend, tiles[0], tiles[1]);
        st.load_mask(d, b, 0, kend);
    }
    v8 q[KS], g[KS];
    load_row<T, KS, WIDTH>(q, static_cast<const T*>(d.q) + b * d.qs[0] + ra.token * d.qs[1] + ra.head * d.qs[2], d.dim, half, valid);
    load_row<T, KS, WIDTH>(g, static_cast<const T*>(d.d_o) + b * d.dos[0] + ra.token * d.dos[1] + ra.head * d.dos[2], d.dim, half, valid);
    float hi, lo, delta = 0.0f;
    row_stats<MASK>(d.stats[sat * 2], d.stats[sat * 2 + 1], hi, lo);
    const float f = d.scale * kLog2e;
    wait_loads();
    if (kend > 0) st.arrive(tiles[0], tiles[1], bias, d.dim);
    lds_barrier();

    f32x16 s[NT], e[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (nt * 32 >= kend) break;
        s[nt] = e[nt] = f32x16{};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            s[nt] = mma(read_rows<T, DP>(tiles[0], nt * 32 + (lane & 31), ks, half), q[ks], s[nt]);
            e[nt] = mma(read_rows<T, DP>(tiles[1], nt * 32 + (lane & 31), ks, half), g[ks], e[nt]);
        }
        if (!MASK && nt * 32 + 32 > kend) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (nt * 32 + 8 * (r >> 2) + 4 * half + (r & 3) >= kend) s[nt][r] = -INFINITY;
        }
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
            float4 bv = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if constexpr (MASK != kNoMask) bv = *reinterpret_cast<const float4*>(&bias[nt * 32 + 8 * g4 + 4 * half]);
            const float bs[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = 4 * g4 + j;
                s[nt][r] = weight<MASK>(s[nt][r], d.scale, f, bs[j], hi, lo);
                delta = fmaf(s[nt][r], e[nt][r], delta);
            }
        }
    }
    delta += __shfl_xor(delta, 32, 64);
    f32x16 acc[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) acc[i] = f32x16{};
    float power = kFirstPower<T>;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        if (nt * 32 >= kend) break;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[nt][r] *= e[nt][r] - delta;
        fit<T>(s[nt], power, acc);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v8 ds = pack<T>(s[nt], t);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mma(read_cols<T, DP>(tiles[0], nt * 32 + t * 16, db, lane), ds, acc[db]);
        }
    }
    if (valid && half == 0) put_stats<T, MASK>(d, b, ra, hi, lo, delta);
    unscale<T>(acc, power);
    T* out = static_cast<T*>(d.dq) + b * d.dqs[0] + ra.token * d.dqs[1] + ra.head * d.dqs[2];
    store_row<T, DB, WIDTH>(out, d.dim, acc, d.scale, half, valid);
}

// dk, dv: a wave owns 32 keys (K and V in registers), tiles of 32 tokens of one query head and their
// statistics pass by, up to three on their way; the heads of the group one after the other. The sizes of dq's
// comments: 132 us over 1541 keys in fp16 (matrix units busy 33%; 416 of the 512 places for blocks are taken), 20 us
// over 77, of which some 15 are a block's start and the writing of its partial sums (with 256 or 768 ranges
// in place of 512: 20.8 and 23.8).
template <class T, int KS, int MASK, int WIDTH>
__global__ __launch_bounds__(kThreads, KS <= 6 ? 2 : 1) void k_cross_dkv(CrossDev d) {
    constexpr int DP = KS <= 4 ? 64 : 128, DB = (KS + 1) / 2, KEYS = 128, ROWS = 32;
    constexpr bool DIRECT = WIDTH == kWhole;
    constexpr int STAGES = DIRECT ? 4 : 2;
    typedef typename Vec<T>::v8 v8;
    typedef Stage<T, DP, ROWS, WIDTH, DIRECT> S;
    __shared__ __align__(16) T tiles[STAGES][2][ROWS * DP];      // [][q, do]
    __shared__ __align__(16) float stat[STAGES][4][256];         // [][wave]: wave 0's holds hi, lo, delta, 32 of each

    const int key_tiles = (d.kv_len + KEYS - 1) / KEYS;
    int id = xcd_order(blockIdx.x, gridDim.x);
    const int tile = id % key_tiles;
    id /= key_tiles;
    const int split = id % d.row_splits, bh = id / d.row_splits;
    const int b = bh / d.kv_heads, hk = bh - b * d.kv_heads;
    const int lane = threadIdx.x & 63, half = lane >> 5, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int key = tile * KEYS + w * 32 + (lane & 31);
    const int klen = sample_keys(d, b);

    const int head_tiles = (d.q_len + ROWS - 1) / ROWS;
    const int tbeg = split * d.split_tiles;
    int tend = d.group * head_tiles;
    if (tend > tbeg + d.split_tiles) tend = tbeg + d.split_tiles;
    if (tile * KEYS >= klen) tend = tbeg;
    const T* qb = static_cast<const T*>(d.q) + b * d.qs[0] + (int64_t)hk * d.group * d.qs[2];
    const T* gb = static_cast<const T*>(d.d_o) + b * d.dos[0] + (int64_t)hk * d.group * d.dos[2];
    S sq(d.dim, d.qs[1]), sg(d.dim, d.dos[1]);
    constexpr int LOADS = 2 * S::kPieces + 1;                    // of a thread for one tile
    auto rows_of = [&](int it) { return d.q_len - it % head_tiles * ROWS; };
    auto load = [&](int it, int p) {
        const int gh = it / head_tiles, r0 = (it - gh * head_tiles) * ROWS;
        sq.load(qb + gh * d.qs[2] + r0 * d.qs[1], d.qs[1], d.q_len - r0, d.dim, tiles[p][0]);
        sg.load(gb + gh * d.dos[2] + r0 * d.dos[1], d.dos[1], d.q_len - r0, d.dim, tiles[p][1]);
        // 96 floats: 24 lanes of wave 0 (the other waves fill their own part with zeros, to issue as many loads).
        load_lds(buffer_at(tile_stats(d, b, {r0, hk * d.group + gh})), stat[p][w], w == 0 && lane < 24 ? lane * 16 : kNowhere, 0);
    };
    auto arrive = [&](int it, int p) {
        sq.arrive(tiles[p][0], d.dim);
        sg.arrive(tiles[p][1], d.dim);
        const int i = threadIdx.x;                               // a row that does not exist sees no key
        if (i < ROWS && i >= rows_of(it)) {
            stat[p][0][i] = MASK ? 0.0f : INFINITY;
            stat[p][0][i + 32] = INFINITY;
            stat[p][0][i + 64] = 0.0f;
        }
    };
#pragma unroll
    for (int i = 0; i < (DIRECT ? STAGES - 1 : 1); ++i)
        if (tbeg + i < tend) load(tbeg + i, i);

    const int at = key < d.kv_len ? key : 0;
    bool seen = key < klen;
    float bias = -INFINITY;                  // of the lane's key
    if constexpr (MASK != kNoMask) {
        const float v = mask_bias<MASK>(mask_load<MASK>(d, b, at));
        bias = seen ? v : -INFINITY;
        seen = bias != -INFINITY;
    }
    v8 kr[KS], vr[KS];
    load_row<T, KS, WIDTH>(kr, static_cast<const T*>(d.k) + b * d.ks[0] + at * d.ks[1] + hk * d.ks[2], d.dim, half, seen);
    load_row<T, KS, WIDTH>(vr, static_cast<const T*>(d.v) + b * d.vs[0] + at * d.vs[1] + hk * d.vs[2], d.dim, half, seen);
    f32x16 ak[DB], av[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i) ak[i] = av[i] = f32x16{};
    float power = kFirstPower<T>;            // of dk
    const float f = d.scale * kLog2e;
    const bool busy = tile * KEYS + w * 32 < klen;       // the wave has keys

    wait_loads();
    if (tbeg < tend) arrive(tbeg, 0);
    if (!DIRECT && tbeg + 1 < tend) load(tbeg + 1, 1);
    lds_barrier();
    for (int it = tbeg; it < tend; ++it) {
        const int p = (it - tbeg) % STAGES, p1 = (it + 1 - tbeg) % STAGES;
        if (DIRECT && it + STAGES - 1 < tend) load(it + STAGES - 1, (it + STAGES - 1 - tbeg) % STAGES);
        const T* qt = tiles[p][0];
        const T* gt = tiles[p][1];
        if (busy) {
            f32x16 s = f32x16{}, e = f32x16{};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                s = mma(read_rows<T, DP>(qt, lane & 31, ks, half), kr[ks], s);
                e = mma(read_rows<T, DP>(gt, lane & 31, ks, half), vr[ks], e);
            }
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4) {
                float4 st[3];
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (MASK || i != 1) st[i] = *reinterpret_cast<const float4*>(&stat[p][0][i * 32 + 8 * g4 + 4 * half]);
                const float hi[4] = {st[0].x, st[0].y, st[0].z, st[0].w}, dl[4] = {st[2].x, st[2].y, st[2].z, st[2].w};
                float lo[4] = {};
                if constexpr (MASK != kNoMask) lo[0] = st[1].x, lo[1] = st[1].y, lo[2] = st[1].z, lo[3] = st[1].w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 4 * g4 + i;
                    s[r] = weight<MASK>(s[r], d.scale, f, bias, hi[i], lo[i]);
                    e[r] = s[r] * (e[r] - dl[i]);
                }
            }
            fit<T>(e, power, ak);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const v8 pw = pack<T>(s, t), ds = pack<T>(e, t);
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    av[db] = mma(read_cols<T, DP>(gt, t * 16, db, lane), pw, av[db]);
                    ak[db] = mma(read_cols<T, DP>(qt, t * 16, db, lane), ds, ak[db]);
                }
            }
        }
        if (it + 1 < tend) {
            if (DIRECT && it + STAGES - 1 < tend) wait_loads<(STAGES - 2) * LOADS>();    // the next tile is there
            else wait_loads();
            arrive(it + 1, p1);
        }
        lds_barrier();
        if (!DIRECT && it + 2 < tend) load(it + 2, p);
    }
    if (!seen) {                             // the lane's columns held weights of a key of zeros
#pragma unroll
        for (int i = 0; i < DB; ++i) ak[i] = av[i] = f32x16{};
    }
    unscale<T>(ak, power * kLifted<T>);
    unscale<T>(av, kLifted<T>);
    const bool valid = key < d.kv_len;
    if (d.row_splits == 1) {
        T* ok = static_cast<T*>(d.dk) + b * d.dks[0] + key * d.dks[1] + hk * d.dks[2];
        T* ov = static_cast<T*>(d.dv) + b * d.dvs[0] + key * d.dvs[1] + hk * d.dvs[2];
        store_row<T, DB, WIDTH>(ok, d.dim, ak, d.scale, half, valid);
        store_row<T, DB, WIDTH>(ov, d.dim, av, 1.0f, half, valid);
    } else if (valid) {
        const int64_t out = ((int64_t)split * d.batch * d.kv_heads + bh) * d.kv_len + key;
        store_row_f32<DB>(d.part_dk + out * d.dim, d.dim, ak, half);
        store_row_f32<DB>(d.part_dv + out * d.dim, d.dim, av, half);
    }
}

// dq of the split row tiles from their key ranges, in a fixed order; four columns a thread. Bound by memory.
template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_sum_dq(CrossDev d) {
    const int quads = (d.dim + 3) / 4;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, r = i / quads;
    const int c = (int)(i - r * quads) * 4;
    const int rt = (int)(r / d.tile_rows), lr = (int)(r - (int64_t)rt * d.tile_rows), t = d.whole + rt;
    if (t >= d.tiles) return;
    const int row_tiles = (d.rows + d.tile_rows - 1) / d.tile_rows, bh = t / row_tiles, row = (t - bh * row_tiles) * d.tile_rows + lr;
    if (row >= d.rows) return;
    const int b = bh / d.kv_heads;
    const RowAt a = row_at(d, bh - b * d.kv_heads, row);
    const float4 s = sum_parts(d.part + ((int64_t)rt * d.splits * d.tile_rows + lr) * d.dim, (int64_t)d.tile_rows * d.dim, d.splits, c, d.dim, [](int) { return 1.0f; });
    store_quad(static_cast<T*>(d.dq) + b * d.dqs[0] + a.token * d.dqs[1] + a.head * d.dqs[2], s, d.scale, c, d.dim);
}

// dk (blockIdx.y 0) and dv (1) from their row ranges, in a fixed order; four columns a thread. Bound by memory:
// 5.2 us for the 77 keys, 7.6 for the 1541.
template <class T>
__global__ __launch_bounds__(kThreads) void k_cross_sum_dkv(CrossDev d) {
    const int quads = (d.dim + 3) / 4;
    const int64_t n = (int64_t)d.batch * d.kv_heads * d.kv_len;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, r = i / quads;
    if (r >= n) return;
    const int c = (int)(i - r * quads) * 4;
    const float4 s = sum_parts((blockIdx.y ? d.part_dv : d.part_dk) + r * d.dim, n * d.dim, d.row_splits, c, d.dim,
                               [](int) { return 1.0f; });
    const int64_t bh = r / d.kv_len, b = bh / d.kv_heads;
    const int hk = (int)(bh - b * d.kv_heads), key = (int)(r - bh * d.kv_len);
    if (blockIdx.y) store_quad(static_cast<T*>(d.dv) + b * d.dvs[0] + key * d.dvs[1] + hk * d.dvs[2], s, 1.0f, c, d.dim);
    else store_quad(static_cast<T*>(d.dk) + b * d.dks[0] + key * d.dks[1] + hk * d.dks[2], s, d.scale, c, d.dim);
}

template <class T, int KS, int MASK, int WIDTH>
hipError_t backward(const CrossDev& d, hipStream_t st) {
    const int64_t bh = (int64_t)d.batch * d.kv_heads;
    hipError_t e = hipSuccess;
    if (d.dq && d.rows > 0) {
        const unsigned blocks = (unsigned)(d.whole + (d.tiles - d.whole) * d.splits);
        if (KS == 4 && d.kv_len <= kShortKeys) k_cross_dq_short<T, MASK, WIDTH><<<blocks, kThreads, 0, st>>>(d);
        else if (d.kv_len <= kExactKeys) k_cross_dq<T, KS, MASK, WIDTH, true><<<blocks, kThreads, 0, st>>>(d);
        else k_cross_dq<T, KS, MASK, WIDTH, false><<<blocks, kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (d.whole < d.tiles) {
            k_cross_sum_dq<T><<<blocks_for((int64_t)(d.tiles - d.whole) * d.tile_rows * ((d.dim + 3) / 4), kThreads), kThreads, 0, st>>>(d);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
    } else if (d.rows > 0) {
        k_cross_stats<T, MASK><<<blocks_for(bh * d.rows, 16), kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (d.dk && d.kv_len > 0) {
        k_cross_dkv<T, KS, MASK, WIDTH><<<(unsigned)((d.kv_len + 127) / 128 * d.row_splits * bh), kThreads, 0, st>>>(d);
        if ((e = hipGetLastError()) != hipSuccess) return e;
        if (d.row_splits > 1) {
            k_cross_sum_dkv<T><<<dim3(blocks_for(bh * d.kv_len * ((d.dim + 3) / 4), kThreads), 2), kThreads, 0, st>>>(d);
            e = hipGetLastError();
        }
    }
    return e;
}

}  // namespace

// Blocks that the machine holds at once: two on each of its 256 CUs.
constexpr int64_t kSlots = 512;

// Splits `length` tiles of an axis over as many ranges as `room` allows, each of at least two tiles.
static void split(int64_t room, int64_t length, int& n, int& each) {
    int64_t want = room < length / 2 ? room : length / 2;
    if (want < 1) want = 1;
    const int64_t per = length > 0 ? (length + want - 1) / want : 1;
    each = (int)per;
    n = length > 0 ? (int)((length + per - 1) / per) : 1;
}

// Row tiles that fill the machine in whole rounds take all keys in one block. The rest, at most half a
// round, would leave most CUs idle for as long as a whole round takes: they are split over the keys, and
// their partial results joined. (2304 tokens, 32 heads, 4096 keys: 576 tiles are one round and 64 more.)
void cross_plan(CrossDev& d, bool backward_pass) {
    const int64_t bh = (int64_t)d.batch * d.kv_heads;
    const int key_tile = !backward_pass && d.rows <= 32 ? 128 : 64;
    d.tile_rows = !backward_pass && d.rows <= 32 ? 32 : 128;
    const int64_t tiles = (d.rows + d.tile_rows - 1) / d.tile_rows * bh, rest = tiles % kSlots;
    d.tiles = (int)tiles;
    d.whole = (int)tiles;
    split(rest > 0 ? kSlots / rest : 1, ((int64_t)d.kv_len + key_tile - 1) / key_tile, d.splits, d.split_keys);
    d.split_keys *= key_tile;
    if (backward_pass && d.kv_len <= kExactKeys) d.splits = 1;      // a block sees all keys
    if (d.splits > 1) d.whole = (int)(tiles - rest);
    // dk, dv: one block a CU above a head width of 96.
    const int64_t key_blocks = ((int64_t)d.kv_len + 127) / 128 * bh;
    split((d.dim <= 96 ? kSlots : kSlots / 2) / (key_blocks > 0 ? key_blocks : 1), (int64_t)d.group * ((d.q_len + 31) / 32),
          d.row_splits, d.split_tiles);
}

hipError_t cross_backward(const CrossDev& d, int dtype, hipStream_t st) {
    return dispatch(d, dtype, [&](auto t, auto ks, auto mk, auto wd) {
        return backward<decltype(t), decltype(ks)::value, decltype(mk)::value, decltype(wd)::value>(d, st);
    });
}

}  // namespace pa
