// Attention of prompt and chunk rows over the 8-bit cache on the matrix cores.
//
// A workgroup takes a tile of up to 128 rows and a query head, each of its four waves 32 rows, and walks the positions 64 (four blocks) at a time.
// Keys and values go through LDS, the next tile's while one is multiplied: keys as they are, values widened to fp16 once for the four waves.
//
//   scores   S^T[pos, row] = K[pos, :] . Q[row, :] in whole numbers (32x32x32, 8 bits): a query is three base-256 digits (24 bits under its largest
//            entry), kept in registers.
//   sums     O^T[d, row] += V^T[d, pos] W^T[pos, row] (32x32x16, fp16): codes are exact in fp16; W = p 2^e 2^x, e the value's exponent and 2^x the power
//            of two that brings the largest p 2^e of the row so far to 2^9 .. 65504, as two fp16 terms (22 bits).
//
// Which position a row of the score tile is, is free: row 8 b + 4 h + i is slot 4 b + i of block h of a pair, so that lane (row, h) ends with the scores of
// block h, slot by slot, which is what it has to bring as the other operand of the sums.
//
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "ld_q8.h"

using namespace ldd;

namespace {

constexpr int TILE = 64, ROWS = 128;
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

template <int HD>
struct Stage {
    uint4 k[4 * HD];        // [position][piece of 16 dims, swizzled]
    f16x8_t v[8 * HD];      // [block][half][dim]: eight slots
    float unit[256];        // 2^e of the keys, 2^(e - E0) of the values; NaN where a vector is not finite; the rest is room for threads without one
};

// Piece p of position r (block r / 16, slot r % 16), so that eight lanes' pieces of a score operand lie in different banks.
template <int HD>
__device__ __forceinline__ int key_piece(int r, int p) {
    constexpr int N = HD / 16;
    return N == 8 ? r * 8 + (p ^ ((r & 3) | ((r >> 2) & 4))) : r * 4 + (p ^ (((r >> 1) & 1) | ((r >> 3) & 2)));
}

// The larger of a lane's and its partner's (lane ^ 32) number.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// The largest of a wave.
__device__ __forceinline__ int wave_max(int x) {
#define LD_ROR(N_) x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x120 + N_, 0xf, 0xf, true))
    LD_ROR(8);
    LD_ROR(4);
    LD_ROR(2);
    LD_ROR(1);
#undef LD_ROR
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((int)r[0], (int)r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane(max((int)q[0], (int)q[1]));
}

struct TileRows { int row, n, pos, seq, first, prefix; };

// Positions that rows r0 .. r1 - 1 of a tile see at least one of.
__device__ __forceinline__ int seen_from(const TileRows &t, int r, int window) { return max(max(t.first, window > 0 ? t.pos + r - window + 1 : 0), 0); }
__device__ __forceinline__ int seen_to(const TileRows &t, int r, int most) { return min(max(t.pos + r, t.prefix - 1), most); }

// Nothing is moved over this line.  The compiler puts matrix instructions next to each other, where each waits for the one before and the vector unit for
// all of them; the parts of a step lie in the order in which they are to be issued.
#define LD_HERE() __builtin_amdgcn_sched_barrier(0)

template <int HD, bool EXTRA>
__global__ __launch_bounds__(256, 2) void k_prefill_q8(Q8Attention a, const int32_t *__restrict__ tiles, int n_tiles, int max_pos, int splits,
                                                       float *__restrict__ part_o, float2 *__restrict__ part_ml) {
    constexpr int KS = HD / 32, ND = HD / 32, NP = HD / 64;
    // the last tiles first (they see the most); KV heads next to each other, so that one cache's L2 serves one of them where there are eight
    int idx = blockIdx.x;
    const int sp = idx % splits;
    idx /= splits;
    const int x = idx % a.H, tile_no = n_tiles - 1 - idx / a.H, G = a.H / a.Hkv, j = x % a.Hkv, h = j * G + x / a.Hkv;
    const int32_t *tp = tiles + 6 * (int64_t)tile_no;
    const TileRows tr{tp[0], min(tp[1], ROWS), tp[2], tp[3], tp[4], tp[5]};
    if (tr.n <= 0) return;
    const int most = (int)min((int64_t)max_pos, (int64_t)a.table_stride * 16 - 1);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hh = lane >> 5;
    const int wlo = seen_from(tr, 0, a.window), whi = seen_to(tr, tr.n - 1, most);      // of the workgroup
    int t0 = wlo >> 6, t1 = whi < wlo ? t0 : (whi >> 6) + 1;
    const int per = (t1 - t0 + splits - 1) / splits;
    t0 += sp * per;
    t1 = min(t1, t0 + per);

    const int r = 32 * wave + r32;
    const bool real = r < tr.n, busy = 32 * wave < tr.n;
    // lanes past the last row do as the last one does
    const int rr = min(r, tr.n - 1), nlast = min(tr.n - 1, 32 * wave + 31);
    const int lo = seen_from(tr, rr, a.window), hi = seen_to(tr, rr, most);
    const int wave_lo = seen_from(tr, 32 * wave, a.window), wave_hi = seen_to(tr, nlast, most);      // any row of the wave (if busy)
    const int all_lo = seen_from(tr, nlast, a.window), all_hi = seen_to(tr, 32 * wave, most);        // every row

    __shared__ __attribute__((aligned(16))) Stage<HD> stage[3];
    const int32_t *trow = a.table + (int64_t)tr.seq * a.table_stride;
    const int last = whi >> 4;
    const int64_t bs = q8_block(a.Hkv, HD);

    // ---- what a thread brings of a tile: NP pieces of keys and of values, and one exponent
    int id[NP], ide;
    uint4 kr[NP], vr[NP];
    int er = 0;
    const int8_t *kbase = a.codes + q8_k(HD, j, 0, 0) + 16 * (tid % HD);      // HD divides 256: the same place in every block
    auto ask = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NP; u++) id[u] = trow[min(4 * tile + (tid + 256 * u) / HD, last)];
        ide = trow[min(4 * tile + (lane >> 4), last)];
    };
    auto load_keys = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NP; u++) kr[u] = *reinterpret_cast<const uint4 *>(kbase + max(id[u], 0) * bs);
    };
    auto load_values = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NP; u++) vr[u] = *reinterpret_cast<const uint4 *>(kbase + (int64_t)a.Hkv * 16 * HD + max(id[u], 0) * bs);
        er = a.expo[(((int64_t)max(ide, 0) * 2 + (wave & 1)) * a.Hkv + j) * 16 + (lane & 15)];
    };
    // bit b: the tile's block b is mapped
    auto mapped_of = [&]() __attribute__((always_inline)) {
        const uint64_t ok = __ballot(ide >= 0);
        return (int)((ok & 1) | (ok >> 15 & 2) | (ok >> 30 & 4) | (ok >> 45 & 8));
    };
    // E0: the largest exponent of the first tile's values (those that are all zero aside); every wave finds it for itself
    int e0 = 0;
    auto store_keys = [&](Stage<HD> &s) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NP; u++) {
            const int i = tid + 256 * u, in = i % HD;
            s.k[key_piece<HD>(i / HD * 16 + in / (HD / 16), in % (HD / 16))] = kr[u];
        }
    };
    // part 0 .. 2 NP - 1: eight slots of a thread's values each; with the last one the unit
    auto store_values = [&](Stage<HD> &s, int part) __attribute__((always_inline)) {
        const int u = part >> 1, i = tid + 256 * u;
        s.v[(2 * (i / HD) + (part & 1)) * HD + i % HD] = part & 1 ? q8_halves(vr[u].z, vr[u].w) : q8_halves(vr[u].x, vr[u].y);
        if (part == 2 * NP - 1) s.unit[tid] = er == Q8_NAN ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, er - (wave & 1 ? e0 : 0));
    };
    auto store_all_values = [&](Stage<HD> &s) __attribute__((always_inline)) {
#pragma unroll
        for (int p = 0; p < 2 * NP; p++) store_values(s, p);
    };

    // ---- queries: dims 32 s + 16 hh .. + 16 of this lane's row
    i32x4_t qd[3][KS];
    float unit;
    {
        const float *qp = a.q + (int64_t)(tr.row + rr) * a.q_stride + h * HD + 16 * hh;
        float v[KS][16];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < KS; s++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                v[s][i] = qp[32 * s + i];
                top = max(top, __float_as_uint(v[s][i]) & 0x7fffffffu);
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, WAVE));
        const Q8Query query = q8_query(top, (EXTRA ? 1.0 : 1.4426950408889634) / sqrt((double)HD));
        unit = ldexpf(query.unit, query.exp);
        unit = unit < 0x1p-126f ? 0x1p-126f : unit;      // not zero: it multiplies -infinity
#pragma unroll
        for (int s = 0; s < KS; s++)
#pragma unroll
            for (int w = 0; w < 4; w++) {
                uint32_t d[3] = {0, 0, 0};
#pragma unroll
                for (int i = 0; i < 4; i++)
#pragma unroll
                    for (int n = 0; n < 3; n++) d[n] |= (uint32_t)(q8_digit(v[s][4 * w + i], query.scale, n) & 255) << (8 * i);
#pragma unroll
                for (int n = 0; n < 3; n++) qd[n][s][w] = (int)d[n];
            }
    }
    const float rs = EXTRA ? 1.f : unit;
    const float slope = EXTRA && a.slopes ? a.slopes[h] * 1.4426950408889634f : 0.f, inv_cap = EXTRA && a.softcap > 0.f ? 1.f / a.softcap : 0.f;

    f32x16_t o[ND];
#pragma unroll
    for (int n = 0; n < ND; n++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[n][i] = 0.f;
    // weights are 2^(score + add), score in the log2 domain; l: their sum over this lane's positions
    constexpr float NONE = 1e30f;      // of a row that has seen no score yet
    float add = NONE, l = 0.f;
    float big = 0.f;      // largest weight times its value's unit

    // A tile is taken in as two halves of 32 positions.  Products of a half's keys and queries: digits 2, and digits 1 and 0 ..
    i32x16_t acc2, acc;
    i32x4_t kf[KS];
    auto ask_keys = [&](const Stage<HD> &st, int u) __attribute__((always_inline)) {
        const int row = (2 * u + ((r32 >> 2) & 1)) * 16 + (r32 >> 3) * 4 + (r32 & 3);
#pragma unroll
        for (int q = 0; q < KS; q++) kf[q] = __builtin_bit_cast(i32x4_t, st.k[key_piece<HD>(row, 2 * q + hh)]);
    };
    auto product = [&](int k) __attribute__((always_inline)) {      // 0 .. 3 KS - 1
        if (k == 0) acc = (i32x16_t){};
        if (k == 1) acc2 = (i32x16_t){};
        if (k < 2 * KS) {
            if (k & 1) acc2 = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[k >> 1], qd[2][k >> 1], acc2, 0, 0, 0);
            else acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[k >> 1], qd[1][k >> 1], acc, 0, 0, 0);
        } else {
            if (k == 2 * KS) {
#pragma unroll
                for (int i = 0; i < 16; i++) acc[i] <<= 8;
            }
            acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[k - 2 * KS], qd[0][k - 2 * KS], acc, 0, 0, 0);
        }
    };
    // .. and the scores that they make (times rs: in the log2 domain), four at a time
    float s[16];
    auto score4 = [&](int i4, const float4 &k4, int at) __attribute__((always_inline)) {
        const float kk[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int i = 4 * i4 + e;
            s[i] = fmaf((float)acc2[i], 65536.f, (float)acc[i]) * kk[e];
            if constexpr (EXTRA) {
                float y = s[i] * unit;
                if (a.softcap > 0.f) y = q8_cap(y, a.softcap, inv_cap);
                s[i] = fmaf(slope, (float)(at + 16 * hh + i - (tr.pos + rr)), y * 1.4426950408889634f);
            }
        }
    };
    // Takes in half u of tile `tile`, whose scores are in s; leaves those of the half behind it (of stage nst) there.  Its weights are formed while the next
    // half's keys are multiplied, its values multiplied while the next half's scores are formed and (to: with the second half) a later tile is stored.
    auto step = [&](const Stage<HD> &st, const Stage<HD> &nst, int tile, int mapped, auto half, Stage<HD> &to) __attribute__((always_inline)) {
        constexpr int u = decltype(half)::value, un = 1 - u;
        const int base = tile * TILE + 32 * u;
        const bool whole = base >= all_lo && base + 31 <= all_hi && (mapped >> (2 * u) & 3) == 3;
        // Keeps the entries whose positions the row sees.  What it compares is hidden from the compiler, which would hold the positions and as many truth
        // values over all of the step otherwise.
        auto keep_seen = [&](float (&x)[16], float other) __attribute__((always_inline)) {
            int at = lo - base - 16 * hh;
            asm volatile("" : "+v"(at));
            const uint32_t range = (uint32_t)(hi - lo);
            const bool there = (mapped >> (2 * u + hh) & 1) && hi >= lo;
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = there && (uint32_t)(i - at) <= range ? x[i] : other;
        };
        ask_keys(nst, un);
        if (!whole) keep_seen(s, -INFINITY);
        float most_s = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; i++) most_s = fmaxf(most_s, s[i]);
        most_s = max_halves(most_s) * rs;
        // the first score makes the largest weight 2^12; one that would be above 2^30 does so too
        if (__any(most_s + add > 30.f)) {
            const float an = most_s + add > 30.f ? 12.f - most_s : add;
            const float keep = add == NONE ? 0.f : fast_exp2(an - add);
            add = an;
            l *= keep;
            big *= keep;
#pragma unroll
            for (int n = 0; n < ND; n++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[n][i] *= keep;
        }
        // ---- weights, beside the next half's products
        const float4 *vu = reinterpret_cast<const float4 *>(st.unit + 64 + 32 * u + 16 * hh);
        float sum = 0.f, top = 0.f;
        float4 v4 = vu[0];
        LD_HERE();
#pragma unroll
        for (int k = 0; k < 2 * KS; k++) {
            product(k);
            constexpr int per = 16 / (2 * KS);      // weights a product
#pragma unroll
            for (int e = 0; e < per; e++) {
                const int i = per * k + e;
                const float vv = (i & 3) == 0 ? v4.x : (i & 3) == 1 ? v4.y : (i & 3) == 2 ? v4.z : v4.w;
                const float p = fast_exp2(fmaf(s[i], rs, add));
                sum += p;
                s[i] = p * vv;
                if ((i & 3) == 3 && i < 15) v4 = vu[(i >> 2) + 1];
            }
            LD_HERE();
        }
        if (!whole) keep_seen(s, 0.f);      // units of positions that are not seen may be anything
        constexpr int PAIRS = ND / 2;
        f16x8_t vf[2][2];      // values of a pair of 32 dimensions, and of the next
        auto ask_values = [&](int g) __attribute__((always_inline)) {
            const int q = g / PAIRS, n = g % PAIRS * 2;
#pragma unroll
            for (int e = 0; e < 2; e++) vf[g & 1][e] = st.v[(2 * (2 * u + hh) + q) * HD + 32 * (n + e) + r32];
        };
        ask_values(0);
        LD_HERE();
#pragma unroll
        for (int k = 2 * KS; k < 3 * KS; k++) {
            product(k);
            constexpr int per = 16 / KS;
#pragma unroll
            for (int e = 0; e < per; e++) top = fmaxf(top, s[per * (k - 2 * KS) + e]);
            LD_HERE();
        }
        top = max_halves(top);
        // the largest product leaves 2^9 .. 65504: scaled to 2^12 .. 2^13, what is there and what comes
        big = fmaxf(big, top);
        if (__any(big > 65504.f || (big > 0.f && big < 512.f))) {
            // the exponent of the exponential's argument stays below 100
            const int x = big > 0.f ? min(12 - ((int)(__float_as_uint(big) >> 23) - 127), (int)fminf(100.f - add - fmaxf(most_s, -1e4f), 126.f)) : 0;
            const float up = ldexpf(1.f, x);
            add += (float)x;
            l *= up;
            sum *= up;
            big *= up;
#pragma unroll
            for (int n = 0; n < ND; n++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[n][i] *= up;
#pragma unroll
            for (int i = 0; i < 16; i++) s[i] *= up;
        }
        l += sum;
        // ---- sums, beside the next half's scores and a later tile
        f16x8_t wh[2], wl[2];
        auto split_pair = [&](int i) __attribute__((always_inline)) {
            uint32_t hi2, lo2;
            split2_halves(s[i], s[i + 1], hi2, lo2);
            const f16x2_t y = __builtin_bit_cast(f16x2_t, hi2), z = __builtin_bit_cast(f16x2_t, lo2);
            wh[i >> 3][i & 7] = y[0];
            wh[i >> 3][(i & 7) + 1] = y[1];
            wl[i >> 3][i & 7] = z[0];
            wl[i >> 3][(i & 7) + 1] = z[1];
        };
#pragma unroll
        for (int i = 0; i < 8; i += 2) split_pair(i);
        const float4 *ku = reinterpret_cast<const float4 *>(nst.unit + 32 * un + 16 * hh);
        float4 k4;
        LD_HERE();
#pragma unroll
        for (int k = 0; k < 4 * ND; k++) {      // pairs of dimensions: both leading terms, then both second ones
            const int g = k >> 2, q = g / PAIRS, n = g % PAIRS * 2 + (k & 1);
            if ((k & 3) == 0 && g + 1 < 2 * PAIRS) ask_values(g + 1);
            o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[g & 1][k & 1], k & 2 ? wl[q] : wh[q], o[n], 0, 0, 0);
            if (k < 4) split_pair(8 + 2 * k);
            constexpr int EVERY = (4 * ND - 4) / 4;      // a score of four each so many products
            if (k >= 4 && (k - 4) % EVERY == EVERY - 1) score4((k - 4) / EVERY, k4, (tile + u) * TILE + 32 * un);
            if (k >= 3 && (k - 3) % EVERY == 0 && (k - 3) / EVERY < 4) k4 = ku[(k - 3) / EVERY];
            if (u == 0 && k == 2) store_keys(to);
            if (u == 1 && k >= 3 && (k - 3) % 3 == 0 && (k - 3) / 3 < 2 * NP) store_values(to, (k - 3) / 3);
            LD_HERE();
        }
    };

    if (t0 < t1) {
        // the tiles that the wave takes in: of those of the workgroup, the ones that one of its rows sees
        const int w0 = busy ? max(t0, wave_lo >> 6) : t1, w1 = busy && wave_hi >= 0 ? min(t1, (wave_hi >> 6) + 1) : w0;
        {
            const int at = t0 * TILE + lane, ph = trow[min(at >> 4, last)];
            const int e = a.expo[(((int64_t)max(ph, 0) * 2 + 1) * a.Hkv + j) * 16 + (lane & 15)];
            const int top = wave_max(at >= wlo && at <= whi && ph >= 0 && e > -126 ? e : -1000);
            e0 = top == -1000 ? 0 : top;
        }
        // With tile t its keys and values and the keys of t + 1 are read, t + 2 is stored (in the place of t - 1): its keys, asked for a half earlier, in the
        // first half, its values in the second, so that few registers hold them.  Past the end the last tile comes again, which nobody reads.
        ask(t0);
        load_keys();
        load_values();
        int map0 = mapped_of(), map1, map2;
        ask(min(t0 + 1, t1 - 1));
        store_keys(stage[0]);
        store_all_values(stage[0]);
        load_keys();
        load_values();
        map1 = mapped_of();
        ask(min(t0 + 2, t1 - 1));
        store_keys(stage[1]);
        store_all_values(stage[1]);
        load_keys();
        lds_barrier();
        int cur = 0;
        for (int tile = t0; tile < t1; tile++) {
            const int nxt = cur == 2 ? 0 : cur + 1, then = nxt == 2 ? 0 : nxt + 1;
            const bool in = tile >= w0 && tile < w1;
            if (in) {
                if (tile == w0) {
                    ask_keys(stage[cur], 0);
#pragma unroll
                    for (int k = 0; k < 3 * KS; k++) product(k);
                    const float4 *ku = reinterpret_cast<const float4 *>(stage[cur].unit + 16 * hh);
#pragma unroll
                    for (int i = 0; i < 4; i++) score4(i, ku[i], tile * TILE);
                }
                step(stage[cur], stage[cur], tile, map0, std::integral_constant<int, 0>{}, stage[then]);
            } else {
                store_keys(stage[then]);
            }
            load_values();
            map2 = mapped_of();
            ask(min(tile + 3, t1 - 1));
            if (in) step(stage[cur], stage[nxt], tile, map0, std::integral_constant<int, 1>{}, stage[then]);
            else store_all_values(stage[then]);
            load_keys();
            map0 = map1;
            map1 = map2;
            lds_barrier();
            cur = nxt;
        }
    }

    l += __shfl_xor(l, 32, WAVE);
    if (!real) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t item = splits == 1 ? (int64_t)(tr.row + r) * a.H + h : (((int64_t)tile_no * a.H + h) * splits + sp) * ROWS + r;
    float *dst = (splits == 1 ? a.out : part_o) + item * HD;
#pragma unroll
    for (int n = 0; n < ND; n++)
#pragma unroll
        for (int b = 0; b < 4; b++) {
            float4_u y;
#pragma unroll
            for (int i = 0; i < 4; i++) y[i] = ldexpf(o[n][4 * b + i] * inv, e0);
            *reinterpret_cast<float4_u *>(dst + 32 * n + 8 * b + 4 * hh) = y;
        }
    if (splits > 1 && hh == 0) part_ml[item] = make_float2(l == 0.f ? -INFINITY : -add, l);
}

// Joins the shares of a row and head, in their order: one wave a row.
template <int HD>
__global__ __launch_bounds__(256) void k_join_prefill_q8(Q8Attention a, const int32_t *__restrict__ tiles, int splits, const float *__restrict__ part_o,
                                                         const float2 *__restrict__ part_ml) {
    const int tile_no = blockIdx.x, h = blockIdx.y, lane = threadIdx.x & 63, r = blockIdx.z * 4 + (threadIdx.x >> 6);
    const int32_t *tp = tiles + 6 * (int64_t)tile_no;
    if (r >= min(tp[1], ROWS)) return;
    const int64_t first = ((int64_t)tile_no * a.H + h) * splits * ROWS + r;
    float M = -INFINITY;
    for (int i = 0; i < splits; i++) M = fmaxf(M, part_ml[first + (int64_t)i * ROWS].x);
    const float ref = M > -INFINITY ? M : 0.f;
    float L = 0.f, acc[HD / 64] = {};
    for (int i = 0; i < splits; i++) {
        const int64_t at = first + (int64_t)i * ROWS;
        const float2 ml = part_ml[at];
        if (ml.y == 0.f) continue;
        const float f = fast_exp2(ml.x - ref) * ml.y;
        L += f;
#pragma unroll
        for (int u = 0; u < HD / 64; u++) acc[u] += f * part_o[at * HD + lane + 64 * u];
    }
#pragma unroll
    for (int u = 0; u < HD / 64; u++) a.out[((int64_t)(tp[0] + r) * a.H + h) * HD + lane + 64 * u] = L == 0.f ? 0.f : acc[u] / L;
}

constexpr int WANT = 512, LEAST = 4;      // workgroups, tiles of positions a share

int shares(int n_tiles, int H, int max_pos) {
    const int64_t pairs = (int64_t)n_tiles * H, kt = ((int64_t)max_pos + TILE) / TILE;
    return (int)std::max<int64_t>(1, std::min<int64_t>((WANT + pairs - 1) / pairs, kt / LEAST));
}

template <int HD>
void launch_prefill(const Q8Attention &a, const int32_t *tiles, int n_tiles, int max_pos, int splits, char *scratch, hipStream_t s) {
    float2 *part_ml = (float2 *)scratch;
    float *part_o = (float *)(scratch + ld::align_up((size_t)n_tiles * a.H * splits * ROWS * 8, 256));
    const dim3 grid((unsigned)((int64_t)n_tiles * a.H * splits)), block(256);
    if (a.softcap > 0.f || a.slopes) LD_LAUNCH((k_prefill_q8<HD, true>), grid, block, 0, s, a, tiles, n_tiles, max_pos, splits, part_o, part_ml);
    else LD_LAUNCH((k_prefill_q8<HD, false>), grid, block, 0, s, a, tiles, n_tiles, max_pos, splits, part_o, part_ml);
    if (splits > 1) LD_LAUNCH(k_join_prefill_q8<HD>, dim3(n_tiles, a.H, ROWS / 4), block, 0, s, a, tiles, splits, part_o, part_ml);
}

}  // namespace

extern "C" {

size_t ldk_prefill_attention_q8_scratch_bytes(int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t max_pos, int32_t window) {
    if (n_tiles <= 0 || H <= 0 || Hkv <= 0 || H % Hkv || (hd != 64 && hd != 128) || max_pos < 0 || window < 0) return 0;
    // no more shares than fill the machine, whatever the number of tiles: pairs * shares < WANT + pairs
    const size_t rows = ((size_t)n_tiles * H + WANT) * ROWS;
    return shares(1, 1, max_pos) == 1 ? 256 : ld::align_up(rows * 8, 256) + rows * hd * 4;
}

ld_status ldk_prefill_attention_q8(const float *q, int32_t q_stride, const int8_t *codes, const int8_t *expo, const int32_t *table,
                                   int32_t table_stride, const int32_t *tiles, int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t window,
                                   float softcap, const float *slopes, int32_t max_pos, float *out, void *scratch, size_t scratch_bytes,
                                   void *stream) {
    if (n_tiles == 0) return LD_OK;
    const Q8Attention a{q, q_stride, codes, expo, table, table_stride, H, Hkv, window, softcap, slopes, out};
    if (n_tiles < 0 || max_pos < 0 || !tiles || bad_attention(a, hd)) return ld::fail(LD_E_INVAL, "ldk_prefill_attention_q8: bad argument");
    const int splits = shares(n_tiles, H, max_pos);
    if (H > 65535 || (int64_t)n_tiles * H * splits > INT32_MAX)
        return ld::fail(LD_E_RANGE, "ldk_prefill_attention_q8: more than 65535 heads, or too many tiles");
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < ldk_prefill_attention_q8_scratch_bytes(n_tiles, H, Hkv, hd, max_pos, window))
        return ld::fail(LD_E_INVAL, "ldk_prefill_attention_q8: scratch too small, or not aligned to 16 bytes");
    hipStream_t s = (hipStream_t)stream;
    if (hd == 128) launch_prefill<128>(a, tiles, n_tiles, max_pos, splits, (char *)scratch, s);
    else launch_prefill<64>(a, tiles, n_tiles, max_pos, splits, (char *)scratch, s);
    return launched("k_prefill_q8");
}

}  // extern "C"
