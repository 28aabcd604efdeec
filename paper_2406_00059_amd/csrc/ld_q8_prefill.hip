// Attention of prompt and chunk rows over the 8-bit cache on the matrix cores.
//
// A workgroup takes a tile of up to 128 rows and a query head, each of its four waves 32 rows, and walks the positions 64 (four blocks) at a time.
// Keys and values go through LDS, the next tile's while one is multiplied: keys as they are, values widened to fp16 once for the four waves.
//
//   scores   S^T[pos, row] = K[pos, :] . Q[row, :] in whole numbers (32x32x32, 8 bits): a query is three base-256 digits (24 bits under its largest
//            entry), kept in registers.
//   sums     O^T[d, row] += V^T[d, pos] W^T[pos, row] (32x32x16, fp16): codes are exact in fp16; W = p 2^e 2^x, e the value's exponent and 2^x the power
//            of two that brings the largest p 2^e of the row so far to 2^13 .. 65504, as two fp16 terms (22 bits).
//
// Which position a row of the score tile is, is free: row 8 b + 4 h + i is slot 4 b + i of block h of a pair, so that lane (row, h) ends with the scores of
// block h, slot by slot, which is what it has to bring as the other operand of the sums.
//
// Units of positions are held by sixteen lanes each and enter products from there (row_newbcast); read by every lane they cost a third of the LDS reads, and
// the registers that brought some of the staged keys into scratch memory (8191 rows below: 812 us).
//
// What bounds it: 64 positions and 32 rows are 56 matrix instructions (1800 cycles of a SIMD) and some 545 vector ones.  With two waves a SIMD, which is what
// the registers allow, matrix instructions take 48 % and vector ones 69 % of the time.  8191 rows of 32 heads in a band of 4096 take 720 - 760 us, some 555 TFLOP/s
// of the formula and 970 of executed products, at a clock that falls to 1.6 - 2.0 GHz meanwhile: vector instructions saved (sums that the matrix cores begin
// at a number whose bits are a float's) and the two kinds of work ordered otherwise (scores of both halves first, wave priorities) no longer change it.
// Measured and not kept, the first two with keys in scratch: scores in fp16 with queries in two terms (five vector instructions an entry less, a third more
// matrix time, registers spilled: 1055 us); one wave a SIMD with the scores of the next tile formed ahead (1794); half tiles whose instructions are
// interleaved by hand (760; four capped observations 170 us against 115); two groups of four waves that take turns at matrix and vector instructions, a
// barrier between (913).
#include <algorithm>
#include <cmath>
#include <utility>
#include "ld_q8.h"

using namespace ldd;

namespace {

constexpr int TILE = 64, ROWS = 128;
// Units of keys are 2^-23 too small and those of queries as much too large, so that a whole-number score (below 2^38) times a key's unit stays in float32 for keys
// up to 2^120; the smallest unit, 2^-149, is still a float.
constexpr int KEY_SHIFT = 23;
typedef int i32x16_t __attribute__((ext_vector_type(16)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

template <int HD>
struct Stage {
    i32x4_t k[4 * HD];             // [position][piece of 16 dims, swizzled]
    f16x8_t v[8 * HD];             // [block][half][dim]: eight slots
    float ku[TILE], vu[TILE];      // units; NaN where a vector is not finite
    int mapped;                    // bit b: block b
};

// Piece p of position r (block r / 16, slot r % 16), so that eight lanes' pieces of a score operand lie in different banks.
template <int HD>
__device__ __forceinline__ int key_piece(int r, int p) {
    constexpr int N = HD / 16;
    return N == 8 ? r * 8 + (p ^ ((r & 3) | ((r >> 2) & 4))) : r * 4 + (p ^ (((r >> 1) & 1) | ((r >> 3) & 2)));
}

// x[i] *= the unit that lane i of these sixteen holds.
template <int... I>
__device__ __forceinline__ void times_units(float (&x)[16], float unit, std::integer_sequence<int, I...>) {
    ((x[I] *= __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(unit), 0x150 + I, 0xf, 0xf, true))), ...);
}

struct TileRows { int row, n, pos, seq, first, prefix; };

// Positions that rows r0 .. r1 - 1 of a tile see at least one of.
__device__ __forceinline__ int seen_from(const TileRows &t, int r, int window) { return max(max(t.first, window > 0 ? t.pos + r - window + 1 : 0), 0); }
__device__ __forceinline__ int seen_to(const TileRows &t, int r, int most) { return min(max(t.pos + r, t.prefix - 1), most); }

// Heads of 64 without caps and slopes fit three waves a SIMD (4096 rows of 32 heads over 8: 183 us, 192 with two).
template <int HD, bool EXTRA>
__global__ __launch_bounds__(256, HD == 64 && !EXTRA ? 3 : 2) void k_prefill_q8(Q8Attention a, const int32_t *__restrict__ tiles, int n_tiles, int max_pos, int splits,
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

    __shared__ __attribute__((aligned(16))) Stage<HD> stage[2];
    __shared__ float froms[256];
    const int32_t *trow = a.table + (int64_t)tr.seq * a.table_stride;
    const int last = whi >> 4;
    const int64_t bs = q8_block(a.Hkv, HD);

    // ---- what a thread brings of a tile: NP pieces of keys and of values, and one exponent
    int id[NP], ide;
    i32x4_t kr[NP], vr[NP];
    int er = 0;
    const uint32_t place = 16 * (tid % HD);
    const int eb = (tid & 63) >> 4;
    auto ask = [&](int tile) {
#pragma unroll
        for (int u = 0; u < NP; u++) id[u] = trow[min(4 * tile + (64 * wave + 256 * u) / HD, last)];      // a wave's pieces lie in one block
        ide = trow[min(4 * tile + eb, last)];
    };
    auto load = [&]() {
#pragma unroll
        for (int u = 0; u < NP; u++) {
            const int8_t *b = a.codes + max(__builtin_amdgcn_readfirstlane(id[u]), 0) * bs + q8_k(HD, j, 0, 0);      // a scalar: the lanes differ by 32 bits
            kr[u] = *reinterpret_cast<const i32x4_t *>(b + place);
            vr[u] = *reinterpret_cast<const i32x4_t *>(b + a.Hkv * 16 * HD + place);
        }
        if (tid < 128) er = a.expo[(((int64_t)max(ide, 0) * 2 + (tid >> 6)) * a.Hkv + j) * 16 + (tid & 15)];
    };
    // E0: the largest exponent of the first tile's values (those that are all zero aside); every wave finds it for itself
    int e0 = 0;
    auto store = [&](Stage<HD> &s, int ide_of) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < NP; u++) {
            const int i = tid + 256 * u, b = i / HD, in = i % HD;
            s.k[key_piece<HD>(b * 16 + in / (HD / 16), in % (HD / 16))] = kr[u];
            s.v[(2 * b) * HD + in] = q8_halves(vr[u][0], vr[u][1]);
            s.v[(2 * b + 1) * HD + in] = q8_halves(vr[u][2], vr[u][3]);
        }
        if (tid < 64) {
            s.ku[tid] = er == Q8_NAN ? __uint_as_float(0x7fc00000u) : ldexpf(1.f, er - KEY_SHIFT);
            const uint64_t ok = __ballot(ide_of >= 0);
            if (tid == 0) s.mapped = (int)((ok & 1) | (ok >> 15 & 2) | (ok >> 30 & 4) | (ok >> 45 & 8));
        } else if (tid < 128) {
            // a zero value (the lowest exponent, and out of range beside these if it is not one) asks for no scaling of a row
            s.vu[tid - 64] = er == Q8_NAN ? __uint_as_float(0x7fc00000u) : er == -126 && e0 > -41 ? 0.f : ldexpf(1.f, er - e0);
        }
    };

    // ---- queries: dims 32 s + 16 hh .. + 16 of this lane's row
    i32x4_t qd[3][KS];
    float unit;
    uint64_t broken;      // lanes whose query is not finite: theirs is taken as zero until the end, where a row that has seen anything becomes NaN
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
        broken = __ballot(top >= 0x7f800000u);
        unit = top >= 0x7f800000u ? 1.f : ldexpf(query.unit, query.exp + KEY_SHIFT);
        unit = unit < 0x1p-149f ? 0x1p-149f : unit;      // not zero: it multiplies -infinity (and sums below 2^128: what a subnormal number lacks in bits shows in no weight)
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
    const float rs = EXTRA ? 1.4426950408889634f : unit;
    const float slope = EXTRA && a.slopes ? a.slopes[h] : 0.f, inv_cap = EXTRA && a.softcap > 0.f ? 1.f / a.softcap : 0.f;

    f32x16_t o[ND];
#pragma unroll
    for (int n = 0; n < ND; n++)
#pragma unroll
        for (int i = 0; i < 16; i++) o[n][i] = 0.f;
    // weights are 2^((s - from) rs + add), s rs a score in the log2 domain; l: their sum over this lane's positions.  from is 0, or a score that is so large that
    // add could not hold it: a product s rs is off by up to 2^-25 of itself from what a multiple of it in add was rounded to, which must not reach an exponent.
    // It seldom is, and has no register: large has a bit for the lanes whose from is in froms.
    constexpr float NONE = 3e38f;         // add of a row that has seen no score yet
    constexpr float LARGE = 32768.f;      // of a score
    float add = NONE, l = 0.f;
    uint64_t large = 0;
    float big = 0.f;      // largest weight times its value's unit

    auto exponent = [](float x) { return (int)(__float_as_uint(x) >> 23) - 127; };      // of x > 0

    auto multiply = [&](const Stage<HD> &st, int tile) {
        const int base = tile * TILE, mapped = __builtin_amdgcn_readfirstlane(st.mapped);
        float s[2][16];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            i32x16_t acc2 = {}, acc = {};
            const int row = (2 * u + ((r32 >> 2) & 1)) * 16 + (r32 >> 3) * 4 + (r32 & 3);
            i32x4_t kf[KS];
#pragma unroll
            for (int q = 0; q < KS; q++) kf[q] = st.k[key_piece<HD>(row, 2 * q + hh)];
#pragma unroll
            for (int q = 0; q < KS; q++) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[q], qd[1][q], acc, 0, 0, 0);
#pragma unroll
            for (int q = 0; q < KS; q++) acc2 = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[q], qd[2][q], acc2, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; i++) acc[i] <<= 8;
#pragma unroll
            for (int q = 0; q < KS; q++) acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(kf[q], qd[0][q], acc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; i++) s[u][i] = fmaf((float)acc2[i], 65536.f, (float)acc[i]);
            times_units(s[u], st.ku[32 * u + 16 * hh + (lane & 15)], std::make_integer_sequence<int, 16>());
        }
        if constexpr (EXTRA) {
            float most = 0.f;
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    s[u][i] *= unit;
                    most = fmaxf(most, fabsf(s[u][i]));
                }
            if (a.softcap > 0.f) {
                if (__any(most * inv_cap >= Q8_SERIES)) {
#pragma unroll
                    for (int u = 0; u < 2; u++)
#pragma unroll
                        for (int i = 0; i < 16; i++) s[u][i] = q8_cap(s[u][i], a.softcap, inv_cap);
                } else {      // scores far below the cap, as they mostly are: a third of the instructions
#pragma unroll
                    for (int u = 0; u < 2; u++)
#pragma unroll
                        for (int i = 0; i < 16; i++) s[u][i] = q8_cap_small(s[u][i], inv_cap);
                }
            }
            if (a.slopes) {
                const float at = (float)(base + 16 * hh - (tr.pos + rr));
#pragma unroll
                for (int u = 0; u < 2; u++)
#pragma unroll
                    for (int i = 0; i < 16; i++) s[u][i] = fmaf(slope, at + (float)(32 * u + i), s[u][i]);
            }
        }
        const bool whole = base >= all_lo && base + TILE - 1 <= all_hi && mapped == 15;
        // Keeps the entries whose positions the row sees.  What it compares is hidden from the compiler, which would hold 32 positions and as many
        // truth values over all of the tile otherwise.
        auto keep_seen = [&](float (&x)[2][16], float other) __attribute__((always_inline)) {
            int at = lo - base - 16 * hh;
            asm volatile("" : "+v"(at));
            const uint32_t range = (uint32_t)(hi - lo);
#pragma unroll
            for (int u = 0; u < 2; u++) {
                const bool there = (mapped >> (2 * u + hh) & 1) && hi >= lo;
#pragma unroll
                for (int i = 0; i < 16; i++) x[u][i] = there && (uint32_t)(32 * u + i - at) <= range ? x[u][i] : other;
            }
        };
        if (!whole) keep_seen(s, -INFINITY);
        float most_s = -INFINITY;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 16; i++) most_s = fmaxf(most_s, s[u][i]);
        most_s = max_halves(most_s);
        float from = 0.f;
        if (__builtin_expect(large != 0, 0)) from = large >> lane & 1 ? froms[tid] : 0.f;
        // the first score makes the largest weight 2^14 (mostly within what the products are held in below); one that would be above 2^30 does so too.  What is
        // seldom taken is told to the compiler, here and below: four capped observations 117.1 -> 114.8 us, 8191 rows 733 -> 728
        const bool lower = fmaf(most_s - from, rs, add) > 30.f;
        if (__builtin_expect(__any(lower), 0)) {
            const float fn = !lower ? from : fabsf(most_s * rs) >= LARGE ? most_s : 0.f, an = lower ? 14.f - (most_s - fn) * rs : add;
            const float keep = add == NONE ? 0.f : fast_exp2(fmaf(from - fn, rs, an - add));
            add = an;
            l *= keep;
            big *= keep;
#pragma unroll
            for (int n = 0; n < ND; n++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[n][i] *= keep;
            large = __ballot(fn != 0.f);
            if (large) froms[tid] = fn;
            from = fn;
        }
        if (__builtin_expect(large != 0, 0)) {
#pragma unroll
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[u][i] -= from;
        }
        float sum = 0.f, top = 0.f;
#pragma unroll
        for (int u = 0; u < 2; u++) {
#pragma unroll
            for (int i = 0; i < 16; i++) {
                s[u][i] = fast_exp2(fmaf(s[u][i], rs, add));
                sum += s[u][i];
            }
            times_units(s[u], st.vu[32 * u + 16 * hh + (lane & 15)], std::make_integer_sequence<int, 16>());
        }
        if (!whole) keep_seen(s, 0.f);      // units of positions that are not seen may be anything
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = fmaxf(top, s[u][i]);
        top = max_halves(top);
        // the largest product leaves 2^13 .. 65504: scaled to 2^13 .. 2^14, what is there and what comes
        big = fmaxf(big, top);
        if (__builtin_expect(__any(big > 65504.f || (big > 0.f && big < 8192.f)), 0)) {
            // the sum of the row's weights, of this tile and of earlier ones, stays below 2^97: where the values that draw most are zero, nothing else holds
            // the weights down
            const int x = big > 0.f ? min(min(13 - exponent(big), 96 - exponent(max_halves(l + sum))), 126) : 0;
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
            for (int u = 0; u < 2; u++)
#pragma unroll
                for (int i = 0; i < 16; i++) s[u][i] *= up;
        }
        l += sum;
#pragma unroll
        for (int u = 0; u < 2; u++) {
            f16x8_t wh[2], wl[2];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                uint32_t hi, lo;
                split2_halves(s[u][i], s[u][i + 1], hi, lo);
                const f16x2_t y = __builtin_bit_cast(f16x2_t, hi), z = __builtin_bit_cast(f16x2_t, lo);
                wh[i >> 3][i & 7] = y[0];
                wh[i >> 3][(i & 7) + 1] = y[1];
                wl[i >> 3][i & 7] = z[0];
                wl[i >> 3][(i & 7) + 1] = z[1];
            }
#pragma unroll
            for (int q = 0; q < 2; q++) {
                f16x8_t vf[ND];
#pragma unroll
                for (int n = 0; n < ND; n++) vf[n] = st.v[(2 * (2 * u + hh) + q) * HD + 32 * n + r32];
#pragma unroll
                for (int n = 0; n < ND; n++) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[n], wh[q], o[n], 0, 0, 0);
#pragma unroll
                for (int n = 0; n < ND; n++) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[n], wl[q], o[n], 0, 0, 0);
            }
        }
    };

    if (t0 < t1) {
        ask(t0);
        load();
        int ide_of = ide;
        {
            const int at = t0 * TILE + lane, ph = trow[min(at >> 4, last)];
            const int e = a.expo[(((int64_t)max(ph, 0) * 2 + 1) * a.Hkv + j) * 16 + (lane & 15)];
            const int top = wave_max(at >= wlo && at <= whi && ph >= 0 && e > -126 ? e : -1000);
            e0 = top == -1000 ? 0 : top;
        }
        if (t0 + 1 < t1) ask(t0 + 1);
        store(stage[0], ide_of);
        if (t0 + 1 < t1) {
            load();
            ide_of = ide;
        }
        if (t0 + 2 < t1) ask(t0 + 2);
        lds_barrier();
        for (int tile = t0; tile < t1; tile++) {
            const int cur = (tile - t0) & 1;
            if (busy && tile * TILE <= wave_hi && tile * TILE + TILE - 1 >= wave_lo) multiply(stage[cur], tile);
            if (tile + 1 < t1) {
                store(stage[cur ^ 1], ide_of);
                if (tile + 2 < t1) {
                    load();
                    ide_of = ide;
                }
                if (tile + 3 < t1) ask(tile + 3);
                lds_barrier();
            }
        }
    }

    l += __shfl_xor(l, 32, WAVE);
    if (!real) return;
    if (l > 0.f && (broken >> lane & 1)) l = __uint_as_float(0x7fc00000u);
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
    if (splits > 1 && hh == 0) {
        // beside a large score add would be lost: it is a whole number there, and goes into the sum
        const bool far = large >> lane & 1;
        part_ml[item] = l == 0.f ? make_float2(-INFINITY, 0.f) : far ? make_float2(froms[tid] * rs, ldexpf(l, -(int)add)) : make_float2(-add, l);
    }
}

// Joins the shares of a row and head, in their order: HD / 4 lanes a row, four shares' loads in flight (5.7 us for the 96 pairs
// below and 11.7 for the 280; a wave a row and one load at a time 8.8 and 16.4).
template <int HD>
__global__ __launch_bounds__(256) void k_join_prefill_q8(Q8Attention a, const int32_t *__restrict__ tiles, int splits, const float *__restrict__ part_o,
                                                         const float2 *__restrict__ part_ml) {
    constexpr int PER = HD / 4;
    const int tile_no = blockIdx.x, h = blockIdx.y, d = threadIdx.x % PER, r = blockIdx.z * (256 / PER) + threadIdx.x / PER;
    const int32_t *tp = tiles + 6 * (int64_t)tile_no;
    if (r >= min(tp[1], ROWS)) return;
    const int64_t first = ((int64_t)tile_no * a.H + h) * splits * ROWS + r;
    const float2 *ml = part_ml + first;
    const float4 *po = reinterpret_cast<const float4 *>(part_o + first * HD) + d;
    // The weights of all shares, together at most 1, so that the sum stays within the values up to the ends of float32: a row's own sums go up to 2^97
    float M = -INFINITY, most = -INFINITY;
#pragma unroll 4
    for (int i = 0; i < splits; i++) {
        const float2 w = ml[i * ROWS];
        M = fmaxf(M, w.x);
        most = fmaxf(most, w.x + __builtin_amdgcn_logf(w.y));
    }
    const float ref = M > -INFINITY ? M : 0.f;
    const float scale = most > -INFINITY ? ldexpf(1.f, -(int)ceilf(most - ref) - (33 - __clz(splits))) : 0.f;
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = 0; i < splits; i++) {
        const float2 w = ml[i * ROWS];
        const float4 o = po[(int64_t)i * ROWS * PER];
        const float f = w.y == 0.f ? 0.f : fast_exp2(w.x - ref) * w.y * scale;      // a share without a position that the row sees left zeros
        L += f;
        acc = make_float4(fmaf(f, o.x, acc.x), fmaf(f, o.y, acc.y), fmaf(f, o.z, acc.z), fmaf(f, o.w, acc.w));
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *reinterpret_cast<float4_u *>(a.out + ((int64_t)(tp[0] + r) * a.H + h) * HD + 4 * d) = (float4_u){acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
}

constexpr int MOST = 1024, LEAST = 4;      // workgroups with shares, 64-position tiles a share

// Shares of a tile's positions, by the number of (tile, head) pairs.  Up to a pair a CU: what fills the CUs once with two workgroups each, or nearly; more: about
// four a CU, so that the last ones do not work alone.  us, 1 / 2 / 3 / 4 / 5 / 6 / 8 shares: 96 pairs of 24 tiles 66 / 45 / 45 / 40 / 41 / 48 / 48, 280 pairs of up to
// 68 tiles 189 / 127 / 130 / 118 / 121 / 123 / 138.
int shares(int n_tiles, int H, int max_pos) {
    const int64_t pairs = (int64_t)n_tiles * H, kt = ((int64_t)max_pos + TILE) / TILE;
    const int64_t n = pairs <= 256 ? std::max<int64_t>(2, 400 / pairs) : (MOST + pairs - 1) / pairs;
    return (int)std::max<int64_t>(1, std::min<int64_t>(n, kt / LEAST));
}

template <int HD>
void launch_prefill(const Q8Attention &a, const int32_t *tiles, int n_tiles, int max_pos, int splits, char *scratch, hipStream_t s) {
    float2 *part_ml = (float2 *)scratch;
    float *part_o = (float *)(scratch + ld::align_up((size_t)n_tiles * a.H * splits * ROWS * 8, 256));
    const dim3 grid((unsigned)((int64_t)n_tiles * a.H * splits)), block(256);
    if (a.softcap > 0.f || a.slopes) LD_LAUNCH((k_prefill_q8<HD, true>), grid, block, 0, s, a, tiles, n_tiles, max_pos, splits, part_o, part_ml);
    else LD_LAUNCH((k_prefill_q8<HD, false>), grid, block, 0, s, a, tiles, n_tiles, max_pos, splits, part_o, part_ml);
    if (splits > 1) LD_LAUNCH(k_join_prefill_q8<HD>, dim3(n_tiles, a.H, ROWS * HD / 1024), block, 0, s, a, tiles, splits, part_o, part_ml);
}

}  // namespace

extern "C" {

size_t ldk_prefill_attention_q8_scratch_bytes(int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t max_pos, int32_t window) {
    if (n_tiles <= 0 || H <= 0 || Hkv <= 0 || H % Hkv || (hd != 64 && hd != 128) || max_pos < 0 || window < 0) return 0;
    // pairs * shares < MOST + pairs, whatever the number of tiles
    const size_t rows = ((size_t)n_tiles * H + MOST) * ROWS;
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
    if (H > 65535 || too_large((int64_t)n_tiles * H * splits, 256))
        return ld::fail(LD_E_RANGE, "ldk_prefill_attention_q8: more than 65535 heads, or too many tiles");
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < ldk_prefill_attention_q8_scratch_bytes(n_tiles, H, Hkv, hd, max_pos, window))
        return ld::fail(LD_E_INVAL, "ldk_prefill_attention_q8: scratch too small, or not aligned to 16 bytes");
    hipStream_t s = (hipStream_t)stream;
    if (hd == 128) launch_prefill<128>(a, tiles, n_tiles, max_pos, splits, (char *)scratch, s);
    else launch_prefill<64>(a, tiles, n_tiles, max_pos, splits, (char *)scratch, s);
    return launched("k_prefill_q8");
}

}  // extern "C"
