// Attention of single tokens over the 8-bit cache on the matrix cores.
//
// A workgroup of four waves takes one row, KV head and chunk of the sequence, a wave 64 positions (four blocks) at a time, which it loads
// straight into operand registers; nothing goes through LDS but the join of the waves.  The G query heads of the KV head, padded to GP = 1, 2, 4, 8 or 16,
// share the 16 columns of a tile with their terms: column c is head c % GP and term c / GP.
//
//   scores   S^T[pos, c] = K[pos, :] . Q[c, :] in whole numbers (16x16x64, 8 bits): a query is three base-256 digits (24 bits under its largest
//            entry), the keys enter as they lie in the cache.  One product where three terms find room beside the heads (GP <= 4), two or three else; a
//            rotation within 16 lanes adds the terms, scaled to float32, so that every column of a head holds its score.
//   sums     O^T[d, c] += V^T[d, pos] W^T[pos, c] (16x16x32, fp16): codes are exact in fp16; W = p 2^(e - k), e the value's exponent and k
//            the running largest of p 2^e in the column, held at 2^13 .. 2^14, as two fp16 terms (22 bits) in two columns.
//
// What bounds it is the cache's stream: 32 rows of 512 - 8192 positions of 32 heads 206 us with the join, 5.5 TB/s (a large copy reaches 5.2); one row of
// 131067 positions of 8 KV heads 58 us, 53 of them the stream.  Heads are next to each other in the grid, for the blocks' sake (344 us with rows next to each other).
// One row of 1520 positions is a chain of loads, a tile and the join: 8.0 and 2.3 us.
//
// Which position a row of the score tile is, is free: row 4 g + i of tile t is slot 4 t + i of block g, so lane (c, g) ends with the scores of
// block g, slot by slot, which is what it has to bring as the other operand of the sums.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "ld_q8.h"

using namespace ldd;

namespace {

constexpr int TILE = 64, WAVES = 4;

// Positions lo .. hi that a row sees; hi < lo: none.
struct Seen { int lo, hi; };
__device__ __forceinline__ Seen seen_of(int ctx_len, int first, int max_ctx, int window, int table_stride) {
    const int ctx = (int)min((int64_t)min(ctx_len, max_ctx), (int64_t)table_stride * 16);
    return {max(max(first, window > 0 ? ctx_len - window : 0), 0), ctx - 1};
}

// x summed over the lanes of 16 that hold the same head's terms; the same bits in all of them.
template <int GP>
__device__ __forceinline__ float sum_terms(float x) {
    if constexpr (GP <= 8) x += __int_as_float(LD_ROR(__float_as_int(x), 8));
    if constexpr (GP <= 4) x += __int_as_float(LD_ROR(__float_as_int(x), 4));
    if constexpr (GP <= 2) x += __int_as_float(LD_ROR(__float_as_int(x), 2));
    if constexpr (GP <= 1) x += __int_as_float(LD_ROR(__float_as_int(x), 1));
    return x;
}

template <int HD, int GP, bool EXTRA>
__global__ __launch_bounds__(64 * WAVES, 2) void k_decode_q8(Q8Attention a, const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ first,
                                                             const int32_t *__restrict__ ctx_len, int max_ctx, int chunk, int chunks, float *__restrict__ part_o,
                                                             float2 *__restrict__ part_ml) {
    constexpr int KS = HD / 64, ND = HD / 16, TERMS = 16 / GP, PASSES = (3 + TERMS - 1) / TERMS;
    // heads next to each other: a block's keys and values of all heads lie together
    const int G = a.H / a.Hkv, parts = (G + 15) / 16, groups = a.Hkv * parts, item = blockIdx.x / groups, t = item / chunks, ch = item % chunks;
    const int hg = blockIdx.x % groups, j = hg / parts, h0 = j * G + hg % parts * 16, heads = min(G - hg % parts * 16, 16);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4, head = c % GP, term = c / GP;
    const int len = ctx_len[t], seq = seq_slot[t];
    const Seen see = seen_of(len, first ? first[t] : 0, max_ctx, a.window, a.table_stride);
    const int t0 = (see.lo >> 6) + ch * chunk, t1 = min(t0 + chunk, (see.hi >> 6) + 1);
    if (see.hi < see.lo || t0 >= t1) {
        if (chunks == 1)
            for (int i = threadIdx.x; i < heads * HD; i += 64 * WAVES) a.out[((int64_t)t * a.H + h0) * HD + i] = 0.f;
        return;
    }
    const int32_t *trow = a.table + (int64_t)seq * a.table_stride;
    const int last = see.hi >> 4;      // last visible block
    const int64_t bs = q8_block(a.Hkv, HD);
    const int8_t *kbase = a.codes + q8_k(HD, j, c & 3, 16 * g), *vbase = a.codes + q8_v(a.Hkv, HD, j, 0, c);

    typename std::conditional<GP == 1, int, u32x4_t>::type ek, ev;      // exponents of position 64 tile + lane, or of block g's
    u32x4_t kf[4][KS], vf[ND];
    int idk, idv;      // blocks of the tile to be loaded: the one of this lane's key rows, and block g
    auto ask = [&](int tile) {
        idk = trow[min(4 * tile + (c >> 2), last)];
        idv = trow[min(4 * tile + g, last)];
    };
    auto load_k = [&]() {
        const int8_t *p = kbase + max(idk, 0) * bs;
#pragma unroll
        for (int s = 0; s < 4; s++)
#pragma unroll
            for (int u = 0; u < KS; u++) kf[s][u] = load_stream16(p + 4 * s * HD + 64 * u);
        const int8_t *e = a.expo + ((int64_t)max(idv, 0) * 2 * a.Hkv + j) * 16 + (GP == 1 ? c : 0);
        if constexpr (GP == 1) {
            ek = e[0];
            ev = e[a.Hkv * 16];
        } else {
            ek = *reinterpret_cast<const u32x4_t *>(e);
            ev = *reinterpret_cast<const u32x4_t *>(e + a.Hkv * 16);
        }
    };
    auto load_v = [&](int id) {
        const int8_t *p = vbase + max(id, 0) * bs;
#pragma unroll
        for (int n = 0; n < ND; n++) vf[n] = load_stream16(p + 256 * n);
    };

    // The first tile is asked for before the queries are made ready
    const int begin = t0 + wave;
    if (begin < t1) {
        ask(begin);
        load_k();
        load_v(idv);
    }

    // Queries: dims 64 s + 16 g .. + 16 of this lane's head and term
    i32x4_t qd[PASSES][KS];
    float weight[PASSES];
    Q8Query query;
    {
        const float *qp = a.q + (int64_t)t * a.q_stride + (h0 + (head < heads ? head : 0)) * HD + 16 * g;
        float x[KS][16];
        uint32_t top = 0;
#pragma unroll
        for (int s = 0; s < KS; s++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                x[s][i] = qp[64 * s + i];
                top = max(top, __float_as_uint(x[s][i]) & 0x7fffffffu);
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, WAVE));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, WAVE));
        query = q8_query(top, (EXTRA ? 1.0 : 1.4426950408889634) / sqrt((double)HD));
#pragma unroll
        for (int p = 0; p < PASSES; p++) {
            const int digit = 2 - p * TERMS - term;
            weight[p] = digit == 2 ? 65536.f : digit == 1 ? 256.f : 1.f;
#pragma unroll
            for (int s = 0; s < KS; s++)
#pragma unroll
                for (int w = 0; w < 4; w++) {
                    uint32_t word = 0;
#pragma unroll
                    for (int i = 0; i < 4; i++) word |= (uint32_t)(q8_digit(x[s][4 * w + i], query.scale, digit) & 255) << (8 * i);
                    qd[p][s][w] = digit >= 0 && head < heads ? (int)word : 0;
                }
        }
    }
    const float slope = EXTRA && a.slopes && head < heads ? a.slopes[h0 + head] * 1.4426950408889634f : 0.f;
    const float inv_cap = EXTRA && a.softcap > 0.f ? 1.f / a.softcap : 0.f;

    f32x4_t o[ND];
#pragma unroll
    for (int n = 0; n < ND; n++) o[n] = (f32x4_t){0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;      // log2 domain; l over this lane's own positions
    int k = -100000;                   // o is in units of 2^(k - 14)

    // A score (in the log2 domain) from a sum of products
    auto score = [&](float x, int kexp, int pos) __attribute__((always_inline)) {
        x = ldexpf(x, kexp + query.exp) * query.unit;
        if constexpr (EXTRA) {
            if (a.softcap > 0.f) x = q8_cap(x, a.softcap, inv_cap);
            x = fmaf(slope, (float)(pos - (len - 1)), x * 1.4426950408889634f);
        }
        return kexp == Q8_NAN ? __uint_as_float(0x7fc00000u) : x;
    };
    // Brings m to the largest score, mb being that of a lane's own positions, then k to (at least) the largest exponent of what a column adds up, top that of
    // p 2^e over a lane's own positions.  The latter is formed from differences to m: beside a score of 2^25 an exponent is lost to rounding.
    float ref = 0.f, keep = 1.f;
    int fall = 0;
    auto raise = [&](float mb) __attribute__((always_inline)) {
        if constexpr (GP == 1) mb = max_of16(mb);
        mb = max_halves(max_quarters(mb));
        const float mn = fmaxf(m, mb);
        ref = mn > -INFINITY ? mn : 0.f;
        keep = fast_exp2(m - ref);
        fall = (int)ceilf(fminf(m > -INFINITY ? ref - m : 0.f, 100000.f));
        m = mn;
    };
    auto rescale = [&](float top) __attribute__((always_inline)) {
        if constexpr (GP == 1) top = max_of16(top);
        top = max_halves(max_quarters(top));
        const int kt = top > -INFINITY ? (int)ceilf(fminf(fmaxf(top, -90000.f), 90000.f)) : -100000;
        const int kn = max(max(k - fall, kt), -100000);
        const float scale = ldexpf(keep, max(min(k - kn, 300), -300));
        l *= keep;
        k = kn;
        if (__any(scale != 1.f)) {
#pragma unroll
            for (int n = 0; n < ND; n++)
#pragma unroll
                for (int i = 0; i < 4; i++) o[n][i] *= scale;
        }
    };
    for (int tile = begin; tile < t1; tile += WAVES) {
        const bool more = tile + WAVES < t1;
        // ---- scores of block g's 16 slots
        float s[16];
        const int at = (4 * tile + g) * 16;      // position of slot 0
        const bool mapped = idv >= 0;
        const auto ekn = ek, evn = ev;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int p = 0; p < PASSES; p++) {
                i32x4_t acc = {0, 0, 0, 0};
#pragma unroll
                for (int u = 0; u < KS; u++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4_t, kf[q][u]), qd[p][u], acc, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; i++) sum[i] = fmaf((float)acc[i], weight[p], sum[i]);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) s[4 * q + i] = sum_terms<GP>(sum[i]);
        }
        if (more) {
            ask(tile + WAVES);
            load_k();
        }
        const int id_next = idv;
        f16x8_t wb[2][GP == 16 ? 2 : 1];
        if constexpr (GP == 1) {
            // One head: every column of 16 holds its score, lane c goes on with slot c's, so that a lane has one position (64 tile + lane), and gets the others'
            // weights back by broadcasts within the 16.
            float x = s[0];
#pragma unroll
            for (int i = 1; i < 16; i++) x = c == i ? s[i] : x;
            const int pos = tile * TILE + lane, kexp = ekn;
            x = score(x, kexp, pos);
            const bool ok = mapped && pos >= see.lo && pos <= see.hi;
            x = ok ? x : -INFINITY;
            const int e = ok ? evn : -1000;
            raise(x);
            x -= ref;
            rescale(x + (float)e);
            const float p = fast_exp2(x);
            l += p;
            float w = ldexpf(p, e - k + 14);
            w = e == Q8_NAN ? __uint_as_float(0x7fc00000u) : w;
            const _Float16 hi = (_Float16)w, lo = (_Float16)(w - (float)hi);
            const int both = (int)((uint32_t)__builtin_bit_cast(uint16_t, hi) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16);
            const uint32_t take = term == 0 ? 0x05040100u : term == 1 ? 0x07060302u : 0x0c0c0c0cu;      // leading terms, second terms, zeros
            uint32_t words[8];
#define LD_PAIR(I_) words[I_] = __builtin_amdgcn_perm((uint32_t)__builtin_amdgcn_update_dpp(0, both, 0x150 + 2 * I_ + 1, 0xf, 0xf, true), \
                                                      (uint32_t)__builtin_amdgcn_update_dpp(0, both, 0x150 + 2 * I_, 0xf, 0xf, true), take)
            LD_PAIR(0); LD_PAIR(1); LD_PAIR(2); LD_PAIR(3); LD_PAIR(4); LD_PAIR(5); LD_PAIR(6); LD_PAIR(7);
#undef LD_PAIR
            wb[0][0] = __builtin_bit_cast(f16x8_t, (u32x4_t){words[0], words[1], words[2], words[3]});
            wb[1][0] = __builtin_bit_cast(f16x8_t, (u32x4_t){words[4], words[5], words[6], words[7]});
        } else {
            // ---- online softmax of this lane's column
            const bool all = mapped && at >= see.lo && at + 15 <= see.hi;
            int e[16];      // exponents of the values
#pragma unroll
            for (int i = 0; i < 16; i++) {
                e[i] = (int)(int8_t)(evn[i >> 2] >> (8 * (i & 3)));
                s[i] = score(s[i], (int)(int8_t)(ekn[i >> 2] >> (8 * (i & 3))), at + i);
            }
            if (!__all(all)) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const bool ok = mapped && at + i >= see.lo && at + i <= see.hi;
                    s[i] = ok ? s[i] : -INFINITY;
                    e[i] = ok ? e[i] : -1000;
                }
            }
            float mb = -INFINITY, top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 16; i++) mb = fmaxf(mb, s[i]);
            raise(mb);
#pragma unroll
            for (int i = 0; i < 16; i++) {
                s[i] -= ref;
                top = fmaxf(top, s[i] + (float)e[i]);
            }
            rescale(top);
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float w[2];
#pragma unroll
                for (int u = 0; u < 2; u++) {
                    const float p = fast_exp2(s[i + u]);
                    l += p;
                    w[u] = ldexpf(p, e[i + u] - k + 14);
                    w[u] = e[i + u] == Q8_NAN ? __uint_as_float(0x7fc00000u) : w[u];
                }
                uint32_t hi, lo;
                split2_halves(w[0], w[1], hi, lo);
                if constexpr (GP == 16) {
                    const f16x2_t y = __builtin_bit_cast(f16x2_t, hi), z = __builtin_bit_cast(f16x2_t, lo);
                    wb[i >> 3][0][i & 7] = y[0];
                    wb[i >> 3][0][(i & 7) + 1] = y[1];
                    wb[i >> 3][1][i & 7] = z[0];
                    wb[i >> 3][1][(i & 7) + 1] = z[1];
                } else {
                    const f16x2_t y = __builtin_bit_cast(f16x2_t, term == 0 ? hi : term == 1 ? lo : 0u);
                    wb[i >> 3][0][i & 7] = y[0];
                    wb[i >> 3][0][(i & 7) + 1] = y[1];
                }
            }
        }
        // ---- sums
#pragma unroll
        for (int n = 0; n < ND; n++) {
            const f16x8_t va = q8_halves(vf[n][0], vf[n][1]), vb = q8_halves(vf[n][2], vf[n][3]);
#pragma unroll
            for (int p = 0; p < (GP == 16 ? 2 : 1); p++) {
                o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, wb[0][p], o[n], 0, 0, 0);
                o[n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vb, wb[1][p], o[n], 0, 0, 0);
            }
        }
        if (more) load_v(id_next);
    }

#pragma unroll
    for (int off = GP == 1 ? 1 : 16; off < 64; off <<= 1) l += __shfl_xor(l, off, WAVE);
    __shared__ __attribute__((aligned(16))) float so[WAVES][GP][HD + 4];
    __shared__ float2 sml[WAVES][GP];
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int n = 0; n < ND; n++) {
        float4 r;
        float *v = &r.x;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            float x = o[n][i];
            if constexpr (GP < 16) {      // its two terms
                const float other = __shfl_xor(x, GP, WAVE);
                x += other;
            }
            v[i] = ldexpf(x * inv, max(min(k - 14, 300), -300));
        }
        if (term == 0) *reinterpret_cast<float4 *>(&so[wave][head][16 * n + 4 * g]) = r;
    }
    if (lane < GP) sml[wave][lane] = make_float2(m, l);
    __syncthreads();
    for (int idx = threadIdx.x; idx < heads * HD; idx += 64 * WAVES) {
        const int hh = idx / HD, d = idx % HD;
        float M = -INFINITY, L = 0.f, r = 0.f, f[WAVES];
#pragma unroll
        for (int w = 0; w < WAVES; w++) M = fmaxf(M, sml[w][hh].x);
        const float ref = M > -INFINITY ? M : 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; w++) {
            const float2 ml = sml[w][hh];
            f[w] = ml.y == 0.f ? 0.f : fast_exp2(ml.x - ref) * ml.y;
            L += f[w];
        }
        // shares of one: the sum stays within the values, up to the ends of float32
        const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
        for (int w = 0; w < WAVES; w++) r = fmaf(f[w] * inv, so[w][hh][d], r);
        const int64_t at = (int64_t)t * a.H + h0 + hh;
        if (chunks == 1) {
            a.out[at * HD + d] = r;
        } else {
            part_o[(at * chunks + ch) * HD + d] = r;
            if (d == 0) part_ml[at * chunks + ch] = make_float2(M, L);
        }
    }
}

// Joins the chunks of a row and head: 256 threads as groups of HD / 4, a group the chunks of its number modulo the groups', so that a chunk's partial sums
// are asked for beside others' (64 chunks of 32 heads, one wave each and a chunk at a time: 37 us).  The order of every sum is fixed.
template <int HD>
__global__ __launch_bounds__(256) void k_join_q8(Q8Attention a, const int32_t *__restrict__ first, const int32_t *__restrict__ ctx_len, int max_ctx, int chunk,
                                                 int chunks, const float *__restrict__ part_o, const float2 *__restrict__ part_ml) {
    constexpr int PER = HD / 4, GROUPS = 256 / PER;
    __shared__ __attribute__((aligned(16))) float4 sum[GROUPS][PER];
    __shared__ float sl[GROUPS];
    const int t = blockIdx.x, h = blockIdx.y, gr = threadIdx.x / PER, d = threadIdx.x % PER;
    const Seen see = seen_of(ctx_len[t], first ? first[t] : 0, max_ctx, a.window, a.table_stride);
    const int64_t item = (int64_t)t * a.H + h;
    const int n = see.hi < see.lo ? 0 : ((see.hi >> 6) - (see.lo >> 6)) / chunk + 1;
    const float2 *ml = part_ml + item * chunks;
    const float4 *po = reinterpret_cast<const float4 *>(part_o + item * chunks * HD) + d;
    float M = -INFINITY;
    for (int i = threadIdx.x & 63; i < n; i += 64) M = fmaxf(M, ml[i].x);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, WAVE));
    const float ref = M > -INFINITY ? M : 0.f;
    // a position weighs at most one, and there are at most max_ctx: all weights together at most 1, so that the sum stays within the values up to the ends of float32
    const float scale = ldexpf(1.f, -(32 - __clz(max_ctx)));
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int i = gr; i < n; i += GROUPS) {
        const float2 w = ml[i];
        const float4 o = po[(int64_t)i * PER];
        const float f = w.y == 0.f ? 0.f : fast_exp2(w.x - ref) * (w.y * scale);      // a chunk without a visible position left zeros
        L += f;
        acc = make_float4(fmaf(f, o.x, acc.x), fmaf(f, o.y, acc.y), fmaf(f, o.z, acc.z), fmaf(f, o.w, acc.w));
    }
    sum[gr][d] = acc;
    if (d == 0) sl[gr] = L;
    __syncthreads();
    if (gr) return;
#pragma unroll
    for (int i = 1; i < GROUPS; i++) {
        const float4 o = sum[i][d];
        acc = make_float4(acc.x + o.x, acc.y + o.y, acc.z + o.z, acc.w + o.w);
        L += sl[i];
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *reinterpret_cast<float4_u *>(a.out + item * HD + 4 * d) = (float4_u){acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv};
}

struct Plan { int chunk, chunks; size_t rows; };

int visible_tiles(int max_ctx, int window) {
    const int64_t all = ((int64_t)max_ctx + TILE - 1) / TILE;
    return (int)(window > 0 ? std::min<int64_t>(all, ((int64_t)window + TILE - 2) / TILE + 1) : all);
}

// us of one row at 1520 positions of 32 heads / one at 131067 of 8 KV heads / 32 of 32 heads at 512 - 8192 / 8 capped ones of 40 heads at 1 - 2048: 256 workgroups
// 11.6 / 59 / 206 / 22.8, 512 11.2 / 59 / 206 / 21.9, 1024 11.6 / 67 / 206 / 25.0, 2048 11.3 / 81 / 206 / 25.9; chunks of at most 16 tiles 11.0 / 66 / 214 / 21.8;
// of at least two a wave 12.5 / 59 / 206 / 21.8.
constexpr int WANT = 512, CHUNK_TILES = 32;

Plan plan(int T, int H, int Hkv, int max_ctx, int window) {
    const int tiles = std::max(1, visible_tiles(max_ctx, window)), G = H / Hkv;
    const int64_t pairs = (int64_t)T * Hkv * ((G + 15) / 16);
    const int64_t want = std::max<int64_t>((WANT + pairs - 1) / pairs, (tiles + CHUNK_TILES - 1) / CHUNK_TILES);
    Plan p;
    p.chunk = (int)std::max<int64_t>(WAVES, (tiles + want - 1) / want);
    p.chunks = (tiles + p.chunk - 1) / p.chunk;
    p.rows = (size_t)T * H * (1 + (tiles + CHUNK_TILES - 1) / CHUNK_TILES) + (size_t)WANT * std::min(G, 16);
    return p;
}

template <int HD, int GP>
void launch_decode(const Q8Attention &a, const int32_t *seq_slot, const int32_t *first, const int32_t *ctx_len, int max_ctx, int T, const Plan &p, char *scratch,
                   hipStream_t s) {
    float *part_o = (float *)(scratch + ld::align_up(p.rows * 8, 256));
    float2 *part_ml = (float2 *)scratch;
    const int parts = (a.H / a.Hkv + 15) / 16;
    const dim3 grid((unsigned)((int64_t)T * p.chunks * a.Hkv * parts)), block(64 * WAVES);
    if (a.softcap > 0.f || a.slopes)
        LD_LAUNCH((k_decode_q8<HD, GP, true>), grid, block, 0, s, a, seq_slot, first, ctx_len, max_ctx, p.chunk, p.chunks, part_o, part_ml);
    else
        LD_LAUNCH((k_decode_q8<HD, GP, false>), grid, block, 0, s, a, seq_slot, first, ctx_len, max_ctx, p.chunk, p.chunks, part_o, part_ml);
    if (p.chunks > 1) LD_LAUNCH(k_join_q8<HD>, dim3(T, a.H), dim3(256), 0, s, a, first, ctx_len, max_ctx, p.chunk, p.chunks, part_o, part_ml);
}

template <int HD>
void launch_decode(const Q8Attention &a, const int32_t *seq_slot, const int32_t *first, const int32_t *ctx_len, int max_ctx, int T, const Plan &p, char *scratch,
                   hipStream_t s) {
    const int G = a.H / a.Hkv;
#define LD_DECODE(GP_) launch_decode<HD, GP_>(a, seq_slot, first, ctx_len, max_ctx, T, p, scratch, s)
    if (G == 1) LD_DECODE(1);
    else if (G == 2) LD_DECODE(2);
    else if (G <= 4) LD_DECODE(4);
    else if (G <= 8) LD_DECODE(8);
    else LD_DECODE(16);
#undef LD_DECODE
}

}  // namespace

extern "C" {

size_t ldk_attention_q8_scratch_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t max_ctx, int32_t window) {
    if (T <= 0 || H <= 0 || Hkv <= 0 || H % Hkv || (hd != 64 && hd != 128) || max_ctx < 0 || window < 0) return 0;
    const size_t rows = plan(T, H, Hkv, max_ctx, window).rows;
    return ld::align_up(rows * 8, 256) + rows * hd * 4;
}

ld_status ldk_paged_attention_q8(const float *q, int32_t q_stride, const int8_t *codes, const int8_t *expo, const int32_t *table,
                                 int32_t table_stride, const int32_t *seq_slot, const int32_t *first, const int32_t *ctx_len, int32_t max_ctx,
                                 int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t window, float softcap, const float *slopes, float *out,
                                 void *scratch, size_t scratch_bytes, void *stream) {
    if (T == 0) return LD_OK;
    const Q8Attention a{q, q_stride, codes, expo, table, table_stride, H, Hkv, window, softcap, slopes, out};
    if (T < 0 || max_ctx < 0 || !seq_slot || !ctx_len || bad_attention(a, hd)) return ld::fail(LD_E_INVAL, "ldk_paged_attention_q8: bad argument");
    const Plan p = plan(T, H, Hkv, max_ctx, window);
    if (H > 65535 || (int64_t)T * p.chunks > INT32_MAX / H || too_large((int64_t)T * p.chunks * Hkv * ((H / Hkv + 15) / 16), 64 * WAVES))
        return ld::fail(LD_E_RANGE, "ldk_paged_attention_q8: more than 65535 heads, or too many rows");
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < ldk_attention_q8_scratch_bytes(T, H, Hkv, hd, max_ctx, window))
        return ld::fail(LD_E_INVAL, "ldk_paged_attention_q8: scratch too small, or not aligned to 16 bytes");
    hipStream_t s = (hipStream_t)stream;
    if (hd == 128) launch_decode<128>(a, seq_slot, first, ctx_len, max_ctx, T, p, (char *)scratch, s);
    else launch_decode<64>(a, seq_slot, first, ctx_len, max_ctx, T, p, (char *)scratch, s);
    return launched("k_decode_q8");
}

}  // extern "C"
