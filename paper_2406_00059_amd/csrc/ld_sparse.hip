// Decode attention over the cache blocks that a cheap score selects for each query, and the bounds it scores with.
//
// A block of 16 positions is described, per KV head, by the largest and the smallest value of its keys in every
// dimension, as 8-bit integers of a power of two: with q rounded to 8-bit integers the same way,
//   score = sum_i (q_i >= 0 ? q_i hi_i : q_i lo_i)
// bounds q.k over the block's positions (up to the rounding of q).  Integer sums and powers of two: a score has one
// value, however the work is cut, and so has the choice.  A block and head cost 2 hd + 4 bytes to score against
// 64 hd to attend to (bf16).
#include "ld_device.h"

#include <algorithm>
#include <cmath>

using namespace ldd;

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

inline ld_status launched(const char *what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        ld::set_error("launch of %s failed: %s", what, hipGetErrorString(e));
        return LD_E_HIP;
    }
    return LD_OK;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t INF_BITS = 0x7f800000u;

// e of the unit 2^e in which a largest magnitude (as bits, finite) counts 64 .. 127: floor(log2 max) - 6, not below -126.
__device__ __forceinline__ int unit_exponent(uint32_t top) { return top ? max(ilogbf(__uint_as_float(top)) - 6, -126) : 0; }

// Maximum and sum over the 16 lanes of a row, in all of them (rotations within the row).
template <int N> __device__ __forceinline__ float row_rotate(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + N, 0xf, 0xf, false));
}
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, row_rotate<8>(v));
    v = fmaxf(v, row_rotate<4>(v));
    v = fmaxf(v, row_rotate<2>(v));
    return fmaxf(v, row_rotate<1>(v));
}
__device__ __forceinline__ float row_sum(float v) {
    v += row_rotate<8>(v);
    v += row_rotate<4>(v);
    v += row_rotate<2>(v);
    return v + row_rotate<1>(v);
}

// ---------------------------------------------------------------- bounds of a block's keys

// One wave a (block, KV head): the 16 key rows, 8 elements a lane and load; rows meet by shuffles.  Bound by the keys' bytes.
template <typename KT, int HD>
__global__ __launch_bounds__(256) void k_kv_summary(const KT *__restrict__ pool, int Hkv, const int32_t *__restrict__ table, int table_stride,
                                                    const int32_t *__restrict__ ranges, int8_t *__restrict__ bounds, float *__restrict__ unit) {
    constexpr int LPR = HD / 8, ROWS = 64 / LPR, PASSES = 16 / ROWS;      // lanes a key row, rows a pass
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int32_t *range = ranges + (int64_t)blockIdx.y * 3;
    const int seq = range[0], first = range[1], end = range[2];
    if (first < 0 || first >= end) return;
    const int64_t b = first / 16 + item / Hkv;
    const int kvh = (int)(item % Hkv);
    if (b * 16 >= end) return;
    const int phys = table[(int64_t)seq * table_stride + b];
    if (phys < 0) return;
    const int real = (int)min((int64_t)16, end - b * 16);
    const KT *keys = pool + (int64_t)phys * kv_block_elems(Hkv, HD) + kv_k_offset(HD, kvh, 0, 0);
    const int d = (lane % LPR) * 8;
    float lo[8], hi[8];
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) { lo[e] = INFINITY; hi[e] = -INFINITY; }
#pragma unroll
    for (int p = 0; p < PASSES; p++) {
        const int slot = p * ROWS + lane / LPR;
        if (slot >= real) continue;
        float v[8];
        load8_stream(keys + (int64_t)slot * HD + d, v);
#pragma unroll
        for (int e = 0; e < 8; e++) {
            lo[e] = fminf(lo[e], v[e]);
            hi[e] = fmaxf(hi[e], v[e]);
            top = max(top, abs_bits(v[e]));      // compared as bits: a NaN stays
        }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
#pragma unroll
    for (int off = LPR; off < 64; off <<= 1)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            lo[e] = fminf(lo[e], __shfl_xor(lo[e], off, WAVE));
            hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], off, WAVE));
        }
    const int64_t at = (int64_t)phys * Hkv + kvh;
    const bool finite = top < INF_BITS;
    const int ue = finite ? unit_exponent(top) : 0;
    if (lane < LPR) {
        union { int8_t c[8]; uint2 u; } up, down;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            up.c[e] = finite ? (int8_t)fminf(ceilf(ldexpf(hi[e], -ue)), 127.f) : 0;
            down.c[e] = finite ? (int8_t)fmaxf(floorf(ldexpf(lo[e], -ue)), -127.f) : 0;
        }
        *reinterpret_cast<uint2 *>(bounds + at * 2 * HD + d) = up.u;
        *reinterpret_cast<uint2 *>(bounds + at * 2 * HD + HD + d) = down.u;
    }
    if (lane == 0) unit[at] = finite ? ldexpf(1.f, ue) : INFINITY;
}

// ---------------------------------------------------------------- visible blocks of a row

struct Visible { int start, b0, n; };      // first visible position, its block, number of blocks
__device__ __forceinline__ Visible visible(int ctx, int window) {
    Visible v;
    v.start = (window > 0 && ctx > window) ? ctx - window : 0;
    v.b0 = v.start >> 4;
    v.n = ctx > 0 ? ((ctx + 15) >> 4) - v.b0 : 0;
    return v;
}

// ---------------------------------------------------------------- scores

// The group's queries as operand columns of the integer matrix instructions: their positive parts against the upper bounds, their
// negative parts against the lower; lane l holds head g0 + l % 16, dimensions 64 j + 16 (l / 16) .. + 16.
template <int HD>
struct ScoreQuery {
    i32x4 b[HD / 32];
    float unit;
    bool real;
    __device__ __forceinline__ void load(const float *__restrict__ q, int64_t head0, int g0, int G, int lane) {      // q: the row; head0: of the group
        constexpr int NJ = HD / 64;
        const int c16 = lane & 15, h = lane >> 4;
        real = g0 + c16 < G;
        const float *qp = q + (head0 + (real ? g0 + c16 : 0)) * HD + 16 * h;
        float f[NJ][16];
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < NJ; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
                f[j][e] = qp[64 * j + e];
                top = max(top, abs_bits(f[j][e]));
            }
        top = max(top, (uint32_t)__shfl_xor((int)top, 16, WAVE));
        top = max(top, (uint32_t)__shfl_xor((int)top, 32, WAVE));
        const bool ok = real && top < INF_BITS;
        const int qe = ok ? unit_exponent(top) : 0;
#pragma unroll
        for (int j = 0; j < NJ; j++)
#pragma unroll
            for (int w = 0; w < 4; w++) {
                uint32_t pos = 0, neg = 0;
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int c = ok ? (int)fminf(fmaxf(rintf(ldexpf(f[j][4 * w + e], -qe)), -127.f), 127.f) : 0;
                    pos |= (uint32_t)(max(c, 0) & 255) << (8 * e);
                    neg |= (uint32_t)(min(c, 0) & 255) << (8 * e);
                }
                b[j][w] = (int32_t)pos;
                b[NJ + j][w] = (int32_t)neg;
            }
        unit = ldexpf(1.f, qe);
    }
};

// Scores of the 16 blocks whose physical ids lanes l % 16 hold: lane l < 64 returns that of block 4 (l / 16) + l % 4.
template <int HD>
__device__ __forceinline__ float score_tile(const ScoreQuery<HD> &q, const int8_t *__restrict__ bounds, const float *__restrict__ unit, int64_t phys,
                                            int Hkv, int kvh, int lane) {
    const int h = lane >> 4;
    const int8_t *rec = bounds + (phys * Hkv + kvh) * 2 * HD + 16 * h;
    i32x4 a[HD / 32];
#pragma unroll
    for (int j = 0; j < HD / 32; j++) a[j] = *reinterpret_cast<const i32x4 *>(rec + 64 * j);
    const float un = unit[phys * Hkv + kvh];
    i32x4 acc = (i32x4){0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < HD / 32; j++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], q.b[j], acc, 0, 0, 0);
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float u = __shfl(un, 4 * h + i, WAVE);
        s[i] = row_max(q.real ? (u < INFINITY ? (float)acc[i] * q.unit * u : INFINITY) : -INFINITY);
    }
    const int i = lane & 3;
    return i == 0 ? s[0] : i == 1 ? s[1] : i == 2 ? s[2] : s[3];
}

// A wave tiles_per_wave tiles of 16 blocks of a (row, KV head).
template <int HD>
__global__ __launch_bounds__(256) void k_sparse_score(const float *__restrict__ q, int q_stride, const int8_t *__restrict__ bounds,
                                                      const float *__restrict__ unit, const int32_t *__restrict__ table, int table_stride,
                                                      const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len, int max_ctx,
                                                      int Hkv, int G, int window, int tiles_per_wave, int stride, float *__restrict__ scores) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.z, kvh = blockIdx.y;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    const int tile0 = (blockIdx.x * 4 + wave) * tiles_per_wave;
    if (tile0 * 16 >= v.n) return;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride + v.b0;
    float *dst = scores + ((int64_t)t * Hkv + kvh) * stride;
    for (int g0 = 0; g0 < G; g0 += 16) {
        ScoreQuery<HD> sq;
        sq.load(q + (int64_t)t * q_stride, (int64_t)kvh * G, g0, G, lane);
        for (int tile = tile0; tile < tile0 + tiles_per_wave && tile * 16 < v.n; tile++) {
            const float x = score_tile<HD>(sq, bounds, unit, trow[min(tile * 16 + (lane & 15), v.n - 1)], Hkv, kvh, lane);
            const int at = tile * 16 + 4 * (lane >> 4) + (lane & 3);
            if ((lane & 15) < 4 && at < v.n) dst[at] = g0 ? fmaxf(dst[at], x) : x;
        }
    }
}

// ---------------------------------------------------------------- selection

__device__ __forceinline__ uint32_t order_key(float f) {
    const uint32_t b = __float_as_uint(f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// The choice among the n > budget visible blocks of a (row, KV head), by WAVES waves that hold KPL scores a lane (block
// j 64 WAVES + thread).  The threshold is searched between the smallest and the largest key by halves, counting in the
// ballots; where a count hits the number wanted the search is over (a bell of scores: after some 10 - 14 steps), otherwise it ends
// at a key that several share, of which the first in index order are taken.  All waves call it; out: list of budget ascending
// logical blocks (LDS or global), sm: 2 WAVES words of LDS where WAVES > 1.
template <int WAVES, int KPL>
__device__ __forceinline__ void select_blocks(const float *sc, int n, int b0, int budget, int keep_first, int keep_last, int32_t *out, int32_t *out2,
                                              uint32_t *sm) {
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? threadIdx.x >> 6 : 0;
    const int c1 = n - keep_last, need = budget - keep_first - keep_last;
    uint32_t key[KPL], lo = 0xffffffffu, hi = 0;
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const int i = (j * WAVES + wave) * 64 + lane;
        const bool cand = i >= keep_first && i < c1;
        key[j] = cand ? order_key(sc[i]) : 0;      // no score has key 0
        if (cand) { lo = min(lo, key[j]); hi = max(hi, key[j]); }
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, off, WAVE));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, off, WAVE));
    }
    if (WAVES > 1) {
        if (lane == 0) { sm[wave] = lo; sm[WAVES + wave] = hi; }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; w++) { lo = min(lo, sm[w]); hi = max(hi, sm[WAVES + w]); }
        __syncthreads();
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    // count over all waves, one barrier each: the halves of sm take turns
    int turn = 0;
    auto total = [&](int c) {
        if (WAVES == 1) return c;
        uint32_t *p = sm + (turn++ & 1) * WAVES;
        if (lane == 0) p[wave] = (uint32_t)c;
        __syncthreads();
        int s = 0;
#pragma unroll
        for (int w = 0; w < WAVES; w++) s += (int)p[w];
        return __builtin_amdgcn_readfirstlane(s);
    };
    uint32_t from = hi;      // keys >= from are taken
    bool exact = need <= 0;
    if (exact) from = 0xffffffffu;
    while (!exact && lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int c = 0;
#pragma unroll
        for (int j = 0; j < KPL; j++) c += __popcll(__ballot(key[j] >= mid));
        c = total(c);
        if (c == need) { from = mid; exact = true; }
        else if (c > need) lo = mid;
        else hi = mid - 1;
    }
    int eq = 0;      // how many of the keys equal to the threshold are taken; where exact, every key >= from is
    if (!exact) {
        from = lo;
        int c = 0;
#pragma unroll
        for (int j = 0; j < KPL; j++) c += __popcll(__ballot(key[j] > from));
        eq = need - total(c);
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int at = 0, met = 0;      // written so far, equal keys met so far
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const int i = (j * WAVES + wave) * 64 + lane;
        if (j * WAVES * 64 >= n) break;
        const bool kept = i < n && (i < keep_first || i >= c1);
        const bool tie = !exact && key[j] == from;
        const uint64_t bt = __ballot(tie);
        int met_here = met;
        if (WAVES > 1 && !exact) {
            __syncthreads();
            if (lane == 0) sm[wave] = (uint32_t)__popcll(bt);
            __syncthreads();
            int all = 0;
            for (int w = 0; w < WAVES; w++) {
                if (w < wave) met_here += (int)sm[w];
                all += (int)sm[w];
            }
            met += all;
        } else {
            met += __popcll(bt);
        }
        const bool take = kept || (exact ? key[j] >= from : key[j] > from || (tie && met_here + __popcll(bt & below) < eq));
        const uint64_t bk = __ballot(take);
        int at_here = at;
        if (WAVES > 1) {
            __syncthreads();
            if (lane == 0) sm[WAVES + wave] = (uint32_t)__popcll(bk);
            __syncthreads();
            int all = 0;
            for (int w = 0; w < WAVES; w++) {
                if (w < wave) at_here += (int)sm[WAVES + w];
                all += (int)sm[WAVES + w];
            }
            at += all;
        } else {
            at += __popcll(bk);
        }
        const int slot = at_here + __popcll(bk & below);
        if (take && slot < budget) {
            out[slot] = b0 + i;
            if (out2) out2[slot] = b0 + i;
        }
    }
}

constexpr int SELECT_KEYS = 16;      // a lane's keys in the launch of its own: 16384 blocks a (row, KV head)

__global__ __launch_bounds__(1024) void k_sparse_select(const float *__restrict__ scores, int stride, const int32_t *__restrict__ ctx_len,
                                                        int max_ctx, int Hkv, int window, int budget, int keep_first, int keep_last,
                                                        int32_t *__restrict__ sel) {
    __shared__ uint32_t sm[32];
    const int t = blockIdx.y, kvh = blockIdx.x;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    int32_t *out = sel + ((int64_t)t * Hkv + kvh) * budget;
    if (v.n <= budget) {
        for (int i = threadIdx.x; i < budget; i += 1024) out[i] = i < v.n ? v.b0 + i : -1;
        return;
    }
    const float *sc = scores + ((int64_t)t * Hkv + kvh) * stride;
    if (v.n <= 2048) select_blocks<16, 2>(sc, v.n, v.b0, budget, keep_first, keep_last, out, nullptr, sm);
    else select_blocks<16, SELECT_KEYS>(sc, v.n, v.b0, budget, keep_first, keep_last, out, nullptr, sm);
}

// The same for more blocks than fit in registers: every step of the search reads the scores again.
__global__ __launch_bounds__(1024) void k_sparse_select_long(const float *__restrict__ scores, int stride, const int32_t *__restrict__ ctx_len,
                                                             int max_ctx, int Hkv, int window, int budget, int keep_first, int keep_last,
                                                             int32_t *__restrict__ sel) {
    __shared__ uint32_t sm[32];
    const int t = blockIdx.y, kvh = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    int32_t *out = sel + ((int64_t)t * Hkv + kvh) * budget;
    if (v.n <= budget) {
        for (int i = threadIdx.x; i < budget; i += 1024) out[i] = i < v.n ? v.b0 + i : -1;
        return;
    }
    const float *sc = scores + ((int64_t)t * Hkv + kvh) * stride;
    const int c0 = keep_first, c1 = v.n - keep_last, need = budget - keep_first - keep_last;
    auto sum = [&](int c) {      // over the workgroup
        for (int off = 32; off > 0; off >>= 1) c += __shfl_xor(c, off, WAVE);
        __syncthreads();
        if (lane == 0) sm[wave] = (uint32_t)c;
        __syncthreads();
        int s = 0;
        for (int w = 0; w < 16; w++) s += (int)sm[w];
        return s;
    };
    // the largest key that at least `need` candidates reach, bit by bit
    uint32_t from = 0;
    for (int bit = 31; bit >= 0; bit--) {
        const uint32_t mid = from | (1u << bit);
        int c = 0;
        for (int i = c0 + threadIdx.x; i < c1; i += 1024) c += order_key(sc[i]) >= mid;
        if (sum(c) >= need) from = mid;
    }
    int c = 0;
    for (int i = c0 + threadIdx.x; i < c1; i += 1024) c += order_key(sc[i]) > from;
    const int eq = need - sum(c);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int at = 0, met = 0;
    for (int base = 0; base < v.n; base += 1024) {
        const int i = base + threadIdx.x;
        const bool cand = i >= c0 && i < c1;
        const uint32_t k = cand ? order_key(sc[i]) : 0;
        const uint64_t bt = __ballot(cand && k == from);
        __syncthreads();
        if (lane == 0) sm[wave] = (uint32_t)__popcll(bt);
        __syncthreads();
        int here = met;
        for (int w = 0; w < 16; w++) {
            if (w < wave) here += (int)sm[w];
            met += (int)sm[w];
        }
        const bool take = i < v.n && (!cand || (need > 0 && (k > from || (k == from && here + __popcll(bt & below) < eq))));
        const uint64_t bk = __ballot(take);
        if (lane == 0) sm[16 + wave] = (uint32_t)__popcll(bk);
        __syncthreads();
        int slot = at + __popcll(bk & below);
        for (int w = 0; w < 16; w++) {
            if (w < wave) slot += (int)sm[16 + w];
            at += (int)sm[16 + w];
        }
        if (take && slot < budget) out[slot] = v.b0 + i;
    }
}

// ---------------------------------------------------------------- attention over the selected blocks

// Eight elements as loaded.
template <typename KT> struct Eight;
template <> struct Eight<bf16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const bf16_t *p) { w = load_stream16(p); }
    __device__ __forceinline__ float at(int e) const { return __uint_as_float((e & 1) ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16); }
};
template <> struct Eight<float> {
    u32x4 w[2];
    __device__ __forceinline__ void load(const float *p) { w[0] = load_stream16(p); w[1] = load_stream16(p + 4); }
    __device__ __forceinline__ float at(int e) const { return __uint_as_float(w[e >> 2][e & 3]); }
};

// What a wave has of GT query heads: the maximum (log2 domain), its lanes' shares of the sum (lane: position l % 16) and of the
// output (lane: dimensions l / 2 + 32 u, eight of a block's positions).
template <int HD, int GT>
struct Share {
    float m[GT], l[GT], o[GT][HD / 32];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int g = 0; g < GT; g++) {
            m[g] = -INFINITY;
            l[g] = 0.f;
#pragma unroll
            for (int u = 0; u < HD / 32; u++) o[g][u] = 0.f;
        }
    }
};

// A block's keys and values as a wave reads them, 1 KB a load: keys: lane = position l % 16, dimensions 32 j + 8 (l / 16) .. + 8;
// values (transposed in the block): lane = dimension l / 2 + 32 u, positions 8 (l % 2) .. + 8.
template <typename KT, int HD>
struct BlockData {
    Eight<KT> k[HD / 32], v[HD / 32];
    __device__ __forceinline__ void load(const KT *blk, int Hkv, int kvh, int lane) {
        const KT *kp = blk + kv_k_offset(HD, kvh, lane & 15, 8 * (lane >> 4));
        const KT *vp = blk + kv_v_offset(Hkv, HD, kvh, 8 * (lane & 1), lane >> 1);
#pragma unroll
        for (int j = 0; j < HD / 32; j++) k[j].load(kp + 32 * j);
#pragma unroll
        for (int u = 0; u < HD / 32; u++) v[u].load(vp + (int64_t)u * 32 * 16);
    }
};

// One block added to the share.  qs: the heads' queries in LDS, scaled by log2(e) / sqrt(hd); pl: 16 floats of LDS of the wave's own.
template <typename KT, int HD, int GT>
__device__ __forceinline__ void attend_block(BlockData<KT, HD> &d, int pos0, int start, int ctx, const float *qs, float *pl, Share<HD, GT> &s, int lane) {
    const int pos = pos0 + (lane & 15);
    const bool ok = pos >= start && pos < ctx, full = pos0 >= start && pos0 + 16 <= ctx;
    float sc[GT];
#pragma unroll
    for (int g = 0; g < GT; g++) {
        float a = 0.f;
#pragma unroll
        for (int j = 0; j < HD / 32; j++) {
            const float4 q0 = *reinterpret_cast<const float4 *>(qs + g * HD + 32 * j + 8 * (lane >> 4));
            const float4 q1 = *reinterpret_cast<const float4 *>(qs + g * HD + 32 * j + 8 * (lane >> 4) + 4);
            const float qv[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
            for (int e = 0; e < 8; e++) a += qv[e] * d.k[j].at(e);
        }
        a += __shfl_xor(a, 16, WAVE);
        a += __shfl_xor(a, 32, WAVE);
        sc[g] = ok ? a : -INFINITY;
    }
#pragma unroll
    for (int g = 0; g < GT; g++) {
        const float m_new = fmaxf(s.m[g], row_max(sc[g]));      // a selected block holds a visible position
        const float corr = fast_exp2(s.m[g] - m_new);
        const float p = ok ? fast_exp2(sc[g] - m_new) : 0.f;
        s.m[g] = m_new;
        s.l[g] = s.l[g] * corr + p;
        if (lane < 16) pl[lane] = p;
        __builtin_amdgcn_wave_barrier();      // a wave's LDS operations execute in order
        const float4 p0 = *reinterpret_cast<const float4 *>(pl + 8 * (lane & 1)), p1 = *reinterpret_cast<const float4 *>(pl + 8 * (lane & 1) + 4);
        __builtin_amdgcn_wave_barrier();
        const float pv[8] = {p0.x, p0.y, p0.z, p0.w, p1.x, p1.y, p1.z, p1.w};
#pragma unroll
        for (int u = 0; u < HD / 32; u++) {
            float a = s.o[g][u] * corr;
            if (full) {
#pragma unroll
                for (int e = 0; e < 8; e++) a += pv[e] * d.v[u].at(e);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) {      // what an unwritten slot holds is not looked at
                    const int ps = pos0 + 8 * (lane & 1) + e;
                    if (ps >= start && ps < ctx) a += pv[e] * d.v[u].at(e);
                }
            }
            s.o[g][u] = a;
        }
    }
}

// The waves' shares into LDS: o [wave][GT][HD], m and l [wave][GT].
template <int HD, int GT>
__device__ __forceinline__ void put_share(const Share<HD, GT> &s, float *o, float *ml, int waves, int wave, int lane) {
#pragma unroll
    for (int g = 0; g < GT; g++) {
        const float l = row_sum(s.l[g]);
#pragma unroll
        for (int u = 0; u < HD / 32; u++) {
            const float a = s.o[g][u] + __shfl_xor(s.o[g][u], 1, WAVE);
            if (!(lane & 1)) o[(wave * GT + g) * HD + (lane >> 1) + 32 * u] = a;
        }
        if (lane == 0) { ml[wave * GT + g] = s.m[g]; ml[(waves + wave) * GT + g] = l; }
    }
}

// Queries of GT heads into LDS, scaled.
template <int HD, int GT>
__device__ __forceinline__ void stage_queries(const float *__restrict__ q, float *qs) {
    const float scale = 1.4426950408889634f / sqrtf((float)HD);
    for (int i = threadIdx.x; i < GT * HD; i += blockDim.x) qs[i] = q[i] * scale;
}

// Split form: a workgroup a chunk of cb selected blocks of a (row, KV head), a wave every fourth block, GT heads at a time.
template <typename KT, int HD, int GT>
__global__ __launch_bounds__(256) void k_sparse_attend(const float *__restrict__ q, int q_stride, const KT *__restrict__ pool, int Hkv,
                                                       const int32_t *__restrict__ table, int table_stride,
                                                       const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len, int max_ctx,
                                                       int G, int window, int budget, const int32_t *__restrict__ sel, int cb,
                                                       float *__restrict__ part_o, float *__restrict__ part_ml) {
    __shared__ __attribute__((aligned(16))) float qs[GT * HD], pl[4][16], so[4 * GT * HD], sml[8 * GT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x, kvh = blockIdx.y, t = blockIdx.z, chunks = gridDim.x;
    const int ctx = min(ctx_len[t], max_ctx);
    const Visible v = visible(ctx, window);
    const int i0 = c * cb, i1 = min(i0 + cb, min(v.n, budget));
    if (i0 >= i1) return;
    const int32_t *list = sel + ((int64_t)t * Hkv + kvh) * budget;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride;
    for (int g0 = 0; g0 < G; g0 += GT) {
        const int64_t head = (int64_t)kvh * G + g0;
        stage_queries<HD, GT>(q + (int64_t)t * q_stride + head * HD, qs);
        __syncthreads();
        Share<HD, GT> s;
        s.clear();
        for (int i = i0 + wave; i < i1; i += 4) {
            const int b = list[i];
            BlockData<KT, HD> d;
            d.load(pool + (int64_t)trow[b] * kv_block_elems(Hkv, HD), Hkv, kvh, lane);
            attend_block<KT, HD, GT>(d, b * 16, v.start, ctx, qs, pl[wave], s, lane);
        }
        put_share<HD, GT>(s, so, sml, 4, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < GT * HD; i += 256) {
            const int g = i / HD;
            const float M = fmaxf(fmaxf(sml[g], sml[GT + g]), fmaxf(sml[2 * GT + g], sml[3 * GT + g]));
            float o = 0.f, L = 0.f;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const float a = fast_exp2(sml[w * GT + g] - M);
                o += a * so[w * GT * HD + i];
                L += a * sml[(4 + w) * GT + g];
            }
            const int64_t item = ((int64_t)t * Hkv * G + head + g) * chunks + c;
            part_o[item * HD + i % HD] = o;
            if (i % HD == 0) { part_ml[item * 2] = M; part_ml[item * 2 + 1] = L; }
        }
        __syncthreads();
    }
}

// Chunks of a (row, head) joined in their order: 256 threads, 256 / hd chunks at a time; a row that sees nothing is 0.
template <int HD>
__global__ __launch_bounds__(256) void k_sparse_join(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                     const int32_t *__restrict__ ctx_len, int max_ctx, int H, int window, int budget, int cb,
                                                     int chunks, float *__restrict__ out) {
    constexpr int LINES = 256 / HD;
    __shared__ float so[256], sl[LINES];
    const int h = blockIdx.x, t = blockIdx.y, d = threadIdx.x % HD, line = threadIdx.x / HD;
    const int n = min(visible(min(ctx_len[t], max_ctx), window).n, budget);
    const int nc = (n + cb - 1) / cb;
    const int64_t base = ((int64_t)t * H + h) * chunks;
    float M = -INFINITY;
    for (int c = threadIdx.x & 63; c < nc; c += 64) M = fmaxf(M, part_ml[(base + c) * 2]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, WAVE));
    float o = 0.f, L = 0.f;
#pragma unroll 8
    for (int c = line; c < nc; c += LINES) {
        const float2 ml = *reinterpret_cast<const float2 *>(part_ml + (base + c) * 2);
        const float a = fast_exp2(ml.x - M);
        o += a * part_o[(base + c) * HD + d];
        L += a * ml.y;
    }
    so[threadIdx.x] = o;
    if (d == 0) sl[line] = L;
    __syncthreads();
    if (line) return;
    L = 0.f; o = 0.f;
#pragma unroll
    for (int i = 0; i < LINES; i++) { o += so[i * HD + d]; L += sl[i]; }
    out[((int64_t)t * H + h) * HD + d] = nc ? o / L : 0.f;
}

// Everything for one (row, KV head) in one workgroup of 16 waves: scores into LDS, the choice, attention, the waves joined.  One launch
// and no scratch, for up to FUSED_BLOCKS visible blocks.
constexpr int FUSED_BLOCKS = 2048, FUSED_BUDGET = 1024;

template <typename KT, int HD, int GT>
__global__ __launch_bounds__(1024) void k_sparse_row(const float *__restrict__ q, int q_stride, const KT *__restrict__ pool,
                                                     const int8_t *__restrict__ bounds, const float *__restrict__ unit, int Hkv,
                                                     const int32_t *__restrict__ table, int table_stride, const int32_t *__restrict__ seq_slot,
                                                     const int32_t *__restrict__ ctx_len, int max_ctx, int G, int window, int budget,
                                                     int keep_first, int keep_last, float *__restrict__ out, int32_t *__restrict__ sel) {
    constexpr int W = 16;
    __shared__ float sc[FUSED_BLOCKS];
    __shared__ int32_t list[FUSED_BUDGET];
    __shared__ uint32_t sm[2 * W];
    __shared__ __attribute__((aligned(16))) float qs[GT * HD], pl[W][16], so[W * GT * HD], sml[2 * W * GT];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int kvh = blockIdx.x, t = blockIdx.y;
    const int ctx = min(ctx_len[t], max_ctx);
    const Visible v = visible(ctx, window);
    const int64_t H = (int64_t)Hkv * G;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride;
    int32_t *gsel = sel + ((int64_t)t * Hkv + kvh) * budget;
    if (v.n > budget) {
        for (int g0 = 0; g0 < G; g0 += 16) {
            ScoreQuery<HD> sq;
            sq.load(q + (int64_t)t * q_stride, (int64_t)kvh * G, g0, G, lane);
            for (int tile = wave; tile * 16 < v.n; tile += W) {
                const float x = score_tile<HD>(sq, bounds, unit, trow[v.b0 + min(tile * 16 + (lane & 15), v.n - 1)], Hkv, kvh, lane);
                const int at = tile * 16 + 4 * (lane >> 4) + (lane & 3);
                if ((lane & 15) < 4 && at < v.n) sc[at] = g0 ? fmaxf(sc[at], x) : x;
            }
        }
        __syncthreads();
        if (v.n <= 512) {
            if (wave == 0) select_blocks<1, 8>(sc, v.n, v.b0, budget, keep_first, keep_last, list, gsel, sm);
        } else {
            select_blocks<W, FUSED_BLOCKS / 1024>(sc, v.n, v.b0, budget, keep_first, keep_last, list, gsel, sm);
        }
    } else {
        for (int i = threadIdx.x; i < budget; i += 1024) {
            if (i < v.n) list[i] = v.b0 + i;
            gsel[i] = i < v.n ? v.b0 + i : -1;
        }
    }
    const int n = min(v.n, budget);
    for (int g0 = 0; g0 < G; g0 += GT) {
        const int64_t head = (int64_t)kvh * G + g0;
        stage_queries<HD, GT>(q + (int64_t)t * q_stride + head * HD, qs);
        __syncthreads();
        Share<HD, GT> s;
        s.clear();
        for (int i = wave; i < n; i += W) {
            const int b = list[i];
            BlockData<KT, HD> d;
            d.load(pool + (int64_t)trow[b] * kv_block_elems(Hkv, HD), Hkv, kvh, lane);
            attend_block<KT, HD, GT>(d, b * 16, v.start, ctx, qs, pl[wave], s, lane);
        }
        put_share<HD, GT>(s, so, sml, W, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < GT * HD; i += 1024) {
            const int g = i / HD;
            float M = -INFINITY, o = 0.f, L = 0.f;
#pragma unroll
            for (int w = 0; w < W; w++) M = fmaxf(M, sml[w * GT + g]);
#pragma unroll
            for (int w = 0; w < W; w++) {
                const float a = fast_exp2(sml[w * GT + g] - M);
                o += a * so[w * GT * HD + i];
                L += a * sml[(W + w) * GT + g];
            }
            out[((int64_t)t * H + head) * HD + i] = n ? o / L : 0.f;
        }
        __syncthreads();
    }
}

int visible_blocks(int max_ctx, int window) {
    const int all = (int)(((int64_t)max_ctx + 15) / 16);
    return window > 0 ? (int)std::min<int64_t>(all, ((int64_t)window + 14) / 16 + 1) : all;
}

// Selected blocks a workgroup attends to: so many that a launch has some two workgroups a CU, in steps of four.
int chunk_blocks(int T, int Hkv, int n) {
    const int64_t cb = ((int64_t)T * Hkv * n + 511) / 512;
    return (int)std::min<int64_t>((std::max<int64_t>(cb, 1) + 3) / 4 * 4, 32);
}

struct SparsePlan { int nb, n, cb, chunks; size_t scores, part_o; };
SparsePlan sparse_plan(int T, int H, int Hkv, int hd, int max_ctx, int window, int budget) {
    SparsePlan p;
    p.nb = visible_blocks(max_ctx, window);
    p.n = std::max(1, std::min(p.nb, budget));
    p.cb = chunk_blocks(T, Hkv, p.n);
    p.chunks = (p.n + p.cb - 1) / p.cb;
    p.scores = p.nb > budget ? ld::align_up((size_t)T * Hkv * p.nb * 4, 256) : 0;
    p.part_o = ld::align_up((size_t)T * H * p.chunks * hd * 4, 256);
    return p;
}

bool fused_form(int T, int Hkv, int nb, int budget) {
    static const int force = ld::env_flag("LD_SPARSE_FUSED", -1);
    if (force >= 0) return force && nb <= FUSED_BLOCKS && std::min(nb, budget) <= FUSED_BUDGET;
    return nb <= FUSED_BLOCKS && std::min(nb, budget) <= FUSED_BUDGET;
}

// Scratch that any call of up to T rows, contexts up to max_ctx and this budget can use.  The number of chunks is not monotonic in
// either, so it is bounded: n / cb <= 512 / (T Hkv) unless cb is at its cap of 32, and cb >= 4.
size_t scratch_bound(int T, int H, int Hkv, int hd, int max_ctx, int window, int budget) {
    const int nb = visible_blocks(max_ctx, window);
    const int64_t n = std::max(1, std::min(nb, budget)), rows = (int64_t)T * H;
    const int64_t items = std::min(rows * ((n + 3) / 4), std::max((int64_t)512 * (H / Hkv) + rows, rows * ((n + 31) / 32)));
    return (nb > budget ? ld::align_up((size_t)T * Hkv * nb * 4, 256) : 0) + ld::align_up((size_t)items * hd * 4, 256) +
           ld::align_up((size_t)items * 8, 256);
}

struct SparseArgs {
    const float *q; int q_stride; const void *pool; const int8_t *bounds; const float *unit; const int32_t *table; int table_stride;
    const int32_t *seq_slot, *ctx_len; int max_ctx, T, H, Hkv, window, budget, keep_first, keep_last; float *out; int32_t *sel; char *scratch;
};

template <typename KT, int HD, int GT>
void launch_sparse(const SparseArgs &a, hipStream_t s) {
    const KT *pool = (const KT *)a.pool;
    const int G = a.H / a.Hkv, nb = visible_blocks(a.max_ctx, a.window);
    if (fused_form(a.T, a.Hkv, nb, a.budget)) {
        LD_LAUNCH((k_sparse_row<KT, HD, GT>), dim3(a.Hkv, a.T), dim3(1024), 0, s, a.q, a.q_stride, pool, a.bounds, a.unit, a.Hkv, a.table,
                  a.table_stride, a.seq_slot, a.ctx_len, a.max_ctx, G, a.window, a.budget, a.keep_first, a.keep_last, a.out, a.sel);
        return;
    }
    const SparsePlan p = sparse_plan(a.T, a.H, a.Hkv, HD, a.max_ctx, a.window, a.budget);
    float *scores = (float *)a.scratch, *part_o = (float *)(a.scratch + p.scores), *part_ml = (float *)(a.scratch + p.scores + p.part_o);
    if (p.nb > a.budget) {
        const int tiles = (p.nb + 15) / 16;
        const int64_t waves = (int64_t)tiles * a.Hkv * a.T;
        const int per = (int)std::max<int64_t>(1, std::min<int64_t>(8, waves / 4096));      // tiles a wave
        LD_LAUNCH(k_sparse_score<HD>, dim3((tiles + 4 * per - 1) / (4 * per), a.Hkv, a.T), dim3(256), 0, s, a.q, a.q_stride, a.bounds, a.unit, a.table,
                  a.table_stride, a.seq_slot, a.ctx_len, a.max_ctx, a.Hkv, G, a.window, per, p.nb, scores);
    }
    if (p.nb <= 1024 * SELECT_KEYS)
        LD_LAUNCH(k_sparse_select, dim3(a.Hkv, a.T), dim3(1024), 0, s, scores, p.nb, a.ctx_len, a.max_ctx, a.Hkv, a.window, a.budget, a.keep_first,
                  a.keep_last, a.sel);
    else
        LD_LAUNCH(k_sparse_select_long, dim3(a.Hkv, a.T), dim3(1024), 0, s, scores, p.nb, a.ctx_len, a.max_ctx, a.Hkv, a.window, a.budget,
                  a.keep_first, a.keep_last, a.sel);
    LD_LAUNCH((k_sparse_attend<KT, HD, GT>), dim3(p.chunks, a.Hkv, a.T), dim3(256), 0, s, a.q, a.q_stride, pool, a.Hkv, a.table, a.table_stride,
              a.seq_slot, a.ctx_len, a.max_ctx, G, a.window, a.budget, a.sel, p.cb, part_o, part_ml);
    LD_LAUNCH(k_sparse_join<HD>, dim3(a.H, a.T), dim3(256), 0, s, part_o, part_ml, a.ctx_len, a.max_ctx, a.H, a.window, a.budget, p.cb, p.chunks, a.out);
}

template <typename KT, int HD>
void launch_sparse(const SparseArgs &a, hipStream_t s) {
    const int G = a.H / a.Hkv;      // heads that share a block's loads: the most of 4, 2, 1 that divide the group
    if (G % 4 == 0) launch_sparse<KT, HD, 4>(a, s);
    else if (G % 2 == 0) launch_sparse<KT, HD, 2>(a, s);
    else launch_sparse<KT, HD, 1>(a, s);
}

}  // namespace

extern "C" {

ld_status ldk_kv_summary(const void *pool_layer, int32_t dtype, const int32_t *table, int32_t table_stride, const int32_t *ranges,
                         int32_t n_ranges, int32_t max_len, int32_t Hkv, int32_t hd, int8_t *bounds, float *unit, void *stream) {
    if (n_ranges == 0 || max_len == 0) return LD_OK;
    if (!pool_layer || !table || !ranges || !bounds || !unit || n_ranges < 0 || max_len < 0 || Hkv <= 0 || (hd != 64 && hd != 128) ||
        (dtype != LD_BF16 && dtype != LD_F32) || ((uintptr_t)pool_layer & 15) || ((uintptr_t)bounds & 15))
        return ld::fail(LD_E_INVAL, "ldk_kv_summary: bad argument");
    if (n_ranges > 65535) return ld::fail(LD_E_RANGE, "ldk_kv_summary: more than 65535 ranges");
    // positions first .. first + max_len - 1 touch at most this many blocks
    const int64_t items = (((int64_t)max_len + 14) / 16 + 1) * Hkv;
    const dim3 grid((unsigned)((items + 3) / 4), n_ranges), block(256);
    hipStream_t s = (hipStream_t)stream;
#define LD_SUM(KT_, HD_) LD_LAUNCH((k_kv_summary<KT_, HD_>), grid, block, 0, s, (const KT_ *)pool_layer, Hkv, table, table_stride, ranges, bounds, unit)
    if (dtype == LD_BF16) { if (hd == 128) LD_SUM(bf16_t, 128); else LD_SUM(bf16_t, 64); }
    else { if (hd == 128) LD_SUM(float, 128); else LD_SUM(float, 64); }
#undef LD_SUM
    return launched("k_kv_summary");
}

size_t ldk_sparse_attention_scratch_bytes(int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t max_ctx, int32_t window, int32_t budget) {
    if (T <= 0 || H <= 0 || Hkv <= 0 || H % Hkv || (hd != 64 && hd != 128) || max_ctx <= 0 || window < 0 || budget <= 0) return 0;
    return scratch_bound(T, H, Hkv, hd, max_ctx, window, budget);
}

ld_status ldk_sparse_attention(const float *q, int32_t q_stride, const void *pool_layer, int32_t dtype, const int8_t *bounds, const float *unit,
                               const int32_t *table, int32_t table_stride, const int32_t *seq_slot, const int32_t *ctx_len, int32_t max_ctx,
                               int32_t T, int32_t H, int32_t Hkv, int32_t hd, int32_t window, int32_t budget, int32_t keep_first,
                               int32_t keep_last, float *out, int32_t *sel, void *scratch, size_t scratch_bytes, void *stream) {
    if (T == 0) return LD_OK;
    if (!q || !pool_layer || !bounds || !unit || !table || !seq_slot || !ctx_len || !out || !sel || !scratch || T < 0 || H <= 0 || Hkv <= 0 ||
        H % Hkv || (hd != 64 && hd != 128) || max_ctx <= 0 || window < 0 || (dtype != LD_BF16 && dtype != LD_F32) ||
        (((uintptr_t)pool_layer | (uintptr_t)bounds | (uintptr_t)scratch) & 15))
        return ld::fail(LD_E_INVAL, "ldk_sparse_attention: bad argument");
    if (keep_first < 0 || keep_last < 1 || budget < 1 || (int64_t)keep_first + keep_last > budget)
        return ld::fail(LD_E_INVAL, "ldk_sparse_attention: the last block is always kept (keep_last >= 1), and the kept blocks must fit the budget");
    if (T > 65535 || Hkv > 65535) return ld::fail(LD_E_RANGE, "ldk_sparse_attention: more than 65535 rows or KV heads");
    if (scratch_bytes < ldk_sparse_attention_scratch_bytes(T, H, Hkv, hd, max_ctx, window, budget))
        return ld::fail(LD_E_INVAL, "ldk_sparse_attention: scratch too small");
    hipStream_t s = (hipStream_t)stream;
    const SparseArgs a{q, q_stride, pool_layer, bounds, unit, table, table_stride, seq_slot, ctx_len, max_ctx, T, H, Hkv, window, budget, keep_first,
                       keep_last, out, sel, (char *)scratch};
    if (dtype == LD_BF16) { if (hd == 128) launch_sparse<bf16_t, 128>(a, s); else launch_sparse<bf16_t, 64>(a, s); }
    else { if (hd == 128) launch_sparse<float, 128>(a, s); else launch_sparse<float, 64>(a, s); }
    return launched("k_sparse_attend");
}

}  // extern "C"
