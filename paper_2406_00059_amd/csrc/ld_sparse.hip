// Decode attention over the cache blocks that a cheap score selects for each query, and the bounds it scores with.
//
// A block of 16 positions is described, per KV head, by the largest and the smallest value of its keys in every
// dimension, as 8-bit integers of a power of two: with q rounded to 8-bit integers the same way,
//   score = sum_i (q_i >= 0 ? q_i hi_i : q_i lo_i)
// is the most that q.k can be over the block's positions, up to the rounding of q and to a magnitude between 127 and 128 units, which counts as 127.
// Integer sums and powers of two, rounded once: a score has one value, however the work is cut, and so has the choice.  A block and head cost 2 hd + 4
// bytes to score against 64 hd to attend to (bf16).
#include "ld_device.h"

#include <algorithm>
#include <cmath>

using namespace ldd;

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int32_t i32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
constexpr uint32_t INF_BITS = 0x7f800000u;

// e of the unit 2^e in which a largest magnitude (as bits, finite) counts 64 .. 127: floor(log2 max) - 6, not below -126.
__device__ __forceinline__ int unit_exponent(uint32_t top) { return top ? max(ilogbf(__uint_as_float(top)) - 6, -126) : 0; }

// Lane exchanges without LDS.  Rotation within a row of 16 lanes; maximum and sum over a row, in all of its lanes.
template <int N, typename T> __device__ __forceinline__ T row_rotate(T v) {
    return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + N, 0xf, 0xf, false));
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
// Minimum, maximum over a wave (uniform).
template <typename F> __device__ __forceinline__ uint32_t wave_reduce(uint32_t v, F f) {
    v = f(v, row_rotate<8>(v));
    v = f(v, row_rotate<4>(v));
    v = f(v, row_rotate<2>(v));
    v = f(v, row_rotate<1>(v));
    auto lane = [&](int l) { return (uint32_t)__builtin_amdgcn_readlane((int)v, l); };
    return f(f(lane(0), lane(16)), f(lane(32), lane(48)));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) { return wave_reduce(v, [](uint32_t a, uint32_t b) { return max(a, b); }); }
__device__ __forceinline__ uint32_t wave_min(uint32_t v) { return wave_reduce(v, [](uint32_t a, uint32_t b) { return min(a, b); }); }
// f over the four rows' lanes of one column, in all of them (exchanges of whole rows).
template <typename F> __device__ __forceinline__ float across_rows(float v, F f) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Inclusive prefix sum over a wave: shifts within the rows, then the rows' last lanes to the rows behind them.
__device__ __forceinline__ uint32_t wave_prefix(uint32_t v) {
#define LD_SHIFTED(ctrl, rows) (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false)
    v += LD_SHIFTED(0x111, 0xf);
    v += LD_SHIFTED(0x112, 0xf);
    v += LD_SHIFTED(0x114, 0xf);
    v += LD_SHIFTED(0x118, 0xf);
    v += LD_SHIFTED(0x142, 0xa);
    v += LD_SHIFTED(0x143, 0xc);
#undef LD_SHIFTED
    return v;
}

// ---------------------------------------------------------------- bounds of a block's keys

// One wave a (block, KV head): the 16 key rows, 8 elements a lane and load; rows meet by lane exchanges.  Bound by the keys' bytes: 16383
// positions of 40 heads of 128 (168 MB) 38 us, 4.7 TB/s, with all of a block's loads in flight (48 us two at a time).
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
    float v[PASSES][8];
#pragma unroll
    for (int p = 0; p < PASSES; p++)      // all in flight; past the last position its key again
        load8_stream(keys + (int64_t)min(p * ROWS + lane / LPR, real - 1) * HD + d, v[p]);
#pragma unroll
    for (int p = 0; p < PASSES; p++)
#pragma unroll
        for (int e = 0; e < 8; e++) {
            lo[e] = fminf(lo[e], v[p][e]);
            hi[e] = fmaxf(hi[e], v[p][e]);
            top = max(top, abs_bits(v[p][e]));      // compared as bits: a NaN stays
        }
    top = wave_max(top);
#pragma unroll
    for (int e = 0; e < 8; e++) {      // over the lanes of the same dimensions
        if (LPR == 8) {
            lo[e] = fminf(lo[e], row_rotate<8>(lo[e]));
            hi[e] = fmaxf(hi[e], row_rotate<8>(hi[e]));
        }
        lo[e] = across_rows(lo[e], [](float a, float b) { return fminf(a, b); });
        hi[e] = across_rows(hi[e], [](float a, float b) { return fmaxf(a, b); });
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

// Up to 16 query heads of a KV head as operand columns of the integer matrix instructions: [head][positive parts, negative parts][hd]
// bytes, and the units' exponents.  The positive parts meet the upper bounds, the negative ones the lower.
template <int HD>
struct ScoreQueries {
    int8_t c[16][2 * HD + 16];      // rows 16 bytes apart from a multiple of the banks
    int unit[16];
};
// A wave a head (q: the first head's); a barrier has to follow.
template <int HD>
__device__ __forceinline__ void quantise_queries(const float *__restrict__ q, int heads, ScoreQueries<HD> &sq, int waves) {
    const int lane = threadIdx.x & 63;
    for (int g = threadIdx.x >> 6; g < heads; g += waves) {
        float f[HD / 64];
        uint32_t top = 0;
#pragma unroll
        for (int u = 0; u < HD / 64; u++) {
            f[u] = q[g * HD + lane + 64 * u];
            top = max(top, abs_bits(f[u]));
        }
        top = wave_max(top);
        const bool ok = top < INF_BITS;
        const int e = ok ? unit_exponent(top) : 0;
#pragma unroll
        for (int u = 0; u < HD / 64; u++) {
            const int c = ok ? (int)fminf(fmaxf(rintf(ldexpf(f[u], -e)), -127.f), 127.f) : 0;
            sq.c[g][lane + 64 * u] = (int8_t)max(c, 0);
            sq.c[g][HD + lane + 64 * u] = (int8_t)min(c, 0);
        }
        if (lane == 0) sq.unit[g] = e;
    }
}
// A wave's operands: lane l holds head l % 16, bytes 64 j + 16 (l / 16) .. + 16.
template <int HD>
struct ScoreOperand {
    i32x4 b[HD / 32];
    int unit;
    bool real;
    __device__ __forceinline__ ScoreOperand(const ScoreQueries<HD> &sq, int heads, int lane) {
        const int g = min(lane & 15, heads - 1);
        real = (lane & 15) < heads;
        unit = sq.unit[g];
#pragma unroll
        for (int j = 0; j < HD / 32; j++) b[j] = *reinterpret_cast<const i32x4 *>(&sq.c[g][64 * j + 16 * (lane >> 4)]);
    }
};

// Scores of the 16 blocks whose physical ids lanes l % 16 hold: lane l < 64 returns that of block 4 (l / 16) + l % 4.
template <int HD>
__device__ __forceinline__ float score_tile(const ScoreOperand<HD> &q, const int8_t *__restrict__ bounds, const float *__restrict__ unit, int64_t phys,
                                            int Hkv, int kvh, int lane) {
    const int h = lane >> 4;
    const int8_t *rec = bounds + (phys * Hkv + kvh) * 2 * HD + 16 * h;
    i32x4 a[HD / 32];
#pragma unroll
    for (int j = 0; j < HD / 32; j++) a[j] = *reinterpret_cast<const i32x4 *>(rec + 64 * j);
    const int un = (int)(__float_as_uint(unit[phys * Hkv + kvh]) >> 23) - 127;      // exponent of a power of two; 128: infinity
    i32x4 acc = (i32x4){0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < HD / 32; j++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], q.b[j], acc, 0, 0, 0);
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int u = __shfl(un, 4 * h + i, WAVE);
        // one scaling by both exponents: after the query's alone a score may lie outside the range that it ends in
        s[i] = row_max(q.real ? (u < 128 ? ldexpf((float)acc[i], q.unit + u) : INFINITY) : -INFINITY);
    }
    const int i = lane & 3;
    return i == 0 ? s[0] : i == 1 ? s[1] : i == 2 ? s[2] : s[3];
}

// A wave tiles_per_wave tiles of 16 blocks of a (row, KV head).  Also clears the tickets of the launch behind it.  8192 blocks of 8 KV heads
// (17 MB of bounds): 5.9 us.
template <int HD>
__global__ __launch_bounds__(256) void k_sparse_score(const float *__restrict__ q, int q_stride, const int8_t *__restrict__ bounds,
                                                      const float *__restrict__ unit, const int32_t *__restrict__ table, int table_stride,
                                                      const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len, int max_ctx,
                                                      int Hkv, int G, int window, int tiles_per_wave, int stride, float *__restrict__ scores,
                                                      int32_t *__restrict__ tickets) {
    if (threadIdx.x == 0 && blockIdx.x == 0) tickets[(int64_t)blockIdx.z * Hkv + blockIdx.y] = 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.z, kvh = blockIdx.y;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    const int tile0 = (blockIdx.x * 4 + wave) * tiles_per_wave;
    if (blockIdx.x * 4 * tiles_per_wave * 16 >= v.n) return;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride + v.b0;
    float *dst = scores + ((int64_t)t * Hkv + kvh) * stride;
    __shared__ __attribute__((aligned(16))) ScoreQueries<HD> qq;
    for (int g0 = 0; g0 < G; g0 += 16) {
        const int heads = min(16, G - g0);
        quantise_queries<HD>(q + (int64_t)t * q_stride + ((int64_t)kvh * G + g0) * HD, heads, qq, 4);
        __syncthreads();
        const ScoreOperand<HD> sq(qq, heads, lane);
        if (g0 + 16 < G) __syncthreads();
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

// The largest key among lo .. hi that at least `need` of a wave's keys reach, by halves with counts from the ballots, and how many of the
// keys equal to it belong to the choice.
template <int N>
__device__ __forceinline__ void search_keys(const uint32_t (&key)[N], uint32_t lo, uint32_t hi, int need, uint32_t &from, int &equal) {
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int c = 0;
#pragma unroll
        for (int j = 0; j < N; j++) c += __popcll(__ballot(key[j] >= mid));
        if (c == need) { from = mid; equal = 1 << 30; return; }      // all that reach it
        if (c > need) lo = mid;
        else hi = mid - 1;
    }
    from = lo;
    int c = 0;
#pragma unroll
    for (int j = 0; j < N; j++) c += __popcll(__ballot(key[j] > lo));
    equal = need - c;
}

// Keys of the choice: kept blocks lie above every score (the largest, +infinity's, is 0xff800000), what is no block below.
constexpr uint32_t KEPT = 0xffffffffu;

// The choice among the n > budget visible blocks of a (row, KV head): writes the `budget` chosen ones, ascending, to out.
// One wave, n <= 64 KPL; lane l holds the blocks j 64 + l.
template <int KPL>
__device__ __forceinline__ void select_by_wave(const float *sc, int n, int budget, int keep_first, int keep_last, int32_t *out) {
    const int lane = threadIdx.x & 63;
    const int c1 = n - keep_last;
    uint32_t key[KPL], lo = KEPT, hi = 0;
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const int i = j * 64 + lane;
        key[j] = i < n ? KEPT : 0;
        if (i >= keep_first && i < c1) {
            key[j] = order_key(sc[i]);
            lo = min(lo, key[j]);
            hi = max(hi, key[j]);
        }
    }
    uint32_t from = KEPT;
    int equal = 1 << 30;
    if (budget > keep_first + keep_last) search_keys<KPL>(key, wave_min(lo), wave_max(hi), budget, from, equal);
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int at = 0, met = 0;      // written so far, equal keys met so far
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const uint64_t bt = __ballot(key[j] == from);
        const bool take = key[j] > from || (key[j] == from && met + __popcll(bt & below) < equal);
        const uint64_t bk = __ballot(take);
        const int slot = at + __popcll(bk & below);
        if (take && slot < budget) out[slot] = j * 64 + lane;
        met += __popcll(bt);
        at += __popcll(bk);
    }
}

// The same by a workgroup of WAVES waves, n <= 64 WAVES KPL; thread i holds the blocks i KPL .. + KPL.  The keys' range is cut into 64 WAVES
// bins, counted in LDS (a bell of scores spreads well over them, its exponent bits alone would not); the bin that the
// threshold falls into holds a few dozen keys, among which every wave searches on its own.  Bins that hold more than 64 keys are cut
// again.  All waves call it; sc may be read up to a multiple of KPL past n; b0 is added to what is written.
template <int WAVES>
struct SelectRoom {
    uint32_t bin[64 * WAVES], wave[2 * WAVES], list[64];
    uint32_t at_bin, above, count;
};
template <int WAVES, int KPL>
__device__ __forceinline__ void select_by_group(const float *sc, int n, int b0, int budget, int keep_first, int keep_last, int32_t *out,
                                                SelectRoom<WAVES> &sm) {
    constexpr int TH = 64 * WAVES;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c1 = n - keep_last, i0 = tid * KPL;
    int need = budget - keep_first - keep_last;
    uint32_t key[KPL], lo = KEPT, hi = 0;
    float raw[KPL];
    if (i0 < n) {
#pragma unroll
        for (int j = 0; j < KPL; j += 4) *reinterpret_cast<float4 *>(raw + j) = *reinterpret_cast<const float4 *>(sc + i0 + j);
    }
    sm.bin[tid] = 0;
    if (tid == 0) sm.count = 0;
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const int i = i0 + j;
        key[j] = i < n ? KEPT : 0;
        if (i >= keep_first && i < c1) {
            key[j] = order_key(raw[j]);
            lo = min(lo, key[j]);
            hi = max(hi, key[j]);
        }
    }
    lo = wave_min(lo);
    hi = wave_max(hi);
    if (lane == 0) { sm.wave[wave] = lo; sm.wave[WAVES + wave] = hi; }
    __syncthreads();
    {
        const uint32_t l = sm.wave[lane % WAVES], h = sm.wave[WAVES + lane % WAVES];
        lo = wave_min(l);
        hi = wave_max(h);
    }
    uint32_t from = KEPT;
    int equal = 1 << 30;
    for (bool first = true; need > 0; first = false) {      // keys in lo .. hi are in question, `need` of them are wanted (all larger ones are)
        if (lo == hi) { from = lo; equal = need; break; }
        const int shift = max(0, 32 - __builtin_clz(hi - lo) - (31 - __builtin_clz(TH)));      // (hi - lo) >> shift < TH
        if (!first) {
            __syncthreads();
            sm.bin[tid] = 0;
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < KPL; j++)
            if (key[j] >= lo && key[j] <= hi) atomicAdd(&sm.bin[(key[j] - lo) >> shift], 1u);
        __syncthreads();
        // thread i: bin TH - 1 - i, so that the prefix counts from the top
        const uint32_t mine = sm.bin[TH - 1 - tid], inc = wave_prefix(mine);
        if (lane == 63) sm.wave[wave] = inc;
        __syncthreads();
        uint32_t upto = inc;
#pragma unroll
        for (int w = 0; w < WAVES; w++) upto += w < wave ? sm.wave[w] : 0;
        if (upto >= (uint32_t)need && upto - mine < (uint32_t)need) { sm.at_bin = TH - 1 - tid; sm.above = upto - mine; }
        __syncthreads();
        const uint32_t bin = sm.at_bin, in_bin = sm.bin[bin];
        need -= (int)sm.above;
        hi = (uint32_t)min((uint64_t)hi, (uint64_t)lo + ((uint64_t)(bin + 1) << shift) - 1);
        lo = lo + (bin << shift);
        if ((int)in_bin == need) { from = lo; break; }      // the whole bin
        if (in_bin <= 64) {
#pragma unroll
            for (int j = 0; j < KPL; j++)
                if (key[j] >= lo && key[j] <= hi) sm.list[atomicAdd(&sm.count, 1u)] = key[j];      // their order does not matter
            __syncthreads();
            const uint32_t one[1] = {lane < (int)in_bin ? sm.list[lane] : 0};
            search_keys<1>(one, lo, hi, need, from, equal);
            break;
        }
    }
    // how many of a thread's blocks are taken for certain (low half) and how many tie; the same before the thread
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < KPL; j++) mine += key[j] > from ? 1u : key[j] == from ? 1u << 16 : 0u;
    const uint32_t inc = wave_prefix(mine);
    __syncthreads();
    if (lane == 63) sm.wave[wave] = inc;
    __syncthreads();
    uint32_t before = inc - mine;
#pragma unroll
    for (int w = 0; w < WAVES; w++) before += w < wave ? sm.wave[w] : 0;
    if (mine == 0) return;
    int met = (int)(before >> 16), slot = (int)(before & 0xffff) + min(met, equal);
#pragma unroll
    for (int j = 0; j < KPL; j++) {
        const bool take = key[j] > from || (key[j] == from && met < equal);
        met += key[j] == from;
        if (take && slot < budget) out[slot] = b0 + i0 + j;
        slot += take;
    }
}

// The choice as a launch of its own, for more blocks than fit in registers: every step of the search reads the scores again.
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

// A wave adds the blocks of the selection two at a time to what it has of some query heads (maximum in the log2 domain, sum, output).
// Two ways of it, with the same shape: load (a pair of blocks), add (the pair), put (the wave's share into LDS: o [wave][HEADS][HD], ml
// [max, sum][wave][HEADS]).  Queries come from LDS, where stage has left them scaled by log2(e) / sqrt(hd).

// bf16: on the matrix cores, four query heads an operand.  Operands of 16 significant bits would cost what float32 keeps, so queries and
// probabilities are split into three bf16 terms (24 bits); column c of an operand is term c / 4 of head c % 4 (columns 12 .. 15 zero), so that
// the three terms cost no more instructions than one, and a block of 8 KB takes 8 + 8 instructions of 16 cycles where converting and
// multiplying on the vector units takes some 200 of 4.
//   S[pos, c]  = K[pos, :] . Q[c, :]    tile 0, row 4 h + i: position 8 (h % 2) + i of block h / 2, tile 1: position 8 (h % 2) + 4 + i
//   O[d, c]   += V^T[d, pos] P^T[pos, c]   so that lane group h = l / 16 holds the eight positions that its operand of V, 16 bytes of one
//                                          dimension of block h / 2, contracts with
template <int HD, int NS>
struct OnMatrixCores {
    typedef bf16_t KT;
    static constexpr int HEADS = 4 * NS;
    static constexpr bool TERMS = true;
    static constexpr int WORKGROUPS = NS == 2 ? 2 : HD == 64 ? 5 : 3;      // of k_sparse_row a CU, by registers
    struct Pair { u32x4 k[2][HD / 32], v[HD / 16]; };
    typedef uint16_t Queries[HEADS][3][HD];      // in LDS: the three terms
    bf16x8 q[NS][HD / 32];
    float m[NS], l[NS];
    f32x4 o[NS][HD / 16];

    static __device__ __forceinline__ uint32_t term2(float a, float b, int term) {      // term 0 .. 2 of two floats as packed bf16, 0 for 3
        uint32_t x = pack2_bf16(a, b);
        const float ra = a - __uint_as_float(x << 16), rb = b - __uint_as_float(x & 0xffff0000u);
        const uint32_t y = pack2_bf16(ra, rb);
        const uint32_t z = pack2_bf16(ra - __uint_as_float(y << 16), rb - __uint_as_float(y & 0xffff0000u));
        return term == 0 ? x : term == 1 ? y : term == 2 ? z : 0u;
    }
    static __device__ __forceinline__ void stage(const float *__restrict__ src, int heads, Queries &qs) {
        const float scale = 1.4426950408889634f / sqrtf((float)HD);
        for (int i = threadIdx.x; i < heads * HD; i += blockDim.x) {
            const float x = src[i] * scale;
#pragma unroll
            for (int t = 0; t < 3; t++) qs[i / HD][t][i % HD] = (uint16_t)term2(x, 0.f, t);
        }
    }
    __device__ __forceinline__ void start(const Queries &qs, int heads, int lane) {
        const int g = lane & 3, term = (lane & 15) >> 2, h = lane >> 4;
#pragma unroll
        for (int n = 0; n < NS; n++) {
            const bool real = 4 * n + g < heads && term < 3;
#pragma unroll
            for (int j = 0; j < HD / 32; j++) {
                u32x4 w = (u32x4){0, 0, 0, 0};
                if (real) w = *reinterpret_cast<const u32x4 *>(&qs[4 * n + g][term][32 * j + 8 * h]);
                q[n][j] = __builtin_bit_cast(bf16x8, w);
            }
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int t = 0; t < HD / 16; t++) o[n][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
        }
    }
    static __device__ __forceinline__ void load(Pair &d, const KT *b0, const KT *b1, int Hkv, int kvh, int lane) {
        const int r = lane & 15, h = lane >> 4;
        const KT *kp = ((r >> 3) ? b1 : b0) + kv_k_offset(HD, kvh, 8 * ((r >> 2) & 1) + (r & 3), 8 * h);
        const KT *vp = ((h >> 1) ? b1 : b0) + kv_v_offset(Hkv, HD, kvh, 8 * (h & 1), r);
#pragma unroll
        for (int t = 0; t < 2; t++)
#pragma unroll
            for (int j = 0; j < HD / 32; j++) d.k[t][j] = load_stream16(kp + 4 * t * HD + 32 * j);
#pragma unroll
        for (int t = 0; t < HD / 16; t++) d.v[t] = load_stream16(vp + t * 16 * 16);
    }
    // pos0, pos1: first positions of the two blocks (pos1 -16: there is no second one, its positions lie before every row's first)
    __device__ __forceinline__ void add(Pair &d, int pos0, int pos1, int start, int ctx, float *, int lane) {
        const int h = lane >> 4, term = (lane & 15) >> 2;
        const int first = ((h >> 1) ? pos1 : pos0) + 8 * (h & 1);      // of the lane's eight positions
        bool ok[8];
#pragma unroll
        for (int e = 0; e < 8; e++) ok[e] = first + e >= start && first + e < ctx;
        const bool full = pos0 >= start && pos1 >= start && pos0 + 16 <= ctx && pos1 + 16 <= ctx;
        if (!full) {      // what an unwritten slot holds, NaN among it, is not looked at
#pragma unroll
            for (int t = 0; t < HD / 16; t++)
#pragma unroll
                for (int w = 0; w < 4; w++) d.v[t][w] &= (ok[2 * w] ? 0x0000ffffu : 0u) | (ok[2 * w + 1] ? 0xffff0000u : 0u);
        }
#pragma unroll
        for (int n = 0; n < NS; n++) {
            float s[8];
#pragma unroll
            for (int t = 0; t < 2; t++) {
                f32x4 a = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < HD / 32; j++) a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, d.k[t][j]), q[n][j], a, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    float x = a[i] + row_rotate<8>(a[i]);      // the terms' columns: all of them get the head's score
                    x += row_rotate<4>(x);
                    s[4 * t + i] = full || ok[4 * t + i] ? x : -INFINITY;
                }
            }
            float mb = s[0];
#pragma unroll
            for (int e = 1; e < 8; e++) mb = fmaxf(mb, s[e]);
            const float m_new = fmaxf(m[n], across_rows(mb, [](float a, float b) { return fmaxf(a, b); }));      // a selected block holds a visible position
            const float corr = fast_exp2(m[n] - m_new);
            m[n] = m_new;
            float p[8], sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) {
                p[e] = full || ok[e] ? fast_exp2(s[e] - m_new) : 0.f;
                sum += p[e];
            }
            l[n] = l[n] * corr + sum;
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; e++) w[e] = term2(p[2 * e], p[2 * e + 1], term);
            const bf16x8 pb = __builtin_bit_cast(bf16x8, w);
            const bool moved = __any(corr != 1.f);
#pragma unroll
            for (int t = 0; t < HD / 16; t++) {
                if (moved) {
#pragma unroll
                    for (int i = 0; i < 4; i++) o[n][t][i] *= corr;
                }
                o[n][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, d.v[t]), pb, o[n][t], 0, 0, 0);
            }
        }
    }
    // Whether the wave's sums are numbers.  An infinite key or value times the terms of unlike sign, or the zero columns, is NaN, where the product
    // itself may be -infinity (no weight) or infinite: attend_plainly then.  (A sum of everything times 0, 0 or NaN: an instruction a value.)
    __device__ __forceinline__ bool finite() const {
        float z = 0.f;
#pragma unroll
        for (int n = 0; n < NS; n++) {
            z = fmaf(l[n], 0.f, z);
#pragma unroll
            for (int t = 0; t < HD / 16; t++)
#pragma unroll
                for (int i = 0; i < 4; i++) z = fmaf(o[n][t][i], 0.f, z);
        }
        return !__any(z != 0.f);
    }
    static __device__ __forceinline__ float query(const Queries &qs, int g, int d) {      // the three terms are the float
        return bf16_to_f32(qs[g][0][d]) + bf16_to_f32(qs[g][1][d]) + bf16_to_f32(qs[g][2][d]);
    }
    __device__ __forceinline__ void put(float *so, float *ml, int waves, int wave, int lane) const {
        const int g = lane & 15, h = lane >> 4;
#pragma unroll
        for (int n = 0; n < NS; n++) {
            const float sum = across_rows(l[n], [](float a, float b) { return a + b; });
#pragma unroll
            for (int t = 0; t < HD / 16; t++) {
                f32x4 v;
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float x = o[n][t][i] + row_rotate<8>(o[n][t][i]);
                    v[i] = x + row_rotate<4>(x);
                }
                if (g < 4) *reinterpret_cast<f32x4 *>(so + (wave * HEADS + 4 * n + g) * HD + 16 * t + 4 * h) = v;
            }
            if (lane < 4) {
                ml[wave * HEADS + 4 * n + lane] = m[n];
                ml[(waves + wave) * HEADS + 4 * n + lane] = sum;
            }
        }
    }
};

// float32 pools (small models): one head on the vector units.  Keys: lane = position l % 16, dimensions 32 j + 8 (l / 16) .. + 8; values
// (transposed in a block): lane = dimension l / 2 + 32 u, positions 8 (l % 2) .. + 8.
template <int HD>
struct OnVectorUnits {
    typedef float KT;
    static constexpr int HEADS = 1;
    static constexpr bool TERMS = false;
    static constexpr int WORKGROUPS = 3;
    struct Block { float k[HD / 32][8], v[HD / 32][8]; };
    struct Pair { Block b[2]; };
    typedef float Queries[HD];
    const float *qs;
    float m, l, o[HD / 32];

    static __device__ __forceinline__ void stage(const float *__restrict__ src, int, Queries &queries) {
        const float scale = 1.4426950408889634f / sqrtf((float)HD);
        for (int i = threadIdx.x; i < HD; i += blockDim.x) queries[i] = src[i] * scale;
    }
    __device__ __forceinline__ void start(const Queries &queries, int, int) {
        qs = queries;
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int u = 0; u < HD / 32; u++) o[u] = 0.f;
    }
    static __device__ __forceinline__ void load(Pair &d, const KT *b0, const KT *b1, int Hkv, int kvh, int lane) {
#pragma unroll
        for (int n = 0; n < 2; n++) {
            const KT *kp = (n ? b1 : b0) + kv_k_offset(HD, kvh, lane & 15, 8 * (lane >> 4));
            const KT *vp = (n ? b1 : b0) + kv_v_offset(Hkv, HD, kvh, 8 * (lane & 1), lane >> 1);
#pragma unroll
            for (int j = 0; j < HD / 32; j++) { load8_stream(kp + 32 * j, d.b[n].k[j]); load8_stream(vp + j * 32 * 16, d.b[n].v[j]); }
        }
    }
    __device__ __forceinline__ void add_block(const Block &d, int pos0, int start, int ctx, float *pl, int lane) {
        const int pos = pos0 + (lane & 15);
        const bool ok = pos >= start && pos < ctx;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < HD / 32; j++)
#pragma unroll
            for (int e = 0; e < 8; e++) s += qs[32 * j + 8 * (lane >> 4) + e] * d.k[j][e];
        s = across_rows(s, [](float a, float b) { return a + b; });
        if (!ok) s = -INFINITY;
        const float m_new = fmaxf(m, row_max(s)), at = m_new > -INFINITY ? m_new : 0.f;      // -inf: keys of -infinity so far, which have no weight
        const float corr = fast_exp2(m - at), p = ok ? fast_exp2(s - at) : 0.f;
        m = m_new;
        l = l * corr + p;
        if (lane < 16) pl[lane] = p;
        __builtin_amdgcn_wave_barrier();      // a wave's LDS operations execute in order
        float pv[8];
#pragma unroll
        for (int e = 0; e < 8; e++) pv[e] = pl[8 * (lane & 1) + e];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < HD / 32; u++) {
            o[u] *= corr;
#pragma unroll
            for (int e = 0; e < 8; e++) {      // what an unwritten slot holds is not looked at
                const int ps = pos0 + 8 * (lane & 1) + e;
                if (ps >= start && ps < ctx) o[u] += pv[e] * d.v[u][e];
            }
        }
    }
    __device__ __forceinline__ void add(Pair &d, int pos0, int pos1, int start, int ctx, float *pl, int lane) {
        add_block(d.b[0], pos0, start, ctx, pl, lane);
        if (pos1 >= 0) add_block(d.b[1], pos1, start, ctx, pl, lane);
    }
    __device__ __forceinline__ void put(float *so, float *ml, int waves, int wave, int lane) const {
        const float sum = row_sum(l);
#pragma unroll
        for (int u = 0; u < HD / 32; u++) {
            const float a = o[u] + __shfl_xor(o[u], 1, WAVE);
            if (!(lane & 1)) so[wave * HD + (lane >> 1) + 32 * u] = a;
        }
        if (lane == 0) { ml[wave] = m; ml[waves + wave] = sum; }
    }
};

// A wave's share again, product by product in float32, for what the terms cannot express (see finite): lane l has position l % 16 of a block and the
// l / 16-th quarter of the dimensions for the scores, the dimensions l + 64 u for the values.  block(i, b, p): logical and physical block i < n.
template <typename A, int HD, int W, typename Block>
__device__ __forceinline__ void attend_plainly(const typename A::Queries &qs, int heads, const typename A::KT *__restrict__ pool, int64_t bs, int Hkv, int kvh,
                                               int n, Block block, int start, int ctx, float *so, float *ml) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));      // nothing of this rare path is computed ahead and kept in registers
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll 1
    for (int g = 0; g < heads; g++) {
        float m = -INFINITY, l = 0.f, o[HD / 64];
        for (int u = 0; u < HD / 64; u++) o[u] = 0.f;
#pragma unroll 1
        for (int i = 2 * wave; i < n; i = (i & 1) ? i + 2 * W - 1 : i + 1) {
            int b;
            int64_t p;
            block(i, b, p);
            const typename A::KT *blk = pool + p * bs;
            const int pos = b * 16 + (lane & 15);
            const bool ok = pos >= start && pos < ctx;
            float s = 0.f;
#pragma unroll 1
            for (int d = (lane >> 4) * (HD / 4); d < ((lane >> 4) + 1) * (HD / 4); d += 8) {
                float v[8];
                load8(blk + kv_k_offset(HD, kvh, lane & 15, d), v);
                for (int e = 0; e < 8; e++) s += A::query(qs, g, d + e) * v[e];
            }
            s = across_rows(s, [](float a, float c) { return a + c; });
            if (!ok) s = -INFINITY;
            const float m_new = fmaxf(m, row_max(s)), at = m_new > -INFINITY ? m_new : 0.f;
            const float corr = fast_exp2(m - at), w = ok ? fast_exp2(s - at) : 0.f;
            m = m_new;
            l = l * corr + w;
            for (int u = 0; u < HD / 64; u++) {
                o[u] *= corr;
                const typename A::KT *vp = blk + kv_v_offset(Hkv, HD, kvh, 0, lane + 64 * u);
#pragma unroll 1
                for (int e = 0; e < 16; e++) {
                    const float we = __shfl(w, e, WAVE);
                    if (b * 16 + e >= start && b * 16 + e < ctx) o[u] += we * bf16_to_f32(vp[e]);
                }
            }
        }
        l = row_sum(l);
        for (int u = 0; u < HD / 64; u++) so[(wave * A::HEADS + g) * HD + lane + 64 * u] = o[u];
        if (lane == 0) {
            ml[wave * A::HEADS + g] = m;
            ml[(W + wave) * A::HEADS + g] = l;
        }
    }
}

template <typename A, int HD, int W, typename Block>
__device__ __forceinline__ void put_wave(const A &a, const typename A::Queries &qs, int heads, const typename A::KT *__restrict__ pool, int64_t bs, int Hkv,
                                         int kvh, int n, Block block, int start, int ctx, float *so, float *ml, int wave, int lane) {
    if constexpr (A::TERMS)
        if (__builtin_expect(!a.finite(), 0)) return attend_plainly<A, HD, W>(qs, heads, pool, bs, Hkv, kvh, n, block, start, ctx, so, ml);
    a.put(so, ml, W, wave, lane);
}

// Output (d of head g) of a workgroup's waves, their sum and their common maximum.
template <int HD, int HEADS, int W>
__device__ __forceinline__ float join_waves(const float *so, const float *ml, int g, int d, float &M, float &L) {
    M = ml[g];
#pragma unroll
    for (int w = 1; w < W; w++) M = fmaxf(M, ml[w * HEADS + g]);      // a wave that had no block: -inf, and its weight 0
    const float at = M > -INFINITY ? M : 0.f;
    float o = 0.f;
    L = 0.f;
#pragma unroll
    for (int w = 0; w < W; w++) {
        const float a = fast_exp2(ml[w * HEADS + g] - at);
        o += a * so[(w * HEADS + g) * HD + d];
        L += a * ml[(W + w) * HEADS + g];
    }
    return o;
}

// Floats that workgroups on other XCDs read in the same launch: stored and loaded at agent scope, past the caches that are not shared, so
// that a writer has only to wait until its stores have arrived before it draws a ticket.  (Fences for ordinary stores write a whole
// L2 back, once a wave: 47 us where the launch takes 8.)
__device__ __forceinline__ void store_shared(float *p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float load_shared(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Second launch of the split form: gridDim.x workgroups a (row, KV head).  Each makes the choice by itself (it is the same in all of them,
// and cheaper than a launch between), attends to its chunk of cb blocks and leaves its share; the one that draws the last ticket
// joins the shares in their order.  chosen: the choice is in sel already (k_sparse_select_long).
// 256 of 8192 blocks of 8 KV heads: 18 us, some 5 of them the choice and 4 the 17 MB of keys and values (the rest not measured apart); both launches 24.
constexpr int SPLIT_WAVES = 8, SPLIT_BLOCKS = 16384, SPLIT_BUDGET = 4096;
template <typename A, int HD>
__global__ __launch_bounds__(64 * SPLIT_WAVES) void k_sparse_attend(const float *__restrict__ q, int q_stride, const typename A::KT *__restrict__ pool,
                                                                    int Hkv, const int32_t *__restrict__ table, int table_stride,
                                                                    const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len,
                                                                    int max_ctx, int G, int window, int budget, int keep_first, int keep_last,
                                                                    const float *__restrict__ scores, int stride, bool chosen, int cb,
                                                                    float *__restrict__ part_o, float *__restrict__ part_ml,
                                                                    int32_t *__restrict__ tickets, float *__restrict__ out, int32_t *__restrict__ sel) {
    constexpr int W = SPLIT_WAVES, TH = 64 * W;
    __shared__ int32_t list[SPLIT_BUDGET];
    __shared__ SelectRoom<W> sm;
    __shared__ __attribute__((aligned(16))) typename A::Queries qs;
    __shared__ __attribute__((aligned(16))) float pl[W][16], so[W * A::HEADS * HD], ml[2 * W * A::HEADS];
    __shared__ int last;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x, kvh = blockIdx.y, t = blockIdx.z, chunks = gridDim.x;
    const int ctx = min(ctx_len[t], max_ctx);
    const Visible v = visible(ctx, window);
    const int n = min(v.n, budget), real = (n + cb - 1) / cb;      // chunks with blocks in them
    int32_t *gsel = sel + ((int64_t)t * Hkv + kvh) * budget;
    const int64_t H = (int64_t)Hkv * G, bs = kv_block_elems(Hkv, HD);
    if (c >= real) {
        if (real == 0 && c == 0) {      // the row sees nothing
            for (int i = threadIdx.x; i < G * HD; i += TH) out[((int64_t)t * H + kvh * G) * HD + i] = 0.f;
            for (int i = threadIdx.x; i < budget; i += TH) gsel[i] = -1;
        }
        return;
    }
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride + v.b0;
    const float *sc = scores + ((int64_t)t * Hkv + kvh) * stride;
    const int i0 = c * cb, i1 = min(i0 + cb, n);
    A::stage(q + (int64_t)t * q_stride + (int64_t)kvh * G * HD, min(A::HEADS, G), qs);
    if (chosen) {
        for (int i = i0 + threadIdx.x; i < i1; i += TH) list[i - i0] = gsel[i] - v.b0;
    } else {
        if (v.n <= budget) for (int i = threadIdx.x; i < n; i += TH) list[i] = i;
        else if (v.n <= 128) { if (wave == 0) select_by_wave<2>(sc, v.n, budget, keep_first, keep_last, list); }
        else if (v.n <= 512) { if (wave == 0) select_by_wave<8>(sc, v.n, budget, keep_first, keep_last, list); }
        else if (v.n <= 2048) select_by_group<W, 4>(sc, v.n, 0, budget, keep_first, keep_last, list, sm);
        else if (v.n <= 8192) select_by_group<W, 16>(sc, v.n, 0, budget, keep_first, keep_last, list, sm);
        else select_by_group<W, 32>(sc, v.n, 0, budget, keep_first, keep_last, list, sm);
    }
    __syncthreads();
    const int32_t *mine = chosen ? list : list + i0;
    for (int g0 = 0; g0 < G; g0 += A::HEADS) {
        const int heads = min(A::HEADS, G - g0);
        const int64_t head = (int64_t)kvh * G + g0;
        if (g0) {
            A::stage(q + (int64_t)t * q_stride + head * HD, heads, qs);
            __syncthreads();
        }
        A a;
        a.start(qs, heads, lane);
        for (int i = 2 * wave; i < i1 - i0; i += 2 * W) {
            const int b0 = mine[i], b1 = i + 1 < i1 - i0 ? mine[i + 1] : -1;
            const int64_t p0 = trow[b0], p1 = b1 >= 0 ? trow[b1] : p0;
            typename A::Pair d;
            A::load(d, pool + p0 * bs, pool + p1 * bs, Hkv, kvh, lane);
            a.add(d, (v.b0 + b0) * 16, b1 >= 0 ? (v.b0 + b1) * 16 : -16, v.start, ctx, pl[wave], lane);
        }
        put_wave<A, HD, W>(a, qs, heads, pool, bs, Hkv, kvh, i1 - i0, [&](int i, int &b, int64_t &p) { b = v.b0 + mine[i]; p = trow[mine[i]]; },
                           v.start, ctx, so, ml, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < heads * HD; i += TH) {
            float M, L;
            const float o = join_waves<HD, A::HEADS, W>(so, ml, i / HD, i % HD, M, L);
            const int64_t item = ((int64_t)t * H + head + i / HD) * chunks + c;
            if (real == 1) { out[((int64_t)t * H + head) * HD + i] = o / L; continue; }
            store_shared(part_o + item * HD + i % HD, o);
            if (i % HD == 0) { store_shared(part_ml + item * 2, M); store_shared(part_ml + item * 2 + 1, L); }
        }
        __syncthreads();
    }
    if (c == 0 && !chosen)
        for (int i = threadIdx.x; i < budget; i += TH) gsel[i] = i < n ? v.b0 + list[i] : -1;
    if (real == 1) return;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // this wave's shares have arrived
    __syncthreads();
    if (threadIdx.x == 0) last = __hip_atomic_fetch_add(&tickets[(int64_t)t * Hkv + kvh], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == real - 1;
    __syncthreads();
    if (!last) return;
    for (int i = threadIdx.x; i < G * HD; i += TH) {
        const int64_t base = ((int64_t)t * H + (int64_t)kvh * G + i / HD) * chunks;
        float M = -INFINITY, o = 0.f, L = 0.f;
#pragma unroll 8
        for (int k = 0; k < real; k++) M = fmaxf(M, load_shared(part_ml + (base + k) * 2));
        M = M > -INFINITY ? M : 0.f;
#pragma unroll 8
        for (int k = 0; k < real; k++) {
            const float w = fast_exp2(load_shared(part_ml + (base + k) * 2) - M);
            o += w * load_shared(part_o + (base + k) * HD + i % HD);
            L += w * load_shared(part_ml + (base + k) * 2 + 1);
        }
        out[((int64_t)t * H + (int64_t)kvh * G) * HD + i] = o / L;
    }
}

__global__ __launch_bounds__(256) void k_sparse_clear(int32_t *__restrict__ tickets, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) tickets[i] = 0;
}

// Everything for one (row, KV head) in one workgroup: scores into LDS, the choice, attention, the waves joined.  One launch and no scratch,
// for up to FUSED_BLOCKS visible blocks.  Four waves, three workgroups a CU (by registers), so that the memory has work while one of them
// chooses: 7B batch 32, 590 MB, 104 us (5.7 TB/s); with eight waves and one workgroup a CU 119.
constexpr int FUSED_BLOCKS = 2048, FUSED_BUDGET = 1024, FUSED_WAVES = 4;

template <typename A, int HD>
__global__ __launch_bounds__(64 * FUSED_WAVES, A::WORKGROUPS) void k_sparse_row(const float *__restrict__ q, int q_stride, const typename A::KT *__restrict__ pool,
                                                                 const int8_t *__restrict__ bounds, const float *__restrict__ unit, int Hkv,
                                                                 const int32_t *__restrict__ table, int table_stride,
                                                                 const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len,
                                                                 int max_ctx, int G, int window, int budget, int keep_first, int keep_last,
                                                                 float *__restrict__ out, int32_t *__restrict__ sel) {
    constexpr int W = FUSED_WAVES;
    __shared__ __attribute__((aligned(16))) float sc[FUSED_BLOCKS];
    __shared__ __attribute__((aligned(16))) ScoreQueries<HD> qq;
    __shared__ int32_t phys[FUSED_BLOCKS], list[FUSED_BUDGET];
    __shared__ SelectRoom<W> sm;
    __shared__ __attribute__((aligned(16))) typename A::Queries qs;
    __shared__ __attribute__((aligned(16))) float pl[W][16], so[W * A::HEADS * HD], ml[2 * W * A::HEADS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int kvh = blockIdx.x, t = blockIdx.y;
    const int ctx = min(ctx_len[t], max_ctx);
    const Visible v = visible(ctx, window);
    const int64_t H = (int64_t)Hkv * G, bs = kv_block_elems(Hkv, HD);
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride + v.b0;
    int32_t *gsel = sel + ((int64_t)t * Hkv + kvh) * budget;
    const int n = min(v.n, budget);
    if (v.n > budget) {
        for (int g0 = 0; g0 < G; g0 += 16) {
            const int heads = min(16, G - g0);
            quantise_queries<HD>(q + (int64_t)t * q_stride + ((int64_t)kvh * G + g0) * HD, heads, qq, W);
            __syncthreads();
            const ScoreOperand<HD> sq(qq, heads, lane);
            if (g0 + 16 < G) __syncthreads();
            for (int tile = wave; tile * 16 < v.n; tile += W) {
                const int blk = tile * 16 + (lane & 15), id = trow[min(blk, v.n - 1)];
                if (lane < 16 && blk < v.n) phys[blk] = id;
                const float x = score_tile<HD>(sq, bounds, unit, id, Hkv, kvh, lane);
                const int at = tile * 16 + 4 * (lane >> 4) + (lane & 3);
                if ((lane & 15) < 4 && at < v.n) sc[at] = g0 ? fmaxf(sc[at], x) : x;
            }
        }
        __syncthreads();
        if (v.n <= 128) {
            if (wave == 0) select_by_wave<2>(sc, v.n, budget, keep_first, keep_last, list);
        } else if (v.n <= 512) {
            if (wave == 0) select_by_wave<8>(sc, v.n, budget, keep_first, keep_last, list);
        } else {
            select_by_group<W, FUSED_BLOCKS / (64 * W)>(sc, v.n, 0, budget, keep_first, keep_last, list, sm);
        }
    } else {
        for (int i = threadIdx.x; i < n; i += 64 * W) { list[i] = i; phys[i] = trow[i]; }
    }
    for (int g0 = 0; g0 < G; g0 += A::HEADS) {
        const int heads = min(A::HEADS, G - g0);
        const int64_t head = (int64_t)kvh * G + g0;
        A::stage(q + (int64_t)t * q_stride + head * HD, heads, qs);
        __syncthreads();
        if (g0 == 0)
            for (int i = threadIdx.x; i < budget; i += 64 * W) gsel[i] = i < n ? v.b0 + list[i] : -1;
        A a;
        a.start(qs, heads, lane);
        for (int i = 2 * wave; i < n; i += 2 * W) {
            const int b0 = list[i], b1 = i + 1 < n ? list[i + 1] : -1;
            const int64_t p0 = phys[b0], p1 = b1 >= 0 ? phys[b1] : p0;
            typename A::Pair d;
            A::load(d, pool + p0 * bs, pool + p1 * bs, Hkv, kvh, lane);
            a.add(d, (v.b0 + b0) * 16, b1 >= 0 ? (v.b0 + b1) * 16 : -16, v.start, ctx, pl[wave], lane);
        }
        put_wave<A, HD, W>(a, qs, heads, pool, bs, Hkv, kvh, n, [&](int i, int &b, int64_t &p) { b = v.b0 + list[i]; p = phys[list[i]]; },
                           v.start, ctx, so, ml, wave, lane);
        __syncthreads();
        for (int i = threadIdx.x; i < heads * HD; i += 64 * W) {
            float M, L;
            const float o = join_waves<HD, A::HEADS, W>(so, ml, i / HD, i % HD, M, L);
            out[((int64_t)t * H + head) * HD + i] = n ? o / L : 0.f;
        }
        __syncthreads();
    }
}

int visible_blocks(int max_ctx, int window) {
    const int all = (int)(((int64_t)max_ctx + 15) / 16);
    return window > 0 ? (int)std::min<int64_t>(all, ((int64_t)window + 14) / 16 + 1) : all;
}

// One launch or two.  A CU alone draws some 50 GB/s, so one workgroup a (row, KV head) is slow where there are few of them and each has much to
// read; two launches and the meeting of the shares cost 4 - 5 us.  us, one / two launches: 32 pairs of 160 KB each 11.5 / 13.0, 40 of 192 KB 15.5 / 16.7, 32 of
// 192 KB 15.1 / 14.7, 80 of 192 KB 18.1 / 17.2, 32 of 256 KB 21.7 / 16.2, 80 of 280 KB 21.6 / 16.4, 192 of 256 KB 26.0 / 21.9; 1024 of 580 KB 104 / 127.
bool fused_form(int T, int Hkv, int hd, int el, int nb, int budget) {
    const int n = std::min(nb, budget);
    if (nb > FUSED_BLOCKS || n > FUSED_BUDGET) return false;
    return (int64_t)T * Hkv >= 256 || (int64_t)(nb > budget ? nb : 0) * 2 * hd + (int64_t)n * 32 * hd * el <= 176 << 10;
}

// Split form: as many chunks a (row, KV head) as bring a workgroup to every CU and, where the pairs alone do not, no CU a second one (80 pairs, 280 KB
// each: 16 us with 240 workgroups, 22 with 320), of two blocks at least.  The scratch holds scores, shares and tickets.
struct SparsePlan { int nb, stride, cb, chunks; size_t scores, part_o, part_ml, total; };
SparsePlan sparse_plan(int T, int H, int Hkv, int hd, int max_ctx, int window, int budget) {
    SparsePlan p;
    p.nb = visible_blocks(max_ctx, window);
    p.stride = (p.nb + 31) / 32 * 32;      // the choice reads whole vectors
    const int n = std::max(1, std::min(p.nb, budget));
    const int64_t pairs = (int64_t)T * Hkv, want = std::max<int64_t>(1, 256 / pairs);
    p.cb = (int)std::min<int64_t>(std::max<int64_t>(2, (n + want - 1) / want), SPLIT_BUDGET);      // a chunk's list fits the LDS
    p.chunks = (n + p.cb - 1) / p.cb;
    const size_t shares = (size_t)H / Hkv * (256 + pairs * ((n + SPLIT_BUDGET - 1) / SPLIT_BUDGET));
    p.scores = p.nb > budget ? ld::align_up((size_t)pairs * p.stride * 4, 256) : 0;
    p.part_o = ld::align_up(shares * hd * 4, 256);
    p.part_ml = ld::align_up(shares * 8, 256);
    p.total = p.scores + p.part_o + p.part_ml + ld::align_up((size_t)pairs * 4, 256);
    return p;
}

struct SparseArgs {
    const float *q; int q_stride; const void *pool; const int8_t *bounds; const float *unit; const int32_t *table; int table_stride;
    const int32_t *seq_slot, *ctx_len; int max_ctx, T, H, Hkv, window, budget, keep_first, keep_last; float *out; int32_t *sel; char *scratch;
};

template <typename A, int HD>
void launch_sparse(const SparseArgs &a, hipStream_t s) {
    const typename A::KT *pool = (const typename A::KT *)a.pool;
    const int G = a.H / a.Hkv, nb = visible_blocks(a.max_ctx, a.window);
    if (fused_form(a.T, a.Hkv, HD, sizeof(typename A::KT), nb, a.budget)) {
        LD_LAUNCH((k_sparse_row<A, HD>), dim3(a.Hkv, a.T), dim3(64 * FUSED_WAVES), 0, s, a.q, a.q_stride, pool, a.bounds, a.unit, a.Hkv, a.table,
                  a.table_stride, a.seq_slot, a.ctx_len, a.max_ctx, G, a.window, a.budget, a.keep_first, a.keep_last, a.out, a.sel);
        return;
    }
    const SparsePlan p = sparse_plan(a.T, a.H, a.Hkv, HD, a.max_ctx, a.window, a.budget);
    char *at = a.scratch;
    float *scores = (float *)at, *part_o = (float *)(at += p.scores), *part_ml = (float *)(at += p.part_o);
    int32_t *tickets = (int32_t *)(at += p.part_ml);
    if (p.nb > a.budget) {
        const int tiles = (p.nb + 15) / 16;
        const int64_t waves = (int64_t)tiles * a.Hkv * a.T;
        const int per = (int)std::max<int64_t>(1, std::min<int64_t>(8, waves / 4096));      // tiles a wave
        LD_LAUNCH(k_sparse_score<HD>, dim3((tiles + 4 * per - 1) / (4 * per), a.Hkv, a.T), dim3(256), 0, s, a.q, a.q_stride, a.bounds, a.unit, a.table,
                  a.table_stride, a.seq_slot, a.ctx_len, a.max_ctx, a.Hkv, G, a.window, per, p.stride, scores, tickets);
    } else {
        LD_LAUNCH(k_sparse_clear, dim3((a.T * a.Hkv + 255) / 256), dim3(256), 0, s, tickets, a.T * a.Hkv);
    }
    const bool long_choice = p.nb > a.budget && (p.nb > SPLIT_BLOCKS || a.budget > SPLIT_BUDGET);
    const bool chosen = long_choice || std::min(p.nb, a.budget) > SPLIT_BUDGET;
    if (chosen)
        LD_LAUNCH(k_sparse_select_long, dim3(a.Hkv, a.T), dim3(1024), 0, s, scores, p.stride, a.ctx_len, a.max_ctx, a.Hkv, a.window, a.budget,
                  a.keep_first, a.keep_last, a.sel);
    LD_LAUNCH((k_sparse_attend<A, HD>), dim3(p.chunks, a.Hkv, a.T), dim3(64 * SPLIT_WAVES), 0, s, a.q, a.q_stride, pool, a.Hkv, a.table,
              a.table_stride, a.seq_slot, a.ctx_len, a.max_ctx, G, a.window, a.budget, a.keep_first, a.keep_last, scores, p.stride, chosen, p.cb, part_o,
              part_ml, tickets, a.out, a.sel);
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
    return sparse_plan(T, H, Hkv, hd, max_ctx, window, budget).total;
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
    const bool many = H / Hkv > 4;      // more than four query heads a KV head: eight at a time
    if (dtype == LD_BF16 && hd == 128) { if (many) launch_sparse<OnMatrixCores<128, 2>, 128>(a, s); else launch_sparse<OnMatrixCores<128, 1>, 128>(a, s); }
    else if (dtype == LD_BF16) { if (many) launch_sparse<OnMatrixCores<64, 2>, 64>(a, s); else launch_sparse<OnMatrixCores<64, 1>, 64>(a, s); }
    else if (hd == 128) launch_sparse<OnVectorUnits<128>, 128>(a, s);
    else launch_sparse<OnVectorUnits<64>, 64>(a, s);
    return launched("k_sparse_attend");
}

}  // extern "C"
