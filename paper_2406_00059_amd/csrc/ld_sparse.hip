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

// One wave 16 blocks at a time on the matrix cores: A = 16 blocks' bounds (upper, then lower: K = 2 hd bytes), B = the group's
// queries as columns (their positive parts against the upper bounds, their negative parts against the lower), 16 at a time.
template <int HD>
__global__ __launch_bounds__(256) void k_sparse_score(const float *__restrict__ q, int q_stride, const int8_t *__restrict__ bounds,
                                                      const float *__restrict__ unit, const int32_t *__restrict__ table, int table_stride,
                                                      const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len, int max_ctx,
                                                      int Hkv, int G, int window, int tiles_per_wave, int stride, float *__restrict__ scores) {
    constexpr int NJ = HD / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.z, kvh = blockIdx.y;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    const int tile0 = (blockIdx.x * 4 + wave) * tiles_per_wave;
    if (tile0 * 16 >= v.n) return;
    const int c16 = lane & 15, h = lane >> 4;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride + v.b0;
    float *dst = scores + ((int64_t)t * Hkv + kvh) * stride;
    for (int g0 = 0; g0 < G; g0 += 16) {
        const bool real = g0 + c16 < G;
        const float *qp = q + (int64_t)t * q_stride + (int64_t)(kvh * G + (real ? g0 + c16 : 0)) * HD + 16 * h;
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
        i32x4 b[2 * NJ];
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
        const float qu = ldexpf(1.f, qe);
        for (int tile = tile0; tile < tile0 + tiles_per_wave && tile * 16 < v.n; tile++) {
            const int blk = tile * 16 + c16;
            const int64_t phys = trow[min(blk, v.n - 1)];
            const int8_t *rec = bounds + (phys * Hkv + kvh) * 2 * HD + 16 * h;
            i32x4 acc = (i32x4){0, 0, 0, 0};
            i32x4 a[2 * NJ];
#pragma unroll
            for (int j = 0; j < 2 * NJ; j++) a[j] = *reinterpret_cast<const i32x4 *>(rec + 64 * j);
            const float un = unit[phys * Hkv + kvh];
#pragma unroll
            for (int j = 0; j < 2 * NJ; j++) acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[j], b[j], acc, 0, 0, 0);
            float s[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const float u = __shfl(un, 4 * h + i, WAVE);      // lane = block of the tile
                float x = u < INFINITY ? (float)acc[i] * qu * u : INFINITY;
                if (!real) x = -INFINITY;
#pragma unroll
                for (int off = 1; off < 16; off <<= 1) x = fmaxf(x, __shfl_xor(x, off, WAVE));
                s[i] = x;
            }
            if (c16 < 4) {
                const int at = tile * 16 + 4 * h + c16;
                const float x = c16 == 0 ? s[0] : c16 == 1 ? s[1] : c16 == 2 ? s[2] : s[3];
                if (at < v.n) dst[at] = g0 ? fmaxf(dst[at], x) : x;
            }
        }
    }
}

// ---------------------------------------------------------------- selection

__device__ __forceinline__ uint32_t order_key(float f) {
    const uint32_t b = __float_as_uint(f);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// One workgroup a (row, KV head): the k-th largest candidate score by its bits, eight at a time from the top; then one walk in
// index order that writes what is larger, and of what is equal the first ones.
__global__ __launch_bounds__(1024) void k_sparse_select(const float *__restrict__ scores, int stride, const int32_t *__restrict__ ctx_len,
                                                        int max_ctx, int Hkv, int window, int budget, int keep_first, int keep_last,
                                                        int32_t *__restrict__ sel) {
    const int t = blockIdx.y, kvh = blockIdx.x;
    const Visible v = visible(min(ctx_len[t], max_ctx), window);
    int32_t *out = sel + ((int64_t)t * Hkv + kvh) * budget;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (v.n <= budget) {
        for (int i = tid; i < budget; i += 1024) out[i] = i < v.n ? v.b0 + i : -1;
        return;
    }
    const float *sc = scores + ((int64_t)t * Hkv + kvh) * stride;
    const int c0 = keep_first, c1 = v.n - keep_last;      // candidates; budget < n, so the kept ones do not overlap
    int need = budget - keep_first - keep_last;
    __shared__ uint32_t hist[256];
    __shared__ uint32_t sm_prefix;
    __shared__ int sm_need;
    uint32_t prefix = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        for (int i = c0 + tid; i < c1; i += 1024) {
            const uint32_t k = order_key(sc[i]);
            if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1u);
        }
        __syncthreads();
        if (tid == 0) {
            int left = need, bin = 255;
            while (bin > 0 && (int)hist[bin] < left) { left -= (int)hist[bin]; bin--; }
            sm_prefix = prefix | ((uint32_t)bin << shift);
            sm_need = left;
        }
        __syncthreads();
        prefix = sm_prefix;
        need = sm_need;
    }
    // need: how many of the scores equal to the threshold belong to the choice (0 only where nothing but the kept blocks does)
    const bool any = budget > keep_first + keep_last;
    __shared__ int w_take[16], w_eq[16];
    int taken = 0, equal = 0;
    for (int base = 0; base < v.n; base += 1024) {
        const int i = base + tid;
        bool gt = false, eq = false;
        if (i < v.n) {
            if (i < c0 || i >= c1) gt = true;
            else if (any) {
                const uint32_t k = order_key(sc[i]);
                gt = k > prefix;
                eq = k == prefix;
            }
        }
        const uint64_t below = ((uint64_t)1 << lane) - 1;
        const uint64_t be = __ballot(eq);
        if (lane == 0) w_eq[wave] = __popcll(be);
        __syncthreads();
        int eq_before = equal, eq_all = 0;
        for (int w = 0; w < 16; w++) {
            if (w < wave) eq_before += w_eq[w];
            eq_all += w_eq[w];
        }
        const bool take = gt || (eq && eq_before + __popcll(be & below) < need);
        const uint64_t bt = __ballot(take);
        if (lane == 0) w_take[wave] = __popcll(bt);
        __syncthreads();
        int at = taken + __popcll(bt & below), all = 0;
        for (int w = 0; w < 16; w++) {
            if (w < wave) at += w_take[w];
            all += w_take[w];
        }
        if (take && at < budget) out[at] = v.b0 + i;
        taken += all;
        equal += eq_all;
    }
}

// ---------------------------------------------------------------- attention over the selected blocks

// One workgroup a (row, KV head, chunk of the selection), a wave one query head of the group at a time.  Scores: lane = position
// l % 16, a quarter of the dimensions; values: lane = dimensions l (and l + 64).
template <typename KT, int HD>
__global__ __launch_bounds__(256) void k_sparse_attend(const float *__restrict__ q, int q_stride, const KT *__restrict__ pool, int Hkv,
                                                       const int32_t *__restrict__ table, int table_stride,
                                                       const int32_t *__restrict__ seq_slot, const int32_t *__restrict__ ctx_len, int max_ctx,
                                                       int G, int window, int budget, const int32_t *__restrict__ sel, int cb,
                                                       float *__restrict__ part_o, float *__restrict__ part_ml) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x, kvh = blockIdx.y, t = blockIdx.z, chunks = gridDim.x;
    const int ctx = min(ctx_len[t], max_ctx);
    const Visible v = visible(ctx, window);
    const int n = min(v.n, budget);
    const int i0 = c * cb, i1 = min(i0 + cb, n);
    if (i0 >= i1) return;
    const int32_t *list = sel + ((int64_t)t * Hkv + kvh) * budget;
    const int32_t *trow = table + (int64_t)seq_slot[t] * table_stride;
    const int pos16 = lane & 15, part = lane >> 4;
    const float scale = 1.4426950408889634f / sqrtf((float)HD);
    for (int g = wave; g < G; g += 4) {
        const int head = kvh * G + g;
        const float *qp = q + (int64_t)t * q_stride + (int64_t)head * HD + part * (HD / 4);
        float qv[HD / 4];
#pragma unroll
        for (int e = 0; e < HD / 4; e++) qv[e] = qp[e] * scale;
        float m = -INFINITY, l = 0.f, o[HD / 64];
#pragma unroll
        for (int u = 0; u < HD / 64; u++) o[u] = 0.f;
        for (int i = i0; i < i1; i++) {
            const int b = list[i];
            const KT *blk = pool + (int64_t)trow[b] * kv_block_elems(Hkv, HD);
            const int pos = b * 16 + pos16;
            const bool ok = pos >= v.start && pos < ctx;
            float s = 0.f;
            if (ok) {
                const KT *kp = blk + kv_k_offset(HD, kvh, pos16, part * (HD / 4));
#pragma unroll
                for (int e = 0; e < HD / 4; e += 8) {
                    float kv[8];
                    load8(kp + e, kv);
#pragma unroll
                    for (int u = 0; u < 8; u++) s += qv[e + u] * kv[u];
                }
            }
            s += __shfl_xor(s, 16, WAVE);
            s += __shfl_xor(s, 32, WAVE);
            if (!ok) s = -INFINITY;
            float mb = s;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) mb = fmaxf(mb, __shfl_xor(mb, off, WAVE));
            const float m_new = fmaxf(m, mb);      // a selected block holds a visible position
            const float corr = fast_exp2(m - m_new);
            const float p = ok ? fast_exp2(s - m_new) : 0.f;
            m = m_new;
            float ps = p;
#pragma unroll
            for (int off = 1; off < 16; off <<= 1) ps += __shfl_xor(ps, off, WAVE);
            l = l * corr + ps;
#pragma unroll
            for (int u = 0; u < HD / 64; u++) {
                const KT *vp = blk + kv_v_offset(Hkv, HD, kvh, 0, lane + 64 * u);
                float a[8], bb[8], sum = 0.f;
                load8(vp, a);
                load8(vp + 8, bb);
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const bool see = b * 16 + e >= v.start && b * 16 + e < ctx;      // what an unwritten slot holds is not looked at
                    const float pe = __shfl(p, e, WAVE);
                    if (see) sum += pe * (e < 8 ? a[e] : bb[e - 8]);
                }
                o[u] = o[u] * corr + sum;
            }
        }
        const int64_t item = ((int64_t)t * Hkv * G + head) * chunks + c;
#pragma unroll
        for (int u = 0; u < HD / 64; u++) part_o[item * HD + lane + 64 * u] = o[u];
        if (lane == 0) { part_ml[item * 2] = m; part_ml[item * 2 + 1] = l; }
    }
}

// Chunks of a (row, head) joined in their order; a row that sees nothing is 0.
template <int HD>
__global__ __launch_bounds__(HD) void k_sparse_join(const float *__restrict__ part_o, const float *__restrict__ part_ml,
                                                    const int32_t *__restrict__ ctx_len, int max_ctx, int H, int window, int budget, int cb,
                                                    int chunks, float *__restrict__ out) {
    const int h = blockIdx.x, t = blockIdx.y, d = threadIdx.x;
    const int n = min(visible(min(ctx_len[t], max_ctx), window).n, budget);
    const int nc = (n + cb - 1) / cb;
    const int64_t base = ((int64_t)t * H + h) * chunks;
    float M = -INFINITY;
    for (int c = 0; c < nc; c++) M = fmaxf(M, part_ml[(base + c) * 2]);
    float o = 0.f, L = 0.f;
    for (int c = 0; c < nc; c++) {
        const float a = fast_exp2(part_ml[(base + c) * 2] - M);
        o += a * part_o[(base + c) * HD + d];
        L += a * part_ml[(base + c) * 2 + 1];
    }
    out[((int64_t)t * H + h) * HD + d] = nc ? o / L : 0.f;
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

// Scratch that any call of up to T rows, contexts up to max_ctx and this budget can use.  The number of chunks is not monotonic in
// either, so it is bounded: n / cb <= 512 / (T Hkv) unless cb is at its cap of 32, and cb >= 4.
size_t scratch_bound(int T, int H, int Hkv, int hd, int max_ctx, int window, int budget) {
    const int nb = visible_blocks(max_ctx, window);
    const int64_t n = std::max(1, std::min(nb, budget)), rows = (int64_t)T * H;
    const int64_t items = std::min(rows * ((n + 3) / 4), std::max((int64_t)512 * (H / Hkv) + rows, rows * ((n + 31) / 32)));
    return (nb > budget ? ld::align_up((size_t)T * Hkv * nb * 4, 256) : 0) + ld::align_up((size_t)items * hd * 4, 256) +
           ld::align_up((size_t)items * 8, 256);
}

template <typename KT, int HD>
void launch_sparse(const float *q, int q_stride, const KT *pool, const int8_t *bounds, const float *unit, const int32_t *table,
                   int table_stride, const int32_t *seq_slot, const int32_t *ctx_len, int max_ctx, int T, int H, int Hkv, int window, int budget,
                   int keep_first, int keep_last, float *out, int32_t *sel, char *scratch, hipStream_t s) {
    const SparsePlan p = sparse_plan(T, H, Hkv, HD, max_ctx, window, budget);
    float *scores = (float *)scratch, *part_o = (float *)(scratch + p.scores), *part_ml = (float *)(scratch + p.scores + p.part_o);
    const int G = H / Hkv;
    if (p.nb > budget) {
        const int tiles = (p.nb + 15) / 16;
        const int64_t waves = (int64_t)tiles * Hkv * T;
        const int per = (int)std::max<int64_t>(1, std::min<int64_t>(8, waves / 4096));      // tiles a wave
        LD_LAUNCH(k_sparse_score<HD>, dim3((tiles + 4 * per - 1) / (4 * per), Hkv, T), dim3(256), 0, s, q, q_stride, bounds, unit, table,
                  table_stride, seq_slot, ctx_len, max_ctx, Hkv, G, window, per, p.nb, scores);
    }
    LD_LAUNCH(k_sparse_select, dim3(Hkv, T), dim3(1024), 0, s, scores, p.nb, ctx_len, max_ctx, Hkv, window, budget, keep_first, keep_last, sel);
    LD_LAUNCH((k_sparse_attend<KT, HD>), dim3(p.chunks, Hkv, T), dim3(256), 0, s, q, q_stride, pool, Hkv, table, table_stride, seq_slot, ctx_len,
              max_ctx, G, window, budget, sel, p.cb, part_o, part_ml);
    LD_LAUNCH(k_sparse_join<HD>, dim3(H, T), dim3(HD), 0, s, part_o, part_ml, ctx_len, max_ctx, H, window, budget, p.cb, p.chunks, out);
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
#define LD_SPARSE(KT_, HD_)                                                                                                                   \
    launch_sparse<KT_, HD_>(q, q_stride, (const KT_ *)pool_layer, bounds, unit, table, table_stride, seq_slot, ctx_len, max_ctx, T, H, Hkv, window, \
                            budget, keep_first, keep_last, out, sel, (char *)scratch, s)
    if (dtype == LD_BF16) { if (hd == 128) LD_SPARSE(bf16_t, 128); else LD_SPARSE(bf16_t, 64); }
    else { if (hd == 128) LD_SPARSE(float, 128); else LD_SPARSE(float, 64); }
#undef LD_SPARSE
    return launched("k_sparse_attend");
}

}  // extern "C"
