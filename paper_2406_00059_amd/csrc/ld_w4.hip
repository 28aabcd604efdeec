// Linear layers on 4-bit weights with group scales: W[n, k] = (c[n, k] - z[n, k / G]) s[n, k / G].
//
// The codes never become floats one by one.  A 16-bit half of a packed word with all but four bits cleared IS an fp16
// number: the bits 0 .. 3 as a subnormal c 2^-24, the bits 4 .. 7 as c 2^-20.  So four masks and one shift turn a word
// into the eight fp16 operands of a 16 x 16 x 32 matrix instruction; the columns that sit in bits 4 .. 7 meet
// activations divided by 16, and 2^24 goes into the row's own power of two.
// Activations: a row is scaled by the power of two that brings its largest magnitude to 2^14 .. 2^15 and split into two
// fp16 terms.  hi is a whole number of a quantum that 128 columns share, 2^-12 of the power of two below their largest magnitude:
// |hi| <= 2^13 quanta, so the sum of 128 products with a code stays below 15 / 16 of 2^24 quanta and is exact in a float32
// accumulator, in any order (the matrix cores cut what an addition shifts out, always downwards in magnitude: sums of unlike
// exponents were 2.4e-6 off, relative 2-norm).  lo is what is left (up to 2.5 quanta, half of one for columns below a quarter of the 128's
// maximum), rounded to fp16: 2^-11 of it gets lost at most, that is 2^-22 and 2^-25 of the maximum, or, below fp16's normal numbers, 2^-25 of a unit, 16
// times that for the columns divided by 16: 2^-35 of the row's largest magnitude.  The two terms meet the same codes in accumulators of their own.
// Per group of G columns:  total[n] += s[n] (sum_k c hi + sum_k c lo - z[n] sum_k (hi + lo)), the sums formed with the split.
// (The products of many rows with narrow groups or zero points take c - z in place of the subnormals, see ld_w4_tile.hip; the exactness of hi is the same.)
//
// Image of a matrix: tiles of 16 rows x 128 columns, 1 KB each, lane l's 16 bytes in a row, the tiles of 16 rows one
// after the other along K: a wave streams consecutive kilobytes.  Word j of lane l holds the columns 32 j + 8 (l / 16)
// .. + 8 of row l % 16, column e of the eight in nibble e / 2 + 4 (e % 2).  Behind the codes the scales
// [row tile][group][16], then (optional) the zero points, one byte each, likewise.
#include "ld_w4_device.h"

#include <algorithm>

using namespace ldd;
using namespace ldw;

namespace {

// ---------------------------------------------------------------- laying a matrix out

__device__ __forceinline__ int nibble_of(int e) { return (e >> 1) + 4 * (e & 1); }

__device__ __forceinline__ void store_scale(void *p, int scale_dtype, int64_t i, float v) {
    if (scale_dtype == LD_BF16) ((bf16_t *)p)[i] = f32_to_bf16(v);
    else ((float *)p)[i] = v;
}
__device__ __forceinline__ float load_scale(const void *p, int scale_dtype, int64_t i) {
    return scale_dtype == LD_BF16 ? bf16_to_f32(((const bf16_t *)p)[i]) : ((const float *)p)[i];
}

// One workgroup a tile, thread (row, octet): eight columns each.  Rows and columns past the matrix get code 0 and scale 0.
__global__ __launch_bounds__(256) void k_w4_pack(const uint8_t *__restrict__ codes, const void *__restrict__ scales, int scale_dtype,
                                                 const uint8_t *__restrict__ zeros, int N, int K, int G, ld::W4Image w) {
    const int kt = blockIdx.x, rt = blockIdx.y, part = blockIdx.z;
    const int row = threadIdx.x >> 4, o = threadIdx.x & 15;
    const int n = rt * 16 + row, k0 = kt * 128 + o * 8;
    const int64_t src = (int64_t)part * N + n;
    const int64_t tile = ((int64_t)part * w.row_tiles + rt) * w.k_tiles + kt;
    uint32_t word = 0;
    if (n < N)
        for (int e = 0; e < 8; e++)
            if (k0 + e < K) {
                const uint8_t b = codes[src * ((K + 1) / 2) + ((k0 + e) >> 1)];
                word |= (uint32_t)((e & 1) ? b >> 4 : b & 15) << (4 * nibble_of(e));
            }
    w.codes[(tile * 64 + row + 16 * (o & 3)) * 4 + (o >> 2)] = word;
    const int per = 128 / G, kg = (K + G - 1) / G;
    if (o < per) {
        const int g = kt * per + o;
        const int64_t at = (((int64_t)part * w.row_tiles + rt) * w.groups + g) * 16 + row;
        const bool real = n < N && g < kg;
        store_scale(w.scales, scale_dtype, at, real ? load_scale(scales, scale_dtype, src * kg + g) : 0.f);
        if (w.zeros) w.zeros[at] = real ? min(zeros[src * kg + g], (uint8_t)15) : 0;
    }
}

// Quantised to nearest.  Without zero points s = max |w| / 7 and c = 8 + w / s; with them s = (max - min) / 15 over the group and
// zero, and z = -min / s.  s is rounded to its type before the codes are formed.  A group of zeros: s = 0, the codes z.
template <typename WT>
__global__ __launch_bounds__(256) void k_w4_quantize(const WT *__restrict__ W, int scale_dtype, int N, int K, int G, ld::W4Image w) {
    const int kt = blockIdx.x, rt = blockIdx.y, part = blockIdx.z;
    const int row = threadIdx.x >> 4, o = threadIdx.x & 15;
    const int n = rt * 16 + row, k0 = kt * 128 + o * 8;
    const int64_t src = (int64_t)part * N + n;
    const int64_t tile = ((int64_t)part * w.row_tiles + rt) * w.k_tiles + kt;
    float v[8], lo = 0.f, hi = 0.f;
    for (int e = 0; e < 8; e++) {
        v[e] = 0.f;
        if (n < N && k0 + e < K) {
            if constexpr (sizeof(WT) == 2) v[e] = bf16_to_f32(W[src * K + k0 + e]);
            else v[e] = W[src * K + k0 + e];
        }
        lo = fminf(lo, v[e]);
        hi = fmaxf(hi, v[e]);
    }
    for (int off = 1; off < G / 8; off <<= 1) {      // the G / 8 threads of a group lie next to each other
        lo = fminf(lo, __shfl_xor(lo, off, WAVE));
        hi = fmaxf(hi, __shfl_xor(hi, off, WAVE));
    }
    float s = w.zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f;
    if (scale_dtype == LD_BF16) s = bf16_to_f32(f32_to_bf16(s));
    int z = 8;
    if (w.zeros) z = s > 0.f ? (int)fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0;
    uint32_t word = 0;
    for (int e = 0; e < 8; e++) {
        const int c = s > 0.f ? (int)fminf(fmaxf(rintf(v[e] / s) + z, 0.f), 15.f) : z;
        word |= (uint32_t)c << (4 * nibble_of(e));
    }
    w.codes[(tile * 64 + row + 16 * (o & 3)) * 4 + (o >> 2)] = word;
    const int per = 128 / G;
    if (o % (G / 8) == 0) {
        const int64_t at = (((int64_t)part * w.row_tiles + rt) * w.groups + kt * per + o / (G / 8)) * 16 + row;
        store_scale(w.scales, scale_dtype, at, s);
        if (w.zeros) w.zeros[at] = (uint8_t)z;
    }
}

// ---------------------------------------------------------------- activations

// Image of the activations: for every 16 rows and 32 columns the hi and the lo operand of one matrix instruction, 1 KB
// each in lane order ([row tile][k / 32][term][lane][8]).  sums [row tile][group][term][16]: 2^-24 times the sums of a group's
// columns (those of hi are exact).  expo[t]: the exponent that takes a finished sum back, or W4_NOT_FINITE.

// One row by a workgroup of THREADS threads: a thread takes four columns at a time, NC times, and keeps them (NC = 0: longer rows, read
// twice).  put(c, hi, lo): columns c .. c + 3 as fp16; put_sums(group, hi, lo), by one thread each.  Returns the row's exponent.
template <int THREADS, int NC>
struct SplitRow {
    static constexpr int STEP = THREADS * 4, WAVES = THREADS / 64;
    f32x4 kept[NC ? NC : 1], weight[NC ? NC : 1];
    const float *row, *gain;
    int K;
    bool quads;
    struct Room { float ss[WAVES]; uint32_t top[WAVES]; };

    __device__ __forceinline__ void fetch(const float *p, int c, f32x4 &v) const {
        if (quads) {
            if (c < K) v = *reinterpret_cast<const f32x4 *>(p + c);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (c + e < K) v[e] = p[c + e];
        }
    }
    __device__ __forceinline__ f32x4 value(int c) const {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        fetch(row, c, v);
        return v;
    }
    __device__ __forceinline__ f32x4 gain_at(int c) const {
        f32x4 g = {1.f, 1.f, 1.f, 1.f};
        if (gain) fetch(gain, c, g);
        return g;
    }
    // Asks for the row (aligned: all rows' starts and the gain are 16-byte aligned).
    __device__ __forceinline__ void load(const float *x, const float *g, int columns, bool aligned) {
        row = x; gain = g; K = columns; quads = aligned;
        if constexpr (NC > 0) {
#pragma unroll
            for (int i = 0; i < NC; i++) {
                kept[i] = value(i * STEP + threadIdx.x * 4);
                weight[i] = gain_at(i * STEP + threadIdx.x * 4);
            }
        }
    }
    template <bool SUBNORMAL, typename Put, typename Sums>
    __device__ __forceinline__ int split(float eps, int Kp, int G, Room &sm, Put put, Sums put_sums) {
        float ss = 0.f;
        uint32_t top = 0;      // largest |x gain|, compared as bits: a NaN stays
        auto look = [&](const f32x4 &v, const f32x4 &g) {
#pragma unroll
            for (int e = 0; e < 4; e++) {
                ss += v[e] * v[e];
                top = max(top, __float_as_uint(v[e] * g[e]) & 0x7fffffffu);
            }
        };
        if constexpr (NC > 0) {
#pragma unroll
            for (int i = 0; i < NC; i++) look(kept[i], weight[i]);
        } else {
            for (int c = threadIdx.x * 4; c < K; c += STEP) look(value(c), gain_at(c));
        }
        ss = lanes_sum(ss, 32);
        ss += swapped_half(ss);
        const float most = max_of_32(__uint_as_float(top));      // as floats here: a NaN is put aside first
        top = __any(top > 0x7f800000u) ? 0x7fc00000u : __float_as_uint(fmaxf(most, swapped_half(most)));
        if ((threadIdx.x & 63) == 0) { sm.ss[threadIdx.x >> 6] = ss; sm.top[threadIdx.x >> 6] = top; }
        lds_barrier();
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; i++) { ss += sm.ss[i]; top = max(top, sm.top[i]); }
        const float inv = gain ? 1.f / sqrtf(ss / K + eps) : 1.f;
        const float m = __uint_as_float(top) * inv;
        const bool finite = m < INFINITY;      // false for NaN
        const int k = row_exponent(m);
        auto part = [&](int c, const f32x4 &raw, const f32x4 &g) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = finite ? raw[e] * inv * g[e] : 0.f;      // in the order of the definition: x / rms, then the gain
            split4<SUBNORMAL>(v, k, c, G, put, put_sums);
        };
        if constexpr (NC > 0) {
#pragma unroll
            for (int i = 0; i < NC; i++)
                if (i * STEP + (int)threadIdx.x * 4 < Kp) part(i * STEP + threadIdx.x * 4, kept[i], weight[i]);
        } else {
            for (int c = threadIdx.x * 4; c < Kp; c += STEP) part(c, value(c), gain_at(c));
        }
        return finite ? (SUBNORMAL ? 24 : 0) - k : ld::W4_NOT_FINITE;
    }
};

// The activations of a product of many rows, a workgroup a row.  Latency at few rows (32 x 4096: 4.4 us), the image's 8-byte pieces
// at many (257 x 11008, 23 MB read and written: 11.4 us, 2 TB/s).
constexpr int SPLIT_THREADS = 512;
template <int NC, bool SUBNORMAL>
__global__ __launch_bounds__(SPLIT_THREADS) void k_w4_split(const float *__restrict__ x, const float *__restrict__ gain, float eps, int T, int K, int G,
                                                            ld::W4Rows r) {
    // the 16 rows of a tile fill the same lines of the image: they go to one XCD (workgroups take turns over eight), whose L2 puts the lines together
    const int t = (int)(blockIdx.x / 128 * 8 + blockIdx.x % 8) * 16 + blockIdx.x / 8 % 16;
    if (t >= T) return;
    __shared__ typename SplitRow<SPLIT_THREADS, NC>::Room sm;
    SplitRow<SPLIT_THREADS, NC> row;
    row.load(x + (int64_t)t * K, gain, K, K % 4 == 0 && (((uintptr_t)x | (uintptr_t)gain) & 15) == 0);
    const int Kp = r.k_tiles * 128, rt = t >> 4, col = t & 15, groups = Kp / G;
    const int expo = row.template split<SUBNORMAL>(
        eps, Kp, G, sm,
        [&](int c, uint2 hi, uint2 lo) {
            const int kb = c >> 5, slot = col + 16 * ((c & 31) >> 3), half = (c & 7) * 2;      // half: bytes into the lane's 16
            char *p = (char *)r.image + (((int64_t)rt * r.k_tiles * 4 + kb) * 128 + slot) * 16 + half;
            *reinterpret_cast<uint2 *>(p) = hi;
            *reinterpret_cast<uint2 *>(p + 1024) = lo;
        },
        [&](int g, float hi, float lo) {
            float *p = r.sums + ((int64_t)rt * groups + g) * 32 + col;
            p[0] = hi;
            p[16] = lo;
        });
    if (threadIdx.x == 0) r.expo[t] = expo;
}

void launch_split(const float *x, const float *g, float eps, int T, int K, int G, bool zeros, const ld::W4Rows &r, hipStream_t s) {
    const dim3 grid((T + 127) / 128 * 128), block(SPLIT_THREADS);
#define LD_SPLIT(NC_)                                                                                          \
    do {                                                                                                       \
        if (ld::w4_subnormal(G, zeros)) LD_LAUNCH((k_w4_split<NC_, true>), grid, block, 0, s, x, g, eps, T, K, G, r); \
        else LD_LAUNCH((k_w4_split<NC_, false>), grid, block, 0, s, x, g, eps, T, K, G, r);                    \
    } while (0)
    if (K <= 2 * 2048) LD_SPLIT(2);
    else if (K <= 7 * 2048) LD_SPLIT(7);
    else LD_SPLIT(0);
#undef LD_SPLIT
}

// ---------------------------------------------------------------- the product, few rows

// One row, or a few short ones.  A workgroup of eight waves splits the rows into LDS by itself, while its first codes are on their way; a launch
// ahead would take longer than the product.  It takes units of R tiles of 16 output rows (SwiGLU: the gate tile and its up tile), every
// gridDim.x-th of them; wave w multiplies the column tiles w, w + 8, .., and the eight sums meet in LDS.  Up to eight rows make one
// operand: columns 0 .. 7 are their hi terms, 8 .. 15 the lo terms, so that both cost what one does.
// AHEAD column tiles are asked for at any time, also over the end of a unit, and without a condition (past an end the last one again): a wait
// for one then leaves the younger ones in flight.
// One row of 4096 columns: 4096 outputs 5.7 us (9 MB), gated 2 x 11008 14.4 us (47 MB: 3.3 TB/s over the call, of which the start and the row's split
// take some 5 us), 32000 outputs 15.0 us; 11008 columns, 4096 outputs 10.4 us.  With the split in a launch ahead each took 3 - 4 us more.
template <int G, int R, int T, int NC, typename ST, bool ZEROS>
__global__ __launch_bounds__(512, 4) void k_w4_rows(ld::W4Image w, const float *__restrict__ x, const float *__restrict__ gain, float eps, int N, int K,
                                                    int epilogue, float *__restrict__ y) {
    constexpr int WAVES = 8, PER = 128 / G;
    constexpr int AHEAD = R == 1 && PER < 4 ? 4 : R * PER * sizeof(ST) < 32 ? 2 : 1;      // by the registers that a column tile takes
    extern __shared__ __attribute__((aligned(16))) char sm_rows[];      // [row][term] of `stride` bytes, then sums [row][group][term]
    __shared__ f32x4 sm[2][WAVES][R][64];
    __shared__ int expo[T];
    __shared__ typename SplitRow<512, NC>::Room room;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, h = lane >> 4;
    const bool pair = epilogue == LDK_SWIGLU;
    const int units = pair ? w.row_tiles : (w.row_tiles + R - 1) / R;
    const int steps = ((w.k_tiles + WAVES - 1) / WAVES + AHEAD - 1) / AHEAD * AHEAD;      // column tiles a wave, up to a multiple of AHEAD
    const int Kp = w.k_tiles * 128, stride = Kp * 2 + 64;      // 64: neighbouring rows' pieces lie in different banks
    float *sm_sums = reinterpret_cast<float *>(sm_rows + 2 * T * stride);

    CodeTile<PER, ST, ZEROS> ring[AHEAD][R];
    // asks for step `at` of a unit, or of the workgroup's next one where the unit ends before it
    auto fill = [&](CodeTile<PER, ST, ZEROS> (&q)[R], int unit, int at) {
        if (at >= steps) { at -= steps; unit += gridDim.x; }
        unit = min(unit, units - 1);
        const int kt = min(wave + at * WAVES, w.k_tiles - 1);
#pragma unroll
        for (int i = 0; i < R; i++) q[i].load(w, pair ? (int64_t)i * w.row_tiles + unit : min(unit * R + i, w.row_tiles - 1), kt, lane);
    };
#pragma unroll
    for (int t = 0; t < T; t++) {
        SplitRow<512, NC> row;
        row.load(x + (int64_t)t * K, gain, K, K % 4 == 0 && (((uintptr_t)x | (uintptr_t)gain) & 15) == 0);
        if (t == 0) {
#pragma unroll
            for (int u = 0; u < AHEAD; u++) fill(ring[u], blockIdx.x, u);
        } else {
            lds_barrier();      // everyone has read the room
        }
        const int e = row.template split<true>(
            eps, Kp, G, room,
            [&](int c, uint2 hi, uint2 lo) {
                *reinterpret_cast<uint2 *>(sm_rows + 2 * t * stride + c * 2) = hi;
                *reinterpret_cast<uint2 *>(sm_rows + (2 * t + 1) * stride + c * 2) = lo;
            },
            [&](int g, float hi, float lo) { *reinterpret_cast<float2 *>(sm_sums + 2 * (t * w.groups + g)) = make_float2(hi, lo); });
        if (threadIdx.x == 0) expo[t] = e;
    }
    lds_barrier();

    f32x4 total[R];
    const int t_col = min(col & 7, T - 1);      // columns past the rows repeat the last one's
    const char *operand = sm_rows + (2 * t_col + (col >> 3)) * stride + 16 * h;
    const float *my_sums = sm_sums + 2 * t_col * w.groups + (col >> 3);
    auto multiply = [&](const CodeTile<PER, ST, ZEROS> (&q)[R], int kt) {
#pragma unroll
        for (int p = 0; p < PER; p++) {
            f32x4 acc[R];
#pragma unroll
            for (int i = 0; i < R; i++) acc[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = p * (G / 32); j < (p + 1) * (G / 32); j++) {
                const f16x8 b = *reinterpret_cast<const f16x8 *>(operand + kt * 256 + 64 * j);
#pragma unroll
                for (int i = 0; i < R; i++) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_as_subnormals(q[i].code[j]), b, acc[i], 0, 0, 0);
            }
            const float sum = my_sums[2 * (kt * PER + p)];
#pragma unroll
            for (int i = 0; i < R; i++)
#pragma unroll
                for (int e = 0; e < 4; e++) total[i][e] += q[i].s(p, e) * (acc[i][e] - q[i].z(p, e) * sum);
        }
    };
    int turn = 0;
    for (int unit = blockIdx.x; unit < units; unit += gridDim.x, turn ^= 1) {
#pragma unroll
        for (int i = 0; i < R; i++) total[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
        for (int at = 0; at < steps; at += AHEAD)
#pragma unroll
            for (int u = 0; u < AHEAD; u++) {
                const int kt = wave + (at + u) * WAVES;
                if (kt < w.k_tiles) multiply(ring[u], kt);
                fill(ring[u], unit, at + u + AHEAD);
            }
#pragma unroll
        for (int i = 0; i < R; i++) sm[turn][wave][i][lane] = total[i];
        lds_barrier();      // the other half of sm is free by the next one: whoever reads it does so ahead of that
        // 16 sums (8 waves, 2 terms) of each of 16 R values a row: one a lane, joined across the 16 lanes of a row of the wave; a value's
        // two halves (R = 2) lie in neighbouring rows
        const int part = R == 2 ? (threadIdx.x >> 4) & 1 : 0, j = threadIdx.x >> (R == 2 ? 5 : 4);
        const int n = (R == 2 && !pair ? unit * 2 + part : unit) * 16 + j;
        if (R == 2 || j < 16)
#pragma unroll
            for (int t = 0; t < T; t++) {
                float v = sm[turn][col & 7][part][(t + (col & 8)) + 16 * (j >> 2)][j & 3];
                v += dpp<0xb1>(v);
                v += dpp<0x4e>(v);
                v += dpp<0x141>(v);
                v += dpp<0x140>(v);
                float out = ld::w4_finish(v, expo[t]);
                if (pair) out = ld::w4_gated(out, other_row(out, [](float, float b) { return b; }));
                if (col == 0 && n < N && !(pair && part)) {
                    float *dst = y + (int64_t)t * N + n;
                    *dst = epilogue == LDK_ADD ? *dst + out : out;
                }
            }
    }
}

struct Few { const float *x, *g; float eps; int T, N, K, epilogue; float *y; };

template <int G, int R, int T, int NC>
void launch_rows(const ld::W4Image &w, int scale_dtype, const Few &a, hipStream_t s) {
    // two workgroups a CU, each with the same number of units
    const int units = a.epilogue == LDK_SWIGLU ? w.row_tiles : (w.row_tiles + R - 1) / R, each = (units + 511) / 512;
    const dim3 grid((units + each - 1) / each), block(512);
    const size_t lds = (size_t)T * (2 * (w.k_tiles * 256 + 64) + w.groups * 8);
#define LD_ROWS(S_, Z_) LD_LAUNCH((k_w4_rows<G, R, T, NC, S_, Z_>), grid, block, lds, s, w, a.x, a.g, a.eps, a.N, a.K, a.epilogue, a.y)
    if (scale_dtype == LD_BF16) { if (w.zeros) LD_ROWS(bf16_t, true); else LD_ROWS(bf16_t, false); }
    else { if (w.zeros) LD_ROWS(float, true); else LD_ROWS(float, false); }
#undef LD_ROWS
}
template <int G, int R>
void launch_rows(const ld::W4Image &w, int scale_dtype, const Few &a, hipStream_t s) {
    if (a.T == 2 && a.K <= 4096) launch_rows<G, R, 2, 2>(w, scale_dtype, a, s);
    else if (a.T == 2) launch_rows<G, R, 2, 3>(w, scale_dtype, a, s);
    else if (a.K <= 4096) launch_rows<G, R, 1, 2>(w, scale_dtype, a, s);
    else if (a.K <= 6144) launch_rows<G, R, 1, 3>(w, scale_dtype, a, s);
    else launch_rows<G, R, 1, 7>(w, scale_dtype, a, s);
}
template <int G>
void launch_group(const ld::W4Image &w, int scale_dtype, const Few &a, hipStream_t s) {
    if (a.epilogue != LDK_SWIGLU && w.row_tiles <= 512) launch_rows<G, 1>(w, scale_dtype, a, s);      // a tile a unit where there are few: more CUs
    else launch_rows<G, 2>(w, scale_dtype, a, s);
}

// Rows that a workgroup splits by itself: one as long as its threads hold it in registers, two up to 6144 columns.  us, by itself / in a launch ahead
// of the tiles, two rows: gated 2 x 13824 x 5120 21 / 27, 15360 x 5120 16 / 19; 4096 x 11008 24 / 21, 4096 x 14336 27 / 24.
bool few_rows(int T, int K) { return (T == 1 && K <= 7 * 2048) || (T == 2 && K <= 3 * 2048); }

constexpr int MOST_ROWS = 1 << 20, MOST_OUTPUTS = 65535 * 16;      // of a call, of a part of an image

bool bad_shape(int N, int K, int group, int parts, int scale_dtype) {
    return N <= 0 || K <= 0 || N > (1 << 28) || K > (1 << 28) || (group != 32 && group != 64 && group != 128) || (parts != 1 && parts != 2) ||
           (scale_dtype != LD_BF16 && scale_dtype != LD_F32);
}

}  // namespace

namespace ld {

W4Image w4_image(const void *image, int N, int K, int group, int parts, int scale_dtype, bool zeros, size_t *bytes) {
    W4Image w{};
    w.row_tiles = (N + 15) / 16;
    w.k_tiles = (K + 127) / 128;
    w.groups = w.k_tiles * (128 / group);
    const size_t tiles = (size_t)parts * w.row_tiles * w.k_tiles, groups = (size_t)parts * w.row_tiles * w.groups * 16;
    char *p = (char *)image;
    w.codes = (uint32_t *)p;
    w.scales = p + tiles * 1024;
    const size_t at = align_up(tiles * 1024 + groups * (scale_dtype == LD_BF16 ? 2 : 4), 256);
    w.zeros = zeros ? (uint8_t *)p + at : nullptr;
    if (bytes) *bytes = at + (zeros ? align_up(groups, 256) : 0);
    return w;
}

W4Rows w4_rows(void *scratch, int T, int K, size_t part_bytes, size_t *bytes) {
    W4Rows r{};
    r.k_tiles = (K + 127) / 128;
    const size_t tiles = (size_t)(T + 15) / 16 * r.k_tiles * 4;      // blocks of 16 rows x 32 columns
    char *p = (char *)scratch;
    r.image = (uint16_t *)p;
    r.sums = (float *)(p + tiles * 2048);                            // at the finest group
    r.expo = (int32_t *)(p + tiles * (2048 + 128));
    const size_t at = align_up(tiles * (2048 + 128) + (size_t)T * 4, 256);
    r.part = (float *)(p + at);
    if (bytes) *bytes = at + part_bytes;
    return r;
}

}  // namespace ld

extern "C" {

size_t ldk_w4_image_bytes(int32_t N, int32_t K, int32_t group, int32_t parts, int32_t scale_dtype, int32_t zeros) {
    if (bad_shape(N, K, group, parts, scale_dtype) || N > MOST_OUTPUTS) return 0;
    size_t bytes = 0;
    ld::w4_image(nullptr, N, K, group, parts, scale_dtype, zeros != 0, &bytes);
    return bytes;
}

ld_status ldk_w4_pack(const uint8_t *codes, const void *scales, int32_t scale_dtype, const uint8_t *zeros, int32_t N, int32_t K,
                      int32_t group, int32_t parts, void *image, size_t image_bytes, void *stream) {
    if (!codes || !scales || !image || ((uintptr_t)image & 15) || bad_shape(N, K, group, parts, scale_dtype))
        return ld::fail(LD_E_INVAL, "ldk_w4_pack: bad argument (group 32, 64 or 128; image 16-byte aligned)");
    size_t need = 0;
    const ld::W4Image w = ld::w4_image(image, N, K, group, parts, scale_dtype, zeros != nullptr, &need);
    if (image_bytes < need) return ld::fail(LD_E_INVAL, "ldk_w4_pack: image too small");
    if (N > MOST_OUTPUTS) return ld::fail(LD_E_RANGE, "ldk_w4_pack: more than 1048560 rows");
    LD_LAUNCH(k_w4_pack, dim3(w.k_tiles, w.row_tiles, parts), dim3(256), 0, (hipStream_t)stream, codes, scales, scale_dtype, zeros, N, K, group, w);
    return launched("k_w4_pack");
}

ld_status ldk_w4_quantize(const void *W, int32_t dtype, int32_t N, int32_t K, int32_t group, int32_t parts, int32_t scale_dtype,
                          int32_t zeros, void *image, size_t image_bytes, void *stream) {
    if (!W || !image || ((uintptr_t)image & 15) || bad_shape(N, K, group, parts, scale_dtype) || (dtype != LD_BF16 && dtype != LD_F32))
        return ld::fail(LD_E_INVAL, "ldk_w4_quantize: bad argument (group 32, 64 or 128; image 16-byte aligned)");
    size_t need = 0;
    const ld::W4Image w = ld::w4_image(image, N, K, group, parts, scale_dtype, zeros != 0, &need);
    if (image_bytes < need) return ld::fail(LD_E_INVAL, "ldk_w4_quantize: image too small");
    if (N > MOST_OUTPUTS) return ld::fail(LD_E_RANGE, "ldk_w4_quantize: more than 1048560 rows");
    const dim3 grid(w.k_tiles, w.row_tiles, parts), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == LD_BF16) LD_LAUNCH(k_w4_quantize<bf16_t>, grid, block, 0, s, (const bf16_t *)W, scale_dtype, N, K, group, w);
    else LD_LAUNCH(k_w4_quantize<float>, grid, block, 0, s, (const float *)W, scale_dtype, N, K, group, w);
    return launched("k_w4_quantize");
}

size_t ldk_linear_w4_scratch_bytes(int32_t T, int32_t N, int32_t K, int32_t epilogue) {
    if (T <= 0 || T > MOST_ROWS || N <= 0 || K <= 0 || N > (1 << 28) || K > (1 << 28)) return 0;
    size_t bytes = 0;
    ld::w4_rows(nullptr, T, K, ld::w4_part_bound(T, N, epilogue), &bytes);
    return bytes;
}

ld_status ldk_linear_w4(const void *image, int32_t scale_dtype, int32_t zeros, int32_t group, const float *x, const float *g, float eps,
                        int32_t T, int32_t N, int32_t K, int32_t epilogue, float *y, void *scratch, size_t scratch_bytes, void *stream) {
    if (T == 0) return LD_OK;
    if (!image || ((uintptr_t)image & 15) || !x || !y || T < 0 || epilogue < 0 || epilogue > 2 ||
        bad_shape(N, K, group, epilogue == LDK_SWIGLU ? 2 : 1, scale_dtype))
        return ld::fail(LD_E_INVAL, "ldk_linear_w4: bad argument (group 32, 64 or 128; image 16-byte aligned)");
    if (T > MOST_ROWS) return ld::fail(LD_E_RANGE, "ldk_linear_w4: more than 1048576 rows");
    const bool few = few_rows(T, K);
    const ld::W4Plan plan = few ? ld::W4Plan{} : ld::w4_plan(T, N, K, epilogue);
    size_t need = 0;
    ld::w4_rows(nullptr, T, K, plan.part_bytes, &need);
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < need)
        return ld::fail(LD_E_INVAL, "ldk_linear_w4: scratch missing, not 16-byte aligned or too small");
    hipStream_t s = (hipStream_t)stream;
    const ld::W4Image w = ld::w4_image(image, N, K, group, epilogue == LDK_SWIGLU ? 2 : 1, scale_dtype, zeros != 0, nullptr);
    const ld::W4Rows r = ld::w4_rows(scratch, T, K, 0, nullptr);
    if (!few) {
        launch_split(x, g, eps, T, K, group, zeros != 0, r, s);
        ld::launch_w4_tile(w, scale_dtype, r, group, T, N, epilogue, plan, y, s);
        return launched("k_w4_tile");
    }
    const Few a{x, g, eps, T, N, K, epilogue, y};
    if (group == 32) launch_group<32>(w, scale_dtype, a, s);
    else if (group == 64) launch_group<64>(w, scale_dtype, a, s);
    else launch_group<128>(w, scale_dtype, a, s);
    return launched("k_w4_rows");
}

}  // extern "C"
