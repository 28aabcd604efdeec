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
// exponents were 2.4e-6 off, relative 2-norm).  lo is what is left, rounded to fp16: at worst 2^-23 of the 128 columns' maximum
// gets lost, 2^-25 for columns below a quarter of it.  The two terms meet the same codes in accumulators of their own.
// Per group of G columns:  total[n] += s[n] (sum_k c hi + sum_k c lo - z[n] sum_k x), the sums of x formed with the split.
//
// Image of a matrix: tiles of 16 rows x 128 columns, 1 KB each, lane l's 16 bytes in a row, the tiles of 16 rows one
// after the other along K: a wave streams consecutive kilobytes.  Word j of lane l holds the columns 32 j + 8 (l / 16)
// .. + 8 of row l % 16, column e of the eight in nibble e / 2 + 4 (e % 2).  Behind the codes the scales
// [row tile][group][16], then (optional) the zero points, one byte each, likewise.
#include "ld_w4.h"
#include "ld_device.h"

#include <algorithm>

using namespace ldd;

namespace {

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

inline ld_status launched(const char *what) {
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) {
        ld::set_error("launch of %s failed: %s", what, hipGetErrorString(e));
        return LD_E_HIP;
    }
    return LD_OK;
}

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
// each in lane order ([row tile][k / 32][term][lane][8]).  Up to eight rows share one operand: columns 0 .. 7 of it are
// the hi terms, 8 .. 15 the lo terms ([k / 32][lane][8]).  sums [row tile][group][term][16]: 2^-24 times the sums of a group's
// columns (packed: [group][16] like the operand; those of hi are exact).  expo[t]: the exponent that takes a finished sum back, or W4_NOT_FINITE.
// One workgroup of 512 threads a row; a thread takes four columns at a time, NC times, and keeps them (NC = 0: longer rows, read twice).
constexpr int SPLIT_THREADS = 512;
template <bool PACKED, int NC>
__global__ __launch_bounds__(SPLIT_THREADS) void k_w4_split(const float *__restrict__ x, const float *__restrict__ gain, float eps, int T, int K, int G,
                                                            ld::W4Rows r) {
    constexpr int STEP = SPLIT_THREADS * 4, WAVES = SPLIT_THREADS / 64;
    // the 16 rows of a tile fill the same lines of the image: they go to one XCD (workgroups take turns over eight), whose L2 puts the lines together
    const int t = PACKED ? blockIdx.x : (int)(blockIdx.x / 128 * 8 + blockIdx.x % 8) * 16 + blockIdx.x / 8 % 16;
    if (t >= T) return;
    const float *row = x + (int64_t)t * K;
    const int Kp = r.k_tiles * 128, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool quads = K % 4 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)gain & 15) == 0;
    auto fetch = [&](const float *p, int c, f32x4 &v) {
        if (quads) {
            if (c < K) v = *reinterpret_cast<const f32x4 *>(p + c);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (c + e < K) v[e] = p[c + e];
        }
    };
    float ss = 0.f;
    uint32_t top = 0;      // largest |x gain|, compared as bits: a NaN stays
    auto look = [&](const f32x4 &v, const f32x4 &g) {
#pragma unroll
        for (int e = 0; e < 4; e++) {
            ss += v[e] * v[e];
            top = max(top, __float_as_uint(v[e] * g[e]) & 0x7fffffffu);
        }
    };
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f}, one = {1.f, 1.f, 1.f, 1.f};
    f32x4 kept[NC ? NC : 1], weight[NC ? NC : 1];
    if constexpr (NC > 0) {
#pragma unroll
        for (int i = 0; i < NC; i++) {
            kept[i] = zero;
            weight[i] = one;
            fetch(row, i * STEP + threadIdx.x * 4, kept[i]);
            if (gain) fetch(gain, i * STEP + threadIdx.x * 4, weight[i]);
        }
#pragma unroll
        for (int i = 0; i < NC; i++) look(kept[i], weight[i]);
    } else {
        for (int c = threadIdx.x * 4; c < K; c += STEP) {
            f32x4 v = zero, g = one;
            fetch(row, c, v);
            if (gain) fetch(gain, c, g);
            look(v, g);
        }
    }
    __shared__ float sm_ss[WAVES];
    __shared__ uint32_t sm_top[WAVES];
    ss = wave_sum(ss);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
    if (lane == 0) { sm_ss[wave] = ss; sm_top[wave] = top; }
    __syncthreads();
    ss = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; i++) { ss += sm_ss[i]; top = max(top, sm_top[i]); }
    const float inv = gain ? 1.f / sqrtf(ss / K + eps) : 1.f;
    const float m = __uint_as_float(top) * inv;
    const bool finite = m < INFINITY;      // false for NaN
    const int k = finite && m > 0.f ? 14 - ilogbf(m) : 0;
    if (threadIdx.x == 0) r.expo[t] = finite ? 24 - k : ld::W4_NOT_FINITE;

    const int rt = t >> 4, col = PACKED ? t : t & 15;
    const int groups = Kp / G;
    auto split = [&](int c, const f32x4 &raw, const f32x4 &g) {
        float v[4], sum_hi = 0.f, sum_lo = 0.f, most = 0.f;
        union { _Float16 h[4]; uint2 u; } hi, lo;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            v[e] = ldexpf(finite ? raw[e] * inv * g[e] : 0.f, k);      // in the order of the definition: x / rms, then the gain
            most = fmaxf(most, fabsf(v[e]));
        }
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) most = fmaxf(most, __shfl_xor(most, off, WAVE));      // 128 columns: 32 lanes
        // quantum: 2^-12 of the power of two at or below the largest magnitude, as its bits; at least fp16's least subnormal
        const float quantum = __uint_as_float(max((int)(__float_as_uint(most) & 0x7f800000u) - (12 << 23), (127 - 24) << 23));
        const float per_quantum = __uint_as_float((254u << 23) - __float_as_uint(quantum));      // its reciprocal
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float h = (float)(_Float16)(rintf(v[e] * per_quantum) * quantum);
            const float f = e < 2 ? 1.f : 0.0625f;      // e >= 2: codes in bits 4 .. 7 (c is a multiple of 4)
            hi.h[e] = (_Float16)(h * f);
            lo.h[e] = (_Float16)((v[e] - h) * f);
            sum_hi += h;
            sum_lo += v[e] - h;
        }
        const int kb = c >> 5, slot = col + 16 * ((c & 31) >> 3), half = (c & 7) * 2;      // half: bytes into the lane's 16
        if (PACKED) {
            char *p = (char *)r.image + ((int64_t)kb * 64 + slot) * 16 + half;
            *reinterpret_cast<uint2 *>(p) = hi.u;
            *reinterpret_cast<uint2 *>(p + 8 * 16) = lo.u;
        } else {
            char *p = (char *)r.image + (((int64_t)rt * r.k_tiles * 4 + kb) * 128 + slot) * 16 + half;
            *reinterpret_cast<uint2 *>(p) = hi.u;
            *reinterpret_cast<uint2 *>(p + 1024) = lo.u;
        }
        for (int off = 1; off < G / 4; off <<= 1) {
            sum_hi += __shfl_xor(sum_hi, off, WAVE);
            sum_lo += __shfl_xor(sum_lo, off, WAVE);
        }
        if (c % G == 0) {
            float *p = r.sums + (PACKED ? (int64_t)(c / G) * 16 : ((int64_t)rt * groups + c / G) * 32) + col;
            p[0] = ldexpf(sum_hi, -24);
            p[PACKED ? 8 : 16] = ldexpf(sum_lo, -24);
        }
    };
    if constexpr (NC > 0) {
#pragma unroll
        for (int i = 0; i < NC; i++)
            if (i * STEP + (int)threadIdx.x * 4 < Kp) split(i * STEP + threadIdx.x * 4, kept[i], weight[i]);
    } else {
        for (int c = threadIdx.x * 4; c < Kp; c += STEP) {
            f32x4 v = zero, g = one;
            fetch(row, c, v);
            if (gain) fetch(gain, c, g);
            split(c, v, g);
        }
    }
}

template <bool PACKED>
void launch_split(const float *x, const float *g, float eps, int T, int K, int G, const ld::W4Rows &r, hipStream_t s) {
    const dim3 grid(PACKED ? T : (T + 127) / 128 * 128), block(SPLIT_THREADS);
    if (K <= 2 * 2048) LD_LAUNCH((k_w4_split<PACKED, 2>), grid, block, 0, s, x, g, eps, T, K, G, r);
    else if (K <= 7 * 2048) LD_LAUNCH((k_w4_split<PACKED, 7>), grid, block, 0, s, x, g, eps, T, K, G, r);
    else LD_LAUNCH((k_w4_split<PACKED, 0>), grid, block, 0, s, x, g, eps, T, K, G, r);
}

// ---------------------------------------------------------------- the product, few rows

__device__ __forceinline__ f16x8 codes_as_f16(uint32_t w) {
    const uint32_t s = w >> 8;
    return __builtin_bit_cast(f16x8, (u32x4){w & 0x000f000fu, w & 0x00f000f0u, s & 0x000f000fu, s & 0x00f000f0u});
}

// A workgroup of eight waves takes R tiles of 16 output rows (SwiGLU: the gate tile and its up tile) and 16 CT activation rows;
// wave w multiplies the column tiles w, w + 8, ..; the eight sums meet in LDS.  PACKED: up to eight activation rows, both terms in
// one operand.
template <int CT, bool PACKED, int G, int R>
__global__ __launch_bounds__(512) void k_w4_rows(ld::W4Image w, int scale_dtype, ld::W4Rows r, int T, int N, int epilogue, float *__restrict__ y) {
    constexpr int WAVES = 8, PER = 128 / G, TERMS = PACKED ? 1 : 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = lane & 15, h = lane >> 4;
    const bool pair = epilogue == LDK_SWIGLU;
    const int rt0 = pair ? blockIdx.x : blockIdx.x * R;
    const int ct0 = blockIdx.y * CT;
    const int ct_all = (T + 15) >> 4;
    int64_t tile0[R], group0[R];
#pragma unroll
    for (int i = 0; i < R; i++) {
        const int64_t t = pair ? (int64_t)i * w.row_tiles + rt0 : min(rt0 + i, w.row_tiles - 1);
        tile0[i] = t * w.k_tiles;
        group0[i] = t * w.groups;
    }
    f32x4 total[R][CT];
#pragma unroll
    for (int i = 0; i < R; i++)
#pragma unroll
        for (int c = 0; c < CT; c++) total[i][c] = (f32x4){0.f, 0.f, 0.f, 0.f};

    for (int kt = wave; kt < w.k_tiles; kt += WAVES) {
        u32x4 code[R];
#pragma unroll
        for (int i = 0; i < R; i++) code[i] = load_stream16(w.codes + ((tile0[i] + kt) * 64 + lane) * 4);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            f32x4 acc[R][CT][TERMS];
#pragma unroll
            for (int i = 0; i < R; i++)
#pragma unroll
                for (int c = 0; c < CT; c++)
#pragma unroll
                    for (int q = 0; q < TERMS; q++) acc[i][c][q] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = p * (G / 32); j < (p + 1) * (G / 32); j++) {
                f16x8 b[CT][TERMS];
#pragma unroll
                for (int c = 0; c < CT; c++)
#pragma unroll
                    for (int q = 0; q < TERMS; q++) {
                        const int ct = min(ct0 + c, ct_all - 1);
                        const int64_t at = PACKED ? ((int64_t)kt * 4 + j) * 64 : (((int64_t)ct * w.k_tiles + kt) * 4 + j) * 128 + q * 64;
                        u32x4 v = {0, 0, 0, 0};
                        if (!PACKED || (col & 7) < T) v = *reinterpret_cast<const u32x4 *>((const char *)r.image + (at + lane) * 16);
                        b[c][q] = __builtin_bit_cast(f16x8, v);
                    }
#pragma unroll
                for (int i = 0; i < R; i++) {
                    const f16x8 a = codes_as_f16(code[i][j]);
#pragma unroll
                    for (int c = 0; c < CT; c++)
#pragma unroll
                        for (int q = 0; q < TERMS; q++) acc[i][c][q] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b[c][q], acc[i][c][q], 0, 0, 0);
                }
            }
            const int g = kt * PER + p;
            float sum[CT];
#pragma unroll
            for (int c = 0; c < CT; c++) {
                sum[c] = 0.f;
                if (PACKED) {
                    if ((col & 7) < T) sum[c] = r.sums[(int64_t)g * 16 + col];
                } else {
                    const float *p = r.sums + ((int64_t)min(ct0 + c, ct_all - 1) * w.groups + g) * 32 + col;
                    sum[c] = p[0] + p[16];
                }
            }
#pragma unroll
            for (int i = 0; i < R; i++) {
                const int64_t at = (group0[i] + g) * 16 + 4 * h;
                float s[4], z[4];
                if (scale_dtype == LD_BF16) {
                    const uint2 v = *reinterpret_cast<const uint2 *>((const bf16_t *)w.scales + at);
                    s[0] = __uint_as_float(v.x << 16); s[1] = __uint_as_float(v.x & 0xffff0000u);
                    s[2] = __uint_as_float(v.y << 16); s[3] = __uint_as_float(v.y & 0xffff0000u);
                } else {
                    const float4 v = *reinterpret_cast<const float4 *>((const float *)w.scales + at);
                    s[0] = v.x; s[1] = v.y; s[2] = v.z; s[3] = v.w;
                }
                uint32_t zw = 0x08080808u;
                if (w.zeros) zw = *reinterpret_cast<const uint32_t *>(w.zeros + at);
#pragma unroll
                for (int e = 0; e < 4; e++) z[e] = (float)((zw >> (8 * e)) & 255u);
#pragma unroll
                for (int c = 0; c < CT; c++)
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        float d = acc[i][c][0][e] - z[e] * sum[c];
                        if (TERMS == 2) d += acc[i][c][TERMS - 1][e];
                        total[i][c][e] += s[e] * d;
                    }
            }
        }
    }

    __shared__ f32x4 sm[WAVES][R][CT][64];
#pragma unroll
    for (int i = 0; i < R; i++)
#pragma unroll
        for (int c = 0; c < CT; c++) sm[wave][i][c][lane] = total[i][c];
    __syncthreads();
    for (int idx = threadIdx.x; idx < (pair ? 1 : R) * CT * 64; idx += WAVES * 64) {
        const int l = idx & 63, c = (idx >> 6) % CT, i = (idx >> 6) / CT;
        const int t = (ct0 + c) * 16 + (l & 15), n = (rt0 + i) * 16 + 4 * (l >> 4);
        if (t >= T || n >= N || (PACKED && (l & 15) >= 8)) continue;
        f32x4 v[2];
#pragma unroll
        for (int u = 0; u < 2; u++) {
            if (u == 1 && !pair) break;
            const int tile = pair ? u : i;
            f32x4 a = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < WAVES; q++) {
                a += sm[q][tile][c][l];
                if (PACKED) a += sm[q][tile][c][l + 8];
            }
            v[u] = a;
        }
        const int expo = r.expo[t];
        float *dst = y + (int64_t)t * N + n;
        float out[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            out[e] = ld::w4_finish(v[0][e], expo);
            if (pair) out[e] = ld::w4_gated(out[e], ld::w4_finish(v[1][e], expo));
        }
        const int m = min(4, N - n);
        for (int e = 0; e < m; e++) dst[e] = epilogue == LDK_ADD ? dst[e] + out[e] : out[e];
    }
}

template <int CT, bool PACKED, int G>
void launch_rows(const ld::W4Image &w, int scale_dtype, const ld::W4Rows &r, int T, int N, int epilogue, float *y, hipStream_t s) {
    const int tiles = epilogue == LDK_SWIGLU ? w.row_tiles : (w.row_tiles + 1) / 2;
    const dim3 grid(tiles, PACKED ? 1 : (T + 16 * CT - 1) / (16 * CT)), block(512);
    LD_LAUNCH((k_w4_rows<CT, PACKED, G, 2>), grid, block, 0, s, w, scale_dtype, r, T, N, epilogue, y);
}

template <int G>
void launch_group(const ld::W4Image &w, int scale_dtype, const ld::W4Rows &r, int T, int N, int epilogue, float *y, hipStream_t s) {
    if (T <= 8) launch_rows<1, true, G>(w, scale_dtype, r, T, N, epilogue, y, s);
    else if (T <= 16) launch_rows<1, false, G>(w, scale_dtype, r, T, N, epilogue, y, s);
    else if (T <= 32) launch_rows<2, false, G>(w, scale_dtype, r, T, N, epilogue, y, s);
    else launch_rows<4, false, G>(w, scale_dtype, r, T, N, epilogue, y, s);
}

constexpr int TILE_ROWS = 65;      // rows from which the tiled product takes over

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
    if (bad_shape(N, K, group, parts, scale_dtype)) return 0;
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
    if (w.row_tiles > 65535) return ld::fail(LD_E_RANGE, "ldk_w4_pack: more than 1048560 rows");
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
    if (w.row_tiles > 65535) return ld::fail(LD_E_RANGE, "ldk_w4_quantize: more than 1048560 rows");
    const dim3 grid(w.k_tiles, w.row_tiles, parts), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == LD_BF16) LD_LAUNCH(k_w4_quantize<bf16_t>, grid, block, 0, s, (const bf16_t *)W, scale_dtype, N, K, group, w);
    else LD_LAUNCH(k_w4_quantize<float>, grid, block, 0, s, (const float *)W, scale_dtype, N, K, group, w);
    return launched("k_w4_quantize");
}

size_t ldk_linear_w4_scratch_bytes(int32_t T, int32_t N, int32_t K, int32_t epilogue) {
    if (T <= 0 || N <= 0 || K <= 0) return 0;
    size_t bytes = 0;
    ld::w4_rows(nullptr, T, K, T >= TILE_ROWS ? ld::w4_part_bound(T, N, epilogue) : 0, &bytes);
    return bytes;
}

ld_status ldk_linear_w4(const void *image, int32_t scale_dtype, int32_t zeros, int32_t group, const float *x, const float *g, float eps,
                        int32_t T, int32_t N, int32_t K, int32_t epilogue, float *y, void *scratch, size_t scratch_bytes, void *stream) {
    if (T == 0) return LD_OK;
    if (!image || ((uintptr_t)image & 15) || !x || !y || T < 0 || epilogue < 0 || epilogue > 2 ||
        bad_shape(N, K, group, epilogue == LDK_SWIGLU ? 2 : 1, scale_dtype))
        return ld::fail(LD_E_INVAL, "ldk_linear_w4: bad argument (group 32, 64 or 128; image 16-byte aligned)");
    const ld::W4Plan plan = T >= TILE_ROWS ? ld::w4_plan(T, N, K, epilogue) : ld::W4Plan{};
    size_t need = 0;
    ld::w4_rows(nullptr, T, K, plan.part_bytes, &need);
    if (!scratch || ((uintptr_t)scratch & 15) || scratch_bytes < need)
        return ld::fail(LD_E_INVAL, "ldk_linear_w4: scratch missing, not 16-byte aligned or too small");
    if (T > 1 << 20) return ld::fail(LD_E_RANGE, "ldk_linear_w4: more than 1048576 rows");
    hipStream_t s = (hipStream_t)stream;
    const ld::W4Image w = ld::w4_image(image, N, K, group, epilogue == LDK_SWIGLU ? 2 : 1, scale_dtype, zeros != 0, nullptr);
    const ld::W4Rows r = ld::w4_rows(scratch, T, K, 0, nullptr);
    if (T <= 8) launch_split<true>(x, g, eps, T, K, group, r, s);
    else launch_split<false>(x, g, eps, T, K, group, r, s);
    if (T >= TILE_ROWS) {
        ld::launch_w4_tile(w, scale_dtype, r, group, T, N, epilogue, plan, y, s);
        return launched("k_w4_tile");
    }
    if (group == 32) launch_group<32>(w, scale_dtype, r, T, N, epilogue, y, s);
    else if (group == 64) launch_group<64>(w, scale_dtype, r, T, N, epilogue, y, s);
    else launch_group<128>(w, scale_dtype, r, T, N, epilogue, y, s);
    return launched("k_w4_rows");
}

}  // extern "C"
