// The 8-bit cache: layout of a layer, and what its kernels share.
#pragma once
#include <cmath>
#include "ld_device.h"

namespace ldd {

constexpr int Q8_NAN = -128;      // exponent of a vector that is not finite

// Offsets in codes (bytes) of a block; its exponents are [2][Hkv][16].
__device__ __forceinline__ int64_t q8_block(int Hkv, int hd) { return (int64_t)2 * Hkv * 16 * hd; }
__device__ __forceinline__ int64_t q8_k(int hd, int kvh, int slot, int dim) { return ((int64_t)kvh * 16 + slot) * hd + dim; }
__device__ __forceinline__ int64_t q8_v(int Hkv, int hd, int kvh, int slot, int dim) { return (int64_t)Hkv * 16 * hd + ((int64_t)kvh * hd + dim) * 16 + slot; }

// 2^e as a float, e in -126 .. 127; the mark of a vector that is not finite gives NaN.
__device__ __forceinline__ float q8_unit(int e) { return e == Q8_NAN ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(e + 127) << 23); }

// Exponent of a vector whose largest |x| has these upper 32 bits as a double (sign cleared): Q8_NAN where that is not a finite float32.
__device__ __forceinline__ int q8_exponent(uint32_t top) {
    const int e = (int)(top >> 20) - 1023;
    return e > 127 ? Q8_NAN : max(e - 6, -126);
}
// The same of floats' bits: only the exponent counts, and subnormals' would be below -126.
__device__ __forceinline__ int q8_exponent32(uint32_t top) {
    const int e = (int)(top >> 23) - 127;
    return e > 127 ? Q8_NAN : max(e - 6, -126);
}
// Codes of eight floats under their exponents, packed.  x 2^-e is exact; adding 1.5 2^23 leaves its nearest whole number (ties to even) in the low bits.
__device__ __forceinline__ uint2 q8_codes8(const float (&x)[8], const int (&e)[8]) {
    uint32_t n[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float u = __uint_as_float((uint32_t)(127 - e[i]) << 23);
        const float c = fminf(fmaxf(x[i] * u, -127.f), 127.f) + 12582912.f;
        n[i] = e[i] == Q8_NAN ? 0u : __float_as_uint(c) & 255u;
    }
    return make_uint2(n[0] | n[1] << 8 | n[2] << 16 | n[3] << 24, n[4] | n[5] << 8 | n[6] << 16 | n[7] << 24);
}

// Code of x under exponent e.
__device__ __forceinline__ int8_t q8_code(double x, int e) {
    if (e == Q8_NAN) return 0;
    const double u = __longlong_as_double((long long)(1023 - e) << 52);
    return (int8_t)(int)fmin(fmax(rint(x * u), -127.0), 127.0);
}

// What the attention kernels are given.
struct Q8Attention {
    const float *q;
    int q_stride;
    const int8_t *codes, *expo;
    const int32_t *table;
    int table_stride, H, Hkv, window;
    float softcap;
    const float *slopes;
    float *out;
};

// A launch has fewer than 2^32 threads in a dimension.
inline bool too_large(int64_t workgroups, int threads) { return workgroups > UINT32_MAX / threads; }

inline bool bad_attention(const Q8Attention &a, int hd) {
    return !a.q || !a.codes || !a.expo || (((uintptr_t)a.codes | (uintptr_t)a.expo) & 15) || !a.table || a.table_stride < 0 || a.H <= 0 || a.Hkv <= 0 ||
           a.H % a.Hkv || (hd != 64 && hd != 128) || (int64_t)a.q_stride < (int64_t)a.H * hd || a.window < 0 || !(a.softcap >= 0.f) ||
           !std::isfinite(a.softcap) || (a.softcap > 0.f && a.softcap < 1e-30f) || !a.out;      // 1 / cap, times a score of zero
}

// cap tanh(s / cap).  |s| below cap / 2: an odd polynomial of the ninth degree, its coefficients fitted so that the largest error there relative to tanh is as small
// as it gets (1.5e-8; 9.5e-8 with the roundings of float32.  The series needs the 13th power for that: 1.3e-7, and two instructions an entry more); above, by the
// exponential, which would cancel below.
constexpr float Q8_SERIES = 0.5f;
__device__ __forceinline__ float q8_cap_small(float s, float inv_cap) {
    const float x = s * inv_cap, x2 = x * x;
    return s * (1.f + x2 * (-0.333331435918808f + x2 * (0.13325878977775574f + x2 * (-0.053045500069856644f + x2 * 0.01724150963127613f))));
}
__device__ __forceinline__ float q8_cap(float s, float cap, float inv_cap) {
    const float x = fabsf(s) * inv_cap, t = fast_exp2(-2.8853900817779268f * x);
    return x < Q8_SERIES ? q8_cap_small(s, inv_cap) : copysignf(cap * ((1.f - t) * __builtin_amdgcn_rcpf(1.f + t)), s);
}

typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float float4_u __attribute__((ext_vector_type(4), aligned(4)));      // four floats at any float's address
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// The larger of a lane's number and its partner's, 32 or 16 lanes away; the largest of 16 lanes.  Vector instructions: no way through LDS.
__device__ __forceinline__ float max_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_quarters(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
#define LD_ROR(X_, N_) __builtin_amdgcn_update_dpp(0, X_, 0x120 + N_, 0xf, 0xf, true)      // X_ of the lane N_ on, within 16
__device__ __forceinline__ float max_of16(float x) {
    x = fmaxf(x, __int_as_float(LD_ROR(__float_as_int(x), 8)));
    x = fmaxf(x, __int_as_float(LD_ROR(__float_as_int(x), 4)));
    x = fmaxf(x, __int_as_float(LD_ROR(__float_as_int(x), 2)));
    return fmaxf(x, __int_as_float(LD_ROR(__float_as_int(x), 1)));
}
__device__ __forceinline__ int wave_max(int x) {
    x = max(x, LD_ROR(x, 8));
    x = max(x, LD_ROR(x, 4));
    x = max(x, LD_ROR(x, 2));
    x = max(x, LD_ROR(x, 1));
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((int)r[0], (int)r[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return __builtin_amdgcn_readfirstlane(max((int)q[0], (int)q[1]));
}

// Eight codes (two words) as fp16, exact: a byte c + 128 under the exponent of 1024 is the fp16 number 1152 + c.
__device__ __forceinline__ f16x8_t q8_halves(uint32_t w0, uint32_t w1) {
    const f16x2_t bias = {(_Float16)1152.f, (_Float16)1152.f};
    const uint32_t a = w0 ^ 0x80808080u, b = w1 ^ 0x80808080u;
    f16x2_t h[4];
    h[0] = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - bias;
    h[1] = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - bias;
    h[2] = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - bias;
    h[3] = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - bias;
    return (f16x8_t){h[0][0], h[0][1], h[1][0], h[1][1], h[2][0], h[2][1], h[3][0], h[3][1]};
}

// a and b as sums of two fp16 numbers each (22 bits), packed in pairs: four instructions (the compiler's own way takes eight).
__device__ __forceinline__ void split2_halves(float a, float b, uint32_t &hi, uint32_t &lo) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    hi = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, f16x2_t));
    float x, y;
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(x) : "v"(hi), "v"(a));
    asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(hi), "v"(b));
    lo = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){x, y}, f16x2_t));
}

// A query as whole numbers n = round(8355711 q / max |q|), three base-256 digits from -128 .. 127 each: q = n unit 2^exp, |n - exact| <= 1/2.
struct Q8Query {
    double scale;      // 8355711 / max |q|, 0 for a query that is zero or not finite
    float unit;        // in 1 .. 2; NaN for a query that is not finite
    int exp;
};
// top: the bits of max |q| (which order as the numbers do; above infinity's: a NaN).  factor: what scores are multiplied by besides.
__device__ __forceinline__ Q8Query q8_query(uint32_t top, double factor) {
    Q8Query r{0.0, 1.f, 0};
    if (top >= 0x7f800000u) {
        r.unit = __uint_as_float(0x7fc00000u);
    } else if (top) {
        const double most = (double)__uint_as_float(top);
        r.scale = 8355711.0 / most;
        const double u = most * factor * (1.0 / 8355711.0);
        r.exp = (int)((__double2hiint(u) >> 20) & 0x7ff) - 1023;
        r.unit = (float)__longlong_as_double((__double_as_longlong(u) & 0xfffffffffffffll) | 0x3ff0000000000000ll);
    }
    return r;
}
// Digit 2 (of 65536), 1 (of 256) or 0.
__device__ __forceinline__ int q8_digit(float q, double scale, int digit) {
    int n = (int)rint(q * scale);
    if (scale == 0.0) n = 0;
    const int d0 = (int8_t)n, n1 = (n - d0) >> 8, d1 = (int8_t)n1, d2 = (n1 - d1) >> 8;
    return digit == 2 ? d2 : digit == 1 ? d1 : d0;
}

}  // namespace ldd
