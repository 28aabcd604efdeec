// The 8-bit cache: layout of a layer, and what its kernels share.
#pragma once
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

// cap tanh(s / cap).  Small arguments by the odd series (next term 2e-9 of the sum at 0.25), the others by the exponential, which would
// cancel there.
__device__ __forceinline__ float q8_cap(float s, float cap, float inv_cap) {
    const float x = fabsf(s) * inv_cap, x2 = x * x;
    const float series = x * (1.f + x2 * (-1.f / 3 + x2 * (2.f / 15 + x2 * (-17.f / 315 + x2 * (62.f / 2835)))));
    const float t = fast_exp2(-2.8853900817779268f * x);
    return copysignf(cap * (x < 0.25f ? series : (1.f - t) / (1.f + t)), s);
}

}  // namespace ldd
