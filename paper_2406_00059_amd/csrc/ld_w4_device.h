// Device code that the kernels of 4-bit linear layers share (see ld_w4.hip).
#pragma once
#include "ld_w4.h"
#include "ld_device.h"

namespace ldw {

using namespace ldd;

typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Sum over 8, 16 or 32 neighbouring lanes, maximum over 32, in all of them: exchanges within the row of 16 lanes, then of whole rows.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
template <typename F> __device__ __forceinline__ float other_row(float v, F f) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float lanes_sum(float v, int lanes) {
    v += dpp<0xb1>(v);       // quads: 1 0 3 2
    v += dpp<0x4e>(v);       // quads: 2 3 0 1
    v += dpp<0x141>(v);      // mirrored halves of a row
    if (lanes > 8) v += dpp<0x140>(v);      // mirrored rows
    if (lanes > 16) v = other_row(v, [](float a, float b) { return a + b; });
    return v;
}
__device__ __forceinline__ float max_of_32(float v) {
    v = fmaxf(v, dpp<0xb1>(v));
    v = fmaxf(v, dpp<0x4e>(v));
    v = fmaxf(v, dpp<0x141>(v));
    v = fmaxf(v, dpp<0x140>(v));
    return other_row(v, [](float a, float b) { return fmaxf(a, b); });
}

// The other half's value, for one that is the same in the 32 lanes of each.
__device__ __forceinline__ float swapped_half(float v) {
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return threadIdx.x & 32 ? __uint_as_float(a[0]) : __uint_as_float(a[1]);
}

// The power of two that brings a row whose largest magnitude is m to 2^14 .. 2^15 (0 for a row of zeros, or one that is not finite).
__device__ __forceinline__ int row_exponent(float m) { return m < INFINITY && m > 0.f ? 14 - ilogbf(m) : 0; }

// Columns c .. c + 3 of a row (c a multiple of 4; the 32 lanes of a half wave hold 128 columns), scaled by 2^k, as two fp16 terms:
// put(c, hi, lo), and the sums of a group of G columns: put_sums(group, hi, lo), by one lane each, of the terms as they are stored, so that a column
// whose code is the zero point leaves nothing behind.  SUBNORMAL: for codes_as_subnormals, the sums 2^-24 times as large.
template <bool SUBNORMAL, typename Put, typename Sums>
__device__ __forceinline__ void split4(float (&v)[4], int k, int c, int G, Put put, Sums put_sums) {
    float sum_hi = 0.f, sum_lo = 0.f, most = 0.f;
    union { _Float16 h[4]; uint2 u; } hi, lo;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        v[e] = ldexpf(v[e], k);
        most = fmaxf(most, fabsf(v[e]));
    }
    most = max_of_32(most);      // 128 columns
    // quantum: 2^-12 of the power of two at or below the largest magnitude, as its bits; at least fp16's least subnormal
    const float quantum = __uint_as_float(max((int)(__float_as_uint(most) & 0x7f800000u) - (12 << 23), (127 - 24) << 23));
    const float per_quantum = __uint_as_float((254u << 23) - __float_as_uint(quantum));      // its reciprocal
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const float f = SUBNORMAL && e >= 2 ? 0.0625f : 1.f;      // e >= 2: codes in bits 4 .. 7
        hi.h[e] = (_Float16)(rintf(v[e] * per_quantum) * quantum * f);
        const float h = (float)hi.h[e] / f;
        lo.h[e] = (_Float16)((v[e] - h) * f);
        sum_hi += h;
        sum_lo += (float)lo.h[e] / f;
    }
    put(c, hi.u, lo.u);
    sum_hi = lanes_sum(sum_hi, G / 4);
    sum_lo = lanes_sum(sum_lo, G / 4);
    if (c % G == 0) put_sums(c / G, SUBNORMAL ? ldexpf(sum_hi, -24) : sum_hi, SUBNORMAL ? ldexpf(sum_lo, -24) : sum_lo);
}

// A word's codes as eight fp16 operands: 2^-24 c and 2^-20 c, a mask each ..
__device__ __forceinline__ f16x8 codes_as_subnormals(uint32_t w) {
    const uint32_t s = w >> 8;
    return __builtin_bit_cast(f16x8, (u32x4){w & 0x000f000fu, w & 0x00f000f0u, s & 0x000f000fu, s & 0x00f000f0u});
}
// .. and c - z, under the exponents of 1024 + c and 1024 + 16 c (all steps exact).  z: 1024 + z in both halves.
__device__ __forceinline__ f16x8 codes_less(uint32_t w, uint32_t z) {
    typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
    const uint32_t s = w >> 8, one = 0x64006400u;
    const f16x2 z0 = __builtin_bit_cast(f16x2, z), z1 = (f16x2){960.f16, 960.f16} - z0;
    auto low = [&](uint32_t v) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, v) - z0); };
    auto high = [&](uint32_t v) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(__builtin_bit_cast(f16x2, v), (f16x2){0.0625f16, 0.0625f16}, z1));
    };
    auto pick = [&](uint32_t v, uint32_t mask) {      // in one instruction, which takes one scalar operand
        uint32_t r;
#if defined(__HIP_DEVICE_COMPILE__)
        asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(v), "s"(mask), "v"(one));
#else
        r = (v & mask) | one;
#endif
        return r;
    };
    return __builtin_bit_cast(f16x8, (u32x4){low(pick(w, 0x000f000fu)), high(pick(w, 0x00f000f0u)), low(pick(s, 0x000f000fu)), high(pick(s, 0x00f000f0u))});
}

// What a wave reads of a tile of 16 rows x 128 columns: its codes, the scales of its lanes' four rows, the zero points.
template <int PER, typename ST, bool ZEROS>
struct CodeTile {
    u32x4 code;
    uint32_t scale[PER][sizeof(ST)], zero[ZEROS ? PER : 1];
    __device__ __forceinline__ void load(const ld::W4Image &w, int64_t tile, int kt, int lane) {
        code = load_stream16(w.codes + ((tile * w.k_tiles + kt) * 64 + lane) * 4);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            const int64_t at = (tile * w.groups + (int64_t)kt * PER + p) * 16 + 4 * (lane >> 4);
            if constexpr (sizeof(ST) == 2) {
                const uint2 v = *reinterpret_cast<const uint2 *>((const bf16_t *)w.scales + at);
                scale[p][0] = v.x; scale[p][1] = v.y;
            } else {
                const uint4 v = *reinterpret_cast<const uint4 *>((const float *)w.scales + at);
                scale[p][0] = v.x; scale[p][1] = v.y; scale[p][2] = v.z; scale[p][3] = v.w;
            }
            if constexpr (ZEROS) zero[p] = *reinterpret_cast<const uint32_t *>(w.zeros + at);
        }
    }
    __device__ __forceinline__ float s(int p, int e) const {
        if constexpr (sizeof(ST) == 4) return __uint_as_float(scale[p][e]);
        else return __uint_as_float((e & 1) ? scale[p][e >> 1] & 0xffff0000u : scale[p][e >> 1] << 16);
    }
    __device__ __forceinline__ float z(int p, int e) const {
        if constexpr (ZEROS) return (float)((zero[p] >> (8 * e)) & 255u);
        else return 8.f;
    }
};

}  // namespace ldw
