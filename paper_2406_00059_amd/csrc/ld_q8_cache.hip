// What is written into the 8-bit cache, and positions that move between it and a pool of the model's type.
#include <cmath>
#include "ld_q8.h"

using namespace ldd;

namespace {

// One angle a thread, in float64: positions up to 2^31 times a frequency keep more digits than the float32 result holds.
__global__ void k_rope_table_scaled(const int32_t *__restrict__ pos, int64_t n, int half, double log2_base, double factor, double low, double high, double turns,
                                    double attention, float2 *__restrict__ cos_sin) {
    const int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (at >= n) return;
    const int i = (int)(at % half);
    const double f = exp2(-log2_base * i / half);
    const double g = turns > 0 ? fmin(fmax((turns * f - low) / (high - low), 0.0), 1.0) : 0.0;
    double s, c;
    sincos(pos[at / half] * (f * ((1.0 - g) / factor + g)), &s, &c);
    cos_sin[at] = make_float2((float)(attention * c), (float)(attention * s));
}

struct WriteArgs {
    const float *qkv;
    int64_t qkv_stride;
    const float *q_gain, *k_gain;
    double eps;
    const float *cos_sin;
    int rot;
    const int32_t *pos, *seq_slot, *table;
    int table_stride;
    int8_t *codes, *expo;
    int H, Hkv;
    float *q_out;
    int64_t q_out_stride;
};

// One wave a row and head, two elements a lane: a rotated pair, or two of the rest.
template <int HD, bool INTERLEAVED>
__global__ __launch_bounds__(64) void k_write_q8(WriteArgs a) {
    const int t = blockIdx.x, hh = blockIdx.y, lane = threadIdx.x;
    const int p = a.pos[t];
    if (p < 0) return;
    const bool live = lane < HD / 2;
    const int j = hh < a.H ? -1 : hh < a.H + a.Hkv ? hh - a.H : hh - a.H - a.Hkv;      // KV head, or a query head
    const bool value = hh >= a.H + a.Hkv, turn = !value && lane < a.rot / 2;
    const bool apart = turn && !INTERLEAVED;
    const int i0 = apart ? lane : turn || value ? 2 * lane : a.rot + 2 * (lane - a.rot / 2), i1 = apart ? lane + a.rot / 2 : i0 + 1;
    double x = 0, y = 0;
    if (live) {
        const float *row = a.qkv + t * a.qkv_stride + hh * HD;
        x = row[i0];
        y = row[i1];
    }
    const float *gain = value ? nullptr : j < 0 ? a.q_gain : a.k_gain;
    if (gain) {
        double ss = x * x + y * y;
        for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off, WAVE);
        const double r = 1.0 / sqrt(ss / HD + a.eps);
        if (live) {
            x *= r * gain[i0];
            y *= r * gain[i1];
        }
    }
    if (turn) {
        const float2 c = reinterpret_cast<const float2 *>(a.cos_sin)[(int64_t)t * (a.rot / 2) + lane];
        const double u = x * c.x - y * c.y;
        y = x * c.y + y * c.x;
        x = u;
    }
    if (j < 0) {
        if (live) {
            float *q = a.q_out + t * a.q_out_stride + hh * HD;
            q[i0] = (float)x;
            q[i1] = (float)y;
        }
        return;
    }
    const int slot = p & 15, b = p >> 4, seq = a.seq_slot[t];
    const int phys = b < a.table_stride && seq >= 0 ? a.table[(int64_t)seq * a.table_stride + b] : -1;
    if (phys < 0) return;
    uint32_t top = max((uint32_t)__double2hiint(x) & 0x7fffffffu, (uint32_t)__double2hiint(y) & 0x7fffffffu);
    for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
    const int e = q8_exponent(top);
    int8_t *blk = a.codes + phys * q8_block(a.Hkv, HD);
    if (live) {
        blk[value ? q8_v(a.Hkv, HD, j, slot, i0) : q8_k(HD, j, slot, i0)] = q8_code(x, e);
        blk[value ? q8_v(a.Hkv, HD, j, slot, i1) : q8_k(HD, j, slot, i1)] = q8_code(y, e);
    }
    if (lane == 0) a.expo[(((int64_t)phys * 2 + value) * a.Hkv + j) * 16 + slot] = (int8_t)e;
}

struct MoveArgs {
    const int32_t *table;
    int table_stride;
    const int32_t *q8_table;
    int q8_table_stride;
    const int32_t *ranges;
    int Hkv, max_len;
};

// Blocks of a range: logical block blockIdx.x of it, in both caches, and the slots [s0, s1) that it moves; false where there are none.
__device__ __forceinline__ bool move_block(const MoveArgs &a, int64_t &full, int64_t &q8, int &s0, int &s1) {
    const int32_t *r = a.ranges + 3 * blockIdx.y;
    const int first = max(r[1], 0);
    const int64_t end = min((int64_t)r[2], (int64_t)r[1] + a.max_len);
    const int b = (first >> 4) + blockIdx.x;
    s0 = max(first - b * 16, 0);
    s1 = (int)min(end - (int64_t)b * 16, (int64_t)16);
    if (s0 >= s1 || r[0] < 0 || b >= a.table_stride || b >= a.q8_table_stride) return false;
    full = a.table[(int64_t)r[0] * a.table_stride + b];
    q8 = a.q8_table[(int64_t)r[0] * a.q8_table_stride + b];
    return full >= 0 && q8 >= 0;
}

__device__ __forceinline__ float elem(const float *p) { return *p; }
__device__ __forceinline__ float elem(const bf16_t *p) { return bf16_to_f32(*p); }

// One wave a block, head, and keys or values; a position at a time.
template <int HD, typename KT>
__global__ __launch_bounds__(64) void k_to_q8(MoveArgs a, const KT *__restrict__ pool, int8_t *__restrict__ codes, int8_t *__restrict__ expo) {
    int64_t full, q8;
    int s0, s1;
    if (!move_block(a, full, q8, s0, s1)) return;
    const int j = blockIdx.z >> 1, value = blockIdx.z & 1, lane = threadIdx.x;
    const KT *src = pool + full * kv_block_elems(a.Hkv, HD);
    int8_t *dst = codes + q8 * q8_block(a.Hkv, HD);
    for (int s = s0; s < s1; s++) {
        float x[HD / 64];
        uint32_t top = 0;
        for (int u = 0; u < HD / 64; u++) {
            const int d = lane + 64 * u;
            x[u] = elem(src + (value ? kv_v_offset(a.Hkv, HD, j, s, d) : kv_k_offset(HD, j, s, d)));
            top = max(top, (uint32_t)__double2hiint((double)x[u]) & 0x7fffffffu);
        }
        for (int off = 32; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
        const int e = q8_exponent(top);
        for (int u = 0; u < HD / 64; u++) {
            const int d = lane + 64 * u;
            dst[value ? q8_v(a.Hkv, HD, j, s, d) : q8_k(HD, j, s, d)] = q8_code(x[u], e);
        }
        if (lane == 0) expo[((q8 * 2 + value) * a.Hkv + j) * 16 + s] = (int8_t)e;
    }
}

template <int HD, typename KT>
__global__ __launch_bounds__(64) void k_from_q8(MoveArgs a, const int8_t *__restrict__ codes, const int8_t *__restrict__ expo, KT *__restrict__ pool) {
    int64_t full, q8;
    int s0, s1;
    if (!move_block(a, full, q8, s0, s1)) return;
    const int j = blockIdx.z >> 1, value = blockIdx.z & 1, lane = threadIdx.x;
    const int8_t *src = codes + q8 * q8_block(a.Hkv, HD);
    KT *dst = pool + full * kv_block_elems(a.Hkv, HD);
    for (int s = s0; s < s1; s++) {
        const float unit = q8_unit(expo[((q8 * 2 + value) * a.Hkv + j) * 16 + s]);
        for (int u = 0; u < HD / 64; u++) {
            const int d = lane + 64 * u;
            store_elem(dst + (value ? kv_v_offset(a.Hkv, HD, j, s, d) : kv_k_offset(HD, j, s, d)),
                       unit * src[value ? q8_v(a.Hkv, HD, j, s, d) : q8_k(HD, j, s, d)]);
        }
    }
}

bool bad_pool(const void *codes, const void *expo) { return !codes || !expo || (((uintptr_t)codes | (uintptr_t)expo) & 15); }

ld_status check_move(const char *what, const void *pool, int dtype, const MoveArgs &a, const void *codes, const void *expo, int n_ranges, int hd) {
    if (!pool || ((uintptr_t)pool & 15) || bad_pool(codes, expo) || !a.table || !a.q8_table || !a.ranges || n_ranges < 0 || a.max_len < 0 || a.Hkv <= 0 ||
        a.table_stride < 0 || a.q8_table_stride < 0 || (hd != 64 && hd != 128) || (dtype != LD_BF16 && dtype != LD_F32)) {
        ld::set_error("%s: bad argument", what);
        return LD_E_INVAL;
    }
    if (n_ranges > 65535 || a.Hkv > 32767) {
        ld::set_error("%s: more than 65535 ranges or 32767 KV heads", what);
        return LD_E_RANGE;
    }
    return LD_OK;
}

}  // namespace

extern "C" {

ld_status ldk_rope_table_scaled(const int32_t *pos, int32_t T, int32_t rot, float rope_base, const ld_rope_scaling *scaling, float *cos_sin,
                                void *stream) {
    const ld_rope_scaling sc = scaling ? *scaling : ld_rope_scaling{1.f, 0.f, 0.f, 0, 1.f};
    if (T < 0 || rot < 2 || rot % 2 || !(rope_base > 0.f) || !std::isfinite(rope_base) || !(sc.factor > 0.f) || !std::isfinite(sc.factor) ||
        !std::isfinite(sc.attention) || sc.original < 0 ||
        (sc.original > 0 && (!(sc.high > sc.low) || !std::isfinite(sc.low) || !std::isfinite(sc.high))))
        return ld::fail(LD_E_INVAL, "ldk_rope_table_scaled: bad argument");
    if (T == 0) return LD_OK;
    if (!pos || !cos_sin) return ld::fail(LD_E_INVAL, "ldk_rope_table_scaled: bad argument");
    const int64_t n = (int64_t)T * (rot / 2);
    if (n > (int64_t)1 << 38) return ld::fail(LD_E_RANGE, "ldk_rope_table_scaled: too many angles");
    LD_LAUNCH(k_rope_table_scaled, dim3((unsigned)((n + 63) / 64)), dim3(64), 0, (hipStream_t)stream, pos, n, rot / 2, std::log2((double)rope_base),
              (double)sc.factor, (double)sc.low, (double)sc.high, sc.original / (2 * M_PI), (double)sc.attention, reinterpret_cast<float2 *>(cos_sin));
    return launched("k_rope_table_scaled");
}

ld_status ldk_rope_kv_write_q8(const float *qkv, int32_t qkv_stride, const float *q_gain, const float *k_gain, float eps, const float *cos_sin,
                               int32_t rot, int32_t interleaved, const int32_t *pos, const int32_t *seq_slot, const int32_t *table,
                               int32_t table_stride, int8_t *codes, int8_t *expo, int32_t T, int32_t H, int32_t Hkv, int32_t hd, float *q_out,
                               int32_t q_out_stride, void *stream) {
    if (T < 0 || H <= 0 || Hkv <= 0 || H % Hkv || (hd != 64 && hd != 128) || rot < 0 || rot > hd || rot % 2 || table_stride < 0 ||
        (int64_t)qkv_stride < ((int64_t)H + 2 * (int64_t)Hkv) * hd || (int64_t)q_out_stride < (int64_t)H * hd ||
        ((q_gain || k_gain) && !(eps >= 0.f && std::isfinite(eps))))
        return ld::fail(LD_E_INVAL, "ldk_rope_kv_write_q8: bad argument");
    if (T == 0) return LD_OK;
    if (!qkv || !pos || !seq_slot || !table || !q_out || (rot && !cos_sin) || bad_pool(codes, expo) || (q_out == qkv && q_out_stride != qkv_stride))
        return ld::fail(LD_E_INVAL, "ldk_rope_kv_write_q8: bad argument");
    if (H + 2 * (int64_t)Hkv > 65535) return ld::fail(LD_E_RANGE, "ldk_rope_kv_write_q8: more than 65535 heads");
    const WriteArgs a{qkv, qkv_stride, q_gain, k_gain, eps, cos_sin, rot, pos, seq_slot, table, table_stride, codes, expo, H, Hkv, q_out, q_out_stride};
    const dim3 grid(T, H + 2 * Hkv), block(64);
    hipStream_t s = (hipStream_t)stream;
    if (hd == 128) { if (interleaved) LD_LAUNCH((k_write_q8<128, true>), grid, block, 0, s, a); else LD_LAUNCH((k_write_q8<128, false>), grid, block, 0, s, a); }
    else { if (interleaved) LD_LAUNCH((k_write_q8<64, true>), grid, block, 0, s, a); else LD_LAUNCH((k_write_q8<64, false>), grid, block, 0, s, a); }
    return launched("k_write_q8");
}

ld_status ldk_kv_to_q8(const void *pool_layer, int32_t dtype, const int32_t *table, int32_t table_stride, int8_t *codes, int8_t *expo,
                       const int32_t *q8_table, int32_t q8_table_stride, const int32_t *ranges, int32_t n_ranges, int32_t max_len, int32_t Hkv,
                       int32_t hd, void *stream) {
    if (n_ranges == 0 || max_len == 0) return LD_OK;
    const MoveArgs a{table, table_stride, q8_table, q8_table_stride, ranges, Hkv, max_len};
    if (const ld_status bad = check_move("ldk_kv_to_q8", pool_layer, dtype, a, codes, expo, n_ranges, hd)) return bad;
    const dim3 grid((unsigned)(((int64_t)max_len + 14) / 16 + 1), n_ranges, 2 * Hkv), block(64);
    hipStream_t s = (hipStream_t)stream;
#define LD_TO(HD_, KT_) LD_LAUNCH((k_to_q8<HD_, KT_>), grid, block, 0, s, a, (const KT_ *)pool_layer, codes, expo)
    if (dtype == LD_BF16) { if (hd == 128) LD_TO(128, bf16_t); else LD_TO(64, bf16_t); }
    else { if (hd == 128) LD_TO(128, float); else LD_TO(64, float); }
#undef LD_TO
    return launched("k_to_q8");
}

ld_status ldk_kv_from_q8(const int8_t *codes, const int8_t *expo, const int32_t *q8_table, int32_t q8_table_stride, void *pool_layer, int32_t dtype,
                         const int32_t *table, int32_t table_stride, const int32_t *ranges, int32_t n_ranges, int32_t max_len, int32_t Hkv,
                         int32_t hd, void *stream) {
    if (n_ranges == 0 || max_len == 0) return LD_OK;
    const MoveArgs a{table, table_stride, q8_table, q8_table_stride, ranges, Hkv, max_len};
    if (const ld_status bad = check_move("ldk_kv_from_q8", pool_layer, dtype, a, codes, expo, n_ranges, hd)) return bad;
    const dim3 grid((unsigned)(((int64_t)max_len + 14) / 16 + 1), n_ranges, 2 * Hkv), block(64);
    hipStream_t s = (hipStream_t)stream;
#define LD_FROM(HD_, KT_) LD_LAUNCH((k_from_q8<HD_, KT_>), grid, block, 0, s, a, codes, expo, (KT_ *)pool_layer)
    if (dtype == LD_BF16) { if (hd == 128) LD_FROM(128, bf16_t); else LD_FROM(64, bf16_t); }
    else { if (hd == 128) LD_FROM(128, float); else LD_FROM(64, float); }
#undef LD_FROM
    return launched("k_from_q8");
}

}  // extern "C"
