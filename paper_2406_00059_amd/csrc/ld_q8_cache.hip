// What is written into the 8-bit cache, and positions that move between it and a pool of the model's type.
#include <cmath>
#include "ld_q8.h"

using namespace ldd;

namespace {

// One angle a thread, in float64: positions up to 2^31 times a frequency keep more digits than the float32 result holds.  2048 angles 2.4 us: a launch.
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

// A rotated pair.  Written out, so that both kernels below round alike: with the sum of squares added in one order they give a row the same codes, however many
// rows a call has.  The order: pairs (of a rotation, or neighbours), then pairs of these, and so on.
__device__ __forceinline__ void turn_pair(double &x, double &y, double c, double s) {
    const double first = fma(x, c, -(y * s));
    y = fma(x, s, y * c);
    x = first;
}

// One wave a row and head, two elements a lane: a rotated pair, or two of the rest.  For few rows, where a launch and its chain of loads count (one row of 96
// heads 2.6 us), and for rotated parts that are no multiple of 8.
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
        for (int off = 1; off < 64; off <<= 1) ss += __shfl_xor(ss, off, WAVE);
        const double r = 1.0 / sqrt(ss / HD + a.eps);
        if (live) {
            x *= r * gain[i0];
            y *= r * gain[i1];
        }
    }
    if (turn) {
        const float2 c = reinterpret_cast<const float2 *>(a.cos_sin)[(int64_t)t * (a.rot / 2) + lane];
        turn_pair(x, y, c.x, c.y);
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

// Sixteen rows of a head a workgroup, HD / 8 lanes a row and eight elements a lane: four rotated pairs, or (lanes i >= rot / 8) the elements from 8 i on, of
// the rest.  rot is a multiple of 8.
// Values go through LDS, from which neighbouring lanes write neighbouring positions: a position's values lie 16 bytes apart in the cache, and a store of
// one of them touches a sector for a byte.  Float64 costs nothing that counts: 1056 rows of 120 heads, 98 MB, 23 us (4.2 TB/s; one row and head a wave 46).
template <int HD, bool INTERLEAVED>
__global__ __launch_bounds__(2 * HD) void k_write_rows_q8(WriteArgs a, int T) {
    constexpr int R = 16, LPR = HD / 8;
    __shared__ __attribute__((aligned(8))) uint8_t vt[R][HD + 8];
    __shared__ int64_t at[R];      // the row's block, -1: not stored
    __shared__ int slots[R];
    const int r = threadIdx.x / LPR, i = threadIdx.x % LPR, t = blockIdx.x * R + r, hh = blockIdx.y;
    const bool value = hh >= a.H + a.Hkv, keep = hh >= a.H;
    const int j = value ? hh - a.H - a.Hkv : hh - a.H;
    const int p = t < T ? a.pos[t] : -1;
    const bool live = p >= 0;
    const int half = a.rot / 2;
    const bool turn = !value && (INTERLEAVED ? 8 * i < a.rot : 4 * i < half);
    const int i0 = INTERLEAVED || value || !turn ? 8 * i : 4 * i, i1 = INTERLEAVED || value || !turn ? 8 * i + 4 : half + 4 * i;
    int phys = -1;
    float4_u x0 = {0.f, 0.f, 0.f, 0.f}, x1 = x0;
    float4_u c0 = x0, c1 = x0;
    if (live) {
        const float *row = a.qkv + t * a.qkv_stride + hh * HD;
        x0 = *reinterpret_cast<const float4_u *>(row + i0);
        x1 = *reinterpret_cast<const float4_u *>(row + i1);
        if (turn) {
            const float *cs = a.cos_sin + ((int64_t)t * half + 4 * i) * 2;
            c0 = *reinterpret_cast<const float4_u *>(cs);
            c1 = *reinterpret_cast<const float4_u *>(cs + 4);
        }
        if (keep) {
            const int b = p >> 4, seq = a.seq_slot[t];
            phys = b < a.table_stride && seq >= 0 ? a.table[(int64_t)seq * a.table_stride + b] : -1;
        }
    }
    const int slot = p & 15;
    if (value) {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 4; e++) top = max(top, max(__float_as_uint(x0[e]) & 0x7f800000u, __float_as_uint(x1[e]) & 0x7f800000u));
#pragma unroll
        for (int off = LPR / 2; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
        const int e1 = q8_exponent32(top);
        const float x[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
        const int e[8] = {e1, e1, e1, e1, e1, e1, e1, e1};
        *reinterpret_cast<uint2 *>(&vt[r][8 * i]) = q8_codes8(x, e);
        if (i == 0) {
            at[r] = phys;
            slots[r] = slot;
            if (phys >= 0) a.expo[(((int64_t)phys * 2 + 1) * a.Hkv + j) * 16 + slot] = (int8_t)e1;
        }
        __syncthreads();
        const int vr = threadIdx.x % R;
        const int64_t b = at[vr];
        if (b < 0) return;
        int8_t *dst = a.codes + b * q8_block(a.Hkv, HD) + q8_v(a.Hkv, HD, j, slots[vr], 0);
        for (int d = threadIdx.x / R; d < HD; d += LPR) dst[16 * d] = (int8_t)vt[vr][d];
        return;
    }
    double y[8] = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
    const float *gain = keep ? a.k_gain : a.q_gain;
    if (gain) {
        double p[4];      // squares of floats are exact
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int u = INTERLEAVED || !turn ? 2 * e : e, w = INTERLEAVED || !turn ? 2 * e + 1 : e + 4;
            p[e] = y[u] * y[u] + y[w] * y[w];
        }
        double ss = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) ss += __shfl_xor(ss, off, WAVE);
        const double n = 1.0 / sqrt(ss / HD + a.eps);
#pragma unroll
        for (int e = 0; e < 8; e++) y[e] *= n * gain[(e < 4 ? i0 : i1) + (e & 3)];
    }
    if (turn) {
        const float cs[8] = {c0[0], c0[1], c0[2], c0[3], c1[0], c1[1], c1[2], c1[3]};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int u = INTERLEAVED ? 2 * e : e, w = INTERLEAVED ? 2 * e + 1 : e + 4;
            turn_pair(y[u], y[w], cs[2 * e], cs[2 * e + 1]);
        }
    }
    if (!keep) {
        if (live) {
            float *q = a.q_out + t * a.q_out_stride + hh * HD;
            *reinterpret_cast<float4_u *>(q + i0) = (float4_u){(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
            *reinterpret_cast<float4_u *>(q + i1) = (float4_u){(float)y[4], (float)y[5], (float)y[6], (float)y[7]};
        }
        return;
    }
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) top = max(top, (uint32_t)__double2hiint(y[e]) & 0x7fffffffu);
#pragma unroll
    for (int off = LPR / 2; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
    if (phys < 0) return;
    const int e1 = q8_exponent(top);
    uint32_t n[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < 8; e++) n[e >> 2] |= (uint32_t)(uint8_t)q8_code(y[e], e1) << (8 * (e & 3));
    int8_t *dst = a.codes + phys * q8_block(a.Hkv, HD) + q8_k(HD, j, slot, 0);
    *reinterpret_cast<uint32_t *>(dst + i0) = n[0];
    *reinterpret_cast<uint32_t *>(dst + i1) = n[1];
    if (i == 0) a.expo[((int64_t)phys * 2 * a.Hkv + j) * 16 + slot] = (int8_t)e1;
}

struct MoveArgs {
    const int32_t *table;
    int table_stride;
    const int32_t *q8_table;
    int q8_table_stride;
    const int32_t *ranges;
    int Hkv, max_len;
};

// What a wave moves: block, KV head and keys or values of item number `item` (blocks, then keys and values, then heads: the order of memory); false where
// the range has no such block or one side does not map it.
struct Moved { int64_t full, q8; int j, value, s0, s1; };      // slots s0 .. s1 - 1
__device__ __forceinline__ bool moved_block(const MoveArgs &a, uint32_t item, Moved &m) {
    const int32_t *r = a.ranges + 3 * (int64_t)blockIdx.y;
    const int first = max(r[1], 0);
    const int64_t end = min((int64_t)r[2], (int64_t)r[1] + a.max_len), b = (int64_t)(first >> 4) + item / (uint32_t)(2 * a.Hkv);
    m.s0 = (int)max(first - b * 16, (int64_t)0);
    m.s1 = (int)min(end - b * 16, (int64_t)16);
    if (m.s0 >= m.s1 || r[0] < 0 || b >= a.table_stride || b >= a.q8_table_stride) return false;
    m.full = a.table[(int64_t)r[0] * a.table_stride + b];
    m.q8 = a.q8_table[(int64_t)r[0] * a.q8_table_stride + b];
    const int part = (int)(item % (uint32_t)(2 * a.Hkv));
    m.value = part >= a.Hkv;
    m.j = part - (m.value ? a.Hkv : 0);
    return m.full >= 0 && m.q8 >= 0;
}

// Eight consecutive elements as floats, and back (rounded to nearest; a code times its unit is exact).
__device__ __forceinline__ void put8(bf16_t *p, const float (&v)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
}
__device__ __forceinline__ void put8(float *p, const float (&v)[8]) {
    reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// A wave an item, eight elements a lane and load: of keys HD / 8 lanes a position, of values two lanes a dimension (slots 0 .. 7, 8 .. 15).  The largest
// exponent is the exponent of the largest.  What bounds it is the traffic; whole blocks leave in 8-byte pieces in the order of memory, of others only
// the range's slots.  Eight sequences of 512 - 8192 positions of 40 heads, 1.3 GB each way: 280 us there, 250 back (a position at a time 1193 and 1251).
template <int HD, typename KT>
__device__ __forceinline__ void move_to(const MoveArgs &a, const Moved &m, const KT *__restrict__ pool, int8_t *__restrict__ codes, int8_t *__restrict__ expo) {
    constexpr int N = HD / 32, LPR = HD / 8;      // loads; lanes a key row
    const int lane = threadIdx.x & 63;
    const KT *src = pool + m.full * kv_block_elems(a.Hkv, HD) + ((int64_t)m.value * a.Hkv + m.j) * 16 * HD + 8 * lane;
    int8_t *dst = codes + m.q8 * q8_block(a.Hkv, HD) + ((int64_t)m.value * a.Hkv + m.j) * 16 * HD + 8 * lane;
    int8_t *ex = expo + ((m.q8 * 2 + m.value) * a.Hkv + m.j) * 16;
    float x[N][8];
#pragma unroll
    for (int n = 0; n < N; n++) load8(src + 512 * n, x[n]);
    if (!m.value) {
#pragma unroll
        for (int n = 0; n < N; n++) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) top = max(top, __float_as_uint(x[n][i]) & 0x7f800000u);
#pragma unroll
            for (int off = LPR / 2; off > 0; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, WAVE));
            const int e1 = q8_exponent32(top), slot = (lane + 64 * n) / LPR;
            const int e[8] = {e1, e1, e1, e1, e1, e1, e1, e1};
            if (slot < m.s0 || slot >= m.s1) continue;
            *reinterpret_cast<uint2 *>(dst + 512 * n) = q8_codes8(x[n], e);
            if (lane % LPR == 0) ex[slot] = (int8_t)e1;
        }
        return;
    }
    uint32_t top[8] = {};
#pragma unroll
    for (int i = 0; i < 8; i++) {
#pragma unroll
        for (int n = 0; n < N; n++) top[i] = max(top[i], __float_as_uint(x[n][i]) & 0x7f800000u);
#pragma unroll
        for (int off = 2; off < 64; off <<= 1) top[i] = max(top[i], (uint32_t)__shfl_xor((int)top[i], off, WAVE));
    }
    int e[8];
#pragma unroll
    for (int i = 0; i < 8; i++) e[i] = q8_exponent32(top[i]);
    const int first = 8 * (lane & 1);
#pragma unroll
    for (int n = 0; n < N; n++) {
        const uint2 c = q8_codes8(x[n], e);
        if (m.s0 == 0 && m.s1 == 16) {
            *reinterpret_cast<uint2 *>(dst + 512 * n) = c;
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (first + i >= m.s0 && first + i < m.s1) dst[512 * n + i] = (int8_t)((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
        }
    }
    if (lane < 2) {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (first + i >= m.s0 && first + i < m.s1) ex[first + i] = (int8_t)e[i];
    }
}

template <int HD, typename KT>
__device__ __forceinline__ void move_from(const MoveArgs &a, const Moved &m, const int8_t *__restrict__ codes, const int8_t *__restrict__ expo, KT *__restrict__ pool) {
    constexpr int N = HD / 32, LPR = HD / 8;
    const int lane = threadIdx.x & 63;
    const int8_t *src = codes + m.q8 * q8_block(a.Hkv, HD) + ((int64_t)m.value * a.Hkv + m.j) * 16 * HD + 8 * lane;
    const int8_t *ex = expo + ((m.q8 * 2 + m.value) * a.Hkv + m.j) * 16;
    KT *dst = pool + m.full * kv_block_elems(a.Hkv, HD) + ((int64_t)m.value * a.Hkv + m.j) * 16 * HD + 8 * lane;
    const int first = 8 * (lane & 1);
    uint2 c[N];
#pragma unroll
    for (int n = 0; n < N; n++) c[n] = *reinterpret_cast<const uint2 *>(src + 512 * n);
    const uint2 ev = *reinterpret_cast<const uint2 *>(ex + first);
#pragma unroll
    for (int n = 0; n < N; n++) {
        const int slot = (lane + 64 * n) / LPR;      // of keys
        const float one = m.value ? 0.f : q8_unit(ex[slot]);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int code = (int)(int8_t)((i < 4 ? c[n].x : c[n].y) >> (8 * (i & 3))), e = (int)(int8_t)((i < 4 ? ev.x : ev.y) >> (8 * (i & 3)));
            v[i] = (float)code * (m.value ? q8_unit(e) : one);
        }
        if (m.value ? m.s0 == 0 && m.s1 == 16 : slot >= m.s0 && slot < m.s1) {
            put8(dst + 512 * n, v);
        } else if (m.value) {
#pragma unroll
            for (int i = 0; i < 8; i++)
                if (first + i >= m.s0 && first + i < m.s1) store_elem(dst + 512 * n + i, v[i]);
        }
    }
}

template <int HD, typename KT, bool TO>
__global__ __launch_bounds__(256) void k_move_q8(MoveArgs a, uint32_t items, KT *__restrict__ pool, int8_t *__restrict__ codes, int8_t *__restrict__ expo) {
    const uint32_t item = blockIdx.x * 4u + (threadIdx.x >> 6);
    Moved m;
    if (item >= items || !moved_block(a, item, m)) return;
    if constexpr (TO) move_to<HD, KT>(a, m, pool, codes, expo);
    else move_from<HD, KT>(a, m, codes, expo, pool);
}

template <bool TO>
ld_status move(const char *what, const MoveArgs &a, int n_ranges, int hd, void *pool, int dtype, int8_t *codes, int8_t *expo, hipStream_t s) {
    const int64_t items = (((int64_t)a.max_len + 14) / 16 + 1) * 2 * a.Hkv;      // positions first .. first + max_len - 1 touch at most so many blocks
    if (too_large((items + 3) / 4, 256)) {
        ld::set_error("%s: too many blocks a range", what);
        return LD_E_RANGE;
    }
    const dim3 grid((unsigned)((items + 3) / 4), n_ranges), block(256);
#define LD_MOVE(HD_, KT_) LD_LAUNCH((k_move_q8<HD_, KT_, TO>), grid, block, 0, s, a, (uint32_t)items, (KT_ *)pool, codes, expo)
    if (dtype == LD_BF16) { if (hd == 128) LD_MOVE(128, bf16_t); else LD_MOVE(64, bf16_t); }
    else { if (hd == 128) LD_MOVE(128, float); else LD_MOVE(64, float); }
#undef LD_MOVE
    return launched("k_move_q8");
}

// From so many rows on sixteen rows a workgroup.  us, one row and head a wave / sixteen rows, 32 + 32 heads: rows of as many sequences 16 3.0 / 3.6, 32 3.5 / 3.8,
// 64 4.7 / 4.4; of one chunk 16 3.0 / 2.9, 32 3.5 / 3.1, 64 4.5 / 3.3, 256 10.7 / 5.4.
constexpr int MANY_ROWS = 48;

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
    if (too_large((n + 63) / 64, 64)) return ld::fail(LD_E_RANGE, "ldk_rope_table_scaled: too many angles");
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
    const bool many = T >= MANY_ROWS && rot % 8 == 0;
    if (H + 2 * (int64_t)Hkv > 65535 || (many ? too_large(((int64_t)T + 15) / 16, 2 * hd) : too_large(T, 64)))
        return ld::fail(LD_E_RANGE, "ldk_rope_kv_write_q8: more than 65535 heads, or too many rows");
    const WriteArgs a{qkv, qkv_stride, q_gain, k_gain, eps, cos_sin, rot, pos, seq_slot, table, table_stride, codes, expo, H, Hkv, q_out, q_out_stride};
    hipStream_t s = (hipStream_t)stream;
    if (many) {
        const dim3 grid((unsigned)(((int64_t)T + 15) / 16), H + 2 * Hkv), block(2 * hd);
#define LD_ROWS(HD_, IL_) LD_LAUNCH((k_write_rows_q8<HD_, IL_>), grid, block, 0, s, a, T)
        if (hd == 128) { if (interleaved) LD_ROWS(128, true); else LD_ROWS(128, false); }
        else { if (interleaved) LD_ROWS(64, true); else LD_ROWS(64, false); }
#undef LD_ROWS
        return launched("k_write_rows_q8");
    }
    const dim3 grid(T, H + 2 * Hkv), block(64);
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
    return move<true>("ldk_kv_to_q8", a, n_ranges, hd, const_cast<void *>(pool_layer), dtype, codes, expo, (hipStream_t)stream);
}

ld_status ldk_kv_from_q8(const int8_t *codes, const int8_t *expo, const int32_t *q8_table, int32_t q8_table_stride, void *pool_layer, int32_t dtype,
                         const int32_t *table, int32_t table_stride, const int32_t *ranges, int32_t n_ranges, int32_t max_len, int32_t Hkv,
                         int32_t hd, void *stream) {
    if (n_ranges == 0 || max_len == 0) return LD_OK;
    const MoveArgs a{table, table_stride, q8_table, q8_table_stride, ranges, Hkv, max_len};
    if (const ld_status bad = check_move("ldk_kv_from_q8", pool_layer, dtype, a, codes, expo, n_ranges, hd)) return bad;
    return move<false>("ldk_kv_from_q8", a, n_ranges, hd, pool_layer, dtype, const_cast<int8_t *>(codes), const_cast<int8_t *>(expo), (hipStream_t)stream);
}

}  // extern "C"
