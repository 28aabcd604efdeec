// Attention over the 8-bit cache, one row and head a wave: a position a lane for the scores, a dimension a lane for the sums.
#include <cmath>
#include "ld_q8.h"

using namespace ldd;

namespace {

// Row `row` of q and out at position p over positions lo .. hi of the sequence whose block-table row is trow.
template <int HD>
__device__ void attend(const Q8Attention &a, int row, int h, int p, int lo, int hi, const int32_t *trow, float *qs, float *ws) {
    const int lane = threadIdx.x, j = h / (a.H / a.Hkv);
    const float scale = 1.f / sqrtf((float)HD), slope = a.slopes ? a.slopes[h] : 0.f, inv_cap = a.softcap > 0.f ? 1.f / a.softcap : 0.f;
    constexpr int N = HD / 64;
    for (int u = 0; u < N; u++) qs[lane + 64 * u] = a.q[(int64_t)row * a.q_stride + h * HD + lane + 64 * u];
    __syncthreads();
    float m = -INFINITY, l = 0.f, o[N] = {};
    for (int base = lo & ~63; base <= hi; base += 64) {
        const int at = base + lane, b = at >> 4;
        const int phys = b < a.table_stride ? trow[b] : -1;
        const bool seen = at >= lo && at <= hi && phys >= 0;
        float s = -INFINITY, unit = 0.f;
        if (seen) {
            const int8_t *k = a.codes + phys * q8_block(a.Hkv, HD) + q8_k(HD, j, at & 15, 0);
            const int8_t *e = a.expo + ((int64_t)phys * 2 * a.Hkv + j) * 16 + (at & 15);
            float dot = 0.f;
            for (int d = 0; d < HD; d++) dot += qs[d] * k[d];
            s = dot * scale * q8_unit(*e);
            unit = q8_unit(e[a.Hkv * 16]);
            if (a.softcap > 0.f) s = q8_cap(s, a.softcap, inv_cap);
            s += slope * (at - p);
        }
        float top = s;
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, WAVE));
        const float M = fmaxf(m, top);
        const float w = seen ? fast_exp2((s - (M > -INFINITY ? M : 0.f)) * 1.4426950408889634f) : 0.f;
        const float keep = m > -INFINITY ? fast_exp2((m - M) * 1.4426950408889634f) : 0.f;
        l = l * keep + wave_sum(w);
        m = M;
        __syncthreads();
        ws[lane] = seen ? w * unit : 0.f;
        __syncthreads();
        for (int u = 0; u < N; u++) {
            o[u] *= keep;
            for (int c = 0; c < 4; c++) {
                const int bb = (base >> 4) + c;
                const int ph = bb < a.table_stride && bb * 16 <= hi ? trow[bb] : -1;
                if (ph < 0) continue;
                const int8_t *v = a.codes + ph * q8_block(a.Hkv, HD) + q8_v(a.Hkv, HD, j, 0, lane + 64 * u);
                for (int i = 0; i < 16; i++) o[u] += ws[16 * c + i] * v[i];
            }
        }
    }
    for (int u = 0; u < N; u++) a.out[((int64_t)row * a.H + h) * HD + lane + 64 * u] = l == 0.f ? 0.f : o[u] / l;
}

template <int HD>
__global__ __launch_bounds__(64) void k_prefill_q8(Q8Attention a, const int32_t *tiles, int max_pos) {
    __shared__ float qs[HD], ws[64];
    const int32_t *tile = tiles + 6 * blockIdx.x;
    const int h = blockIdx.y, r = blockIdx.z;
    if (r >= tile[1]) return;
    const int p = tile[2] + r;
    const int lo = max(max(tile[4], a.window > 0 ? p - a.window + 1 : 0), 0);
    attend<HD>(a, tile[0] + r, h, p, lo, min(max(p, tile[5] - 1), max_pos), a.table + (int64_t)tile[3] * a.table_stride, qs, ws);
}

}  // namespace

extern "C" {

size_t ldk_prefill_attention_q8_scratch_bytes(int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t max_pos, int32_t window) { return 0; }

ld_status ldk_prefill_attention_q8(const float *q, int32_t q_stride, const int8_t *codes, const int8_t *expo, const int32_t *table,
                                   int32_t table_stride, const int32_t *tiles, int32_t n_tiles, int32_t H, int32_t Hkv, int32_t hd, int32_t window,
                                   float softcap, const float *slopes, int32_t max_pos, float *out, void *scratch, size_t scratch_bytes,
                                   void *stream) {
    if (n_tiles == 0) return LD_OK;
    const Q8Attention a{q, q_stride, codes, expo, table, table_stride, H, Hkv, window, softcap, slopes, out};
    if (n_tiles < 0 || max_pos < 0 || !tiles || bad_attention(a, hd))
        return ld::fail(LD_E_INVAL, "ldk_prefill_attention_q8: bad argument");
    if (H > 65535) return ld::fail(LD_E_RANGE, "ldk_prefill_attention_q8: more than 65535 heads");
    hipStream_t s = (hipStream_t)stream;
    if (hd == 128) LD_LAUNCH(k_prefill_q8<128>, dim3(n_tiles, H, 128), dim3(64), 0, s, a, tiles, max_pos);
    else LD_LAUNCH(k_prefill_q8<64>, dim3(n_tiles, H, 128), dim3(64), 0, s, a, tiles, max_pos);
    return launched("k_prefill_q8");
}

}  // extern "C"
