// Token choice under rules: penalties for repeated tokens, biases, a grammar's mask, then the arg-max or a draw.
//
// A workgroup takes a slice of one row's vocabulary.  It counts the history's tokens that lie in the slice in LDS (integer
// atomics, whose order cannot matter) and notes the last bias entry of each token, walks the slice's logits once, and leaves
// its best token; a second launch joins the slices.  No count table outlives a call: a sequence that is forked, swapped or
// rolled back needs nothing but its token history.  Latency at few rows (the chain of loads, the launch behind: one row of 32000 5.9 + 2 us
// in the two kernels).  32 rows with histories of 512 to 8192 tokens: slices 10.9 us, of which 6.0 remain without any rule, 2 - 3 are the history and up to 1.4
// the noise of a draw; 2.8 the join.
#include "ld_device.h"

#include <algorithm>

using namespace ldd;

namespace {

constexpr int THREADS = 1024, PER = 4;                        // tokens a thread has at once
constexpr int LEAST = 2048, MOST = 8192;                      // tokens of a slice: 16 - 64 KB of LDS
// Slices of a row, of whole thousands of tokens: up to a workgroup for every CU, but none of less than LEAST (one row of 32000: 16).  A history is read
// once a slice.
int slice_tokens(int R, int V) {
    const int64_t want = ((int64_t)R * V + 255) / 256;
    return (int)std::min<int64_t>(MOST, std::max<int64_t>(LEAST, (want + 1023) / 1024 * 1024));
}
int slices_of(int R, int V) { const int s = slice_tokens(R, V); return (V + s - 1) / s; }
constexpr uint32_t SEEN = 0x80000000u;
constexpr int MOST_TOKENS = 1 << 30;

struct Best { float v; int i; };
// The larger score, the lower index among equal ones; i < 0: nothing yet.
__device__ __forceinline__ void better(Best &a, float v, int i) {
    if (i >= 0 && (a.i < 0 || v > a.v || (v == a.v && i < a.i))) { a.v = v; a.i = i; }
}
__device__ __forceinline__ void wave_best(Best &b) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) {
        const float v = __shfl_xor(b.v, off, WAVE);
        const int i = __shfl_xor(b.i, off, WAVE);
        better(b, v, i);
    }
}

__global__ __launch_bounds__(THREADS) void k_choose_slice(const float *logits, int V, int slice, ld_token_rules rules,
                                                          const float *__restrict__ temperature, const uint64_t *__restrict__ seed,
                                                          const int32_t *__restrict__ pos, float *adjusted, Best *__restrict__ part) {
    extern __shared__ uint32_t sm_tokens[];
    __shared__ Best sm[THREADS / 64];
    uint32_t *seen = sm_tokens;                              // bit 31: in the history; the rest: times in its answer part
    uint32_t *bias_at = sm_tokens + slice;                   // last entry naming the token, + 1
    const int r = blockIdx.y, base = blockIdx.x * slice, tid = threadIdx.x;
    const int size = min(slice, V - base);
    const bool counted = rules.history && rules.penalties, biased = rules.bias != nullptr;
    const float *row = logits + (int64_t)r * V + base;
    // what the walk needs first is asked for first, and its history likewise
    float l[PER];
#pragma unroll
    for (int u = 0; u < PER; u++) l[u] = tid + u * THREADS < size ? row[tid + u * THREADS] : 0.f;
    const int32_t *h = counted ? rules.history + (int64_t)r * rules.history_stride : nullptr;
    const int n = counted ? min(rules.history_len[r], rules.history_stride) : 0, answer = counted && rules.n_prompt ? rules.n_prompt[r] : 0;
    const int b0 = biased ? rules.bias_start[r] : 0, b1 = biased ? rules.bias_start[r + 1] : 0;
    float rep = 1.f, pres = 0.f, freq = 0.f;
    if (counted) { rep = rules.penalties[3 * r]; pres = rules.penalties[3 * r + 1]; freq = rules.penalties[3 * r + 2]; }
    const int mrow = rules.mask ? (rules.mask_row ? rules.mask_row[r] : r) : -1;
    const float temp = temperature ? temperature[r] : 0.f;
    const uint64_t sd = temp > 0.f ? seed[r] : 0, ctr = temp > 0.f ? (uint64_t)pos[r] * (uint64_t)V : 0;
    for (int i = tid; i < slice; i += THREADS) { seen[i] = 0; bias_at[i] = 0; }
    __syncthreads();
    for (int j0 = 0; j0 < n; j0 += 4 * THREADS) {
        uint32_t k[4];
#pragma unroll
        for (int u = 0; u < 4; u++) {
            const int j = j0 + u * THREADS + tid;
            k[u] = j < n ? (uint32_t)h[j] - (uint32_t)base : 0xffffffffu;
        }
#pragma unroll
        for (int u = 0; u < 4; u++)
            if (k[u] < (uint32_t)size) {      // a token outside the vocabulary lies in no slice
                atomicOr(&seen[k[u]], SEEN);
                if (j0 + u * THREADS + tid >= answer) atomicAdd(&seen[k[u]], 1u);
            }
    }
    for (int j = b0 + tid; j < b1; j += THREADS) {
        const uint32_t k = (uint32_t)rules.bias_token[j] - (uint32_t)base;
        if (k < (uint32_t)size) atomicMax(&bias_at[k], (uint32_t)(j - b0 + 1));
    }
    __syncthreads();
    const uint32_t *mask = mrow >= 0 && mrow < rules.mask_rows ? rules.mask + (int64_t)mrow * ((V + 31) / 32) : nullptr;
    const bool nothing = mrow >= 0 && !mask;      // a row of the mask that does not exist allows no token
    const float inv_t = temp > 0.f ? 1.0f / temp : 1.0f;
    Best best{-INFINITY, -1};
    auto take = [&](int k, float l) {
        const int i = base + k;
        const uint32_t c = seen[k];
        if (c) {
            const float n = (float)(c & ~SEEN);
            l = l > 0.f ? l / rep : l * rep;
            l = l - (freq * n + (n > 0.f ? pres : 0.f));
        }
        if (bias_at[k]) l += rules.bias[b0 + (int)bias_at[k] - 1];
        if (nothing || (mask && !((mask[i >> 5] >> (i & 31)) & 1u))) l = -INFINITY;
        if (adjusted) adjusted[(int64_t)r * V + i] = l;
        if (!(l > -INFINITY)) return;      // neither -inf nor NaN
        better(best, temp > 0.f ? l * inv_t + gumbel_noise(sd, ctr + i) : l, i);
    };
#pragma unroll
    for (int u = 0; u < PER; u++)
        if (tid + u * THREADS < size) take(tid + u * THREADS, l[u]);
    for (int k = tid + PER * THREADS; k < size; k += THREADS) take(k, row[k]);
    wave_best(best);
    if ((tid & 63) == 0) sm[tid >> 6] = best;
    __syncthreads();
    if (tid < 64) {
        best = tid < THREADS / 64 ? sm[tid] : Best{-INFINITY, -1};
        wave_best(best);
        if (tid == 0) part[(int64_t)r * gridDim.x + blockIdx.x] = best;
    }
}

__global__ __launch_bounds__(64) void k_choose_join(const Best *__restrict__ part, int slices, int32_t *__restrict__ token) {
    const int r = blockIdx.x;
    Best best{-INFINITY, -1};
    for (int i = threadIdx.x; i < slices; i += 64) {
        const Best b = part[(int64_t)r * slices + i];
        better(best, b.v, b.i);
    }
    wave_best(best);
    if (threadIdx.x == 0) token[r] = best.i;
}

}  // namespace

extern "C" {

size_t ldk_choose_scratch_bytes(int32_t R, int32_t V) {
    return R > 0 && V > 0 && V <= MOST_TOKENS ? (size_t)R * ((V + LEAST - 1) / LEAST) * sizeof(Best) : 0;      // the most slices
}

ld_status ldk_choose(const float *logits, int32_t R, int32_t V, const ld_token_rules *rules, const float *temperature, const uint64_t *seed,
                     const int32_t *pos, float *adjusted, int32_t *token, void *scratch, size_t scratch_bytes, void *stream) {
    if (R == 0) return LD_OK;
    if (!logits || !token || R < 0 || V <= 0 || (temperature && (!seed || !pos)))
        return ld::fail(LD_E_INVAL, "ldk_choose: bad argument (a temperature needs seed and pos)");
    const ld_token_rules none{};
    const ld_token_rules &u = rules ? *rules : none;
    if ((u.history && (!u.history_len || !u.penalties || u.history_stride < 0)) || (u.penalties && !u.history) ||
        (u.bias && (!u.bias_start || !u.bias_token)) || (u.mask && u.mask_rows <= 0) || (u.mask && !u.mask_row && u.mask_rows < R))
        return ld::fail(LD_E_INVAL, "ldk_choose: bad argument (history comes with history_len and penalties, bias with bias_start and "
                                    "bias_token, mask with mask_rows and, unless it has a row for each of the logits', mask_row)");
    if (R > 65535 || V > MOST_TOKENS) return ld::fail(LD_E_RANGE, "ldk_choose: more than 65535 rows or 2^30 tokens");
    if (!scratch || ((uintptr_t)scratch & 7) || scratch_bytes < ldk_choose_scratch_bytes(R, V))
        return ld::fail(LD_E_INVAL, "ldk_choose: scratch missing, not 8-byte aligned or too small");
    const int slice = slice_tokens(R, V), slices = slices_of(R, V);
    hipStream_t s = (hipStream_t)stream;
    LD_LAUNCH(k_choose_slice, dim3(slices, R), dim3(THREADS), (size_t)slice * 8, s, logits, V, slice, u, temperature, seed, pos, adjusted, (Best *)scratch);
    LD_LAUNCH(k_choose_join, dim3(R), dim3(64), 0, s, (const Best *)scratch, slices, token);
    return launched("k_choose");
}

}  // extern "C"
