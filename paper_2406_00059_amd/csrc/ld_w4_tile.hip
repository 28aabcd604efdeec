// Linear layers on 4-bit weights for many rows: the operands and the arithmetic are those of ld_w4.hip.
//
// A workgroup of four waves multiplies 16 tiles of 16 output rows (SwiGLU: 8 gate tiles and their up tiles) with 16 TT activation
// rows, a wave 4 tiles with all of them.  The activations of 128 columns (8 KB per 16 rows, both terms) are copied straight into
// LDS in operand order, two stages, and every wave reads them all; codes go from memory into registers, a column tile ahead, are
// unpacked once per group and meet TT x 2 operands there.
// Groups of 128 take the codes as subnormals: 80 vector instructions for TT x 32 matrix instructions; what a group's sums owe to the zero
// point 8 enters as the first matrix instruction's addend, and a group costs 2 vector instructions a value (add, multiply-add with the scale).
// Groups of 32 and 64 have that cost four and two times as often, zero points that are given would meet both terms' sums apart (2 more, for they
// have to be taken off the hi sums while those are exact), and little of it runs beside the matrix instructions of the other wave of a
// SIMD here (counters of 4096 x 11008, groups of 32, 257 rows: 47 k cycles a SIMD of vector and 50 k of matrix instructions in 114 k that a CU is
// busy).  These take c - z (64 instructions more a column tile) and add the lo products to the exact sum of the hi products: 1 vector instruction a
// value, no addend to prepare.
// At 1056 rows the matrix cores bound it: 13B gate/up (2 x 13824 x 5120, groups of 128) 497 us, 601 TFLOP/s of the product, two terms executed: 1.2 PFLOP/s
// (a large library product in fp16: 1.1 - 1.5).  4096 x 11008, groups of 32, 257 rows: 72 us with split and join.
#include "ld_w4_device.h"

#include <algorithm>

using namespace ldd;
using namespace ldw;

namespace {

constexpr int NT = 4;      // tiles of 16 output rows a wave

// 1 KB from src + 16 lane into LDS, in lane order.
__device__ __forceinline__ void copy_kb(const char *src, char *dst, int lane) {
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(src + lane * 16),
                                     (__attribute__((address_space(3))) void *)dst, 16, 0, 0);
#endif
}

// Workgroups go to the 8 XCDs in turn.  An XCD takes whole columns of the grid, all rows' blocks of an output block one after
// the other: its 64 workgroups stand at much the same place along K, and its 4 MB of L2 hold what they share there (the codes of some three
// output blocks and the activations of all rows), so that codes leave the memory once and not once a row block.  13B gate/up of 1056 rows:
// 505 us, 632 with workgroups in the grid's order.
__device__ __forceinline__ void block_of(int id, int n_blocks, int t_blocks, int &nb, int &tb) {
    const int whole = n_blocks / 8 * 8;
    if (id < whole * t_blocks) {
        nb = id % 8 + 8 * (id / 8 / t_blocks);
        tb = id / 8 % t_blocks;
    } else {
        nb = whole + (id - whole * t_blocks) / t_blocks;
        tb = (id - whole * t_blocks) % t_blocks;
    }
}

template <int TT, int G, bool ZEROS, typename ST>
__global__ __launch_bounds__(256, 2) void k_w4_tile(ld::W4Image w, ld::W4Rows r, int T, int N, int epilogue, int n_blocks, int t_blocks, int slabs,
                                                    float *__restrict__ y, float *__restrict__ part) {
    constexpr int PER = 128 / G, JG = G / 32;
    constexpr bool SUBNORMAL = ld::w4_subnormal(G, ZEROS);
    __shared__ __attribute__((aligned(16))) char sm_x[2][TT * 8192];
    __shared__ float sm_s[2][SUBNORMAL ? TT * PER * 32 : 1];
    __shared__ __attribute__((aligned(16))) float sm_w[2][PER][256];      // scales
    __shared__ __attribute__((aligned(16))) uint32_t sm_z[2][PER][ZEROS ? 256 : 4];      // zero points: 1024 + z as two fp16
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col = lane & 15, h = lane >> 4;
    const bool pair = epilogue == LDK_SWIGLU;
    const int slab = blockIdx.y;
    int nb, tb;
    block_of(blockIdx.x, n_blocks, t_blocks, nb, tb);
    const int rt_all = (T + 15) >> 4;
    const int k0 = (int)((int64_t)w.k_tiles * slab / slabs), k1 = (int)((int64_t)w.k_tiles * (slab + 1) / slabs);
    // this wave's tiles: pairs: gate 8 nb + 2 wave + (0, 1), then their up tiles; otherwise 16 nb + 4 wave + i
    int tile_of[NT];
    int64_t tile[NT];
#pragma unroll
    for (int i = 0; i < NT; i++) {
        tile_of[i] = pair ? nb * 8 + wave * 2 + (i & 1) : nb * 16 + wave * 4 + i;
        tile[i] = (int64_t)(pair && i >= 2 ? w.row_tiles : 0) + min(tile_of[i], w.row_tiles - 1);
    }
    auto copy_x = [&](int kt, int stage) {
#pragma unroll
        for (int u = 0; u < 2 * TT; u++) {
            const int piece = u * 4 + wave, tt = piece >> 3;      // 8 KB a row tile, 1 KB a copy
            const int64_t rt = min(tb * TT + tt, rt_all - 1);
            copy_kb((const char *)r.image + (rt * w.k_tiles + kt) * 8192 + (piece & 7) * 1024, sm_x[stage] + piece * 1024, lane);
        }
    };
    // What belongs to a column tile beside codes and operands goes through LDS: the sums of the activations, and the scales (and zero points)
    // of 256 output rows, a row a thread.  Nothing else is loaded inside a tile's products, so that no wait there drains the copies.
    constexpr int SUMS = SUBNORMAL ? (TT * PER * 32 + 255) / 256 : 0;
    struct Small { float sum[SUMS ? SUMS : 1]; ST scale[PER]; uint8_t zero[PER]; };
    const int my = threadIdx.x >> 4;      // row tile of the workgroup's 16: wave my / 4, its tile my % 4
    const int64_t my_tile = pair ? (int64_t)((my & 3) >= 2 ? w.row_tiles : 0) + min(nb * 8 + (my >> 2) * 2 + (my & 1), w.row_tiles - 1)
                                 : min(nb * 16 + my, w.row_tiles - 1);
    auto load_small = [&](int kt, Small &v) {
#pragma unroll
        for (int u = 0; u < SUMS; u++) {
            const int i = min(u * 256 + (int)threadIdx.x, TT * PER * 32 - 1);
            const int64_t rt = min(tb * TT + i / (PER * 32), rt_all - 1);
            v.sum[u] = r.sums[(rt * w.groups + (int64_t)kt * PER) * 32 + i % (PER * 32)];
        }
#pragma unroll
        for (int p = 0; p < PER; p++) {
            const int64_t at = (my_tile * w.groups + (int64_t)kt * PER + p) * 16 + (threadIdx.x & 15);
            v.scale[p] = ((const ST *)w.scales)[at];
            if constexpr (ZEROS) v.zero[p] = w.zeros[at];
        }
    };
    auto put_small = [&](int stage, const Small &v) {
#pragma unroll
        for (int u = 0; u < SUMS; u++)
            if (u * 256 + (int)threadIdx.x < TT * PER * 32) sm_s[stage][u * 256 + threadIdx.x] = v.sum[u];
#pragma unroll
        for (int p = 0; p < PER; p++) {
            if constexpr (sizeof(ST) == 2) sm_w[stage][p][threadIdx.x] = bf16_to_f32(v.scale[p]);
            else sm_w[stage][p][threadIdx.x] = v.scale[p];
            if constexpr (ZEROS) sm_z[stage][p][threadIdx.x] = 0x64006400u | v.zero[p] * 0x10001u;
        }
    };
    auto load_codes = [&](int kt, u32x4 (&c)[NT]) {
#pragma unroll
        for (int i = 0; i < NT; i++) c[i] = *reinterpret_cast<const u32x4 *>(w.codes + ((tile[i] * w.k_tiles + kt) * 64 + lane) * 4);
    };

    f32x4 total[NT][TT];
#pragma unroll
    for (int i = 0; i < NT; i++)
#pragma unroll
        for (int t = 0; t < TT; t++) total[i][t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    u32x4 code[NT];
    Small small;
    copy_x(k0, 0);
    load_codes(k0, code);
    load_small(k0, small);
    for (int kt = k0; kt < k1; kt++) {
        const int stage = (kt - k0) & 1;
        put_small(stage, small);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        lds_barrier();      // this tile's copies have arrived, everyone is done with the other stage
        u32x4 next[NT];
        const int ahead = min(kt + 1, k1 - 1);
        if (kt + 1 < k1) copy_x(ahead, stage ^ 1);
        load_codes(ahead, next);
        load_small(ahead, small);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            f16x8 a[NT][JG];
#pragma unroll
            for (int i = 0; i < NT; i++) {
                uint32_t z = 0x64086408u;      // 8
                if constexpr (ZEROS) z = sm_z[stage][p][(wave * NT + i) * 16 + col];
#pragma unroll
                for (int j = 0; j < JG; j++) a[i][j] = SUBNORMAL ? codes_as_subnormals(code[i][p * JG + j]) : codes_less(code[i][p * JG + j], z);
            }
            f32x4 sc[NT];
#pragma unroll
            for (int i = 0; i < NT; i++) sc[i] = *reinterpret_cast<const f32x4 *>(&sm_w[stage][p][(wave * NT + i) * 16 + 4 * h]);
#pragma unroll
            for (int t = 0; t < TT; t++) {
                float s_hi = 0.f, s_lo = 0.f;
                if constexpr (SUBNORMAL) {
                    s_hi = sm_s[stage][(t * PER + p) * 32 + col];
                    s_lo = sm_s[stage][(t * PER + p) * 32 + 16 + col];
                }
                auto operand = [&](int j, int term) {
                    return *reinterpret_cast<const f16x8 *>(sm_x[stage] + (t * 4 + p * JG + j) * 2048 + term * 1024 + lane * 16);
                };
                f32x4 d[NT];
                if constexpr (SUBNORMAL) {
                    const float c_hi = -8.f * s_hi, c_lo = -8.f * s_lo;      // what the sums owe to the zero point 8
                    f32x4 lo[NT];
#pragma unroll
                    for (int i = 0; i < NT; i++) {
                        d[i] = (f32x4){c_hi, c_hi, c_hi, c_hi};
                        lo[i] = (f32x4){c_lo, c_lo, c_lo, c_lo};
                    }
#pragma unroll
                    for (int j = 0; j < JG; j++) {
                        const f16x8 bh = operand(j, 0), bl = operand(j, 1);
#pragma unroll
                        for (int i = 0; i < NT; i++) d[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][j], bh, d[i], 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < NT; i++) lo[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][j], bl, lo[i], 0, 0, 0);
                    }
#pragma unroll
                    for (int i = 0; i < NT; i++) d[i] += lo[i];
                } else {
#pragma unroll
                    for (int i = 0; i < NT; i++) d[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int term = 0; term < 2; term++)      // all hi products first: their sum is exact, the lo products are added to it
#pragma unroll
                        for (int j = 0; j < JG; j++) {
                            const f16x8 b = operand(j, term);
#pragma unroll
                            for (int i = 0; i < NT; i++) d[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[i][j], b, d[i], 0, 0, 0);
                        }
                }
#pragma unroll
                for (int i = 0; i < NT; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) total[i][t][e] += sc[i][e] * d[i][e];
            }
        }
#pragma unroll
        for (int i = 0; i < NT; i++) code[i] = next[i];
    }

    const int np = w.row_tiles * 16;      // rows of a part, padded
#pragma unroll
    for (int t = 0; t < TT; t++) {
        const int row = (tb * TT + t) * 16 + col;
        if (row >= T) continue;
        if (slabs > 1) {
#pragma unroll
            for (int i = 0; i < NT; i++)
                if (tile_of[i] < w.row_tiles)
                    *reinterpret_cast<f32x4 *>(part + (((int64_t)slab * T + row) * (pair ? 2 : 1) + (pair && i >= 2 ? 1 : 0)) * np + tile_of[i] * 16 + 4 * h) =
                        total[i][t];
            continue;
        }
        const int expo = r.expo[row];
#pragma unroll
        for (int i = 0; i < NT; i++) {
            if (pair && i >= 2) break;
            const int n = tile_of[i] * 16 + 4 * h;
            float *dst = y + (int64_t)row * N + n;
            float out[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                out[e] = ld::w4_finish(total[i][t][e], expo);
                if (pair) out[e] = ld::w4_gated(out[e], ld::w4_finish(total[(i + 2) % NT][t][e], expo));
            }
            if (n + 4 <= N && N % 4 == 0 && !((uintptr_t)y & 15)) {
                float4 v = make_float4(out[0], out[1], out[2], out[3]);
                if (epilogue == LDK_ADD) {
                    const float4 o = *reinterpret_cast<const float4 *>(dst);
                    v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
                }
                *reinterpret_cast<float4 *>(dst) = v;
            } else {
                for (int e = 0; e < 4; e++)
                    if (n + e < N) dst[e] = epilogue == LDK_ADD ? dst[e] + out[e] : out[e];
            }
        }
    }
}

// The slabs' sums added in their order, then the epilogue.  A thread four outputs of a row.  16 slabs of 32 x 6144 sums (12.6 MB): 4.3 us.
__global__ __launch_bounds__(256) void k_w4_join(const float *__restrict__ part, const int32_t *__restrict__ expo, int T, int N, int np, int slabs,
                                                 int epilogue, float *__restrict__ y) {
    const int quads = np / 4;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(id / quads), n = (int)(id % quads) * 4;
    if (row >= T || n >= N) return;
    const bool pair = epilogue == LDK_SWIGLU;
    const int64_t wide = (int64_t)np * (pair ? 2 : 1);
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const f32x4 a = slab_sum(reinterpret_cast<const f32x4 *>(part + row * wide + n), T * wide / 4, slabs, zero);
    const f32x4 b = pair ? slab_sum(reinterpret_cast<const f32x4 *>(part + row * wide + np + n), T * wide / 4, slabs, zero) : zero;
    const int e2 = expo[row];
    float *dst = y + (int64_t)row * N + n;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        if (n + e >= N) break;
        float v = ld::w4_finish(a[e], e2);
        if (pair) v = ld::w4_gated(v, ld::w4_finish(b[e], e2));
        dst[e] = epilogue == LDK_ADD ? dst[e] + v : v;
    }
}

template <int TT, int G>
void launch_tile(const ld::W4Image &w, int scale_dtype, const ld::W4Rows &r, int T, int N, int epilogue, const ld::W4Plan &p, float *y, hipStream_t s) {
    const dim3 grid(p.n_blocks * p.t_blocks, p.slabs), block(256);
#define LD_TILE(Z_, S_) LD_LAUNCH((k_w4_tile<TT, G, Z_, S_>), grid, block, 0, s, w, r, T, N, epilogue, p.n_blocks, p.t_blocks, p.slabs, y, r.part)
    if (scale_dtype == LD_BF16) { if (w.zeros) LD_TILE(true, bf16_t); else LD_TILE(false, bf16_t); }
    else { if (w.zeros) LD_TILE(true, float); else LD_TILE(false, float); }
#undef LD_TILE
}
template <int G>
void launch_group(const ld::W4Image &w, int scale_dtype, const ld::W4Rows &r, int T, int N, int epilogue, const ld::W4Plan &p, float *y, hipStream_t s) {
    if (p.tt == 1) launch_tile<1, G>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    else if (p.tt == 2) launch_tile<2, G>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    else if (p.tt == 3) launch_tile<3, G>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    else launch_tile<4, G>(w, scale_dtype, r, T, N, epilogue, p, y, s);
}

}  // namespace

namespace ld {

constexpr int MOST_SLABS = 16, MOST_GROUPS = 1024;      // slabs, and workgroups of a launch with slabs

size_t w4_part_bound(int T, int N, int epilogue) {
    // n_blocks t_blocks slabs <= MOST_GROUPS, and a workgroup leaves at most 64 rows of 256 sums
    const size_t row = (size_t)((N + 15) / 16 * 16) * (epilogue == LDK_SWIGLU ? 2 : 1) * 4;
    return std::min((size_t)MOST_SLABS * T * row, (size_t)MOST_GROUPS * 64 * 256 * 4);
}

// Tile and slabs.  Up to 128 rows: 16 of them a workgroup (four workgroups a CU), and as many slabs as bring some 1024 workgroups
// and leave each two column tiles.  More rows: the least of rounds x (column tiles + 3.3, what begins and ends a workgroup) x the time of a column
// tile of 32, 48 or 64 rows, a last round that leaves half the CUs one workgroup taking 0.84 of one; slabs cost a launch and their sums' way
// out and back, 5.9 column tiles of 32 rows.  Both fitted to 110 sizes (3 .. 1056 rows of the decoder shapes' matrices, each in up to 20
// forms): the times of the forms taken are 2 % and 0.2 % above the best ones' in the mean.
W4Plan w4_plan(int T, int N, int K, int epilogue) {
    const int row_tiles = (N + 15) / 16, k_tiles = (K + 127) / 128, per_block = epilogue == LDK_SWIGLU ? 8 : 16;
    W4Plan best{};
    best.n_blocks = (row_tiles + per_block - 1) / per_block;
    if (T <= 128) {
        best.tt = 1;
        best.t_blocks = (T + 15) / 16;
        best.slabs = (int)std::max<int64_t>(1, std::min<int64_t>({MOST_SLABS, k_tiles / 2, MOST_GROUPS / ((int64_t)best.n_blocks * best.t_blocks)}));
    } else {
        const double tile[3] = {1.0, 1.28, 1.72};
        double cost = 0;
        for (int tt = 2; tt <= 4; tt++)
            for (int slabs = 1; slabs <= MOST_SLABS && slabs <= k_tiles; slabs++) {
                const int t_blocks = (T + 16 * tt - 1) / (16 * tt);
                const int64_t groups = (int64_t)best.n_blocks * t_blocks * slabs, rest = groups % 512;
                if (slabs > 1 && groups > MOST_GROUPS) break;
                const double rounds = (double)(groups / 512) + (rest == 0 ? 0 : rest <= 256 ? 0.84 : 1);
                const double c = rounds * ((k_tiles + slabs - 1) / slabs + 3.3) * tile[tt - 2] + (slabs > 1 ? 5.9 : 0);
                if (cost == 0 || c < cost) {
                    cost = c;
                    best.tt = tt;
                    best.t_blocks = t_blocks;
                    best.slabs = slabs;
                }
            }
    }
    best.part_bytes = best.slabs > 1 ? (size_t)best.slabs * T * row_tiles * 16 * (epilogue == LDK_SWIGLU ? 2 : 1) * 4 : 0;
    return best;
}

void launch_w4_tile(const W4Image &w, int scale_dtype, const W4Rows &r, int group, int T, int N, int epilogue, const W4Plan &p, float *y, hipStream_t s) {
    if (group == 32) launch_group<32>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    else if (group == 64) launch_group<64>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    else launch_group<128>(w, scale_dtype, r, T, N, epilogue, p, y, s);
    if (p.slabs > 1) {
        const int np = w.row_tiles * 16;
        LD_LAUNCH(k_w4_join, dim3((unsigned)(((int64_t)T * (np / 4) + 255) / 256)), dim3(256), 0, s, r.part, r.expo, T, N, np, p.slabs, epilogue, y);
    }
}

}  // namespace ld
