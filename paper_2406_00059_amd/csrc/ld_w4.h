// Linear layers on 4-bit weights: the image of a matrix and the image of the activations (see ld_w4.hip).
#pragma once
#include <cstddef>
#include <cstdint>
#include "ld_internal.h"

namespace ld {

struct W4Image {
    uint32_t *codes;       // [part][row tile][k tile][lane][4]
    void *scales;          // [part][row tile][group][16]
    uint8_t *zeros;        // the same, or null: 8 everywhere
    int row_tiles, k_tiles, groups;      // of one part; groups: k_tiles * 128 / G
};

constexpr int W4_NOT_FINITE = 1 << 20;

// How the products of many rows take the codes: as subnormals (fewest instructions a code) with wide groups and zero points 8, as c - z (fewest a group's
// sum, and zero points cost nothing more) otherwise.  us, subnormals / c - z: 4096 x 11008 with groups of 32, 300 rows 95 / 80; 6144 x 4096 with groups of 64, 512 rows
// 77 / 71; gated 2 x 13824 x 5120 with groups of 128, 1056 rows 494 / 523, with zero points given 592 / 528.
constexpr bool w4_subnormal(int group, bool zeros) { return group == 128 && !zeros; }

struct W4Rows {
    uint16_t *image;       // fp16 operands
    float *sums;
    int32_t *expo;
    float *part;           // sums of slabs of K
    int k_tiles;
};

// A product of many rows: workgroups of 16 tt rows and 256 outputs (128 gated ones), K in slabs.
struct W4Plan {
    int tt, slabs, n_blocks, t_blocks;
    size_t part_bytes;
};
W4Plan w4_plan(int T, int N, int K, int epilogue);
size_t w4_part_bound(int T, int N, int epilogue);      // of any plan of up to T rows
void launch_w4_tile(const W4Image &w, int scale_dtype, const W4Rows &r, int group, int T, int N, int epilogue, const W4Plan &p, float *y, hipStream_t s);

#if defined(__HIPCC__)
// A finished sum of a row in units of 1, and the gated activation.
__device__ __forceinline__ float w4_finish(float v, int expo) { return expo == W4_NOT_FINITE ? NAN : ldexpf(v, expo); }
__device__ __forceinline__ float w4_gated(float gate, float up) { return gate / (1.f + expf(-gate)) * up; }
#endif

// The regions of an image, and its size.
W4Image w4_image(const void *image, int N, int K, int group, int parts, int scale_dtype, bool zeros, size_t *bytes);
// The regions of the scratch for T rows of K columns, and their size.
W4Rows w4_rows(void *scratch, int T, int K, size_t part_bytes, size_t *bytes);

}  // namespace ld
