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

struct W4Rows {
    uint16_t *image;       // fp16 operands
    float *sums;
    int32_t *expo;
    int k_tiles;
};

// The regions of an image, and its size.
W4Image w4_image(const void *image, int N, int K, int group, int parts, int scale_dtype, bool zeros, size_t *bytes);
// The regions of the scratch for T rows of K columns, and their size.
W4Rows w4_rows(void *scratch, int T, int K, size_t *bytes);

}  // namespace ld
