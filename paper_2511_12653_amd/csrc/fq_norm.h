// Internal interface between the host side of layer norm (fq_norm_api.cpp) and its gfx950 kernels (fq_norm.hip).
// Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr long long kNormMostWidth = 1LL << 24;
constexpr int kNormHeldWidth = 16384;            // rows of up to so many values stay in a block's registers
constexpr int kNormStrip = 512;                  // columns of a block where they do not (backward)

struct NormArgs {
    const void *x, *w, *b;     // w, b: null for 1 and 0
    void *y;
    float *ys, *stats;
    const void *gy;
    void *gx, *gw, *gb;
    float *partial;            // [parts][2][width] sums of the rows' shares of gweight and gbias
    long long rows;
    long long ldx, ldy, ldgy, ldgx;
    int width, parts, blocks;
    int lanes, vecs;           // that a row has; vectors of eight values that a lane has
    float eps;
    double inverse;            // 1 / width
    int x16, y16, codes, w16;  // 1: FP16 (else FP32); y is codes
};

constexpr int norm_threads(int lanes) { return lanes > 64 ? lanes : 256; }       // of a block

int launch_norm_forward(const NormArgs &a, void *stream);
int launch_norm_backward(const NormArgs &a, void *stream);

}  // namespace fq
