// Internal interface between the host side of the int8 linear layer (fq_linear_api.cpp) and its gfx950 kernels
// (fq_linear.hip).  Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr long long kLinearMostK = 131071;       // k * 128 * 128 < 2^31
constexpr long long kCodePitch = 128;            // rows of codes in the workspace: a multiple of this, zeros behind k

constexpr int kFewLds = 150 << 10;               // most LDS of a block of few tokens
constexpr int kFewMostN = 16 * 256;              // most channels there: a block to a compute unit

struct LinearArgs {
    const int8_t *x;           // codes
    const void *raw;           // instead of x: values that the kernel quantizes itself (see linear_quantizes)
    const float *xs;
    const int8_t *w;
    const float *ws;
    const float *bias;
    void *y;
    long long ldx, ldw, ldy;
    int m, n, k;
    int kx;                    // codes of a row of x that may be read: k, or up to the pitch where zeros lie behind k
    int xs_step, ws_step;
    int y16;                   // 1: y is FP16
    int y_vec;                 // 1: rows of y begin on 16-byte boundaries
    int x16, x_vec;            // of raw, 1: FP16; rows begin on 16-byte boundaries
    int w_fits;                // 1: rows of w begin on 16-byte boundaries, k is a multiple of 16, the pitch is at most 2^22
    int aligned;               // 1: so do those of x
};

struct QuantizeArgs {
    const void *x;
    long long ldx;
    int m, k;
    int x16;                   // 1: x is FP16
    int vec;                   // 1: rows of x begin on 16-byte boundaries
    int8_t *q;                 // [m][pitch]
    float *s;                  // [m]
    long long pitch;
};

bool linear_quantizes(const LinearArgs &a);      // whether the kernel for these sizes takes values of x
int launch_quantize_rows(const QuantizeArgs &a, void *stream);
int launch_linear(const LinearArgs &a, void *stream);

}  // namespace fq
