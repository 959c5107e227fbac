// Internal interface between the host side of the int8 linear layer (fq_linear_api.cpp) and its gfx950 kernels
// (fq_linear.hip).  Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr long long kLinearMostK = 131071;       // k * 128 * 128 < 2^31
constexpr long long kCodePitch = 128;            // rows of codes in the workspace: a multiple of this, zeros behind k

constexpr long long kMostPitch = 1 << 22;        // of rows of codes that the tiles take: 256 of them have 32-bit offsets
constexpr int kFewLds = 150 << 10;               // most LDS of a block of few tokens
constexpr int kFewLdsOfTwo = 78 << 10;           // most of a block that leaves room for another
constexpr int kFewMostN = 16 * 256;              // channels there of a block to a compute unit

struct LinearArgs {
    const int8_t *x;           // codes, in rows that fit (see w_fits) but in the kernel of few tokens
    const void *raw;           // instead of x: values for the kernel of few tokens
    const float *xs;
    const int8_t *w;
    const float *ws;
    const float *bias;
    void *y;
    long long ldx, ldw, ldy;
    int m, n, k;
    int kx, kw;                // codes of a row of x and w that the tiles read: whole 16; k, or more where zeros lie behind k
    int xs_step, ws_step;
    int x16, x_vec;            // of raw, 1: FP16; rows on 16-byte boundaries
    int y16, y_lines;          // 1: y is FP16; its rows begin on 128-byte lines
    int x_fits;                // 1: so do rows of x, where it is codes
    int w_fits;                // 1: rows of w begin on 16-byte boundaries, k is a multiple of 16, the pitch is at most kMostPitch
};

struct QuantizeArgs {
    const void *x;
    long long ldx;
    int m, k;
    int x16;                   // 1: x is FP16
    int8_t *q;                 // [m][pitch]
    float *s;                  // [m]
    long long pitch;
};

struct AlignArgs {
    const int8_t *from;
    int8_t *to;                // [rows][pitch]
    long long rows, ld, pitch;
    int k;
};

bool linear_few(const LinearArgs &a, int size);   // whether x with elements of so many bytes may be given as raw (or as x)
bool linear_rows(const LinearArgs &a);            // whether x may be given as raw for its short rows
bool linear_rows_as_they_lie(const LinearArgs &a);     // whether w then is best read so; else its rows are laid out anew first
// (`other`: rows of codes to lay out anew by the same launch; none if it has no rows)
int launch_quantize_rows(const QuantizeArgs &a, const AlignArgs &other, void *stream);
int launch_align_rows(const AlignArgs &a, const AlignArgs &other, void *stream);
int launch_linear(const LinearArgs &a, void *stream);

}  // namespace fq
