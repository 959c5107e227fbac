// Internal interface between the host side of the adapters (fq_adapters_api.cpp) and their gfx950 kernels (fq_adapters.hip).
// Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr long long kAdaptersMostWidth = 1LL << 20;
constexpr int kAdaptersMostRank = 256;

struct AdapterArgs {
    const void *x;
    const float *xs;
    const int32_t *ids;
    const void *a, *b;
    const float *scale;
    const void *base;
    void *y;
    float *t;                  // [m][rank]
    long long ldx, ldy, ldbase;
    int m, n, k, count, rank;
    int xs_step;
    int x_type;                // fq_dtype
    int y16, base16;
};

int launch_adapters(const AdapterArgs &a, void *stream);

}  // namespace fq
