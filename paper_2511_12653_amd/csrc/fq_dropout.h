// Internal interface between the host side of dropout (fq_dropout_api.cpp) and its gfx950 kernel (fq_dropout.hip).
// Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

struct DropoutArgs {
    const void *x, *residual;
    void *y;
    const uint64_t *step_on_device;
    uint64_t seed, step;
    long long n;
    unsigned threshold;        // kept: 31 random bits of at least this
    float scale;
    int x16, y16;
};

int launch_dropout(const DropoutArgs &a, void *stream);

}  // namespace fq
