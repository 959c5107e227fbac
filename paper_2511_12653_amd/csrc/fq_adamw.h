// Internal interface between the host side of the AdamW step (fq_adamw_api.cpp) and its gfx950 kernel
// (fq_adamw.hip).  Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr int kAdamwThreads = 256;               // four wavefronts
constexpr unsigned kStateBlock = 256;            // elements that share a scale: one wavefront's, four to a lane
constexpr unsigned kAdamwRowElems = 4 * kAdamwThreads;   // elements of a grid block's row, four state blocks

struct AdamwTensor {
    void *p;
    const void *g;
    void *p16;
    void *m, *v;
    float *m_scale, *v_scale;
    long long n;
    float lr_scale, weight_decay;
    unsigned first;            // first grid block
    unsigned place;            // 256 * (state blocks of the tensors before), modulo 2^32
    unsigned char p16_type, g16_type;     // 1: p (g) is FP16
    unsigned char f8;                     // 1: FP8 states
    unsigned char vec;                    // 1: every pointer allows a load of four elements
};

// Step constants, rounded on the host.
struct AdamwStep {
    float beta1, one_minus_beta1, beta2, one_minus_beta2;
    float lr, lr_corrected;    // lr and lr / (1 - beta1^t)
    float root_factor, eps;    // 1 / sqrt(1 - beta2^t)
    unsigned key;
    const float *grad_scale;
};

// table: the n descriptors, and behind them (at `first`) their first grid blocks; or, with no `first`, a descriptor for each
// grid block.  rows: rows of a grid block, 1 or 2 (1 without `first`).
int launch_adamw(const AdamwTensor *table, const unsigned *first, int n, const AdamwStep &s, unsigned blocks, int rows,
                 void *stream);

}  // namespace fq
