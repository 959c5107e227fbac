// Internal interface between the host side of the adapters (fq_adapters_api.cpp) and their gfx950 kernels (fq_adapters.hip).
// Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace fq {

constexpr long long kAdaptersMostWidth = 1LL << 20;
constexpr int kAdaptersMostRank = 256;
constexpr int kWindow = 64;                      // tokens that a wavefront sorts out by itself
constexpr long long kAdaptersMostTokens = 1 << 16;       // of a launch
constexpr int kSorted = 4096, kFewSorted = 1024;   // tokens that a block sorts out by itself; that cost it less
constexpr int kMostGrouped = 1024;               // adapters that tokens are sorted by

enum AdapterWay { kWindows, kSorting, kList };   // how a block comes to its tokens

struct AdapterTile {                             // tokens of one adapter
    int id, first, count;                        // adapter (-1: none); places in `order`
};

struct AdapterArgs {
    const void *x;
    const float *xs;
    const int32_t *ids;
    const void *a, *b;
    const float *scale;
    const void *base;
    void *y;
    float *t;                  // [splits][m][pitch] sums over a part of k each
    int *order;                // kList: [m] tokens by adapter
    AdapterTile *tiles;        // kList: [tiles_most]
    int *found;                // kSorting: [tiles_most][2 + 16 token_tiles], a tile's count, adapter and tokens
    long long ldx, ldy, ldbase;
    int m, n, k, count, rank;
    int pitch;                 // of a row of t: whole 16 values
    int way;                   // AdapterWay
    int tiles_most;            // tiles there can be
    int token_tiles;           // tokens of a tile in 16s: 1, 2 or (with rank_tiles 4, FP16 and codes that fit) 4
    int rank_tiles;            // ranks of a block in 16s: 1, 2 or 4
    int splits, chunks;        // parts of k; of the ranks
    int wide, groups;          // channels of a wavefront at a time in 16s: 2 or 4; blocks that share a tile's channels
    unsigned x_bytes;          // of all rows of x where x and a fit the loads into LDS, else 0
    int xs_step;
    int x_type;                // fq_dtype
    int y16, base16, no_base;  // no_base: base is y, of which nothing counts
};

int launch_adapters(const AdapterArgs &a, void *stream);

}  // namespace fq
