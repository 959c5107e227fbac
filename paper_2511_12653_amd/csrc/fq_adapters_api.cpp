// Host side of the adapters: validation, workspace and launches (declared in include/fq.h).
#include <cstring>

#include "../../include/fq.h"
#include "fq_adapters.h"
#include "fq_extent.h"
#include "fq_internal.h"

namespace fq {
namespace {

constexpr size_t kAlign = 256;
constexpr long long kMostSplits = 8;

fq_status validate(const fq_adapters &d)
{
    if (d.x_dtype != FQ_F16 && d.x_dtype != FQ_F32 && d.x_dtype != FQ_I8) return FQ_ERR_DTYPE;
    if ((d.y_dtype != FQ_F16 && d.y_dtype != FQ_F32) || (d.base_dtype != FQ_F16 && d.base_dtype != FQ_F32)) return FQ_ERR_DTYPE;
    if (d.m < 0 || d.n < 0 || d.k < 0 || d.count < 0 || d.rank < 0 || d.m > 0x7fffff00LL || d.n > kAdaptersMostWidth ||
        d.k > kAdaptersMostWidth || d.count > 0x7fffff00LL || d.rank > kAdaptersMostRank)
        return FQ_ERR_SHAPE;
    if (!pitch_fits(d.m, d.ldx, d.k) || !pitch_fits(d.m, d.ldy, d.n) || (d.base && !pitch_fits(d.m, d.ldbase, d.n))) return FQ_ERR_SHAPE;
    if (d.xs_step != 0 && d.xs_step != 1) return FQ_ERR_SHAPE;
    const size_t xb = size_of(d.x_dtype), yb = size_of(d.y_dtype), bb = size_of(d.base_dtype);
    if (!aligned(d.x, xb) || !aligned(d.xs, 4) || !aligned(d.ids, 4) || !aligned(d.a, 2) || !aligned(d.b, 2) || !aligned(d.scale, 4) ||
        !aligned(d.base, bb) || !aligned(d.y, yb))
        return FQ_ERR_ALIGN;
    if (d.m == 0 || d.n == 0) return FQ_OK;
    const bool some = d.count > 0 && d.rank > 0;
    if (!d.y || !d.ids || (d.x_dtype == FQ_I8 && !d.xs) || (d.k > 0 && !d.x) || (some && (!d.b || (d.k > 0 && !d.a)))) return FQ_ERR_NULL;
    const size_t m = (size_t)d.m, n = (size_t)d.n, k = (size_t)d.k, count = (size_t)d.count, all = count * (size_t)d.rank * 2;
    const auto line = [](const void *p, size_t bytes) { return Rows{(uintptr_t)p, bytes, bytes, 1}; };
    const Rows y = {(uintptr_t)d.y, n * yb, (size_t)d.ldy * yb, m}, base = {(uintptr_t)d.base, n * bb, (size_t)d.ldbase * bb, m};
    if (overlap(y, base) && !(y.at == base.at && y.width == base.width && (y.pitch == base.pitch || m == 1))) return FQ_ERR_ALIAS;
    const Rows in[] = {{(uintptr_t)d.x, k * xb, (size_t)d.ldx * xb, m}, line(d.x_dtype == FQ_I8 ? d.xs : nullptr, (d.xs_step ? m : 1) * 4),
                       line(d.ids, m * 4), line(d.a, all * k), line(d.b, all * n), line(d.scale, count * 4)};
    for (const Rows &r : in)
        if (overlap(y, r)) return FQ_ERR_ALIAS;
    return FQ_OK;
}

long long at_most(long long v, long long most) { return v < most ? v : most; }
long long at_least(long long v, long long least) { return v > least ? v : least; }
long long ceiling(long long v, long long by) { return (v + by - 1) / by; }

// Bytes of m rows of x where these and a's begin on 16-byte boundaries and have offsets of 32 bits (else 0).  (So rows end with 16 bytes, too.)
unsigned fitting_bytes(const fq_adapters &d, long long m)
{
    const long long size = (long long)size_of(d.x_dtype);
    if (!aligned(d.x, 16) || !aligned(d.a, 16) || d.ldx * size % 16 != 0 || d.k * (size < 2 ? size : 2) % 16 != 0 || d.k < 16 || d.ldx > (1LL << 31)) return 0;
    const long long bytes = ((m - 1) * d.ldx + d.k) * size;
    return bytes < (1LL << 32) - 4096 ? (unsigned)bytes : 0;
}

// How m tokens of the call are cut up.  Tiles of 32 tokens read the adapters half as often as those of 16, but leave compute units without
// work where there are few (us, 4096 x 4096 by 16 ranks, 4 adapters, tiles of 16 / 32 / 64: 512 tokens 15.4 / 16.9 / 27, 2048 tokens 28.4 / 26.0 / 33,
// 8192 tokens 76 / 65.8 / 66.7); those of 64 pay where an adapter has many bytes (8192 tokens, 64 ranks: 144 / 87 / 80.5).  k goes in as
// many parts as make a block for each compute unit (512 tokens: 15.4 in eight parts, 21 in one).  Channels go in as many
// groups as make two blocks for each, and up to eight as long as a wavefront has two strips one after the other (us, in 4 / 8 / 16 / 32 groups:
// 512 tokens 18 / 15.5 / 14.9 / 15; 2048 tokens 29.6 / 27.1 / 29.2 / 29.2; 8192 x 8192 by 64 ranks 132 / 124.6 / 122 / 130).
AdapterArgs plan_of(const fq_adapters &d, long long m)
{
    AdapterArgs a;
    std::memset(&a, 0, sizeof a);
    a.m = (int)m; a.n = (int)d.n; a.k = (int)d.k; a.count = d.rank > 0 ? (int)d.count : 0; a.rank = (int)d.rank;
    a.pitch = (int)ceiling(d.rank, 16) * 16;
    a.x_bytes = fitting_bytes(d, m);
    const bool large = a.x_bytes > 0 && d.x_dtype != FQ_F32 && d.rank > 32 && d.rank <= 64 && m >= 64LL * a.count && m >= 4096;
    a.token_tiles = m < 1024 || m < 16LL * a.count || d.k < 16 || d.n < 4 ? 1 : large ? 4 : 2;
    a.rank_tiles = d.rank <= 16 || d.k < 16 ? 1 : d.rank <= 32 ? 2 : 4;
    a.chunks = (int)ceiling(d.rank, 16 * a.rank_tiles);
    const long long tile = 16 * a.token_tiles, some = at_most(a.count + 1LL, m);
    a.way = m <= kWindow || a.count == 0 || a.count > kMostGrouped ? kWindows : m <= kSorted ? kSorting : kList;
    a.tiles_most = (int)(a.way != kWindows ? m / tile + some : ceiling(m, kWindow) * at_most(m, kWindow));
    const long long tiles = at_least(m / tile + at_most(a.count, m), 1), parts = tiles * at_least(a.chunks, 1);
    a.splits = (int)at_least(at_most(at_most((kComputeUnits + parts / 2) / parts, ceiling(d.k, 256)), kMostSplits), 1);
    a.wide = d.n >= 4 && (a.token_tiles > 1 || tiles * ceiling(d.n, 64) > 4 * kComputeUnits) ? 4 : 2;
    const long long strips = ceiling(d.n, 64 * a.wide);          // that a block of four wavefronts takes at a time
    a.groups = 1;
    while ((a.groups * tiles < 2 * kComputeUnits && a.groups < strips) || (a.groups * tiles < 8 * kComputeUnits && a.groups * 4 <= strips))
        a.groups *= 2;
    if (a.groups > strips) a.groups = (int)strips;
    return a;
}

struct Workspace {
    size_t order = 0, tiles = 0, t = 0, bytes = kAlign;
};

size_t list_bytes(const AdapterArgs &a)
{
    if (a.way == kWindows) return 0;
    return (size_t)a.tiles_most * (a.way == kList ? sizeof(AdapterTile) : (size_t)(2 + 16 * a.token_tiles) * sizeof(int));
}

Workspace workspace_of(const fq_adapters &d)
{
    Workspace at;
    if (d.m == 0 || d.n == 0 || d.count == 0 || d.rank == 0) return at;
    const AdapterArgs a = plan_of(d, at_most(d.m, kAdaptersMostTokens));
    at.tiles = round_up((size_t)a.m * sizeof(int), kAlign);
    size_t list = list_bytes(a);
    if (d.m > kAdaptersMostTokens && d.m % kAdaptersMostTokens != 0) {          // (the last tokens come in a launch of fewer)
        const size_t last = list_bytes(plan_of(d, d.m % kAdaptersMostTokens));
        if (last > list) list = last;
    }
    at.t = at.tiles + round_up(list, kAlign);
    // (calls of several launches do not cut up k)
    at.bytes = at.t + round_up((size_t)a.m * (size_t)a.pitch * sizeof(float) * (size_t)(d.m > kAdaptersMostTokens ? 1 : a.splits), kAlign);
    return at;
}

AdapterArgs args_of(const fq_adapters &d, long long m, void *workspace)
{
    AdapterArgs a = plan_of(d, m);
    const Workspace at = workspace_of(d);
    if (d.m > kAdaptersMostTokens) a.splits = 1;
    char *const ws = (char *)workspace;
    if (a.count > 0) {
        a.order = (int *)(ws + at.order);
        a.tiles = (AdapterTile *)(ws + at.tiles);
        a.found = (int *)(ws + at.tiles);
        a.t = (float *)(ws + at.t);
    }
    a.a = d.a; a.b = d.b; a.scale = d.scale;
    a.ldx = d.ldx; a.ldy = d.ldy; a.ldbase = d.ldbase;
    a.xs_step = d.xs_step; a.x_type = d.x_dtype; a.y16 = d.y_dtype == FQ_F16; a.base16 = d.base_dtype == FQ_F16;
    if (!d.base) {
        a.no_base = 1;
        a.ldbase = a.ldy;
        a.base16 = a.y16;
    }
    return a;
}

}  // namespace
}  // namespace fq

extern "C" {

size_t fq_adapters_workspace_bytes(const fq_adapters *d)
{
    return d && fq::validate(*d) == FQ_OK ? fq::workspace_of(*d).bytes : 0;
}

fq_status fq_adapters_forward(const fq_adapters *d, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    const fq_status st = fq::validate(*d);
    if (st != FQ_OK || d->m == 0 || d->n == 0) return st;
    if (!workspace || ws_bytes < fq::workspace_of(*d).bytes) return FQ_ERR_WORKSPACE;
    if (!fq::aligned(workspace, fq::kAlign)) return FQ_ERR_ALIGN;
    for (long long row = 0; row < d->m; row += fq::kAdaptersMostTokens) {
        fq::AdapterArgs a = fq::args_of(*d, fq::at_most(d->m - row, fq::kAdaptersMostTokens), workspace);
        a.x = d->x ? (const char *)d->x + (size_t)(row * d->ldx) * fq::size_of(d->x_dtype) : nullptr;
        a.xs = d->x_dtype == FQ_I8 ? d->xs + row * d->xs_step : nullptr;
        a.ids = d->ids + row;
        a.base = d->base ? (const char *)d->base + (size_t)(row * d->ldbase) * fq::size_of(d->base_dtype) : nullptr;
        a.y = (char *)d->y + (size_t)(row * d->ldy) * fq::size_of(d->y_dtype);
        if (a.no_base) a.base = a.y;
        if (fq::launch_adapters(a, hip_stream) != 0) return FQ_ERR_LAUNCH;
    }
    return FQ_OK;
}

}  // extern "C"
