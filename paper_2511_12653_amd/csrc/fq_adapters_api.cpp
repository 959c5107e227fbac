// Host side of the adapters: validation, workspace and launches (declared in include/fq.h).
#include <cstring>

#include "../../include/fq.h"
#include "fq_adapters.h"
#include "fq_extent.h"

namespace fq {
namespace {

constexpr size_t kAlign = 256;
constexpr long long kMostBlocks = 1LL << 22;     // of a launch, each at least 256 channels of a token

// Tokens of a launch.
long long tokens_of(const fq_adapters &d)
{
    const long long strips = (d.n + 255) / 256, most = kMostBlocks / (strips > 0 ? strips : 1);
    return d.m < most ? d.m : most;
}

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

size_t workspace_of(const fq_adapters &d)
{
    const size_t bytes = round_up((size_t)tokens_of(d) * (size_t)d.rank * sizeof(float), kAlign);
    return d.n > 0 && bytes > kAlign ? bytes : kAlign;
}

AdapterArgs args_of(const fq_adapters &d, void *workspace)
{
    AdapterArgs a;
    std::memset(&a, 0, sizeof a);
    a.ids = d.ids; a.a = d.a; a.b = d.b; a.scale = d.scale; a.t = (float *)workspace;
    a.ldx = d.ldx; a.ldy = d.ldy; a.ldbase = d.ldbase;
    a.n = (int)d.n; a.k = (int)d.k; a.count = d.rank > 0 ? (int)d.count : 0; a.rank = (int)d.rank;
    a.xs_step = d.xs_step; a.x_type = d.x_dtype; a.y16 = d.y_dtype == FQ_F16; a.base16 = d.base_dtype == FQ_F16;
    return a;
}

}  // namespace
}  // namespace fq

extern "C" {

size_t fq_adapters_workspace_bytes(const fq_adapters *d)
{
    return d && fq::validate(*d) == FQ_OK ? fq::workspace_of(*d) : 0;
}

fq_status fq_adapters_forward(const fq_adapters *d, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    const fq_status st = fq::validate(*d);
    if (st != FQ_OK || d->m == 0 || d->n == 0) return st;
    if (!workspace || ws_bytes < fq::workspace_of(*d)) return FQ_ERR_WORKSPACE;
    if (!fq::aligned(workspace, fq::kAlign)) return FQ_ERR_ALIGN;
    fq::AdapterArgs a = fq::args_of(*d, workspace);
    const long long tokens = fq::tokens_of(*d);
    for (long long row = 0; row < d->m; row += tokens) {
        a.m = (int)(d->m - row < tokens ? d->m - row : tokens);
        a.x = d->x ? (const char *)d->x + (size_t)(row * d->ldx) * fq::size_of(d->x_dtype) : nullptr;
        a.xs = d->x_dtype == FQ_I8 ? d->xs + row * d->xs_step : nullptr;
        a.ids = d->ids + row;
        a.base = d->base ? (const char *)d->base + (size_t)(row * d->ldbase) * fq::size_of(d->base_dtype) : nullptr;
        a.y = (char *)d->y + (size_t)(row * d->ldy) * fq::size_of(d->y_dtype);
        if (fq::launch_adapters(a, hip_stream) != 0) return FQ_ERR_LAUNCH;
    }
    return FQ_OK;
}

}  // extern "C"
