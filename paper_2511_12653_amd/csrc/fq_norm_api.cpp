// Host side of layer norm: validation, workspace and launches (declared in include/fq.h).
#include <cmath>
#include <cstring>

#include "../../include/fq.h"
#include "fq_extent.h"
#include "fq_internal.h"
#include "fq_norm.h"

namespace fq {
namespace {

constexpr size_t kAlign = 256;
constexpr long long kMostRows = 1LL << 36, kMostRowsOfPart = 256, kMostParts = 1LL << 21;

bool float_type(int32_t dtype) { return dtype == FQ_F16 || dtype == FQ_F32; }

// One row of `count` values.
Rows line(const void *p, size_t count, size_t size) { return {(uintptr_t)p, count * size, count * size, 1}; }

bool same(const Rows &a, const Rows &b) { return a.at == b.at && a.width == b.width && (a.pitch == b.pitch || a.count == 1); }

// Whether what is written (`out`) shares memory with anything else; `in_place`: the inputs that it may be.
bool alias(const Rows *out, int outs, const Rows *in, int ins, int in_place)
{
    for (int i = 0; i < outs; ++i) {
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return true;
        for (int j = 0; j < ins; ++j)
            if (overlap(out[i], in[j]) && !(i == 0 && j < in_place && same(out[i], in[j]))) return true;
    }
    return false;
}

fq_status validate(const fq_norm &d, bool backward)
{
    if (!float_type(d.x_dtype) || !float_type(d.w_dtype)) return FQ_ERR_DTYPE;
    if (!float_type(d.y_dtype) && (backward || d.y_dtype != FQ_I8)) return FQ_ERR_DTYPE;
    if (d.rows < 0 || d.width < 0 || d.rows > kMostRows || d.width > kNormMostWidth) return FQ_ERR_SHAPE;
    if (!pitch_fits(d.rows, d.ldx, d.width)) return FQ_ERR_SHAPE;
    if (!backward && !pitch_fits(d.rows, d.ldy, d.width)) return FQ_ERR_SHAPE;
    if (backward && (!pitch_fits(d.rows, d.ldgy, d.width) || (d.gx && !pitch_fits(d.rows, d.ldgx, d.width)))) return FQ_ERR_SHAPE;
    if (!std::isfinite(d.eps) || d.eps < 0.0f) return FQ_ERR_SCALE_PARAMS;
    const size_t xb = size_of(d.x_dtype), yb = size_of(d.y_dtype), wb = size_of(d.w_dtype);
    if (!aligned(d.x, xb) || !aligned(d.weight, wb) || !aligned(d.bias, wb) || !aligned(d.stats, 4)) return FQ_ERR_ALIGN;
    const size_t m = (size_t)d.rows, k = (size_t)d.width;
    if (!backward) {
        if (!aligned(d.y, yb) || !aligned(d.ys, 4)) return FQ_ERR_ALIGN;
        if (d.rows == 0 || d.width == 0) return FQ_OK;
        if (!d.x || !d.y || (d.y_dtype == FQ_I8 && !d.ys)) return FQ_ERR_NULL;
        const Rows out[] = {{(uintptr_t)d.y, k * yb, (size_t)d.ldy * yb, m}, line(d.y_dtype == FQ_I8 ? d.ys : nullptr, m, 4),
                            line(d.stats, m, 8)};
        const Rows in[] = {{(uintptr_t)d.x, k * xb, (size_t)d.ldx * xb, m}, line(d.weight, k, wb), line(d.bias, k, wb)};
        return alias(out, 3, in, 3, 1) ? FQ_ERR_ALIAS : FQ_OK;
    }
    if (!aligned(d.gy, yb) || !aligned(d.gx, xb) || !aligned(d.gweight, wb) || !aligned(d.gbias, wb)) return FQ_ERR_ALIGN;
    if (d.width == 0) return FQ_OK;
    if (d.rows > 0 && (!d.x || !d.gy || !d.stats)) return FQ_ERR_NULL;
    const Rows out[] = {{(uintptr_t)d.gx, k * xb, (size_t)d.ldgx * xb, m}, line(d.gweight, k, wb), line(d.gbias, k, wb)};
    const Rows in[] = {{(uintptr_t)d.x, k * xb, (size_t)d.ldx * xb, m}, {(uintptr_t)d.gy, k * yb, (size_t)d.ldgy * yb, m},
                       line(d.weight, k, wb), line(d.stats, m, 8)};
    return alias(out, 3, in, 4, 2) ? FQ_ERR_ALIAS : FQ_OK;
}

// How rows are spread over the chip: lanes of a row, vectors of eight values to a lane, blocks to a compute unit, which then go from row
// to row.  What a row costs beside its values (its sums over the lanes, its root) is paid by every wavefront that has a part of it, so
// lanes have as many values as registers allow; more blocks hide more of it, fewer ask for weight and bias less often.  FP16, us, with the
// shape here / others: forward 19200 x 384 (16, 3, 3) 7.6 / (64, 1) 11.2; 16384 x 2048 (64, 4, 2) 26.3 / (256, 1) 36.2; 32768 x 8192 (256, 4, 1)
// 176 / (256, 4, 2) 195 / (512, 2, 2) 191; codes 16384 x 4096 (256, 2, 6) 58.2 / (256, 2, 2) 70 / (512, 2) 80; backward 19200 x 384 (64, 1, 2)
// 15.5 / (16, 3, 2) 17.3; 1201 x 1155 (256, 1, 1) 11.4 / (64, 3, 1) 12.0; 32768 x 8192 (256, 4, 1) 285 / (512, 2, 1) 293.  A vector that
// no lane needs costs its registers and, in codes, its arithmetic: codes of FP32 8000 x 5120 (256, 3, 2) 45.7 / (256, 4, 6) 75, of 4000 x 12288
// (512, 3, 1) 56 / (512, 4, 1) 105; backward 8000 x 5120 (256, 3, 1) 59 / (256, 4, 1) 68.
struct Shape {
    int lanes, vecs, blocks;
    int rows() const { return norm_threads(lanes) / lanes; }         // of a block at a time
};

Shape shape_of(const fq_norm &d, bool backward)
{
    const long long width = d.width;
    if (width > kNormHeldWidth) return {1024, 2, 2};
    if (width < 8) return {16, 1, 4};
    if (backward) {
        if (width <= 256) return {16, width <= 128 ? 1 : 2, 2};
        if (width <= 1024) return {64, width <= 512 ? 1 : 2, 2};
        if (width <= 2048) return {256, 1, 2};
        if (width <= 4096) return {256, 2, 2};
        if (width <= 8192) return {256, width <= 6144 ? 3 : 4, 1};
        return {512, width <= 12288 ? 3 : 4, 1};
    }
    const bool codes = d.y_dtype == FQ_I8;
    if (width <= 128) return {16, 1, 6};
    if (width <= 512) return {16, width <= 256 ? 2 : width <= 384 ? 3 : 4, codes ? 2 : 3};
    if (width <= 1536) return {64, width <= 1024 ? 2 : 3, codes ? 6 : 2};
    if (width <= 2048) return {64, 4, 2};
    if (width <= 4096) return {256, 2, codes ? 6 : 2};
    if (width <= 6144) return {256, 3, codes || d.x_dtype == FQ_F16 ? 2 : 1};
    if (width <= 8192) return {256, 4, codes ? 6 : 1};
    return {512, width <= 12288 ? 3 : 4, 1};
}

// Blocks of the backward pass, each of which makes a partial sum of every column: as many as the chip holds, and enough for no
// more than kMostRowsOfPart rows to one (those are added in binary32, the parts in binary64).  Rows that no block holds go in
// strips of columns: so many blocks to a part.  A few rows are one part, which needs no second launch.
int parts_of(const fq_norm &d)
{
    const Shape s = shape_of(d, true);
    const long long groups = (d.rows + s.rows() - 1) / s.rows(), least = (groups + kMostRowsOfPart - 1) / kMostRowsOfPart;
    const bool held = d.width <= kNormHeldWidth;
    // (us, in one part / in one for each group of rows a block has at a time: 4 x 1155 4.5 / 5.7, 6 x 1155 6.0 / 5.7, 3 x 4096 5.4 / 5.9, 4 x 4096 6.5 / 6.1,
    // 2 x 9305 7.0 / 8.2, 3 x 9305 8.8 / 8.3)
    if (held && groups <= (s.vecs == 1 ? 4 : s.vecs == 2 ? 3 : 2)) return 1;
    const long long strips = held ? 1 : (d.width + kNormStrip - 1) / kNormStrip;
    long long chip = held ? (long long)s.blocks * kComputeUnits : strips < 2 * kComputeUnits ? 2 * kComputeUnits / strips : 1;
    // (a part of a wide row's width is as much to write, and to read again, as two or three rows: 403 x 4096 FP16 13.2 us in 128 parts, 17.7 in 403)
    if (held && s.rows() == 1 && groups / 3 < chip) chip = groups / 3 > 128 ? groups / 3 : 128;
    const long long parts = groups < chip ? groups : least > chip ? least : chip, most = kMostParts / strips;
    return (int)(parts < most ? parts : most);
}

size_t workspace_of(const fq_norm &d)
{
    if (d.rows == 0 || d.width == 0 || (!d.gweight && !d.gbias)) return kAlign;
    return round_up((size_t)parts_of(d) * 2 * (size_t)d.width * sizeof(float), kAlign);
}

NormArgs args_of(const fq_norm &d, bool backward)
{
    NormArgs a;
    std::memset(&a, 0, sizeof a);
    a.x = d.x; a.w = d.weight; a.b = d.bias; a.y = d.y; a.stats = d.stats;
    a.ys = d.ys; a.gy = d.gy; a.gx = d.gx; a.gw = d.gweight; a.gb = d.gbias;
    a.rows = d.rows; a.width = (int)d.width; a.eps = d.eps; a.inverse = 1.0 / (double)d.width;
    a.ldx = d.ldx; a.ldy = d.ldy; a.ldgy = d.ldgy; a.ldgx = d.ldgx;
    a.x16 = d.x_dtype == FQ_F16; a.y16 = d.y_dtype == FQ_F16; a.codes = d.y_dtype == FQ_I8; a.w16 = d.w_dtype == FQ_F16;
    const Shape s = shape_of(d, backward);
    const long long groups = (d.rows + s.rows() - 1) / s.rows(), chip = (long long)s.blocks * kComputeUnits;
    a.lanes = s.lanes; a.vecs = s.vecs;
    a.blocks = (int)(groups < chip ? groups : chip);
    return a;
}

}  // namespace
}  // namespace fq

extern "C" {

fq_status fq_norm_forward(const fq_norm *d, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    const fq_status st = fq::validate(*d, false);
    if (st != FQ_OK || d->rows == 0 || d->width == 0) return st;
    return fq::launch_norm_forward(fq::args_of(*d, false), hip_stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
}

size_t fq_norm_workspace_bytes(const fq_norm *d)
{
    return d && fq::validate(*d, true) == FQ_OK ? fq::workspace_of(*d) : 0;
}

fq_status fq_norm_backward(const fq_norm *d, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    const fq_status st = fq::validate(*d, true);
    if (st != FQ_OK || d->width == 0 || (!d->gx && !d->gweight && !d->gbias)) return st;
    fq::NormArgs a = fq::args_of(*d, true);
    if (d->rows > 0 && (d->gweight || d->gbias)) {
        if (!workspace || ws_bytes < fq::workspace_of(*d)) return FQ_ERR_WORKSPACE;
        if (!fq::aligned(workspace, fq::kAlign)) return FQ_ERR_ALIGN;
        a.partial = (float *)workspace;
        a.parts = fq::parts_of(*d);
    }
    if (d->rows == 0 && !d->gweight && !d->gbias) return FQ_OK;
    if (a.partial && d->width <= fq::kNormHeldWidth) a.blocks = a.parts;
    return fq::launch_norm_backward(a, hip_stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
}

}  // extern "C"
