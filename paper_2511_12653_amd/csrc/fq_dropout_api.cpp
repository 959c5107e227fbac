// Host side of dropout: validation and launch (declared in include/fq.h).
#include <cmath>
#include <cstring>

#include "../../include/fq.h"
#include "fq_dropout.h"
#include "fq_extent.h"

namespace fq {
namespace {

fq_status validate(const fq_dropout_args &d)
{
    if ((d.x_dtype != FQ_F16 && d.x_dtype != FQ_F32) || (d.y_dtype != FQ_F16 && d.y_dtype != FQ_F32)) return FQ_ERR_DTYPE;
    if (d.n < 0 || d.n > (1LL << 35)) return FQ_ERR_SHAPE;
    if (!(d.p >= 0.0 && d.p <= 1.0)) return FQ_ERR_SCALE_PARAMS;
    const size_t n = (size_t)d.n, xb = size_of(d.x_dtype), yb = size_of(d.y_dtype);
    if (!aligned(d.x, xb) || !aligned(d.residual, yb) || !aligned(d.y, yb) || !aligned(d.step_on_device, 8)) return FQ_ERR_ALIGN;
    if (d.n == 0) return FQ_OK;
    if (!d.x || !d.y) return FQ_ERR_NULL;
    const Rows y = {(uintptr_t)d.y, n * yb, n * yb, 1}, step = {(uintptr_t)d.step_on_device, 8, 8, 1};
    const Rows in[] = {{(uintptr_t)d.x, n * xb, n * xb, 1}, {(uintptr_t)d.residual, n * yb, n * yb, 1}};
    for (const Rows &r : in)
        if (overlap(y, r) && !(y.at == r.at && y.width == r.width)) return FQ_ERR_ALIAS;
    return overlap(y, step) ? FQ_ERR_ALIAS : FQ_OK;
}

}  // namespace
}  // namespace fq

extern "C" fq_status fq_dropout(const fq_dropout_args *d, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    const fq_status st = fq::validate(*d);
    if (st != FQ_OK || d->n == 0) return st;
    fq::DropoutArgs a;
    std::memset(&a, 0, sizeof a);
    a.x = d->x; a.residual = d->residual; a.y = d->y; a.step_on_device = d->step_on_device;
    a.seed = d->seed; a.step = d->step; a.n = d->n;
    a.threshold = (unsigned)std::nearbyint(d->p * 2147483648.0);
    a.scale = d->p < 1.0 ? (float)(1.0 / (1.0 - d->p)) : 0.0f;
    a.x16 = d->x_dtype == FQ_F16; a.y16 = d->y_dtype == FQ_F16;
    return fq::launch_dropout(a, hip_stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
}
