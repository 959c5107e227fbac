// Host side of the AdamW step: validation, the table and its plan (declared in include/fq.h).
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/fq.h"
#include "fq_adamw.h"
#include "fq_internal.h"

namespace fq {
namespace {

constexpr size_t kAlign = 256;
// Two rows to a grid block for lists with FP8 states of more elements than this, else one.  us, one row / two / four: 6.0M elements
// with FP8 states 21.2 / 20.5 / 23.6, 20M FP16 ones 46.8 / 42.1 / 50.3, 240M 657 / 649 / 672; 120M with FP32 states 565 / 586 / 593.
constexpr long long kAdamwOneRow = 1 << 21;
// Up to so many grid blocks the table has a descriptor for each: the search for the block's tensor, a trip to memory in front
// of all others, falls away (88 tensors, 436 blocks: the kernel 2.8 us at best, with the search 3.7).
constexpr long long kAdamwBlockTable = 2048;
constexpr long long kAdamwMostBlocks = 0xffffffffLL / kAdamwThreads;      // a grid has less than 2^32 threads

struct Range {
    uintptr_t at;
    size_t bytes;
};

bool overlap(const Range &a, const Range &b)
{
    return a.at && b.at && a.bytes && b.bytes && a.at < b.at + b.bytes && b.at < a.at + a.bytes;
}

bool float_type(int32_t dtype) { return dtype == FQ_F16 || dtype == FQ_F32; }

bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }

fq_status validate(const fq_param &t)
{
    if (!float_type(t.p_dtype) || !float_type(t.g_dtype)) return FQ_ERR_DTYPE;
    if (t.state != FQ_STATE_F32 && t.state != FQ_STATE_F8) return FQ_ERR_DTYPE;
    if (t.p16 && t.p_dtype != FQ_F32) return FQ_ERR_DTYPE;
    if (t.n < 0 || t.n > (1LL << 40)) return FQ_ERR_SHAPE;
    if (!std::isfinite(t.lr_scale) || !std::isfinite(t.weight_decay)) return FQ_ERR_OPTIMIZER;
    if (t.n == 0) return FQ_OK;
    const bool f8 = t.state == FQ_STATE_F8;
    if (!t.p || !t.g || !t.m || !t.v || (f8 && (!t.m_scale || !t.v_scale))) return FQ_ERR_NULL;
    const size_t n = (size_t)t.n, pb = t.p_dtype == FQ_F16 ? 2 : 4, gb = t.g_dtype == FQ_F16 ? 2 : 4, sb = f8 ? 1 : 4;
    const size_t scales = f8 ? (n + kStateBlock - 1) / kStateBlock * sizeof(float) : 0;
    if (!aligned(t.p, pb) || !aligned(t.g, gb) || !aligned(t.p16, 2) || !aligned(t.m, sb) || !aligned(t.v, sb) ||
        (f8 && (!aligned(t.m_scale, 4) || !aligned(t.v_scale, 4))))
        return FQ_ERR_ALIGN;
    const Range part[] = {{(uintptr_t)t.p, n * pb}, {(uintptr_t)t.g, n * gb}, {(uintptr_t)t.p16, n * 2}, {(uintptr_t)t.m, n * sb},
                          {(uintptr_t)t.v, n * sb}, {(uintptr_t)t.m_scale, scales}, {(uintptr_t)t.v_scale, scales}};
    for (size_t i = 0; i < sizeof part / sizeof part[0]; ++i)
        for (size_t j = 0; j < i; ++j)
            if (overlap(part[i], part[j])) return FQ_ERR_ALIAS;
    return FQ_OK;
}

struct Shape {
    long long blocks = 0;
    int rows = 1;
    long long entries = 0;           // descriptors in the table
    bool by_block = false;           // one for each grid block
    size_t first_off = 0, bytes = 0;
};

fq_status shape_of(const fq_param *ps, int n, Shape &shape)
{
    if (n < 0) return FQ_ERR_SHAPE;
    if (n > 0 && !ps) return FQ_ERR_NULL;
    long long rows = 0;
    bool f8 = false;
    for (int i = 0; i < n; ++i) {
        const fq_status st = validate(ps[i]);
        if (st != FQ_OK) return st;
        rows += (ps[i].n + kAdamwRowElems - 1) / kAdamwRowElems;
        f8 = f8 || ps[i].state == FQ_STATE_F8;
    }
    shape.rows = f8 && rows * (long long)kAdamwRowElems > kAdamwOneRow ? 2 : 1;
    const long long per = (long long)kAdamwRowElems * shape.rows;
    for (int i = 0; i < n; ++i) {
        shape.blocks += (ps[i].n + per - 1) / per;
        if (shape.blocks > kAdamwMostBlocks) return FQ_ERR_SHAPE;
    }
    shape.by_block = shape.rows == 1 && shape.blocks <= kAdamwBlockTable;
    shape.entries = shape.by_block ? shape.blocks : n;
    shape.first_off = (size_t)shape.entries * sizeof(AdamwTensor);
    shape.bytes = (shape.first_off + (shape.by_block ? 0 : (size_t)n * sizeof(unsigned)) + kAlign - 1) / kAlign * kAlign;
    if (shape.bytes == 0) shape.bytes = kAlign;
    return FQ_OK;
}

uint64_t mixed_key(uint64_t seed, int64_t step)
{
    uint64_t k = seed * 0x9E3779B97F4A7C15ull + (uint64_t)step * 0xD1B54A32D192ED03ull;
    k = (k ^ (k >> 32)) * 0x9E3779B97F4A7C15ull;
    return k >> 32;
}

}  // namespace
}  // namespace fq

struct fq_adamw_plan {
    const fq::AdamwTensor *table = nullptr;      // device
    const unsigned *first = nullptr;             // device
    int n = 0;
    fq::Shape shape;
};

namespace {

fq_status fill(fq_adamw_plan *plan, const fq_param *ps, int n, void *workspace, size_t ws_bytes, void *stream)
{
    fq_status st = fq::shape_of(ps, n, plan->shape);
    if (st != FQ_OK) return st;
    plan->n = n;
    if (plan->shape.blocks == 0) return FQ_OK;
    if (!workspace || ws_bytes < plan->shape.bytes) return FQ_ERR_WORKSPACE;
    if (!fq::aligned(workspace, fq::kAlign)) return FQ_ERR_ALIGN;
    std::vector<char> image(plan->shape.bytes, 0);
    const long long per = (long long)fq::kAdamwRowElems * plan->shape.rows;
    unsigned block = 0, place = 0;
    for (int i = 0; i < n; ++i) {
        const fq_param &t = ps[i];
        fq::AdamwTensor d;
        std::memset(&d, 0, sizeof d);
        const bool f8 = t.state == FQ_STATE_F8;
        d.p = t.p; d.g = t.g; d.p16 = t.p16; d.m = t.m; d.v = t.v;
        d.m_scale = f8 ? t.m_scale : nullptr;
        d.v_scale = f8 ? t.v_scale : nullptr;
        d.n = t.n;
        d.lr_scale = t.lr_scale;
        d.weight_decay = t.weight_decay;
        d.first = block;
        d.place = place;
        d.p16_type = t.p_dtype == FQ_F16;
        d.g16_type = t.g_dtype == FQ_F16;
        d.f8 = f8;
        d.vec = fq::aligned(t.p, d.p16_type ? 8 : 16) && fq::aligned(t.g, d.g16_type ? 8 : 16) && fq::aligned(t.p16, 8) &&
                fq::aligned(t.m, f8 ? 4 : 16) && fq::aligned(t.v, f8 ? 4 : 16);
        const unsigned blocks = (unsigned)((t.n + per - 1) / per);
        if (plan->shape.by_block) {
            for (unsigned b = block; b < block + blocks; ++b) std::memcpy(image.data() + (size_t)b * sizeof d, &d, sizeof d);
        } else {
            std::memcpy(image.data() + (size_t)i * sizeof d, &d, sizeof d);
            std::memcpy(image.data() + plan->shape.first_off + (size_t)i * sizeof block, &block, sizeof block);
        }
        block += blocks;
        place += (unsigned)((t.n + fq::kStateBlock - 1) / fq::kStateBlock * fq::kStateBlock);
    }
    if (fq::copy_table_async(workspace, image.data(), image.size(), stream) != 0) return FQ_ERR_LAUNCH;
    plan->table = (const fq::AdamwTensor *)workspace;
    plan->first = plan->shape.by_block ? nullptr : (const unsigned *)((const char *)workspace + plan->shape.first_off);
    return FQ_OK;
}

}  // namespace

extern "C" {

size_t fq_adamw_workspace_bytes(const fq_param *ps, int n)
{
    fq::Shape shape;
    return fq::shape_of(ps, n, shape) == FQ_OK ? shape.bytes : 0;
}

fq_status fq_adamw_create(const fq_param *ps, int n, void *workspace, size_t ws_bytes, void *hip_stream,
                          fq_adamw_plan **plan)
{
    if (!plan) return FQ_ERR_NULL;
    *plan = nullptr;
    fq_adamw_plan *p = new (std::nothrow) fq_adamw_plan();
    if (!p) return FQ_ERR_LAUNCH;
    fq_status st;
    try {
        st = fill(p, ps, n, workspace, ws_bytes, hip_stream);
    } catch (...) {
        st = FQ_ERR_LAUNCH;
    }
    if (st != FQ_OK) {
        delete p;
        return st;
    }
    *plan = p;
    return FQ_OK;
}

fq_status fq_adamw_step(const fq_adamw_plan *plan, const fq_adamw *h, void *hip_stream)
{
    if (!plan || !h) return FQ_ERR_NULL;
    if (h->step < 1 || !(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) ||
        !std::isfinite(h->lr) || !std::isfinite(h->eps) || h->eps < 0.0)
        return FQ_ERR_OPTIMIZER;
    if (!fq::aligned(h->grad_scale, 4)) return FQ_ERR_ALIGN;
    if (plan->shape.blocks == 0) return FQ_OK;
    fq::AdamwStep s;
    s.beta1 = (float)h->beta1;
    s.one_minus_beta1 = (float)(1.0 - h->beta1);
    s.beta2 = (float)h->beta2;
    s.one_minus_beta2 = (float)(1.0 - h->beta2);
    s.lr = (float)h->lr;
    s.lr_corrected = (float)(h->lr / (1.0 - std::pow(h->beta1, (double)h->step)));
    s.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
    s.eps = (float)h->eps;
    s.key = (unsigned)fq::mixed_key(h->seed, h->step);
    s.grad_scale = h->grad_scale;
    return fq::launch_adamw(plan->table, plan->first, plan->n, s, (unsigned)plan->shape.blocks, plan->shape.rows,
                            hip_stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
}

void fq_adamw_destroy(fq_adamw_plan *plan) { delete plan; }

}  // extern "C"
