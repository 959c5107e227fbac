// Low-rank adapters of many requests beside a shared layer (declared in include/fq.h).
//
//   t = x a^T (* xs),   y = base + scale * t b^T      a, b: those of the token's adapter
#include "fq_adapters.h"
#include "fq_rows.h"

namespace fq {
namespace {

using namespace dev;

// A token to a block, a rank at a time to each of its wavefronts.
template <typename X> __global__ __launch_bounds__(256) void adapter_down_kernel(AdapterArgs a)
{
    const int token = blockIdx.x, id = a.ids[token], lane = threadIdx.x & 63;
    if (id < 0 || id >= a.count) return;
    const X *x = (const X *)a.x + token * a.ldx;
    const float xs = a.xs ? a.xs[(long long)token * a.xs_step] : 1.0f;
    for (int l = threadIdx.x >> 6; l < a.rank; l += 4) {
        const _Float16 *row = (const _Float16 *)a.a + ((long long)id * a.rank + l) * a.k;
        double s = 0.0;
        for (int i = lane; i < a.k; i += 64) s += (double)(float)ld_global(x + i) * (double)(float)ld_global(row + i);
        s = wave_sum(s);
        if (lane == kSumLane) st_global(a.t + (long long)token * a.rank + l, (float)(s * xs));
    }
}

// A token and 256 channels to a block.
template <typename Y, typename B> __global__ __launch_bounds__(256) void adapter_up_kernel(AdapterArgs a, int strips)
{
    const int token = blockIdx.x / strips, j = blockIdx.x % strips * 256 + threadIdx.x, id = a.ids[token];
    if (j >= a.n) return;
    float y = a.base ? (float)ld_global((const B *)a.base + token * a.ldbase + j) : 0.0f;
    if (id >= 0 && id < a.count) {
        const _Float16 *row = (const _Float16 *)a.b + ((long long)id * a.n + j) * a.rank;
        const float *t = a.t + (long long)token * a.rank;
        float s = 0.0f;
        for (int l = 0; l < a.rank; ++l) s = __builtin_fmaf(ld_global(t + l), (float)ld_global(row + l), s);
        y += (a.scale ? a.scale[id] : 1.0f) * s;
    }
    st_global((Y *)a.y + token * a.ldy + j, (Y)y);
}

}  // namespace

int launch_adapters(const AdapterArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.count > 0) {
        if (a.x_type == 0) adapter_down_kernel<_Float16><<<a.m, 256, 0, s>>>(a);
        else if (a.x_type == 1) adapter_down_kernel<float><<<a.m, 256, 0, s>>>(a);
        else adapter_down_kernel<int8_t><<<a.m, 256, 0, s>>>(a);
        const int err = (int)hipGetLastError();
        if (err != 0) return err;
    }
    const int strips = (a.n + 255) / 256;
    const unsigned blocks = (unsigned)a.m * (unsigned)strips;
    if (a.y16) {
        if (a.base16) adapter_up_kernel<_Float16, _Float16><<<blocks, 256, 0, s>>>(a, strips);
        else adapter_up_kernel<_Float16, float><<<blocks, 256, 0, s>>>(a, strips);
    } else {
        if (a.base16) adapter_up_kernel<float, _Float16><<<blocks, 256, 0, s>>>(a, strips);
        else adapter_up_kernel<float, float><<<blocks, 256, 0, s>>>(a, strips);
    }
    return (int)hipGetLastError();
}

}  // namespace fq
