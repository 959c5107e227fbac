// Int8 linear layer with a scale per token and per channel (declared in include/fq.h).
#include <hip/hip_fp16.h>

#include "fq_device.h"
#include "fq_linear.h"

namespace fq {
namespace {

using namespace dev;

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------------------------
// Codes and scale of a row of x: a block per row, which reads it twice (the second time from the caches).
__device__ __forceinline__ unsigned wave_umax(unsigned v)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v = max(v, (unsigned)__shfl_xor((int)v, d));
    return v;
}

template <typename T>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a)
{
    __shared__ unsigned top[4];
    const long long row = blockIdx.x;
    const T *x = (const T *)a.x + row * a.ldx;
    unsigned most = 0;
    for (int i = threadIdx.x; i < a.k; i += 256)
        most = max(most, __builtin_bit_cast(unsigned, (float)ld_global(x + i)) & 0x7FFFFFFFu);
    most = wave_umax(most);
    if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = most;
    __syncthreads();
    most = max(max(top[0], top[1]), max(top[2], top[3]));
    const float largest = __builtin_bit_cast(float, most);
    const bool fine = most < 0x7F800000u;                    // no NaN and no infinity (magnitudes order like their bits)
    const bool zero = largest < 127.0f * 0x1p-126f;
    const float s = !fine ? __builtin_nanf("") : zero ? 0.0f : largest / 127.0f;
    if (threadIdx.x == 0) st_global(a.s + row, s);
    for (int i = threadIdx.x; i < a.pitch; i += 256) {
        float q = 0.0f;
        if (fine && !zero && i < a.k) q = __builtin_fminf(__builtin_fmaxf(__builtin_rintf((float)ld_global(x + i) / s), -127.0f), 127.0f);
        st_global(a.q + row * a.pitch + i, (int8_t)q);
    }
}

// ---------------------------------------------------------------------------------------------
// 16 codes of a row of k from l on; zeros behind its end.
__device__ __forceinline__ i32x4 load16(const int8_t *row, int l, int k)
{
    i32x4 r = {0, 0, 0, 0};
    if (l + 16 <= k) {
        __builtin_memcpy(&r, (const FQ_GLOBAL int8_t *)row + l, 16);
        return r;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (l + j < k) r[j / 4] |= (int)((unsigned)(unsigned char)ld_global(row + l + j) << (8 * (j % 4)));
    return r;
}

// A wavefront multiplies 16 channels by 16 tokens: lane l holds 16 codes of channel l % 16 and of token l % 16 for each
// matrix instruction, and of its sums those of token l % 16 and of channels 4 * (l / 16) to 4 * (l / 16) + 3.
__global__ __launch_bounds__(256) void linear_kernel(LinearArgs a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tiles_n = (a.n + 31) / 32;
    const int n0 = (int)(blockIdx.x % (unsigned)tiles_n) * 32 + (wave & 1) * 16;
    const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * 32 + (wave >> 1) * 16;
    const int8_t *w = a.w + (long long)min(n0 + lane % 16, a.n - 1) * a.ldw;
    const int8_t *x = a.x + (long long)min(m0 + lane % 16, a.m - 1) * a.ldx;
    i32x4 sum = {0, 0, 0, 0};
    for (int l = lane / 16 * 16; l - lane / 16 * 16 < a.k; l += 64)
        sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(load16(w, l, a.k), load16(x, l, a.k), sum, 0, 0, 0);
    const int i = m0 + lane % 16;
    if (i >= a.m) return;
    const float xs = ld_global(a.xs + (long long)i * a.xs_step);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int j = n0 + lane / 16 * 4 + r;
        if (j >= a.n) continue;
        float y = (float)sum[r] * (xs * ld_global(a.ws + (long long)j * a.ws_step));
        if (a.bias) y += ld_global(a.bias + j);
        if (a.y16) st_global((_Float16 *)a.y + (long long)i * a.ldy + j, (_Float16)y);
        else st_global((float *)a.y + (long long)i * a.ldy + j, y);
    }
}

}  // namespace

int launch_quantize_rows(const QuantizeArgs &a, void *stream)
{
    if (a.x16) quantize_rows_kernel<_Float16><<<(unsigned)a.m, 256, 0, (hipStream_t)stream>>>(a);
    else quantize_rows_kernel<float><<<(unsigned)a.m, 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

int launch_linear(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)((a.n + 31) / 32) * (unsigned)((a.m + 31) / 32);
    linear_kernel<<<blocks, 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace fq
