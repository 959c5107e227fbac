// Dropout whose mask is never stored (declared in include/fq.h).
//
//   y_i = (h_i >> 1 >= round(p 2^31) ? x_i / (1 - p) : 0) + residual_i,   h_i a hash of i under two keys of seed and step
//
// Bound by memory: x (and the residual) are read once, y is written once: 36.9M FP16 values with a residual (221 MB) take 39 us, 5.6 TB/s.
// The hash is two 32-bit products and six other instructions, all at the full rate; with the rest an element costs some fifteen, which
// are 480 cycles of a SIMD for a wavefront's 512 elements, where memory takes 1350 (FP16 with a residual).
#include "fq_dropout.h"
#include "fq_rows.h"

namespace fq {
namespace {

using namespace dev;

struct Keys {
    unsigned first, second;
};

__device__ __forceinline__ Keys keys_of(uint64_t seed, uint64_t step, unsigned high)
{
    uint64_t k = seed * 0x9E3779B97F4A7C15ull + step * 0xD1B54A32D192ED03ull + high * 0x8CB92BA72F3D8DD7ull;
    k = (k ^ (k >> 32)) * 0x9E3779B97F4A7C15ull;
    k = (k ^ (k >> 29)) * 0xD1B54A32D192ED03ull;
    return {(unsigned)(k >> 32), (unsigned)(k ^ (k >> 32))};
}

__device__ __forceinline__ unsigned bits_of(unsigned place, const Keys &k)
{
    unsigned h = place * 0x9E3779B1u + k.first;
    h = (h ^ (h >> 16)) * 0x6A09E667u;
    h = ((h ^ (h >> 15)) + k.second) * 0xBB67AE85u;
    return h >> 1;
}

// x * scale as a binary32 value.  (The product and its conversion to FP16 would otherwise become one instruction, which rounds
// once where the definition rounds twice.)
__device__ __forceinline__ float scaled(float x, float scale)
{
    float v = x * scale;
    asm("" : "+v"(v));
    return v;
}

template <typename T> __device__ __forceinline__ Eight<T> ask(const T *p)
{
    Eight<T> r;
    __builtin_memcpy(&r, (const FQ_GLOBAL T *)p, sizeof r);
    return r;
}

// A thread has eight neighbouring elements, a block a run of 2048, all with the same upper 32 bits of their places.  (The 221 MB above:
// 39.2 us; 40.2 with sixteen elements a thread, 42.4 with 32; 41 to 43 with 1024 to 4096 blocks that go from run to run.  Stores
// past the caches make it 37.6, but then who reads y pays: a layer norm of the result of 16384 x 4096 128 us with it, 123 without.)
constexpr int kBlockElems = 256 * 8;
constexpr unsigned kMostAcross = 1u << 23;         // blocks along x: a grid has fewer than 2^32 threads along each of its sides

template <typename X, typename Y, bool ADD> __global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a)
{
    const long long begin = (long long)(blockIdx.y * gridDim.x + blockIdx.x) * kBlockElems;
    if (begin >= a.n) return;
    const X *x = (const X *)a.x + begin;
    const Y *r = (const Y *)a.residual + begin;
    Y *y = (Y *)a.y + begin;
    uint64_t step = a.step;
    if (a.step_on_device) step += *a.step_on_device;
    const Keys keys = keys_of(a.seed, step, (unsigned)((uint64_t)begin >> 32));
    const unsigned place = (unsigned)begin;
    const int left = a.n - begin < kBlockElems ? (int)(a.n - begin) : kBlockElems;
    const int at = (int)threadIdx.x * 8;
    if (at + 8 <= left) {
        const auto from = __builtin_bit_cast(typename Values<X>::type, ask(x + at));
        typename Values<Y>::type to;
        if constexpr (ADD) to = __builtin_bit_cast(typename Values<Y>::type, ask(r + at));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = bits_of(place + at + e, keys) >= a.threshold ? scaled((float)from[e], a.scale) : 0.0f;
            if constexpr (ADD) v += (float)to[e];
            to[e] = (Y)v;
        }
        __builtin_memcpy((FQ_GLOBAL Y *)(y + at), &to, sizeof to);
    } else {
        for (int i = at; i < left; ++i) {
            float v = bits_of(place + i, keys) >= a.threshold ? scaled((float)ld_global(x + i), a.scale) : 0.0f;
            if constexpr (ADD) v += (float)ld_global(r + i);
            st_global(y + i, (Y)v);
        }
    }
}

template <typename X, typename Y> int dropout(const DropoutArgs &a, hipStream_t stream)
{
    const unsigned runs = (unsigned)((a.n + kBlockElems - 1) / kBlockElems);       // 2^24 at most
    const dim3 blocks(runs < kMostAcross ? runs : kMostAcross, (runs + kMostAcross - 1) / kMostAcross);
    if (a.residual) dropout_kernel<X, Y, true><<<blocks, 256, 0, stream>>>(a);
    else dropout_kernel<X, Y, false><<<blocks, 256, 0, stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

int launch_dropout(const DropoutArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.x16) return a.y16 ? dropout<_Float16, _Float16>(a, s) : dropout<_Float16, float>(a, s);
    return a.y16 ? dropout<float, _Float16>(a, s) : dropout<float, float>(a, s);
}

}  // namespace fq
