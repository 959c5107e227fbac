// Device helpers of the kernels that work on rows of values: loads of eight at any address, the codes of a row, and loads straight into LDS.  Included by
// .hip files only; not part of the C ABI.
#pragma once
#include "fq_device.h"

namespace fq {
namespace dev {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Codes and scale of a row of x.
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// L lanes have a row, V vectors of eight values each: vectors l, l + L, l + 2 L, ... to lane l.  All of them are asked for at
// once, by loads that no lane branches round (any address will do; lanes without eight values take the row's first, which
// leaves its greatest magnitude as it is, and with k < 8, where a row need not have as many, all take zeros: with k = 0 they
// are the row).  An odd end is fetched value by value.
template <typename T> struct Eight { i32x4 w[sizeof(T) / 2]; };
template <typename T> struct Values { typedef T type __attribute__((ext_vector_type(8))); };

__constant__ const int kZeros[8] = {};

template <typename T> __device__ __forceinline__ Eight<T> ask8(const T *row, int at, int k)
{
    Eight<T> r;
    const T *p = k >= 8 ? row + (at + 8 <= k ? at : 0) : (const T *)kZeros;
    __builtin_memcpy(&r, (const FQ_GLOBAL T *)p, sizeof r);
    return r;
}

template <typename T> __device__ __forceinline__ void odd_end(Eight<T> &r, const T *row, int at, int k)
{
    if (k % 8 == 0 || at + 8 <= k) return;
    typename Values<T>::type h = (typename Values<T>::type)(T)0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < k) h[e] = ld_global(row + at + e);
    r = __builtin_bit_cast(Eight<T>, h);
}

// Greatest magnitude of the vectors, as the bits of a float (magnitudes order like their bits: numbers, infinity, NaN).
template <typename T, int V> __device__ __forceinline__ unsigned most_of(const Eight<T> (&r)[V])
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    unsigned most = 0;
    if constexpr (sizeof(T) == 2) {
        u16x2 both = (u16x2)(unsigned short)0;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) both = __builtin_elementwise_max(both, __builtin_bit_cast(u16x2, r[j].w[0][e] & 0x7FFF7FFF));
        const unsigned short half = both[0] > both[1] ? both[0] : both[1];
        most = __builtin_bit_cast(unsigned, (float)__builtin_bit_cast(_Float16, half));
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, (unsigned)r[j].w[e / 4][e % 4] & 0x7FFFFFFFu);
    }
    return most;
}

// The greatest of the 16 lanes' values that a row of the DPP unit holds, in all of them.
__device__ __forceinline__ unsigned max16(unsigned v)
{
    v = dpp_max<0xB1, 0xf>(v);
    v = dpp_max<0x4E, 0xf>(v);
    v = dpp_max<0x141, 0xf>(v);
    return dpp_max<0x140, 0xf>(v);
}

struct RowScale {
    float s, inverse;                  // inverse 0: the row's codes are 0
};

__device__ __forceinline__ RowScale row_scale(unsigned most)
{
    const float largest = __builtin_bit_cast(float, most);
    if (most >= 0x7F800000u) return {__builtin_nanf(""), 0.0f};
    if (largest < 127.0f * 0x1p-126f) return {0.0f, 0.0f};
    const float s = largest / 127.0f;
    return {s, 1.0f / s};
}

// Codes of eight values.  x * (1 / s) is within 127 * 2^-23 of the quotient x / s as it is rounded, so unless it lies that near
// to a half (a few vectors of a row) it rounds to the same integer.  Adding 1.5 * 2^23 rounds it, to even, and leaves the code
// in the low byte; the product is not rounded before (one instruction, FP16 operands and all).  No code leaves
// [-127, 127]: no |x| is over 127 * s * (1 + 2^-24).
template <typename T> __device__ __forceinline__ u32x2 codes8(const Eight<T> &r, RowScale scale, bool none)
{
    constexpr float kMagic = 0x1.8p23f;
    const auto v = __builtin_bit_cast(typename Values<T>::type, r);
    unsigned b[8];
    float near = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float f = __builtin_fmaf((float)v[e], scale.inverse, kMagic);
        b[e] = __builtin_bit_cast(unsigned, f);
        near = __builtin_fmaxf(near, __builtin_fabsf(__builtin_fmaf((float)v[e], scale.inverse, kMagic - f)));
    }
    if (near > 0.49995f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = __builtin_bit_cast(unsigned, (float)v[e] / scale.s + kMagic);
    }
    const auto pack = [](unsigned p, unsigned q, unsigned s, unsigned t) {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t, s, 0x0c0c0400u), __builtin_amdgcn_perm(q, p, 0x0c0c0400u), 0x05040100u);
    };
    u32x2 w = u32x2{pack(b[0], b[1], b[2], b[3]), pack(b[4], b[5], b[6], b[7])};
    if (none || scale.inverse == 0.0f) w = (u32x2)0u;
    return w;
}

#define FQ_LDS __attribute__((address_space(3)))

// 16 bytes per lane from `off` of a buffer to LDS, in lane order from `to` on (uniform).  No builtin: with one the compiler
// waits for all such loads in front of a read of LDS wherever it loses sight of which array they go to.  The kernel
// waits itself (as by loads_but); the compiler's own waits for other loads only become longer.
__device__ __forceinline__ void load_lds(i32x4 buffer, unsigned off, int8_t *to)
{
    const unsigned at = (unsigned)(uintptr_t)(FQ_LDS int8_t *)to;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(at), "v"(off), "s"(buffer) : "memory", "m0");
}

// The last LEFT loads of this wavefront may be on their way, all others and all its LDS reads are done.
template <int LEFT> __device__ __forceinline__ void loads_but()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(LEFT) : "memory");
}

}  // namespace dev
}  // namespace fq
