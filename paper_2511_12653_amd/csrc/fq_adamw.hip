// AdamW over a list of tensors in one launch, moments in FP32 or in FP8 (declared in include/fq.h).
//
//   m' = beta1 m + (1 - beta1) g,  v' = beta2 v + (1 - beta2) g^2,  p' = p (1 - lr wd) - lr / (1 - beta1^t) m' / (sqrt(v') /
//   sqrt(1 - beta2^t) + eps)
//
// Every element is read and written once and depends on no other; in FP8 the 256 elements of a state block share a scale, which is known
// when all their new moments are.  Hence a state block to a wavefront, four elements to a lane: the block's greatest moments are one
// reduction in registers, and no LDS or barrier is needed.  A grid block has one tensor, so all branches on types are uniform.
//
// With FP32 states memory bounds it: 120 million elements 544 us, 6.2 TB/s.  In FP8 it is memory too where the elements have many
// bytes (240 million, FP32 p, FP16 g and copy: 16 bytes each, 640 us, 6.0 TB/s), and arithmetic where they have few (20 million in FP16: 10
// bytes each, 43 to 45 us, 4.5 TB/s).  Short lists cost the launch and a trip to memory or two (88 tensors, 0.4 million elements: 4.2 us).
#include <hip/hip_fp16.h>

#include "fq_adamw.h"
#include "fq_device.h"

namespace fq {
namespace {

using namespace dev;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef unsigned char u8x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Four;
template <> struct Four<float> { typedef f32x4 type; };
template <> struct Four<_Float16> { typedef f16x4 type; };
template <> struct Four<unsigned char> { typedef u8x4 type; };

// Elements i to i + 3 of a tensor that has `left` of them from i on; zeros behind its end.
template <typename T> __device__ __forceinline__ typename Four<T>::type load4(const void *base, long long i, bool vec, long long left)
{
    typedef typename Four<T>::type V;
    const T *p = (const T *)base + i;
    V r = (V)(T)0;
    if (vec && left >= 4) return ld_stream((const V *)p);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) r[j] = ld_global(p + j);
    return r;
}

template <typename T> __device__ __forceinline__ void store4(void *base, long long i, bool vec, long long left, typename Four<T>::type r)
{
    typedef typename Four<T>::type V;
    T *p = (T *)base + i;
    if (vec && left >= 4) {
        st_stream((V *)p, r);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) st_global(p + j, (T)r[j]);
}

// The greater of each 16-bit half, over the wavefront.
template <int CTRL, int ROW_MASK> __device__ __forceinline__ unsigned max_step(unsigned v)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    const unsigned w = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, false);
    return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, v), __builtin_bit_cast(u16x2, w)));
}

__device__ __forceinline__ unsigned halves_max(unsigned v)
{
    v = max_step<0xB1, 0xf>(v);
    v = max_step<0x4E, 0xf>(v);
    v = max_step<0x141, 0xf>(v);
    v = max_step<0x140, 0xf>(v);
    v = max_step<0x142, 0xa>(v);
    v = max_step<0x143, 0xc>(v);
    return (unsigned)__builtin_amdgcn_readlane((int)v, kSumLane);
}

constexpr unsigned kPlace = 0x9E3779B1u;          // x = place * kPlace + key is what is mixed

__device__ __forceinline__ unsigned mix(unsigned x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}

// The e4m3 value at or below a (0 <= a <= 448) raised by (u + 1/2) / 2^16 of the step between codes: adding that
// to the 20 mantissa bits that a code lacks, and cutting them off.  Below 2^-6 the steps stay those of the binade
// above, where adding 2^-6 puts a.  more: 16 u + 8.  near: the least distance, plus 2, of the sums from a multiple of 2^20 so far.
__device__ __forceinline__ float round_code(float a, unsigned more, unsigned &near)
{
    const float low = a < 0x1p-6f ? 0x1p-6f : 0.0f;
    const unsigned z = __builtin_bit_cast(unsigned, a + low) + more, far = (z + 2u) & 0xFFFFFu;
    near = near < far ? near : far;
    return __builtin_bit_cast(float, z & 0xFFF00000u) - low;
}

__device__ __forceinline__ unsigned pack4(const float *c)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
}

__device__ __forceinline__ void unpack4(u8x4 codes, float *c)
{
    const int w = __builtin_bit_cast(int, codes);
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    c[0] = a[0]; c[1] = a[1]; c[2] = b[0]; c[3] = b[1];
}

__device__ __forceinline__ float power_of_two(int e) { return __builtin_bit_cast(float, (unsigned)(e + 127) << 23); }

// A grid block's ROWS rows of one tensor.  All loads go out before the first use.
template <typename P, typename G, bool F8, int ROWS>
__device__ __forceinline__ void step_rows(const AdamwTensor &t, const AdamwStep &s, float gs, unsigned chunk)
{
    typedef typename Four<P>::type P4;
    typedef typename Four<G>::type G4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool vec = t.vec;
    const float lr = s.lr * t.lr_scale, lrc = s.lr_corrected * t.lr_scale, keep = 1.0f - lr * t.weight_decay;

    P4 p4[ROWS];
    G4 g4[ROWS];
    f32x4 mf[ROWS], vf[ROWS];
    u8x4 m8[ROWS], v8[ROWS];
    float ms[ROWS], vs[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long block = ((long long)chunk * ROWS + r) * (kAdamwRowElems / kStateBlock) + wave;
        const long long i = block * kStateBlock + 4 * lane, left = t.n - i;
        if (block * kStateBlock >= t.n) continue;
        p4[r] = load4<P>(t.p, i, vec, left);
        g4[r] = load4<G>(t.g, i, vec, left);
        if (F8) {
            ms[r] = ld_global(t.m_scale + block);
            vs[r] = ld_global(t.v_scale + block);
            m8[r] = load4<unsigned char>(t.m, i, vec, left);
            v8[r] = load4<unsigned char>(t.v, i, vec, left);
        } else {
            mf[r] = load4<float>(t.m, i, vec, left);
            vf[r] = load4<float>(t.v, i, vec, left);
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long block = ((long long)chunk * ROWS + r) * (kAdamwRowElems / kStateBlock) + wave;
        const long long i = block * kStateBlock + 4 * lane, left = t.n - i;
        if (block * kStateBlock >= t.n) continue;
        if constexpr (!F8) {
            P4 pn;
            f16x4 copy;
            f32x4 mn, vn;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = (float)g4[r][j] * gs, m0 = mf[r][j], v0 = vf[r][j], p0 = (float)p4[r][j];
                const float m1 = s.beta1 * m0 + s.one_minus_beta1 * g;
                const float v1 = s.beta2 * v0 + (s.one_minus_beta2 * g) * g;
                const bool fine = __builtin_fabsf(v1) < __builtin_inff();
                mn[j] = fine ? m1 : m0;
                vn[j] = fine ? v1 : v0;
                const float p1 = p0 * keep - lrc * (m1 / (__builtin_sqrtf(v1) * s.root_factor + s.eps));
                const float p = fine ? p1 : p0;
                pn[j] = (P)p;
                copy[j] = (_Float16)p;
            }
            store4<P>(t.p, i, vec, left, pn);
            if (t.p16) store4<_Float16>(t.p16, i, vec, left, copy);
            store4<float>(t.m, i, vec, left, mn);
            store4<float>(t.v, i, vec, left, vn);
            continue;
        }
        // What bounds this is the arithmetic (about 75 instructions an element; with the compiler's root and quotient, a
        // guard per element and four products to a hash it was 114: 20 million FP16 elements 53 us, now 43 to 45).
        float m[4], v[4];
        unsigned both;
        auto moments = [&](bool guarded) {
            unpack4(m8[r], m);
            unpack4(v8[r], v);
            unsigned am = 0, av = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = (float)g4[r][j] * gs, m0 = m[j] * ms[r], r0 = v[j] * vs[r], v0 = r0 * r0;
                m[j] = s.beta1 * m0 + s.one_minus_beta1 * g;
                v[j] = s.beta2 * v0 + (s.one_minus_beta2 * g) * g;
                if (guarded && !(__builtin_fabsf(v[j]) < __builtin_inff())) {
                    m[j] = m0;
                    v[j] = v0;
                }
                am = max(am, __builtin_bit_cast(unsigned, m[j]) & 0x7FFFFFFFu);
                av = max(av, __builtin_bit_cast(unsigned, v[j]) & 0x7FFFFFFFu);
            }
            // exponents (biased) of the least powers of two that reach the greatest |m| / 1.75 and v / 1.53125: the
            // mantissas of 448 = 1.75 * 2^8 and of 448^2 = 1.53125 * 2^17
            both = halves_max(((am + 0x1FFFFFu) >> 23) | ((av + 0x3BFFFFu) >> 23) << 16);
        };
        moments(false);
        const bool odd = both >> 16 >= 255u;                    // some v is not finite
        if (odd) moments(true);
        const int em = max((int)(both & 0xFFFFu) - 127 - 8, -126);
        const int e2 = max((int)(both >> 16) - 127 - 17, -126);
        const int ev = (e2 + 1) >> 1;
        const float down_m = power_of_two(-em), down_v = power_of_two(-2 * ev), up = power_of_two(ev) * s.root_factor;
        const unsigned place = (t.place + (unsigned)i) * kPlace + s.key;
        float cm[4], cv[4];
        P4 pn;
        f16x4 copy;
        unsigned near = ~0u, nothing = 0;
        // The root in units of the scale: the rounding of a scaled number is that of the number.
        auto codes = [&](int j, float root) {
            const unsigned bits = mix(place + (unsigned)j * kPlace);
            cm[j] = __builtin_copysignf(round_code(__builtin_fabsf(m[j]) * down_m, (bits & 0xFFFFu) << 4 | 8u, nothing), m[j]);
            cv[j] = __builtin_fmaxf(round_code(root, (bits >> 12 & 0xFFFF0u) | 8u, near), v[j] > 0.0f ? 0x1p-9f : 0.0f);
        };
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float root = __builtin_amdgcn_sqrtf(v[j] * down_v);
            const float p = (float)p4[r][j] * keep - lrc * (m[j] * __builtin_amdgcn_rcpf(root * up + s.eps));
            pn[j] = (P)p;
            copy[j] = (_Float16)p;
            codes(j, root);
        }
        // The hardware's root is one unit off at most.  Where that may make another code, which has to follow from the
        // rounded root alone, it is worked out again; few wavefronts are.  So they are where the greatest v is large or eps tiny: a
        // root over 2^62 times smaller than the greatest is lost in the units, which otherwise does not matter beside eps.
        if (__builtin_expect(odd || !(up * 0x1p-62f <= s.eps * 0x1p-26f) || __ballot(near <= 4u), 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float g = (float)g4[r][j] * gs, p0 = (float)p4[r][j];
                float m0[4], v0[4];
                unpack4(m8[r], m0);
                unpack4(v8[r], v0);
                const float r0 = v0[j] * vs[r], v1 = s.beta2 * (r0 * r0) + (s.one_minus_beta2 * g) * g;
                const float root = __builtin_sqrtf(v[j]);
                float p = p0 * keep - lrc * (m[j] / (root * s.root_factor + s.eps));
                if (!(__builtin_fabsf(v1) < __builtin_inff())) p = p0;    // (a gradient that was not finite leaves no trace in m and v)
                pn[j] = (P)p;
                copy[j] = (_Float16)p;
                codes(j, __builtin_sqrtf(v[j] * down_v));
            }
        }
        store4<P>(t.p, i, vec, left, pn);
        if (t.p16) store4<_Float16>(t.p16, i, vec, left, copy);
        store4<unsigned char>(t.m, i, vec, left, __builtin_bit_cast(u8x4, pack4(cm)));
        store4<unsigned char>(t.v, i, vec, left, __builtin_bit_cast(u8x4, pack4(cv)));
        if (lane == 0) {
            st_global(t.m_scale + block, power_of_two(em));
            st_global(t.v_scale + block, power_of_two(ev));
        }
    }
}

// The tensor of a grid block: the last whose first block is not behind it.  Every wavefront looks at 64 first blocks
// at a time, an even sample of those still in question, so one look for up to 64 tensors and two for up to 4096.
__device__ __forceinline__ unsigned find_tensor(const unsigned *first, unsigned n, unsigned block)
{
    const unsigned lane = threadIdx.x & 63;
    unsigned begin = 0, count = n;
    for (;;) {
        const unsigned stride = (count + 63) / 64, at = begin + lane * stride;
        const bool before = lane * stride < count && ld_global(first + at) <= block;
        const unsigned ahead = (unsigned)__popcll(__ballot(before));   // lane 0 is always among them
        if (stride == 1) return begin + ahead - 1;
        begin += (ahead - 1) * stride;
        count = min(stride, n - begin);
    }
}

__device__ __forceinline__ AdamwTensor descriptor(const AdamwTensor *p)
{
    unsigned w[sizeof(AdamwTensor) / 4];
#pragma unroll
    for (unsigned i = 0; i < sizeof w / sizeof w[0]; ++i) w[i] = ld_uniform((const unsigned *)p + i);
    AdamwTensor t;
    __builtin_memcpy(&t, w, sizeof t);
    return t;
}

// FIND: the table has a descriptor per tensor, else one per grid block.
template <int ROWS, bool FIND>
__global__ __launch_bounds__(kAdamwThreads) void adamw_kernel(const AdamwTensor *table, const unsigned *first, unsigned n, AdamwStep s)
{
    const unsigned which = FIND ? __builtin_amdgcn_readfirstlane(find_tensor(first, n, blockIdx.x)) : blockIdx.x;
    const AdamwTensor t = descriptor(table + which);
    const float gs = s.grad_scale ? ld_uniform(s.grad_scale) : 1.0f;
    const unsigned chunk = blockIdx.x - t.first;
    switch (t.p16_type | t.g16_type << 1 | t.f8 << 2) {
    case 0: return step_rows<float, float, false, ROWS>(t, s, gs, chunk);
    case 1: return step_rows<_Float16, float, false, ROWS>(t, s, gs, chunk);
    case 2: return step_rows<float, _Float16, false, ROWS>(t, s, gs, chunk);
    case 3: return step_rows<_Float16, _Float16, false, ROWS>(t, s, gs, chunk);
    case 4: return step_rows<float, float, true, ROWS>(t, s, gs, chunk);
    case 5: return step_rows<_Float16, float, true, ROWS>(t, s, gs, chunk);
    case 6: return step_rows<float, _Float16, true, ROWS>(t, s, gs, chunk);
    default: return step_rows<_Float16, _Float16, true, ROWS>(t, s, gs, chunk);
    }
}

}  // namespace

int launch_adamw(const AdamwTensor *table, const unsigned *first, int n, const AdamwStep &s, unsigned blocks, int rows,
                 void *stream)
{
    if (!first) adamw_kernel<1, false><<<blocks, kAdamwThreads, 0, (hipStream_t)stream>>>(table, first, (unsigned)n, s);
    else if (rows == 1) adamw_kernel<1, true><<<blocks, kAdamwThreads, 0, (hipStream_t)stream>>>(table, first, (unsigned)n, s);
    else adamw_kernel<2, true><<<blocks, kAdamwThreads, 0, (hipStream_t)stream>>>(table, first, (unsigned)n, s);
    return (int)hipGetLastError();
}

}  // namespace fq
