// Layer norm over rows, forward and backward, and with codes for the int8 linear layer (declared in include/fq.h).
//
//   mean = sum x / k,  rstd = 1 / sqrt(sum (x - mean)^2 / k + eps),  h = (x - mean) rstd,  y = h w + b
//   a = gy w,  gx = rstd (a - sum a / k - h sum a h / k),  gw = sum over rows of gy h,  gb = sum over rows of gy
//
// Bound by memory: x is read once and y written once, x and gy read once and gx written once.  So a row stays in registers from its
// load to its store.  Its two sums are taken together, of e = x - x0 and e^2 with x0 the row's first value, in binary64:
//   mean = x0 + S1 / k,   sum (x - mean)^2 = S2 - S1^2 / k
// is right to 2^-52 (1 + (mean - x0)^2 / var), so one reduction over the lanes does where mean and deviation one after the other take
// two.  (binary64 additions run at the rate of binary32 ones here.)
#include <type_traits>

#include "fq_norm.h"
#include "fq_rows.h"

namespace fq {
namespace {

using namespace dev;

typedef double f64x2 __attribute__((ext_vector_type(2)));

// Another lane's value (every lane has one, so nothing has to be there before).
template <int CTRL> __device__ __forceinline__ double from_lane(double v)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    i32x2 w = __builtin_bit_cast(i32x2, v);
    w[0] = __builtin_amdgcn_mov_dpp(w[0], CTRL, 0xf, 0xf, true);
    w[1] = __builtin_amdgcn_mov_dpp(w[1], CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, w);
}

// The sum over 16 lanes, in all of them.
__device__ __forceinline__ double sum16(double v)
{
    v += from_lane<0xB1>(v);
    v += from_lane<0x4E>(v);
    v += from_lane<0x141>(v);
    return v + from_lane<0x140>(v);
}

// The sums of both values over a wavefront, a's in lanes 0 to 31 and b's in the others: the first step leaves one value to a lane.
__device__ __forceinline__ double wave_sums(double a, double b)
{
    typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
    u32x2 p = __builtin_bit_cast(u32x2, a), q = __builtin_bit_cast(u32x2, b);
    auto low = __builtin_amdgcn_permlane32_swap(p[0], q[0], false, false);
    auto high = __builtin_amdgcn_permlane32_swap(p[1], q[1], false, false);
    const double v = __builtin_bit_cast(double, u32x2{low[0], high[0]}) + __builtin_bit_cast(double, u32x2{low[1], high[1]});
    p = __builtin_bit_cast(u32x2, v);
    low = __builtin_amdgcn_permlane16_swap(p[0], p[0], false, false);
    high = __builtin_amdgcn_permlane16_swap(p[1], p[1], false, false);
    return sum16(__builtin_bit_cast(double, u32x2{low[0], high[0]}) + __builtin_bit_cast(double, u32x2{low[1], high[1]}));
}

__device__ __forceinline__ double lane_value(double v, int lane)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    i32x2 w = __builtin_bit_cast(i32x2, v);
    w[0] = __builtin_amdgcn_readlane(w[0], lane);
    w[1] = __builtin_amdgcn_readlane(w[1], lane);
    return __builtin_bit_cast(double, w);
}

// What the wavefronts of a row that has more than one hand each other: each sum has its place, and two of them, which the rows take
// in turn, so that one barrier is enough.
template <int L> struct Shared {
    f64x2 sums[2][L / 64];
    unsigned most[2][L / 64];
};
template <> struct Shared<16> {};
template <> struct Shared<64> {};

// Sums of both values over the L lanes of a row, in all of them.
template <int L> __device__ __forceinline__ void row_sums(double &a, double &b, Shared<L> &s, int turn)
{
    if constexpr (L == 16) {
        a = sum16(a);
        b = sum16(b);
    } else {
        const double v = wave_sums(a, b);
        if constexpr (L == 64) {
            a = lane_value(v, 0);
            b = lane_value(v, 32);
        } else {
            if ((threadIdx.x & 31) == 0) ((double *)&s.sums[turn][threadIdx.x >> 6])[threadIdx.x >> 5 & 1] = v;
            __syncthreads();
            f64x2 sum = s.sums[turn][0];
#pragma unroll
            for (int i = 1; i < L / 64; ++i) sum += s.sums[turn][i];
            a = sum[0];
            b = sum[1];
        }
    }
}

template <int L> __device__ __forceinline__ unsigned row_most(unsigned v, Shared<L> &s, int turn)
{
    if constexpr (L == 16) return max16(v);
    v = wave_max(v);
    if constexpr (L > 64) {
        if ((threadIdx.x & 63) == 0) s.most[turn][threadIdx.x >> 6] = v;
        __syncthreads();
        v = s.most[turn][0];
#pragma unroll
        for (int i = 1; i < L / 64; ++i) v = max(v, s.most[turn][i]);
    }
    return v;
}

// The places behind a row's end (of a vector that begins at `at`) take `value`.
template <typename T> __device__ __forceinline__ void fill_end(Eight<T> &r, int at, int k, T value)
{
    if (at + 8 <= k) return;
    auto v = __builtin_bit_cast(typename Values<T>::type, r);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e >= k) v[e] = value;
    r = __builtin_bit_cast(Eight<T>, v);
}

// Eight values of a row, `value` behind its end.
template <typename T> __device__ __forceinline__ Eight<T> load8(const T *row, int at, int k, T value)
{
    Eight<T> r = ask8(row, at, k);
    odd_end(r, row, at, k);
    fill_end(r, at, k, value);
    return r;
}

template <typename T> __device__ __forceinline__ void store8(T *row, int at, int k, const float *y)
{
    if (at + 8 <= k) {
        typename Values<T>::type v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (T)y[e];
        __builtin_memcpy((FQ_GLOBAL T *)(row + at), &v, sizeof v);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < k) st_global(row + at + e, (T)y[e]);
}

__device__ __forceinline__ void store_codes(int8_t *row, int at, int k, u32x2 q)
{
    if (at + 8 <= k) {
        __builtin_memcpy((FQ_GLOBAL int8_t *)(row + at), &q, sizeof q);
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < k) st_global(row + at + e, (int8_t)(q[e / 4] >> (8 * (e % 4))));
}

// Eight weights or biases; `none` where there are none, 0 behind the end.
__device__ __forceinline__ void weights8(float *to, const void *from, int at, int k, int w16, float none)
{
    if (!from) {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = at + e < k ? none : 0.0f;
    } else if (w16) {
        const auto v = __builtin_bit_cast(Values<_Float16>::type, load8((const _Float16 *)from, at, k, (_Float16)0.0f));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = (float)v[e];
    } else {
        const auto v = __builtin_bit_cast(Values<float>::type, load8((const float *)from, at, k, 0.0f));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = v[e];
    }
}

struct Moments {
    double mean, rstd;
    float high, low, scale;          // mean as a sum of two floats; rstd
};

// 1 / sqrt(v): the hardware's, right to 2^-24 or so, and two of Newton's steps.
__device__ __forceinline__ double reciprocal_root(double v)
{
    double r = __builtin_amdgcn_rsq(v);
    const double half = 0.5 * v;
#pragma unroll
    for (int i = 0; i < 2; ++i) r = __builtin_fma(r, __builtin_fma(-half * r, r, 0.5), r);
    return v == 0.0 ? __builtin_inf() : r;
}

// inverse: 1 / k
__device__ __forceinline__ Moments moments(double x0, double s1, double s2, double inverse, float eps)
{
    const double off = s1 * inverse;
    double var = (s2 - s1 * off) * inverse;
    if (var < 0.0) var = 0.0;                      // (rounding; a NaN stays)
    const double mean = x0 + off, rstd = reciprocal_root(var + (double)eps);
    const float high = (float)mean;
    return {mean, rstd, high, (float)(mean - (double)high), (float)rstd};
}

template <typename X> __device__ __forceinline__ void add_moments(const Eight<X> &r, float x0, double &s1, double &s2)
{
    const auto x = __builtin_bit_cast(typename Values<X>::type, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double d = (double)(float)x[e] - (double)x0;
        s1 += d;
        s2 = __builtin_fma(d, d, s2);
    }
}

// y of eight values.  EXACT: in binary64, rounded once, since a value next to the border of two codes decides between them.  Else in
// binary32, where x - mean is right to half a step (the mean comes in two parts, so that it is also where the row lies far from zero) and
// no conversions to binary64 and back, of twice the cycles of other instructions, are needed.
template <bool EXACT, typename X>
__device__ __forceinline__ void normed(float *y, const Eight<X> &r, const Moments &m, const float *w, const float *b)
{
    const auto x = __builtin_bit_cast(typename Values<X>::type, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (EXACT) y[e] = (float)__builtin_fma(((double)(float)x[e] - m.mean) * m.rstd, (double)w[e], (double)b[e]);
        else y[e] = __builtin_fmaf((((float)x[e] - m.high) - m.low) * m.scale, w[e], b[e]);
    }
}

// Where a lane's vector of eight values lies in a row that is held: vector i of k values begins at 8 i, the last one at k - 8, so that all
// loads and stores are whole vectors at any address.  `twice` of its first values are the vector's before, too: they are worked out and
// stored by both lanes, to the same bits, and are taken out of the sums again.
struct Place {
    int at, twice;
    bool there;
};

__device__ __forceinline__ Place place_of(int i, int k)
{
    const int at = i * 8, over = max(at + 8 - k, 0);
    return {at - over, over, at < k};
}

template <typename T> __device__ __forceinline__ Eight<T> held8(const T *row, int at)
{
    Eight<T> r;
    __builtin_memcpy(&r, (const FQ_GLOBAL T *)(row + at), sizeof r);
    return r;
}

template <typename T> __device__ __forceinline__ void put8(T *row, int at, const float *y)
{
    typename Values<T>::type v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (T)y[e];
    __builtin_memcpy((FQ_GLOBAL T *)(row + at), &v, sizeof v);
}

__device__ __forceinline__ void put_codes(int8_t *row, int at, u32x2 q) { __builtin_memcpy((FQ_GLOBAL int8_t *)(row + at), &q, sizeof q); }

__device__ __forceinline__ Eight<float> as_eight(const float *y)
{
    Eight<float> r;
    __builtin_memcpy(&r, y, sizeof r);
    return r;
}

__device__ __forceinline__ void held_weights(float *to, const void *from, int at, int w16, float none)
{
    if (!from) {
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = none;
    } else if (w16) {
        const auto v = __builtin_bit_cast(Values<_Float16>::type, held8((const _Float16 *)from, at));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = (float)v[e];
    } else {
        const auto v = __builtin_bit_cast(Values<float>::type, held8((const float *)from, at));
#pragma unroll
        for (int e = 0; e < 8; ++e) to[e] = v[e];
    }
}

// A row of 8 to 8 L V values to L lanes, V vectors to each; weight and bias stay in registers while the block goes from row to row, and
// the next row is on its way while this one is worked on.
template <typename X, typename Y, int L, int V>
__global__ __launch_bounds__(norm_threads(L)) void norm_forward_kernel(NormArgs a)
{
    constexpr int kRows = norm_threads(L) / L;
    constexpr bool kCodes = std::is_same<Y, int8_t>::value;
    __shared__ Shared<L> shared;
    const int lane = (int)threadIdx.x % L, k = a.width;
    Place p[V];
    float w[V][8], b[V][8];
    const long long stride = (long long)gridDim.x * kRows, sub = threadIdx.x / L;
    long long first = (long long)blockIdx.x * kRows;
    const auto row_at = [&](long long f) { return (const X *)a.x + min(f + sub, a.rows - 1) * a.ldx; };
    const X *x = row_at(first);
    Eight<X> next[V];
    X begin_next = ld_global(x);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        p[j] = place_of(j * L + lane, k);
        next[j] = held8(x, p[j].there ? p[j].at : 0);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        held_weights(w[j], a.w, p[j].there ? p[j].at : 0, a.w16, 1.0f);
        held_weights(b[j], a.b, p[j].there ? p[j].at : 0, a.w16, 0.0f);
    }
    int turn = 0;
    for (; first < a.rows; first += stride) {
        const long long row = first + sub;
        const bool there = row < a.rows;
        Eight<X> raw[V];
        const float begin = (float)begin_next;
#pragma unroll
        for (int j = 0; j < V; ++j) raw[j] = next[j];
        if (first + stride < a.rows) {
            x = row_at(first + stride);
            begin_next = ld_global(x);
#pragma unroll
            for (int j = 0; j < V; ++j) next[j] = held8(x, p[j].there ? p[j].at : 0);
        }
        double s1 = 0.0, s2 = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!p[j].there) continue;
            add_moments(raw[j], begin, s1, s2);
            if (p[j].twice) {
                const auto v = __builtin_bit_cast(typename Values<X>::type, raw[j]);
#pragma unroll
                for (int e = 0; e < 7; ++e) {
                    const double d = e < p[j].twice ? (double)(float)v[e] - (double)begin : 0.0;
                    s1 -= d;
                    s2 = __builtin_fma(-d, d, s2);
                }
            }
        }
        row_sums<L>(s1, s2, shared, turn);
        const Moments m = moments((double)begin, s1, s2, a.inverse, a.eps);
        if (a.stats && there && lane == 0) {
            st_global(a.stats + 2 * row, (float)m.mean);
            st_global(a.stats + 2 * row + 1, (float)m.rstd);
        }
        float y[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j) normed<kCodes>(y[j], raw[j], m, w[j], b[j]);
        if constexpr (!kCodes) {
            Y *to = (Y *)a.y + row * a.ldy;
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (there && p[j].there) put8(to, p[j].at, y[j]);
        } else {
            Eight<float> held[V];
            unsigned most = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                held[j] = as_eight(y[j]);
                Eight<float> one[1] = {held[j]};
                if (p[j].there) most = max(most, most_of(one));
            }
            const RowScale r = row_scale(row_most<L>(most, shared, turn));
            if (there && lane == 0) st_global(a.ys + row, r.s);
            int8_t *to = (int8_t *)a.y + row * a.ldy;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const u32x2 q = codes8(held[j], r, false);
                if (there && p[j].there) put_codes(to, p[j].at, q);
            }
        }
        turn ^= 1;
    }
}

// A row of any width to L lanes: V vectors of eight values to each, and of what is more read again from the caches.
template <typename X, typename Y, int L, int V>
__global__ __launch_bounds__(norm_threads(L)) void norm_forward_any_kernel(NormArgs a)
{
    constexpr int kRows = norm_threads(L) / L, kHeld = 8 * L * V;
    constexpr bool kCodes = std::is_same<Y, int8_t>::value;
    __shared__ Shared<L> shared;
    const int at = (int)threadIdx.x % L * 8, k = a.width;
    float w[V][8], b[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        weights8(w[j], a.w, j * L * 8 + at, k, a.w16, 1.0f);
        weights8(b[j], a.b, j * L * 8 + at, k, a.w16, 0.0f);
    }
    int turn = 0;
    for (long long first = (long long)blockIdx.x * kRows; first < a.rows; first += (long long)gridDim.x * kRows) {
        const long long row = first + threadIdx.x / L;
        const bool there = row < a.rows;
        const long long from = there ? row : a.rows - 1;
        const X *x = (const X *)a.x + from * a.ldx;
        const X begin = ld_global(x);
        Eight<X> raw[V];
#pragma unroll
        for (int j = 0; j < V; ++j) raw[j] = ask8(x, j * L * 8 + at, k);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            odd_end(raw[j], x, j * L * 8 + at, k);
            fill_end(raw[j], j * L * 8 + at, k, begin);
        }
        double s1 = 0.0, s2 = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) add_moments(raw[j], (float)begin, s1, s2);
        for (int i = kHeld + at; i < k; i += L * 8) add_moments(load8(x, i, k, begin), (float)begin, s1, s2);
        row_sums<L>(s1, s2, shared, turn);
        const Moments m = moments((double)(float)begin, s1, s2, a.inverse, a.eps);
        if (a.stats && there && at == 0) {
            st_global(a.stats + 2 * row, (float)m.mean);
            st_global(a.stats + 2 * row + 1, (float)m.rstd);
        }
        float y[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j) normed<kCodes>(y[j], raw[j], m, w[j], b[j]);
        if constexpr (!kCodes) {
            if (there) {
                Y *to = (Y *)a.y + row * a.ldy;
#pragma unroll
                for (int j = 0; j < V; ++j) store8(to, j * L * 8 + at, k, y[j]);
                for (int i = kHeld + at; i < k; i += L * 8) {
                    float wi[8], bi[8], yi[8];
                    weights8(wi, a.w, i, k, a.w16, 1.0f);
                    weights8(bi, a.b, i, k, a.w16, 0.0f);
                    normed<kCodes>(yi, load8(x, i, k, begin), m, wi, bi);
                    store8(to, i, k, yi);
                }
            }
        } else {
            Eight<float> held[V];
#pragma unroll
            for (int j = 0; j < V; ++j) __builtin_memcpy(&held[j], y[j], sizeof held[j]);
            unsigned most = most_of(held);
            for (int i = kHeld + at; i < k; i += L * 8) {
                float wi[8], bi[8], yi[8];
                weights8(wi, a.w, i, k, a.w16, 1.0f);
                weights8(bi, a.b, i, k, a.w16, 0.0f);
                normed<kCodes>(yi, load8(x, i, k, begin), m, wi, bi);
                Eight<float> more[1];
                __builtin_memcpy(&more[0], yi, sizeof more[0]);
                most = max(most, most_of(more));
            }
            const RowScale r = row_scale(row_most<L>(most, shared, turn));
            if (there) {
                if (at == 0) st_global(a.ys + row, r.s);
                int8_t *to = (int8_t *)a.y + row * a.ldy;
#pragma unroll
                for (int j = 0; j < V; ++j) store_codes(to, j * L * 8 + at, k, codes8(held[j], r, false));
                for (int i = kHeld + at; i < k; i += L * 8) {
                    float wi[8], bi[8], yi[8];
                    weights8(wi, a.w, i, k, a.w16, 1.0f);
                    weights8(bi, a.b, i, k, a.w16, 0.0f);
                    normed<kCodes>(yi, load8(x, i, k, begin), m, wi, bi);
                    Eight<float> more;
                    __builtin_memcpy(&more, yi, sizeof more);
                    store_codes(to, i, k, codes8(more, r, false));
                }
            }
        }
        turn ^= 1;
    }
}

template <typename X, typename G>
__device__ __forceinline__ void halves(float *x, float *g, const Eight<X> &rx, const Eight<G> &rg)
{
    const auto vx = __builtin_bit_cast(typename Values<X>::type, rx);
    const auto vg = __builtin_bit_cast(typename Values<G>::type, rg);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        x[e] = (float)vx[e];
        g[e] = (float)vg[e];
    }
}

__device__ __forceinline__ void put_gradient(void *to, int at, float v, int w16)
{
    if (!to) return;
    if (w16) st_global((_Float16 *)to + at, (_Float16)v);
    else st_global((float *)to + at, v);
}

__device__ __forceinline__ void put_gradients(void *to, int at, const float *v, int w16)
{
    if (!to) return;
    if (w16) put8((_Float16 *)to, at, v);
    else put8((float *)to, at, v);
}

// gx of a row of 8 to 8 L V values to L lanes, and the block's share of gw and gb: a lane adds up those of its columns over the block's rows.
template <typename X, typename G, int L, int V>
__global__ __launch_bounds__(norm_threads(L)) void norm_backward_kernel(NormArgs a)
{
    constexpr int kRows = norm_threads(L) / L;
    __shared__ Shared<L> shared;
    __shared__ float part[L <= 64 ? 4 : 1][L <= 64 ? 8 * L * V : 1];
    const int lane = (int)threadIdx.x % L, k = a.width;
    const long long stride = (long long)gridDim.x * kRows, sub = threadIdx.x / L;
    long long first = (long long)blockIdx.x * kRows;
    Place p[V];
    float w[V][8], gw[V][8], gb[V][8];
    Eight<X> next_x[V];
    Eight<G> next_g[V];
    float next_mean, next_rstd;
    const auto ask = [&](long long f) {
        const long long row = min(f + sub, a.rows - 1);
        const X *x = (const X *)a.x + row * a.ldx;
        const G *gy = (const G *)a.gy + row * a.ldgy;
        next_mean = ld_global(a.stats + 2 * row);
        next_rstd = ld_global(a.stats + 2 * row + 1);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            next_x[j] = held8(x, p[j].there ? p[j].at : 0);
            next_g[j] = held8(gy, p[j].there ? p[j].at : 0);
        }
    };
#pragma unroll
    for (int j = 0; j < V; ++j) p[j] = place_of(j * L + lane, k);
    ask(first);
#pragma unroll
    for (int j = 0; j < V; ++j) {
        held_weights(w[j], a.w, p[j].there ? p[j].at : 0, a.w16, 1.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) gw[j][e] = gb[j][e] = 0.0f;
    }
    int turn = 0;
    for (; first < a.rows; first += stride) {
        const long long row = first + sub;
        const bool there = row < a.rows;
        Eight<X> rx[V];
        Eight<G> rg[V];
        const float mean = next_mean, rstd = next_rstd;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            rx[j] = next_x[j];
            rg[j] = next_g[j];
        }
        if (first + stride < a.rows) ask(first + stride);
        float t1 = 0.0f, t2 = 0.0f;
        double s1 = 0.0, s2 = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!there || !p[j].there) continue;
            float xs[8], g[8];
            halves(xs, g, rx[j], rg[j]);
            t1 = t2 = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = (xs[e] - mean) * rstd, c = g[e] * w[j][e];
                t1 += c;
                t2 = __builtin_fmaf(c, h, t2);
                gw[j][e] = __builtin_fmaf(g[e], h, gw[j][e]);
                gb[j][e] += g[e];
            }
            if (p[j].twice) {
                t1 = t2 = 0.0f;
#pragma unroll
                for (int e = 1; e < 8; ++e) {
                    if (e < p[j].twice) continue;
                    const float h = (xs[e] - mean) * rstd, c = g[e] * w[j][e];
                    t1 += c;
                    t2 = __builtin_fmaf(c, h, t2);
                }
            }
            s1 += (double)t1;
            s2 += (double)t2;
        }
        if (!a.gx) continue;
        row_sums<L>(s1, s2, shared, turn);
        turn ^= 1;
        const float c1 = (float)(s1 * a.inverse), c2 = (float)(s2 * a.inverse);
        X *to = (X *)a.gx + row * a.ldgx;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float xs[8], g[8];
            halves(xs, g, rx[j], rg[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) xs[e] = rstd * ((g[e] * w[j][e] - c1) - (xs[e] - mean) * rstd * c2);
            if (there && p[j].there) put8(to, p[j].at, xs);
        }
    }
    if (!a.partial) return;
    float *to = a.partial + (long long)blockIdx.x * 2 * k;
    if constexpr (L > 64) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!p[j].there) continue;
            if (a.parts == 1) {
                // (what two vectors share is worked out and written by both, to the same bits)
                put_gradients(a.gw, p[j].at, gw[j], a.w16);
                put_gradients(a.gb, p[j].at, gb[j], a.w16);
            } else if (!p[j].twice) {
                put8(to, p[j].at, gw[j]);
                put8(to + k, p[j].at, gb[j]);
            } else {
#pragma unroll
                for (int e = 1; e < 8; ++e) {
                    if (e < p[j].twice) continue;
                    st_global(to + p[j].at + e, gw[j][e]);
                    st_global(to + k + p[j].at + e, gb[j][e]);
                }
            }
        }
    } else {
        // a block's rows side by side: those of a wavefront by its lanes, those of the four through LDS (columns of the last
        // vector by its lane's places)
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = which ? gb[j][e] : gw[j][e];
                    if constexpr (L == 16) {
                        v += __shfl_xor(v, 16);
                        v += __shfl_xor(v, 32);
                    }
                    if ((threadIdx.x & 63) < L && p[j].there && e >= p[j].twice) part[threadIdx.x >> 6][p[j].at + e] = v;
                }
            __syncthreads();
            for (int i = threadIdx.x; i < k; i += 256) {
                const float v = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
                if (a.parts == 1) put_gradient(which ? a.gb : a.gw, i, v, a.w16);
                else st_global(to + which * k + i, v);
            }
            __syncthreads();
        }
    }
}

// The same of rows of any width: those that are no whole of a block's registers are read again and leave gw and gb to
// norm_columns_kernel.
template <typename X, typename G, int L, int V>
__global__ __launch_bounds__(norm_threads(L)) void norm_backward_any_kernel(NormArgs a)
{
    constexpr int kRows = norm_threads(L) / L, kHeld = 8 * L * V;
    __shared__ Shared<L> shared;
    __shared__ float part[L <= 64 ? 4 : 1][L <= 64 ? kHeld : 1];
    const int at = (int)threadIdx.x % L * 8, k = a.width;
    float w[V][8], gw[V][8], gb[V][8];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        weights8(w[j], a.w, j * L * 8 + at, k, a.w16, 1.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) gw[j][e] = gb[j][e] = 0.0f;
    }
    int turn = 0;
    for (long long first = (long long)blockIdx.x * kRows; first < a.rows; first += (long long)gridDim.x * kRows) {
        const long long row = first + threadIdx.x / L;
        const bool there = row < a.rows;
        const long long from = there ? row : a.rows - 1;
        const X *x = (const X *)a.x + from * a.ldx;
        const G *gy = (const G *)a.gy + from * a.ldgy;
        const float mean = ld_global(a.stats + 2 * from), rstd = ld_global(a.stats + 2 * from + 1);
        Eight<X> rx[V];
        Eight<G> rg[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            rx[j] = ask8(x, j * L * 8 + at, k);
            rg[j] = ask8(gy, j * L * 8 + at, k);
        }
        double s1 = 0.0, s2 = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            odd_end(rx[j], x, j * L * 8 + at, k);
            odd_end(rg[j], gy, j * L * 8 + at, k);
            if (!there || j * L * 8 + at >= k) continue;
            float xs[8], g[8], t1 = 0.0f, t2 = 0.0f;
            halves(xs, g, rx[j], rg[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = (xs[e] - mean) * rstd, c = g[e] * w[j][e];
                t1 += c;
                t2 = __builtin_fmaf(c, h, t2);
                gw[j][e] = __builtin_fmaf(g[e], h, gw[j][e]);
                gb[j][e] += g[e];
            }
            s1 += (double)t1;
            s2 += (double)t2;
        }
        for (int i = kHeld + at; i < k; i += L * 8) {
            float xs[8], g[8], wi[8], t1 = 0.0f, t2 = 0.0f;
            weights8(wi, a.w, i, k, a.w16, 1.0f);
            halves(xs, g, load8(x, i, k, (X)0.0f), load8(gy, i, k, (G)0.0f));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float h = (xs[e] - mean) * rstd, c = g[e] * wi[e];
                t1 += c;
                t2 = __builtin_fmaf(c, h, t2);
            }
            s1 += (double)t1;
            s2 += (double)t2;
        }
        if (!a.gx) continue;
        row_sums<L>(s1, s2, shared, turn);
        turn ^= 1;
        if (!there) continue;
        const float c1 = (float)(s1 * a.inverse), c2 = (float)(s2 * a.inverse);
        X *to = (X *)a.gx + row * a.ldgx;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (j * L * 8 + at >= k) continue;
            float xs[8], g[8];
            halves(xs, g, rx[j], rg[j]);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                xs[e] = rstd * ((g[e] * w[j][e] - c1) - (xs[e] - mean) * rstd * c2);
            store8(to, j * L * 8 + at, k, xs);
        }
        for (int i = kHeld + at; i < k; i += L * 8) {
            float xs[8], g[8], wi[8];
            weights8(wi, a.w, i, k, a.w16, 1.0f);
            halves(xs, g, load8(x, i, k, (X)0.0f), load8(gy, i, k, (G)0.0f));
#pragma unroll
            for (int e = 0; e < 8; ++e) xs[e] = rstd * ((g[e] * wi[e] - c1) - (xs[e] - mean) * rstd * c2);
            store8(to, i, k, xs);
        }
    }
    if constexpr (L <= 64) {
        if (!a.partial) return;
        float *to = a.partial + (long long)blockIdx.x * 2 * k;
        // a block's rows side by side: those of a wavefront by its lanes, those of the four through LDS
#pragma unroll
        for (int which = 0; which < 2; ++which) {
#pragma unroll
            for (int j = 0; j < V; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = which ? gb[j][e] : gw[j][e];
                    if constexpr (L == 16) {
                        v += __shfl_xor(v, 16);
                        v += __shfl_xor(v, 32);
                    }
                    if ((threadIdx.x & 63) < L) part[threadIdx.x >> 6][j * L * 8 + at + e] = v;
                }
            __syncthreads();
            for (int i = threadIdx.x; i < k; i += 256) {
                const float v = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
                if (a.parts == 1) put_gradient(which ? a.gb : a.gw, i, v, a.w16);
                else st_global(to + which * k + i, v);
            }
            __syncthreads();
        }
    }
}

// Shares of gw and gb of rows that no block holds: a strip of columns of every parts-th four rows, one row to a wavefront, eight
// columns to a lane.
template <typename X, typename G> __global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a)
{
    __shared__ float part[4][kNormStrip];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = a.width;
    const int strips = (k + kNormStrip - 1) / kNormStrip, piece = (int)blockIdx.x / strips;
    const int base = (int)blockIdx.x % strips * kNormStrip, at = base + lane * 8;
    float gw[8], gb[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) gw[e] = gb[e] = 0.0f;
    if (at < k) {
        for (long long row = piece * 4LL + wave; row < a.rows; row += a.parts * 4LL) {
            const float mean = ld_global(a.stats + 2 * row), rstd = ld_global(a.stats + 2 * row + 1);
            float x[8], g[8];
            halves(x, g, load8((const X *)a.x + row * a.ldx, at, k, (X)0.0f), load8((const G *)a.gy + row * a.ldgy, at, k, (G)0.0f));
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                gw[e] = __builtin_fmaf(g[e], (x[e] - mean) * rstd, gw[e]);
                gb[e] += g[e];
            }
        }
    }
    float *to = a.partial + (long long)piece * 2 * k;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
#pragma unroll
        for (int e = 0; e < 8; ++e) part[wave][lane * 8 + e] = which ? gb[e] : gw[e];
        __syncthreads();
        for (int i = threadIdx.x; i < kNormStrip && base + i < k; i += 256)
            st_global(to + which * (long long)k + base + i, (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]));
        __syncthreads();
    }
}

// The sums of the parts, in binary64: COLUMNS columns to a block, 1024 / COLUMNS threads to a column, each with every so manieth part,
// eight on their way at a time.
constexpr int kJoinThreads = 1024;

template <typename W, int COLUMNS> __global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(NormArgs a)
{
    constexpr int kGroups = kJoinThreads / COLUMNS;
    __shared__ double part[kGroups][COLUMNS];
    const int k = a.width, column = threadIdx.x % COLUMNS, group = threadIdx.x / COLUMNS;
    const long long at = min((long long)blockIdx.x * COLUMNS + column, 2LL * k - 1);
    double s = 0.0;
    for (int i = group; i < a.parts; i += 8 * kGroups) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ld_global(a.partial + (long long)min(i + j * kGroups, a.parts - 1) * 2 * k + at);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += i + j * kGroups < a.parts ? (double)v[j] : 0.0;
    }
    part[group][column] = s;
    __syncthreads();
    const long long to = (long long)blockIdx.x * COLUMNS + threadIdx.x;
    if (threadIdx.x >= COLUMNS || to >= 2LL * k) return;
    s = 0.0;
#pragma unroll 16
    for (int i = 0; i < kGroups; ++i) s += part[i][threadIdx.x];
    W *const out = (W *)(to < k ? a.gw : a.gb);
    if (out) st_global(out + (to < k ? to : to - k), (W)s);
}

// (few parts leave most threads of a column without any: 6 x 11377 FP16 11.9 us with 16 columns to a block, 9.9 with 256)
template <typename W> void join(const NormArgs &a, hipStream_t s)
{
    if (a.parts <= 32) norm_join_kernel<W, 256><<<(unsigned)((2LL * a.width + 255) / 256), kJoinThreads, 0, s>>>(a);
    else norm_join_kernel<W, 16><<<(unsigned)((2LL * a.width + 15) / 16), kJoinThreads, 0, s>>>(a);
}

template <typename W> __global__ __launch_bounds__(256) void norm_zero_kernel(NormArgs a)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.width) return;
    if (a.gw) st_global((W *)a.gw + at, (W)0.0f);
    if (a.gb) st_global((W *)a.gb + at, (W)0.0f);
}

template <typename X, typename Y, int L, int V> void forward_by(const NormArgs &a, hipStream_t stream)
{
    norm_forward_kernel<X, Y, L, V><<<(unsigned)a.blocks, norm_threads(L), 0, stream>>>(a);
}

template <typename X, typename Y> int forward(const NormArgs &a, hipStream_t stream)
{
    if (a.width < 8) norm_forward_any_kernel<X, Y, 16, 1><<<(unsigned)a.blocks, 256, 0, stream>>>(a);
    else if (a.width > kNormHeldWidth) norm_forward_any_kernel<X, Y, 1024, 2><<<(unsigned)a.blocks, 1024, 0, stream>>>(a);
    else if (a.lanes == 16 && a.vecs == 1) forward_by<X, Y, 16, 1>(a, stream);
    else if (a.lanes == 16 && a.vecs == 2) forward_by<X, Y, 16, 2>(a, stream);
    else if (a.lanes == 16 && a.vecs == 3) forward_by<X, Y, 16, 3>(a, stream);
    else if (a.lanes == 16 && a.vecs == 4) forward_by<X, Y, 16, 4>(a, stream);
    else if (a.lanes == 64 && a.vecs == 2) forward_by<X, Y, 64, 2>(a, stream);
    else if (a.lanes == 64 && a.vecs == 3) forward_by<X, Y, 64, 3>(a, stream);
    else if (a.lanes == 64 && a.vecs == 4) forward_by<X, Y, 64, 4>(a, stream);
    else if (a.lanes == 256 && a.vecs == 2) forward_by<X, Y, 256, 2>(a, stream);
    else if (a.lanes == 256 && a.vecs == 3) forward_by<X, Y, 256, 3>(a, stream);
    else if (a.lanes == 256 && a.vecs == 4) forward_by<X, Y, 256, 4>(a, stream);
    else if (a.lanes == 512 && a.vecs == 3) forward_by<X, Y, 512, 3>(a, stream);
    else if (a.lanes == 512 && a.vecs == 4) forward_by<X, Y, 512, 4>(a, stream);
    else return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}

template <typename X, typename G, int L, int V> void backward_by(const NormArgs &a, hipStream_t stream)
{
    norm_backward_kernel<X, G, L, V><<<(unsigned)a.blocks, norm_threads(L), 0, stream>>>(a);
}

template <typename X, typename G> int backward(const NormArgs &a, hipStream_t stream)
{
    if (a.width > kNormHeldWidth) {
        // (the columns' sums in front of gx, which may be x or gy itself)
        if (a.partial) norm_columns_kernel<X, G><<<(unsigned)((a.width + kNormStrip - 1) / kNormStrip * a.parts), 256, 0, stream>>>(a);
        if (a.gx) norm_backward_any_kernel<X, G, 1024, 2><<<(unsigned)a.blocks, 1024, 0, stream>>>(a);
    } else if (a.width < 8) norm_backward_any_kernel<X, G, 16, 1><<<(unsigned)a.blocks, 256, 0, stream>>>(a);
    else if (a.lanes == 16 && a.vecs == 1) backward_by<X, G, 16, 1>(a, stream);
    else if (a.lanes == 16 && a.vecs == 2) backward_by<X, G, 16, 2>(a, stream);
    else if (a.lanes == 64 && a.vecs == 1) backward_by<X, G, 64, 1>(a, stream);
    else if (a.lanes == 64 && a.vecs == 2) backward_by<X, G, 64, 2>(a, stream);
    else if (a.lanes == 256 && a.vecs == 1) backward_by<X, G, 256, 1>(a, stream);
    else if (a.lanes == 256 && a.vecs == 2) backward_by<X, G, 256, 2>(a, stream);
    else if (a.lanes == 256 && a.vecs == 3) backward_by<X, G, 256, 3>(a, stream);
    else if (a.lanes == 256 && a.vecs == 4) backward_by<X, G, 256, 4>(a, stream);
    else if (a.lanes == 512 && a.vecs == 3) backward_by<X, G, 512, 3>(a, stream);
    else if (a.lanes == 512 && a.vecs == 4) backward_by<X, G, 512, 4>(a, stream);
    else return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}

}  // namespace

int launch_norm_forward(const NormArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.codes) return a.x16 ? forward<_Float16, int8_t>(a, s) : forward<float, int8_t>(a, s);
    if (a.y16) return a.x16 ? forward<_Float16, _Float16>(a, s) : forward<float, _Float16>(a, s);
    return a.x16 ? forward<_Float16, float>(a, s) : forward<float, float>(a, s);
}

int launch_norm_backward(const NormArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.rows == 0) {
        const unsigned blocks = (unsigned)((a.width + 255) / 256);
        if (a.w16) norm_zero_kernel<_Float16><<<blocks, 256, 0, s>>>(a);
        else norm_zero_kernel<float><<<blocks, 256, 0, s>>>(a);
        return (int)hipGetLastError();
    }
    const int err = a.x16 ? (a.y16 ? backward<_Float16, _Float16>(a, s) : backward<_Float16, float>(a, s))
                          : (a.y16 ? backward<float, _Float16>(a, s) : backward<float, float>(a, s));
    if (err != 0 || !a.partial || (a.parts == 1 && a.width <= kNormHeldWidth)) return err;
    if (a.w16) join<_Float16>(a, s);
    else join<float>(a, s);
    return (int)hipGetLastError();
}

}  // namespace fq
