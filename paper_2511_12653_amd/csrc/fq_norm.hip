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

__device__ __forceinline__ double sum16(double v)
{
    v += dpp_move<0xB1, 0xf>(v);
    v += dpp_move<0x4E, 0xf>(v);
    v += dpp_move<0x141, 0xf>(v);
    return v + dpp_move<0x140, 0xf>(v);
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
    double sums[2][2][16];
    unsigned most[2][16];
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
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (L == 64) {
            a = lane_value(a, kSumLane);
            b = lane_value(b, kSumLane);
        } else {
            if ((threadIdx.x & 63) == kSumLane) {
                s.sums[turn][0][threadIdx.x >> 6] = a;
                s.sums[turn][1][threadIdx.x >> 6] = b;
            }
            __syncthreads();
            // (as many lanes as wavefronts have a sum each, the others of 16 zero)
            const int i = threadIdx.x & 15;
            a = sum16(i < L / 64 ? s.sums[turn][0][i] : 0.0);
            b = sum16(i < L / 64 ? s.sums[turn][1][i] : 0.0);
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
        const int i = threadIdx.x & 15;
        v = max16(i < L / 64 ? s.most[turn][i] : 0u);
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
};

__device__ __forceinline__ Moments moments(double x0, double s1, double s2, int k, float eps)
{
    const double off = s1 / k;
    double var = (s2 - s1 * off) / k;
    if (var < 0.0) var = 0.0;                      // (rounding; a NaN stays)
    return {x0 + off, 1.0 / sqrt(var + (double)eps)};
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

template <typename X>
__device__ __forceinline__ void normed(float *y, const Eight<X> &r, const Moments &m, const float *w, const float *b)
{
    const auto x = __builtin_bit_cast(typename Values<X>::type, r);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        y[e] = (float)__builtin_fma(((double)(float)x[e] - m.mean) * m.rstd, (double)w[e], (double)b[e]);
}

// A row to L lanes, V vectors of eight values to each; rows of more are read again from the caches.
template <typename X, typename Y, int L, int V>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_forward_kernel(NormArgs a)
{
    constexpr int kRows = L < 256 ? 256 / L : 1, kHeld = 8 * L * V;
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
        const Moments m = moments((double)(float)begin, s1, s2, k, a.eps);
        if (a.stats && there && at == 0) {
            st_global(a.stats + 2 * row, (float)m.mean);
            st_global(a.stats + 2 * row + 1, (float)m.rstd);
        }
        float y[V][8];
#pragma unroll
        for (int j = 0; j < V; ++j) normed(y[j], raw[j], m, w[j], b[j]);
        if constexpr (!kCodes) {
            if (there) {
                Y *to = (Y *)a.y + row * a.ldy;
#pragma unroll
                for (int j = 0; j < V; ++j) store8(to, j * L * 8 + at, k, y[j]);
                for (int i = kHeld + at; i < k; i += L * 8) {
                    float wi[8], bi[8], yi[8];
                    weights8(wi, a.w, i, k, a.w16, 1.0f);
                    weights8(bi, a.b, i, k, a.w16, 0.0f);
                    normed(yi, load8(x, i, k, begin), m, wi, bi);
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
                normed(yi, load8(x, i, k, begin), m, wi, bi);
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
                    normed(yi, load8(x, i, k, begin), m, wi, bi);
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

// gx of a row to L lanes, and the block's share of gw and gb: a lane adds up those of its columns over the block's rows.  Rows
// that are no whole of a block's registers are read again and leave gw and gb to norm_columns_kernel.
template <typename X, typename G, int L, int V>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_backward_kernel(NormArgs a)
{
    constexpr int kRows = L < 256 ? 256 / L : 1, kHeld = 8 * L * V;
    __shared__ Shared<L> shared;
    __shared__ float part[L < 64 ? 4 : L < 256 ? 4 : 1][L < 256 ? kHeld : 1];
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
        const float c1 = (float)(s1 / k), c2 = (float)(s2 / k);
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
    if (!a.partial || k > kNormHeldWidth) return;
    float *to = a.partial + (long long)blockIdx.x * 2 * k;
    if constexpr (L >= 256) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (j * L * 8 + at >= k) continue;
            store8(to, j * L * 8 + at, k, gw[j]);
            store8(to + k, j * L * 8 + at, k, gb[j]);
        }
    } else {
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
            for (int i = threadIdx.x; i < k; i += 256)
                st_global(to + which * k + i, (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]));
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

// The sums of the parts, in binary64: 32 columns to a block, 32 threads to a column.
constexpr int kJoinColumns = 32, kJoinThreads = 1024;

template <typename W> __global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(NormArgs a)
{
    __shared__ double part[kJoinThreads / kJoinColumns][kJoinColumns + 1];
    const int k = a.width, column = threadIdx.x % kJoinColumns, group = threadIdx.x / kJoinColumns;
    const long long at = (long long)blockIdx.x * kJoinColumns + column;
    double s = 0.0;
    if (at < 2LL * k)
        for (int i = group; i < a.parts; i += kJoinThreads / kJoinColumns) s += (double)ld_global(a.partial + (long long)i * 2 * k + at);
    part[group][column] = s;
    __syncthreads();
    if (group != 0 || at >= 2LL * k) return;
#pragma unroll
    for (int i = 1; i < kJoinThreads / kJoinColumns; ++i) s += part[i][column];
    W *const to = (W *)(at < k ? a.gw : a.gb);
    if (to) st_global(to + (at < k ? at : at - k), (W)s);
}

template <typename W> __global__ __launch_bounds__(256) void norm_zero_kernel(NormArgs a)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= a.width) return;
    if (a.gw) st_global((W *)a.gw + at, (W)0.0f);
    if (a.gb) st_global((W *)a.gb + at, (W)0.0f);
}

constexpr long long kMostBlocks = 1 << 21;       // a grid has less than 2^32 threads

template <typename X, typename Y, int L, int V> void forward_by(const NormArgs &a, hipStream_t stream)
{
    constexpr int kRows = L < 256 ? 256 / L : 1;
    const long long groups = (a.rows + kRows - 1) / kRows;
    norm_forward_kernel<X, Y, L, V><<<(unsigned)(groups < kMostBlocks ? groups : kMostBlocks), L < 256 ? 256 : L, 0, stream>>>(a);
}

template <typename X, typename Y> int forward(const NormArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.width);
    if (s.lanes == 16) (s.vecs == 1 ? forward_by<X, Y, 16, 1> : s.vecs == 2 ? forward_by<X, Y, 16, 2> : forward_by<X, Y, 16, 3>)(a, stream);
    else if (s.lanes == 64) (s.vecs == 1 ? forward_by<X, Y, 64, 1> : forward_by<X, Y, 64, 2>)(a, stream);
    else if (s.lanes == 256) (s.vecs == 1 ? forward_by<X, Y, 256, 1> : forward_by<X, Y, 256, 2>)(a, stream);
    else if (s.lanes == 512) forward_by<X, Y, 512, 2>(a, stream);
    else forward_by<X, Y, 1024, 2>(a, stream);
    return (int)hipGetLastError();
}

template <typename X, typename G, int L, int V> void backward_by(const NormArgs &a, hipStream_t stream)
{
    constexpr int kRows = L < 256 ? 256 / L : 1;
    const long long groups = (a.rows + kRows - 1) / kRows;
    const bool held = a.width <= kNormHeldWidth;
    const long long blocks = a.partial && held ? a.parts : groups < kMostBlocks ? groups : kMostBlocks;
    norm_backward_kernel<X, G, L, V><<<(unsigned)blocks, L < 256 ? 256 : L, 0, stream>>>(a);
}

template <typename X, typename G> int backward(const NormArgs &a, hipStream_t stream)
{
    const NormShape s = norm_shape(a.width);
    const bool held = a.width <= kNormHeldWidth;
    // (in front of gx, which may be x or gy itself)
    if (a.partial && !held) norm_columns_kernel<X, G><<<(unsigned)((a.width + kNormStrip - 1) / kNormStrip * a.parts), 256, 0, stream>>>(a);
    if (a.gx || held) {
        if (s.lanes == 16) (s.vecs == 1 ? backward_by<X, G, 16, 1> : s.vecs == 2 ? backward_by<X, G, 16, 2> : backward_by<X, G, 16, 3>)(a, stream);
        else if (s.lanes == 64) (s.vecs == 1 ? backward_by<X, G, 64, 1> : backward_by<X, G, 64, 2>)(a, stream);
        else if (s.lanes == 256) (s.vecs == 1 ? backward_by<X, G, 256, 1> : backward_by<X, G, 256, 2>)(a, stream);
        else if (s.lanes == 512) backward_by<X, G, 512, 2>(a, stream);
        else backward_by<X, G, 1024, 2>(a, stream);
    }
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
    if (err != 0 || !a.partial) return err;
    const unsigned blocks = (unsigned)((2LL * a.width + kJoinColumns - 1) / kJoinColumns);
    if (a.w16) norm_join_kernel<_Float16><<<blocks, kJoinThreads, 0, s>>>(a);
    else norm_join_kernel<float><<<blocks, kJoinThreads, 0, s>>>(a);
    return (int)hipGetLastError();
}

}  // namespace fq
