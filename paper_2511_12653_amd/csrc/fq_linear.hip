// Int8 linear layer with a scale per token and per channel (declared in include/fq.h).
#include <hip/hip_fp16.h>

#include "fq_device.h"
#include "fq_linear.h"

namespace fq {
namespace {

using namespace dev;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------------------------
// Codes and scale of a row of x.
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// Values [at, at + 8) of a row of k; zeros behind its end.
template <typename T> __device__ __forceinline__ void load8(const T *row, int at, int k, bool vec, float *v)
{
    if (vec && at + 8 <= k) {
        if constexpr (sizeof(T) == 2) {
            const f16x8 h = *(const FQ_GLOBAL f16x8 *)(row + at);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)h[e];
        } else {
            const f32x4 a = *(const FQ_GLOBAL f32x4 *)(row + at), b = *(const FQ_GLOBAL f32x4 *)(row + at + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[e + 4] = b[e]; }
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = at + e < k ? (float)ld_global(row + at + e) : 0.0f;
}

// Greatest magnitude of eight values, as bits (magnitudes order like their bits: NaN, infinity, numbers).
__device__ __forceinline__ unsigned most8(const float *v)
{
    unsigned most = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(unsigned, v[e]) & 0x7FFFFFFFu);
    return most;
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

// Codes of eight values.  x * (1 / s) is within 127 * 2^-22.4 of the quotient x / s, so unless it lies that near to a
// half (a few vectors of a row) it rounds to the same integer.  Adding 1.5 * 2^23 rounds it, to even, and leaves the code in
// the low byte.  No code leaves [-127, 127]: no |x| is over 127 * s * (1 + 2^-24).
__device__ __forceinline__ u32x2 codes8(const float *v, RowScale r)
{
    constexpr float kMagic = 0x1.8p23f;
    unsigned b[8];
    float near = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = v[e] * r.inverse, f = t + kMagic;
        b[e] = __builtin_bit_cast(unsigned, f);
        near = __builtin_fmaxf(near, __builtin_fabsf(t - (f - kMagic)));
    }
    if (near > 0.49995f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = __builtin_bit_cast(unsigned, v[e] / r.s + kMagic);
    }
    const auto pack = [](unsigned p, unsigned q, unsigned s, unsigned t) {
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t, s, 0x0c0c0400u), __builtin_amdgcn_perm(q, p, 0x0c0c0400u), 0x05040100u);
    };
    u32x2 w = u32x2{pack(b[0], b[1], b[2], b[3]), pack(b[4], b[5], b[6], b[7])};
    if (r.inverse == 0.0f) w = (u32x2)0u;
    return w;
}

// THREADS of a block have a row, HELD vectors of eight each: read once, kept in registers.  Longer rows are read again
// for the codes.
template <typename T, int THREADS, int HELD>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a)
{
    __shared__ unsigned top[4];
    const int at = threadIdx.x % THREADS;
    const long long row = (long long)blockIdx.x * (256 / THREADS) + threadIdx.x / THREADS;
    if (THREADS < 256 && row >= a.m) return;
    const T *x = (const T *)a.x + row * a.ldx;
    float v[HELD][8];
    unsigned most = 0;
#pragma unroll
    for (int j = 0; j < HELD; ++j) load8(x, (j * THREADS + at) * 8, a.k, a.vec, v[j]);
#pragma unroll
    for (int j = 0; j < HELD; ++j) most = max(most, most8(v[j]));
    for (int i = (HELD * THREADS + at) * 8; i < a.k; i += THREADS * 8) {
        float more[8];
        load8(x, i, a.k, a.vec, more);
        most = max(most, most8(more));
    }
    most = wave_max(most);
    if (THREADS == 256) {
        if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(top[0], top[1]), max(top[2], top[3]));
    }
    const RowScale r = row_scale(most);
    if (at == 0) st_global(a.s + row, r.s);
    int8_t *q = a.q + row * a.pitch;
#pragma unroll
    for (int j = 0; j < HELD; ++j) {
        const int i = (j * THREADS + at) * 8;
        if (i < a.pitch) *(FQ_GLOBAL u32x2 *)(q + i) = codes8(v[j], r);
    }
    for (int i = (HELD * THREADS + at) * 8; i < a.pitch; i += THREADS * 8) {
        float more[8];
        load8(x, i, a.k, a.vec, more);
        *(FQ_GLOBAL u32x2 *)(q + i) = codes8(more, r);
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

// ---------------------------------------------------------------------------------------------
// Product of a tile of BM tokens by BN channels.  BM / WM by BN / WN of it belong to a wavefront, which builds them from
// 32 x 32 matrix instructions: lane l holds 16 codes of channel l % 32 and of token l % 32, and of the sums those of token
// l % 32 and channels 8 g + 4 (l / 32) + 0..3, g = 0..3.
//
// 128 codes of every row of the tile are in LDS at a time, twice over: while the matrix cores work on one, the loads of the
// next 128 go straight from memory into the other.  A load instruction fills 1 KiB of LDS in lane order, eight rows; which
// 16 codes a lane fetches is free, and lane 8 r + c fetches those at c ^ r, so that eight lanes that read the same 16 codes of
// eight neighbouring rows find them in eight different places of the banks.
constexpr int kDepth = 128;                                     // codes of a row per step
constexpr unsigned kNowhere = 0x7FFFFFF0u;                      // beyond the end of any buffer: reads as zeros

#define FQ_LDS __attribute__((address_space(3)))

struct Panel {                                                  // rows of one operand that a block multiplies
    const int8_t *at;
    unsigned bytes;                                             // from `at` to the end of the last row
};

__device__ __forceinline__ Panel panel(const int8_t *base, long long ld, int row0, int rows, int left, int k)
{
    return {base + (long long)row0 * ld, (unsigned)(min(rows, left) - 1) * (unsigned)ld + (unsigned)k};
}

template <int N, int WAVES> struct Staging {                    // N wavefront loads of a panel per wavefront and step
    unsigned off[N];
    i32x4 held[N];

    __device__ __forceinline__ void place(long long ld, int lane, int wave)
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
            off[j] = (unsigned)((j * WAVES + wave) * 8 + lane / 8) * (unsigned)ld + (unsigned)((lane % 8) ^ (lane / 8)) * 16;
    }
    // Codes [at, at + kDepth) of the panel's rows into LDS; with `tail`, those from `at + left` on as zeros.
    __device__ __forceinline__ void fetch(const Panel &p, int at, int8_t *to, int wave, bool tail, int left, int lane)
    {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)(p.at + at), (short)0, (int)(p.bytes - (unsigned)at), 0x00027000);
        const bool none = tail && ((lane % 8) ^ (lane / 8)) * 16 >= left;
#pragma unroll
        for (int j = 0; j < N; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (FQ_LDS void *)(to + (j * WAVES + wave) * 1024), 16, none ? kNowhere : off[j], 0, 0, 0);
    }
    // The same by way of registers, for rows at any address.
    __device__ __forceinline__ void request(const int8_t *base, long long ld, int row0, int rows, int at, int k, int lane, int wave)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = min(row0 + (j * WAVES + wave) * 8 + lane / 8, rows - 1);
            held[j] = load16(base + (long long)row * ld, at + ((lane % 8) ^ (lane / 8)) * 16, k);
        }
    }
    __device__ __forceinline__ void put(int8_t *to, int lane, int wave)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) *(i32x4 *)(to + (j * WAVES + wave) * 1024 + lane * 16) = held[j];
    }
};

// What a wavefront's lanes have written to LDS before is what its lanes read behind.
__device__ __forceinline__ void lanes_in_step()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// y of 8 channels from j on, of token i.
__device__ __forceinline__ void store8(const LinearArgs &a, long long i, int j, const float *y)
{
    if (a.y16) {
        _Float16 *to = (_Float16 *)a.y + i * a.ldy + j;
        f16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (_Float16)y[e];
        if (a.y_vec && j + 8 <= a.n) {
            *(FQ_GLOBAL f16x8 *)to = v;
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e < a.n) st_global(to + e, v[e]);
        return;
    }
    float *to = (float *)a.y + i * a.ldy + j;
    if (a.y_vec && j + 8 <= a.n) {
        *(FQ_GLOBAL f32x4 *)to = f32x4{y[0], y[1], y[2], y[3]};
        *(FQ_GLOBAL f32x4 *)(to + 4) = f32x4{y[4], y[5], y[6], y[7]};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (j + e < a.n) st_global(to + e, y[e]);
}

// Tile of a block.  Blocks go to the eight XCDs in turn: each gets neighbouring tiles, in groups kGroup token tiles
// high, so that what its L2 holds of x and w serves many of them.
constexpr int kXcds = 8, kGroup = 4;

__device__ __forceinline__ void tile_of(unsigned block, unsigned blocks, unsigned tiles_m, unsigned tiles_n, unsigned &tm, unsigned &tn)
{
    const unsigned xcd = block % kXcds, each = blocks / kXcds, more = blocks % kXcds;
    const unsigned t = xcd * each + min(xcd, more) + block / kXcds;
    const unsigned group = t / (kGroup * tiles_n), in = t % (kGroup * tiles_n), high = min((unsigned)kGroup, tiles_m - group * kGroup);
    tm = group * kGroup + in % high;
    tn = in / high;
}

template <int BM, int BN, int WM, int WN, bool ALIGNED>
__global__ __launch_bounds__(WM * WN * 64) void linear_tile_kernel(LinearArgs a)
{
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kPitch = TN * 32 + 4;                         // of the sums in LDS
    constexpr int kStage = (BM + BN) * kDepth;
    static_assert(WAVES * 32 * kPitch * 4 <= 2 * kStage, "the sums of a wavefront's 32 tokens fit in its share");
    __shared__ __attribute__((aligned(1024))) int8_t even[kStage], odd[kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned tile_m, tile_n;
    tile_of(blockIdx.x, gridDim.x, (a.m + BM - 1) / BM, (a.n + BN - 1) / BN, tile_m, tile_n);
    const int m0 = (int)tile_m * BM, n0 = (int)tile_n * BN;
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

    Staging<BN / 8 / WAVES, WAVES> w;
    Staging<BM / 8 / WAVES, WAVES> x;
    const Panel pw = panel(a.w, a.ldw, n0, BN, a.n - n0, a.k), px = panel(a.x, a.ldx, m0, BM, a.m - m0, a.kx);
    if constexpr (ALIGNED) {
        w.place(a.ldw, lane, wave);
        x.place(a.ldx, lane, wave);
    }
    const int steps = (a.k + kDepth - 1) / kDepth;
    auto ask = [&](int step, int8_t *to) {
        if (step >= steps) return;
        const int at = step * kDepth;
        if constexpr (ALIGNED) {
            w.fetch(pw, at, to, wave, false, 0, lane);
            x.fetch(px, at, to + BN * kDepth, wave, at + kDepth > a.kx, a.kx - at, lane);
        } else {
            w.request(a.w, a.ldw, n0, a.n, at, a.k, lane, wave);
            x.request(a.x, a.ldx, m0, a.m, at, a.k, lane, wave);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto have = [&](int step, int8_t *to) {
        if (!ALIGNED && step < steps) {
            w.put(to, lane, wave);
            x.put(to + BN * kDepth, lane, wave);
        }
        __syncthreads();
    };
    i32x16 sum[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) sum[j][i] = (i32x16)0;
    auto multiply = [&](const int8_t *from) {
        const int8_t *fw = from + (wn + lane % 32) * kDepth, *fx = from + (BN + wm + lane % 32) * kDepth;
#pragma unroll
        for (int s = 0; s < kDepth / 32; ++s) {
            const int at = ((2 * s + lane / 32) ^ (lane % 8)) * 16;
            i32x4 cw[TN], cx[TM];
#pragma unroll
            for (int j = 0; j < TN; ++j) cw[j] = *(const i32x4 *)(fw + j * 32 * kDepth + at);
#pragma unroll
            for (int i = 0; i < TM; ++i) cx[i] = *(const i32x4 *)(fx + i * 32 * kDepth + at);
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) sum[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(cw[j], cx[i], sum[j][i], 0, 0, 0);
        }
    };
    ask(0, even);
    have(0, even);
    int step = 0;
    for (; step + 1 < steps; step += 2) {
        ask(step + 1, odd);
        multiply(even);
        have(step + 1, odd);
        ask(step + 2, even);
        multiply(odd);
        have(step + 2, even);
    }
    if (step < steps) {
        multiply(even);
        __syncthreads();
    }

    // 32 tokens at a time: the sums change places through LDS, so that a lane has 8 neighbouring channels of a token and
    // a store instruction whole lines.
    constexpr int kLanes = TN * 32 / 8;                         // that hold a token
    int *const mine = (int *)(wave < WAVES / 2 ? even : odd) + (wave % (WAVES / 2)) * (32 * kPitch);
    const int n = n0 + wn + lane % kLanes * 8;
    float ws[8], bias[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int j = min(n + e, a.n - 1);
        ws[e] = ld_global(a.ws + (long long)j * a.ws_step);
        bias[e] = a.bias ? ld_global(a.bias + j) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(i32x4 *)(mine + (lane % 32) * kPitch + j * 32 + g * 8 + lane / 32 * 4) =
                    i32x4{sum[j][i][4 * g], sum[j][i][4 * g + 1], sum[j][i][4 * g + 2], sum[j][i][4 * g + 3]};
        lanes_in_step();
#pragma unroll
        for (int t = 0; t < 32; t += 64 / kLanes) {
            const int row = t + lane / kLanes, m = m0 + wm + i * 32 + row;
            const int *from = mine + row * kPitch + lane % kLanes * 8;
            const i32x4 low = *(const i32x4 *)from, high = *(const i32x4 *)(from + 4);
            if (m >= a.m || n >= a.n) continue;
            const float xs = ld_global(a.xs + (long long)m * a.xs_step);
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = (float)(e < 4 ? low[e] : high[e - 4]) * (xs * ws[e]);
                if (a.bias) y[e] += bias[e];
            }
            store8(a, m, n, y);
        }
        lanes_in_step();
    }
}

// ---------------------------------------------------------------------------------------------
// Few tokens: what counts is to stream w once.  A block multiplies 16 * CH channels by all tokens (TOK times 16, lanes past
// the last repeat it); its wavefronts share the codes of a row, a run of whole steps of 64 each, and their sums meet in
// LDS.  w goes straight from memory into registers, kAhead steps of it requested before the first is used: 16 rows x 64
// bytes to a load instruction.  With X FP16 or FP32 the block first turns the rows of x into codes in LDS, while the first
// codes of w are on their way; with X int8 the codes of x come from memory like those of w.
template <typename X, int TOK, int CH, int WAVES, bool ALIGNED>
__global__ __launch_bounds__(WAVES * 64) void linear_few_kernel(LinearArgs a)
{
    constexpr bool kQuantize = sizeof(X) > 1;
    constexpr int kAhead = 8 / CH, kPitch = 20;                  // (of 16 channels' sums in LDS)
    extern __shared__ __attribute__((aligned(16))) int8_t lds[];
    __shared__ int sums[WAVES * TOK * CH * 16 * kPitch];
    __shared__ unsigned top[TOK * 16];
    __shared__ float scales[TOK * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (int)blockIdx.x * (16 * CH);
    const int steps = (a.k + 63) / 64, each = (steps + WAVES - 1) / WAVES;
    const int begin = wave * each * 64, end = min(steps, (wave + 1) * each) * 64;
    const int8_t *w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = a.w + (long long)min(n0 + c * 16 + lane % 16, a.n - 1) * a.ldw;
    // Behind the end of a row: with ALIGNED any codes (those of x are 0 there).
    auto load_w = [&](int c, int l) {
        const int at = l + lane / 16 * 16;
        return ALIGNED ? ld_stream((const i32x4 *)(w[c] + min(at, a.k - 16))) : load16(w[c], at, a.k);
    };
    i32x4 cw[kAhead][CH];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (begin + j * 64 < end) cw[j][c] = load_w(c, begin + j * 64);

    const int8_t *x[TOK];
    const int pitch = steps * 64 + 16;                           // of a row of codes in LDS: rows of a 16 begin in different banks
    if constexpr (kQuantize) {
        __builtin_amdgcn_sched_barrier(0);
        // (row, part) pairs go round the wavefronts
        const int parts = max(1, WAVES / a.m), span = ((a.k + parts - 1) / parts + 511) / 512 * 512;
        const X *rows = (const X *)a.raw;
        if (threadIdx.x < TOK * 16) top[threadIdx.x] = 0;
        __syncthreads();
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span;
            unsigned most = 0;
            for (int at = from + lane * 8; at < min(from + span, a.k); at += 512) {
                float v[8];
                load8(rows + row * a.ldx, at, a.k, a.x_vec, v);
                most = max(most, most8(v));
            }
            most = wave_max(most);
            if (lane == 0) atomicMax(&top[row], most);
        }
        __syncthreads();
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span;
            const RowScale r = row_scale(top[row]);
            if (lane == 0) scales[row] = r.s;
            for (int at = from + lane * 8; at < min(from + span, steps * 64); at += 512) {
                float v[8];
                load8(rows + row * a.ldx, at, a.k, a.x_vec, v);
                *(u32x2 *)(lds + row * pitch + at) = codes8(v, r);
            }
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TOK; ++t) x[t] = lds + min(t * 16 + lane % 16, a.m - 1) * pitch;
    } else {
#pragma unroll
        for (int t = 0; t < TOK; ++t) x[t] = a.x + (long long)min(t * 16 + lane % 16, a.m - 1) * a.ldx;
    }
    auto load_x = [&](int t, int l) {
        const int at = l + lane / 16 * 16;
        if constexpr (kQuantize) return *(const i32x4 *)(x[t] + at);
        if (!ALIGNED) return load16(x[t], at, a.k);
        return at < a.kx ? ld_global((const i32x4 *)(x[t] + at)) : (i32x4)0;
    };

    i32x4 sum[CH][TOK];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int t = 0; t < TOK; ++t) sum[c][t] = (i32x4)0;
    for (int l = begin; l < end; l += kAhead * 64) {
        i32x4 cx[kAhead][TOK];
        if (!kQuantize) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
#pragma unroll
                for (int t = 0; t < TOK; ++t)
                    if (l + j * 64 < end) cx[j][t] = load_x(t, l + j * 64);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int at = l + j * 64;
            if (at >= end) break;
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                const i32x4 codes = kQuantize ? load_x(t, at) : cx[j][t];
#pragma unroll
                for (int c = 0; c < CH; ++c) sum[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cw[j][c], codes, sum[c][t], 0, 0, 0);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c)
                if (at + kAhead * 64 < end) cw[j][c] = load_w(c, at + kAhead * 64);
        }
    }
    // lane l has channels 4 (l / 16) to 4 (l / 16) + 3 of token l % 16
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int t = 0; t < TOK; ++t)
            *(i32x4 *)(sums + (((wave * CH + c) * TOK + t) * 16 + lane % 16) * kPitch + lane / 16 * 4) = sum[c][t];
    __syncthreads();
    // four channels of a token to a thread
    for (int i = threadIdx.x; i < CH * TOK * 64; i += WAVES * 64) {
        const int group = i % 4, c = i / 4 % CH, m = i / (4 * CH), n = n0 + c * 16 + group * 4;
        if (m >= a.m || n >= a.n) continue;
        i32x4 all = (i32x4)0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) all += *(const i32x4 *)(sums + ((v * CH + c) * TOK * 16 + m) * kPitch + group * 4);
        const float xs = kQuantize ? scales[m] : ld_global(a.xs + (long long)m * a.xs_step);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = n + e;
            if (j >= a.n) break;
            float y = (float)all[e] * (xs * ld_global(a.ws + (long long)j * a.ws_step));
            if (a.bias) y += ld_global(a.bias + j);
            if (a.y16) st_global((_Float16 *)a.y + (long long)m * a.ldy + j, (_Float16)y);
            else st_global((float *)a.y + (long long)m * a.ldy + j, y);
        }
    }
}

template <typename X, int TOK, int CH> int launch_few(const LinearArgs &a, void *stream)
{
    constexpr int WAVES = 8;
    const unsigned blocks = (unsigned)((a.n + 16 * CH - 1) / (16 * CH));
    const size_t lds = sizeof(X) > 1 ? (size_t)a.m * (size_t)((a.k + 63) / 64 * 64 + 16) : 0;
    if (a.aligned) linear_few_kernel<X, TOK, CH, WAVES, true><<<blocks, WAVES * 64, lds, (hipStream_t)stream>>>(a);
    else linear_few_kernel<X, TOK, CH, WAVES, false><<<blocks, WAVES * 64, lds, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

template <int BM, int BN, int WM, int WN> int launch_tiles(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + BM - 1) / BM * (((long long)a.n + BN - 1) / BN));
    if (a.aligned) linear_tile_kernel<BM, BN, WM, WN, true><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    else linear_tile_kernel<BM, BN, WM, WN, false><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

template <typename T> static int quantize_rows(const QuantizeArgs &a, void *stream)
{
    if (a.k <= 512) quantize_rows_kernel<T, 64, 1><<<((unsigned)a.m + 3) / 4, 256, 0, (hipStream_t)stream>>>(a);
    else if (a.k <= 2048) quantize_rows_kernel<T, 64, 4><<<((unsigned)a.m + 3) / 4, 256, 0, (hipStream_t)stream>>>(a);
    else quantize_rows_kernel<T, 256, 4><<<(unsigned)a.m, 256, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

int launch_quantize_rows(const QuantizeArgs &a, void *stream)
{
    return a.x16 ? quantize_rows<_Float16>(a, stream) : quantize_rows<float>(a, stream);
}

bool linear_quantizes(const LinearArgs &a)
{
    return a.k > 0 && a.m <= 16 && (long long)a.m * (a.k + 80) <= kFewLds;
}

int launch_linear(const LinearArgs &a, void *stream)
{
    if (a.raw) {
        if (a.x16) return launch_few<_Float16, 1, 1>(a, stream);
        return launch_few<float, 1, 1>(a, stream);
    }
    if (a.m <= 64 && a.k > 0) {
        const bool wide = a.n >= 32 * 2 * kComputeUnits;
        if (a.m <= 16) return wide ? launch_few<int8_t, 1, 2>(a, stream) : launch_few<int8_t, 1, 1>(a, stream);
        if (a.m <= 32) return wide ? launch_few<int8_t, 2, 2>(a, stream) : launch_few<int8_t, 2, 1>(a, stream);
        return wide ? launch_few<int8_t, 4, 2>(a, stream) : launch_few<int8_t, 4, 1>(a, stream);
    }
    const long long large = ((long long)a.m + 255) / 256 * (((long long)a.n + 255) / 256);
    if (large >= kComputeUnits) return launch_tiles<256, 256, 2, 4>(a, stream);
    const long long medium = ((long long)a.m + 127) / 128 * (((long long)a.n + 127) / 128);
    if (medium >= kComputeUnits / 2) return launch_tiles<128, 128, 2, 2>(a, stream);
    return launch_tiles<64, 64, 2, 2>(a, stream);
}

}  // namespace fq
