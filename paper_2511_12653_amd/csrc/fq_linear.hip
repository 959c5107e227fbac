// Int8 linear layer with a scale per token and per channel (declared in include/fq.h).
#include <type_traits>

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
// 16 codes at any address.
__device__ __forceinline__ i32x4 load16(const int8_t *p)
{
    i32x4 r;
    __builtin_memcpy(&r, (const FQ_GLOBAL int8_t *)p, 16);
    return r;
}

// 16 codes of a row of k from l on; zeros behind its end.
__device__ __forceinline__ i32x4 load16(const int8_t *row, int l, int k)
{
    i32x4 r = {0, 0, 0, 0};
    if (l + 16 <= k) return load16(row + l);
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
// 128 codes of every row of the tile make a step; LDS holds STAGES of them.  While the matrix cores work on one, the loads of
// the STAGES - 1 next go straight from memory into the others.  A load instruction fills 1 KiB of LDS in lane order, eight rows; which
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

// 16 bytes per lane from `off` of a buffer to LDS, in lane order from `to` on (uniform).  No builtin: with one the compiler
// waits for all such loads in front of a read of LDS wherever it loses sight of which array they go to.  The kernel
// waits itself (loads_and_barrier); the compiler's own waits for other loads only become longer.
__device__ __forceinline__ void load_lds(i32x4 buffer, unsigned off, int8_t *to)
{
    const unsigned at = (unsigned)(uintptr_t)(FQ_LDS int8_t *)to;
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(at), "v"(off), "s"(buffer) : "memory", "m0");
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
    // Load J of codes [at, at + kDepth) of the panel's rows into LDS; lanes with `none` fetch zeros.
    __device__ __forceinline__ void fetch(const Panel &p, int at, int j, int8_t *to, int wave, bool none)
    {
        // (descriptor of a raw buffer: the hardware answers loads behind its end with zeros)
        const uint64_t from = (uint64_t)(p.at + at);
        const i32x4 r = {(int)from, (int)(from >> 32) & 0xFFFF, (int)(p.bytes - (unsigned)at), 0x00027000};
        load_lds(r, none ? kNowhere : off[j], to + (j * WAVES + wave) * 1024);
    }
    // The same by way of registers, for rows at any address.
    __device__ __forceinline__ void request(const int8_t *base, long long ld, int row0, int rows, int at, int k, int lane, int wave)
    {
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int row = min(row0 + (j * WAVES + wave) * 8 + lane / 8, rows - 1);
            const int8_t *from = base + (long long)row * ld;
            const int l = at + ((lane % 8) ^ (lane / 8)) * 16;
            held[j] = at + kDepth <= k ? load16(from + l) : load16(from, l, k);
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

// All loads but the last LEFT of a wavefront have arrived, its reads of LDS are done; and so for all wavefronts.
template <int LEFT> __device__ __forceinline__ void loads_and_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(LEFT) : "memory");
}

template <int BM, int BN, int WM, int WN, int STAGES, bool ALIGNED>
__global__ __launch_bounds__(WM * WN * 64) void linear_tile_kernel(LinearArgs a)
{
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kPitch = TN * 32 + 4;                         // of the sums in LDS
    constexpr int kStage = (BM + BN) * kDepth, kLoads = (BM + BN) / 8 / WAVES;
    static_assert(STAGES >= 2 && STAGES <= 4 && (STAGES == 2 || ALIGNED), "stages");
    static_assert(WAVES * 32 * kPitch * 4 <= 2 * kStage, "the sums of a wavefront's 32 tokens fit in its share");
    // (separate arrays: the compiler then knows that a write of one leaves the others alone)
    __shared__ __attribute__((aligned(1024))) int8_t stage0[kStage], stage1[kStage], stage2[STAGES > 2 ? kStage : 16], stage3[STAGES > 3 ? kStage : 16];
    auto stage = [&](auto i) {
        constexpr int which = i % STAGES;
        if constexpr (which == 0) return &stage0[0];
        else if constexpr (which == 1) return &stage1[0];
        else if constexpr (which == 2) return &stage2[0];
        else return &stage3[0];
    };
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
    const int mine16 = ((lane % 8) ^ (lane / 8)) * 16;          // where in a step this lane's 16 codes lie
    // Loads [from, to) of the kLoads of a step.
    auto ask = [&](auto sure, int step, int8_t *into, int from, int to) {
        if (!sure && step >= steps) return;
        const int at = step * kDepth;
        const bool none = !sure && at + mine16 >= a.kx;
#pragma unroll
        for (int i = from; i < to; ++i) {
            if (i < BN / 8 / WAVES) w.fetch(pw, at, i, into, wave, false);
            else x.fetch(px, at, i - BN / 8 / WAVES, into + BN * kDepth, wave, none);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto ask_slowly = [&](int step) {
        if (step >= steps) return;
        w.request(a.w, a.ldw, n0, a.n, step * kDepth, a.k, lane, wave);
        x.request(a.x, a.ldx, m0, a.m, step * kDepth, a.k, lane, wave);
        __builtin_amdgcn_sched_barrier(0);
    };
    // The codes of step `step` are in LDS for all; those of the STAGES - 2 steps behind it may be on their way.
    auto have = [&](auto sure, int step, int8_t *to) {
        if constexpr (!ALIGNED) {
            if (step < steps) {
                w.put(to, lane, wave);
                x.put(to + BN * kDepth, lane, wave);
            }
            __syncthreads();
        } else if (sure || step + STAGES - 2 < steps) {
            loads_and_barrier<(STAGES - 2) * kLoads>();
        } else {
            loads_and_barrier<0>();
        }
    };
    i32x16 sum[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) sum[j][i] = (i32x16)0;
    // The codes of the next 32 are read from LDS before the products of these 32 are begun; so are the first of the next
    // step, behind the barrier, in front of the last products of this one.
    struct Codes { i32x4 w[TN], x[TM]; } now, then;
    auto read = [&](const int8_t *from, int s, Codes &c) {
        const int8_t *fw = from + (wn + lane % 32) * kDepth, *fx = from + (BN + wm + lane % 32) * kDepth;
        const int at = ((2 * s + lane / 32) ^ (lane % 8)) * 16;
#pragma unroll
        for (int j = 0; j < TN; ++j) c.w[j] = *(const i32x4 *)(fw + j * 32 * kDepth + at);
#pragma unroll
        for (int i = 0; i < TM; ++i) c.x[i] = *(const i32x4 *)(fx + i * 32 * kDepth + at);
        __builtin_amdgcn_sched_barrier(0);
    };
    // Products of quarter q of a step.  Between them, spread over the first three quarters, go the loads of the step that is
    // STAGES - 1 ahead: a wavefront issues them while its matrix core is busy.  (With two stages they have only this step to
    // arrive and go out at its begin: 8192 x 8192 x 8192 471 us against 481 to 504.)
    auto multiply = [&](auto sure, auto q, const Codes &c, int step, int8_t *into) {
        constexpr int kOf = 3 * TM * TN;
#pragma unroll
        for (int p = 0; p < TM * TN; ++p) {
            const int j = p / TM, i = p % TM, at = q * TM * TN + p;
            sum[j][i] = __builtin_amdgcn_mfma_i32_32x32x32_i8(c.w[j], c.x[i], sum[j][i], 0, 0, 0);
            if constexpr (ALIGNED && STAGES > 2 && q < 3) {
                __builtin_amdgcn_sched_barrier(0);
                ask(sure, step, into, at * kLoads / kOf, (at + 1) * kLoads / kOf);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::true_type sure{};
    constexpr std::false_type maybe{};
    constexpr std::integral_constant<int, 0> k0{};
    constexpr std::integral_constant<int, 1> k1{};
    constexpr std::integral_constant<int, 2> k2{};
    constexpr std::integral_constant<int, 3> k3{};
    // Step `step`, in stage i.  Into the stage that the step before has read from, and all wavefronts are past that, go the
    // loads of a later one.  `sure`: a whole step STAGES - 1 ahead is there to be loaded.
    auto advance = [&](auto all, auto i, int step) {
        constexpr std::integral_constant<int, i + 1> ahead{};
        constexpr std::integral_constant<int, i + STAGES - 1> last{};
        const int8_t *from = stage(i);
        int8_t *next = stage(ahead), *into = stage(last);
        if constexpr (!ALIGNED) ask_slowly(step + 1);
        else if constexpr (STAGES == 2) ask(all, step + 1, into, 0, kLoads);
        read(from, 1, then);
        multiply(all, k0, now, step + STAGES - 1, into);
        read(from, 2, now);
        multiply(all, k1, then, step + STAGES - 1, into);
        read(from, 3, then);
        multiply(all, k2, now, step + STAGES - 1, into);
        have(all, step + 1, next);
        read(next, 0, now);
        multiply(all, k3, then, 0, nullptr);
    };
    if constexpr (ALIGNED) {
        ask(maybe, 0, stage0, 0, kLoads);
        if constexpr (STAGES > 2) ask(maybe, 1, stage1, 0, kLoads);
        if constexpr (STAGES > 3) ask(maybe, 2, stage2, 0, kLoads);
    } else {
        ask_slowly(0);
    }
    have(maybe, 0, stage0);
    read(stage0, 0, now);
    int step = 0;
    auto round = [&](auto all) {
        advance(all, k0, step);
        advance(all, k1, step + 1);
        if constexpr (STAGES > 2) advance(all, k2, step + 2);
        if constexpr (STAGES > 3) advance(all, k3, step + 3);
    };
    const int whole = min(a.k, a.kx) / kDepth;                  // whole steps
    for (; step + 2 * STAGES - 2 < whole; step += STAGES) round(sure);
    for (; step + STAGES - 1 < steps; step += STAGES) round(maybe);
    if (step < steps) advance(maybe, k0, step);
    if (STAGES > 2 && step + 1 < steps) advance(maybe, k1, step + 1);
    if constexpr (STAGES > 3) {
        if (step + 2 < steps) advance(maybe, k2, step + 2);
    }
    __syncthreads();

    // 32 tokens at a time: the sums change places through LDS, so that a lane has 8 neighbouring channels of a token and
    // a store instruction whole lines.
    constexpr int kLanes = TN * 32 / 8;                         // that hold a token
    int *const mine = (int *)(wave < WAVES / 2 ? stage0 : stage1) + (wave % (WAVES / 2)) * (32 * kPitch);
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
// Up to 16 tokens: what counts is to stream w once.  A block multiplies 16 channels by all tokens (lanes past the last
// repeat it); its wavefronts share the codes of a row, a run of whole steps of 128 each, and their sums meet in LDS.  Every
// wavefront has kRing steps of w of its own in LDS or on their way there, so it waits for nobody; the layout is that of the
// tiles above.  x lies in LDS as a whole: fetched in front of w, and with X FP16 or FP32 turned into codes by the block while
// w is still coming.
constexpr int kFewWaves = 8, kRing = 4;

struct FewLds {                                                 // where things lie, in bytes behind the rings
    int raw_pitch, raw, code_pitch, codes, total;
};

__host__ __device__ constexpr FewLds few_lds(int m, int k, int size)
{
    FewLds l = {};
    const int ring = kFewWaves * kRing * 16 * kDepth;
    l.raw = ring;
    l.raw_pitch = (k * size + 1023) / 1024 * 1024 + 16;          // (rows of 16 lanes begin in different banks)
    l.code_pitch = size > 1 ? (k + kDepth - 1) / kDepth * kDepth + 16 : l.raw_pitch;
    l.codes = size > 1 ? l.raw + m * l.raw_pitch : l.raw;
    l.total = l.codes + m * l.code_pitch;
    return l;
}

// The last LEFT loads of this wavefront may be on their way, all others and all its LDS reads are done.
template <int LEFT> __device__ __forceinline__ void loads_but()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(LEFT) : "memory");
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

template <typename X>
__global__ __launch_bounds__(kFewWaves * 64) void linear_few_kernel(LinearArgs a)
{
    constexpr int WAVES = kFewWaves, kPitch = 17;                // (of 16 channels' sums in LDS)
    constexpr bool kQuantize = sizeof(X) > 1;
    extern __shared__ __attribute__((aligned(1024))) int8_t lds[];
    __shared__ int sums[16 * kPitch];
    __shared__ unsigned top[16];
    __shared__ float scales[16];
    const FewLds at = few_lds(a.m, a.k, sizeof(X));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (int)blockIdx.x * 16;
    // this thread's output: asked for first, used last
    const int out_m = threadIdx.x / 16, out_n = n0 + (int)threadIdx.x % 16;
    const bool writes = out_m < a.m && out_n < a.n;
    float ws = 0.0f, bias = 0.0f, xs = 0.0f;
    if (writes) {
        ws = ld_global(a.ws + (long long)out_n * a.ws_step);
        if (a.bias) bias = ld_global(a.bias + out_n);
        if (!kQuantize) xs = ld_global(a.xs + (long long)out_m * a.xs_step);
    }
    if (threadIdx.x < 16 * kPitch) sums[threadIdx.x] = 0;
    if (threadIdx.x < 16) top[threadIdx.x] = 0;

    // x: 1 KiB of a row to a load, zeros behind its end
    const int row_bytes = a.k * (int)sizeof(X), pieces = (row_bytes + 1023) / 1024;
    const int8_t *xb = kQuantize ? (const int8_t *)a.raw : a.x;
    for (int i = wave; i < a.m * pieces; i += WAVES) {
        const int row = i / pieces, from = i % pieces * 1024;
        const uint64_t p = (uint64_t)(xb + (long long)row * a.ldx * (int)sizeof(X) + from);
        const i32x4 r = {(int)p, (int)(p >> 32) & 0xFFFF, row_bytes - from, 0x00027000};
        load_lds(r, (unsigned)lane * 16, lds + at.raw + row * at.raw_pitch + from);
    }
    // w
    const int steps = (a.k + kDepth - 1) / kDepth, each = (steps + WAVES - 1) / WAVES;
    const int begin = min(steps, wave * each), end = min(steps, begin + each);
    int8_t *const ring = lds + wave * (kRing * 16 * kDepth);
    const Panel pw = panel(a.w, a.ldw, n0, 16, a.n - n0, a.k);
    Staging<2, 1> w;
    w.place(a.ldw, lane, 0);
    auto ask = [&](int step) {
        if (step >= end) return;
        int8_t *to = ring + (step - begin) % kRing * (16 * kDepth);
        w.fetch(pw, step * kDepth, 0, to, 0, false);
        w.fetch(pw, step * kDepth, 1, to, 0, false);
    };
#pragma unroll
    for (int j = 0; j < kRing; ++j) ask(begin + j);
    // what is left on its way when x has come: the steps of w
    auto arrived = [&](int steps_left) {
        if (steps_left >= 4) loads_but<8>();
        else if (steps_left == 3) loads_but<6>();
        else if (steps_left == 2) loads_but<4>();
        else if (steps_left == 1) loads_but<2>();
        else loads_but<0>();
    };
    arrived(min(kRing, end - begin));
    lds_barrier();

    if constexpr (kQuantize) {
        // (row, part) pairs go round the wavefronts
        constexpr int kEach = 8;
        const int parts = max(1, WAVES / a.m), span = ((a.k + parts - 1) / parts + 511) / 512 * 512;
        auto values = [&](int row, int from, float *v) {
            const X *p = (const X *)(lds + at.raw + row * at.raw_pitch) + from;
#pragma unroll
            for (int e = 0; e < kEach; ++e) v[e] = (float)p[e];
        };
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span;
            unsigned most = 0;
            for (int l = from + lane * kEach; l < min(from + span, a.k); l += 64 * kEach) {
                float v[kEach];
                values(row, l, v);
                most = max(most, most8(v));
            }
            most = wave_max(most);
            if (lane == 0) atomicMax(&top[row], most);
        }
        lds_barrier();
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span;
            const RowScale r = row_scale(top[row]);
            if (lane == 0) scales[row] = r.s;
            for (int l = from + lane * kEach; l < min(from + span, steps * kDepth); l += 64 * kEach) {
                float v[kEach];
                if (l < a.k) values(row, l, v);
                else
#pragma unroll
                    for (int e = 0; e < kEach; ++e) v[e] = 0.0f;
                *(u32x2 *)(lds + at.codes + row * at.code_pitch + l) = codes8(v, r);
            }
        }
        lds_barrier();
    }

    const int8_t *x = lds + at.codes + min(lane % 16, a.m - 1) * at.code_pitch + lane / 16 * 16;
    i32x4 sum = (i32x4)0;
    for (int step = begin; step < end; ++step) {
        arrived(min(kRing - 1, end - 1 - step));
        const int8_t *from = ring + (step - begin) % kRing * (16 * kDepth) + lane % 16 * kDepth;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const i32x4 cw = *(const i32x4 *)(from + ((4 * s + lane / 16) ^ (lane % 8)) * 16);
            const i32x4 cx = *(const i32x4 *)(x + step * kDepth + 64 * s);
            sum = __builtin_amdgcn_mfma_i32_16x16x64_i8(cw, cx, sum, 0, 0, 0);
        }
        if (step + kRing < end) {
            loads_but<63>();                                    // (the reads of this step are done)
            ask(step + kRing);
        }
    }
    // lane l has channels 4 (l / 16) to 4 (l / 16) + 3 of token l % 16
#pragma unroll
    for (int e = 0; e < 4; ++e) atomicAdd(sums + lane % 16 * kPitch + lane / 16 * 4 + e, sum[e]);
    __syncthreads();
    if (!writes) return;
    if (kQuantize) xs = scales[out_m];
    float y = (float)sums[out_m * kPitch + threadIdx.x % 16] * (xs * ws);
    if (a.bias) y += bias;
    if (a.y16) st_global((_Float16 *)a.y + (long long)out_m * a.ldy + out_n, (_Float16)y);
    else st_global((float *)a.y + (long long)out_m * a.ldy + out_n, y);
}

template <typename X> int launch_few(const LinearArgs &a, void *stream)
{
    const int lds = few_lds(a.m, a.k, sizeof(X)).total;
    linear_few_kernel<X><<<((unsigned)a.n + 15) / 16, kFewWaves * 64, (size_t)lds, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int STAGES> int launch_tiles(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + BM - 1) / BM * (((long long)a.n + BN - 1) / BN));
    if (a.aligned) linear_tile_kernel<BM, BN, WM, WN, STAGES, true><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    else linear_tile_kernel<BM, BN, WM, WN, 2, false><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
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

// Up to 16 tokens whose x fits into LDS beside the rings; rows of x and w on 16-byte boundaries and of whole 16 bytes.
static bool takes_few(const LinearArgs &a, int size, bool x_fits)
{
    return a.k > 0 && a.m <= 16 && a.w_fits && x_fits && (long long)a.k * 4 * a.m < (1 << 20) &&
           few_lds(a.m, a.k, size).total <= kFewLds && a.n <= kFewMostN;
}

bool linear_quantizes(const LinearArgs &a) { return takes_few(a, a.x16 ? 2 : 4, a.x_vec && a.k % 16 == 0); }

// The tiles, and what a step of 128 codes of a block takes: at least `wait`, and `work` for each block that a compute unit
// holds at once (`resident` of them at most); `ends` for what is in front of the first step and behind the last (us).
struct Tile {
    int m, n, stages, resident;
    double wait, work, ends;
    int (*launch)(const LinearArgs &, void *);
};

static const Tile kTiles[] = {
    {256, 256, 2, 1, 1.80, 1.80, 2.0, launch_tiles<256, 256, 2, 4, 2>},
    {256, 128, 3, 1, 0.70, 0.98, 2.0, launch_tiles<256, 128, 4, 2, 3>},
    {128, 128, 2, 2, 0.80, 0.56, 2.0, launch_tiles<128, 128, 2, 2, 2>},
    {128, 128, 4, 1, 0.46, 0.56, 2.5, launch_tiles<128, 128, 2, 2, 4>},
    {64, 64, 4, 2, 0.19, 0.21, 1.0, launch_tiles<64, 64, 2, 2, 4>},
    {32, 64, 4, 3, 0.19, 0.12, 1.0, launch_tiles<32, 64, 1, 2, 4>},
};

static double tile_time(const LinearArgs &a, const Tile &t)
{
    const long long blocks = ((long long)a.m + t.m - 1) / t.m * (((long long)a.n + t.n - 1) / t.n);
    const long long once = (long long)kComputeUnits * t.resident, rounds = blocks / once, left = blocks % once;
    const double steps = (double)((a.k + kDepth - 1) / kDepth);
    double time = (double)rounds * (steps * (t.wait > t.resident * t.work ? t.wait : t.resident * t.work) + t.ends);
    if (left) {
        const double each = (double)((left + kComputeUnits - 1) / kComputeUnits) * t.work;
        time += steps * (t.wait > each ? t.wait : each) + t.ends;
    }
    return time;
}

int launch_linear(const LinearArgs &a, void *stream)
{
    if (a.raw) return a.x16 ? launch_few<_Float16>(a, stream) : launch_few<float>(a, stream);
    if (takes_few(a, 1, a.aligned)) return launch_few<int8_t>(a, stream);
#ifdef FQ_V
    if (FQ_V == 1) return launch_tiles<256, 256, 2, 4, 2>(a, stream);
    if (FQ_V == 2) return launch_tiles<256, 128, 4, 2, 3>(a, stream);
    if (FQ_V == 3) return launch_tiles<128, 128, 2, 2, 2>(a, stream);
    if (FQ_V == 4) return launch_tiles<128, 128, 2, 2, 4>(a, stream);
    if (FQ_V == 5) return launch_tiles<64, 64, 2, 2, 4>(a, stream);
    if (FQ_V == 6) return launch_tiles<64, 128, 1, 4, 3>(a, stream);
    if (FQ_V == 14) return launch_tiles<32, 64, 1, 2, 4>(a, stream);
    if (FQ_V == 15) return launch_tiles<32, 128, 1, 4, 4>(a, stream);
    if (FQ_V == 16) return launch_tiles<32, 64, 1, 2, 3>(a, stream);
#endif
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < (int)(sizeof kTiles / sizeof kTiles[0]); ++i) {
        if (!a.aligned && kTiles[i].stages > 2 && kTiles[i].m != 64) continue;   // (64 x 64: launched with two)
        const double t = tile_time(a, kTiles[i]);
        if (least == 0.0 || t < least) { least = t; best = i; }
    }
    return kTiles[best].launch(a, stream);
}

}  // namespace fq
