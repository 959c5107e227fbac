// Int8 linear layer with a scale per token and per channel (declared in include/fq.h).
//
//   y_ij = (sum_k q_ik w_jk) * (xs_i * ws_j) + bias_j          the sum exact in 32 bits, the rest in binary32
//   xs_i = max_k |x_ik| / 127,  q_ik = round(x_ik / xs_i)      where x comes in FP16 or FP32
//
// Few tokens: linear_few_kernel, which with up to 16 and room for them in LDS does all of it in one launch, bound by the stream of w.
// Short rows and few channels: linear_rows_kernel, one launch, bound by x and y.  All else: quantize_rows_kernel, bound by memory, and
// linear_tile_kernel, bound by the matrix cores or, in few tiles, by what a compute unit can load.  Quantizing inside the tiles would do
// it again for every tile of channels: n / 256 times.  Sizes below are m x n x k, tokens by channels by values of a row.
#include <type_traits>

#include "fq_device.h"
#include "fq_linear.h"
#include "fq_rows.h"

namespace fq {
namespace {

using namespace dev;

typedef int i32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------------------------
// Rows of codes at any address, laid out anew for the tiles: on 16-byte boundaries, zeros behind k.  A thread moves 16.
__device__ __forceinline__ void align_rows(const AlignArgs &a, unsigned block)
{
    const unsigned each = (unsigned)(a.pitch / 16);
    const unsigned long long i = (unsigned long long)block * 256 + threadIdx.x;
    const long long row = (long long)(i / each);
    const int l = (int)(i % each) * 16;
    if (row >= a.rows) return;
    const int8_t *from = a.from + row * a.ld + l;
    i32x4 r = {0, 0, 0, 0};
    if (l + 16 <= a.k) {
        __builtin_memcpy(&r, (const FQ_GLOBAL int8_t *)from, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (l + j < a.k) r[j / 4] |= (int)((unsigned)(unsigned char)ld_global(from + j) << (8 * (j % 4)));
    }
    *(FQ_GLOBAL i32x4 *)(a.to + row * a.pitch + l) = r;
}

__global__ __launch_bounds__(256) void align_rows_kernel(AlignArgs a, unsigned blocks, AlignArgs other)
{
    if (blockIdx.x < blocks) align_rows(a, blockIdx.x);
    else align_rows(other, blockIdx.x - blocks);
}

// A row to L lanes, from the loads to the codes in their registers: x is read once.  (Rows of more than 8 * L * V values are read
// again for the codes; the second time they come from the caches.)  Bound by memory: 8192 x 8192 FP16 31.4 us, 6.4 TB/s; 600 x 4096
// 5.0 us, mostly the way to memory and back.  Short rows share a wavefront: what a row costs beside its values is paid
// once for four (19200 x 384 5.6 us).
//
// The blocks behind the first `blocks` lay out w instead, where its rows begin at any address: 301 x 600 x 437 FP32 7.9 us
// against 10.4 with a launch of its own for that.
template <typename T, int L, int V>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantizeArgs a, unsigned blocks, AlignArgs other)
{
    if (blockIdx.x >= blocks) {
        align_rows(other, blockIdx.x - blocks);
        return;
    }
    __shared__ unsigned top[4];
    const int at = threadIdx.x % L * 8;
    const long long row = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
    const T *x = (const T *)a.x + min(row, (long long)a.m - 1) * a.ldx;
    Eight<T> raw[V];
#pragma unroll
    for (int j = 0; j < V; ++j) raw[j] = ask8(x, j * L * 8 + at, a.k);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < V; ++j) odd_end(raw[j], x, j * L * 8 + at, a.k);
    unsigned most = most_of(raw);
    for (int i = V * L * 8 + at; i < a.k; i += L * 8) {
        Eight<T> more[1] = {ask8(x, i, a.k)};
        odd_end(more[0], x, i, a.k);
        most = max(most, most_of(more));
    }
    most = L == 16 ? max16(most) : wave_max(most);
    if (L == 256) {
        if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = most;
        __syncthreads();
        most = max(max(top[0], top[1]), max(top[2], top[3]));
    }
    const RowScale r = row_scale(most);
    if (row >= a.m) return;
    if (at == 0) st_global(a.s + row, r.s);
    int8_t *q = a.q + row * a.pitch;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int i = j * L * 8 + at;
        if (i < a.pitch) *(FQ_GLOBAL u32x2 *)(q + i) = codes8(raw[j], r, i >= a.k);
    }
    for (int i = V * L * 8 + at; i < a.pitch; i += L * 8) {
        Eight<T> more = ask8(x, i, a.k);
        odd_end(more, x, i, a.k);
        *(FQ_GLOBAL u32x2 *)(q + i) = codes8(more, r, i >= a.k);
    }
}

// ---------------------------------------------------------------------------------------------
// Product of a tile of BM tokens by BN channels.  What bounds it, by tile: 256 x 256 the matrix cores, which are busy 65 % of the
// cycles at a clock that their power holds down (8192 x 8192 x 8192 460 us, 2.39 POP/s; codes that are all zero are 12 to 25 % faster);
// the smaller ones, taken where large ones leave compute units without work, what a compute unit can move by itself: a 128 x 128 step, 32 KiB
// from the L2s and 96 through LDS, takes 0.30 us with 32 or 64 blocks on the chip and 0.36 with 160 (the matrix cores work 0.21 of it), a 64 x 64
// step of 16 KiB 0.15.  More stages, and codes read from LDS a whole step ahead, change neither (5 % either way).
//
// BM / WM by BN / WN of it belong to a wavefront, which builds them from
// 32 x 32 matrix instructions: lane l holds 16 codes of channel l % 32 and of token l % 32, and of the sums those of token
// l % 32 and channels 8 g + 4 (l / 32) + 0..3, g = 0..3.
//
// 128 codes of every row of the tile make a step; LDS holds STAGES of them.  While the matrix cores work on one, the loads of
// the STAGES - 1 next go straight from memory into the others.  A load instruction fills 1 KiB of LDS in lane order, eight rows; which
// 16 codes a lane fetches is free.  LDS answers 16 lanes at a time, from 64 banks: 16 places of 16 bytes, two rows of them.  So
// the codes at 16 c of row r lie at place c ^ (r / 2 % 8) of it: 16 neighbouring rows have theirs in 16 places.  (At
// c ^ (r % 8) half of the cycles that LDS worked were conflicts.  The times are the same: not LDS bounds these kernels.)
constexpr int kDepth = 128;                                     // codes of a row per step

__device__ __forceinline__ int place_of(int chunk, int row) { return chunk ^ (row / 2 & 7); }      // (its own inverse in chunk)
constexpr unsigned kNowhere = 0x7FFFFFF0u;                      // beyond the end of any buffer: reads as zeros

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

    // (shift: where in 16 bytes the first row begins; a row's loads begin at the boundary in front of it)
    __device__ __forceinline__ void place(long long ld, int lane, int wave, unsigned shift = 0)
    {
#pragma unroll
        for (int j = 0; j < N; ++j)
            off[j] = (((unsigned)((j * WAVES + wave) * 8 + lane / 8) * (unsigned)ld + shift) & ~15u) +
                     (unsigned)place_of(lane % 8, (j * WAVES + wave) * 8 + lane / 8) * 16;
    }
    // Load J of codes [at, at + kDepth) of the panel's rows into LDS; lanes with `none` fetch zeros.
    __device__ __forceinline__ void fetch(const Panel &p, int at, int j, int8_t *to, int wave, bool none)
    {
        // (descriptor of a raw buffer: the hardware answers loads behind its end with zeros)
        const uint64_t from = (uint64_t)(p.at + at);
        const i32x4 r = {(int)from, (int)(from >> 32) & 0xFFFF, (int)(p.bytes - (unsigned)at), 0x00027000};
        load_lds(r, none ? kNowhere : off[j], to + (j * WAVES + wave) * 1024);
    }
};

// What a wavefront's lanes have written to LDS before is what its lanes read behind.
__device__ __forceinline__ void lanes_in_step()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// N neighbouring channels of a token, `left` of which there are (WHOLE: all).  Vector stores take any address.  LINES: the
// lanes of this one instruction write whole lines, which then need not wait in the caches for the rest of them: 19200 x 384 x 384
// of codes 10.2 -> 8.7 us, 8192 x 8192 x 8192 479 -> 470, 12000 x 2048 x 600 FP32 44.8 -> 40.9; for parts of lines it is the other way, 20000 x
// 1000 x 64 FP32 28.7 -> 48.9.
template <bool HALF, bool WHOLE, bool LINES, int N> __device__ __forceinline__ void store_channels(char *at, const float *y, int left)
{
    typedef typename std::conditional<HALF, _Float16, float>::type T;
    typedef T V __attribute__((ext_vector_type(HALF ? N : 4)));
    if (WHOLE || left >= N) {
#pragma unroll
        for (int p = 0; p < (HALF ? 1 : N / 4); ++p) {
            V v;
#pragma unroll
            for (int e = 0; e < (HALF ? N : 4); ++e) v[e] = (T)y[p * 4 + e];
            if constexpr (LINES) __builtin_nontemporal_store(v, (FQ_GLOBAL V *)((FQ_GLOBAL char *)at + p * sizeof v));
            else __builtin_memcpy((FQ_GLOBAL char *)at + p * sizeof v, &v, sizeof v);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < left) st_global((T *)at + e, (T)y[e]);
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

template <int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void linear_tile_kernel(LinearArgs a)
{
    constexpr int WAVES = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
    constexpr int kPitch = TN * 32 + 4;                         // of the sums in LDS
    constexpr int kStage = (BM + BN) * kDepth, kLoads = (BM + BN) / 8 / WAVES;
    static_assert(STAGES >= 2 && STAGES <= 4, "stages");
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
    const Panel pw = panel(a.w, a.ldw, n0, BN, a.n - n0, a.kw), px = panel(a.x, a.ldx, m0, BM, a.m - m0, a.kx);
    w.place(a.ldw, lane, wave);
    x.place(a.ldx, lane, wave);
    const int steps = (a.k + kDepth - 1) / kDepth;
    static_assert(WAVES % 2 == 0, "a wavefront's loads differ by multiples of 16 rows");
    const int mine16 = place_of(lane % 8, wave * 8 + lane / 8) * 16;     // where in a step this lane's 16 codes lie
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
    // The codes of step `step` are in LDS for all; those of the STAGES - 2 steps behind it may be on their way.
    auto have = [&](auto sure, int step) {
        if (sure || step + STAGES - 2 < steps) loads_and_barrier<(STAGES - 2) * kLoads>();
        else loads_and_barrier<0>();
    };
    i32x16 sum[TN][TM];
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int i = 0; i < TM; ++i) sum[j][i] = (i32x16)0;
    // What the end needs, asked for at the begin where there are registers for it.  A lane ends with eight channels of tokens m_lane +
    // kTokens * (0, 1, ...): n_lane to n_lane + 3 and `apart` behind them, so that the lanes of a store have neighbouring 16 bytes
    // (12000 x 2048 x 600 FP32 53.0 us with 32 bytes of a lane in two stores, 44.8 so).
    constexpr int kLanes = TN * 32 / 8, kTokens = 64 / kLanes, kRows = 32 / kTokens;      // lanes of a token, tokens at once, times
    constexpr bool kEarly = TM * TN <= 4;
    const int apart = a.y16 ? 4 : kLanes * 4, at_lane = lane % kLanes * (a.y16 ? 8 : 4), n_lane = n0 + wn + at_lane, m_lane = m0 + wm + lane / kLanes;
    float ws[8], bias[8], xs[TM * kRows];
    auto ask_scales = [&] {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = min(n_lane + e % 4 + e / 4 * apart, a.n - 1);
            ws[e] = ld_global(a.ws + (long long)j * a.ws_step);
            bias[e] = a.bias ? ld_global(a.bias + j) : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < TM * kRows; ++i)
            xs[i] = ld_global(a.xs + (long long)min(m_lane + i / kRows * 32 + i % kRows * kTokens, a.m - 1) * a.xs_step);
        __builtin_amdgcn_sched_barrier(0);
    };
    if constexpr (kEarly) ask_scales();
    // The codes of the next 32 are read from LDS before the products of these 32 are begun; so are the first of the next
    // step, behind the barrier, in front of the last products of this one.
    struct Codes { i32x4 w[TN], x[TM]; } now, then;
    auto read = [&](const int8_t *from, int s, Codes &c) {
        const int8_t *fw = from + (wn + lane % 32) * kDepth, *fx = from + (BN + wm + lane % 32) * kDepth;
        const int at = place_of(2 * s + lane / 32, lane % 32) * 16;
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
            if constexpr (STAGES > 2 && q < 3) {
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
        const int8_t *next = stage(ahead);
        int8_t *into = stage(last);
        if constexpr (STAGES == 2) ask(all, step + 1, into, 0, kLoads);
        read(from, 1, then);
        multiply(all, k0, now, step + STAGES - 1, into);
        read(from, 2, now);
        multiply(all, k1, then, step + STAGES - 1, into);
        read(from, 3, then);
        multiply(all, k2, now, step + STAGES - 1, into);
        have(all, step + 1);
        read(next, 0, now);
        multiply(all, k3, then, 0, nullptr);
    };
    ask(maybe, 0, stage0, 0, kLoads);
    if constexpr (STAGES > 2) ask(maybe, 1, stage1, 0, kLoads);
    if constexpr (STAGES > 3) ask(maybe, 2, stage2, 0, kLoads);
    have(maybe, 0);
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
    int *const mine = (int *)(wave < WAVES / 2 ? stage0 : stage1) + (wave % (WAVES / 2)) * (32 * kPitch);
    if constexpr (!kEarly) ask_scales();
    auto finish = [&](auto half, auto whole, auto lines) {
        const long long row_bytes = a.ldy * (half ? 2 : 4);
        char *const y0 = (char *)a.y + (long long)m_lane * row_bytes + (long long)n_lane * (half ? 2 : 4);
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
            for (int t = 0; t < kRows; ++t) {
                const int row = i * 32 + t * kTokens;
                const int *from = mine + (t * kTokens + lane / kLanes) * kPitch + at_lane;
                const i32x4 low = *(const i32x4 *)from, high = *(const i32x4 *)(from + apart);
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = (float)(e < 4 ? low[e] : high[e - 4]) * (xs[i * kRows + t] * ws[e]);
                if (a.bias)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] += bias[e];
                if (m_lane + row >= a.m) continue;
                if constexpr (half) {
                    store_channels<true, whole, lines, 8>(y0 + row * row_bytes, y, a.n - n_lane);
                } else {
                    store_channels<false, whole, lines, 4>(y0 + row * row_bytes, y, a.n - n_lane);
                    store_channels<false, whole, lines, 4>(y0 + row * row_bytes + apart * 4, y + 4, a.n - n_lane - apart);
                }
            }
            lanes_in_step();
        }
    };
    constexpr std::bool_constant<TN == 2> line{};               // 64 channels of FP16, 32 of FP32
    if (n0 + wn + TN * 32 <= a.n) {
        if (a.y16 && line && a.y_lines) finish(sure, sure, line);
        else if (a.y16) finish(sure, sure, maybe);
        else if (line && a.y_lines) finish(maybe, sure, line);
        else finish(maybe, sure, maybe);
    } else {
        if (a.y16) finish(sure, maybe, maybe);
        else finish(maybe, maybe, maybe);
    }
}

// ---------------------------------------------------------------------------------------------
// Few tokens: what counts is to stream w once (1 x 4096 x 4096 FP16 5.4 us a call, 16.8 MB of w, of which the launch
// of an empty kernel is 1.7).  A block multiplies 16 channels by all tokens, up to 16 (lanes past the last
// repeat it); its wavefronts share the codes of a row, a run of whole steps of 128 each, and their sums meet in LDS.  Every
// wavefront has kRing steps of w of its own in LDS or on their way there, so it waits for nobody; the layout is that of the
// tiles above.  x lies in LDS as a whole: fetched in front of w, and with X FP16 or FP32 turned into codes by the block while
// w is still coming.
// Rows that do not begin on 16-byte boundaries (SHIFTED: of w or x) are fetched from the boundary in front of them on.  A step then
// is 112 codes, and the 16 of a lane are cut out of two neighbouring 16 bytes; the last quarter of the second product has
// zeros for x.
// Codes of x that leave no room in LDS, and those of more tokens (RINGED: 16, or 32 to a block and more along blockIdx.y), come
// through the rings, too, step by step beside those of w, and may lie at any address like those (16 x 1000 x 1155 codes 4.3 us, laid
// out anew first 7.5).
constexpr int kFewWaves = 8, kRing = 4;

// What the rings hold: 16 rows of w, and with x in them 16 or 32 of x; three steps of the latter.
constexpr int few_slot(int of_x) { return (16 + of_x) * kDepth; }
constexpr int few_ring(int of_x) { return of_x > 16 ? kRing - 1 : kRing; }
constexpr int few_ringed(int of_x) { return kFewWaves * few_ring(of_x) * few_slot(of_x); }

struct FewLds {                                                 // where things lie, in bytes behind the rings
    int use, steps, pieces, raw_pitch, raw, code_pitch, codes, total;
};

__host__ __device__ constexpr FewLds few_lds(int m, int k, int size, bool shifted)
{
    FewLds l = {};
    l.use = shifted ? kDepth - 16 : kDepth;
    l.steps = (k + l.use - 1) / l.use;
    l.raw = kFewWaves * kRing * 16 * kDepth;
    // (of a row of x: values as they lie in memory from a 16-byte boundary on, or codes with zeros to the end of the last step)
    l.pieces = ((size > 1 ? k * size + 15 : l.steps * l.use) + 1023) / 1024;
    l.raw_pitch = l.pieces * 1024 + 16;                          // (rows of 16 lanes begin in different banks)
    l.code_pitch = size > 1 ? l.steps * l.use + 32 - (l.steps * l.use % 32 == 0 ? 16 : 0) : l.raw_pitch;
    l.codes = size > 1 ? l.raw + m * l.raw_pitch : l.raw;
    l.total = l.codes + m * l.code_pitch + 32;                   // (a shifted last step reads 16 codes more)
    return l;
}

__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// Bytes [o, o + 16) of 32.
__device__ __forceinline__ i32x4 cut16(i32x4 low, i32x4 high, int o)
{
    const auto pick = [](int which, int no, int yes) { return which ? yes : no; };
    int t[7], e[5];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        t[j] = pick(o & 4, low[j], low[j + 1]);
        t[j + 4] = pick(o & 4, high[j], high[j + 1]);
    }
    t[3] = pick(o & 4, low[3], high[0]);
#pragma unroll
    for (int j = 0; j < 5; ++j) e[j] = pick(o & 8, t[j], t[j + 2]);
    i32x4 r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = (int)__builtin_amdgcn_alignbyte((unsigned)e[j + 1], (unsigned)e[j], (unsigned)o & 3u);
    return r;
}

// The first n bytes of 16, zeros behind them.
__device__ __forceinline__ i32x4 first16(i32x4 v, int n)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int bits = min(max(n - 4 * j, 0), 4) * 8;
        v[j] &= (int)(unsigned)((1ull << bits) - 1);
    }
    return v;
}

template <typename X, bool SHIFTED, int RINGED = 0>
__global__ __launch_bounds__(kFewWaves * 64) void linear_few_kernel(LinearArgs a)
{
    static_assert(!RINGED || sizeof(X) == 1, "values to quantize lie in LDS");
    constexpr int WAVES = kFewWaves, kPitch = 17, kGroups = RINGED > 16 ? 2 : 1;      // (pitch of 16 channels' sums in LDS; 16 tokens each)
    constexpr bool kQuantize = sizeof(X) > 1;
    constexpr int kUse = SHIFTED ? kDepth - 16 : kDepth, kDeep = few_ring(RINGED), kSlot = few_slot(RINGED), kLoads = kSlot / 1024;
    extern __shared__ __attribute__((aligned(1024))) int8_t lds[];
    __shared__ int sums[kGroups * 16 * kPitch];
    __shared__ unsigned top[16];
    __shared__ float scales[16];
    const FewLds at = few_lds(RINGED ? 0 : a.m, a.k, sizeof(X), SHIFTED);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = (int)blockIdx.x * 16;
    const int m0 = RINGED ? (int)blockIdx.y * RINGED : 0;
    // this thread's output: asked for first, used last
    const int out_m = m0 + (int)threadIdx.x / 16, out_n = n0 + (int)threadIdx.x % 16;
    const bool writes = out_m < a.m && out_n < a.n && (!RINGED || (int)threadIdx.x < RINGED * 16);
    float ws = 0.0f, bias = 0.0f, xs = 0.0f;
    if (writes) {
        ws = ld_global(a.ws + (long long)out_n * a.ws_step);
        if (a.bias) bias = ld_global(a.bias + out_n);
        if (!kQuantize) xs = ld_global(a.xs + (long long)out_m * a.xs_step);
    }
    for (int i = threadIdx.x; i < kGroups * 16 * kPitch; i += WAVES * 64) sums[i] = 0;
    if (threadIdx.x < 16) top[threadIdx.x] = 0;

    // x: 1 KiB of a row to a load, zeros behind the 16 bytes with its end
    auto row_of_x = [&](int row) { return (uint64_t)(kQuantize ? (const int8_t *)a.raw : a.x) + (uint64_t)row * (uint64_t)a.ldx * sizeof(X); };
    for (int i = wave; !RINGED && i < a.m * at.pieces; i += WAVES) {
        const int row = i / at.pieces, from = i % at.pieces * 1024;
        const uint64_t begins = row_of_x(row), p = (begins & ~15ull) + from;
        const int bytes = max(0, ((int)(begins & 15) + a.k * (int)sizeof(X) + 15) / 16 * 16 - from);
        const i32x4 r = {(int)p, (int)(p >> 32) & 0xFFFF, bytes, 0x00027000};
        load_lds(r, (unsigned)lane * 16, lds + at.raw + row * at.raw_pitch + from);
    }
    // w
    const int each = (at.steps + WAVES - 1) / WAVES;
    const int begin = min(at.steps, wave * each), end = min(at.steps, begin + each);
    int8_t *const ring = lds + wave * (kDeep * kSlot);
    const int8_t *const w0 = a.w + (long long)n0 * a.ldw;
    const int shift0 = SHIFTED ? (int)((uint64_t)w0 & 15) : 0;
    const Panel pw = {w0 - shift0, ((unsigned)(min(16, a.n - n0) - 1) * (unsigned)a.ldw + (unsigned)(shift0 + a.k) + 15) / 16 * 16};
    Staging<2, 1> w;
    w.place(a.ldw, lane, 0, (unsigned)shift0);
    const int8_t *const x0 = a.x + (long long)m0 * a.ldx;
    const int front = RINGED && SHIFTED ? (int)((uint64_t)x0 & 15) : 0;       // (0 where rows of x fit)
    const Panel px = {x0 - front, ((unsigned)(min(kGroups * 16, a.m - m0) - 1) * (unsigned)a.ldx + (unsigned)(front + a.kx) + 15) / 16 * 16};
    Staging<2 * kGroups, 1> rows;
    if (RINGED) rows.place(a.ldx, lane, 0, (unsigned)front);
    auto ask = [&](int step) {
        if (step >= end) return;
        int8_t *to = ring + (step - begin) % kDeep * kSlot;
        w.fetch(pw, step * kUse, 0, to, 0, false);
        w.fetch(pw, step * kUse, 1, to, 0, false);
        if (RINGED) {
#pragma unroll
            for (int j = 0; j < 2 * kGroups; ++j)
                rows.fetch(px, step * kUse, j, to + 16 * kDepth, 0, a.x_fits && step * kUse + place_of(lane % 8, j * 8 + lane / 8) * 16 >= a.kx);
        }
    };
#pragma unroll
    for (int j = 0; j < kDeep; ++j) ask(begin + j);
    // what is left on its way when x has come: the steps of w
    auto arrived = [&](int steps_left) {
        if (steps_left >= 4) loads_but<4 * kLoads>();
        else if (steps_left == 3) loads_but<3 * kLoads>();
        else if (steps_left == 2) loads_but<2 * kLoads>();
        else if (steps_left == 1) loads_but<kLoads>();
        else loads_but<0>();
    };
    arrived(min(kDeep, end - begin));
    lds_barrier();

    if constexpr (kQuantize) {
        // (row, part) pairs go round the wavefronts
        const int parts = max(1, WAVES / a.m), span = ((a.k + parts - 1) / parts + 511) / 512 * 512;
        auto values = [&](const X *p, bool whole, int from) {
            if (!SHIFTED || (whole && from + 8 <= a.k)) return *(const Eight<X> *)__builtin_assume_aligned(p + from, 16);
            typename Values<X>::type v;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = from + e < a.k ? p[from + e] : (X)0;
            return __builtin_bit_cast(Eight<X>, v);
        };
        const int padded = at.steps * kUse;
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span, shift = (int)(row_of_x(row) & 15);
            const X *p = (const X *)(lds + at.raw + row * at.raw_pitch + shift);
            unsigned most = 0;
            for (int l = from + lane * 8; l < min(from + span, a.k); l += 512) {
                const Eight<X> v[1] = {values(p, shift == 0, l)};
                most = max(most, most_of(v));
            }
            most = wave_max(most);
            if (lane == 0) atomicMax(&top[row], most);
        }
        lds_barrier();
        for (int i = wave; i < a.m * parts; i += WAVES) {
            const int row = i / parts, from = i % parts * span, shift = (int)(row_of_x(row) & 15);
            const X *p = (const X *)(lds + at.raw + row * at.raw_pitch + shift);
            const RowScale r = row_scale(top[row]);
            if (lane == 0) scales[row] = r.s;
            // (the last part also fills up the last step)
            const int to = i % parts == parts - 1 ? padded : min(from + span, padded);
            for (int l = from + lane * 8; l < to; l += 512)
                *(u32x2 *)(lds + at.codes + row * at.code_pitch + l) = codes8(values(p, shift == 0, min(l, a.k)), r, l >= a.k);
        }
        lds_barrier();
    }

    const int8_t *x = lds + at.codes + min(lane % 16, a.m - 1) * at.code_pitch + lane / 16 * 16;
    const int shift = SHIFTED ? (int)((uint64_t)(w0 + (long long)(lane % 16) * a.ldw) & 15) : 0;
    i32x4 sum[kGroups];
#pragma unroll
    for (int g = 0; g < kGroups; ++g) sum[g] = (i32x4)0;
    for (int step = begin; step < end; ++step) {
        arrived(min(kDeep - 1, end - 1 - step));
        const int8_t *from = ring + (step - begin) % kDeep * kSlot + lane % 16 * kDepth;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int c = 4 * s + lane / 16;
            i32x4 cw = *(const i32x4 *)(from + place_of(c, lane % 16) * 16);
            if (SHIFTED) cw = cut16(cw, *(const i32x4 *)(from + place_of((c + 1) & 7, lane % 16) * 16), shift);
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                i32x4 cx = *(const i32x4 *)(RINGED ? from + (g + 1) * 16 * kDepth + place_of(c, lane % 16) * 16 : x + step * kUse + 64 * s);
                if (SHIFTED && RINGED && !a.x_fits) {
                    const int8_t *more = from + (g + 1) * 16 * kDepth + place_of((c + 1) & 7, lane % 16) * 16;
                    cx = first16(cut16(cx, *(const i32x4 *)more, (int)((uint64_t)(x0 + (long long)(g * 16 + lane % 16) * a.ldx) & 15)),
                                 a.k - step * kUse - c * 16);
                }
                if (SHIFTED && c == 7) cx = (i32x4)0;
                sum[g] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cw, cx, sum[g], 0, 0, 0);
            }
        }
        if (step + kDeep < end) {
            loads_but<63>();                                    // (the reads of this step are done)
            ask(step + kDeep);
        }
    }
    // lane l has channels 4 (l / 16) to 4 (l / 16) + 3 of token l % 16
#pragma unroll
    for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int e = 0; e < 4; ++e) atomicAdd(sums + (g * 16 + lane % 16) * kPitch + lane / 16 * 4 + e, sum[g][e]);
    __syncthreads();
    if (!writes) return;
    if (kQuantize) xs = scales[out_m];
    float y = (float)sums[threadIdx.x / 16 * kPitch + threadIdx.x % 16] * (xs * ws);
    if (a.bias) y += bias;
    if (a.y16) st_global((_Float16 *)a.y + (long long)out_m * a.ldy + out_n, (_Float16)y);
    else st_global((float *)a.y + (long long)out_m * a.ldy + out_n, y);
}

// Whether all rows of x and w begin on 16-byte boundaries and consist of whole 16 values.
bool few_fits(const LinearArgs &a) { return a.w_fits && (!a.raw || a.x_vec); }

// LDS of a block with x as a whole there, at any alignment; more than there is for more than 16 tokens.
long long few_most(const LinearArgs &a, int size)
{
    return a.m > 16 || (long long)a.m * a.k * size > kFewLds ? kFewLds + 1 : few_lds(a.m, a.k, size, true).total;
}

template <int RINGED> int launch_ringed(const LinearArgs &a, unsigned blocks, void *stream)
{
    const dim3 grid(blocks, ((unsigned)a.m + RINGED - 1) / RINGED);
    if (a.w_fits && a.x_fits) linear_few_kernel<int8_t, false, RINGED><<<grid, kFewWaves * 64, few_ringed(RINGED), (hipStream_t)stream>>>(a);
    else linear_few_kernel<int8_t, true, RINGED><<<grid, kFewWaves * 64, few_ringed(RINGED), (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

template <typename X> int launch_few(const LinearArgs &a, void *stream)
{
    const unsigned blocks = ((unsigned)a.n + 15) / 16;
    // (32 tokens to a block where 16 would make more blocks than compute units.  us, 32 / 16 where they do not: 385 x 64 x 6448 codes 7.4 / 5.6,
    // 32 x 2048 x 14336 10.2 / 8.2, 112 x 384 x 668 4.4 / 4.4.)
    if constexpr (sizeof(X) == 1)
        if (few_most(a, 1) > kFewLds || !a.x_fits)
            return ((long long)a.m + 15) / 16 * blocks <= kComputeUnits || a.m <= 16 ? launch_ringed<16>(a, blocks, stream) : launch_ringed<32>(a, blocks, stream);
    const size_t lds = (size_t)few_lds(a.m, a.k, sizeof(X), !few_fits(a)).total;
    if (few_fits(a)) linear_few_kernel<X, false><<<blocks, kFewWaves * 64, lds, (hipStream_t)stream>>>(a);
    else linear_few_kernel<X, true><<<blocks, kFewWaves * 64, lds, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

// ---------------------------------------------------------------------------------------------
// Short rows, many tokens: x is read once and its codes never leave the compute unit (288000 x 128 x 128 FP16 50.0 us, 2.9 TB/s of x and
// y; codes by a launch of their own and tiles 58.5).  A block has TOK * 16 tokens.  It turns
// them into codes in LDS, a row to 16 lanes, V vectors each, with all of a wavefront's rows requested before the first is
// looked at; then every wavefront multiplies all of them by 16 * CH channels at a time.  w, small enough to stay in the L2s,
// goes from there into registers, whole rows of it: the first before x is quantized, the next as the last are used up.  Which rows
// make one matrix instruction's 16 is free: those with which a store's lanes have the longest runs, 4 * CH channels of a token to a
// lane of FP16 (20000 x 1000 x 64 16.4 -> 14.8 us), 4 with the neighbouring lanes' behind them of FP32 (the other way 19.1 -> 22.9).
//
// w may lie at any address: where k is no multiple of 16, its last codes are fetched as those of the 16 that end with the row, and the
// codes of x are laid out for that (end_behind).  With many channels and few tokens, blockIdx.y shares the channels out: x, small then,
// is quantized once for each.
constexpr int kRowsWaves = 8, kRowsLeastK = 16, kRowsMostK = 512;

// Codes l to l + 7 of a row of k, no multiple of 16, in lanes of which an even and the odd one behind it have 16; of the row's last k % 16 codes the
// 16 end with them instead of beginning with them, zeros in front.
__device__ __forceinline__ u32x2 end_behind(u32x2 c, int l, int k)
{
    const auto swap = [](unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false); };
    const u32x2 o = u32x2{swap(c[0]), swap(c[1])};
    const uint64_t own = __builtin_bit_cast(uint64_t, c), other = __builtin_bit_cast(uint64_t, o);
    const uint64_t first = l & 8 ? other : own, second = l & 8 ? own : other;
    const int by = 128 - k % 16 * 8;                            // bits, 8 to 120
    const uint64_t low = by < 64 ? first << by : 0;
    const uint64_t high = by < 64 ? second << by | first >> (64 - by) : first << (by - 64);
    return (l & ~15) == (k & ~15) ? __builtin_bit_cast(u32x2, l & 8 ? high : low) : c;
}

template <typename X, int TOK, int CH, int V>
__global__ __launch_bounds__(kRowsWaves * 64) void linear_rows_kernel(LinearArgs a)
{
    constexpr int WAVES = kRowsWaves, kRows = TOK * 16, kPasses = (kRows + 4 * WAVES - 1) / (4 * WAVES), kSteps = V * 2;
    __shared__ __attribute__((aligned(16))) int8_t codes[kRows * (kSteps * 64 + 16)];
    __shared__ float scales[kRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m0 = (int)blockIdx.x * kRows, steps = (a.k + 63) / 64, pitch = steps * 64 + 16;

    auto row_of = [&](int r) { return (r * WAVES + wave) * 4 + lane / 16; };
    auto row_of_x = [&](int r) { return (const X *)a.raw + (long long)min(m0 + row_of(r), a.m - 1) * a.ldx; };
    Eight<X> raw[kPasses][V];
#pragma unroll
    for (int r = 0; r < kPasses; ++r)
        if ((r * WAVES + wave) * 4 < kRows)
#pragma unroll
            for (int j = 0; j < V; ++j) raw[r][j] = ask8(row_of_x(r), (j * 16 + lane % 16) * 8, a.k);
    __builtin_amdgcn_sched_barrier(0);
    const int tiles = (a.n + 16 * CH - 1) / (16 * CH);
    i32x4 cw[kSteps][CH];
    const int by_c = a.y16 ? 4 : 16, by_group = a.y16 ? 4 * CH : 4;
    auto load_w = [&](int tile, int step) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int8_t *row = a.w + (long long)min(tile * 16 * CH + lane % 16 / 4 * by_group + c * by_c + lane % 4, a.n - 1) * a.ldw;
            __builtin_memcpy(&cw[step][c], (const FQ_GLOBAL int8_t *)(row + min(step * 64 + lane / 16 * 16, a.k - 16)), 16);      // (behind k the codes of x are 0)
        }
    };
    const int first = (int)blockIdx.y * WAVES + wave, stride = (int)gridDim.y * WAVES;
    if (first < tiles)
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
            if (j < steps) load_w(first, j);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int r = 0; r < kPasses; ++r) {
        if ((r * WAVES + wave) * 4 >= kRows) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) odd_end(raw[r][j], row_of_x(r), (j * 16 + lane % 16) * 8, a.k);
        const RowScale scale = row_scale(max16(most_of(raw[r])));
        if (lane % 16 == 0) scales[row_of(r)] = scale.s;
        u32x2 c[V];
#pragma unroll
        for (int j = 0; j < V; ++j) c[j] = codes8(raw[r][j], scale, (j * 16 + lane % 16) * 8 >= a.k);
        if (a.k % 16 != 0)
#pragma unroll
            for (int j = 0; j < V; ++j) c[j] = end_behind(c[j], (j * 16 + lane % 16) * 8, a.k);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int l = (j * 16 + lane % 16) * 8;
            if (l < steps * 64) *(u32x2 *)(codes + row_of(r) * pitch + l) = c[j];
        }
    }
    __syncthreads();

    const int8_t *x = codes + lane % 16 * pitch + lane / 16 * 16;
    for (int tile = first; tile < tiles; tile += stride) {
        i32x4 sum[CH][TOK];
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int t = 0; t < TOK; ++t) sum[c][t] = (i32x4)0;
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            if (j >= steps) continue;
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                const i32x4 cx = *(const i32x4 *)(x + t * 16 * pitch + j * 64);
#pragma unroll
                for (int c = 0; c < CH; ++c) sum[c][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(cw[j][c], cx, sum[c][t], 0, 0, 0);
            }
            if (tile + stride < tiles) load_w(tile + stride, j);
        }
        const int n = tile * 16 * CH + lane / 16 * by_group;
        float ws[CH * 4], bias[CH * 4];
#pragma unroll
        for (int e = 0; e < CH * 4; ++e) {
            const int j = min(n + e / 4 * by_c + e % 4, a.n - 1);
            ws[e] = ld_global(a.ws + (long long)j * a.ws_step);
            bias[e] = a.bias ? ld_global(a.bias + j) : 0.0f;
        }
        auto finish = [&](auto half, auto whole) {
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                const int m = m0 + t * 16 + lane % 16;
                const float xs = scales[t * 16 + lane % 16];
                char *const to = (char *)a.y + ((long long)m * a.ldy + n) * (half ? 2 : 4);
                if (m >= a.m) continue;
                float y[CH * 4];
#pragma unroll
                for (int e = 0; e < CH * 4; ++e) y[e] = (float)sum[e / 4][t][e % 4] * (xs * ws[e]);
                if (a.bias)
#pragma unroll
                    for (int e = 0; e < CH * 4; ++e) y[e] += bias[e];
                if constexpr (half) {
                    store_channels<true, whole, false, CH * 4>(to, y, a.n - n);
                } else {
#pragma unroll
                    for (int c = 0; c < CH; ++c) store_channels<false, whole, false, 4>(to + c * 64, y + c * 4, a.n - n - c * 16);
                }
            }
        };
        if ((tile + 1) * CH * 16 <= a.n) {
            if (a.y16) finish(std::true_type{}, std::true_type{});
            else finish(std::false_type{}, std::true_type{});
        } else {
            if (a.y16) finish(std::true_type{}, std::false_type{});
            else finish(std::false_type{}, std::false_type{});
        }
    }
}

template <typename X, int TOK, int CH> int launch_rows_of(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + TOK * 16 - 1) / (TOK * 16));
    const unsigned passes = (unsigned)(((long long)a.n + kRowsWaves * 16 * CH - 1) / (kRowsWaves * 16 * CH));
    const dim3 grid(blocks, blocks < kComputeUnits ? min(passes, kComputeUnits / blocks) : 1);
    if (a.k <= 256) linear_rows_kernel<X, TOK, CH, 2><<<grid, kRowsWaves * 64, 0, (hipStream_t)stream>>>(a);
    else if (a.k <= 384) linear_rows_kernel<X, TOK, CH, 3><<<grid, kRowsWaves * 64, 0, (hipStream_t)stream>>>(a);
    else linear_rows_kernel<X, TOK, CH, 4><<<grid, kRowsWaves * 64, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

template <int BM, int BN, int WM, int WN, int STAGES> int launch_tiles(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + BM - 1) / BM * (((long long)a.n + BN - 1) / BN));
    linear_tile_kernel<BM, BN, WM, WN, STAGES><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
}

}  // namespace

static unsigned align_blocks(const AlignArgs &a)
{
    return (unsigned)(((unsigned long long)a.rows * (unsigned long long)(a.pitch / 16) + 255) / 256);
}

int launch_align_rows(const AlignArgs &a, const AlignArgs &other, void *stream)
{
    const unsigned blocks = align_blocks(a);
    align_rows_kernel<<<blocks + align_blocks(other), 256, 0, (hipStream_t)stream>>>(a, blocks, other);
    return (int)hipGetLastError();
}

template <typename T, int L, int V> static int quantize_rows_by(const QuantizeArgs &a, const AlignArgs &other, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + 256 / L - 1) / (256 / L));
    quantize_rows_kernel<T, L, V><<<blocks + align_blocks(other), 256, 0, (hipStream_t)stream>>>(a, blocks, other);
    return (int)hipGetLastError();
}

template <typename T> static int quantize_rows(const QuantizeArgs &a, const AlignArgs &other, void *stream)
{
    if (a.k <= 128) return quantize_rows_by<T, 16, 1>(a, other, stream);
    if (a.k <= 256) return quantize_rows_by<T, 16, 2>(a, other, stream);
    if (a.k <= 384) return quantize_rows_by<T, 16, 3>(a, other, stream);
    if (a.k <= 512) return quantize_rows_by<T, 16, 4>(a, other, stream);
    if (a.k <= 2048) return quantize_rows_by<T, 64, 4>(a, other, stream);
    return quantize_rows_by<T, 256, 4>(a, other, stream);
}

int launch_quantize_rows(const QuantizeArgs &a, const AlignArgs &other, void *stream)
{
    return a.x16 ? quantize_rows<_Float16>(a, other, stream) : quantize_rows<float>(a, other, stream);
}

// The tiles, and what a step of 128 codes of a block takes: at least `wait`, and `work` for each block that a compute unit
// holds at once (`resident` of them at most); in us.  What is in front of the first step and behind the last takes kEnds and the time of the
// blocks' parts of y at 5 TB/s (with few steps the most of it: 11707 x 9600 x 272 89 us in 256 x 256, 45 of them for y).  The tile
// with the least sum is taken.  (Sums are up to 1.5 times off, either way: 600 x 4096 x 4096 in 256 x 256 60 for 41, 20 x 16384 x 4096 in 32 x 64 7.8
// for 12.5.  The tiles chosen below are the best or within 2 % of it.)  Measured, codes at aligned rows, us, the tiles in the order of the table (- : not in question):
//   8192 x 8192 x 8192   461   483   565   582   856   1091
//   2048 x 4096 x 4096  44.5  34.0  37.0  38.3  55.0   73.9
//   19200 x 384 x 384   12.3   8.8   8.6  11.1  14.4   16.9
//   600 x 4096 x 4096   41.2  23.1  27.0  17.0  21.6   26.9
//   256 x 4096 x 4096      -     -     -  15.7  10.3   12.1
//   446 x 503 x 6144       -     -     -  22.7  12.3   11.3
//   20 x 16384 x 4096   40.3  22.2  26.2  15.0  12.8   12.5
//   12814 x 166 x 1040, FP32 y  23.3  15.6  13.8  11.7  -  14.7
struct Tile {
    int m, n, resident;
    double wait, work;
    int (*launch)(const LinearArgs &, void *);
};

constexpr double kEnds = 1.5, kStoreRate = 5e6;                  // us, bytes a us

static const Tile kTiles[] = {
    {256, 256, 1, 1.80, 1.80, launch_tiles<256, 256, 2, 4, 2>},
    {256, 128, 1, 0.70, 0.98, launch_tiles<256, 128, 4, 2, 3>},
    {128, 128, 2, 0.80, 0.56, launch_tiles<128, 128, 2, 2, 2>},
    {128, 128, 1, 0.46, 0.56, launch_tiles<128, 128, 2, 2, 4>},
    {64, 64, 2, 0.19, 0.21, launch_tiles<64, 64, 2, 2, 4>},
    {32, 64, 3, 0.19, 0.12, launch_tiles<32, 64, 1, 2, 4>},
};

static double tile_time(const LinearArgs &a, const Tile &t)
{
    const long long blocks = ((long long)a.m + t.m - 1) / t.m * (((long long)a.n + t.n - 1) / t.n);
    const long long once = (long long)kComputeUnits * t.resident, rounds = blocks / once, left = blocks % once;
    const double steps = (double)((a.k + kDepth - 1) / kDepth), store = (double)t.m * t.n * (a.y16 ? 2 : 4) / kStoreRate;
    double time = (double)rounds * (steps * (t.wait > t.resident * t.work ? t.wait : t.resident * t.work) + kEnds + (double)once * store);
    if (left) {
        const double each = (double)((left + kComputeUnits - 1) / kComputeUnits) * t.work;
        time += steps * (t.wait > each ? t.wait : each) + kEnds + (double)left * store;
    }
    return time;
}

// Whether the kernel of few tokens takes x of this element size: values fit into LDS beside the rings (codes need not), and all
// blocks are on the chip at once, or there are at most 16 tokens and w does not fit the tiles.  us, this / quantizing and tiles: 1 x 4096 x 4096 FP16 5.4 / 10.7, 16 x 4096 x 4096 8.9 / 11.0, 4 x 4096 x 8192
// 10.5 / 16.2; two blocks to a compute unit: 1 x 8192 x 4096 8.4 / 11.0, 1 x 8192 x 64 4.6 / 7.6, codes 3 x 8192 x 2048 4.8 / 6.2; codes
// through the rings, x quantized by a launch of its own in both: 16 x 4096 x 14336 15.8 / 25.5, 32 x 4096 x 4096 8.3 / 11.3, 128 x 1024 x 2352
// 6.9 / 9.7, 1000 x 128 x 4096 11.4 / 13.2, codes 224 x 503 x 6144 5.9 / 11.1, 33 x 16 x 16 4.4 / 4.4; not at once: 4 x 8192 x 4096 15.1 / 11.2, 1201
// x 257 x 1155 14.0 / 10.2, codes 16 x 16384 x 4096 20.7 / 12.4, 446 x 503 x 6144 10.4 / 11.3.
bool linear_few(const LinearArgs &a, int size)
{
    if (a.k <= 0 || a.ldw > kMostPitch || (size == 1 && !a.x_fits && a.ldx > kMostPitch)) return false;
    if (a.m > 16) return size == 1 && ((long long)a.m + 31) / 32 * (((long long)a.n + 15) / 16) <= kComputeUnits;
    const long long lds = few_most(a, size);
    return (lds <= kFewLds || size == 1) && (!a.w_fits || a.n <= (lds <= kFewLdsOfTwo ? 2 : 1) * kFewMostN);
}

// Work that a launch and a trip of the codes to memory would be much of, and x with few channels.  us, codes by a kernel of their own and
// tiles / this: 348 x 37 x 16 5.8 / 3.5, 1000 x 1000 x 128 7.3 / 4.5, 100 x 8000 x 320 7.4 / 5.4, 1024 x 512 x 512 7.7 / 6.5; 2048 x 256 x 256 7.1 / 6.1,
// 19200 x 128 x 384 14.5 / 10.6, 288000 x 128 x 128 58.5 / 50.0; not: 900 x 1100 x 512 FP32 8.5 / 10.9, 12032 x 2277 x 64 26.2 / 30.8, 2000 x 2000 x 384
// 11.3 / 12.2.
bool linear_rows(const LinearArgs &a)
{
    if (a.k < kRowsLeastK || a.k > kRowsMostK) return false;
    return (a.m >= 1024 && (long long)a.n * a.k <= (1 << 16)) || ((double)a.m * a.n * a.k <= 0x1p28 && linear_rows_as_they_lie(a));
}

// Loads of 16 bytes that begin between words take twice the time, which is nothing for few.  us, w laid out and tiles (the last:
// this kernel) / as it lies: 500 x 1000 x 63 7.6 / 5.1, 200 x 1000 x 127 7.4 / 6.4, 400 x 300 x 255 7.5 / 7.5, 200 x 300 x 511 8.5 / 12.7, 900 x 1100
// x 127 7.9 / 8.3, 100000 x 64 x 255 29.2 / 33.4.
bool linear_rows_as_they_lie(const LinearArgs &a)
{
    return ((uintptr_t)a.w | (uintptr_t)a.ldw) % 4 == 0 || (a.k <= 256 && (double)a.m * a.n * a.k <= 0x1p26);
}

template <typename X, int TOK> static int launch_rows_by(const LinearArgs &a, void *stream)
{
    const long long pairs = ((long long)a.m + TOK * 16 - 1) / (TOK * 16) * (((long long)a.n + 32 * kRowsWaves - 1) / (32 * kRowsWaves));
    return a.n <= 16 * kRowsWaves || pairs < kComputeUnits ? launch_rows_of<X, TOK, 1>(a, stream) : launch_rows_of<X, TOK, 2>(a, stream);
}

// 32 tokens to a block while they are that few that longer blocks leave compute units without one, else 80.
template <typename X> static int launch_rows(const LinearArgs &a, void *stream)
{
    return a.m <= 32 * kComputeUnits ? launch_rows_by<X, 2>(a, stream) : launch_rows_by<X, 5>(a, stream);
}

int launch_linear(const LinearArgs &a, void *stream)
{
    // (x given as raw for its short rows goes there also with 16 tokens or fewer: offsets into rows of w beyond kMostPitch need 64 bits, and
    // blocks that are not all on the chip at once cost.  us, few tokens / short rows: 16 x 16384 x 512 17.4 / 6.0, 1 x 16384 x 64 6.5 / 4.1,
    // 1 x 16384 x 512 6.6 / 5.7, 1 x 8208 x 512 5.2 / 5.4.)
    if (a.raw && linear_few(a, a.x16 ? 2 : 4)) return a.x16 ? launch_few<_Float16>(a, stream) : launch_few<float>(a, stream);
    if (a.raw) return a.x16 ? launch_rows<_Float16>(a, stream) : launch_rows<float>(a, stream);
    if (linear_few(a, 1)) return launch_few<int8_t>(a, stream);
    int best = 0;
    double least = 0.0;
    for (int i = 0; i < (int)(sizeof kTiles / sizeof kTiles[0]); ++i) {
        const double t = tile_time(a, kTiles[i]);
        if (least == 0.0 || t < least) { least = t; best = i; }
    }
    return kTiles[best].launch(a, stream);
}

}  // namespace fq
