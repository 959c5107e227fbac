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
        typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
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
    typedef float f32x4 __attribute__((ext_vector_type(4)));
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

template <int BM, int BN, int WM, int WN> int launch_tiles(const LinearArgs &a, void *stream)
{
    const unsigned blocks = (unsigned)(((long long)a.m + BM - 1) / BM * (((long long)a.n + BN - 1) / BN));
    if (a.aligned) linear_tile_kernel<BM, BN, WM, WN, true><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    else linear_tile_kernel<BM, BN, WM, WN, false><<<blocks, WM * WN * 64, 0, (hipStream_t)stream>>>(a);
    return (int)hipGetLastError();
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
    const long long large = ((long long)a.m + 255) / 256 * (((long long)a.n + 255) / 256);
    if (large >= kComputeUnits) return launch_tiles<256, 256, 2, 4>(a, stream);
    const long long medium = ((long long)a.m + 127) / 128 * (((long long)a.n + 127) / 128);
    if (medium >= kComputeUnits / 2) return launch_tiles<128, 128, 2, 2>(a, stream);
    return launch_tiles<64, 64, 2, 2>(a, stream);
}

}  // namespace fq
