// Low-rank adapters of many requests beside a shared layer (declared in include/fq.h).
//
//   t = x a^T,   y = base + (xs scale) t b^T      a, b: those of the token's adapter
//
// Two steps, since all of t is needed for any y: adapter_down_kernel makes t, in parts of k where there are few tiles, and
// adapter_up_kernel adds them up and makes y.  Both work on tiles of up to 16 (64) tokens of one adapter, whose rows they pick out
// by a list: with up to 64 tokens a wavefront finds those of one adapter by itself; with more, adapter_group_kernel orders them first.
// Products go to the matrix cores.  Bound by memory (x, base and y once each: few operations to a byte, 2 rank of them) and, for few tokens,
// by the launches.
#include <type_traits>

#include "fq_adapters.h"
#include "fq_rows.h"

namespace fq {
namespace {

using namespace dev;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bool has_adapter(int id, int count) { return id >= 0 && id < count; }

// ---------------------------------------------------------------------------------------------
// Tokens in the order of their adapters (those without one behind all others), and the tiles of up to `tile` of each.  One block:
// ids are read twice.  Places of one adapter's tokens are handed out by an atomic counter, so which tile a token is in may differ from
// run to run; what is worked out for it does not depend on that.
constexpr int kGroupThreads = 1024;

__global__ __launch_bounds__(kGroupThreads) void adapter_group_kernel(AdapterArgs a)
{
    extern __shared__ int counts[];              // [count + 1]: of tokens, then the next free place
    __shared__ int sums[2][kGroupThreads / 64];
    const int groups = a.count + 1, thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    const int tile = 16 * a.token_tiles;
    for (int i = thread; i < groups; i += kGroupThreads) counts[i] = 0;
    __syncthreads();
    // (tokens of one request come one after the other: then all lanes of a wavefront count for the same adapter)
    const auto group_of = [&](int i) {
        const int id = ld_global(a.ids + i);
        return has_adapter(id, a.count) ? id : a.count;
    };
    for (int i = thread; i < a.m; i += kGroupThreads) {
        const int g = group_of(i), leader = __builtin_amdgcn_readfirstlane(g);
        const unsigned long long same = __ballot(g == leader), all = __ballot(1);
        if (same == all) {
            if (lane == __builtin_ctzll(all)) atomicAdd(counts + leader, __popcll(all));
        } else {
            atomicAdd(counts + g, 1);
        }
    }
    __syncthreads();
    // first places and first tiles of the groups: each thread has a run of them
    const int each = (groups + kGroupThreads - 1) / kGroupThreads, from = min(thread * each, groups), to = min(from + each, groups);
    int tokens = 0, tiles = 0;
    for (int g = from; g < to; ++g) {
        tokens += counts[g];
        tiles += (counts[g] + tile - 1) / tile;
    }
    int token_at = tokens, tile_at = tiles;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const int p = __shfl_up(token_at, step), q = __shfl_up(tile_at, step);
        if (lane >= step) {
            token_at += p;
            tile_at += q;
        }
    }
    if (lane == 63) {
        sums[0][wave] = token_at;
        sums[1][wave] = tile_at;
    }
    __syncthreads();
    token_at -= tokens;
    tile_at -= tiles;
    int all_tiles = 0;
    for (int w = 0; w < kGroupThreads / 64; ++w) {
        if (w < wave) {
            token_at += sums[0][w];
            tile_at += sums[1][w];
        }
        all_tiles += sums[1][w];
    }
    for (int g = from; g < to; ++g) {
        const int count = counts[g];
        for (int i = 0; i < count; i += tile) {
            const AdapterTile t = {g < a.count ? g : -1, token_at + i, min(tile, count - i)};
            a.tiles[tile_at++] = t;
        }
        counts[g] = token_at;
        token_at += count;
    }
    for (int i = all_tiles + thread; i < a.tiles_most; i += kGroupThreads) a.tiles[i] = AdapterTile{-1, 0, 0};
    __syncthreads();
    for (int i = thread; i < a.m; i += kGroupThreads) {
        const int g = group_of(i), leader = __builtin_amdgcn_readfirstlane(g);
        const unsigned long long same = __ballot(g == leader), all = __ballot(1);
        int place;
        if (same == all) {
            int base = 0;
            if (lane == __builtin_ctzll(all)) base = atomicAdd(counts + leader, __popcll(all));
            place = __shfl(base, __builtin_ctzll(all)) + __popcll(all & ((1ull << lane) - 1));
        } else {
            place = atomicAdd(counts + g, 1);
        }
        a.order[place] = i;
    }
}

// ---------------------------------------------------------------------------------------------
// The tile of a block: its adapter, its tokens (up to kWindow, in `tokens`) and where its rows of t begin; t's rows are in the order of the
// tokens' places.  `window`: the tokens that have the adapter of token `index` of theirs, if that is the first to have it (so every
// adapter of the window has one block).
struct Tile {
    int id, first, count;
};

__device__ __forceinline__ Tile find_tile(const AdapterArgs &a, int index, int *tokens)
{
    const int lane = threadIdx.x & 63;
    Tile t;
    if (a.grouped) {
        const AdapterTile f = a.tiles[index];
        t = {f.id, f.first, f.count};
        if (threadIdx.x < (unsigned)t.count) tokens[threadIdx.x] = ld_global(a.order + t.first + threadIdx.x);
    } else {
        const int slots = min(a.m, kWindow), begin = index / slots * kWindow, slot = index % slots;
        const int token = begin + lane, left = min(a.m - begin, kWindow);
        int id = lane < left ? ld_global(a.ids + token) : -2;
        if (lane < left && !has_adapter(id, a.count)) id = -1;
        t.id = __builtin_amdgcn_readlane(id, slot);
        const unsigned long long mine = __ballot(id == t.id);
        t.first = begin;
        t.count = slot < left && __builtin_ctzll(mine) == slot ? __popcll(mine) : 0;
        if (threadIdx.x < 64 && (mine >> lane & 1)) tokens[__popcll(mine & ((1ull << lane) - 1))] = token;
    }
    __syncthreads();
    return t;
}

// The row of t of token i of the tile.
__device__ __forceinline__ int row_of(const AdapterArgs &a, const Tile &t, const int *tokens, int i)
{
    return a.grouped ? t.first + i : tokens[i];
}

// Eight values of a row from `at` on, zeros behind its end.
template <typename T> __device__ __forceinline__ Eight<T> row8(const T *row, int at, int k, bool whole)
{
    Eight<T> r;
    if (whole || at + 8 <= k) {
        __builtin_memcpy(&r, (const FQ_GLOBAL T *)(row + at), sizeof r);
        return r;
    }
    typename Values<T>::type v = (typename Values<T>::type)(T)0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (at + e < k) v[e] = ld_global(row + at + e);
    return __builtin_bit_cast(Eight<T>, v);
}

struct Codes16 { i32x4 w; };

__device__ __forceinline__ Codes16 codes16(const int8_t *row, int at, int k, bool whole)
{
    Codes16 r;
    if (whole || at + 16 <= k) {
        __builtin_memcpy(&r, (const FQ_GLOBAL int8_t *)(row + at), sizeof r);
        return r;
    }
    r.w = (i32x4)0;
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (at + e < k) r.w[e / 4] |= (int)((unsigned)(unsigned char)ld_global(row + at + e) << (8 * (e % 4)));
    return r;
}

// Eight codes as FP16: 1024 + (code + 128) has the code's byte, its top bit turned, as its lower byte.
__device__ __forceinline__ f16x8 halves_of(int low, int high)
{
    f16x8 v;
    const unsigned bytes[2] = {(unsigned)low ^ 0x80808080u, (unsigned)high ^ 0x80808080u};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned pair = __builtin_amdgcn_perm(0x64646464u, bytes[i / 2], i % 2 ? 0x04030402u : 0x04010400u);
        const f16x2 h = __builtin_bit_cast(f16x2, pair) - (f16x2)(_Float16)1152.0f;
        v[2 * i] = h[0];
        v[2 * i + 1] = h[1];
    }
    return v;
}

// 64 values of k of a wavefront's rows: a lane has 16 neighbouring ones of a token, and of a rank.
template <typename X> struct Piece;
template <> struct Piece<_Float16> {
    Eight<_Float16> w[2];
    __device__ __forceinline__ void fetch(const _Float16 *row, int at, int k, bool whole)
    {
        w[0] = row8(row, at, k, whole);
        w[1] = row8(row, at + 8, k, whole);
    }
    __device__ __forceinline__ f16x8 half(int i) const { return __builtin_bit_cast(f16x8, w[i]); }
};
template <> struct Piece<int8_t> {
    Codes16 c;
    __device__ __forceinline__ void fetch(const int8_t *row, int at, int k, bool whole) { c = codes16(row, at, k, whole); }
    __device__ __forceinline__ f16x8 half(int i) const { return halves_of(c.w[2 * i], c.w[2 * i + 1]); }
};
template <> struct Piece<float> {
    Eight<float> w[2];
    __device__ __forceinline__ void fetch(const float *row, int at, int k, bool whole)
    {
        w[0] = row8(row, at, k, whole);
        w[1] = row8(row, at + 8, k, whole);
    }
    __device__ __forceinline__ float value(int i) const { return __builtin_bit_cast(Values<float>::type, w[i / 8])[i % 8]; }
};

// t of a tile: NT x 16 tokens by NR x 16 ranks.  The wavefronts of a block take 64 values of k in turn; their sums meet in LDS.  Loads go
// straight into the registers that the matrix instructions take (lane l: token l % 16, and rank l % 16, values 16 (l / 16) and on of the
// 64), those of the next 64 while these are multiplied.
constexpr int kDownWaves = 4, kDepth = 64;

template <typename X, int NT, int NR> __global__ __launch_bounds__(64 * kDownWaves) void adapter_down_kernel(AdapterArgs a)
{
    __shared__ f32x4 part[kDownWaves][NT * NR][64];
    __shared__ int tokens[kWindow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int split = blockIdx.x % a.splits, chunk = blockIdx.x / a.splits % a.chunks;
    const Tile tile = find_tile(a, blockIdx.x / a.splits / a.chunks, tokens);
    if (tile.id < 0 || tile.count == 0) return;
    const int steps = (a.k + kDepth - 1) / kDepth;
    const int begin = (int)((long long)steps * split / a.splits), end = (int)((long long)steps * (split + 1) / a.splits);
    const _Float16 *ranks[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r)
        ranks[r] = (const _Float16 *)a.a + ((long long)tile.id * a.rank + min(chunk * 64 + r * 16 + lane % 16, a.rank - 1)) * a.k;
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        const X *rows[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) rows[n] = (const X *)a.x + tokens[min(sub + n * 16 + lane % 16, tile.count - 1)] * a.ldx;
        f32x4 sum[NT][NR];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) sum[n][r] = (f32x4)0.0f;
        Piece<X> x[2][NT];
        Piece<_Float16> w[2][NR];
        const auto fetch = [&](int buffer, int step) {
            const int at = step * kDepth + lane / 16 * 16;
            const bool whole = (step + 1) * kDepth <= a.k;
#pragma unroll
            for (int n = 0; n < NT; ++n) x[buffer][n].fetch(rows[n], at, a.k, whole);
#pragma unroll
            for (int r = 0; r < NR; ++r) w[buffer][r].fetch(ranks[r], at, a.k, whole);
        };
        const auto multiply = [&](int buffer) {
            if constexpr (std::is_same<X, float>::value) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        const float v = (float)w[buffer][r].half(e / 8)[e % 8];
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            sum[n][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[buffer][n].value(e), sum[n][r], 0, 0, 0);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    f16x8 v[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) v[n] = x[buffer][n].half(i);
#pragma unroll
                    for (int r = 0; r < NR; ++r)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            sum[n][r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[buffer][r].half(i), v[n], sum[n][r], 0, 0, 0);
                }
            }
        };
        int step = begin + wave;
        if (step < end) fetch(0, step);
        while (step < end) {
            if (step + kDownWaves < end) fetch(1, step + kDownWaves);
            multiply(0);
            step += kDownWaves;
            if (step >= end) break;
            if (step + kDownWaves < end) fetch(0, step + kDownWaves);
            multiply(1);
            step += kDownWaves;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) part[wave][n * NR + r][lane] = sum[n][r];
        __syncthreads();
        // lane l's four sums: token l % 16, ranks 4 (l / 16) and on
        for (int i = threadIdx.x; i < NT * NR * 64; i += 64 * kDownWaves) {
            const int n = i / 64 / NR, r = i / 64 % NR, l = i % 64;
            const int token = sub + n * 16 + l % 16, rank = chunk * 64 + r * 16 + l / 16 * 4;
            f32x4 s = part[0][n * NR + r][l];
#pragma unroll
            for (int v = 1; v < kDownWaves; ++v) s += part[v][n * NR + r][l];
            if (token < tile.count && rank < a.pitch)
                st_global((f32x4 *)(a.t + ((long long)split * a.m + row_of(a, tile, tokens, token)) * a.pitch + rank), s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// y of a tile of NT x 16 tokens, in strips of CT x 16 channels to each of four wavefronts.  First the block adds up t (of all its
// parts) and puts it into LDS as two FP16 numbers to a value: t 2^-e to 11 bits and the rest to 11 more, 2^e the power of two that
// brings the row's greatest into [2^14, 2^15), so that nothing overflows and 22 bits of each are kept, or 2^-39 of the greatest.  (FP16
// products cost a quarter of the matrix cores' time that binary32 ones take.)  Then a wavefront has channels for the rows of its products and
// tokens for the columns: lane l has 4 CT neighbouring channels of token l % 16, whole lines of y from four lanes.
constexpr int kUpWaves = 4;

__device__ __forceinline__ f32x4 product(f16x8 b, f16x8 t, f32x4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(b, t, sum, 0, 0, 0); }

template <typename T, int N> __device__ __forceinline__ void load_channels(float *to, const T *at, int left)
{
    typedef T V __attribute__((ext_vector_type(N)));
    if (left >= N) {
        V v;
        __builtin_memcpy(&v, (const FQ_GLOBAL T *)at, sizeof(T) * N);
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = (float)v[e];
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) to[e] = e < left ? (float)ld_global(at + e) : 0.0f;
}

template <typename T, int N> __device__ __forceinline__ void store_channels(T *at, const float *y, int left)
{
    typedef T V __attribute__((ext_vector_type(N)));
    if (left >= N) {
        V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = (T)y[e];
        __builtin_memcpy((FQ_GLOBAL T *)at, &v, sizeof(T) * N);
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (e < left) st_global(at + e, (T)y[e]);
}

template <typename Y, typename B, int NT, int CT> __global__ __launch_bounds__(64 * kUpWaves) void adapter_up_kernel(AdapterArgs a)
{
    extern __shared__ __attribute__((aligned(16))) _Float16 shared[];          // [2][NT * 16][row]
    __shared__ int tokens[kWindow];
    __shared__ float factor[NT * 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Tile tile = find_tile(a, blockIdx.x / a.groups, tokens);
    const int deep = (a.rank + 31) / 32, row = deep * 32 + 8;
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        if (tile.id >= 0) {
            // four lanes to a token
            for (int i = threadIdx.x / 4; i < NT * 16; i += 16 * kUpWaves) {
                const int token = min(sub + i, tile.count - 1), part = threadIdx.x % 4;
                const float *t = a.t + (long long)row_of(a, tile, tokens, token) * a.pitch;
                float most = 0.0f;
                f32x4 held[8];                   // (ranks up to 128; of more, the rest is added up again)
                const auto ask = [&](int l) {
                    f32x4 s = (f32x4)0.0f;
                    if (l < a.pitch) {
                        s = ld_global((const f32x4 *)(t + l));
                        for (int p = 1; p < a.splits; ++p) s += ld_global((const f32x4 *)(t + (long long)p * a.m * a.pitch + l));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (l + e >= a.rank) s[e] = 0.0f;
                    return s;
                };
                const auto greatest = [&](f32x4 s) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(s[e]));
                };
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < deep * 2) greatest(held[j] = ask(j * 16 + part * 4));
                for (int j = 8; j < deep * 2; ++j) greatest(ask(j * 16 + part * 4));
                most = __builtin_fmaxf(most, __shfl_xor(most, 1));
                most = __builtin_fmaxf(most, __shfl_xor(most, 2));
                const int e2 = most > 0.0f && most < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(most) : 0;
                const auto put = [&](int j, f32x4 s) {
                    f16x4 high, low;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = __builtin_ldexpf(s[e], e2);
                        high[e] = (_Float16)v;
                        const float rest = v - (float)high[e];
                        low[e] = (_Float16)(__builtin_fabsf(rest) < __builtin_inff() ? rest : 0.0f);
                    }
                    *(f16x4 *)(shared + i * row + j * 16 + part * 4) = high;
                    *(f16x4 *)(shared + (NT * 16 + i) * row + j * 16 + part * 4) = low;
                };
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < deep * 2) put(j, held[j]);
                for (int j = 8; j < deep * 2; ++j) put(j, ask(j * 16 + part * 4));
                if (part == 0) {
                    const int at = tokens[token];
                    const float s = (a.scale ? ld_global(a.scale + tile.id) : 1.0f) * (a.xs ? ld_global(a.xs + (long long)at * a.xs_step) : 1.0f);
                    factor[i] = __builtin_ldexpf(s, -e2);
                }
            }
        }
        __syncthreads();
        const bool copy = tile.id < 0;
        if (!(copy && a.base == a.y)) {
            for (int strip = (int)(blockIdx.x % a.groups) * kUpWaves + wave; strip * CT * 16 < a.n; strip += a.groups * kUpWaves) {
                const int mine = strip * CT * 16 + lane / 16 * CT * 4;         // the lane's first channel
                float y[NT][CT * 4];
                f32x4 sum[NT][CT];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int token = sub + n * 16 + lane % 16;
                    if (a.base && token < tile.count)
                        load_channels<B, CT * 4>(y[n], (const B *)a.base + tokens[token] * a.ldbase + mine, a.n - mine);
                    else
#pragma unroll
                        for (int e = 0; e < CT * 4; ++e) y[n][e] = 0.0f;
#pragma unroll
                    for (int c = 0; c < CT; ++c) sum[n][c] = (f32x4)0.0f;
                }
                if (!copy) {
                    for (int d = 0; d < deep; ++d) {
                        f16x8 b[CT];
#pragma unroll
                        for (int c = 0; c < CT; ++c) {
                            // row i of the product's 16: channel (i / 4) 4 CT + 4 c + i % 4 of the strip
                            const int channel = min(strip * CT * 16 + lane % 16 / 4 * CT * 4 + c * 4 + lane % 4, a.n - 1);
                            const _Float16 *from = (const _Float16 *)a.b + ((long long)tile.id * a.n + channel) * a.rank;
                            b[c] = __builtin_bit_cast(f16x8, row8(from, d * 32 + lane / 16 * 8, a.rank, false));
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const _Float16 *at = shared + (n * 16 + lane % 16) * row + d * 32 + lane / 16 * 8;
                            const f16x8 high = *(const f16x8 *)at, low = *(const f16x8 *)(at + NT * 16 * row);
#pragma unroll
                            for (int c = 0; c < CT; ++c) sum[n][c] = product(b[c], low, product(b[c], high, sum[n][c]));
                        }
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const int token = sub + n * 16 + lane % 16;
                    if (token >= tile.count) continue;
                    if (!copy) {
                        const float f = factor[n * 16 + lane % 16];
#pragma unroll
                        for (int e = 0; e < CT * 4; ++e) y[n][e] += f * sum[n][e / 4][e % 4];
                    }
                    store_channels<Y, CT * 4>((Y *)a.y + tokens[token] * a.ldy + mine, y[n], a.n - mine);
                }
            }
        }
        __syncthreads();
    }
}

template <typename X, int NT> void down_by(const AdapterArgs &a, unsigned blocks, hipStream_t stream)
{
    if (a.rank <= 16) adapter_down_kernel<X, NT, 1><<<blocks, 64 * kDownWaves, 0, stream>>>(a);
    else if (a.rank <= 32) adapter_down_kernel<X, NT, 2><<<blocks, 64 * kDownWaves, 0, stream>>>(a);
    else adapter_down_kernel<X, NT, 4><<<blocks, 64 * kDownWaves, 0, stream>>>(a);
}

template <typename X> void down(const AdapterArgs &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)a.tiles_most * (unsigned)a.splits * (unsigned)a.chunks;
    if (a.token_tiles == 1) down_by<X, 1>(a, blocks, stream);
    else down_by<X, 4>(a, blocks, stream);
}

template <typename Y, typename B> void up(const AdapterArgs &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)a.tiles_most * (unsigned)a.groups;
    const size_t lds = a.count > 0 ? (size_t)2 * 16 * a.token_tiles * ((a.rank + 31) / 32 * 32 + 8) * sizeof(_Float16) : 0;
    if (a.token_tiles == 4) adapter_up_kernel<Y, B, 4, 4><<<blocks, 64 * kUpWaves, lds, stream>>>(a);
    else if (a.wide == 4) adapter_up_kernel<Y, B, 1, 4><<<blocks, 64 * kUpWaves, lds, stream>>>(a);
    else adapter_up_kernel<Y, B, 1, 1><<<blocks, 64 * kUpWaves, lds, stream>>>(a);
}

}  // namespace

int launch_adapters(const AdapterArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.count > 0) {
        if (a.grouped) adapter_group_kernel<<<1, kGroupThreads, (size_t)(a.count + 1) * sizeof(int), s>>>(a);
        if (a.x_type == 0) down<_Float16>(a, s);
        else if (a.x_type == 1) down<float>(a, s);
        else down<int8_t>(a, s);
        const int err = (int)hipGetLastError();
        if (err != 0) return err;
    }
    if (a.y16) {
        if (a.base16) up<_Float16, _Float16>(a, s);
        else up<_Float16, float>(a, s);
    } else {
        if (a.base16) up<float, _Float16>(a, s);
        else up<float, float>(a, s);
    }
    return (int)hipGetLastError();
}

}  // namespace fq
