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
constexpr int kGroupThreads = 1024, kHeldIds = 8;

__device__ __forceinline__ int group_of(const AdapterArgs &a, int token)
{
    const int id = token < a.m ? ld_global(a.ids + token) : -1;
    return has_adapter(id, a.count) ? id : a.count;
}

// Counts the lanes with `some` for their groups; the number that were counted there before a lane's.  (Tokens of one request come one
// after the other: then the wavefront counts for one adapter, once.)
__device__ __forceinline__ int count_in(int *counts, int group, bool some, int lane)
{
    const unsigned long long all = __ballot(some);
    if (all == 0) return 0;
    const int first = __builtin_ctzll(all), leader = __builtin_amdgcn_readlane(group, first);
    if (__ballot(some && group == leader) == all) {
        int before = 0;
        if (lane == first) before = atomicAdd(counts + leader, __popcll(all));
        return __builtin_amdgcn_readlane(before, first) + __popcll(all & ((1ull << lane) - 1));
    }
    return some ? atomicAdd(counts + group, 1) : 0;
}

// Sums of both values over the threads of a block before this one, and of all (in `total`, of the second).
template <int WAVES> __device__ __forceinline__ void sums_before(int &a, int &b, int &total, int (&sums)[2][WAVES], int lane, int wave)
{
    int x = a, y = b;
#pragma unroll
    for (int step = 1; step < 64; step *= 2) {
        const int p = __shfl_up(x, step), q = __shfl_up(y, step);
        if (lane >= step) {
            x += p;
            y += q;
        }
    }
    if (lane == 63) {
        sums[0][wave] = x;
        sums[1][wave] = y;
    }
    __syncthreads();
    a = x - a;
    b = y - b;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        a += w < wave ? sums[0][w] : 0;
        b += w < wave ? sums[1][w] : 0;
        total += sums[1][w];
    }
}

__global__ __launch_bounds__(kGroupThreads) void adapter_group_kernel(AdapterArgs a)
{
    extern __shared__ int counts[];              // [count + 1]: of tokens, then the next free place
    __shared__ int sums[2][kGroupThreads / 64];
    const int groups = a.count + 1, thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    const int tile = 16 * a.token_tiles;
    constexpr int kRun = kGroupThreads * kHeldIds;
    int held[kHeldIds];
    const auto ask = [&](int from) {
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) held[j] = group_of(a, from + j * kGroupThreads + thread);
    };
    ask(0);
    for (int i = thread; i < groups; i += kGroupThreads) counts[i] = 0;
    __syncthreads();
    for (int from = 0; from < a.m; from += kRun) {
        if (from > 0) ask(from);
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) count_in(counts, held[j], from + j * kGroupThreads + thread < a.m, lane);
    }
    __syncthreads();
    // first places and first tiles of the groups: each thread has a run of them
    const int each = (groups + kGroupThreads - 1) / kGroupThreads, begin = min(thread * each, groups), end = min(begin + each, groups);
    int token_at = 0, tile_at = 0, all_tiles;
    for (int g = begin; g < end; ++g) {
        token_at += counts[g];
        tile_at += (counts[g] + tile - 1) / tile;
    }
    sums_before(token_at, tile_at, all_tiles, sums, lane, wave);
    for (int g = begin; g < end; ++g) {
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
    for (int from = 0; from < a.m; from += kRun) {
        if (a.m > kRun) ask(from);
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) {
            const int token = from + j * kGroupThreads + thread;
            const int place = count_in(counts, held[j], token < a.m, lane);
            if (token < a.m) a.order[place] = token;
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The tile of a block: its adapter (-1: none) and its tokens, which go to `tokens`.  Three ways:
//   windows   up to kWindow tokens (or windows of so many): those that have the adapter of token `slot` of theirs, if that is the first to have
//             it; so every adapter of the window has one block, which takes them by tiles one after the other
//   sorting   up to kSorted tokens and adapters: the block counts the tokens of each adapter by itself, which costs less than a launch in
//             front and the two trips to memory for its results
//   list      tile and tokens are what adapter_group_kernel has written
struct Tile {
    int id, count;
};

struct Finding {
    int tokens[kWindow];
    int counts[kSorted + 1];
    int sums[2][kBlock / 64], parts[kSorted / 64];
    Tile tile;
    int first;
};

__device__ __forceinline__ Tile find_tile(const AdapterArgs &a, int index, Finding &s)
{
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    Tile t = {-1, 0};
    if (a.way == kWindows) {
        const int slots = min(a.m, kWindow), begin = index / slots * kWindow, slot = index % slots;
        const int left = min(a.m - begin, kWindow);
        int id = lane < left ? ld_global(a.ids + begin + lane) : -2;
        if (lane < left && !has_adapter(id, a.count)) id = -1;
        t.id = __builtin_amdgcn_readlane(id, slot);
        const unsigned long long mine = __ballot(id == t.id);
        t.count = slot < left && __builtin_ctzll(mine) == slot ? __popcll(mine) : 0;
        if (thread < 64 && (mine >> lane & 1)) s.tokens[__popcll(mine & ((1ull << lane) - 1))] = begin + lane;
    } else if (a.way == kSorting) {
        constexpr int kIds = kSorted / kBlock;
        const int groups = a.count + 1, tile = 16 * a.token_tiles;
        int id[kIds];
#pragma unroll
        for (int j = 0; j < kIds; ++j) id[j] = group_of(a, j * kBlock + thread);
        for (int i = thread; i < groups; i += kBlock) s.counts[i] = 0;
        if (thread == 0) s.tile = t;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kIds; ++j) count_in(s.counts, id[j], j * kBlock + thread < a.m, lane);
        __syncthreads();
        const int each = (groups + kBlock - 1) / kBlock, begin = min(thread * each, groups), end = min(begin + each, groups);
        int at = 0, none = 0, all;
        for (int g = begin; g < end; ++g) at += (s.counts[g] + tile - 1) / tile;
        sums_before(none, at, all, s.sums, lane, wave);
        for (int g = begin; g < end; ++g) {
            const int count = s.counts[g], tiles = (count + tile - 1) / tile;
            if (index >= at && index < at + tiles) {
                s.tile = {g < a.count ? g : -1, min(tile, count - (index - at) * tile)};
                s.first = (index - at) * tile;
            }
            at += tiles;
        }
        __syncthreads();
        t = s.tile;
        if (t.count == 0) return t;
        const int group = t.id < 0 ? a.count : t.id;
        unsigned long long mine[kIds];
#pragma unroll
        for (int j = 0; j < kIds; ++j) {
            mine[j] = __ballot(j * kBlock + thread < a.m && id[j] == group);
            if (lane == 0) s.parts[j * (kBlock / 64) + wave] = __popcll(mine[j]);
        }
        __syncthreads();
        int before = -s.first;
#pragma unroll
        for (int j = 0; j < kIds; ++j)
#pragma unroll
            for (int w = 0; w < kBlock / 64; ++w) {
                const int place = before + __popcll(mine[j] & ((1ull << lane) - 1));
                if (w == wave && (mine[j] >> lane & 1) && place >= 0 && place < t.count) s.tokens[place] = j * kBlock + thread;
                before += s.parts[j * (kBlock / 64) + w];
            }
    } else {
        const AdapterTile f = a.tiles[index];
        t = {f.id, f.count};
        if (thread < t.count) s.tokens[thread] = ld_global(a.order + f.first + thread);
    }
    __syncthreads();
    return t;
}

// All loads are of whole vectors, and no lane branches round one (else each would be waited for before the next is asked for): a vector that
// would go over the end of a row of N or more values begins N before it instead, and what it then has of the vector before counts as
// zero in one of the two factors.  SHORT: rows of less, value by value.
__device__ __forceinline__ int begin_of(int at, int n, int width) { return max(min(at, width - n), 0); }

template <int N, bool SHORT, typename T> __device__ __forceinline__ void load(T *to, const T *row, int at, int width)
{
    if constexpr (!SHORT) {
        __builtin_memcpy(to, (const FQ_GLOBAL T *)(row + at), sizeof(T) * N);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) to[e] = ld_global(row + min(at + e, width - 1));
    }
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

// 16 neighbouring values of a row.
template <typename X> struct Piece {
    X v[16];
    template <bool SHORT> __device__ __forceinline__ void fetch(const X *row, int at, int k) { load<16, SHORT>(v, row, at, k); }
    // only those from `first` to `last` count
    __device__ __forceinline__ void keep(int first, int last)
    {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = e >= first && e <= last ? v[e] : (X)0;
    }
    __device__ __forceinline__ f16x8 half(int i) const
    {
        f16x8 h;
        if constexpr (sizeof(X) == 1) {
            int w[4];
            __builtin_memcpy(w, v, sizeof w);
            h = halves_of(w[2 * i], w[2 * i + 1]);
        } else {
            __builtin_memcpy(&h, v + 8 * i, sizeof h);
        }
        return h;
    }
};

// t of a tile: NT x 16 tokens by NR x 16 ranks.  The wavefronts of a block take 64 values of k in turn; their sums meet in LDS.  Loads go
// straight into the registers that the matrix instructions take (lane l: token l % 16, and rank l % 16, values 16 (l / 16) and on of the
// 64: whole lines from four lanes).  Small tiles have the loads of the next 64 on their way while these are multiplied; large ones
// would need more registers for that than four blocks on a compute unit have, and those cover for each other.
constexpr int kDownWaves = kBlock / 64, kDepth = 64;

template <typename X, int NT, int NR, bool SHORT>
__global__ __launch_bounds__(kBlock, NT * NR == 1 ? 1 : 4) void adapter_down_kernel(AdapterArgs a)
{
    constexpr int kAhead = NT * NR == 1 ? 2 : 1;                   // steps whose loads are on their way at a time
    __shared__ f32x4 part[kDownWaves][NT * NR][64];
    __shared__ Finding finding;
    const int *tokens = finding.tokens;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int split = blockIdx.x % a.splits, chunk = blockIdx.x / a.splits % a.chunks;
    const Tile tile = find_tile(a, blockIdx.x / a.splits / a.chunks, finding);
    if (tile.id < 0 || tile.count == 0) return;
    const int steps = (a.k + kDepth - 1) / kDepth;
    const int begin = (int)((long long)steps * split / a.splits), end = (int)((long long)steps * (split + 1) / a.splits);
    const _Float16 *ranks[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r)
        ranks[r] = (const _Float16 *)a.a + ((long long)tile.id * a.rank + min((chunk * NR + r) * 16 + lane % 16, a.rank - 1)) * a.k;
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        const X *rows[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) rows[n] = (const X *)a.x + tokens[min(sub + n * 16 + lane % 16, tile.count - 1)] * a.ldx;
        f32x4 sum[NT][NR];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) sum[n][r] = (f32x4)0.0f;
        Piece<X> x[kAhead][NT];
        Piece<_Float16> w[kAhead][NR];
        const auto fetch = [&](int buffer, int step) {
            const int at = begin_of(step * kDepth + lane / 16 * 16, 16, a.k);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[buffer][n].template fetch<SHORT>(rows[n], at, a.k);
#pragma unroll
            for (int r = 0; r < NR; ++r) w[buffer][r].template fetch<SHORT>(ranks[r], at, a.k);
        };
        const auto multiply = [&](int buffer, int step) {
            if ((step + 1) * kDepth > a.k) {
                const int at = step * kDepth + lane / 16 * 16, from = begin_of(at, 16, a.k);
#pragma unroll
                for (int n = 0; n < NT; ++n) x[buffer][n].keep(at - from, a.k - 1 - from);
            }
            if constexpr (std::is_same<X, float>::value) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
#pragma unroll
                    for (int r = 0; r < NR; ++r) {
                        const float v = (float)w[buffer][r].v[e];
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            sum[n][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[buffer][n].v[e], sum[n][r], 0, 0, 0);
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
        if constexpr (kAhead == 2) {
            if (step < end) fetch(0, step);
            while (step < end) {
                if (step + kDownWaves < end) fetch(1, step + kDownWaves);
                multiply(0, step);
                step += kDownWaves;
                if (step >= end) break;
                if (step + kDownWaves < end) fetch(0, step + kDownWaves);
                multiply(1, step);
                step += kDownWaves;
            }
        } else {
            for (; step < end; step += kDownWaves) {
                fetch(0, step);
                multiply(0, step);
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) part[wave][n * NR + r][lane] = sum[n][r];
        __syncthreads();
        // lane l's four sums: token l % 16, ranks 4 (l / 16) and on
        for (int i = threadIdx.x; i < NT * NR * 64; i += kBlock) {
            const int n = i / 64 / NR, r = i / 64 % NR, l = i % 64;
            const int token = sub + n * 16 + l % 16, rank = (chunk * NR + r) * 16 + l / 16 * 4;
            f32x4 s = part[0][n * NR + r][l];
#pragma unroll
            for (int v = 1; v < kDownWaves; ++v) s += part[v][n * NR + r][l];
            if (token < tile.count && rank < a.pitch)
                st_global((f32x4 *)(a.t + ((long long)split * a.m + tokens[token]) * a.pitch + rank), s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------
// y of a tile of NT x 16 tokens, in strips of CT x 16 channels to each of four wavefronts.  First the block adds up t (of all its
// parts) and puts it into LDS as two FP16 numbers to a value: t 2^-e to 11 bits and the rest to 11 more, 2^e the power of two that
// brings the row's greatest into [2^14, 2^15), so that nothing overflows and 22 bits of each are kept, or 2^-39 of the greatest.  (FP16
// products cost a quarter of the matrix cores' time that binary32 ones take.)  Then a wavefront has channels for the rows of its products and
// tokens for the columns: lane l has, of token l % 16, groups of 8 (CT 1: of 4) neighbouring channels, and four lanes 64 bytes of FP16.
constexpr int kUpWaves = kBlock / 64;

__device__ __forceinline__ f32x4 product(f16x8 b, f16x8 t, f32x4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(b, t, sum, 0, 0, 0); }

// N neighbouring channels.  Where a row ends within them they begin N before its end (see begin_of); those of them that are
// others' are left to those.
template <typename T, int N> struct Channels {
    T v[N];
    __device__ __forceinline__ void store(T *row, int at, int n) const
    {
        if (at + N <= n) {
            __builtin_memcpy((FQ_GLOBAL T *)(row + at), v, sizeof v);
            return;
        }
        const int begin = begin_of(at, N, n);
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (begin + e >= at && begin + e < n) st_global(row + begin + e, v[e]);
    }
};

// Where rank l of t lies in LDS, so that eight places are the ranks of one vector of b (which begins eight before the end of a row where it
// would go over it): the last ranks at the end of their vector, what would be before them behind it.  (Places of no rank hold zeros.)
__device__ __forceinline__ int place_of_rank(int l, int rank)
{
    const int last = rank / 8 * 8, off = rank % 8;
    if (rank < 8 || off == 0 || l < last) return l;
    return l < rank ? l + 8 - off : l < last + 8 ? l - off : l;
}

// y's kernel takes t in units of four ranks, eight lanes to a token: unit u, u + 8, ... to lane u.  J units of a lane, of all parts: eight
// loads on their way at a time.
template <int J> __device__ __forceinline__ void sum_of_parts(f32x4 (&s)[J], const AdapterArgs &a, const float *t, int unit)
{
    constexpr int P = 8 / J;
    const long long part = (long long)a.m * a.pitch;
#pragma unroll
    for (int j = 0; j < J; ++j) s[j] = (f32x4)0.0f;
    for (int p = 0; p < a.splits; p += P) {
        f32x4 v[P][J];
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) v[i][j] = ld_global((const f32x4 *)(t + min(p + i, a.splits - 1) * part + min((j * 8 + unit) * 4, a.pitch - 4)));
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j)
                if (p + i < a.splits) s[j] += v[i][j];
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[j][e] = (j * 8 + unit) * 4 + e < a.rank ? s[j][e] : 0.0f;
}

// FEW: channels, fewer than N; SHORT: rows of b, fewer than eight ranks; J: of t's units, 32 J ranks at most.
template <typename Y, typename B, int NT, int CT, int J, bool FEW, bool SHORT>
__global__ __launch_bounds__(kBlock, J == 8 ? 2 : 4) void adapter_up_kernel(AdapterArgs a)
{
    constexpr int N = CT == 1 ? 4 : 8, G = CT == 1 ? 1 : CT / 2;      // channels of a lane that are neighbours, and groups of them
    extern __shared__ __attribute__((aligned(16))) _Float16 shared[];          // [2][NT * 16][row]
    __shared__ Finding finding;
    __shared__ float factor[NT * 16];
    const int *tokens = finding.tokens;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Tile tile = find_tile(a, blockIdx.x / a.groups, finding);
    const int deep = (a.rank + 31) / 32, row = deep * 32 + 8;
    const bool copy = tile.id < 0;
    if (copy && a.base == a.y) return;
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        int strip = (int)(blockIdx.x % a.groups) * kUpWaves + wave;
        long long from[NT], to[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int token = tokens[min(sub + n * 16 + lane % 16, tile.count - 1)];
            from[n] = token * a.ldbase;
            to[n] = token * a.ldy;
        }
        Channels<B, N> base[NT][G];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int e = 0; e < N; ++e) base[n][g].v[e] = (B)0.0f;
        const auto ask = [&]() {
            if (!a.base) return;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int at = begin_of(strip * CT * 16 + g * 32 + lane / 16 * N, N, a.n);
#pragma unroll
                for (int n = 0; n < NT; ++n) load<N, FEW>(base[n][g].v, (const B *)a.base + from[n], at, a.n);
            }
        };
        if (strip * CT * 16 < a.n) ask();
        if (!copy) {
            const int i = threadIdx.x / 8, unit = threadIdx.x % 8;
            if (i < NT * 16) {
                const int token = tokens[min(sub + i, tile.count - 1)];
                f32x4 s[J];
                sum_of_parts<J>(s, a, a.t + (long long)token * a.pitch, unit);
                float most = 0.0f;
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(s[j][e]));
                most = __builtin_fmaxf(most, __shfl_xor(most, 1));
                most = __builtin_fmaxf(most, __shfl_xor(most, 2));
                most = __builtin_fmaxf(most, __shfl_xor(most, 4));
                const int e2 = most > 0.0f && most < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(most) : 0;
                _Float16 *const heads = shared + i * row, *const rests = heads + NT * 16 * row;
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int l = (j * 8 + unit) * 4;
                    if (l >= deep * 32) continue;
                    f16x4 high, low;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float v = __builtin_ldexpf(s[j][e], e2);
                        high[e] = (_Float16)v;
                        const float off = v - (float)high[e];
                        low[e] = (_Float16)(__builtin_fabsf(off) < __builtin_inff() ? off : 0.0f);
                    }
                    if (a.rank % 4 == 0) {       // (neighbours stay neighbours)
                        const int at = place_of_rank(l, a.rank);
                        *(f16x4 *)(heads + at) = high;
                        *(f16x4 *)(rests + at) = low;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            heads[place_of_rank(l + e, a.rank)] = high[e];
                            rests[place_of_rank(l + e, a.rank)] = low[e];
                        }
                    }
                }
                if (unit == 0) {
                    const float f = (a.scale ? ld_global(a.scale + tile.id) : 1.0f) * (a.xs ? ld_global(a.xs + (long long)token * a.xs_step) : 1.0f);
                    factor[i] = __builtin_ldexpf(f, -e2);
                }
            }
        }
        __syncthreads();
        while (strip * CT * 16 < a.n) {
            f32x4 sum[NT][CT];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < CT; ++c) sum[n][c] = (f32x4)0.0f;
            if (!copy) {
                const _Float16 *channel[CT];
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    // row i of product c: channel i / 4 of four groups of N, half c % 2 of it, i % 4 of that
                    const int first = begin_of(strip * CT * 16 + c / 2 * 32 + lane % 16 / 4 * N, N, a.n);
                    channel[c] = (const _Float16 *)a.b + ((long long)tile.id * a.n + min(first + c % 2 * 4 + lane % 4, a.n - 1)) * a.rank;
                }
                for (int d = 0; d < deep; ++d) {
                    f16x8 b[CT];
#pragma unroll
                    for (int c = 0; c < CT; ++c) load<8, SHORT>((_Float16 *)&b[c], channel[c], begin_of(d * 32 + lane / 16 * 8, 8, a.rank), a.rank);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const _Float16 *at = shared + (n * 16 + lane % 16) * row + d * 32 + lane / 16 * 8;
                        const f16x8 high = *(const f16x8 *)at, low = *(const f16x8 *)(at + NT * 16 * row);
#pragma unroll
                        for (int c = 0; c < CT; ++c) sum[n][c] = product(b[c], low, product(b[c], high, sum[n][c]));
                    }
                }
            }
            Channels<Y, N> y[NT][G];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float f = copy ? 0.0f : factor[n * 16 + lane % 16];
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float v = (float)base[n][g].v[e];
                        y[n][g].v[e] = (Y)(copy ? v : v + f * sum[n][g * 2 + e / 4][e % 4]);
                    }
            }
            const int done = strip;
            strip += a.groups * kUpWaves;
            if (strip * CT * 16 < a.n) ask();
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (sub + n * 16 + lane % 16 >= tile.count) continue;
#pragma unroll
                for (int g = 0; g < G; ++g) y[n][g].store((Y *)a.y + to[n], done * CT * 16 + g * 32 + lane / 16 * N, a.n);
            }
        }
        __syncthreads();
    }
}

template <typename X> int down(const AdapterArgs &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)a.tiles_most * (unsigned)a.splits * (unsigned)a.chunks;
    const int shape = a.token_tiles * 10 + a.rank_tiles;
    if (a.k < 16) adapter_down_kernel<X, 1, 1, true><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 11) adapter_down_kernel<X, 1, 1, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 12) adapter_down_kernel<X, 1, 2, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 14) adapter_down_kernel<X, 1, 4, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 21) adapter_down_kernel<X, 2, 1, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 22) adapter_down_kernel<X, 2, 2, false><<<blocks, kBlock, 0, stream>>>(a);
    else adapter_down_kernel<X, 2, 4, false><<<blocks, kBlock, 0, stream>>>(a);
    return (int)hipGetLastError();
}

template <typename Y, typename B, int NT, int CT> void up_by(const AdapterArgs &a, unsigned blocks, size_t lds, hipStream_t stream)
{
    if (a.rank < 8) adapter_up_kernel<Y, B, NT, CT, 1, false, true><<<blocks, kBlock, lds, stream>>>(a);
    else if (a.rank <= 64) adapter_up_kernel<Y, B, NT, CT, 2, false, false><<<blocks, kBlock, lds, stream>>>(a);
    else adapter_up_kernel<Y, B, NT, CT, 8, false, false><<<blocks, kBlock, lds, stream>>>(a);
}

template <typename Y, typename B> void up(const AdapterArgs &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)a.tiles_most * (unsigned)a.groups;
    const size_t lds = a.count > 0 ? (size_t)2 * 16 * a.token_tiles * ((a.rank + 31) / 32 * 32 + 8) * sizeof(_Float16) : 0;
    if (a.n < 8) adapter_up_kernel<Y, B, 1, 1, 8, true, true><<<blocks, kBlock, lds, stream>>>(a);
    else if (a.token_tiles == 2) up_by<Y, B, 2, 4>(a, blocks, lds, stream);
    else if (a.wide == 4) up_by<Y, B, 1, 4>(a, blocks, lds, stream);
    else up_by<Y, B, 1, 1>(a, blocks, lds, stream);
}

}  // namespace

int launch_adapters(const AdapterArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.count > 0) {
        if (a.way == kList) adapter_group_kernel<<<1, kGroupThreads, (size_t)(a.count + 1) * sizeof(int), s>>>(a);
        const int err = a.x_type == 0 ? down<_Float16>(a, s) : a.x_type == 1 ? down<float>(a, s) : down<int8_t>(a, s);
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
