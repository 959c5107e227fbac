// Low-rank adapters of many requests beside a shared layer (declared in include/fq.h).
//
//   t = x a^T,   y = base + (xs scale) t b^T      a, b: those of the token's adapter
//
// Two steps, since all of t is needed for any y: adapter_down_kernel makes t, in parts of k where there are few tiles, and
// adapter_up_kernel adds them up and makes y.  Both work on tiles of 16, 32 or 64 tokens of one adapter, whose rows they pick out by a
// list.  Up to 64 tokens, and any number for more than 1024 adapters, go in windows of 64, in which a wavefront finds those of an adapter by itself;
// up to 4096 are sorted by the first kernel's blocks, which leave the second what they have found; more are ordered by adapter_group_kernel first.
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
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ bool has_adapter(int id, int count) { return id >= 0 && id < count; }

// ---------------------------------------------------------------------------------------------
// Tokens in the order of their adapters (those without one behind all others), those of an adapter in the order that they come in, and
// the tiles of each.  One block, each of whose wavefronts has a run of tokens and counters of its own: what each adds to them is known from
// the lanes with the same adapter, so places do not depend on which wavefront is first.
constexpr int kGroupThreads = 1024, kGroupWaves = kGroupThreads / 64, kHeldIds = 8;
constexpr int kGroupBits = 11;                   // of a group's number: kMostGrouped and one more
static_assert(kMostGrouped < (1 << kGroupBits), "groups have numbers of kGroupBits");

__device__ __forceinline__ int group_of(const AdapterArgs &a, int token)
{
    const int id = token < a.m ? ld_global(a.ids + token) : -1;
    return has_adapter(id, a.count) ? id : a.count;
}

// The lanes with `some` that have this lane's group.
__device__ __forceinline__ unsigned long long peers(int group, bool some)
{
    unsigned long long mine = __ballot(some);
    if (mine == 0) return 0;
    const int leader = __builtin_amdgcn_readlane(group, __builtin_ctzll(mine));
    if (__ballot(some && group == leader) == mine) return mine;          // (tokens of one request come one after the other)
#pragma unroll
    for (int bit = 0; bit < kGroupBits; ++bit) {
        const unsigned long long set = __ballot(group >> bit & 1);
        mine &= group >> bit & 1 ? set : ~set;
    }
    return mine;
}

__device__ __forceinline__ int before(unsigned long long lanes, int lane) { return __popcll(lanes & ((1ull << lane) - 1)); }

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
    extern __shared__ int counts[];              // [kGroupWaves][count + 1]: of tokens, then the next free place
    __shared__ int sums[2][kGroupWaves];
    const int groups = a.count + 1, thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    const int tile = 16 * a.token_tiles, run = (a.m + kGroupThreads - 1) / kGroupThreads * 64;
    const int first = wave * run, last = min(first + run, a.m);
    volatile int *const own = counts + wave * groups;
    int held[kHeldIds];
    const auto ask = [&](int from) {
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) held[j] = group_of(a, min(from + j * 64 + lane, last));
    };
    ask(first);
    for (int i = thread; i < groups * kGroupWaves; i += kGroupThreads) counts[i] = 0;
    __syncthreads();
    for (int from = first; from < last; from += 64 * kHeldIds) {
        if (from > first) ask(from);
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) {
            const unsigned long long mine = peers(held[j], from + j * 64 + lane < last);
            if ((mine >> lane & 1) && before(mine, lane) == 0) own[held[j]] = own[held[j]] + __popcll(mine);
        }
    }
    __syncthreads();
    // first places and first tiles of the groups: each thread has a run of them
    const int each = (groups + kGroupThreads - 1) / kGroupThreads, begin = min(thread * each, groups), end = min(begin + each, groups);
    int token_at = 0, tile_at = 0, all_tiles;
    for (int g = begin; g < end; ++g) {
        int count = 0;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) count += counts[w * groups + g];
        token_at += count;
        tile_at += (count + tile - 1) / tile;
    }
    sums_before(token_at, tile_at, all_tiles, sums, lane, wave);
    for (int g = begin; g < end; ++g) {
        const int start = token_at;
#pragma unroll
        for (int w = 0; w < kGroupWaves; ++w) {
            const int count = counts[w * groups + g];
            counts[w * groups + g] = token_at;
            token_at += count;
        }
        for (int i = start; i < token_at; i += tile) a.tiles[tile_at++] = AdapterTile{g < a.count ? g : -1, i, min(tile, token_at - i)};
    }
    for (int i = all_tiles + thread; i < a.tiles_most; i += kGroupThreads) a.tiles[i] = AdapterTile{-1, 0, 0};
    __syncthreads();
    for (int from = first; from < last; from += 64 * kHeldIds) {
        if (run > 64 * kHeldIds) ask(from);
#pragma unroll
        for (int j = 0; j < kHeldIds; ++j) {
            const int token = from + j * 64 + lane;
            const unsigned long long mine = peers(held[j], token < last);
            if (mine >> lane & 1) {
                const int place = own[held[j]], rank = before(mine, lane);
                a.order[place + rank] = token;
                if (rank == 0) own[held[j]] = place + __popcll(mine);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The tile of a block: its adapter (-1: none) and its tokens, which go to `tokens`.  Three ways:
//   windows   up to kWindow tokens (or windows of so many): those that have the adapter of token `slot` of theirs, if that is the first to have
//             it; so every adapter of the window has one block, which takes them by tiles one after the other
//   sorting   up to kSorted tokens: the block counts the tokens of each adapter by itself, which costs less than a launch in
//             front and the two trips to memory for its results (us, 4096 x 4096 by 16 ranks: 2048 tokens 23.2, 27.1 with a list; 4000
//             tokens 33.8, 36.8; 8192 x 8192 by 64 ranks, 8192 tokens: 122.8, 120.4); adapter_down_kernel then leaves what it has found to adapter_up_kernel
//   list      tile and tokens are what adapter_group_kernel has written
struct Tile {
    int id, count;
};

struct Finding {
    int tokens[kWindow];
    int counts[kMostGrouped + 1];
    int sums[2][kBlock / 64], parts[kSorted / 64];
    Tile tile;
    int first;
};

// Sorting (see find_tile), IDS tokens to a thread.
template <int IDS> __device__ __forceinline__ Tile sorted_tile(const AdapterArgs &a, int index, Finding &s)
{
    const int thread = threadIdx.x, lane = thread & 63, wave = thread >> 6;
    Tile t = {-1, 0};
    const int groups = a.count + 1, tile = 16 * a.token_tiles;
    int id[IDS];
#pragma unroll
    for (int j = 0; j < IDS; ++j) id[j] = group_of(a, j * kBlock + thread);
    for (int i = thread; i < groups; i += kBlock) s.counts[i] = 0;
    if (thread == 0) s.tile = t;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < IDS; ++j) {
        // (tokens of one request come one after the other: then the wavefront counts once)
        const bool some = j * kBlock + thread < a.m;
        const unsigned long long mine = __ballot(some);
        if (mine == 0) continue;
        const int leader = __builtin_amdgcn_readlane(id[j], __builtin_ctzll(mine));
        if (__ballot(some && id[j] == leader) == mine) {
            if (lane == 0) atomicAdd(s.counts + leader, __popcll(mine));
        } else if (some) {
            atomicAdd(s.counts + id[j], 1);
        }
    }
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
    unsigned long long mine[IDS];
#pragma unroll
    for (int j = 0; j < IDS; ++j) {
        mine[j] = __ballot(j * kBlock + thread < a.m && id[j] == group);
        if (lane == 0) s.parts[j * (kBlock / 64) + wave] = __popcll(mine[j]);
    }
    __syncthreads();
    int place = -s.first;
#pragma unroll
    for (int j = 0; j < IDS; ++j) {
        if (j * kBlock >= a.m || place >= t.count) continue;
#pragma unroll
        for (int w = 0; w < kBlock / 64; ++w) {
            const int own = place + before(mine[j], lane);
            if (w == wave && (mine[j] >> lane & 1) && own >= 0 && own < t.count) s.tokens[own] = j * kBlock + thread;
            place += s.parts[j * (kBlock / 64) + w];
        }
    }
    return t;
}

// What adapter_down_kernel's block of a tile has found: count, adapter and tokens.
__device__ __forceinline__ int *record_of(const AdapterArgs &a, int index) { return a.found + index * (2 + 16 * a.token_tiles); }

__device__ __forceinline__ void leave_tile(const AdapterArgs &a, int index, const Tile &t, const Finding &s)
{
    int *const record = record_of(a, index);
    if (threadIdx.x < 2) st_global(record + threadIdx.x, threadIdx.x ? t.id : t.count);
    if ((int)threadIdx.x < t.count) st_global(record + 2 + threadIdx.x, s.tokens[threadIdx.x]);
}

__device__ __forceinline__ Tile left_tile(const AdapterArgs &a, int index, Finding &s)
{
    const int thread = threadIdx.x, v = thread < 2 + 16 * a.token_tiles ? ld_global(record_of(a, index) + thread) : 0;
    if (thread == 0) s.tile.count = v;
    else if (thread == 1) s.tile.id = v;
    else if (thread < 2 + kWindow) s.tokens[thread - 2] = v;
    __syncthreads();
    return s.tile;
}

__device__ __forceinline__ Tile find_tile(const AdapterArgs &a, int index, Finding &s)
{
    const int thread = threadIdx.x, lane = thread & 63;
    Tile t = {-1, 0};
    if (a.way == kWindows) {
        const int slots = min(a.m, kWindow), begin = index / slots * kWindow, slot = index % slots;
        const int left = min(a.m - begin, kWindow);
        int id = lane < left ? ld_global(a.ids + begin + lane) : -2;
        if (lane < left && !has_adapter(id, a.count)) id = -1;
        t.id = __builtin_amdgcn_readlane(id, slot);
        const unsigned long long mine = __ballot(id == t.id);
        t.count = slot < left && __builtin_ctzll(mine) == slot ? __popcll(mine) : 0;
        if (thread < 64 && (mine >> lane & 1)) s.tokens[before(mine, lane)] = begin + lane;
    } else if (a.way == kSorting) {
        t = a.m <= kFewSorted ? sorted_tile<kFewSorted / kBlock>(a, index, s) : sorted_tile<kSorted / kBlock>(a, index, s);
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
// zero: for t in both factors (an infinity in one would make the other's zero NaN), for y in t.  SHORT: rows of less, value by value.
__device__ __forceinline__ int begin_of(int at, int n, int width) { return max(min(at, width - n), 0); }

// N values, in the words that they are loaded in.  (As an array of values they would be taken apart into a register each.)
template <typename T, int N> struct Words {
    static constexpr int kWords = (int)sizeof(T) * N / 4;
    typedef T V __attribute__((ext_vector_type(N)));
    typedef int W __attribute__((ext_vector_type(kWords)));
    W w;
    __device__ __forceinline__ V values() const { return __builtin_bit_cast(V, w); }
};

template <bool SHORT, typename T, int N> __device__ __forceinline__ void load(Words<T, N> &to, const T *row, int at, int width)
{
    if constexpr (!SHORT) {
        __builtin_memcpy(&to, (const FQ_GLOBAL T *)(row + at), sizeof to);
    } else {
        typename Words<T, N>::V v;
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = ld_global(row + min(at + e, width - 1));
        to.w = __builtin_bit_cast(typename Words<T, N>::W, v);
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
    Words<X, 16> p;
    template <bool SHORT> __device__ __forceinline__ void fetch(const X *row, int at, int k) { load<SHORT>(p, row, at, k); }
    __device__ __forceinline__ f16x8 half(int i) const
    {
        if constexpr (sizeof(X) == 1) return halves_of(p.w[2 * i], p.w[2 * i + 1]);
        else return __builtin_bit_cast(f16x8, i32x4{p.w[4 * i], p.w[4 * i + 1], p.w[4 * i + 2], p.w[4 * i + 3]});
    }
    __device__ __forceinline__ X value(int e) const { return p.values()[e]; }
};

// Only the values from `first` to `last` of each piece count.
template <typename X, int N> __device__ __forceinline__ void keep(Piece<X> (&pieces)[N], int first, int last)
{
    constexpr int kEach = 4 / (int)sizeof(X), kBits = 8 * (int)sizeof(X);
#pragma unroll
    for (int d = 0; d < Words<X, 16>::kWords; ++d) {
        unsigned mask = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            mask |= d * kEach + e >= first && d * kEach + e <= last ? (unsigned)((1ull << kBits) - 1) << (e * kBits) : 0u;
#pragma unroll
        for (int n = 0; n < N; ++n) pieces[n].p.w[d] &= (int)mask;
    }
}

// The products of 64 values of k: a lane has 16 neighbouring ones of a token, and of a rank.
template <typename X, int NT, int NR> __device__ __forceinline__ void multiply(f32x4 (&sum)[NT][NR], const Piece<X> (&x)[NT], const Piece<_Float16> (&w)[NR])
{
    if constexpr (std::is_same<X, float>::value) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const float v = (float)w[r].value(e);
#pragma unroll
                for (int n = 0; n < NT; ++n) sum[n][r] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, x[n].value(e), sum[n][r], 0, 0, 0);
            }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f16x8 v[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) v[n] = x[n].half(i);
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int n = 0; n < NT; ++n) sum[n][r] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[r].half(i), v[n], sum[n][r], 0, 0, 0);
        }
    }
}

// The sums of a block's wavefronts, added up and written to t.  Lane l's four: token l % 16, ranks 4 (l / 16) and on.
constexpr int kDownWaves = kBlock / 64, kDepth = 64;

template <int NT, int NR>
__device__ __forceinline__ void join(const AdapterArgs &a, f32x4 (*part)[NT * NR][64], const f32x4 (&sum)[NT][NR], const int *tokens, int sub, int count,
                                     int split, int chunk)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int r = 0; r < NR; ++r) part[wave][n * NR + r][lane] = sum[n][r];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * NR * 64; i += kBlock) {
        const int n = i / 64 / NR, r = i / 64 % NR, l = i % 64;
        const int token = sub + n * 16 + l % 16, rank = (chunk * NR + r) * 16 + l / 16 * 4;
        f32x4 s = part[0][n * NR + r][l];
#pragma unroll
        for (int v = 1; v < kDownWaves; ++v) s += part[v][n * NR + r][l];
        if (token < count && rank < a.pitch) st_global((f32x4 *)(a.t + ((long long)split * a.m + tokens[token]) * a.pitch + rank), s);
    }
    __syncthreads();
}

// What a block of the kernels below works on: a tile, a part of the ranks, and steps [begin, begin + length) of 64 values of k.  Each tile
// begins elsewhere in its part and goes round (`turn`), so that blocks do not all ask for the same columns at a time.
struct Share {
    int index, split, chunk, begin, length, turn;
    __device__ __forceinline__ explicit Share(const AdapterArgs &a)
    {
        split = blockIdx.x % a.splits;
        chunk = blockIdx.x / a.splits % a.chunks;
        index = blockIdx.x / a.splits / a.chunks;
        const int steps = (a.k + kDepth - 1) / kDepth;
        begin = (int)((long long)steps * split / a.splits);
        length = (int)((long long)steps * (split + 1) / a.splits) - begin;
        turn = length > 0 ? (int)((unsigned)index * 2654435769u >> 16) % length : 0;
    }
    __device__ __forceinline__ int step(int i) const { return begin + (i + turn < length ? i + turn : i + turn - length); }
};

// t of a tile: NT x 16 tokens by NR x 16 ranks.  The wavefronts of a block take 64 values of k in turn.  Here the loads go
// straight into the registers that the matrix instructions take (lane l: token l % 16, and rank l % 16, values 16 (l / 16) and on of the
// 64), from rows at any address: for few tokens, and where rows do not fit adapter_down_ring_kernel.
template <typename X, int NT, int NR, bool SHORT>
__global__ __launch_bounds__(kBlock, SHORT ? 2 : 4) void adapter_down_kernel(AdapterArgs a)
{
    __shared__ f32x4 part[kDownWaves][NT * NR][64];
    __shared__ Finding finding;
    const int *tokens = finding.tokens;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Share share(a);
    const Tile tile = find_tile(a, share.index, finding);
    if (a.way == kSorting && share.split == 0 && share.chunk == 0) leave_tile(a, share.index, tile, finding);
    if (tile.id < 0 || tile.count == 0) return;
    const _Float16 *ranks[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r)
        ranks[r] = (const _Float16 *)a.a + ((long long)tile.id * a.rank + min((share.chunk * NR + r) * 16 + lane % 16, a.rank - 1)) * a.k;
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        const X *rows[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) rows[n] = (const X *)a.x + tokens[min(sub + n * 16 + lane % 16, tile.count - 1)] * a.ldx;
        f32x4 sum[NT][NR];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) sum[n][r] = (f32x4)0.0f;
        for (int i = wave; i < share.length; i += kDownWaves) {
            Piece<X> x[NT];
            Piece<_Float16> w[NR];
            const int at = share.step(i) * kDepth + lane / 16 * 16, from = begin_of(at, 16, a.k);
#pragma unroll
            for (int n = 0; n < NT; ++n) x[n].template fetch<SHORT>(rows[n], from, a.k);
#pragma unroll
            for (int r = 0; r < NR; ++r) w[r].template fetch<SHORT>(ranks[r], from, a.k);
            if (share.step(i) * kDepth + kDepth > a.k) {
                keep(x, at - from, a.k - 1 - from);
                keep(w, at - from, a.k - 1 - from);
            }
            multiply<X, NT, NR>(sum, x, w);
        }
        join<NT, NR>(a, part, sum, tokens, sub, tile.count, share.split, share.chunk);
    }
}

// The same by way of LDS: loads of whole lines, eight neighbouring lanes to one, go straight there, each wavefront's into a ring of its own
// whose slots hold 64 values of k of all rows, and the lanes pick out what the matrix instructions take.  (8192 x 8192 FP16 by 64 ranks:
// 36 us, 3.7 TB/s; 48 with lanes of one load in 16 rows, as above, which are looked up in the caches one by one.)  A slot's rows of C
// chunks of 16 bytes lie one behind the other, chunk c of row r at place c ^ (r C / 16 modulo C): LDS answers 16 lanes at a time from
// 256 bytes, and 16 neighbouring rows then have theirs in 16 places.
template <int C> __device__ __forceinline__ int place_in_row(int chunk, int row) { return chunk ^ (row * C / 16 & (C - 1)); }

template <typename X, int NT, int NR> constexpr int ring_slot() { return (NT * (int)sizeof(X) + NR * 2) * 1024; }
template <typename X, int NT, int NR> constexpr int ring_slots() { return ring_slot<X, NT, NR>() <= 6144 ? 3 : 2; }

template <typename X, int NT, int NR>
__global__ __launch_bounds__(kBlock) void adapter_down_ring_kernel(AdapterArgs a)
{
    constexpr int kSlot = ring_slot<X, NT, NR>(), kSlots = ring_slots<X, NT, NR>(), kX = NT * (int)sizeof(X), kW = NR * 2, kLoads = kX + kW;
    constexpr int kChunks = 4 * (int)sizeof(X);                    // of 16 bytes, of a row of x in a slot; of a rank's: 8
    extern __shared__ __attribute__((aligned(1024))) int8_t ring[];            // [wavefronts][slots][x, a]
    static_assert(kDownWaves * kSlots * kSlot >= kDownWaves * NT * NR * 1024, "the sums of all wavefronts fit in the rings");
    __shared__ Finding finding;
    const int *tokens = finding.tokens;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Share share(a);
    const Tile tile = find_tile(a, share.index, finding);
    if (a.way == kSorting && share.split == 0 && share.chunk == 0) leave_tile(a, share.index, tile, finding);
    if (tile.id < 0 || tile.count == 0) return;
    const uint64_t x_at = (uint64_t)a.x, a_at = (uint64_t)a.a + (uint64_t)tile.id * (uint64_t)a.rank * (uint64_t)a.k * 2;
    // descriptors of raw buffers: the hardware answers loads behind their ends with zeros
    const i32x4 x_buffer = {(int)x_at, (int)(x_at >> 32) & 0xFFFF, (int)a.x_bytes, 0x00027000};
    const i32x4 a_buffer = {__builtin_amdgcn_readfirstlane((int)a_at), __builtin_amdgcn_readfirstlane((int)(a_at >> 32) & 0xFFFF), a.rank * a.k * 2, 0x00027000};
    unsigned w_off[kW];
#pragma unroll
    for (int j = 0; j < kW; ++j) {
        const int row = j * 8 + lane / 8;
        w_off[j] = (unsigned)min(share.chunk * NR * 16 + row, a.rank - 1) * (unsigned)a.k * 2 + (unsigned)place_in_row<8>(lane % 8, row) * 16;
    }
    int8_t *const own = ring + wave * (kSlots * kSlot);
    for (int sub = 0; sub < tile.count; sub += NT * 16) {
        unsigned x_off[kX];
#pragma unroll
        for (int j = 0; j < kX; ++j) {
            const int row = (j * 64 + lane) / kChunks;
            x_off[j] = (unsigned)tokens[min(sub + row, tile.count - 1)] * (unsigned)(a.ldx * (int)sizeof(X)) +
                       (unsigned)place_in_row<kChunks>(lane % kChunks, row) * 16;
        }
        constexpr unsigned kNowhere = 0xFFFFFFF0u;                 // behind the end of any buffer
        const auto ask = [&](int i) {
            const bool none = i >= share.length;
            const unsigned step = none ? 0 : (unsigned)share.step(i);
            int8_t *const to = own + i / kDownWaves % kSlots * kSlot;
#pragma unroll
            for (int j = 0; j < kX; ++j) load_lds(x_buffer, none ? kNowhere : x_off[j] + step * (kDepth * (unsigned)sizeof(X)), to + j * 1024);
#pragma unroll
            for (int j = 0; j < kW; ++j) load_lds(a_buffer, none ? kNowhere : w_off[j] + step * (kDepth * 2u), to + (kX + j) * 1024);
        };
        f32x4 sum[NT][NR];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < NR; ++r) sum[n][r] = (f32x4)0.0f;
#pragma unroll
        for (int s = 0; s < kSlots; ++s) ask(wave + s * kDownWaves);
        for (int i = wave; i < share.length; i += kDownWaves) {
            loads_but<(kSlots - 1) * kLoads>();
            const int8_t *const from = own + i / kDownWaves % kSlots * kSlot;
            Piece<X> x[NT];
            Piece<_Float16> w[NR];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int row = n * 16 + lane % 16;
#pragma unroll
                for (int c = 0; c < (int)sizeof(X); ++c) {
                    const i32x4 v = *(const i32x4 *)(from + (row * kChunks + place_in_row<kChunks>(lane / 16 * (int)sizeof(X) + c, row)) * 16);
#pragma unroll
                    for (int d = 0; d < 4; ++d) x[n].p.w[4 * c + d] = v[d];
                }
            }
#pragma unroll
            for (int r = 0; r < NR; ++r) {
                const int row = r * 16 + lane % 16;
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const i32x4 v = *(const i32x4 *)(from + kX * 1024 + (row * 8 + place_in_row<8>(lane / 16 * 2 + c, row)) * 16);
#pragma unroll
                    for (int d = 0; d < 4; ++d) w[r].p.w[4 * c + d] = v[d];
                }
            }
            if (share.step(i) * kDepth + kDepth > a.k) {           // (what lies behind a row's end is the next row's)
                const int at = share.step(i) * kDepth + lane / 16 * 16;
                keep(x, 0, a.k - 1 - at);
                keep(w, 0, a.k - 1 - at);
            }
            multiply<X, NT, NR>(sum, x, w);
            loads_but<63>();                                       // (the reads of this slot are done)
            ask(i + kSlots * kDownWaves);
        }
        loads_but<0>();
        __syncthreads();
        join<NT, NR>(a, (f32x4(*)[NT * NR][64])ring, sum, tokens, sub, tile.count, share.split, share.chunk);
    }
}

// ---------------------------------------------------------------------------------------------
// y of a tile of up to 64 tokens, in strips of 16 N channels to each of four wavefronts.  First the block adds up t (of all its
// parts) and puts it into LDS as two FP16 numbers to a value: t 2^-e to 11 bits and the rest to 11 more, 2^e the power of two that
// brings the row's greatest into [2^14, 2^15), so that nothing overflows and 22 bits of each are kept, or 2^-39 of the greatest.  (FP16
// products cost a quarter of the matrix cores' time that binary32 ones take.)  Then a wavefront has tokens for the rows of its products and
// channels for the columns, the N products' columns N apart: lane l has N neighbouring channels of four tokens, and the 16 lanes of a token
// have neighbouring ones, so a load or store is of runs of 32 N bytes.  (8192 x 8192 FP16 by 64 ranks: 69 us, 3.9 TB/s; 80 with lanes of one
// instruction in 16 rows, 16 bytes each, whose addresses are looked up one by one.  Eight channels to a lane: as four.)
//
// Infinities.  One among a token's t has 0 for its second number, and e goes by the others.  In b one times 0 - t's second number where the first is all
// of it, or a place of no rank - would be NaN where the formula has an infinity: a wavefront that finds one in its vectors of b (it looks once a strip,
// which costs 0 to 3 % of a call) leaves that strip to plain_strip.  A NaN does no harm: y of its channel is NaN in any case.
constexpr int kUpWaves = kBlock / 64;

// Adds 0 times all values of v, which is NaN where one is not finite.
template <int N> __device__ __forceinline__ void look_at(f16x2 &wild, const Words<_Float16, 8> (&v)[N])
{
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) wild = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (int)v[c].w[w]), (f16x2)(_Float16)0.0f, wild);
}

template <int N> __device__ __forceinline__ bool has_infinity(const Words<_Float16, 8> (&v)[N])
{
    bool some = false;
#pragma unroll
    for (int c = 0; c < N; ++c)
#pragma unroll
        for (int w = 0; w < 4; ++w) some |= (v[c].w[w] & 0x7FFF) == 0x7C00 || (v[c].w[w] >> 16 & 0x7FFF) == 0x7C00;
    return some;
}

__device__ __forceinline__ f32x4 product(f16x8 t, f16x8 b, f32x4 sum) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(t, b, sum, 0, 0, 0); }

// Stores N neighbouring channels.  Where a row ends within them they begin N before its end (see begin_of); those of them that are
// others' are left to those.
template <typename T, int N> __device__ __forceinline__ void store_channels(T *row, int at, int n, const typename Words<T, N>::V &v)
{
    if (at + N <= n) {
        __builtin_memcpy((FQ_GLOBAL T *)(row + at), &v, sizeof v);
        return;
    }
    const int begin = begin_of(at, N, n);
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (begin + e >= at && begin + e < n) st_global(row + begin + e, v[e]);
}

// Where rank l of t lies in LDS, so that eight places are the ranks of one vector of b (which begins eight before the end of a row where it
// would go over it): the last ranks at the end of their vector, what would be before them behind it.  (Places of no rank hold zeros.)
__device__ __forceinline__ int place_of_rank(int l, int rank)
{
    const int last = rank / 8 * 8, off = rank % 8;
    if (rank < 8 || off == 0 || l < last) return l;
    return l < rank ? l + 8 - off : l < last + 8 ? l - off : l;
}

// y's kernel takes t in units of four ranks, eight lanes to a token: unit u, u + 8, ... to lane u.  J units of a lane, of all parts, several
// loads on their way at a time.
template <int J> __device__ __forceinline__ void sum_of_parts(f32x4 (&s)[J], const AdapterArgs &a, const float *t, int unit)
{
    constexpr int P = J == 2 ? 2 : 8 / J;
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

// Rows of b of fewer than eight ranks, that of channel c in the first places and zeros behind it: they lie one behind the other, so a whole vector
// from there on has it, or at the end of the adapter's one that begins up to seven values before.  (By single values, us: 27 tokens, 7953 channels
// and 4 ranks 17.4, so 10.6; 3818 x 2501 x 7056 with 4 ranks 77, so 51 to 55.)
__device__ __forceinline__ void short_row(Words<_Float16, 8> &to, const _Float16 *b, int c, int n, int rank, bool some)
{
    const int at = c * rank, from = min(at, n * rank - 8), off = (at - from) * 16;
    __builtin_memcpy(&to, (const FQ_GLOBAL _Float16 *)(b + from), sizeof to);
    const auto v = __builtin_bit_cast(u64x2, to.w);
    const uint64_t high = off < 64 ? v[1] >> off : 0, low = off < 64 ? v[0] >> off | (v[1] << 1) << (63 - off) : v[1] >> (off - 64);
    const int bits = some ? rank * 16 : 0;
    const uint64_t keep_low = bits >= 64 ? ~0ull : (1ull << bits) - 1, keep_high = bits > 64 ? (1ull << (bits - 64)) - 1 : 0;
    to.w = __builtin_bit_cast(typename Words<_Float16, 8>::W, u64x2{low & keep_low, high & keep_high});
}

// A value that the compiler takes for another at each use.  (What follows from it is then worked out where it is needed: the addresses of all
// rows of a tile, kept over its strips, would take 64 registers.)
__device__ __forceinline__ int anew(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// Values from a row of t in LDS to the next: whole 32 ranks, and eight more so that rows begin in different banks.
__host__ __device__ constexpr int row_of_t(int rank) { return (rank + 31) / 32 * 32 + 8; }

// scale xs 2^-e of a token: a number, and a power of two that its finished sums are multiplied by.  By itself the product may be beyond binary32's range
// where y is not (t of 2^-120 and b of 2^15); as a rule it is well within, and the power is 2^0.  Tiles with another go to plain_strip (to multiply all
// sums by a power made 8192^3 by 64 ranks 2 % slower).
struct Factors {
    float number[kWindow];
    int power[kWindow];
};

__device__ __forceinline__ void set_factor(Factors &to, int i, float scale, float xs, int e)
{
    float number = scale * xs;
    const bool fits = __builtin_isnormal(number);
    number = __builtin_ldexpf(number, -e);
    int power = 0;
    if (__builtin_expect(!fits || !__builtin_isnormal(number), 0)) {
        number = __builtin_amdgcn_frexp_mantf(scale) * __builtin_amdgcn_frexp_mantf(xs);
        power = __builtin_amdgcn_frexp_expf(scale) + __builtin_amdgcn_frexp_expf(xs) - e;
        if (power >= -100 && power <= 100) {
            number = __builtin_ldexpf(number, power);
            power = 0;
        }
    }
    to.number[i] = number;
    to.power[i] = power;
}

// The greatest of the eight lanes that have a token's t, none of them negative or NaN.
__device__ __forceinline__ float most_of_token(float most)
{
    unsigned v = __builtin_bit_cast(unsigned, most);
    v = dpp_max<0xB1, 0xf>(v);
    v = dpp_max<0x4E, 0xf>(v);
    return __builtin_bit_cast(float, dpp_max<0x141, 0xf>(v));
}

// y of a strip by sums of binary32 products, one channel after the other: of the lane's N from `first` on, as elsewhere.  (Slow, but rare and
// out of the way: by matrix instructions with masked vectors the kernel took 10 to 120 registers more.)
template <typename Y, typename B, int N, int TT>
__device__ __forceinline__ void plain_strip(const AdapterArgs &a, int id, const _Float16 *heads, int row, const Factors &factors, const int *tokens, int count,
                                            int first)
{
    const _Float16 *const rests = heads + TT * 16 * row, *const b = (const _Float16 *)a.b + (long long)id * a.n * a.rank;
#pragma unroll 1
    for (int i = 0; i < TT * 4 * N; ++i) {
        const int token = i / (4 * N) * 16 + (threadIdx.x & 63) / 16 * 4 + i / N % 4, c = first + i % N;
        if (token >= count || c >= a.n) continue;
        float sum = 0.0f;
#pragma unroll 4
        for (int l = 0; l < a.rank; ++l) {
            const int at = token * row + place_of_rank(l, a.rank);
            sum += ((float)heads[at] + (float)rests[at]) * (float)ld_global(b + (long long)c * a.rank + l);
        }
        const float v = a.no_base ? 0.0f : (float)ld_global((const B *)a.base + tokens[token] * a.ldbase + c);
        st_global((Y *)a.y + tokens[token] * a.ldy + c, (Y)(v + __builtin_ldexpf(factors.number[token] * sum, factors.power[token])));
    }
}

// TT: tokens of a tile in 16s, at most; J: of t's units, 32 J ranks at most; SHORT: rows of b, fewer than eight ranks; FEW: channels, fewer
// than N, or values of b of an adapter, fewer than eight.  Wavefronts to a SIMD: as many as leave each its registers (32 tokens with an FP32 base, whose two
// tiles are 32 of them: 2048 x 4096 x 4096 by 16 ranks 27.4 us with three, 29.6 with four).
template <typename Y, typename B, int N, int TT, int J, bool FEW, bool SHORT>
__global__ __launch_bounds__(kBlock, J == 8 || (J == 4 && N == 4) ? 2 : J == 4 ? 3 : N == 2 || (J == 1 && (TT == 1 || sizeof(B) == 2)) ? 4 : 3) void adapter_up_kernel(AdapterArgs a)
{
    constexpr int kHeld = J == 8 ? 1 : J;                             // vectors of b of a channel that are held: all, or one at a time
    constexpr int kAhead = TT > 1 ? 2 : 1;                            // tokens' tiles whose base is held
    extern __shared__ __attribute__((aligned(16))) _Float16 shared[];          // [2][tile][row]
    __shared__ Finding finding;
    __shared__ Factors factors;
    const int *tokens = finding.tokens;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int index = (int)(blockIdx.x / a.groups);
    const Tile tile = a.way == kSorting ? left_tile(a, index, finding) : find_tile(a, index, finding);
    const int deep = (a.rank + 31) / 32, row = row_of_t(a.rank), most_tokens = TT * 16;
    const bool copy = tile.id < 0;
    if (copy && a.base == a.y && !a.no_base) return;
    for (int sub = 0; sub < tile.count; sub += most_tokens) {
        const int count = min(tile.count - sub, most_tokens);
        int strip = (int)(blockIdx.x % a.groups) * kUpWaves + wave;
        const auto first_of = [&](int of) { return of * 16 * N + lane % 16 * N; };
        Words<_Float16, 8> b[kHeld][N];
        const auto channel = [&](int c, int of) {
            return (const _Float16 *)a.b + ((long long)tile.id * a.n + begin_of(first_of(of), N, a.n) + (FEW ? min(c, a.n - 1) : c)) * a.rank;
        };
        const auto ask_b = [&](int of) {
#pragma unroll
            for (int c = 0; c < N; ++c) {
                if constexpr (SHORT && !FEW) {
                    short_row(b[0][c], (const _Float16 *)a.b + (long long)tile.id * a.n * a.rank, begin_of(first_of(of), N, a.n) + c, a.n, a.rank, lane < 16);
                } else {
                    const _Float16 *from = channel(c, of);
#pragma unroll
                    for (int d = 0; d < kHeld; ++d) load<SHORT>(b[d][c], from, begin_of(d * 32 + lane / 16 * 8, 8, a.rank), a.rank);
                }
            }
        };
        Words<B, N> base[kAhead][4];
        const auto ask_base = [&](int n, int of) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const B *from = (const B *)a.base + tokens[anew(sub + min(n * 16 + lane / 16 * 4 + i, count - 1))] * a.ldbase;
                load<FEW>(base[n % kAhead][i], from, begin_of(first_of(of), N, a.n), a.n);
            }
        };
        // (J == 8: vectors of b come one after the other, each for all tokens of the tile while the next is on its way)
        Words<_Float16, 8> odd[kHeld][N];
        const auto ask_deep = [&](Words<_Float16, 8> (&to)[N], int d, int of) {
#pragma unroll
            for (int c = 0; c < N; ++c) load<SHORT>(to[c], channel(c, of), begin_of(min(d, deep - 1) * 32 + lane / 16 * 8, 8, a.rank), a.rank);
        };
        // (strips behind the last clamp to the end of the row: loads of what is left unused)
        if (!copy && J < 8) ask_b(strip);
        ask_base(0, strip);
        if (J == 8) {
            if (TT == 2) ask_base(1, strip);
            if (!copy) ask_deep(b[0], 0, strip);
        }
        if (!copy) {
            const int unit = threadIdx.x % 8;
            for (int i = threadIdx.x / 8; i < most_tokens; i += kBlock / 8) {
                const int token = tokens[sub + min(i, count - 1)];
                const float scale = a.scale ? ld_global(a.scale + tile.id) : 1.0f, xs = a.xs ? ld_global(a.xs + (long long)token * a.xs_step) : 1.0f;
                f32x4 s[J];
                sum_of_parts<J>(s, a, a.t + (long long)token * a.pitch, unit);
                float most = 0.0f;
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = __builtin_fmaxf(most, __builtin_fabsf(s[j][e]));
                most = most_of_token(most);
                if (__builtin_expect(most == __builtin_inff(), 0)) {            // (of all eight lanes of a token, or of none)
                    most = 0.0f;
#pragma unroll
                    for (int j = 0; j < J; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float size = __builtin_fabsf(s[j][e]);
                            most = __builtin_fmaxf(most, size < __builtin_inff() ? size : 0.0f);
                        }
                    most = most_of_token(most);
                }
                const int e2 = most > 0.0f ? 15 - __builtin_amdgcn_frexp_expf(most) : 0;
                _Float16 *const heads = shared + i * row, *const rests = heads + most_tokens * row;
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
                if (unit == 0) set_factor(factors, i, scale, xs, e2);
            }
        }
        __syncthreads();
        while (strip * 16 * N < a.n) {
            const int after = strip + a.groups * kUpWaves;
            f16x2 wild = (f16x2)(_Float16)0.0f;
            bool matrix = true;                                           // whether the matrix instructions make the y of this strip
            f32x4 sums[J == 8 ? TT : 1][N];
            if (J == 8) {
#pragma unroll
                for (int n = 0; n < TT; ++n)
#pragma unroll
                    for (int c = 0; c < N; ++c) sums[n][c] = (f32x4)0.0f;
                if (!copy) {
                    const auto multiply_all = [&](const Words<_Float16, 8> (&by)[N], int d) {
                        look_at(wild, by);
#pragma unroll
                        for (int n = 0; n < TT; ++n) {
                            const _Float16 *t = shared + (n * 16 + lane % 16) * row + lane / 16 * 8 + d * 32;
                            const f16x8 high = *(const f16x8 *)t, low = *(const f16x8 *)(t + most_tokens * row);
#pragma unroll
                            for (int c = 0; c < N; ++c) sums[n][c] = product(low, by[c].values(), product(high, by[c].values(), sums[n][c]));
                        }
                    };
                    for (int d = 0; d < deep; d += 2) {
                        ask_deep(odd[0], d + 1, strip);
                        multiply_all(b[0], d);
                        ask_deep(b[0], d + 2, strip);
                        if (d + 1 < deep) multiply_all(odd[0], d + 1);
                    }
                    ask_deep(b[0], 0, after);
                }
            }
#pragma unroll
            for (int n = 0; n < TT; ++n) {
                if (TT > 1 && J < 8) {
                    if (n + 1 < TT) ask_base(n + 1, strip);
                    else ask_base(0, after);
                }
                f32x4 sum[N];
#pragma unroll
                for (int c = 0; c < N; ++c) sum[c] = J == 8 ? sums[J == 8 ? n : 0][c] : (f32x4)0.0f;
                if (!copy && J < 8) {
                    const _Float16 *t = shared + (n * 16 + lane % 16) * row + lane / 16 * 8;
#pragma unroll
                    for (int d = 0; d < kHeld; ++d) {
                        if (d >= deep) continue;
                        const f16x8 high = *(const f16x8 *)(t + d * 32), low = *(const f16x8 *)(t + d * 32 + most_tokens * row);
#pragma unroll
                        for (int c = 0; c < N; ++c) sum[c] = product(low, b[d][c].values(), product(high, b[d][c].values(), sum[c]));
                    }
                }
                if (n == 0) {
                    if (!copy && J < 8) {
#pragma unroll
                        for (int d = 0; d < kHeld; ++d) look_at(wild, b[d]);
                    }
                    const int power = copy ? 0 : factors.power[lane % most_tokens];
                    if (__builtin_expect(__ballot(wild[0] != 0 || wild[1] != 0 || power != 0) != 0, 0)) {
                        bool some = J == 8 || power != 0;                     // (the vectors of J == 8 are no longer there)
                        if (J < 8) {
#pragma unroll
                            for (int d = 0; d < kHeld; ++d) some |= has_infinity(b[d]);
                        }
                        if (__ballot(some)) matrix = false;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int token = n * 16 + lane / 16 * 4 + i;
                    const float f = copy ? 0.0f : factors.number[token];
                    const auto from = base[n % kAhead][i].values();
                    typename Words<Y, N>::V y;
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const float v = a.no_base ? 0.0f : (float)from[e];
                        y[e] = (Y)(copy ? v : v + f * sum[e][i]);
                    }
                    if (token < count && matrix) store_channels<Y, N>((Y *)a.y + tokens[anew(sub + token)] * a.ldy, first_of(strip), a.n, y);
                }
                if (TT == 1 || J == 8) ask_base(n, after);
            }
            if (__builtin_expect(!matrix, 0)) {
                plain_strip<Y, B, N, TT>(a, tile.id, shared, row, factors, tokens + sub, count, first_of(strip));
#pragma unroll
                for (int n = 0; n < kAhead; ++n)
                    if (n == 0 || J == 8) ask_base(n, after);
            }
            strip = after;
            if (!copy && J < 8) ask_b(strip);
        }
        __syncthreads();
    }
}

template <typename X, int NT, int NR> void ring_by(const AdapterArgs &a, unsigned blocks, hipStream_t stream)
{
    adapter_down_ring_kernel<X, NT, NR><<<blocks, kBlock, kDownWaves * ring_slots<X, NT, NR>() * ring_slot<X, NT, NR>(), stream>>>(a);
}

template <typename X> int down(const AdapterArgs &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)a.tiles_most * (unsigned)a.splits * (unsigned)a.chunks;
    const int shape = (a.x_bytes ? 100 : 0) + a.token_tiles * 10 + a.rank_tiles;
    if (a.k < 16) adapter_down_kernel<X, 1, 1, true><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 11) adapter_down_kernel<X, 1, 1, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 12) adapter_down_kernel<X, 1, 2, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 14) adapter_down_kernel<X, 1, 4, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 21) adapter_down_kernel<X, 2, 1, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 22) adapter_down_kernel<X, 2, 2, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 24) adapter_down_kernel<X, 2, 4, false><<<blocks, kBlock, 0, stream>>>(a);
    else if (shape == 111) ring_by<X, 1, 1>(a, blocks, stream);
    else if (shape == 112) ring_by<X, 1, 2>(a, blocks, stream);
    else if (shape == 114) ring_by<X, 1, 4>(a, blocks, stream);
    else if (shape == 121) ring_by<X, 2, 1>(a, blocks, stream);
    else if (shape == 122) ring_by<X, 2, 2>(a, blocks, stream);
    else if (shape == 124) ring_by<X, 2, 4>(a, blocks, stream);
    else if constexpr (sizeof(X) == 4) return (int)hipErrorInvalidValue;
    else if (shape == 144) ring_by<X, 4, 4>(a, blocks, stream);
    else return (int)hipErrorInvalidValue;
    return (int)hipGetLastError();
}

template <typename Y, typename B, int N, int TT, int J, bool FEW, bool SHORT> void up_with(const AdapterArgs &a, hipStream_t stream)
{
    const size_t lds = (size_t)2 * 16 * TT * row_of_t(a.rank) * sizeof(_Float16);         // (what the kernel keeps goes by its own TT)
    adapter_up_kernel<Y, B, N, TT, J, FEW, SHORT><<<(unsigned)a.tiles_most * (unsigned)a.groups, kBlock, lds, stream>>>(a);
}

template <typename Y, typename B, int N, int TT> void up_by(const AdapterArgs &a, hipStream_t stream)
{
    if (a.rank < 8) up_with<Y, B, N, TT, 1, false, true>(a, stream);
    else if (a.rank <= 32) up_with<Y, B, N, TT, 1, false, false>(a, stream);
    else if (a.rank <= 64) up_with<Y, B, N, TT, 2, false, false>(a, stream);
    else if (a.rank <= 128) up_with<Y, B, N, TT, 4, false, false>(a, stream);
    else up_with<Y, B, N, TT, 8, false, false>(a, stream);
}

template <typename Y, typename B> void up(const AdapterArgs &a, hipStream_t stream)
{
    if (a.n < 2 || a.n * a.rank < 8) up_with<Y, B, 2, 1, 8, true, true>(a, stream);
    else if (a.wide == 2) up_by<Y, B, 2, 1>(a, stream);
    else if (a.token_tiles == 1) up_by<Y, B, 4, 1>(a, stream);
    else if (a.token_tiles == 2) up_by<Y, B, 4, 2>(a, stream);
    else up_with<Y, B, 4, 4, 2, false, false>(a, stream);
}

}  // namespace

int launch_adapters(const AdapterArgs &a, void *stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.count > 0) {
        if (a.way == kList) adapter_group_kernel<<<1, kGroupThreads, (size_t)(a.count + 1) * kGroupWaves * sizeof(int), s>>>(a);
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
