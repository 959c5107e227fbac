// Host side of layer norm, dropout and the adapters under sanitizers, from no tokens to the largest extents: launchers are stubs that check
// what they are given, where it lies in the workspace and how many threads it asks for.
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <initializer_list>

#include "../../include/fq.h"
#include "../../paper_2511_12653_amd/csrc/fq_adapters.h"
#include "../../paper_2511_12653_amd/csrc/fq_dropout.h"
#include "../../paper_2511_12653_amd/csrc/fq_norm.h"

static int failures = 0, launches = 0;
#define CHECK(c) do { if (!(c)) { ++failures; std::printf("%s:%d: %s (%lld %lld %lld, %lld by %lld)\n", __FILE__, __LINE__, #c, shown[0], shown[1], shown[2], shown[3], shown[4]); } } while (0)
static long long shown[5];

static char *ws_begin, *ws_end;
static long long tokens;                           // of the adapters' call so far
static void grid(unsigned long long threads) { CHECK(threads > 0 && threads < 1ull << 32); }
static void inside(const void *p, unsigned long long bytes)
{
    CHECK((const char *)p >= ws_begin && (const char *)p <= ws_end && bytes <= (unsigned long long)(ws_end - (const char *)p));
}
static long long ceiling(long long v, long long by) { return (v + by - 1) / by; }

namespace fq {

int launch_norm_forward(const NormArgs &a, void *)
{
    ++launches;
    CHECK(a.rows > 0 && a.width > 0 && a.blocks > 0);
    const long long held = (long long)a.lanes * a.vecs * 8;
    CHECK(a.width > kNormHeldWidth || a.width < 8 || a.width <= held);
    grid((unsigned long long)a.blocks * (unsigned)norm_threads(a.lanes));
    return 0;
}

int launch_norm_backward(const NormArgs &a, void *)
{
    ++launches;
    CHECK(a.width > 0);
    if (a.rows == 0) return 0;
    CHECK(a.blocks > 0);
    grid((unsigned long long)a.blocks * (unsigned)norm_threads(a.lanes));
    if (a.partial) {
        CHECK(a.parts > 0);
        if (a.parts > 1 || a.width > kNormHeldWidth) inside(a.partial, (unsigned long long)a.parts * 2 * (unsigned)a.width * 4);
        grid((unsigned long long)(a.width > kNormHeldWidth ? ceiling(a.width, kNormStrip) : 1) * (unsigned)a.parts * 512);
        grid((unsigned long long)ceiling(2LL * a.width, 16) * 256);
    } else {
        CHECK(!a.gw && !a.gb);
    }
    return 0;
}

int launch_dropout(const DropoutArgs &a, void *)
{
    ++launches;
    CHECK(a.n > 0 && a.n <= 1LL << 35 && a.threshold <= 1u << 31);
    return 0;
}

int launch_adapters(const AdapterArgs &a, void *)
{
    ++launches;
    CHECK(a.m > 0 && a.n > 0 && a.m <= kAdaptersMostTokens && a.groups > 0 && a.base);
    CHECK((a.token_tiles == 1 || a.token_tiles == 2 || (a.token_tiles == 4 && a.x_bytes && a.x_type != FQ_F32 && a.rank_tiles == 4)) && (a.wide == 2 || a.wide == 4));
    CHECK(a.wide == 2 || a.n >= 4);
    CHECK(a.token_tiles == 1 || a.wide == 4);
    grid((unsigned long long)a.tiles_most * (unsigned)a.groups * 256);
    tokens += a.m;
    if (a.count == 0) {
        CHECK(a.way == kWindows);
        return 0;
    }
    CHECK(a.splits > 0 && a.chunks * a.rank_tiles * 16 >= a.rank && a.pitch >= a.rank && a.pitch % 16 == 0);
    grid((unsigned long long)a.tiles_most * (unsigned)a.splits * (unsigned)a.chunks * 256);
    inside(a.t, (unsigned long long)a.splits * (unsigned)a.m * (unsigned)a.pitch * 4);
    CHECK((uintptr_t)a.t % 256 == 0);
    if (a.way == kList) {
        CHECK(a.count <= kMostGrouped);
        inside(a.order, (unsigned long long)a.m * 4);
        inside(a.tiles, (unsigned long long)a.tiles_most * sizeof(AdapterTile));
        CHECK((char *)a.order + (size_t)a.m * 4 <= (char *)a.tiles && (char *)a.tiles + (size_t)a.tiles_most * sizeof(AdapterTile) <= (char *)a.t);
        CHECK(a.tiles_most >= ceiling(a.m, 16 * a.token_tiles));
    } else {
        CHECK(a.way == kWindows ? a.tiles_most >= ceiling(a.m, kWindow) : a.m <= kSorted);
        if (a.way == kSorting) {
            const unsigned long long records = (unsigned long long)a.tiles_most * (unsigned)(2 + 16 * a.token_tiles) * 4;
            inside(a.found, records);
            CHECK((char *)a.found + records <= (char *)a.t);
        }
    }
    if (a.x_bytes) CHECK((unsigned long long)a.x_bytes >= (unsigned long long)(a.m - 1) * (unsigned long long)a.ldx && a.k >= 16 && (uintptr_t)a.x % 16 == 0);
    return 0;
}

}  // namespace fq

// Addresses that nothing touches, far enough from each other for every extent here.
static char *at(int i) { return (char *)(uintptr_t)((unsigned long long)i << 56); }

static unsigned long long state = 1;
static long long pick(long long most)
{
    state = state * 6364136223846793005ull + 1442695040888963407ull;
    const int bits = (int)((state >> 40) % 63);
    const unsigned long long r = (state >> 20) ^ (state << 37);
    return (long long)(r & ((1ull << bits) - 1)) % (most + 1);
}

static void norm(long long rows, long long width, int type)
{
    shown[0] = rows; shown[1] = width; shown[2] = type;
    if ((double)rows * (double)width * 8 > 7e16) return;                // (more than lies between two of the addresses)
    fq_norm d;
    std::memset(&d, 0, sizeof d);
    d.rows = rows; d.width = width; d.x_dtype = type & 1; d.y_dtype = type >> 1 & 1; d.w_dtype = type >> 2 & 1; d.eps = 1e-5f;
    d.ldx = d.ldy = d.ldgy = d.ldgx = width;
    d.x = at(1); d.y = at(2); d.stats = (float *)at(3); d.gy = at(4); d.gx = type & 8 ? nullptr : at(5); d.gweight = type & 16 ? nullptr : at(6); d.gbias = type & 32 ? nullptr : at(7);
    d.weight = at(8); d.bias = at(9);
    CHECK(fq_norm_forward(&d, nullptr) == FQ_OK);
    const size_t bytes = fq_norm_workspace_bytes(&d);
    CHECK(bytes > 0);
    ws_begin = at(10); ws_end = ws_begin + bytes;
    CHECK(fq_norm_backward(&d, ws_begin, bytes, nullptr) == FQ_OK);
    CHECK(fq_norm_backward(&d, ws_begin, bytes - 1, nullptr) == (width == 0 || rows == 0 || !(d.gweight || d.gbias) ? FQ_OK : FQ_ERR_WORKSPACE));
    d.y_dtype = FQ_I8; d.ys = (float *)at(11);
    CHECK(fq_norm_forward(&d, nullptr) == FQ_OK);
}

static void adapters(long long m, long long n, long long k, long long count, long long rank, int type)
{
    shown[0] = m; shown[1] = n; shown[2] = k; shown[3] = count; shown[4] = rank;
    fq_adapters d;
    std::memset(&d, 0, sizeof d);
    d.m = m; d.n = n; d.k = k; d.count = count; d.rank = rank;
    d.x_dtype = type % 3; d.y_dtype = type >> 2 & 1; d.base_dtype = type >> 3 & 1; d.xs_step = 1;
    d.ldx = k + (type >> 4 & 1); d.ldy = n; d.ldbase = n;
    d.x = at(1); d.xs = (float *)at(2); d.ids = (int32_t *)at(3); d.a = at(4) + (type >> 5 & 1) * 2; d.b = at(5); d.scale = (float *)at(6);
    d.base = type & 64 ? nullptr : at(7); d.y = at(8);
    const size_t bytes = fq_adapters_workspace_bytes(&d);
    CHECK(bytes > 0);
    ws_begin = at(9); ws_end = ws_begin + bytes;
    tokens = 0;
    CHECK(fq_adapters_forward(&d, ws_begin, bytes, nullptr) == FQ_OK);
    CHECK(tokens == (n == 0 ? 0 : m));
    CHECK(fq_adapters_forward(&d, ws_begin, bytes - 1, nullptr) == (m == 0 || n == 0 ? FQ_OK : FQ_ERR_WORKSPACE));
}

int main()
{
    for (long long rows : {0LL, 1LL, 2LL, 600LL, 70000LL, 1LL << 26, 1LL << 36})
        for (long long width : {0LL, 1LL, 7LL, 8LL, 128LL, 129LL, 4096LL, 16384LL, 16385LL, 65536LL, 1LL << 24})
            for (int type = 0; type < 64; type += 7) norm(rows, width, type);
    for (int i = 0; i < 4000; ++i) norm(pick(1LL << 36), pick(1LL << 24), (int)pick(63));
    for (long long n : {0LL, 1LL, 2048LL, 1LL << 34, 1LL << 35})
        for (double p : {0.0, 0.1, 1.0}) {
            fq_dropout_args d;
            std::memset(&d, 0, sizeof d);
            d.n = n; d.p = p; d.x = at(1); d.y = at(2); d.residual = at(3);
            CHECK(fq_dropout(&d, nullptr) == FQ_OK);
        }
    for (long long m : {0LL, 1LL, 16LL, 64LL, 65LL, 1024LL, 1025LL, 4096LL, 65536LL, 65537LL, 140001LL})
        for (long long n : {0LL, 1LL, 4LL, 1000LL, 1LL << 20})
            for (long long k : {0LL, 1LL, 16LL, 4096LL, 1LL << 20})
                for (long long count : {0LL, 1LL, 8LL, 1024LL, 1025LL, 1LL << 26})
                    for (long long rank : {0LL, 1LL, 16LL, 33LL, 64LL, 256LL}) adapters(m, n, k, count, rank, (int)pick(127));
    for (int i = 0; i < 20000; ++i) adapters(pick(1000000), pick(1LL << 20), pick(1LL << 20), pick(100000), pick(256), (int)pick(127));
    adapters(0x7fffff00LL, 1, 16, 1024, 256, 0);
    std::printf("more operators: %d failures, %d launches\n", failures, launches);
    return failures != 0;
}
