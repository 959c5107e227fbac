// Host side of the int8 linear layer and of the AdamW step under sanitizers: launchers are stubs that check what they are given.
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <vector>

#include "../../include/fq.h"
#include "../../paper_2511_12653_amd/csrc/fq_adamw.h"
#include "../../paper_2511_12653_amd/csrc/fq_internal.h"
#include "../../paper_2511_12653_amd/csrc/fq_linear.h"

static int failures = 0;
#define CHECK(c) do { if (!(c)) { ++failures; std::printf("%s:%d: %s\n", __FILE__, __LINE__, #c); } } while (0)

static std::vector<char> table;                    // what the last create copied
static const void *table_at;
static char *ws_begin, *ws_end;
static int launches;

static bool inside(const void *p, size_t bytes) { return (const char *)p >= ws_begin && (const char *)p + bytes <= ws_end; }

namespace fq {

int copy_table_async(void *dst, const void *src, size_t bytes, void *)
{
    CHECK(inside(dst, bytes));
    table.assign((const char *)src, (const char *)src + bytes);
    table_at = dst;
    return 0;
}

int launch_adamw(const AdamwTensor *t, const unsigned *first, int n, const AdamwStep &s, unsigned blocks, int rows, void *)
{
    ++launches;
    CHECK(t == table_at && blocks > 0 && (rows == 1 || rows == 2) && s.beta1 >= 0 && std::isfinite(s.root_factor));
    const AdamwTensor *host = (const AdamwTensor *)table.data();
    const long long per = (long long)kAdamwRowElems * rows;
    if (!first) {                                  // a descriptor per block: block b works on elements (b - first) * per of its tensor
        CHECK(rows == 1 && blocks * sizeof(AdamwTensor) <= table.size());
        for (unsigned b = 0; b < blocks; ++b)
            CHECK(host[b].first <= b && (long long)(b - host[b].first) * per < host[b].n);
        return 0;
    }
    CHECK((const char *)first >= (const char *)table_at + (size_t)n * sizeof(AdamwTensor));
    const unsigned *f = (const unsigned *)(table.data() + ((const char *)first - (const char *)table_at));
    CHECK((const char *)(f + n) <= table.data() + table.size());
    long long block = 0, place = 0;
    for (int i = 0; i < n; ++i) {
        CHECK(f[i] == (unsigned)block && host[i].first == f[i] && host[i].place == (unsigned)place);
        block += (host[i].n + per - 1) / per;
        place += (host[i].n + 255) / 256 * 256;
    }
    CHECK(block == (long long)blocks);
    return 0;
}

bool linear_few(const LinearArgs &a, int size) { return a.k > 0 && a.m <= 16 && (long long)a.m * a.k * size < 40000; }
bool linear_rows(const LinearArgs &a) { return a.k >= 16 && a.k <= 512 && a.m >= 1024; }
bool linear_rows_as_they_lie(const LinearArgs &a) { return ((uintptr_t)a.w | (uintptr_t)a.ldw) % 4 == 0; }

static void check_aligned(const AlignArgs &a)
{
    CHECK(a.pitch % 128 == 0 && a.pitch >= a.k && a.ld >= a.k && a.rows > 0 && inside(a.to, (size_t)a.rows * (size_t)a.pitch));
}

int launch_quantize_rows(const QuantizeArgs &a, const AlignArgs &other, void *)
{
    ++launches;
    CHECK(a.pitch % 128 == 0 && a.pitch >= a.k && inside(a.q, (size_t)a.m * (size_t)a.pitch) && inside(a.s, (size_t)a.m * 4));
    CHECK((char *)a.s >= (char *)a.q + (size_t)a.m * (size_t)a.pitch);
    if (other.rows) {
        check_aligned(other);
        CHECK((char *)other.to >= (char *)(a.s + a.m));
    }
    return 0;
}

int launch_align_rows(const AlignArgs &a, const AlignArgs &other, void *)
{
    ++launches;
    CHECK(a.rows || other.rows);
    if (a.rows) check_aligned(a);
    if (other.rows) check_aligned(other);
    if (a.rows && other.rows) CHECK((char *)other.to >= (char *)a.to + (size_t)a.rows * (size_t)a.pitch);
    return 0;
}

int launch_linear(const LinearArgs &a, void *)
{
    ++launches;
    CHECK(a.m > 0 && a.n > 0 && a.y && (a.raw || a.k == 0 || a.x) && (a.raw || a.xs));
    if (a.raw && linear_few(a, a.x16 ? 2 : 4)) return 0;
    if (!a.raw && linear_few(a, 1)) return 0;
    if (a.raw && linear_rows(a) && linear_rows_as_they_lie(a)) return 0;       // reads inside the rows of w
    // the tiles read whole 16 bytes of rows on 16-byte boundaries
    if (a.k > 0) CHECK((uintptr_t)a.w % 16 == 0 && a.ldw % 16 == 0 && a.kw % 16 == 0 && a.kw >= a.k && a.kw <= a.ldw && a.ldw <= kMostPitch);
    if (a.k > 0 && !a.raw) CHECK((uintptr_t)a.x % 16 == 0 && a.ldx % 16 == 0 && a.kx % 16 == 0 && a.kx >= a.k && a.kx <= a.ldx && a.ldx <= kMostPitch);
    return 0;
}

}  // namespace fq

static unsigned long long seed = 88172645463325252ull;
static unsigned next_random() { seed ^= seed << 13; seed ^= seed >> 7; seed ^= seed << 17; return (unsigned)(seed >> 16); }
static long long pick(long long lo, long long hi) { return lo + (long long)(next_random() % (unsigned long long)(hi - lo + 1)); }

static void linear()
{
    CHECK(fq_linear_workspace_bytes(nullptr) == 0 && fq_linear_forward(nullptr, nullptr, 0, nullptr) == FQ_ERR_NULL);
    const long long edges[] = {LLONG_MIN, -1, 0, 1, 15, 16, 131071, 131072, 1LL << 31, 1LL << 40, LLONG_MAX};
    for (long long m : edges)
        for (long long n : edges)
            for (long long k : edges)
                for (long long ld : edges) {
                    fq_linear d;
                    std::memset(&d, 0, sizeof d);
                    d.m = m; d.n = n; d.k = k; d.ldx = d.ldw = d.ldy = ld; d.x_dtype = (int)(next_random() % 3); d.y_dtype = (int)(next_random() % 2);
                    d.x = (void *)(1LL << 30); d.w = (int8_t *)(1LL << 32); d.ws = (float *)(1LL << 20); d.xs = (float *)(1LL << 21); d.y = (void *)(1LL << 62);
                    (void)fq_linear_workspace_bytes(&d);
                }
    for (int i = 0; i < 20000; ++i) {
        fq_linear d;
        std::memset(&d, 0, sizeof d);
        d.m = pick(0, 40) * (next_random() % 8 ? 1 : 60); d.n = pick(0, 300); d.k = pick(0, 3) ? pick(0, 700) : 16 * pick(0, 60);
        d.x_dtype = (int)(next_random() % 3); d.y_dtype = (int)(next_random() % 2);
        d.ldx = d.k + (next_random() % 2 ? 0 : pick(0, 40)); d.ldw = d.k + (next_random() % 2 ? 0 : pick(0, 40)); d.ldy = d.n + pick(0, 5);
        const int size = d.x_dtype == FQ_I8 ? 1 : d.x_dtype == FQ_F16 ? 2 : 4;
        d.x = (char *)(1LL << 40) + size * pick(0, 20); d.w = (int8_t *)(1LL << 41) + pick(0, 20); d.y = (char *)(1LL << 42) + 4 * pick(0, 9);
        d.ws = (float *)(1LL << 43); d.xs = (float *)(1LL << 44); d.xs_step = (int)(next_random() % 2); d.ws_step = (int)(next_random() % 2);
        const size_t bytes = fq_linear_workspace_bytes(&d);
        CHECK(bytes >= 256 && bytes % 256 == 0);
        ws_begin = (char *)(1LL << 45);
        ws_end = ws_begin + bytes;
        launches = 0;
        CHECK(fq_linear_forward(&d, ws_begin, bytes, nullptr) == FQ_OK);
        CHECK(launches <= 3 && (launches > 0) == (d.m > 0 && d.n > 0));
    }
}

static void adamw()
{
    for (int turn = 0; turn < 300; ++turn) {
        std::vector<fq_param> ps((size_t)pick(0, turn % 10 == 0 ? 3000 : 40));
        uintptr_t at = 1ull << 40;
        auto room = [&](size_t bytes) { const uintptr_t p = at; at += (bytes + 63) / 64 * 64 + 64; return (void *)p; };
        for (fq_param &p : ps) {
            std::memset(&p, 0, sizeof p);
            p.n = pick(0, 3) ? pick(0, 3000) : pick(0, 2000000);
            p.p_dtype = (int)(next_random() % 2); p.g_dtype = (int)(next_random() % 2); p.state = (int)(next_random() % 2); p.lr_scale = 1.0f;
            const size_t n = (size_t)p.n;
            p.p = room(4 * n); p.g = room(4 * n); p.m = room(4 * n); p.v = room(4 * n);
            if (p.state == FQ_STATE_F8) { p.m_scale = (float *)room(n); p.v_scale = (float *)room(n); }
            if (p.p_dtype == FQ_F32 && next_random() % 2) p.p16 = room(2 * n);
        }
        const int n = (int)ps.size();
        const size_t bytes = fq_adamw_workspace_bytes(ps.data(), n);
        CHECK(bytes >= 256 && bytes % 256 == 0);
        ws_begin = (char *)(1LL << 45);
        ws_end = ws_begin + bytes;
        fq_adamw_plan *plan = nullptr;
        CHECK(fq_adamw_create(ps.data(), n, ws_begin, bytes, nullptr, &plan) == FQ_OK && plan);
        fq_adamw h = {1e-3, 0.9, 0.999, 1e-8, 1 + turn, 7, nullptr};
        CHECK(fq_adamw_step(plan, &h, nullptr) == FQ_OK);
        h.step = 0;
        CHECK(fq_adamw_step(plan, &h, nullptr) == FQ_ERR_OPTIMIZER);
        fq_adamw_destroy(plan);
    }
    const long long edges[] = {LLONG_MIN, -1, 1LL << 40, (1LL << 40) + 1, LLONG_MAX};
    for (long long n : edges) {
        fq_param p;
        std::memset(&p, 0, sizeof p);
        p.n = n; p.lr_scale = 1.0f; p.p = (void *)64; p.g = (void *)(1LL << 43); p.m = (void *)(1LL << 44); p.v = (void *)(1LL << 45);
        std::vector<fq_param> many(5000, p);
        (void)fq_adamw_workspace_bytes(&p, 1);
        CHECK(fq_adamw_workspace_bytes(many.data(), 5000) == 0);       // too many blocks, or a size that is refused
    }
    fq_adamw_destroy(nullptr);
}

int main()
{
    linear();
    adamw();
    std::printf("operators' host side: %d failures\n", failures);
    return failures != 0;
}
