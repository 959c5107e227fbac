// Extents of the int8 linear layer at which a launch would have more threads than a grid may (2^32 along x): launchers are stubs
// that count the threads of what they are given, and which part of y it is.
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "../../include/fq.h"
#include "../../paper_2511_12653_amd/csrc/fq_linear.h"

static int failures = 0;
#define CHECK(c) do { if (!(c)) { ++failures; std::printf("%s:%d: %s\n", __FILE__, __LINE__, #c); } } while (0)

static const fq_linear *given;
static char *ws_begin, *ws_end;
static double covered;                             // elements of y so far
static int few;                                    // 1: up to 16 tokens go to the kernel of few

static void grid(unsigned long long threads) { CHECK(threads > 0 && threads < 1ull << 32); }
static unsigned long long layout(const fq::AlignArgs &a)
{
    if (!a.rows) return 0;
    CHECK((char *)a.to >= ws_begin && (char *)a.to + (size_t)a.rows * (size_t)a.pitch <= ws_end);
    return ((unsigned long long)a.rows * (unsigned long long)a.pitch / 16 + 255) / 256 * 256;
}

namespace fq {

bool linear_few(const LinearArgs &a, int) { return few && a.k > 0 && a.m <= 16; }
bool linear_rows(const LinearArgs &) { return false; }
bool linear_rows_as_they_lie(const LinearArgs &) { return false; }

int launch_quantize_rows(const QuantizeArgs &a, const AlignArgs &other, void *)
{
    CHECK((char *)a.q >= ws_begin && (char *)(a.s + a.m) <= ws_end);
    grid((unsigned long long)a.m * 256 + layout(other));
    return 0;
}

int launch_align_rows(const AlignArgs &a, const AlignArgs &other, void *)
{
    grid(layout(a) + layout(other));
    return 0;
}

int launch_linear(const LinearArgs &a, void *)
{
    const fq_linear &d = *given;
    const size_t size = d.y_dtype == FQ_F16 ? 2 : 4, off = (size_t)((char *)a.y - (char *)d.y) / size;
    const long long row = (long long)(off / (size_t)d.ldy), column = (long long)(off % (size_t)d.ldy);
    CHECK(a.m > 0 && a.n > 0 && row + a.m <= d.m && column + a.n <= d.n);
    CHECK(a.ws == d.ws + column * d.ws_step && a.bias == (d.bias ? d.bias + column : nullptr));
    if ((char *)a.w < ws_begin || (char *)a.w >= ws_end) CHECK(a.w == d.w + column * d.ldw);
    if (d.x_dtype == FQ_I8) CHECK(a.xs == d.xs + row * d.xs_step);
    if (a.raw) CHECK(a.raw == (const char *)d.x + row * d.ldx * (d.x_dtype == FQ_F16 ? 2 : 4));
    if (few && a.k > 0 && a.m <= 16) grid(((unsigned long long)a.n + 15) / 16 * 512);
    covered += (double)a.m * (double)a.n;
    return 0;
}

}  // namespace fq

static void run(long long m, long long n, long long k, int x_dtype, int off, int bias)
{
    for (few = 0; few < 2; ++few) {
        fq_linear d;
        std::memset(&d, 0, sizeof d);
        d.m = m; d.n = n; d.k = k; d.ldx = k + off; d.ldw = k + off; d.ldy = n + off;
        d.x_dtype = x_dtype; d.y_dtype = FQ_F16; d.ws_step = 1; d.xs_step = 1;
        d.x = (char *)(1LL << 50) + 4 * off; d.w = (int8_t *)(1LL << 51) + off; d.y = (void *)(1LL << 52);
        d.ws = (float *)(1LL << 49); d.xs = (float *)(1LL << 48);
        if (bias) d.bias = (float *)(1LL << 47);
        given = &d;
        const size_t bytes = fq_linear_workspace_bytes(&d);
        CHECK(bytes >= 256);
        ws_begin = (char *)(1LL << 53);
        ws_end = ws_begin + bytes;
        covered = 0;
        std::printf("m %lld n %lld k %lld x %d off %d few %d\n", m, n, k, x_dtype, off, few);
        CHECK(fq_linear_forward(&d, ws_begin, bytes, nullptr) == FQ_OK);
        CHECK(covered == (double)m * (double)n);
    }
}

int main()
{
    const long long most = 0x7fffff00LL;
    for (int x_dtype : {FQ_F16, FQ_F32, FQ_I8})
        for (int off : {0, 1}) {
            const int bias = off ^ (x_dtype == FQ_I8);
            for (long long n : {(1LL << 26) - 1, 1LL << 26, 1LL << 27, (1LL << 27) + 5, 1LL << 29, most})
                for (long long k : {5LL, 16LL, 200LL}) run(1, n, k, x_dtype, off, bias);
            for (long long n : {1LL << 17, (1LL << 19) + 3, 1LL << 21}) run(3, n, 131071, x_dtype, off, bias);
            for (long long m : {1LL << 17, (1LL << 19) + 3, 1LL << 21}) run(m, 3, 131071, x_dtype, off, bias);
            for (long long m : {(1LL << 23) + 1, 1LL << 27, most}) run(m, 3, 100, x_dtype, off, bias);
            run(1 << 19, 1 << 19, 131056, x_dtype, off, bias);
            run(40, 1 << 27, 0, x_dtype, off, bias);
        }
    std::printf("extents: %d failures\n", failures);
    return failures != 0;
}
