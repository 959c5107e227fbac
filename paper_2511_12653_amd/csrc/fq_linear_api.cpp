// Host side of the int8 linear layer: validation, workspace and launches (declared in include/fq.h).
#include <cstring>

#include "../../include/fq.h"
#include "fq_linear.h"

namespace fq {
namespace {

constexpr size_t kAlign = 256;
// What a launch takes, so that its grid has less than 2^32 threads: rows of x, up to 256 threads to one; channels, 512 to 16 of them;
// bytes of codes that are laid out anew, of x and w each, a thread to 16.
constexpr long long kMostRows = 1LL << 23, kMostChannels = 1LL << 26, kMostCodes = 1LL << 34;

size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }

size_t size_of(int32_t dtype) { return dtype == FQ_I8 ? 1 : dtype == FQ_F16 ? 2 : 4; }

// Rows of a matrix in memory: bytes of one, from one to the next, and how many.
struct Rows {
    uintptr_t at;
    size_t width, pitch, count;
    size_t span() const { return count ? (count - 1) * pitch + width : 0; }
};

// Whether two matrices share memory.  Columns of one buffer (equal pitches, rows that fall into each other's gaps) do not.
bool overlap(const Rows &a, const Rows &b)
{
    if (!a.at || !b.at || !a.width || !b.width || !a.count || !b.count) return false;
    if (a.at >= b.at + b.span() || b.at >= a.at + a.span()) return false;
    if (a.pitch == b.pitch) {
        const size_t off = a.at <= b.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
        if (off >= a.width && off + b.width <= a.pitch) return false;
    }
    return true;
}

// Whether the tiles take rows of codes as they lie.
bool fits(const void *p, long long ld, long long k)
{
    return aligned(p, 16) && ld % 16 == 0 && ld <= kMostPitch && k % 16 == 0;
}

// [codes of x][scales of x][codes of w], each only where it is needed: x is quantized or laid out anew, w laid out anew.
struct Workspace {
    long long pitch = 0;             // of a row of codes
    size_t scales = 0, w = 0, bytes = kAlign;
};

Workspace workspace_of(const fq_linear &d)
{
    Workspace at;
    at.pitch = (d.k + kCodePitch - 1) / kCodePitch * kCodePitch;
    if (d.m == 0 || d.n == 0 || d.k == 0) at.pitch = 0;
    size_t end = 0;
    if (d.x_dtype != FQ_I8 || !fits(d.x, d.ldx, d.k)) end += round_up((size_t)d.m * (size_t)at.pitch, kAlign);
    at.scales = end;
    if (d.x_dtype != FQ_I8) end += round_up((size_t)d.m * sizeof(float), kAlign);
    at.w = end;
    if (!fits(d.w, d.ldw, d.k)) end += round_up((size_t)d.n * (size_t)at.pitch, kAlign);
    if (end > at.bytes) at.bytes = end;
    return at;
}

bool pitch_fits(long long rows, long long pitch, long long width)
{
    return pitch >= width && pitch <= (1LL << 56) / (rows > 0 ? rows : 1);
}

fq_status validate(const fq_linear &d)
{
    if (d.x_dtype != FQ_F16 && d.x_dtype != FQ_F32 && d.x_dtype != FQ_I8) return FQ_ERR_DTYPE;
    if (d.y_dtype != FQ_F16 && d.y_dtype != FQ_F32) return FQ_ERR_DTYPE;
    if (d.m < 0 || d.n < 0 || d.k < 0 || d.m > 0x7fffff00LL || d.n > 0x7fffff00LL || d.k > kLinearMostK) return FQ_ERR_SHAPE;
    if (!pitch_fits(d.m, d.ldx, d.k) || !pitch_fits(d.n, d.ldw, d.k) || !pitch_fits(d.m, d.ldy, d.n)) return FQ_ERR_SHAPE;
    if ((d.xs_step != 0 && d.xs_step != 1) || (d.ws_step != 0 && d.ws_step != 1)) return FQ_ERR_SHAPE;
    if (((d.m + 31) / 32) * ((d.n + 31) / 32) > 0x7fffffffLL) return FQ_ERR_SHAPE;
    const size_t xb = size_of(d.x_dtype), yb = size_of(d.y_dtype);
    if (!aligned(d.x, xb) || !aligned(d.xs, 4) || !aligned(d.ws, 4) || !aligned(d.bias, 4) || !aligned(d.y, yb)) return FQ_ERR_ALIGN;
    if (d.m == 0 || d.n == 0) return FQ_OK;
    if (!d.y || !d.ws || (d.x_dtype == FQ_I8 && !d.xs) || (d.k > 0 && (!d.x || !d.w))) return FQ_ERR_NULL;
    const size_t m = (size_t)d.m, n = (size_t)d.n, k = (size_t)d.k;
    const Rows y = {(uintptr_t)d.y, n * yb, (size_t)d.ldy * yb, m};
    const Rows in[] = {{(uintptr_t)d.x, k * xb, (size_t)d.ldx * xb, m}, {(uintptr_t)d.w, k, (size_t)d.ldw, n},
                       {(uintptr_t)d.ws, (d.ws_step ? n : 1) * 4, 0, 1}, {(uintptr_t)d.bias, n * 4, 0, 1},
                       {d.x_dtype == FQ_I8 ? (uintptr_t)d.xs : 0, (d.xs_step ? m : 1) * 4, 0, 1}};
    for (const Rows &r : in)
        if (overlap(y, r)) return FQ_ERR_ALIAS;
    return FQ_OK;
}

fq_status run(const fq_linear &d, void *workspace, void *stream)
{
    const Workspace at = workspace_of(d);
    const bool quantize = d.x_dtype != FQ_I8, x_fits = !quantize && fits(d.x, d.ldx, d.k), w_fits = fits(d.w, d.ldw, d.k);
    LinearArgs a;
    std::memset(&a, 0, sizeof a);
    a.x = (const int8_t *)d.x; a.xs = d.xs; a.ldx = d.ldx; a.xs_step = d.xs_step;
    a.w = d.w; a.ws = d.ws; a.ldw = d.ldw; a.ws_step = d.ws_step;
    a.bias = d.bias; a.y = d.y; a.ldy = d.ldy; a.y16 = d.y_dtype == FQ_F16;
    a.m = (int)d.m; a.n = (int)d.n; a.k = a.kx = a.kw = (int)d.k;
    a.y_lines = aligned(a.y, 128) && (size_t)a.ldy * size_of(d.y_dtype) % 128 == 0;
    a.x_fits = x_fits || quantize;                   // (codes in the workspace fit)
    a.w_fits = w_fits;
    a.x16 = d.x_dtype == FQ_F16;
    a.x_vec = aligned(d.x, 16) && (size_t)d.ldx * size_of(d.x_dtype) % 16 == 0;
    if (quantize && linear_few(a, (int)size_of(d.x_dtype))) {
        a.raw = d.x;
        return launch_linear(a, stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
    }
    int8_t *const codes = (int8_t *)workspace;
    AlignArgs w;
    std::memset(&w, 0, sizeof w);
    const bool rows = quantize && linear_rows(a);
    if (!w_fits && a.k > 0 && !(rows ? linear_rows_as_they_lie(a) : linear_few(a, 1))) {
        w = {a.w, codes + at.w, d.n, d.ldw, at.pitch, a.k};
        a.w = w.to;
        a.ldw = at.pitch;
        a.kw = (int)at.pitch;
    }
    if (rows) {
        a.raw = d.x;
        if (w.rows && launch_align_rows(w, {}, stream) != 0) return FQ_ERR_LAUNCH;
    } else if (quantize) {
        QuantizeArgs q;
        std::memset(&q, 0, sizeof q);
        q.x = d.x; q.ldx = d.ldx; q.m = a.m; q.k = a.k; q.x16 = a.x16;
        q.q = codes; q.s = (float *)(codes + at.scales); q.pitch = at.pitch;
        if (launch_quantize_rows(q, w, stream) != 0) return FQ_ERR_LAUNCH;
        a.xs = q.s;
        a.xs_step = 1;
    } else if (!x_fits && linear_few(a, 1)) {
        return launch_linear(a, stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
    } else if (a.k > 0 && (!x_fits || w.rows)) {
        a.x_fits = 1;
        const AlignArgs x = {a.x, codes, x_fits ? 0 : d.m, d.ldx, at.pitch, a.k};
        if (launch_align_rows(x, w, stream) != 0) return FQ_ERR_LAUNCH;
    }
    if (!x_fits && !a.raw) {
        a.x = codes;
        a.ldx = at.pitch;
        a.kx = (int)at.pitch;
    }
    return launch_linear(a, stream) == 0 ? FQ_OK : FQ_ERR_LAUNCH;
}

fq_status forward(const fq_linear &d, void *workspace, size_t ws_bytes, void *stream)
{
    const fq_status st = validate(d);
    if (st != FQ_OK || d.m == 0 || d.n == 0) return st;
    if (d.x_dtype != FQ_I8 || !fits(d.x, d.ldx, d.k) || !fits(d.w, d.ldw, d.k)) {
        if (!workspace || ws_bytes < workspace_of(d).bytes) return FQ_ERR_WORKSPACE;
        if (!aligned(workspace, kAlign)) return FQ_ERR_ALIGN;
    }
    const long long most = kMostCodes / (workspace_of(d).pitch ? workspace_of(d).pitch : 1);
    const long long rows = most < kMostRows ? most : kMostRows, channels = most < kMostChannels ? most : kMostChannels;
    for (long long row = 0; row < d.m; row += rows)
        for (long long column = 0; column < d.n; column += channels) {
            fq_linear part = d;
            part.m = d.m - row < rows ? d.m - row : rows;
            part.n = d.n - column < channels ? d.n - column : channels;
            part.x = d.x ? (const char *)d.x + (size_t)(row * d.ldx) * size_of(d.x_dtype) : nullptr;
            part.xs = d.xs ? d.xs + row * d.xs_step : nullptr;
            part.w = d.w ? d.w + column * d.ldw : nullptr;
            part.ws = d.ws + column * d.ws_step;
            part.bias = d.bias ? d.bias + column : nullptr;
            part.y = (char *)d.y + (size_t)(row * d.ldy + column) * size_of(d.y_dtype);
            const fq_status ran = run(part, workspace, stream);
            if (ran != FQ_OK) return ran;
        }
    return FQ_OK;
}

}  // namespace
}  // namespace fq

extern "C" {

size_t fq_linear_workspace_bytes(const fq_linear *d)
{
    return d && fq::validate(*d) == FQ_OK ? fq::workspace_of(*d).bytes : 0;
}

fq_status fq_linear_forward(const fq_linear *d, void *workspace, size_t ws_bytes, void *hip_stream)
{
    if (!d) return FQ_ERR_NULL;
    return fq::forward(*d, workspace, ws_bytes, hip_stream);
}

}  // extern "C"
