// What the host sides check of matrices in memory.  Not part of the C ABI.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/fq.h"

namespace fq {

inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

inline bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }

inline size_t size_of(int32_t dtype) { return dtype == FQ_I8 ? 1 : dtype == FQ_F16 ? 2 : 4; }

// Rows of a matrix in memory: bytes of one, from one to the next, and how many.
struct Rows {
    uintptr_t at;
    size_t width, pitch, count;
    size_t span() const { return count ? (count - 1) * pitch + width : 0; }
};

// Whether two matrices share memory.  Columns of one buffer (equal pitches, rows that fall into each other's gaps) do not.
inline bool overlap(const Rows &a, const Rows &b)
{
    if (!a.at || !b.at || !a.width || !b.width || !a.count || !b.count) return false;
    if (a.at >= b.at + b.span() || b.at >= a.at + a.span()) return false;
    if (a.pitch == b.pitch) {
        const size_t off = a.at <= b.at ? (b.at - a.at) % a.pitch : (a.pitch - (a.at - b.at) % a.pitch) % a.pitch;
        if (off >= a.width && off + b.width <= a.pitch) return false;
    }
    return true;
}

inline bool pitch_fits(long long rows, long long pitch, long long width)
{
    return pitch >= width && pitch <= (1LL << 56) / (rows > 0 ? rows : 1);
}

}  // namespace fq
