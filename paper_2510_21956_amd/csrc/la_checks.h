// Argument checks that the entry points share (host).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "la.h"

namespace la {

static inline size_t round_up(size_t x, size_t m) { return (x + m - 1) / m * m; }

struct Range {
    const void *p;
    size_t bytes;
};
static inline bool overlap(const Range &x, const Range &y)
{
    if (!x.p || !y.p || !x.bytes || !y.bytes) return false;
    const uintptr_t a0 = (uintptr_t)x.p, a1 = a0 + x.bytes, b0 = (uintptr_t)y.p, b1 = b0 + y.bytes;
    return a0 < b1 && b0 < a1;
}
// No written buffer (outs) may overlap any other buffer of the call.
static inline bool any_alias(const Range *ins, int nin, const Range *outs, int nout)
{
    for (int i = 0; i < nout; ++i) {
        for (int j = 0; j < nin; ++j)
            if (overlap(outs[i], ins[j])) return true;
        for (int j = i + 1; j < nout; ++j)
            if (overlap(outs[i], outs[j])) return true;
    }
    return false;
}

static inline bool real_type(la_dtype t) { return t == LA_F32 || t == LA_BF16; }
static inline bool eight_bits(la_dtype t) { return t == LA_E4M3 || t == LA_I8; }
static inline size_t size_of(la_dtype t) { return t == LA_F32 ? 4 : t == LA_BF16 ? 2 : 1; }
static inline bool aligned_to(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace la
