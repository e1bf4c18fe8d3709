// Rows in 8 bits: the block format of the OCP microscaling (MX) specification, 32 neighbours to a power
// of two.  Powers of two multiply exactly, so the codes are roundings of the elements themselves, whatever
// computes them, and what they stand for has at most seven bits: a bfloat16.
#pragma once

#include "la_common.h"

namespace la {

constexpr int kGroup = 32;

// Eight neighbours, one lane's share of a row, in registers.
struct Eight {
    float x[8];
};

// The same as they are stored.
template <typename T>
struct Stored {
    uint32_t w[2 * sizeof(T)];
};
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2)));  // at any element's address

// A lane's place in a row of C elements: eight from element c on, `valid` of them in the row (none where the row is not
// `here`).  Eight elements of the row are loaded in one go whatever the place, the row's last ones from its end on, and
// moved down by `shift` once they are there: loads that only some lanes make, or of single elements, cost branches
// and waits for every row (30000 rows of 771, bf16, backward 45 us; with both 83).
struct Span {
    int c, valid, shift;
    __device__ __forceinline__ Span(int c, int C, bool here = true)
        : c(c), valid(here ? C - c : 0), shift(valid >= 8 ? 0 : valid <= 0 ? 8 : 8 - valid)
    {
    }
    __device__ __forceinline__ int from(int C) const { return min(c, C - 8); }
};

// The span of the row at p.  SHORT: the row may have less than eight elements, which are loaded one by one.
template <bool SHORT, typename T>
__device__ __forceinline__ Stored<T> request8(const T *p, const Span &s, int C)
{
    Stored<T> r;
    if (!SHORT || C >= 8) {
        __builtin_memcpy(&r, p + s.from(C), sizeof r);
    } else {  // as if the row's end were where it is in a row of eight
        T c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = j - (8 - C) >= 0 ? p[j - (8 - C)] : (T)0;
        __builtin_memcpy(&r, c, sizeof r);
    }
    return r;
}
// Its elements; those behind the row's end are zero.
template <typename T>
__device__ __forceinline__ Eight widen(const Stored<T> &s)
{
    Eight r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (sizeof(T) == 4) r.x[j] = __uint_as_float(s.w[j]);
        else r.x[j] = __uint_as_float(j & 1 ? s.w[j / 2] & 0xffff0000u : s.w[j / 2] << 16);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ Eight widen(const Stored<T> &s, const Span &at)
{
    Eight r = widen<T>(s);
    if (at.shift) {
#pragma unroll
        for (int m = 1; m <= 8; m *= 2)
#pragma unroll
            for (int j = 0; j < 8; ++j) r.x[j] = at.shift & m ? (j + m < 8 ? r.x[j + m] : 0.f) : r.x[j];
    }
    return r;
}
template <bool SHORT, typename T>
__device__ __forceinline__ Eight load8(const T *p, const Span &s, int C)
{
    return widen<T>(request8<SHORT>(p, s, C), s);
}
template <typename T>
__device__ __forceinline__ Stored<T> narrow(const Eight &r)
{
    Stored<T> s;
#pragma unroll
    for (int j = 0; j < (int)(2 * sizeof(T)); ++j) {
        if (sizeof(T) == 4) s.w[j] = __float_as_uint(r.x[j]);
        else {
            const __bf16 c[2] = {(__bf16)r.x[2 * j], (__bf16)r.x[2 * j + 1]};
            __builtin_memcpy(&s.w[j], c, 4);
        }
    }
    return s;
}
// STREAM: non-temporal.  What a forward pass over the rows writes is more than it reads again, and a cache line that
// is written whole costs less when it is not kept: 16384 rows of 2048, bf16, two tensors in and two out 50 and 41 us
// (with a reader of y behind it 84 and 75, of y and s 102 and 99).  Not in float32, whose lanes' 32 bytes are two
// stores of half lines (47 and 51), and not in the backward pass, which reads three tensors for one (55 and 62).
template <bool STREAM, typename T>
__device__ __forceinline__ void store8(T *row, const Eight &r, const Span &at)
{
    const Stored<T> s = narrow<T>(r);
    T *p = row + at.c;
    if (at.valid >= 8) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) {
            const words4 v = {s.w[4 * k], s.w[4 * k + 1], s.w[4 * k + 2], s.w[4 * k + 3]};
            if (STREAM && sizeof(T) == 2) __builtin_nontemporal_store(v, (words4 *)p + k);
            else ((words4 *)p)[k] = v;
        }
    } else {
        T c[8];
        __builtin_memcpy(c, &s, sizeof c);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < at.valid) p[j] = c[j];
    }
}

// The largest magnitude of a group, as bits (a NaN is larger than infinity), from its four lanes' shares.
__device__ __forceinline__ uint32_t group_most(const Eight &r)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(r.x[j]) & 0x7fffffffu);
    m = max(m, (uint32_t)__shfl_xor((int)m, 1));
    return max(m, (uint32_t)__shfl_xor((int)m, 2));
}
// The power k of a group: the least with which its largest magnitude fits.  A group of zeros gets that of
// 2^-1, a group that is not finite 128, whose byte stands for NaN.
__device__ __forceinline__ int group_power(uint32_t most, bool ints)
{
    if (most >= 0x7f800000u) return 128;
    const float m = __uint_as_float(most), part = __builtin_amdgcn_frexp_mantf(m);  // m = part 2^e, 1/2 <= part < 1
    const int e = __builtin_amdgcn_frexp_expf(m);
    const int k = ints ? e - 1 + (part > 127.f / 128.f) : e - 9 + (part > 448.f / 512.f);
    return min(max(k, -127), 127);
}
__device__ __forceinline__ uint2 codes_of(const Eight &r, int k, bool ints)
{
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float *x = r.x + 4 * h;
        if (ints) {
            uint32_t c = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = (int)rintf(__builtin_amdgcn_ldexpf(x[j], 6 - k));
                c |= (uint32_t)(min(max(i, -127), 127) & 255) << (8 * j);
            }
            w[h] = c;
        } else {
            int c = 0;
            c = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_ldexpf(x[0], -k), __builtin_amdgcn_ldexpf(x[1], -k), c, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_ldexpf(x[2], -k), __builtin_amdgcn_ldexpf(x[3], -k), c, true);
            w[h] = (uint32_t)c;
        }
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ Eight values_of(uint2 c, int e, bool ints)
{
    Eight r;
    const int k = e - 127;
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float *x = r.x + 4 * h;
        if (ints) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_ldexpf((float)(int)(int8_t)(w[h] >> (8 * j)), k - 6);
        } else {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[h], true);
            x[0] = __builtin_amdgcn_ldexpf(lo[0], k), x[1] = __builtin_amdgcn_ldexpf(lo[1], k);
            x[2] = __builtin_amdgcn_ldexpf(hi[0], k), x[3] = __builtin_amdgcn_ldexpf(hi[1], k);
        }
        if (e == 255) x[0] = x[1] = x[2] = x[3] = __builtin_nanf("");
    }
    return r;
}
template <bool SHORT>
__device__ __forceinline__ uint2 request_codes(const uint8_t *p, const Span &s, int C)
{
    uint32_t w[2] = {0, 0};
    if (!SHORT || C >= 8) __builtin_memcpy(w, p + s.from(C), 8);
    else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j - (8 - C) >= 0) w[j / 4] |= (uint32_t)p[j - (8 - C)] << (8 * (j % 4));
    }
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint2 settle(uint2 c, const Span &s)
{
    const uint64_t v = s.shift < 8 ? ((uint64_t)c.y << 32 | c.x) >> (8 * s.shift) : 0;
    return make_uint2((uint32_t)v, (uint32_t)(v >> 32));
}
__device__ __forceinline__ void store_codes(uint8_t *p, uint2 c, int valid)
{
    if (valid >= 8) __builtin_memcpy(p, &c, 8);
    else {
        const uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) p[j] = (uint8_t)(w[j / 4] >> (8 * (j % 4)));
    }
}

// A span into its codes; the group's first lane leaves the power.  The four lanes of a group call it together.
// `codes`, `powers`: the row's.
__device__ __forceinline__ void pack8(const Eight &r, uint8_t *codes, uint8_t *powers, const Span &at, bool ints)
{
    const int k = group_power(group_most(r), ints);
    if (at.valid <= 0) return;
    store_codes(codes + at.c, codes_of(r, k, ints), at.valid);
    if (at.c % kGroup == 0) powers[at.c / kGroup] = (uint8_t)(k + 127);
}

}  // namespace la
