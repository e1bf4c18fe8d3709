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

// Elements from `valid` on (a row's end) are zero.
template <typename T>
__device__ __forceinline__ Stored<T> request8(const T *p, int valid)
{
    Stored<T> r;
    if (valid >= 8) {
        __builtin_memcpy(&r, p, sizeof r);
    } else {
        T c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = j < valid ? p[j] : (T)0;
        __builtin_memcpy(&r, c, sizeof r);
    }
    return r;
}
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
__device__ __forceinline__ Eight load8(const T *p, int valid)
{
    return widen<T>(request8(p, valid));
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
__device__ __forceinline__ void store8(T *p, const Eight &r, int valid)
{
    const Stored<T> s = narrow<T>(r);
    if (valid >= 8) {
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
            if (j < valid) p[j] = c[j];
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
__device__ __forceinline__ uint2 load_codes(const uint8_t *p, int valid)
{
    uint2 c = make_uint2(0, 0);
    if (valid >= 8) __builtin_memcpy(&c, p, 8);
    else {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < valid) w[j / 4] |= (uint32_t)p[j] << (8 * (j % 4));
        c = make_uint2(w[0], w[1]);
    }
    return c;
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

// Eight neighbours of a row of C elements from element `at` on, at % 8 == 0, into its codes; the group's first
// lane leaves the power.  The four lanes of a group call it together.  `groups`: the row's powers.
__device__ __forceinline__ void pack8(const Eight &r, uint8_t *codes, uint8_t *powers, int at, int valid, bool ints)
{
    const int k = group_power(group_most(r), ints);
    if (valid <= 0) return;
    store_codes(codes + at, codes_of(r, k, ints), valid);
    if (at % kGroup == 0) powers[at / kGroup] = (uint8_t)(k + 127);
}

}  // namespace la
