// Selective state space scan: S states to a channel, h[s] -> exp(d A[s]) h[s] + d x B[s], read out by C: forward, backward,
// in steps.
//
// A lane holds one channel, a wave P of its states in registers, a workgroup's W waves all S <= P W of them; it walks a
// sequence (or a segment of one) in tiles of rows.  The waves share a tile's rows: each forms d and d x of its rows
// and leaves them in LDS, with the tile's B and C; then every wave walks all rows with its states, and at last each
// wave adds up the waves' shares of its rows' outputs.
#include "la_checks.h"
#include "la_common.h"
#include "la_scalar.h"

namespace la {
namespace {

constexpr int kMostStates = 128;
constexpr int kRows = 16;  // of a tile
// What the backward pass keeps of kCells / P rows, h and exp(d A) of every row and state, fills 128 registers, and its 64
// sums over a wave's channels of either kind are one to a lane.  Where a tile has more rows they are taken in
// parts, the states before a part formed once more from those before the tile.
constexpr int kCells = 64;

struct Scan {
    const void *X, *Dt, *Bm, *Cm;
    size_t xs, ts, bs, cs;
    const float *A, *D, *bias;
    const float *first;  // forward: h0; backward: dlast; [B, C, S]
    float *end;          // forward: last; backward: dh0
    void *Y;
    float *saved;        // [B, tiles, S, C] the states before every tile
    const int *lengths;
    const void *dY;
    void *dX, *dDt;
    float *shares;       // [B, columns, tiles, W, parts, 2, 64] sums over a column's channels for dB, dC
    float *dA, *dd;      // [B * segs, S, C], [B * segs, 2, C] a segment's sums for dA; for dD and dbias
    float *sums, *spans; // [B, segs, S, C] what a segment makes of zero states, [B, segs, C] the sum of its d
    int B, N, C, S, G, group, per, columns;  // channels of a group; columns of 64 channels to it, in all
    int tiles, seg, segs;                    // tiles of the sequence; rows of a segment, segments
    int step;
};

// Where a workgroup is: its sequence, channels and rows.
struct Spot {
    int b, column, g, c, seg, n, r0, r1;
    bool live;
    __device__ __forceinline__ Spot(const Scan &a, int lane)
    {
        const unsigned k = blockIdx.x / a.segs;
        seg = (int)(blockIdx.x % a.segs);
        column = (int)(k % a.columns), b = (int)(k / a.columns);
        g = column / a.per;
        c = g * a.group + column % a.per * 64 + lane;
        const int behind = (g + 1) * a.group;
        live = c < behind;
        c = min(c, behind - 1);  // lanes behind the group's last channel read that one
        n = a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
        r0 = min(seg * a.seg, a.N);
        r1 = min(n, r0 + a.seg);
    }
};

// d and, for the backward pass, its derivative by dt.
template <bool FINE>
__device__ __forceinline__ float step_of(float dt, int step, float &slope)
{
    slope = 1.f;
    if (step == LA_STEP_VALUE) return dt;
    const float E = exp_down<FINE>(dt);
    float rest;
    sigmoid_of(dt, E, slope, rest);
    return softplus_of(dt, E);
}

// A tile's B and C on their way to LDS: R rows of [B | C], P W of each, zeros behind the last state and row.
template <typename T, int P, int W, int R>
struct Vectors {
    static constexpr int COUNT = 2 * R * P / 64;
    T v[COUNT];
    __device__ __forceinline__ void load(const Scan &a, const Spot &p, int t)
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) {
            const int k = threadIdx.x + i * 64 * W, row = k / (2 * P * W), s = k % (P * W);
            const bool c = k % (2 * P * W) >= P * W;
            v[i] = (T)0;
            if (s < a.S && t + row < p.n) {
                const size_t r = (size_t)p.b * a.N + t + row;
                v[i] = c ? ((const T *)a.Cm)[r * a.cs + p.g * a.S + s] : ((const T *)a.Bm)[r * a.bs + p.g * a.S + s];
            }
        }
    }
    __device__ __forceinline__ void leave(float *to) const
    {
#pragma unroll
        for (int i = 0; i < COUNT; ++i) to[threadIdx.x + i * 64 * W] = load_elem(v, i);
    }
};

template <int P>
__device__ __forceinline__ void decays(const Scan &a, const Spot &p, int wave, float (&A)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int s = wave * P + j;
        A[j] = s < a.S ? a.A[(size_t)p.c * a.S + s] * kLog2e : 0.f;
    }
}
template <int P>
__device__ __forceinline__ void states_from(const float *from, const Scan &a, const Spot &p, int wave, float (&h)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int s = wave * P + j;
        h[j] = from && p.live && s < a.S ? from[((size_t)p.b * a.C + p.c) * a.S + s] : 0.f;
    }
}
template <int P>
__device__ __forceinline__ void states_to(float *to, const Scan &a, const Spot &p, int wave, const float (&h)[P])
{
    if (!to || !p.live) return;
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int s = wave * P + j;
        if (s < a.S) to[((size_t)p.b * a.C + p.c) * a.S + s] = h[j];
    }
}
// The states that the segments before (BWD: behind) this one leave.
template <int P, bool BWD>
__device__ __forceinline__ void walk_segments(const Scan &a, const Spot &p, int wave, const float (&A)[P], float (&h)[P])
{
    const int end = BWD ? (p.n + a.seg - 1) / a.seg - 1 : 0;  // the last segment with rows
    for (int k = end; BWD ? k > p.seg : k < p.seg; k += BWD ? -1 : 1) {
        const size_t at = (size_t)p.b * a.segs + k;
        const float span = a.spans[at * a.C + p.c];
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int s = wave * P + j;
            if (s < a.S) h[j] = fmaf(__builtin_amdgcn_exp2f(span * A[j]), h[j], a.sums[(at * a.S + s) * a.C + p.c]);
        }
    }
}

// FULL: outputs.  Else what the segment makes of zero states.
template <typename T, int P, int W, bool FULL>
__global__ void __launch_bounds__(64 * W) k_selective(Scan a)
{
    constexpr int R = kRows, OWN = (R + W - 1) / W;  // rows of a tile, of a wave
    __shared__ float2 du[R][64];
    __shared__ float ys[W][R][64];
    __shared__ __align__(16) float bc[R][2][P * W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Spot p(a, lane);
    float A[P], h[P], span = 0.f;
    decays<P>(a, p, wave, A);
    states_from<P>(FULL ? a.first : nullptr, a, p, wave, h);
    if (FULL) walk_segments<P, false>(a, p, wave, A, h);
    const float bias = a.bias ? a.bias[p.c] : 0.f, D = a.D ? a.D[p.c] : 0.f;
    T x[OWN], dt[OWN];
    Vectors<T, P, W, R> vec;
    auto request = [&](int t) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = wave + i * W;
            if (R % W && r >= R) break;
            const size_t row = (size_t)p.b * a.N + min(t + r, p.n - 1);
            x[i] = ((const T *)a.X)[row * a.xs + p.c];
            dt[i] = ((const T *)a.Dt)[row * a.ts + p.c];
        }
        vec.load(a, p, t);
    };
    if (p.r0 < p.r1) request(p.r0);
    for (int t = p.r0; t < p.r1; t += R) {
        float xw[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = wave + i * W;
            if (R % W && r >= R) break;
            float slope;
            const float d = t + r < p.n ? step_of<sizeof(T) == 4>(load_elem(dt, i) + bias, a.step, slope) : 0.f;
            xw[i] = t + r < p.n ? load_elem(x, i) : 0.f;
            du[r][lane] = make_float2(d, d * xw[i]);
        }
        vec.leave(&bc[0][0][0]);
        block_sync();
        if (t + R < p.r1) request(t + R);
        if (FULL && a.saved && p.live) {
            float *to = a.saved + ((size_t)p.b * a.tiles + t / R) * a.S * a.C + p.c;
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (wave * P + j < a.S) to[(size_t)(wave * P + j) * a.C] = h[j];
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float2 s = du[r][lane];
            const float *Bt = &bc[r][0][wave * P], *Ct = &bc[r][1][wave * P];
            float y = 0.f;
#pragma unroll
            for (int j = 0; j < P; ++j) {
                h[j] = fmaf(__builtin_amdgcn_exp2f(s.x * A[j]), h[j], s.y * Bt[j]);
                if (FULL) y = fmaf(Ct[j], h[j], y);
            }
            if (FULL) ys[wave][r][lane] = y;
            else span += s.x;
        }
        block_sync();
        if (FULL) {
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int r = wave + i * W;
                if (R % W && r >= R) break;
                float y = D * xw[i];
#pragma unroll
                for (int w = 0; w < W; ++w) y += ys[w][r][lane];
                if (p.live && t + r < p.n) store_elem((T *)a.Y, ((size_t)p.b * a.N + t + r) * a.C + p.c, y);
            }
        }
    }
    if (FULL) {
        if (p.live)
            for (int t = max(p.r0, p.n) + wave; t < min(a.N, p.r0 + a.seg); t += W)  // padding
                store_elem((T *)a.Y, ((size_t)p.b * a.N + t) * a.C + p.c, 0.f);
        if (p.seg == max(p.n - 1, 0) / a.seg) states_to<P>(a.end, a, p, wave, h);
    } else if (p.live) {
        const size_t at = (size_t)p.b * a.segs + p.seg;
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (wave * P + j < a.S) a.sums[(at * a.S + wave * P + j) * a.C + p.c] = h[j];
        if (wave == 0) a.spans[at * a.C + p.c] = span;
    }
}

// 64 values a lane, added up over the lanes: lane l gets the sum of value l.  Halves, then quarters of the values are
// exchanged between the lanes' halves and quarters, so that every step halves what a lane has to add.
__device__ __forceinline__ float over_lanes(float (&v)[64], int lane)
{
#pragma unroll
    for (int m = 32; m >= 1; m /= 2) {
        const bool up = lane & m;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float keep = up ? v[i + m] : v[i], send = up ? v[i] : v[i + m];
            v[i] = keep + __shfl_xor(send, m);
        }
    }
    return v[0];
}

// Backward.  FULL: outputs, walking the tiles from the far end: states from the saved ones before the tile on, then the rows in
// reverse.  Else what the segment hands to the rows before it from nothing behind it.
template <typename T, int P, int W, bool FULL>
__global__ void __launch_bounds__(64 * W) k_selective_back(Scan a)
{
    constexpr int R = kRows, OWN = (R + W - 1) / W, PART = kCells / P;
    __shared__ float2 du[R][64];
    __shared__ float dys[R][64];
    __shared__ float2 gs[FULL ? W : 1][R][64];
    __shared__ __align__(16) float bc[R][2][P * W];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Spot p(a, lane);
    float A[P], carry[P], dA[P], before[P], dD = 0.f, db = 0.f, span = 0.f;
    decays<P>(a, p, wave, A);
#pragma unroll
    for (int j = 0; j < P; ++j) dA[j] = 0.f;
    states_from<P>(FULL ? a.first : nullptr, a, p, wave, carry);
    if (FULL) walk_segments<P, true>(a, p, wave, A, carry);
    const float bias = a.bias ? a.bias[p.c] : 0.f, D = a.D ? a.D[p.c] : 0.f;
    T x[OWN], dt[OWN], dy[OWN];
    Vectors<T, P, W, R> vec;
    auto request = [&](int t) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = wave + i * W;
            if (R % W && r >= R) break;
            const size_t row = (size_t)p.b * a.N + min(t + r, p.n - 1);
            if (FULL) x[i] = ((const T *)a.X)[row * a.xs + p.c];
            dt[i] = ((const T *)a.Dt)[row * a.ts + p.c];
            dy[i] = ((const T *)a.dY)[row * a.C + p.c];
        }
        vec.load(a, p, t);
        if (FULL) {
            const float *from = a.saved + ((size_t)p.b * a.tiles + t / R) * a.S * a.C + p.c;
#pragma unroll
            for (int j = 0; j < P; ++j) before[j] = p.live && wave * P + j < a.S ? from[(size_t)(wave * P + j) * a.C] : 0.f;
        }
    };
    const int last = p.r0 + (p.r1 - p.r0 - 1) / R * R;
    if (p.r0 < p.r1) request(last);
    for (int t = last; p.r0 < p.r1 && t >= p.r0; t -= R) {
        float xw[OWN], slope[OWN];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int r = wave + i * W;
            if (R % W && r >= R) break;
            const bool here = p.live && t + r < p.n;
            const float d = step_of<sizeof(T) == 4>(load_elem(dt, i) + bias, a.step, slope[i]);
            xw[i] = FULL && here ? load_elem(x, i) : 0.f;
            du[r][lane] = make_float2(here ? d : 0.f, here ? d * xw[i] : 0.f);
            dys[r][lane] = here ? load_elem(dy, i) : 0.f;
        }
        vec.leave(&bc[0][0][0]);
        block_sync();
        if constexpr (FULL) {
            float begin[P];
#pragma unroll
            for (int j = 0; j < P; ++j) begin[j] = before[j];
            if (t > p.r0) request(t - R);
            float *to = a.shares + ((((size_t)p.b * a.columns + p.column) * a.tiles + t / R) * W + wave) * (R / PART) * 128;
#pragma unroll 1
            for (int r0 = R - PART; r0 >= 0; r0 -= PART) {
                float h[kCells], f[kCells], h0[P];
#pragma unroll
                for (int j = 0; j < P; ++j) h0[j] = begin[j];
                for (int r = 0; r < r0; ++r) {
                    const float2 s = du[r][lane];
#pragma unroll
                    for (int j = 0; j < P; ++j) h0[j] = fmaf(__builtin_amdgcn_exp2f(s.x * A[j]), h0[j], s.y * bc[r][0][wave * P + j]);
                }
#pragma unroll
                for (int r = 0; r < PART; ++r) {
                    const float2 s = du[r0 + r][lane];
                    const float *Bt = &bc[r0 + r][0][wave * P];
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        f[r * P + j] = __builtin_amdgcn_exp2f(s.x * A[j]);
                        h[r * P + j] = fmaf(f[r * P + j], r ? h[(r - 1) * P + j] : h0[j], s.y * Bt[j]);
                    }
                }
#pragma unroll
                for (int r = PART - 1; r >= 0; --r) {
                    const float2 s = du[r0 + r][lane];
                    const float y = dys[r0 + r][lane];
                    const float *Bt = &bc[r0 + r][0][wave * P], *Ct = &bc[r0 + r][1][wave * P];
                    float gu = 0.f, gd = 0.f;
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        const float g = fmaf(Ct[j], y, carry[j]);
                        gu = fmaf(g, Bt[j], gu);
                        carry[j] = g * f[r * P + j];
                        const float e = carry[j] * (r ? h[(r - 1) * P + j] : h0[j]);
                        gd = fmaf(e, A[j], gd);
                        dA[j] = fmaf(e, s.x, dA[j]);
                        f[r * P + j] = g * s.y;
                        h[r * P + j] *= y;
                    }
                    gs[wave][r0 + r][lane] = make_float2(gu, gd * kLn2);
                }
                to[r0 / PART * 128 + lane] = over_lanes(f, lane);
                to[r0 / PART * 128 + 64 + lane] = over_lanes(h, lane);
            }
        } else {
            if (t > p.r0) request(t - R);
#pragma unroll
            for (int r = R - 1; r >= 0; --r) {
                const float2 s = du[r][lane];
                const float y = dys[r][lane];
                const float *Ct = &bc[r][1][wave * P];
#pragma unroll
                for (int j = 0; j < P; ++j) carry[j] = fmaf(Ct[j], y, carry[j]) * __builtin_amdgcn_exp2f(s.x * A[j]);
                span += s.x;
            }
        }
        block_sync();
        if constexpr (FULL) {
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int r = wave + i * W;
                if (R % W && r >= R) break;
                float gu = 0.f, gd = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float2 g = gs[w][r][lane];
                    gu += g.x, gd += g.y;
                }
                const float y = dys[r][lane], dd = fmaf(xw[i], gu, gd) * slope[i];
                if (p.live && t + r < p.n) {
                    const size_t at = ((size_t)p.b * a.N + t + r) * a.C + p.c;
                    store_elem((T *)a.dX, at, fmaf(du[r][lane].x, gu, D * y));
                    store_elem((T *)a.dDt, at, dd);
                    dD = fmaf(y, xw[i], dD);
                    db += dd;
                }
            }
        }
    }
    const size_t at = (size_t)p.b * a.segs + p.seg;
    if constexpr (FULL) {
        if (p.live)
            for (int t = max(p.r0, p.n) + wave; t < min(a.N, p.r0 + a.seg); t += W) {  // padding
                const size_t k = ((size_t)p.b * a.N + t) * a.C + p.c;
                store_elem((T *)a.dX, k, 0.f);
                store_elem((T *)a.dDt, k, 0.f);
            }
        if (p.seg == 0) states_to<P>(a.end, a, p, wave, carry);
        block_sync();
        gs[wave][0][lane] = make_float2(dD, db);
        block_sync();
        if (!p.live) return;
        if (a.dA)
#pragma unroll
            for (int j = 0; j < P; ++j)
                if (wave * P + j < a.S) a.dA[(at * a.S + wave * P + j) * a.C + p.c] = dA[j];
        if (wave == 0) {
            float2 s = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) s.x += gs[w][0][lane].x, s.y += gs[w][0][lane].y;
            a.dd[at * 2 * a.C + p.c] = s.x;
            a.dd[(at * 2 + 1) * a.C + p.c] = s.y;
        }
    } else if (p.live) {
#pragma unroll
        for (int j = 0; j < P; ++j)
            if (wave * P + j < a.S) a.sums[(at * a.S + wave * P + j) * a.C + p.c] = carry[j];
        if (wave == 0) a.spans[at * a.C + p.c] = span;
    }
}

// dB and dC from the columns' shares: a lane to a value, the columns of a group in order.
template <typename T, int P, int W>
__global__ void __launch_bounds__(256) k_selective_vectors(Scan a, T *dB, T *dC)
{
    constexpr int PART = kCells / P, EACH = W * (kRows / PART) * 128;  // values of a tile
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)a.B * a.G * a.tiles * EACH; i += (size_t)gridDim.x * 256) {
        const size_t k = i / EACH;
        const int v = (int)(i % EACH), m = v % 64, part = v / 128 % (kRows / PART), w = v / 128 / (kRows / PART);
        const int tile = (int)(k % a.tiles), g = (int)(k / a.tiles % a.G), b = (int)(k / a.tiles / a.G);
        const int t = tile * kRows + part * PART + m / P, s = w * P + m % P;
        if (t >= a.N || s >= a.S) continue;
        const int n = a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
        float sum = 0.f;
        if (t < n)
            for (int c = 0; c < a.per; ++c) sum += a.shares[(((size_t)b * a.columns + g * a.per + c) * a.tiles + tile) * EACH + v];
        store_elem(v % 128 < 64 ? dB : dC, (((size_t)b * a.N + t) * a.G + g) * a.S + s, sum);
    }
}

// dA, dD and dbias from the segments' sums: 64 channels and one row of the sums a workgroup, its waves take every 4th
// segment each.
__global__ void __launch_bounds__(256) k_selective_join(Scan a, float *dA, float *dD, float *db)
{
    __shared__ float sums[4][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane, s = blockIdx.y;
    const int rows = s < a.S ? a.S : 2;
    const float *from = s < a.S ? a.dA + (size_t)s * a.C : a.dd + (size_t)(s - a.S) * a.C;
    if (s < a.S && !dA) return;
    float sum = 0.f;
    if (c < a.C)
        for (int k = wave; k < a.B * a.segs; k += 4) sum += from[(size_t)k * rows * a.C + c];
    sums[wave][lane] = sum;
    block_sync();
    if (wave || c >= a.C) return;
    sum = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    if (s < a.S) dA[(size_t)c * a.S + s] = sum;
    else if (s == a.S) {
        if (dD) dD[c] = sum;
    } else if (db) db[c] = sum;
}

// T rows on a carried state, L lanes to a channel, P states a lane.
template <typename T, int P>
__global__ void __launch_bounds__(256) k_selective_step(Scan a, float *state, int L)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    const int l = (int)(i % L);
    const size_t k = i / L;
    if (k >= (size_t)a.B * a.C) return;
    const int b = (int)(k / a.C), c = (int)(k - (size_t)b * a.C), g = c / a.group;
    float A[P], h[P];
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int s = l * P + j;
        A[j] = s < a.S ? a.A[(size_t)c * a.S + s] * kLog2e : 0.f;
        h[j] = s < a.S ? state[k * a.S + s] : 0.f;
    }
    const float bias = a.bias ? a.bias[c] : 0.f, D = a.D ? a.D[c] : 0.f;
    for (int t = 0; t < a.N; ++t) {
        const size_t row = (size_t)b * a.N + t;
        const float x = load_elem((const T *)a.X, row * a.xs + c);
        float slope;
        const float d = step_of<sizeof(T) == 4>(load_elem((const T *)a.Dt, row * a.ts + c) + bias, a.step, slope), u = d * x;
        float y = 0.f;
#pragma unroll
        for (int j = 0; j < P; ++j) {
            const int s = l * P + j;
            const float Bt = s < a.S ? load_elem((const T *)a.Bm, row * a.bs + g * a.S + s) : 0.f;
            const float Ct = s < a.S ? load_elem((const T *)a.Cm, row * a.cs + g * a.S + s) : 0.f;
            h[j] = fmaf(__builtin_amdgcn_exp2f(d * A[j]), h[j], u * Bt);
            y = fmaf(Ct, h[j], y);
        }
        for (int m = 1; m < L; m *= 2) y += __shfl_xor(y, m);
        if (l == 0) store_elem((T *)a.Y, row * a.C + c, fmaf(D, x, y));
    }
#pragma unroll
    for (int j = 0; j < P; ++j)
        if (l * P + j < a.S) state[k * a.S + l * P + j] = h[j];
}

// States of a wave and waves of a workgroup.
struct Shape {
    int P, W;
};
Shape shape_of(int S)
{
    if (S <= 32) return {4, S <= 4 ? 1 : S <= 8 ? 2 : S <= 12 ? 3 : S <= 16 ? 4 : S <= 24 ? 6 : 8};
    if (S <= 64) return {8, S <= 48 ? 6 : 8};
    return {16, S <= 96 ? 6 : 8};
}
// f(states as a constant, waves as a constant)
template <typename F>
void by_shape(int S, F f)
{
    const Shape s = shape_of(S);
    auto with = [&](auto P, auto W) {
        if (s.P == decltype(P)::value && s.W == decltype(W)::value) f(P, W);
    };
    auto four = std::integral_constant<int, 4>();
    auto eight = std::integral_constant<int, 8>();
    auto more = std::integral_constant<int, 16>();
    with(four, std::integral_constant<int, 1>());
    with(four, std::integral_constant<int, 2>());
    with(four, std::integral_constant<int, 3>());
    with(four, std::integral_constant<int, 4>());
    with(four, std::integral_constant<int, 6>());
    with(four, std::integral_constant<int, 8>());
    with(eight, std::integral_constant<int, 6>());
    with(eight, std::integral_constant<int, 8>());
    with(more, std::integral_constant<int, 6>());
    with(more, std::integral_constant<int, 8>());
}

la_status check_shape(int B, int N, int C, int S, int G)
{
    if (B < 1 || N < 1 || C < 1 || S < 1 || G < 1 || N > 1 << 30 || S > kMostStates || C % G) return LA_ERR_SHAPE;
    const double columns = (double)B * G * ((C / G + 63) / 64);
    if (columns >= 2097152.0 || columns * ((N + 15) / 16) >= 2147483648.0) return LA_ERR_SHAPE;  // 2^21, 2^31
    return LA_OK;
}
la_status check(const Scan &a, la_step step, la_dtype dt)
{
    const la_status s = check_shape(a.B, a.N, a.C, a.S, a.G);
    if (s != LA_OK) return s;
    const size_t vec = (size_t)a.G * a.S;
    if (a.xs < (size_t)a.C || a.ts < (size_t)a.C || a.bs < vec || a.cs < vec) return LA_ERR_SHAPE;
    for (size_t n : {a.xs, a.ts, a.bs, a.cs, vec})
        if ((double)a.B * a.N * (double)n >= 1099511627776.0) return LA_ERR_SHAPE;  // 2^40
    if (!real_type(dt) || (step != LA_STEP_VALUE && step != LA_STEP_SOFTPLUS)) return LA_ERR_UNSUPPORTED;
    if (!a.X || !a.Dt || !a.A || !a.Bm || !a.Cm) return LA_ERR_NULL;
    const size_t e = size_of(dt);
    for (const void *p : {a.X, a.Dt, a.Bm, a.Cm, (const void *)a.Y, a.dY, (const void *)a.dX, (const void *)a.dDt})
        if (!aligned_to(p, e)) return LA_ERR_ALIGN;
    for (const void *p : {(const void *)a.A, (const void *)a.D, (const void *)a.bias, (const void *)a.first, (const void *)a.end, (const void *)a.lengths})
        if (!aligned_to(p, 4)) return LA_ERR_ALIGN;
    return LA_OK;
}
// The tensors that every call reads.
struct Inputs {
    Range r[9];
    Inputs(const Scan &a, la_dtype dt)
    {
        const size_t e = size_of(dt), rows = (size_t)a.B * a.N - 1, vec = (size_t)a.G * a.S;
        r[0] = {a.X, (rows * a.xs + a.C) * e}, r[1] = {a.Dt, (rows * a.ts + a.C) * e};
        r[2] = {a.Bm, (rows * a.bs + vec) * e}, r[3] = {a.Cm, (rows * a.cs + vec) * e};
        r[4] = {a.A, (size_t)a.C * a.S * 4}, r[5] = {a.D, (size_t)a.C * 4}, r[6] = {a.bias, (size_t)a.C * 4};
        r[7] = {a.first, (size_t)a.B * a.C * a.S * 4}, r[8] = {a.lengths, (size_t)a.B * 4};
    }
};
void lay_out(Scan &a)
{
    a.group = a.C / a.G;
    a.per = (a.group + 63) / 64;
    a.columns = a.G * a.per;
    a.tiles = (a.N + kRows - 1) / kRows;
    a.seg = a.tiles * kRows;
    a.segs = 1;
}
Scan scan_of(const void *X, size_t xs, const void *Dt, size_t ts, const float *A, const void *Bm, size_t bs, const void *Cm, size_t cs,
             const float *D, const float *bias, int B, int N, int C, int S, int G, la_step step)
{
    Scan a{};
    a.X = X, a.xs = xs, a.Dt = Dt, a.ts = ts, a.A = A, a.Bm = Bm, a.bs = bs, a.Cm = Cm, a.cs = cs, a.D = D, a.bias = bias;
    a.B = B, a.N = N, a.C = C, a.S = S, a.G = G, a.step = step;
    return a;
}

// Floats of a tile's shares: kRows rows of the P W states of a workgroup, for dB and for dC.
size_t shares_of(int S) { return (size_t)shape_of(S).P * shape_of(S).W * kRows * 2; }

// What a call keeps in its workspace, in floats.
struct Room {
    size_t shares, dA, dd, sums, spans, bytes;
    Room(const Scan &a, bool back)
    {
        size_t at = 0;
        auto take = [&](size_t n) {
            const size_t here = at;
            at += round_up(n, 64);
            return here;
        };
        const size_t segs = (size_t)a.B * a.segs;
        const bool cut = a.segs > 1;
        sums = take(cut ? segs * a.S * a.C : 0);
        spans = take(cut ? segs * a.C : 0);
        shares = take(back ? (size_t)a.B * a.columns * a.tiles * shares_of(a.S) : 0);
        dA = take(back ? segs * a.S * a.C : 0);
        dd = take(back ? segs * 2 * a.C : 0);
        bytes = at * 4;
    }
};

la_status done() { return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH; }

}  // namespace
}  // namespace la

extern "C" {

size_t la_selective_workspace_bytes(int B, int N, int C, int S, int G, int is_backward)
{
    if (la::check_shape(B, N, C, S, G) != LA_OK) return 0;
    la::Scan a{};
    a.B = B, a.N = N, a.C = C, a.S = S, a.G = G;
    la::lay_out(a);
    return la::Room(a, is_backward != 0).bytes;
}

size_t la_selective_saved_bytes(int B, int N, int C, int S)
{
    if (la::check_shape(B, N, C, S, 1) != LA_OK) return 0;
    return la::round_up((size_t)B * ((N + la::kRows - 1) / la::kRows) * S * C * 4, 256);
}

la_status la_selective_forward(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                               const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D,
                               const float *bias, const float *h0, void *Y, float *last, void *saved, size_t saved_bytes,
                               const int *lengths, int B, int N, int C, int S, int G, la_step step, la_dtype dt,
                               void *workspace, size_t workspace_bytes, void *hip_stream)
{
    la::Scan a = la::scan_of(X, x_stride, Dt, dt_stride, A, Bm, b_stride, Cm, c_stride, D, bias, B, N, C, S, G, step);
    a.first = h0, a.end = last, a.Y = Y, a.lengths = lengths, a.saved = (float *)saved;
    const la_status s = la::check(a, step, dt);
    if (s != LA_OK) return s;
    if (!Y) return LA_ERR_NULL;
    la::lay_out(a);
    const la::Room room(a, false);
    const size_t kept = la_selective_saved_bytes(B, N, C, S);
    if (room.bytes && (!workspace || workspace_bytes < room.bytes || !la::aligned_to(workspace, 256))) return LA_ERR_WORKSPACE;
    if (saved && (saved_bytes < kept || !la::aligned_to(saved, 256))) return LA_ERR_WORKSPACE;
    const la::Inputs in(a, dt);
    const la::Range outs[] = {{Y, (size_t)B * N * C * la::size_of(dt)}, {last, (size_t)B * C * S * 4}, {saved, kept}, {workspace, room.bytes}};
    if (la::any_alias(in.r, 9, outs, 4)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    a.sums = (float *)workspace + room.sums, a.spans = (float *)workspace + room.spans;
    const dim3 grid((unsigned)((size_t)B * a.columns * a.segs));
    const hipStream_t st = (hipStream_t)hip_stream;
    la::by_shape(S, [&](auto P, auto W) {
        constexpr int p = decltype(P)::value, w = decltype(W)::value;
        if (dt == LA_F32) {
            if (a.segs > 1) la::k_selective<float, p, w, false><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective<float, p, w, true><<<grid, dim3(64 * w), 0, st>>>(a);
        } else {
            if (a.segs > 1) la::k_selective<la::bf16_t, p, w, false><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective<la::bf16_t, p, w, true><<<grid, dim3(64 * w), 0, st>>>(a);
        }
    });
    return la::done();
}

la_status la_selective_backward(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                                const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D,
                                const float *bias, const void *saved, size_t saved_bytes, const void *dY, const float *dlast,
                                void *dX, void *dDt, float *dA, void *dBm, void *dCm, float *dD, float *dbias, float *dh0,
                                const int *lengths, int B, int N, int C, int S, int G, la_step step, la_dtype dt,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    la::Scan a = la::scan_of(X, x_stride, Dt, dt_stride, A, Bm, b_stride, Cm, c_stride, D, bias, B, N, C, S, G, step);
    a.first = dlast, a.end = dh0, a.dY = dY, a.dX = dX, a.dDt = dDt, a.lengths = lengths, a.saved = (float *)saved;
    const la_status s = la::check(a, step, dt);
    if (s != LA_OK) return s;
    if (!dY || !dX || !dDt || !dBm || !dCm) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), tb = (size_t)B * N * C * e, vb = (size_t)B * N * G * S * e;
    if (!la::aligned_to(dBm, e) || !la::aligned_to(dCm, e) || !la::aligned_to(dA, 4) || !la::aligned_to(dD, 4) || !la::aligned_to(dbias, 4))
        return LA_ERR_ALIGN;
    la::lay_out(a);
    const la::Room room(a, true);
    const size_t kept = la_selective_saved_bytes(B, N, C, S);
    if (!workspace || workspace_bytes < room.bytes || !la::aligned_to(workspace, 256)) return LA_ERR_WORKSPACE;
    if (!saved || saved_bytes < kept || !la::aligned_to(saved, 256)) return LA_ERR_WORKSPACE;
    const la::Inputs in(a, dt);
    la::Range ins[11];
    for (int k = 0; k < 9; ++k) ins[k] = in.r[k];
    ins[9] = {dY, tb}, ins[10] = {saved, kept};
    const la::Range outs[] = {{dX, tb}, {dDt, tb}, {dA, (size_t)C * S * 4}, {dBm, vb}, {dCm, vb}, {dD, (size_t)C * 4},
                              {dbias, (size_t)C * 4}, {dh0, (size_t)B * C * S * 4}, {workspace, room.bytes}};
    if (la::any_alias(ins, 11, outs, 9)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    float *const ws = (float *)workspace;
    a.sums = ws + room.sums, a.spans = ws + room.spans, a.shares = ws + room.shares;
    a.dA = dA ? ws + room.dA : nullptr, a.dd = ws + room.dd;
    const dim3 grid((unsigned)((size_t)B * a.columns * a.segs));
    const hipStream_t st = (hipStream_t)hip_stream;
    la::by_shape(S, [&](auto P, auto W) {
        constexpr int p = decltype(P)::value, w = decltype(W)::value;
        const size_t values = ((size_t)B * G * a.tiles * la::shares_of(S) + 255) / 256;
        const dim3 all((unsigned)(values < 1 << 20 ? values : 1 << 20));
        if (dt == LA_F32) {
            if (a.segs > 1) la::k_selective_back<float, p, w, false><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective_back<float, p, w, true><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective_vectors<float, p, w><<<all, dim3(256), 0, st>>>(a, (float *)dBm, (float *)dCm);
        } else {
            if (a.segs > 1) la::k_selective_back<la::bf16_t, p, w, false><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective_back<la::bf16_t, p, w, true><<<grid, dim3(64 * w), 0, st>>>(a);
            la::k_selective_vectors<la::bf16_t, p, w><<<all, dim3(256), 0, st>>>(a, (la::bf16_t *)dBm, (la::bf16_t *)dCm);
        }
    });
    if (dA || dD || dbias) la::k_selective_join<<<dim3((C + 63) / 64, S + 2), dim3(256), 0, st>>>(a, dA, dD, dbias);
    return la::done();
}

la_status la_selective_step(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                            const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D,
                            const float *bias, float *state, void *Y, int B, int T, int C, int S, int G, la_step step,
                            la_dtype dt, void *hip_stream)
{
    la::Scan a = la::scan_of(X, x_stride, Dt, dt_stride, A, Bm, b_stride, Cm, c_stride, D, bias, B, T, C, S, G, step);
    a.Y = Y, a.end = state;
    const la_status s = la::check(a, step, dt);
    if (s != LA_OK) return s;
    if (!state || !Y) return LA_ERR_NULL;
    const la::Inputs in(a, dt);
    const la::Range outs[] = {{Y, (size_t)B * T * C * la::size_of(dt)}, {state, (size_t)B * C * S * 4}};
    if (la::any_alias(in.r, 9, outs, 2)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    a.group = C / G;
    int L = 1;
    while (L * 4 < S) L *= 2;
    const dim3 grid((unsigned)(((size_t)B * C * L + 255) / 256)), block(256);
    if (dt == LA_F32) la::k_selective_step<float, 4><<<grid, block, 0, (hipStream_t)hip_stream>>>(a, state, L);
    else la::k_selective_step<la::bf16_t, 4><<<grid, block, 0, (hipStream_t)hip_stream>>>(a, state, L);
    return la::done();
}

}  // extern "C"
