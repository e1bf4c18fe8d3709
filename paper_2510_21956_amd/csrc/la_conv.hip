// Short causal convolution along the rows, one filter of W taps a channel, with an activation: forward, backward, in steps.
//
// A lane takes V neighbouring channels down a run of rows and keeps the W - 1 rows before the current one in
// registers: every row is read once, but for the W - 1 rows in front of a run.  Rows may start at any element: the
// lane at a row's end takes its last V channels once more.
//
// Bound by HBM: 2 W operations and the activation a row and channel, twice to three times that backward, for two tensors
// moved forward and three backward.  8 x 2048 rows of 2048 channels, 4 taps, bf16: forward 28 us, 4.8 TB/s; backward 55,
// 3.7 TB/s, with the join of dw 4 of them; 32 x 2048 of 4096, 213 and 351, 5.0 and 4.6 TB/s.
#include <limits.h>

#include "la_checks.h"
#include "la_common.h"
#include "la_scalar.h"

namespace la {
namespace {

// V neighbouring channels, as they are stored and in registers.
template <typename T, int V>
struct Piece {
    T x[V];
};
template <int V>
struct Wide {
    float x[V];
};
template <typename T, int V>
__device__ __forceinline__ Piece<T, V> fetch(const void *p)
{
    Piece<T, V> r;
    __builtin_memcpy(&r, p, sizeof r);
    return r;
}
template <typename T, int V>
__device__ __forceinline__ Wide<V> widened(const Piece<T, V> &p)
{
    Wide<V> r;
#pragma unroll
    for (int k = 0; k < V; ++k) r.x[k] = load_elem(p.x, k);
    return r;
}
template <typename T, int V>
__device__ __forceinline__ void put(void *p, const Wide<V> &r)
{
    Piece<T, V> s;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if constexpr (sizeof(T) == 4) s.x[k] = r.x[k];
        else {
            const __bf16 c = (__bf16)r.x[k];
            __builtin_memcpy(&s.x[k], &c, 2);
        }
    }
    __builtin_memcpy(p, &s, sizeof s);
}

struct Conv {
    const void *X, *Wt, *bias, *state;
    void *Y, *last;               // forward
    const void *dY, *dlast;       // backward
    void *dX, *dstate;
    float *shares;                // [shares, W + 1, C] sums of dw and dbias
    const int *lengths;
    size_t xs, items, from;       // from: the launch's first item
    int B, N, C, run, runs, lanes, columns;
};
// Pieces of V channels in a row.
__host__ __device__ __forceinline__ int pieces_of(int C, int V) { return (C - 1) / V + 1; }
__device__ __forceinline__ int rows_of(const Conv &a, int b)
{
    return a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
}

// Taps and bias of a lane's channels.
template <typename WT, int V, int W>
struct Taps {
    Wide<V> w[W], bias;
    __device__ __forceinline__ Taps(const Conv &a, int c)
    {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            bias.x[k] = a.bias ? load_elem((const WT *)a.bias, c + k) : 0.f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j].x[k] = load_elem((const WT *)a.Wt, (size_t)(c + k) * W + j);
        }
    }
};

// Row t of the sequence, t < n; rows before the first are the carried ones.
template <typename T, int V, int W>
__device__ __forceinline__ Piece<T, V> row_at(const Conv &a, int b, int t, int c)
{
    if (t >= 0) return fetch<T, V>((const T *)a.X + ((size_t)b * a.N + t) * a.xs + c);
    if (a.state) return fetch<T, V>((const T *)a.state + ((size_t)b * (W - 1) + t + W - 1) * a.C + c);
    return Piece<T, V>{};
}

// What the activation is given, of rows that stand in a ring of W, the oldest at I % W.
template <int I, typename WT, int V, int W>
__device__ __forceinline__ Wide<V> before_act(const Taps<WT, V, W> &taps, const Wide<V> (&past)[W])
{
    Wide<V> v = taps.bias;
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
        for (int k = 0; k < V; ++k) v.x[k] = fmaf(taps.w[j].x[k], past[(I + j) % W].x[k], v.x[k]);
    return v;
}
// Rows that a loop takes together: whole turns of the ring, four at least, and as many are asked for ahead.
template <int W>
constexpr int rows_together = W >= 4 ? W : W == 3 ? 6 : 4;

// Items: (sequence, run of rows, V channels), then (sequence, carried row, V channels) where `last` is wanted.
template <typename T, typename WT, int V, int W, int ACT>
__global__ void __launch_bounds__(256) k_conv(Conv a)
{
    const size_t i = a.from + (size_t)blockIdx.x * 256 + threadIdx.x;
    const int pieces = pieces_of(a.C, V);
    if (i >= a.items) {
        const size_t k = i - a.items;
        if (!a.last || k >= (size_t)a.B * (W - 1) * pieces) return;
        const int c = min((int)(k % pieces) * V, a.C - V), j = (int)(k / pieces % (W - 1)), b = (int)(k / pieces / (W - 1));
        const Piece<T, V> p = row_at<T, V, W>(a, b, rows_of(a, b) - (W - 1) + j, c);
        __builtin_memcpy((T *)a.last + ((size_t)b * (W - 1) + j) * a.C + c, &p, sizeof p);
        return;
    }
    const int c = min((int)(i % pieces) * V, a.C - V), r = (int)(i / pieces % a.runs), b = (int)(i / pieces / a.runs);
    const int n = rows_of(a, b), t0 = r * a.run, end = min(a.N, t0 + a.run), stop = min(n, end);
    T *Y = (T *)a.Y + ((size_t)b * a.N + t0) * a.C + c;
    int t = t0;
    if (t < stop) {
        const Taps<WT, V, W> taps(a, c);
        Wide<V> past[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) past[j] = widened(row_at<T, V, W>(a, b, t0 - (W - 1) + j, c));
        const T *X = (const T *)a.X + ((size_t)b * a.N + t0) * a.xs + c;
        constexpr int U = rows_together<W>;
        Piece<T, V> next[U];
#pragma unroll
        for (int k = 0; k < U; ++k) next[k] = fetch<T, V>(X + (size_t)min(k, stop - 1 - t0) * a.xs);
        for (; t < stop; t += U)
            each<U>([&](auto k_) {
                constexpr int k = decltype(k_)::value;
                if (t + k >= stop) return;
                past[(k + W - 1) % W] = widened(next[k]);
                next[k] = fetch<T, V>(X + (size_t)(min(t + k + U, stop - 1) - t0) * a.xs);
                Wide<V> v = before_act<k>(taps, past);
                if (ACT == LA_ACT_SILU)
#pragma unroll
                    for (int m = 0; m < V; ++m) {
                        float f, rest;
                        sigmoid<sizeof(T) == 4>(v.x[m], f, rest);
                        v.x[m] *= f;
                    }
                put<T, V>(Y, v);
                Y += a.C;
            });
        t = stop;
    }
    for (; t < end; ++t) {
        put<T, V>(Y, Wide<V>{});
        Y += a.C;
    }
}

// Backward.  A workgroup's four waves take runs of rows that follow one another, `lanes` lanes to a run; e of the W - 1
// rows behind a run is formed once more.  Sums of dw and dbias: a lane's rows, then the runs of a wave and of the
// workgroup, whose share k_conv_join adds to the others'.
template <typename T, typename WT, int V, int W, int U, int ACT>
__global__ void __launch_bounds__(256) k_conv_back(Conv a)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, per = 64 / a.lanes;
    const int column = (int)(blockIdx.x % a.columns), share = (int)(blockIdx.x / a.columns);
    const int cv = column * a.lanes + lane % a.lanes;
    const int pieces = pieces_of(a.C, V);
    const bool mine = cv < pieces;  // else a channel behind the last: that of the lane before
    const int cw = min(cv, pieces - 1) * V, c = min(cw, a.C - V), first = cw - c;  // channels before `first` are another lane's
    const size_t q = ((size_t)share * 4 + wave) * per + lane / a.lanes;  // the run
    Wide<V> dw[W], db{};
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j] = Wide<V>{};
    if (mine && q < (size_t)a.B * a.runs) {
        const int b = (int)(q / a.runs), t0 = (int)(q % a.runs) * a.run, end = min(a.N, t0 + a.run), n = rows_of(a, b);
        const size_t row0 = (size_t)b * a.N;
        const Taps<WT, V, W> taps(a, c);
        const int own = min(n, end), stop = min(n, end + W - 1);  // e of rows [t0, stop)
        // e and x of the last W rows, in rings
        Wide<V> e[W], past[W];
#pragma unroll
        for (int j = 0; j < W; ++j) e[j] = Wide<V>{};
        if (t0 < stop)
#pragma unroll
            for (int j = 0; j < W - 1; ++j) past[j] = widened(row_at<T, V, W>(a, b, t0 - (W - 1) + j, c));
        const T *X = (const T *)a.X + row0 * a.xs + c, *dY = (const T *)a.dY + row0 * a.C + c;
        T *dX = (T *)a.dX + row0 * a.C + c;
        Piece<T, V> nx[U], ny[U];
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (t0 < stop) {
                const int m = min(t0 + k, stop - 1);
                nx[k] = fetch<T, V>(X + (size_t)m * a.xs), ny[k] = fetch<T, V>(dY + (size_t)m * a.C);
            }
        // dx of row s = t - (W - 1) is complete once e_t is there; rows before the first are the carried ones
        const int from = n - (W - 1);  // the first row that is carried on
        const T *Xt = X + (size_t)(t0 + U) * a.xs, *dYt = dY + (size_t)(t0 + U) * a.C;  // rows asked for next
        T *dXt = dX + (ptrdiff_t)(t0 - (W - 1)) * a.C;
        bool endless = false;  // a tap of the wave's is infinite, or NaN: 0 times that is not 0
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int q = 0; q < V; ++q) endless = endless || !(fabsf(taps.w[j].x[q]) < INFINITY);
        endless = __any(endless);
        // PLAIN: all rows of the turn are the run's own, and so is what they complete and ask for
        auto turn = [&](int t1, auto plain_) {
            constexpr bool PLAIN = decltype(plain_)::value;
            each<U>([&](auto k_) {
                constexpr int k = decltype(k_)::value, now = (k + W - 1) % W;
                const int t = t1 + k;
                if (!PLAIN && t >= end + W - 1) return;
                if (!PLAIN) e[now] = Wide<V>{};
                if (PLAIN || t < stop) {
                    past[now] = widened(nx[k]);
                    Wide<V> g = widened(ny[k]);
                    if (PLAIN) nx[k] = fetch<T, V>(Xt), ny[k] = fetch<T, V>(dYt);
                    else {
                        const int m = min(t + U, stop - 1);
                        nx[k] = fetch<T, V>(X + (size_t)m * a.xs), ny[k] = fetch<T, V>(dY + (size_t)m * a.C);
                    }
                    if (ACT == LA_ACT_SILU) {
                        const Wide<V> v = before_act<k>(taps, past);
#pragma unroll
                        for (int q = 0; q < V; ++q) {
                            float f, rest;
                            sigmoid<sizeof(T) == 4>(v.x[q], f, rest);
                            g.x[q] *= f * fmaf(v.x[q], rest, 1.f);
                        }
                    }
                    e[now] = g;
                    if (PLAIN || t < own) {
#pragma unroll
                        for (int q = 0; q < V; ++q) {
                            db.x[q] += g.x[q];
#pragma unroll
                            for (int j = 0; j < W; ++j) dw[j].x[q] = fmaf(g.x[q], past[(k + j) % W].x[q], dw[j].x[q]);
                        }
                    }
                }
                T *const to = dXt;
                Xt += a.xs, dYt += a.C, dXt += a.C;
                const int s = t - (W - 1);
                if (!PLAIN && s < t0 && (t0 > 0 || !a.dstate)) return;
                // e of row s + j is in place (k + j) % W
                Wide<V> d{};
#pragma unroll
                for (int j = 0; j < W; ++j)
#pragma unroll
                    for (int q = 0; q < V; ++q) d.x[q] = fmaf(taps.w[W - 1 - j].x[q], e[(k + j) % W].x[q], d.x[q]);
                if (!PLAIN && endless) {  // without the products with rows that there are not
                    d = Wide<V>{};
#pragma unroll
                    for (int j = 0; j < W; ++j)
#pragma unroll
                        for (int q = 0; q < V; ++q)
                            if (s + j >= 0 && s + j < n) d.x[q] = fmaf(taps.w[W - 1 - j].x[q], e[(k + j) % W].x[q], d.x[q]);
                }
                if (!PLAIN && a.dlast && s >= from && s < n) {
                    const Wide<V> l = widened(fetch<T, V>((const T *)a.dlast + ((size_t)b * (W - 1) + s - from) * a.C + c));
#pragma unroll
                    for (int q = 0; q < V; ++q) d.x[q] += l.x[q];
                }
                if (PLAIN || s >= 0) put<T, V>(to, d);
                else put<T, V>((T *)a.dstate + ((size_t)b * (W - 1) + s + W - 1) * a.C + c, d);
            });
        };
        const int plain = min(own, min(stop - U, from + W - 1));  // up to where
        for (int t1 = t0; t1 < end + W - 1; t1 += U) {
            if (__all(t1 >= t0 + W - 1 && t1 + U <= plain)) turn(t1, std::true_type());
            else turn(t1, std::false_type());
        }
    }
    if (!a.shares) return;
    __shared__ float sums[4][W + 1][64][V];
    for (int m = a.lanes; m < 64; m *= 2)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            db.x[k] += __shfl_xor(db.x[k], m);
#pragma unroll
            for (int j = 0; j < W; ++j) dw[j].x[k] += __shfl_xor(dw[j].x[k], m);
        }
    if (lane < a.lanes)
#pragma unroll
        for (int k = 0; k < V; ++k) {
            sums[wave][W][lane][k] = db.x[k];
#pragma unroll
            for (int j = 0; j < W; ++j) sums[wave][j][lane][k] = dw[j].x[k];
        }
    block_sync();
    if (wave == 0 && lane < a.lanes && mine)
#pragma unroll
        for (int j = 0; j <= W; ++j)
#pragma unroll
            for (int k = 0; k < V; ++k)
                if (k >= first)
                    a.shares[((size_t)share * (W + 1) + j) * a.C + c + k] =
                        (sums[0][j][lane][k] + sums[1][j][lane][k]) + (sums[2][j][lane][k] + sums[3][j][lane][k]);
}

// dw and dbias from the workgroups' shares: 64 channels a workgroup, from c0 on, its waves take every 16th share each.
template <int W>
__global__ void __launch_bounds__(1024) k_conv_join(const float *shares, float *dW, float *db, int count, int C, int c0)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = c0 + blockIdx.x * 64 + lane, j = blockIdx.y;
    float s = 0.f;
    if (c < C)
        for (int k = wave; k < count; k += 16) s += shares[((size_t)k * (W + 1) + j) * C + c];
    sums[wave][lane] = s;
    block_sync();
    if (wave || c >= C) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += sums[k][lane];
    if (j < W) {
        if (dW) dW[(size_t)c * W + j] = s;
    } else if (db) db[c] = s;
}

// T rows on the carried ones: one channel a lane.
template <typename T, typename WT, int W, int ACT>
__global__ void __launch_bounds__(256) k_conv_step(Conv a)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)a.B * a.C) return;
    const int b = (int)(i / a.C), c = (int)(i - (size_t)b * a.C);
    const Taps<WT, 1, W> taps(a, c);
    T *state = (T *)a.last + (size_t)b * (W - 1) * a.C + c;
    T kept[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) kept[j] = state[(size_t)j * a.C];
    for (int t = 0; t < a.N; ++t) {
        kept[W - 1] = ((const T *)a.X)[((size_t)b * a.N + t) * a.xs + c];
        float v = taps.bias.x[0];
#pragma unroll
        for (int j = 0; j < W; ++j) v = fmaf(taps.w[j].x[0], load_elem(kept, j), v);
        if (ACT == LA_ACT_SILU) {
            float f, rest;
            sigmoid<sizeof(T) == 4>(v, f, rest);
            v *= f;
        }
        store_elem((T *)a.Y, ((size_t)b * a.N + t) * a.C + c, v);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) kept[j] = kept[j + 1];
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) state[(size_t)j * a.C] = kept[j];
}

constexpr int kMostTaps = 8;
constexpr size_t kMostItems = 1u << 31;  // of a launch, whose threads are counted in 32 bits: with `last`, up to 7 * 2^31 in all
constexpr int kMostJoined = 1 << 27;         // channels of a launch of k_conv_join, 16 threads each

// Channels a lane takes: four, two where the taps would fill the registers, backward two; one where a row is shorter.  More of
// them leave fewer waves, whose loads are not enough: 8 x 2048 rows of 2048, bf16, forward 28 us, with eight 36; backward
// 55, with four 74 and with eight 85.
template <int W>
constexpr int wide_of = W > 4 ? 2 : 4;
constexpr int kWideBack = 2;

// Backward, up to four taps: twice the rows together where a run has as many as this (8 x 2048 rows of 2048, runs of 128:
// 55 us, else 60; 2 x 3001 rows, runs of 32: 26 us, with twice the rows together 27).
constexpr int kLongRun = 64;

// Rows of a run: enough waves to fill the chip, and few rows read twice.  4096 waves forward, 2048 backward, whose rows
// behind a run cost more (2 x 3001 rows of 2048, bf16: 13 us forward, with 2048 waves 14; 26 backward, with 4096 32).
int run_rows(int B, int N, size_t pieces, int waves)
{
    int run = 128;
    while (run > 16 && (double)B * ((N + run - 1) / run) * pieces < 64.0 * waves) run /= 2;
    return run;
}

template <int W, typename F>
void by_taps(int taps, F f)
{
    if (taps == W) f(std::integral_constant<int, W>());
    else if constexpr (W < kMostTaps) by_taps<W + 1>(taps, f);
}
// f(T *, WT *, activation as a constant, taps as a constant)
template <typename F>
void by_kind(la_dtype dt, la_dtype wt, la_act act, int taps, F f)
{
    auto with = [&](auto *t, auto *w) {
        by_taps<2>(taps, [&](auto W) {
            if (act == LA_ACT_SILU) f(t, w, std::integral_constant<int, LA_ACT_SILU>(), W);
            else f(t, w, std::integral_constant<int, LA_ACT_NONE>(), W);
        });
    };
    if (dt == LA_F32) with((float *)nullptr, (float *)nullptr);
    else if (wt == LA_F32) with((bf16_t *)nullptr, (float *)nullptr);
    else with((bf16_t *)nullptr, (bf16_t *)nullptr);
}

la_status check(size_t stride, int B, int N, int C, int W, la_act act, la_dtype dt, la_dtype wt)
{
    if (B < 1 || N < 1 || C < 1 || N > 1 << 30 || C > INT_MAX - 256 || W < 2 || W > kMostTaps || stride < (size_t)C) return LA_ERR_SHAPE;
    if (!real_type(dt) || (wt != LA_F32 && wt != dt) || (act != LA_ACT_NONE && act != LA_ACT_SILU)) return LA_ERR_UNSUPPORTED;
    if ((double)B * N * (double)stride >= 1099511627776.0) return LA_ERR_SHAPE;             // 2^40
    if ((double)B * C * ((N + 15) / 16) >= 2147483648.0) return LA_ERR_SHAPE;  // runs' channels
    return LA_OK;
}
size_t span_of(size_t rows, size_t stride, int C, size_t e) { return ((rows - 1) * stride + C) * e; }

la_status done() { return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH; }

// How the backward pass is laid out.
struct Back {
    int V, lanes, run, runs, columns, count;  // count: workgroups down the runs, shares
};
Back back_of(int B, int N, int C, int most)
{
    Back p;
    p.V = C < most ? 1 : most;
    const int pieces = pieces_of(C, p.V);
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < pieces) p.lanes *= 2;
    p.columns = (pieces + p.lanes - 1) / p.lanes;
    p.run = run_rows(B, N, (size_t)p.columns * p.lanes, 2048);
    p.runs = (N + p.run - 1) / p.run;
    const int of = 4 * (64 / p.lanes);
    p.count = (int)(((size_t)B * p.runs + of - 1) / of);
    return p;
}

}  // namespace
}  // namespace la

extern "C" {

size_t la_conv_workspace_bytes(int B, int N, int C, int W)
{
    if (la::check(C < 1 ? 1 : C, B, N, C, W, LA_ACT_NONE, LA_F32, LA_F32) != LA_OK) return 0;
    return la::round_up((size_t)la::back_of(B, N, C, la::kWideBack).count * (W + 1) * C * 4, 256);
}

la_status la_conv_forward(const void *X, size_t x_stride, const void *Wt, const void *bias, const void *state, void *Y, void *last,
                          const int *lengths, int B, int N, int C, int W, la_act act, la_dtype dt, la_dtype wt, void *hip_stream)
{
    const la_status s = la::check(x_stride, B, N, C, W, act, dt, wt);
    if (s != LA_OK) return s;
    if (!X || !Wt || !Y) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), we = la::size_of(wt), tb = (size_t)B * N * C * e, sb = (size_t)B * (W - 1) * C * e;
    for (const void *p : {X, state, (const void *)Y, (const void *)last})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if (!la::aligned_to(Wt, we) || !la::aligned_to(bias, we) || !la::aligned_to(lengths, 4)) return LA_ERR_ALIGN;
    const la::Range ins[] = {{X, la::span_of((size_t)B * N, x_stride, C, e)}, {Wt, (size_t)C * W * we}, {bias, C * we}, {state, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{Y, tb}, {last, sb}};
    if (la::any_alias(ins, 5, outs, 2)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Conv a{};
    a.X = X, a.xs = x_stride, a.Wt = Wt, a.bias = bias, a.state = state, a.Y = Y, a.last = last, a.lengths = lengths;
    a.B = B, a.N = N, a.C = C;
    la::by_kind(dt, wt, act, W, [&](auto *t, auto *w, auto act_, auto taps) {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(w)> WT;
        constexpr int K = decltype(taps)::value, V = la::wide_of<K>;
        auto go = [&](auto wide) {
            constexpr int U = decltype(wide)::value;
            const size_t each = la::pieces_of(C, U);
            a.run = la::run_rows(B, N, each, 4096);
            a.runs = (N + a.run - 1) / a.run;
            a.items = (size_t)B * a.runs * each;
            const size_t all = a.items + (last ? (size_t)B * (K - 1) * each : 0);
            for (a.from = 0; a.from < all; a.from += la::kMostItems) {
                const size_t n = all - a.from < la::kMostItems ? all - a.from : la::kMostItems;
                la::k_conv<T, WT, U, K, decltype(act_)::value><<<dim3((unsigned)((n + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream>>>(a);
            }
        };
        if (C >= V) go(std::integral_constant<int, V>());
        else go(std::integral_constant<int, 1>());
    });
    return la::done();
}

la_status la_conv_backward(const void *X, size_t x_stride, const void *Wt, const void *bias, const void *state, const void *dY,
                           const void *dlast, void *dX, float *dW, float *dbias, void *dstate, const int *lengths,
                           int B, int N, int C, int W, la_act act, la_dtype dt, la_dtype wt,
                           void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const la_status s = la::check(x_stride, B, N, C, W, act, dt, wt);
    if (s != LA_OK) return s;
    if (!X || !Wt || !dY || !dX) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), we = la::size_of(wt), tb = (size_t)B * N * C * e, sb = (size_t)B * (W - 1) * C * e;
    for (const void *p : {X, state, dY, dlast, (const void *)dX, (const void *)dstate})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if (!la::aligned_to(Wt, we) || !la::aligned_to(bias, we) || !la::aligned_to(lengths, 4) || !la::aligned_to(dW, 4) || !la::aligned_to(dbias, 4))
        return LA_ERR_ALIGN;
    const size_t need = dW || dbias ? la_conv_workspace_bytes(B, N, C, W) : 0;
    if (need && (!workspace || workspace_bytes < need || !la::aligned_to(workspace, 256))) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{X, la::span_of((size_t)B * N, x_stride, C, e)}, {Wt, (size_t)C * W * we}, {bias, C * we}, {state, sb},
                             {dY, tb}, {dlast, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{dX, tb}, {dW, (size_t)C * W * 4}, {dbias, (size_t)C * 4}, {dstate, sb}, {workspace, need}};
    if (la::any_alias(ins, 7, outs, 5)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Conv a{};
    a.X = X, a.xs = x_stride, a.Wt = Wt, a.bias = bias, a.state = state, a.lengths = lengths;
    a.dY = dY, a.dlast = dlast, a.dX = dX, a.dstate = dstate, a.shares = need ? (float *)workspace : nullptr;
    a.B = B, a.N = N, a.C = C;
    const hipStream_t st = (hipStream_t)hip_stream;
    la::by_kind(dt, wt, act, W, [&](auto *t, auto *w, auto act_, auto taps) {
        typedef std::remove_pointer_t<decltype(t)> T;
        typedef std::remove_pointer_t<decltype(w)> WT;
        constexpr int K = decltype(taps)::value, V = la::kWideBack;
        const la::Back p = la::back_of(B, N, C, V);
        a.lanes = p.lanes, a.columns = p.columns, a.run = p.run, a.runs = p.runs;
        auto go = [&](auto wide, auto rows) {
            la::k_conv_back<T, WT, decltype(wide)::value, K, decltype(rows)::value, decltype(act_)::value>
                <<<dim3((unsigned)p.columns * p.count), dim3(256), 0, st>>>(a);
        };
        const std::integral_constant<int, la::rows_together<K>> few;
        const std::integral_constant<int, la::rows_together<K> * (K > 4 ? 1 : 2)> many;
        if (C < V) go(std::integral_constant<int, 1>(), few);
        else if (p.run >= la::kLongRun) go(std::integral_constant<int, V>(), many);
        else go(std::integral_constant<int, V>(), few);
        if (need)
            for (int c0 = 0; c0 < C; c0 += la::kMostJoined) {
                const int n = C - c0 < la::kMostJoined ? C - c0 : la::kMostJoined;
                la::k_conv_join<K><<<dim3((n + 63) / 64, K + 1), dim3(1024), 0, st>>>(a.shares, dW, dbias, p.count, C, c0);
                if (n < la::kMostJoined) break;
            }
    });
    return la::done();
}

la_status la_conv_step(const void *X, size_t x_stride, const void *Wt, const void *bias, void *state, void *Y, int B, int T, int C,
                       int W, la_act act, la_dtype dt, la_dtype wt, void *hip_stream)
{
    const la_status s = la::check(x_stride, B, T, C, W, act, dt, wt);
    if (s != LA_OK) return s;
    if (!X || !Wt || !state || !Y) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), we = la::size_of(wt), tb = (size_t)B * T * C * e, sb = (size_t)B * (W - 1) * C * e;
    for (const void *p : {X, (const void *)state, (const void *)Y})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if (!la::aligned_to(Wt, we) || !la::aligned_to(bias, we)) return LA_ERR_ALIGN;
    const la::Range ins[] = {{X, la::span_of((size_t)B * T, x_stride, C, e)}, {Wt, (size_t)C * W * we}, {bias, C * we}};
    const la::Range outs[] = {{Y, tb}, {state, sb}};
    if (la::any_alias(ins, 3, outs, 2)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Conv a{};
    a.X = X, a.xs = x_stride, a.Wt = Wt, a.bias = bias, a.last = state, a.Y = Y;
    a.B = B, a.N = T, a.C = C;
    la::by_kind(dt, wt, act, W, [&](auto *t, auto *w, auto act_, auto taps) {
        typedef std::remove_pointer_t<decltype(t)> E;
        typedef std::remove_pointer_t<decltype(w)> WT;
        la::k_conv_step<E, WT, decltype(taps)::value, decltype(act_)::value>
            <<<dim3((unsigned)(((size_t)B * C + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream>>>(a);
    });
    return la::done();
}

}  // extern "C"
