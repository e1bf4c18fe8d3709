// Root-mean-square norm of rows with the residual's addition, its backward pass, and rows in 8 bits.
//
// All of it is one pass over the rows, bound by HBM: a row stays in the registers of the lanes that share it
// (8 to 1024 of them, eight neighbouring elements to a lane and step), from the sum of its squares to the
// normalised row; nothing is read twice.
#include "la_checks.h"
#include "la_eight.h"

namespace la {
namespace {

// L lanes share a row and take K steps of 8 L elements each; a workgroup has max(L, 256) lanes.  L = 0: the whole
// workgroup shares a row, as many waves as it takes.
template <int L>
struct Share {
    static constexpr int NT = L > 256 || L == 0 ? 1024 : 256, ROWS = L ? NT / L : 1;
};
template <int L>
__device__ __forceinline__ int row_lanes()
{
    return L ? L : (int)blockDim.x;
}

// The sum over the lanes that share a row, in every one of them.
template <int L>
__device__ __forceinline__ float row_sum(float s, float *lds)
{
#pragma unroll
    for (int m = (L < 64 && L ? L : 64) / 2; m >= 1; m >>= 1) s += __shfl_xor(s, m);
    if constexpr (L > 64 || L == 0) {
        const int wave = threadIdx.x / 64, waves = row_lanes<L>() / 64;
        block_sync();  // the shares of the row before have been read
        if (threadIdx.x % 64 == 0) lds[wave] = s;
        block_sync();
        const int first = wave / waves * waves;
        s = 0.f;
        for (int v = 0; v < waves; ++v) s += lds[first + v];
    }
    return s;
}

struct Norm {
    const void *X, *R, *W;
    void *Y, *S;
    uint8_t *Yp, *K, *Kp;
    float *rstd;
    size_t rows;
    int C;
    float eps;
    int yt, kt;  // la_dtype
};

template <typename T, typename TW, int L, int K>
__global__ void __launch_bounds__(Share<L>::NT) k_norm(Norm a)
{
    constexpr bool SHORT = L == 8;
    __shared__ float lds[Share<L>::NT / 64];
    const int lanes = row_lanes<L>(), lane = threadIdx.x % lanes, C = a.C, G = (C + kGroup - 1) / kGroup;
    const size_t step = (size_t)gridDim.x * Share<L>::ROWS;
    for (size_t base = (size_t)blockIdx.x * Share<L>::ROWS; base < a.rows; base += step) {
        const size_t row = base + threadIdx.x / lanes;
        const bool here = row < a.rows;
        const size_t at = (here ? row : 0) * C;
        Eight t[K];
        float ss = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Span p((k * lanes + lane) * 8, C, here);
            t[k] = load8<SHORT>((const T *)a.X + at, p, C);
            if (a.R) {
                const Eight r = load8<SHORT>((const T *)a.R + at, p, C);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[k].x[j] += r.x[j];
                t[k] = widen<T>(narrow<T>(t[k]));  // as it is stored: what the backward pass will read
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) ss += t[k].x[j] * t[k].x[j];
        }
        ss = row_sum<L>(ss, lds);
        const float rstd = 1.f / sqrtf(ss / (float)C + a.eps);
        if (here && lane == 0 && a.rstd) a.rstd[row] = rstd;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Span p((k * lanes + lane) * 8, C, here);
            if (a.S) store8<true>((T *)a.S + at, t[k], p);
            if (a.K) pack8(t[k], a.K + at, a.Kp + (here ? row : 0) * G, p, a.kt == LA_I8);
            Eight y = t[k];
            if (a.W) {
                const Eight w = load8<SHORT>((const TW *)a.W, p, C);
#pragma unroll
                for (int j = 0; j < 8; ++j) y.x[j] = y.x[j] * rstd * w.x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) y.x[j] *= rstd;
            }
            if (a.Yp) pack8(y, (uint8_t *)a.Y + at, a.Yp + (here ? row : 0) * G, p, a.yt == LA_I8);
            else store8<true>((T *)a.Y + at, y, p);
        }
    }
}

struct NormBack {
    const void *S, *W, *dY, *dS;
    const uint8_t *Sp;
    const float *rstd;
    void *dX;
    float *parts;  // [gridDim.x, C] shares of dw
    size_t rows;
    int C, st;
};

// A row's tensors as they are stored, one lane's share.  Where the sum was kept in 8 bits its codes and power take
// the place of its elements.
template <typename T, int K>
struct Row {
    Stored<T> s[K], d[K], g[K];
    float rstd;
};

// Rows are requested AHEAD rows before they are worked on, as far as there are registers to hold them: 16384 rows of
// 2056, bf16, one row ahead 79 us, two 61 (of 2048, four waves to a row, 58 either way); 30000 of 770, fp32, one 78,
// two, for which fewer workgroups run at once, 88.
template <typename T, typename TW, int L, int K>
__global__ void __launch_bounds__(Share<L>::NT) k_norm_back(NormBack a)
{
    constexpr int AHEAD = K > 1 ? 0 : sizeof(T) == 2 ? 2 : 1, TURNS = AHEAD ? AHEAD : 1;
    constexpr bool HOLD = K == 1;  // registers for the weights as well
    constexpr bool SHORT = L == 8;
    __shared__ float lds[Share<L>::NT / 64];
    __shared__ float shares[Share<L>::ROWS > 1 ? Share<L>::NT * 8 * K : 1];
    const int lanes = row_lanes<L>(), lane = threadIdx.x % lanes, C = a.C, G = (C + kGroup - 1) / kGroup;
    const size_t step = (size_t)gridDim.x * Share<L>::ROWS;
    const auto weights = [&](int k) {
        Eight w;
        if (a.W) w = load8<SHORT>((const TW *)a.W, Span((k * lanes + lane) * 8, C), C);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) w.x[j] = 1.f;
        return w;
    };
    Eight w[K], dw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (HOLD) w[k] = weights(k);
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[k].x[j] = 0.f;
    }
    const auto request = [&](size_t row) {
        Row<T, K> r;
        const bool here = row < a.rows;
        const size_t at = (here ? row : 0) * C;
        r.rstd = a.rstd[here ? row : 0];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Span p((k * lanes + lane) * 8, C, here);
            if (a.Sp) {
                const uint2 c = request_codes<SHORT>((const uint8_t *)a.S + at, p, C);
                r.s[k].w[0] = c.x, r.s[k].w[1] = c.y;
                r.s[k].w[2] = a.Sp[(here ? row : 0) * G + min(p.c / kGroup, G - 1)];
            } else r.s[k] = request8<SHORT>((const T *)a.S + at, p, C);
            r.d[k] = request8<SHORT>((const T *)a.dY + at, p, C);
            if (a.dS) r.g[k] = request8<SHORT>((const T *)a.dS + at, p, C);
        }
        return r;
    };
    Row<T, K> rows[TURNS];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        rows[u] = request((size_t)blockIdx.x * Share<L>::ROWS + threadIdx.x / lanes + u * step);
    for (size_t first = (size_t)blockIdx.x * Share<L>::ROWS; first < a.rows; first += TURNS * step)
#pragma unroll
        for (int u = 0; u < TURNS; ++u) {
            const size_t base = first + u * step;
            if (base >= a.rows) break;
            const size_t row = base + threadIdx.x / lanes;
            const bool here = row < a.rows;
            const size_t at = (here ? row : 0) * C;
            if (AHEAD == 0) rows[u] = request(row);
            const float rstd = rows[u].rstd;
            Eight n[K], d[K];
            Stored<T> g[K];
            float m = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Span p((k * lanes + lane) * 8, C, here);
                const Stored<T> &s = rows[u].s[k];
                n[k] = a.Sp ? values_of(settle(make_uint2(s.w[0], s.w[1]), p), s.w[2], a.st == LA_I8) : widen<T>(s, p);
                d[k] = widen<T>(rows[u].d[k], p);
                g[k] = rows[u].g[k];
            }
            if (AHEAD) rows[u] = request(row + AHEAD * step);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!HOLD) w[k] = weights(k);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    n[k].x[j] *= rstd;
                    dw[k].x[j] += d[k].x[j] * n[k].x[j];
                    d[k].x[j] *= w[k].x[j];
                    m += d[k].x[j] * n[k].x[j];
                }
            }
            const float mean = row_sum<L>(m, lds) / (float)C;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const Span p((k * lanes + lane) * 8, C, here);
#pragma unroll
                for (int j = 0; j < 8; ++j) d[k].x[j] = rstd * (d[k].x[j] - n[k].x[j] * mean);
                if (a.dS) {
                    const Eight s = widen<T>(g[k], p);
#pragma unroll
                    for (int j = 0; j < 8; ++j) d[k].x[j] += s.x[j];
                }
                store8<false>((T *)a.dX + at, d[k], p);
            }
        }
    if (!a.parts) return;
    float *out = a.parts + (size_t)blockIdx.x * C;
    if constexpr (Share<L>::ROWS > 1) {  // the workgroup's rows, in their order
        constexpr int W8 = L * 8 * K;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) shares[threadIdx.x / lanes * W8 + (k * lanes + lane) * 8 + j] = dw[k].x[j];
        block_sync();
        for (int c = threadIdx.x; c < C; c += Share<L>::NT) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < Share<L>::ROWS; ++r) s += shares[r * W8 + c];
            out[c] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            store8<false>(out, dw[k], Span((k * lanes + lane) * 8, C));
        }
    }
}

// dw from its shares, in a fixed order: sixteen channels a workgroup, whose 64 groups of lanes take a run of shares
// each (1024 shares of 2048 channels: 5.2 us, 7.0 with 64 channels and 16 runs).
__global__ void __launch_bounds__(1024) k_norm_join(const float *parts, float *dW, int n, int C)
{
    __shared__ float lds[64][16];
    const int channel = threadIdx.x % 16, run = threadIdx.x / 16, c = blockIdx.x * 16 + channel;
    const int per = (n + 63) / 64, end = min(n, (run + 1) * per);
    float s = 0.f;
    if (c < C)
#pragma unroll 8
        for (int i = run * per; i < end; ++i) s += parts[(size_t)i * C + c];
    lds[run][channel] = s;
    block_sync();
    if (run < 4) {  // one wave
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) s += lds[run * 16 + r][channel];
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if (run == 0 && c < C) dW[c] = s;
    }
}

// Tensors of one shape, blockIdx.y of them.
constexpr int kMostTensors = 4;
struct Batch {
    const void *X[kMostTensors];
    uint8_t *codes[kMostTensors], *powers[kMostTensors];
};

// Eight elements a lane; four lanes to a group, and as many to the last group of a row however short it is.
template <typename T>
__global__ void __launch_bounds__(256) k_pack(Batch a, size_t rows, int C, int ints)
{
    const T *X = (const T *)a.X[blockIdx.y];
    uint8_t *codes = a.codes[blockIdx.y], *powers = a.powers[blockIdx.y];
    const int G = (C + kGroup - 1) / kGroup, lanes = G * 4;
    const size_t total = rows * lanes, step = (size_t)gridDim.x * 256;
    for (size_t base = (size_t)blockIdx.x * 256; base < total; base += step) {
        const size_t i = base + threadIdx.x;
        const bool here = i < total;
        const size_t row = here ? i / lanes : 0;
        const Span p(here ? (int)(i - row * lanes) * 8 : 0, C, here);
        pack8(load8<true>(X + row * C, p, C), codes + row * C, powers + row * G, p, ints);
    }
}
template <typename T>
__global__ void __launch_bounds__(256) k_unpack(const uint8_t *codes, const uint8_t *powers, T *X, size_t rows, int C, int ints)
{
    const int G = (C + kGroup - 1) / kGroup, lanes = G * 4;
    const size_t total = rows * lanes, step = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
        const size_t row = i / lanes;
        const Span p((int)(i - row * lanes) * 8, C);
        if (p.valid > 0)
            store8<true>(X + row * C, values_of(settle(request_codes<true>(codes + row * C, p, C), p), powers[row * G + p.c / kGroup], ints), p);
    }
}

constexpr int kMostColumns = 16384;  // of the norm, whose rows stay in registers

// Lanes that share a row of C elements, and steps.  Forward: two steps a lane, which leaves few lanes waiting
// for a row's sum; backward: one, whose registers hold the next rows as well, up to 8192 columns.  From 1024 columns on
// a workgroup to a row, of as many waves as hold it.
template <int L, int K>
struct Shape {
    static constexpr int l = L, k = K;
    int C;
    int lanes() const { return L ? Share<L>::NT : (C + 512 * K - 1) / (512 * K) * 64; }  // of a workgroup
    int rows() const { return Share<L>::ROWS; }
};
template <bool BACKWARD, typename F>
void by_width(int C, F f)
{
    if (C <= 64) f(Shape<8, 1>{C});
    else if (C <= 128) f(Shape<16, 1>{C});
    else if (C <= 256) f(Shape<32, 1>{C});
    else if (C <= 512) f(Shape<64, 1>{C});
    else if constexpr (BACKWARD) {
        if (C <= 1024) f(Shape<128, 1>{C});
        else if (C <= 8192) f(Shape<0, 1>{C});
        else f(Shape<0, 2>{C});
    } else {
        if (C <= 1024) f(Shape<64, 2>{C});
        else f(Shape<0, 2>{C});
    }
}
// Workgroups that take all rows in one go.
template <typename S>
size_t row_groups(size_t rows, S shape)
{
    return (rows + shape.rows() - 1) / shape.rows();
}
// Workgroups of the backward pass: as many as run at once (four waves of its registers to a SIMD, whose share of a
// workgroup's waves is rounded up), each with a share of dw, and fewer, down to one for each of the 256 compute units, where
// each would get less than four rows to itself: 16384 rows of 2056, bf16, 512 workgroups 61 us, 1024 87; 1000 of 2048, 256
// workgroups 11.0, 1000 16.3.
int back_blocks(size_t rows, int C)
{
    int n = 0;
    by_width<true>(C, [&](auto shape) {
        const size_t g = row_groups(rows, shape), most = 256 * (4 / ((shape.lanes() / 64 + 3) / 4));
        const size_t few = g / 4 > 256 ? g / 4 : 256;
        n = (int)(g < few ? g : few < most ? few : most);
    });
    return n;
}

template <typename F>
void by_types(la_dtype dt, la_dtype wt, F f)
{
    if (dt == LA_F32) f((float *)nullptr, (float *)nullptr);
    else if (wt == LA_F32) f((bf16_t *)nullptr, (float *)nullptr);
    else f((bf16_t *)nullptr, (bf16_t *)nullptr);
}

la_status check_rows(size_t rows, int C, int most)
{
    if (rows < 1 || C < 1) return LA_ERR_SHAPE;
    if (C > most || (double)rows * C >= 1099511627776.0) return LA_ERR_SHAPE;  // 2^40
    return LA_OK;
}
size_t powers_bytes(size_t rows, int C) { return rows * ((C + kGroup - 1) / kGroup); }
la_status done() { return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH; }

unsigned rows_blocks(size_t rows, int C)
{
    const size_t blocks = (powers_bytes(rows, C) * 4 + 255) / 256;
    return (unsigned)(blocks < 16384 ? blocks : 16384);
}

}  // namespace
}  // namespace la

extern "C" {

la_status la_pack_tensors(int count, const void *const *X, void *const *codes, void *const *scales, size_t rows, int C,
                          la_dtype dt, la_dtype code, void *hip_stream)
{
    const la_status s = la::check_rows(rows, C, 2147483647 - 64);
    if (s != LA_OK) return s;
    if (count < 1 || count > la::kMostTensors) return LA_ERR_SHAPE;
    if (!la::real_type(dt) || !la::eight_bits(code)) return LA_ERR_UNSUPPORTED;
    if (!X || !codes || !scales) return LA_ERR_NULL;
    la::Batch a{};
    la::Range ins[la::kMostTensors], outs[2 * la::kMostTensors];
    for (int i = 0; i < count; ++i) {
        if (!X[i] || !codes[i] || !scales[i]) return LA_ERR_NULL;
        if (!la::aligned_to(X[i], la::size_of(dt))) return LA_ERR_ALIGN;
        a.X[i] = X[i], a.codes[i] = (uint8_t *)codes[i], a.powers[i] = (uint8_t *)scales[i];
        ins[i] = {X[i], rows * C * la::size_of(dt)};
        outs[2 * i] = {codes[i], rows * C};
        outs[2 * i + 1] = {scales[i], la::powers_bytes(rows, C)};
    }
    if (la::any_alias(ins, count, outs, 2 * count)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    const dim3 grid(la::rows_blocks(rows, C), count), block(256);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (dt == LA_F32) la::k_pack<float><<<grid, block, 0, st>>>(a, rows, C, code == LA_I8);
    else la::k_pack<la::bf16_t><<<grid, block, 0, st>>>(a, rows, C, code == LA_I8);
    return la::done();
}

la_status la_pack_rows(const void *X, void *codes, void *scales, size_t rows, int C, la_dtype dt, la_dtype code,
                       void *hip_stream)
{
    return la_pack_tensors(1, &X, &codes, &scales, rows, C, dt, code, hip_stream);
}

la_status la_unpack_rows(const void *codes, const void *scales, void *X, size_t rows, int C, la_dtype code,
                         la_dtype dt, void *hip_stream)
{
    const la_status s = la::check_rows(rows, C, 2147483647 - 64);
    if (s != LA_OK) return s;
    if (!la::real_type(dt) || !la::eight_bits(code)) return LA_ERR_UNSUPPORTED;
    if (!X || !codes || !scales) return LA_ERR_NULL;
    if (!la::aligned_to(X, la::size_of(dt))) return LA_ERR_ALIGN;
    const la::Range ins[] = {{codes, rows * C}, {scales, la::powers_bytes(rows, C)}};
    const la::Range outs[] = {{X, rows * C * la::size_of(dt)}};
    if (la::any_alias(ins, 2, outs, 1)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    const dim3 grid(la::rows_blocks(rows, C)), block(256);
    const hipStream_t st = (hipStream_t)hip_stream;
    const uint8_t *c = (const uint8_t *)codes, *p = (const uint8_t *)scales;
    if (dt == LA_F32) la::k_unpack<float><<<grid, block, 0, st>>>(c, p, (float *)X, rows, C, code == LA_I8);
    else la::k_unpack<la::bf16_t><<<grid, block, 0, st>>>(c, p, (la::bf16_t *)X, rows, C, code == LA_I8);
    return la::done();
}

size_t la_rmsnorm_workspace_bytes(size_t rows, int C)
{
    if (la::check_rows(rows, C, la::kMostColumns) != LA_OK) return 0;
    return la::round_up((size_t)la::back_blocks(rows, C) * C * 4, 256);
}

la_status la_rmsnorm_forward(const void *X, const void *R, const void *W, void *Y, void *Yscale, void *S, void *Kept,
                             void *Kscale, float *rstd, size_t rows, int C, float eps, la_dtype dt, la_dtype wt,
                             la_dtype yt, la_dtype kt, void *hip_stream)
{
    const la_status s = la::check_rows(rows, C, la::kMostColumns);
    if (s != LA_OK) return s;
    if (!la::real_type(dt) || (W && wt != LA_F32 && wt != dt)) return LA_ERR_UNSUPPORTED;
    if ((yt != dt && !la::eight_bits(yt)) || (Kept && !la::eight_bits(kt))) return LA_ERR_UNSUPPORTED;
    if (!X || !Y || (yt != dt) != (Yscale != nullptr) || (Kept != nullptr) != (Kscale != nullptr) ||
        (R != nullptr) != (S != nullptr))
        return LA_ERR_NULL;
    const size_t e = la::size_of(dt), n = rows * C, pb = la::powers_bytes(rows, C);
    for (const void *p : {X, R, (const void *)S, yt == dt ? (const void *)Y : nullptr})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if ((W && !la::aligned_to(W, la::size_of(wt))) || !la::aligned_to(rstd, 4)) return LA_ERR_ALIGN;
    const la::Range ins[] = {{X, n * e}, {R, S == R ? 0 : n * e}, {W, W ? C * la::size_of(wt) : 0}};
    const la::Range outs[] = {{Y, n * la::size_of(yt)}, {Yscale, pb}, {S, n * e}, {Kept, n}, {Kscale, pb}, {rstd, rows * 4}};
    if (la::any_alias(ins, 3, outs, 6)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    const la::Norm a{X, R, W, Y, S, (uint8_t *)Yscale, (uint8_t *)Kept, (uint8_t *)Kscale, rstd, rows, C, eps, yt, kt};
    la::by_types(dt, wt, [&](auto *t, auto *w) {
        la::by_width<false>(C, [&](auto shape) {
            typedef decltype(shape) Sh;
            const size_t groups = la::row_groups(rows, shape);
            const dim3 grid((unsigned)(groups < 65536 ? groups : 65536));
            la::k_norm<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>, Sh::l, Sh::k>
                <<<grid, dim3(shape.lanes()), 0, (hipStream_t)hip_stream>>>(a);
        });
    });
    return la::done();
}

la_status la_rmsnorm_backward(const void *S, const void *Sscale, const void *W, const float *rstd, const void *dY,
                              const void *dS, void *dX, float *dW, size_t rows, int C, la_dtype dt, la_dtype wt,
                              la_dtype st, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const la_status s = la::check_rows(rows, C, la::kMostColumns);
    if (s != LA_OK) return s;
    if (!la::real_type(dt) || (W && wt != LA_F32 && wt != dt)) return LA_ERR_UNSUPPORTED;
    if (st != dt && !la::eight_bits(st)) return LA_ERR_UNSUPPORTED;
    if (!S || !rstd || !dY || !dX || (st != dt) != (Sscale != nullptr) || (dW && !W)) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), n = rows * C, need = dW ? la_rmsnorm_workspace_bytes(rows, C) : 0;
    for (const void *p : {st == dt ? S : nullptr, dY, dS, (const void *)dX})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if ((W && !la::aligned_to(W, la::size_of(wt))) || !la::aligned_to(rstd, 4) || !la::aligned_to(dW, 4))
        return LA_ERR_ALIGN;
    if (need && (!workspace || workspace_bytes < need || !la::aligned_to(workspace, 256))) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{S, n * la::size_of(st)}, {Sscale, la::powers_bytes(rows, C)}, {W, W ? C * la::size_of(wt) : 0},
                             {rstd, rows * 4}, {dY, n * e}, {dS, n * e}};
    const la::Range outs[] = {{dX, n * e}, {dW, (size_t)C * 4}, {workspace, need}};
    if (la::any_alias(ins, 6, outs, 3)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    const la::NormBack a{S, W, dY, dS, (const uint8_t *)Sscale, rstd, dX, dW ? (float *)workspace : nullptr, rows, C, st};
    const int blocks = la::back_blocks(rows, C);
    const hipStream_t stream = (hipStream_t)hip_stream;
    la::by_types(dt, wt, [&](auto *t, auto *w) {
        la::by_width<true>(C, [&](auto shape) {
            typedef decltype(shape) Sh;
            la::k_norm_back<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>, Sh::l, Sh::k>
                <<<dim3(blocks), dim3(shape.lanes()), 0, stream>>>(a);
        });
    });
    if (dW) la::k_norm_join<<<dim3((C + 15) / 16), dim3(1024), 0, stream>>>((const float *)workspace, dW, blocks, C);
    return la::done();
}

}  // extern "C"
