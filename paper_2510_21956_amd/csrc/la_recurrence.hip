// Gated linear recurrence h_t = f_t h_{t-1} + u_t per channel, forward, backward and in steps.
//
// One wave takes 64 V neighbouring channels of one segment of a sequence and walks its rows; what a
// segment does to a state is h -> P h + q, P the product of its gates, q its result from zero.  Where
// sequences are cut, one launch finds (P, q) of every segment, and every wave of the next joins those
// of the segments before its own, in their order, and walks its rows again from there.  The backward pass
// is the same walk from the far end with e_t = f_t (dh_t + e_{t+1}): what row t hands to row t-1.
#include "la_checks.h"
#include "la_common.h"

namespace la {
namespace {

constexpr int kBatch = 8;  // rows requested together

// V neighbouring channels of a row, one lane's share.
template <typename T, int V>
struct Cells {
    T x[V];
};
template <typename T, int V>
__device__ __forceinline__ Cells<T, V> request(const T *p)
{
    Cells<T, V> c;
    __builtin_memcpy(&c, p, sizeof c);
    return c;
}
template <typename T, int V>
__device__ __forceinline__ void leave(T *p, const float (&x)[V])
{
    Cells<T, V> c;
#pragma unroll
    for (int j = 0; j < V; ++j) store_elem(c.x, j, x[j]);
    __builtin_memcpy(p, &c, sizeof c);
}

// f and 1 - f of a stored gate, both from the smaller one's exponential: neither loses digits to a difference,
// and infinite gates give 0 and 1.
template <int GATE>
__device__ __forceinline__ void open_gate(float g, float &f, float &rest)
{
    if (GATE == LA_GATE_SIGMOID) {
        const float E = expf(-fabsf(g)), large = __builtin_amdgcn_rcpf(1.f + E), small = E * large;
        f = g >= 0.f ? large : small;
        rest = g >= 0.f ? small : large;
    } else {
        f = g;
        rest = 1.f;
    }
}

struct Walk {
    const void *X, *Gate, *H, *dH;
    void *out0, *out1;  // forward: h; backward: dx, dgate
    const float *first; // forward: h0; backward: dlast
    const float *h0;
    float *last;        // forward: last; backward: dh0
    const int *lengths;
    float *sums;        // [B, nseg, 2, C]
    int B, N, C, nseg, seg_len, groups;
};

__device__ __forceinline__ int rows_of(const Walk &w, int b)
{
    if (!w.lengths) return w.N;
    const int n = w.lengths[b];
    return n < 0 ? 0 : n > w.N ? w.N : n;
}

// Segment seg of sequence b, channels [c, c + V): found from the wave's number.  The lanes behind the last
// channel take the last V channels once more: they write what their neighbour writes.
template <int V>
__device__ __forceinline__ bool locate(const Walk &w, int &b, int &seg, int &c)
{
    const int u = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (u >= w.B * w.groups * w.nseg) return false;
    seg = u % w.nseg;
    const int bg = u / w.nseg;
    b = bg / w.groups;
    c = (bg % w.groups * 64 + lane) * V;
    if (c > w.C - V) c = w.C - V;
    return true;
}

template <typename T, int V, int GATE, bool BWD>
__global__ void __launch_bounds__(256) k_sums(Walk w)
{
    int b, seg, c;
    if (!locate<V>(w, b, seg, c)) return;
    const int n = rows_of(w, b), r0 = seg * w.seg_len, r1 = min(n, r0 + w.seg_len);
    const size_t at = ((size_t)b * w.N) * w.C + c;
    const T *G = (const T *)w.Gate + at, *X = (const T *)(BWD ? w.dH : w.X) + at;
    float P[V], q[V];
#pragma unroll
    for (int j = 0; j < V; ++j) P[j] = 1.f, q[j] = 0.f;
    for (int r = r0; r < r1; r += kBatch) {
        Cells<T, V> g[kBatch], x[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int s = min(r + k, r1 - 1), t = BWD ? r1 - 1 - (s - r0) : s;
            g[k] = request<T, V>(G + (size_t)t * w.C);
            x[k] = request<T, V>(X + (size_t)t * w.C);
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (r + k < r1) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, rest;
                    open_gate<GATE>(load_elem(g[k].x, j), f, rest);
                    const float v = load_elem(x[k].x, j);
                    q[j] = BWD ? f * (q[j] + v) : f * q[j] + (GATE == LA_GATE_SIGMOID ? rest * v : v);
                    P[j] *= f;
                }
            }
    }
    float *s = w.sums + ((size_t)b * w.nseg + seg) * 2 * w.C + c;
    leave<float, V>(s, P);
    leave<float, V>(s + w.C, q);
}

template <typename T, int V, int GATE, bool BWD>
__global__ void __launch_bounds__(256) k_walk(Walk w)
{
    int b, seg, c;
    if (!locate<V>(w, b, seg, c)) return;
    const int n = rows_of(w, b), r0 = seg * w.seg_len, end = min(w.N, r0 + w.seg_len), r1 = min(n, end);
    const size_t at = ((size_t)b * w.N) * w.C + c, bc = (size_t)b * w.C + c;
    const T *G = (const T *)w.Gate + at, *X = (const T *)w.X + at, *H = (const T *)w.H + at,
            *D = (const T *)w.dH + at;
    T *O0 = (T *)w.out0 + at, *O1 = (T *)w.out1 + at;
    float zero[V], e[V], before[V];
#pragma unroll
    for (int j = 0; j < V; ++j) zero[j] = 0.f, e[j] = 0.f, before[j] = 0.f;
    for (int t = max(r0, n); t < end; ++t) {
        leave<T, V>(O0 + (size_t)t * w.C, zero);
        if (BWD) leave<T, V>(O1 + (size_t)t * w.C, zero);
    }
    if (w.first) {
        const Cells<float, V> s = request<float, V>(w.first + bc);
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = s.x[j];
    }
    if (BWD && w.h0) {
        const Cells<float, V> s = request<float, V>(w.h0 + bc);
#pragma unroll
        for (int j = 0; j < V; ++j) before[j] = s.x[j];
    }
    if (n == 0 && seg == 0 && w.last) leave<float, V>(w.last + bc, e);
    if (r0 >= r1) return;
    // the segments before this one in the order of the walk; all of them have rows
    const int from = BWD ? (n - 1) / w.seg_len : 0;
    for (int s = from; s != seg; s += BWD ? -1 : 1) {
        const float *p = w.sums + ((size_t)b * w.nseg + s) * 2 * w.C + c;
        const Cells<float, V> P = request<float, V>(p), q = request<float, V>(p + w.C);
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = P.x[j] * e[j] + q.x[j];
    }
    for (int r = r0; r < r1; r += kBatch) {
        Cells<T, V> g[kBatch], x[kBatch], h[kBatch], d[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int s = min(r + k, r1 - 1), t = BWD ? r1 - 1 - (s - r0) : s;
            g[k] = request<T, V>(G + (size_t)t * w.C);
            if (!BWD || GATE == LA_GATE_SIGMOID) x[k] = request<T, V>(X + (size_t)t * w.C);
            if (BWD) {
                h[k] = request<T, V>(H + (size_t)(t ? t - 1 : 0) * w.C);
                d[k] = request<T, V>(D + (size_t)t * w.C);
            }
        }
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            if (r + k < r1) {
                const int t = BWD ? r1 - 1 - (r + k - r0) : r + k;
                float o0[V], o1[V];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, rest;
                    open_gate<GATE>(load_elem(g[k].x, j), f, rest);
                    const float v = load_elem(x[k].x, j);
                    if (!BWD) {
                        e[j] = f * e[j] + (GATE == LA_GATE_SIGMOID ? rest * v : v);
                        o0[j] = e[j];
                    } else {
                        const float dt = load_elem(d[k].x, j) + e[j];
                        const float prev = t ? load_elem(h[k].x, j) : before[j];
                        o0[j] = GATE == LA_GATE_SIGMOID ? rest * dt : dt;
                        o1[j] = GATE == LA_GATE_SIGMOID ? dt * (prev - v) * (f * rest) : dt * prev;
                        e[j] = f * dt;
                    }
                }
                leave<T, V>(O0 + (size_t)t * w.C, o0);
                if (BWD) leave<T, V>(O1 + (size_t)t * w.C, o1);
            }
    }
    if (w.last && (BWD ? r0 == 0 : r1 == n)) leave<float, V>(w.last + bc, e);
}

// T rows on a carried state.  One channel a lane: the state is updated in place.
template <typename T, int GATE>
__global__ void __launch_bounds__(256) k_step(const T *X, const T *G, T *H, float *state, int B, int Tn, int C)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)B * C) return;
    const size_t b = i / C, at = b * Tn * C + (i - b * C);
    float h = state[i];
    for (int t = 0; t < Tn; ++t) {
        float f, rest;
        open_gate<GATE>(load_elem(G, at + (size_t)t * C), f, rest);
        const float x = load_elem(X, at + (size_t)t * C);
        h = f * h + (GATE == LA_GATE_SIGMOID ? rest * x : x);
        store_elem(H, at + (size_t)t * C, h);
    }
    state[i] = h;
}

struct Cut1 {
    int nseg, seg_len, groups, V;
    size_t bytes;
};

// Segments so that some 4096 waves, sixteen a compute unit, have work; 32 rows at least.
Cut1 cut_of(int B, int N, int C, la_dtype dt)
{
    Cut1 p;
    p.V = dt == LA_BF16 && C >= 2 ? 2 : 1;
    p.groups = (C + 64 * p.V - 1) / (64 * p.V);
    const long waves = (long)B * p.groups, want = (4096 + waves - 1) / waves, most = (N + 31) / 32;
    const long nseg = want < most ? want : most;
    p.seg_len = (int)((N + nseg - 1) / nseg);
    p.nseg = (N + p.seg_len - 1) / p.seg_len;
    p.bytes = p.nseg > 1 ? round_up((size_t)B * p.nseg * 2 * C * 4, 256) : 0;
    return p;
}

la_status check_shape(int B, int N, int C, la_gate gate, la_dtype dt)
{
    if (B < 1 || N < 1 || C < 1) return LA_ERR_SHAPE;
    if (!real_type(dt) || (gate != LA_GATE_VALUE && gate != LA_GATE_SIGMOID)) return LA_ERR_UNSUPPORTED;
    if ((double)B * N * C >= 1099511627776.0) return LA_ERR_SHAPE;          // 2^40
    if ((double)B * ((C + 63) / 64) >= 8388608.0) return LA_ERR_SHAPE;  // 2^23
    return LA_OK;
}

template <typename T, int V, int GATE, bool BWD>
void launch(const Walk &w, hipStream_t st)
{
    const dim3 grid((unsigned)(((long)w.B * w.groups * w.nseg + 3) / 4)), block(256);
    if (w.nseg > 1) k_sums<T, V, GATE, BWD><<<grid, block, 0, st>>>(w);
    k_walk<T, V, GATE, BWD><<<grid, block, 0, st>>>(w);
}
template <bool BWD>
la_status run(Walk w, const Cut1 &p, la_gate gate, la_dtype dt, hipStream_t st)
{
    w.nseg = p.nseg;
    w.seg_len = p.seg_len;
    w.groups = p.groups;
    const bool s = gate == LA_GATE_SIGMOID;
    if (dt == LA_F32) s ? launch<float, 1, LA_GATE_SIGMOID, BWD>(w, st) : launch<float, 1, LA_GATE_VALUE, BWD>(w, st);
    else if (p.V == 2)
        s ? launch<bf16_t, 2, LA_GATE_SIGMOID, BWD>(w, st) : launch<bf16_t, 2, LA_GATE_VALUE, BWD>(w, st);
    else s ? launch<bf16_t, 1, LA_GATE_SIGMOID, BWD>(w, st) : launch<bf16_t, 1, LA_GATE_VALUE, BWD>(w, st);
    return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

bool bad_workspace(const void *ws, size_t bytes, size_t need)
{
    return need && (!ws || bytes < need || !aligned_to(ws, 256));
}

}  // namespace
}  // namespace la

extern "C" {

size_t la_recurrence_workspace_bytes(int B, int N, int C, la_dtype dt, int is_backward)
{
    (void)is_backward;
    if (la::check_shape(B, N, C, LA_GATE_VALUE, dt) != LA_OK) return 0;
    return la::cut_of(B, N, C, dt).bytes;
}

la_status la_recurrence_forward(const void *X, const void *Gate, const float *h0, void *Hs, float *last,
                                const int *lengths, int B, int N, int C, la_gate gate, la_dtype dt,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const la_status s = la::check_shape(B, N, C, gate, dt);
    if (s != LA_OK) return s;
    if (!X || !Gate || !Hs) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), tb = (size_t)B * N * C * e, sb = (size_t)B * C * 4;
    for (const void *p : {X, Gate, (const void *)Hs})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    for (const void *p : {(const void *)h0, (const void *)last, (const void *)lengths})
        if (!la::aligned_to(p, 4)) return LA_ERR_ALIGN;
    const la::Cut1 p = la::cut_of(B, N, C, dt);
    if (la::bad_workspace(workspace, workspace_bytes, p.bytes)) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{X, tb}, {Gate, tb}, {h0, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{Hs, tb}, {last, sb}, {workspace, p.bytes}};
    if (la::any_alias(ins, 4, outs, 3)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Walk w{};
    w.X = X, w.Gate = Gate, w.out0 = Hs, w.out1 = Hs, w.first = h0, w.last = last, w.lengths = lengths;
    w.sums = (float *)workspace;
    w.B = B, w.N = N, w.C = C;
    return la::run<false>(w, p, gate, dt, (hipStream_t)hip_stream);
}

la_status la_recurrence_backward(const void *X, const void *Gate, const float *h0, const void *Hs,
                                 const void *dHs, const float *dlast, void *dX, void *dGate, float *dh0,
                                 const int *lengths, int B, int N, int C, la_gate gate, la_dtype dt,
                                 void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const la_status s = la::check_shape(B, N, C, gate, dt);
    if (s != LA_OK) return s;
    if (!X || !Gate || !Hs || !dHs || !dX || !dGate) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), tb = (size_t)B * N * C * e, sb = (size_t)B * C * 4;
    for (const void *p : {X, Gate, Hs, dHs, (const void *)dX, (const void *)dGate})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    for (const void *p : {(const void *)h0, (const void *)dlast, (const void *)dh0, (const void *)lengths})
        if (!la::aligned_to(p, 4)) return LA_ERR_ALIGN;
    const la::Cut1 p = la::cut_of(B, N, C, dt);
    if (la::bad_workspace(workspace, workspace_bytes, p.bytes)) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{X, tb}, {Gate, tb}, {h0, sb}, {Hs, tb}, {dHs, tb}, {dlast, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{dX, tb}, {dGate, tb}, {dh0, sb}, {workspace, p.bytes}};
    if (la::any_alias(ins, 7, outs, 4)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Walk w{};
    w.X = X, w.Gate = Gate, w.H = Hs, w.dH = dHs, w.out0 = dX, w.out1 = dGate, w.first = dlast, w.h0 = h0;
    w.last = dh0, w.lengths = lengths, w.sums = (float *)workspace;
    w.B = B, w.N = N, w.C = C;
    return la::run<true>(w, p, gate, dt, (hipStream_t)hip_stream);
}

la_status la_recurrence_step(const void *X, const void *Gate, void *Hs, float *state, int B, int T, int C,
                             la_gate gate, la_dtype dt, void *hip_stream)
{
    const la_status s = la::check_shape(B, T, C, gate, dt);
    if (s != LA_OK) return s;
    if (!X || !Gate || !Hs || !state) return LA_ERR_NULL;
    const size_t e = la::size_of(dt), tb = (size_t)B * T * C * e, sb = (size_t)B * C * 4;
    for (const void *p : {X, Gate, (const void *)Hs})
        if (!la::aligned_to(p, e)) return LA_ERR_ALIGN;
    if (!la::aligned_to(state, 4)) return LA_ERR_ALIGN;
    const la::Range ins[] = {{X, tb}, {Gate, tb}};
    const la::Range outs[] = {{Hs, tb}, {state, sb}};
    if (la::any_alias(ins, 2, outs, 2)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    const dim3 grid((unsigned)(((size_t)B * C + 255) / 256)), block(256);
    const hipStream_t st = (hipStream_t)hip_stream;
    const bool sg = gate == LA_GATE_SIGMOID;
    if (dt == LA_F32)
        (sg ? la::k_step<float, LA_GATE_SIGMOID> : la::k_step<float, LA_GATE_VALUE>)<<<grid, block, 0, st>>>(
            (const float *)X, (const float *)Gate, (float *)Hs, state, B, T, C);
    else
        (sg ? la::k_step<la::bf16_t, LA_GATE_SIGMOID> : la::k_step<la::bf16_t, LA_GATE_VALUE>)<<<grid, block, 0, st>>>(
            (const la::bf16_t *)X, (const la::bf16_t *)Gate, (la::bf16_t *)Hs, state, B, T, C);
    return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH;
}

}  // extern "C"
