// Gated linear recurrence h_t = f_t h_{t-1} + u_t per channel, forward, backward and in steps.
//
// What a run of rows does to a state is h -> P h + q, P the product of its gates, q its result from zero.  A
// workgroup takes tiles, W R rows of 64 V neighbouring channels, into registers (R rows to each of W waves), finds
// every wave's (P, q), learns the state that the tiles before it hand over, and walks its rows once more in
// registers: every tensor moves once.  Tiles of a sequence are joined in blocks of `span`: a tile publishes its
// (P, q) as soon as it has them, reads those of its block's tiles before it and the state that the block
// before left, and the block's last tile publishes the state for the next.  So sums are joined in a fixed order
// (two runs give the same bits), and only every span-th tile waits for a chain of states.
//
// Bound by HBM: forward 3 elements moved a row and channel, backward 5 or 6.  One sequence of 131072 rows, bf16, 2048
// channels, sigmoid gates: forward 312 us (5.2 TB/s), backward 660 (4.9); short calls by the clearing launch
// and a chain of tiles (2 x 3001 rows, 22 us; 3 x 5003 rows of 771 channels, 25 and 44, half the rate).
//
// Tiles are handed out by a counter, in an order in which a tile waits for earlier ones only: those are done or in
// hand of a workgroup that waits for still earlier ones at most, whatever the order in which workgroups
// start, so every wait ends.  A published word is 64 bits that carry their own mark of being there (the
// workspace is filled with ones first): no fence is needed between data and flag, and stores and loads of
// device scope keep the eight L2 caches out of it.
//
// The backward pass is the same walk from the far end with e_t = f_t (dh_t + e_{t+1}): what row t hands to
// row t-1.
#include "la_checks.h"
#include "la_common.h"

namespace la {
namespace {

constexpr int kRowsFwd = 16, kRowsBack = 8;  // of a wave

// V neighbouring channels of a row, one lane's share, as they are stored: two bfloat16 stay one register.
template <typename T, int V>
struct Cells {
    T x[V];
    __device__ __forceinline__ float at(int j) const { return load_elem(x, j); }
};
template <>
struct Cells<bf16_t, 2> {
    uint32_t x;
    __device__ __forceinline__ float at(int j) const { return __uint_as_float(j ? x & 0xffff0000u : x << 16); }
};
// From a row's address, the same in all lanes, and the lane's channel.
template <typename T, int V>
__device__ __forceinline__ Cells<T, V> request(const void *row, unsigned channel)
{
    Cells<T, V> c;
    __builtin_memcpy(&c, (const char *)row + channel * (unsigned)sizeof(T), sizeof c);
    return c;
}
// STREAM: non-temporal, the backward pass's gradients, two tensors for three or four read (4 x 4096 rows of 1024, fp32, 83
// and 70 us; 8 x 2048 of 2048, bf16, 91 and 84; a forward pass 36.2 and 35.4, whose reader follows).
template <typename T, int V, bool STREAM = false>
__device__ __forceinline__ void leave(void *row, unsigned channel, const float (&x)[V])
{
    Cells<T, V> c;
    if constexpr (sizeof(T) == 2 && V == 2) {
        const __bf16 y[2] = {(__bf16)x[0], (__bf16)x[1]};
        __builtin_memcpy(&c, y, sizeof c);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) store_elem(c.x, j, x[j]);
    }
    char *p = (char *)row + channel * (unsigned)sizeof(T);
    if constexpr (STREAM && sizeof c == 4) {
        typedef uint32_t word __attribute__((aligned(2)));
        uint32_t w;
        __builtin_memcpy(&w, &c, 4);
        __builtin_nontemporal_store(w, (word *)p);
    } else __builtin_memcpy(p, &c, sizeof c);
}

// f and 1 - f of a stored gate, both from the smaller one's exponential: neither loses digits to a difference,
// and infinite gates give 0 and 1.  The exponential's argument in base 2 is rounded, an error of up to |g| U
// relative to it: float32 adds what the rounding lost, bfloat16 rounds to 2^-8 what that is far below.
template <int GATE, bool FINE>
__device__ __forceinline__ void open_gate(float g, float &f, float &rest)
{
    if (GATE == LA_GATE_SIGMOID) {
        constexpr float L = 1.44269504f, Lrest = 1.92596299e-8f, ln2 = 0.693147181f;  // log2(e) in two parts
        const float y = -fabsf(g), t = y * L;
        float E = __builtin_amdgcn_exp2f(t);
        if (FINE) {
            const float lost = fmaf(y, Lrest, fmaf(y, L, -t));
            E = fmaf(E, (y > -128.f ? lost : 0.f) * ln2, E);
        }
        const float large = __builtin_amdgcn_rcpf(1.f + E), small = E * large;
        f = g >= 0.f ? large : small;
        rest = g >= 0.f ? small : large;
    } else {
        f = g;
        rest = 1.f;
    }
}

struct Walk {
    const void *X, *Gate, *H, *dH;
    void *out0, *out1;   // forward: h; backward: dx, dgate
    const float *first;  // forward: h0; backward: dlast
    const float *h0;
    float *last;         // forward: last; backward: dh0
    const int *lengths;
    uint64_t *sums, *states;  // [B, tiles, C] words (P, q); [B, blocks, C] words (state, 0)
    unsigned *ticket;
    int B, N, C, lanes, groups, chains, tiles, blocks, span, lots;
};
constexpr uint32_t kNothing = 0xffffffffu;
constexpr int kMostLooks = 1 << 21;
constexpr int kMostSpan = 32, kLots = 8, kCounters = kLots * 64;

// Rows of sequence b.  `held`: the length of sequence `lane`, where a wave holds all of them: asked for before the wave
// knows which one is its own.
__device__ __forceinline__ int rows_of(const Walk &w, int b, int held)
{
    if (!w.lengths) return w.N;
    const int n = w.B <= 64 ? __builtin_amdgcn_readlane(held, b) : __builtin_amdgcn_readfirstlane(w.lengths[b]);
    return n < 0 ? 0 : n > w.N ? w.N : n;
}

__device__ __forceinline__ void publish(uint64_t *p, uint32_t mark, float x)
{
    __hip_atomic_store(p, (uint64_t)mark << 32 | __float_as_uint(x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t peek(const uint64_t *p)
{
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// A word that was peeked at, once it is there.  Within one call every wait ends (above) in microseconds; where two calls
// overlap on one workspace, against the rules, one may wipe out what the other waits for: after some seconds of looking
// a wait ends with what is there, ones, which are NaN in either half.  That ends the kernel and tells nothing: such calls
// may as well take each other's finite words, or leave out the tiles whose tickets the other drew.
__device__ __forceinline__ uint64_t await(const uint64_t *p, uint64_t word)
{
    for (int looks = 0; (uint32_t)(word >> 32) == kNothing && looks < kMostLooks; ++looks) {
        __builtin_amdgcn_s_sleep(1);
        word = peek(p);
    }
    return word;
}

// One tile: rows [r0, r0 + count) of sequence b (and padding up to `end`), channels c on.  `order` counts the tiles
// of a sequence that have rows as the walk meets them.
template <bool BWD>
struct Place {
    unsigned at;  // of this lane's channels, from the address of row t of sequence b on
    int c, own;   // its first channel, its sequence
    int b, n, r0, end, count, tile, tiles, order;
    bool goes_on;  // there is a tile after it
    // the s-th row of the walk through the tile (its last one for s behind it)
    __device__ __forceinline__ int row(int s) const
    {
        s = min(s, count - 1);
        return BWD ? r0 + count - 1 - s : r0 + s;
    }
};
template <int V, int ROWS, bool BWD>
__device__ __forceinline__ Place<BWD> place_of(const Walk &a, unsigned k, unsigned chain, int lane, int held)
{
    Place<BWD> p;
    const int together = 64 / a.lanes;  // narrow sequences that share a wave, all of one length
    p.b = __builtin_amdgcn_readfirstlane(chain / a.groups * together);
    p.tile = __builtin_amdgcn_readfirstlane(BWD ? a.tiles - 1 - (int)k : (int)k);
    // the lanes behind the last channel take the last V channels once more, those behind the last sequence that
    // one: they write what their neighbour writes
    const int other = min(lane / a.lanes, a.B - 1 - p.b);
    p.c = min(((int)(chain % a.groups) * 64 + lane % a.lanes) * V, a.C - V);
    p.own = p.b + other;
    p.at = (unsigned)other * (unsigned)a.N * (unsigned)a.C + p.c;
    p.n = rows_of(a, p.b, held);
    p.r0 = p.tile * ROWS;
    p.end = min(a.N, p.r0 + ROWS);
    p.count = min(p.n, p.end) - p.r0;
    p.tiles = (p.n + ROWS - 1) / ROWS;
    p.order = BWD ? p.tiles - 1 - p.tile : p.tile;
    p.goes_on = p.order < p.tiles - 1;
    return p;
}

// R rows of a tile as they are stored, for one lane: those from the first-th of the walk on.
template <typename T, int V, int GATE, bool BWD, int R>
struct Rows {
    Cells<T, V> g[R], x[R], h[R], d[R];
    __device__ __forceinline__ void load(const Walk &a, const Place<BWD> &p, int first)
    {
        int t = p.row(first);
        size_t o = ((size_t)p.b * a.N + t) * a.C;  // the same in all lanes
#pragma unroll
        for (int i = 0; i < R; ++i) {
            g[i] = request<T, V>((const T *)a.Gate + o, p.at);
            if (BWD) d[i] = request<T, V>((const T *)a.dH + o, p.at);
            if (!BWD || GATE == LA_GATE_SIGMOID) x[i] = request<T, V>((const T *)a.X + o, p.at);
            if (BWD) h[i] = request<T, V>((const T *)a.H + (t ? o - a.C : o), p.at);
            if (first + i + 1 < p.count) {  // behind the tile's last row: that row once more
                o = BWD ? o - a.C : o + a.C;
                t += BWD ? -1 : 1;
            }
        }
    }
};

template <typename T, int V, int GATE, bool BWD, int W, int R>
__global__ void __launch_bounds__(W * 64, 4) k_walk(Walk a)
{
    __shared__ float2 sums[W][64 * V], blocks[kMostSpan][64 * V];
    __shared__ float state[64 * V];
    __shared__ unsigned ticket;
    constexpr int ROWS = W * R;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, first = wave * R;
    // every lot's counter hands out the tiles of its own chains, neighbouring ones
    const unsigned group = blockIdx.y * gridDim.x + blockIdx.x;
    const unsigned chains = (unsigned)a.chains, lot = group % a.lots, per = (chains + a.lots - 1) / a.lots;
    const unsigned mine = lot * per < chains ? min(per, chains - lot * per) : 0;
    unsigned k = group / a.lots;
    const int held = a.lengths && a.B <= 64 ? a.lengths[min(lane, a.B - 1)] : 0;
    if (a.tiles > 1) {
        if (threadIdx.x == 0) ticket = atomicAdd(a.ticket + 16 * lot, 1u);
        block_sync();
        k = __builtin_amdgcn_readfirstlane(ticket);
    }
    if (k >= mine * a.tiles) return;
    const Place<BWD> p = place_of<V, ROWS, BWD>(a, k / mine, lot * per + k % mine, lane, held);
    T *O0 = (T *)a.out0, *O1 = (T *)a.out1;
    Rows<T, V, GATE, BWD, R> r;
    if (p.count > 0) r.load(a, p, first);
    float P[V], q[V], e[V], f[R][V], u[R][V], rest[R][V];
#pragma unroll
    for (int j = 0; j < V; ++j) P[j] = 1.f, q[j] = e[j] = 0.f;
    for (int t = max(p.r0, p.n) + wave; t < p.end; t += W) {  // padding
        const size_t o = ((size_t)p.b * a.N + t) * a.C;
        leave<T, V>(O0 + o, p.at, q);
        if (BWD) leave<T, V>(O1 + o, p.at, q);
    }
    if (a.first) {
        const Cells<float, V> s = request<float, V>(a.first + (size_t)p.own * a.C, p.c);
#pragma unroll
        for (int j = 0; j < V; ++j) e[j] = s.at(j);
    }
    if (p.n == 0 && p.tile == 0 && wave == 0 && a.last) leave<float, V>(a.last + (size_t)p.own * a.C, p.c, e);
    if (p.count <= 0) return;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const bool live = first + i < p.count;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            open_gate<GATE, sizeof(T) == 4>(r.g[i].at(j), f[i][j], rest[i][j]);
            if (BWD) u[i][j] = r.d[i].at(j);
            else u[i][j] = GATE == LA_GATE_SIGMOID ? rest[i][j] * r.x[i].at(j) : r.x[i].at(j);
            if (live) {
                q[j] = BWD ? f[i][j] * (q[j] + u[i][j]) : f[i][j] * q[j] + u[i][j];
                P[j] *= f[i][j];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) sums[wave][lane * V + j] = make_float2(P[j], q[j]);
    block_sync();

    const int block = p.order / a.span, start = block * a.span;
    const bool ends = p.order - start == a.span - 1;
    if (wave == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            P[j] = 1.f, q[j] = 0.f;
#pragma unroll
            for (int v = 0; v < W; ++v) {
                const float2 s = sums[v][lane * V + j];
                q[j] = s.x * q[j] + s.y;
                P[j] *= s.x;
            }
            if (p.goes_on && !ends) {
                const uint32_t bits = __float_as_uint(P[j]);
                publish(a.sums + ((size_t)p.own * a.tiles + p.tile) * a.C + p.c + j, bits == kNothing ? 0x7fc00000u : bits, q[j]);
            }
        }
    }
    if (p.order > 0) {
        const uint64_t *from = a.states + ((size_t)p.own * a.blocks + block - 1) * a.C + p.c;
        uint64_t word[V];
        const bool last_wave = block > 0 && wave == W - 1;
        if (last_wave)
#pragma unroll
            for (int j = 0; j < V; ++j) word[j] = peek(from + j);
        for (int s = start + wave; s < p.order; s += W) {
            const uint64_t *f = a.sums + ((size_t)p.own * a.tiles + (BWD ? p.tiles - 1 - s : s)) * a.C + p.c;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const uint64_t w = await(f + j, peek(f + j));
                blocks[s - start][lane * V + j] = make_float2(__uint_as_float((uint32_t)(w >> 32)), __uint_as_float((uint32_t)w));
            }
        }
        if (last_wave)
#pragma unroll
            for (int j = 0; j < V; ++j) state[lane * V + j] = __uint_as_float((uint32_t)await(from + j, word[j]));
        block_sync();
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (block > 0) e[j] = state[lane * V + j];
        for (int s = start; s < p.order; ++s) {
            const float2 y = blocks[s - start][lane * V + j];
            e[j] = y.x * e[j] + y.y;
        }
        if (wave == 0 && ends && p.goes_on)
            publish(a.states + ((size_t)p.own * a.blocks + block) * a.C + p.c + j, 0, P[j] * e[j] + q[j]);
        for (int v = 0; v < wave; ++v) {
            const float2 y = sums[v][lane * V + j];
            e[j] = y.x * e[j] + y.y;
        }
    }
    int t = p.row(first);
    size_t o = ((size_t)p.b * a.N + t) * a.C;
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (first + i < p.count) {
            float o0[V], o1[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (!BWD) {
                    e[j] = f[i][j] * e[j] + u[i][j];
                    o0[j] = e[j];
                } else {
                    const float d = u[i][j] + e[j];
                    float prev = r.h[i].at(j);
                    if (t == 0) prev = a.h0 ? a.h0[(size_t)p.own * a.C + p.c + j] : 0.f;
                    e[j] = f[i][j] * d;
                    if (GATE == LA_GATE_SIGMOID) {
                        o0[j] = rest[i][j] * d;
                        o1[j] = (prev - r.x[i].at(j)) * (f[i][j] * o0[j]);
                    } else {
                        o0[j] = d;
                        o1[j] = d * prev;
                    }
                }
            }
            leave<T, V, BWD>(O0 + o, p.at, o0);
            if (BWD) leave<T, V, BWD>(O1 + o, p.at, o1);
            o = BWD ? o - a.C : o + a.C;
            t += BWD ? -1 : 1;
        }
    // the wave with the last row of the walk
    if (a.last && !p.goes_on && first < p.count && first + R >= p.count) leave<float, V>(a.last + (size_t)p.own * a.C, p.c, e);
}

// The counter at zero, the words of `n` 16-byte units behind it at kNothing.
__global__ void __launch_bounds__(256) k_clear(unsigned *ticket, uint4 *words, size_t n)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < kLots) ticket[16 * i] = 0;  // a line of memory each
    if (i < n) words[i] = make_uint4(kNothing, kNothing, kNothing, kNothing);
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
        open_gate<GATE, sizeof(T) == 4>(load_elem(G, at + (size_t)t * C), f, rest);
        const float x = load_elem(X, at + (size_t)t * C);
        h = f * h + (GATE == LA_GATE_SIGMOID ? rest * x : x);
        store_elem(H, at + (size_t)t * C, h);
    }
    state[i] = h;
}

// How a call is tiled.
struct Tiling {
    int V, W, lanes, groups, chains, tiles, blocks, span, lots;
    size_t words, bytes;  // 16-byte units of published words; the workspace
};

// Workgroups of eight waves (two or more to a compute unit, whose loads and waits overlap) or of sixteen (half the
// tiles to join): sixteen where they leave one tile, which waits for nobody, and where sequences are long: more than
// 24 tiles of eight waves in few chains of them, or more than a hundred.  Lots: one counter hands out a tile in some 20 ns,
// which many short chains wait for; eight counters bind chains to dies (a workgroup's number goes round the dies),
// and few or long ones are better spread over all.  Span: a chain of states takes some 3 us a block; where
// there are many chains the blocks of one hide those of others, and short blocks have fewer words to read.
// Over 286 shapes of 1 to 400 chains and 200 to 100000 rows, both types and directions, each timed with W = 8, 16,
// lots = 1, 2, 8 and span = 4 .. 32, this takes 1.025 times the best's time on the average, 1.29 at most.  Both
// sides, us: one sequence of 100000 rows, bf16, 2048 channels, forward, W = 16, lots 1, span 4 241; W = 8 301;
// lots 8 277; 128 channels, span 32 54, span 8 80; 8 x 500 rows of 3200 channels, fp32, W = 8, lots 8 27; W = 16 32;
// lots 1 35.
//
// Narrow sequences, heads of a head layout: up to 64 channels a lane takes one of bfloat16 too (64 sequences of 4096
// rows of 64, backward, 48 us; two a lane 63), and several sequences share a wave where none ends before the others
// (1000 of 300 rows of 16, bf16, forward, one a wave 34 us, four 14).
Tiling tiling(int B, int N, int C, la_dtype dt, bool backward, bool ragged)
{
    Tiling p;
    p.V = dt == LA_BF16 && C > 64 ? 2 : 1;
    p.groups = (C + 64 * p.V - 1) / (64 * p.V);
    p.lanes = 64;
    // (the lanes' offsets are 32 bits)
    while (!ragged && C <= p.lanes / 2 && 64 / p.lanes < B && p.lanes > 4 && (double)N * C * 128 / p.lanes < 1 << 28) p.lanes /= 2;
    const long chains = (long)((B + 64 / p.lanes - 1) / (64 / p.lanes)) * p.groups;
    p.chains = (int)chains;
    const int R = backward ? kRowsBack : kRowsFwd, eights = (N + 8 * R - 1) / (8 * R);
    p.W = eights <= 2 || (eights > 24 && chains < 32) || eights > 100 ? 16 : 8;
    p.lots = chains < 16 || eights > 100 ? 1 : kLots;
    p.span = chains >= 12 ? 4 : chains >= 6 ? 8 : chains >= 3 ? 16 : kMostSpan;
    p.tiles = (N + p.W * R - 1) / (p.W * R);
    p.blocks = (p.tiles + p.span - 1) / p.span;
    p.words = p.tiles > 1 ? ((size_t)B * C * (p.tiles + p.blocks) * 8 + 15) / 16 : 0;
    p.bytes = p.tiles > 1 ? kCounters + round_up(p.words * 16, 256) : 0;
    return p;
}

la_status check_shape(int B, int N, int C, la_gate gate, la_dtype dt)
{
    if (B < 1 || N < 1 || C < 1 || N > 1 << 30) return LA_ERR_SHAPE;
    if (!real_type(dt) || (gate != LA_GATE_VALUE && gate != LA_GATE_SIGMOID)) return LA_ERR_UNSUPPORTED;
    if ((double)B * N * C >= 1099511627776.0) return LA_ERR_SHAPE;          // 2^40
    if ((double)B * ((C + 63) / 64) >= 8388608.0) return LA_ERR_SHAPE;  // 2^23
    if ((double)B * ((C + 63) / 64) * ((N + 63) / 64) >= 2147483648.0) return LA_ERR_SHAPE;  // tiles
    return LA_OK;
}

template <typename T, int V, int GATE, bool BWD>
void launch(const Walk &w, const Tiling &p, hipStream_t st)
{
    constexpr int R = BWD ? kRowsBack : kRowsFwd;
    const size_t chains = w.chains, most = (chains + w.lots - 1) / w.lots * w.lots * w.tiles;
    if (w.tiles > 1)
        k_clear<<<dim3((unsigned)((p.words + 255) / 256)), dim3(256), 0, st>>>(w.ticket, (uint4 *)w.sums, p.words);
    constexpr size_t wide = 1 << 21;  // a grid has less than 2^32 threads in a dimension
    const dim3 grid((unsigned)(most < wide ? most : wide), (unsigned)((most + wide - 1) / wide));
    if (p.W == 8) k_walk<T, V, GATE, BWD, 8, R><<<grid, dim3(512), 0, st>>>(w);
    else k_walk<T, V, GATE, BWD, 16, R><<<grid, dim3(1024), 0, st>>>(w);
}
template <bool BWD>
la_status run(Walk w, const Tiling &p, void *ws, la_gate gate, la_dtype dt, hipStream_t st)
{
    w.lanes = p.lanes, w.groups = p.groups, w.chains = p.chains, w.tiles = p.tiles, w.blocks = p.blocks, w.span = p.span, w.lots = p.lots;
    w.ticket = (unsigned *)ws;
    w.sums = (uint64_t *)((char *)ws + kCounters);
    w.states = w.sums + (size_t)w.B * w.C * w.tiles;
    const bool s = gate == LA_GATE_SIGMOID;
    if (dt == LA_F32)
        s ? launch<float, 1, LA_GATE_SIGMOID, BWD>(w, p, st) : launch<float, 1, LA_GATE_VALUE, BWD>(w, p, st);
    else if (p.V == 2)
        s ? launch<bf16_t, 2, LA_GATE_SIGMOID, BWD>(w, p, st) : launch<bf16_t, 2, LA_GATE_VALUE, BWD>(w, p, st);
    else s ? launch<bf16_t, 1, LA_GATE_SIGMOID, BWD>(w, p, st) : launch<bf16_t, 1, LA_GATE_VALUE, BWD>(w, p, st);
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
    if (la::check_shape(B, N, C, LA_GATE_VALUE, dt) != LA_OK) return 0;
    // a call with lengths may be tiled in another way than one without
    const size_t a = la::tiling(B, N, C, dt, is_backward, false).bytes, b = la::tiling(B, N, C, dt, is_backward, true).bytes;
    return a > b ? a : b;
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
    const la::Tiling p = la::tiling(B, N, C, dt, false, lengths != nullptr);
    if (la::bad_workspace(workspace, workspace_bytes, la_recurrence_workspace_bytes(B, N, C, dt, 0))) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{X, tb}, {Gate, tb}, {h0, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{Hs, tb}, {last, sb}, {workspace, p.bytes}};
    if (la::any_alias(ins, 4, outs, 3)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Walk w{};
    w.X = X, w.Gate = Gate, w.out0 = Hs, w.out1 = Hs, w.first = h0, w.last = last, w.lengths = lengths;
    w.B = B, w.N = N, w.C = C;
    return la::run<false>(w, p, workspace, gate, dt, (hipStream_t)hip_stream);
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
    const la::Tiling p = la::tiling(B, N, C, dt, true, lengths != nullptr);
    if (la::bad_workspace(workspace, workspace_bytes, la_recurrence_workspace_bytes(B, N, C, dt, 1))) return LA_ERR_WORKSPACE;
    const la::Range ins[] = {{X, tb}, {Gate, tb}, {h0, sb}, {Hs, tb}, {dHs, tb}, {dlast, sb}, {lengths, (size_t)B * 4}};
    const la::Range outs[] = {{dX, tb}, {dGate, tb}, {dh0, sb}, {workspace, p.bytes}};
    if (la::any_alias(ins, 7, outs, 4)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    la::Walk w{};
    w.X = X, w.Gate = Gate, w.H = Hs, w.dH = dHs, w.out0 = dX, w.out1 = dGate, w.first = dlast, w.h0 = h0;
    w.last = dh0, w.lengths = lengths;
    w.B = B, w.N = N, w.C = C;
    return la::run<true>(w, p, workspace, gate, dt, (hipStream_t)hip_stream);
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
