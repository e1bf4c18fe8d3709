// Selective state space scan: S states to a channel, h[s] -> exp(d A[s]) h[s] + d x B[s], read out by C: forward, backward,
// in steps.
//
// A lane holds one channel, a wave P of its states in registers, a workgroup's W waves all S <= P W of them; it walks a
// sequence (or a segment of one) in tiles of 16 rows.  The waves share a tile's rows: each forms d and d x of its rows
// and leaves them in LDS; then every wave walks all rows with its states, and at last each wave adds up the waves'
// shares of its rows' outputs.  B and C of a row are the same for all channels: a wave keeps a tile's as one value a lane, and the
// instruction that needs one reads the lane that has it (through LDS every wave would read them back 64 times over; through
// scalar loads 8 x 2048 rows took 373 us, this way 302 when both were tried).  Where there are few sequences and channels,
// these are cut into segments, walked side by side from zero states first to learn where each of them starts (lay_out).
//
// The backward pass goes by the states before every tile, which the forward pass keeps (S / 4 bytes an element of X): a
// tile is walked forward once more, half of it at a time with all its states and decays in registers, then back.
//
// Bound by the vector ALU: a state and row of 64 channels takes 21 cycles of a SIMD forward (an exponential 7, two products, a
// sum, the read-out; reading another lane's value doubles an instruction's time) and 65 backward (states one and a half times, eight operations,
// sums over the channels 16 to 19).  8 x 2048 rows of 2048 channels, 16 states, bf16: 82 and 254 us of that at 2.1 GHz, 105 us of bytes,
// 220 and 470 measured (there are 256 chains, two waves to a SIMD); 64 x 512 rows, 164 and 508, 265 and 769.
#include "la_checks.h"
#include "la_common.h"
#include "la_scalar.h"

namespace la {
namespace {

constexpr int kMostStates = 128;
constexpr int kRows = 16, kPairs = kRows / 2;  // of a tile
// What the backward pass keeps of kCells / P rows, h and exp(d A) of every row and state: 64 registers, and its 64
// sums over a wave's channels, of either kind, are folded together.  Where a tile has more rows they are taken in parts,
// the states before a part formed once more from those before the tile.
constexpr int kCells = 32;

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
    float *shares;       // [B, columns, tiles, W, parts, 2, kCells] sums over a column's channels for dB, dC
    float *dA, *dd;      // [B * segs, S, C], [B * segs, 2, C] a segment's sums for dA; for dD and dbias
    float *sums, *spans; // [B, segs, S, C] what a segment makes of zero states, then the states it starts from; [B, segs, C] the sum of its d
    int B, N, C, S, G, group, per, columns;  // channels of a group; columns of 64 channels to it, in all
    int tiles, seg, segs;                    // tiles of the sequence; rows of a segment, segments
    int step;
};

__device__ __forceinline__ int rows_of(const Scan &a, int b)
{
    return a.lengths ? min(max(a.lengths[b], 0), a.N) : a.N;
}
// Where a workgroup is: its sequence, channels and rows.
struct Spot {
    int b, column, g, seg, n, r0, r1;
    unsigned c;
    bool live;
    __device__ __forceinline__ Spot(const Scan &a, int lane)
    {
        const unsigned k = blockIdx.x / a.segs;
        seg = (int)(blockIdx.x % a.segs);
        column = (int)(k % a.columns), b = (int)(k / a.columns);
        g = column / a.per;
        const int mine = g * a.group + column % a.per * 64 + lane, behind = (g + 1) * a.group;
        live = mine < behind;
        c = (unsigned)min(mine, behind - 1);  // lanes behind the group's last channel read that one
        n = a.lengths ? min(max(__builtin_amdgcn_readfirstlane(a.lengths[b]), 0), a.N) : a.N;
        r0 = min(seg * a.seg, a.N);
        r1 = min(n, r0 + a.seg);
    }
};

// The rows of a tensor from the tile's first on, by a buffer's descriptor: a scalar address, a scalar offset of the row and a
// lane's place in it in 32 bits, so that no lane adds up addresses.  (The descriptor is not asked to check: rows are
// clamped to those that there are.)
template <typename T>
struct Rows {
    char *tile;
    unsigned stride, lane;  // bytes
    __device__ __forceinline__ Rows(const void *p, size_t row, size_t stride, size_t column, unsigned lane)
        : tile((char *)p + (row * stride + column) * sizeof(T)), stride((unsigned)(stride * sizeof(T))), lane(lane * (unsigned)sizeof(T))
    {
    }
    __device__ __forceinline__ void move(int tiles) { tile += (ptrdiff_t)tiles * kRows * (ptrdiff_t)stride; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer() const
    {
        return __builtin_amdgcn_make_buffer_rsrc(tile, 0, 0x7fffffff, 0x00020000);
    }
    __device__ __forceinline__ T operator[](int row) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(buffer(), lane, row * stride, 0));
        else return __builtin_amdgcn_raw_buffer_load_b16(buffer(), lane, row * stride, 0);
    }
    __device__ __forceinline__ void put(int row, float x) const
    {
        if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), buffer(), lane, row * stride, 0);
        else {
            const __bf16 c = (__bf16)x;
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(short, c), buffer(), lane, row * stride, 0);
        }
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

// What stands before it in the source comes before what stands behind it: the compiler would ask for all of a tile's rows first
// and hold them in registers.
__device__ __forceinline__ void keep_order()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// x is there here, and not where it is used: what it was made from is let go of.
__device__ __forceinline__ void settle(float &x) { asm volatile("" : "+v"(x)); }

// B or C of a tile for the P states of a wave: value P row + state stands in lane (P row + state) % 16 of every 16 lanes of a
// register, from where the instruction that needs it reads it for all of them; zeros behind the last state and row.
template <typename T, int P>
struct Vector {
    static constexpr int REGS = kRows * P / 16, STEP = 16 / P;  // rows of a register
    Rows<T> from;
    uint32_t mask;
    int row;
    uint32_t raw[REGS];
    float v[REGS];
    __device__ __forceinline__ Vector(const void *p, size_t row0, size_t stride, const Scan &a, const Spot &s, int wave, int lane)
        : from(p, row0, stride, (size_t)s.g * a.S, 0)
    {
        const int k = lane % 16, state = wave * P + k % P;
        mask = state < a.S ? 0xffffffffu : 0;
        row = k / P;
        from.lane = (unsigned)row * from.stride + (unsigned)min(state, a.S - 1) * (unsigned)sizeof(T);
    }
    // rows: how many of the tile's there are
    __device__ __forceinline__ void request(int rows)
    {
        if (rows >= kRows) {
#pragma unroll
            for (int i = 0; i < REGS; ++i) raw[i] = widen(from[STEP * i]);
        } else {
#pragma unroll
            for (int i = 0; i < REGS; ++i) {
                raw[i] = 0;
                if (STEP * i + row < rows) raw[i] = widen(from[STEP * i]);
            }
        }
    }
    static __device__ __forceinline__ uint32_t widen(float x) { return __float_as_uint(x); }
    static __device__ __forceinline__ uint32_t widen(bf16_t x) { return x; }
    __device__ __forceinline__ void arrive()
    {
#pragma unroll
        for (int i = 0; i < REGS; ++i) v[i] = __uint_as_float((sizeof(T) == 4 ? raw[i] : raw[i] << 16) & mask);
    }
};
// The value of lane K of 16.
template <int K>
__device__ __forceinline__ float of_lane(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x150 + K, 0xf, 0xf, true));
}
// acc_j += v_{K+j} x, and sum_j v_{K+j} x_j, v_k being the value of lane k of 16.  (A register that another lane's value is read
// from is ready two instructions after it was written.)
#define LA_OF_LANE(op, acc, x, k) "v_" op "_f32_dpp " acc ", %[v], " x " row_newbcast:" k " row_mask:0xf bank_mask:0xf\n\t"
template <int K, int P, int J = 0>
__device__ __forceinline__ void fma_each(float (&acc)[P], float v, float x)
{
    if constexpr (P == 2)
        asm("s_nop 1\n\t" LA_OF_LANE("fmac", "%0", "%[x]", "%[k0]") LA_OF_LANE("fmac", "%1", "%[x]", "%[k1]")
            : "+v"(acc[0]), "+v"(acc[1]) : [v] "v"(v), [x] "v"(x), [k0] "n"(K), [k1] "n"(K + 1));
    else {
        asm("s_nop 1\n\t" LA_OF_LANE("fmac", "%0", "%[x]", "%[k0]") LA_OF_LANE("fmac", "%1", "%[x]", "%[k1]")
            LA_OF_LANE("fmac", "%2", "%[x]", "%[k2]") LA_OF_LANE("fmac", "%3", "%[x]", "%[k3]")
            : "+v"(acc[J]), "+v"(acc[J + 1]), "+v"(acc[J + 2]), "+v"(acc[J + 3])
            : [v] "v"(v), [x] "v"(x), [k0] "n"(K + J), [k1] "n"(K + J + 1), [k2] "n"(K + J + 2), [k3] "n"(K + J + 3));
        if constexpr (J + 4 < P) fma_each<K, P, J + 4>(acc, v, x);
    }
}
template <int K, int P, int J = 0>
__device__ __forceinline__ float sum_all(float v, const float (&x)[P])
{
    float a, b = 0.f;
    if constexpr (P == 2)
        asm("s_nop 1\n\t" LA_OF_LANE("mul", "%0", "%[x0]", "%[k0]") LA_OF_LANE("fmac", "%0", "%[x1]", "%[k1]")
            : "=&v"(a) : [v] "v"(v), [x0] "v"(x[0]), [x1] "v"(x[1]), [k0] "n"(K), [k1] "n"(K + 1));
    else {
        asm("s_nop 1\n\t" LA_OF_LANE("mul", "%0", "%[x0]", "%[k0]") LA_OF_LANE("mul", "%1", "%[x1]", "%[k1]")
            LA_OF_LANE("fmac", "%0", "%[x2]", "%[k2]") LA_OF_LANE("fmac", "%1", "%[x3]", "%[k3]")
            : "=&v"(a), "=&v"(b)
            : [v] "v"(v), [x0] "v"(x[J]), [x1] "v"(x[J + 1]), [x2] "v"(x[J + 2]), [x3] "v"(x[J + 3]), [k0] "n"(K + J), [k1] "n"(K + J + 1),
              [k2] "n"(K + J + 2), [k3] "n"(K + J + 3));
        a += b;
        if constexpr (J + 4 < P) a += sum_all<K, P, J + 4>(v, x);
    }
    return a;
}
#undef LA_OF_LANE

// A[s] in powers of two.  Finite, where it is not NaN, so that a row that is not there (d = 0) leaves the state as it is; below
// the lowest number any d > 2^-120 forgets the state.
__device__ __forceinline__ float decay_of(float A)
{
    const float x = A * kLog2e, low = -0x1.fffffep127f;
    return x < low ? low : x;
}
// (Places behind the last state have its decay: a number wherever that is one.)
template <int P>
__device__ __forceinline__ void decays(const Scan &a, const Spot &p, int wave, float (&A)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        A[j] = decay_of(a.A[(size_t)p.c * a.S + min(wave * P + j, a.S - 1)]);
    }
}
// v, or 0 where the mask is 0, also of an infinity.
__device__ __forceinline__ float held(float v, uint32_t mask) { return __uint_as_float(__float_as_uint(v) & mask); }
// Whether the states fill the waves' places: kAll; kWaves, some waves hold none, and leave zeros; kPlaces, a wave holds fewer than P.  Places
// without a state have B = 0 and C = 0, and what would be an infinity times these is taken out.
enum Fill { kAll, kWaves, kPlaces };
template <int P, Fill FILL>
struct Places {
    uint32_t mask[P];
    __device__ __forceinline__ Places(const Scan &a, int wave)
    {
#pragma unroll
        for (int j = 0; j < P; ++j) mask[j] = wave * P + j < a.S ? 0xffffffffu : 0;
    }
    __device__ __forceinline__ float of(float v, int j) const { return FILL == kPlaces ? held(v, mask[j]) : v; }
};
// The states that the walk starts from: the caller's, or those that k_selective_chain left for the segment.
template <int P>
__device__ __forceinline__ void states_from(const Scan &a, const Spot &p, int wave, float (&h)[P])
{
#pragma unroll
    for (int j = 0; j < P; ++j) {
        const int s = wave * P + j;
        h[j] = 0.f;
        if (!p.live || s >= a.S) continue;
        if (a.segs > 1) h[j] = a.sums[(((size_t)p.b * a.segs + p.seg) * a.S + s) * a.C + p.c];
        else if (a.first) h[j] = a.first[((size_t)p.b * a.C + p.c) * a.S + s];
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
// The sum of a segment's d from those of its tiles (pairs of rows, then eight of these: 8 U), with what every addition loses: within
// 10 U of it however many rows the segment has.  One serial sum of a thousand equal d is off by some 250 U, which exp(A sum d) has of
// a state that the segment carries on.
struct Span {
    float large = 0.f, lost = 0.f;
    __device__ __forceinline__ void add(float x)
    {
        const float s = large + x, taken = s - large;
        lost += (large - (s - taken)) + (x - taken);
        large = s;
    }
    __device__ __forceinline__ float sum() const { return lost == lost ? large + lost : large; }  // infinities lose NaN
};
template <int P>
__device__ __forceinline__ void leave_sums(const Scan &a, const Spot &p, int wave, const float (&h)[P], float span)
{
    if (!p.live) return;
    const size_t at = (size_t)p.b * a.segs + p.seg;
#pragma unroll
    for (int j = 0; j < P; ++j)
        if (wave * P + j < a.S) a.sums[(at * a.S + wave * P + j) * a.C + p.c] = h[j];
    if (wave == 0) a.spans[at * a.C + p.c] = span;
}

// The states that every segment starts from, in place of what it makes of zero states: a lane to a state of a channel.
template <bool BWD>
__global__ void __launch_bounds__(256) k_selective_chain(Scan a)
{
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (size_t)a.B * a.S * a.C) return;
    const int c = (int)(i % a.C), s = (int)(i / a.C % a.S), b = (int)(i / a.C / a.S);
    const float A = decay_of(a.A[(size_t)c * a.S + s]);
    float h = a.first ? a.first[((size_t)b * a.C + c) * a.S + s] : 0.f;
    constexpr int AHEAD = 16;  // segments whose words are asked for together
    for (int k0 = 0; k0 < a.segs; k0 += AHEAD) {
        float own[AHEAD], span[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int k = min(k0 + i, a.segs - 1);
            const size_t at = (size_t)b * a.segs + (BWD ? a.segs - 1 - k : k);
            own[i] = a.sums[(at * a.S + s) * a.C + c], span[i] = a.spans[at * a.C + c];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (k0 + i >= a.segs) break;
            const size_t at = (size_t)b * a.segs + (BWD ? a.segs - 1 - k0 - i : k0 + i);
            a.sums[(at * a.S + s) * a.C + c] = h;
            const float f = __builtin_amdgcn_exp2f(span[i] * A);  // 0 behind many rows, of which none had 0
            h = fabsf(h) == INFINITY && f == 0.f ? h + own[i] : fmaf(f, h, own[i]);
        }
    }
}

// FULL: outputs.  Else what the segment makes of zero states.
template <typename T, int P, int W, bool FULL, Fill FILL>
__global__ void __launch_bounds__(64 * W) k_selective(Scan a)
{
    constexpr int OWN = (kPairs + W - 1) / W;  // pairs of rows that a wave prepares
    __shared__ float4 du[kPairs][64];
    __shared__ float2 ys[FULL ? W : 1][kPairs][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Spot p(a, lane);
    const Places<P, FILL> places(a, wave);
    float A[P], h[P];
    Span span;
    decays<P>(a, p, wave, A);
    if (FULL) states_from<P>(a, p, wave, h);
    else
#pragma unroll
        for (int j = 0; j < P; ++j) h[j] = 0.f;
    const float bias = a.bias ? a.bias[p.c] : 0.f, D = a.D ? a.D[p.c] : 0.f;
    const size_t row0 = (size_t)p.b * a.N + p.r0;
    Rows<T> X(a.X, row0, a.xs, 0, p.c), Dt(a.Dt, row0, a.ts, 0, p.c), Y(a.Y, row0, a.C, 0, p.c);
    Vector<T, P> B(a.Bm, row0, a.bs, a, p, wave, lane), C(a.Cm, row0, a.cs, a, p, wave, lane);
    float *saved = a.saved ? a.saved + (((size_t)p.b * a.tiles + p.r0 / kRows) * a.S + wave * P) * a.C : nullptr;
    T x[OWN][2], dt[OWN][2];
    auto request = [&](int rows) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int q = wave + i * W;
            if (kPairs % W && q >= kPairs) break;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = min(2 * q + r, rows - 1);
                x[i][r] = X[row], dt[i][r] = Dt[row];
            }
        }
        B.request(rows);
        if (FULL) C.request(rows);
    };
    if (p.r0 < p.r1) request(p.r1 - p.r0);
    for (int t = p.r0; t < p.r1; t += kRows) {
        const int rows = p.r1 - t;
        float xw[OWN][2];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int q = wave + i * W;
            if (kPairs % W && q >= kPairs) break;
            float d[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float slope;
                d[r] = step_of<sizeof(T) == 4>(load_elem(dt[i], r) + bias, a.step, slope);
                xw[i][r] = load_elem(x[i], r);
                if (2 * q + r >= rows) d[r] = xw[i][r] = 0.f;
            }
            du[q][lane] = make_float4(d[0], d[0] * xw[i][0], d[1], d[1] * xw[i][1]);
        }
        B.arrive();
        if (FULL) C.arrive();
        block_sync();
        if (rows > kRows) {
            X.move(1), Dt.move(1), B.from.move(1), C.from.move(1);
            request(rows - kRows);
        }
        if (FULL && a.saved) {
            if (p.live)
#pragma unroll
                for (int j = 0; j < P; ++j)
                    if (wave * P + j < a.S) saved[(size_t)j * a.C + p.c] = h[j];
            saved += (size_t)a.S * a.C;
        }
        float4 s = du[0][lane], next = du[1][lane];
        float of_tile = 0.f;  // the sum of d
        float f[2 * P], g[2 * P];  // exp(d A) of a pair of rows, and of the next
        auto open = [&](float (&f)[2 * P], const float4 &s) {
#pragma unroll
            for (int j = 0; j < 2 * P; ++j) f[j] = __builtin_amdgcn_exp2f((j < P ? s.x : s.z) * A[j % P]);
        };
        open(f, s);
        each<kPairs>([&](auto q_) {
            constexpr int q = decltype(q_)::value;
            const float4 after = du[q + 2 < kPairs ? q + 2 : kPairs - 1][lane];
            float y[2];
            if constexpr (q + 1 < kPairs) open(g, next);
            each<2>([&](auto r_) {
                constexpr int r = decltype(r_)::value, k = (2 * q + r) * P;
                each<P>([&](auto j) {
                    const float u = places.of(r ? s.w : s.y, j);
                    h[j] = fmaf(f[r * P + j], h[j], u * of_lane<k % 16 + decltype(j)::value>(B.v[k / 16]));
                });
                if (FULL) y[r] = sum_all<k % 16>(C.v[k / 16], h);
            });
            if (!FULL) of_tile += s.x + s.z;
            if (FULL) ys[wave][q][lane] = make_float2(y[0], y[1]);
            s = next, next = after;
#pragma unroll
            for (int j = 0; j < 2 * P; ++j) f[j] = g[j];
            keep_order();
        });
        if (!FULL) span.add(of_tile);
        if (FULL && FILL != kAll && wave * P >= a.S)
            for (int q = 0; q < kPairs; ++q) ys[wave][q][lane] = make_float2(0.f, 0.f);
        block_sync();
        if (FULL) {
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int q = wave + i * W;
                if (kPairs % W && q >= kPairs) break;
                float y[2] = {D * xw[i][0], D * xw[i][1]};
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float2 v = ys[w][q][lane];
                    y[0] += v.x, y[1] += v.y;
                }
                if (p.live) {
                    if (2 * q < rows) Y.put(2 * q, y[0]);
                    if (2 * q + 1 < rows) Y.put(2 * q + 1, y[1]);
                }
            }
            Y.move(1);
        }
    }
    if (FULL) {
        if (p.live)
            for (int t = max(p.r0, p.n) + wave; t < min(a.N, p.r0 + a.seg); t += W)  // padding
                store_elem((T *)a.Y, ((size_t)p.b * a.N + t) * a.C + p.c, 0.f);
        if (p.seg == max(p.n - 1, 0) / a.seg) states_to<P>(a.end, a, p, wave, h);
    } else leave_sums<P>(a, p, wave, h, span.sum());
}

// 64 values a lane, added up over the wave's lanes.  At every step a lane keeps half of its values, by a bit of its
// number, and adds the partner's share of them, so that 64 sums take a lane 116 additions and not 6 each.  First the partners
// within 16 lanes (rotated by 8, mirrored in 8), whose shares the additions read in place, the kept half chosen by
// the instruction's mask of banks, two additions a value; then halves and quarters of the wave change places, one instruction for two values; the
// last four values are added up over four neighbours.  Lane l ends with values 32 l3 + 16 l2 + 8 l5 + 4 l4 + (0 .. 3), l3 being bit 3
// of l.  An instruction that reads another lane's register needs two others behind the one that wrote it.
#define LA_FOLD(to, from, how, banks) "v_add_f32_dpp " to ", " to ", " to " " how " row_mask:0xf bank_mask:0xf\n\t" \
                                     "v_add_f32_dpp " to ", " from ", " from " " how " row_mask:0xf bank_mask:" banks "\n\t"
__device__ __forceinline__ float4 over_lanes(float (&v)[64])
{
#pragma unroll
    for (int i = 0; i < 32; i += 4)
        asm("s_nop 1\n\t" LA_FOLD("%0", "%4", "row_ror:8", "0xc") LA_FOLD("%1", "%5", "row_ror:8", "0xc")
            LA_FOLD("%2", "%6", "row_ror:8", "0xc") LA_FOLD("%3", "%7", "row_ror:8", "0xc")
            : "+v"(v[i]), "+v"(v[i + 1]), "+v"(v[i + 2]), "+v"(v[i + 3])
            : "v"(v[i + 32]), "v"(v[i + 33]), "v"(v[i + 34]), "v"(v[i + 35]));
#pragma unroll
    for (int i = 0; i < 16; i += 4)
        asm("s_nop 1\n\t" LA_FOLD("%0", "%4", "row_half_mirror", "0xa") LA_FOLD("%1", "%5", "row_half_mirror", "0xa")
            LA_FOLD("%2", "%6", "row_half_mirror", "0xa") LA_FOLD("%3", "%7", "row_half_mirror", "0xa")
            : "+v"(v[i]), "+v"(v[i + 1]), "+v"(v[i + 2]), "+v"(v[i + 3])
            : "v"(v[i + 16]), "v"(v[i + 17]), "v"(v[i + 18]), "v"(v[i + 19]));
#pragma unroll
    for (int i = 0; i < 8; i += 4)  // the compiler does not see what the instructions above wrote: it would not wait
        asm("s_nop 1" : "+v"(v[i]), "+v"(v[i + 1]), "+v"(v[i + 2]), "+v"(v[i + 3]), "+v"(v[i + 8]), "+v"(v[i + 9]), "+v"(v[i + 10]), "+v"(v[i + 11]));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
        v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 4]), false, false);
        v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
        v[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[i]), 0xb1, 0xf, 0xf, true));
        v[i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[i]), 0x4e, 0xf, 0xf, true));
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}
#undef LA_FOLD

// Backward.  FULL: outputs, walking the tiles from the far end: states from the saved ones before the tile on, then the rows in
// reverse.  Else what the segment hands to the rows before it from nothing behind it.
// Registers, of as many waves to a SIMD as the attribute says: 168 for three (two, four and six waves a workgroup spill 12 to 20 bytes a
// lane, for 170 and two waves to a SIMD they would not; twelve waves of eight states 184); eight waves, of which four to a SIMD would have 128 and spill 136 bytes, run
// two to a SIMD (4 x 2048 rows of 1024, 32 states, fp32: 280 us, with four 379); 16 waves a workgroup can't have more than 128 (380 bytes
// of spills).
template <typename T, int P, int W, bool FULL, Fill FILL>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(!FULL || W == 16 ? 4 : W == 8 ? 2 : 3))) k_selective_back(Scan a)
{
    constexpr int OWN = (kPairs + W - 1) / W, PART = kCells / P, PARTS = kRows / PART;
    __shared__ float4 du[kPairs][64];
    __shared__ float2 dys[kPairs][64];
    __shared__ float4 gs[FULL ? W : 1][kPairs][64];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
    const Spot p(a, lane);
    const Places<P, FILL> places(a, wave);
    float A[P], carry[P], dA[P], before[P], dD = 0.f, db = 0.f;
    Span span;
    decays<P>(a, p, wave, A);
    if (FULL) states_from<P>(a, p, wave, carry);
#pragma unroll
    for (int j = 0; j < P; ++j) {
        dA[j] = 0.f;
        if (!FULL) carry[j] = 0.f;
    }
    const float bias = a.bias ? a.bias[p.c] : 0.f, D = a.D ? a.D[p.c] : 0.f;
    const int tiles = p.r0 < p.r1 ? (p.r1 - p.r0 + kRows - 1) / kRows : 0, last = p.r0 + max(tiles - 1, 0) * kRows;
    const size_t row0 = (size_t)p.b * a.N + last;
    Rows<T> X(a.X, row0, a.xs, 0, p.c), Dt(a.Dt, row0, a.ts, 0, p.c), dY(a.dY, row0, a.C, 0, p.c), dX(a.dX, row0, a.C, 0, p.c), dDt(a.dDt, row0, a.C, 0, p.c);
    Vector<T, P> B(a.Bm, row0, a.bs, a, p, wave, lane), C(a.Cm, row0, a.cs, a, p, wave, lane);
    const float *saved = a.saved + (((size_t)p.b * a.tiles + last / kRows) * a.S + wave * P) * a.C;
    float *shares = a.shares + ((((size_t)p.b * a.columns + p.column) * a.tiles + last / kRows) * W + wave) * PARTS * 64;
    T x[OWN][2], dt[OWN][2], dy[OWN][2];
    auto request = [&](int rows) {
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int q = wave + i * W;
            if (kPairs % W && q >= kPairs) break;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = min(2 * q + r, rows - 1);
                if (FULL) x[i][r] = X[row];
                dt[i][r] = Dt[row], dy[i][r] = dY[row];
            }
        }
        if (FULL) B.request(rows);
        C.request(rows);
        if (FULL)
#pragma unroll
            for (int j = 0; j < P; ++j) before[j] = p.live && wave * P + j < a.S ? saved[(size_t)j * a.C + p.c] : 0.f;
    };
    // lanes without a channel of their own have no share in the sums over channels
    const uint32_t mask = p.live ? 0xffffffffu : 0;
    auto of_live = [&](float v) { return held(v, mask); };
    if (tiles) request(p.r1 - last);
    for (int k = 0, rows = p.r1 - last; k < tiles; ++k, rows = kRows) {
        float xw[OWN][2], slope[OWN][2];
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            const int q = wave + i * W;
            if (kPairs % W && q >= kPairs) break;
            float d[2], y[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                d[r] = of_live(step_of<sizeof(T) == 4>(load_elem(dt[i], r) + bias, a.step, slope[i][r]));
                xw[i][r] = FULL ? of_live(load_elem(x[i], r)) : 0.f;
                y[r] = of_live(load_elem(dy[i], r));
                if (2 * q + r >= rows) d[r] = xw[i][r] = y[r] = 0.f;
            }
            du[q][lane] = make_float4(d[0], d[0] * xw[i][0], d[1], d[1] * xw[i][1]);
            dys[q][lane] = make_float2(y[0], y[1]);
        }
        if (FULL) B.arrive();
        C.arrive();
        float begin[P];
#pragma unroll
        for (int j = 0; j < P; ++j) begin[j] = FULL ? before[j] : 0.f;
        block_sync();
        if (k + 1 < tiles) {
            X.move(-1), Dt.move(-1), dY.move(-1), B.from.move(-1), C.from.move(-1);
            saved -= (size_t)a.S * a.C;
            request(kRows);
        }
        if constexpr (FULL) {
            each<PARTS>([&](auto part_) {
                constexpr int part = PARTS - 1 - decltype(part_)::value, first = part * PART / 2;  // pair
                float v[64], h0[P], own[P];  // f: exp(d A), then shares of dB; h, then shares of dC
                float *const f = v, *const h = v + kCells;
#pragma unroll
                for (int j = 0; j < P; ++j) h0[j] = begin[j], own[j] = 0.f;
                each<first>([&](auto q_) {
                    constexpr int q = decltype(q_)::value;
                    const float4 s = du[q][lane];
                    each<2 * P>([&](auto i) {
                        constexpr int r = decltype(i)::value / P, j = decltype(i)::value % P, k = (2 * q + r) * P + j;
                        h0[j] = fmaf(__builtin_amdgcn_exp2f((r ? s.z : s.x) * A[j]), h0[j], (r ? s.w : s.y) * of_lane<k % 16>(B.v[k / 16]));
                    });
                    if (q % 2) keep_order();
                });
#pragma unroll
                for (int j = 0; j < P; ++j) h0[j] = places.of(h0[j], j);
                float4 s = du[first][lane];
                each<PART / 2>([&](auto q_) {
                    constexpr int q = decltype(q_)::value;
                    const float4 next = du[first + (q + 1 < PART / 2 ? q + 1 : q)][lane];
                    each<2 * P>([&](auto i) {
                        constexpr int r = decltype(i)::value / P, j = decltype(i)::value % P, k = (2 * q + r) * P + j, at = k + 2 * first * P;
                        const float u = places.of(r ? s.w : s.y, j);
                        f[k] = __builtin_amdgcn_exp2f((r ? s.z : s.x) * A[j]);
                        h[k] = fmaf(f[k], k >= P ? h[k - P] : h0[j], u * of_lane<at % 16>(B.v[at / 16]));
                        settle(f[k]), settle(h[k]);
                    });
                    s = next;
                    keep_order();
                });
                float2 y2 = dys[first + PART / 2 - 1][lane];
                each<PART / 2>([&](auto q_) {
                    constexpr int q = PART / 2 - 1 - decltype(q_)::value;
                    const float4 next = du[first + (q ? q - 1 : q)][lane];
                    const float2 nexty = dys[first + (q ? q - 1 : q)][lane];
                    float gu[2], gd[2];
                    each<2>([&](auto r_) {
                        constexpr int r = 1 - decltype(r_)::value, k = (2 * q + r) * P, at = k + 2 * first * P;
                        const float d = r ? s.z : s.x, u = r ? s.w : s.y, y = r ? y2.y : y2.x;
                        fma_each<at % 16>(carry, C.v[at / 16], y);
#pragma unroll
                        for (int j = 0; j < P; ++j) carry[j] = places.of(carry[j], j);
                        gu[r] = sum_all<at % 16>(B.v[at / 16], carry);
#pragma unroll
                        for (int j = 0; j < P; ++j) {
                            const float g = carry[j];
                            carry[j] = g * f[k + j];
                            const float e = carry[j] * (k ? h[k - P + j] : h0[j]);
                            gd[r] = j ? fmaf(e, A[j], gd[r]) : e * A[j];
                            own[j] = fmaf(e, d, own[j]);
                            f[k + j] = g * u;
                            h[k + j] *= y;
                            settle(f[k + j]), settle(h[k + j]), settle(own[j]), settle(carry[j]);
                        }
                    });
                    gs[wave][first + q][lane] = make_float4(gu[0], gd[0], gu[1], gd[1]);
                    s = next, y2 = nexty;
                    keep_order();
                });
#pragma unroll
                for (int j = 0; j < P; ++j) dA[j] += own[j];
                // lanes without a channel: B or C may be infinite.  Columns that have none skip this.
                if (!p.live)
#pragma unroll
                    for (int i = 0; i < 64; ++i) asm volatile("v_mov_b32 %0, 0" : "=v"(v[i]));
                const float4 sum = over_lanes(v);
                if (lane % 4 == 0)
                    *(float4 *)(shares + part * 64 + (lane & 8) * 4 + (lane & 4) * 4 + (lane & 32) / 4 + (lane & 16) / 4) = sum;
            });
            shares -= W * PARTS * 64;
            if (FILL != kAll && wave * P >= a.S)
                for (int q = 0; q < kPairs; ++q) gs[wave][q][lane] = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
            float of_tile = 0.f;
            each<kPairs>([&](auto q_) {
                constexpr int q = kPairs - 1 - decltype(q_)::value;
                const float4 s = du[q][lane];
                const float2 y = dys[q][lane];
                each<2>([&](auto r_) {
                    constexpr int r = 1 - decltype(r_)::value, k = (2 * q + r) * P;
                    fma_each<k % 16>(carry, C.v[k / 16], r ? y.y : y.x);
#pragma unroll
                    for (int j = 0; j < P; ++j) carry[j] *= __builtin_amdgcn_exp2f((r ? s.z : s.x) * A[j]);
                });
                of_tile += s.x + s.z;
            });
            span.add(of_tile);
        }
        block_sync();
        if constexpr (FULL) {
            float dDt_ = 0.f, db_ = 0.f;
#pragma unroll
            for (int i = 0; i < OWN; ++i) {
                const int q = wave + i * W;
                if (kPairs % W && q >= kPairs) break;
                float4 g = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < W; ++w) {
                    const float4 o = gs[w][q][lane];
                    g.x += o.x, g.y += o.y, g.z += o.z, g.w += o.w;
                }
                const float4 s = du[q][lane];
                const float2 y2 = dys[q][lane];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float gu = r ? g.z : g.x, gd = r ? g.w : g.y, y = r ? y2.y : y2.x;
                    const float dd = fmaf(xw[i][r], gu, gd * kLn2) * slope[i][r];
                    if (p.live && 2 * q + r < rows) {
                        dX.put(2 * q + r, fmaf(r ? s.z : s.x, gu, D * y));
                        dDt.put(2 * q + r, dd);
                        dDt_ = fmaf(y, xw[i][r], dDt_);
                        db_ += dd;
                    }
                }
            }
            dD += dDt_, db += db_;
            dX.move(-1), dDt.move(-1);
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
        gs[wave][0][lane] = make_float4(dD, db, 0.f, 0.f);
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
    } else leave_sums<P>(a, p, wave, carry, span.sum());
}

// dB and dC from the columns' shares: a lane to a value, the columns of a group in order.
template <typename T>
__global__ void __launch_bounds__(256) k_selective_shares(Scan a, T *dB, T *dC, int P, int W)
{
    const int part = kCells / P, parts = kRows / part, each = W * parts * 64;  // values of a tile
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < (size_t)a.B * a.G * a.tiles * each; i += (size_t)gridDim.x * 256) {
        const size_t k = i / each;
        const int v = (int)(i - k * each), m = v % kCells, w = v / 64 / parts;
        const int tile = (int)(k % a.tiles), g = (int)(k / a.tiles % a.G), b = (int)(k / a.tiles / a.G);
        const int t = tile * kRows + v / 64 % parts * part + m / P, s = w * P + m % P;
        if (t >= a.N || s >= a.S) continue;
        const int n = rows_of(a, b);
        float sum = 0.f;
        if (t < n) {
            const size_t step = (size_t)a.tiles * each;
            const float *from = a.shares + ((size_t)b * a.columns + g * a.per) * step + (size_t)tile * each + v;
            int c = 0;
            for (; c + 8 <= a.per; c += 8, from += 8 * step) {  // asked for together, added in order
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = from[k * step];
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += x[k];
            }
            for (; c < a.per; ++c, from += step) sum += *from;
        }
        store_elem(v % 64 < kCells ? dB : dC, (((size_t)b * a.N + t) * a.G + g) * a.S + s, sum);
    }
}

// dA of the rows [r0, n) of a sequence's last segment, one at a time, as far as it is a number.  The walk gives the rows that the last tile
// has room for behind them d = 0, which leaves nothing of these in the sums but where the state there or its gradient is not finite.
template <typename T>
__device__ float sum_of_rows(const Scan &a, int b, int r0, int n, int s, int c)
{
    const int g = c / a.group;
    const float A = decay_of(a.A[(size_t)c * a.S + s]), bias = a.bias ? a.bias[c] : 0.f;
    auto step = [&](size_t row) {
        float slope;
        return step_of<sizeof(T) == 4>(load_elem((const T *)a.Dt, row * a.ts + c) + bias, a.step, slope);
    };
    float carry = a.segs > 1 ? a.sums[(((size_t)b * a.segs + r0 / a.seg) * a.S + s) * a.C + c] : a.first ? a.first[((size_t)b * a.C + c) * a.S + s] : 0.f;
    float sum = 0.f;
    for (int t = n - 1; t >= r0 && sum == sum; --t) {
        const size_t row0 = (size_t)b * a.N, row = row0 + t;
        float h = a.saved[(((size_t)b * a.tiles + t / kRows) * a.S + s) * a.C + c];  // before row t, from the tile's first on
        for (size_t k = row0 + t / kRows * kRows; k < row; ++k) {
            const float d = step(k), u = d * load_elem((const T *)a.X, k * a.xs + c);
            h = fmaf(__builtin_amdgcn_exp2f(d * A), h, u * load_elem((const T *)a.Bm, k * a.bs + g * a.S + s));
        }
        const float d = step(row), C = load_elem((const T *)a.Cm, row * a.cs + g * a.S + s);
        carry = fmaf(C, load_elem((const T *)a.dY, row * a.C + c), carry) * __builtin_amdgcn_exp2f(d * A);
        sum = fmaf(carry * h, d, sum);
    }
    return sum;
}

// dA, dD and dbias from the segments' sums: 64 channels and one row of the sums a workgroup, its waves take every 16th
// segment each, eight of them asked for together.
template <typename T>
__global__ void __launch_bounds__(1024) k_selective_join(Scan a, float *dA, float *dD, float *db)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane, s = blockIdx.y;
    const int rows = s < a.S ? a.S : 2;
    const float *from = s < a.S ? a.dA + (size_t)s * a.C : a.dd + (size_t)(s - a.S) * a.C;
    if (s < a.S && !dA) return;
    float sum = 0.f;
    if (c < a.C) {
        const int count = a.B * a.segs;
        const size_t step = (size_t)rows * a.C;
        int k = wave;
        for (; k + 7 * 16 < count; k += 8 * 16) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = from[(size_t)(k + 16 * i) * step + c];
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += x[i];
        }
        for (; k < count; k += 16) sum += from[(size_t)k * step + c];
        if (sum != sum && s < a.S) {  // once more, with those that rows behind a sequence may have spoilt by themselves
            sum = 0.f;
            for (k = wave; k < count; k += 16) {
                const int b = k / a.segs, r0 = k % a.segs * a.seg, n = rows_of(a, b);
                float x = from[(size_t)k * step + c];
                if (x != x && n % kRows && n > r0 && n - r0 <= a.seg) x = sum_of_rows<T>(a, b, r0, n, s, c);
                sum += x;
            }
        }
    }
    sums[wave][lane] = sum;
    block_sync();
    if (wave || c >= a.C) return;
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) sum += sums[k][lane];
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
        A[j] = decay_of(a.A[(size_t)c * a.S + min(s, a.S - 1)]);
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
            h[j] = fmaf(__builtin_amdgcn_exp2f(d * A[j]), h[j], s < a.S ? u * Bt : 0.f);
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
// Backward, 16 waves have too few registers for four states each (128, 136 bytes of spills a lane): more than 48 states take
// 8 waves of eight.  2 x 2048 rows of 1024, 64 states, fp32: 320 us, with 16 waves 369; 16 x 1024, bf16: 955 and 1113.
Shape shape_of(int S, bool two, bool backward)
{
    if (backward && S > 48 && S <= 64) return {8, 8};
    if (S <= 8 || (S <= 16 && two)) return {2, S <= 2 ? 1 : S <= 4 ? 2 : S <= 8 ? 4 : S <= 12 ? 6 : 8};
    if (S <= 64) return {4, S <= 16 ? 4 : S <= 24 ? 6 : S <= 32 ? 8 : S <= 48 ? 12 : 16};
    return {8, S <= 96 ? 12 : 16};
}
// f(states as a constant, waves as a constant), of the shapes that the pass takes
template <bool BWD, typename F>
void by_shape(const Shape &s, F f)
{
    auto with = [&](auto P, auto W) {
        if (s.P == decltype(P)::value && s.W == decltype(W)::value) f(P, W);
    };
    auto two = std::integral_constant<int, 2>();
    auto four = std::integral_constant<int, 4>();
    auto eight = std::integral_constant<int, 8>();
    with(two, std::integral_constant<int, 1>());
    with(two, two);
    with(two, four);
    if constexpr (BWD) with(eight, eight);
    else {
        with(two, std::integral_constant<int, 6>());
        with(four, std::integral_constant<int, 16>());
    }
    with(two, eight);
    with(four, four);
    with(four, std::integral_constant<int, 6>());
    with(four, eight);
    with(four, std::integral_constant<int, 12>());
    with(eight, std::integral_constant<int, 12>());
    with(eight, std::integral_constant<int, 16>());
}

// f(how S states fill W waves of P as a constant)
template <int P, int W, typename F>
void by_fill(int S, F f)
{
    if (S == P * W) f(std::integral_constant<Fill, kAll>());
    else if (S % P) f(std::integral_constant<Fill, kPlaces>());
    else if constexpr (W > 2) f(std::integral_constant<Fill, kWaves>());  // (one wave or two hold a state each: shape_of)
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
    for (size_t n : {a.xs, a.ts, a.bs, a.cs, vec, (size_t)a.C})
        if (n >= 1 << 24) return LA_ERR_SHAPE;  // a tile's rows in 32 bits
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
// How a call is laid out: the states of a wave, and the segments that sequences are cut into, whose start states two more launches
// find (what every segment makes of zero states, an exponential and three operations for every row and state once more, and
// the walk along the segments).  512 rows take, in us, with w waves on every SIMD of the busiest compute units (S = 16, bf16):
// 39 + 29 w forward (31 + 35 w with two states a wave), 100 + 80 w backward (5 + 117 w), what the segments make of zero states 28 + 23 w and 31 + 21 w.  Segments fill the
// compute units once forward, about twice backward (5 waves to a SIMD at once, backward 2 to 4), and have 32 rows at least; one
// piece where that takes less.  Of 1 to 96 segments, on 10 shapes of 1 to 256 chains, this takes 1.04 times the best on the average.  The
// constants are those of 16 states; of 1 to 128 segments, on 5 shapes of 8 to 512 chains, other numbers of states take, forward and backward, 1.11
// and 1.14 times the best with 4 (at most 1.4: one sequence of 8192 rows), 1.02 and 1.07 with 8, 1.07 and 1.02 with 24, 1.02 and 1.01 with 32,
// 1.00 and 1.01 at most with 64, 100 and 128.
// One piece and few waves: two states a wave instead of four, whose twice as many waves hide each other's
// waits (8 x 2048 rows of 2048 channels 222 us forward, with four 260, in 8 segments 240; backward 484, in 3 segments
// 546; with 12 states backward 543 and 529: only from 13 on).
Shape lay_out(Scan &a, bool backward)
{
    a.group = a.C / a.G;
    a.per = (a.group + 63) / 64;
    a.columns = a.G * a.per;
    a.tiles = (a.N + kRows - 1) / kRows;
    const Shape s = shape_of(a.S, false, backward);
    const double chains = (double)a.B * a.columns, waves = chains * s.W / 1024.0, rows = a.N / 512.0;
    const int slots = 256 * ((!backward ? 20 : s.W == 16 ? 16 : s.W == 8 ? 8 : 12) / s.W);  // workgroups at once
    const int rounds = (int)((!backward ? 1536.0 : s.W == 8 ? 1024.0 : 1792.0) * 4 / s.W / slots + 0.4);
    const double most = (rounds ? rounds : 1) * (double)slots / chains;
    int segs = (int)(most < 256.0 ? most : 256.0);
    if (segs > a.N / 32) segs = a.N / 32;
    const double busiest = (double)(int)((chains + 255) / 256) * s.W / 4.0;
    const double fours = backward ? 100 + 80 * busiest : 39 + 29 * busiest, twos = backward ? 5 + 117 * busiest : 31 + 35 * busiest;
    const bool two = a.S <= 16 && (a.S > 12 || !backward) && twos < fours;
    const double whole = rows * (two ? twos : fours);
    const double cut = 8.0 + rows * (backward ? 101 * waves + 131.0 / segs : 52 * waves + 67.0 / segs);
    if (segs < 2 || whole <= cut) segs = 1;
    const int of = (a.tiles + segs - 1) / segs;
    a.seg = of * kRows;
    a.segs = (a.tiles + of - 1) / of;
    return shape_of(a.S, two && a.segs == 1, backward);
}
Scan scan_of(const void *X, size_t xs, const void *Dt, size_t ts, const float *A, const void *Bm, size_t bs, const void *Cm, size_t cs,
             const float *D, const float *bias, int B, int N, int C, int S, int G, la_step step)
{
    Scan a{};
    a.X = X, a.xs = xs, a.Dt = Dt, a.ts = ts, a.A = A, a.Bm = Bm, a.bs = bs, a.Cm = Cm, a.cs = cs, a.D = D, a.bias = bias;
    a.B = B, a.N = N, a.C = C, a.S = S, a.G = G, a.step = step;
    return a;
}

// Floats of a tile's shares of dB and dC.
size_t shares_of(const Shape &s) { return (size_t)s.W * (kRows * s.P / kCells) * 64; }

// What a call keeps in its workspace, in floats.
struct Room {
    size_t shares, dA, dd, sums, spans, bytes;
    Room(const Scan &a, const Shape &shape, bool back)
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
        shares = take(back ? (size_t)a.B * a.columns * a.tiles * shares_of(shape) : 0);
        dA = take(back ? segs * a.S * a.C : 0);
        dd = take(back ? segs * 2 * a.C : 0);
        bytes = at * 4;
    }
};

// Workgroups of 256 for n values, which walk the values where a grid would be too large.
dim3 blocks_of(size_t n)
{
    const size_t k = (n + 255) / 256;
    return dim3((unsigned)(k < 1 << 20 ? k : 1 << 20));
}
la_status done() { return hipGetLastError() == hipSuccess ? LA_OK : LA_ERR_LAUNCH; }

}  // namespace
}  // namespace la

extern "C" {

size_t la_selective_workspace_bytes(int B, int N, int C, int S, int G, int is_backward)
{
    if (la::check_shape(B, N, C, S, G) != LA_OK) return 0;
    la::Scan a{};
    a.B = B, a.N = N, a.C = C, a.S = S, a.G = G;
    const la::Shape shape = la::lay_out(a, is_backward != 0);
    return la::Room(a, shape, is_backward != 0).bytes;
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
    const la::Shape shape = la::lay_out(a, false);
    const la::Room room(a, shape, false);
    const size_t kept = la_selective_saved_bytes(B, N, C, S);
    if (room.bytes && (!workspace || workspace_bytes < room.bytes || !la::aligned_to(workspace, 256))) return LA_ERR_WORKSPACE;
    if (saved && (saved_bytes < kept || !la::aligned_to(saved, 256))) return LA_ERR_WORKSPACE;
    const la::Inputs in(a, dt);
    const la::Range outs[] = {{Y, (size_t)B * N * C * la::size_of(dt)}, {last, (size_t)B * C * S * 4}, {saved, kept}, {workspace, room.bytes}};
    if (la::any_alias(in.r, 9, outs, 4)) return LA_ERR_ALIAS;
    if (hipPeekAtLastError() != hipSuccess) return LA_ERR_LAUNCH;
    a.sums = (float *)workspace + room.sums, a.spans = (float *)workspace + room.spans;
    const dim3 grid((unsigned)((size_t)B * a.columns * a.segs)), chain((unsigned)(((size_t)B * C * S + 255) / 256));
    const hipStream_t st = (hipStream_t)hip_stream;
    auto run = [&](auto *t, auto P, auto W) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int p = decltype(P)::value, w = decltype(W)::value;
        if constexpr (p > 2 || w <= 4) {  // (else two states a wave of one piece: lay_out)
            if (a.segs > 1) {
                la::k_selective<T, p, w, false, la::kAll><<<grid, dim3(64 * w), 0, st>>>(a);
                la::k_selective_chain<false><<<chain, dim3(256), 0, st>>>(a);
            }
        }
        la::by_fill<p, w>(S, [&](auto F) { la::k_selective<T, p, w, true, decltype(F)::value><<<grid, dim3(64 * w), 0, st>>>(a); });
    };
    la::by_shape<false>(shape, [&](auto P, auto W) {
        if (dt == LA_F32) run((float *)nullptr, P, W);
        else run((la::bf16_t *)nullptr, P, W);
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
    const la::Shape shape = la::lay_out(a, true);
    const la::Room room(a, shape, true);
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
    const dim3 grid((unsigned)((size_t)B * a.columns * a.segs)), chain((unsigned)(((size_t)B * C * S + 255) / 256));
    const hipStream_t st = (hipStream_t)hip_stream;
    auto run = [&](auto *t, auto P, auto W) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int p = decltype(P)::value, w = decltype(W)::value;
        if constexpr (p > 2 || w <= 4) {
            if (a.segs > 1) {
                la::k_selective_back<T, p, w, false, la::kAll><<<grid, dim3(64 * w), 0, st>>>(a);
                la::k_selective_chain<true><<<chain, dim3(256), 0, st>>>(a);
            }
        }
        la::by_fill<p, w>(S, [&](auto F) { la::k_selective_back<T, p, w, true, decltype(F)::value><<<grid, dim3(64 * w), 0, st>>>(a); });
    };
    la::by_shape<true>(shape, [&](auto P, auto W) {
        if (dt == LA_F32) run((float *)nullptr, P, W);
        else run((la::bf16_t *)nullptr, P, W);
    });
    const dim3 all = la::blocks_of((size_t)B * G * a.tiles * la::shares_of(shape));
    if (dt == LA_F32) la::k_selective_shares<float><<<all, dim3(256), 0, st>>>(a, (float *)dBm, (float *)dCm, shape.P, shape.W);
    else la::k_selective_shares<la::bf16_t><<<all, dim3(256), 0, st>>>(a, (la::bf16_t *)dBm, (la::bf16_t *)dCm, shape.P, shape.W);
    const dim3 joined((C + 63) / 64, S + 2);
    if (!dA && !dD && !dbias) return la::done();
    if (dt == LA_F32) la::k_selective_join<float><<<joined, dim3(1024), 0, st>>>(a, dA, dD, dbias);
    else la::k_selective_join<la::bf16_t><<<joined, dim3(1024), 0, st>>>(a, dA, dD, dbias);
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
