/*
 * la.h -- C ABI of the MI355X (gfx950) linear-attention library.
 *
 * The attention comes first; the operators around it (gated recurrences, rows in 8 bits, the norm with
 * the residual's addition) have their own conventions about shapes and alignment at the end, and
 * share the rest with it: caller-owned buffers, streams, errors, no written buffer over another.
 *
 * Linear attention with kernel f(x) = a + b*x (Sec. 2.2): for every (batch,
 * head) slice with rows q_i, k_i, v_i in R^D, i = 0..N-1,
 *
 *     w_in = a + b * (q_i . k_n)
 *     g_i  = sum_{n in A(i)} w_in
 *     o_i  = sum_{n in A(i)} w_in * v_n / g_i
 *
 * where A(i) = {0..i} with the causal mask and {0..N-1} without it.  The
 * library evaluates this in O(N D^2) time and O(N D) memory through the
 * running sums of Sec. 3.1 (forward, Eq. fglast / xy) and Sec. 3.2 (backward,
 * Eq. back1 / back2 / endd), carried chunk by chunk.
 *
 * Conventions common to every entry point
 *   - All tensor arguments are DEVICE pointers to dense row-major arrays
 *     [B, H, N, D] with D contiguous (the paper's [B*H, N, D] storage, Sec. 4);
 *     G is [B, H, N] float32.  Every pointer must be 16-byte aligned.
 *   - `dt` is the element type of Q, K, V, O, dO, dQ, dK, dV: LA_F32 (float) or
 *     LA_BF16 (bfloat16 bit patterns, round-to-nearest-even on store).  All
 *     accumulation is float32; G is always float32.
 *   - The caller owns every buffer, including the workspace.  The library
 *     allocates no memory and keeps no state between calls (the one exception
 *     is the test hook la_debug_override below); calls on different buffers
 *     may run concurrently.  Calls that share a workspace must not overlap in
 *     time.
 *   - Work is enqueued on `hip_stream` (a hipStream_t passed as void*; NULL is
 *     the default stream).  The call returns without synchronising.
 *   - Outputs are overwritten, never accumulated into.  No written buffer
 *     (outputs, workspace, hand-over buffer) may overlap any other buffer of
 *     the call: this is checked and reported as LA_ERR_ALIAS.
 *   - Supported: D in {16, 32, 64, 128, 256}; B, H, N >= 1 with B*H*N*D < 2^40;
 *     any N (a ragged last chunk is handled).
 *   - Errors are reported by return code only.  Every argument check happens
 *     before anything is enqueued, so a failed call has no side effect.
 *     LA_ERR_LAUNCH carries a failed kernel enqueue (hipGetLastError).  A HIP
 *     error already pending on the calling thread when the call is made is
 *     also reported as LA_ERR_LAUNCH; it is left pending and nothing is
 *     enqueued.
 *   - Numerical precondition (not checked): g_i != 0.  It holds when
 *     a > |b| * max|q.k|, e.g. unit-norm rows of Q and K (the normalisation of
 *     Sec. 3.3, which is the caller's job) with a = 1, b = 0.5.
 *   - Range of float32 tensors: an element is carried exactly for
 *     magnitudes from 2^-109 (1.5e-33) to the largest float; below, it keeps
 *     an absolute error of up to 2^-134 (so 10 bits are left at 2^-124).
 *     An infinity or a NaN in V or dO spoils its column of O and dV from the
 *     row's aligned block of 32 rows on (for dV: up to it), earlier rows of
 *     that block included; in fp32 an infinity in V is an infinity in the rows
 *     of its block that see it where all their weights are of one sign.
 */
#ifndef LA_H_
#define LA_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LA_API __attribute__((visibility("default")))

typedef enum la_status {
    LA_OK = 0,
    LA_ERR_NULL = 1,        /* a required pointer is NULL                      */
    LA_ERR_SHAPE = 2,       /* B, H, N or D out of range                       */
    LA_ERR_UNSUPPORTED = 3, /* D or dtype not supported                        */
    LA_ERR_ALIGN = 4,       /* a pointer is not 16-byte aligned                */
    LA_ERR_WORKSPACE = 5,   /* workspace NULL or smaller than required         */
    LA_ERR_LAUNCH = 6,      /* a kernel enqueue failed                         */
    LA_ERR_ALIAS = 7        /* an output overlaps another buffer of the call   */
} la_status;

typedef enum la_dtype {
    LA_F32 = 0,
    LA_BF16 = 1,
    LA_E4M3 = 2,  /* 8-bit rows (la_pack_rows); no type of the attention's tensors */
    LA_I8 = 3     /* the same with integers                                        */
} la_dtype;

struct la_trace; /* per-kernel timing hook, defined further down */

/* Library version: major*10000 + minor*100 + patch. */
LA_API int la_version(void);

/* Static, human-readable name of a status code. */
LA_API const char *la_status_string(la_status s);

/*
 * Bytes of device workspace la_forward (is_backward = 0) or la_backward
 * (is_backward = 1; is_backward = 2: la_backward called with O or G NULL, which
 * recomputes them; is_backward = 3: la_backward_ab) needs for this problem.  Returns 0 for invalid or
 * unsupported arguments.  The workspace holds the per-segment running-sum
 * states (S = sum k v^T, z = sum k, p = sum v of Eq. xy; and the reverse sums
 * of Eq. endd for the backward pass) that let segments of one sequence run in
 * parallel; its size is O(B*H*(N/segment)*D^2 + B*H*N).  D = 256 runs on
 * blocks of 128 columns; with bf16 tensors the shares that one launch hands to the next stay
 * in float32 in the workspace: 1024 more bytes per token-head for la_forward, 3072 for
 * la_backward.
 *
 * The sizes do not grow steadily with N: a sequence is cut into the number of segments that
 * costs least, and a longer one may be cut into fewer (bf16, D = 32, 156 slices: 8.8 MB at
 * N = 773, 2.7 MB at 1165).  A caller that keeps one buffer for several lengths takes the
 * largest of their sizes, or, for every length up to N, this bound (in bytes, plus 1024):
 *     la_forward   4 M E (E + 2)       + at D = 256 B*H*N * 4, in bf16 * 1028
 *     la_backward  4 M E (2 E + 4)     + B*H*N * 4, at D = 256 B*H*(N + 1) * 8, in bf16 * 3080
 *     hand-over    4 M E (E + 2)       + at D = 256 B*H * 1024      (la_saved_state_bytes)
 * with E = 32, 32, 64, 128, 128 and M = max(B*H, 3072), max(B*H, 3072), max(B*H, 1536),
 * max(B*H, 768), 4 max(B*H, 128) at D = 16, 32, 64, 128, 256.
 */
LA_API size_t la_workspace_bytes(int B, int H, int N, int D, la_dtype dt, int causal,
                          int is_backward);

/*
 * Forward pass (Sec. 3.1: Eq. div, fglast, xy).
 *   in : Q, K, V   [B,H,N,D] of `dt`
 *   out: O         [B,H,N,D] of `dt`      o_i = f_i / g_i
 *        G         [B,H,N]   float32      g_i, the denominators; part of the
 *                                         set {Q,K,V,O,g} kept for the
 *                                         backward pass (Sec. 3.2).  May be
 *                                         NULL: g is then not stored, and
 *                                         la_backward must recompute it.
 *   a, b   : kernel coefficients; causal != 0 applies the causal mask.
 *   workspace / workspace_bytes: device scratch of at least
 *            la_workspace_bytes(..., 0) bytes, 256-byte aligned.
 */
LA_API la_status la_forward(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Backward pass (Sec. 3.2: Eq. bound, back1, back2, endd).
 *   in : Q, K, V, O, dO [B,H,N,D] of `dt`; G [B,H,N] float32 -- O and G exactly
 *        as written by la_forward for the same Q, K, V, a, b, causal.
 *        O and/or G may be NULL (a caller that keeps only {Q,K,V} of the saved
 *        set of Sec. 3.2): the forward pass is then run again inside the call,
 *        into the workspace, and whichever of the two was NULL takes its
 *        result.  That costs one forward pass and O(B*H*N*D) workspace.
 *   out: dQ, dK, dV     [B,H,N,D] of `dt`: gradients of sum(O * dO).
 *   workspace: 256-byte aligned; at least la_workspace_bytes(..., 1) bytes, or
 *        la_workspace_bytes(..., 2) bytes when O or G is NULL.
 */
LA_API la_status la_backward(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO,
                      void *dQ, void *dK, void *dV,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Forward and backward pass with the row normalisation of Sec. 3.3 inside the call: Q and K
 * are the raw rows, every kernel scales them to unit length (qhat = q / ||q||, khat = k /
 * ||k||) as it stages them, so that no normalised copy of Q and K is ever written or read
 * back, and la_backward_qknorm returns the gradients for the raw rows,
 *     dq = (dqhat - qhat (qhat . dqhat)) / ||q||   (likewise dk):
 * the kernels pass their dqhat, dkhat through that map before they store them.
 * Arguments, workspace sizes (la_workspace_bytes with is_backward 0 / 1, or 2 when O or G is
 * NULL) and error behaviour as for la_forward_traced / la_backward_traced; O and G are those
 * of la_forward_qknorm.  A row of zeros stays a row of zeros (and makes g_i = a n_i for it).
 * With bfloat16 tensors the rows stay as they are on chip and the factors 1/||q||, 1/||k|| go
 * to quantities that are float32 anyway, so that the normalised rows are not rounded to
 * bfloat16 again (about 1.8 times the time of the plain bfloat16 calls at D = 128).
 * The squared length of a row has to be a float: lengths from 1e-19 (fewer digits down to 1e-22) to
 * 1.8e19.
 */
LA_API la_status la_forward_qknorm(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream,
                     struct la_trace *trace);

LA_API la_status la_backward_qknorm(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO,
                      void *dQ, void *dK, void *dV,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes, void *hip_stream,
                      struct la_trace *trace);

/*
 * The same pair with the hand-over of la_forward_save / la_backward_saved: the running
 * sums of the normalised rows at the segment boundaries go from the forward call to the
 * backward call through `saved` (la_saved_state_bytes bytes, 256-byte aligned; NULL where
 * that size is 0), which then skips their recomputation.  What a training step with the
 * normalisation of Sec. 3.3 runs.
 */
LA_API la_status la_forward_qknorm_save(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt,
                     void *workspace, size_t workspace_bytes,
                     void *saved, size_t saved_bytes, void *hip_stream,
                     struct la_trace *trace);

LA_API la_status la_backward_qknorm_saved(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO,
                      void *dQ, void *dK, void *dV,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes,
                      const void *saved, size_t saved_bytes, void *hip_stream,
                      struct la_trace *trace);

/*
 * Gradients of sum(O * dO) with respect to the kernel's own coefficients, which
 * Sec. 2.2 allows to be learnable.  With dL/dw_in = OmegaHat_i . v_n - delta_i
 * (Eq. bound divided by b; OmegaHat = dO / g, delta_i = o_i . OmegaHat_i) and
 * w_in = a + b q_i . k_n:
 *     dL/db = sum_{i, n in A(i)} dL/dw_in (q_i . k_n) = sum_i q_i . dq_i / b,
 *     dL/da = sum_{i, n in A(i)} dL/dw_in             = -(b / a) dL/db
 * (O depends on a and b through their ratio only).  The call runs the ascending
 * sweep of the backward pass (Eq. back1) once with unit b and reduces q . dq over
 * all elements in a fixed order, so b = 0 is allowed; a = 0 is LA_ERR_UNSUPPORTED.
 *   in : Q, K, V, O, dO, G as for la_backward (O, G required).
 *   out: dab: device pointer to two floats, 8-byte aligned: dab[0] = dL/da,
 *        dab[1] = dL/db, summed over every batch, head and row.
 *   workspace: at least la_workspace_bytes(..., 3) bytes, 256-byte aligned.
 */
LA_API la_status la_backward_ab(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO, float *dab,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Incremental (decode) form: the recurrence of App. B.1 (Table 3, row 2: S_t =
 * S_{t-1} + k_t v_t^T, z_t = z_{t-1} + k_t) for the kernel a + b x, i.e. Eq. xy /
 * fglast with the running sums carried across calls instead of across chunks.
 *
 *   state: device memory, caller-owned, float32, la_decode_state_bytes(B, H, D)
 *       bytes, 256-byte aligned; per (batch, head) slice [S (D*D, row r column j =
 *       sum k_r v_j) | z (D) | p (D) | count (1)], padded to a multiple of 64
 *       floats.  All zeros stands for an empty prefix (the caller clears it).
 *   la_decode_step: appends T >= 1 rows per slice -- q, k, v, o are [B,H,T,D] of
 *       `dt`, g is [B,H,T] float32 or NULL -- each row is added to the sums and
 *       then read out (a row attends to the prefix and to itself), and the state
 *       is updated in place.  D in {16, 32, 64, 128, 256}.  Calls that share a
 *       state must not overlap in time.
 *   la_decode_prefill: sets (accumulate = 0) or adds to (accumulate != 0) the
 *       state the sums over the N rows of K, V [B,H,N,D] in one parallel pass:
 *       the state after a prompt that was run through la_forward.  workspace as
 *       for la_forward without the mask: la_workspace_bytes(B,H,N,D,dt,0,0).
 * Error behaviour as for la_forward; a missing, misaligned or short state is
 * LA_ERR_WORKSPACE.
 */
LA_API size_t la_decode_state_bytes(int B, int H, int D);

LA_API la_status la_decode_step(const void *q, const void *k, const void *v,
                     void *o, float *g, float *state, size_t state_bytes,
                     int B, int H, int T, int D,
                     float a, float b, la_dtype dt, void *hip_stream);

LA_API la_status la_decode_prefill(const void *K, const void *V,
                     float *state, size_t state_bytes,
                     int B, int H, int N, int D, la_dtype dt, int accumulate,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * la_forward for callers that cannot allocate or pass a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same computation as la_forward, with the workspace in a static
 * device array inside the library (LA_STATIC_SCRATCH_BYTES per GPU, held until
 * the process ends).  The call allocates nothing and frees nothing.  Where
 * la_workspace_bytes(..., 0) fits LA_STATIC_SCRATCH_BYTES (the five benchmark
 * configurations do) the results are la_forward's, bit for bit.  Where it does
 * not, the call cuts the sequences into fewer, longer segments, at D = 256 works
 * on one block of columns after another, and at D = 16 takes kernels with a
 * quarter of the workspace (up to 26214 slices): the results then differ from
 * la_forward's by the order of the sums.  What does not fit even so is rejected
 * with LA_ERR_WORKSPACE (nothing enqueued).  All calls on one GPU share the array:
 * calls that overlap in time on one GPU (different streams, different threads) race,
 * and the caller must order them.  The first call on each GPU resolves the
 * array's device address (make it outside graph capture); if that fails the
 * call returns LA_ERR_LAUNCH.
 */
#define LA_STATIC_SCRATCH_BYTES (32u << 20)
LA_API la_status la_forward_static(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt, void *hip_stream);

/*
 * Test and profiling hook -- the only process-wide state of the library.
 * seg_len > 0 forces the number of rows per segment (rounded up to a multiple
 * of 64; 0 restores the automatic choice); force_generic != 0 routes every
 * head size to the plain-ALU kernels.  Both change la_workspace_bytes and
 * la_saved_state_bytes and the private layout of those buffers, so a size
 * query and the calls that use its result must see the same setting; a buffer
 * filled by la_forward_save under one setting must not be given to
 * la_backward_saved under another.  Not synchronised with calls in flight on
 * other threads.  Production callers never call it.
 */
LA_API void la_debug_override(int seg_len, int force_generic);

/*
 * Optional hand-over of the forward pass's running sums to the backward pass.
 *
 * The ascending sweep of the backward pass (dQ, Eq. back1) starts every segment
 * from the same sums S = sum k v^T, z = sum k (Eq. xy) that the forward pass
 * carries through the sequence.  la_backward recomputes them from K and V;
 * a caller that runs the two passes as a pair (a training step) can let
 * la_forward_save write them out at the segment boundaries and hand them to
 * la_backward_saved, which then skips that recomputation.  This is an
 * addition to the set {Q,K,V,O,g} that Sec. 3.2 keeps: O(B*H*(N/segment)*D^2)
 * floats, small next to the tensors where these are large (8 to 17 MB at D = 64
 * and 128 where the segments just fill the GPU, up to three times that where three
 * rounds of them do; 34 MB at D = 256), but larger than
 * a tensor where sequences are short.
 *
 *   la_saved_state_bytes: size of the `saved` buffer for this problem (it does not grow
 *       steadily with N either: see la_workspace_bytes; 0 for
 *       invalid arguments, and 0 when the library would not use one -- D = 16,
 *       and D = 256 where it would exceed both 96 MB and one tensor's bytes;
 *       a zero-size buffer may be NULL).
 *   la_forward_save:   la_forward, and additionally fills `saved` (device
 *       memory, 256-byte aligned, at least la_saved_state_bytes bytes).
 *   la_backward_saved: la_backward, reading `saved` as written by
 *       la_forward_save for the same Q, K, V, B, H, N, D, dt, a, b, causal.
 *       Results agree with la_backward up to fp32 rounding order.
 * `saved` is caller-owned like every other buffer; its layout is private to
 * the library and to this library version.  `trace` is the timing hook
 * described below and may be NULL.  Error behaviour as for la_forward /
 * la_backward; a missing, misaligned or short `saved` is LA_ERR_WORKSPACE, except
 * at D = 256, where the hand-over is optional: such a buffer, or one that overlaps
 * another buffer of the call, is left unused by both calls (callers that pass NULL
 * there need not change), and la_backward_saved finds out whether the sums in the
 * one it is given are those of its inputs (by the last row of every slice of O,
 * which la_forward_save leaves in the buffer); where they are not, it forms its own.
 */
LA_API size_t la_saved_state_bytes(int B, int H, int N, int D, la_dtype dt, int causal);

LA_API la_status la_forward_save(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt,
                     void *workspace, size_t workspace_bytes,
                     void *saved, size_t saved_bytes,
                     void *hip_stream, struct la_trace *trace);

LA_API la_status la_backward_saved(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO,
                      void *dQ, void *dK, void *dV,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes,
                      const void *saved, size_t saved_bytes,
                      void *hip_stream, struct la_trace *trace);

/*
 * Per-kernel timing hook for benchmarks and profiles.  The caller creates
 * `capacity` hipEvent_t handles (timing enabled) and passes them in `events`;
 * the traced entry points record events[0] on the stream before their first
 * kernel and events[k] right after their k-th kernel, and fill `names[k-1]`
 * with a static string naming that kernel.  `recorded` receives the number of
 * events recorded (kernels + 1); if `capacity` is too small only the first
 * `capacity` events are recorded.  No call has more than LA_MAX_TRACE entries: at
 * D = 256 the forward pass that la_backward runs again (O or G NULL) is one entry, and
 * so are the two kernels that form the sums of slices whose hand-over does not hold.
 * The caller synchronises and reads the
 * intervals with hipEventElapsedTime.  The library never waits on the events.
 */
#define LA_MAX_TRACE 8
typedef struct la_trace {
    void **events;                    /* in : caller-owned hipEvent_t handles     */
    int capacity;                     /* in : number of handles in `events`       */
    int recorded;                     /* out: number of events recorded           */
    const char *names[LA_MAX_TRACE];  /* out: names[k] = kernel between events k, k+1 */
} la_trace;

/* la_forward / la_backward with the timing hook; `trace` may be NULL, which
 * makes them identical to the plain entry points. */
LA_API la_status la_forward_traced(const void *Q, const void *K, const void *V,
                     void *O, float *G,
                     int B, int H, int N, int D,
                     float a, float b, int causal, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream,
                     la_trace *trace);

LA_API la_status la_backward_traced(const void *Q, const void *K, const void *V,
                      const void *O, const float *G, const void *dO,
                      void *dQ, void *dK, void *dV,
                      int B, int H, int N, int D,
                      float a, float b, int causal, la_dtype dt,
                      void *workspace, size_t workspace_bytes, void *hip_stream,
                      la_trace *trace);

/*
 * Gated linear recurrence: the recurrence of App. B.1 with a gate per row and channel, on a vector state (not
 * the matrix states of the gated rows of Table 3).  For each of B sequences of N rows with C channels
 *
 *     h_t = f_t h_{t-1} + u_t          (element-wise, t = 0 .. N-1, h_{-1} = h0)
 *     LA_GATE_VALUE:    f_t = g_t,             u_t = x_t
 *     LA_GATE_SIGMOID:  f_t = 1/(1+exp(-g_t)), u_t = (1 - f_t) x_t
 *
 * and backward, d_t being the gradient that reaches h_t from its own output and from all later rows,
 *
 *     d_t = dh_t + f_{t+1} d_{t+1}  (d_{N-1} = dh_{N-1} + dlast),   dh0 = f_0 d_0
 *     LA_GATE_VALUE:    dx_t = d_t,            dg_t = d_t h_{t-1}
 *     LA_GATE_SIGMOID:  dx_t = (1 - f_t) d_t,  dg_t = d_t (h_{t-1} - x_t) f_t (1 - f_t)
 *
 * The sequence is cut into segments that run in parallel, as in the attention's passes: what a segment
 * does to a state is the product of its gates and its own sum.  States and sums are float32; h is
 * stored in the tensors' type, and the backward pass goes by the stored h.
 *
 *   X, Gate, Hs, dHs, dX, dGate: [B, N, C] of `dt`, dense, C contiguous.  A head layout [B, H, N, D]
 *       is B*H sequences of D channels.  Addresses are those of elements: no further alignment.
 *   h0, last, dlast, dh0: [B, C] float32.  h0 NULL: zeros; last (the state after the last row) NULL:
 *       not wanted; dlast NULL: zeros; dh0 NULL: not wanted.
 *   lengths: NULL, or B ints on the device.  Rows from lengths[b] on are padding: they are not read,
 *       every output is zero there, and `last` is the state before them (a length of 0 or less leaves
 *       h0, one of N or more is N).
 *   workspace: at least la_recurrence_workspace_bytes(..., is_backward) bytes, 256-byte aligned; NULL
 *       where that is 0.  Nothing in it has to start at zero.
 * A gate of zero (LA_GATE_SIGMOID: -infinity) starts anew: packed documents need no lengths.  The product
 * of a run of gates has to be a float (gates of magnitude up to 1 are); an infinity or a NaN spoils its
 * channel from its row on (backward: up to it), whatever the gates after it.
 * Calls that share a workspace must not overlap in time, two captured graphs' neither: workgroups of one
 * call wait for words that others of it leave there.  Results of calls that overlap all the same are undefined: wrong
 * finite values, rows left unwritten or NaN, with LA_OK; the waits are bounded only so that the kernels end.
 * Limits: B, N, C >= 1, N <= 2^30, B*N*C < 2^40, B * ceil(C / 64) < 2^23 and, times ceil(N / 64), < 2^31.
 *
 * la_recurrence_step appends T rows to a carried state, [B, C] float32, and updates it in place: the
 * form for single tokens.  No workspace; rows are walked one after another, T is meant to be small.
 * Calls that share a state must not overlap in time.
 * Error behaviour as for la_forward; an unknown gate is LA_ERR_UNSUPPORTED.
 */
typedef enum la_gate {
    LA_GATE_VALUE = 0,
    LA_GATE_SIGMOID = 1
} la_gate;

LA_API size_t la_recurrence_workspace_bytes(int B, int N, int C, la_dtype dt, int is_backward);

LA_API la_status la_recurrence_forward(const void *X, const void *Gate, const float *h0,
                     void *Hs, float *last, const int *lengths,
                     int B, int N, int C, la_gate gate, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

LA_API la_status la_recurrence_backward(const void *X, const void *Gate, const float *h0,
                      const void *Hs, const void *dHs, const float *dlast,
                      void *dX, void *dGate, float *dh0, const int *lengths,
                      int B, int N, int C, la_gate gate, la_dtype dt,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

LA_API la_status la_recurrence_step(const void *X, const void *Gate, void *Hs, float *state,
                     int B, int T, int C, la_gate gate, la_dtype dt, void *hip_stream);

/*
 * Rows in 8 bits: groups of 32 neighbours of a row (the last group of a row may be shorter) share a
 * power of two, kept as one byte e that stands for 2^(e - 127): the block format of the OCP
 * microscaling (MX) specification, which the matrix cores of gfx950 read as it stands.
 *     LA_E4M3: codes are OCP e4m3 numbers;        the least power with  max |x| <= 448    2^(e - 127)
 *     LA_I8:   codes are integers, 64ths of the power; the least with  max |x| <= 127/64 2^(e - 127)
 * Elements are rounded to nearest, ties to even; e is held to 0 .. 254.  Every finite value that the
 * codes stand for is a bfloat16 number, so that unpacking rounds nothing (below 2^-126 it may; with
 * LA_E4M3 magnitudes from 1.9375 2^127 on round to 2^128 and come back as infinities).  A group with
 * an infinity or a NaN gets e = 255 and comes back as NaN.
 *
 *   la_pack_rows:   X [rows, C] of `dt` (LA_F32 / LA_BF16) -> codes [rows, C], scales
 *                   [rows, ceil(C / 32)] bytes
 *   la_pack_tensors: the same for `count` tensors of one shape (1 to 4), whose addresses are read
 *                   before the call returns.
 *   la_unpack_rows: the way back.
 * One byte and 1/32 an element instead of two or four: what a backward pass keeps of a forward pass
 * where memory is short (la_rmsnorm_backward reads the codes themselves).
 * Addresses are those of elements.  Limits: rows, C >= 1, rows * C < 2^40.
 */
LA_API la_status la_pack_rows(const void *X, void *codes, void *scales, size_t rows, int C,
                     la_dtype dt, la_dtype code, void *hip_stream);

LA_API la_status la_pack_tensors(int count, const void *const *X, void *const *codes, void *const *scales,
                     size_t rows, int C, la_dtype dt, la_dtype code, void *hip_stream);

LA_API la_status la_unpack_rows(const void *codes, const void *scales, void *X, size_t rows, int C,
                     la_dtype code, la_dtype dt, void *hip_stream);

/*
 * Root-mean-square norm of rows, with the residual's addition in front of it:
 *
 *     s = x + r (rounded to `dt`, as it is stored),  rstd = 1 / sqrt(mean(s^2) + eps),
 *     y = w s rstd
 * and backward, with n = s rstd and the gradients dy of y and ds of s (where s has other readers, as
 * a residual stream has)
 *     dx = dr = rstd (w dy - n mean(w dy n)) + ds,   dw = sum over the rows of dy n.
 *
 *   X, R, S, dY, dS, dX: [rows, C] of `dt` (LA_F32 / LA_BF16); W: [C] of `wt`, LA_F32 or `dt`.
 *   R NULL: no residual, s is x; S must then be NULL too.  S may be R itself (updated in place).
 *   W NULL: ones.  dS NULL: zeros.  dW: [C] float32, or NULL where it is not wanted (or W is NULL).
 *   Y: [rows, C] of `yt`: `dt`, or LA_E4M3 / LA_I8, the codes of la_pack_rows with Yscale for their
 *       powers (NULL otherwise): what a matrix product on 8-bit operands takes.
 *   Kept, Kscale: NULL, or s in 8 bits of type `kt` for the backward pass, in the same pass over the rows.
 *   rstd: [rows] float32, or NULL where no backward pass follows.
 *   la_rmsnorm_backward: `st` is the type of S: `dt`, with Sscale NULL, or LA_E4M3 / LA_I8 (Kept,
 *       Kscale of the forward call), whose values then stand for s.
 *   workspace (only where dW is wanted): at least la_rmsnorm_workspace_bytes(rows, C) bytes, 256-byte
 *       aligned.
 * Sums are float32, those of dW in a fixed order.  The mean square of a row has to be a float.
 * Addresses are those of elements.  Limits: rows >= 1, 1 <= C <= 16384, rows * C < 2^40.
 */
LA_API size_t la_rmsnorm_workspace_bytes(size_t rows, int C);

LA_API la_status la_rmsnorm_forward(const void *X, const void *R, const void *W,
                     void *Y, void *Yscale, void *S, void *Kept, void *Kscale, float *rstd,
                     size_t rows, int C, float eps,
                     la_dtype dt, la_dtype wt, la_dtype yt, la_dtype kt, void *hip_stream);

LA_API la_status la_rmsnorm_backward(const void *S, const void *Sscale, const void *W, const float *rstd,
                      const void *dY, const void *dS, void *dX, float *dW,
                      size_t rows, int C, la_dtype dt, la_dtype wt, la_dtype st,
                      void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Short causal convolution along the rows, one filter of W taps a channel, with an activation: what stands in front of
 * a selective scan.  For each of B sequences of N rows with C channels
 *
 *     v_t = bias + sum_{j < W} w_j x_{t-(W-1)+j},   y_t = v_t (LA_ACT_NONE) or v_t / (1 + exp(-v_t)) (LA_ACT_SILU)
 *
 * where the W - 1 rows before the first are `state`, the rows carried from an earlier call, or zeros; and backward,
 * with e_t = dy_t dy/dv (zero outside of the sequence),
 *
 *     dx_t = sum_j w_j e_{t+(W-1)-j},   dw_j = sum_t e_t x_{t-(W-1)+j},   dbias = sum_t e_t   (over the sequences too)
 *
 *   X: B * N rows of C elements of `dt` (LA_F32 / LA_BF16), x_stride >= C elements from one row to the next: a part of wider
 *       rows may be given as it is.  Y, dY, dX: [B, N, C] of `dt`, dense.
 *   Wt: [C, W]; bias: [C], or NULL for zeros; both of `wt`, LA_F32 or `dt`.  2 <= W <= 8.
 *   state: [B, W - 1, C] of `dt`, oldest row first, NULL: zeros.  last: the W - 1 rows to carry on, NULL: not wanted; where a
 *       sequence has fewer rows than that, those of `state` move up.  last must not be state itself.
 *   dlast, dstate: their gradients, [B, W - 1, C] of `dt`; dlast NULL: zeros, dstate NULL: not wanted.
 *   dW: [C, W] float32, dbias: [C] float32, or NULL where they are not wanted.
 *   lengths: NULL, or B ints on the device.  Rows from lengths[b] on are padding: they are not read, every output is zero there
 *       (a length of 0 or less: `last` is `state`; one of N or more is N).
 *   workspace (only where dW or dbias is wanted): at least la_conv_workspace_bytes(B, N, C, W) bytes, 256-byte aligned.
 * Sums are float32, those of dW and dbias in a fixed order.  Addresses are those of elements.
 * Limits: B, N, C >= 1, N <= 2^30, B * N * x_stride < 2^40, B * C * ceil(N / 16) < 2^31, C < 2^31 - 256.
 *
 * la_conv_step appends T rows to the carried ones, which it updates in place: the form for single tokens.  Rows are walked one
 * after another, T is meant to be small.  Calls that share a state must not overlap in time.
 * Error behaviour as for la_forward; an unknown activation is LA_ERR_UNSUPPORTED.
 */
typedef enum la_act {
    LA_ACT_NONE = 0,
    LA_ACT_SILU = 1
} la_act;

LA_API size_t la_conv_workspace_bytes(int B, int N, int C, int W);

LA_API la_status la_conv_forward(const void *X, size_t x_stride, const void *Wt, const void *bias, const void *state,
                     void *Y, void *last, const int *lengths,
                     int B, int N, int C, int W, la_act act, la_dtype dt, la_dtype wt, void *hip_stream);

LA_API la_status la_conv_backward(const void *X, size_t x_stride, const void *Wt, const void *bias, const void *state,
                     const void *dY, const void *dlast, void *dX, float *dW, float *dbias, void *dstate,
                     const int *lengths, int B, int N, int C, int W, la_act act, la_dtype dt, la_dtype wt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

LA_API la_status la_conv_step(const void *X, size_t x_stride, const void *Wt, const void *bias, void *state, void *Y,
                     int B, int T, int C, int W, la_act act, la_dtype dt, la_dtype wt, void *hip_stream);

/*
 * Selective state space scan: a recurrence with S states to a channel, whose decays and inputs depend on the row, read out by a
 * vector that does too.  For each of B sequences of N rows with C channels c, in G groups of C / G neighbours that share
 * B_t and C_t, and states s < S
 *
 *     d_t[c] = softplus(dt_t[c] + bias[c]) (LA_STEP_SOFTPLUS: log(1 + exp(.))) or dt_t[c] + bias[c] (LA_STEP_VALUE)
 *     h_t[c,s] = exp(d_t[c] A[c,s]) h_{t-1}[c,s] + d_t[c] x_t[c] B_t[s],     y_t[c] = sum_s C_t[s] h_t[c,s] + D[c] x_t[c]
 *
 * and backward, with g_t = C_t dy_t + exp(d_{t+1} A) g_{t+1} (from dlast behind the last row) and e_t = g_t exp(d_t A) h_{t-1},
 *
 *     dx_t = d_t sum_s g_t B_t + D dy_t,     dd_t = x_t sum_s g_t B_t + sum_s e_t A,     ddt_t = dd_t or dd_t / (1 + exp(-dt_t - bias))
 *     dB_t = sum_c g_t d_t x_t,   dC_t = sum_c dy_t h_t   (over the channels of the group),   dh0 = exp(d_0 A) g_0
 *     dA = sum_t e_t d_t,   dD = sum_t dy_t x_t,   dbias = sum_t ddt_t   (over the sequences too)
 *
 *   X, Dt: B * N rows of C elements of `dt` (LA_F32 / LA_BF16), Bm, Cm: B * N rows of G * S; x_stride, dt_stride, b_stride,
 *       c_stride elements from one row to the next: parts of wider rows may be given as they are.
 *       Y, dY, dX, dDt: [B, N, C], dBm, dCm: [B, N, G, S] of `dt`, dense.
 *   A: [C, S] float32 (the decays exp(d A) have to be floats, and so has their product over a run of rows: A < 0 with d >= 0).
 *       D, bias: [C] float32, or NULL for zeros.  dA, dD, dbias: their gradients, float32, or NULL where they are not wanted.
 *   h0, last, dlast, dh0: [B, C, S] float32.  h0 NULL: zeros; last (the state after the last row) NULL: not wanted; dlast NULL:
 *       zeros; dh0 NULL: not wanted.
 *   saved: states that the forward call leaves for the backward call with the same arguments, those before every 16th row,
 *       la_selective_saved_bytes(B, N, C, S) bytes (S / 4 for every element of X), 256-byte aligned; NULL in a forward call that no
 *       backward call follows.  Its layout is private to the library.
 *   lengths: NULL, or B ints on the device.  Rows from lengths[b] on are padding: they are not read, every output is zero there, and
 *       `last` is the state before them (a length of 0 or less leaves h0, one of N or more is N).
 *   workspace: at least la_selective_workspace_bytes(B, N, C, S, G, is_backward) bytes, 256-byte aligned; NULL where that is 0.
 *       Nothing in it has to start at zero.  Calls that share one must not overlap in time, two captured graphs' neither.
 * States, products and sums are float32, the sums in a fixed order: two runs give the same bits.  Infinities and NaN go where the
 * formulas take them, a decay that is too small for a float being 0.  Addresses are those of elements.
 * Limits: B, N, C, S, G >= 1, N <= 2^30, S <= 128, C a multiple of G, every stride, C and G * S < 2^24, B * N * stride < 2^40
 * for every tensor, B * G * ceil(C / G / 64) * ceil(N / 16) < 2^31 and, without the last factor, < 2^21.
 *
 * la_selective_step appends T rows to a carried state, [B, C, S] float32, and updates it in place: the form for single
 * tokens.  No workspace; rows are walked one after another, T is meant to be small.  Calls that share a state must not overlap in time.
 * Error behaviour as for la_forward; an unknown step is LA_ERR_UNSUPPORTED.
 */
typedef enum la_step {
    LA_STEP_VALUE = 0,
    LA_STEP_SOFTPLUS = 1
} la_step;

LA_API size_t la_selective_workspace_bytes(int B, int N, int C, int S, int G, int is_backward);
LA_API size_t la_selective_saved_bytes(int B, int N, int C, int S);

LA_API la_status la_selective_forward(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                     const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D, const float *bias,
                     const float *h0, void *Y, float *last, void *saved, size_t saved_bytes, const int *lengths,
                     int B, int N, int C, int S, int G, la_step step, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

LA_API la_status la_selective_backward(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                     const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D, const float *bias,
                     const void *saved, size_t saved_bytes, const void *dY, const float *dlast,
                     void *dX, void *dDt, float *dA, void *dBm, void *dCm, float *dD, float *dbias, float *dh0,
                     const int *lengths, int B, int N, int C, int S, int G, la_step step, la_dtype dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

LA_API la_status la_selective_step(const void *X, size_t x_stride, const void *Dt, size_t dt_stride, const float *A,
                     const void *Bm, size_t b_stride, const void *Cm, size_t c_stride, const float *D, const float *bias,
                     float *state, void *Y, int B, int T, int C, int S, int G, la_step step, la_dtype dt, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* LA_H_ */
