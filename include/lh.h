/*
 * lh.h -- C ABI of the distilled modal recurrence on AMD MI355X (gfx950).
 *
 * The operation (Laughing Hyena distillation, Sec. 3.4 "Deploying the
 * recurrence", Proposition "modal_realization", App. B.1):
 *
 *   every channel c of a bank of D distilled filters carries d complex modes
 *   with poles lambda[c,n], residues R[c,n] and a real pass-through h0[c];
 *   its filter is h_0 = h0, h_t = Re sum_n R[c,n] lambda[c,n]^(t-1) (t >= 1,
 *   eq. "modal_impulse").  Its state-space form is A = diag(lambda), B = 1,
 *   C = R, D = h0 (eq. "dtssm"):
 *
 *       y_t     = Re( sum_n R[c,n] x_t[n] ) + h0[c] u_t      (reads x_t)
 *       x_{t+1} = lambda[c,n] x_t[n] + u_t                     (then updates)
 *
 *   so that, from x_0 = 0, y is the causal convolution of h with u
 *   (eq. "cnn") and x_T[n] = sum_{k<T} lambda[c,n]^(T-1-k) u_k.
 *
 * Prefill (lh_prefill) processes a prompt of T tokens: all outputs y_0..y_{T-1}
 * and the post-prompt state x_T.  Decode (lh_step) advances the state by one
 * token per call and returns that token's output; a step right after a prefill
 * of T tokens returns y_T.
 *
 * Layouts (all row-major, contiguous, caller-owned device memory):
 *   lambda, R : [D, d]    complex64, interleaved (re, im)        (lh_c32)
 *   h0        : [D]       float32
 *   u, y      : [B, T, D] float32 or bfloat16 (io_dtype), channel fastest
 *   state     : [B, D, d] complex64, mode fastest
 *   u_t, y_t  : [B, D]    float32 or bfloat16 (io_dtype)
 * All arithmetic is float32; bfloat16 inputs are widened exactly and bfloat16
 * outputs are rounded to nearest, ties to even.
 *
 * Ownership and execution: the library never allocates, frees or keeps a
 * pointer; it holds no state between calls and is re-entrant.  Work is enqueued
 * asynchronously on `stream` (a hipStream_t; NULL is the null stream) and the
 * call returns without synchronising.  Calls on the same buffers must be
 * ordered by the caller (same stream, or events).
 *
 * Errors: every argument is checked on the host before any device work is
 * enqueued; on a non-LH_OK status nothing has been enqueued and no buffer has
 * been touched.  Faults during execution surface at the caller's next
 * synchronisation of `stream`.  No call aborts and no C++ exception crosses
 * this interface.  lh_last_error() returns a thread-local description of the
 * most recent failure in the calling thread.
 */
#ifndef LH_H
#define LH_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LH_ABI_VERSION 2

/* complex64, interleaved real and imaginary parts */
typedef struct lh_c32 {
    float re;
    float im;
} lh_c32;

/* element type of u / y (and u_t / y_t); lambda, R, h0 and the state are
 * always float32-based */
typedef enum lh_dtype {
    LH_F32 = 0,
    LH_BF16 = 1
} lh_dtype;

typedef enum lh_status {
    LH_OK = 0,
    LH_ERR_INVALID_ARG = 1,       /* null pointer, bad size, size overflow,
                                     pointer not accessible from the device */
    LH_ERR_OVERLAP = 2,           /* an output buffer overlaps another buffer */
    LH_ERR_UNSUPPORTED_DTYPE = 3, /* io_dtype is not LH_F32 or LH_BF16 */
    LH_ERR_NO_DEVICE = 4,         /* no HIP device is visible */
    LH_ERR_WORKSPACE = 5,         /* workspace null or smaller than required */
    LH_ERR_HIP = 6                /* the HIP runtime refused a launch */
} lh_status;

/* Largest supported number of modes per channel. */
#define LH_MAX_MODES 1024

/* LH_ABI_VERSION of the built library. */
int lh_abi_version(void);

/* Static description of a status code (never NULL). */
const char* lh_status_string(lh_status status);

/* Thread-local detail of the most recent non-LH_OK status returned in the
 * calling thread ("" if none). */
const char* lh_last_error(void);

/*
 * Workspace bytes lh_prefill needs for these sizes, for either input type
 * (the larger of the float32 and bfloat16 plans' needs).  Returns 0 when the
 * plan needs no workspace and (size_t)-1 when the arguments are invalid.
 * Pure function of its arguments; host only.
 */
size_t lh_prefill_workspace_bytes(int64_t B, int64_t D, int64_t d, int64_t T);

/*
 * Prefill (Sec. 3.4, "fast pre-filling"; states start at x_0 = 0): outputs
 * y[b,t,c] for t < T and the post-prompt state state[b,c,n] = x_T.
 *
 *   lambda, R, h0 : inputs as laid out above
 *   u             : [B,T,D] prompt inputs (io_dtype)
 *   B, D, d, T    : B >= 1, D >= 1, 1 <= d <= LH_MAX_MODES, T >= 0
 *   io_dtype      : LH_F32 or LH_BF16 (u and y)
 *   state         : out, [B,D,d] complex64 (overwritten, not read)
 *   y             : out, [B,T,D] (io_dtype); may be NULL only when T == 0
 *   workspace     : device scratch of at least
 *                   lh_prefill_workspace_bytes(B,D,d,T) bytes, 256-byte
 *                   aligned; may be NULL when that size is 0.  Its contents
 *                   on entry are ignored and on exit undefined.
 *
 * The library picks the plan (lh_prefill_plan with plan = LH_PREFILL_AUTO
 * reports which): the matrix-core plan over the whole prompt where its
 * workgroups fill the GPU, the segmented matrix-core plan where the prompt
 * must be split in time to fill it, else the general chunked scan, which runs
 * on the matrix cores too where its sizes allow and that is faster (see
 * lh_prefill_with_plan for what each computes and needs).  Every plan gives
 * the same results within the accuracy of its arithmetic: float32 rounding, but
 * for plans named LH_PLAN_MFMA and LH_PLAN_MFMA_SEG with 16-byte aligned u and y
 * the two-term operands described at lh_prefill_with_plan.  An input that is not
 * finite affects its (row, channel) from its own step on; in those two plans, with
 * such u and y, from the start of its 16-step chunk on (the outputs before it in
 * the chunk are lost too).
 * T == 0 zeroes the state and leaves y untouched.  y must not overlap u,
 * state, lambda, R, h0 or workspace; state must not overlap any input.
 */
lh_status lh_prefill(const lh_c32* lambda, const lh_c32* R, const float* h0,
                     const void* u, int64_t B, int64_t D, int64_t d, int64_t T,
                     lh_dtype io_dtype, lh_c32* state, void* y,
                     void* workspace, size_t workspace_bytes, void* stream);

/* Scratch bytes lh_prefill_noalloc holds per GPU (64 MiB). */
#define LH_NOALLOC_SCRATCH_BYTES (UINT64_C(64) << 20)

/*
 * lh_prefill for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid allocation): the
 * same arguments, ownership and errors as lh_prefill, with no workspace
 * argument.  The plan's scratch is a static array of
 * LH_NOALLOC_SCRATCH_BYTES that the library holds on each GPU it runs on
 * until the process ends; this call allocates nothing and makes no
 * allocating runtime call.  Its results are lh_prefill's, bit for bit, where
 * lh_prefill_workspace_bytes(B,D,d,T) <= LH_NOALLOC_SCRATCH_BYTES.  Larger plans
 * named LH_PLAN_SCAN run the VALU scan if its own states fit, with its rounding;
 * all others return LH_ERR_WORKSPACE before anything is enqueued.  Every call
 * on one GPU shares that GPU's array, which keeps the last call's contents (no
 * plan reads scratch it has not written in the same call): calls that overlap
 * on one GPU (on different streams, or from several threads without ordering)
 * race on it and must not be made.
 */
lh_status lh_prefill_noalloc(const lh_c32* lambda, const lh_c32* R, const float* h0,
                             const void* u, int64_t B, int64_t D, int64_t d, int64_t T,
                             lh_dtype io_dtype, lh_c32* state, void* y, void* stream);

/* Plan requests of lh_prefill_with_plan (values > 0 are VALU chunk lengths). */
#define LH_PREFILL_AUTO 0
#define LH_PREFILL_MFMA (-1)
#define LH_PREFILL_MFMA_SEG (-2)

/* Prefill plans: names that fix a call's workspace.  lh_prefill_path tells what
 * runs inside it. */
typedef enum {
    LH_PLAN_SCAN = 0,      /* general chunked scan */
    LH_PLAN_MFMA = 1,      /* matrix-core plan over the whole prompt */
    LH_PLAN_MFMA_SEG = 2   /* segmented matrix-core plan */
} lh_prefill_plan_kind;

/*
 * The plan of a prefill with these sizes, plan request and input type.
 * Returns an lh_prefill_plan_kind, or -1 when the arguments are invalid or no
 * plan exists (as the prefill would fail).  Pure function of its arguments;
 * host only, no device call.
 */
int lh_prefill_plan(int64_t B, int64_t D, int64_t d, int64_t T, int64_t plan,
                    lh_dtype io_dtype);

/*
 * What such a call executes with a workspace of at least
 * lh_prefill_with_plan_workspace_bytes bytes and 16-byte aligned u and y.
 * Returns 1 for the matrix cores, 0 for the VALU scan, -1 where
 * lh_prefill_plan does.  *columns (unless NULL): on the matrix cores the
 * consecutive 16-step chunks of a row that a product takes side by side (1, 2, 4
 * or 16 of its 16 columns), else 1.  *segments (unless NULL): the time segments
 * processed in parallel (1: the prompt in one pass).  The name of a plan does not
 * tell: the scan runs on the matrix cores where that is the faster way, a
 * whole-prompt plan may be cut into segments and a segmented one may not, and
 * past 2^31 bytes in 257 steps of a row every plan runs on the VALU.  Pure
 * function of its arguments; host only, no device call.
 */
int lh_prefill_path(int64_t B, int64_t D, int64_t d, int64_t T, int64_t plan,
                    lh_dtype io_dtype, int64_t* columns, int64_t* segments);

/*
 * Workspace bytes of lh_prefill_with_plan for this plan request (as
 * lh_prefill_workspace_bytes; plan = LH_PREFILL_AUTO gives the same value).
 */
size_t lh_prefill_with_plan_workspace_bytes(int64_t B, int64_t D, int64_t d, int64_t T,
                                            int64_t plan);

/*
 * lh_prefill with the plan named by the caller instead of chosen by the
 * library: for callers that compare plans (tests, benchmarks).  Same results,
 * arguments, ownership and errors as lh_prefill, with
 *
 *   plan = LH_PREFILL_AUTO (0): the automatic plan (lh_prefill itself);
 *   plan > 0: the VALU chunked scan with this time-chunk length (the prompt
 *            is cut into ceil(T/plan) chunks processed in parallel: each
 *            chunk's end state from zero, a carry across chunks with
 *            lambda^plan formed in float64, then the outputs from each chunk's
 *            entry state; plan >= T means one sequential pass per row);
 *   plan = LH_PREFILL_MFMA: the matrix-core plan (chunks of 16 steps as dense
 *            contractions on the MFMA units: outputs Y = T U + W X_in, chunk
 *            end states S = P U and the carry X_in <- lambda^16 X_in + S; the
 *            16 columns of a product are batch rows, or fewer rows and several
 *            chunks of each; with
 *            the float32 operands split into bfloat16 terms: three with
 *            float32 u/y, but two of X_in (error of the outputs near 2e-6 of
 *            their norm); two for the outputs and three for the state with
 *            bfloat16 u/y; d = 16 or 32 require D % 8 == 0, d = 64 requires
 *            float32 u/y and D % 4 == 0; always T >= 1 and 16-byte aligned u and
 *            y, else LH_ERR_INVALID_ARG).  The automatic plan, which takes any
 *            alignment of u and y, uses it where
 *            supported and either ceil(D/16) * ceil(B/32) >= 256 (enough
 *            workgroups to fill the GPU without splitting the prompt in time)
 *            or a count of the 32-step chunks each compute unit walks puts
 *            it within 7/5 of the segmented plan below (the count depends
 *            on the input type, so float32 and bfloat16 calls may take
 *            different plans); at d = 64 also when T does not split into
 *            segments and B >= 4 or ceil(D/4) * ceil(B/16) >= 256, and never
 *            when B < 4 and B * T <= 1024;
 *   plan = LH_PREFILL_MFMA_SEG: the segmented matrix-core plan: its workspace
 *            holds the states of 2^k segments of T / 2^k steps (a multiple of
 *            32, at least 256), the fewest whose (batch row, segment) pairs
 *            fill the GPU.  The prompt is cut into at most that many where the
 *            chunks of a row side by side in a product do not fill the GPU
 *            already: a matrix-core pass computes each segment's end state from
 *            zero, a carry gives each segment its entry state, and a second
 *            matrix-core pass computes the outputs (same operand splitting
 *            and requirements as LH_PREFILL_MFMA, and such a T).  The
 *            automatic plan takes it where the whole-prompt matrix-core plan
 *            is supported but not chosen and T splits this way (at d = 64
 *            only when B * T > 1024).
 * Elsewhere an automatic call runs the general chunked scan: the matrix-core
 * pass above, every operand in three terms, where d <= 64 and a fitted estimate
 * of both times favours it, else, or with a workspace that does not hold its
 * tables (but the VALU scan's states, if it has any), the VALU scan.  A named
 * automatic plan whose u or y is not 16-byte aligned takes three terms too.
 * workspace: at least lh_prefill_with_plan_workspace_bytes(B,D,d,T,plan)
 * bytes.  A plan request the sizes do not support returns LH_ERR_INVALID_ARG.
 */
lh_status lh_prefill_with_plan(const lh_c32* lambda, const lh_c32* R, const float* h0,
                               const void* u, int64_t B, int64_t D, int64_t d, int64_t T,
                               lh_dtype io_dtype, lh_c32* state, void* y, int64_t plan,
                               void* workspace, size_t workspace_bytes, void* stream);

/* Longest prompt lh_prefill_fft accepts (transforms of at most 2^20 points). */
#define LH_FFT_MAX_T (INT64_C(1) << 19)

/*
 * Workspace bytes lh_prefill_fft needs for these sizes; 0 when T == 0 and
 * (size_t)-1 when the arguments are invalid or T > LH_FFT_MAX_T.  Pure
 * function of its arguments.  About (2 + 2 ceil(B/2)) N D 4 bytes, with N the
 * transform length below, plus partial states and small tables.
 */
size_t lh_prefill_fft_workspace_bytes(int64_t B, int64_t D, int64_t d, int64_t T);

/*
 * Prefill by FFT convolution (Sec. 3.4, fast pre-filling "via convolutions"):
 * the same results as lh_prefill (outputs y[b,t,c] for t < T and state = x_T),
 * computed the other way the paper describes:
 *
 *   hhat_0 = h0[c],  hhat_t = Re sum_n R[c,n] lambda[c,n]^(t-1)   (t < T; the
 *       O(dT) evaluation of Lemma "ssmd_impulse")
 *   y[b,t,c]     = sum_{j<=t} hhat_{t-j} u[b,j,c]   (eq. "cnn"), by N-point
 *       FFTs with N the smallest power of two >= 2T - 1
 *   state[b,c,n] = sum_{k<T} lambda[c,n]^(T-1-k) u[b,k,c]  (Vandermonde
 *       contraction)
 *
 * Arguments, layouts, ownership and errors as lh_prefill, with
 *   T          : 0 <= T <= LH_FFT_MAX_T
 *   workspace  : at least lh_prefill_fft_workspace_bytes(B,D,d,T) bytes,
 *                256-byte aligned (NULL allowed when that size is 0)
 * The rounding differs from the scan's (float32 transforms: an error near
 * 1e-7 log2(N) of the largest outputs of a row, spread over the row).
 */
lh_status lh_prefill_fft(const lh_c32* lambda, const lh_c32* R, const float* h0,
                         const void* u, int64_t B, int64_t D, int64_t d, int64_t T,
                         lh_dtype io_dtype, lh_c32* state, void* y,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Decode step (Proposition "modal_realization"; App. B.1 for the real part):
 *   y_t[b,c]     = Re(sum_n R[c,n] state[b,c,n]) + h0[c] u_t[b,c]
 *   state[b,c,n] = lambda[c,n] state[b,c,n] + u_t[b,c]      (in place)
 *
 *   state : in/out [B,D,d] complex64
 *   u_t   : [B,D] (io_dtype);  y_t : out [B,D] (io_dtype)
 * y_t must not overlap any other buffer; state must not overlap lambda, R,
 * h0 or u_t.  O(d) work per (b, c); one kernel launch; no workspace.
 */
lh_status lh_step(const lh_c32* lambda, const lh_c32* R, const float* h0,
                  lh_c32* state, const void* u_t, void* y_t,
                  int64_t B, int64_t D, int64_t d, lh_dtype io_dtype,
                  void* stream);

/* Largest modal order the companion form accepts (companion order 2d <= 32). */
#define LH_COMPANION_MAX_MODES 16

/*
 * Companion (rational) form of the distilled filters (App. "From Transfer
 * Function to State-Space", eq. "ssm_canon"; canonization of a modal SSM).
 * The real filter h_0 = h0, h_t = Re sum_n R_n lambda_n^(t-1) is the impulse
 * response of a real system of order 2d (each pole with its conjugate,
 * residues R_n / 2 and conj(R_n) / 2, App. B.1) whose transfer function in
 * w = z^-1 is
 *
 *   H(w) = h0 + (beta_1 w + ... + beta_2d w^2d) / (1 + a_1 w + ... + a_2d w^2d)
 *
 * This call writes, per channel, a[c, m-1] = a_m and beta[c, m-1] = beta_m
 * (m = 1..2d), computed in float64 from the complex64 poles and residues.
 *
 *   lambda, R : [D, d] complex64;  a, beta : out [D, 2d] float64
 *   D >= 1, 1 <= d <= LH_COMPANION_MAX_MODES
 * Outputs must not overlap each other or the inputs.  One kernel launch; no
 * workspace; same execution and error rules as lh_step.
 *
 * Numerical range: p's coefficients grow like binomial coefficients and the
 * companion state like the impulse response of 1/p, far beyond the outputs it
 * combines, so even in float64 the form meets a 1e-4 relative accuracy only
 * for small orders (measured over 1500 steps with pole angles spread over
 * [0, pi]: d <= 8 at pole radii up to 0.9999; d = 16 loses it near the unit
 * circle).  The modal calls above do not have this limit.
 */
lh_status lh_companion_coeffs(const lh_c32* lambda, const lh_c32* R, int64_t D, int64_t d,
                              double* a, double* beta, void* stream);

/*
 * Companion decode step (Lemma "efficient_recurrence"), per (b, c):
 *   y_t[b,c]      = sum_m beta[c,m] state[b,c,m] + h0[c] u_t[b,c]
 *   state[b,c,:]  = (u_t[b,c] - sum_m a[c,m] state[b,c,m], state[b,c,0], ...,
 *                    state[b,c,2d-2])                               (in place)
 * in float64, y_t rounded to io_dtype.
 *
 *   a, beta : [D, 2d] float64 (lh_companion_coeffs), 16-byte aligned
 *   h0      : [D] float32
 *   state   : in/out [B, D, 2d] float64, 16-byte aligned
 *   u_t, y_t: [B, D] (io_dtype)
 * y_t must not overlap any other buffer; state must not overlap a, beta, h0
 * or u_t.  One kernel launch; no workspace; same execution and error rules
 * as lh_step.
 */
lh_status lh_companion_step(const double* a, const double* beta, const float* h0,
                            double* state, const void* u_t, void* y_t,
                            int64_t B, int64_t D, int64_t d, lh_dtype io_dtype, void* stream);

/* Workspace bytes of lh_companion_init: T D 8 (the taps of 1/p); 0 when
 * T == 0, (size_t)-1 for invalid sizes. */
size_t lh_companion_init_workspace_bytes(int64_t D, int64_t d, int64_t T);

/*
 * Companion state after a prompt without stepping (Proposition "fast_init"):
 *   state[b,c,j] = v_{T-1-j},  v = g * u[b,:,c],  j = 0..2d-1
 * with g the impulse response of 1/p (g_0 = 1, g_t = -sum_m a_m g_{t-m}) and
 * v_t = 0 for t < 0; the state lh_companion_step reaches from zero after the
 * T prompt inputs.  Prompt outputs come from lh_prefill or lh_prefill_fft
 * (the same filter).
 *
 *   a        : [D, 2d] float64;  u : [B, T, D] (io_dtype)
 *   state    : out [B, D, 2d] float64, 16-byte aligned
 *   workspace: lh_companion_init_workspace_bytes(D, d, T) bytes, 256-byte
 *              aligned (NULL allowed when that is 0)
 *   T >= 0; T == 0 zeroes the state
 * state and workspace must not overlap each other or the inputs.  Two kernel
 * launches; same execution and error rules as lh_prefill.
 */
lh_status lh_companion_init(const double* a, const void* u, int64_t B, int64_t D, int64_t d,
                            int64_t T, lh_dtype io_dtype, double* state, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * Multi-head decode step (Sec. 5, "Multi-head Long Convolutions": the
 * projections q, k, v of width D = M N are split into M heads of N channels;
 * per head the outer product z = k (x) v is convolved entry by entry with the
 * head's distilled filter and the result multiplies q).  Every entry (i, j)
 * of head m carries the d-mode state of Proposition "modal_realization":
 *
 *   z[i,j]          = k[b, mN+i] v[b, mN+j]
 *   y[b, mN+i]      = sum_j q[b, mN+j] ( Re(sum_n R[m,n] state[b,m,i,j,n])
 *                                        + h0[m] z[i,j] )          (reads state)
 *   state[b,m,i,j,n] = lambda[m,n] state[b,m,i,j,n] + z[i,j]       (in place)
 *
 * The q contraction runs over the second (value) index of z; exchanging the
 * k and v arguments gives the other orientation (q against the key index).
 *
 *   lambda, R : [M, d] complex64;  h0 : [M] float32 (one filter per head)
 *   state     : in/out [B, M, N, N, d] complex64, mode fastest
 *   q, k, v   : [B, M N] (io_dtype);  y : out [B, M N] (io_dtype)
 *   B, M, N   : >= 1;  1 <= d <= LH_MAX_MODES
 * y must not overlap any other buffer; state must not overlap lambda, R, h0,
 * q, k or v.  One kernel launch; no workspace; same execution and error
 * rules as lh_step.
 */
lh_status lh_mh_step(const lh_c32* lambda, const lh_c32* R, const float* h0,
                     lh_c32* state, const void* q, const void* k, const void* v, void* y,
                     int64_t B, int64_t M, int64_t N, int64_t d, lh_dtype io_dtype,
                     void* stream);

/*
 * Distillation objective of the modal form (Sec. 3.2, "Modal canonical
 * form"; the O(dL) filter evaluation of Lemma "ssmd_impulse").  Per channel c,
 * poles in polar form lambda = A e^{i theta} and residues R (cartesian) are
 * fitted to a real target filter h_1 .. h_L by the squared l2 interpolation
 * error:
 *
 *   hhat_t = Re sum_n R[c,n] lambda[c,n]^(t-1)   (t = 1..L)
 *   loss[c] = sum_t (hhat_t - h_t)^2
 *
 * with its gradients with respect to A, theta, Re R and Im R (dR holds
 * d/dRe R + i d/dIm R).  The pass-through h0 is matched by h_0 and is not
 * part of the objective.
 *
 *   A, theta : [D, d] float32 (polar poles);  R : [D, d] complex64
 *   target   : [D, L] float32, target[c, t-1] = h_t
 *   loss     : out [D];  dA, dtheta : out [D, d];  dR : out [D, d] complex64
 *   hhat     : out [D, L] (the materialised filter) or NULL
 *   D >= 1, 1 <= d <= LH_MAX_MODES, L >= 1
 * Outputs must not overlap each other or the inputs.  One kernel launch; no
 * workspace; same execution and error rules as lh_step.
 */
lh_status lh_distill(const float* A, const float* theta, const lh_c32* R, const float* target,
                     int64_t D, int64_t d, int64_t L, float* loss, float* dA, float* dtheta,
                     lh_c32* dR, float* hhat, void* stream);

/*
 * The selective block: layer norm, a short causal convolution per channel and the
 * selective state-space scan, the input-dependent sibling of the recurrence above,
 * for prompts, single tokens and training.
 *
 * Rows: an input x [B, T, D] of these calls whose argument has an `ld` is read from
 * rows of D consecutive elements, ld >= D elements apart: token t of batch row b is
 * row b T + t (a slice of a projection's output needs no copy).  Outputs are
 * contiguous.  Any element alignment is taken.  An output must not overlap any other
 * buffer (a strided input is taken as the whole range from its first to its last
 * element) but for the pairs named below, which may be the same buffer.
 *
 * lengths ([B] int32, or NULL): a right-padded batch; row b has lengths[b] tokens (a
 * value outside [0, T] is taken as the nearer end).  Tokens past them are not read
 * (the memory must be accessible all the same), their outputs and gradients are 0, and
 * they leave the state alone.
 *
 * Sums, statistics and states are float32; bfloat16 outputs are rounded once, to
 * nearest even.  Every call gives the same bits for the same inputs.  Sizes that need
 * 2^32 threads or more in one launch return LH_ERR_INVALID_ARG (layer norm and the
 * convolution count the launches of their gradients, and a thread for each channel).
 */

/*
 * Layer norm over the last axis:
 *   s = x (+ residual),  y = (s - mean s) / sqrt(var s + eps) * w + b
 *
 *   x, residual : [rows, D] (io_dtype); residual may be NULL
 *   w, b        : [D] float32; b may be NULL
 *   rows >= 0, D >= 1, eps >= 0
 *   y           : out [rows, D] (io_dtype)
 *   total       : out [rows, D] (io_dtype), s rounded; NULL, or with a residual (it may
 *                 be the buffer of x or of residual).  y is formed from s unrounded.
 *   mean, rstd  : out [rows] float32, mean s and 1 / sqrt(var s + eps), which the
 *                 gradient takes; NULL where not needed
 * One kernel launch; no workspace; same execution and error rules as lh_step.
 */
lh_status lh_layer_norm(const void* x, const void* residual, const float* w, const float* b,
                        int64_t rows, int64_t D, float eps, lh_dtype io_dtype, void* y,
                        void* total, float* mean, float* rstd, void* stream);

/* Workspace bytes of lh_layer_norm_backward; (size_t)-1 for invalid sizes. */
size_t lh_layer_norm_backward_workspace_bytes(int64_t rows, int64_t D);

/*
 * Gradients of lh_layer_norm, from what went in (x is s, the total where there was a
 * residual) and its mean and rstd:
 *   h = (x - mean) rstd,  g = dy w
 *   dx = rstd (g - mean g - h mean(g h)) (+ dtotal),  dw = sum dy h,  db = sum dy
 *
 *   dy, x, dtotal : [rows, D] (io_dtype); dtotal, the gradient of total, may be NULL
 *   dx            : out [rows, D] (io_dtype), of x and of residual alike; it may be the
 *                   buffer of dtotal
 *   dw, db        : out [D] float32; db may be NULL
 *   workspace     : lh_layer_norm_backward_workspace_bytes bytes, 256-byte aligned (NULL
 *                   allowed when that is 0)
 */
lh_status lh_layer_norm_backward(const void* dy, const void* x, const float* w, const float* mean,
                                 const float* rstd, const void* dtotal, int64_t rows, int64_t D,
                                 lh_dtype io_dtype, void* dx, float* dw, float* db,
                                 void* workspace, size_t workspace_bytes, void* stream);

/* Largest number of taps of the short convolution. */
#define LH_SHORT_CONV_MAX_TAPS 8

/*
 * Short causal convolution, one filter of K taps per channel:
 *   o_t = bias + sum_k w[c, k] x_(t - K + 1 + k),   y_t = silu ? o_t sigmoid(o_t) : o_t
 * (w[c, K - 1] meets the current token).
 *
 *   x       : [B, T, D] (io_dtype), rows ld_x apart
 *   w, bias : [D, K] and [D] float32; bias may be NULL
 *   lengths : [B] int32 or NULL
 *   B >= 1, T >= 0, D >= 1, 1 <= K <= LH_SHORT_CONV_MAX_TAPS
 *   resume  : the inputs before the first token are the state's (else zeros, and the
 *             state is not read)
 *   state   : in/out [B, K - 1, D] (io_dtype): the last K - 1 inputs, oldest first
 *             (NULL allowed when K = 1)
 *   y       : out [B, T, D] (io_dtype)
 * One kernel launch; no workspace.
 */
lh_status lh_short_conv_prefill(const void* x, int64_t ld_x, const float* w, const float* bias,
                                const int32_t* lengths, int64_t B, int64_t T, int64_t D, int64_t K,
                                lh_dtype io_dtype, int silu, int resume, void* state, void* y,
                                void* stream);

/* One token per batch row, x_t and y_t [B, D], the state in place: the outputs of a
 * prefill that resumes with T = 1. */
lh_status lh_short_conv_step(const void* x_t, int64_t ld_x, const float* w, const float* bias,
                             int64_t B, int64_t D, int64_t K, lh_dtype io_dtype, int silu,
                             void* state, void* y_t, void* stream);

/* Workspace bytes of lh_short_conv_backward; (size_t)-1 for invalid sizes. */
size_t lh_short_conv_backward_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t K);

/*
 * Gradients of lh_short_conv_prefill without resume: dx [B, T, D] (io_dtype), dw [D, K]
 * and dbias [D] float32 (dbias may be NULL) from dy [B, T, D] (io_dtype) and the inputs.
 * workspace as in lh_layer_norm_backward.
 */
lh_status lh_short_conv_backward(const void* dy, const void* x, int64_t ld_x, const float* w,
                                 const float* bias, const int32_t* lengths, int64_t B, int64_t T,
                                 int64_t D, int64_t K, lh_dtype io_dtype, int silu, void* dx,
                                 float* dw, float* dbias, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* Largest number of states per channel of the selective scan. */
#define LH_SELECTIVE_MAX_STATES 128

/*
 * Selective state-space scan.  Per batch row, channel c and state n, g = c / (D / G):
 *
 *   delta = log(1 + exp(dt[b,t,c] + dt_bias[c]))
 *   x[n]  = exp(delta A[c,n]) x[n] + delta Bm[b,t,g,n] u[b,t,c]
 *   y     = sum_n Cm[b,t,g,n] x[n] + h0[c] u[b,t,c],  times z sigmoid(z) where z is given
 *
 * (the output reads the state after the update, unlike lh_step's.)  A <= 0, -infinity among
 * them: a state that decays, or with A = 0 a sum.  Prompts and gradients multiply decays over
 * up to a whole prompt, so with A > 0 results are only right while e^(A sum delta) is finite.
 */
typedef struct lh_selective_inputs {
    const float* A;         /* [D, N] */
    const float* dt_bias;   /* [D] or NULL (0) */
    const float* h0;        /* [D] or NULL (0) */
    const void* dt;         /* [B, T, D] (io_dtype), rows ld_dt apart */
    const void* u;          /* [B, T, D] (io_dtype), rows ld_u apart */
    const void* z;          /* [B, T, D] (io_dtype), rows ld_z apart; NULL: no gate */
    const void* Bm;         /* [B, T, G, N] (io_dtype), rows of G N elements ld_B apart */
    const void* Cm;         /* [B, T, G, N] (io_dtype), rows of G N elements ld_C apart */
    const int32_t* lengths; /* [B] or NULL */
    int64_t ld_dt, ld_u, ld_z, ld_B, ld_C;
    int64_t B, T, D, N, G;  /* B >= 1, T >= 0, D >= 1, 1 <= N <= LH_SELECTIVE_MAX_STATES,
                               G >= 1 divides D */
    lh_dtype io_dtype;
} lh_selective_inputs;

/* Workspace bytes of lh_selective_prefill; (size_t)-1 for invalid sizes. */
size_t lh_selective_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t N, int64_t G);

/*
 * The scan over a prompt.
 *   resume    : start from the state (else from zero, and the state is not read)
 *   state     : in/out [B, D, N] float32, after each row's last token
 *   y         : out [B, T, D] (io_dtype)
 *   workspace : lh_selective_workspace_bytes bytes, 256-byte aligned (NULL allowed when
 *               that is 0)
 * Every ld must be less than 2^26 here (not in a step or in the gradient).
 * One kernel launch, or two or three where the prompt is cut into chunks.
 */
lh_status lh_selective_prefill(const lh_selective_inputs* in, int resume, float* state, void* y,
                               void* workspace, size_t workspace_bytes, void* stream);

/* One token per batch row (T = 1, lengths NULL): y_t [B, D] and the state in place.  One
 * kernel launch; no workspace. */
lh_status lh_selective_step(const lh_selective_inputs* in, float* state, void* y_t, void* stream);

/* What lh_selective_backward takes and gives beside the inputs. */
typedef struct lh_selective_grads {
    const void* dy;  /* [B, T, D] (io_dtype): the gradient of y */
    void* ddt;       /* out [B, T, D] (io_dtype) */
    void* du;        /* out [B, T, D] (io_dtype) */
    void* dz;        /* out [B, T, D] (io_dtype); NULL where z is NULL, and only there */
    void* dBm;       /* out [B, T, G, N] (io_dtype) */
    void* dCm;       /* out [B, T, G, N] (io_dtype) */
    float* dA;       /* out [D, N] */
    float* dh0;      /* out [D], or NULL */
    float* ddt_bias; /* out [D], or NULL */
} lh_selective_grads;

/* Workspace bytes of lh_selective_backward; (size_t)-1 for invalid sizes.  About
 * 5/16 B T D N bytes up to 32 states and 1/2 B T D N beyond: states and gradients of
 * each chunk, and partial sums (16 x 4096 x 2048: 0.7 GB with 16 states, 4.3 GB with 64).
 */
size_t lh_selective_backward_workspace_bytes(int64_t B, int64_t T, int64_t D, int64_t N,
                                             int64_t G);

/* Gradients of lh_selective_prefill without resume, from its inputs alone (the states
 * are formed again).  workspace as there. */
lh_status lh_selective_backward(const lh_selective_inputs* in, const lh_selective_grads* grads,
                                void* workspace, size_t workspace_bytes, void* stream);

/*
 * The ends of a recurrent language model and its gated recurrence: token embedding, a
 * gated linear recurrence, distillation from a teacher's top logits, and the verification
 * of drafted tokens.  Rows, lengths, overlaps, types and the order of sums are as said at
 * the selective block above.  Token ids are int32.
 */

/* The gated recurrence keeps the state before every LH_GATED_MARK-th token for its gradient. */
#define LH_GATED_MARK 8

/*
 * Gated linear recurrence.  Per batch row and channel c:
 *
 *   f = sigmoid(r[b,t,c] + r_bias[c]),  p = sigmoid(i[b,t,c] + i_bias[c])
 *   a = exp(-rate[c] f),  h <- a h + sqrt(1 - a^2) p u[b,t,c]
 *   y = h,  times z sigmoid(z) where z is given
 *
 * rate >= 0 and finite: how fast a channel can forget (0: it holds its state; below 0 the
 * results are NaN).  A gate below 2^-126 (x below about -87.3) is 0.  A state that is not finite
 * stays so (where tokens follow an infinity, it may be NaN).
 */
typedef struct lh_gated_inputs {
    const float* rate;      /* [D] */
    const float* r_bias;    /* [D] or NULL (0) */
    const float* i_bias;    /* [D] or NULL (0) */
    const void* r;          /* [B, T, D] (io_dtype), rows ld_r apart */
    const void* i;          /* [B, T, D] (io_dtype), rows ld_i apart */
    const void* u;          /* [B, T, D] (io_dtype), rows ld_u apart */
    const void* z;          /* [B, T, D] (io_dtype), rows ld_z apart; NULL: no gate */
    const int32_t* lengths; /* [B] or NULL */
    int64_t ld_r, ld_i, ld_u, ld_z;
    int64_t B, T, D;        /* B >= 1, T >= 0, D >= 1 */
    lh_dtype io_dtype;
} lh_gated_inputs;

/* Workspace bytes of lh_gated_prefill; (size_t)-1 for invalid sizes. */
size_t lh_gated_workspace_bytes(int64_t B, int64_t T, int64_t D);

/*
 * The recurrence over a prompt.
 *   resume    : start from the state (else from zero, and the state is not read)
 *   state     : in/out [B, D] float32, after each row's last token
 *   y         : out [B, T, D] (io_dtype)
 *   marks     : out [B, ceil(T / LH_GATED_MARK), D] float32, the state before the tokens 0,
 *               LH_GATED_MARK, 2 LH_GATED_MARK, ..., which the gradient takes; not written
 *               where a row has no such token; NULL where not needed
 *   workspace : lh_gated_workspace_bytes bytes, 256-byte aligned (NULL allowed when that
 *               is 0), of one call at a time: calls that may run at once, graphs among them,
 *               need one each
 * Every ld must be less than 2^26 here and in the gradient (not in a step).
 * One kernel launch, or two where rows are few and workgroups share a prompt's blocks.
 */
lh_status lh_gated_prefill(const lh_gated_inputs* in, int resume, float* state, void* y,
                           float* marks, void* workspace, size_t workspace_bytes, void* stream);

/* One token per batch row (T = 1, lengths NULL): y_t [B, D] and the state in place.  One
 * kernel launch; no workspace. */
lh_status lh_gated_step(const lh_gated_inputs* in, float* state, void* y_t, void* stream);

/* What lh_gated_backward takes and gives beside the inputs. */
typedef struct lh_gated_grads {
    const void* dy;     /* [B, T, D] (io_dtype): the gradient of y */
    const float* marks; /* what lh_gated_prefill left, with resume or without */
    const float* dlast; /* [B, D]: the gradient of the state after the prompt; NULL: 0 */
    void* dr;           /* out [B, T, D] (io_dtype) */
    void* di;           /* out [B, T, D] (io_dtype) */
    void* du;           /* out [B, T, D] (io_dtype) */
    void* dz;           /* out [B, T, D] (io_dtype); NULL where z is NULL, and only there */
    float* drate;       /* out [D]; 0 where rate is 0 (the slope of the square root there
                           has no bound) */
    float* dr_bias;     /* out [D], or NULL */
    float* di_bias;     /* out [D], or NULL */
    float* dfirst;      /* out [B, D]: the gradient of the state before the prompt; or NULL */
} lh_gated_grads;

/* Workspace bytes of lh_gated_backward; (size_t)-1 for invalid sizes. */
size_t lh_gated_backward_workspace_bytes(int64_t B, int64_t T, int64_t D);

/* Gradients of lh_gated_prefill.  workspace as there. */
lh_status lh_gated_backward(const lh_gated_inputs* in, const lh_gated_grads* grads,
                            void* workspace, size_t workspace_bytes, void* stream);

/*
 * Embedding: y[k] = scale W[ids[k]], in float32, rounded once.
 *
 *   W      : [V, D] (table_dtype);  ids : [n] int32
 *   y      : out [n, D] (io_dtype)
 *   n >= 0, V >= 1, D >= 1; n and V < 2^31; each type LH_F32 or LH_BF16
 * An id outside [0, V) gives a row of zeros.  One kernel launch; no workspace.
 */
lh_status lh_embed(const void* W, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                   lh_dtype table_dtype, lh_dtype io_dtype, float scale, void* y, void* stream);

/* Workspace bytes of lh_embed_backward; (size_t)-1 for invalid sizes.  Each array in it begins
 * on a border of 256 bytes: four of 4 n bytes; above 8192 tokens the counts of the sort, up
 * to 256 KiB; and 8 D bytes for each 16 tokens or part of them (64, above 8192 tokens). */
size_t lh_embed_backward_workspace_bytes(int64_t n, int64_t V, int64_t D);

/*
 * The table's gradient: dW[v] = scale sum over k with ids[k] = v of dy[k], the tokens sorted
 * by id and added in a fixed order.
 *
 *   dy         : [n, D] (io_dtype);  dW : out [V, D] float32
 *   accumulate : dW is added to (rows without a token are not touched); else every row is
 *                written
 * Ids outside [0, V) take no part.  The same inputs give the same bits; other tokens beside a
 * row's may group its sum otherwise.  workspace as in lh_gated_prefill.  A launch holds fewer
 * than 2^32 threads: n is below 2^28 for D <= 1024, below 2^27 for D <= 2048, and so on.
 */
lh_status lh_embed_backward(const void* dy, const int32_t* ids, int64_t n, int64_t V, int64_t D,
                            lh_dtype io_dtype, float scale, int accumulate, float* dW,
                            void* workspace, size_t workspace_bytes, void* stream);

/* Largest number of a teacher's logits per row. */
#define LH_DISTILL_MAX_TOP 1024

/* Workspace bytes of lh_distill_logits, at present 0; (size_t)-1 for invalid sizes. */
size_t lh_distill_logits_workspace_bytes(int64_t rows, int64_t V, int64_t K);

/*
 * Distillation from a teacher's top logits.  Per row, with t = values / tau over the slots
 * k whose id is in [0, V) and whose value is not -infinity, and x = logits / tau:
 *
 *   p = softmax(t),  q = softmax(x)
 *   loss = scale tau^2 sum_k p_k (log p_k - log q[id_k])
 *   dlogits[j] = scale tau (q[j] - sum of p_k with id_k = j)
 *   lse = log sum_j exp(x_j)
 *
 * (an id given twice counts twice).  A row without such a slot, or whose scale is 0, has
 * loss and gradient 0 and its logits are not read (the memory must be accessible all the
 * same); its lse is 0.  A row whose logits are all -infinity has q = 0.  The sums are float32,
 * and the loss is a difference of logarithms: it is off by some 2^-20 scale tau^2, which is
 * much of it where tau is large and p near q.
 *
 *   logits  : [rows, V] (io_dtype), rows ld_logits apart
 *   values  : [rows, K] float32;  ids : [rows, K] int32
 *   scale   : [rows] float32, or NULL (1)
 *   rows >= 0, V >= 1, 1 <= K <= LH_DISTILL_MAX_TOP, 2^-60 <= tau <= 2^60; V < 2^31
 *   loss    : out [rows] float32
 *   lse     : out [rows] float32, which lh_distill_logits_backward takes; or NULL
 *   dlogits : out [rows, V] (io_dtype), rows ld_dlogits apart, the gradient of the sum of
 *             the losses; or NULL.  It may be the buffer of logits (with the same ld).
 *   workspace as in lh_gated_prefill
 * One kernel launch.
 */
lh_status lh_distill_logits(const void* logits, int64_t ld_logits, const float* values,
                            const int32_t* ids, const float* scale, int64_t rows, int64_t V,
                            int64_t K, lh_dtype io_dtype, float tau, float* loss, float* lse,
                            void* dlogits, int64_t ld_dlogits, void* workspace,
                            size_t workspace_bytes, void* stream);

/* The gradient for an upstream gradient dloss [rows] (float32) of the losses: dlogits of
 * lh_distill_logits times dloss, from its lse.  Where |lse| > 16 its rounding would count
 * for more than that of the exponentials: there the row's sum is formed again, and lse only
 * says so.  One kernel launch; no workspace. */
lh_status lh_distill_logits_backward(const float* dloss, const void* logits, int64_t ld_logits,
                                     const float* values, const int32_t* ids, const float* scale,
                                     const float* lse, int64_t rows, int64_t V, int64_t K,
                                     lh_dtype io_dtype, float tau, void* dlogits,
                                     int64_t ld_dlogits, void* stream);

/* Largest number of drafted tokens per row. */
#define LH_VERIFY_MAX_DRAFT 64

/* Workspace bytes of lh_verify_draft; (size_t)-1 for invalid sizes. */
size_t lh_verify_draft_workspace_bytes(int64_t B, int64_t K, int64_t V);

/*
 * Verification of drafted tokens: tokens distributed as the target's, of which as many of
 * the drafted ones as the given random numbers accept.  Row b has n = lengths[b] drafted
 * tokens t_0 .. t_(n-1) (n outside [0, K] is taken as the nearer end), drawn from q_i =
 * draft_p[b, i]; p_i = target_p[b, i] are the target's probabilities after i of them.
 *
 *   token i is accepted while u[b,i] q_i(t_i) < p_i(t_i);  m = the first that is not, or n
 *   w = max(p_m - q_m, 0) where m < n, p_n where m = n
 *   next token = the lowest j with  w_0 + ... + w_j > u_last[b] (w_0 + ... + w_(V-1))
 *
 * Differences and sums are float64.  A drafted token outside [0, V) is not accepted (and
 * with draft_p = NULL takes nothing from w).  Entries of w that are negative or NaN count
 * as 0; where nothing of w is left, w = p_m; where nothing of that is left either, the next
 * token is -1.  Probabilities need not sum to 1; they must be finite.
 *
 *   drafted  : [B, K] int32;  lengths : [B] int32 or NULL (K)
 *   draft_p  : [B, K, V] (io_dtype), rows ld_draft apart; NULL: the draft is certain of its
 *              tokens (q_i is 1 at t_i and 0 elsewhere)
 *   target_p : [B, K + 1, V] (io_dtype), rows ld_target apart
 *   u        : [B, K] float32;  u_last : [B] float32, in [0, 1)
 *   B >= 1, 1 <= K <= LH_VERIFY_MAX_DRAFT, V >= 1; V < 2^31
 *   accepted : out [B] int32, m
 *   tokens   : out [B, K + 1] int32: the m accepted tokens, the next token, then -1
 *   workspace as in lh_gated_prefill
 */
lh_status lh_verify_draft(const int32_t* drafted, const int32_t* lengths, const void* draft_p,
                          int64_t ld_draft, const void* target_p, int64_t ld_target,
                          const float* u, const float* u_last, int64_t B, int64_t K, int64_t V,
                          lh_dtype io_dtype, int32_t* accepted, int32_t* tokens, void* workspace,
                          size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LH_H */
