/*
 * lordba.h -- C ABI of the B200 (sm_100a) LoRDBA adapter-forward library.
 *
 * The library evaluates the unmerged low-rank double-binary adapter branch
 *
 *     y[t,:] += s_out * ( B_sign ( s_r * ( A_sign ( s_in * x[t,:] ) ) ) )      t < T
 *
 * i.e. the paper's Delta-W(theta) = D_alpha B1 D_beta B2 D_gamma (Def. 1, Eq. 4,
 * canonical l = 1) applied in the evaluation order of Eq. 8 with both binary
 * products done as the sign accumulation of Eq. 9, and added to the buffer that
 * already holds the frozen base projection's output (Eq. 2).
 *
 *     paper              here
 *     N, M, R            d_in, d_out, r
 *     B1 (N x R)         A_sign = B1^T   (r x d_in,   +-1)
 *     B2 (R x M)         B_sign = B2^T   (d_out x r,  +-1)
 *     alpha, beta, gamma s_in (d_in), s_r (r), s_out (d_out), float32
 *     X (T x N)          x, row-major, one token per row
 *
 * The paper's Def. 1 carries no scalar LoRA alpha/r factor; a caller that has
 * one multiplies it into s_r.
 *
 * Conventions for every entry point
 *   - Pointers marked [device] are caller-owned device memory of the current
 *     CUDA device; [host] pointers are ordinary host memory.  The library keeps
 *     no pointer after a call returns.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the legacy default
 *     stream).  Calls enqueue work on it and return without synchronising,
 *     except where stated.
 *   - Return value: a lordba_status.  Argument errors are detected on the host
 *     and nothing is launched.  There is no CPU fallback: without a usable CUDA
 *     device the calls return LORDBA_ECUDA.
 *   - Supported rank: 1 <= r <= 64.  A call takes at most LORDBA_MAX_PROJS projections
 *     (LORDBA_EUNSUPPORTED beyond that).
 *   - No entry point allocates host or device memory.
 *
 * Bit-packed carriers (the paper says only "bit-packed"; this layout is the
 * library's own).  Bit 1 <=> +1, bit 0 <=> -1, 32-bit little-endian words,
 * pad bits are 0:
 *   role 0, A carrier (r x d_in): the columns are cut into blocks of 64; block b
 *       holds r consecutive 64-bit groups, one per row k, each stored as two
 *       words (low word first).  Entry (k,i) is bit (i mod 32) of word
 *       ((i/64)*r + k)*2 + (i mod 64)/32; ceil(d_in/64)*r*2 words.  (One block is
 *       exactly what the kernels need next to one 64-column tile of x.)
 *   role 1, B carrier (d_out x r): one dense bit stream of the row-major
 *       matrix; entry (j,k) is bit (b mod 32) of word b/32 with b = j*r + k.
 */
#ifndef LORDBA_H_
#define LORDBA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define LORDBA_MAX_PROJS 4096

typedef enum {
    LORDBA_F32 = 0,   /* x and y are float32                                   */
    LORDBA_BF16 = 1,  /* x and y are bfloat16; all accumulation is in float32  */
    LORDBA_F16 = 2    /* x and y are IEEE half (the precision the method exports its adapters in:
                         Sec. "Training and export", fp16 scales and activations); accumulation
                         in float32.  s_in is used as a pair of halves here: |s_in| must stay below
                         65504, and entries below 2^-14 are used with fewer than 22 bits */
} lordba_dtype;

typedef enum {
    LORDBA_OK = 0,
    LORDBA_EINVAL = 1,        /* null pointer, negative size, ld < width, x aliases y ...   */
    LORDBA_EUNSUPPORTED = 2,  /* rank outside 1..64, unknown dtype / role / variant         */
    LORDBA_EALIGN = 3,        /* a pointer is not aligned to its element type               */
    LORDBA_ECUDA = 4,         /* a CUDA runtime call or the launch failed                   */
    LORDBA_ETIMEOUT = 5,      /* a bounded device-side wait gave up (see lordba_device_status) */
    LORDBA_ETOOLARGE = 6      /* the call needs more than the library's built-in scratch buffer */
} lordba_status;

/* Kernel families the forward entry points can be pinned to (default AUTO). */
typedef enum {
    LORDBA_VARIANT_AUTO = 0,  /* the library's choice: streaming kernel where the shape allows  */
                              /* it; tcgen05 kernel for rank (x envelopes) > 16 once a call has */
                              /* enough 128-token tiles (> 32: 32 tiles, else eight per SM), and */
                              /* for widths that are not multiples of 64 from 128 tokens up     */
                              /* (rank a multiple of 8); else FMA.  lordba_query_variant tells  */
                              /* which one a given call gets                                   */
    LORDBA_VARIANT_FMA = 1,   /* CUDA-core float32 FMA kernel (always used for LORDBA_F32)  */
    LORDBA_VARIANT_TC = 2,    /* tcgen05/TMA cluster kernel; LORDBA_EUNSUPPORTED if the     */
                              /* shape or alignment rules it out                            */
    LORDBA_VARIANT_MMA = 3    /* TMA-fed streaming mma.sync kernel; LORDBA_EUNSUPPORTED if   */
                              /* the shape or alignment rules it out                        */
} lordba_variant;

/* One adapted projection for the _ex and _batched entry points.  ldx / ldy are
 * row pitches in elements (ldx >= d_in, ldy >= d_out).  Elements of y behind a row's d_out are not written. */
typedef struct lordba_proj {
    const void     *x;          /* [device] T x d_in,  pitch ldx                */
    const uint32_t *packed_A;   /* [device] role-0 words of A_sign (r x d_in)   */
    const uint32_t *packed_B;   /* [device] role-1 words of B_sign (d_out x r)  */
    const float    *s_in;       /* [device] d_in                                */
    const float    *s_r;        /* [device] r                                   */
    const float    *s_out;      /* [device] d_out                               */
    void           *y;          /* [device] T x d_out, pitch ldy, updated in place */
    int64_t d_in, d_out, ldx, ldy;
    int32_t r;
    int32_t flags;              /* LORDBA_PROJ_OVERLAP, _X_READY, _SCALES_F16, LORDBA_PROJ_ELL(ell); other bits 0 */
} lordba_proj;

/*
 * Multi-envelope adapters (Def. 1 / Eq. 4 with ell > 1): Delta-W is the sum of ell terms that
 * share the two sign carriers and differ in their scale triples.  A projection made with
 * LORDBA_PROJ_ELL(ell) in its flags, 1 <= ell <= LORDBA_MAX_ELL, takes s_in as ell x d_in,
 * s_r as ell x r and s_out as ell x d_out (row-major, envelope e in row e), and the call adds
 *     sum_e  s_out[e] * ( B_sign ( s_r[e] * ( A_sign ( s_in[e] * x[t,:] ) ) ) )
 * to y[t,:] with one rounding.  Flags without this field mean ell = 1.  Every envelope count at
 * every rank runs on the tensor cores (streaming kernel; two envelopes with ell * r <= 64 also
 * in the tcgen05 kernel, which the library takes for them by the same rule as for one envelope
 * of rank ell * r); the cost is about that of one envelope at rank ell * r.
 */
#define LORDBA_MAX_ELL 8
#define LORDBA_PROJ_ELL(ell) ((((ell) - 1) & 0xf) << 8)

/*
 * lordba_proj.flags: a promise by the caller that lets consecutive calls overlap on the GPU.
 * A call (all of its projections) made with LORDBA_PROJ_OVERLAP may start while the library
 * calls before it on the same stream are still running, back to and including the most recent
 * call made WITHOUT the flag.  The caller guarantees that, within such a run of calls, no call
 * reads what another one writes (a y buffer) and no call writes what another one reads or
 * writes, and that nothing else was enqueued on the stream in between.  Example: the q, k and v
 * adapters of one layer read the same x and update three different y buffers; the first is
 * called without the flag (it must see the kernel that produced x), the other two with it.
 * Work enqueued after the run is ordered after all of it, as usual.  Only the streaming
 * kernel acts on the flag; elsewhere it is accepted and ignored.
 */
#define LORDBA_PROJ_OVERLAP 1

/*
 * lordba_proj.flags: a weaker promise for a call that does depend on its predecessor, as an
 * adapter call does that follows the base projection which produced y (Eq. 2: y = W x, then
 * y += Delta-W x).  With LORDBA_PROJ_X_READY on every projection of a call made WITHOUT
 * LORDBA_PROJ_OVERLAP the caller guarantees that x, the packed carriers and the three scale
 * vectors were final before the previous piece of work on the stream began (the base projection
 * reads x itself, so this is the normal case); only y may still be in the making.  The call then
 * requests x and runs the first product (Eq. 8, u = A_sign (s_in * x)) while its predecessor
 * finishes, and touches y only once the predecessor is complete.  Only the streaming kernel acts
 * on the flag; elsewhere, and together with LORDBA_PROJ_OVERLAP, it is accepted and ignored.
 */
#define LORDBA_PROJ_X_READY 4

/*
 * lordba_proj.flags: the caller states that every entry of s_in is exactly representable as an
 * IEEE half, which is the case for an adapter exported with fp16 scales (Section 3.2: the scales
 * are trained in float32 and leave training as halves) and widened by lordba_scales_from_f16.  With
 * LORDBA_F16 activations the streaming kernel then forms x * s_in in one tensor-core pass
 * instead of two; with a false statement the low bits of s_in beyond a half are ignored, nothing
 * else.  Other kernels and dtypes accept the flag and ignore it.
 */
#define LORDBA_PROJ_SCALES_F16 2

/*
 * Widens n IEEE-half scales (the storage format of an exported adapter, 2 bytes per scale as in
 * the method's footprint count, Eq. 5) to the float32 arrays that the forward calls take.  Once
 * per adapter, like packing.  src: [device] n halves, 2-byte aligned; dst: [device] n floats.
 * Exact (every half is a float).  Asynchronous on stream.  n = 0 is a no-op; n < 0 or a null
 * pointer with n > 0 is LORDBA_EINVAL.
 */
int lordba_scales_from_f16(const uint16_t *src, float *dst, int64_t n, void *stream);

/* Number of uint32 words of a packed carrier (layout above); -1 on bad arguments. */
int64_t lordba_packed_words(int64_t rows, int64_t cols, int role);

/*
 * Bit-pack a sign matrix: the two sign carriers are kept as one bit per entry and packed
 * once per adapter (Section 3.3).  signs: [device] int8, rows x cols row-major; an entry < 0 packs
 * as -1, anything else (0 included: sign(0) = +1) as +1.  role 0: rows = r,
 * cols = d_in.  role 1: rows = d_out, cols = r.  packed: [device], at least
 * lordba_packed_words() words, fully overwritten (pad bits 0).
 */
int lordba_pack_signs(const int8_t *signs, int64_t rows, int64_t cols, int role,
                      uint32_t *packed, void *stream);

/* Inverse of lordba_pack_signs: writes +1 / -1 into signs [device] (rows x cols). */
int lordba_unpack_signs(const uint32_t *packed, int64_t rows, int64_t cols, int role,
                        int8_t *signs, void *stream);

/*
 * Adapter forward, Eq. 8 / Eq. 9, bfloat16 activations, dense rows
 * (ldx = d_in, ldy = d_out).  All pointers [device].  y is read, the adapter
 * term is added in float32 and the sum is rounded once to bfloat16.  x and y
 * must not overlap.  T = 0 is a no-op.
 */
int lordba_adapter_forward(const void *x, const uint32_t *packed_A, const uint32_t *packed_B,
                           const float *s_in, const float *s_r, const float *s_out, void *y,
                           int64_t T, int64_t d_in, int64_t d_out, int r, void *stream);

/* Same operation with float32 x and y (float32 arithmetic throughout). */
int lordba_adapter_forward_f32(const float *x, const uint32_t *packed_A, const uint32_t *packed_B,
                               const float *s_in, const float *s_r, const float *s_out, float *y,
                               int64_t T, int64_t d_in, int64_t d_out, int r, void *stream);

/*
 * Multi-envelope form of the two calls above (Eq. 4, ell >= 1), dense rows: s_in is ell x d_in,
 * s_r ell x r, s_out ell x d_out.  dtype: LORDBA_BF16, LORDBA_F16 or LORDBA_F32.
 */
int lordba_adapter_forward_ell(const void *x, const uint32_t *packed_A, const uint32_t *packed_B,
                               const float *s_in, const float *s_r, const float *s_out, void *y,
                               int64_t T, int64_t d_in, int64_t d_out, int r, int ell, int dtype,
                               void *stream);

/* Same operation with explicit row pitches and dtype.  p: [host]. */
int lordba_adapter_forward_ex(const lordba_proj *p, int64_t T, int dtype, void *stream);

/*
 * The adapter forward of n_proj projections that share T and dtype (for
 * instance the seven adapted projections q,k,v,o,gate,up,down of one decoder
 * layer, Section 5 Setup) in as few launches as the kernel-parameter space
 * allows.  projs: [host] array, read before the call returns.  The projections
 * are treated as simultaneous: their y buffers must be pairwise disjoint and no
 * projection's x may overlap any projection's y (LORDBA_EINVAL otherwise); the
 * launches of one call may therefore overlap on the GPU.
 */
int lordba_adapter_forward_batched(const lordba_proj *projs, int n_proj, int64_t T, int dtype,
                                   void *stream);

/*
 * Multi-adapter batch (Section 2, adapter-mode deployment, condition A4: many task adapters
 * served over one frozen base): segment i is tokens[i] consecutive token rows that go through their own adapter.
 * segs[i].x / .y point at the segment's first row (usually into one shared x / y matrix),
 * the other fields name the segment's adapter; several segments may share an adapter.
 * segs, tokens: [host] arrays of n_seg entries, read before the call returns.  Segments are
 * treated as simultaneous (same disjointness rules as the batched call); empty segments are
 * skipped.  One launch per 24 segments of equal padded rank (per 96 on the tcgen05 kernel).
 */
int lordba_adapter_forward_segments(const lordba_proj *segs, const int64_t *tokens, int n_seg, int dtype,
                                    void *stream);

/*
 * Host-buffer form of lordba_adapter_forward{,_f32}: x_host and y_host are
 * [host] (pinned memory makes the copies asynchronous), dense rows; the carriers
 * and scales stay [device] because they are loaded once per adapter.
 * workspace: [device], at least lordba_host_workspace_bytes() bytes, 256-byte
 * aligned.  Enqueues H2D(x), H2D(y), the forward kernel and D2H(y) on `stream`;
 * y_host is valid once the stream has been synchronised.
 */
size_t lordba_host_workspace_bytes(int64_t T, int64_t d_in, int64_t d_out, int dtype);
int lordba_adapter_forward_host(const void *x_host, const uint32_t *packed_A,
                                const uint32_t *packed_B, const float *s_in, const float *s_r,
                                const float *s_out, void *y_host, int64_t T, int64_t d_in,
                                int64_t d_out, int r, int dtype, void *workspace,
                                size_t workspace_bytes, void *stream);

/*
 * lordba_adapter_forward_host without a caller-supplied workspace (an addition of this library;
 * the paper has no counterpart).
 *
 * For callers that have host activations but are not in a position to obtain device memory: code
 * that runs where cudaMalloc is off limits (inside a latency-critical loop, since an allocation
 * can synchronise the whole device; under a host framework that owns all device memory and hands
 * none to plug-ins; in a process whose memory budget was fixed at start-up).  The device staging
 * area for x and y is a buffer of LORDBA_STATIC_SCRATCH_BYTES that is part of the library image:
 * every GPU on which the library is loaded holds it until the process exits, and this call
 * allocates nothing and frees nothing.
 *
 *   - Same arguments, order of work and result as lordba_adapter_forward_host, minus the
 *     workspace.  If lordba_host_workspace_bytes(T, d_in, d_out, dtype) exceeds
 *     LORDBA_STATIC_SCRATCH_BYTES the call returns LORDBA_ETOOLARGE and does nothing.
 *   - The first call on a device looks up the buffer's device address (with that device current)
 *     and remembers it.  If nothing of the library has run on that device yet, this lookup is
 *     also the moment at which the CUDA runtime loads the library's device code there, which
 *     reserves the buffer and may synchronise the device: make that first call at start-up,
 *     outside any stream capture and outside latency-critical code.
 *   - All calls on a device share the one buffer.  It still holds the previous call's x and y;
 *     nothing in it has to start at zero, because every byte that is read was copied in by the
 *     same call first.  Two calls whose work overlaps on the GPU (different streams, no
 *     ordering between them) would overwrite each other's staging data: order them.
 */
#define LORDBA_STATIC_SCRATCH_BYTES (8u << 20)
int lordba_adapter_forward_host_static(const void *x_host, const uint32_t *packed_A,
                                       const uint32_t *packed_B, const float *s_in, const float *s_r,
                                       const float *s_out, void *y_host, int64_t T, int64_t d_in,
                                       int64_t d_out, int r, int dtype, void *stream);

/*
 * Which kernel family a call would run each projection on, without launching anything: the
 * answer of lordba_adapter_forward_batched (tokens == NULL: every projection has T rows) or of
 * lordba_adapter_forward_segments (tokens[i] rows each) for the same arguments and the current
 * lordba_set_variant setting.  variants: [host] n_proj entries, each set to LORDBA_VARIANT_FMA,
 * _TC or _MMA (0 for a projection without rows).  The CUDA-core kernel (FMA) takes every shape but
 * runs an order of magnitude below the tensor-core kernels, which want bf16 / float16 activations,
 * d_in and d_out multiples of 64, row pitches multiples of 8 elements and 16-byte aligned x, y,
 * scales and carriers: a caller can see that fallback coming here.  Returns the status the call
 * itself would return for bad arguments.
 */
int lordba_query_variant(const lordba_proj *projs, int n_proj, int64_t T, const int64_t *tokens, int dtype,
                         int *variants);

/*
 * Prepared calls.  Every forward call builds its launch parameters on the host first (tensor maps
 * for the copy engine, six per projection in the streaming kernel).  A caller that repeats a call
 * with the same pointers and sizes (a layer's adapters over fixed activation buffers, step after
 * step) can have that done once:
 *
 *   lordba_plan_bytes   the storage a plan for these arguments needs (0 on bad arguments);
 *   lordba_plan_init    validates the arguments exactly like lordba_adapter_forward_batched
 *                       (tokens == NULL) or lordba_adapter_forward_segments (tokens given), chooses
 *                       the kernels and writes the prepared launches into plan: [host], 64-byte
 *                       aligned, caller-owned, plan_bytes long (LORDBA_ETOOLARGE if too short).
 *                       Nothing is launched;
 *   lordba_adapter_forward_planned   enqueues the prepared launches on stream: the same kernels
 *                       with the same arguments as the unprepared call.
 *
 * A plan holds device addresses: it belongs to the device that was current at lordba_plan_init
 * (LORDBA_EINVAL on another one), stays valid while the buffers it names are, and may be replayed
 * any number of times, from any stream; it holds no resources and needs no release.
 * LORDBA_PROJ_OVERLAP and LORDBA_PROJ_X_READY in the projections' flags are part of the plan.
 */
size_t lordba_plan_bytes(const lordba_proj *projs, int n_proj, int64_t T, const int64_t *tokens, int dtype);
int lordba_plan_init(void *plan, size_t plan_bytes, const lordba_proj *projs, int n_proj, int64_t T,
                     const int64_t *tokens, int dtype);
int lordba_adapter_forward_planned(const void *plan, void *stream);
/* Kernel launches a plan holds (-1 if plan is not a plan). */
int lordba_plan_launches(const void *plan);

/*
 * Closed-form scale updates of the adapter fit (Appendix "Closed-form scale updates for
 * PTQ-LoRDBA"; the scale step Eq. scales-step of the PTQ-LoRDBA iteration, and the sweep that
 * initialises the scales after the SVD warm start, Eq. svd-init).  With the packed carriers held
 * fixed, `sweeps` block-coordinate sweeps of
 *
 *     min  1/2 || target - diag(s_in) A_sign^T diag(s_r) B_sign^T diag(s_out) ||_F^2
 *
 * each sweep updating s_in (Eq. alpha-update: one scalar least squares per row of the target), then
 * s_r (Eq. beta-gram and Eq. beta-pinv: the r x r normal equations G = (P^T P) o (Q Q^T), solved
 * by the Moore-Penrose pseudo-inverse, eigenvalues below r * 2^-52 * lambda_max dropped), then
 * s_out (Eq. gamma-update: one scalar least squares per column); a row or column whose model is
 * identically zero gets 0.  axes: which of the three a sweep updates (LORDBA_FIT_ALPHA | _BETA |
 * _GAMMA; LORDBA_FIT_ALL for the full sweep), always in that order.
 *
 * target: [device] float32, d_in x d_out row-major with row pitch ld >= d_out elements (the dense
 * adapter Delta-W* that is being fitted, in the orientation y = x Delta-W); read only.  packed_A,
 * packed_B: the carriers as lordba_pack_signs makes them.  s_in (d_in), s_r (r), s_out (d_out):
 * [device] float32, read as the starting point and overwritten with the result.  workspace:
 * [device], 256-byte aligned, at least lordba_fit_workspace_bytes() bytes (LORDBA_EINVAL if
 * shorter); its contents need not be initialised and are not meaningful afterwards.  The passes
 * over the target accumulate in float32, everything of size r x r and the quotients in float64;
 * results are deterministic.  Asynchronous on stream; sweeps = 0 is a no-op.
 */
#define LORDBA_FIT_ALPHA 1
#define LORDBA_FIT_BETA 2
#define LORDBA_FIT_GAMMA 4
#define LORDBA_FIT_ALL 7
size_t lordba_fit_workspace_bytes(int64_t d_in, int64_t d_out, int r);
int lordba_fit_scales(const float *target, int64_t ld, const uint32_t *packed_A, const uint32_t *packed_B,
                      float *s_in, float *s_r, float *s_out, int64_t d_in, int64_t d_out, int r, int sweeps,
                      int axes, void *workspace, size_t workspace_bytes, void *stream);

/*
 * ---- The frozen base projection in 8-bit integers ------------------------------------------------
 *
 * y[t,n] = s_x[t] * s_w[n] * sum_k x[t,k] w[n,k]: x holds a token's activations as integers with one
 * scale a token, w a weight matrix (d_out x d_in row-major, the contraction contiguous) with one scale
 * an output channel.  The sum is exact in 32-bit integers (d_in <= LORDBA_INT8_MAX_DIN, all values
 * -128 ... 127 allowed); float32(sum) * s_x * s_w is rounded once to the type of y.  y is overwritten:
 * this is the base output of Eq. 2, to which the adapter forward then adds its term.
 *
 * lordba_int8_quantize_rows makes x and s_x from activations: s_x[t] = max_k |x[t,k]| / 127 and
 * q = rint(x * (127 / max)), ties to even.  A row whose largest magnitude is below 2^-120 (zero rows
 * among them) becomes zeros with scale 0; a row that holds an infinity or a NaN becomes zeros with
 * scale NaN, so that its outputs are NaN and no other row's are touched.
 *
 * The gradient to x of a frozen projection is the same product with w transposed (laid out once) and
 * dy * s_w quantised per token.
 *
 * dtype: the type of y (and of the activations that are quantised): LORDBA_BF16, LORDBA_F16 or
 * LORDBA_F32.  Any sizes, pitches and alignments are taken; operands whose base or pitch is not a
 * multiple of 16 bytes cost more time and may be copied into the workspace first.  T = 0 is a no-op.
 */
#define LORDBA_INT8_MAX_DIN 131071
typedef struct lordba_int8_proj {
    const int8_t *x;            /* [device] T x d_in, pitch ldx                 */
    const float  *s_x;          /* [device] T                                   */
    const int8_t *w;            /* [device] d_out x d_in, pitch ldw             */
    const float  *s_w;          /* [device] d_out                               */
    void         *y;            /* [device] T x d_out, pitch ldy, overwritten   */
    int64_t d_in, d_out, ldx, ldw, ldy;      /* pitches in elements              */
} lordba_int8_proj;

int lordba_int8_quantize_rows(const void *x, int64_t ldx, int8_t *q, int64_t ldq, float *scale, int64_t T,
                              int64_t d, int dtype, void *stream);
/* Bytes of workspace the call needs: [device], 256-byte aligned; 0 for most calls (the workspace may then be
 * NULL), not 0 where operands are copied or a long sum with few results is split and joined.  LORDBA_EINVAL
 * from the call when the workspace given is shorter.
 *
 * The answer holds for the very call: the query wants the struct as the call will get it, every pointer (NULL counts as
 * aligned, and what is NULL is not made) and every pitch, with the same current device.  Another slice of the same
 * shape may need another size, because alignment decides on copies and on the kernel.  This goes for the queries of
 * lordba_gated_forward and lordba_gated_backward too. */
size_t lordba_int8_linear_workspace_bytes(const lordba_int8_proj *p, int64_t T);
int lordba_int8_linear(const lordba_int8_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes,
                       void *stream);

/*
 * ---- The gated feed-forward block -----------------------------------------------------------------
 *
 *     g = x w_gate^T + gate_add        u = x w_up^T + up_add        h = act(g) * u
 *
 * both projections, the activation and the product in one kernel.  x is T x d_in, w_gate and w_up are
 * d_hidden x d_in (contraction contiguous), h is T x d_hidden.  gate_add / up_add (both or neither) are
 * added to the sums in float32: the terms that the adapters of the two projections put into zeroed
 * buffers.  gate / up (both or neither) receive g and u rounded once, which is what the backward pass
 * takes; they may be the buffers of gate_add / up_add.  h is computed from the unrounded g and u.
 *
 * act: LORDBA_ACT_SILU  act(g) = g s(g), s the logistic function;
 *      LORDBA_ACT_GELU_TANH  act(g) = g (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2.
 *
 * dtype: LORDBA_BF16 or LORDBA_F16, the type of every matrix.  With LORDBA_GATED_INT8 in flags x, w_gate
 * and w_up are int8 and s_x (T), s_gate, s_up (d_hidden) their scales, as in lordba_int8_linear; dtype is
 * then the type of the other matrices.  LORDBA_F32 is LORDBA_EUNSUPPORTED.  Workspace as above.
 */
typedef enum { LORDBA_ACT_SILU = 0, LORDBA_ACT_GELU_TANH = 1 } lordba_activation;
#define LORDBA_GATED_INT8 1
typedef struct lordba_gated {
    const void  *x, *w_gate, *w_up;          /* [device] pitches ldx, ldw, ldw                        */
    const float *s_x, *s_gate, *s_up;        /* [device] scales, LORDBA_GATED_INT8 only, else NULL    */
    const void  *gate_add, *up_add;          /* [device] T x d_hidden, pitch ld_add, or both NULL     */
    void        *gate, *up;                  /* [device] T x d_hidden, pitch ld_pre, or both NULL     */
    void        *h;                          /* [device] T x d_hidden, pitch ldh                      */
    int64_t d_in, d_hidden, ldx, ldw, ld_add, ld_pre, ldh;
    int32_t act, flags;
} lordba_gated;

size_t lordba_gated_workspace_bytes(const lordba_gated *g, int64_t T);
int lordba_gated_forward(const lordba_gated *g, int64_t T, int dtype, void *workspace, size_t workspace_bytes,
                         void *stream);

/*
 * Backward pass of lordba_gated_forward from the gradient dh of h and the stored gate / up:
 *
 *     dgate = dh * up * act'(gate)           dup = dh * act(gate)
 *     dx = dgate w_gate + dup w_up           dw_gate = dgate^T x       dw_up = dup^T x
 *
 * dgate and dup (T x d_hidden) are always written: they are the gradients of gate_add and up_add, where
 * the adapters' own gradients start.  dx is skipped when its pointer is NULL (w_gate and w_up are then
 * not read), dw_gate / dw_up when both of theirs are (x is then not read).  Every sum is float32.  dgate
 * and dup enter the products in the matrices' type, because that is what the tensor cores take: as written
 * for more than 64 tokens, with the rest that their rounding left as a second term up to there (where it
 * costs nothing; dx of more than 65535 * 128 columns goes without).  The result is the same from run to run.  T = 0 writes zeros into dw_gate and dw_up.
 * dtype: LORDBA_BF16 or LORDBA_F16.
 */
typedef struct lordba_gated_grad {
    const void *dh, *gate, *up;              /* [device] T x d_hidden, pitches ld_dh, ld_pre, ld_pre  */
    const void *x;                           /* [device] T x d_in, pitch ldx                          */
    const void *w_gate, *w_up;               /* [device] d_hidden x d_in, pitch ldw                   */
    void       *dgate, *dup;                 /* [device] T x d_hidden, pitch ld_dpre                  */
    void       *dx;                          /* [device] T x d_in, pitch ld_dx, or NULL               */
    void       *dw_gate, *dw_up;             /* [device] d_hidden x d_in, pitch ld_dw, or both NULL   */
    int64_t d_in, d_hidden, ld_dh, ld_pre, ldx, ldw, ld_dpre, ld_dx, ld_dw;
    int32_t act, flags;                      /* flags: 0                                              */
} lordba_gated_grad;

size_t lordba_gated_backward_workspace_bytes(const lordba_gated_grad *g, int64_t T);
int lordba_gated_backward(const lordba_gated_grad *g, int64_t T, int dtype, void *workspace, size_t workspace_bytes,
                          void *stream);

/*
 * ---- Dropout --------------------------------------------------------------------------------------
 *
 * out[t,c] = residual[t,c] + (keep(t,c) ? x[t,c] * 65536 / (65536 - n) : 0),  n = rint(65536 p)
 *
 * keep is a function of (t, c, seed, offset) alone and is never stored: the sixteen-bit number of
 * element (t,c) is at least n.  The numbers are those of Philox4x32-10 (Salmon, Moraes, Dror and Shaw, SC
 * 2011) with key (seed low, seed high) and counter (c / 8, t, offset low, offset high): the 128-bit
 * output holds the numbers of columns 8 (c/8) ... 8 (c/8) + 7, lowest bits first.  So the backward pass is
 * the same call on the gradient (residual NULL), whatever the pitches.  0 <= p <= 1; the probability is
 * taken to the nearest 1/65536.  A dropped element contributes an exact zero, also where x is not finite.
 *
 * residual may be NULL; out may be x or residual (same pitch), nothing else may overlap it.  dtype: all
 * three matrices.  T < 2^32, d < 2^34.  One rounding, of the sum.  T = 0 is a no-op.
 */
int lordba_dropout(const void *x, int64_t ldx, const void *residual, int64_t ldr, void *out, int64_t ldo, int64_t T,
                   int64_t d, float p, uint64_t seed, uint64_t offset, int dtype, void *stream);

/*
 * ---- The frozen base projection in 4-bit integers with group scales --------------------------------
 *
 * w[n,k] = scale[n, k/group] * (u[n,k] - zero[n, k/group]),  u = 0 ... 15, zero = 8 where it is NULL: a
 * weight matrix (d_out x d_in) of which `group` neighbouring columns of a row share a scale.
 *
 *     lordba_int4_linear             y[t,n]  = sum_k x[t,k] w[n,k]
 *     lordba_int4_linear_backward    dx[t,k] = sum_n dy[t,n] w[n,k]
 *
 * The first is a base output of Eq. 2 over a 4-bit base, to which the adapter forward adds its term; the
 * second is the gradient that the frozen projection hands down to its input.
 *
 * The carrier q: blocks of 128 columns, 64 bytes each, ceil(d_in / 128) blocks a row.  A block is sixteen
 * little-endian 32-bit words; word 4 t + j (t, j = 0 ... 3) holds columns 32 j + 8 t ... 32 j + 8 t + 7 of
 * the block, column c of these eight in bits 4 (c / 2) + 16 (c % 2) ... + 3.  So a 16-byte piece holds
 * every fourth run of eight columns, and a word masked with 0x000f000f << 4 i is a pair of neighbours.
 * What stands in columns from d_in on is not looked at.  q lies on a 16-byte boundary and its pitch is a
 * multiple of 16 bytes (LORDBA_EALIGN).
 *
 * group: a power of two, at least 32; a group of at least d_in columns is one scale a row.  scale and zero
 * are d_out x ceil(d_in / group), row-major with pitches of their own.  scale has the type of x and y; of
 * a zero's byte the low four bits count.
 *
 * dtype: LORDBA_BF16 or LORDBA_F16, the type of the activations, the results and the scales (LORDBA_F32 is
 * LORDBA_EUNSUPPORTED).  Every sum is float32, results are rounded once.  A forward call of few tokens
 * (now up to 32) multiplies the integers themselves (they are exact in 16 bits) and scales the sum of each
 * group; others multiply weights that were rounded to the type of x, because that is what the tensor cores
 * take (the error of y is then up to 1.4 times that of rounding y alone).  So a float16 weight beyond 65504 (a scale above 65504 / 15 can
 * make one) is infinite in gradients and for many tokens, as it is for lordba_int4_dequantize, though not for few.  A scale that is not
 * finite spoils its row of y (of dx: the columns of its group) and nothing else.  T = 0 is a no-op.
 */
typedef struct lordba_int4_proj {
    const void    *in;          /* [device] x, T x d_in  (backward: dy, T x d_out), pitch ld_in                  */
    void          *out;         /* [device] y, T x d_out (backward: dx, T x d_in), pitch ld_out, overwritten     */
    const uint8_t *q;           /* [device] carrier, d_out rows, pitch ldq bytes                                 */
    const void    *scale;       /* [device] d_out x groups, pitch ld_scale                                       */
    const uint8_t *zero;        /* [device] d_out x groups, pitch ld_zero, or NULL                               */
    int64_t d_in, d_out, ld_in, ld_out, ldq, ld_scale, ld_zero;
    int32_t group, flags;       /* flags: 0                                                                      */
} lordba_int4_proj;

/* Bytes of a row of the carrier: 64 for each 128 columns begun (-1 on a bad size). */
int64_t lordba_int4_row_bytes(int64_t d_in);

/* values (d_out x d_in bytes, of which the low four bits count) -> the carrier. */
int lordba_int4_pack(const uint8_t *values, int64_t ldv, uint8_t *q, int64_t ldq, int64_t d_out, int64_t d_in, void *stream);

/*
 * Weights -> carrier, scales and, where zero is not NULL, zeros; wdtype: the type of w, dtype that of scale
 * (LORDBA_BF16 or LORDBA_F16).  Of a group, in float32:
 *
 *     without zeros   scale = max |w| / 7               u = 8 + rint(w / scale)
 *     with zeros      scale = (max(w, 0) - min(w, 0)) / 15,  zero = rint(-min(w, 0) / scale),  u = zero + rint(w / scale)
 *
 * scale is rounded to its type first, zero and u are what the rounded scale gives (exact quotients, ties to
 * even), clamped to 0 ... 15.  A group whose scale rounds to zero gets u = 8 (zero = 8) throughout, and scale 0; one
 * that holds an infinity or a NaN, or whose scale overflows, the same with scale NaN.
 */
int lordba_int4_quantize(const void *w, int64_t ldw, int wdtype, uint8_t *q, int64_t ldq, void *scale, int64_t ld_scale,
                         uint8_t *zero, int64_t ld_zero, int64_t d_out, int64_t d_in, int group, int dtype, void *stream);

/* The weights that p's carrier, scales and zeros stand for, rounded to dtype: out is d_out x d_in, pitch ld_out (in is
 * not looked at).  A base's rest, which an adapter is fitted to, is the original less these. */
int lordba_int4_dequantize(const lordba_int4_proj *p, int dtype, void *stream);

/* Workspace as for lordba_int8_linear: the queries answer for the call with the very pointers and pitches. */
size_t lordba_int4_linear_workspace_bytes(const lordba_int4_proj *p, int64_t T);
int lordba_int4_linear(const lordba_int4_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream);
size_t lordba_int4_linear_backward_workspace_bytes(const lordba_int4_proj *p, int64_t T);
int lordba_int4_linear_backward(const lordba_int4_proj *p, int64_t T, int dtype, void *workspace, size_t workspace_bytes,
                                void *stream);

/*
 * ---- Norms of queries and keys, and the rotation by position -----------------------------------------
 *
 * What happens to the results of the query and key projections before attention, for every head vector x of
 * d entries (queries and keys in one launch):
 *
 *     n_i = x_i w_i / sqrt(mean_j x_j^2 + eps)                          (LORDBA_ROPE_NO_NORM: n = x)
 *     y_a = n_a cos(f) - n_b sin(f),  y_b = n_b cos(f) + n_a sin(f),    f = positions[t] * inv_freq[i]
 *
 * for the pairs (a, b) = (i, i + rotary/2), or (2 i, 2 i + 1) with LORDBA_ROPE_INTERLEAVED, i < rotary/2;
 * y = n from entry `rotary` on.  rotary = 0 is the norm alone.  The angle is the product of any 64-bit position and a frequency (up to
 * 16 in size) less its whole turns, good to 2^-40 of a turn.  Everything else is float32, y is rounded once.
 *
 * Tensors are [token][head][entry] with any distances between tokens and between heads and the entries
 * side by side (slices of a joint projection's output are read in place).  q_out may be q and k_out may be
 * k with the same distances; otherwise outputs meet nothing.  heads_k = 0: there are no keys, and
 * nothing of theirs is looked at.  w_q, w_k: d values of type w_dtype, or NULL for ones.  d <= LORDBA_ROPE_MAX_D.
 * dtype: all of q, k, q_out, k_out: LORDBA_BF16, LORDBA_F16 or LORDBA_F32.  T = 0 is a no-op.
 */
#define LORDBA_ROPE_MAX_D 512
#define LORDBA_ROPE_NO_NORM 1
#define LORDBA_ROPE_INTERLEAVED 2
typedef struct lordba_heads {           /* head vectors of T tokens; distances in entries */
    const void *p;
    int64_t token, head;
} lordba_heads;
typedef struct lordba_norm_rope_args {
    lordba_heads q, k, q_out, k_out;         /* [device]                                            */
    const void *w_q, *w_k;                   /* [device] d values of w_dtype, or NULL               */
    const int64_t *positions;                /* [device] T, may be negative                         */
    const float *inv_freq;                   /* [device] rotary/2                                   */
    int32_t heads_q, heads_k, d, rotary, w_dtype, flags;
    float eps;
} lordba_norm_rope_args;
int lordba_norm_rope(const lordba_norm_rope_args *a, int64_t T, int dtype, void *stream);

/*
 * Its backward pass: f.q, f.k are the inputs of the forward call, f.q_out, f.k_out the gradients of its
 * results (read), dq, dk receive the gradients of q and k, and dw_q, dw_k (float32, d values each, NULL where
 * not wanted) those of w_q and w_k, summed over all tokens and heads in a fixed order and overwritten.
 *
 *     g = the gradient turned back by -f,  r = 1 / sqrt(mean x^2 + eps)
 *     dw_i = sum g_i x_i r        dx = r (g w - x r^2 mean(g w x))       (without norm: dx = g)
 *
 * dq may be q or the gradient q_out (same distances), and dk likewise.  dw_q and dw_k need the norm (with
 * LORDBA_ROPE_NO_NORM they must be NULL).  The workspace holds the partial sums of dw: [device], 256-byte
 * aligned, 0 bytes where no dw is wanted.  T = 0 writes zeros into dw_q and dw_k.
 */
typedef struct lordba_norm_rope_grad_args {
    lordba_norm_rope_args f;
    lordba_heads dq, dk;
    float *dw_q, *dw_k;
} lordba_norm_rope_grad_args;
size_t lordba_norm_rope_backward_workspace_bytes(const lordba_norm_rope_grad_args *a, int64_t T);
int lordba_norm_rope_backward(const lordba_norm_rope_grad_args *a, int64_t T, int dtype, void *workspace, size_t workspace_bytes,
                              void *stream);

/*
 * ---- Distillation from a teacher's top logits ----------------------------------------------------------
 *
 * The loss that an adapter over a quantised base is trained with: the divergence of the student's
 * distribution over `vocab` classes from the teacher's, of which the `top` largest logits were kept.
 *
 *     p = softmax of the row's present teacher logits / temperature      lse[t] = log sum_i exp(logits[t,i] / temperature)
 *     loss[t] = weight[t] temperature^2 sum_j p_j (log p_j - logits[t, ids[t,j]] / temperature + lse[t])
 *     dlogits[t,i] = weight[t] temperature (exp(logits[t,i] / temperature - lse[t]) - sum over j with ids[t,j] = i of p_j)
 *
 * An entry is present where 0 <= ids[t,j] < vocab; an index may stand in a row more than once.  An entry
 * of teacher logit minus infinity has p = 0 and adds nothing, whatever the student's logit.  A row without
 * an entry of p > 0, and one of weight 0, has loss 0 and gradient 0, whatever stands in its logits.  A
 * student's logit of minus infinity, or of any number so low that its power is nothing beside the row's largest, has probability 0.
 * Sums and exponents are float32, and relative to the row's largest logit: loss and the gradient of lordba_distill_loss do not
 * depend on how far from zero a row lies.  lse is float32 too (infinite where logits / temperature pass its range), and the gradient made
 * from it is off by its rounding.
 *
 * lordba_distill_loss writes loss and lse and, where dlogits is not NULL, the gradient in the same pass
 * over the logits (the weights of the rows, such as 1 over the number of tokens, are then the gradients of
 * the losses).  lordba_distill_backward makes dlogits from lse and the gradients of the losses, which it takes
 * in `weight`; loss is not looked at.  weight may be NULL: ones.  dlogits may be logits (same pitch).
 *
 * dtype: logits and dlogits; teacher_dtype: teacher.  Each LORDBA_BF16, LORDBA_F16 or LORDBA_F32.  1 <= top <=
 * LORDBA_DISTILL_MAX_TOP.  temperature > 0.  T = 0 is a no-op.  The workspace (the same for both calls, 0 bytes for few
 * rows) holds the teacher's part of every row: [device], 256-byte aligned.
 */
#define LORDBA_DISTILL_MAX_TOP 256
#define LORDBA_DISTILL_IDS_64 1
typedef struct lordba_distill {
    const void  *logits;        /* [device] T x vocab, pitch ld_logits                                           */
    const void  *ids;           /* [device] T x top, pitch ld_ids: int32, or int64 with LORDBA_DISTILL_IDS_64    */
    const void  *teacher;       /* [device] T x top, pitch ld_teacher                                            */
    const float *weight;        /* [device] T, or NULL                                                           */
    float       *loss, *lse;    /* [device] T (lse is read by the backward call)                                 */
    void        *dlogits;       /* [device] T x vocab, pitch ld_dlogits, or NULL                                 */
    int64_t vocab, top, ld_logits, ld_ids, ld_teacher, ld_dlogits;
    float   temperature;
    int32_t teacher_dtype, flags;
} lordba_distill;
size_t lordba_distill_workspace_bytes(const lordba_distill *d, int64_t T);
int lordba_distill_loss(const lordba_distill *d, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream);
int lordba_distill_backward(const lordba_distill *d, int64_t T, int dtype, void *workspace, size_t workspace_bytes, void *stream);

/* Storage of one adapter in bits, Eq. 5: r(d_in+d_out) + 16 ell (d_in+r+d_out). */
int64_t lordba_adapter_bits(int64_t d_in, int64_t d_out, int r, int ell);

/* Pin the kernel family used by the forward entry points (process-wide). */
int lordba_set_variant(int variant);
int lordba_get_variant(void);

/*
 * Bounded device-side waits (TMA / MMA completion barriers) record a non-zero
 * code in a device status word instead of spinning forever.  This call
 * synchronises `stream`, copies the word to *code, clears it, and returns
 * LORDBA_ETIMEOUT if it was non-zero.
 */
int lordba_device_status(int *code, void *stream);

/* Kernels launched by this library in this process so far. */
int64_t lordba_launch_count(void);

const char *lordba_status_string(int status);
const char *lordba_version(void);

#ifdef __cplusplus
}
#endif
#endif /* LORDBA_H_ */
