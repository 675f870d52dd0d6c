/*
 * scanweaver.h -- C ABI of libscanweaver.so, the MI355X (gfx950) library for
 * the forward affine recurrence and the Mamba-style fused selective scan.
 *
 * The operation (ScanWeaver, Sec. 3.1-3.2): for every independent channel,
 *
 *     h_t = a_t * h_{t-1} + bx_t                                   Eq. (3)
 *
 * evaluated as a prefix scan over the affine pairs (A_t, U_t) = (a_t, bx_t)
 * of Eq. (6) under the composition of Eq. (7),
 *
 *     (A2, U2) (+) (A1, U1) = (A2*A1, A2*U1 + U2)   (left = later segment),
 *
 * so that h_t = A_{1:t} h_0 + U_{1:t}.  The library returns the inclusive
 * states h_1..h_L, i.e. exactly what a sequential traversal produces
 * (Sec. 3.2), for every (b, d) row.
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Arrays are caller-owned DEVICE pointers (hipMalloc / torch CUDA tensors)
 *    on the current HIP device, dense and row-major; the library never frees
 *    or keeps them.  Host pointers are rejected with SW_ERR_INVALID_ARG.
 *  - Alignment: natural alignment of the element type is required (4 bytes for
 *    fp32/int32, 2 bytes for bf16).  Wider vector loads are used when every
 *    pointer is 16-byte aligned and L allows it; results do not depend on it.
 *  - Calls are asynchronous: SW_OK means the work was enqueued on the stream
 *    set with sw_set_stream() for the calling thread (default: the null
 *    stream).  Faults surface at the caller's next synchronisation.
 *  - Validation happens before anything is enqueued: on any non-OK return no
 *    output has been written and nothing is launched.  sw_last_error() gives
 *    a message for the last non-OK return on the calling thread.
 *  - Negative sizes are SW_ERR_INVALID_ARG.  A call whose output is empty
 *    (B*D == 0, or L == 0 for the bare scan) returns SW_OK and touches
 *    nothing; pointers are not inspected in that case.
 *  - Outputs must not overlap inputs or each other (SW_ERR_INVALID_ARG).
 *  - Scratch memory: calls whose sequences are split across workgroups use
 *    a small scratch per (device, stream) -- carry words and a ticket
 *    counter -- allocated from the device's default stream-ordered pool on
 *    the first such call on that stream, kept for later calls (grown when a
 *    call needs more) and never freed by the library.  Where the caller hands
 *    none over, the backward pass takes a per-call workspace, and a forward
 *    with N > 16 its planes of y (ceil(N/16) B*D*L fp32, at most 1 GiB), from
 *    the same pool on the same stream and releases it, stream-ordered, before
 *    returning.  The library raises that pool's release threshold so freed
 *    blocks stay cached for the next call (a process-wide setting of the
 *    device's default pool).  SW_ERR_ALLOC if an allocation fails, except that
 *    of the planes: the call then takes a kernel that needs none, whose y
 *    agrees within fp32 rounding.
 *  - Threads using distinct streams may call concurrently.
 *  - HIP graph capture: a call that uses neither the scratch nor a workspace
 *    can be captured and replayed: it launches kernels only.  Such calls are
 *    the fused forward at N = 16 with L a multiple of 8 for bf16 or of 4 for
 *    fp32, 16-byte aligned arrays and a workgroup's byte offsets below 2^31;
 *    the bare scan and its projection form when a row fits one chunk
 *    (L <= 2048) or the rows alone fill the GPU (B*D >= 8 per compute unit);
 *    sw_affine_scan_noalloc on every path (its tickets and records live in
 *    a static array, of which each call first clears what it uses with a fill
 *    kernel, so a replay repeats the call exactly); and
 *    the Blelloch schedule entry points.  A call that uses the scratch
 *    is not replay-safe (a replay would repeat the ticket range and epoch the
 *    host gave the captured launch), and the backward allocates a workspace
 *    per call: while the stream is capturing, those calls return
 *    SW_ERR_UNSUPPORTED before enqueuing anything.
 */
#ifndef SCANWEAVER_H
#define SCANWEAVER_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum sw_status {
  SW_OK = 0,              /* enqueued */
  SW_ERR_INVALID_ARG = 1, /* NULL / host / misaligned / overlapping pointer, negative size */
  SW_ERR_UNSUPPORTED = 2, /* a size outside what the kernels handle (e.g. N > 64) */
  SW_ERR_HIP = 3,         /* a HIP runtime call or launch failed */
  SW_ERR_ALLOC = 4        /* scratch allocation failed */
} sw_status;

/* Version of this ABI, major*10000 + minor*100 + patch (200: the training
 * forward and the backward exchange the pre-gate output, s_pre). */
int sw_version(void);

/*
 * Bare affine scan, fp32 (Eq. (3); pairs Eq. (6); composition Eq. (7)).
 *   a, bx, h_out : (B, D, L) fp32, L fastest.  h_out[b,d,t] is the state
 *                  after step t, i.e. a[b,d,t]*h_out[b,d,t-1] + bx[b,d,t].
 *   h0           : (B, D) fp32 initial state h[b,d,-1], or NULL for zero.
 * Arithmetic is fp32 (the composition is evaluated in an order that differs
 * from the sequential loop, so results are not bitwise equal to it; they
 * agree to within the rounding of fp32 affine compositions).
 */
int sw_affine_scan(const float* a, const float* bx, const float* h0, float* h_out, int64_t B,
                   int64_t D, int64_t L);

/*
 * Bare affine scan in the int32 wraparound ring Z/2^32: the same recurrence
 * on two's-complement bit patterns with arithmetic modulo 2^32.  The ring is
 * exact under any association order, so the result is bit-identical to the
 * sequential loop for every schedule.
 *   a, bx, h_out : (B, D, L) int32;  h0 : (B, D) int32 or NULL for zero.
 */
int sw_affine_scan_i32(const int32_t* a, const int32_t* bx, const int32_t* h0, int32_t* h_out,
                       int64_t B, int64_t D, int64_t L);

/*
 * sw_affine_scan for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same arguments, layout, results (within fp32 rounding of the same
 * schedule) and errors as sw_affine_scan, but no hipMalloc, hipFree or
 * allocating library routine is called: the tickets and records of rows cut
 * into segments live in a static array in the library's device code (32 KiB +
 * 24 bytes per chunk, 1.5 MiB for SW_NOALLOC_MAX_CHUNKS chunks), one copy per
 * GPU, held until the process ends; its address is looked up on the first
 * call on each device (make that call before capturing one into a HIP
 * graph).  Each call clears the part it uses, tickets and records, with a fill
 * kernel on the call's stream before the scan: what an earlier call left there
 * does not matter.
 *   - Calls with L > 2048, B*D < 8 * (compute units) and more than
 *     SW_NOALLOC_MAX_CHUNKS chunks, B * D * ceil(L / 2048), return
 *     SW_ERR_UNSUPPORTED before enqueuing anything.  Other calls (one chunk
 *     per row, or enough rows to give each its own workgroup) use no scratch
 *     and have no limit beyond sw_affine_scan's.
 *   - Every call on one GPU shares that GPU's array: two calls that may run
 *     at the same time on one GPU (on different streams, or from different
 *     host threads without ordering) race and give wrong results.  Order
 *     them on one stream.
 */
#define SW_NOALLOC_MAX_CHUNKS 65536
int sw_affine_scan_noalloc(const float* a, const float* bx, const float* h0, float* h_out,
                           int64_t B, int64_t D, int64_t L);

/* Scan schedules of sw_affine_scan_schedule. */
enum {
  SW_SCHED_DEFAULT = 0,  /* the library's: lane-sequential composition, DPP wavefront scan,
                            LDS combine, rows walked chunk by chunk, few long rows in
                            segments (what sw_affine_scan runs) */
  SW_SCHED_BLELLOCH = 1  /* the paper's (Sec. 3.3): a Blelloch upsweep / root / downsweep tree
                            over 2048-pair chunks in LDS, then affine-prefix reconstruction;
                            one workgroup per row, chunk carries in registers */
};

/*
 * sw_affine_scan (fp32) and sw_affine_scan_i32 with an explicit scan
 * schedule, for comparing schedules on the same recurrence.  Same arguments,
 * layout, results (bit-identical in int32; within fp32 rounding in fp32) and
 * errors, plus SW_ERR_INVALID_ARG for an unknown schedule.  The Blelloch
 * schedule gives each (b,d) row one workgroup, so it fills the GPU only when
 * there are many rows.
 */
int sw_affine_scan_schedule(const float* a, const float* bx, const float* h0, float* h_out,
                            int64_t B, int64_t D, int64_t L, int schedule);
int sw_affine_scan_schedule_i32(const int32_t* a, const int32_t* bx, const int32_t* h0,
                                int32_t* h_out, int64_t B, int64_t D, int64_t L, int schedule);

/*
 * The fused selective scan (plain form: fp32 y, zero initial state, no
 * options) with an explicit schedule.  SW_SCHED_DEFAULT is
 * sw_selective_scan_fwd / _bf16 (in_dtype F32 / BF16).  SW_SCHED_BLELLOCH
 * scans every (b,d,n) recurrence over t with the paper's Blelloch tree in LDS
 * (2048-step chunks, one workgroup per row looping over the states,
 * y accumulated in registers), for comparing schedules on the method's own
 * workload.  Arguments, layouts, results (within fp32 rounding) and errors
 * as for sw_selective_scan_fwd, plus SW_ERR_INVALID_ARG for an unknown dtype
 * or schedule.
 */
int sw_selective_scan_fwd_schedule(const void* x, const void* delta, const float* A,
                                   const void* Bm, const void* Cm, const float* Dskip, float* y,
                                   float* h_last, int64_t B, int64_t D, int64_t N, int64_t L,
                                   int in_dtype, int schedule);

/*
 * Recurrence with input and output projections, elementwise (Eq. (3)-(4)):
 *   h[b,d,t] = a[b,d,t] * h[b,d,t-1] + b[b,d,t] * x[b,d,t]      (h[b,d,-1] = h0)
 *   y[b,d,t] = c[b,d,t] * h[b,d,t]
 * The weighted prefix of Eq. (10) is the case x = 1, c = 1 (alpha -> a,
 * beta -> b).
 *   a, b, y      : (B, D, L) fp32, L fastest, required.
 *   x, c         : (B, D, L) fp32, or NULL for all ones.
 *   h0           : (B, D) fp32 initial state, or NULL for zero.
 *   h_last       : (B, D) fp32, receives h[b,d,L-1] (h0, or zero, when
 *                  L == 0), or NULL.
 * b*x and c*h are each rounded to fp32 once; the scan itself is that of
 * sw_affine_scan on the pairs (a, b*x), so with x and c NULL, y equals the
 * h_out of sw_affine_scan bit for bit.  Same conventions as sw_affine_scan
 * otherwise: caller-owned device pointers, outputs may not overlap inputs,
 * SW_ERR_INVALID_ARG for a NULL required pointer, misalignment, foreign or
 * host memory, negative sizes or overlap; SW_ERR_UNSUPPORTED when B*D*L
 * overflows.
 */
int sw_affine_scan_proj(const float* a, const float* b, const float* x, const float* c,
                        const float* h0, float* y, float* h_last, int64_t B, int64_t D,
                        int64_t L);

/*
 * The same in the int32 wraparound ring: b*x, the recurrence and c*h modulo
 * 2^32 on two's-complement bit patterns; bit-identical to the sequential loop.
 */
int sw_affine_scan_proj_i32(const int32_t* a, const int32_t* b, const int32_t* x,
                            const int32_t* c, const int32_t* h0, int32_t* y, int32_t* h_last,
                            int64_t B, int64_t D, int64_t L);

/*
 * Fused selective scan, forward, fp32 inputs (the Mamba-style instance of
 * Eq. (3) that motivates the method, Sec. 1 and Sec. 3.1), zero initial state:
 *
 *   a[b,d,t,n]  = exp(delta[b,d,t] * A[d,n])
 *   u[b,d,t,n]  = delta[b,d,t] * Bm[b,t,n] * x[b,d,t]
 *   h[b,d,t,n]  = a * h[b,d,t-1,n] + u                 (h[.,-1,.] = 0)
 *   y[b,d,t]    = sum_n Cm[b,t,n] * h[b,d,t,n] + Dskip[d] * x[b,d,t]
 *   h_last      = h[b,d,L-1,:]
 *
 *   x, delta : (B, D, L) fp32          A      : (D, N) fp32
 *   Bm, Cm   : (B, L, N) fp32          Dskip  : (D) fp32, or NULL for no skip
 *   y        : (B, D, L) fp32 output   h_last : (B, D, N) fp32 output or NULL
 * 1 <= N <= 64, else SW_ERR_UNSUPPORTED.  State and accumulation are fp32.
 * With L == 0 and B*D > 0, h_last (if given) is set to zero.
 * With N = 16, a call whose rows leave SIMDs idle or unevenly loaded may
 * split each row into up to 16 segments composed with Eq. (7), and may walk
 * each row with four lanes (four states each) instead of sixteen (fp32 y,
 * L a multiple of 32).  The library prices each choice with a model of its
 * launches on the device (per-step times measured per layout and occupancy)
 * and takes the cheapest; calls that write checkpoints walk whole rows.
 * Segments take one of two forms.  Correction form (fp32 y): every segment
 * walks from a zero state, a fold composes the carries, and each later
 * segment is walked again from its composed state only until the part
 * carried in has faded below 2^-26 of the magnitude of the state's own
 * terms (the whole segment when it does not fade).  Records form: each
 * segment's carry is formed first, then every segment walks once from its
 * initial state.  Results of both agree with a whole-row walk within fp32
 * rounding, not bit for bit.  The environment variables SW_SS_QUAD (0: never
 * four lanes per row, 1: whenever the call allows), SW_SS_SEGMENTS (the
 * count, 1: whole rows) and SW_SS_SEGFORM (1: records, 2: correction), read
 * per call, force the choice; sw_last_launch() names what a call enqueued.
 * A count k gives segments of L / k steps rounded up to the layout's
 * granularity (a 64- or 128-step super-tile with sixteen lanes per row, 64
 * steps with four), the last one the rest (a rest shorter than that
 * granularity joins the segment before, or, with four lanes per row, the
 * length is rounded down instead).
 * y's memory holds the segments' carries between the call's kernels, so y
 * must not be read until the call completes on its stream (as for any
 * output).
 */
int sw_selective_scan_fwd(const float* x, const float* delta, const float* A, const float* Bm,
                          const float* Cm, const float* Dskip, float* y, float* h_last,
                          int64_t B, int64_t D, int64_t N, int64_t L);

/*
 * As sw_selective_scan_fwd, with x, delta, Bm and Cm given as bf16 (raw
 * uint16 bit patterns, widened exactly to fp32 inside the kernel).  A, Dskip,
 * the state, y and h_last are fp32.
 */
int sw_selective_scan_fwd_bf16(const uint16_t* x, const uint16_t* delta, const float* A,
                               const uint16_t* Bm, const uint16_t* Cm, const float* Dskip,
                               float* y, float* h_last, int64_t B, int64_t D, int64_t N,
                               int64_t L);

/* Element types of sw_selective_scan_fwd_ex's arrays. */
typedef enum sw_dtype {
  SW_DTYPE_F32 = 0,  /* fp32 */
  SW_DTYPE_BF16 = 1  /* bf16, as raw uint16 bit patterns */
} sw_dtype;

/* Flags of sw_selective_scan_fwd_ex. */
enum { SW_DELTA_SOFTPLUS = 1 /* delta' = softplus(delta + delta_bias) */ };

/*
 * Fused selective scan, forward, with the optional inputs of a Mamba block
 * (the production kernel the method is measured against fuses the same
 * pieces; Sec. 1, Sec. 6.3).  With z, delta_bias, h0 NULL and flags 0 it is
 * sw_selective_scan_fwd (in_dtype F32) or sw_selective_scan_fwd_bf16 (BF16):
 *
 *   delta'[b,d,t] = delta[b,d,t] + delta_bias[d]        (bias: 0 if NULL)
 *                   then softplus(v) = log(1 + e^v)      if flags & SW_DELTA_SOFTPLUS
 *   a = exp(delta' * A[d,n]),  u = delta' * Bm[b,t,n] * x[b,d,t]
 *   h[b,d,-1,n] = h0[b,d,n]                              (0 if h0 is NULL)
 *   h[b,d,t,n] = a * h[b,d,t-1,n] + u                    (Eq. (3))
 *   y[b,d,t] = sum_n Cm[b,t,n] h[b,d,t,n] + Dskip[d] x[b,d,t]
 *   y[b,d,t] *= silu(z[b,d,t]) = z / (1 + e^-z)           if z is not NULL
 *   h_last[b,d,n] = h[b,d,L-1,n]
 *
 *   x, delta, z : (B, D, L) of in_dtype        Bm, Cm : (B, L, N) of in_dtype
 *   A : (D, N) fp32      Dskip, delta_bias : (D) fp32 or NULL
 *   h0, h_last : (B, D, N) fp32 or NULL        y : (B, D, L) of out_dtype
 * bf16 y is the fp32 result rounded to nearest even.  Softplus and silu are
 * evaluated in fp32 (a few ulps).  h0 may be the h_last of the previous
 * chunk of the same sequences, which continues the scan across calls; with
 * L == 0, h_last receives h0 (or zeros).  Unknown dtypes or flags:
 * SW_ERR_INVALID_ARG.  Other conventions as for sw_selective_scan_fwd.
 */
int sw_selective_scan_fwd_ex(const void* x, const void* delta, const float* A, const void* Bm,
                             const void* Cm, const float* Dskip, const void* z,
                             const float* delta_bias, const float* h0, void* y, float* h_last,
                             int64_t B, int64_t D, int64_t N, int64_t L, int in_dtype,
                             int out_dtype, int flags);

/*
 * sw_selective_scan_fwd_ex with workspace, 16-byte aligned device memory of at
 * least sw_selective_scan_fwd_workspace bytes that nothing else uses until the
 * call completes on its stream (SW_ERR_INVALID_ARG if the call needs more), or
 * NULL: taken from the device's stream-ordered pool for the call.
 */
int sw_selective_scan_fwd_ws(const void* x, const void* delta, const float* A, const void* Bm,
                             const void* Cm, const float* Dskip, const void* z,
                             const float* delta_bias, const float* h0, void* y, float* h_last,
                             int64_t B, int64_t D, int64_t N, int64_t L, int in_dtype,
                             int out_dtype, int flags, void* workspace, int64_t workspace_bytes);

/*
 * Bytes of the workspace of a forward of these sizes on the current device,
 * with (nonzero) or without z, with all arrays 16-byte aligned (nonzero) or not
 * (then what the call may need at most).  0 for N <= 16, for calls that need
 * none and for an empty or invalid call.
 */
int64_t sw_selective_scan_fwd_workspace(int64_t B, int64_t D, int64_t N, int64_t L, int in_dtype,
                                        int z, int aligned);

/*
 * sw_selective_scan_fwd_ex that also keeps what the backward pass needs
 * (training; always walks whole rows, so y is bit-identical to that of
 * sw_selective_scan_fwd_ex run with SW_SS_SEGMENTS=1): ckpt (B, D,
 * ceil(L/8), 16) fp32, required, receives the state
 * h[b,d,8k-1,n] before step 8k (h0, or zero, for k = 0) in slot
 * [b, d, k, n]; slots n >= N hold no state.  N <= 16 (SW_ERR_UNSUPPORTED
 * above).  s_pre (B, D, L) fp32, or NULL, receives y before the output gate
 * (y = s_pre * silu(z); without z, s_pre = y in fp32).  Handing ckpt (and,
 * with z, s_pre) to sw_selective_scan_bwd with the same inputs spares the
 * backward its own forward sweep (and its forward without the gate).
 * Otherwise as sw_selective_scan_fwd_ex.
 */
int sw_selective_scan_fwd_train(const void* x, const void* delta, const float* A, const void* Bm,
                                const void* Cm, const float* Dskip, const void* z,
                                const float* delta_bias, const float* h0, void* y, float* h_last,
                                float* ckpt, float* s_pre, int64_t B, int64_t D, int64_t N,
                                int64_t L, int in_dtype, int out_dtype, int flags);

/*
 * sw_selective_scan_fwd_train that may cut each row into segments where its
 * rows leave the GPU idle (N = 16 and the even N below 16 that take the
 * 16-lane kernels; the records form of sw_selective_scan_fwd, whose last launch
 * walks every segment from its composed state and writes its checkpoints): y,
 * s_pre, h_last and ckpt agree with those of sw_selective_scan_fwd_train within
 * fp32 rounding, not bit for bit.
 */
int sw_selective_scan_fwd_train_seg(const void* x, const void* delta, const float* A,
                                    const void* Bm, const void* Cm, const float* Dskip,
                                    const void* z, const float* delta_bias, const float* h0,
                                    void* y, float* h_last, float* ckpt, float* s_pre, int64_t B,
                                    int64_t D, int64_t N, int64_t L, int in_dtype, int out_dtype,
                                    int flags);

/*
 * Backward of sw_selective_scan_fwd_ex: the gradients of
 *   sum_{b,d,t} dy[b,d,t] y[b,d,t] + sum_{b,d,n} dh_last[b,d,n] h_last[b,d,n]
 * with respect to every input, by the chain rule through Eq. (3).  The
 * paper gives the forward only; the adjoint lam = dL/dh is the same affine
 * recurrence run backwards in time (Eq. (6)-(7) with the order reversed):
 *   ds_t = dy_t silu(z_t) (dy_t without z),  lam_t = ds_t Cm_t + a_{t+1} lam_{t+1}
 * and every gradient follows from lam, h and the inputs (see the oracle's
 * documentation for the full list of formulas).
 *
 * Inputs: as for sw_selective_scan_fwd_ex (same dtypes, same flags), plus
 *   dy      : (B, D, L) of dy_dtype (fp32 or bf16), required
 *   dh_last : (B, D, N) fp32 or NULL (zero)
 *   ckpt    : the ckpt of sw_selective_scan_fwd_train on the same inputs,
 *             or NULL (the backward then rebuilds it in its workspace: for
 *             N = 16 where the forward takes its 16-lane layout, with the
 *             forward's walk without y; else in its own kernel; the results
 *             are the same bits either way)
 *   s_pre   : with z, the s_pre of sw_selective_scan_fwd_train on the same
 *             inputs, or NULL (the backward then reruns the forward without
 *             the gate, which also writes the checkpoints when N <= 16);
 *             SW_ERR_INVALID_ARG without z
 * Outputs (fp32, overwritten, never accumulated into):
 *   dx, ddelta : (B, D, L), required; ddelta is with respect to the delta
 *                passed in (before bias and softplus)
 *   dA : (D, N), dB, dC : (B, L, N), required (sums over b, resp. over d)
 *   dDskip, ddelta_bias : (D) or NULL (not written); each is the gradient at
 *                the given value (at zero when the input is NULL)
 *   dz : (B, D, L), or NULL; requires z
 *   dh0 : (B, D, N) or NULL; the gradient with respect to the initial state
 *                (h0, or the zero state when h0 is NULL)
 * With L == 0 (or B*D == 0) the sums are zero and dh0 = dh_last.
 * Results are deterministic: cross-row sums are added in a fixed order.
 * N in [1, 64] (states above 16 run as further passes over the sequence,
 * 16 states each); with ckpt, N <= 16.  A workspace of about
 * (B*D*L*8 without ckpt + B*ceil(D/16)*L*128 + B*D*L*4 if z without s_pre) bytes,
 * where N > 32 with z at most ceil(N/16)*B*D*L*4 in place of the first term, is
 * taken from the device's stream-ordered pool for the call.  Other conventions (and
 * errors) as for sw_selective_scan_fwd_ex.
 */
int sw_selective_scan_bwd(const void* x, const void* delta, const float* A, const void* Bm,
                          const void* Cm, const float* Dskip, const void* z,
                          const float* delta_bias, const float* h0, const void* dy,
                          const float* dh_last, const float* ckpt, const float* s_pre,
                          float* dx, float* ddelta,
                          float* dA, float* dB,
                          float* dC, float* dDskip, float* dz, float* ddelta_bias, float* dh0,
                          int64_t B, int64_t D, int64_t N, int64_t L, int in_dtype, int dy_dtype,
                          int flags);

/*
 * sw_selective_scan_bwd with the type of the gradients that follow the inputs'
 * type: dx, ddelta, dB, dC and dz are of grad_dtype (bf16: the fp32 gradient
 * rounded once to nearest even; bf16 inputs, fp32 dy and N <= 16 only, else
 * SW_ERR_UNSUPPORTED); dA, dDskip, ddelta_bias and dh0 stay fp32.
 * workspace: 16-byte aligned device memory of at least
 * sw_selective_scan_bwd_workspace bytes that nothing else uses until the call
 * completes on its stream (SW_ERR_INVALID_ARG if smaller), or NULL: taken
 * from the device's stream-ordered pool for the call.
 */
int sw_selective_scan_bwd_ex(const void* x, const void* delta, const float* A, const void* Bm,
                             const void* Cm, const float* Dskip, const void* z,
                             const float* delta_bias, const float* h0, const void* dy,
                             const float* dh_last, const float* ckpt, const float* s_pre,
                             void* dx, void* ddelta, float* dA, void* dB, void* dC,
                             float* dDskip, void* dz, float* ddelta_bias, float* dh0, int64_t B,
                             int64_t D, int64_t N, int64_t L, int in_dtype, int dy_dtype,
                             int grad_dtype, int flags, void* workspace,
                             int64_t workspace_bytes);

/*
 * Bytes of the workspace of a backward call of these sizes on the current
 * device, with (nonzero) or without ckpt, z and s_pre (0 for an empty or
 * invalid call).
 */
int64_t sw_selective_scan_bwd_workspace(int64_t B, int64_t D, int64_t N, int64_t L, int ckpt,
                                        int z, int s_pre);

/*
 * Linear attention with a log decay for each head: the affine recurrence with a
 * K x V matrix as each head's state,
 *
 *   S_t = e^{g_t} S_{t-1} + k_t v_t^T        (Eq. (3) with a_t = e^{g_t})
 *   o_t = scale * S_t^T q_t
 *   h_last = the state after the last step; S_{-1} = h0, or zero
 *
 *   q, k : (B, L, Hk, K) of dtype      v : (B, L, H, V) of dtype
 *   g    : (B, L, H) fp32 log decays, or, with SW_LINEAR_G_HEAD, (H) fp32, one
 *          for all of a head's steps.  g <= 0 decays, and e^g is zero for
 *          g < -104 (as it is in fp32), -inf included.  g > 0 grows the state:
 *          where those of steps in a row add up to more than 87 (e^88 is more
 *          than fp32 holds), results may be infinite or NaN.
 *   o    : (B, L, H, V) of dtype, dense
 *   h0, h_last : (nseq, H, K, V) fp32, dense, or NULL
 * H is a multiple of Hk; head h reads the q and k of head h / (H / Hk).
 * 1 <= K, V <= 256, else SW_ERR_UNSUPPORTED.
 *
 * strides: host array of element strides, all >= 0, of q, k, v and g in turn,
 * each over (B, L, heads); the width is contiguous (parts of a fused
 * projection, broadcast inputs and transposed orders need no copy).  Loads are
 * 16 bytes wide where address, strides and width allow it; results do not
 * depend on it.
 *
 * cu_seqlens: NULL (then nseq = B), or (nseq + 1) int32 device values, ascending
 * within [0, L]: B = 1 and the row of L steps holds nseq sequences, sequence n the
 * steps cu_seqlens[n] .. cu_seqlens[n+1] - 1, each with its own state.  They are
 * read by the kernels only and held to [0, L].  Steps that no sequence covers (a
 * row padded to a fixed length) read as zero in o, and in every gradient; what q,
 * k, v, g and dout hold there is not used.  A sequence may be empty: its h_last is
 * its h0 (or zero).
 *
 * The state and all sums are fp32; bf16 inputs run on bf16 matrix instructions
 * with the states, the state's increments and the chunk's weights split in bf16
 * parts: o is rounded once, at its end, whatever the sizes of the call.
 * An infinity or NaN in q, k, v or g reaches the steps from its own on, as in
 * the recurrence, and no earlier one.
 *
 * workspace: 16-byte aligned device memory of at least
 * sw_linear_attn_fwd_workspace bytes (flags as for the call; packed nonzero with
 * cu_seqlens) that nothing else uses until the call completes on its stream
 * (SW_ERR_INVALID_ARG if the call needs more), or NULL: taken from the device's
 * stream-ordered pool for the call (then the call cannot be captured into a HIP
 * graph; otherwise it can).  Other conventions as above.
 */
enum { SW_LINEAR_G_HEAD = 1 /* g is (H): one log decay for a head */ };
int sw_linear_attn_fwd(const void* q, const void* k, const void* v, const float* g,
                       const float* h0, const int32_t* cu_seqlens, void* o, float* h_last,
                       int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K, int64_t V,
                       int64_t nseq, const int64_t* strides, int dtype, int flags, float scale,
                       void* workspace, int64_t workspace_bytes);
int64_t sw_linear_attn_fwd_workspace(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K,
                                     int64_t V, int64_t nseq, int dtype, int flags, int packed);

/*
 * Backward of sw_linear_attn_fwd: the gradients of sum(dout * o) +
 * sum(dh_last * h_last).  With dS_t the gradient with respect to S_t,
 *
 *   dS_t = scale q_t dout_t^T + e^{g_{t+1}} dS_{t+1}    (the last step's: + dh_last)
 *   dq_t = scale S_t dout_t,  dk_t = dS_t v_t  (summed over the heads that share them)
 *   dv_t = dS_t^T k_t,  dg_t = e^{g_t} <dS_t, S_{t-1}>,  dh0 = e^{g_0} dS_0
 *
 *   dout : (B, L, H, V) of dtype; its strides follow g's in `strides` (15 values)
 *   dh_last : (nseq, H, K, V) fp32 or NULL (zero)
 *   dq, dk, dv : dense, of dtype, rounded once from fp32;  dg : (B, L, H) fp32, or
 *   (H) with SW_LINEAR_G_HEAD;  dh0 : (nseq, H, K, V) fp32 or NULL
 * The states in dq, dk and dg keep fp32 accuracy.  dg is a sum of products of
 * steps before t with steps from t on, without a difference, so that it keeps its
 * digits where a step forgets nearly everything; it is zero where g < -104.  An
 * infinity or NaN reaches the steps that it reaches through these sums.  Results
 * are deterministic.  With no steps, dg (H) is zero and dh0 = dh_last.
 * The workspace holds a state of each head for every 64 steps (32 for fp32 inputs):
 * 4 H K V / 64 bytes a step, 2.7 GB at L = 65536, H = 40, K = V = 128; and fp32
 * gradients of q and k for every head where heads share them.  Otherwise as
 * sw_linear_attn_fwd.
 */
int sw_linear_attn_bwd(const void* q, const void* k, const void* v, const float* g,
                       const float* h0, const int32_t* cu_seqlens, const void* dout,
                       const float* dh_last, void* dq, void* dk, void* dv, float* dg, float* dh0,
                       int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K, int64_t V,
                       int64_t nseq, const int64_t* strides, int dtype, int flags, float scale,
                       void* workspace, int64_t workspace_bytes);
int64_t sw_linear_attn_bwd_workspace(int64_t B, int64_t L, int64_t Hk, int64_t H, int64_t K,
                                     int64_t V, int64_t nseq, int dtype, int flags, int packed);

/*
 * One step of B sequences, their states updated in place (serving):
 *   S <- e^g S + k v^T,  o = scale * S^T q
 *   q, k : (B, Hk, K), v : (B, H, V), o : (B, H, V) dense, all of dtype
 *   g : (B, H) fp32, or (H) with SW_LINEAR_G_HEAD
 *   state : (pool, H, K, V) fp32;  slots : (B) int32 device values or NULL.
 * Sequence b's state is state[slots[b]] (state[b] if NULL; pool >= B then).  A
 * slot outside [0, pool) is no sequence: its o is zero and no state changes.
 * Two sequences must not share a slot.  strides: element strides of q, k, v and
 * g over (B, heads), 8 values >= 0.  Launches one kernel; can be captured.
 */
int sw_linear_attn_step(const void* q, const void* k, const void* v, const float* g, float* state,
                        const int32_t* slots, void* o, int64_t B, int64_t Hk, int64_t H, int64_t K,
                        int64_t V, int64_t pool, const int64_t* strides, int dtype, int flags,
                        float scale);

/*
 * The norm before a block, with the residual addition and its scale:
 *   R' = R + res_scale * x      (rounded to res_dtype, in residual_out)
 *   y  = weight * R' / sqrt(mean(R'^2) + eps)
 * over M rows of D columns, 1 <= D <= 16384.  y is the norm of R' as stored.
 *   x, y : dtype     residual, residual_out : res_dtype (dtype, or fp32)
 *   weight, res_scale : (D) fp32; res_scale may be NULL (ones)
 * residual NULL: y is the norm of x; residual_out and res_scale are NULL then.
 * x and residual have their rows x_stride, residual_stride elements apart; the
 * outputs are dense.  Sums are fp32, outputs rounded once.  One launch; can be
 * captured.  Other conventions as above.
 */
int sw_residual_norm_fwd(const void* x, const void* residual, const float* weight,
                         const float* res_scale, void* y, void* residual_out, int64_t M, int64_t D,
                         int64_t x_stride, int64_t residual_stride, int dtype, int res_dtype,
                         float eps);

/*
 * Backward: given dy, dres (of y and residual_out; dres may be NULL) and
 * residual_out (x itself, with res_dtype = dtype, where there was no residual),
 * with n = R' / rms:
 *   dR' = dres + (weight dy - n mean(weight dy n)) / rms
 *   dresidual = dR', dx = res_scale * dR', dweight = sum dy n, dres_scale = sum x dR'
 * dx and dresidual may be NULL (not written; without res_scale and with equal
 * types they are the same values); x is needed with res_scale only.  The sums
 * over rows are added in a fixed order.  workspace: 16-byte aligned, at least
 * sw_norm_bwd_workspace(M, D, D, 1, or 2 with res_scale) bytes, or NULL: from
 * the device's stream-ordered pool for the call (no capture then).
 */
int sw_residual_norm_bwd(const void* dy, const void* dres, const void* residual_out,
                         const float* weight, const void* x, const float* res_scale, void* dx,
                         void* dresidual, float* dweight, float* dres_scale, int64_t M, int64_t D,
                         int64_t dy_stride, int64_t dres_stride, int64_t residual_out_stride,
                         int64_t x_stride, int dtype, int res_dtype, float eps, void* workspace,
                         int64_t workspace_bytes);
int64_t sw_norm_bwd_workspace(int64_t M, int64_t D, int64_t width, int grads);

/*
 * The norm after a block's mixer, with its gate, over groups of `group` columns
 * (group = D: the whole row; the width of a head: a norm for each head):
 *   y = weight * u / sqrt(mean_group(u^2) + eps),  u = x silu(z)
 *   with SW_GATE_AFTER:  y = weight * x / sqrt(mean_group(x^2) + eps) * silu(z)
 * x, z, y : M rows of D of dtype, D a multiple of group, 1 <= group <= 16384; z
 * NULL: no gate.  weight : (D) fp32.  Rows of x and z lie x_stride, z_stride
 * elements apart.  Otherwise as sw_residual_norm_fwd.
 */
enum { SW_GATE_AFTER = 1 /* the gate multiplies the normed values */ };
int sw_gated_norm_fwd(const void* x, const void* z, const float* weight, void* y, int64_t M,
                      int64_t D, int64_t group, int64_t x_stride, int64_t z_stride, int dtype,
                      int flags, float eps);

/*
 * Its gradients: dx, dz (with z) dense, of dtype; dweight (D) fp32, its sums over
 * the rows in a fixed order.  workspace as for sw_residual_norm_bwd, of
 * sw_norm_bwd_workspace(M, D, group, 1) bytes.
 */
int sw_gated_norm_bwd(const void* dy, const void* x, const void* z, const float* weight, void* dx,
                      void* dz, float* dweight, int64_t M, int64_t D, int64_t group,
                      int64_t dy_stride, int64_t x_stride, int64_t z_stride, int dtype, int flags,
                      float eps, void* workspace, int64_t workspace_bytes);

/*
 * Gated linear recurrence: the affine recurrence of Eq. (3) with one state for
 * each channel and gates that make its pairs,
 *
 *   m_t = c softplus(lam) sigmoid(r_t),  a_t = e^{-m_t}
 *   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t
 *   h_last = the state after the last step; h_{-1} = h0, or zero
 *
 *   x, r, i : (B, L, D) of dtype, r and i before their sigmoids
 *   lam     : (D) fp32;  c > 0 and finite
 *   h       : (B, L, D) of dtype, dense, rounded once from fp32; NULL: not written
 *   h0, h_last : (nseq, D) fp32, dense, or NULL
 *   ckpt    : (B, ceil(L / SW_GATED_CKPT), D) fp32 or NULL: the state before every
 *             SW_GATED_CKPT-th step, for the backward
 * strides: host array of 6 element strides >= 0, over (B, L) of x, r and i in turn;
 * the D channels of a step are contiguous.
 *
 * cu_seqlens: NULL (then nseq = B), or (nseq + 1) int32 device values, ascending
 * within [0, L], B = 1: sequences packed into one row, as for sw_linear_attn_fwd.
 * Steps that no sequence covers read as zero in h and in every gradient, whatever
 * x, r and i hold there; an empty sequence's h_last is its h0 (or zero).
 *
 * The state, the gates and all sums are fp32.  sqrt(1 - a^2) is formed from m, so
 * that it keeps its digits as a nears 1; it is off by some 2^-20 of itself for bf16
 * inputs, whose series is shorter, and 2^-22 for fp32 ones, and the sigmoid of a bf16 v
 * by at most (|v| + 4) 2^-24 (a step's input in all: 1.2e-6 and 3.1e-7 of itself, measured
 * over |r|, |i| <= 8 and lam from -12 to 4).  An infinity or NaN in a step's inputs
 * makes that step and those after it in its channel and sequence infinite or NaN,
 * as far as the recurrence carries it, and touches no other.
 *
 * workspace: 16-byte aligned, at least sw_gated_scan_fwd_workspace bytes, that nothing
 * else uses until the call completes, or NULL: from the device's stream-ordered
 * pool for the call (no capture then).  The words that chunks of a row hand on lie
 * there; a call whose words take at most 16 MiB keeps them in the per-stream scratch
 * instead, which spares a launch that clears them, except while its stream is
 * capturing.  Rows of at most 256 steps need none.  Results depend on neither; every
 * call of the same inputs gives the same bits.
 */
enum { SW_GATED_CKPT = 64 };
int sw_gated_scan_fwd(const void* x, const void* r, const void* i, const float* lam,
                      const float* h0, const int32_t* cu_seqlens, void* h, float* h_last,
                      float* ckpt, int64_t B, int64_t L, int64_t D, int64_t nseq,
                      const int64_t* strides, int dtype, float c, void* workspace,
                      int64_t workspace_bytes);
int64_t sw_gated_scan_fwd_workspace(int64_t B, int64_t L, int64_t D);

/*
 * Backward: the gradients of sum(dh * h) + sum(dh_last * h_last).  With g_t that with
 * respect to h_t, g_t = dh_t + a_{t+1} g_{t+1} (the last step's: + dh_last), b =
 * sqrt(1 - a^2), s = sigmoid(i) and
 *   e_t = g_t (a^2 (m / b) s x - m a h_{t-1}):
 *   dx = g b s,  di = g b s (1 - s) x,  dr = e (1 - sigmoid(r)),
 *   dlam = sum e * sigmoid(lam) / softplus(lam),  dh0 = a_0 g_0
 * (m / b tends to sqrt(m / 2) where a nears 1, so nothing here is singular).
 *   dh : (B, L, D) of dtype; its strides follow i's in `strides` (8 values)
 *   dx, dr, di : (B, L, D) of dtype, dense;  dlam : (D) fp32;  dh0 : (nseq, D) fp32 or
 *   NULL;  ckpt : the forward's, or NULL (formed again)
 * Sums run in a fixed order.  With no steps dlam is zero and dh0 = dh_last.
 */
int sw_gated_scan_bwd(const void* x, const void* r, const void* i, const float* lam,
                      const float* h0, const int32_t* cu_seqlens, const float* ckpt,
                      const void* dh, const float* dh_last, void* dx, void* dr, void* di,
                      float* dlam, float* dh0, int64_t B, int64_t L, int64_t D, int64_t nseq,
                      const int64_t* strides, int dtype, float c, void* workspace,
                      int64_t workspace_bytes);
int64_t sw_gated_scan_bwd_workspace(int64_t B, int64_t L, int64_t D, int ckpt);

/*
 * One step of B sequences, their states updated in place (serving): x, r, i (B, D)
 * of dtype, rows strides[0..2] apart; h (B, D) of dtype, dense; state (pool, D)
 * fp32; slots : (B) int32 device values or NULL, as for sw_linear_attn_step.
 */
int sw_gated_scan_step(const void* x, const void* r, const void* i, const float* lam,
                       float* state, const int32_t* slots, void* h, int64_t B, int64_t D,
                       int64_t pool, const int64_t* strides, int dtype, float c);

/*
 * The norm of each head's query and key, with the rotation by the token's position:
 *   u = w * x / sqrt(mean(x^2) + eps)   over the K columns of a head
 *   y = u with its first R columns turned, pair j by the angle position * inv_freq[j]:
 *       (p, q) -> (p cos - q sin, q cos + p sin)
 * where pair j is columns (j, j + R / 2), or, with SW_HEAD_ADJACENT, (2 j, 2 j + 1).
 *   q, yq : (B, L, H, K);  k, yk : (B, L, Hk, K), of dtype; 1 <= K <= 256.  The
 *           outputs are dense.  H and Hk may be any, zero among them.
 *   wq, wk : (K) fp32 or NULL (ones)
 *   inv_freq : (R / 2) fp32; R even, at most K; R = 0: no rotation (inv_freq unused)
 *   positions : (B, L) int32, with SW_HEAD_POS_I64 int64 values, of any sign; NULL: l
 * Angles are formed and reduced in 64 bits, so that far positions keep theirs to
 * fp32.  Sums are fp32, outputs rounded once.
 * strides: host array of 8 element strides >= 0: q's and k's over (B, L, heads), then
 * positions' over (B, L).  One launch; can be captured.
 */
enum { SW_HEAD_ADJACENT = 1, SW_HEAD_POS_I64 = 2 };
int sw_head_norm_fwd(const void* q, const void* k, const float* wq, const float* wk,
                     const void* positions, const float* inv_freq, void* yq, void* yk, int64_t B,
                     int64_t L, int64_t H, int64_t Hk, int64_t K, int64_t R,
                     const int64_t* strides, int dtype, int flags, float eps);

/*
 * Its gradients: dq and dk dense, of dtype; dwq, dwk (K) fp32 (both or neither NULL),
 * their sums over tokens and heads in a fixed order.  strides: dyq's, dyk's, q's and
 * k's over (B, L, heads), then positions' (14 values).  workspace as for
 * sw_residual_norm_bwd, of sw_head_norm_bwd_workspace bytes; none without dwq.
 */
int sw_head_norm_bwd(const void* dyq, const void* dyk, const void* q, const void* k,
                     const float* wq, const float* wk, const void* positions,
                     const float* inv_freq, void* dq, void* dk, float* dwq, float* dwk, int64_t B,
                     int64_t L, int64_t H, int64_t Hk, int64_t K, int64_t R,
                     const int64_t* strides, int dtype, int flags, float eps, void* workspace,
                     int64_t workspace_bytes);
int64_t sw_head_norm_bwd_workspace(int64_t B, int64_t L, int64_t H, int64_t Hk, int64_t K);

/*
 * Rows of a table by token, scaled: y_t = scale * table[token_t], rounded once.
 *   tokens : (T) int32, or int64 with SW_EMBED_TOKENS_I64; one outside [0, V) is no
 *            token (padding): its row is zero
 *   table  : (V, D) of table_dtype, dense;  y : (T, D) of y_dtype, dense
 * One launch; can be captured.
 */
enum { SW_EMBED_TOKENS_I64 = 1 };
int sw_embedding_fwd(const void* tokens, const void* table, void* y, int64_t T, int64_t V,
                     int64_t D, int table_dtype, int y_dtype, int flags, float scale);

/*
 * The table's gradient, dense: dtable[v] = scale * (the sum of dy_t over the t with
 * token_t = v), rounded once to table_dtype; zero where there is none.  Sums are fp32,
 * in an order that T, D and the tokens alone fix: the same inputs give the same bits.
 * dy : T rows of D of dy_dtype, dy_stride elements apart.  T < 2^31.  workspace: 16-byte aligned,
 * at least sw_embedding_bwd_workspace bytes, or NULL: from the device's
 * stream-ordered pool (no capture then).
 */
int sw_embedding_bwd(const void* tokens, const void* dy, void* dtable, int64_t T, int64_t V,
                     int64_t D, int64_t dy_stride, int dy_dtype, int table_dtype, int flags,
                     float scale, void* workspace, int64_t workspace_bytes);
int64_t sw_embedding_bwd_workspace(int64_t T, int64_t V, int64_t D);

/* Stream used by the calling thread's subsequent calls (a hipStream_t;
 * NULL = the null stream).  Always SW_OK. */
int sw_set_stream(void* hip_stream);
void* sw_get_stream(void);

/* Static text for a status code; never NULL. */
const char* sw_status_string(int status);

/* Message for the calling thread's last non-OK return ("" if none). */
const char* sw_last_error(void);

/*
 * The kernels sw_selective_scan_fwd_ex (train = 0) or
 * sw_selective_scan_fwd_train (train = 1) would enqueue for these sizes and
 * dtypes, with 16-byte aligned arrays, on a part with `cus` compute units
 * (cus <= 0: the current device's), under the same SW_SS_* environment;
 * nothing is launched and no device memory is touched, so with cus > 0 it
 * needs no GPU.  Outputs (all required):
 *   layout : 16 (one lane per state), 4 (four lanes per row, four states
 *            each), 8 (the kernels for any N, whose segments are not planned
 *            here: one for at most 16 steps, one that chains its own sequence
 *            chunks, and the 16-lane kernels on groups of states), or 0 when there is nothing to launch (B*D or L zero)
 *   nseg, lseg : the row is walked as nseg segments of lseg steps, the last
 *            taking the rest (1 and L: whole rows; 0 and 0 with layout 0)
 *   form   : 0 whole rows, 1 records form, 2 correction form (see
 *            sw_selective_scan_fwd)
 * Errors as the forward call's for the same sizes: SW_ERR_INVALID_ARG
 * (unknown dtype, negative size, NULL output), SW_ERR_UNSUPPORTED (N outside
 * [1, 64], train with N > 16, sizes past the launch limits); SW_ERR_HIP when
 * cus <= 0 and the device cannot be queried.
 */
int sw_selective_scan_plan(int64_t B, int64_t D, int64_t N, int64_t L, int in_dtype,
                           int out_dtype, int train, int cus, int* layout, int64_t* nseg,
                           int64_t* lseg, int* form);

/* Which kernels the calling thread's last successful fused forward or
 * backward call (sw_selective_scan_fwd*, sw_selective_scan_bwd; "" before
 * any) enqueued: for the forward the layout, and for a call split into
 * segments their count, length and form -- e.g. "selective_quad_kernel: 9
 * segments of 7296 steps, correction form (3 launches)"; for the backward
 * where its checkpoints came from.  For tuning and benchmarks; the text is
 * not a stable format. */
const char* sw_last_launch(void);

#ifdef __cplusplus
}
#endif

#endif /* SCANWEAVER_H */
