/*
 * gla.h - C ABI of the MI355X (gfx950) implementation of the gated-linear-attention
 * (GLA) token mixer used in the DiG diffusion backbone: the forward pass (gla_fwd*),
 * its variants with the gate prologue and output epilogue (gla_fwd_fused) and with
 * several scan orders summed (gla_fwd_multi), the backward pass (gla_bwd*), the same
 * with the full gate matrix alpha_t^T beta_t (gla_fwd_gates, gla_fwd_fused_gates,
 * gla_bwd_gates), and the depth-wise convolution of the DiG block's reorientation
 * module (gla_srem_dwconv).  Beside them stands a mixer with one decay a head for
 * sequences of any kind: the recurrence itself (gla_decay_fwd, gla_decay_bwd, and
 * gla_decay_step for single tokens), the rotation of its queries and keys by the
 * tokens' positions (gla_rope), and the layer norm of its outputs or of the tokens
 * with and without the output gate, both directions (gla_norm_fwd, gla_norm_bwd).
 *
 * Operation (DiG paper, Sec. 3.1 "Gated Linear Attention Transformer",
 * Eq. (attn_gla), rows 1-3, with the gate G_t reduced to its key-side factor
 * alpha_t, i.e. beta_t = 1, except in the *_gates entry points):
 *
 *     S_t = diag(alpha_t) S_{t-1} + k_t^T v_t ,     o_t = q_t S_t ,     S_0 = 0
 *
 * per (batch, head), S in R^{dk x dv}, evaluated in the chunk-parallel form of
 * Sec. 3.5 ("Efficiency Analysis": the sequence is cut into chunks that are
 * computed on-chip, cost O(T M D + T D^2)).  The tokens of one image form a
 * grid_h x grid_w grid; the recurrence runs along one of the four scan orders
 * that the DiG block obtains by alternately transposing and flipping the token
 * grid (Sec. 3.3, Algorithm 1; operators of the supplementary Algorithms 2-4).
 * The permutation is folded into the kernels' address arithmetic: tensors stay
 * in canonical order and nothing is transposed in memory.
 *
 * Conventions common to every entry point
 * ---------------------------------------
 * Pointers marked DEVICE are device (HBM) addresses owned by the caller; the
 * library never frees, reallocates or retains them.  All tensors are dense,
 * row-major, in canonical token order n = r * grid_w + c for every scan order:
 *
 *     q, k        : [B, H, T, dk]   element type qkv_dtype (bf16 or fp32)
 *     log_alpha   : [B, H, T, dk]   fp32, log(alpha_t) <= 0 (e.g. logsigmoid(z)/tau)
 *     v           : [B, H, T, dv]   element type qkv_dtype
 *     out         : [B, H, T, dv]   element type out_dtype; out[n] = o at token n
 *     final_state : [B, H, dk, dv]  fp32, the state after the last scan step; may be NULL
 *
 * T must equal grid_h * grid_w.  No 1/sqrt(dk) scale is applied (the recurrence
 * has none); scale q beforehand.  Supported head sizes: 1 <= dk <= 64,
 * 1 <= dv <= 128.  T need not be a multiple of the chunk length.
 *
 * Calls enqueue work on `stream` (a hipStream_t passed as void*, NULL = the
 * default stream) and return without synchronising the host; results are valid
 * once the stream reaches that point.  Inputs must stay unmodified until then.
 * Outputs must not alias inputs.  The current HIP device must be the one that
 * owns the buffers.
 *
 * Every function returns a gla_status (0 = success).  An argument error (every
 * status but GLA_ERR_HIP) is found before anything is enqueued: no kernel has
 * run and no output byte has been written.  GLA_ERR_HIP reports a failed runtime
 * call or launch; a call is several kernels, so the earlier ones of that call
 * may already be enqueued and the outputs are then undefined.
 *
 * Preconditions that are not checked: log_alpha <= 0 and finite inputs.  Further
 * limits of the engines (see gla_engine):
 *  - bf16 hi/lo MFMA engine: the summed |log_alpha| over any 64 consecutive scan
 *    steps of one key channel stays below 80 (true for alpha = sigmoid(z)^(1/16)
 *    whenever z > -20).  GLA_ENGINE_RECURRENT has no such limit.  Beyond it, up to a gate
 *    of exactly zero (log_alpha = -inf), what that channel adds inside the 64-step chunk is
 *    lost or wrong, but finite: later chunks lack it as far as it would not have decayed.
 *    With the two-sided gate the bound is on the sum of both sides' |log|, and what lies beyond it need not be finite.
 *  - fp16 MFMA engine (what GLA_ENGINE_AUTO takes for the plain forward pass, and for
 *    gla_fwd_fused without the output epilogue, on bf16 inputs with 17..64 key
 *    channels and more than four chunks, unless the single-launch kernels take the call (see gla_engine), or
 *    the last span of the launch plan would
 *    be a single chunk of fewer than 64 tokens, or the call is a large column scan or
 *    [B,T,H,d] call of 33 to 36 key channels: such calls run on the bf16 hi/lo kernels, see gla_engine): its operands
 *    cover a decay of at most 2^-11 per key channel over 32 consecutive scan steps
 *    (alpha above about 0.79 on average; sigmoid(z)^(1/16) with z > -3.7) and
 *    inputs whose largest |q|, |k| lie in [2^-8, 8] and |v| in [2^-8, 2^14].  This
 *    IS checked, on the device: a (batch, head) sequence outside the range is
 *    recomputed in the same call by the bf16 hi/lo kernel, one work-group walking
 *    the whole sequence - correct, but many times slower for that sequence.
 *    Callers whose gates close faster than that as a rule should select
 *    GLA_ENGINE_MFMA.
 *  - Where the output pass chains the span states itself (gla_carry), a thread
 *    stops adding earlier spans once the decay accumulated on its key channels is
 *    below 2^-40: what is left out is at most 2^-40 of what those earlier states
 *    hold.  The bound is relative to the earlier states, not to the sum so far
 *    (a thread whose sum is still exactly zero, e.g. behind a padded tail of
 *    all-zero k or v, does go on: with the two-sided gate, in the single-launch kernels, and in the kernels that the
 *    heads of 33 to 36 key channels have, the 2^-40 then count from behind the zeros;
 *    in the others with one gate, which these heads share for their shortest spans, it
 *    stops after the group of up to 32 spans that ended them): sequences whose later spans are many orders
 *    of magnitude smaller than the earlier ones lose the decayed remainder of
 *    the earlier ones.  GLA_CARRY_KERNEL has no cut-off.
 *
 * The entry points that take a caller workspace only enqueue kernels, with two
 * exceptions: the first use of a kernel instantiation on a device raises its
 * dynamic-LDS limit (hipFuncSetAttribute), and a forward call in one launch asks
 * whether its stream is being recorded (hipStreamIsCapturing; a recorded call has
 * one small kernel more, which clears its flags).  Before capturing calls into a HIP
 * graph, or entering a region that must not touch the runtime, run each call
 * once with the same shapes and options.
 */
#ifndef GLA_H_
#define GLA_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    GLA_OK = 0,
    GLA_ERR_NULL = 1,        /* a required pointer is NULL */
    GLA_ERR_SHAPE = 2,       /* non-positive size, grid_h*grid_w != T, or a bad enum value */
    GLA_ERR_UNSUPPORTED = 3, /* dk > 64, dv > 128, or a dtype / engine combination not built */
    GLA_ERR_ALIGN = 4,       /* a base pointer is not 16-byte aligned */
    GLA_ERR_WORKSPACE = 5,   /* workspace NULL or smaller than gla_fwd_workspace_bytes() */
    GLA_ERR_HIP = 6          /* the HIP runtime reported an error (allocation or launch) */
} gla_status;

/* Scan orders (Sec. 3.3 / Algorithm 1).  Scan step s visits canonical token n:
 *   ROW_FWD  n = s                       ROW_REV  n = T-1-s
 *   COL_FWD  n = (s % grid_h) * grid_w + s / grid_h   (down a column, then the next column)
 *   COL_REV  the COL_FWD sequence read from its last step backwards              */
typedef enum { GLA_SCAN_ROW_FWD = 0, GLA_SCAN_ROW_REV = 1,
               GLA_SCAN_COL_FWD = 2, GLA_SCAN_COL_REV = 3 } gla_scan_dir;

typedef enum { GLA_DT_F32 = 0, GLA_DT_BF16 = 1 } gla_dtype;

/* Options for gla_set_option (process-wide, meant for tuning and tests). */
typedef enum {
    GLA_OPT_CHUNKS_PER_SPAN = 0, /* 0 = choose automatically; n > 0 = n 64-token chunks per work-group */
    GLA_OPT_ENGINE = 1,          /* gla_engine */
    GLA_OPT_CARRY = 2,           /* gla_carry */
    GLA_OPT_BWD_SPLIT = 3,       /* 0 = the backward pass computes dk and dv of a chunk in one kernel (MFMA engine);
                                    1 = in two kernels (the forward output pass for dv, the row read for dk) */
    GLA_OPT_LOOK_BACK_POLLS = 5, /* how often a wave of the single-launch forward kernels (gla_recur_fwd's too, but for calls in
                                    place, which have no inputs left to start from) polls for the state of an earlier span
                                    before it forms the state entering its own from the inputs (default 32768: tens of
                                    milliseconds, which only runs out where other work keeps the earlier spans off the
                                    GPU; 0 = never, for tests) */
    GLA_OPT_GLU_SPLIT = 6,       /* 1 = gla_glu_bwd takes dg and du of bf16 calls as two bf16 numbers each into the second pair of
                                    products: gradients are off by their own rounding alone, for twice that pair's operations and
                                    twice the workspace's two arrays (gla_glu_bwd_workspace_bytes goes by it too); 0 (default) =
                                    as one */
    GLA_OPT_RANGE_FALLBACK = 4   /* 1 (default) = after the fp16 engine's passes, the (batch, head) sequences that
                                    left its range are recomputed by the bf16 hi/lo kernel (one more launch, whose
                                    work-groups return at once when no flag is raised); 0 = that launch is skipped
                                    (for callers that know their gates and inputs stay in range, and for
                                    measurements) */
} gla_option;
typedef enum {
    GLA_ENGINE_AUTO = 0,      /* bf16 inputs with dk % 4 == 0 and dv % 8 == 0 -> an MFMA engine (the fp16 one for the
                                 plain forward pass and for gla_fwd_fused without r_pre, with 17..64 key channels
                                 and more than four chunks, else the bf16 hi/lo one), otherwise recurrent.  A call
                                 whose last span would be one chunk of fewer than 64 tokens (T % 64 != 0, and 64-token
                                 chunks before it that the plan's chunks per span divide) runs on the bf16 hi/lo kernels
                                 instead of the fp16 ones, and so does the plain forward pass with 33 to 36 key channels
                                 (or up to 36 and 65 to 80 value columns) of a column scan or of [B,T,H,d] tensors from
                                 3000 chunks of 64 tokens on, over all batches and heads; in gla_fwd_static only if their plan fits its array.
                                 Of heads of 17 to 36 key channels and 33 to 72 value columns, forward calls with one gate from about
                                 512 chunks (320 for sequences of up to ten, 288 for up to 32 / 64 channels; with the output epilogue
                                 48 to 192) up to about 2048, and larger ones of 8 to 128 sequences up to 4096 (from about 3000), run on
                                 kernels with the bf16 hi/lo operands that read their inputs once, in one launch; so do sequences of four
                                 chunks (with the epilogue of three) and, from 288 chunks on, the two-sided gate's of up to 128 sequences.
                                 Long sequences only up to a number of spans (of four or eight chunks) that depends on the kind of call: 48 to
                                 128, and 24 to 64 where not all spans are worked on at once.  Not with
                                 GLA_OPT_CHUNKS_PER_SPAN or GLA_CARRY_KERNEL set */
    GLA_ENGINE_RECURRENT = 1, /* fp32 token-by-token arithmetic inside each span; any dtype, any gates */
    GLA_ENGINE_MFMA = 2,      /* bf16 hi/lo MFMA chunk form (Sec. 3.5) in every pass, or in the one there is; bf16 inputs only */
    GLA_ENGINE_MFMA_FP16 = 3  /* fp16 operands in both passes of the plain forward call and of gla_fwd_fused without
                                 r_pre (producer / consumer waves), the bf16 hi/lo kernel as range fallback;
                                 GLA_ERR_UNSUPPORTED where it does not apply (the output epilogue, other entry
                                 points, fp32 inputs, fewer than 17 key channels) */
} gla_engine;

/* Where the states of the spans of one (batch, head) are chained, S_start(r+1) = diag(Gamma_r) S_start(r) + U_r
 * (the recurrence of Eq. (attn_gla) applied span by span). */
typedef enum {
    GLA_CARRY_AUTO = 0,          /* in the output pass when an MFMA engine runs with at most 128 spans per head */
    GLA_CARRY_KERNEL = 1,        /* a kernel of its own between the two passes */
    GLA_CARRY_IN_OUTPUT_PASS = 2 /* each output work-group chains the local states before its span, whatever the
                                    span count (the recurrent engine has no such path and keeps the kernel) */
} gla_carry;

typedef void *gla_stream_t; /* a hipStream_t */

/*
 * gla_fwd - GLA forward for bf16 q/k/v, fp32 log_alpha, fp32 out
 * (Eq. (attn_gla) rows 1-3 along `scan_dir`; chunk form of Sec. 3.5).
 *
 *   q, k, v      DEVICE, bf16, layouts above            (read)
 *   log_alpha    DEVICE, fp32                           (read)
 *   out          DEVICE, fp32 [B,H,T,dv]                (written)
 *   final_state  DEVICE, fp32 [B,H,dk,dv] or NULL       (written if not NULL)
 *
 * Uses a library-owned scratch buffer per device that grows on demand with
 * hipMalloc (which synchronises the device the first time a larger problem is
 * seen) and is kept until the process ends; concurrent calls on different
 * streams of one device would share it and are not supported - use gla_fwd_ex
 * with separate workspaces for that.
 */
int gla_fwd(const void *q, const void *k, const void *v, const float *log_alpha,
            int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
            float *out, float *final_state, gla_stream_t stream);

/*
 * gla_fwd_static - gla_fwd for callers that cannot allocate device memory: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same
 * arguments, results and status codes as gla_fwd; the span states live in a static
 * device array of GLA_STATIC_SCRATCH_BYTES that every GPU the library runs on holds
 * until the process ends.  The call itself makes no hipMalloc / hipFree and uses no
 * allocating library routine; the kernels it launches are gla_fwd's.
 *
 * GLA_ERR_WORKSPACE if the launch plan of the problem needs more than the array holds
 * (B * H * spans * (dk * dv + dk + dv + 1) floats, spans = 64-token chunks / chunks per
 * work-group; the DiG-XL/2 shape at 2048 px uses about 7 MiB); nothing is enqueued then.
 * (A call in one launch needs some bytes more for its flags, and runs in two passes where
 * those do not fit.)
 * All calls on one GPU share that GPU's array: calls that overlap on one GPU (different
 * streams or threads) race.  Nothing in it needs clearing between calls: every call
 * writes the span states before it reads them.  As for every entry point that takes a
 * workspace, the first call of a kernel variant in the process configures it
 * (hipFuncSetAttribute); make one call outside graph capture before capturing.
 */
#define GLA_STATIC_SCRATCH_BYTES (16u << 20)
int gla_fwd_static(const void *q, const void *k, const void *v, const float *log_alpha,
                   int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                   float *out, float *final_state, gla_stream_t stream);

/*
 * gla_fwd_ex - the same operation with explicit element types and a caller-owned
 * workspace; never allocates.
 *
 *   qkv_dtype        gla_dtype of q, k, v
 *   out_dtype        gla_dtype of out (final_state is always fp32)
 *   workspace        DEVICE, 16-byte aligned, at least gla_fwd_workspace_bytes(...) bytes;
 *                    contents on entry are ignored, contents on return are unspecified
 */
int gla_fwd_ex(const void *q, const void *k, const void *v, const float *log_alpha,
               int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
               int qkv_dtype, int out_dtype, void *out, float *final_state,
               void *workspace, size_t workspace_bytes, gla_stream_t stream);

/* Memory order of q, k, log_alpha ([.., dk]) and v, out ([.., dv]); final_state and initial_state are always
 * [B,H,dk,dv].  BTHD is the (B, T, D) token stream of Algorithm 1 with D = H * d seen per head. */
typedef enum { GLA_LAYOUT_BHTD = 0, GLA_LAYOUT_BTHD = 1 } gla_layout;

/*
 * gla_fwd_layout - gla_fwd_ex for either memory order, starting from a given state
 * (Eq. (attn_gla) row 1 with S_0 = initial_state instead of zero: the recurrence
 * continued from an earlier call's final_state, e.g. a sequence fed in pieces).
 *
 *   layout           gla_layout of q, k, v, log_alpha and out (dense, no padding)
 *   initial_state    DEVICE, fp32 [B,H,dk,dv], 16-byte aligned, or NULL for a zero state   (read)
 *
 * Everything else as gla_fwd_ex; GLA_ERR_SHAPE for an unknown layout.  With the MFMA
 * engine a (batch, head) view must span less than 2 GiB (T * H * max(dk, dv) * 4 bytes
 * in BTHD order), otherwise the call falls back to the recurrent engine.
 */
int gla_fwd_layout(const void *q, const void *k, const void *v, const float *log_alpha,
                   int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                   int qkv_dtype, int out_dtype, int layout, const float *initial_state,
                   void *out, float *final_state,
                   void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_fwd_gates - the recurrence with the full gate matrix of Sec. 3.1, G_t = alpha_t^T beta_t
 * (Eq. (gate_gla) for the key side, Eq. (gate_gla_2) for the value side), applied element-wise
 * in Eq. (attn_gla) row 1:   S_t = (alpha_t^T beta_t) * S_{t-1} + k_t^T v_t ,  o_t = q_t S_t.
 *
 *   log_beta         DEVICE, fp32, shaped and laid out like v ([B,H,T,dv] or [B,T,H,dv]), 16-byte
 *                    aligned; log of the value-side gate, <= 0                                  (read)
 *
 * Everything else as gla_fwd_layout (log_beta = 0 gives its result).  bf16 q, k, v with
 * dk % 4 == 0, dv % 8 == 0, dk <= 40 and dv <= 80 run on the MFMA engine (chunk form with both
 * decays factorised: the values are gated like the keys and carried as bf16 hi/lo pairs); every
 * other element type and head size runs on the token-by-token fp32 engine.
 * GLA_ERR_UNSUPPORTED if the engine option forces the MFMA engine
 * onto a case it does not cover, GLA_ERR_NULL for a NULL log_beta.
 */
int gla_fwd_gates(const void *q, const void *k, const void *v, const float *log_alpha, const float *log_beta,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, int out_dtype, int layout, const float *initial_state,
                  void *out, float *final_state, void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_bwd - gradients of a scalar loss L that depends on `out` of gla_fwd_ex (zero initial
 * state, [B,H,T,d] order) with respect to q, k, v and log_alpha: Eq. (attn_gla) rows 1-3
 * differentiated in reverse mode.  With S_s the state after scan step s and
 * G_s = q_s^T dO_s + diag(alpha_{s+1}) G_{s+1} the gradient that reaches it:
 *   dq_s = S_s dO_s^T,  dk_s = G_s v_s^T,  dv_s = k_s G_s,
 *   dlog_alpha_s = sum over scan steps s' >= s of (q_s' * dq_s' - k_s' * dk_s').
 *
 *   q, k, v, d_out   DEVICE, qkv_dtype (d_out = dL/d out, shaped like v)              (read)
 *   log_alpha        DEVICE, fp32                                                     (read)
 *   dq, dk_grad, dlog_alpha   DEVICE, fp32 [B,H,T,dk];  dv_grad  DEVICE, fp32 [B,H,T,dv]   (written)
 *   workspace        DEVICE, 16-byte aligned, gla_bwd_workspace_bytes(...) bytes.  (From fwd_workspace_bytes plus
 *                    4 dk B H ceil(T / 256) bytes, both rounded up to 256, on the call works as well; where what one
 *                    walk leaves for the other then has no room it takes three kernels more.)
 *
 * Same status codes as gla_fwd_ex.  Never allocates.
 */
int gla_bwd(const void *q, const void *k, const void *v, const float *log_alpha, const void *d_out,
            int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir, int qkv_dtype,
            float *dq, float *dk_grad, float *dv_grad, float *dlog_alpha,
            void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_bwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype);

/*
 * gla_bwd_gates - gla_bwd for the recurrence of gla_fwd_gates (two-sided gate alpha_t^T beta_t,
 * zero initial state, [B,H,T,d] order).  The gradient that reaches the state obeys
 * G_s = q_s^T dO_s + (alpha_{s+1}^T beta_{s+1}) * G_{s+1}; dq, dk, dv as in gla_bwd, and
 *   dlog_alpha_s = sum over s' >= s of (q_s' * dq_s' - k_s' * dk_s'),
 *   dlog_beta_s  = sum over s' >= s of (o_s' * dO_s' - v_s' * dv_s')      (o = the forward outputs,
 *                                                                           recomputed in the workspace).
 *
 *   log_beta         DEVICE, fp32 [B,H,T,dv]                                           (read)
 *   out_fwd          DEVICE, fp32 [B,H,T,dv]: `out` of gla_fwd_gates on the same inputs, or NULL
 *                    (the outputs are then recomputed, one more pass over the sequence)          (read)
 *   dlog_beta        DEVICE, fp32 [B,H,T,dv]                                           (written)
 *   workspace        DEVICE, 16-byte aligned, gla_bwd_gates_workspace_bytes(...) bytes.  (From fwd_workspace_bytes plus
 *                    4 max(dk, dv) B H ceil(T / 256) bytes plus 4 dv B H T bytes, each rounded up to 256, on the call
 *                    works as well; where what one walk leaves for the other then has no room it takes more kernels.)
 *
 * Everything else as gla_bwd.  Engines as gla_fwd_gates (MFMA chunk form for bf16 rows with
 * dk % 4 == 0, dv % 8 == 0, dk <= 40, dv <= 80; token by token in fp32 otherwise).  Never allocates.
 */
int gla_bwd_gates(const void *q, const void *k, const void *v, const float *log_alpha, const float *log_beta,
                  const void *d_out, const float *out_fwd, int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, float *dq, float *dk_grad, float *dv_grad, float *dlog_alpha, float *dlog_beta,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_bwd_gates_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype);

/*
 * gla_bwd_reuse - gla_bwd that takes the span states of S from the workspace of the forward
 * call instead of recomputing them (one of the two state passes of the backward pass is the
 * state pass of the forward pass).
 *
 *   fwd_workspace        DEVICE, the workspace that gla_fwd_ex / gla_fwd_layout (same layout, no
 *                        initial state) / gla_fwd_multi's last scan order used for the SAME
 *                        q, k, v, log_alpha, sizes and scan_dir, untouched since that call, and
 *                        with the same gla_set_option values in force as then               (read)
 *   fwd_workspace_bytes  its size, at least gla_fwd_workspace_bytes(...)
 *
 * Everything else as gla_bwd; `workspace` must be a different buffer.  The library cannot
 * check that the forward workspace belongs to these tensors: a stale one gives wrong dq.
 * Of a (batch, head) sequence that left the range of the fp16 MFMA engine (see above) the forward
 * call's outputs are right, but the span states that its fp16 passes left are not: where gates
 * close that fast, take gla_bwd, or GLA_ENGINE_MFMA for both calls; dq and dlog_alpha of such a
 * sequence can be wrong or not finite otherwise.
 */
int gla_bwd_reuse(const void *q, const void *k, const void *v, const float *log_alpha, const void *d_out,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir, int qkv_dtype,
                  const void *fwd_workspace, size_t fwd_workspace_bytes,
                  float *dq, float *dk_grad, float *dv_grad, float *dlog_alpha,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_bwd_layout - gla_bwd / gla_bwd_reuse for either memory order: the backward pass of
 * gla_fwd_layout with a zero initial state (Eq. (attn_gla) rows 1-3 differentiated).
 *
 *   layout           gla_layout of q, k, v, log_alpha, d_out and of the four gradients
 *   fwd_workspace    as in gla_bwd_reuse, or NULL to recompute the span states (then
 *                    fwd_workspace_bytes is ignored)
 *
 * Everything else as gla_bwd; GLA_ERR_SHAPE for an unknown layout.
 */
int gla_bwd_layout(const void *q, const void *k, const void *v, const float *log_alpha, const void *d_out,
                   int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir, int qkv_dtype,
                   int layout, const void *fwd_workspace, size_t fwd_workspace_bytes,
                   float *dq, float *dk_grad, float *dv_grad, float *dlog_alpha,
                   void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_srem_dwconv - the 3x3 depth-wise convolution of the spatial reorient & enhancement
 * module (Sec. 3.3, Algorithm 1: DWConv2d on the 2-D token matrix; every channel has its own
 * 3x3 kernel, zero padding of one token, stride one; the paper initialises it to the identity).
 *   y[b, r, c, d] = bias[d] + sum over dy, dx in {-1,0,1} of weight[d, dy+1, dx+1] * x[b, r+dy, c+dx, d]
 * for orient = 0.  The paper permutes the token sequence between blocks; here tensors stay in
 * canonical row-major order and `orient` (a gla_scan_dir) names the order the paper's sequence
 * would be in, so that the result equals: permute, reshape to 2-D, convolve, flatten, un-permute.
 *
 *   x        DEVICE, x_dtype [B, grid_h*grid_w, D], 16-byte aligned                  (read)
 *   weight   DEVICE, fp32 [D, 3, 3]                                                  (read)
 *   bias     DEVICE, fp32 [D], or NULL                                               (read)
 *   y        DEVICE, y_dtype [B, grid_h*grid_w, D], 16-byte aligned, not x           (written)
 *
 * Status codes as gla_fwd_ex.  Needs no workspace and never allocates.
 */
int gla_srem_dwconv(const void *x, const float *weight, const float *bias, int B, int grid_h, int grid_w, int D,
                    int orient, int x_dtype, int y_dtype, void *y, gla_stream_t stream);

/*
 * gla_fwd_multi - multi-directional scanning (supplement, Algorithms 2 and 3): the sum over
 * several scan orders of the outputs of gla_fwd_ex on the same q, k, v, log_alpha, every
 * term in canonical token order:  out = sum over d in scan_mask of gla_fwd_ex(..., scan_dir = d).
 *
 *   scan_mask   bit d set (d = gla_scan_dir): scan order d takes part; 0x3 is the
 *               bidirectional variant, 0xF the 4-directional one; 1..15
 *   out         DEVICE, fp32 [B,H,T,dv]                                              (written)
 *
 * q, k, v, log_alpha, sizes, workspace (gla_fwd_workspace_bytes) and stream as gla_fwd_ex;
 * no final state is returned (each scan order ends in its own).  The scan orders run one
 * after the other on `stream`; the first writes `out`, the others add to it.  Same status
 * codes as gla_fwd_ex, GLA_ERR_SHAPE for a mask outside 1..15.  Never allocates.
 */
int gla_fwd_multi(const void *q, const void *k, const void *v, const float *log_alpha,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, unsigned scan_mask,
                  int qkv_dtype, float *out, void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_fwd_fused - gla_fwd_ex with the gate computed from its pre-activation inside the kernels
 * and, optionally, the output gate and normalisation applied before the store:
 *   log alpha_t = logsigmoid(z_t) / tau                  (Eq. (gate_gla), alpha = sigmoid(z)^(1/tau))
 *   y_t = Swish(r_t) * LN(o_t),  Swish(x) = x sigmoid(x)  (Eq. (attn_gla) rows 4-5, up to the projection W_O)
 * LN takes mean and (biased) variance over the dv entries of one head's o_t, adds ln_eps
 * under the square root, and applies weight and bias rows of that head.
 *
 *   z_alpha     DEVICE, qkv_dtype [B,H,T,dk]: X W_alpha + b_alpha                         (read)
 *   tau         temperature, > 0 (the DiG configurations use 16)
 *   r_pre       DEVICE, qkv_dtype [B,H,T,dv]: X W_r + b_r, or NULL: no epilogue, `out`
 *               receives o_t as in gla_fwd_ex (the three ln_ arguments are then ignored)    (read)
 *   ln_weight, ln_bias   DEVICE, fp32 [H,dv], or NULL for all ones / all zeros            (read)
 *   ln_eps      >= 0
 *
 * Everything else as gla_fwd_ex ([B,H,T,d] order, zero initial state); same status codes,
 * GLA_ERR_SHAPE also for tau <= 0 or ln_eps < 0.  Never allocates.
 */
int gla_fwd_fused(const void *q, const void *k, const void *v, const void *z_alpha, float tau,
                  const void *r_pre, const float *ln_weight, const float *ln_bias, float ln_eps,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, int out_dtype, void *out, float *final_state,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_fwd_fused_gates - gla_fwd_fused with the value-side gate as well, also from its
 * pre-activation (Eq. (gate_gla_2): beta = sigmoid(z_beta)^(1/tau), same temperature):
 * the mixer of Sec. 3.1 from the projections' outputs to the input of W_O in one call.
 *
 *   z_beta      DEVICE, qkv_dtype [B,H,T,dv]: X W_beta + b_beta, 16-byte aligned          (read)
 *
 * Everything else as gla_fwd_fused; engines as gla_fwd_gates.  GLA_ERR_NULL for a NULL z_beta.
 */
int gla_fwd_fused_gates(const void *q, const void *k, const void *v, const void *z_alpha, const void *z_beta, float tau,
                        const void *r_pre, const float *ln_weight, const float *ln_bias, float ln_eps,
                        int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                        int qkv_dtype, int out_dtype, void *out, float *final_state,
                        void *workspace, size_t workspace_bytes, gla_stream_t stream);

/*
 * gla_decay_fwd - linear attention with one decay a head:
 *
 *     S_t = a_t S_{t-1} + k_t^T v_t ,     o_t = q_t S_t ,     S_0 = initial_state or zero
 *
 * with a_t = exp(log_decay) a number: Eq. (attn_gla) with the gate row alpha_t replaced by one decay, constant for a
 * head or given for each token.  No gate rows are read, queries and keys may be rotated (gla_rope; a scalar commutes
 * with the rotation, a gate row does not), and heads may be wider: 1 <= dk, dv <= 128.
 *
 *   q, k, v        DEVICE, qkv_dtype, in `layout` ([B,H,T,d] or [B,T,H,d])                                    (read)
 *   log_decay      DEVICE, fp32, 16-byte aligned, <= 0 down to -inf (a gate of zero)                          (read)
 *   decay_kind     a gla_decay_kind: log_decay is [H], or one for each token in the order of `layout`
 *                  ([B,H,T] or [B,T,H])
 *   seq_lens       DEVICE, int32 [B], 0 .. T, or NULL: all T.  Sequence b ends after seq_lens[b] tokens: it is walked
 *                  as if it were that long (ROW_REV begins at its own last token), its final state is the one after
 *                  them, the rows behind them may hold anything and those of `out` are left as they were.  A length of
 *                  0 gives the initial state as final state.  Values outside 0 .. T count as the nearer end.
 *                  Row scans only (GLA_ERR_UNSUPPORTED)                                                       (read)
 *   grid_h, grid_w, scan_dir   as in gla_fwd; for text and the like grid_h = 1, grid_w = T, GLA_SCAN_ROW_FWD
 *   initial_state  DEVICE, fp32 [B,H,dk,dv] or NULL                                                           (read)
 *   out            DEVICE, out_dtype, shaped and laid out like v                                              (written)
 *   final_state    DEVICE, fp32 [B,H,dk,dv] or NULL; may be initial_state, GLA_ERR_SHAPE where the two overlap
 *                  otherwise                                                                                  (written)
 *   workspace      DEVICE, 16-byte aligned, gla_decay_fwd_workspace_bytes(...) bytes (0 for many sequences: then it
 *                  may be NULL)
 *
 * bf16 calls run on bf16 MFMA with every factor that is not an input carried as two bf16 numbers: fp32 outputs are within
 * 3e-6 of their size (2-norm).  With a final state what the states take up is three, and final states are as exact as
 * fp32 arithmetic leaves them (4e-7).  fp32 calls run on fp32 MFMA; pass bf16 rows as fp32 for these digits throughout.
 * Gates have no lower limit; one that is NaN makes NaN of all that it has a part in.  Inputs of visited rows have to be
 * finite.  T is at most 2^30.  Tuning options have no effect.
 * Never allocates; nothing is kept between calls.  `out` must not overlap the inputs.  Calls that may overlap, captured ones
 * among them, need workspaces of their own.
 */
typedef enum { GLA_DECAY_HEAD = 0, GLA_DECAY_TOKEN = 1 } gla_decay_kind;
int gla_decay_fwd(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind, const int *seq_lens,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, int out_dtype, int layout, const float *initial_state, void *out, float *final_state,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_decay_fwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype);

/*
 * gla_decay_bwd - gradients of a loss that depends on `out` and, through d_final_state, on the final state of
 * gla_decay_fwd.  With G_t = q_t^T dO_t + a_{t+1} G_{t+1} the adjoint state (behind the last token d_final_state):
 *   dq_t = S_t dO_t^T,  dk_t = G_t v_t^T,  dv_t = k_t G_t,  dlog a_t = <a_t S_{t-1}, G_t>,  d S_0 = a_1 G_1.
 *
 *   d_out            DEVICE, qkv_dtype, like v                                                                (read)
 *   d_final_state    DEVICE, fp32 [B,H,dk,dv] or NULL: zero                                                   (read)
 *   dq, dk_grad, dv_grad   DEVICE, grad_dtype, like q, k, v; rows behind a sequence's end are cleared         (written)
 *   dlog_decay       DEVICE, fp32, like log_decay (cleared behind a sequence's end; for GLA_DECAY_HEAD the sum over
 *                    batches and tokens, always added in one order), or NULL: not wanted                      (written)
 *   d_initial_state  DEVICE, fp32 [B,H,dk,dv], or NULL: not wanted                                            (written)
 *   workspace        DEVICE, 16-byte aligned, gla_decay_bwd_workspace_bytes(...) bytes
 *
 * With dlog_decay of GLA_DECAY_HEAD bf16 calls carry three bf16 numbers instead of two throughout (45 % more time): that sum over
 * all steps would add up the errors of two.  With GLA_DECAY_TOKEN it is within 1e-5 of its size from bf16 rows, 1e-6 from fp32;
 * a gate's gradient is as exact as the largest of its 256 steps.  d_initial_state is as exact as a final state.  Everything
 * else as gla_decay_fwd.  Outputs must not alias inputs.
 */
int gla_decay_bwd(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind, const int *seq_lens,
                  const void *d_out, const float *initial_state, const float *d_final_state,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, int grad_dtype, int layout, void *dq, void *dk_grad, void *dv_grad, float *dlog_decay,
                  float *d_initial_state, void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_decay_bwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype);

/*
 * gla_decay_step - one token of gla_decay_fwd for each of B sequences:
 *   state_out = a state + k^T v,   out = q state_out.
 *
 *   q, k [B,H,dk], v [B,H,dv]   DEVICE, qkv_dtype                                                             (read)
 *   log_decay   DEVICE, fp32 [H] or (GLA_DECAY_TOKEN) [B,H]                                                   (read)
 *   state       DEVICE, fp32 [B,H,dk,dv], 16-byte aligned                                                     (read)
 *   state_out   the same; may be `state` (in place), GLA_ERR_SHAPE where the two overlap otherwise            (written)
 *   out         DEVICE, out_dtype [B,H,dv]                                                                    (written)
 *
 * q, k, v, log_decay and out may begin at any element.  Arithmetic in fp32.  Needs no workspace and never allocates.
 */
int gla_decay_step(const void *q, const void *k, const void *v, const float *log_decay, int decay_kind,
                   int B, int H, int dk, int dv, int qkv_dtype, int out_dtype, const float *state, float *state_out,
                   void *out, gla_stream_t stream);

/*
 * gla_rope - rotary positions with one or several axes.  The first channels of a head fall into sections, one an axis;
 * pair i of the section of axis x with w channels is turned by the angle position_x * base^(-2 i / w):
 *   (u, v) -> (u cos - v sin, v cos + u sin).
 * Channels behind the sections are copied.
 *
 *   q, k        DEVICE, dtype, [B,H,T,d] or [B,T,H,d] by `layout`; k (and out_k) may be NULL                  (read)
 *   positions   DEVICE, int32 [B,T,axes], or NULL: from the grid, for one axis the token's number, for two its row and
 *               column (T = grid_h * grid_w), for three frame, row and column (T a multiple of it)            (read)
 *   sections    HOST, axes even numbers whose sum is at most d
 *   axes        1 .. 4 (1 .. 3 without positions)
 *   base        > 0, finite; 10000 as a rule
 *   pairing     a gla_rope_pairing: a pair is two neighbouring channels, or channel i and i + w/2 of a section
 *   inverse     not 0: turned back, which is also the backward pass
 *   out_q, out_k   DEVICE, dtype, like q and k; may be q and k (GLA_ERR_SHAPE: out_q = k, out_k = q or out_q = out_k, and where an
 *               output overlaps another tensor otherwise)                                                       (written)
 *
 * 1 <= d <= 256.  Frequencies restart with every section.  Angles are formed and reduced from frequencies in two 64-bit numbers: with a base of 1 or
 * more every position of 32 bits is as exact as the first, with less an angle is off by up to 2^-25 / base besides.  grid_h, grid_w are
 * ignored with positions or one axis.  Needs no workspace and never allocates.
 */
typedef enum { GLA_ROPE_ADJACENT = 0, GLA_ROPE_HALVES = 1 } gla_rope_pairing;
int gla_rope(const void *q, const void *k, const int *positions, const int *sections, int axes, float base, int pairing,
             int inverse, int B, int H, int T, int d, int grid_h, int grid_w, int dtype, int layout,
             void *out_q, void *out_k, gla_stream_t stream);

/*
 * gla_norm_fwd - layer norm of rows of D channels, and with r_pre the output gate behind it (Eq. (attn_gla) rows 4-5, what
 * gla_fwd_fused has as its epilogue):   y = LN(x) weight + bias,   out = y, or Swish(r) y.
 *
 *   x           DEVICE, x_dtype, [B,H,T,D] or [B,T,H,D] by `layout`; H = 1 for tokens                         (read)
 *   weight, bias   DEVICE, fp32 [H,D], or NULL: ones, zeros                                                   (read)
 *   eps         >= 0, under the square root
 *   r_pre       DEVICE, x_dtype, like x, or NULL: no gate                                                     (read)
 *   out         DEVICE, out_dtype, like x; may be x or r_pre if the element types agree, GLA_ERR_SHAPE where it overlaps
 *               them otherwise                                                                                  (written)
 *
 * 1 <= D <= 8192.  Statistics in fp32.  Needs no workspace and never allocates.
 */
int gla_norm_fwd(const void *x, const float *weight, const float *bias, float eps, const void *r_pre,
                 int B, int H, int T, int D, int x_dtype, int out_dtype, int layout, void *out, gla_stream_t stream);

/*
 * gla_norm_bwd - gradients of gla_norm_fwd; mean and variance are taken from x again.
 *
 *   d_out           DEVICE, x_dtype, like x                                                                   (read)
 *   dx              DEVICE, grad_dtype, like x                                                                (written)
 *   dr              DEVICE, grad_dtype, like x; NULL exactly if r_pre is                                      (written)
 *   dweight, dbias  DEVICE, fp32 [H,D], both or neither (NULL: not wanted); sums over batches and tokens, always added in
 *                   one order                                                                                 (written)
 *   workspace       DEVICE, 16-byte aligned, gla_norm_bwd_workspace_bytes(...) bytes (written only for dweight, dbias)
 *
 * Everything else as gla_norm_fwd.  Outputs must not alias inputs.
 */
int gla_norm_bwd(const void *x, const void *d_out, const float *weight, const float *bias, float eps, const void *r_pre,
                 int B, int H, int T, int D, int x_dtype, int grad_dtype, int layout, void *dx, void *dr,
                 float *dweight, float *dbias, void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_norm_bwd_workspace_bytes(int B, int H, int T, int D);

/*
 * gla_recur_fwd - gated recurrence of channels:
 *
 *     h_t = a_t h_{t-1} + u_t ,     u_t = x_t or (1 - a_t) x_t ,     out = h ,     h_0 = initial_state or zero
 *
 * with a gate a_t for every channel and token: a mixer whose state is one number a channel.
 *
 *   x              DEVICE, x_dtype, [B,T,D]                                                                   (read)
 *   gate           DEVICE, [B,T,D] (read): by gate_kind (a gla_gate_kind)
 *                  GLA_GATE_LOG: log a in fp32, <= 0 down to -inf (a gate of zero)
 *                  GLA_GATE_PRE: z in x_dtype, a = sigmoid(z)^(1/tau)   (Eq. (gate_gla))
 *   tau            from 2^-64 on, finite; ignored for GLA_GATE_LOG
 *   complement     not 0: u_t = (1 - a_t) x_t
 *   seq_lens       DEVICE, int32 [B], 0 .. T, or NULL: all T; as in gla_decay_fwd (row scans only): rows behind a sequence's end may hold
 *                  anything and those of `out` are left as they were                                          (read)
 *   grid_h, grid_w, scan_dir   as in gla_fwd; for text and the like grid_h = 1, grid_w = T, GLA_SCAN_ROW_FWD
 *   initial_state  DEVICE, fp32 [B,D] or NULL                                                                 (read)
 *   out            DEVICE, out_dtype, [B,T,D]; may be x or the gate if the element types agree, GLA_ERR_SHAPE where it overlaps them
 *                  otherwise                                                                                  (written)
 *   final_state    DEVICE, fp32 [B,D] or NULL; may be initial_state, GLA_ERR_SHAPE where the two overlap otherwise   (written)
 *   workspace      DEVICE, 16-byte aligned, gla_recur_fwd_workspace_bytes(...) bytes (0: may be NULL)
 *
 * Arithmetic in fp32, gates summed as logarithms: memories of any length are as exact as short ones.  Inputs of visited rows have to be
 * finite, but for gates of zero; a NaN makes NaN of what comes after it in its channel.  Tensors 16-byte aligned.  Never
 * allocates; nothing is kept between calls.  Calls that may overlap, captured ones among them, need workspaces of their own.
 *
 * T up to 2^30, D up to 2^26, and with c = ceil(D / 128) for even D, ceil(D / 64) for odd D: B c < 2^23, where T > 256 and B D < 2^15 (odd D: 2^14) also
 * B c ceil(T / 128) < 2^23; gla_recur_bwd: B c ceil(T / 64) < 2^23, and for T > 64 B ceil(D / 64) < 2^22.  Others are refused (GLA_ERR_UNSUPPORTED), but
 * for some of few channels, of which several sequences share a work-group.
 */
typedef enum { GLA_GATE_LOG = 0, GLA_GATE_PRE = 1 } gla_gate_kind;
int gla_recur_fwd(const void *x, const void *gate, int gate_kind, float tau, int complement, const int *seq_lens,
                  int B, int T, int D, int grid_h, int grid_w, int scan_dir, int x_dtype, int out_dtype,
                  const float *initial_state, void *out, float *final_state, void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_recur_fwd_workspace_bytes(int B, int T, int D);

/*
 * gla_recur_bwd - gradients of a loss that depends on `out` and, through d_final_state, on the final state of gla_recur_fwd.  With
 * G_t = dO_t + a_{t+1} G_{t+1} (behind the last token d_final_state):
 *   dx_t = G_t or (1 - a_t) G_t,  dlog a_t = a_t (h_{t-1} - (0 or x_t)) G_t,  dz_t = dlog a_t sigmoid(-z_t) / tau,  d h_0 = a_1 G_1.
 *
 *   d_out            DEVICE, x_dtype, like x                                                                  (read)
 *   d_final_state    DEVICE, fp32 [B,D] or NULL: zero                                                         (read)
 *   dx, d_gate       DEVICE, grad_dtype, [B,T,D]; the gradient of what `gate` holds; rows behind a sequence's end are cleared   (written)
 *   d_initial_state  DEVICE, fp32 [B,D], or NULL: not wanted                                                  (written)
 *   workspace        DEVICE, 16-byte aligned, gla_recur_bwd_workspace_bytes(...) bytes (0: may be NULL)
 *
 * The states are formed again from x and the gates.  Everything else as gla_recur_fwd.  Outputs must not overlap inputs (GLA_ERR_SHAPE).
 */
int gla_recur_bwd(const void *x, const void *gate, int gate_kind, float tau, int complement, const int *seq_lens, const void *d_out,
                  const float *initial_state, const float *d_final_state, int B, int T, int D, int grid_h, int grid_w, int scan_dir,
                  int x_dtype, int grad_dtype, void *dx, void *d_gate, float *d_initial_state,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_recur_bwd_workspace_bytes(int B, int T, int D);

/*
 * gla_recur_step - one token of gla_recur_fwd for each of B sequences: state_out = a state + u, out = state_out.
 *
 *   x [B,D], gate [B,D], state [B,D]   DEVICE, as in gla_recur_fwd                                            (read)
 *   state_out   DEVICE, fp32 [B,D]; may be `state` (in place), GLA_ERR_SHAPE where the two overlap otherwise  (written)
 *   out         DEVICE, out_dtype [B,D]; must not overlap the others (GLA_ERR_SHAPE)                          (written)
 *
 * x, gate and out may begin at any element, the states at 16 bytes.  Needs no workspace and never allocates.
 */
int gla_recur_step(const void *x, const void *gate, int gate_kind, float tau, int complement, int B, int D, int x_dtype, int out_dtype,
                   const float *state, float *state_out, void *out, gla_stream_t stream);

/*
 * gla_qk_norm_fwd - norm of each head's query and key row by its root mean square, and the rotation of gla_rope behind it, in one pass:
 *   n = x / sqrt(mean(x^2) + eps),   y = R (n weight).
 *
 *   q, k        DEVICE, dtype, rows of d channels: B x H x T of queries, B x Hk x T of keys; k (and out_k) may be NULL   (read)
 *   q_strides, k_strides   HOST, elements from one batch, head and token to the next (0 and more; a packed projection's rows, say), or
 *               NULL: dense, [B,H,T,d] or [B,T,H,d] by `layout`
 *   q_weight, k_weight   DEVICE, fp32 [d], shared by the heads, or NULL: ones                                 (read)
 *   eps         >= 0, finite, under the square root
 *   positions, sections, axes, base, pairing, grid_h, grid_w   as in gla_rope; axes = 0: no rotation (sections may be NULL)
 *   out_q, out_k   DEVICE, out_dtype, dense in `layout`; may be q and k if these are dense and the element types agree, GLA_ERR_SHAPE where
 *               they overlap the inputs or each other otherwise                                                 (written)
 *
 * 1 <= d <= 256.  q and k may begin at any element, the other tensors at 16 bytes.  Sums and angles as in gla_norm_fwd and gla_rope; a row's
 * squares have to add up to a finite fp32 number, and their mean and eps to no less than 2^-126: a row that is all but zero needs an eps.  Needs no workspace and never allocates.
 */
int gla_qk_norm_fwd(const void *q, const long long *q_strides, int H, const void *k, const long long *k_strides, int Hk, const float *q_weight,
                    const float *k_weight, float eps, const int *positions, const int *sections, int axes, float base, int pairing,
                    int B, int T, int d, int grid_h, int grid_w, int dtype, int out_dtype, int layout, void *out_q, void *out_k,
                    gla_stream_t stream);

/*
 * gla_qk_norm_bwd - gradients of gla_qk_norm_fwd; norms and angles are formed again.
 *
 *   d_out_q, d_out_k   DEVICE, dtype, dense in `layout`; the latter NULL exactly if k is                      (read)
 *   dq, dk      DEVICE, grad_dtype, dense in `layout`                                                         (written)
 *   dq_weight, dk_weight   DEVICE, fp32 [d], or NULL: not wanted; sums over batches, heads and tokens, always added in one order   (written)
 *   workspace   DEVICE, 16-byte aligned, gla_qk_norm_bwd_workspace_bytes(...) bytes (Hk = 0 without keys); may be NULL where neither
 *               weight's gradient is wanted
 *
 * Everything else as gla_qk_norm_fwd.  Outputs must not overlap inputs (GLA_ERR_SHAPE).
 */
int gla_qk_norm_bwd(const void *q, const long long *q_strides, int H, const void *k, const long long *k_strides, int Hk,
                    const void *d_out_q, const void *d_out_k, const float *q_weight, const float *k_weight, float eps,
                    const int *positions, const int *sections, int axes, float base, int pairing, int B, int T, int d, int grid_h, int grid_w,
                    int dtype, int grad_dtype, int layout, void *dq, void *dk, float *dq_weight, float *dk_weight,
                    void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_qk_norm_bwd_workspace_bytes(int B, int H, int Hk, int T, int d);

/*
 * gla_glu_fwd - gated feed-forward product: both projections of M tokens, the activation and the product, without the projections' way through memory:
 *   out = act(x w_gate^T) * (x w_up^T).
 *
 *   x              DEVICE, dtype, [M,K]                                                                       (read)
 *   w_gate, w_up   DEVICE, dtype, [F,K]                                                                       (read)
 *   act            a gla_activation: Swish(g) = g sigmoid(g), GELU g Phi(g), or GELU with
 *                  Phi(g) ~ (1 + tanh(sqrt(2/pi) (g + 0.044715 g^3))) / 2
 *   out            DEVICE, out_dtype, [M,F]                                                                   (written)
 *   pre            DEVICE, fp32 [2,M,F], or NULL: the two products before the activation, for gla_glu_bwd     (written)
 *   workspace      DEVICE, 16-byte aligned, gla_glu_fwd_workspace_bytes(...) bytes (0 where rows of K are whole pieces of 16 bytes: may be
 *                  NULL; else for copies whose rows are)
 *
 * Sums in fp32 (bf16 or fp32 MFMA).  Tensors 16-byte aligned.  Outputs must not overlap inputs or each other (GLA_ERR_SHAPE).  K, F up to 2^20,
 * M up to 2^28, M (max(K, F) + 8) < 2^34 and F (K + 8) < 2^32: others are refused (GLA_ERR_UNSUPPORTED).  Never allocates;
 * nothing is kept between calls.  Calls that may overlap, captured ones among them, need workspaces of their own.
 */
typedef enum { GLA_ACT_SILU = 0, GLA_ACT_GELU = 1, GLA_ACT_GELU_TANH = 2 } gla_activation;
int gla_glu_fwd(const void *x, const void *w_gate, const void *w_up, int M, int K, int F, int act, int dtype, int out_dtype,
                void *out, float *pre, void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_glu_fwd_workspace_bytes(int M, int K, int F, int dtype);

/*
 * gla_glu_bwd - gradients of gla_glu_fwd.  With g, u the two products, dg = d_out u act'(g) and du = d_out act(g):
 *   dx = dg w_gate + du w_up,   dw_gate = dg^T x,   dw_up = du^T x.
 *
 *   d_out       DEVICE, dtype, [M,F]                                                                          (read)
 *   pre         DEVICE, what gla_glu_fwd left there for the same inputs, or NULL: the products are formed again   (read)
 *   dx          DEVICE, dtype, [M,K], or NULL: not wanted                                                     (written)
 *   dw_gate, dw_up   DEVICE, dtype, [F,K], both or neither (NULL: not wanted)                                 (written)
 *   workspace   DEVICE, 16-byte aligned, gla_glu_bwd_workspace_bytes(...) bytes
 *
 * Gradients have the inputs' element type.  From bf16, dg and du are rounded to bf16 once as operands: gradients are off by 1.4 times what
 * their own rounding takes (2.3e-3 in the 2-norm, not 1.7e-3); GLA_OPT_GLU_SPLIT takes them as two numbers each.  Sums are always added in
 * one order.  Everything else as gla_glu_fwd.
 */
int gla_glu_bwd(const void *x, const void *w_gate, const void *w_up, const void *d_out, const float *pre, int M, int K, int F, int act,
                int dtype, void *dx, void *dw_gate, void *dw_up, void *workspace, size_t workspace_bytes, gla_stream_t stream);
size_t gla_glu_bwd_workspace_bytes(int M, int K, int F, int dtype);

/* Bytes of workspace gla_fwd_ex / gla_fwd_layout need for this problem (an upper bound over all
 * launch plans, so it does not depend on tuning options).  0 on invalid sizes. */
size_t gla_fwd_workspace_bytes(int B, int H, int T, int dk, int dv, int qkv_dtype);

/*
 * gla_fwd_timed - measurement aid: runs gla_fwd_ex `iters` times on `stream`
 * with HIP events around each of the three phases of the chunk-parallel plan
 * (Sec. 3.5 cut into spans: local span states, carry across spans, outputs) and
 * returns mean milliseconds per call in phase_ms (HOST pointer to 4 floats:
 * span-state kernel, carry kernel, output kernel, whole call).  Synchronises
 * the stream before returning.  Phases a plan skips report 0 (a call in one launch has
 * an output kernel only).
 */
int gla_fwd_timed(const void *q, const void *k, const void *v, const float *log_alpha,
                  int B, int H, int T, int dk, int dv, int grid_h, int grid_w, int scan_dir,
                  int qkv_dtype, int out_dtype, void *out, float *final_state,
                  void *workspace, size_t workspace_bytes, gla_stream_t stream,
                  int iters, float *phase_ms);

/*
 * gla_calibrate_mfma - measurement aid: the rate at which this GPU retires v_mfma_f32_16x16x32_bf16 when nothing
 * else limits it (every wave of a grid that fills the chip runs a loop of eight independent accumulator chains
 * held in registers, no memory traffic), in TFLOP/s (2 flops per multiply-add), written to *tflops (HOST pointer).
 * It is the figure to hold next to the published dense bf16 peak when a kernel's MFMA rate is priced.  Runs on
 * `stream`, synchronises it before returning, allocates 4 KiB of device memory for the duration of the call.
 * GLA_ERR_NULL for a NULL pointer, GLA_ERR_HIP if a runtime call fails.
 */
int gla_calibrate_mfma(double *tflops, gla_stream_t stream);

/* Process-wide tuning knobs; returns GLA_ERR_SHAPE for an unknown option or value.  They are plain process
 * globals read at the start of every call: set them before, not while, other threads call the library. */
int gla_set_option(int option, int value);
int gla_get_option(int option);

/*
 * gla_block_scan_dir - the scan order that DiG block `block` uses (Sec. 3.3, Algorithm 1: after every block the
 * token matrix is transposed, for even block indices, or the sequence flipped, for odd ones; supplement,
 * Algorithm 4 states the same schedule with the parities swapped).  This library leaves the tokens in canonical
 * row-major order and folds those permutations into `scan_dir` of the gla_fwd* / gla_bwd* calls and `orient` of
 * gla_srem_dwconv; this function names the order a block sees:
 *   GLA_SCHEDULE_BLOCK_PROCESS (Algorithm 1):  block 1, 2, 3, 4, 5 ... -> ROW_FWD, ROW_REV, COL_REV, COL_FWD, ROW_FWD ...
 *   GLA_SCHEDULE_BLOCK_SCAN    (Algorithm 4):  block 1, 2, 3, 4, 5 ... -> ROW_FWD, COL_FWD, COL_REV, ROW_REV, ROW_FWD ...
 * (the paper's reshape2d takes a square token matrix; on a grid_h x grid_w grid the orders are those of
 * gla_scan_dir on that grid).  Host only, no GPU work.
 *
 *   block      1-based index of the block (the paper's l)
 *   schedule   a gla_schedule
 * Returns the gla_scan_dir, or -1 for block < 1 or an unknown schedule.
 */
typedef enum { GLA_SCHEDULE_BLOCK_PROCESS = 0, GLA_SCHEDULE_BLOCK_SCAN = 1 } gla_schedule;
int gla_block_scan_dir(int block, int schedule);

/* Static, NUL-terminated description of a status code. */
const char *gla_status_string(int status);

/* Library version: major * 10000 + minor * 100 + patch. */
int gla_version(void);

#ifdef __cplusplus
}
#endif
#endif /* GLA_H_ */
