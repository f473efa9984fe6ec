/*
 * hla.h -- C ABI of the GB300 (sm_103a) implementation of Higher-order Linear
 * Attention (Zhang, Qin, Wang, Gu, "Higher-order Linear Attention").
 *
 * All entry points take plain pointers and sizes.  Device pointers refer to
 * memory of the current CUDA device; the caller owns every buffer (inputs,
 * outputs, states and the scratch workspace) and the library allocates no
 * device memory.  Work is enqueued asynchronously on `stream`; host-side
 * argument errors are returned synchronously before anything is launched.
 *
 * Common conventions
 * ------------------
 * Tokens are row vectors.  q, k are [B, H, n, d] and v, out are [B, H, n, dv],
 * contiguous, in the element type `dt` (out has the same type as the inputs).
 * Base pointers must be 16-byte aligned.
 *
 * Second-order state of one head (fp32, row-major), the tuple of Fig. 1(A):
 *   [ S (d*d) | C (d*dv) | m (d) | G (d*dv) | h (d) ]
 * with S = sum k k^T, C = sum q v^T, m = sum q, G = sum_i k_i k_i^T C_{i-1},
 * h = sum_i k_i k_i^T m_{i-1} (Sec. 3 and Sec. 3.2).  States of B*H heads are
 * stored back to back in [B, H] order.  With masked = 0 the operator does not
 * use G and h: they are ignored on input and written as zeros on output.
 *
 * Supported shapes: d, dv in {16, 32, 64, 128}; 1 <= chunk <= 128 (chunk is
 * the scan granularity of Theorem 2; the result does not depend on it up to
 * rounding); n >= 0 with any remainder n % chunk (a ragged last chunk).
 * Other values return HLA_ERR_UNSUPPORTED.
 */
#ifndef HLA_H_
#define HLA_H_

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

struct CUstream_st;
/* A CUDA stream (the same object as cudaStream_t); NULL is the legacy default stream. */
typedef struct CUstream_st *hla_stream_t;

typedef enum {
    HLA_OK = 0,
    HLA_ERR_INVALID_ARGUMENT = 1, /* null pointer, negative size, misaligned pointer, bad flag */
    HLA_ERR_UNSUPPORTED = 2,      /* valid request outside the supported shapes/types        */
    HLA_ERR_CUDA = 3,             /* a CUDA runtime call or kernel launch failed              */
    HLA_ERR_TIMEOUT = 4,          /* a device-side wait ran past its budget (hla_poll_error)  */
    HLA_ERR_WORKSPACE = 5         /* workspace missing or smaller than the required size      */
} hla_status;

typedef enum {
    HLA_F32 = 0,  /* IEEE float32 tokens */
    HLA_BF16 = 1  /* bfloat16 tokens (fp32 accumulation everywhere) */
} hla_dtype;

/* Human-readable name of a status code (static storage). */
const char *hla_status_string(hla_status status);

/* Detail of the last error returned on the calling host thread (static,
 * thread-local storage; empty string if none). */
const char *hla_last_error(void);

/* Number of floats of one head's second-order state tuple: d*d + 2*d*dv + 2*d. */
size_t hla2_state_floats(int d, int dv);

/* Bytes of scratch workspace hla2_forward needs for these sizes (any flags).
 * Returns 0 for unsupported sizes. */
size_t hla2_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, hla_dtype dt);

/*
 * hla2_forward -- chunk-parallel forward of second-order HLA over n tokens.
 *
 * Operator (per head, t = 1..n):
 *   masked = 1 (strictly causal, Theorem 1, Eq. masked-unnorm / Eq. masked):
 *     num_t = q_t^T (S_t C_t - G_t),   den_t = q_t^T (S_t m_t - h_t)
 *     = sum_{j<=t} sum_{i<=j} (q_t.k_i)(q_j.k_i) v_j   (and v_j -> 1 for den)
 *   masked = 0 (Eq. hla-unnorm / Eq. hla-row):
 *     num_t = q_t^T S_t C_t,           den_t = q_t^T S_t m_t
 *   out_t = num_t                       if normalized == 0 (the default operator)
 *   out_t = num_t / (den_t + eps)       if normalized == 1 (no clamp, no abs)
 * where the states include token t (inclusive) and start from state_in.  The
 * result equals the serial recurrence (online updates after Theorem 1) by
 * Theorem 2; chunking only changes rounding.
 *
 * q, k, v : device, [B, H, n, d] / [B, H, n, d] / [B, H, n, dv] of type dt (read only)
 * out     : device, [B, H, n, dv] of type dt (written)
 * state_in  : device fp32 [B*H * hla2_state_floats(d,dv)] or NULL (= zero state)
 * state_out : device fp32, same size, or NULL (= not written); receives the
 *             state after token n (Eq. semidirect applied to the whole
 *             sequence).  May equal state_in (read before written).
 * eps     : the stability constant of the normalised output (finite)
 * workspace / workspace_bytes : device scratch of at least
 *             hla2_workspace_bytes(B,H,n,d,dv,chunk,dt) bytes, 256-byte
 *             aligned; its contents on entry are ignored.  Calls that share a
 *             workspace must be ordered on one stream.
 * Errors: HLA_ERR_INVALID_ARGUMENT / UNSUPPORTED / WORKSPACE before launch;
 * HLA_ERR_CUDA if a launch fails.  A device-side wait that exceeds its budget
 * sets a flag in the workspace that hla_poll_error reports as HLA_ERR_TIMEOUT.
 */
hla_status hla2_forward(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                        int B, int H, int n, int d, int dv, int masked, int normalized, float eps,
                        int chunk, const float *state_in, float *state_out,
                        void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * hla2_step -- one streaming decode step of second-order HLA for B*H heads.
 *
 * For each head, with the state tuple (S, C, m, G, h) before the token
 * (online updates after Theorem 1; outputs of Theorem 1 / Eq. hla-row):
 *   masked:  G += k (k^T C),  h += k (k^T m)          (previous C and m)
 *   S += k k^T,  C += q v^T,  m += q
 *   masked:   num = (q^T S) C - q^T G,  den = (q^T S) m - q^T h
 *   unmasked: num = (q^T S) C,          den = (q^T S) m   (G, h untouched)
 *   out = num, or num / (den + eps) if normalized.
 *
 * q, k : device [B, H, d] of type dt; v : device [B, H, dv] of type dt
 * out  : device [B, H, dv] of type dt
 * state: device fp32 [B*H * hla2_state_floats(d,dv)], updated in place
 * Errors as for hla2_forward (no workspace, no device-side waits).
 */
hla_status hla2_step(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                     int B, int H, int d, int dv, int masked, int normalized, float eps,
                     float *state, hla_stream_t stream);

/* Bytes of scratch workspace hla2_backward needs (0 if unsupported). */
size_t hla2_backward_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, hla_dtype dt);

/*
 * hla2_backward -- gradients of the masked second-order forward (from a zero
 * state) for L = sum_t dout_t . out_t: dq, dk, dv.  The paper's training
 * route (Sec. "Chunk-parallel training via associative scans"): the forward
 * prefixes are checkpointed at chunk boundaries and recomputed within a
 * chunk, and the gradient suffixes are carried by a reverse scan with the
 * adjoint of the semidirect product (Eq. semidirect); the result equals the
 * gradients of the serial recurrence (Theorem 2 and the chain rule) up to
 * rounding.  normalized selects out = num / (den + eps) (Eq. masked).
 * q, k, v : device [B, H, n, d] / [B, H, n, d] / [B, H, n, dv] of type dt
 * dout    : device [B, H, n, dv] of type dt (the gradient of the output)
 * dq, dk  : device [B, H, n, d] of type dt (written); dv : [B, H, n, dv] (written)
 * workspace : at least hla2_backward_workspace_bytes(...) bytes, 256-byte aligned.
 * Errors as for hla2_forward.
 */
hla_status hla2_backward(const void *q, const void *k, const void *v, const void *dout, void *dq, void *dk,
                         void *dv, hla_dtype dt, int B, int H, int n, int d, int dv_size, int normalized,
                         float eps, int chunk, void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * The (S, D, e) decode state of the masked operator (no counterpart printed in
 * the paper; it follows from Theorem 1 and Eq. semidirect).  With
 * D = S C - G (d x dv) and e = S m - h (d), Theorem 1's outputs read
 * num_t = q_t^T D_t and den_t = q_t^T e_t, and the online updates after
 * Theorem 1 collapse to
 *   S' = S + k k^T,   x = S' q,   D' = D + x v^T,   e' = e + x.
 * Per head (fp32, row-major): [ S (d*d) | D (d*dv) | e (d) ], heads in [B, H]
 * order.  It carries exactly what the masked outputs need with d*d + d*dv + d
 * floats instead of the tuple's d*d + 2*d*dv + 2*d (a third fewer bytes per
 * decode step at d = dv); the tuple cannot be recovered from it (C, m, G, h
 * are folded together).  This is one of the state-format options of the
 * paper's implementation considerations (Sec. "Implementation details and
 * complexity").
 */
size_t hla2_sde_state_floats(int d, int dv);

/*
 * hla2_state_to_sde -- convert B*H masked second-order tuples (S, C, m, G, h)
 * (hla2_state_floats each, e.g. a state_out of hla2_forward) into (S, D, e)
 * states: D = S C - G, e = S m - h, fp32 on the device.
 * state : device fp32 [B*H * hla2_state_floats(d,dv)] (read only)
 * sde   : device fp32 [B*H * hla2_sde_state_floats(d,dv)] (written); must not
 *         overlap state.  Both 16-byte aligned.
 * Errors: HLA_ERR_INVALID_ARGUMENT (null, misaligned, overlapping),
 * HLA_ERR_UNSUPPORTED (d, dv outside {16, 32, 64, 128}), HLA_ERR_CUDA.
 */
hla_status hla2_state_to_sde(const float *state, float *sde, int B, int H, int d, int dv, hla_stream_t stream);

/*
 * hla2_step_sde -- hla2_step of the masked operator on (S, D, e) states:
 *   S += k k^T;  x = S q;  D += x v^T;  e += x;
 *   num = q^T D,  den = q^T e,  out = num or num / (den + eps).
 * q, k : device [B, H, d] of type dt; v, out : device [B, H, dv] of type dt
 * sde  : device fp32 [B*H * hla2_sde_state_floats(d,dv)], updated in place
 * Errors as for hla2_step.
 */
hla_status hla2_step_sde(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                         int B, int H, int d, int dv, int normalized, float eps,
                         float *sde, hla_stream_t stream);

/*
 * hla2_forward_path -- which CUDA path hla2_forward takes for these arguments
 * on the current device, without launching anything:
 *   0  generic path: fp32 CUDA-core kernels (every supported shape);
 *   1  fused path: one persistent tcgen05/TMA kernel (bf16 tokens, d and dv
 *      in {64, 128}; masked: state_in only with d = dv = 128; unmasked: the
 *      plain output, no states, one SM per head) on sm_103, plus two small kernels for
 *      state_out (C = Q^T V and m = Q^T 1 on the tensor cores, then
 *      G = S C - D, h = S m - e from the forward's prefixes).  It works in
 *      128-token tiles whatever chunk is (chunk only changes the rounding,
 *      Theorem 2);
 *  -1  the arguments are not supported.
 * *launches (if not NULL) receives the number of kernels the call launches.
 */
int hla2_forward_path(int B, int H, int n, int d, int dv, int masked, int normalized, int chunk, hla_dtype dt,
                      int has_state_in, int has_state_out, int *launches);

/* Number of floats of one head's third-order state tuple (Theorem 3):
 * [ SK d*d | SQ d*d | P d*dv | mK d | G1 d*dv | G2 d*dv | G3 d*dv | h1 d | h2 d | h3 d ]. */
size_t hla3_state_floats(int d, int dv);

/* Bytes of scratch workspace hla3_forward needs (0 if unsupported). */
size_t hla3_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, hla_dtype dt);

/*
 * hla3_forward -- forward of third-order HLA (Sec. 7).
 *
 *   masked = 1 (Theorem 3, Algorithm 3 at gamma = 1):
 *     num_t = q_t^T (S^K_t S^Q_t P^KV_t - G1_t - G2_t - G3_t)
 *     den_t = q_t^T (S^K_t S^Q_t m^K_t  - h1_t - h2_t - h3_t)
 *   masked = 0: num_t = q_t^T S^K_t S^Q_t P^KV_t, den_t = q_t^T S^K_t S^Q_t m^K_t
 *   out_t = num_t, or num_t / (den_t + eps) if normalized.
 * Arguments as for hla2_forward, with the third-order state layout.
 */
hla_status hla3_forward(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                        int B, int H, int n, int d, int dv, int masked, int normalized, float eps,
                        int chunk, const float *state_in, float *state_out,
                        void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * hla3_forward_path -- which CUDA path hla3_forward takes for these arguments on
 * the current device, without launching anything: 2 the tensor-core kernels
 * (fp32 tokens, d = dv = 32, masked = 1, normalized = 0, no states, an sm_103
 * device), 1 the chunk-parallel fp32 kernels, 0 the serial kernel, -1 the
 * arguments are not supported.  *launches (if not null) receives the number of
 * kernel launches of one call (0 when B*H = 0).
 */
int hla3_forward_path(int B, int H, int n, int d, int dv, int masked, int normalized, int chunk, hla_dtype dt,
                      int has_state_in, int has_state_out, int *launches);

/*
 * hla2_backward_path -- which CUDA path hla2_backward takes for these arguments
 * on the current device, without launching anything: 1 the tensor-core kernel
 * (bf16 tokens, d = dv = 64, normalized = 0, an sm_103 device; one launch),
 * 0 the fp32 CUDA-core kernels (five launches), -1 the arguments are not
 * supported.
 */
int hla2_backward_path(int B, int H, int n, int d, int dv, int normalized, int chunk, hla_dtype dt);

/*
 * hla2_forward_noalloc -- hla2_forward for callers that cannot allocate device
 * memory (no counterpart in the paper: it only changes where scratch lives).
 *
 * Some callers cannot call cudaMalloc or hand over a workspace: code that runs
 * under an allocator it does not own (a framework's caching pool, a memory
 * budget that forbids extra reservations), or host code that links this
 * library without any device-memory management of its own.  This entry point
 * computes exactly what hla2_forward computes (same arguments, minus the
 * workspace and state_out) and allocates nothing: its scratch is a 16 MiB
 * array in device memory that belongs to the library.  Every GPU on which the
 * library is used holds that array until the process exits.
 *
 * Scope: the arguments for which hla2_forward_path returns 1 without a final
 * state (the fused path: bf16 tokens, d and dv in {64, 128}, masked = 1,
 * state_in only with d = dv = 128, an sm_103 device); other arguments return
 * HLA_ERR_UNSUPPORTED.  Sizes whose scratch exceeds 16 MiB (it grows with
 * B*H, about 263 KiB per head, and with B*H*n*4 bytes when normalized) return
 * HLA_ERR_WORKSPACE before anything is launched.
 * Set-up: the first call on a device looks up the array's device address
 * (cudaGetSymbolAddress) with that device current; make that first call before
 * any stream capture.
 * Sharing: all calls use the same array and it keeps the last call's contents
 * (each call clears what must start at zero).  Calls whose kernels overlap on
 * the GPU (different streams, or several host threads) race on it: order them
 * on one stream.  A device-side wait that exceeds its budget sets the error
 * word at the start of the array; hla_poll_error_noalloc reads it.
 * An empty problem (B*H = 0 or n = 0) returns HLA_OK without launching.
 */
hla_status hla2_forward_noalloc(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                                int B, int H, int n, int d, int dv, int masked, int normalized, float eps,
                                int chunk, const float *state_in, hla_stream_t stream);

/*
 * Asymmetric second-order HLA (AHLA), Sec. "Asymmetric Higher-order Linear
 * Attention".  The operator is always causal:
 *   o_t = sum_{j<=t} sum_{i=j..t} (q_t.k_i)(q_i.k_j) v_j   (Eq. AHLA-explicit),
 * computed as q_t^T E_t with the streaming state of Theorem AHLA:
 *   P_t = P_{t-1} + k_t v_t^T,  m_t = m_{t-1} + k_t,
 *   E_t = E_{t-1} + k_t (q_t^T P_t),  n_t = n_{t-1} + k_t (q_t^T m_t),
 *   out_t = q_t^T E_t, or q_t^T E_t / (q_t^T n_t + eps) if normalized.
 * State of one head (fp32, row-major): [ P (d*dv) | m (d) | E (d*dv) | n (d) ].
 */
size_t ahla_state_floats(int d, int dv);

/* Bytes of scratch workspace ahla_forward needs (0 if unsupported). */
size_t ahla_workspace_bytes(int B, int H, int n, int d, int dv, int chunk, hla_dtype dt);

/*
 * ahla_forward -- chunk-parallel AHLA forward: chunk summaries composed with
 * the AHLA semidirect product (Eq. AHLA-semidirect, with the segment cross
 * moment R^KQ = sum k q^T of the later segment), which reproduces the serial
 * recurrence (scan equivalence); chunk is the scan granularity (results do not
 * depend on it up to rounding).  Arguments, layouts, shapes and errors as for
 * hla2_forward (no masked flag), with the AHLA state layout for state_in /
 * state_out (state_out may equal state_in).  bf16 tokens with d and dv in
 * {64, 128}, the plain output and no states run on the tensor cores (one
 * persistent tcgen05 kernel sweeping each head's 128-token tiles with the P
 * and E carries in tensor memory); every other call runs three fp32 kernels.
 * A device-side wait that exceeds its budget sets the flag hla_poll_error reads.
 */
hla_status ahla_forward(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                        int B, int H, int n, int d, int dv, int normalized, float eps, int chunk,
                        const float *state_in, float *state_out,
                        void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * ahla_forward_path -- which CUDA path ahla_forward takes for these arguments on
 * the current device, without launching anything: 1 the tensor-core kernel,
 * 0 the fp32 kernels, -1 the arguments are not supported.
 */
int ahla_forward_path(int B, int H, int n, int d, int dv, int normalized, int chunk, hla_dtype dt, int has_state_in,
                      int has_state_out);

/*
 * ahla_step -- one AHLA decode step for B*H heads (the online updates of
 * Theorem AHLA; Algorithm AHLA-stream at gamma = 1): q, k [B, H, d], v, out
 * [B, H, dv] of type dt; state fp32 [B*H * ahla_state_floats(d,dv)], updated
 * in place.  Errors as for hla2_step.
 */
hla_status ahla_step(const void *q, const void *k, const void *v, void *out, hla_dtype dt,
                     int B, int H, int d, int dv, int normalized, float eps,
                     float *state, hla_stream_t stream);

/*
 * Around the mixers: a short convolution, a selective scan, norms with rotation
 * ------------------------------------------------------------------------------
 * The operators below stand before and beside the HLA mixers in one layer (no
 * counterpart in the paper).  They read and write rows of projections, so a
 * token tensor is given by a base pointer and a row stride in elements: token t
 * of sequence b is row b*n + t (the step functions: row b), and a row holds its
 * heads or channels contiguously.  A row stride is at least the row's width, so
 * a tensor may be a slice of a wider projection.  No alignment beyond the
 * element's is asked of these rows (16-byte aligned rows take the wide path);
 * [B, H, n, d] tensors, fp32 states and tables are 16-byte aligned.
 * lengths: device int32 [B] or NULL (= n everywhere), clamped to 0..n: tokens at
 * and after a sequence's length are not read, give zeros in the outputs, and
 * leave the state as it is.
 * A buffer that is written may not overlap one that is read, except where said.
 */

/*
 * hla_conv_forward -- causal depthwise convolution of a few taps:
 *   pre_t = bias + sum_{j<width} w[c][j] x_{t-(width-1)+j},
 *   out_t = pre_t * sigmoid(pre_t) if silu, else pre_t,
 * rows before the first being state_in's.
 * x      : device [B, n, C], row stride x_stride, of type dt
 * w      : device [C, width] of type dt; bias: device [C] of type dt, or NULL (= 0)
 * out    : device [B, n, C], row stride out_stride (written)
 * state_in  : device [B, width-1, C] of type dt, the rows before the call, or NULL (= 0)
 * state_out : device [B, width-1, C] of type dt or NULL; receives the last
 *             width-1 rows (after lengths[b] tokens).  May equal state_in.
 * width in {2, 3, 4}.  Errors: HLA_ERR_INVALID_ARGUMENT, HLA_ERR_UNSUPPORTED
 * before anything is launched, HLA_ERR_CUDA.
 */
hla_status hla_conv_forward(const void *x, const void *w, const void *bias, void *out, hla_dtype dt, int B, int n,
                            int C, int width, long long x_stride, long long out_stride, int silu, const int *lengths,
                            const void *state_in, void *state_out, hla_stream_t stream);

/*
 * hla_conv_step -- hla_conv_forward of one token a sequence, the state updated
 * in place.  x, out: device [B, C], row strides x_stride, out_stride (out may
 * equal x); state: device [B, width-1, C] of type dt.
 */
hla_status hla_conv_step(const void *x, const void *w, const void *bias, void *out, hla_dtype dt, int B, int C,
                         int width, long long x_stride, long long out_stride, int silu, void *state,
                         hla_stream_t stream);

/* Bytes of scratch workspace hla_conv_backward needs (0 if unsupported). */
size_t hla_conv_backward_workspace_bytes(int B, int n, int C, int width, hla_dtype dt);

/*
 * hla_conv_backward -- gradients of hla_conv_forward (from a zero state) for
 * L = sum dout . out:  dx, dw and, if not NULL, dbias.
 * dout: device [B, n, C], row stride dout_stride; dx: device [B, n, C], row stride
 * dx_stride (written); dw: device fp32 [C, width] (written); dbias: device fp32
 * [C] or NULL.  Weight gradients are summed in a fixed order: equal inputs give
 * equal bits.  workspace: 256-byte aligned.
 */
hla_status hla_conv_backward(const void *x, const void *w, const void *bias, const void *dout, void *dx, float *dw,
                             float *dbias, hla_dtype dt, int B, int n, int C, int width, long long x_stride,
                             long long dout_stride, long long dx_stride, int silu, const int *lengths,
                             void *workspace, size_t workspace_bytes, hla_stream_t stream);

/* Bytes of scratch workspace hla_ssm_forward needs (0 if unsupported). */
size_t hla_ssm_workspace_bytes(int B, int n, int H, int P, int G, int N, hla_dtype dt);

/*
 * hla_ssm_forward -- selective state space scan over a prompt.  Per head h of
 * group g = h / (H / G), with the N x P state s:
 *   delta_t = softplus(raw_t + delta_bias_h)   (raw_t + delta_bias_h if softplus == 0)
 *   s_t = exp(a_h delta_t) s_{t-1} + delta_t b_t x_t^T,   y_t = s_t^T c_t + skip_h x_t
 * x, y  : device [B, n, H, P], row strides x_stride, y_stride, of type dt
 * delta : device [B, n, H], row stride delta_stride, of type dt (the raw step sizes)
 * b, c  : device [B, n, G, N], row strides b_stride, c_stride, of type dt
 * a     : device fp32 [H], not above 0 (with delta not below 0: the state does not grow)
 *         (bf16 tokens: products c_t . b_u delta_u, taken before x_u, have to stay in range)
 * skip, delta_bias : device fp32 [H] or NULL (= 0)
 * state_in  : device fp32 [B, H, N, P] or NULL (= 0)
 * state_out : device fp32 [B, H, N, P] or NULL; the state after lengths[b] tokens.
 *             May equal state_in.
 * P, N in {16, 32, 64, 128}; H a multiple of G.
 * workspace : at least hla_ssm_workspace_bytes(...) bytes, 256-byte aligned; calls
 *             that share one are ordered on one stream; hla_poll_error reads its flag.
 * fp32 tokens: fp32 throughout.  bf16 tokens with 16-byte aligned rows: sums and
 * states are fp32 sums of products of bf16 pairs (16 bits: a state is about 4e-6
 * from the exact one), and outputs, rounded to bf16, may differ by that rounding.
 * A NaN or infinity in a token reaches the outputs of that token and later ones,
 * where it enters them (there as NaN, or infinity), and the state.
 */
hla_status hla_ssm_forward(const void *x, const void *delta, const float *a, const void *b, const void *c,
                           const float *skip, const float *delta_bias, void *y, hla_dtype dt, int B, int n, int H,
                           int P, int G, int N, long long x_stride, long long delta_stride, long long b_stride,
                           long long c_stride, long long y_stride, int softplus, const int *lengths,
                           const float *state_in, float *state_out, void *workspace, size_t workspace_bytes,
                           hla_stream_t stream);

/*
 * hla_ssm_forward_path -- which CUDA path hla_ssm_forward takes for these arguments
 * on the current device, without launching anything: 1 the tensor-core kernels
 * (bf16 tokens, rows of x, b, c and y 16-byte aligned: aligned_rows = 1, an sm_103
 * device), 0 the fp32 kernels, -1 the arguments are not supported.  *launches (if
 * not NULL) receives the number of kernels the call launches (0 for an empty one).
 */
int hla_ssm_forward_path(int B, int n, int H, int P, int G, int N, hla_dtype dt, int aligned_rows, int *launches);

/*
 * hla_ssm_step -- hla_ssm_forward of one token a sequence: x, y [B, H, P], delta
 * [B, H], b, c [B, G, N] with their row strides; state fp32 [B, H, N, P], updated
 * in place.  y may equal x.  No workspace.
 */
hla_status hla_ssm_step(const void *x, const void *delta, const float *a, const void *b, const void *c,
                        const float *skip, const float *delta_bias, void *y, hla_dtype dt, int B, int H, int P, int G,
                        int N, long long x_stride, long long delta_stride, long long b_stride, long long c_stride,
                        long long y_stride, int softplus, float *state, hla_stream_t stream);

/*
 * hla_qk_norm_forward -- RMS norm of every query and key head, the rotation of
 * its first rot components by the token's position, and the change of layout to
 * the one the mixers read:
 *   y = x / sqrt(mean(x^2) + eps) * w                          (over the d components)
 *   out_i = y_i cos - y_j sin,  out_j = y_j cos + y_i sin      for each pair (i, j)
 * pairs (i, i + rot/2), or (2i, 2i+1) if interleaved; pair i takes column i of the
 * tables.  q has H heads, k has Hk; key head h is written for the H/Hk query
 * heads h*H/Hk .. that share it.
 * q, k  : device [B, n, H, d], [B, n, Hk, d], row strides q_stride, k_stride
 * wq, wk: device [d] of type dt, or NULL (= 1)
 * cos, sin : device fp32 [table_rows, rot/2] (NULL if rot == 0), 16-byte aligned
 * positions: device int32 [B, n], the tables' rows; NULL: token t has row pos0 + t.
 *            A position outside the tables gives NaN in the rotated components.
 * q_out, k_out : device [B, H, n, d] of type dt, 16-byte aligned (written)
 * d in {16, 32, 64, 128}; rot a multiple of 8, 0..d; H a multiple of Hk; eps >= 0.
 */
hla_status hla_qk_norm_forward(const void *q, const void *k, const void *wq, const void *wk, const float *cos,
                               const float *sin, const int *positions, void *q_out, void *k_out, hla_dtype dt, int B,
                               int n, int H, int Hk, int d, int rot, int interleaved, long long q_stride,
                               long long k_stride, int pos0, int table_rows, float eps, hla_stream_t stream);

/* Bytes of scratch workspace hla_qk_norm_backward needs (0 if unsupported). */
size_t hla_qk_norm_backward_workspace_bytes(int B, int n, int H, int Hk, int d, hla_dtype dt);

/*
 * hla_qk_norm_backward -- gradients of hla_qk_norm_forward: dq, dk (rows like q,
 * k, strides dq_stride, dk_stride) and the weights' dwq, dwk (device fp32 [d] or
 * NULL) from dq_out, dk_out [B, H, n, d].  A key head's gradient is the sum over
 * the query heads that share it.  Sums in a fixed order: equal inputs give equal bits.
 */
hla_status hla_qk_norm_backward(const void *q, const void *k, const void *wq, const void *wk, const float *cos,
                                const float *sin, const int *positions, const void *dq_out, const void *dk_out,
                                void *dq, void *dk, float *dwq, float *dwk, hla_dtype dt, int B, int n, int H, int Hk,
                                int d, int rot, int interleaved, long long q_stride, long long k_stride,
                                long long dq_stride, long long dk_stride, int pos0, int table_rows, float eps,
                                void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * The rest of a block: a gated recurrence, norms around it, a gated feed-forward part
 * ----------------------------------------------------------------------------------
 * Operators that stand beside the mixers and after them (no counterpart in the paper).
 * Rows, strides, lengths and overlap are as above: token t of sequence b is row
 * b*n + t at a row stride in elements, and no alignment beyond the element's is
 * asked of rows.  Sums over tokens are made in a fixed order: equal inputs give
 * equal bits.  Exponentials (of gates, of decays) are made in fp32, for fp32 tokens to the last bits, for bf16
 * tokens to 2^-23 |v| of e^v.  Calls that share a workspace run one after another, on one stream or ordered by
 * events; a captured graph's workspace stays its own while the graph may run.  No call's workspace
 * keeps anything from one call for the next.
 */

/* Activations of a gate (also the slopes of the gradients). */
typedef enum {
    HLA_LINEAR = 0,  /* v */
    HLA_SIGMOID = 1, /* 1 / (1 + e^-v) */
    HLA_SILU = 2     /* v / (1 + e^-v) */
} hla_act;

/* Number of marks of n tokens: states that hla_glr_forward leaves for hla_glr_backward. */
int hla_glr_marks(int n);

/*
 * hla_glr_forward -- gated linear recurrence over a prompt, for each channel:
 *   s_t = sigmoid(r_t),  a_t = exp(decay s_t),  i_t = sigmoid(g_t),
 *   h_t = a_t h_{t-1} + sqrt(1 - a_t^2) i_t x_t,   y_t = h_t
 * x, r, g, y : device [B, n, C], row strides x_stride, r_stride, g_stride, y_stride, of type dt
 * decay : device fp32 [C], finite and below 0 (where it is 0, gradients of r and decay are unbounded)
 * state_in  : device fp32 [B, C] or NULL (= 0)
 * state_out : device fp32 [B, C] or NULL; the state after lengths[b] tokens.  May equal state_in.
 * marks     : device fp32 [B, hla_glr_marks(n), C] or NULL; receives the state before
 *             every 32nd token, which hla_glr_backward reads
 * decay, states and marks are 16-byte aligned.
 * No workspace (should a wait between the blocks of one sequence run past its limit of 2 s, the state behind
 * the sequence is NaN, and so are the outputs and marks that are not known without it).  fp32 throughout for both types; i_t below 1e-19 counts as 0, and a token
 * whose gates are both shut (r and g far below 0, minus infinity too) leaves the state as it is.  A NaN
 * or infinity in a token reaches that token's output and, where it enters the state, later ones, and no
 * earlier one.
 */
hla_status hla_glr_forward(const void *x, const void *r, const void *g, const float *decay, void *y, hla_dtype dt, int B,
                           int n, int C, long long x_stride, long long r_stride, long long g_stride, long long y_stride,
                           const int *lengths, const float *state_in, float *state_out, float *marks,
                           hla_stream_t stream);

/*
 * hla_glr_step -- hla_glr_forward of one token a sequence: x, r, g, y [B, C] with their
 * row strides; state fp32 [B, C], updated in place.  y may equal x, r or g.  No workspace.
 */
hla_status hla_glr_step(const void *x, const void *r, const void *g, const float *decay, void *y, hla_dtype dt, int B, int C,
                        long long x_stride, long long r_stride, long long g_stride, long long y_stride, float *state,
                        hla_stream_t stream);

/* Bytes of scratch workspace hla_glr_backward needs (0 if unsupported). */
size_t hla_glr_backward_workspace_bytes(int B, int n, int C, hla_dtype dt);

/*
 * hla_glr_backward -- gradients of hla_glr_forward for L = sum dy . y + sum dstate_out . state_out:
 * dx, dr, dg (rows like x, r, g, with their strides; zero at and after a length), ddecay
 * (device fp32 [C]) and, if not NULL, dstate_in (device fp32 [B, C]).
 * dy: device [B, n, C], row stride dy_stride; dstate_out: device fp32 [B, C] or NULL (= 0; may
 * equal dstate_in); marks: those that the forward with the same x, r, g, decay, lengths and
 * state_in left.  decay, states, marks and ddecay are 16-byte aligned.  workspace: 256-byte aligned;
 * hla_poll_error reads its flag (a wait that ran out; what is not known without it, dstate_in and ddecay among it, is NaN).
 */
hla_status hla_glr_backward(const void *x, const void *r, const void *g, const float *decay, const void *dy,
                            const float *marks, void *dx, void *dr, void *dg, float *ddecay, hla_dtype dt, int B, int n,
                            int C, long long x_stride, long long r_stride, long long g_stride, long long dy_stride,
                            long long dx_stride, long long dr_stride, long long dg_stride, const int *lengths,
                            const float *dstate_out, float *dstate_in, void *workspace, size_t workspace_bytes,
                            hla_stream_t stream);

/*
 * hla_block_norm_forward -- what stands between two blocks: the norm of a block's output y with
 * its gate, residual scale and dropout, the residual sum, and the norm before the next block:
 *   x' = alpha x + k scale act(gate) u w_post,   u = y / sqrt(mean(y^2) + eps), or y if post_norm == 0
 *   h  = x' / sqrt(mean(x'^2) + eps) w_pre       if pre_norm   (of x' before it is rounded)
 * means over a row's C columns; k = 1 without dropout, else 0 or 1 / (1 - dropout): value (row,
 * column) is dropped where its 32 random bits are below floor(dropout 2^32), bits that
 * Philox4x32-10 gives for the counter (column / 4, row, offset low, offset high) and the key (seed
 * low, seed high), word column % 4.  The mask is not stored: the gradient makes it again.  Where a value
 * is dropped, y and gate may hold anything, NaN and infinities too (y without post_norm, whose mean has it).
 * x, y, gate : device [rows, C], row strides x_stride, y_stride, gate_stride, of type dt; gate may be NULL (= 1)
 * w_post, scale, w_pre : device [C] of type dt, or NULL (= 1; w_post and w_pre are not read without their norm)
 * x_out : device [rows, C], row stride x_out_stride (written; may equal x, with its stride)
 * h     : device [rows, C], row stride h_stride (written; not read or written without pre_norm)
 * 0 <= dropout < 1; eps >= 0 finite; alpha finite; offset and seed: any 64 bits.
 */
hla_status hla_block_norm_forward(const void *x, const void *y, const void *gate, const void *w_post, const void *scale,
                                  const void *w_pre, void *x_out, void *h, hla_dtype dt, int rows, int C,
                                  long long x_stride, long long y_stride, long long gate_stride, long long x_out_stride,
                                  long long h_stride, int post_norm, int pre_norm, int act, float alpha, float eps,
                                  double dropout, unsigned long long seed, unsigned long long offset, hla_stream_t stream);

/* Bytes of scratch workspace hla_block_norm_backward needs (0 if unsupported). */
size_t hla_block_norm_backward_workspace_bytes(int rows, int C, hla_dtype dt);

/*
 * hla_block_norm_backward -- gradients of hla_block_norm_forward for L = sum dx_out . x_out + sum dh . h:
 * dx, dy, dgate (rows like x, y, gate, with their strides; dgate NULL without a gate) and, where not
 * NULL, dw_post, dscale, dw_pre (device fp32 [C]; zeros where a norm is off).
 * dx_out, dh: device [rows, C] with their row strides; dh is not read without pre_norm.
 * dx may equal dx_out, with its stride.
 */
hla_status hla_block_norm_backward(const void *x, const void *y, const void *gate, const void *w_post, const void *scale,
                                   const void *w_pre, const void *dx_out, const void *dh, void *dx, void *dy, void *dgate,
                                   float *dw_post, float *dscale, float *dw_pre, hla_dtype dt, int rows, int C,
                                   long long x_stride, long long y_stride, long long gate_stride, long long dx_out_stride,
                                   long long dh_stride, long long dx_stride, long long dy_stride, long long dgate_stride,
                                   int post_norm, int pre_norm, int act, float alpha, float eps, double dropout,
                                   unsigned long long seed, unsigned long long offset, void *workspace,
                                   size_t workspace_bytes, hla_stream_t stream);

/* Bytes of scratch workspace hla_ffn_forward and hla_ffn_backward need (0 if unsupported). */
size_t hla_ffn_workspace_bytes(int rows, int K, int F, hla_dtype dt);
size_t hla_ffn_backward_workspace_bytes(int rows, int K, int F, hla_dtype dt);

/*
 * hla_ffn_forward -- gated feed-forward projections, activation and product:
 *   out = act(x Wg^T) (x Wu^T)
 * x   : device [rows, K], row stride x_stride, of type dt
 * w   : device [2, F, K] of type dt: Wg, then Wu
 * out : device [rows, F], row stride out_stride, of type dt (written)
 * The products are rounded once, after the activation.  workspace: 256-byte aligned; hla_poll_error
 * reads its flag.
 */
hla_status hla_ffn_forward(const void *x, const void *w, void *out, hla_dtype dt, int rows, int K, int F,
                           long long x_stride, long long out_stride, int act, void *workspace, size_t workspace_bytes,
                           hla_stream_t stream);

/*
 * hla_ffn_backward -- gradients of hla_ffn_forward for L = sum dout . out, which computes the
 * projections again: dx (device [rows, K], row stride dx_stride) and dw (device [2, F, K]), of type dt.
 * dout: device [rows, F], row stride dout_stride.  bf16: the projections' gradients are rounded to bf16
 * once between the products, which makes the error of dx and dw against 64 bits 1.4 times what their own
 * rounding alone makes (0.0023 of their norm instead of 0.0017).
 */
hla_status hla_ffn_backward(const void *x, const void *w, const void *dout, void *dx, void *dw, hla_dtype dt, int rows,
                            int K, int F, long long x_stride, long long dout_stride, long long dx_stride, int act,
                            void *workspace, size_t workspace_bytes, hla_stream_t stream);

/*
 * hla_poll_error_noalloc -- hla_poll_error for hla2_forward_noalloc (no
 * counterpart in the paper): waits for `stream`, then reports and clears the
 * device-side error word of the library's scratch array on the current device:
 * HLA_OK, or HLA_ERR_TIMEOUT if a device-side wait of the last no-alloc call
 * gave up.  Returns HLA_ERR_CUDA if synchronisation or the read fails.
 */
hla_status hla_poll_error_noalloc(hla_stream_t stream);

/*
 * hla_poll_error -- wait for `stream`, then report the device-side error flag
 * kept in `workspace` by the last forward call that used it: HLA_OK, or
 * HLA_ERR_TIMEOUT if a device-side wait gave up.  Clears the flag.
 * Returns HLA_ERR_CUDA if synchronisation or the read fails.
 */
hla_status hla_poll_error(void *workspace, hla_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* HLA_H_ */
