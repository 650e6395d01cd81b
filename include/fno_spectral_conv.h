/*
 * fno_spectral_conv.h — C ABI of the half-precision FNO spectral-convolution
 * layer for AMD Instinct MI355X (gfx950).
 *
 * The layer is the Fourier convolution operator of Tu et al., "Guaranteed
 * Approximation Bounds for Mixed-Precision Neural Operators" (ICLR 2024),
 * Sec. 2 ("FNO and extensions"):
 *
 *     (K v)(x) = F^-1( R . T_K( F tanh(v) ) )(x)
 *
 * with the tanh pre-activation of Sec. 4.3 in half-precision mode, the
 * forward transform normalised as the Riemann sum of Sec. 3 (1/N), the
 * truncation T_K keeping the m_j lowest non-negative and m_j highest negative
 * frequencies on every axis but the last and k = 0..m_d-1 on the last
 * (real-FFT) axis, a complex per-mode channel mixing R (dense, or Tucker
 * factorised as in the tensorised FNO of Sec. 2, contracted pairwise in the
 * greedy order of Sec. 4.2), and the inverse
 *
 *     y[x] = sum_t c(k_d(t)) Re( Yhat[t] exp(+2 pi i <k(t), x / N>) ),
 *
 * c = 1 on the k_d = 0 and Nyquist planes and 2 elsewhere.  Gradients follow
 * the real-gradient convention g = dL/dRe + i dL/dIm.
 *
 * Conventions for every entry point
 *   - Tensors are device pointers to contiguous row-major arrays, last axis
 *     fastest.  Complex values are interleaved (re, im) pairs of the element
 *     type.  Every device pointer must be 16-byte aligned.
 *   - Element type: FNO_PREC_FP16_TANH stores x, y, gy, gx and the weights as
 *     IEEE fp16 (round-to-nearest-even stores, fp32 accumulation inside the
 *     kernels); FNO_PREC_FP32 stores them as fp32.  Weight gradients are always
 *     fp32 complex.
 *   - The caller owns all device memory, including the workspace.  The library
 *     owns only per-descriptor plan tables (twiddles, index maps, the Tucker
 *     path); they are built, with a blocking upload, on the first call for a
 *     descriptor on a device and kept until fno_release_caches() or unload.
 *     Later calls allocate nothing.  Issue one warm-up call before capturing
 *     calls into a HIP graph.
 *   - All argument checks run on the host before anything is enqueued; a
 *     rejected call enqueues nothing.  Calls are asynchronous on `stream`.
 *   - A transform's output (y, gx) may hold intermediate sums of the call
 *     before its results are written, where its memory overlaps none of the
 *     call's inputs.
 *   - The plan cache is mutex-guarded; concurrent calls on different streams
 *     are safe as long as their workspaces and outputs do not overlap.
 *   - Calls run on the current device, whose stream `stream` must be.  With
 *     Tucker or CP weights the forward, data-gradient, weight-gradient and
 *     combined backward calls run part of their steps on up to three more
 *     streams of the library's own (default priority, one set per device,
 *     created on the first such call outside a stream capture and kept until
 *     the process ends).  Those streams fork from and join `stream` through
 *     events, so the whole call stays ordered on `stream`: work enqueued on
 *     `stream` afterwards sees every result, and a stream capture records
 *     every branch.
 */
#ifndef FNO_SPECTRAL_CONV_H_
#define FNO_SPECTRAL_CONV_H_

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FNO_OK = 0,
  FNO_ERR_INVALID_ARGUMENT = 1,   /* null/misaligned pointer, bad size or mode count */
  FNO_ERR_UNSUPPORTED = 2,        /* valid request outside what the kernels handle */
  FNO_ERR_WORKSPACE_TOO_SMALL = 3,
  FNO_ERR_HIP = 4,                /* a HIP runtime call or launch failed          */
  FNO_ERR_INTERNAL = 5
} fno_status;

/* Storage precision, and the pre-activation that FNO_PREACT_DEFAULT selects. */
typedef enum {
  FNO_PREC_FP32 = 0,        /* fp32 storage and math, no pre-activation        */
  FNO_PREC_FP16_TANH = 1    /* fp16 storage, fp32 accumulation, tanh (Sec. 4.3) */
} fno_precision;

/* Pre-activation u = f(x) applied to the input before the forward transform
 * (the stabiliser of Sec. 4.3, and the pre-FFT alternatives compared in
 * App. B.6); bwd_data multiplies the transformed gradient by f'(x).  Any
 * choice combines with either storage precision: FP32 with TANH is the
 * full-precision + tanh ablation of App. B.8, FP16_TANH with NONE the
 * unstabilised half-precision baseline, and HARD_CLIP with clip = 57344 the
 * clipping of out-of-range values to the FP8-E5M2 limits (Sec. 4.6,
 * App. B.11).
 *   NONE      : f(x) = x
 *   TANH      : f(x) = tanh(x),  f'(x) = 1 - tanh(x)^2
 *   HARD_CLIP : f(x) = min(max(x, -clip), clip),  f'(x) = 1 for |x| <= clip,
 *               0 otherwise (the bound's own point counts as inside)
 *   SIGMA_CLIP: the statistics-based clip of App. B.6 (with clip = 2 its
 *               2-sigma clip): every (batch, channel) plane of x is clipped
 *               to [mu - clip sigma, mu + clip sigma], mu and sigma the mean
 *               and the population standard deviation of that plane's N
 *               values (computed in double); f'(x) = 1 inside the bounds
 *               (their own points included), 0 outside: the bounds are held
 *               constant in the gradient (no gradient through mu and sigma).
 *               A plane holding a non-finite value has NaN bounds and gives
 *               NaN throughout.  The comparisons with the bounds are made in
 *               double.  The forward, data-gradient and (without caches)
 *               weight-gradient calls compute the statistics themselves
 *               (one extra read of x); their workspaces grow by 16 bytes per
 *               (batch, input channel) plane.  The plane transforms then run
 *               on the table-free kernels.
 * NaN inputs give NaN in f and f'.  In fp16 storage f(x) is rounded once to
 * fp16 before the transform. */
typedef enum {
  FNO_PREACT_DEFAULT = 0,   /* TANH for FNO_PREC_FP16_TANH, NONE for FNO_PREC_FP32 */
  FNO_PREACT_NONE = 1,
  FNO_PREACT_TANH = 2,
  FNO_PREACT_HARD_CLIP = 3,
  FNO_PREACT_SIGMA_CLIP = 4 /* clip each (batch, channel) plane to mean +- clip * sigma */
} fno_preactivation;

/* Spectral weight parameterisation: dense, Tucker (the tensorised FNO of
 * Sec. 2) or CP (canonical polyadic, the factorisation of the Navier-Stokes
 * and Darcy runs of Sec. 4.6). */
typedef enum {
  FNO_WEIGHT_DENSE = 0,
  FNO_WEIGHT_TUCKER = 1,
  FNO_WEIGHT_CP = 2
} fno_weight_kind;

/* Greedy rule for the Tucker and CP contraction order (Sec. 4.2).  MIN_RESULT takes
 * the pair whose intermediate has the fewest elements; MIN_NET the pair that
 * minimises (result - both inputs).  Ties go to the lexicographically smallest
 * pair of the current operand list. */
typedef enum { FNO_PATH_MIN_RESULT = 0, FNO_PATH_MIN_NET = 1 } fno_path_policy;

typedef enum {
  FNO_OP_FWD = 0,
  FNO_OP_BWD_DATA = 1,
  FNO_OP_BWD_WEIGHT = 2,
  FNO_OP_BWD = 3      /* data and weight gradient in one call (fno_spectral_conv_bwd) */
} fno_op;

/* Layer descriptor.  Spatial extents n[0..ndim-1] (N_1..N_d), retained mode
 * counts modes[0..ndim-1]: axes j < d keep K_j = 2 m_j slots (2 m_j <= N_j),
 * the last axis keeps K_d = m_d slots (1 <= m_d <= N_d/2 + 1).  Retained slot
 * t on a leading axis is FFT index k = t for t < m, k = N - 2m + t otherwise.
 * rank = (r_in, r_out, r_1..r_d) for Tucker weights, rank[0] = R for CP
 * weights, ignored for dense.  preact: fno_preactivation (0 = the precision's
 * default); clip: the HARD_CLIP bound, positive and finite (at most 65504 in
 * fp16 storage), ignored otherwise; FNO_ERR_INVALID_ARGUMENT when out of range. */
typedef struct {
  int32_t ndim;          /* 1, 2 or 3                      */
  int32_t precision;     /* fno_precision                  */
  int32_t weight_kind;   /* fno_weight_kind                */
  int32_t path_policy;   /* fno_path_policy (Tucker, CP)   */
  int64_t batch;
  int64_t c_in;
  int64_t c_out;
  int64_t n[3];
  int64_t modes[3];
  int64_t rank[5];
  int32_t preact;        /* fno_preactivation              */
  float clip;            /* bound of FNO_PREACT_HARD_CLIP; number of standard
                            deviations of FNO_PREACT_SIGMA_CLIP (both > 0) */
} fno_conv_desc;

/* Spectral weights R (device pointers, element type of the precision mode).
 *   dense  : [c_in, c_out, K_1..K_d] complex
 * Tucker:
 *   core   : [r_in, r_out, r_1..r_d] complex
 *   u_in   : [c_in, r_in] complex,  u_out: [c_out, r_out] complex
 *   u_mode : u_mode[j] is [K_j, r_j] complex
 *   W[i,o,t] = sum core[a,e,c..] u_in[i,a] u_out[o,e] prod_j u_mode[j][t_j,c_j]
 * CP (rank R = rank[0]; `core` holds the weights lambda):
 *   core   : lambda [R] complex
 *   u_in   : [c_in, R], u_out: [c_out, R], u_mode[j]: [K_j, R], all complex
 *   W[i,o,t] = sum_r lambda[r] u_in[i,r] u_out[o,r] prod_j u_mode[j][t_j,r] */
typedef struct {
  const void *dense;
  const void *core;
  const void *u_in;
  const void *u_out;
  const void *u_mode[3];
} fno_weights;

/* Weight gradients, same shapes as fno_weights, always fp32 complex.  Dense
 * uses `dense`; Tucker and CP use core (CP: the lambda gradient), u_in, u_out
 * and u_mode[0..d-1]. */
typedef struct {
  void *dense;
  void *core;
  void *u_in;
  void *u_out;
  void *u_mode[3];
} fno_weight_grads;

/* Bytes of workspace `op` needs for this descriptor (>= 256, multiple of 256).
 * The size for FNO_OP_BWD_WEIGHT assumes both spectral caches are supplied
 * (for FNO_OP_BWD: the input-spectrum cache);
 * fno_spectral_conv_workspace_size_nocache gives the size when they are not. */
fno_status fno_spectral_conv_workspace_size(const fno_conv_desc *desc, fno_op op,
                                            size_t *bytes);
fno_status fno_spectral_conv_workspace_size_nocache(const fno_conv_desc *desc,
                                                    fno_op op, size_t *bytes);

/* Bytes of one spectral cache: the truncated spectrum [batch, channels, K...]
 * of the precision's element type.  `which` is 0 for the input spectrum
 * Xhat = (1/N) sum_x f(x) e^{-i theta} (c_in channels, f the pre-activation) and 1 for the
 * gradient spectrum (1/sqrt(N)) sum_x gy e^{-i theta} (c_out channels).  The
 * contents are produced and consumed by this library only. */
fno_status fno_spectrum_bytes(const fno_conv_desc *desc, int which, size_t *bytes);

/* Forward: y[batch, c_out, N...] = K x  (x: [batch, c_in, N...]).
 * x_hat_out: optional (NULL to skip) spectral cache for bwd_weight, written
 * with the input spectrum.  Errors: FNO_ERR_INVALID_ARGUMENT (bad descriptor,
 * null or misaligned pointers), FNO_ERR_UNSUPPORTED, FNO_ERR_WORKSPACE_TOO_SMALL,
 * FNO_ERR_HIP. */
fno_status fno_spectral_conv_fwd(const fno_conv_desc *desc, const void *x,
                                 const fno_weights *w, void *y, void *x_hat_out,
                                 void *workspace, size_t workspace_bytes,
                                 hipStream_t stream);

/* Allocation-free forward call, for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid allocation).  Same arguments and results as fno_spectral_conv_fwd
 * without the workspace: the library's own fixed device array of
 * FNO_NOALLOC_SCRATCH_BYTES per GPU (held until the process ends) takes its
 * place.  The call allocates no device memory and creates no events:
 *   - the descriptor's plan must already exist on the current device (make
 *     one ordinary call with it first, e.g. fno_spectral_conv_fwd);
 *     otherwise FNO_ERR_INVALID_ARGUMENT and nothing is enqueued;
 *   - a descriptor whose forward workspace
 *     (fno_spectral_conv_workspace_size(desc, FNO_OP_FWD)) exceeds
 *     FNO_NOALLOC_SCRATCH_BYTES is rejected with FNO_ERR_WORKSPACE_TOO_SMALL
 *     before anything is enqueued.
 * Every call on a GPU uses the same array, which keeps the last call's
 * contents: calls that overlap on one GPU (other streams, other threads)
 * race; serialise them. */
#define FNO_NOALLOC_SCRATCH_BYTES ((size_t)64 << 20)
fno_status fno_spectral_conv_fwd_noalloc(const fno_conv_desc *desc, const void *x,
                                         const fno_weights *w, void *y, void *x_hat_out,
                                         hipStream_t stream);

/* Data gradient: gx[batch, c_in, N...] from gy[batch, c_out, N...]:
 * G = c(k) sum_x gy e^{-i theta}, gXhat = sum_o G conj(W),
 * gx = (1/N) sum_t Re(gXhat e^{+i theta}) * f'(x) with f the pre-activation
 * (x is read only for f' and may be NULL when the pre-activation is NONE).
 * gy_hat_out: optional spectral cache (gradient spectrum) for bwd_weight. */
fno_status fno_spectral_conv_bwd_data(const fno_conv_desc *desc, const void *x,
                                      const fno_weights *w, const void *gy, void *gx,
                                      void *gy_hat_out, void *workspace,
                                      size_t workspace_bytes, hipStream_t stream);

/* Weight gradient: dense gW[i,o,t] = sum_b conj(Xhat[b,i,t]) G[b,o,t]; Tucker:
 * the chain rule through the multilinear map onto core and factors.  Outputs
 * are overwritten (fp32 complex).  x_hat / gy_hat: spectral caches from fwd /
 * bwd_data of the same descriptor and inputs, or NULL to recompute them from
 * x / gy (which may then not be NULL).  The batch reduction has a fixed order:
 * results are bitwise reproducible. */
fno_status fno_spectral_conv_bwd_weight(const fno_conv_desc *desc, const void *x,
                                        const void *gy, const fno_weights *w,
                                        const void *x_hat, const void *gy_hat,
                                        fno_weight_grads *gw, void *workspace,
                                        size_t workspace_bytes, hipStream_t stream);

/* Data and weight gradients in one call: the results of
 * fno_spectral_conv_bwd_data (gx, optional gy_hat_out) followed by
 * fno_spectral_conv_bwd_weight (gw), with the adjoint contraction and the
 * dense weight gradient sharing one launch when the element type is fp16 and
 * the retained-mode count is a multiple of 16 (elsewhere the two run one after
 * the other, as in the separate calls).  x_hat: the forward's input-spectrum
 * cache (fno_spectral_conv_fwd's x_hat_out) or NULL to recompute it from x.
 * Workspace: fno_spectral_conv_workspace_size(desc, FNO_OP_BWD) when x_hat is
 * given, the _nocache size otherwise.  Errors as for the separate calls. */
fno_status fno_spectral_conv_bwd(const fno_conv_desc *desc, const void *x,
                                 const fno_weights *w, const void *gy, const void *x_hat,
                                 void *gx, fno_weight_grads *gw, void *gy_hat_out,
                                 void *workspace, size_t workspace_bytes, hipStream_t stream);

/* Host-only: FFT index k of retained slot t on `axis` (0-based) — the
 * truncation map of Sec. 2 as described above. */
fno_status fno_mode_frequency(const fno_conv_desc *desc, int32_t axis, int64_t t,
                              int64_t *k);

/* Host-only: the pairwise contraction order of Tucker or CP weights for
 * FNO_OP_FWD or FNO_OP_BWD_DATA (the greedy rule of Sec. 4.2 under
 * desc->path_policy).  Writes 3 int32 per step: p, q (positions in the
 * current operand list, p < q; the two leave the list and the result is
 * appended) and the bit mask of the result's indices: bit 0 batch, 1 c_in,
 * 2 c_out, 3 r_in, 4 r_out, 5+j spatial axis j, 8+j rank of axis j (Tucker),
 * 11 the CP rank.  The initial list is [spectrum, core (CP: lambda), u_in,
 * u_out, u_1..u_d].  FNO_ERR_INVALID_ARGUMENT for dense weights.  `cap` is
 * the capacity in steps. */
fno_status fno_contraction_path(const fno_conv_desc *desc, fno_op op, int32_t *steps,
                                int32_t cap, int32_t *n_steps);

/* Host-only: total complex multiply-adds of that path and its largest
 * intermediate (elements). */
fno_status fno_contraction_path_cost(const fno_conv_desc *desc, fno_op op,
                                     int64_t *macs, int64_t *peak_elems);

/* ------------------------------------------------------------------------
 * The rest of the FNO block (Sec. 2): one block maps v to
 *
 *     out = act( W_skip v + b + K v )  (+ v with a residual connection)
 *
 * with K the spectral convolution above, W_skip v + b a pointwise linear map
 * over the channels (a 1x1 convolution with bias: the skip path) and act a
 * pointwise nonlinearity.  Sec. 4.2 leaves these real-valued operations to
 * automatic mixed precision; here they are one fused pass after K (and two
 * around K's backward) instead of separate convolution, add, activation and
 * residual kernels.  In fp16 mode the channel mix multiplies fp16 operands
 * with fp32 accumulation (as mixed precision runs a 1x1 convolution); the
 * sums, the activation and the residual stay in fp32 registers and the
 * results are rounded once to fp16.
 *
 * Layouts: x [batch][c_in][points], y and out [batch][c_out][points] (points
 * = the product of the spatial extents, the layout of the spectral
 * convolution's tensors), w_skip [c_out][c_in], b [c_out], all of the
 * precision's element type; the parameter gradients g_w_skip [c_out][c_in]
 * and g_b [c_out] are fp32 and overwritten (not accumulated).
 *
 * One block's training step:
 *   fno_spectral_conv_fwd(x -> y);  fno_block_epilogue_fwd(x, y -> out, z)
 *   fno_block_epilogue_bwd_weight(x, z, g_out -> g_z, g_w_skip, g_b)
 *   fno_spectral_conv_bwd(x, gy = g_z -> gx_spec, g_w)
 *   fno_block_epilogue_bwd_data(g_z, w_skip, gx_spec, g_out -> gx)
 * ------------------------------------------------------------------------ */
typedef enum {
  FNO_EPI_ACT_NONE = 0,
  FNO_EPI_ACT_GELU = 1  /* z Phi(z), Phi the exact normal distribution function */
} fno_epi_activation;

typedef struct {
  int32_t precision;   /* FNO_PREC_FP16_TANH: fp16 tensors; FNO_PREC_FP32: fp32 */
  int64_t batch, c_in, c_out;
  int64_t points;      /* grid points of one channel, >= 1 */
  int32_t activation;  /* fno_epi_activation */
  int32_t residual;    /* 1: add x after the activation (needs c_in == c_out) */
} fno_block_desc;

/* Workspace bytes of an epilogue call: FNO_OP_BWD_WEIGHT needs one (the
 * partial sums of the parameter gradients, reduced in a fixed order so that
 * results are bit-identical from run to run); FNO_OP_FWD and
 * FNO_OP_BWD_DATA need none (0).  FNO_ERR_INVALID_ARGUMENT for a malformed
 * descriptor (c_in, c_out up to 65536 with c_out (c_in + 1) <= 65535 x 256;
 * batch x points x channels up to 2^38; a residual with c_in != c_out) or
 * another op. */
fno_status fno_block_epilogue_workspace_size(const fno_block_desc *desc, fno_op op,
                                             size_t *bytes);

/* Forward (Sec. 2, the FNO block after K): z = W_skip x + b + y and
 * out = act(z) (+ x).  b may be null (no bias).  z_out, if not null,
 * receives z (the backward's input when act is GELU; may be null for
 * act NONE or for inference).  out must not alias x or y. */
fno_status fno_block_epilogue_fwd(const fno_block_desc *desc, const void *x, const void *y,
                                  const void *w_skip, const void *b, void *out, void *z_out,
                                  hipStream_t stream);

/* First backward step (chain rule through the epilogue): g_z = g_out act'(z),
 * which is also dL/dy and so the spectral convolution's output gradient, and
 * the parameter gradients g_w_skip[o][i] = sum over batch and points of
 * g_z[o] x[i], g_b[o] = sum of g_z[o].  With act GELU, z (from the forward)
 * and g_z are required; with act NONE g_z equals g_out, z and g_z may be null
 * and nothing is written there.  g_b may be null (no bias).  The workspace
 * is the size fno_block_epilogue_workspace_size gives for FNO_OP_BWD_WEIGHT. */
fno_status fno_block_epilogue_bwd_weight(const fno_block_desc *desc, const void *x,
                                         const void *z, const void *g_out, void *g_z,
                                         float *g_w_skip, float *g_b, void *ws, size_t ws_len,
                                         hipStream_t stream);

/* Last backward step: gx = gx_spec + W_skip^T g_z (+ g_out with a residual),
 * gx_spec the spectral convolution's input gradient (taken at g_z).  g_out
 * is read only with a residual (may be null otherwise).  gx may be the same
 * buffer as gx_spec (in place). */
fno_status fno_block_epilogue_bwd_data(const fno_block_desc *desc, const void *g_z,
                                       const void *w_skip, const void *gx_spec,
                                       const void *g_out, void *gx, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Group norm with an activation, for the blocks' outputs (z of the epilogue
 * with act NONE, or any activation tensor of a model around the layers):
 *
 *     xh = (x - mean) / sqrt(var + eps),  out = act(gamma xh + beta) (+ residual)
 *
 * mean and var (the population variance) over all points of the channels of
 * one group of one sample: groups equal consecutive sets of channels / groups
 * channels (groups = channels normalises every plane by itself, groups = 1 a
 * whole sample).
 *
 * Tensors x, residual, out, g_out, gx are of one element type (fno_dtype) and
 * one layout: CHANNELS_FIRST [batch][channels][points], the layout of the
 * spectral convolution's tensors, or CHANNELS_LAST [batch][points][channels].
 * gamma, beta [channels] and their gradients are fp32, and so are the
 * statistics [batch][groups][2] = (mean, 1 / sqrt(var + eps)).  Sums are
 * formed in at least fp32, the statistics joined in double, results rounded
 * once.  Every sum has a fixed order: results are bit-identical from run to
 * run.  A group that holds a non-finite value gives NaN throughout; so does, in
 * the backward behind an activation, the group of a channel whose gamma or beta
 * is not finite.
 * ------------------------------------------------------------------------ */
typedef enum { FNO_DTYPE_F32 = 0, FNO_DTYPE_F16 = 1, FNO_DTYPE_BF16 = 2 } fno_dtype;

typedef enum { FNO_LAYOUT_CHANNELS_FIRST = 0, FNO_LAYOUT_CHANNELS_LAST = 1 } fno_layout;

typedef enum {
  FNO_NORM_ACT_NONE = 0,
  FNO_NORM_ACT_GELU = 1,  /* z Phi(z), Phi the exact normal distribution function */
  FNO_NORM_ACT_SILU = 2   /* z / (1 + exp(-z)) */
} fno_norm_activation;

typedef struct {
  int32_t dtype;       /* fno_dtype of the tensors */
  int32_t layout;      /* fno_layout */
  int32_t activation;  /* fno_norm_activation */
  float eps;           /* >= 0, finite */
  int64_t batch, points, channels;
  int64_t groups;      /* divides channels */
} fno_norm_desc;

/* Workspace bytes of a call, FNO_OP_FWD or FNO_OP_BWD (>= 256).
 * FNO_ERR_INVALID_ARGUMENT for a malformed descriptor (extents of at least 1,
 * channels up to 65536, batch x points x channels up to 2^38) or another op. */
fno_status fno_group_norm_act_workspace_size(const fno_norm_desc *desc, fno_op op,
                                             size_t *bytes);

/* Forward.  gamma and beta may be null (1 and 0), residual too (none added).
 * stats, if not null, receives the statistics that the backward takes (null
 * for inference).  out may be the same buffer as x or residual (in place). */
fno_status fno_group_norm_act_fwd(const fno_norm_desc *desc, const void *x,
                                  const float *gamma, const float *beta, const void *residual,
                                  void *out, float *stats, void *ws, size_t ws_len,
                                  hipStream_t stream);

/* Backward, from the forward's x, gamma, beta and stats and the output's
 * gradient: gx, and the parameter gradients g_gamma, g_beta (each may be null;
 * overwritten, not accumulated).  The residual's gradient is g_out itself.
 * gx may be the same buffer as g_out or x. */
fno_status fno_group_norm_act_bwd(const fno_norm_desc *desc, const void *x,
                                  const float *gamma, const float *beta, const float *stats,
                                  const void *g_out, void *gx, float *g_gamma, float *g_beta,
                                  void *ws, size_t ws_len, hipStream_t stream);

/* ------------------------------------------------------------------------
 * The optimizer step over all tensors of a model at once: AdamW (Adam with
 * decoupled weight decay), element by element
 *
 *     g = grad s;  m = b1 m + (1 - b1) g;  v = b2 v + (1 - b2) g^2
 *     p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
 *
 * in fp32, t the step's number (from 1).  Complex weights are their
 * interleaved (re, im) pairs, each a parameter of its own.  A list holds any
 * number of tensors of any sizes and types; one launch takes up to
 * FNO_ADAMW_LAUNCH_TENSORS of them.
 *
 * Parameters are fp32, or of a 16-bit type; then `master`, if not null, holds
 * the fp32 values that the step works on and `param` receives them rounded
 * (without a master the step works on the 16-bit values themselves, and
 * updates below half their last place are lost).  Gradients are fp32 (as the
 * weight gradients of this library are) or of the parameter's type.
 *
 * Moments take 32 bits each (exp_avg = m, exp_avg_sq = v, fp32 [n]) or 8 bits:
 * codes [n] with one fp32 scale per FNO_ADAMW_BLOCK consecutive elements of
 * the tensor (the last block may be short),
 *     m       = (A / 127^2) q |q|  int8 q,   A = max |m| of the block
 *     sqrt(v) = (B / 255^2) q^2    uint8 q,  B = max sqrt(v) of the block
 * rounded to nearest in the square root of the value, with q >= 1 wherever
 * v > 0: a second moment that is not zero does not become zero (but where
 * B < 2^-59, the square of whose smallest fraction leaves fp32), so that the
 * next step's quotient stays bounded.  The step itself uses the new moments
 * before they are rounded.  A block that holds a non-finite moment stands for
 * non-finite values throughout.
 *
 * An element's update has one fixed order of rounded operations and no sum
 * over other elements (8-bit blocks: a maximum), so it does not depend on how
 * a list is split.  Tensors of a list must not overlap.
 * ------------------------------------------------------------------------ */
#define FNO_ADAMW_BLOCK 256
#define FNO_ADAMW_LAUNCH_TENSORS 40

typedef struct {
  void *param;              /* [n] of param_dtype */
  float *master;            /* [n], or null; null where param_dtype is F32 */
  const void *grad;         /* [n] of grad_dtype */
  void *exp_avg;            /* [n] fp32, or int8 codes */
  void *exp_avg_sq;         /* [n] fp32, or uint8 codes */
  float *exp_avg_scale;     /* 8-bit states: [ceil(n / 256)], else null */
  float *exp_avg_sq_scale;  /* 8-bit states: [ceil(n / 256)], else null */
  int64_t n;                /* elements, 0 .. 2^34 (0: nothing is read or written) */
  int32_t param_dtype;      /* fno_dtype */
  int32_t grad_dtype;       /* FNO_DTYPE_F32 or param_dtype */
  int32_t state_bits;       /* 32 or 8 */
  float weight_decay;       /* >= 0, finite */
} fno_adamw_tensor;

typedef struct {
  double lr;          /* >= 0, finite */
  double beta1;       /* [0, 1) */
  double beta2;       /* [0, 1) */
  double eps;         /* >= 0, finite */
} fno_adamw_desc;

/* What steps of one optimizer share on the device, for training without a
 * host read between backward and update, and under HIP graph capture: 64
 * bytes of device memory, zeroed by the caller before first use (and after a
 * call that failed) except for lr_factor = 1 and, to go on from a checkpoint,
 * step.  fno_grad_norm writes all but lr_factor; its calls with one block
 * belong on one stream. */
typedef struct {
  int64_t step;       /* steps taken */
  int64_t skipped;    /* steps left out for non-finite gradients */
  double bias1;       /* 1 / (1 - beta1^step) */
  double bias2;       /* 1 / sqrt(1 - beta2^step) */
  float grad_norm;    /* L2 norm of the unscaled gradients of the last call */
  float grad_scale;   /* what the step multiplies gradients with */
  int32_t skip;       /* 1: the last gradients were not finite */
  float lr_factor;    /* multiplies lr (the caller's: a schedule under replay) */
  int32_t arrived;    /* the library's own; 0 between calls */
  int32_t reserved[3];
} fno_adamw_control;

/* The global gradient norm with clip, loss-scale removal and non-finite check:
 * over all gradients of the list (read only; the tensors' other pointers are
 * ignored),
 *     grad_norm  = inv_loss_scale sqrt(sum grad^2)      (sum in double)
 *     grad_scale = inv_loss_scale min(1, max_norm / grad_norm)
 * into `control`, step += 1 and the new step's bias corrections (desc's beta1
 * and beta2); where the sum is not finite instead skip = 1 and skipped += 1,
 * and the fno_adamw_step that follows changes nothing.  max_norm > 0
 * (INFINITY: no clip), inv_loss_scale > 0 and at most 3.4e38 (grad_scale is
 * fp32).  The sum has a fixed order: bit-identical from run to run. */
fno_status fno_grad_norm_workspace_size(const fno_adamw_tensor *tensors, int64_t count,
                                        size_t *bytes);
fno_status fno_grad_norm(const fno_adamw_desc *desc, const fno_adamw_tensor *tensors,
                         int64_t count, double max_norm, double inv_loss_scale,
                         fno_adamw_control *control, void *ws, size_t ws_len,
                         hipStream_t stream);

/* One step.  control null: step number `step` (>= 1) with gradients as they
 * are (s = 1).  control (device memory) not null: the step number, s and skip
 * that fno_grad_norm left there (each step needs a norm of its own before it: a
 * block that none has filled holds no bias corrections); `step` is ignored.
 * `tensors` is read during the call only.  count 0 does nothing. */
fno_status fno_adamw_step(const fno_adamw_desc *desc, const fno_adamw_tensor *tensors,
                          int64_t count, int64_t step, const fno_adamw_control *control,
                          hipStream_t stream);

/* Reads 8-bit moments out as the values they stand for, of element type
 * `dtype`: exp_avg_out[i], exp_avg_sq_out[i] (arrays of device pointers, [n]
 * each) for tensor i of the list (for checkpoints, or to go on with 32-bit
 * states).  Entries with 32-bit states are FNO_ERR_INVALID_ARGUMENT. */
fno_status fno_adamw_moments(const fno_adamw_tensor *tensors, int64_t count, fno_dtype dtype,
                             void *const *exp_avg_out, void *const *exp_avg_sq_out,
                             hipStream_t stream);

/* ------------------------------------------------------------------------
 * The norms around a block with its gate and residual scale, rows of `channels`
 * values (a grid's points, channels last, or any other rows):
 *
 *     n = post_w norm(u) + post_b          u: the block's output
 *     y = scale x + gate n                 x: the residual stream before it
 *     h = pre_w norm(y) + pre_b            h: the next block's input
 *
 *     norm(v) = (v - mean) / sqrt(var + eps)     FNO_ROW_NORM_LAYER
 *             = v / sqrt(mean(v^2) + eps)        FNO_ROW_NORM_RMS
 *
 * over the channels of each row, in one pass over the rows.  Without u it is
 * the norm before the first block, h = pre_w norm(x) + pre_b; without h the
 * join behind the last.  Rows x, u, y, h and their gradients are [rows][channels]
 * of one type (dtype).  Parameters are fp32 [channels], null ones are 1
 * (post_w, scale, pre_w) or 0 (post_b, pre_b).  The gate is [gate_rows][channels],
 * fp32 or of the rows' type; gate_rows divides rows, and each of its rows serves
 * rows / gate_rows consecutive rows: 1 (one gate for all), one per sample, or
 * one per row.  gate_rows 0: no gate (1).
 *
 * A row's sums are fp32; the parameters' are fp32 chains of at most 128
 * additions, joined in double.  Every sum has a fixed order: results are
 * bit-identical from run to run.  h is formed from y before its rounding.  A row with a
 * value that is not finite, or with LAYER a distance from its mean past fp32's
 * largest, gives NaN throughout; rows up to that size keep fp32's precision but for
 * two bits of 1 / sqrt(var), which is subnormal beyond 2^126.
 * ------------------------------------------------------------------------ */
typedef enum { FNO_ROW_NORM_LAYER = 0, FNO_ROW_NORM_RMS = 1 } fno_row_norm;

typedef struct {
  int32_t dtype;       /* fno_dtype of the rows */
  int32_t norm;        /* fno_row_norm */
  int32_t gate_dtype;  /* FNO_DTYPE_F32 or dtype */
  float eps;           /* >= 0, finite */
  int64_t rows;        /* 1 .. 2^40, rows x channels up to 2^42; a backward of
                          2^29 rows and more: FNO_ERR_UNSUPPORTED where one launch
                          does not hold it */
  int64_t channels;    /* 1 .. 16384 */
  int64_t gate_rows;   /* 0, or a divisor of rows; up to 2^22 - 1 unless it is
                          rows (FNO_ERR_UNSUPPORTED) */
} fno_residual_norm_desc;

typedef struct {
  const float *post_w, *post_b;
  const void *gate;  /* null if and only if gate_rows is 0 or there is no u */
  const float *scale, *pre_w, *pre_b;
} fno_residual_norm_params;

/* Gradients of the parameters, each null (not wanted) or of its parameter's
 * shape and type; overwritten, not accumulated. */
typedef struct {
  float *post_w, *post_b;
  void *gate;
  float *scale, *pre_w, *pre_b;
} fno_residual_norm_grads;

/* Forward.  u null: y, gate, scale, post_w, post_b are null too.  h null: pre_w
 * and pre_b are null too.  y may be the buffer of x or u, h that of u. */
fno_status fno_residual_norm_fwd(const fno_residual_norm_desc *desc,
                                 const fno_residual_norm_params *params, const void *x,
                                 const void *u, void *y, void *h, hipStream_t stream);

/* Backward, from the gradients g_y of y (null: zeros) and g_h of h (null: there
 * was no h), not both null:
 *     G = g_y + (gradient of the second norm at y)(g_h),   g_x = scale G,
 *     g_u = (gradient of the first norm at u)(gate G),
 * and the parameters' gradients, sums over rows.  y (the forward's) is needed
 * with g_h, x only for the scale's gradient.  Without u, x takes the place of y
 * and g_u is null.  g_x may be the buffer of g_y or g_h, g_u that of u or g_h; no
 * two results share a buffer. */
fno_status fno_residual_norm_workspace_size(const fno_residual_norm_desc *desc, size_t *bytes);
fno_status fno_residual_norm_bwd(const fno_residual_norm_desc *desc,
                                 const fno_residual_norm_params *params, const void *x,
                                 const void *u, const void *y, const void *g_y, const void *g_h,
                                 void *g_x, void *g_u, const fno_residual_norm_grads *grads,
                                 void *ws, size_t ws_len, hipStream_t stream);

/* ------------------------------------------------------------------------
 * Products in 8-bit floating point with a scale for each block of 128.
 *
 * A matrix [rows][cols] is held as codes of e4m3 (largest value 448, no
 * infinity) or e5m2 (57344), one byte each, rows of fno_fp8_pitch(cols) =
 * cols rounded up to 16 codes (zeros behind cols), and one scale for each block:
 *     FNO_BLOCKS_ROW   128 consecutive columns of one row: [ceil(cols/128)][rows]
 *     FNO_BLOCKS_TILE  128 x 128:           [ceil(cols/128)][ceil(rows/128)]
 * (the last blocks may be short).  A value is its code times its block's scale.
 * Scales are powers of two held in one byte, 2^(byte - 127) (FNO_SCALE_POW2; 255
 * stands for NaN), or fp32 numbers (FNO_SCALE_F32).
 * ------------------------------------------------------------------------ */
#define FNO_FP8_BLOCK 128
typedef enum { FNO_FP8_E4M3 = 0, FNO_FP8_E5M2 = 1 } fno_fp8_format;
typedef enum { FNO_SCALE_POW2 = 0, FNO_SCALE_F32 = 1 } fno_scale_type;
typedef enum { FNO_BLOCKS_ROW = 0, FNO_BLOCKS_TILE = 1 } fno_fp8_blocks;

typedef struct {
  int32_t dtype;       /* fno_dtype of x */
  int32_t format;      /* fno_fp8_format of the codes */
  int32_t scale_type;  /* fno_scale_type */
  int32_t blocks;      /* fno_fp8_blocks */
  int32_t activation;  /* fno_norm_activation */
  int64_t rows, cols;  /* >= 1, each up to 2^31 - 1; rows x cols below 2^38
                          (FNO_ERR_UNSUPPORTED) */
} fno_fp8_quantize_desc;

/* x [rows][cols] to the codes of v = act(x): `codes` [rows][pitch(cols)] with
 * blocks along its rows (or tiles), and `codes_t`, those of the transpose
 * [cols][pitch(rows)] with blocks along its own rows (the columns of x).
 * Either pair of codes and scales may be null.  With F the format's largest
 * value and a the largest size of a block's finite values, the scale is
 *     POW2   2^max(e, -126), e the least with a <= F 2^e
 *     F32    max(a (1 / F), 2^-126), both operations in fp32 (at most one unit in
 *            the last place from the rounded quotient: what torch makes, on the
 *            GPU, of a tensor divided by a number, so that codes formed so agree),
 * 1 where a = 0; the code is v times the scale's reciprocal (an fp32 product)
 * rounded to nearest, ties to even.  NaN stays NaN; an infinity becomes NaN in
 * e4m3.  col_sums, if not null, receives the sums of v over rows (fp32 [cols],
 * fixed order: what a bias's gradient is).  No two results share a buffer. */
int64_t fno_fp8_pitch(int64_t cols);
fno_status fno_fp8_quantize_workspace_size(const fno_fp8_quantize_desc *desc, size_t *bytes);
fno_status fno_fp8_quantize(const fno_fp8_quantize_desc *desc, const void *x, void *codes,
                            void *scale, void *codes_t, void *scale_t, float *col_sums, void *ws,
                            size_t ws_len, hipStream_t stream);

typedef struct {
  int32_t format_a, format_b;  /* fno_fp8_format */
  int32_t scale_type;          /* fno_scale_type of both */
  int32_t blocks_a, blocks_b;  /* fno_fp8_blocks */
  int32_t out_dtype;           /* fno_dtype of out and z */
  int32_t activation;          /* fno_norm_activation: whose derivative multiplies */
  int64_t rows, cols, inner;   /* >= 1, each up to 2^31 - 1, with rows x cols
                                  below 2^37 (FNO_ERR_UNSUPPORTED where one
                                  launch does not hold the tiles) */
} fno_fp8_matmul_desc;

/* out = (A B^T) act'(z) + bias:  A [rows][inner] and B [cols][inner] in codes,
 * out and z [rows][cols], bias fp32 [cols] (null: none).  z is null if and only
 * if the activation is NONE.  Sums are fp32 in a fixed order, with one rounding to
 * out_dtype.  For out_dtype F32 every product enters them exactly; for 16-bit
 * results the matrix instruction for 8-bit codes joins eight consecutive products
 * at a time, each cut towards zero to a multiple of 2^-13 of the power of two below
 * the largest of the eight.  For F32 with powers of two, values (codes times their
 * scales) below 2^-126 count as the nearest multiple of 2^-133, past fp32's largest
 * as infinite; with fp32 scales the product of two scales is an fp32 number.  A row
 * of codes is read whole, fno_fp8_pitch(inner) bytes: what stands behind `inner` has
 * to be zero. */
fno_status fno_fp8_matmul_workspace_size(const fno_fp8_matmul_desc *desc, size_t *bytes);
fno_status fno_fp8_matmul(const fno_fp8_matmul_desc *desc, const void *a, const void *scale_a,
                          const void *b, const void *scale_b, const void *z, const float *bias,
                          void *out, void *ws, size_t ws_len, hipStream_t stream);

/* Per-kernel timing with HIP events (a profiling aid, off by default).
 * While enabled, every kernel the library launches is bracketed by a pair of
 * HIP events recorded on the launch stream (events are created per launch, so
 * this mode allocates and is not for graph capture).  fno_profile_read
 * synchronises the pending events and returns, for the index-th kernel name
 * seen (0-based, in order of first launch), its name, launch count and total
 * elapsed milliseconds; FNO_ERR_INVALID_ARGUMENT past the last name. */
fno_status fno_profile_enable(int32_t enable);
fno_status fno_profile_reset(void);
fno_status fno_profile_read(int32_t index, char *name, int32_t name_cap, int64_t *launches,
                            double *total_ms);

/* Drops every cached plan (device tables) of this process.  A plan that a
 * call on another thread is using stays alive until that call returns;
 * every other plan's tables are freed here.  The tables may still be read by
 * kernels already enqueued: call this only when no work issued through the
 * library is in flight (after a device or stream synchronisation).  HIP
 * graphs captured earlier hold the freed table addresses: re-capture them
 * (after one warm-up call) once the caches have been released. */
fno_status fno_release_caches(void);

const char *fno_status_string(fno_status status);

/* Detail of the last FNO_ERR_HIP returned on the calling thread: the HIP
 * error's name and code and the step that failed (a kernel name or a HIP
 * call).  Empty if no call on this thread has returned FNO_ERR_HIP.  The
 * string is owned by the library and valid until the thread's next failing
 * call. */
const char *fno_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* FNO_SPECTRAL_CONV_H_ */
