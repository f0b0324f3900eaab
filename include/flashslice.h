/*
 * flashslice.h -- C ABI of the GB300 slice -> token mix -> deslice library.
 *
 * The operation is the coupling of Transolver's physics-attention sublayer
 * with a constant token core (paper Sec. 2 "The Transolver layer" and Eq. (1);
 * Appendix G.1 "Single-tile kernels" / "G-blocked kernels").  Per batch b and
 * head h, with x = x_mid[b,:,h,:] (N x d), f = fx[b,:,h,:] (N x d),
 * W = W_slice[h] (d x G), beta = bias[h] (G), tau = tau[h]:
 *
 *   a_ng   = (x_n . W[:,g] + beta_g) / tau           slice logits
 *   w_ng   = exp(a_ng - lse_n),  lse_n = log sum_g exp(a_ng)
 *   S_g    = sum_n w_ng,   U_g = sum_n w_ng f_n      (partials over points)
 *   z_g    = U_g / (S_g + eps)                       tokens
 *   z'_g   = sum_k M[g,k] z_k                        constant G x G mix
 *   out_n  = sum_g w_ng z'_g                         deslice, tied weights
 *
 * The N x H x G weight tensor w is never written to memory: every pass
 * recomputes it tile by tile from x_mid and the per-point statistic lse.
 *
 * Conventions for every entry point
 *  - All tensor pointers are DEVICE pointers owned by the caller.  The library
 *    never allocates, frees or synchronises (except fs_device_status, which
 *    synchronises `stream` to read the status word).  Every call is
 *    asynchronous on `stream` (a cudaStream_t; NULL = legacy default stream).
 *  - Layouts are dense, row-major, contiguous:
 *      x_mid, fx, out, dout, dx_mid, dfx : [B, N, H, d]   dtype of the shape
 *      W_slice, dW                       : [H, d, G]      fp32
 *      bias, dbias                       : [H, G]         fp32
 *      tau, dtau                         : [H]            fp32
 *      M, dM                             : [H, G, G]      fp32, M[h][g][k]
 *      tokens, tokens_mixed, d_tokens*   : [B, H, G, d]   fp32
 *      wsum                              : [B, H, G]      fp32
 *      lse                               : [B, H, N]      fp32, natural log
 *    Channel c of a point's C = H*d features is head c / d, lane c % d.
 *  - A bias of -inf, or one that overflows to it in the scaling by 1/tau, masks its slot: weight 0
 *    for every point, gradients 0.  Each head needs at least one slot that is not masked.
 *  - Every pointer must be 16-byte aligned.
 *  - `ws` is caller-owned scratch of at least fs_workspace_bytes(shape, op)
 *    bytes (16-byte aligned).  Its first word is a device status word that
 *    each call resets; fs_device_status reads it.
 *  - Host-side validation fails with FS_ERR_INVALID / FS_ERR_UNSUPPORTED
 *    before anything is launched.  Device-side problems (tau <= 0 or not
 *    finite; a bounded wait that gave up) are written to the status word and
 *    the affected kernel skips its work; no kernel traps.
 *  - Results are deterministic: no floating-point atomics; partial sums over
 *    points are reduced in a fixed order, so repeated calls on the same
 *    device agree bit for bit.
 *  - Supported: d in {16, 32, 64}; G in [1, 4096]; B*H <= 65535; B*N*H*d < 2^40.
 *    Kernels (fs_path_for_shape, fs_backward_path_for_shape say which):
 *      FS_BF16, d = 32, G <= 1024: the forward on tcgen05 tensor cores, fp32
 *        accumulation, at the dot level of fs_shape.dot (below).
 *      FS_BF16, d = 32, N >= 2 (any supported G): the backward on tensor cores,
 *        always with split products; past G = 640 its passes run over ranges of
 *        at most 640 slots, whose dx_mid and dfx contributions are summed in bf16.
 *      FS_F32, d = 32, G <= 1024, B*N*H*G >= 2^24: the forward on tensor cores
 *        with every operand split into two bf16 halves (normwise relative error
 *        ~1e-5); the backward in fp32 FMA.
 *      everything else: fp32 FMA (SIMT) kernels.
 *
 * Call sequence of one coupling (a training step):
 *   fs_slice_fwd   (x_mid, fx)            -> tokens, wsum, lse
 *   fs_mix         (M, tokens)            -> tokens_mixed   (or fs_mix_channels, or the
 *                                            original layer's attention, fs_attn_fwd)
 *   fs_deslice_fwd (x_mid, tokens_mixed, lse) -> out
 *   fs_deslice_bwd (..., dout)            -> d_tokens_mixed, dx_mid, dW, dbias, dtau
 *   fs_mix_bwd     (M, tokens, d_tokens_mixed) -> d_tokens, dM
 *   fs_slice_bwd   (..., d_tokens, accumulate = 1) -> dfx; adds to dx_mid, dW, dbias, dtau
 * Each call that takes `ws` gets scratch sized by fs_workspace_bytes for its op.
 */
#ifndef FLASHSLICE_H
#define FLASHSLICE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* fs_stream_t; /* identical to cudaStream_t */

typedef enum fs_status {
  FS_OK = 0,
  FS_ERR_INVALID = 1,     /* null/misaligned pointer, bad size, workspace too small */
  FS_ERR_UNSUPPORTED = 2, /* well-formed shape that no kernel implements (e.g. d = 48) */
  FS_ERR_CUDA = 3,        /* a CUDA runtime call or kernel launch failed */
  FS_ERR_TIMEOUT = 4,     /* device: a bounded wait gave up (status word only) */
  FS_ERR_BAD_TAU = 5,     /* device: some tau[h] <= 0 or not finite (status word only) */
  FS_ERR_SCRATCH_TOO_SMALL = 6 /* fs_slice_fwd_noalloc: the shape needs more than its fixed scratch */
} fs_status;

typedef enum fs_dtype { FS_F32 = 0, FS_BF16 = 1 } fs_dtype;

/* Arithmetic of the point-by-slot products for FS_BF16 shapes on the tensor
 * cores (the paper's "dot levels", App. G.2; fp32 accumulation throughout):
 *   FS_DOT_BF16   both operands of every product in bf16: W log2(e)/tau and the
 *                 slice weights rounded to bf16 (the paper's "bf16" level).
 *                 Outputs within ~1e-2 relative of exact.
 *   FS_DOT_BF16X2 W log2(e)/tau and the slice weights each carried as two bf16
 *                 halves (hi + lo, ~2^-16 relative) in the statistics and slice
 *                 passes, and in the deslice where its images fit in shared
 *                 memory (G <= 768): tokens, weight sums and lse to ~1e-4,
 *                 which the temperature gradient needs (a near-cancelling sum).
 *                 Slower: two more K-steps per logits block, twice the slice
 *                 products.
 * Ignored for FS_F32 shapes (split into bf16 halves on the tensor cores, or
 * fp32 FMA) and on the SIMT path. */
typedef enum fs_dot { FS_DOT_BF16 = 0, FS_DOT_BF16X2 = 1 } fs_dot;

typedef struct fs_shape {
  int64_t B;     /* batch size, >= 1 */
  int64_t N;     /* points per sample, >= 1 */
  int32_t H;     /* heads, >= 1 */
  int32_t d;     /* head width (value width equals it), 16, 32 or 64 */
  int32_t G;     /* slices per head, 1..4096 */
  int32_t dtype; /* fs_dtype of the [B,N,H,d] point tensors */
  float eps;     /* added to the weight sums before normalising, >= 0 (paper: 1e-5) */
  int32_t dot;   /* fs_dot: product arithmetic of the tensor-core path */
} fs_shape;

typedef enum fs_op {
  FS_OP_SLICE_FWD = 0,
  FS_OP_DESLICE_FWD = 1,
  FS_OP_DESLICE_BWD = 2,
  FS_OP_SLICE_BWD = 3,
  FS_OP_STATS = 4,
  FS_OP_COUPLING_BWD = 5
} fs_op;

/* Bytes of scratch `ws` that entry point `op` needs for this shape on the
 * current device (0 for an invalid shape).  Depends on the device's SM count. */
size_t fs_workspace_bytes(const fs_shape* s, int op);

/* Slice (Sec. 2; App. G.1 "G-blocked kernels": statistics, slot-owned partial
 * numerators and weight sums, normalisation after the partials are combined).
 *   in : x_mid, fx [B,N,H,d]; W_slice [H,d,G]; bias [H,G]; tau [H]
 *   out: tokens [B,H,G,d] = U/(S+eps) if finalize != 0, else the unnormalised
 *        numerators U (for a cross-device sum before fs_slice_finalize);
 *        wsum [B,H,G] = S; lse [B,H,N] (may be NULL: then kept in ws only). */
fs_status fs_slice_fwd(const fs_shape* s, const void* x_mid, const void* fx,
                       const float* W_slice, const float* bias, const float* tau,
                       float* tokens, float* wsum, float* lse, int finalize,
                       void* ws, size_t ws_bytes, fs_stream_t stream);

/* The statistics pass alone (App. G.1, the per-point statistic of the G-blocked
 * kernels): lse [B,H,N] (natural log) of the logits of these weights, exactly as
 * fs_slice_fwd writes it.  With fs_slice_fwd_lse it splits fs_slice_fwd in two,
 * so that fx can still be on its way to the device while the statistics run;
 * it also gives an untied deslice or a FrozenSlice layer its statistics.
 * ws: FS_OP_STATS's workspace. */
fs_status fs_stats(const fs_shape* s, const void* x_mid, const float* W_slice,
                   const float* bias, const float* tau, float* lse, void* ws,
                   size_t ws_bytes, fs_stream_t stream);

/* Slice given its statistics: fs_slice_fwd with lse [B,H,N] an input (as
 * fs_slice_fwd writes it, natural log) and no statistics pass.  For the
 * FrozenSlice variant (Sec. 3, the variants table: the slice weights of layer 1
 * reused by every layer), where a later layer slices its own fx with the
 * layer-1 logits input, weights and statistics; and for any caller that
 * already holds lse for these weights.  ws: FS_OP_SLICE_FWD's workspace. */
fs_status fs_slice_fwd_lse(const fs_shape* s, const void* x_mid, const void* fx,
                           const float* W_slice, const float* bias, const float* tau,
                           const float* lse, float* tokens, float* wsum, int finalize,
                           void* ws, size_t ws_bytes, fs_stream_t stream);

/* tokens <- tokens / (wsum + eps), in place ("column normalisation after
 * partials have been combined", App. G.1). */
fs_status fs_slice_finalize(const fs_shape* s, float* tokens, const float* wsum,
                            fs_stream_t stream);

/* Constant token mix, the core of Eq. (1) acting on the slot index:
 * tokens_mixed[b,h,g,:] = sum_k M[h,g,k] tokens[b,h,k,:].  Out-of-place only: an
 * output that shares any byte with an input is rejected (FS_ERR_INVALID). */
fs_status fs_mix(const fs_shape* s, const float* M, const float* tokens,
                 float* tokens_mixed, fs_stream_t stream);

/* The attention-free core (Sec. 2 after Eq. (1); "NoTokenAttn" in the Sec. 3
 * variants table): A is the identity, so the tokens do not interact, and a
 * learned linear map acts on the channels of each token, one per head:
 * tokens_mixed[b,h,g,c] = sum_k Wc[h,c,k] tokens[b,h,g,k].  Wc [H,d,d] fp32.
 * Out-of-place only (overlapping input and output: FS_ERR_INVALID).  It may
 * replace fs_mix, or follow it (the two commute). */
fs_status fs_mix_channels(const fs_shape* s, const float* Wc, const float* tokens,
                          float* tokens_mixed, fs_stream_t stream);

/* Backward of fs_mix_channels: d_tokens[b,h,g,k] = sum_c Wc[h,c,k]
 * d_tokens_mixed[b,h,g,c] (overwritten); dWc [H,d,d] = sum over b and g of
 * d_tokens_mixed tokens^T (overwritten).  Outputs that overlap an input or each
 * other: FS_ERR_INVALID. */
fs_status fs_mix_channels_bwd(const fs_shape* s, const float* Wc, const float* tokens,
                              const float* d_tokens_mixed, float* d_tokens, float* dWc,
                              fs_stream_t stream);

/* The same with d_tokens added to, for tokens that several maps read (the query, key and value
 * maps of the token attention); dWc is overwritten. */
fs_status fs_mix_channels_bwd_add(const fs_shape* s, const float* Wc, const float* tokens,
                                  const float* d_tokens_mixed, float* d_tokens, float* dWc,
                                  fs_stream_t stream);

/* Deslice with tied weights (Sec. 2; App. G.1): out[b,n,h,:] = sum_g w z'_g.
 *   lse: statistics from fs_slice_fwd; NULL makes the call compute them first
 *   (into ws).  out has the dtype of the shape.  The Untied variant (Sec. 3, the
 *   variants table: the deslice gets its own projection and temperature) passes
 *   its own W_slice, bias, tau and lse = NULL. */
fs_status fs_deslice_fwd(const fs_shape* s, const void* x_mid, const float* W_slice,
                         const float* bias, const float* tau, const float* tokens_mixed,
                         const float* lse, void* out, void* ws, size_t ws_bytes,
                         fs_stream_t stream);

/* Backward of the deslice given dout (App. G.1 "Backward uses separate
 * point-owned and slot-owned kernels"; temperature gradient App. G.2):
 *   d_tokens_mixed [B,H,G,d] = sum_n w_ng dout_n  (always overwritten)
 *   dx_mid [B,N,H,d], dW [H,d,G], dbias [H,G], dtau [H]: the contribution of
 *   the deslice weights; written if accumulate == 0, added if accumulate != 0.
 *   lse: the statistics of these weights from the forward, or NULL (an untied
 *   deslice, which kept none): the call then computes them into ws.  The backward
 *   forms its weights from fp32 logits and needs lse to ~1e-5: on tensor-core
 *   shapes (fs_path_for_shape == 1) with dot = FS_DOT_BF16, whose lse comes
 *   from logits with bf16-rounded W log2(e)/tau, it recomputes lse with split
 *   products into ws; otherwise it uses the caller's lse. */
fs_status fs_deslice_bwd(const fs_shape* s, const void* x_mid, const float* W_slice,
                         const float* bias, const float* tau, const float* tokens_mixed,
                         const float* lse, const void* dout, float* d_tokens_mixed,
                         void* dx_mid, float* dW, float* dbias, float* dtau,
                         int accumulate, void* ws, size_t ws_bytes, fs_stream_t stream);

/* Backward of the mix: d_tokens = M^T d_tokens_mixed per (b,h) (overwritten);
 * dM [H,G,G] = sum_b d_tokens_mixed tokens^T (overwritten).  Outputs that overlap
 * an input or each other: FS_ERR_INVALID. */
fs_status fs_mix_bwd(const fs_shape* s, const float* M, const float* tokens,
                     const float* d_tokens_mixed, float* d_tokens, float* dM,
                     fs_stream_t stream);

/* Backward of the slice given d_tokens (the gradient w.r.t. the normalised
 * tokens); tokens and wsum are the forward's normalised tokens and S; lse as
 * in fs_deslice_bwd (NULL: computed; recomputed with split products for
 * FS_DOT_BF16).
 *   dfx [B,N,H,d] (overwritten); dx_mid, dW, dbias, dtau: written if
 *   accumulate == 0, added if accumulate != 0. */
fs_status fs_slice_bwd(const fs_shape* s, const void* x_mid, const void* fx,
                       const float* W_slice, const float* bias, const float* tau,
                       const float* tokens, const float* wsum, const float* lse,
                       const float* d_tokens, void* dx_mid, void* dfx, float* dW,
                       float* dbias, float* dtau, int accumulate, void* ws,
                       size_t ws_bytes, fs_stream_t stream);

/* The whole backward of one coupling in one call: the results of
 *   fs_deslice_bwd(..., accumulate) ; fs_mix_bwd ; fs_slice_bwd(..., accumulate = 1)
 * (App. G.1 backward; App. G.2 temperature gradient; the mix backward of Eq. (1)).
 *   d_tokens_mixed, d_tokens [B,H,G,d], dfx [B,N,H,d], dM [H,G,G]: overwritten;
 *   dx_mid [B,N,H,d], dW [H,d,G], dbias [H,G], dtau [H]: the sum of both calls'
 *   contributions, written if accumulate == 0, added if accumulate != 0.
 *   tokens, wsum, tokens_mixed, lse: the forward's (lse may be NULL, as in the
 *   separate calls).  ws: fs_workspace_bytes(s, FS_OP_COUPLING_BWD).
 * The two calls' da_ng share the weights, so one point pass over (point, slot)
 * forms da_D + da_S and dx from it, and one slot pass dW, dbias, dtau, instead of
 * one of each per call; d_tokens_mixed comes first, as the slice's unnormalised
 * numerators with dout for fx.  This holds on the tensor-core backward
 * (fs_backward_path_for_shape == 1) and on the fp32 SIMT one.  Results agree with
 * the separate calls to rounding (for instance dx is summed before its one rounding
 * to the input dtype instead of after each call's).  M, tokens and tokens_mixed
 * overlapping an output, or two outputs overlapping each other: FS_ERR_INVALID. */
fs_status fs_coupling_bwd(const fs_shape* s, const void* x_mid, const void* fx,
                          const float* W_slice, const float* bias, const float* tau,
                          const float* M, const float* tokens, const float* wsum,
                          const float* tokens_mixed, const float* lse, const void* dout,
                          float* d_tokens_mixed, float* d_tokens, void* dx_mid, void* dfx,
                          float* dW, float* dbias, float* dtau, float* dM, int accumulate,
                          void* ws, size_t ws_bytes, fs_stream_t stream);

/* ---- Self-attention of the slice tokens --------------------------------------------------
 *
 * The token operation of the original layer (Sec. 2, "The Transolver layer"; the "baseline"
 * of the Sec. 3 variants table), in place of fs_mix: the core of Eq. (1) depends on the
 * tokens.  q, k, v are the tokens' projections (fs_mix_channels makes them).  Per batch b
 * and head h, with key head h / (H / Hkv), query i and key j:
 *
 *   s_ij = scale q_i . k_j
 *   c_ij = cap tanh(s_ij / cap)  if cap > 0, else s_ij           capped scores
 *   a_ij = c_ij - slopes[h] |pos_q[b,i] - pos_k[b,j]|            distance bias
 *   a masked pair has weight 0
 *   lse_i = log sum_j exp(a_ij),  p_ij = exp(a_ij - lse_i),  out_i = sum_j p_ij v_j
 *
 * Masks (a pair is seen if every mask in use allows it):
 *   documents: doc_q[b,i] == doc_k[b,j] and doc_k[b,j] >= 0.  Tokens of several bodies or
 *     samples share a batch entry this way, in any order; a negative number marks a token
 *     that is not in use (a slot that no point fills).
 *   FS_MASK_PREFIX: key j <= i + (Gk - Gq), or j < prefix[b] (NULL: 0, each query sees its
 *     own and earlier keys).  The queries are the last Gq of the Gk tokens; Gq <= Gk.
 * A query that sees no key (or only keys with a score of -infinity) has out = 0, lse =
 * -infinity and gradients 0.  What masked tokens hold, NaN and infinities included, reaches
 * no result of a query or key that does not see them.
 *
 * Everything is fp32: [B, H, Gq, d] for q, out, dout, dq; [B, Hkv, Gk, d] for k, v, dk, dv;
 * lse [B, H, Gq].  The products run on the tensor cores with every operand split into two
 * tf32 parts (2^-22 relative, where an fp32 product rounds by 2^-24), the exponential is the
 * hardware's 2^x (2^-22 relative), accumulation is fp32.  A pair whose weight
 * underflows to 0 adds nothing, whatever its tokens hold.  Hkv divides H; heads that share a key
 * head have their dk and dv summed.  Supported: d in {16, 32, 64}; Gk and (H / Hkv) Gq up to
 * 2^20; B*H <= 65535; B*H*max(Gq, Gk)*d < 2^40.  No output may share a byte with an input or
 * another output (FS_ERR_INVALID). */
typedef enum fs_mask { FS_MASK_NONE = 0, FS_MASK_PREFIX = 1 } fs_mask;

typedef struct fs_attn_shape {
  int64_t B;    /* batch size, >= 1 */
  int32_t H;    /* query heads */
  int32_t Hkv;  /* key and value heads, divides H */
  int32_t Gq;   /* queries per head */
  int32_t Gk;   /* keys per head */
  int32_t d;    /* head width, 16, 32 or 64 */
  int32_t mask; /* fs_mask */
  float scale;  /* finite, as is scale log2(e) */
  float cap;    /* >= 0; 0: scores are not capped.  scale / cap is finite, and so is cap log2(e)
                 * unless |scale / cap| < 2^-126, where a cap has no effect and is not applied */
} fs_attn_shape;

/* Device pointers, 4-byte aligned, each may be NULL; the struct itself is read on the host
 * during the call. */
typedef struct fs_attn_mask {
  const float* slopes;  /* [H]: the distance bias; constants, no gradient */
  const float* pos_q;   /* [B, Gq], with slopes and pos_k only; NULL: i + (Gk - Gq) */
  const float* pos_k;   /* [B, Gk]; NULL: j */
  const int32_t* doc_q; /* [B, Gq], together with doc_k */
  const int32_t* doc_k; /* [B, Gk] */
  const int32_t* prefix; /* [B], under FS_MASK_PREFIX only */
} fs_attn_mask;

/* mask may be NULL (no bias, no documents).  ws: fs_attn_workspace_bytes(s, 0). */
fs_status fs_attn_fwd(const fs_attn_shape* s, const float* q, const float* k, const float* v,
                      const fs_attn_mask* mask, float* out, float* lse, void* ws, size_t ws_bytes,
                      fs_stream_t stream);

/* Gradients for dout, with out and lse of the forward; all overwritten.
 * ws: fs_attn_workspace_bytes(s, 1). */
fs_status fs_attn_bwd(const fs_attn_shape* s, const float* q, const float* k, const float* v,
                      const fs_attn_mask* mask, const float* out, const float* lse,
                      const float* dout, float* dq, float* dk, float* dv, void* ws,
                      size_t ws_bytes, fs_stream_t stream);

/* Bytes of scratch on the current device; 0 for an invalid or unsupported shape. */
size_t fs_attn_workspace_bytes(const fs_attn_shape* s, int backward);

/* Kernel path of fs_attn_fwd, or of fs_attn_bwd (backward != 0), for this shape: 0 = warps of 16
 * rows, 1 = tcgen05 tiles of 128 rows; -1 for an invalid or unsupported shape.  For tests and
 * benchmarks. */
int fs_attn_path_for_shape(const fs_attn_shape* s, int backward);

/* ---- Layer norm and 8-bit checkpoints of point features ----------------------------------
 *
 * The original layer normalises the residual stream before the coupling's projections
 * (Sec. 2 "The Transolver layer"), and a training step keeps its activations for the
 * backward pass.  These calls work on `rows` rows of C channels (the B*N points' C = H*d
 * features; or the B*H*G tokens' d channels), dense and row-major, in the dtype of the
 * fs_rows; gamma, beta, mean, rstd and their gradients are fp32.
 *
 * An 8-bit checkpoint of x [rows, C] is q8 [rows, C] (int8) with e8 [rows, ceil(C / 32)]
 * (uint8): each block of 32 channels of a row (the last one may be shorter) is kept as
 * x ~ q 2^s with e8 = s + 127; q is x 2^-s rounded to nearest, ties to even, and s is the
 * smallest >= -126 at which the ROUNDED largest magnitude of the block is at most 127 (so up to
 * just below 127.5 steps).  Each value is off by at most half a step, 2^(s-1), which is at most
 * 1/127.5 = 2^-6.994 of the block's largest magnitude (where s is -126: 2^-127).
 * A block that holds NaN or infinity has e8 = 255 and restores to NaN.  The values are exact
 * in both dtypes.
 *
 * Supported: rows >= 1, C in [1, 8192], rows*C < 2^40.  Pointers as above: device,
 * 16-byte aligned, asynchronous on `stream`.  Outputs may not share a byte with an input or
 * another output, except where a call says so (FS_ERR_INVALID). */
typedef struct fs_rows {
  int64_t rows;  /* >= 1 */
  int32_t C;     /* channels of a row, 1..8192 */
  int32_t dtype; /* fs_dtype of the rows */
} fs_rows;

/* Layer norm of v = x + res over each row's channels:
 *   y = (v - mean) rstd gamma + beta,  rstd = 1 / sqrt(var + eps)  (var over C, biased)
 *   res: NULL for v = x.  With it v is rounded to the dtype, and that value is normalised.
 *   sum: NULL, or receives v (only with res; may be x or res itself: the stream in place).
 *   gamma, beta [C]: NULL stands for 1 and 0.  mean, rstd [rows]: NULL to leave them out.
 *   q8, e8: both NULL, or receive v's 8-bit checkpoint.
 * One kernel: each input is read once, each output written once. */
fs_status fs_norm_fwd(const fs_rows* s, const void* x, const void* res, const float* gamma,
                      const float* beta, float eps, void* sum, void* y, float* mean, float* rstd,
                      int8_t* q8, uint8_t* e8, fs_stream_t stream);

/* Backward of fs_norm_fwd given dy: with xh = (v - mean) rstd and g = dy gamma,
 *   dv = rstd (g - avg_c(g) - xh avg_c(g xh)) + dres,  dgamma = sum_rows dy xh,
 *   dbeta = sum_rows dy.
 *   v: the normalised rows, or NULL and their checkpoint q8, e8 (xh is then formed from the
 *   values that it stands for).  mean, rstd: the forward's.
 *   dres: NULL, or the gradient that reaches v along the residual stream.
 *   dv may be dy or dres itself.  dv is the gradient of x and of res.
 *   dgamma, dbeta: both NULL, or written (accumulate == 0) or added to (accumulate != 0).
 * ws: fs_norm_workspace_bytes(s). */
fs_status fs_norm_bwd(const fs_rows* s, const void* v, const int8_t* q8, const uint8_t* e8,
                      const float* gamma, const float* mean, const float* rstd, const void* dy,
                      const void* dres, void* dv, float* dgamma, float* dbeta, int accumulate,
                      void* ws, size_t ws_bytes, fs_stream_t stream);

/* Bytes of scratch that fs_norm_bwd needs on the current device; 0 for invalid or
 * unsupported rows. */
size_t fs_norm_workspace_bytes(const fs_rows* s);

/* x into its 8-bit checkpoint (q8, e8), and back into the values that it stands for. */
fs_status fs_ckpt_pack(const fs_rows* s, const void* x, int8_t* q8, uint8_t* e8, fs_stream_t stream);
fs_status fs_ckpt_unpack(const fs_rows* s, const int8_t* q8, const uint8_t* e8, void* x,
                         fs_stream_t stream);

/* ---- Linear maps of rows, and dropout -----------------------------------------------------
 *
 * Around the coupling, the original layer (Sec. 2 "The Transolver layer") projects the normalised
 * stream to x_mid and fx, projects the coupling's output back and adds it to the stream, and ends
 * with a two-layer MLP, dropout behind each.  One call does a product with all that follows it:
 *   u = x W^T + bias,   y = res + drop(act(u))
 *   x [rows, Cin], res, y [rows, Cout] in the dtype; W [Cout, Cin] in the dtype; bias [Cout] fp32.
 *   pre: NULL, or receives u (rounded to the dtype), which the backward of an activation needs.
 *   bias, res: NULL for none.  res may be y itself (the stream in place).
 * Activations: NONE; RELU; GELU u Phi(u), Phi the normal distribution's function; SILU u / (1 + e^-u).
 *
 * Dropout: drop(a) = a / (1 - p) where the value is kept, 0 where it is not (what it holds, NaN and
 * infinities included, is not looked at).  p in [0, 1); 0: none, rng may be NULL.  The mask is
 * never stored: channel c of row r is kept if word c % 4 of Philox 4x32-10 (Salmon et al., 2011),
 * with the key rng[0] and the 128-bit counter (r ceil(C / 4) + c / 4) + 2^64 rng[1], is at least
 * floor(p 2^32); C: the row's channels.  rng: two 64-bit words {seed, offset} in DEVICE memory, so
 * that a captured graph draws anew when the caller advances the offset.  A call whose backward
 * shall see its mask gets the same two words there; calls that shall not share a mask (another
 * layer, another step) get different offsets.
 *
 * Sums are fp32.  FS_BF16: products of bf16 values, exact; GELU and SILU to 2^-16 of themselves (where
 * they are below 2^-119: to 2^-119), their derivatives to 2^-19; y, pre and dx rounded to bf16.  FS_F32:
 * fp32 throughout; on tensor cores operands in three bf16 parts, which leave out at most 2^-25 of a value, or
 * 2^-134 where that is more.  A sum of K products whose magnitudes add up to S is off by at most
 * (180 + K / 128) 2^-24 S where the result is fp32 (dW and dbias always), and (180 + K / 8) 2^-24 S before it is
 * rounded to bf16.  Of terms of random sign, up to a million, fp32 results measure within 5e-7 of their norm, dW of
 * bf16 rows within 1e-6.
 * Infinities and NaN in x, W, g or a bias go through sums, activations and residuals as in fp32 arithmetic, and to no
 * results that they do not enter; a dropped value is 0 whatever it was.
 *
 * Supported: rows >= 1; Cin, Cout in [1, 8192]; rows*max(Cin, Cout) < 2^40.  No output may share a
 * byte with an input or another output, except where a call says so (FS_ERR_INVALID). */
typedef enum fs_act { FS_ACT_NONE = 0, FS_ACT_RELU = 1, FS_ACT_GELU = 2, FS_ACT_SILU = 3 } fs_act;

typedef struct fs_linear {
  int64_t rows;  /* >= 1 */
  int32_t Cin;   /* channels of x, 1..8192 */
  int32_t Cout;  /* channels of y, 1..8192 */
  int32_t dtype; /* fs_dtype of x, W, y */
} fs_linear;

/* ws: fs_linear_workspace_bytes(s, 0). */
fs_status fs_linear_fwd(const fs_linear* s, const void* x, const void* W, const float* bias, int act, float p,
                        const uint64_t* rng, const void* res, void* y, void* pre, void* ws, size_t ws_bytes,
                        fs_stream_t stream);

/* Gradients given g [rows, Cout], the gradient of u:
 *   dx = drop'(g W) act'(pre) + dres,   dW = g^T x,   dbias = sum_rows g
 *   act, p, rng, pre [rows, Cin]: those of the call that made x (y there), so that dx is the
 *   gradient of ITS u, ready for its own backward; FS_ACT_NONE, 0, NULL, NULL where x came from
 *   elsewhere.  drop' keeps what that call's dropout kept, times 1 / (1 - p).
 *   dres: NULL, or a gradient that reaches x along another way; may be dx itself.
 *   A layer's own residual takes the gradient of y as it is; where the call that made y had an
 *   activation or dropout, fs_dropout_bwd makes g from the gradient of y.
 *   dx: NULL to leave it out (W is then not read).  dW, dbias (fp32): NULL to leave them out
 *   (dbias only with dW), else written (accumulate == 0) or added to (accumulate != 0).
 * ws: fs_linear_workspace_bytes(s, 1). */
fs_status fs_linear_bwd(const fs_linear* s, const void* x, const void* W, const void* g, int act, float p,
                        const uint64_t* rng, const void* pre, const void* dres, void* dx, float* dW, float* dbias,
                        int accumulate, void* ws, size_t ws_bytes, fs_stream_t stream);

/* Bytes of scratch on the current device; 0 for an invalid or unsupported shape. */
size_t fs_linear_workspace_bytes(const fs_linear* s, int backward);

/* Kernel path of fs_linear_fwd, or of fs_linear_bwd's dx (backward != 0), for this shape: 0 = fp32
 * multiply-adds, 1 = tcgen05; -1 for an invalid or unsupported shape.  For tests and benchmarks. */
int fs_linear_path_for_shape(const fs_linear* s, int backward);

/* Dropout alone: y = res + drop(act(x)) over rows of C channels.  res: NULL for none; y may be x or
 * res. */
fs_status fs_dropout_fwd(const fs_rows* s, const void* x, int act, float p, const uint64_t* rng, const void* res, void* y,
                         fs_stream_t stream);
/* Its backward: dx = drop'(dy) act'(pre), pre what the activation saw (not read, and may be NULL, for
 * FS_ACT_NONE).  dx may be dy or pre. */
fs_status fs_dropout_bwd(const fs_rows* s, const void* dy, int act, float p, const uint64_t* rng, const void* pre,
                         void* dx, fs_stream_t stream);

/* Fixed-scratch variant of fs_slice_fwd.  The paper has no counterpart.
 *
 * For callers that cannot give the library device memory at the call site: a
 * program that lays out all of its device memory once at start-up and may not
 * allocate afterwards, or a caller (a plain C host, a foreign-language binding)
 * that holds no device allocator of its own.  Instead of a workspace argument,
 * this entry point uses one scratch buffer of FS_NOALLOC_SCRATCH_BYTES that is
 * part of the library's device code (a static device array), so neither the
 * caller nor the library allocates anything for the call.
 *   - Arguments, outputs and numerics are those of fs_slice_fwd (it runs the
 *     same kernels).  A shape whose fs_workspace_bytes(s, FS_OP_SLICE_FWD)
 *     exceeds FS_NOALLOC_SCRATCH_BYTES is rejected with
 *     FS_ERR_SCRATCH_TOO_SMALL before anything is launched; invalid or
 *     unsupported shapes give fs_slice_fwd's errors.
 *   - The first call on a device (with that device current) looks up the
 *     scratch's device address through the CUDA runtime; later calls on that
 *     device reuse it while the device's context stays the same.  After a
 *     cudaDeviceReset, or with another context current, the next call looks the
 *     address up again.  Make each call that does the lookup (the first one, and
 *     the first after a reset or context change) before any stream capture.
 *   - Each call clears the status word at the start of the scratch; nothing
 *     else in the scratch has to start at zero.
 *   - There is ONE scratch per device.  Calls that can overlap in time (on
 *     different streams, or from different host threads) race on it and
 *     corrupt each other's results: serialise them.
 *   - scratch: if not NULL, receives the scratch's device address, which
 *     fs_device_status accepts to read the call's device status. */
#define FS_NOALLOC_SCRATCH_BYTES ((size_t)16 << 20)
fs_status fs_slice_fwd_noalloc(const fs_shape* s, const void* x_mid, const void* fx,
                               const float* W_slice, const float* bias, const float* tau,
                               float* tokens, float* wsum, float* lse, int finalize,
                               const void** scratch, fs_stream_t stream);

/* Synchronises `stream` and returns the device status word of `ws`
 * (FS_OK, FS_ERR_TIMEOUT or FS_ERR_BAD_TAU), or FS_ERR_CUDA. */
fs_status fs_device_status(const void* ws, fs_stream_t stream);

/* Static, human-readable name of a status code. */
const char* fs_status_string(fs_status st);

/* Kernel path the library takes for this shape: 0 = SIMT fp32 kernels,
 * 1 = tcgen05 tensor-core kernels.  For tests and benchmarks. */
int fs_path_for_shape(const fs_shape* s);

/* Kernel path of the backward (fs_deslice_bwd, fs_slice_bwd) for this shape:
 * 0 = SIMT fp32 kernels, 1 = tcgen05 tensor-core kernels (bf16, d = 32,
 * N >= 2, any supported G, over slot ranges past G = 640; the weights with split
 * products whatever s->dot says).
 * For tests and benchmarks. */
int fs_backward_path_for_shape(const fs_shape* s);

/* Number of kernels the forward (slice + mix + deslice) launches for this shape. */
int fs_forward_launch_count(const fs_shape* s);

/* Number of kernels the backward (fs_deslice_bwd + fs_mix_bwd + fs_slice_bwd)
 * launches for this shape.  lse_given: nonzero when both backward calls get the
 * forward's lse (each call that must recompute the statistics launches that pass
 * again).  Memsets are not counted.  -1 for an invalid or unsupported shape. */
int fs_backward_launch_count(const fs_shape* s, int lse_given);

/* Number of kernels fs_coupling_bwd launches for this shape (lse_given as above;
 * the one call recomputes the statistics at most once).  -1 for an invalid or
 * unsupported shape. */
int fs_coupling_bwd_launch_count(const fs_shape* s, int lse_given);

#ifdef __cplusplus
}
#endif

#endif /* FLASHSLICE_H */
