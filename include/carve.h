/*
 * carve.h -- C ABI of libcarve: the chunked CARVE layer (arXiv 2606.27229)
 * forward and backward on AMD Instinct MI355X (gfx950).
 *
 * What the library computes (one layer, every batch element b and head h,
 * recurrent state S in R^{Dv x Dk}):
 *
 *   Sec. 4, Eq. carve_state (boxed): per token t
 *       S_t = S_{t-1} diag(exp g_t) diag(1 - b_t) + beta_t (w_t * v_t - S_{t-1} k_t) k_t^T
 *       o_t = S_t q_t
 *     with key-axis decay g_t (log domain, <= 0) and erase gate b_t, a
 *     per-token write strength beta_t, and a value-axis write gate w_t that
 *     scales v_t only (Alg. WYChunkDelta step 3).
 *   Sec. 4.2, Eq. content_readout / erase_gate: the gates of every token of
 *     chunk c (tokens [cL, (c+1)L)) read the state carried out of chunk c-1
 *     (S0 for chunk 0), folded once per chunk:
 *       F = [Ub; Uw] S_{c-1}           (2R x Dk)
 *       tau_b = tanh(F_b q_t), tau_w = tanh(F_w q_t)
 *       b_t = sigmoid(bx_t + Vb tau_b),  w_t = sigmoid(wx_t + Vw tau_w)
 *   Sec. 6.2, Alg. WYChunkDelta: evaluated chunk-parallel in WY form (one
 *     shared unit-lower-triangular solve per chunk, Thm. chunkability).
 *   App. Alg. backward / megakernel_bwd: the exact gradient of
 *       loss = <dO, o> + <dS_T, S_T>
 *     with respect to every input, including the chunk-boundary "glue"
 *     through the folded read-out and the parameter gradients reduced over
 *     batch, heads and chunks.
 *
 * Conventions
 *   - All tensors are dense, row-major and live in DEVICE memory owned by
 *     the caller.  Token tensors are [B, T, H, D] (q, k, bx, g: D = Dk;
 *     v, wx, o: D = Dv); beta is [B, T, H]; states are [B, H, Dv, Dk];
 *     S_chunks is [B, H, T/L, Dv, Dk] and holds the state at the start of
 *     every chunk; Ub, Uw are [R, Dv]; Vb is [Dk, R]; Vw is [Dv, R].
 *     Ub, Uw, Vb, Vw are shared by all heads.
 *   - dtype (CARVE_F32 or CARVE_BF16) is the element type of q, k, v, beta,
 *     bx, wx, o, dO and of dq, dk, dv, dbeta, dbx, dwx.  g, the parameters,
 *     the states and dg, dUb, dUw, dVb, dVw, dS0, dS_T are always f32.  All
 *     arithmetic is f32 (bf16 operands on the matrix cores in bf16 mode).
 *   - Every call is asynchronous on `stream` (a hipStream_t; NULL = the
 *     default stream) and never synchronises.  The return value reports
 *     argument validation and launch errors only.
 *   - Outputs are overwritten, never accumulated (parameter gradients too).
 *   - The library allocates no device memory and keeps no state between
 *     calls except the cached kernel attributes; concurrent calls on
 *     different streams must use different workspaces.
 *   - Supported shapes: Dk == Dv in {32, 64, 128}; 1 <= R <= 64;
 *     L in {16, 32, 64, 128}; T a positive multiple of L; B, H >= 1.
 *     Not built (their LDS layouts exceed 160 KB): the forward with f32
 *     token tensors at Dk = 128 and R > 32; the backward with f32 token
 *     tensors at Dk = 128, and with R > 32 at Dk = 128 (bf16) or Dk = 64
 *     (f32).  These, and other shapes, return CARVE_ERR_UNSUPPORTED
 *     (CARVE_ERR_SHAPE when T % L != 0 or a size is non-positive).
 *   - Every pointer must be 16-byte aligned (CARVE_ERR_ALIGN).
 *   - Inputs are assumed finite with g <= 0; NaN/Inf propagate.  Numerical
 *     range (log retention l = g - softplus(z_b) per key channel): the
 *     forward evaluates WY blocks of up to 64 tokens; a key channel whose
 *     sum of l over a block stays above -160 is taken relative to the middle
 *     of that block's range, any other channel relative to the middle of
 *     each 16-token tile's range, with the products across tiles formed from
 *     operands no larger than the raw token values.  The sum of l over every
 *     16-token tile must stay above about -150 (-170 where a block is a
 *     single tile).  The backward evaluates blocks of up to 64 tokens
 *     relative to the middle of their range, 16-token tile by tile where some
 *     channel sums below -80 over the block, with factors up to e^{|sum of l|
 *     / 2}, so each 16-token tile must sum above about -170.
 */
#ifndef CARVE_H
#define CARVE_H

#include <stddef.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { CARVE_F32 = 0, CARVE_BF16 = 1 } carve_dtype_t;

typedef struct {
  int B, T, H, Dk, Dv, R, L;
  carve_dtype_t dtype;
} carve_dims_t;

enum {
  CARVE_OK = 0,
  CARVE_ERR_NULL = -1,        /* a required pointer is NULL */
  CARVE_ERR_SHAPE = -2,       /* non-positive size or T % L != 0 */
  CARVE_ERR_UNSUPPORTED = -3, /* valid but not built: see "Supported shapes" */
  CARVE_ERR_ALIGN = -4,       /* a pointer is not 16-byte aligned */
  CARVE_ERR_WORKSPACE = -5,   /* workspace NULL or smaller than carve_workspace_size */
  CARVE_ERR_HIP = -6,         /* a HIP runtime call failed */
  CARVE_ERR_ARG = -7          /* conflicting or invalid argument values (g and f both given; eps) */
};

/* Bytes of device workspace the forward (for_backward = 0) or the backward
 * (for_backward = 1) needs for these dims; 0 means none.  Returns 0 for
 * dims that fail validation.  The workspace holds the per-chunk records of
 * the recompute (fold, tau, WY factors and block start states), the partial
 * parameter gradients and the chunk ready flags of the fused recompute +
 * adjoint launch (the same size for the gated backward). */
size_t carve_workspace_size(const carve_dims_t* d, int for_backward);

/* Forward (Alg. carve_fwd with the WY solve of Alg. WYChunkDelta).
 * In:  q, k [B,T,H,Dk]; v [B,T,H,Dv]; beta [B,T,H]; g [B,T,H,Dk] (f32);
 *      bx [B,T,H,Dk]; wx [B,T,H,Dv]; Ub, Uw, Vb, Vw (f32);
 *      S0 [B,H,Dv,Dk] f32 or NULL (= zeros).
 * Out: o [B,T,H,Dv]; S_T [B,H,Dv,Dk] or NULL; S_chunks [B,H,T/L,Dv,Dk] or
 *      NULL (needed by carve_chunk_bwd).
 * workspace may be NULL when carve_workspace_size(d, 0) == 0. */
int carve_chunk_fwd(const carve_dims_t* d, const void* q, const void* k, const void* v,
                    const void* beta, const float* g, const void* bx, const void* wx,
                    const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                    const float* S0, void* o, float* S_T, float* S_chunks, void* workspace,
                    size_t workspace_bytes, hipStream_t stream);

/* Backward of carve_chunk_fwd for loss <dO, o> + <dS_T, S_T>.
 * In:  the forward inputs; S_chunks as written by carve_chunk_fwd on the
 *      same inputs; dO [B,T,H,Dv]; dS_T [B,H,Dv,Dk] f32 or NULL (= zeros).
 * Out: dq, dk [B,T,H,Dk]; dv [B,T,H,Dv]; dbeta [B,T,H]; dg [B,T,H,Dk] f32;
 *      dbx [B,T,H,Dk]; dwx [B,T,H,Dv]; dUb, dUw [R,Dv]; dVb [Dk,R];
 *      dVw [Dv,R]; dS0 [B,H,Dv,Dk] or NULL.  (S0 itself is not needed: the
 *      chunk-start states are read from S_chunks.)
 * The parameter gradients are reduced over batch, heads and chunks in a
 * fixed order, so reruns are bitwise identical. */
int carve_chunk_bwd(const carve_dims_t* d, const void* q, const void* k, const void* v,
                    const void* beta, const float* g, const void* bx, const void* wx,
                    const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                    const float* S_chunks, const void* dO, const float* dS_T, void* dq, void* dk,
                    void* dv, void* dbeta, float* dg, void* dbx, void* dwx, float* dUb,
                    float* dUw, float* dVb, float* dVw, float* dS0, void* workspace,
                    size_t workspace_bytes, hipStream_t stream);

/* The same layer with the key-axis decay computed from its raw logit inside
 * the kernels (Sec. decay_gate, Eq. decay_gate: "gate-in-kernel" fusion):
 *     g[b,t,h,j] = -exp(A[h][j]) * softplus(f[b,t,h,j] + tau_f[h][j])
 * In:  f [B,T,H,Dk] in the call's dtype (the raw decay logit, replacing g);
 *      A, tau_f [H,Dk] f32: learned log-amplitudes and biases of the gate
 *      (tau_f is the bias the paper calls tau in Eq. decay_gate, not the
 *      content read-out tau of Eq. content_readout); the other arguments are
 *      those of carve_chunk_fwd.  g is never materialised.
 * The numerical-range precondition applies to the g so formed. */
int carve_chunk_fwd_gated(const carve_dims_t* d, const void* q, const void* k, const void* v,
                          const void* beta, const void* f, const float* A, const float* tau_f,
                          const void* bx, const void* wx, const float* Ub, const float* Uw,
                          const float* Vb, const float* Vw, const float* S0, void* o, float* S_T,
                          float* S_chunks, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Backward of carve_chunk_fwd_gated for loss <dO, o> + <dS_T, S_T>.  Outputs
 * as carve_chunk_bwd, with dg replaced by:
 *   df [B,T,H,Dk] in the call's dtype: dL/df = dL/dg * (-exp(A)) * sigmoid(f + tau_f);
 *   dA, dtau [H,Dk] f32: sums over batch and tokens of dL/dg * g and of dL/df,
 *   reduced in a fixed order (bitwise-reproducible reruns).
 * The workspace is the one carve_workspace_size(d, 1) reports. */
int carve_chunk_bwd_gated(const carve_dims_t* d, const void* q, const void* k, const void* v,
                          const void* beta, const void* f, const float* A, const float* tau_f,
                          const void* bx, const void* wx, const float* Ub, const float* Uw,
                          const float* Vb, const float* Vw, const float* S_chunks, const void* dO,
                          const float* dS_T, void* dq, void* dk, void* dv, void* dbeta, void* df,
                          float* dA, float* dtau, void* dbx, void* dwx, float* dUb, float* dUw,
                          float* dVb, float* dVw, float* dS0, void* workspace, size_t workspace_bytes,
                          hipStream_t stream);

/* The layer with the scalar write gate (Sec. scalar write gate, the deployment
 * variant of the ablation rows "scalar write" of Table attribution): one write
 * logit per token and head, broadcast over the value channels, and no content
 * term on the write side:
 *     w_t = sigmoid(wx[b,t,h]) on every one of the Dv channels,
 *     b_t = sigmoid(bx_t + Vb tanh(F_b q_t)) with F_b = Ub S_{c-1} (as before).
 * The fold has R rows instead of 2R; there is no Uw, Vw.
 * In:  wx [B,T,H] in the call's dtype (replacing the [B,T,H,Dv] logits);
 *      the decay either as g [B,T,H,Dk] f32 (f = A = tau_f = NULL) or from its
 *      raw logit as in carve_chunk_fwd_gated (g = NULL; f, A, tau_f given);
 *      the other arguments are those of carve_chunk_fwd.
 * Returns CARVE_ERR_NULL when neither g nor f is given, CARVE_ERR_ARG when
 * both are.  Ub = 0 gives the ablation's row with no content at all. */
int carve_chunk_fwd_sw(const carve_dims_t* d, const void* q, const void* k, const void* v,
                       const void* beta, const float* g, const void* f, const float* A,
                       const float* tau_f, const void* bx, const void* wx, const float* Ub,
                       const float* Vb, const float* S0, void* o, float* S_T, float* S_chunks,
                       void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Backward of carve_chunk_fwd_sw for loss <dO, o> + <dS_T, S_T>.  Outputs as
 * carve_chunk_bwd (dg with the g form; df, dA, dtau as carve_chunk_bwd_gated
 * with the f form; the other decay outputs may be NULL), except:
 *   dwx [B,T,H] in the call's dtype: the sum over the value channels of the
 *   per-channel write-logit gradient, dL/dwx_t = sum_v dL/dw_tv * w_t (1 - w_t);
 *   no dUw, dVw.
 * The workspace is the one carve_workspace_size(d, 1) reports; the launch
 * sequence (and the measurement hook's events) is that of the matching
 * carve_chunk_bwd or carve_chunk_bwd_gated call. */
int carve_chunk_bwd_sw(const carve_dims_t* d, const void* q, const void* k, const void* v,
                       const void* beta, const float* g, const void* f, const float* A,
                       const float* tau_f, const void* bx, const void* wx, const float* Ub,
                       const float* Vb, const float* S_chunks, const void* dO, const float* dS_T,
                       void* dq, void* dk, void* dv, void* dbeta, float* dg, void* df, float* dA,
                       float* dtau, void* dbx, void* dwx, float* dUb, float* dVb, float* dS0,
                       void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The layer with its input activations inside the kernels (Sec. input
 * projections, Fig. carve_block, the chunk-local normalisation of
 * Alg. megakernel fused into the chunk loads):
 *     q = SiLU(q_raw) / sqrt(|SiLU(q_raw)|^2 + 1e-6)   per (token, head) over Dk,
 *     k likewise from k_raw, v = SiLU(v_raw).
 * In:  q, k, v are the raw projections q_raw, k_raw, v_raw (same shapes and
 *      dtype as in carve_chunk_fwd); every other argument is that of
 *      carve_chunk_fwd.  The activated q, k, v are never written to memory. */
int carve_chunk_fwd_act(const carve_dims_t* d, const void* q, const void* k, const void* v,
                        const void* beta, const float* g, const void* bx, const void* wx,
                        const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                        const float* S0, void* o, float* S_T, float* S_chunks, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* Backward of carve_chunk_fwd_act for loss <dO, o> + <dS_T, S_T>.  Outputs as
 * carve_chunk_bwd, with dq, dk, dv the gradients with respect to q_raw, k_raw,
 * v_raw.  The backward makes one more launch than carve_chunk_bwd (the last:
 * dq, dk taken through the L2 normalisation and SiLU in place). */
int carve_chunk_bwd_act(const carve_dims_t* d, const void* q, const void* k, const void* v,
                        const void* beta, const float* g, const void* bx, const void* wx,
                        const float* Ub, const float* Uw, const float* Vb, const float* Vw,
                        const float* S_chunks, const void* dO, const float* dS_T, void* dq, void* dk,
                        void* dv, void* dbeta, float* dg, void* dbx, void* dwx, float* dUb,
                        float* dUw, float* dVb, float* dVw, float* dS0, void* workspace,
                        size_t workspace_bytes, hipStream_t stream);

/* Output RMS normalisation, the step that closes Alg. carve_fwd:
 *     y = W_O RMSNorm(reshape(o)),
 * without W_O (a plain GEMM outside the recurrence).  Alg. megakernel runs it
 * as one hoisted launch over the assembled o, and Alg. megakernel_bwd mirrors
 * it with one hoisted launch of its gradient; these entry points are those
 * launches.  A token's row is reshape(o)[b, t, :], the N = H * Dv values of
 * all its heads ([B, T, H, Dv] row-major viewed as [B*T, N]):
 *     y[row, i] = o[row, i] / sqrt(mean_i o[row, i]^2 + eps) * weight[i]
 * The paper gives no eps; the Python binding passes 1e-6.
 * Only B, T, H, Dv and dtype of d are read (Dk, R and L are not; T need not be
 * a multiple of L).  Supported: N a multiple of 8 (bf16) or 4 (f32) with
 * N <= 4096 (bf16) or 2048 (f32), else CARVE_ERR_UNSUPPORTED; eps finite and
 * >= 0, else CARVE_ERR_ARG.  A row of zeros with eps = 0 gives NaN.
 * In:  o [B,T,H,Dv] in the call's dtype (as written by carve_chunk_fwd);
 *      weight [H*Dv] f32.
 * Out: y [B,T,H,Dv] in the call's dtype (must not overlap o or weight).
 * One launch; asynchronous on stream. */
int carve_rmsnorm_fwd(const carve_dims_t* d, const void* o, const float* weight, float eps, void* y,
                      hipStream_t stream);

/* Bytes of device workspace carve_rmsnorm_bwd needs for these dims (one f32
 * partial row of dweight per workgroup of its first launch, at most 1024);
 * 0 for dims that fail validation. */
size_t carve_rmsnorm_workspace_size(const carve_dims_t* d);

/* Backward of carve_rmsnorm_fwd for loss <dy, y>:
 *     r = 1 / sqrt(mean_i o_i^2 + eps),  n = o r,  dn = dy * weight,
 *     d_o = r (dn - n mean_i(dn_i n_i)),  dweight = sum over rows of dy * n.
 * In:  o, weight, eps as given to the forward; dy [B,T,H,Dv] in the call's dtype.
 * Out: d_o [B,T,H,Dv] in the call's dtype; dweight [H*Dv] f32 (overwritten,
 *      reduced over the rows in a fixed order: reruns are bitwise identical).
 * workspace: at least carve_rmsnorm_workspace_size(d) bytes, else
 * CARVE_ERR_WORKSPACE.  Two launches (the rows, then the fixed-order sum of
 * the workgroups' dweight partials); no output may overlap an input or the
 * workspace. */
int carve_rmsnorm_bwd(const carve_dims_t* d, const void* o, const float* weight, float eps, const void* dy,
                      void* d_o, float* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* carve_rmsnorm_bwd without a workspace argument, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  It allocates nothing: the dweight
 * partials go to a static device array of the library, 16 MiB (1024 partial
 * rows of up to 4096 floats), which every supported shape fits; each GPU the
 * library runs on holds its own copy until the process ends.  Its device
 * address is looked up once per device, on the first call made with that
 * device current (CARVE_ERR_HIP if the lookup fails).  Arguments, outputs and
 * errors are those of carve_rmsnorm_bwd; the results are bitwise those of
 * carve_rmsnorm_bwd.  Every call on one GPU shares that GPU's array: calls
 * that overlap in time on one GPU (different streams, or different threads
 * without ordering) race on it and must not be made. */
int carve_rmsnorm_bwd_noalloc(const carve_dims_t* d, const void* o, const float* weight, float eps,
                              const void* dy, void* d_o, float* dweight, hipStream_t stream);

/* ---- the gated delta rule (scalar decay) ------------------------------------
 *
 * The scalar-gated delta rule that the CARVE layer is compared with, per
 * sequence and value head (key head hv / (Hv / Hk); S in R^{Dv x Dk}, f32):
 *     S~ = exp(g_t) S_{t-1},  u_t = beta_t (v_t - S~ k_t),
 *     S_t = S~ + u_t k_t^T,   o_t = scale S_t q_t
 * with one log decay g_t <= 0 and one write strength beta_t per token and
 * value head, and the decay before the prediction.  carve_gdr_chunk_fwd and
 * carve_gdr_chunk_bwd evaluate it in chunks of 64 tokens (any T; no padding),
 * carve_gdr_step token by token on a pool of states.
 *
 *   - q, k are [B, T, Hk, Dk] and v is [B, T, Hv, Dv] with the strides of
 *     carve_gdr_dims_t (in elements; the last dimension is contiguous), so that
 *     they may be slices of a fused projection.  beta [B, T, Hv] (token dtype),
 *     g [B, T, Hv] (f32), o and dO [B, T, Hv, Dv] and every gradient are dense.
 *     The strides may not be negative; a stride of 0 is a broadcast input, whose
 *     gradient is still written per element.  A token's stride is less than 16 MB.
 *   - Packed sequences: with N > 0, B must be 1 and the T rows hold N sequences,
 *     sequence n being rows [offsets[n], offsets[n + 1]); offsets is a device
 *     array of N + 1 ints, non-decreasing from >= 0 to <= T.  Sequences may be
 *     empty or of one token.  Rows of o and of the gradients that belong to no
 *     sequence are left as they were.  Offsets are not read on the host: values
 *     outside this contract stay within the tensors, with unspecified results.
 *     With N = 0, offsets must be NULL and every batch element is a sequence.
 *   - S0, S_T, dS_T, dS0: [sequences, Hv, Dv, Dk] f32.  The state of an empty
 *     sequence passes through.  S_chunks: [carve_gdr_chunk_count(d), Hv, Dv, Dk]
 *     f32, the state at the start of every chunk, written by carve_gdr_chunk_fwd for
 *     carve_gdr_chunk_bwd (slots of no chunk are left as they were).
 *   - Supported: Dk in {32, 64, 128}; Dv in {32, 64, 128, 256}; Hv a multiple of
 *     Hk, at most 65535; dtype f32 or bf16.  In the chunk form sequences * Hv *
 *     Dv / 32 (sequences * Hv rounded up to eights) and the chunk count are less
 *     than 2^23 each.  scale is finite.  q, k, v and their
 *     strides are 16-byte aligned, like every other pointer.
 *   - Inputs are finite with g <= 0; g = -inf is a reset (decay 0).  NaN and
 *     infinities propagate within their sequence, also to tokens before them in
 *     the same chunk.  With bf16 tokens the chunk form carries f32 intermediates
 *     through the matrix cores as sums of bf16 values, three towards f32 outputs
 *     (states, dg: f32 accuracy) and two towards bf16 outputs; with f32 tokens
 *     all products are f32.
 *   - No output may overlap an input, another output or the workspace
 *     (CARVE_ERR_UNSUPPORTED): S_T is not written over S0.  Only the pool of
 *     carve_gdr_step is updated in place.
 */
typedef struct {
  int B, T;            /* dense: B sequences of T tokens; packed: B = 1, T rows */
  int N;               /* packed: number of sequences; dense: 0 */
  int Hk, Hv, Dk, Dv;
  carve_dtype_t dtype;
  float scale;
  long long q_batch, q_token, q_head;   /* strides in elements */
  long long k_batch, k_token, k_head;
  long long v_batch, v_token, v_head;
} carve_gdr_dims_t;

/* Chunks that S_chunks has room for (the same as a program needs to allocate;
 * dense: B ceil(T / 64); packed: floor(T / 64) + N); 0 for invalid dims. */
size_t carve_gdr_chunk_count(const carve_gdr_dims_t* d);

/* Bytes of device workspace of carve_gdr_chunk_fwd (for_backward = 0) and
 * carve_gdr_chunk_bwd (1); 0 for invalid dims.  Nothing in it is kept between calls;
 * calls that overlap in time need workspaces of their own, and so do captured
 * graphs that may run at once. */
size_t carve_gdr_workspace_size(const carve_gdr_dims_t* d, int for_backward);

/* Forward.  S0, S_T, S_chunks may be NULL (zeros; not wanted).  Two launches.
 * The strides of q, k, v are those of d. */
int carve_gdr_chunk_fwd(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                        const void* beta, const float* S0, const int* offsets, void* o, float* S_T,
                        float* S_chunks, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Backward for loss <dO, o> + <dS_T, S_T>.  In: the forward's inputs (S0 only
 * through S_chunks), S_chunks as carve_gdr_chunk_fwd wrote it, dO, dS_T or NULL (zeros).
 * Out: dq, dk [B,T,Hk,Dk], dv [B,T,Hv,Dv], dbeta [B,T,Hv] (token dtype), dg
 * [B,T,Hv] f32, dS0 or NULL.  dq and dk are summed over the value heads of their
 * key head in order: reruns are bitwise identical.  Three launches. */
int carve_gdr_chunk_bwd(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                        const void* beta, const float* S_chunks, const int* offsets, const void* dO,
                        const float* dS_T, void* dq, void* dk, void* dv, float* dg, void* dbeta, float* dS0,
                        void* workspace, size_t workspace_bytes, hipStream_t stream);

/* T tokens for each of B sequences (d->N = 0), token by token in f32: state is a
 * pool of `pool` states [pool, Hv, Dv, Dk] f32, updated in place; sequence b's
 * state is state[slots[b]] (slots: [B] device ints), or state[b] with slots NULL
 * (then pool >= B).  The state left is that behind the last of the T tokens.  A sequence whose slot is outside [0, pool) is a padding
 * entry: its state and its rows of o are left as they were.  Two sequences of one
 * call may not have the same slot (their results are then unspecified).  B is at
 * most 65535.  One launch, no workspace. */
int carve_gdr_step(const carve_gdr_dims_t* d, const void* q, const void* k, const void* v, const float* g,
                   const void* beta, const int* slots, int pool, float* state, void* o, hipStream_t stream);

/* ---- the norms around a block, with its gate and residual scale ---------------
 *
 * Rows of N values, statistics and parameters in f32 (see also carve_rmsnorm_fwd,
 * the plain norm of the layer's output):
 *     n = y / sqrt(mean(y^2 over its group) + eps) * weight
 *     t = n * act(gate)                    (gate given; act: SiLU or sigmoid)
 *     x = alpha * residual + scale * t     (residual, scale given)
 *     h = x / sqrt(mean(x^2) + eps) * next_weight       (next_weight given)
 * y is a block's output; n its norm over `groups` equal groups of a row (1: the
 * row; H: per head, with N = H Dv); x the residual stream; h the next block's
 * input.  One pass: h is formed from x before x is rounded to its dtype.
 * Rows of any finite size are normalised, also where their squares leave the
 * range of f32 (and, with eps = 0, small ones): they are summed in another unit.
 * weight, scale, next_weight: [N] f32.  y, gate, residual have row strides (in
 * elements, >= 0, 16-byte aligned), every other tensor is dense.
 * Supported: N a multiple of 8 (bf16) or 4 (f32), at most 8192; with groups > 1,
 * N / groups must be 16 bytes times a power of two up to 64; eps finite and >= 0,
 * alpha finite.  No output may overlap an input, another output or the workspace
 * (CARVE_ERR_UNSUPPORTED): x is not written over residual. */
enum { CARVE_GATE_SILU = 1, CARVE_GATE_SIGMOID = 2 };
typedef struct {
  long long rows;
  int N, groups;
  carve_dtype_t dtype;
  int gate_act;        /* CARVE_GATE_*, read where gate is given */
  float eps, alpha;    /* alpha is read where residual is given */
  long long y_stride, gate_stride, residual_stride;
} carve_block_norm_dims_t;

/* gate, residual, scale may be NULL (left out); next_weight and h are both given
 * or both NULL.  One launch. */
int carve_block_norm_fwd(const carve_block_norm_dims_t* d, const void* y, const float* weight, const void* gate,
                         const void* residual, const float* scale, const float* next_weight, void* x, void* h,
                         hipStream_t stream);

/* Bytes of device workspace of carve_block_norm_bwd; 0 for invalid dims. */
size_t carve_block_norm_workspace_size(const carve_block_norm_dims_t* d);

/* Backward for loss <dx, x> + <dh, h>: in the forward's inputs (x is formed again,
 * unrounded) and dx, dh (dx may be NULL, zeros, where dh is given; dh is given
 * exactly where next_weight is).  Out: dy, dgate and dresidual (exactly where gate
 * and residual are given) in the token dtype; dweight, dscale, dnext_weight [N]
 * f32 (exactly where their inputs are given), summed over the rows in a fixed
 * order (reruns are bitwise identical).  Two launches. */
int carve_block_norm_bwd(const carve_block_norm_dims_t* d, const void* y, const float* weight, const void* gate,
                         const void* residual, const float* scale, const float* next_weight, const void* dx,
                         const void* dh, void* dy, void* dgate, void* dresidual, float* dweight, float* dscale,
                         float* dnext_weight, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Measurement hook (not part of the computation).  Arms the next
 * carve_chunk_*, carve_rmsnorm_*, carve_gdr_* or carve_block_norm_* call made
 * on the calling thread to record events[0] on its stream before its first kernel launch and events[i] after
 * its i-th launch (the forward makes 1 launch; the backward 4: clear of the
 * chunk ready flags, chunk recompute fused with the adjoint, the partials of
 * d[Ub;Uw] and dVb/dVw, their fixed-order reductions; the gated backward
 * a 5th, the reduction of dA, dtau over the batch; the backward with the
 * input activations a 5th, the activation gradient of dq, dk; the norm's
 * forward 1, its backward 2; the gated delta rule's forward 2, chunk triangles
 * and chain, its backward 3, triangles, chain and gradients, its step 1; the
 * block norm's forward 1, its backward 2),
 * up to `capacity` events.  `events` are hipEvent_t handles created by the
 * caller (hipEventCreate) and owned by the caller; the handles are copied
 * here (the array may be freed after this call) and the events are only
 * recorded, never synchronised.  The hook covers exactly one call and is
 * cleared when that call returns, whatever its status; capacity 0 disarms
 * it.  Returns CARVE_ERR_NULL for a NULL array with capacity > 0 or a
 * negative capacity, CARVE_ERR_UNSUPPORTED for capacity > 16. */
int carve_profile_events(hipEvent_t* events, int capacity);

/* Diagnostic of the backward's wait for the chunk records (not part of the
 * computation).  In carve_chunk_bwd and its variants, each adjoint wave waits
 * for the records of the next chunks with a bounded poll of their ready flags
 * (by default 2^20 polls, about a second; a correct launch never reaches it,
 * since a chunk is recomputed in tens of microseconds by a workgroup that is
 * already running and whose own wait is shorter and made once).  If the bound
 * runs out, the wave fills its state gradient
 * with NaN, so the gradients of all earlier tokens come out NaN, waits no
 * more, and sets a timeout word in the workspace's synchronisation area.  The
 * call itself still returns CARVE_OK, as kernel completion is asynchronous.
 * This reads that word for the last backward enqueued with `workspace` and
 * the same dims `d`: *timed_out = 1 if a wait ran out, 0 otherwise.  The word
 * is cleared at the start of every backward.  It copies 4 bytes to the host on
 * `stream` and synchronises `stream`: the only call of this library that
 * synchronises.  Errors: CARVE_ERR_NULL for a NULL argument;
 * CARVE_ERR_SHAPE / CARVE_ERR_UNSUPPORTED for dims no backward accepts;
 * CARVE_ERR_HIP if the copy fails. */
int carve_bwd_wait_status(const carve_dims_t* d, const void* workspace, hipStream_t stream, int* timed_out);

/* Test hook for the timeout path above: sets the bound of that wait, in polls,
 * for the backward calls made on the calling thread from then on.  0 makes
 * every wait give up at once (the kernels still run to completion and the
 * results are NaN); a negative value restores the default.  Returns the
 * previous bound.  Not for production use. */
int carve_set_ready_wait_limit(int polls);

/* Static description of a status code. */
const char* carve_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* CARVE_H */
