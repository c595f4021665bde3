/*
 * scd.h -- C ABI of the SCD KV-state codec on MI355X (gfx950).
 *
 * Semantic Cache Distillation moves a consumer model's prefix KV cache as compact codes:
 * the producer encodes each Reuse layer's de-RoPE'd keys and its values onto low-rank bases and
 * each Patch layer's normalised attention input onto a code (Section 4.3.2, Eq. encode_z_kv;
 * Section 4.4.1); the consumer decodes Reuse layers as code x basis (+ offset) and re-applies
 * RoPE to keys (Eq. decode_kv), and regenerates Patch layers' KV by pushing the predicted
 * normalised input through its own W_K / W_V with RoPE on keys (Section 4.4.2,
 * Eq. kv_from_patch).  Algorithm 1 ("Split Inference with Reuse and Patch") fixes the order
 * and the routing.  Every entry point below computes one of those steps on the GPU.
 *
 * Conventions shared by every entry point
 * ----------------------------------------
 *  - All tensors are dense, row-major and contiguous, in the model's dtype (scd_dtype_t):
 *    fp32, or bf16 with fp32 accumulation and a single round-to-nearest-even at the store.
 *  - Matrices use the [out, in] layout of a linear layer's weight, so every map is y = x W^T
 *    (the paper writes x W with W of shape [in, out]; the maps are the same).
 *  - The KV cache of one layer and branch is [T, H, d_h] (token-major, heads contiguous inside a
 *    token), T = total packed tokens of the batch.  The consumer owns it; the library writes each
 *    slot of a routed layer exactly once and never touches other layers.
 *  - A basis of width w acts on rows of w consecutive channels: one token of D = H*d_h channels
 *    is g = D / w code rows (w = D: one row per token; w = d_h: the head-shared basis, where
 *    batch x heads x tokens form one sample axis, Section 4.1).  Codes are [T*g, r].
 *  - Per-layer tensors are passed as HOST arrays of length n_layers holding DEVICE pointers.
 *    Entries of layers the call does not route are ignored and may be NULL.  When the batch has
 *    no tokens every call is a no-op, and buffers sized by the token count may be NULL.
 *  - RoPE pairs channel i of a head with channel i + d_h/2 and rotates the pair by
 *    p * theta^(-2i/d_h), p the token's position in its own request (Section 4.1 names RoPE and
 *    deRoPE as forward and inverse; Appendix F.2 keeps the framework's own cache positions).
 *  - Device pointers must be 16-byte aligned.  Calls are asynchronous on the given stream, never
 *    synchronise, and allocate nothing: the caller owns every buffer.
 *  - Every argument is validated before any launch.  A non-OK status means nothing was launched
 *    and no output was written; scd_last_error() then describes the problem.  Device-side
 *    contents (cu_seqlens, pos0) are not validated: they must be non-decreasing with
 *    cu_seqlens[0] = 0 and cu_seqlens[B] = n_tokens; positions at or beyond the RoPE table's
 *    max_position give unspecified values (never an out-of-bounds access).
 */
#ifndef SCD_H_
#define SCD_H_

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SCD_OK = 0,
  SCD_ERR_NULL = 1,         /* a required pointer is NULL */
  SCD_ERR_SHAPE = 2,        /* inconsistent or out-of-range sizes */
  SCD_ERR_SCHEDULE = 3,     /* bad layer routing or ranks */
  SCD_ERR_ALIGN = 4,        /* a device pointer is not 16-byte aligned */
  SCD_ERR_UNSUPPORTED = 5,  /* valid per the paper but outside what the kernels implement */
  SCD_ERR_WORKSPACE = 6,    /* RoPE table missing or too small */
  SCD_ERR_HIP = 7           /* a HIP runtime call or kernel launch failed */
} scd_status_t;

typedef enum { SCD_F32 = 0, SCD_BF16 = 1 } scd_dtype_t;

/* Model pair description (host memory, read only during the call).
 * Section 4.1: layers 0..L-1 (0-based here); L_patch = {l : is_patch[l] != 0}, L_reuse its
 * complement; independent branch ranks r_K, r_V, r_H.
 * Supported by the kernels: head_dim 32, 64 or 128; basis_width a multiple of head_dim that
 * divides D; every rank routed by a call a multiple of 16 with
 * 16 <= rank_k, rank_v <= min(basis_width, 256) and 16 <= rank_h <= min(d_model, 256);
 * d_model a multiple of 32. */
typedef struct {
  int32_t n_layers;
  int32_t d_model;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t basis_width;     /* w */
  int32_t dtype;           /* scd_dtype_t: dtype of every tensor argument */
  double rope_theta;
  const uint8_t* is_patch; /* [n_layers] */
  const int32_t* rank_k;   /* [n_layers] */
  const int32_t* rank_v;   /* [n_layers] */
  const int32_t* rank_h;   /* [n_layers] */
} scd_model_t;

/* A packed batch of B requests, T tokens in total (request b owns tokens
 * [cu_seqlens[b], cu_seqlens[b+1])).  Positions restart at pos0[b] (0 when pos0 is NULL) for
 * every request. */
typedef struct {
  int32_t n_seqs;              /* B >= 1 */
  int64_t n_tokens;            /* T >= 0 */
  const int32_t* cu_seqlens;   /* DEVICE [B+1], or NULL when B == 1 (one request of T tokens) */
  const int32_t* pos0;         /* DEVICE [B], or NULL */
} scd_batch_t;

/* ---- RoPE table ------------------------------------------------------------------------------
 * Opaque device table of rotation cosines and sines for positions [0, max_position), evaluated in
 * fp64 and rounded once to fp32 (fp32-evaluated angles lose ~1e-5 absolute accuracy by position
 * 512 and ~2e-3 by 32K).  It depends only on (head_dim, rope_theta, max_position): build it once
 * per model and reuse it.  scd_rope_table_bytes returns its size; scd_rope_table fills it.  The
 * entry points that take a table trust the (table, max_position) pair they are given: it must be a
 * table this model's head_dim and rope_theta built for that max_position, holding
 * scd_rope_table_bytes(model, max_position) bytes (the C calls cannot see its size; the Python
 * binding records head_dim, theta and max_position with the table and checks them). */
size_t scd_rope_table_bytes(const scd_model_t* model, int64_t max_position);
scd_status_t scd_rope_table(const scd_model_t* model, int64_t max_position, void* table,
                            size_t table_bytes, hipStream_t stream);

/* ---- a1: token positions ---------------------------------------------------------------------
 * pos_out[t] = t - cu_seqlens[b] + pos0[b] for every packed token t (DEVICE int32 [n_tokens]).
 * The same mapping every RoPE/deRoPE step below uses internally. */
scd_status_t scd_positions(const scd_batch_t* batch, int32_t* pos_out, hipStream_t stream);

/* ---- a0: routing and payload (host only) -------------------------------------------------------
 * scd_schedule writes the Reuse and Patch layer lists in increasing order (Section 4.5: the sets
 * are fixed inputs, membership is a constant-time lookup).  Output arrays hold n_layers entries.
 * scd_payload_bytes returns the bytes of the transmitted code set of Algorithm 1
 * ({Z_K, Z_V} per Reuse layer, Z_H per Patch layer; O(T r), Section 4.5) for n_tokens tokens and,
 * when offsets is not NULL, fills offsets[0..n_layers] with each layer's start in one packed buffer
 * (layer order, K codes before V codes).  Returns 0 on invalid input. */
scd_status_t scd_schedule(const scd_model_t* model, int32_t* reuse_layers, int32_t* n_reuse,
                          int32_t* patch_layers, int32_t* n_patch);
size_t scd_payload_bytes(const scd_model_t* model, int64_t n_tokens, int64_t* offsets);

/* ---- a2-a4: producer encode (Section 4.3.2, Eq. encode_z_kv; Section 4.4.1; Algorithm 1) ----
 * For every Reuse layer l:
 *   z_k[l] = (rows(deRoPE(k_in[l])) - mu_k[l]) w_enc_k[l]^T      [T*g, rank_k[l]]
 *   z_v[l] = (rows(v_in[l]) - mu_v[l]) w_enc_v[l]^T              [T*g, rank_v[l]]
 * with k_in, v_in [T, H, d_h], w_enc_k [rank_k, w], w_enc_v [rank_v, w], mu [w] (the optional
 * producer-side offset; NULL array or NULL entry = 0, which is the paper's equation).
 * For every Patch layer l:  z_h[l] = h_in[l] w_enc_h[l]^T  with h_in [T, d_model] (the producer's
 * normalised attention input) and w_enc_h [rank_h, d_model]; z_h [T, rank_h].
 * bf16 keys: the de-rotated input is rounded to bf16 once before the product; the offset enters as
 * the fp32 term mu w_enc^T subtracted from the accumulator, so it is never rounded. */
scd_status_t scd_encode(const scd_model_t* model, const scd_batch_t* batch,
                        const void* rope_table, int64_t max_position,
                        const void* const* k_in, const void* const* v_in,
                        const void* const* h_in,
                        const void* const* w_enc_k, const void* const* w_enc_v,
                        const void* const* w_enc_h,
                        const void* const* mu_k, const void* const* mu_v,
                        void* const* z_k, void* const* z_v, void* const* z_h,
                        hipStream_t stream);

/* ---- a5-a6, a8: consumer Reuse decode (Section 4.3.2, Eq. decode_kv; Algorithm 1) ------------
 * For every Reuse layer l, written straight into the consumer's cache:
 *   k_cache[l] = RoPE(unrows(z_k[l] w_dec_k[l]^T + mu_k[l]))     [T, H, d_h]
 *   v_cache[l] = unrows(z_v[l] w_dec_v[l]^T + mu_v[l])           [T, H, d_h]
 * with z [T*g, rank], w_dec [w, rank] and mu [w] the optional consumer-side offset (NULL = 0).
 * The paper writes one W_dec,B for both branches; keys and values are fitted independently
 * (Section 4.3.1), so each branch takes its own decoder.  Patch layers are not touched. */
scd_status_t scd_reuse_decode(const scd_model_t* model, const scd_batch_t* batch,
                              const void* rope_table, int64_t max_position,
                              const void* const* z_k, const void* const* z_v,
                              const void* const* w_dec_k, const void* const* w_dec_v,
                              const void* const* mu_k, const void* const* mu_v,
                              void* const* k_cache, void* const* v_cache, hipStream_t stream);

/* ---- a7, a8: consumer Patch (Section 4.4.2, Eq. kv_from_patch; Appendix F.2; Algorithm 1) ----
 * For every Patch layer l, written straight into the consumer's cache:
 *   k_cache[l] = RoPE(h_hat[l] w_k[l]^T + b_k[l]),   v_cache[l] = h_hat[l] w_v[l]^T + b_v[l]
 * with h_hat [T, d_model] the predicted normalised attention input (the aligner's output; this
 * call does not normalise), w_k, w_v [D, d_model] the consumer's own key/value projection weights
 * and b_k, b_v [D] optional projection biases (NULL array or NULL entry = none, as in the paper).
 * Reuse layers are not touched. */
scd_status_t scd_patch_kv(const scd_model_t* model, const scd_batch_t* batch,
                          const void* rope_table, int64_t max_position,
                          const void* const* h_hat,
                          const void* const* w_k, const void* const* w_v,
                          const void* const* b_k, const void* const* b_v,
                          void* const* k_cache, void* const* v_cache, hipStream_t stream);

/* ---- Patch aligner (Section 4.4.2, Eq. aligner) --------------------------------------------------
 * The consumer's aligner g_theta maps each Patch layer's code to a predicted normalised attention
 * input, the input of scd_patch_kv:
 *   act[l]   = SiLU(z_h[l] w1[l]^T + b1[l])           [T, hidden]
 *   h_hat[l] = act[l] w2[l]^T + b2[l]                 [T, d_model]
 * with z_h [T, rank_h[l]] (the transmitted code), w1 [hidden, rank_h[l]], w2 [d_model, hidden]
 * (nn.Linear layout), b1 [hidden] and b2 [d_model] optional (NULL array or entry = none) and
 * SiLU(x) = x / (1 + e^-x), evaluated in fp32 before the one rounding of each product.  The paper
 * calls g_theta an MLP and fixes neither its depth, width nor activation: this is a two-layer MLP
 * of width `hidden` (16 <= hidden, hidden % 16 == 0) with the backbone's SiLU.  act[l] holds layer
 * l's hidden activations: caller-owned, one buffer per Patch layer, distinct (the call writes them
 * all before it reads them); an act buffer that repeats returns SCD_ERR_SHAPE.  Reuse layers are
 * not touched. */
scd_status_t scd_patch_align(const scd_model_t* model, const scd_batch_t* batch, int32_t hidden,
                             const void* const* z_h,
                             const void* const* w1, const void* const* b1,
                             const void* const* w2, const void* const* b2,
                             void* const* act, void* const* h_hat, hipStream_t stream);

/* ---- Patch from the codes, with the aligner's output layer folded (Section 4.4.2) -------------
 * Eq. aligner ends in an affine layer (h_hat = act w2^T + b2) and Eq. kv_from_patch applies the
 * consumer's projections to h_hat with no nonlinearity in between, so for P = K, V:
 *   h_hat w_p^T + b_p = act (w_p w2)^T + (w_p b2 + b_p).
 * scd_patch_fold forms, once per model pair, for every Patch layer l:
 *   w_fold_k[l] = w_k[l] w2[l]   [D, hidden],    c_k[l] = w_k[l] b2[l] + b_k[l]   [D]
 *   w_fold_v[l] = w_v[l] w2[l]   [D, hidden],    c_v[l] = w_v[l] b2[l] + b_v[l]   [D]
 * with w2 [d_model, hidden] and b2 [d_model] the aligner's output layer (scd_patch_align's), w_k,
 * w_v [D, d_model] and b_k, b_v [D] the consumer's projections (b2, b_k, b_v optional: NULL array
 * or entry = 0), accumulated in fp32 and rounded once to the model's dtype.  Every output buffer
 * is written whole; outputs must not repeat across layers or branches (SCD_ERR_SHAPE) nor overlap
 * the inputs.  hidden % 16 == 0.  The batch plays no part.
 *
 * scd_patch_kv_from_codes is the consumer's Patch from the transmitted codes (Algorithm 1): for
 * every Patch layer l, in layer order,
 *   act[l]     = SiLU(z_h[l] w1[l]^T + b1[l])                 [T, hidden]
 *   k_cache[l] = RoPE(act[l] w_fold_k[l]^T + c_k[l]),   v_cache[l] = act[l] w_fold_v[l]^T + c_v[l]
 * which equals scd_patch_align followed by scd_patch_kv up to rounding, without forming h_hat
 * (its product of inner dimension d_model disappears).  act holds caller-owned [T, hidden]
 * activations and may repeat across layers: a run of consecutive Patch layers with distinct act
 * buffers is computed together (one launch of each product), and a buffer that repeats starts a
 * new run after the previous one has consumed it, so one buffer can serve every layer (at the
 * cost of a launch pair per layer).  c_k, c_v are optional (NULL = 0).  Other arguments and
 * limits as scd_patch_align and scd_patch_kv.  Reuse layers are not touched. */
scd_status_t scd_patch_fold(const scd_model_t* model, int32_t hidden,
                            const void* const* w2, const void* const* b2,
                            const void* const* w_k, const void* const* w_v,
                            const void* const* b_k, const void* const* b_v,
                            void* const* w_fold_k, void* const* w_fold_v,
                            void* const* c_k, void* const* c_v, hipStream_t stream);
scd_status_t scd_patch_kv_from_codes(const scd_model_t* model, const scd_batch_t* batch,
                                     const void* rope_table, int64_t max_position, int32_t hidden,
                                     const void* const* z_h,
                                     const void* const* w1, const void* const* b1,
                                     const void* const* w_fold_k, const void* const* w_fold_v,
                                     const void* const* c_k, const void* const* c_v,
                                     void* const* act, void* const* k_cache, void* const* v_cache,
                                     hipStream_t stream);

/* ---- packed payload and streamed receipt (Algorithm 1's transmitted set; Section 4.5) ---------
 * The codes Algorithm 1 sends travel as one contiguous buffer in the layout scd_payload_bytes
 * describes: layers in order, a Reuse layer's K codes [T*g, rank_k] then its V codes
 * [T*g, rank_v], a Patch layer's code [T, rank_h], no padding.
 *
 * scd_payload_views (host only, touches no memory) fills z_k, z_v, z_h [n_layers] with the
 * addresses of each layer's codes inside `payload` (any 16-byte aligned buffer of
 * scd_payload_bytes bytes), NULL for the branches a layer does not have.  The arrays can be passed
 * as they are to scd_encode (which then writes the packed payload), scd_reuse_decode and
 * scd_patch_align.
 *
 * scd_reuse_decode_streamed is the consumer's receipt: it copies the whole payload from
 * payload_src (pinned host memory, or device memory of this or a peer device; any address
 * hipMemcpyDefault accepts; pageable host memory works but serialises the copies) to payload_dst
 * (device, 16-byte aligned, scd_payload_bytes bytes, not overlapping payload_src) in groups of
 * layers_per_group layers on copy_stream, and enqueues the Reuse decode of each group (as
 * scd_reuse_decode, reading the codes from payload_dst) on `stream` behind that group's copy, so
 * the decode of one group overlaps the copy of the next.  The copies start after the work already
 * queued on `stream`; on return `stream` is ordered after every copy, so work queued on it next
 * (the aligner and scd_patch_kv on the Patch layers' codes) sees the whole payload.  copy_stream
 * may equal `stream` (no overlap).  With no tokens the payload is empty and both payload
 * pointers may be NULL.  The other arguments are scd_reuse_decode's.  SCD_ERR_HIP can leave
 * earlier groups enqueued; every other error means nothing was enqueued. */
scd_status_t scd_payload_views(const scd_model_t* model, int64_t n_tokens, void* payload,
                               void** z_k, void** z_v, void** z_h);
scd_status_t scd_reuse_decode_streamed(const scd_model_t* model, const scd_batch_t* batch,
                                       const void* rope_table, int64_t max_position,
                                       const void* payload_src, void* payload_dst,
                                       int32_t layers_per_group,
                                       const void* const* w_dec_k, const void* const* w_dec_v,
                                       const void* const* mu_k, const void* const* mu_v,
                                       void* const* k_cache, void* const* v_cache,
                                       hipStream_t copy_stream, hipStream_t stream);

/* ---- Offline Reuse fit (Section 4.3.1 "Joint Subspace Learning"; Appendix F.1) ---------------
 * Fits one branch's Reuse translators for every Reuse layer from paired calibration caches: the
 * producer's a_in[l] and the consumer's b_in[l], both [T, H, d_h] over the same packed batch of
 * prefixes (positions as everywhere else).  With rows A, B [N, w] (N = T*g; keys de-rotated first)
 * and X = [A B]:
 *   centring (optional):  mu_enc = mean of A's rows, mu_dec = mean of B's rows; A, B lose them;
 *   truncated SVD:        V_r = the top-r right singular vectors of X (r = rank_k or rank_v of
 *                         the layer), each with its largest-magnitude entry positive; Z = X V_r;
 *   ridge encoder:        E = argmin ||A E - Z||^2 + lambda ||E||^2   -> w_enc [r, w] = E^T;
 *   ridge decoder:        F = argmin ||Z F - B||^2 + lambda ||F||^2   -> w_dec [w, r] = F^T.
 * The outputs are exactly the w_enc / mu_enc the encoder takes and the w_dec / mu_dec the Reuse
 * decoder takes (the paper leaves the latent scale, the decoder's fit and the centring open: Z
 * carries the singular values, the decoder is a ridge fit with the same lambda, and centring is a
 * flag).
 *
 * The fit runs in two calls, stream-ordered:
 *  - scd_fit_gram accumulates, per Reuse layer, gram[l] = X^T X (fp32 [2w, 2w], symmetric) and
 *    colsum[l] = 1^T X (fp32 [2w]) on the matrix cores (bf16: keys de-rotated and rounded to bf16
 *    once, fp32 accumulation; fp32: fp32 products).  Rows are split into slices whose partial sums
 *    go to `workspace` and are added in a fixed order, so the result is deterministic.  branch 0 =
 *    keys (de-rotated; rope_table required), 1 = values.  Needs basis_width % 64 == 0 and at least
 *    one token.
 *  - scd_fit_solve takes those sums for N = n_rows rows (n_tokens * g) and solves the fit in fp64
 *    (Householder tridiagonalisation of the centred Gram, bisection and inverse iteration for its
 *    top r eigenpairs, Cholesky ridge solves; each stage one launch over all layers, except the
 *    tridiagonalisation, one launch per column until at most 256 rows remain, and the Cholesky,
 *    two launches per 64 columns), writing w_enc, w_dec and, when
 *    center = 1, mu_enc and mu_dec in the model's dtype (rounded once).  Needs basis_width <= 1024
 *    and 16 <= rank <= basis_width, rank % 16 == 0, lambda >= 0.  lambda = 0 with a singular
 *    A^T A (fewer independent rows than w) leaves NaN in the layer's outputs.  Eigenvalues within
 *    1e-7 ||G_c|| of each other are solved as a cluster by one thread in turn (slow only for large
 *    clusters, e.g. a rank above the calibration rows' own rank).
 * `workspace` (device, 16-byte aligned, caller-owned, contents undefined on entry and exit, not
 * overlapping any argument) must hold scd_fit_workspace_bytes(model, n_tokens) bytes; one buffer
 * serves both calls.  Each layer's outputs need buffers of their own (a buffer that repeats across
 * layers returns SCD_ERR_SHAPE).  Layers run 64 per launch; the calls never synchronise.  Patch
 * layers are not touched. */
size_t scd_fit_workspace_bytes(const scd_model_t* model, int64_t n_tokens);
scd_status_t scd_fit_gram(const scd_model_t* model, const scd_batch_t* batch,
                          const void* rope_table, int64_t max_position, int32_t branch,
                          const void* const* a_in, const void* const* b_in,
                          float* const* gram, float* const* colsum, void* workspace,
                          size_t workspace_bytes, hipStream_t stream);
scd_status_t scd_fit_solve(const scd_model_t* model, int32_t branch, int64_t n_rows,
                           double ridge_lambda, int32_t center, const float* const* gram,
                           const float* const* colsum, void* const* w_enc, void* const* w_dec,
                           void* const* mu_enc, void* const* mu_dec, void* workspace,
                           size_t workspace_bytes, hipStream_t stream);

/* ---- Allocation-free fit solve -----------------------------------------------------------------
 * For callers that cannot allocate device memory or hand over a workspace (code under stream
 * capture, serving loops, harnesses that forbid allocation): scd_fit_solve without the workspace
 * arguments.  Same arguments, validation and results (bit-identical) as scd_fit_solve.  The
 * solve's fp64 matrices live in a device-resident scratch array of
 * scd_fit_solve_noalloc_max_bytes() bytes (64 MiB) that the library holds on each GPU it runs on
 * until the process ends; layers are solved in as many stream-ordered rounds of launches as that
 * array needs (4 (2w)^2 + 8 (2w) fp64 values per layer).  A basis width whose per-layer matrices
 * exceed the array (w > 512) returns SCD_ERR_WORKSPACE.  The call uses the calling thread's
 * current device, which must own the stream and the buffers; its first call on a device looks the
 * array's address up.  It allocates
 * nothing and never synchronises.  Every call on one GPU shares that GPU's array: calls that may
 * run at the same time on one GPU (different streams, or other threads) race on it and must be
 * serialised by the caller. */
size_t scd_fit_solve_noalloc_max_bytes(void);
scd_status_t scd_fit_solve_noalloc(const scd_model_t* model, int32_t branch, int64_t n_rows,
                                   double ridge_lambda, int32_t center, const float* const* gram,
                                   const float* const* colsum, void* const* w_enc,
                                   void* const* w_dec, void* const* mu_enc, void* const* mu_dec,
                                   hipStream_t stream);

/* ---- Serving the rebuilt cache: rotary positions, a paged 8-bit cache, attention over it -------
 * What a consumer does with its KV cache once the codec has rebuilt it (the decode loop that follows
 * Algorithm 1, Appendix F.2's cache positions): rows go into pages, new tokens' queries and keys are
 * rotated to their positions, and the tokens attend to everything their request holds.  The calls
 * below take a batch of new tokens: request b owns rows [cu_seqlens[b], cu_seqlens[b+1]) and already
 * holds pos0[b] tokens, so row i of the request has position pos0[b] + i.
 *
 * scd_rows_t describes the rows of one tensor: channel c of head h of token t is element
 * t * token_stride + h * head_stride + c of `data` (the model's dtype).  Any strides are taken, such
 * as slices of a fused projection's rows or a head-major layout; rows whose addresses and strides
 * are multiples of 16 bytes are read and written 16 bytes at a time.  `data` need only be aligned to
 * its element (scd_rows_t is the exception to the 16-byte rule above). */
typedef struct {
  void* data;            /* DEVICE */
  int32_t n_heads;
  int64_t token_stride;  /* elements */
  int64_t head_stride;   /* elements */
} scd_rows_t;

/* Rotary positions: pair i of a head (i < rotary_dim / 2) turns by p * w_i at position p.  Channels
 * from rotary_dim on pass through.  HALF pairs channel i with i + rotary_dim / 2 (the codec's own
 * layout), INTERLEAVED pairs 2i with 2i + 1.  With w_i = theta^(-2i / rotary_dim) the frequencies
 * are, by `scaling`:
 *   NONE      w_i
 *   LINEAR    w_i / factor                                    (positions interpolated)
 *   NTK       w_i of the base theta * factor^(rotary_dim / (rotary_dim - 2))
 *   BY_PARTS  (1 - g) w_i / factor + g w_i, g = clamp((n - low) / (high - low), 0, 1) with
 *             n = trained_positions w_i / 2 pi the turns pair i makes over the trained context
 *   GIVEN     frequencies[i] (host array, read during scd_rotary_table)
 * Cosines and sines are multiplied by attention_factor (1 = none). */
typedef enum { SCD_ROTARY_HALF = 0, SCD_ROTARY_INTERLEAVED = 1 } scd_rotary_layout_t;
typedef enum {
  SCD_ROTARY_NONE = 0,
  SCD_ROTARY_LINEAR = 1,
  SCD_ROTARY_NTK = 2,
  SCD_ROTARY_BY_PARTS = 3,
  SCD_ROTARY_GIVEN = 4
} scd_rotary_scaling_t;

typedef struct {
  int32_t head_dim;             /* even, at most 512 */
  int32_t rotary_dim;           /* even, 2 <= rotary_dim <= head_dim */
  int32_t layout;               /* scd_rotary_layout_t */
  int32_t scaling;              /* scd_rotary_scaling_t */
  double theta;                 /* > 1 */
  double factor;                /* > 0; read by LINEAR, NTK, BY_PARTS */
  double low, high;             /* low < high; read by BY_PARTS */
  double attention_factor;      /* > 0 */
  int64_t trained_positions;    /* >= 1; read by BY_PARTS */
  const double* frequencies;    /* HOST [rotary_dim / 2]; read by GIVEN */
} scd_rotary_t;

/* Table of (cos, sin) for positions [0, max_position), fp32 [max_position][rotary_dim / 2][2],
 * evaluated in fp64 and rounded once; built once per (rotary, max_position) and passed with the same
 * pair to the calls below, which trust it as the codec's calls trust theirs. */
size_t scd_rotary_table_bytes(const scd_rotary_t* rotary, int64_t max_position);
scd_status_t scd_rotary_table(const scd_rotary_t* rotary, int64_t max_position, void* table,
                              size_t table_bytes, hipStream_t stream);

/* q_out = R(p) q and k_out = R(p) k for every row, in fp32, rounded once to dtype.  k and k_out may
 * both be NULL.  transpose = 1 applies R(p)^T instead: the gradient of the call with respect to q and
 * k, and, where attention_factor is 1, its inverse.  An output may be its input (same data and
 * strides); otherwise outputs must not overlap inputs. */
scd_status_t scd_rotary(const scd_rotary_t* rotary, const scd_batch_t* batch, const void* table,
                        int64_t max_position, int32_t dtype, int32_t transpose,
                        const scd_rows_t* q, const scd_rows_t* k, const scd_rows_t* q_out,
                        const scd_rows_t* k_out, hipStream_t stream);

/* Paged 8-bit cache of one layer.  A page holds page_tokens consecutive positions of one request, for
 * every KV head: k_pages and v_pages are int8 [n_pages, n_kv_heads, page_tokens, head_dim], and a
 * value stands for q * scale with the page's and head's scale in k_scales, v_scales
 * [n_pages, n_kv_heads] (fp32).  page_table [n_seqs, max_pages] (device, aligned to its entries, so
 * rows of a larger table will do) names the page of each run of page_tokens positions of each request.
 * An entry outside [0, n_pages) is a hole: rows appended there are dropped, rows read there are zero,
 * and attention leaves its positions out; so are positions from max_pages * page_tokens on and negative
 * ones.  Pages that several requests name (a shared prefix) can be read, and must not be appended to.
 * head_dim 32, 64 or 128; page_tokens 16, 32, 64 or 128. */
typedef struct {
  int32_t n_pages;
  int32_t page_tokens;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t max_pages;
  int8_t* k_pages;
  int8_t* v_pages;
  float* k_scales;
  float* v_scales;
  const int32_t* page_table;
} scd_cache_t;

/* Appends rows k, v [n_tokens, n_kv_heads, head_dim] at positions pos0[b] + i.  With `rotary` the
 * keys are rotated to their positions on the way, in fp32, with no rounding before the quantisation
 * (rotary NULL: as they are, for keys that the codec's decode or scd_rotary has rotated; table and
 * max_position are then not read).
 * For each page and head that new rows touch, with a = the largest magnitude of the new values:
 *   scale = max(scale, a / 127)   (the old scale counts only if the page holds earlier positions)
 *   q     = round(x / scale), ties to even, in [-127, 127]   (as x times the fp32 1 / scale)
 * and where the scale grew the page's earlier values are rounded again to the new one (so a value is
 * rounded at most once more per growth).  Scales below 2^-126 become 0 and their values 0.  A value
 * that is not finite makes the scale of its page and head NaN, and with it all the page holds of that
 * head, until the page is begun again.  Slots past the last row keep what they held. */
scd_status_t scd_cache_append(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                              const scd_rows_t* k, const scd_rows_t* v,
                              const scd_rotary_t* rotary, const void* table,
                              int64_t max_position, hipStream_t stream);

/* Reads positions pos0[b] + i (pos0 NULL: from the start) of every request back as dense rows: what
 * scd_encode takes from a producer that serves from pages.  Each value is q * scale in fp32, rounded
 * once to dtype. */
scd_status_t scd_cache_read(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                            const scd_rows_t* k_out, const scd_rows_t* v_out, hipStream_t stream);

/* Causal attention of the new tokens over the cache, which already holds them (append first).  For
 * query row i of request b and query head h (of KV head h / (q.n_heads / n_kv_heads)):
 *   out = sum_j p_j v_j,  p = softmax over j of softmax_scale * (q . k_j),  j in [0, pos0[b] + i]
 * One token per request and whole prompts are the same call, which one kernel takes, chosen by the mean of
 * rows a request: a step's prompts and its single tokens are faster as two calls.  Sums, running maxima and
 * the softmax are fp32, and positions count in it whatever their page's value scale (0, or any from 2^-126
 * on, as scd_cache_append stores them; never negative).  Weights multiply the values with 24 bits in fp32
 * calls and 16 or, in prompts, 11 in bf16 calls: there a weight times its value scale that is below 2^-25 of
 * the row's largest has fewer.  A row with no position to attend to (a hole at every one) is zero.
 * q [n_tokens, n_heads, head_dim], n_heads a multiple of n_kv_heads; out alike, not overlapping q.
 * n_tokens * n_heads must be below 2^31 (else SCD_ERR_UNSUPPORTED), and cached positions from 2^31 - 64
 * on are left out.
 * `workspace` (device, 16-byte aligned, caller-owned) holds
 * scd_cache_attend_workspace_bytes(cache, batch, q.n_heads) bytes; when that is 0 it may be NULL.  Its
 * first SCD_ATTEND_COUNTER_BYTES (or all of it, if less) must be zero before its first use; every call
 * leaves them zero, so one buffer serves calls of any shapes one after another, and the rest may hold
 * anything.  The size depends on n_tokens, n_seqs, max_pages and the heads, not on device contents, so a
 * captured call can be replayed while lengths grow.  Calls that may overlap need one each. */
#define SCD_ATTEND_COUNTER_BYTES 2048
size_t scd_cache_attend_workspace_bytes(const scd_cache_t* cache, const scd_batch_t* batch,
                                        int32_t n_q_heads);
scd_status_t scd_cache_attend(const scd_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                              double softmax_scale, const scd_rows_t* q, const scd_rows_t* out,
                              void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---- A latent cache: one low-rank row a token instead of keys and values ------------------------
 * A model whose layers project every token to one latent c [latent_dim] and one key k [turned_dim] that all
 * heads share has, for head h,
 *   keys  [ W_k,h c | k ]  (plain_dim + turned_dim channels, k rotated to its position),
 *   values  W_v,h c        (value_dim channels),
 * as the codec's decoder has rows from codes.  Only (c, k) are cached, in the model's dtype: pages is
 * [n_pages, page_tokens, latent_dim + turned_dim], page_table as of scd_cache_t, holes and positions outside
 * the table likewise.  latent_dim a multiple of 32 up to 512, turned_dim 32 or 64, page_tokens 16, 32, 64 or
 * 128; plain_dim and value_dim multiples of 32 up to 256.  w_k [n_heads, plain_dim, latent_dim] and
 * w_v [n_heads, value_dim, latent_dim] are contiguous, 16-byte aligned, in the model's dtype. */
typedef struct {
  int32_t n_pages;
  int32_t page_tokens;
  int32_t latent_dim;
  int32_t turned_dim;
  int32_t max_pages;
  void* pages;
  const int32_t* page_table;
} scd_latent_cache_t;

/* Appends rows latent [n_tokens, 1, latent_dim] and turned [n_tokens, 1, turned_dim] at positions pos0[b] + i.
 * With `rotary` (head_dim = turned_dim) the shared keys are rotated to them on the way, in fp32, rounded once;
 * NULL: as they are.  Latents keep their bits.  Rows behind the last request are left alone, and pages that
 * several requests name must not be appended to (scd_pages_reserve sees to it). */
scd_status_t scd_latent_append(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               const scd_rows_t* latent, const scd_rows_t* turned, const scd_rotary_t* rotary,
                               const void* table, int64_t max_position, hipStream_t stream);

/* Causal attention of the new tokens over the cache, which already holds them, with nothing expanded: for query
 * row q_i,h [plain_dim + turned_dim] (its last turned_dim channels rotated: scd_rotary takes them as strided rows)
 *   a = W_k,h^T q_i,h[:plain_dim],  s_j = softmax_scale (a . c_j + q_i,h[plain_dim:] . k_j),  j <= pos0[b] + i
 *   out_i,h = W_v,h sum_j p_j c_j,  p = softmax(s)
 * q [n_tokens, n_heads, plain_dim + turned_dim], out [n_tokens, n_heads, value_dim], not overlapping q.  Sums and
 * the softmax are fp32.  In bf16 calls queries in the latents' space, the softmax's weights and the weighted latents
 * are held as two bf16 summands, 16 bits.  A row with no position to attend to is zero.  A position whose latent or key
 * is not finite reaches the rows that attend to it (which it makes not finite, unless its scores are -inf and its latent
 * finite: that takes it out of them), and no others.  One call takes one
 * token a request or a chunk of them.  scd_latent_expand and scd_rows_attend take (plain_dim + turned_dim + value_dim) /
 * (2 latent_dim + turned_dim) of the arithmetic, and the expansion beside it: less only where 2 latent_dim is well above
 * plain_dim + value_dim and new tokens are many for the positions expanded (32 heads of 128 + 64 and 128 channels,
 * latent_dim 256: from about 100 tokens behind 2000 positions, from fewer than 16 behind 200).
 * n_tokens up to 65535, n_tokens * n_heads below 2^27, cached positions below 2^31 - 128.
 * `workspace` (device, 16-byte aligned, caller-owned, any contents) holds
 * scd_latent_attend_workspace_bytes(cache, batch, dtype, n_heads) bytes, which depend on the sizes alone, so
 * that a captured call can be replayed while lengths grow.  Calls that may overlap need one each. */
size_t scd_latent_attend_workspace_bytes(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                                         int32_t n_heads);
scd_status_t scd_latent_attend(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               double softmax_scale, int32_t plain_dim, int32_t value_dim, const void* w_k,
                               const void* w_v, const scd_rows_t* q, const scd_rows_t* out, void* workspace,
                               size_t workspace_bytes, hipStream_t stream);

/* The dense keys and values of cached positions pos0[b] + i (pos0 NULL: from the start): k_out
 * [n_tokens, n_heads, plain_dim + turned_dim], v_out [n_tokens, n_heads, value_dim], products in fp32 and rounded
 * once, shared keys with their bits.  A position in a hole or outside the table gives zeros, and rows behind the
 * last request are left alone. */
scd_status_t scd_latent_expand(const scd_latent_cache_t* cache, const scd_batch_t* batch, int32_t dtype,
                               int32_t n_heads, int32_t plain_dim, int32_t value_dim, const void* w_k, const void* w_v,
                               const scd_rows_t* k_out, const scd_rows_t* v_out, hipStream_t stream);

/* Causal attention over dense rows: those that scd_latent_expand writes, or the caches that the codec's decode and
 * Patch write.  `held` names the key and value rows of every request as `batch` names its query rows: row j of
 * request b has position held.pos0[b] + j (NULL: j), row i of its queries position batch.pos0[b] + i.
 *   out_i = sum_j p_j v_j,  p = softmax over j of softmax_scale (q_i . k_j),  position j <= position i
 * q [batch.n_tokens, n_heads, key_dim], k [held.n_tokens, n_kv_heads, key_dim], v [.., n_kv_heads, value_dim], query
 * head h reads KV head h / (n_heads / n_kv_heads); out [batch.n_tokens, n_heads, value_dim], overlapping no input.
 * key_dim a multiple of 32 up to 192, value_dim up to 128.  Sums and the softmax are fp32.  In bf16 calls its weights
 * are held as two bf16 summands, 16 bits; calls of more than 64 query rows a KV head and request on average, of 16-byte
 * rows, round them to bf16 once (the sum that divides is of unrounded ones).  A row with no position to attend to is
 * zero.  Keys and values behind a row's position do not reach it, whatever they hold; a value that is not finite makes
 * its channel not finite in the rows that attend to it, a key whose scores are -inf takes its position out of them.
 * Fastest where all rows and strides are multiples of 16 bytes.  The workspace is as of scd_latent_attend; where it is
 * 0 bytes it may be NULL. */
size_t scd_rows_attend_workspace_bytes(const scd_batch_t* batch, const scd_batch_t* held, int32_t dtype, int32_t n_heads,
                                       int32_t n_kv_heads, int32_t key_dim, int32_t value_dim);
scd_status_t scd_rows_attend(const scd_batch_t* batch, const scd_batch_t* held, int32_t dtype, double softmax_scale,
                             int32_t key_dim, int32_t value_dim, const scd_rows_t* q, const scd_rows_t* k,
                             const scd_rows_t* v, const scd_rows_t* out, void* workspace, size_t workspace_bytes,
                             hipStream_t stream);

/* ---- Pages of caches: given back, shared, reserved, moved -------------------------------------------
 * One pool of pages serves the caches of all layers: page id p is page p of every layer's scd_cache_t or
 * scd_latent_cache_t, and page_table [n_seqs, max_pages] names a request's pages for all of them.  refs [n_pages]
 * counts the table entries that name a page (0: free), held [n_seqs] is what every request holds (its pos0 in the
 * next batch).  All are int32 in device memory; an entry outside [0, n_pages) names nothing.  Fresh pages are the
 * lowest free ones, to requests in their order and a request's positions in theirs, so results depend on the arguments
 * alone.  The calls take a pool one after another: on one stream, or ordered by the caller.  n_pages, n_seqs and
 * max_pages are up to 2^30. */
typedef struct {
  int32_t n_pages;
  int32_t n_seqs;
  int32_t max_pages;
  int32_t page_tokens;
  int32_t* refs;
  int32_t* page_table;
  int32_t* held;
} scd_pages_t;

/* Pages whose contents are to be moved, from pairs[2 k] to pairs[2 k + 1] for k < status[0], written by the two
 * calls that say so and read by scd_pages_copy.  No page is both.  status [4] (device): the count of moves; pages in
 * use (scd_pages_compact); pages that are missing; requests whose tokens do not fit the table.  Where one of the last
 * two is not zero the call has changed nothing else.  Pairs past the count keep what they held. */
typedef struct {
  int32_t capacity;     /* pairs */
  int32_t* pairs;       /* DEVICE [capacity, 2] */
  int32_t* status;      /* DEVICE [4] */
} scd_moves_t;

/* Requests seqs[0 .. n) (device) give their pages back: every page they name is counted down, their table entries
 * become -1, held 0.  A request named twice counts once; one outside [0, n_seqs) is passed over. */
scd_status_t scd_pages_free(const scd_pages_t* pages, int32_t n, const int32_t* seqs, hipStream_t stream);

/* Request dst[i] becomes a copy of src[i] without any contents moved: it names the pages that src[i] holds tokens in
 * (the last one too, though it be begun only: scd_pages_reserve separates them once one writes), which are counted
 * up, and holds as many tokens.  A pair is passed over where either is outside [0, n_seqs), where dst[i] holds tokens,
 * names a page or is the target of an earlier pair, and where src[i] is the target of any pair. */
scd_status_t scd_pages_fork(const scd_pages_t* pages, int32_t n, const int32_t* src, const int32_t* dst,
                            hipStream_t stream);

/* Makes the positions held[b] .. held[b] + n_b - 1 of every request writable, n_b its rows in `batch` (whose pos0 is
 * not read): missing pages are taken, and pages that others name too are replaced by fresh ones, with a move
 * where such a page holds earlier positions.  Of requests that all write to one page the last keeps it, if no other
 * names it.  held stays: the caller counts it up with the tokens.  moves holds n_seqs pairs or more. */
size_t scd_pages_workspace_bytes(const scd_pages_t* pages);  /* of the two calls below; any contents */
scd_status_t scd_pages_reserve(const scd_pages_t* pages, const scd_batch_t* batch, const scd_moves_t* moves,
                               void* workspace, size_t workspace_bytes, hipStream_t stream);

/* The n pages in use become pages 0 .. n - 1: the k-th of those behind moves to the k-th free page in front. Table and
 * counts are written to `out` (NULL or equal pointers: in place; its held is not written).  moves holds n_pages / 2
 * pairs or more. */
scd_status_t scd_pages_compact(const scd_pages_t* pages, const scd_pages_t* out, const scd_moves_t* moves,
                               void* workspace, size_t workspace_bytes, hipStream_t stream);

/* Moves the contents of the listed pages in every plane: page p of a plane is page_bytes bytes (a multiple of 4) at
 * data + p * page_bytes, data 16-byte aligned.  A scd_cache_t is four planes (k_pages, v_pages, k_scales, v_scales), a
 * latent cache one.  A move that names a page outside [0, n_pages) is passed over. */
typedef struct {
  void* data;           /* DEVICE */
  int64_t page_bytes;
} scd_plane_t;
scd_status_t scd_pages_copy(int32_t n_planes, const scd_plane_t* planes, int32_t n_pages, const scd_moves_t* moves,
                            hipStream_t stream);

/* ---- diagnostics ---------------------------------------------------------------------------- */
const char* scd_status_string(scd_status_t status);
/* Detail of the last non-OK status returned on the calling thread ("" if none). */
const char* scd_last_error(void);
/* ABI version: bumped whenever a signature or a struct above changes. */
int32_t scd_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SCD_H_ */
