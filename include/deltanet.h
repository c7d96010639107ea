/*
 * deltanet.h - C ABI of the MI355X (gfx950) chunkwise-parallel DeltaNet layer.
 *
 * The operation is the DeltaNet token mixer of "Parallelizing Linear Transformers with the Delta
 * Rule over Sequence Length": per (sequence, head) chain, with a state S in R^{d_k x d_v},
 *
 *     S_t = S_{t-1} + beta_t k_t (v_t - S_{t-1}^T k_t)^T ,   o_t = S_t^T q_t
 *
 * (section 2.2, the delta update rule and read-out; section 3.1 writes the same update as a
 * generalized Householder transition S_{t-1}(I - beta k k^T) + beta v k^T; the state is kept in the
 * orientation of the paper's pseudocode listing, d_k rows by d_v columns).  It is evaluated in the
 * chunkwise-parallel form of section 3.2 (Eq. 8-9: inter-chunk state carry plus causal intra-chunk
 * output) with the per-chunk WY factors W, U built by the UT transform (Eq. 10-11).  No scale
 * factor is applied to q; normalising q, k and squashing beta are the caller's job.
 *
 * Conventions common to every call
 *  - All data pointers are DEVICE pointers unless a name ends in _host.  The caller owns every
 *    buffer; the library never allocates, frees or synchronises.  All work is enqueued on
 *    `hip_stream` (a hipStream_t passed as void*; NULL = the default stream).
 *  - Dense layout: q,k [B,L,H,d_k]; v,o,do [B,L,H,d_v]; beta [B,L,H]; states [B,H,d_k,d_v].
 *    Packed layout (cu_seqlens != NULL): B must be 1, L is the total token count, sequence n
 *    covers rows cu_seqlens[n] .. cu_seqlens[n+1]-1, the state is reset at every sequence start and
 *    states are [num_seqs,H,d_k,d_v].  All tensors are contiguous and row-major.
 *  - q,k,v,beta,o,do,dq,dk,dv have element type `dtype` (fp32, or bf16 with fp32 accumulation);
 *    states, state gradients and dbeta are always fp32.
 *  - Every data pointer must be 16-byte aligned.
 *  - `workspace` is caller-provided device scratch of at least deltanet_workspace_bytes();
 *    its contents are undefined afterwards.  (For few long sequences the passes cut the sequences into
 *    segments that are scanned side by side; the per-segment states this needs are part of that size.)
 *  - Return value: DN_OK (0) or a negative dn_status.  All validation happens before the first
 *    launch; on a validation error nothing has been enqueued.  No exceptions, no abort.
 *  - Packed layout without cu_seqlens_host: nothing can be validated on the host; the kernels then work on the
 *    running maximum of the device array held inside [0, L] (the array itself if it is valid), so a malformed array
 *    gives meaningless results but no access outside the tensors or the workspace.
 *  - A tensor without rows (B * L == 0) may come with a NULL pointer; final_state is then initial_state (or zero).
 *  - Sequences of length 0 are allowed in the packed layout; lengths need not be multiples of
 *    the chunk size (a ragged last chunk is handled exactly, as beta = 0 leaves the state
 *    unchanged, section 2.2).
 */
#ifndef DELTANET_H_
#define DELTANET_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { DN_F32 = 0, DN_BF16 = 1, DN_FP8 = 2 /* e4m3; pages of a cache only */, DN_FP4 = 4 /* e2m1, likewise */ } dn_dtype;

typedef enum {
    DN_OK = 0,
    DN_ERR_NULL = -1,        /* a required pointer is NULL */
    DN_ERR_SHAPE = -2,       /* a size is non-positive or inconsistent */
    DN_ERR_UNSUPPORTED = -3, /* (dtype, d_k, d_v, chunk), or the attention's (types, d, page size, rot), has no compiled kernel */
    DN_ERR_ALIGN = -4,       /* a data pointer is not 16-byte aligned */
    DN_ERR_WORKSPACE = -5,   /* workspace is NULL or too small */
    DN_ERR_CUSEQLENS = -6,   /* cu_seqlens_host is not 0 = c[0] <= c[1] <= ... <= c[N] = L */
    DN_ERR_LAUNCH = -7       /* the HIP runtime reported an error at launch */
} dn_status;

typedef struct {
    int32_t B, L, H, d_k, d_v;
    int32_t chunk;                   /* C of section 3.2; 64 is the compiled value */
    int32_t dtype;                   /* dn_dtype */
    int32_t num_seqs;                /* packed layout only: N */
    const int32_t *cu_seqlens;       /* DEVICE int32 [N+1], or NULL for the dense layout */
    const int32_t *cu_seqlens_host;  /* optional HOST copy of the same array; if given it is
                                        validated (DN_ERR_CUSEQLENS) and never dereferenced later */
} dn_shape;

/* Bytes of device scratch that deltanet_fwd (want_bwd = 0) or deltanet_bwd (want_bwd != 0) needs
 * for this shape.  Host-only; touches no device. */
int deltanet_workspace_bytes(const dn_shape *shape, int want_bwd, size_t *out_bytes);

/*
 * Forward pass (Eq. 8-11).  initial_state may be NULL (zeros).  final_state may be NULL (not
 * written).  Outputs: o (element type dtype), final_state (fp32).
 * Compiled (d_k, d_v): fp32 (64,64), (32,64), (64,32); bf16 (128,128), (64,64), (64,128), (128,64)
 * and (256,256); every entry point below runs at each of them.
 */
int deltanet_fwd(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                 const float *initial_state, void *o, float *final_state, void *workspace,
                 size_t workspace_bytes, void *hip_stream);

/*
 * deltanet_fwd for callers that cannot allocate device memory: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments, results and errors as deltanet_fwd, minus the workspace: the
 * scratch the pass needs is a device array of DN_STATIC_SCRATCH_BYTES that is part of the library (every GPU the
 * library runs on holds its own copy until the process ends).  The call allocates and frees nothing.  Shapes whose
 * deltanet_workspace_bytes(shape, 0) exceeds DN_STATIC_SCRATCH_BYTES are refused with DN_ERR_WORKSPACE before anything
 * is enqueued (one C x C tile per chunk and head: 36 MiB covers 16 384 tokens x 16 heads in bf16, half as many in
 * fp32).  All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two streams, two
 * threads) race on it; calls on one stream, or otherwise ordered, do not.  Nothing in the array needs clearing
 * between calls.
 */
#define DN_STATIC_SCRATCH_BYTES (36u << 20)
int deltanet_fwd_static(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                        const float *initial_state, void *o, float *final_state, void *hip_stream);

/*
 * Backward pass: exact gradient of  sum(o * d_o) + sum(final_state * dfinal_state)  with respect to
 * q, k, v, beta and initial_state.  Self-contained: chunk states are recomputed from the inputs
 * (section 3.2, "hidden states recomputed during the backward pass"), so nothing from the forward
 * call has to be kept.  dfinal_state may be NULL (zeros); dinitial_state may be NULL (not written).
 * Outputs: dq, dk, dv (element type dtype), dbeta (fp32, shape of beta), dinitial_state (fp32).
 * dq, dk and dv may each take the place of a whole input of the same shape (dq over q, dk over k, dv over v or d_o, ...);
 * dv then costs one more copy.  No output may overlap another one, or an input in any other way.  This holds for every
 * backward pass below.
 */
int deltanet_bwd(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                 const float *initial_state, const void *d_o, const float *dfinal_state, void *dq,
                 void *dk, void *dv, float *dbeta, float *dinitial_state, void *workspace,
                 size_t workspace_bytes, void *hip_stream);

/*
 * The same forward and backward pass for a training step that keeps the forward pass's per-chunk
 * results instead of recomputing them (the other side of the trade section 3.2 describes: with
 * hundreds of GB of HBM the chunk states of a layer, d_k * d_v * 2 bytes per 64 tokens and head in
 * bf16, are cheap to keep, and the backward pass then skips the UT transform and the forward scan).
 * deltanet_fwd_save computes what deltanet_fwd computes and leaves T of Eq. 10, the
 * chunk-initial states and U - W S of Eq. 8 in `saved`; deltanet_bwd_saved computes what deltanet_bwd
 * computes from the same q, k, v, beta and that buffer, which it also uses as scratch (afterwards the
 * buffer can serve another deltanet_fwd_save, not another deltanet_bwd_saved).  `saved` is
 * caller-provided device memory of deltanet_workspace_bytes(shape, 1) bytes; its layout is private to
 * the library, and it must stay untouched between the two calls.  The initial state is not an argument
 * of deltanet_bwd_saved: it is the first saved chunk state.  Everything else is as for deltanet_fwd /
 * deltanet_bwd; head sizes without a backward pass return DN_ERR_UNSUPPORTED.
 */
int deltanet_fwd_save(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                      const float *initial_state, void *o, float *final_state, void *saved, size_t saved_bytes,
                      void *hip_stream);
int deltanet_bwd_saved(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                       const void *d_o, const float *dfinal_state, void *dq, void *dk, void *dv, float *dbeta,
                       float *dinitial_state, void *saved, size_t saved_bytes, void *hip_stream);

/*
 * The same passes with the layer's prologue fused into the load path (section 3.3, "Feature map and
 * normalization", and the writing strength of section 2.2): the caller hands over the pre-activations
 * q_pre, k_pre (layouts and element type of q, k) and the logits beta_logit (layout and element type of
 * beta), and the kernels form
 *
 *     q_t = SiLU(q_pre_t) / ||SiLU(q_pre_t)||_2 ,  k_t likewise,  beta_t = sigmoid(beta_logit_t)
 *
 * per token and head (fp32 arithmetic, result rounded to the element type).  The kernel that builds T
 * maps q and k once and leaves them in the workspace for the chain scans and the backward's chunk kernel, which
 * sends dq, dk back through the map on their way out, so the gradients never reach HBM in the mapped coordinates
 * and no separate elementwise pass runs in either direction.  A row whose SiLU image is exactly zero maps to zero
 * (the paper gives no epsilon).
 * deltanet_fused_bwd returns the gradients with respect to q_pre, k_pre and beta_logit (through the
 * normalisation, the SiLU and the sigmoid) in dq_pre, dk_pre (element type dtype) and dbeta_logit
 * (fp32); dv and dinitial_state are as for deltanet_bwd.  Workspace (and `saved`) sizes come from
 * deltanet_fused_workspace_bytes: the plain sizes plus the mapped q and k.  deltanet_fused_fwd_save /
 * deltanet_fused_bwd_saved are the pair that keeps the forward pass's per-chunk results, as
 * deltanet_fwd_save / deltanet_bwd_saved.  Everything else is as for the plain calls.
 */
int deltanet_fused_workspace_bytes(const dn_shape *shape, int want_bwd, size_t *out_bytes);
int deltanet_fused_fwd(const dn_shape *shape, const void *q_pre, const void *k_pre, const void *v, const void *beta_logit,
                       const float *initial_state, void *o, float *final_state, void *workspace, size_t workspace_bytes,
                       void *hip_stream);
int deltanet_fused_bwd(const dn_shape *shape, const void *q_pre, const void *k_pre, const void *v, const void *beta_logit,
                       const float *initial_state, const void *d_o, const float *dfinal_state, void *dq_pre, void *dk_pre,
                       void *dv, float *dbeta_logit, float *dinitial_state, void *workspace, size_t workspace_bytes,
                       void *hip_stream);
int deltanet_fused_fwd_save(const dn_shape *shape, const void *q_pre, const void *k_pre, const void *v,
                            const void *beta_logit, const float *initial_state, void *o, float *final_state, void *saved,
                            size_t saved_bytes, void *hip_stream);
int deltanet_fused_bwd_saved(const dn_shape *shape, const void *q_pre, const void *k_pre, const void *v,
                             const void *beta_logit, const void *d_o, const float *dfinal_state, void *dq_pre, void *dk_pre,
                             void *dv, float *dbeta_logit, float *dinitial_state, void *saved, size_t saved_bytes,
                             void *hip_stream);

/*
 * Forward pass in the recurrent (token-serial) form: the delta-rule update and read-out of
 * section 2.2 applied one token after the other, state in fp32 registers, no chunking, no matrix
 * cores and no workspace.  It computes the same o and final_state as deltanet_fwd (fp32 arithmetic
 * on the fp32 or bf16 inputs) and is what a decoder calls with L = 1 per step, handing
 * final_state back in as initial_state; it is also the baseline the paper's chunkwise form is
 * timed against (section 3.3).  Same layouts, pointer rules and return codes as deltanet_fwd.
 * Compiled for d_k in {32, 64, 128, 256} and any d_v that is a multiple of 16, both dtypes
 * (else DN_ERR_UNSUPPORTED).  `chunk` is not used but must hold a supported value.
 * initial_state may be NULL (zeros); final_state may be NULL (not written); the two may alias.
 */
int deltanet_recurrent_fwd(const dn_shape *shape, const void *q, const void *k, const void *v,
                           const void *beta, const float *initial_state, void *o, float *final_state,
                           void *hip_stream);

/*
 * Gated variant: the last row of the paper's overview table of linear recurrent models (section 6),
 * which its limitations section names as the way to add the decay DeltaNet lacks.  A scalar decay
 * alpha_t = exp(g_t) per token and head multiplies the transition,
 *
 *     S_t = alpha_t (S_{t-1} - beta_t k_t (S_{t-1}^T k_t)^T) + beta_t k_t v_t^T ,   o_t = S_t^T q_t
 *
 * (state orientation as above; g = 0 is the plain delta rule).  g is fp32 [B,L,H] (packed: [L,H]),
 * g <= 0 expected; inside one chunk of 64 tokens the sum of |g| must stay below about 160 (a mean alpha
 * of about 0.08), as the kernels work with exp(+-(sum g) / 2) in fp32.  Evaluated chunkwise like
 * deltanet_fwd / deltanet_bwd: with gamma_i the running product of alpha inside a chunk, taken relative
 * to the chunk's geometric middle, S_i / gamma_i follows the plain delta rule on the values
 * v_i / gamma_i, so Eq. 8-11 apply unchanged to rescaled rows.  In bf16 the gate gradient dg, a
 * difference of nearly equal sums of rounded gradients, loses relative accuracy as the decay grows.  deltanet_gated_bwd also
 * returns dg (fp32, shape of g).  Workspace sizes come from deltanet_gated_workspace_bytes; everything
 * else (layouts, nullable states, return codes) is as for the plain calls.
 * deltanet_gated_recurrent_fwd is the token-serial form (decode steps), as deltanet_recurrent_fwd.
 */
int deltanet_gated_workspace_bytes(const dn_shape *shape, int want_bwd, size_t *out_bytes);
int deltanet_gated_fwd(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                       const float *g, const float *initial_state, void *o, float *final_state, void *workspace,
                       size_t workspace_bytes, void *hip_stream);
int deltanet_gated_bwd(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                       const float *g, const float *initial_state, const void *d_o, const float *dfinal_state,
                       void *dq, void *dk, void *dv, float *dbeta, float *dg, float *dinitial_state, void *workspace,
                       size_t workspace_bytes, void *hip_stream);
int deltanet_gated_recurrent_fwd(const dn_shape *shape, const void *q, const void *k, const void *v,
                                 const void *beta, const float *g, const float *initial_state, void *o,
                                 float *final_state, void *hip_stream);
/* The gated pair that keeps the forward pass's per-chunk results, as deltanet_fwd_save / deltanet_bwd_saved;
 * `saved` holds deltanet_gated_workspace_bytes(shape, 1) bytes. */
int deltanet_gated_fwd_save(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                            const float *g, const float *initial_state, void *o, float *final_state, void *saved,
                            size_t saved_bytes, void *hip_stream);
int deltanet_gated_bwd_saved(const dn_shape *shape, const void *q, const void *k, const void *v, const void *beta,
                             const float *g, const void *d_o, const float *dfinal_state, void *dq, void *dk, void *dv,
                             float *dbeta, float *dg, float *dinitial_state, void *saved, size_t saved_bytes,
                             void *hip_stream);

/*
 * The attention layers of a hybrid model (the paper's hybrids put sliding-window attention between DeltaNet layers, or replace
 * two of those by global attention): the pass between the projections and the attention, a paged cache of keys and
 * values, and the attention of new tokens over that cache.  The conventions above hold (device pointers, caller-owned
 * buffers, the caller's stream, validation before the first launch, 16-byte alignment); what differs:
 *  - Batches are packed: T rows in all, row t of a tensor with H heads is [H, d] at t * stride elements, so that q, k and v may
 *    be the column blocks of one projection's output.  A stride is at least H * d elements and a multiple of 16 bytes.
 *    Outputs are contiguous.
 *  - Query heads share key/value heads in equal groups: Hq is a multiple of Hkv, query head h reads head h / (Hq / Hkv).
 *
 * Norm and rotation.  Per token and head, with x a row of q or k and w the weight of the layer,
 *
 *     z = x / sqrt(mean(x^2) + eps) * w ,    y_a = z_a cos - z_b sin ,  y_b = z_b cos + z_a sin
 *
 * for the pairs (a, b) among the first `rot` elements; the others stay z.  Pairs are (i, i + rot / 2), or (2i, 2i + 1) if
 * `interleaved`; cos_sin (fp32 [max_pos, rot]) holds for each position the rot / 2 cosines, then the rot / 2 sines, of those
 * pairs' angles.  Arithmetic is fp32 (a row the sum of whose squares is past its range becomes zero); y is rounded once.  Weights have the element type of q and k; a NULL weight is all ones.
 * Positions outside [0, max_pos) read the table's nearest row.
 * Compiled: d = 32, 64, 128, 256 in fp32 and bf16; rot a multiple of 16 up to d, or 0 (no rotation; cos_sin may be NULL).
 */
typedef struct {
    int32_t rot, interleaved, max_pos;
    float eps; /* finite, >= 0 */
} dn_rope;

typedef struct {
    int32_t T, Hq, Hkv, d;               /* T <= 2^30, T * Hq < 2^31 */
    int32_t dtype;                       /* DN_F32 or DN_BF16 */
    int32_t seq_len;                     /* without a positions array: row t has position t % seq_len */
    int64_t q_stride, k_stride;          /* elements between rows of q and k */
} dn_qk_shape;

/* y for every row of q and of k.  positions: int32 [T], or NULL. */
int deltanet_qk_norm_rope_fwd(const dn_qk_shape *shape, const dn_rope *rope, const void *q, const void *k,
                              const void *q_weight, const void *k_weight, const float *cos_sin, const int32_t *positions,
                              void *q_out, void *k_out, void *hip_stream);

/*
 * Its gradient: from dq_out [T, Hq, d], dk_out [T, Hkv, d] (contiguous, element type dtype) and the q, k, weights and positions of
 * the forward call (nothing of which has to be kept), dq and dk in the element type, and the weights' gradients dq_weight,
 * dk_weight (fp32 [d]; NULL where not wanted), summed over rows and heads in fp32 in an order that the sizes alone decide.
 * dq may take the place of dq_out and dk that of dk_out.  Workspace: deltanet_qk_norm_rope_workspace_bytes.
 */
int deltanet_qk_norm_rope_workspace_bytes(const dn_qk_shape *shape, size_t *out_bytes);
int deltanet_qk_norm_rope_bwd(const dn_qk_shape *shape, const dn_rope *rope, const void *q, const void *k,
                              const void *dq_out, const void *dk_out, const void *q_weight, const void *k_weight,
                              const float *cos_sin, const int32_t *positions, void *dq, void *dk, float *dq_weight,
                              float *dk_weight, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * The paged cache of a layer: k_pages, v_pages [num_pages, Hkv, page_size, d] of type cache_dtype, which is the tensors' type
 * or, for bf16 tensors, DN_FP8 or DN_FP4.  With DN_FP8, k_scale, v_scale (fp32 [num_pages, Hkv, page_size]) hold a factor per token and head,
 * max |x| / 448 over the row, and the pages the e4m3 numbers nearest to x / factor, divided in fp32 (a row whose largest magnitude is under
 * 2^-100 is held as zeros, factor 0; one with an infinity reads back as NaN); or DN_FP4: k_pages, v_pages [.., d / 2] hold two e2m1 numbers a byte (magnitudes 0, 0.5, 1, 1.5, 2, 3, 4, 6; the sign in
 * a number's highest bit), the first one in the low half, and k_scale, v_scale (bytes [num_pages, Hkv, page_size, d / 32]) a factor for each group of 32 along d, 2^(byte - 127), the least power of two of which
 * six are no less than the group's largest magnitude; a number is the nearest to x / factor, ties to even (magnitudes over 1.5 * 2^127 are held as that; a group under 2^-100 is held as zeros, factor 1; one with an infinity or NaN, byte 255, reads back as
 * NaN).  These values are bf16 numbers, so that attention over them rounds nothing that it would not round in bf16.  page_size is 16, 32, 64, 128 or 256.
 * Sequence n of the batch has kv_len[n] tokens in the cache, the new ones of this step included; its token p stands in page
 * page_table[n][p / page_size], slot p % page_size (entries past its last page may hold anything).  Its new tokens are rows
 * cu_q[n] .. cu_q[n + 1] - 1 of the packed tensors, the last of them at position kv_len[n] - 1.  Rows in front of cu_q[0] and from cu_q[num_seqs] on
 * lie in no sequence (the arrays may be a part of a larger batch's).
 * These arrays live on the device and are not validated: kernels work on the first max_kv tokens of longer contexts (whose rows keep their positions) and on the rows that
 * lie in the tensors, drop writes to pages outside [0, num_pages) and read page 0 or num_pages - 1 in the place of such ones,
 * so that a malformed array gives meaningless results but no access outside the buffers.
 */
typedef struct {
    int32_t num_seqs, T;                 /* T: rows of q (k, v): the new tokens of all sequences */
    int32_t Hq, Hkv, d;
    int32_t dtype, cache_dtype;
    int32_t page_size, num_pages, max_pages; /* max_pages: columns of page_table */
    int32_t max_q, max_kv;               /* bounds: no sequence has more new tokens or a longer context; max_q <= T, max_kv <= max_pages * page_size,
                                            T and max_kv <= 2^30, T * Hq < 2^31 */
    const int32_t *cu_q;                 /* DEVICE int32 [num_seqs + 1] */
    const int32_t *kv_len;               /* DEVICE int32 [num_seqs] */
    const int32_t *page_table;           /* DEVICE int32 [num_seqs, max_pages] */
    int64_t q_stride, k_stride, v_stride;
} dn_paged_shape;                        /* every call checks Hq, T and the bounds, used or not, and the strides of the tensors that it has */

typedef struct { void *k_pages, *v_pages, *k_scale, *v_scale; } dn_paged_cache; /* scales: NULL unless DN_FP8 (fp32) or DN_FP4 (bytes) */

/* Writes the new tokens' k and v to the cache.  Rows whose position is negative (a context shorter than the chunk) or for which there is no room (max_kv and
 * more), and rows in no sequence, are not written.  q_stride is not used, max_q and Hq only checked. d as for the attention below. */
int deltanet_paged_append(const dn_paged_shape *shape, const void *k, const void *v, const dn_paged_cache *cache,
                          void *hip_stream);

/* The serving form of the norm and rotation: q_out [T, Hq, d] = y of q, and y of k, unrounded until it takes the pages' type, and v go
 * to the cache, in one launch.  Positions are those in the sequences. */
int deltanet_paged_norm_rope_append(const dn_paged_shape *shape, const dn_rope *rope, const void *q, const void *k,
                                    const void *v, const void *q_weight, const void *k_weight, const float *cos_sin,
                                    void *q_out, const dn_paged_cache *cache, void *hip_stream);

/* Reads tokens back: rows cu_out[n] .. cu_out[n + 1] - 1 of k_out, v_out [T_out, Hkv, d] (element type dtype) become the last ones of
 * sequence n's context (all of it, if that many); T_out <= 2^30, T_out * Hkv < 2^31.  A row in front of the context's start, past max_kv, or in no sequence, becomes zero. */
int deltanet_paged_read(const dn_paged_shape *shape, const dn_paged_cache *cache, const int32_t *cu_out, int32_t T_out,
                        void *k_out, void *v_out, void *hip_stream);

/*
 * Attention of the new tokens over the cache, which holds their own keys and values already: for the row at position p
 *
 *     o = sum_j exp(scale q . k_j) v_j / sum_j exp(scale q . k_j) ,   max(0, p - window + 1) <= j <= p
 *
 * (window = 0: the whole past).  A row without a position in its context (p < 0), or in no sequence, becomes zero.  Scores, the running maximum and sum and the output
 * are held in fp32, and scores of any size that fp32 holds are told apart (one that is 2^128 or more under its row's largest weighs nothing; a row all of whose scores are -infinity becomes zero); in bf16 the probabilities, multiplied by the cache's factors, enter the product with v as bf16 (in chunks of many rows
 * rounded, for few rows as two terms).  scale > 0.  Nothing at or past kv_len, nor before the windows of all of a sequence's new tokens, reaches a
 * result, whatever the pages hold there (values that one new token sees and another does not are given the weight zero in the other's row: an
 * infinity or NaN among THOSE may reach both).  Deterministic: the order of every sum depends on the sizes and lengths alone.
 * Compiled: d = 64, 128, 256 in bf16, with bf16, DN_FP8 or DN_FP4 pages; d = 32, 64, 128 in fp32 (the precision mode; max_q * Hq < 2^26 there).
 * Workspace: deltanet_paged_attn_workspace_bytes (it depends on num_seqs, T, the heads, d, the types, max_q, max_kv and window).
 */
int deltanet_paged_attn_workspace_bytes(const dn_paged_shape *shape, int32_t window, size_t *out_bytes);
int deltanet_paged_attn_fwd(const dn_paged_shape *shape, const void *q, const dn_paged_cache *cache, float scale,
                            int32_t window, void *o, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Around a mixer: the short convolution in front of it, the norm of its output with its gate, and what stands between two blocks.  The conventions at the top hold; rows
 * may be strided where a stride is given (elements, a multiple of 16 bytes), so that inputs and gradients may be column blocks of a projection's; other tensors are contiguous.
 * Sums are fp32 and in an order that the sizes, and of packed sequences the offsets, decide.  Sigmoids are those of the hardware's exponential and reciprocal: within (|g| + 16) 2^-24 of their value, and
 * zero in the place of one under 2^-126.
 *
 * Short convolution.  Causal and per channel, with W taps (2, 3 or 4; the last one meets the present row): with X_t the sequence's rows, in front of its first row those of
 * initial_state (zeros where there is none),
 *
 *     z_t = bias + sum_{j < W} weight_j X_{t-W+1+j} ,    y = z , or SiLU(z) = z sigmoid(z)
 *
 * x is dense [B, L, C] or packed [L, C] with cu_seqlens, as q above; weight [C, W], bias [C] or NULL, states [N, W - 1, C] (the last W - 1 rows of X, oldest first, which continue the
 * sequence in another call), all of type dtype: a state is a copy of rows, not a sum.  The C channels are one to three parts (q, k and v side by side in a projection's output, say), each
 * with an output of its own, [.., width] contiguous, and activated or not.  cu_seqlens_host is optional and validated if given; without it rows that lie in no sequence become zero, in y
 * and in dx, and malformed offsets give meaningless results but no access outside the tensors.
 * final_state may be initial_state itself (generation), otherwise no output may overlap an input.  C <= 2^20, B L <= 2^30.
 */
typedef struct {
    int32_t B, L, C, W;
    int32_t dtype;
    int32_t num_seqs;                /* packed layout only: N */
    const int32_t *cu_seqlens;       /* DEVICE int32 [N + 1], or NULL for the dense layout */
    const int32_t *cu_seqlens_host;  /* optional HOST copy */
    int32_t parts;                   /* 1 to 3 */
    int32_t width[3], silu[3];       /* of each part: channels (a multiple of 16 bytes, C in all), whether SiLU is applied */
    int64_t x_stride, dx_stride;     /* elements between rows; dx_stride: backward only */
} dn_conv_shape;

/* y: HOST array of `parts` device pointers.  final_state may be NULL (not written). */
int deltanet_short_conv_fwd(const dn_conv_shape *shape, const void *x, const void *weight, const void *bias, const void *initial_state,
                            void *const *y, void *final_state, void *hip_stream);

/* Its gradient: from dy (HOST array of `parts` device pointers) and dfinal_state (NULL: zeros), dx and dinitial_state (element type; the latter NULL where not wanted), dweight (fp32
 * [C, W]) and dbias (fp32 [C]; NULL where not wanted, also dweight). */
int deltanet_short_conv_workspace_bytes(const dn_conv_shape *shape, size_t *out_bytes);
int deltanet_short_conv_bwd(const dn_conv_shape *shape, const void *x, const void *weight, const void *const *dy, const void *bias,
                            const void *initial_state, const void *dfinal_state, void *dx, float *dweight, float *dbias,
                            void *dinitial_state, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Output norm.  Per token and head, with o a row of the mixer's output, g its gate's row and w a weight of d elements (NULL: ones),
 *
 *     y = o / sqrt(mean(o^2) + eps) * w * act(g) ,    act(g) = g sigmoid(g) or sigmoid(g)    (gate NULL: no such factor)
 *
 * o, gate and dgate are [T, H, d] with their strides between tokens, y, dy and d_o contiguous.  d = 32, 64, 128, 256 in fp32 and bf16; T <= 2^30, T * H < 2^31.
 * Backward: d_o and dgate (element type; NULL where there is no gate), dweight (fp32 [d]; NULL where not wanted).  d_o may take the place of dy, and y that of a contiguous o.
 */
typedef enum { DN_ACT_SILU = 1, DN_ACT_SIGMOID = 2 } dn_act;
typedef struct {
    int32_t T, H, d;
    int32_t dtype, act;              /* act: dn_act */
    float eps;                       /* finite, >= 0 */
    int64_t o_stride, gate_stride, dgate_stride; /* the latter two: where there is a gate; dgate_stride: backward only */
} dn_out_norm_shape;
int deltanet_out_norm_fwd(const dn_out_norm_shape *shape, const void *o, const void *gate, const void *weight, void *y, void *hip_stream);
int deltanet_out_norm_workspace_bytes(const dn_out_norm_shape *shape, size_t *out_bytes);
int deltanet_out_norm_bwd(const dn_out_norm_shape *shape, const void *o, const void *dy, const void *gate, const void *weight, void *d_o,
                          void *dgate, float *dweight, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Block norm.  What stands between two blocks: the branch x that a block adds to the residual stream, its own norm (post_norm) and gate u per channel (NULL: ones), the sum, and the norm
 * in front of the next block, with weight w (NULL: ones),
 *
 *     h = residual_scale * residual + scale * u * m ,  m = x , or x / sqrt(mean(x^2) + eps) ;    y = h / sqrt(mean(h^2) + eps) * w
 *
 * for T rows of D elements.  x, y, the vectors and their rows' gradients dy, dx are of type dtype; residual, h, dh and dresidual of stream_dtype (dtype, or DN_F32 for bf16 tensors).  y comes from
 * the sum before it is rounded to h.  residual may be NULL (zeros), and h (not written).  D: a multiple of 8, at most 8192; T <= 2^30.
 * Backward, from dy, dh (NULL: zeros), the h that the forward call left and (with post_norm or a gate) x: dx, dresidual, dweight and dgate (fp32 [D]), each NULL where not wanted.  A
 * row's outputs may take the place of an input row of the same type and layout (y of x, h of residual, dx of dy, dresidual of dh).
 */
typedef struct {
    int32_t T, D;
    int32_t dtype, stream_dtype;
    int32_t post_norm;
    float scale, residual_scale;     /* finite */
    float eps;                       /* finite, >= 0 */
    int64_t x_stride, residual_stride;
} dn_block_norm_shape;
int deltanet_block_norm_fwd(const dn_block_norm_shape *shape, const void *x, const void *residual, const void *weight, const void *gate,
                            void *y, void *h, void *hip_stream);
int deltanet_block_norm_workspace_bytes(const dn_block_norm_shape *shape, size_t *out_bytes);
int deltanet_block_norm_bwd(const dn_block_norm_shape *shape, const void *dy, const void *dh, const void *h, const void *x,
                            const void *weight, const void *gate, void *dx, void *dresidual, float *dweight, float *dgate,
                            void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Measurement aid (not part of the method): per-kernel device time.  After
 * deltanet_profile_enable(1), every kernel launch of deltanet_fwd / deltanet_bwd is bracketed by a
 * pair of HIP events recorded on the launch stream.  deltanet_profile_collect waits for those
 * events, sums the elapsed milliseconds per kernel name into `out` (at most max_entries distinct
 * kernels; HOST memory), stores the number of entries and forgets the records.  Events cost a few
 * microseconds per launch, so whole-pass timings should be taken with profiling disabled.
 */
typedef struct {
    char name[96];    /* kernel name with its template arguments, as written in the source */
    double total_ms;  /* summed device time between the two events */
    int32_t launches;
} dn_kernel_time;
int deltanet_profile_enable(int on);
int deltanet_profile_collect(dn_kernel_time *out, int max_entries, int *num_entries);

/*
 * Process-wide options (each 0 by default).
 *  DN_OPT_STREAMED_CHUNK_KERNEL: accepted and without effect.  It chose a chunk kernel that read the chunk states in
 *    blocks of state columns; the one chunk kernel there is now does that for every rule, type and head size.
 *    Unknown options return DN_ERR_UNSUPPORTED.
 */
typedef enum { DN_OPT_STREAMED_CHUNK_KERNEL = 0 } dn_option;
int deltanet_set_option(int option, int value);

/*
 * Measurement aid (not part of the method): one launch of a probe kernel that repeats, `iters` times, ONE of the LDS
 * access patterns the kernels are built from (pattern 0..17: operand-fragment reads in both storage orders, accumulator
 * and register tiles written to LDS, row-segment reads; the list is in csrc/dn_lds_probe.hip), so that a profiler's LDS
 * counters can be read per pattern.  256 workgroups of 512 threads, no global memory traffic.  iters in [0, 2^20];
 * DN_ERR_UNSUPPORTED for an unknown pattern.  The launch is enqueued on hip_stream.
 */
int deltanet_lds_probe(int pattern, int iters, void *hip_stream);

/* Static, NUL-terminated description of a dn_status value. */
const char *deltanet_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* DELTANET_H_ */
