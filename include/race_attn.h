/*
 * race_attn.h - C ABI of the MI355X (gfx950) RACE Attention library.
 *
 * RACE Attention (arXiv 2510.04008) replaces softmax attention by a linear-time estimator
 * of sharpened angular-kernel attention.  For every head, L independent tables each draw
 * P Gaussian hyperplanes; a query or key x is softly assigned to the R = 2^P corners of
 * the hypercube, phi_r(x) = softmax_r(beta * tanh(W x) . v_r)  (Algorithm 1, steps 2-4);
 * keys and values are accumulated into per-table bucket statistics A = Phi_K^T 1 and
 * B = Phi_K^T V (step 5); every query reads them back, Num = (1/L) sum_l Phi_Q B,
 * Den = (1/L) sum_l Phi_Q A, O = Num / Den (steps 7-8).  The causal variant
 * (Algorithm 2, appendix "Causal RACE Attention") lets query t read the statistics of
 * keys 1..t only (inclusive: token t is added before it reads).
 *
 * Conventions common to all entry points
 *   - Tensors Q, K, V, O, dO, dQ, dK, dV are DEVICE pointers to (B, H, N, d) arrays,
 *     row-major with d contiguous, of the element type named by desc->dtype.
 *     den is a DEVICE pointer to (B, H, N) float.  Buffers must not overlap.
 *   - proj_seeds is a HOST pointer to H 64-bit seeds, one per head, read during the call.
 *     W is shared by the batch.  Head h uses the (L*P, d) matrix whose row l*P+t is
 *     hyperplane t of table l, drawn i.i.d. N(0,1) (Algorithm 1, step 2) by the generator
 *     documented at race_attn_expand_projection().
 *   - Corner r of the hypercube has v_{r,t} = +1 iff bit t of r is set (t = 0 is the least
 *     significant bit and belongs to row l*P+0 of W).
 *   - sharpening is the temperature beta of Algorithms 1/2.  Q and K are used as given:
 *     no 1/sqrt(d) scaling happens inside the layer, and no normalisation unless desc->unit_qk
 *     asks for it.  With unit_qk = 1 every entry point that hashes rows of Q or K (passes, taps,
 *     state_init, step) uses x / max(|x|, 1e-12) in place of the row x, in fp32 from the stored
 *     elements; the backward passes carry the chain rule through that map, (I - xhat xhat^T) / |x|.
 *     beta = +infinity selects the hard hash h(x) = sign(W x) that Section 3.3 starts from
 *     (bit t of the bucket is [<w_t, x> >= 0]; counters instead of soft masses), for inference:
 *     the forward pass, the taps and incremental decoding accept it, the backward passes return
 *     RACE_ERR_UNSUPPORTED (the hard hash is piecewise constant).  A query all of whose buckets
 *     are empty has den = 0 and gets O = 0 (non-causal only; the soft layer never has den = 0).
 *   - The caller owns every buffer, including the workspace (device memory, 256-byte
 *     aligned, at least race_attn_workspace_bytes() bytes; contents are scratch).  The
 *     library allocates no device memory, never synchronises the stream and launches all
 *     work on the given stream.  Calls that share a workspace must be stream-ordered.
 *   - The host keeps one pinned image of the packed W per distinct (proj_seeds, H, d, L, P, dtype) for the life of
 *     the process (asynchronous copies and captured graphs may read it at any time; a few KB to ~100 KB each).
 *     The 4097th distinct combination in one process is refused with RACE_ERR_HIP.
 *   - Every argument is checked before anything is launched; on any error status other
 *     than RACE_ERR_HIP the outputs are untouched.  N == 0 is a valid no-op.
 *   - Arithmetic: products of bf16 operands are accumulated in fp32; the fp32 element
 *     type computes in fp32 throughout.
 *   - Infinities and NaNs: a non-finite element of V reaches the outputs of the tokens that read it, a non-finite element of dO
 *     the gradients of the tokens its row depends on; in the causal case the generic kernels (race_attn_kernel_family() == 1)
 *     keep it to those, the bf16 MFMA kernels may spread it over the other tokens of its tile (32 tokens from a multiple of 32
 *     within a segment).  With a non-finite element in Q or K a token's assignments are arbitrary but finite; its own row's
 *     gradient (and dbeta) is not.
 */
#ifndef RACE_ATTN_H
#define RACE_ATTN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RACE_OK = 0,
    RACE_ERR_INVALID_ARG = 1, /* null pointer, non-positive size, non-finite beta, bad enum   */
    RACE_ERR_UNSUPPORTED = 2, /* a valid shape outside what the kernels were built for         */
    RACE_ERR_WORKSPACE = 3,   /* workspace null, misaligned or smaller than required           */
    RACE_ERR_HIP = 4,         /* a HIP call failed; text from race_attn_last_error()           */
    RACE_ERR_NOT_READY = 5    /* a call that prepares this one has not been made (see the entry
                                 point); text from race_attn_last_error()                       */
} race_status_t;

typedef enum { RACE_F32 = 0, RACE_BF16 = 1 } race_dtype_t;

/* ABI-identical to hipStream_t (a pointer to HIP's opaque stream object); 0 = default stream. */
typedef struct ihipStream_t *race_stream_t;

/* Problem statement of Algorithms 1/2: inputs Q, K, V in R^{N x d}, L tables, P hyperplanes,
 * temperature beta; batched over (B, H). */
typedef struct {
    int32_t B, H;     /* batch, heads (>= 1)                                                   */
    int64_t N;        /* tokens per sequence (>= 0)                                            */
    int32_t d;        /* head dimension: multiple of 8, 8 <= d <= 256                          */
    int32_t L, P;     /* tables (>= 1), hyperplanes per table (1..8); R = 1 << P               */
    float sharpening; /* beta > 0; +infinity = hard hash (forward only)                        */
    int32_t causal;   /* 0: Algorithm 1 (all keys); 1: Algorithm 2 (keys j <= i)               */
    int32_t dtype;    /* race_dtype_t of Q, K, V, O, dO, dQ, dK, dV                            */
    int64_t chunk;    /* tokens per scan segment: the sequence is cut into segments whose
                         bucket statistics are combined by a prefix scan; 0 = choose           */
    int32_t unit_qk;  /* 0: Q and K enter the projection as given (Algorithm 1, step 4);
                         1: every row of Q and K is first divided by its Euclidean norm, the
                         setting |Q_i| = |K_j| = 1 of Theorem 1's proof (Appendix, "Setup and
                         assumptions"); dQ and dK are then the cotangents of the rows as given  */
} race_attn_desc_t;

/* Bytes of device workspace that race_attn_fwd / race_attn_bwd / race_attn_debug_buckets need
 * for this descriptor (one figure covers all three).  Returns 0 for an invalid or unsupported
 * descriptor (and for N == 0). */
size_t race_attn_workspace_bytes(const race_attn_desc_t *desc);

/* Forward pass, Algorithm 1 (causal == 0) or Algorithm 2 (causal == 1).
 * in : Q, K, V (device), proj_seeds (host, H entries)
 * out: O (device, same type as V), den (device, float (B,H,N)): Den_i including the 1/L of
 *      Algorithm 1 step 7; the backward pass needs O and den. */
race_status_t race_attn_fwd(const race_attn_desc_t *desc, const void *Q, const void *K, const void *V,
                            const uint64_t *proj_seeds, void *O, float *den,
                            void *workspace, size_t workspace_bytes, race_stream_t stream);

/* For callers that cannot allocate (code under HIP graph capture, tight serving loops, harnesses that forbid
 * hipMalloc): race_attn_fwd without a workspace argument.  The kernels are race_attn_fwd's; their scratch (the
 * packed W, the per-segment bucket statistics, the hashed rows) lives in an array of 48 MiB that is part of the library's code
 * object, one copy per GPU, held until the process ends.  The call allocates nothing, on the host or on the device.
 *   - Size limit: 32 MiB, counted as W, one segment's statistics per (batch, head) and per token and head the hashed rows of
 *     Q and K; beyond it RACE_ERR_WORKSPACE.  At d = 128, L = 8, P = 6 (bf16) the statistics take 258 KiB and the hashed
 *     rows 384 bytes: B*H*(258 KiB + N * 384 B) < 32 MiB.  The generic kernels are charged two sets of statistics and
 *     12*L*d bytes per token and head.  Within the limit, the sequence is cut into fewer, longer scan segments
 *     (desc->chunk doubled as often as needed) where race_attn_fwd's own would not fit the array; O and den then differ
 *     from race_attn_fwd's by the rounding of a different summation order only.
 *   - The pinned host image of W for (proj_seeds, shape) must exist already, because making it allocates: any
 *     earlier call of another entry point with the same H, d, L, P, dtype and proj_seeds (race_attn_fwd,
 *     race_attn_debug_hash, ...) leaves it in the library's host cache for the life of the process.  Otherwise
 *     RACE_ERR_NOT_READY, and nothing is launched.
 *   - All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (different streams or
 *     threads) race; stream-ordered calls are fine.  Nothing in the array needs clearing between calls (every
 *     element read by a kernel has been written earlier in the same call).
 * Everything else (arguments, outputs, errors) is as for race_attn_fwd.  There is no race_attn_bwd_saved on this
 * scratch: the next call overwrites it. */
race_status_t race_attn_fwd_static(const race_attn_desc_t *desc, const void *Q, const void *K, const void *V,
                                   const uint64_t *proj_seeds, void *O, float *den, race_stream_t stream);

/* Backward pass of the same operator: given dO = d(loss)/dO, O and den from race_attn_fwd on the
 * same inputs, writes dQ, dK, dV.  The paper trains through the differentiable soft assignment
 * (Section 3.3) and prints no gradient; the formulas are the chain rule through Algorithms 1/2:
 * read-out, bucket accumulation (a suffix scan in the causal case), corner softmax, tanh and W.
 * W is a fixed random matrix and gets no gradient. */
race_status_t race_attn_bwd(const race_attn_desc_t *desc, const void *Q, const void *K, const void *V,
                            const void *O, const float *den, const void *dO,
                            const uint64_t *proj_seeds, void *dQ, void *dK, void *dV,
                            void *workspace, size_t workspace_bytes, race_stream_t stream);

/* The same backward pass, which also returns the cotangent of the temperature: the paper's experiments train
 * beta (Section 4), and with W fixed and random it is the layer's only parameter.  The corner logits of Algorithm 1, step 4 are beta * (tanh(W x) . v_r), so
 * d(loss)/d(beta) = sum over Q and K tokens, tables and corners of dlogit_r * (tanh(W x) . v_r).
 * dbeta: DEVICE float (B, H), one partial derivative per (batch, head), written (not accumulated); the
 * derivative with respect to a beta shared by all of them is the sum of the entries.  NULL = not wanted, which
 * makes this call identical to race_attn_bwd.  Sums are formed in a fixed order (bit-reproducible).  Needs no
 * more workspace than race_attn_bwd.  N == 0 writes nothing. */
race_status_t race_attn_bwd_beta(const race_attn_desc_t *desc, const void *Q, const void *K, const void *V,
                                 const void *O, const float *den, const void *dO,
                                 const uint64_t *proj_seeds, void *dQ, void *dK, void *dV, float *dbeta,
                                 void *workspace, size_t workspace_bytes, race_stream_t stream);

/* The backward pass for a caller that kept the forward's workspace.  race_attn_fwd leaves in the workspace what
 * the backward pass would otherwise derive again from Q, K and V: the packed W, the hashed rows of Q and K (one
 * float per token, table and hyperplane: all that the soft assignment of Algorithm 1, step 4 depends on) and the
 * key/value bucket statistics (A, B of Algorithm 1, step 5; in the causal case Algorithm 2's running statistics at
 * the start of every scan segment).  This entry point reads them instead of recomputing them: one projection pass
 * over Q and K and one accumulation pass over K and V fewer.
 * Contract: `workspace` is the buffer that the last race_attn_fwd with the same desc, Q, K, V and proj_seeds wrote,
 * nothing has written to it since, and this call is stream-ordered after that forward.  A workspace that does not
 * hold that forward's data gives wrong gradients, never an out-of-bounds access.  Arguments, outputs, dbeta
 * (may be NULL) and error behaviour are those of race_attn_bwd_beta, whose results it reproduces bit for bit.
 * Both kernel families keep them. */
race_status_t race_attn_bwd_saved(const race_attn_desc_t *desc, const void *Q, const void *K, const void *V,
                                  const void *O, const float *den, const void *dO,
                                  const uint64_t *proj_seeds, void *dQ, void *dK, void *dV, float *dbeta,
                                  void *workspace, size_t workspace_bytes, race_stream_t stream);

/* Host-only: expands the seeds into W_host (HOST, float, (H, L*P, d)), the values the kernels
 * multiply with (Algorithm 1, step 2).  Generator: element e = row*d + col of head h is Gaussian
 * number (e mod 4) of block e/4 of Philox-4x32-10 with key = (low, high) 32 bits of the head's
 * seed and counter = (block low, block high, 0, 0); the block's words (x0,x1,x2,x3) give
 * Box-Muller pairs from (x0,x1) and (x2,x3) with u = (x + 0.5) / 2^32, evaluated in fp64:
 * sqrt(-2 ln u1) * (cos, sin)(2 pi u2); rounded to fp32 (nearest even), and for RACE_BF16 once
 * more to bf16 (nearest even, returned widened to float).  Only H, L, P, d, dtype of desc are used. */
race_status_t race_attn_expand_projection(const race_attn_desc_t *desc, const uint64_t *proj_seeds,
                                          float *W_host);

/* Debug tap of the projection and soft assignment (Algorithm 1, steps 2-4) of one tensor X (Q or K):
 * codes (device, uint8 (B,H,N,L)): bit t = [<w_t, x> >= 0], i.e. the hard hash sign(W x) of
 * Section 3.3, which is also the arg-max corner of phi;  phi (device, float (B,H,N,L,R)) or NULL.
 * Runs the projection arithmetic of the production kernels.  Needs no workspace beyond
 * H*L*P*d floats + 256 bytes. */
race_status_t race_attn_debug_hash(const race_attn_desc_t *desc, const void *X, const uint64_t *proj_seeds,
                                   uint8_t *codes, float *phi,
                                   void *workspace, size_t workspace_bytes, race_stream_t stream);

/* Debug tap of the bucket statistics of Algorithm 1, step 5, over all N keys (whatever causal
 * says): A (device, float (B,H,L,R)) and Bsum (device, float (B,H,L,R,d)). */
race_status_t race_attn_debug_buckets(const race_attn_desc_t *desc, const void *K, const void *V,
                                      const uint64_t *proj_seeds, float *A, float *Bsum,
                                      void *workspace, size_t workspace_bytes, race_stream_t stream);

/* ---- Incremental decoding: the bucket statistics as the carried state (Algorithm 2, one loop iteration per
 * call).  The state plays the part of a key/value cache whose size does not grow with the context:
 * state = DEVICE float (B, H, L, R, d+1), row-major; per bucket row the d sums of phi_K * V (B of Algorithm 1,
 * step 5) followed by the mass (A).  The caller owns it; a zero-filled state is the empty context. */

/* Bytes of one state for this descriptor (B, H, d, L, P are used); 0 for an invalid descriptor. */
size_t race_attn_state_bytes(const race_attn_desc_t *desc);

/* Prefill: state <- statistics of the desc->N keys and values in K, V (DEVICE (B, H, N, d) of desc->dtype);
 * N == 0 zero-fills it.  Workspace as for race_attn_fwd (race_attn_workspace_bytes; none needed for N == 0). */
race_status_t race_attn_state_init(const race_attn_desc_t *desc, const void *K, const void *V,
                                   const uint64_t *proj_seeds, float *state,
                                   void *workspace, size_t workspace_bytes, race_stream_t stream);

/* Bytes of device workspace race_attn_step needs (independent of desc->N). */
size_t race_attn_step_workspace_bytes(const race_attn_desc_t *desc);

/* One new token per (batch, head): q, k, v are DEVICE (B, H, d) rows of desc->dtype.  The state is updated in
 * place with (k, v) first, then q reads it (the loop body of Algorithm 2): o (DEVICE (B, H, d), desc->dtype) and
 * den (DEVICE float (B, H), with the 1/L of Algorithm 1 step 7).  desc->N, desc->causal and desc->chunk are
 * ignored.  Arithmetic is fp32 on the values as given.  Cost O(L R d) per token and head; one kernel launch.
 * The call expands proj_seeds into the workspace (a copy from pinned host memory) and leaves W and cleared arrival counters
 * there: a later step with the same desc, except that B may be another (the workspace must be large enough for it), on a
 * workspace nobody else has written to since may pass proj_seeds = NULL and skips the copy. */
race_status_t race_attn_step(const race_attn_desc_t *desc, const void *q, const void *k, const void *v,
                             const uint64_t *proj_seeds, float *state, void *o, float *den,
                             void *workspace, size_t workspace_bytes, race_stream_t stream);

/* ---- The gated delta rule: a second linear-time layer with a carried state, for models that hold layers of both kinds.
 * Per value head, with decay a_t = exp(g_t) and write strength b_t = beta_t, from the state S_0 in R^{dk x dv}:
 *     S_t = a_t S_{t-1} + k_t b_t (v_t - a_t S_{t-1}^T k_t)^T,     o_t = scale * S_t^T q_t.
 * Conventions
 *   - Q, K, dQ, dK are DEVICE (B, Hk, N, dk), V, O, dO, dV DEVICE (B, H, N, dv) arrays, row-major, of the element type desc->dtype;
 *     g, beta, dg, dbeta are DEVICE float (B, H, N); states are DEVICE float (B, H, dk, dv).  Value head h reads the queries and keys of
 *     head h / (H / Hk); their gradients are summed over the value heads that share them.
 *   - g is the logarithm of the decay, usually <= 0; -infinity (every value below -1e5) empties the state before the token is written.  beta is
 *     used as given (0 where |beta| < 2^-100).  Rows of Q and K are used as given: a bounded state wants |k| <= 1 with beta in [0, 2] (race_qk_rotary_fwd makes such rows).
 *   - A padding token is one with g = 0 and beta = 0: the state passes it unchanged, whatever its rows of K and V hold, as long as it is finite, and so do the other tokens'
 *     outputs and, where its dO is 0, gradients.  Its own output reads the state with its query, whose products with keys and states have to stay finite.
 *     Its rows of dK and dV are 0; its dbeta is what the formula makes of its rows.
 *   - Chunks of 64 tokens are worked on at once; state, sums and decays are held in fp32 (decays are summed in fp64; a sum over part of 64 tokens has to stay
 *     below 88, where exp leaves fp32).  The bf16 type multiplies fp32 values as sums of three bf16, all 24 bits; O, dQ, dK and dV are rounded to bf16 at the end.
 *   - A non-finite element of Q, K, V or dO reaches what depends on it, and may spread over the 64 tokens of its chunk, for bf16 and
 *     fp32 alike; it does not reach another head or sequence (Q, K: other than those that share them).  (The dbeta of a token of strength zero may stay finite: what its
 *     key makes of cotangents is cut off at 2^60.)
 *   - Pointers need be aligned to their elements only.  Buffers must not overlap, except that a state may be carried in place: state_out
 *     may be state_in, dstate_in may be dstate_out.
 *   - Everything else (workspace, streams, errors, capture into a graph) as above.  Results are the same bits every time. */
typedef struct {
    int32_t B, H, Hk; /* batch, value heads, heads of queries and keys (H a multiple of Hk); B * H up to 65535 */
    int64_t N;        /* tokens per sequence (>= 0); B * H * N up to 2^36                               */
    int32_t dk, dv;   /* multiples of 8, 8 .. 128.  (A wider value row: two value heads of half of it, with the same g, beta and shared q, k) */
    float scale;      /* of the outputs, finite                                                         */
    int32_t dtype;    /* race_dtype_t                                                                   */
    int64_t chunk;    /* tokens per scan segment, rounded up to whole chunks; 0 = choose                */
} race_delta_desc_t;

/* Bytes of device workspace of race_delta_fwd and of race_delta_bwd.  0 for an invalid or unsupported descriptor and for N == 0.
 * A long sequence is worked on in windows of at most 4 GiB, which follow one another in the same memory, but no window is less than one segment of every head: with
 * desc->chunk = N all of the sequence's chunks of 64 tokens are held at once (dk = dv = 128: 17 KB each, backward 0.26 MB, with shared heads 0.32 MB).  What is held of
 * every segment of the sequence is one state a head, backward also its transition (dk = 128: 64 KB). */
size_t race_delta_workspace_bytes(const race_delta_desc_t *desc);
size_t race_delta_bwd_workspace_bytes(const race_delta_desc_t *desc);
/* Bytes of one state (B, H, dk, dv are used); 0 for an invalid descriptor. */
size_t race_delta_state_bytes(const race_delta_desc_t *desc);
/* Tokens per scan segment that race_delta_fwd uses for this descriptor (race_delta_bwd chooses its own with chunk = 0: its windows hold fewer chunks).
 * Informational.  0 = invalid. */
int64_t race_delta_segment_tokens(const race_delta_desc_t *desc);

/* Forward pass.  state_in: state before the first token, NULL = zero.  state_out: state behind the last token, NULL = not wanted.
 * N == 0: state_out is state_in. */
race_status_t race_delta_fwd(const race_delta_desc_t *desc, const void *Q, const void *K, const void *V, const float *g, const float *beta,
                             const float *state_in, void *O, float *state_out, void *workspace, size_t workspace_bytes,
                             race_stream_t stream);

/* Backward pass on the forward pass's inputs (it needs nothing that the forward pass left behind).  dstate_out: cotangent of state_out,
 * NULL = zero.  dstate_in: cotangent of state_in, NULL = not wanted.  N == 0: dstate_in is dstate_out. */
race_status_t race_delta_bwd(const race_delta_desc_t *desc, const void *Q, const void *K, const void *V, const float *g, const float *beta,
                             const float *state_in, const void *dO, const float *dstate_out, void *dQ, void *dK, void *dV, float *dg,
                             float *dbeta, float *dstate_in, void *workspace, size_t workspace_bytes, race_stream_t stream);

/* One token per sequence: q, k DEVICE (B, Hk, dk), v, o DEVICE (B, H, dv), g, beta DEVICE float (B, H); the state is updated in place and then read.
 * desc->N and desc->chunk are ignored.  One kernel, no workspace. */
race_status_t race_delta_step(const race_delta_desc_t *desc, const void *q, const void *k, const void *v, const float *g, const float *beta,
                              float *state, void *o, race_stream_t stream);

/* ---- Rows of queries and keys for the layers above: norm for each head and position rotation in one pass.
 * The row x (d elements) of a token and head becomes rotate(x * r * w), r = 1 / sqrt(mean x^2 + eps) (RACE_NORM_RMS), 1 / sqrt(sum x^2 + eps)
 * (RACE_NORM_L2) or 1; rotate turns pair i = 0 .. rot/2 - 1 of the first rot elements, (x_i, x_{i + rot/2}) or with
 * neighbours = 1 (x_{2i}, x_{2i+1}), by the angle position * inv_freq[i]: (m cos - n sin, n cos + m sin).
 *   - The rows as given are read where they lie, e.g. in the output (B, N, heads * d) of a fused projection: element e of the row of (b, n, head) is
 *     at b * strides[0] + n * strides[1] + head * strides[2] + e.  Q and K are contiguous (B, Hq, N, d) and (B, Hk, N, d), as the layers take them.
 *   - wq, wk: DEVICE float (d), NULL = ones.  inv_freq: HOST, rot/2 finite doubles, read during the call.  positions: DEVICE int64 (B, N), NULL =
 *     pos0 + n.  Angles are formed in fp64.
 *   - Arithmetic is fp32, rounded once to desc->dtype.  A non-finite element spreads over its own row.  Pointers need be aligned to their elements only. */
typedef enum { RACE_NORM_NONE = 0, RACE_NORM_RMS = 1, RACE_NORM_L2 = 2 } race_norm_t;
typedef struct {
    int32_t B, Hq, Hk;     /* batch, heads of queries (>= 1) and keys (>= 0), Hq + Hk up to 65535             */
    int64_t N;             /* tokens per sequence (>= 0); B * N up to 2^31                                    */
    int32_t d, rot;        /* row: multiple of 8, 8 .. 256; rotated elements: even, 0 .. d                    */
    int32_t norm;          /* race_norm_t                                                                     */
    int32_t neighbours;    /* 0: pairs (i, i + rot/2), 1: pairs (2i, 2i + 1)                                  */
    float eps;             /* >= 0, finite                                                                    */
    int32_t dtype;         /* race_dtype_t of rows, Q, K and their cotangents                                 */
    int64_t pos0;          /* position of token 0 where positions is NULL: pos0 + N up to 2^63 - 1            */
    int64_t q_strides[3], k_strides[3];    /* batch, token, head of the rows as given, elements, >= 0         */
    int64_t dq_strides[3], dk_strides[3];  /* the same of their cotangents (backward only): rows must not overlap */
} race_rotary_desc_t;

/* k, K, wk may be NULL with Hk = 0. */
race_status_t race_qk_rotary_fwd(const race_rotary_desc_t *desc, const void *q, const void *k, const float *wq, const float *wk,
                                 const double *inv_freq, const int64_t *positions, void *Q, void *K, race_stream_t stream);

/* Backward pass: dq, dk from dQ, dK and the rows as given.  dwq, dwk (DEVICE float (d)): NULL = not wanted; sums in a fixed
 * order.  Workspace: race_qk_rotary_workspace_bytes(), needed only with dwq or dwk. */
size_t race_qk_rotary_workspace_bytes(const race_rotary_desc_t *desc);
race_status_t race_qk_rotary_bwd(const race_rotary_desc_t *desc, const void *q, const void *k, const float *wq, const float *wk,
                                 const double *inv_freq, const int64_t *positions, const void *dQ, const void *dK, void *dq, void *dk,
                                 float *dwq, float *dwk, void *workspace, size_t workspace_bytes, race_stream_t stream);

/* Static, never-null description of a status code. */
const char *race_status_string(race_status_t status);

/* Text of the most recent failure that has one, as seen by the calling thread ("" if none): the HIP error behind
 * RACE_ERR_HIP, the reason for RACE_ERR_NOT_READY, the limit behind race_attn_fwd_static's RACE_ERR_WORKSPACE. */
const char *race_attn_last_error(void);

/* Which kernel family a descriptor is served by: 0 = invalid/unsupported, 1 = generic fp32-math
 * kernels, 2 = bf16 MFMA kernels.  Informational (benchmarks and tests report it).
 * The generic kernels serve fp32 tensors and every bf16 shape without an MFMA instantiation (P = 8: d <= 152); they are not a long-context
 * path, and a descriptor with 3 * B*H*L*N*d floats beyond 16 GiB is RACE_ERR_UNSUPPORTED (e.g. fp32, d = 64, L = 4: B*H*N
 * beyond 5.6 million).
 * Test switch: with RACE_ATTN_FORCE_GENERIC=1 in the environment every descriptor is planned on the generic kernels
 * (the tests use it to run one problem on both families; it is read at every call). */
int race_attn_kernel_family(const race_attn_desc_t *desc);

/* Tokens per scan segment the library uses for this descriptor (desc->chunk rounded to what the kernels take, or
 * the library's own choice for chunk = 0): segment s covers tokens [s * len, min(N, (s + 1) * len)), and the
 * statistics at segment boundaries are what the prefix scan of Algorithm 2's cumulative arrays hands from one
 * workgroup to the next.  Informational (tests place their windows across these boundaries).  0 = invalid. */
int64_t race_attn_segment_tokens(const race_attn_desc_t *desc);

/* Benchmark aid (no passage of the paper; callers: benchmarks and profilers).  While enabled for the
 * calling thread, every kernel the library launches is bracketed by a pair of HIP events recorded on the
 * call's own stream.  race_attn_profile_read() waits for the recorded events, adds up the elapsed time per
 * kernel name since the previous read, writes up to max_entries results (names are static strings, total_ms
 * in milliseconds, launches = number of launches) and returns how many distinct kernels ran.  Enabling
 * creates HIP events (host allocations); results are discarded by disabling. */
void race_attn_profile_enable(int on);
int race_attn_profile_read(int max_entries, const char **names, float *total_ms, int *launches);

/* Benchmark aid (no passage of the paper; callers: counter calibration).  Copies `bytes` bytes (a multiple
 * of 16) from src to dst (DEVICE pointers, 16-byte aligned, not overlapping) with one plain grid-stride kernel
 * named calibration_copy_kernel that reads every byte once and writes every byte once: a dispatch of known HBM
 * traffic against which hardware byte counters of the other kernels are scaled.  bytes == 0 is a no-op. */
race_status_t race_attn_calibration_copy(void *dst, const void *src, size_t bytes, race_stream_t stream);

/* Benchmark aid (no passage of the paper; callers: benchmarks that report the attainable matrix rate next to the
 * published peak).  Launches calibration_mfma_kernel: `workgroups` workgroups of 256 threads, each wavefront
 * issuing `iters` rounds of four independent v_mfma_f32_32x32x16_bf16 on register operands, i.e.
 * workgroups * 4 * iters * 4 * 32768 floating-point operations in all; every lane then stores one float to
 * sink (DEVICE, workgroups * 256 floats) so that the work cannot be optimised away.  vector_ops (0, 4, 8 or 16):
 * that many independent v_mul_f32 on registers of the same wavefront follow every matrix instruction, which
 * measures how much vector work the matrix pipeline hides (the flop count returned by the binding counts the
 * matrix instructions only).  workgroups and iters must be in 1 .. 2^20. */
race_status_t race_attn_calibration_mfma(int workgroups, int iters, int vector_ops, float *sink, race_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* RACE_ATTN_H */
