/*
 * arl2.h -- C ABI of the MI355X (gfx950) library for the ARL^2 hybrid attention step
 * of "Attend Locally, Remember Linearly" (paper Sec. 3.2, Sec. 3.3, Alg. 1).
 *
 * Two operations make up the step:
 *
 *   arl2_hybrid_attn_fwd   one read-only denoising pass:
 *                            out = softmax(q k^T * sm_scale) v  +  g * L2Norm(q) S
 *                          (intra-chunk softmax branch Eq. (2); feature map Eq. (3);
 *                           linear readout of the shared pre-update state Eq. (5), (7);
 *                           headwise gate broadcast over the head dimension Eq. (6)).
 *                          S is never written by this call (Sec. 3.3, clean-pass update).
 *
 *   arl2_state_commit      once per chunk, after the last denoising pass:
 *                            S <- gate * S + sum_i L2Norm(k_i)^T v_i
 *                          (Eq. (4) with beta = 1 and without the delta-correction term;
 *                           the gate multiplies the old state only).
 *
 *   arl2_state_commit_delta the same update with Eq. (4)'s delta-correction term and learning rate.
 *
 *   arl2_state_commit_gdn  Eq. (4) applied token by token in order, with per-token gates.
 *
 *   arl2_feature_map       the learned per-head maps and RoPE of Eq. (3) for the linear branch;
 *   arl2_hybrid_attn_fwd_ex  the readout pass with the linear branch's own query;
 *   arl2_hybrid_attn_fwd_fm  the readout pass that computes that query itself (fused feature map);
 *   arl2_gate_proj         the gate G = sigmoid(x W_g) of Eq. (6): headwise, one per token or element-wise.
 *
 *   arl2_kv_append, arl2_kv_read, arl2_kv_attn_fwd   for layers that keep softmax over everything generated so far
 *                          (Eq. (1)): a paged key/value cache held in 4 bits, and the attention that reads it.
 *
 *   arl2_scan_fwd, arl2_scan_bwd   the linear branch as a causal recurrence over tokens (Eq. (4) without the correction term,
 *                          every token reading the state that it leaves), and its gradients;
 *   arl2_rope_fwd, arl2_rope_bwd   queries and keys normalised and rotated by positions on several axes, and the gradients.
 *
 * Reading of the feature map: q and k arrive after RoPE, the learned 1x1 maps are
 * the identity, so phi is the L2 normalisation over the head dimension,
 * x / sqrt(sum x^2 + l2_eps), and V' = v.
 *
 * All data pointers are DEVICE pointers owned by the caller, 16-byte aligned and
 * contiguous in the layouts below.  The library never allocates, frees or
 * synchronises: every call validates its arguments on the host (sizes, alignment, overlapping
 * buffers, limits of the kernels), enqueues its kernels on desc->stream and returns.  A call that
 * returns ARL2_ERR_INVALID_ARG, ARL2_ERR_UNSUPPORTED or ARL2_ERR_WORKSPACE has launched nothing.
 * ARL2_ERR_DEVICE reports that the runtime refused a launch: a call made of several kernels
 * (the state commits) may then have enqueued the earlier ones, and S is undefined.
 * The kernels address one stream's k, v (the whole x for arl2_feature_map and arl2_gate_proj) with
 * 32-bit byte offsets: such an array must stay below 2 GiB, larger problems return ARL2_ERR_UNSUPPORTED
 * (fp32 inputs: H and B below 65536 instead).
 *
 * Layouts (row-major):
 *   q, out      [B][Lq ][H][D]   io_dtype
 *   k, v        [B][Lkv][H][D]   io_dtype
 *   g           [B][Lq ][H]      g_dtype, values in [0,1]      (branch-mix gate, Eq. (6); other
 *                                granularities: see arl2_gate_mode)
 *   S           [B][H][D][D]     fp32, S[d_k][d_v]; readout contracts d_k
 *   gate        [B][H]           fp32                          (forget gate alpha, Eq. (4))
 */
#ifndef ARL2_H
#define ARL2_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    ARL2_OK = 0,
    ARL2_ERR_INVALID_ARG = 1,   /* NULL/misaligned pointer, non-positive size, bad enum    */
    ARL2_ERR_UNSUPPORTED = 2,   /* valid request outside what the kernels implement        */
    ARL2_ERR_WORKSPACE = 3,     /* workspace missing or smaller than arl2_workspace_bytes  */
    ARL2_ERR_DEVICE = 4         /* a HIP launch failed; see arl2_last_error()              */
} arl2_status;

typedef enum { ARL2_F32 = 0, ARL2_BF16 = 1 } arl2_dtype;

/* Granularity of the branch-mix gate g of the readout pass.  The paper's gate is headwise (Eq. (6),
 * g of shape [B][Lq][H]); its gate ablation (Tab. 4) also has one gate per output feature
 * (ARL2_GATE_PER_ELEMENT, g of shape [B][Lq][H][D], 16-byte aligned) and a scalar gate, one per token
 * shared by the heads (ARL2_GATE_PER_TOKEN, g of shape [B][Lq]). */
typedef enum { ARL2_GATE_PER_HEAD = 0, ARL2_GATE_PER_ELEMENT = 1, ARL2_GATE_PER_TOKEN = 2 } arl2_gate_mode;

typedef struct {
    int32_t B;            /* independent streams, >= 1                                      */
    int32_t H;            /* heads, >= 1                                                    */
    int32_t Lq;           /* query tokens of the chunk, >= 1                                */
    int32_t Lkv;          /* key/value tokens; must equal Lq when S != NULL or in commit.   */
                          /* Lkv != Lq (any value >= 1) is allowed for pure softmax, S NULL */
    int32_t D;            /* head dimension d_k = d_v: 64 or 128                            */
    int32_t io_dtype;     /* arl2_dtype of q, k, v, out                                     */
    int32_t g_dtype;      /* arl2_dtype of g (ignored when g == NULL)                       */
    float sm_scale;       /* softmax logit scale; 0 selects 1/sqrt(D)   (Eq. (1))           */
    float l2_eps;         /* epsilon inside L2Norm's square root; 0 selects 1e-6            */
    int32_t g_mode;       /* arl2_gate_mode of g; 0 (zero-initialised descriptor) is headwise */
    void *workspace;      /* device scratch for arl2_state_commit, >= arl2_workspace_bytes  */
    size_t workspace_bytes;
    void *stream;         /* hipStream_t; NULL is the default stream                        */
} arl2_desc;

/* Device scratch that arl2_state_commit / arl2_state_commit_delta / arl2_state_commit_fm take for this
 * descriptor (bf16: token-split partial sums; fp32: B * Lq * H * 4 bytes, which have to be given but
 * are not used).  arl2_hybrid_attn_fwd needs none.  Returns 0 for an invalid descriptor.            */
size_t arl2_workspace_bytes(const arl2_desc *desc);

/*
 * Read-only denoising pass (paper Eq. (2), (3), (5), (6), (7); Alg. 1 inner loop).
 *   q, k, v   device, io_dtype, layouts above; not modified.
 *   S         device fp32 [B][H][D][D], READ-ONLY; NULL means a zero state (pure softmax,
 *             used for layers that keep softmax over a KV cache, Eq. (1) with every cached
 *             token visible).
 *   g         device [B][Lq][H]; NULL means a gate of one.
 *   out       device, io_dtype [B][Lq][H][D]; fully overwritten; must not alias an input.
 * bf16 I/O runs on bf16 MFMA with fp32 accumulation and fp32 softmax statistics;
 * fp32 I/O: sums, softmax statistics and the state are fp32.  Small launches multiply fp32 operands; launches
 * that fill the chip take every operand as the sum of two scaled halves (23 of its 24 bits) and a product
 * as three of halves, wherever that is no further from 64-bit arithmetic than fp32 products are; values
 * that two halves do not stand for (infinities, NaN, sizes too far apart) are found and multiplied in fp32.
 * What is not found: single values of a feature of v beside ones more than 2^10 times as large, which are
 * exact to 2^-34 of the largest among the first 128 keys.
 */
arl2_status arl2_hybrid_attn_fwd(const arl2_desc *desc,
                                 const void *q, const void *k, const void *v,
                                 const float *S, const void *g, void *out);

/*
 * The same pass with a query of its own for the linear branch (paper Eq. (3), (5)): the inter branch
 * normalises and multiplies with S the rows of q_lin, e.g. RoPE(phi_q(Q)) written by arl2_feature_map,
 * while the softmax branch keeps q (Eq. (2)).
 *   q_lin     device, io_dtype [B][Lq][H][D]; NULL means q (then this is arl2_hybrid_attn_fwd).
 *             Not read when S is NULL.
 */
arl2_status arl2_hybrid_attn_fwd_ex(const arl2_desc *desc,
                                    const void *q, const void *k, const void *v, const void *q_lin,
                                    const float *S, const void *g, void *out);

/*
 * The readout pass with the query feature map of the linear branch fused in (paper Eq. (2), (3), (5),
 * (6)): the inter branch reads L2Norm(RoPE(Wq[h] xq)), computed inside the kernel and never stored;
 * equal to arl2_feature_map(xq, Wq, ...) followed by arl2_hybrid_attn_fwd_ex, without the intermediate
 * array and the second launch.
 *   q, k, v   as in arl2_hybrid_attn_fwd (the softmax branch's inputs), bf16 only.
 *   xq        device bf16 [B][Lq][H][D]: the projection the feature map acts on (before RoPE).
 *   Wq, rope_cos, rope_sin   as in arl2_feature_map.
 *   S         device fp32 [B][H][D][D], READ-ONLY, must not be NULL (without a state there is no
 *             linear branch: use arl2_hybrid_attn_fwd).
 */
arl2_status arl2_hybrid_attn_fwd_fm(const arl2_desc *desc,
                                    const void *q, const void *k, const void *v,
                                    const void *xq, const void *Wq,
                                    const float *rope_cos, const float *rope_sin,
                                    const float *S, const void *g, void *out);

/*
 * Per-head feature map of the linear branch, paper Eq. (3) without its L2Norm (the readout and the
 * commits normalise the rows they are given):
 *     y[b][l][h][:] = RoPE_l( W[h] x[b][l][h][:] )
 *   x         device bf16 [B][Lq][H][D] (desc->io_dtype must be ARL2_BF16; Lkv is not used).
 *   W         device bf16 [H][D][D], per head the D x D matrix of the grouped 1 x 1 map, indexed
 *             [head][out][in].
 *   rope_cos, rope_sin   device fp32 [Lq][D/2], 8-byte aligned: cosine and sine of the angle by which
 *             the pair (y[2i], y[2i+1]) of token l is rotated, shared by all streams and heads; which
 *             positions and frequencies they encode is the caller's choice.  Both NULL: no rotation
 *             (the value map phi_v).
 *   y         device bf16 [B][Lq][H][D], fully overwritten; must not alias x or W.
 * fp32 accumulation and rotation, one rounding to bf16 on output.
 */
arl2_status arl2_feature_map(const arl2_desc *desc, const void *x, const void *W,
                             const float *rope_cos, const float *rope_sin, void *y);

/*
 * Branch-mix gate, paper Eq. (6): G = sigmoid(x W_g), the g argument of the readout pass.
 *   x         device bf16 [B][Lq][H*D], the layer's hidden state (desc->io_dtype must be ARL2_BF16).
 *   Wg        device bf16 [n][H*D], one row per gate output: n = H for desc->g_mode == ARL2_GATE_PER_HEAD
 *             (row h is column h of the paper's (H*D) x H matrix W_g), n = 1 for ARL2_GATE_PER_TOKEN and
 *             n = H*D for ARL2_GATE_PER_ELEMENT (the scalar and the element-wise gate of the paper's gate
 *             ablation, Tab. 4; row h*D + e is the gate of feature e of head h).  Below 2 GiB.
 *   g         device [B][Lq][n] in desc->g_dtype ([B][Lq][H][D] element-wise), fully overwritten; must
 *             not alias an input.
 * fp32 accumulation and sigmoid.  Up to 32 outputs per token the call is bound by reading x once; beyond
 * that it is a dense matrix product on the matrix cores.
 */
arl2_status arl2_gate_proj(const arl2_desc *desc, const void *x, const void *Wg, void *g);

/*
 * Post-denoise state update (paper Eq. (3), Eq. (4); Alg. 1 clean pass).
 *   k, v      device, io_dtype [B][Lq][H][D] of the clean pass (desc->Lkv must equal Lq).
 *   gate      device fp32 [B][H].
 *   S         device fp32 [B][H][D][D], updated IN PLACE.
 * The token-split partial sums are reduced in a fixed order: results are bit-identical
 * from run to run.  Uses desc->workspace.
 */
arl2_status arl2_state_commit(const arl2_desc *desc,
                              const void *k, const void *v,
                              const float *gate, float *S);

/*
 * arl2_state_commit for callers that can neither allocate device memory nor bring a workspace: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, same kernels
 * and bit-identical results; desc->workspace and desc->workspace_bytes are ignored, the token-split
 * partial sums go to a fixed array in device memory that the library holds on every GPU it runs on
 * (arl2_static_scratch_bytes(), 16 MiB).  A problem that needs more returns ARL2_ERR_UNSUPPORTED
 * (bf16: B * H * splits * D * D * 4 bytes, 12 MiB at B = 1, H = 12, Lq = 4680, D = 128; fp32: B * Lq * H * 4
 * bytes, as for arl2_state_commit).  The call allocates and frees nothing and does not synchronise.  All calls on one GPU share that
 * GPU's array: two calls that overlap in time on one GPU (different streams, or threads) race; calls on
 * one stream, or ordered by events, do not.  Nothing in the array has to survive between calls or to be
 * cleared: every call writes each partial sum before it reads it.
 */
size_t arl2_static_scratch_bytes(void);
arl2_status arl2_state_commit_static(const arl2_desc *desc,
                                     const void *k, const void *v,
                                     const float *gate, float *S);

/*
 * arl2_state_commit with the key and value feature maps of the linear branch fused in (paper Eq. (3),
 * Eq. (4); Alg. 1 clean pass):
 *     S <- gate * S + sum_i L2Norm(RoPE_i(Wk[h] xk_i))^T (Wv[h] xv_i)
 * equal to arl2_feature_map(xk, Wk, rope_cos, rope_sin), arl2_feature_map(xv, Wv, NULL, NULL) and
 * arl2_state_commit on their outputs, without the two intermediate arrays and their launches.  The mapped
 * key is rounded to bf16 once, as arl2_feature_map would store it, and normalised as rounded; the mapped
 * value stays in fp32 until it is scaled by the key's inverse norm (it is not rounded to bf16 on its own,
 * so the result is closer to exact arithmetic than the three calls, not bit-identical to them).
 *   xk, xv    device bf16 [B][Lq][H][D]: the clean pass's projections the maps act on (desc->io_dtype must
 *             be ARL2_BF16, desc->Lkv must equal Lq).
 *   Wk, Wv    device bf16 [H][D][D], indexed [head][out][in], as in arl2_feature_map.
 *   rope_cos, rope_sin   device fp32 [Lq][D/2], 8-byte aligned: the key map's rotation, as in
 *             arl2_feature_map; both NULL: no rotation.  The value map is never rotated.
 *   gate      device fp32 [B][H].
 *   S         device fp32 [B][H][D][D], updated IN PLACE.
 * Deterministic.  Uses desc->workspace (arl2_workspace_bytes covers it).
 */
arl2_status arl2_state_commit_fm(const arl2_desc *desc,
                                 const void *xk, const void *Wk,
                                 const float *rope_cos, const float *rope_sin,
                                 const void *xv, const void *Wv,
                                 const float *gate, float *S);

/*
 * Post-denoise state update with the delta-correction term: paper Eq. (4) taken literally at
 * frame level,
 *     S <- alpha * S + beta * K'^T (V - K' S),      K' = L2Norm(k) per token (Eq. (3)),
 * every token's correction using the same pre-update S (frame-level access, Sec. 3.3).
 *   k, v      device bf16 [B][Lq][H][D] of the clean pass (desc->io_dtype must be ARL2_BF16,
 *             desc->Lkv must equal Lq); fp32 inputs return ARL2_ERR_UNSUPPORTED.
 *   gate      device fp32 [B][H], the forget gate alpha.
 *   beta      device fp32 [B][H], the learning rate.  With all L tokens written at once the update
 *             is a contraction only for beta below about 2 D / L; that is the caller's choice.
 *   S         device fp32 [B][H][D][D], updated IN PLACE.
 * Deterministic like arl2_state_commit.  Uses desc->workspace (arl2_workspace_bytes covers it).
 */
arl2_status arl2_state_commit_delta(const arl2_desc *desc,
                                    const void *k, const void *v,
                                    const float *gate, const float *beta, float *S);

/*
 * Token-sequential gated delta rule: paper Eq. (4) applied to one token at a time, in token order,
 * with per-token gates (Sec. 3.2, remark after Eq. (4); Alg. 1, clean pass).  For j = 1..Lq
 *     S <- alpha_j * S + beta_j * k'_j^T (v_j - k'_j S),      k'_j = L2Norm(k_j)  (Eq. (3)),
 * the correction of token j reading the state as token j-1 left it.
 *   k, v      device bf16 [B][Lq][H][D] of the clean pass (desc->io_dtype must be ARL2_BF16,
 *             desc->Lkv must equal Lq); fp32 inputs return ARL2_ERR_UNSUPPORTED.
 *   alpha     device fp32 [B][Lq][H], per-token forget gates.
 *   beta      device fp32 [B][Lq][H], per-token learning rates; each step is a contraction for
 *             0 <= beta_j <= 1 and 0 <= alpha_j <= 1.
 *   S         device fp32 [B][H][D][D], updated IN PLACE.
 * desc->workspace must hold arl2_gdn_workspace_bytes(desc) bytes (per block of 64 tokens and head the
 * operands of its transition, 65 KiB at D = 128, plus up to 7 composed D x D maps of 128 KiB per head).
 * Deterministic.
 */
size_t arl2_gdn_workspace_bytes(const arl2_desc *desc);
arl2_status arl2_state_commit_gdn(const arl2_desc *desc,
                                  const void *k, const void *v,
                                  const float *alpha, const float *beta, float *S);

/*
 * ---- paged 4-bit key/value cache -----------------------------------------------------------------------
 * The cache of a layer that keeps softmax (paper Eq. (1)): rows of Hkv stored heads, in pages of page_size tokens
 * that a block table places anywhere in a pool, in 4 bits a feature and 8 more per 32 features: 68 bytes for a
 * key row of 128 features, of which bf16 takes 256.  The pool is one array of arl2_kv_cache_bytes(desc) bytes, 16-byte aligned,
 * whose layout is the library's own; bytes that no token was written to may hold anything.
 *
 * Format (the OCP microscaling format e2m1 with a power-of-two scale): 32 features of a token and head share
 * an exponent e, the least one in [-120, 125] with max |x| <= 7 * 2^e (125 beyond), and each is stored as the nearest of
 * 2^e * {0, 1/2, 1, 3/2, 2, 3, 4, 6} and their negatives (ties to the even code).  A group with a NaN or an
 * infinity is stored as NaN.  The stored values are exact in bf16.
 *
 * Device-side indexes, int32, read when the kernels run (so a captured graph follows them):
 *   block_table [B][max_pages]   page of the pool that holds tokens i * page_size .. + page_size - 1 of a stream.
 *                                An entry outside [0, n_pages) holds no tokens: nothing is written there, zeros are
 *                                read, attention does not see them (tokens that a sliding window dropped).
 *                                Streams may share pages that are only read (a common prompt); if one call appends
 *                                different rows to the same place of a page, what is stored there may mix their bytes.
 *   start, count, kv_len, q_len  [B] as described below.  Values beyond what the arrays hold are cut to it: count
 *                                and q_len to [0, Lq], kv_len to [0, max_pages * page_size].
 */
typedef struct {
    int32_t B;            /* streams, >= 1                                                       */
    int32_t H;            /* query heads, a multiple of Hkv (query head h reads stored head      */
                          /* h / (H / Hkv)); attention only                                      */
    int32_t Hkv;          /* stored heads, >= 1                                                  */
    int32_t Lq;           /* tokens per stream of the call's dense arrays, >= 1                  */
    int32_t D;            /* head dimension: 64 or 128                                           */
    int32_t page_size;    /* tokens per page: 16, 32, 64, 128 or 256                             */
    int32_t n_pages;      /* pages of the pool, >= 1                                             */
    int32_t max_pages;    /* block table entries per stream, >= 1; max_pages * page_size <= 2^30 */
    int32_t causal;       /* attention: 0 every stored token is seen; 1 see arl2_kv_attn_fwd     */
    float sm_scale;       /* attention: logit scale, at most 2^127; 0 selects 1/sqrt(D)          */
    void *workspace;      /* attention: device scratch, >= arl2_kv_workspace_bytes               */
    size_t workspace_bytes;
    void *stream;         /* hipStream_t; NULL is the default stream                             */
} arl2_kv_desc;

/* Bytes of the pool, and the scratch that arl2_kv_attn_fwd takes for this descriptor (0: none is needed; it depends on the sizes
 * alone, not on kv_len).  Both return 0 for an invalid descriptor. */
size_t arl2_kv_cache_bytes(const arl2_kv_desc *desc);
size_t arl2_kv_workspace_bytes(const arl2_kv_desc *desc);

/*
 * Writes new rows into the cache: token i < count[b] of stream b goes to position start[b] + i, over what was there.
 *   k, v      device bf16 [B][Lq][Hkv][D]; rows from count[b] on are not read.
 *   rope_cos, rope_sin   device fp32 [max_pages * page_size][D/2], 16-byte aligned, indexed by position: the key's pair
 *             (k[2i], k[2i+1]) is rotated by that angle (computed in fp64, rounded once to fp32) before it is
 *             stored.  Both NULL: no rotation.  Values are never rotated.
 *   start     device int32 [B].       count   device int32 [B], or NULL: Lq for all.
 *   cache     the pool.  Tokens outside [0, max_pages * page_size) and pages outside the pool are skipped; every
 *             other byte of the pool keeps its value.
 */
arl2_status arl2_kv_append(const arl2_kv_desc *desc, const void *k, const void *v,
                           const float *rope_cos, const float *rope_sin,
                           const int32_t *block_table, const int32_t *start, const int32_t *count, void *cache);

/*
 * Gives the values that stored rows stand for: k, v [B][Lq][Hkv][D] bf16, token i < count[b] from position start[b] + i.
 * Rows from count[b] on are left as they were; a row without a place in the cache is zero.
 */
arl2_status arl2_kv_read(const arl2_kv_desc *desc, const void *cache,
                         const int32_t *block_table, const int32_t *start, const int32_t *count, void *k, void *v);

/*
 * out_i = softmax_j(sm_scale * q_i.K_j) V_j over the stored tokens j < kv_len[b] of the stream, for its query tokens
 * i < q_len[b].  desc->causal: query i stands at position kv_len[b] - q_len[b] + i and sees the tokens up to it (the queries are
 * the last tokens stored).  A query that sees no token gives zeros.
 *   q         device bf16 [B][Lq][H][D]; rows from q_len[b] on are not read.  A row with a NaN or an infinity gives NaN
 *             if it sees a token.
 *   kv_len    device int32 [B].       q_len   device int32 [B], or NULL: Lq for all.
 *   out       device bf16 [B][Lq][H][D]; rows from q_len[b] on are left as they were.  Must not overlap an input.
 * Products q_i.K_j and logits have to lie in fp32's range, +-2^127.
 * fp32 accumulation, softmax statistics and joins of the key axis, which is divided the same way for the same descriptor:
 * results are bit-identical from run to run.  Probabilities are rounded to bf16 for the second product, and with more than 64
 * query rows (Lq * H / Hkv) a query row may be taken to within 2^-9 of its length, half of what rounding it to bf16 may have taken, or
 * a feature to within 2^-112, whichever is more.  What the other queries of the call hold does not change a bit of a query's output.
 * That division goes by max_pages * page_size, the longest history that the table could hold; parts beyond kv_len are left empty.  Where
 * histories are far shorter, fewer workgroups share them: 1560 queries of 12 heads over 10920 tokens took 99 us with a table of
 * that width and 215 with one four or twelve times as wide, single tokens of 16 streams of 8192 tokens 35, 42 and 74 us with tables of
 * 8192, 32768 and 131072.
 * Uses desc->workspace; calls that overlap in time need one each.
 */
arl2_status arl2_kv_attn_fwd(const arl2_kv_desc *desc, const void *q, const void *cache,
                             const int32_t *block_table, const int32_t *kv_len, const int32_t *q_len, void *out);

/*
 * ---- the linear branch as a causal recurrence ---------------------------------------------------------------
 * For t = 1..len of every stream and head, k'_t = L2Norm(k_t), q'_t = L2Norm(q_t) (Eq. (3)) or the rows as they are,
 *     S_t = exp(log_alpha_t) S_{t-1} + k'_t^T v_t,        out_t = q'_t S_t:
 * Eq. (4) with beta = 1 and without the delta-correction term, token by token, and Eq. (5) with the state that a token leaves
 * instead of a state that its chunk shares: what a causal model trains on and generates with.
 */
typedef struct {
    int32_t B, H, L, D;   /* streams, heads, tokens: >= 1; D: 64 or 128.  L*H*D must stay below 2^30                    */
    int32_t raw_rows;     /* 0: rows of q and k are divided by sqrt(|row|^2 + l2_eps); 1: they are taken as they are   */
    float l2_eps;         /* >= 1e-30; 0 selects 1e-6                                                                  */
    void *workspace;      /* device scratch, >= arl2_scan_workspace_bytes or arl2_scan_bwd_workspace_bytes, 16-byte     */
    size_t workspace_bytes;  /* aligned; one for each call in flight                                                   */
    void *stream;         /* hipStream_t; NULL is the default stream                                                   */
} arl2_scan_desc;

/* Scratch of the two calls (it depends on the sizes alone; 0: none is needed, or the descriptor is invalid). */
size_t arl2_scan_workspace_bytes(const arl2_scan_desc *desc);
size_t arl2_scan_bwd_workspace_bytes(const arl2_scan_desc *desc);

/*
 *   q, k, v   device bf16 [B][L][H][D].
 *   log_alpha device fp32 [B][L][H]: natural logarithms of the gates, in [-inf, 0].  -inf (and what is below -2839) is a gate of zero: the state
 *             begins anew with that token.  Values above 0 are taken as 0.  NULL: all gates are one.
 *   seq_len   device int32 [B], read when the kernels run, cut to [0, L], or NULL: L for all.  Rows from seq_len[b] on are not read,
 *             and left as they were in what is written.
 *   S0        device fp32 [B][H][D][D], the state before the first token; NULL: zeros.
 *   out       device bf16 [B][L][H][D]; must not overlap an input.
 *   S         device fp32 [B][H][D][D], the state after the last token (S0 where there is none); NULL: it is not wanted.  May be S0 itself
 *             (the state is updated in place), else it must not overlap an input.
 * States, decays and sums are fp32 (a block's decays come from sums in fp64).  On the matrix cores rows enter the state as two bf16 parts (to
 * 2^-17 of each value: S is off by 2.5e-6 in the 2-norm), and out's rows take the state's features and the products q'.k' within a block of 64 tokens
 * rounded to bf16 once.
 * Features of rows have to be below 2^16, the state below 2^48 (products of three of them have decays taken out, up to 2^64, before fp32 holds them).
 * Up to 8 tokens are computed in fp32 throughout, with the state read and written once.  A NaN or an infinity in
 * a token's rows or gate reaches outputs of that token and of later ones (in v: that feature alone), and the state, which keeps it also behind a gate of zero, which multiplies by zero.
 * Deterministic.
 */
arl2_status arl2_scan_fwd(const arl2_scan_desc *desc, const void *q, const void *k, const void *v, const float *log_alpha,
                          const int32_t *seq_len, const float *S0, void *out, float *S);

/*
 * Gradients of arl2_scan_fwd's arguments, of those that are given:
 *   dout      device bf16 [B][L][H][D], gradient of out.
 *   dS        device fp32 [B][H][D][D], gradient of the last state; NULL: zeros.
 *   dq, dk, dv  device bf16 [B][L][H][D], written (through the normalisation where there is one).
 *   dlog_alpha  device fp32 [B][L][H], written: the gradient of log_alpha as if it had no upper limit; zero at a gate of zero.  NULL: it is not wanted.
 *   dS0       device fp32 [B][H][D][D], written; NULL: it is not wanted.
 * Features of rows and of dout have to be below 2^15 (a row's product with its gradient holds four of them and a decay taken out), states and their gradients below 2^48.
 * Where l2_eps is below 1e-14, products dout.v have to be below 2^63 sqrt(l2_eps) too, and the gradients of normalised rows, before the normalisation, below 2^127 l2_eps.
 * Of what the matrix cores take, dv and dS0 are rounded as out and S are; dq and dk, whose products with q' and k' add up to dlog_alpha over up to 1024
 * tokens, take the states and what enters them in three bf16 parts (to 2^-25; dlog_alpha is off by 5.5e-6 in the 2-norm at
 * most where it was looked at, by 8.1e-6 in one head; a sum of such products that cancel, it is off by more of itself where gates leave next to nothing of the state).  A NaN or an infinity in a row
 * reaches gradients of its own stream and head alone, of tokens on either side of it.
 * What is written must overlap neither an input nor what else is written.  Deterministic.
 */
arl2_status arl2_scan_bwd(const arl2_scan_desc *desc, const void *q, const void *k, const void *v, const float *log_alpha,
                          const int32_t *seq_len, const float *S0, const void *dout, const float *dS,
                          void *dq, void *dk, void *dv, float *dlog_alpha, float *dS0);

/*
 * ---- rotary positions on several axes -------------------------------------------------------------------------
 * Rows of queries and keys as attention and the linear branch take them: y = R(pos) (w . x / sqrt(mean(x^2) + norm_eps)).
 * The features of a head are D / 2 pairs; axis a turns the next axis_pairs[a] of them, its pair i by the angle
 * pos[a] * theta[a]^(-i / axis_pairs[a]):  (x0, x1) -> (x0 cos - x1 sin, x0 sin + x1 cos).  Pairs beyond the axes' are not turned.
 */
typedef enum { ARL2_NORM_NONE = 0, ARL2_NORM_HEAD = 1, ARL2_NORM_ROW = 2 } arl2_norm_mode;

typedef struct {
    int32_t B, H, L, D;   /* streams, query heads, tokens: >= 1; D: 64 or 128                                          */
    int32_t Hk;           /* key heads, >= 0 (0: there are no keys, their arrays are NULL); (H + Hk) * D <= 24576       */
    int32_t io_dtype;     /* arl2_dtype of rows, weights and gradients of rows                                        */
    int32_t norm;         /* arl2_norm_mode: the mean over a head's features, over all features of a token's          */
                          /* queries (and of its keys), or no norm and no weights                                    */
    int32_t halves;       /* pairs are 0: features (2i, 2i + 1), 1: features (i, i + D / 2)                           */
    int32_t pos_per_stream;  /* pos is 0: [L][n_axes], 1: [B][L][n_axes]                                              */
    int32_t n_axes;       /* 1 to 4                                                                                  */
    int32_t axis_pairs[4];   /* each >= 1, together <= D / 2                                                          */
    double theta[4];      /* 1e-3 to 1e30; 0 selects 10000                                                           */
    float norm_eps;       /* >= 1e-30; 0 selects 1e-6                                                                */
    void *workspace;      /* arl2_rope_bwd with weights' gradients: >= arl2_rope_workspace_bytes, 16-byte aligned     */
    size_t workspace_bytes;
    void *stream;         /* hipStream_t; NULL is the default stream                                                 */
} arl2_rope_desc;

/* Scratch of arl2_rope_bwd where it writes weights' gradients (it depends on B, H, Hk, L and D alone; 0: the descriptor is invalid). */
size_t arl2_rope_workspace_bytes(const arl2_rope_desc *desc);

/*
 *   q, k      device, io_dtype [B][L][H][D] and [B][L][Hk][D].
 *   wq, wk    device, io_dtype: [D] and [D] (ARL2_NORM_HEAD, shared by the heads), [H*D] and [Hk*D] (ARL2_NORM_ROW); NULL: ones.
 *   pos       device int32, any values: angles are computed in fp64.
 *   seq_len   device int32 [B], or NULL: L for all.  Rows from seq_len[b] on are not read, and left as they were in what is written.
 *   yq, yk    device, like q and k.  yq may be q and yk may be k (in place); else they must overlap neither an input nor each other.
 * fp32 arithmetic, one rounding to io_dtype.  Where there is a norm, the sums of a row's squares (and of its products with dy and the weights) have to lie in
 * fp32's range; a NaN or an infinity reaches the rows that share its norm.
 */
arl2_status arl2_rope_fwd(const arl2_rope_desc *desc, const void *q, const void *k, const void *wq, const void *wk,
                          const int32_t *pos, const int32_t *seq_len, void *yq, void *yk);

/*
 * Gradients: dyq, dyk of yq, yk are given; dq, dk are written (they may be dyq and dyk), and the weights' gradients dwq, dwk, fp32, summed over the tokens
 * that there are (and over the heads: ARL2_NORM_HEAD), each where it is not NULL and the rows have a norm.  Without a norm q and k are not read and may be NULL.
 * Deterministic.
 */
arl2_status arl2_rope_bwd(const arl2_rope_desc *desc, const void *q, const void *k, const void *wq, const void *wk,
                          const int32_t *pos, const int32_t *seq_len, const void *dyq, const void *dyk,
                          void *dq, void *dk, float *dwq, float *dwk);

const char *arl2_status_string(arl2_status s);

/* Thread-local detail of the last call that failed on this thread ("" if none has failed yet); a later
 * successful call does not clear it: read it right after a call that returned an error. */
const char *arl2_last_error(void);

/* Library version, major * 10000 + minor * 100 + patch. */
int arl2_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ARL2_H */
