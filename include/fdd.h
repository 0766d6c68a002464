/*
 * fdd.h -- C ABI of the MI355X (gfx950) block-diffusion denoise-step library.
 *
 * One denoising step of a section-aligned block, as the paper describes it:
 *   - block-causal attention (Preliminaries, "Block-Causal Diffusion"): a
 *     block attends bidirectionally to itself and causally to the prompt and
 *     all earlier blocks, whose KV cache is reused without recomputation
 *     ("Section Diffusion (SD)");
 *   - N rollouts forked from one shared KV cache (test-time scaling section,
 *     "Shared prefix"): every rollout owns a private block and they all read
 *     the single prefix, which is never copied per rollout;
 *   - confidence-threshold unmasking of still-masked value positions, with
 *     the structural scaffold frozen (Eq. 2 and the scaffold construction
 *     paragraph; "iteratively unmasks value positions").
 *
 * Conventions common to every call
 *   - Every data pointer is a DEVICE pointer owned by the caller (HBM of the
 *     current HIP device); the parameter structs themselves live on the host.
 *     The library allocates no device memory, never copies the prefix and
 *     never synchronises.  Work is enqueued on `stream` (a hipStream_t passed
 *     as void*; NULL = the default stream) and the call returns at once.
 *   - Arrays are dense, row-major, in the index order written next to them.
 *   - The return code covers what the host can see: NULL pointers, shapes,
 *     element type, workspace size, launch failure.  On error nothing is
 *     launched and fdd_last_error() holds a message (thread-local).
 *   - Inputs are never modified, except arrays documented as in/out.
 *   - Scratch (`workspace`) must be at least what the matching
 *     *_workspace() call returns for the same params, 256-byte aligned;
 *     its contents before and after a call are unspecified.  Calls that
 *     share a workspace must be ordered on one stream.
 */
#ifndef FDD_H
#define FDD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    FDD_OK = 0,
    FDD_ERR_NULL = 1,        /* a required pointer is NULL */
    FDD_ERR_SHAPE = 2,       /* non-positive size, Hq % Hkv != 0, ... */
    FDD_ERR_DTYPE = 3,       /* element type not FDD_F32 / FDD_BF16 */
    FDD_ERR_UNSUPPORTED = 4, /* head size or option outside the supported set */
    FDD_ERR_WORKSPACE = 5,   /* workspace missing, misaligned or too small */
    FDD_ERR_LAUNCH = 6       /* the HIP runtime refused a launch */
} fdd_status;

typedef enum { FDD_F32 = 0, FDD_BF16 = 1 } fdd_dtype;

/* ------------------------------------------------------------------------
 * fdd_block_attn: shared-prefix block-causal attention for N rollouts.
 *
 * For rollout n, block position b, query head h (KV head kh = h / (Hq/Hkv)):
 *   keys   = prefix_k[0..L) ++ block_k[n, 0..B)      (head kh)
 *   values = prefix_v[0..L) ++ block_v[n, 0..B)
 *   out[n,b,h,:] = softmax(scale * q[n,b,h,:] . keys^T) values
 * Every one of the L+B keys is visible (bidirectional inside the block,
 * causal to the prefix); other rollouts' blocks are not.  This is the
 * attention rule of "Block-Causal Diffusion" applied to rollouts that were
 * forked from one cache ("Shared prefix").  Position encoding is outside
 * this call: q and k arrive already rotated.
 *
 * scaffold_mask does not enter the arithmetic: scaffold tokens are ordinary
 * visible tokens of the block (pre-filled, never masked), both as keys and
 * as queries.  It is accepted so the signature matches the step's problem
 * statement, may be NULL, and the output is the same for any value.
 *
 * dtype FDD_BF16: q/k/v/out are bfloat16, products on the matrix cores with
 * fp32 accumulation, softmax in fp32.  dtype FDD_F32: fp32 storage and
 * arithmetic (calls of many rows and keys take each product as six exact
 * products of bf16 parts: to 2^-24 of its factors' powers of two, fp32 sums).
 * D must be 64 or 128.  L may be 0.  `out` must not alias an input.  splits:
 * number of pieces the prefix is cut into along L, with FDD_F32 all keys of a
 * query row (0 = chosen by the library); the result does not depend on it
 * beyond fp32 rounding.
 *
 * Values: q, k and v finite, scores within fp32's range.  For others nothing
 * is read or written out of bounds.  FDD_F32 passes a NaN or an infinity on
 * as arithmetic gives it, to the rows that see it (with
 * FDD_ATTN_CAUSAL_BLOCK also to earlier rows of its block), and such a
 * call may take up to three times as long.  FDD_BF16: the
 * rows that see one, and up to 31 rows stacked next to them, which may
 * belong to another rollout, are undefined.
 */
/* In-block attention is causal instead of bidirectional: block position b sees
 * the prefix and block positions <= b of its own rollout.  This is the verify
 * pass of Scaffold Speculative Decoding (paper, "Scaffold Speculative Decoding
 * (SS)", step 3: "a causal forward pass over the entire block"); the draft pass
 * of step 2 is the default bidirectional form. */
#define FDD_ATTN_CAUSAL_BLOCK 1

typedef struct fdd_attn_params {
    int32_t N, B, L, Hq, Hkv, D;
    int32_t dtype;                 /* fdd_dtype of q, k, v and out */
    float scale;                   /* softmax scale; <= 0 selects 1/sqrt(D) */
    const void *q;                 /* [N,B,Hq,D] */
    const void *prefix_k;          /* [L,Hkv,D]  one copy for all rollouts; may be NULL iff L == 0 */
    const void *prefix_v;          /* [L,Hkv,D] */
    const void *block_k;           /* [N,B,Hkv,D] */
    const void *block_v;           /* [N,B,Hkv,D] */
    const uint8_t *scaffold_mask;  /* [N,B] 1 = frozen scaffold token; may be NULL */
    void *out;                     /* [N,B,Hq,D] */
    void *workspace;               /* >= fdd_block_attn_workspace() bytes */
    size_t workspace_bytes;
    void *stream;                  /* hipStream_t */
    int32_t splits;                /* 0 = automatic */
    int32_t flags;                 /* FDD_ATTN_* bits; unknown bits are rejected */
    const void *prefix_v_packed;   /* optional: output of fdd_prefix_pack for this prefix_v, or NULL */
    /* Per-rollout extension: the blocks rollout n has finished since the fork ("Shared prefix": the
     * trajectory section is continued N times and spans several blocks; "Block-Causal Diffusion": a block
     * attends causally to all earlier blocks).  Rows ext[n, 0..E) are keys of rollout n only, between
     * the shared prefix and the live block; they are fully visible, also with FDD_ATTN_CAUSAL_BLOCK.
     * E = 0 (pointers may then be NULL) is the plain two-run form. */
    const void *ext_k;             /* [N, ext_capacity, Hkv, D] */
    const void *ext_v;             /* [N, ext_capacity, Hkv, D] */
    int32_t E;                     /* valid extension rows per rollout, 0 <= E <= ext_capacity */
    int32_t ext_capacity;          /* rows allocated per rollout */
    /* Batch of independent problems of one shape in a single launch (for callers whose problems are each
     * too small to fill the chip: several requests, each with its own prefix).  Problem i uses the arrays
     * at q + i*q_batch_stride, prefix_k/prefix_v + i*prefix_batch_stride, block_k/block_v +
     * i*block_batch_stride, ext_k/ext_v + i*ext_batch_stride, out + i*out_batch_stride (strides in
     * elements, multiples of 8, at least the size of one problem's array) and prefix_v_packed +
     * i*packed_batch_stride (bytes, a multiple of 256).  batch <= 1 is the single problem and the strides
     * are ignored.  Nothing is shared between the problems of a batch. */
    int32_t batch;
    int32_t n_q_positions;         /* 0: every position is computed; see q_positions */
    int64_t q_batch_stride, prefix_batch_stride, block_batch_stride, ext_batch_stride, out_batch_stride;
    size_t packed_batch_stride;
    /* Only some block positions as queries ("Scaffold": scaffold tokens are given, never predicted, so
     * where nothing but the logits of a layer's output is read - the last layer - their rows are not
     * needed).  q_positions is a DEVICE array of n_q_positions flat positions n*B + b in strictly ascending
     * order, each in [0, N*B); the rows out[n, b, :, :] of these positions are computed exactly as without
     * the list, every other row of `out` is left as it was.  Keys are not affected: block_k / block_v
     * still hold all B positions of every rollout.  With `batch`, the one list serves every problem.
     * The library cannot read the list on the host: entries out of range are clamped into it by the
     * kernels (no access out of bounds), an order other than ascending gives undefined values in `out`. */
    const int32_t *q_positions;
} fdd_attn_params;

/* Bytes of scratch fdd_block_attn needs for these params (host-only
 * arithmetic, no device is touched).  Returns 0 if the params are invalid.
 * The figure serves the same call with and without prefix_v_packed, except
 * that a very large call without it also needs room for the copy of V that
 * it then makes. */
size_t fdd_block_attn_workspace(const fdd_attn_params *p);
fdd_status fdd_block_attn(const fdd_attn_params *p);

/* ------------------------------------------------------------------------
 * fdd_prefix_pack: one-time relayout of the prefix V for the bf16 kernel.
 *
 * The prefix KV cache does not change while a block is denoised and is shared
 * by all rollouts (paper: KV caches of the prompt and of earlier blocks are
 * reused without recomputation).  The bf16 attention kernel reads the full
 * 64-key tiles of prefix V in an order that has the key index contiguous;
 * when several workgroups stream the same V, fdd_block_attn repacks V into
 * its workspace on every call.  A caller that runs many steps on one prefix
 * can do that once: fdd_prefix_pack writes the repacked copy (a few percent
 * of a step's time) and every later fdd_block_attn on the same prefix takes
 * it through prefix_v_packed.  prefix_v itself must still be passed (the
 * ragged last tile is read from it).  The packed copy belongs to exactly the
 * (prefix_v contents, L, Hkv, D) it was made from.
 *
 * fdd_prefix_pack_bytes: size of the packed copy, 256-byte granular; 0 when
 * nothing would be packed (fp32, or L < 64).  Host-only arithmetic.
 */
size_t fdd_prefix_pack_bytes(int32_t L, int32_t Hkv, int32_t D, int32_t dtype);
fdd_status fdd_prefix_pack(const void *prefix_v, int32_t L, int32_t Hkv, int32_t D, int32_t dtype,
                           void *packed, size_t packed_bytes, void *stream);

/* ------------------------------------------------------------------------
 * A prefix cache in 8 bits.
 *
 * K and V of the shared prefix as e4m3 codes (4 bits of exponent, 3 of mantissa, largest value 448, no
 * infinities) with one scale for every FDD_QUANT_BLOCK rows of a KV head: half the bytes of bf16.  The
 * value of an element is code * scale.  A scale is a power of two, the smallest one that brings the largest
 * magnitude of its rows to 448 or less, but at least 2^-117 and at most 2^119.  Scaling is therefore exact:
 * an element is rounded once, to the nearest code and to even on ties (relative error 2^-4 at most, 2^-10
 * of the scale for codes below 2^-6), and its value is exact in bf16 and fp32.
 *
 * A head's rows lie together, so that the tile of FDD_QUANT_BLOCK keys that attention works on is one
 * piece of memory.  Rows behind the last one written, and their scales, are never used.
 */
#define FDD_QUANT_BLOCK 64
typedef struct fdd_quant_cache {
    void *k;                       /* [Hkv,capacity,D] e4m3 */
    void *v;                       /* [Hkv,capacity,D] e4m3 */
    float *k_scale;                /* [Hkv,capacity/FDD_QUANT_BLOCK] */
    float *v_scale;
    int32_t Hkv, D;                /* D 64 or 128 */
    int32_t capacity;              /* rows allocated per head, a multiple of FDD_QUANT_BLOCK */
    int32_t reserved;              /* must be 0 */
    int64_t batch_stride;          /* fdd_block_attn_quant with batch > 1: elements from one problem's codes to the next's */
    int64_t scale_batch_stride;    /* likewise scales */
} fdd_quant_cache;

/* Rows of K and V in their own precision: the source of fdd_prefix_quantize, the destination of
 * fdd_prefix_dequantize. */
typedef struct fdd_quant_rows {
    void *k;                       /* [rows,Hkv,D], consecutive rows k_row_stride apart; only read by fdd_prefix_quantize */
    void *v;
    int64_t k_row_stride;          /* elements; at least Hkv*D, rows 16-byte aligned; 0 = Hkv*D */
    int64_t v_row_stride;
    int32_t rows;                  /* may be 0 */
    int32_t dtype;                 /* fdd_dtype */
} fdd_quant_rows;

/* fdd_prefix_quantize: the rows become rows [row0, row0 + rows) of the cache, which then ends with them: a
 * prompt (row0 = 0), or a finished block behind the rows that are there (row0 = their number).  Where row0
 * lies inside a block of the cache, the block's scale may grow: the rows in front are then rounded again,
 * to the codes of the new scale (exact, except for codes that fall below 2^-6), else they are left as they
 * are.  It does not shrink.  (All rows of that block in front of row0 and its scale have to be there: a scale is a power of two from
 * 2^-117 to 2^119, also in a cache that was filled by other means.)  Codes behind row0 + rows and scales of later blocks are left as they were.
 * Values: an infinity or a magnitude above 448 * 2^119 is stored as the largest code, a NaN as a NaN;
 * infinities and NaN have no part in the scale.  The source must not overlap the cache, nor the cache's arrays one another.
 *
 * fdd_prefix_dequantize: rows [row0, row0 + rows) of the cache are read back, exactly.  Rows of k and v must not overlap; they may
 * interleave. */
fdd_status fdd_prefix_quantize(const fdd_quant_cache *cache, int32_t row0, const fdd_quant_rows *src, void *stream);
fdd_status fdd_prefix_dequantize(const fdd_quant_cache *cache, int32_t row0, const fdd_quant_rows *dst, void *stream);

/* fdd_block_attn_quant: fdd_block_attn with the prefix in a cache of 8 bits.  `p` as for fdd_block_attn,
 * except that prefix_k, prefix_v and prefix_v_packed are NULL (prefix_batch_stride and packed_batch_stride
 * are ignored): the L keys and values of the prefix are rows [0, L) of `cache`, L <= cache->capacity,
 * converted without an error.  Queries, blocks, extensions and outputs are of type p->dtype.  The result is
 * that of fdd_block_attn on the rows as fdd_prefix_dequantize returns them, up to the order of sums and, in bf16,
 * to the 16 bits of averages: where a row's keys are cut into pieces (by `splits` or by the library), each piece's
 * average is off by 2^-11 of itself, by 2^-39 of the row's largest element of it or by 2^-126, whichever is most.
 * `cache` may be NULL iff L == 0.  The workspace is fdd_block_attn_quant_workspace(p), no less: a bf16 call converts the
 * prefix tile by tile on its way to the matrix pipe and needs no room for it; an fp32 call converts it first and
 * needs room for its K and V in fp32.  Values and q_positions as with fdd_block_attn, a NaN in the cache being one
 * among the values: fp32 passes it on, bf16 leaves the rows that see it undefined. */
size_t fdd_block_attn_quant_workspace(const fdd_attn_params *p);
fdd_status fdd_block_attn_quant(const fdd_attn_params *p, const fdd_quant_cache *cache);

/* ------------------------------------------------------------------------
 * fdd_unmask_step: one confidence-threshold unmask iteration over N blocks.
 *
 * A position (n,b) is eligible when mask[n,b] == 1 and scaffold_mask[n,b]
 * == 0: diffusion acts on the editable set only and visible tokens stay
 * fixed (paper, Eq. 2; "Masked Diffusion Language Models").  For every
 * eligible position
 *     cand = lowest id attaining max_v logits[n,b,v]
 *     conf = 1 / sum_v exp(logits[n,b,v] - max)      (largest softmax prob.)
 * Block n commits every eligible position with conf >= tau; if none reaches
 * tau and the block has an eligible position, it commits the eligible
 * position of highest conf (lowest b on ties), so each call makes progress.
 * Committing writes tokens[n,b] = cand and clears mask[n,b].  All other
 * positions of tokens and mask are left as they were; a mask bit set on a
 * scaffold position is ignored (the scaffold wins).
 *
 * Only the logits rows of eligible positions are read.  The arg max is taken
 * on the stored logits (exact); exp and the sum run in fp32.
 *
 * Logits: finite values, and -inf for entries that can never be chosen (their
 * probability is exactly 0; a row needs at least one finite entry).  NaN and
 * +inf are not supported: the outputs of a row that holds one are undefined
 * (nothing is read or written out of bounds).  The same holds for the logits
 * of fdd_verify_step.
 */
typedef struct fdd_unmask_params {
    int32_t N, B;
    int64_t V;
    int32_t dtype;                 /* fdd_dtype of logits */
    float tau;
    const void *logits;            /* [N,B,V] */
    const uint8_t *scaffold_mask;  /* [N,B]; may be NULL (= no scaffold) */
    uint8_t *mask;                 /* [N,B] in/out, 1 = still masked */
    int32_t *tokens;               /* [N,B] in/out */
    float *confidences;            /* [N,B] out: conf of eligible positions, -inf elsewhere */
    int32_t *n_unmasked;           /* [N] out, commits per block; may be NULL */
    uint8_t *committed;            /* [N,B] out, 1 = committed by this call; may be NULL */
    void *workspace;               /* >= fdd_unmask_workspace() bytes */
    size_t workspace_bytes;
    void *stream;
    /* Optional K/V refresh of the positions this call commits, done by the same kernel that takes the
     * commit decisions: exactly what fdd_block_kv_update would do right afterwards with this call's
     * `tokens` and `committed` (one launch less per denoise step).  All four pointers NULL (and the
     * sizes 0): no refresh.  Otherwise all four must be given, 16-byte aligned, with a row of
     * refresh_Hkv * refresh_D elements of refresh_dtype being a multiple of 16 bytes. */
    const void *refresh_table_k;   /* [refresh_T, refresh_Hkv, refresh_D] */
    const void *refresh_table_v;
    void *refresh_block_k;         /* [N, B, refresh_Hkv, refresh_D] in/out */
    void *refresh_block_v;
    int32_t refresh_Hkv, refresh_D, refresh_T;
    int32_t refresh_dtype;         /* fdd_dtype of the tables and the block K/V */
} fdd_unmask_params;

size_t fdd_unmask_workspace(const fdd_unmask_params *p);
fdd_status fdd_unmask_step(const fdd_unmask_params *p);

/* fdd_unmask_step_static: fdd_unmask_step for callers that cannot allocate
 * device memory and carry no workspace: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Same arguments, same
 * results bit for bit; `workspace` and `workspace_bytes` are ignored.  The
 * per-piece partial results of the vocabulary reduction go to a fixed array of
 * FDD_STATIC_SCRATCH_BYTES inside the library's device image instead (every GPU
 * the library runs on holds one copy until the process ends).  The call
 * allocates nothing and frees nothing.  Shapes whose partials do not fit
 * (N*B*pieces > FDD_STATIC_SCRATCH_BYTES / 16, i.e. fdd_unmask_workspace() above
 * that size; 1024 positions over V = 152064 need 64 KiB) are rejected with
 * FDD_ERR_WORKSPACE and nothing is launched.  All calls on one GPU share that
 * GPU's array: two calls that overlap in time on one GPU (different streams,
 * different threads) race and give wrong results; calls ordered on one stream
 * are safe.  Nothing in the array has to be cleared between calls: every
 * record a call reads was written by that call.  The current device must be
 * the one `stream` belongs to.
 */
#define FDD_STATIC_SCRATCH_BYTES ((size_t)1 << 20)
fdd_status fdd_unmask_step_static(const fdd_unmask_params *p);

/* ------------------------------------------------------------------------
 * fdd_verify_step: accept scan of Scaffold Speculative Decoding over N blocks
 * (paper, "Scaffold Speculative Decoding (SS)", steps 1 and 3).
 *
 * Draft positions are those with mask[n,b] == 1 and scaffold_mask[n,b] == 0;
 * scaffold positions are auto-accepted and take no part.  ar_logits[n,b,:] is
 * the AR head's distribution for the token AT position b (the caller applies
 * the usual one-position shift).  Draft positions are visited left to right:
 * while the lowest id attaining max_v ar_logits[n,b,v] equals draft[n,b], the
 * draft is accepted (tokens[n,b] = draft[n,b], mask cleared).  At the first
 * mismatch the AR token replaces the draft (tokens[n,b] = arg max, mask
 * cleared: the one bonus token) and every later draft position of the block
 * is discarded: its mask bit stays 1 and its tokens entry is not touched.
 * n_accepted[n] counts the positions unmasked by this call; accepted[n,b] is
 * 1 for an accepted draft, 2 for the replaced position, 0 otherwise.
 * Only the logits rows of draft positions are read.
 *
 * Sampled verifier (paper, "Trajectory-only stochasticity": in the trajectory
 * section the verifier samples from its softmax, which is what makes forked
 * rollouts differ).  With temperature > 0 the verifier's token at a draft
 * position is a sample of softmax(ar_logits[n,b,:] / temperature) instead of
 * the arg max, drawn by the Gumbel-max rule
 *     token = lowest id attaining max_v key(v),
 *     key(v) = fma(x_v, c, -flog2(-flog2(u_v)))          (binary32 throughout)
 *     c   = (float)(log2(e) / (double)temperature)
 *     u_v = ((r_v >> 9) + 0.5) * 2^-23
 *     r_v = word (v mod 4) of Philox-4x32-10(counter = (v div 4, n*B + b, 0, 0),
 *                                            key = (seed low word, seed high word))
 *     flog2(y) = e + f P(f) for y = m 2^e, m in [1/sqrt 2, sqrt 2), f = m - 1, with
 *                the degree-8 polynomial P listed in csrc/unmask.hip, evaluated
 *                by Horner's rule in fused multiply-adds.
 * Every step is an exactly rounded binary32 operation, so a (seed, row, logits)
 * triple names one token on any conforming implementation.  The same seed
 * gives the same tokens; rollouts differ because their rows n*B + b differ.
 * temperature == 0 selects the greedy verifier; negative or non-finite values
 * are rejected with FDD_ERR_UNSUPPORTED.
 */
typedef struct fdd_verify_params {
    int32_t N, B;
    int64_t V;
    int32_t dtype;                 /* fdd_dtype of ar_logits */
    float temperature;             /* 0 = greedy verifier, > 0 = sampled verifier */
    const void *ar_logits;         /* [N,B,V] */
    const uint8_t *scaffold_mask;  /* [N,B]; may be NULL */
    const int32_t *draft;          /* [N,B] draft tokens (used at draft positions only) */
    uint8_t *mask;                 /* [N,B] in/out */
    int32_t *tokens;               /* [N,B] in/out */
    int32_t *n_accepted;           /* [N] out; may be NULL */
    uint8_t *accepted;             /* [N,B] out; may be NULL */
    void *workspace;               /* >= fdd_verify_workspace() bytes */
    size_t workspace_bytes;
    void *stream;
    uint64_t seed;                 /* sampled verifier: key of the random stream */
} fdd_verify_params;

/* Bytes of scratch for these params (host-only arithmetic; 0 if they are invalid).  The figure depends on
 * `temperature`: the greedy verifier cuts a row into more pieces than the sampled one. */
size_t fdd_verify_workspace(const fdd_verify_params *p);
fdd_status fdd_verify_step(const fdd_verify_params *p);

/* ------------------------------------------------------------------------
 * fdd_token_logprobs: what a row of logits says about a token, without a sample or a decision.
 *
 * With p = softmax(logits[n,b,:] / temperature), for every selected position (row_mask NULL, or
 * row_mask[n,b] == 1):
 *     logprobs[n,b]       = ln p[tokens[n,b]]; -inf for a token outside [0, V)
 *     entropy[n,b]        = -sum_v p[v] ln p[v]   (nats; entries of probability 0 contribute nothing)
 *     top_ids[n,b,0..top) = the ids of the `top` largest logits, largest first, the lowest id first among
 *                           equal ones; top_logprobs their ln p
 * Positions that are not selected keep what their outputs held, and their logits are not read.  An output
 * that is NULL is not computed (top_ids and top_logprobs both or neither).
 *
 * The sums run in fp32 over pieces of a row, which are joined in fp64; the largest term is kept out of the
 * sum and joins in ln(1 + rest), so that the log probability of a token that is nearly certain keeps its
 * digits.  Logits: finite values, down to the type's lowest number, and -inf for entries that can never be chosen; a
 * log probability below fp32's lowest number is -inf.  A row without a
 * finite entry has no softmax: its logprobs, entropy and top_logprobs are NaN, its top_ids 0..top-1.  NaN and
 * +inf are not supported: such a row's outputs are undefined (nothing is read or written out of bounds).
 */
#define FDD_LOGPROBS_MAX_TOP 32
typedef struct fdd_logprob_params {
    int32_t N, B;
    int64_t V;
    int32_t dtype;                 /* fdd_dtype of logits */
    int32_t top;                   /* 0 .. min(V, FDD_LOGPROBS_MAX_TOP) */
    float temperature;             /* positive, at most 2^120, and 1.5 / temperature finite (4.41e-39 and more) */
    int32_t reserved;              /* must be 0 */
    const void *logits;            /* [N,B,V] */
    const int32_t *tokens;         /* [N,B]; may be NULL iff logprobs is */
    const uint8_t *row_mask;       /* [N,B], 1 = selected; may be NULL (= all) */
    float *logprobs;               /* [N,B] out; may be NULL */
    float *entropy;                /* [N,B] out; may be NULL */
    int32_t *top_ids;              /* [N,B,top] out; may be NULL */
    float *top_logprobs;           /* [N,B,top] out; may be NULL */
    void *workspace;               /* >= fdd_token_logprobs_workspace() bytes */
    size_t workspace_bytes;
    void *stream;
} fdd_logprob_params;

size_t fdd_token_logprobs_workspace(const fdd_logprob_params *p);
fdd_status fdd_token_logprobs(const fdd_logprob_params *p);

/* ------------------------------------------------------------------------
 * Rotary positions.
 *
 * Channel pair i of a head, i < rot_dim / 2, is the point (x, y) = channels (i, i + rot_dim / 2), or (2i, 2i + 1) with
 * `interleaved`; at position p it becomes
 *     magnitude * (x cos a - y sin a, y cos a + x sin a),      a = p w_i;
 * channels from rot_dim on stay as they are.  With w = base^(-2i / rot_dim), by `scaling`:
 *     FDD_ROPE_NONE     w_i = w
 *     FDD_ROPE_LINEAR   w_i = w / stretch
 *     FDD_ROPE_BASE     w_i = (base * stretch^(rot_dim / (rot_dim - 2)))^(-2i / rot_dim): the last pair as with LINEAR, the first
 *                       as without
 *     FDD_ROPE_PARTS    w_i = g w + (1 - g) w / stretch, g = clamp((original w / 2 pi - 1) / 31, 0, 1): pairs that turn 32 times
 *                       and more over the `original` length stay, those that turn once or less are stretched; magnitude is
 *                       0.1 ln(stretch) + 1  ("YaRN: Efficient Context Window Extension of Large Language Models", arXiv
 *                       2309.00071: its interpolation by parts and its temperature)
 * and magnitude 1 where none is named.
 *
 * A frequency is held as the part of a turn that one position makes, turns[i] = round(w_i / 2 pi * 2^64) mod 2^64.  A position
 * times it, modulo 2^64, is the angle without the whole turns: to 2^-31 of a turn at every int32 position, also negative
 * ones.  Sine and cosine are within 2^-23 of theirs, all arithmetic is fp32, the result is rounded once.
 *
 * fdd_rope_turns: turns (a HOST array of rot_dim / 2) and magnitude of the table; host-only arithmetic.  A caller
 * copies them to the device once, or fills a table of its own.
 */
enum { FDD_ROPE_NONE = 0, FDD_ROPE_LINEAR = 1, FDD_ROPE_BASE = 2, FDD_ROPE_PARTS = 3 };
typedef struct fdd_rope_scaling {
    int32_t rot_dim;               /* even, 2 .. 1024; FDD_ROPE_BASE: 4 and more */
    int32_t scaling;               /* FDD_ROPE_* */
    double base;                   /* above 1, finite */
    double stretch;                /* at least 1, finite; ignored with FDD_ROPE_NONE */
    double original;               /* positive, finite; FDD_ROPE_PARTS only */
} fdd_rope_scaling;
fdd_status fdd_rope_turns(const fdd_rope_scaling *p, uint64_t *turns, float *magnitude);

typedef struct fdd_rope_table {
    const uint64_t *turns;         /* [rot_dim / 2], 8-byte aligned */
    int32_t rot_dim;               /* even, at least 2, at most the head size */
    int32_t interleaved;           /* 0: pairs (i, i + rot_dim / 2); 1: pairs (2i, 2i + 1) */
    float magnitude;               /* finite */
    int32_t reserved;              /* must be 0 */
} fdd_rope_table;

/* fdd_rope: rows of queries and, if k is given, of keys are rotated, each row at its position.  Consecutive rows of an array
 * lie `stride` elements apart (0 = dense); heads and channels of a row are dense.  q_out may be q itself with the same stride (in
 * place), and k_out k; otherwise no output overlaps anything.  Any alignment of the type; 16-byte aligned rows and a rot_dim
 * whose half is a multiple of 16 bytes are faster.  rows = 0 is a call that does nothing.
 * FDD_ROPE_INVERSE turns the other way, by the same magnitude: the gradient of the rows with respect to what was rotated.
 * A row has one position.  Rows of several (time, row and column of an image's token), each with pairs of its own, take a call in
 * place for each, whose table has 0 for the frequencies of the other pairs, which stay as they are (and magnitude 1 in all calls but one). */
#define FDD_ROPE_INVERSE 1
typedef struct fdd_rope_params {
    int32_t rows, Hq, Hk, D;       /* Hk: heads of k, ignored where k is NULL; D at most 1024 */
    int32_t dtype;                 /* fdd_dtype */
    int32_t flags;                 /* FDD_ROPE_INVERSE */
    fdd_rope_table table;
    const int32_t *positions;      /* [rows] */
    const void *q;                 /* [rows,Hq,D] */
    void *q_out;
    const void *k;                 /* [rows,Hk,D]; may be NULL */
    void *k_out;
    int64_t q_stride, q_out_stride, k_stride, k_out_stride;
    void *stream;
} fdd_rope_params;
fdd_status fdd_rope(const fdd_rope_params *p);

/* ------------------------------------------------------------------------
 * A paged cache.
 *
 * K and V of N requests in pages of page_size rows that any request may take: a head's rows of a page lie together.  Row r of
 * request n is row r mod page_size of page page_table[n][r / page_size].  lens[n] rows are held.  Both lists are DEVICE memory,
 * read when the call runs: a captured call follows them.  What lies behind a request's last row, in pages nobody lists and in
 * entries of the table behind the last page is never used.
 * The library cannot read the lists on the host.  A length is clamped into [0, max_pages * page_size]; rows of a page outside
 * [0, pages) are not written, and read as those of the nearest page there is (nothing is accessed out of bounds).
 */
typedef struct fdd_paged_cache {
    void *k;                       /* [pages,Hkv,page_size,D] */
    void *v;
    const int32_t *page_table;     /* [N,max_pages] */
    const int32_t *lens;           /* [N] */
    int32_t N;
    int32_t pages;
    int32_t page_size;             /* a power of two, 16 .. 1024 */
    int32_t max_pages;             /* max_pages * page_size below 2^30 */
    int32_t Hkv, D;                /* D 64 or 128 */
    int32_t dtype;                 /* fdd_dtype */
    int32_t reserved;              /* must be 0 */
} fdd_paged_cache;

/* fdd_paged_append: rows join the cache behind those that each request holds.  For j in [0, n_rows[n]) source row
 * i = rows[n][j] (rows NULL: i = j) of request n becomes row lens[n] + j, k rotated by `rope` (NULL: as it is) at position
 * positions[n][i], or lens[n] + j where positions is NULL.  lens is not changed: the calls of all layers of a step read the same
 * ones, and the caller adds n_rows once they have been made.  Rows that would lie behind the table's last page and rows
 * whose i is outside [0, B) are not written.  n_rows is clamped into [0, B].  No page may be listed at two places that a call
 * writes.  The source must not overlap the cache, nor K's pages V's. */
typedef struct fdd_paged_append_params {
    int32_t B;                     /* source rows per request */
    int32_t reserved;              /* must be 0 */
    const void *k;                 /* [N,B,Hkv,D]: token (n,b) at (n*B + b) * k_stride */
    const void *v;
    int64_t k_stride, v_stride;    /* elements, rows 16-byte aligned; 0 = Hkv*D */
    const fdd_rope_table *rope;    /* a host struct; may be NULL */
    const int32_t *positions;      /* [N,B]; may be NULL */
    const int32_t *rows;           /* [N,B]; may be NULL */
    const int32_t *n_rows;         /* [N]; may be NULL (= B) */
    void *stream;
} fdd_paged_append_params;
fdd_status fdd_paged_append(const fdd_paged_cache *cache, const fdd_paged_append_params *p);

/* ------------------------------------------------------------------------
 * Trees of drafted tokens.
 *
 * The B tokens of a request are a tree: token 0 is its root, the last token that is certain, and token i > 0 follows token
 * parents[n][i], which is in [0, i).  (A token whose entry is not has no parent: it sees itself only and is never accepted.  The
 * entry of token 0 is not used.)  n_tokens[n] of the B tokens are there, clamped into [0, B].
 *
 * fdd_tree_mask: bit j mod 64 of mask[n][i][j / 64] is set where token j is i itself or one that it follows, through any number of
 * steps; positions[n][i] = lens[n] + the number of those steps.  Tokens that are not there have no bits and position 0.  Outputs
 * overlap nothing.
 */
#define FDD_TREE_MAX 1024
typedef struct fdd_tree_mask_params {
    int32_t N, B;                  /* B at most FDD_TREE_MAX */
    const int32_t *parents;        /* [N,B], or [B] for all requests */
    int64_t parents_stride;        /* entries between requests: at least B, or 0 = one tree for all */
    const int32_t *lens;           /* [N]; may be NULL (= 0) */
    const int32_t *n_tokens;       /* [N]; may be NULL (= B) */
    uint64_t *mask;                /* [N,B,ceil(B/64)] out; may be NULL if positions is not */
    int32_t *positions;            /* [N,B] out; may be NULL if mask is not */
    void *stream;
} fdd_tree_mask_params;
fdd_status fdd_tree_mask(const fdd_tree_mask_params *p);

/* ------------------------------------------------------------------------
 * fdd_paged_attn: attention of every request's new tokens over its paged cache and over one another.
 *
 * For request n, token b < n_tokens[n], query head h (KV head kh = h / (Hq/Hkv)):
 *   keys   = rows [0, lens[n]) of the cache ++ block_k[n, j] for the tokens j < n_tokens[n] that b sees
 *   out[n,b,h,:] = softmax(scale * q[n,b,h,:] . keys^T) values
 * All rows of the cache are seen.  Token b sees token j where bit j mod 64 of mask[n][b][j / 64] is set (fdd_tree_mask, or any
 * other pattern); without a mask all tokens, as in fdd_block_attn, or with FDD_ATTN_CAUSAL_BLOCK those up to b itself.  One token
 * per request (B = 1) is the ordinary decoding step.  Tokens n_tokens[n] .. B are not there: their K and V are not
 * used and their rows of `out` stay as they were.  `out` overlaps nothing.  A row that sees nothing (no cache, no bit) is 0.  Queries and keys arrive rotated.
 *
 * FDD_BF16: products on the matrix cores with fp32 accumulation, softmax in fp32, probabilities rounded to bf16; where a request's
 * keys are cut into pieces, each piece's average is off by 2^-11 of itself or 2^-39 of the row's largest element of it.  FDD_F32: fp32
 * products and sums.  The order of sums depends on lens, n_tokens and max_len of all requests, and on nothing else.
 *
 * Values: q, k and v finite, scores within fp32's range, for what is seen; keys that a row does not see may hold anything.  A NaN
 * or an infinity in V of a token that is there, or in a cached row, reaches all rows of its request and KV head.  FDD_F32 passes a
 * NaN or an infinity in q or in a key on as arithmetic gives it, to the rows that see it (a row whose scores are all -inf is 0).
 * FDD_BF16: such rows are undefined.
 */
typedef struct fdd_paged_attn_params {
    int32_t B, Hq;
    int32_t flags;                 /* FDD_ATTN_CAUSAL_BLOCK; not together with mask */
    int32_t max_len;               /* no request holds more rows (longer ones are cut there); 0 = max_pages * page_size.  Sizes the workspace. */
    float scale;                   /* softmax scale; <= 0 selects 1/sqrt(D) */
    int32_t reserved;              /* must be 0 */
    const void *q;                 /* [N,B,Hq,D]: token (n,b) at (n*B + b) * q_stride; likewise block_k, block_v */
    const void *block_k;           /* [N,B,Hkv,D] */
    const void *block_v;
    int64_t q_stride, k_stride, v_stride;   /* elements, tokens 16-byte aligned; 0 = dense */
    const uint64_t *mask;          /* [N,B,ceil(B/64)], or [B,ceil(B/64)] for all requests; may be NULL */
    int64_t mask_stride;           /* words between requests: at least B*ceil(B/64), or 0 = one mask for all */
    const int32_t *n_tokens;       /* [N]; may be NULL (= B) */
    void *out;                     /* [N,B,Hq,D] */
    void *workspace;               /* >= fdd_paged_attn_workspace() bytes */
    size_t workspace_bytes;
    void *stream;
} fdd_paged_attn_params;
/* Bytes of scratch (host-only arithmetic; 0 for invalid params and for calls that need none). */
size_t fdd_paged_attn_workspace(const fdd_paged_cache *cache, const fdd_paged_attn_params *p);
fdd_status fdd_paged_attn(const fdd_paged_cache *cache, const fdd_paged_attn_params *p);

/* ------------------------------------------------------------------------
 * fdd_tree_verify: which drafted tokens stand, from given random numbers, so that what is emitted is distributed as if the target
 * model had drawn token after token.
 *
 * logits[n,i,:] is the target's distribution of the token behind token i: p_i = softmax(logits[n,i,:] / temperature).  A walk
 * starts at token 0.  At token i its children (tokens j with parents[n][j] == i, lowest j first) are tried:
 *   temperature 0      child j stands where tokens[n][j] is the lowest id attaining the largest logit; if none does, that id is
 *                      emitted and the walk ends.
 *   temperature > 0    w = p_i, W = 1.  Child j with token x stands where  uniforms[n][j][0] * q(x) * W < w(x),  with q(x) = 1, or
 *                      with draft_logits q_i = softmax(draft_logits[n,i,:] / draft_temperature), from which x was drawn.
 *                      Otherwise what the draft accounts for is taken out: w(x) = 0, or with draft_logits
 *                      w = max(p_i - q_i, 0); W = sum w.  If none stands, the token drawn from w by uniforms[n][i][1] = u
 *                      is emitted, the lowest id v with w(0) + .. + w(v) > u * W, and the walk ends; where W < 2^-40 it is drawn
 *                      from p_i instead.
 * A child that stands is emitted and the walk goes on there.  So a walk of k tokens emits k: path[n] = (0, the tokens that
 * stand), n_path[n] = k, emitted[n] = (what stands, the token drawn at the end); entries of path and emitted behind k are -1.  A
 * request without tokens gets n_path 0.  The accepted rows of K and V are path's: `rows` and `n_rows` of fdd_paged_append.
 * chances[n][j] is the probability with which token j stands when it is tried first: min(1, p(x) / q(x)); 1 for token 0, 0
 * for tokens that are not there or have no parent; with temperature 0 it is 1 or 0.
 *
 * draft_logits go with chains only (parents NULL: token j follows j - 1); tokens of a tree count as chosen, not drawn.  With
 * temperature 0 they have no part.  Only rows of tokens that are there are read, of draft_logits only those that another
 * token follows.  Tokens outside [0, V) never stand (with q(x) = 1 they take nothing out).  Uniforms are in [0, 1).
 *
 * In a test or a chance p(x) and q(x) are off by 2^-16 of themselves, however small they are, and W, without draft_logits, by 2^-16 of
 * what was taken out of it (a row's fp32 exponentials are summed in fp64, all else is fp64; chances are rounded to fp32); what the last token is
 * drawn from is fp64 throughout.  Logits: finite values and -inf for entries that can never be
 * chosen, a row that is read needs one finite entry.  NaN and +inf are not supported: such a request's outputs are undefined
 * (ids stay in range).  Outputs overlap nothing.
 */
typedef struct fdd_tree_verify_params {
    int32_t N, B;                  /* B at most FDD_TREE_MAX */
    int64_t V;                     /* at most 2^30 */
    int32_t dtype;                 /* fdd_dtype of logits and draft_logits */
    float temperature;             /* 0, or 2^-20 .. 2^20 */
    float draft_temperature;       /* 2^-20 .. 2^20; draft_logits only */
    int32_t reserved;              /* must be 0 */
    const void *logits;            /* [N,B,V] */
    const void *draft_logits;      /* [N,B,V]; may be NULL; ignored with temperature 0 */
    const int32_t *tokens;         /* [N,B] */
    const int32_t *parents;        /* [N,B], or [B] for all requests; may be NULL (= a chain) */
    int64_t parents_stride;        /* entries between requests: at least B, or 0 = one tree for all */
    const float *uniforms;         /* [N,B,2]; may be NULL with temperature 0 */
    const int32_t *n_tokens;       /* [N]; may be NULL (= B) */
    int32_t *path;                 /* [N,B] out */
    int32_t *n_path;               /* [N] out */
    int32_t *emitted;              /* [N,B] out */
    float *chances;                /* [N,B] out; may be NULL */
    void *workspace;               /* >= fdd_tree_verify_workspace() bytes */
    size_t workspace_bytes;
    void *stream;
} fdd_tree_verify_params;
size_t fdd_tree_verify_workspace(const fdd_tree_verify_params *p);
fdd_status fdd_tree_verify(const fdd_tree_verify_params *p);

/* ------------------------------------------------------------------------
 * Rollout-fork bookkeeping ("fork the KV cache N times").
 *
 * fdd_fork_block: dst[n] = src for n in [0,N), `bytes` bytes each: the
 * private per-rollout state (block K/V, tokens, mask) of the forked
 * rollouts.  The prefix is shared by pointer and is not an argument.
 * bytes must be a multiple of 4; src and dst must not overlap.
 */
fdd_status fdd_fork_block(int32_t N, size_t bytes, const void *src, void *dst, void *stream);

/* fdd_block_commit: a finished block joins its rollout's extension,
 * ext_k[n, E..E+B) = block_k[n], ext_v likewise; the caller then passes E + B as
 * the extension length of the next block's attention calls.  E + B must not
 * exceed ext_capacity; pointers 16-byte aligned; the arrays must not overlap. */
typedef struct fdd_commit_params {
    int32_t N, B, Hkv, D;
    int32_t dtype;
    int32_t E;                     /* rows already in the extension */
    int32_t ext_capacity;
    int32_t reserved;              /* must be 0 */
    const void *block_k;           /* [N,B,Hkv,D] */
    const void *block_v;
    void *ext_k;                   /* [N,ext_capacity,Hkv,D] in/out */
    void *ext_v;
    void *stream;
} fdd_commit_params;

fdd_status fdd_block_commit(const fdd_commit_params *p);

/* fdd_traj_mean: trajectory averaging (paper, "Trajectory averaging", the merge
 * equation): out[p] = (1/N) sum_n traj[n,p], p in [0,P), P = waypoints x
 * coordinates.  fp32 in and out; the sum runs over n in ascending order in
 * fp32, so the result is reproducible and within N * 2^-24 relative of the
 * exact mean of the absolute values.  (The jerk-minimizing fit that produces
 * the waypoints of a rollout is not specified by the paper and is not here.) */
fdd_status fdd_traj_mean(int32_t N, int32_t P, const float *traj, float *out, void *stream);

/* fdd_block_kv_update: refresh the K/V rows of positions committed by the
 * last unmask step.  No model is inside this library, so the new row of a
 * position holding token t is row (t mod T) of caller-provided tables: a
 * stand-in for embedding + projection.  Rows of other positions are not
 * touched. */
typedef struct fdd_kv_update_params {
    int32_t N, B, Hkv, D, T;
    int32_t dtype;                 /* fdd_dtype of the tables and the block K/V */
    const int32_t *tokens;         /* [N,B] */
    const uint8_t *committed;      /* [N,B] as written by fdd_unmask_step */
    const void *table_k;           /* [T,Hkv,D] */
    const void *table_v;           /* [T,Hkv,D] */
    void *block_k;                 /* [N,B,Hkv,D] in/out */
    void *block_v;                 /* [N,B,Hkv,D] in/out */
    void *stream;
} fdd_kv_update_params;

fdd_status fdd_block_kv_update(const fdd_kv_update_params *p);

/* ------------------------------------------------------------------------
 * Timing hook for benchmarks.  While set (both non-NULL), every
 * fdd_block_attn call made by this host thread records `start` on the call's
 * stream right before the main attention kernel (after the pre-pass that
 * repacks V, when there is one) and `stop` right after it (before the small
 * merge kernel), so hipEventElapsedTime(start, stop) is that kernel's
 * duration.  Both are hipEvent_t passed as void*, owned by the
 * caller.  Pass NULL, NULL to clear.  Not meant for production loops.
 */
fdd_status fdd_profile_attn_events(void *start, void *stop);

/* Message of the last failing call on this thread ("" if none). */
const char *fdd_last_error(void);
/* major*10000 + minor*100 + patch */
int fdd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* FDD_H */
