/*
 * dit_attn.h - C ABI of the MI355X (gfx950) DiT denoising-step self-attention.
 *
 * One call computes, for a packed batch of independent token sequences, the
 * self-attention of a DiT block during one denoising step:
 *
 *     for every sequence i with rows R_i = [cu_seqlens[i], cu_seqlens[i+1]),
 *     every head h and every query row r in R_i:
 *         O[r,h,:] = sum_{j in R_i} softmax_j( scale * <Q[r,h,:], K[j,h,:]> ) * V[j,h,:]
 *
 * The batch is what the paper's serving loop hands to a GPU for one step:
 * same-resolution image requests coalesced into one call (paper Section 4.3,
 * "SLO-aware Dynamic Batching"), a whole video request (Section 4.4, one
 * request per GPU set), or one GPU's head subset of a sequence-parallel video
 * (Section 5, Unified Sequence Parallel attention; Section 4.3, "Elastic
 * Sequence Parallelism").  Attention is bidirectional inside a sequence and
 * never crosses sequences.  Text and latent tokens are ordinary rows.
 *
 * Precision: bf16 inputs, fp32 scores / softmax state / accumulators, the
 * probabilities are rounded to bf16 (nearest-even) before the second
 * contraction and the row sum l is taken over the rounded values (O / l is
 * then a convex combination of V rows whatever the rounding did; lse carries
 * at most their 2^-8 relative error, i.e. 4e-3 absolute), bf16 output
 * (nearest-even).  The softmax reference value of a row follows its running
 * maximum lazily (it moves when exceeded by more than 8 in the base-2
 * exponent); the quotient O / l does not depend on it.
 *
 * All functions are thread-compatible, not thread-safe: one context must not
 * be used from two host threads, or for two streams, at the same time.
 * No C++ exception crosses this boundary.
 */
#ifndef DIT_ATTN_H_
#define DIT_ATTN_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes. */
#define DIT_ATTN_OK                 0
#define DIT_ATTN_ERR_NULL          (-1)  /* a required pointer is NULL */
#define DIT_ATTN_ERR_HEAD_DIM      (-2)  /* head_dim is not 64 or 128 */
#define DIT_ATTN_ERR_CU_SEQLENS    (-3)  /* cu_seqlens[0] != 0, decreasing, or n_seqs < 0 */
#define DIT_ATTN_ERR_HIP           (-4)  /* a HIP runtime call failed; see dit_attn_last_error */
#define DIT_ATTN_ERR_SCALE         (-5)  /* scale is NaN or infinite */
#define DIT_ATTN_ERR_N_HEADS       (-6)  /* n_heads < 1 or > 65535 */
#define DIT_ATTN_ERR_ALIGN         (-7)  /* q, k, v or out is not 16-byte aligned */
#define DIT_ATTN_ERR_CAPACITY      (-8)  /* output buffer of dit_attn_plan too small */
#define DIT_ATTN_ERR_KERNEL        (-9)  /* dit_attn_set_kernel: no such kernel */
#define DIT_ATTN_ERR_PARTS         (-10) /* dit_attn_merge: n_parts outside 1..8 */
#define DIT_ATTN_ERR_LIMIT         (-11) /* dit_attn_varlen_fwd_noalloc: the pack exceeds the fixed scratch limits; elsewhere: more rows than a launch takes */
#define DIT_ATTN_ERR_CAPTURE       (-12) /* the stream is capturing and the call would have to allocate or copy */
#define DIT_ATTN_ERR_MASK          (-13) /* dit_attn_mask: a field out of range, or one without the one it belongs to */
#define DIT_ATTN_ERR_ROPE          (-14) /* dit_attn_rope, rot_dim or layout out of range */
#define DIT_ATTN_ERR_NORM          (-15) /* no such norm, eps out of range, or weights without a norm */
#define DIT_ATTN_ERR_STRIDE        (-16) /* a row stride that is no multiple of 8, too short for a row or too long; one side's rows are the other's */

typedef struct dit_attn_ctx dit_attn_ctx; /* opaque */

/*
 * Create a context bound to HIP device `device_id` (host call).
 * The context owns a small amount of device memory: cached work-lists (one per
 * distinct (cu_seqlens, n_heads, head_dim) seen, 16 bytes per work item) and a
 * work counter.  *out_ctx is written only on success.
 * Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL, or DIT_ATTN_ERR_HIP (no such device,
 * not a gfx950 device, allocation failure).
 */
int dit_attn_create(dit_attn_ctx** out_ctx, int device_id);

/*
 * One denoising-step attention call over a packed variable-length batch
 * (paper Sections 4.3 and 5; the math is the definition at the top of this file).
 *
 *   q, k, v     DEVICE pointers, bf16, shape [T, n_heads, head_dim], contiguous
 *               (row stride n_heads*head_dim elements), T = cu_seqlens[n_seqs].
 *               16-byte aligned.  Read only.
 *   cu_seqlens  HOST pointer, n_seqs + 1 int32 entries, cu_seqlens[0] == 0,
 *               non-decreasing.  Read during the call only (the batch is formed
 *               by host code, which knows the lengths).  Zero-length sequences
 *               are legal and contribute no rows.
 *   n_seqs      number of sequences, >= 0.  n_seqs == 0 or T == 0: returns
 *               DIT_ATTN_OK and launches nothing.
 *   n_heads     heads in q, k and v alike (no grouped-query sharing), 1..65535.
 *   head_dim    64 or 128.
 *   scale       multiplies the fp32 scores before the softmax; any finite value
 *               (zero and negative included).
 *   out         DEVICE pointer, bf16, same shape and layout as q; must not
 *               overlap q, k or v.  Exactly the rows [0, T) are written.
 *   stream      a hipStream_t (as void*); NULL is the default stream.
 *
 * The work is enqueued on `stream`; the call does not synchronise.  The first
 * call with a new (cu_seqlens, n_heads, head_dim) builds a work-list on the host
 * and uploads it (one device allocation and one synchronous copy); later
 * calls with the same pack reuse it and do no host work beyond a compare.
 * Under HIP graph capture only such a later call is possible (else DIT_ATTN_ERR_CAPTURE); the captured pack stays
 * cached until the context is destroyed (see dit_attn_plan_cache_victim).
 * The caller keeps ownership of every buffer.  Validation precedes any launch:
 * on a non-zero return `out` is untouched.
 */
int dit_attn_varlen_fwd(dit_attn_ctx* ctx,
                        const void* q, const void* k, const void* v,
                        const int32_t* cu_seqlens, int32_t n_seqs,
                        int32_t n_heads, int32_t head_dim, float scale,
                        void* out, void* stream);

/*
 * For callers that cannot allocate device memory: code being recorded into a HIP graph that meets a pack for the first
 * time, tight serving loops, harnesses that forbid hipMalloc.  The same operation as dit_attn_varlen_fwd, same
 * arguments, same result bit for bit, but the call allocates nothing and copies nothing: the work-list is written by a
 * small kernel on `stream` (the sequence boundaries travel as its argument) into a fixed device array of the library
 * (256 KB + 256 B per GPU, held until the process ends), which also holds the kernels' work counters.  A pack of at most
 * 16 sequences whose items all start at once touches no part of that array: its boundaries travel with the attention
 * kernel.
 * Limits: n_seqs <= 64 and at most 16384 work items per pack (an item is 256 query rows of one head, 128 for packs that
 * the 128-row kernel runs; the five benchmark configurations need 64 to 4632); beyond them DIT_ATTN_ERR_LIMIT, `out`
 * untouched.  Unless a kernel is forced, a pack that exceeds the limit only in 128-row items runs the ping-pong kernel.
 * No split-KV, no plan cache, dit_attn_last_launch_clock is not updated.
 * The other packs on a GPU share that GPU's array: calls with such packs that overlap on one GPU (two streams, contexts or
 * threads) race; calls on one stream are ordered and safe.  Other return codes as dit_attn_varlen_fwd.
 */
int dit_attn_varlen_fwd_noalloc(dit_attn_ctx* ctx,
                                const void* q, const void* k, const void* v,
                                const int32_t* cu_seqlens, int32_t n_seqs,
                                int32_t n_heads, int32_t head_dim, float scale,
                                void* out, void* stream);

/*
 * Destroy a context and free its device memory (host call).  The caller must
 * have synchronised every stream the context was used on.  NULL is a no-op.
 */
void dit_attn_destroy(dit_attn_ctx* ctx);

/*
 * The same operation, also returning the row-wise log-sum-exp
 *     lse[r, h] = ln sum_j exp(scale * <Q[r,h,:], K[j,h,:]>)     (natural log, fp32, [T, H] contiguous, DEVICE)
 * which is what makes results over disjoint key sets combinable (dit_attn_merge).  Sequence parallelism along the
 * sequence - the ring half of the unified sequence parallelism that the paper's elastic SP builds on (Section 5,
 * Section 4.3) - hands a GPU one block of keys per step and needs exactly this pair per block.
 * lse must be 4-byte aligned and hold total_tokens * n_heads floats; everything else as dit_attn_varlen_fwd.
 * Accuracy contract: |lse - exact| <= 4e-3.  The sum inside the logarithm is taken over the probabilities as rounded to
 * bf16 for the second contraction (each within 2^-8 relative, all positive), so lse is within ln(1 + 2^-8) = 3.9e-3
 * of the exact value plus ~1e-5 of fp32 arithmetic; the bound is approached only by rows that one key dominates
 * (typically < 1e-3).  In exchange a merge that uses these lse values reproduces exactly the quotient that a single
 * pass over all keys forms from the same rounded probabilities.
 */
int dit_attn_varlen_fwd_lse(dit_attn_ctx* ctx,
                            const void* q, const void* k, const void* v,
                            const int32_t* cu_seqlens, int32_t n_seqs,
                            int32_t n_heads, int32_t head_dim, float scale,
                            void* out, float* lse, void* stream);

/*
 * Cross-attention over a packed batch (paper Section 2.1: the DiT blocks also attend to the text tokens for text
 * alignment): queries and keys have separate boundaries.  Sequence i's query rows
 * cu_seqlens_q[i] .. cu_seqlens_q[i+1] of q ([Tq, H, D]) see key rows cu_seqlens_k[i] .. cu_seqlens_k[i+1] of k and v
 * ([Tk, H, D]); both arrays are HOST pointers with n_seqs + 1 entries starting at 0, non-decreasing.  out is
 * [Tq, H, D]; lse ([Tq, H], DEVICE) may be NULL.  Query rows of a sequence that has no keys get O = 0 and
 * lse = -inf (an empty sum).  Errors and all other arguments as dit_attn_varlen_fwd.
 */
int dit_attn_cross_varlen_fwd(dit_attn_ctx* ctx,
                              const void* q, const void* k, const void* v,
                              const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t n_seqs,
                              int32_t n_heads, int32_t head_dim, float scale,
                              void* out, float* lse, void* stream);

/*
 * Merge n_parts (1..8) partial results of the SAME queries over DISJOINT key sets (paper Section 5: sequence
 * parallelism splits a long video's sequence over GPUs; each block of keys yields one partial result):
 *     lse = ln sum_p exp(lse_p),     O = sum_p exp(lse_p - lse) O_p.
 * o_parts / lse_parts: HOST arrays of n_parts DEVICE pointers, each to bf16 [total_rows, H, D] / fp32
 * [total_rows, H] as written by dit_attn_varlen_fwd_lse or dit_attn_cross_varlen_fwd.  A part whose lse is -inf in a
 * row has weight 0 there; a row whose parts are all -inf becomes 0 with lse -inf.  out may alias one of the parts;
 * lse_out may be NULL.  fp32 arithmetic, bf16 output rounded to nearest even.  Enqueues one kernel on `stream`.
 * Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL, _HEAD_DIM, _N_HEADS, _PARTS, _CU_SEQLENS (total_rows < 0), _ALIGN, _HIP.
 */
int dit_attn_merge(dit_attn_ctx* ctx,
                   const void* const* o_parts, const float* const* lse_parts, int32_t n_parts,
                   int64_t total_rows, int32_t n_heads, int32_t head_dim,
                   void* out, float* lse_out, void* stream);

/*
 * Single-GPU halves of the head-split sequence-parallel exchange (paper Section 4.3: elastic sequence parallelism
 * gives a video p in {1,2,4,8} GPUs; Section 5: the head-split half of the unified sequence parallelism).  A rank
 * holds n_rows rows of the sequence with all n_heads heads; attention needs the whole sequence for n_heads / p heads.
 *     pack:    src [n_rows, H, D]        -> dst [p, n_rows, H/p, D]   dst[g, r, h, :] = src[r, g*H/p + h, :]
 *     unpack:  src [p, n_rows, H/p, D]   -> dst [n_rows, H, D]        dst[r, g*H/p + h, :] = src[g, r, h, :]
 * Block g of pack's output is what goes to rank g before attention (the blocks a rank receives, in source-rank order,
 * are its [L, H/p, D] input without further copying); unpack's input is the blocks a rank receives after attention,
 * in source-rank order.  bf16, DEVICE buffers, 16-byte aligned, src and dst must not overlap.  sp_degree (p) >= 1 must
 * divide n_heads.  Enqueues one kernel on `stream`; moves every byte once (HBM bound).
 * Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL, _HEAD_DIM, _N_HEADS (also: p does not divide n_heads), _CU_SEQLENS
 * (n_rows < 0), _ALIGN, _HIP.
 */
int dit_attn_sp_pack_heads(dit_attn_ctx* ctx, const void* src, void* dst, int64_t n_rows,
                           int32_t n_heads, int32_t head_dim, int32_t sp_degree, void* stream);
int dit_attn_sp_unpack_heads(dit_attn_ctx* ctx, const void* src, void* dst, int64_t n_rows,
                             int32_t n_heads, int32_t head_dim, int32_t sp_degree, void* stream);

/*
 * Rotation table of token positions: what dit_attn_qk_norm_rope turns queries and keys by.  A DiT's tokens have positions on
 * several axes (text; frame, row, column), each of which rotates a share of a head's elements.  The table is a function of the
 * positions alone: made once for a pack, it serves every block of every denoising step.
 *     table[r, pair] = magnitude * (cos, sin)(positions[r, axis of pair] * f(pair))
 * The pairs of axis 0 come first.  With d = axis_dim[a] elements (d / 2 pairs j) and base theta[a]:
 *     DIT_ATTN_ROPE_PLAIN    f = theta^(-2j/d)
 *     DIT_ATTN_ROPE_LINEAR   f = theta^(-2j/d) / factor                    positions squeezed into the trained range
 *     DIT_ATTN_ROPE_BASE     f = (theta * factor^(d/(d-2)))^(-2j/d)        fast pairs kept, slow ones squeezed (d = 2: plain)
 *     DIT_ATTN_ROPE_BANDS    f = theta^(-2j/d) * (g + (1-g) / factor),     pairs that turn `high` times and more over
 *                            g = clamp((turns - low) / (high - low)),      original_length kept, those under `low` squeezed,
 *                            turns = original_length * theta^(-2j/d) / 2pi   a blend in between
 * Angles are computed in double precision: any int32 position has a table entry within a few units of fp32 rounding.
 *   positions  DEVICE int32 [n_rows, n_axes], contiguous.      n_rows >= 0 (0: nothing is launched).
 *   rope       HOST, read during the call.
 *   table      DEVICE fp32 [n_rows, sum of axis_dim / 2, 2] (cos, sin), 16-byte aligned.
 * Enqueues one kernel on `stream`; allocates nothing.  Returns DIT_ATTN_OK, _ERR_NULL, _ROPE, _CU_SEQLENS (n_rows < 0), _ALIGN,
 * _LIMIT (over 2^34 rows, or more than a launch takes: with 64 pairs 2^29) or _HIP.
 */
#define DIT_ATTN_ROPE_PLAIN   0
#define DIT_ATTN_ROPE_LINEAR  1
#define DIT_ATTN_ROPE_BASE    2
#define DIT_ATTN_ROPE_BANDS   3
typedef struct dit_attn_rope {
  int32_t n_axes;              /* 1..4 */
  int32_t scaling;             /* DIT_ATTN_ROPE_PLAIN .. DIT_ATTN_ROPE_BANDS */
  int32_t axis_dim[4];         /* rotated elements of an axis: even, at least 2; at most 128 together */
  double theta[4];             /* base of an axis, at least 1 */
  double factor[4];            /* at least 1; not read with DIT_ATTN_ROPE_PLAIN */
  double original_length[4];   /* DIT_ATTN_ROPE_BANDS: positions of the trained range */
  double low, high;            /* DIT_ATTN_ROPE_BANDS: low < high */
  double magnitude;            /* multiplies both values; 1 for a rotation */
} dit_attn_rope;
int dit_attn_rope_table(dit_attn_ctx* ctx, const int32_t* positions, int64_t n_rows, const dit_attn_rope* rope,
                        float* table, void* stream);

/*
 * Norm of queries and keys for each head and rotation by position in one pass, as a DiT block does right before its attention
 * (paper Section 2.1: the denoising steps' attention over text and latent tokens).  For each row and head, in fp32:
 *     DIT_ATTN_NORM_RMS     y = x * rsqrt(mean(x^2) + eps) * weight + bias
 *     DIT_ATTN_NORM_LAYER   y = (x - mean(x)) * rsqrt(var(x) + eps) * weight + bias       (var: mean of squares)
 *     DIT_ATTN_NORM_NONE    y = x
 * (means are over the elements of one head: a norm over all heads of a row is another operation)
 * then the first rot_dim elements are turned in pairs, (a, b) -> (a cos - b sin, b cos + a sin) with the row's table entry of
 * the pair, and the result is rounded once to bf16.  Pair j is
 *     DIT_ATTN_ROPE_INTERLEAVED  (2j, 2j + 1)          DIT_ATTN_ROPE_HALF  (j, j + rot_dim / 2)
 *   q, k        HOST structures, read during the call; one of them may be NULL (only the other side is done).
 *     x, out    DEVICE bf16, n_rows rows of n_heads * head_dim elements, 16-byte aligned, row_stride / out_row_stride elements
 *               apart (0: contiguous; a multiple of 8).  So x may lie in the output of a fused projection.  out == x (with equal
 *               strides) replaces the rows in place; otherwise no out overlaps any input.
 *     weight, bias  DEVICE fp32 [head_dim], 16-byte aligned, or NULL (1 and 0).
 *   n_rows      >= 0 (0: nothing is launched).      head_dim  64 or 128.      eps  finite, not negative.
 *   table       DEVICE fp32 [n_rows, rot_dim / 2, 2] (cos, sin) as dit_attn_rope_table writes it, 16-byte aligned; not read with
 *               rot_dim == 0.
 *   rot_dim     rotated elements of a head, a multiple of 8 up to head_dim; the others are only normed.
 * Enqueues one kernel on `stream`; allocates nothing.  Returns DIT_ATTN_OK, _ERR_NULL, _HEAD_DIM, _N_HEADS, _NORM, _ROPE,
 * _STRIDE, _CU_SEQLENS (n_rows < 0), _ALIGN, _LIMIT (over 2^34 rows, or more than a launch takes: 2^24 groups of up to four heads
 * of one side and 2048 / head_dim rows) or _HIP.
 */
#define DIT_ATTN_NORM_NONE          0
#define DIT_ATTN_NORM_RMS           1
#define DIT_ATTN_NORM_LAYER         2
#define DIT_ATTN_ROPE_INTERLEAVED   0
#define DIT_ATTN_ROPE_HALF          1
typedef struct dit_attn_norm_heads {
  const void* x;
  void* out;
  int64_t row_stride, out_row_stride;
  const float* weight;
  const float* bias;
  int32_t n_heads;             /* 1..65535 */
} dit_attn_norm_heads;
int dit_attn_qk_norm_rope(dit_attn_ctx* ctx, const dit_attn_norm_heads* q, const dit_attn_norm_heads* k, int64_t n_rows,
                          int32_t head_dim, int32_t norm, float eps, const float* table, int32_t rot_dim, int32_t layout,
                          void* stream);

/*
 * Attention with masks, capped scores and a distance bias, over a pack with separate query and key boundaries and key heads
 * shared by groups of query heads.  Row i of a sequence with lq queries and lk keys has position pos = i + lk - lq (its
 * queries are the last of its keys: one new token has lq = 1); head h reads key head h / (n_heads / n_kv_heads).
 *     s = scale * <q, k_j>;   softcap C > 0: s = C * tanh(s / C);   slopes: s = s - slopes[h] * |pos - j|
 *     key j is seen  iff  (not causal, or j <= pos, or j < prefix of the sequence)
 *                     and (no ids, or q_doc of the row == k_doc of the key, and that id is not negative)
 *     out = sum over seen keys exp(s - lse) v_j,     lse = ln sum over seen keys exp(s)
 * Scores are fp32: a capped one is within 1e-6 of its value, a biased one within a few roundings of the bias.
 * A row that sees no key gets 0 and -inf.  What lies in keys and values that a row does not see (NaN and infinities too) has no
 * effect on it.  So a padded batch gives its padding rows negative ids, several documents of a sequence get an id each (in any
 * order), and text that all of an ordered sequence sees is its prefix.
 *   q           DEVICE bf16 [Tq, n_heads, head_dim];  k, v  DEVICE bf16 [Tk, n_kv_heads, head_dim];  16-byte aligned.
 *   row_strides HOST, elements from row to row of q, k and v (multiples of 8, at most 2^24; 0: contiguous), or NULL: contiguous.
 *               The heads of a row are contiguous.
 *   cu_seqlens_q, cu_seqlens_k   HOST, as dit_attn_cross_varlen_fwd; cu_seqlens_k may be NULL: keys share the query boundaries.
 *               Any number of sequences.  The keys of a sequence follow those of the one before it: there is no room between
 *               caches to grow into, so a program that adds a token to each either moves them or makes a call for each.
 *   n_kv_heads  divides n_heads.      head_dim  64 or 128.      scale  finite.
 *   mask        HOST structure, read during the call, or NULL: every key is seen.
 *   out         DEVICE bf16 [Tq, n_heads, head_dim], contiguous, overlapping no input.  Exactly the rows [0, Tq) are written.
 *   lse         DEVICE fp32 [Tq, n_heads] or NULL.  Its sum is taken over fp32 probabilities (the products with v take them as
 *               bf16, and out is divided by the sum of those).
 * The call reads no work-list and builds none: boundaries travel with the kernel.  Sequences with few rows or packs with few
 * items have their keys split over the compute units and the parts joined by a second kernel, in a fixed order (the same pack
 * gives the same bits; a sequence's bits depend on what it is packed with).  The parts, and the id ranges of key tiles, lie in
 * the context's workspace, which grows with hipMalloc when a call needs more (DIT_ATTN_ERR_CAPTURE on a capturing stream: call
 * once outside the capture first).  As with every use of a context, calls and replays of captured calls that use the workspace
 * must not overlap.
 * Returns DIT_ATTN_OK, _ERR_NULL, _HEAD_DIM, _N_HEADS, _CU_SEQLENS, _SCALE, _MASK, _STRIDE, _ALIGN, _LIMIT (2^31 work items),
 * _CAPTURE or _HIP; validation precedes any launch.
 */
typedef struct dit_attn_mask {
  int32_t causal;              /* 0 or 1 */
  float softcap;               /* C, or 0: scores are not capped */
  const int32_t* prefix;       /* HOST [n_seqs], not negative, with causal = 1; or NULL: 0 */
  const float* slopes;         /* DEVICE fp32 [n_heads], or NULL: no bias */
  const int32_t* q_doc;        /* DEVICE int32 [Tq] and [Tk], or both NULL (one of no elements may be NULL too) */
  const int32_t* k_doc;
} dit_attn_mask;
int dit_attn_masked_varlen_fwd(dit_attn_ctx* ctx,
                               const void* q, const void* k, const void* v, const int64_t* row_strides,
                               const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t n_seqs,
                               int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, float scale,
                               const dit_attn_mask* mask, void* out, float* lse, void* stream);

/*
 * Kernel choice of a context.  The library has two kernels for the same
 * operation (which one is fastest depends on the pack, Section 4.3 / Table 3:
 * image steps are short, video steps long):
 *     DIT_ATTN_KERNEL_AUTO   (-1) chosen per pack from the lengths, n_heads and
 *                                 head_dim (and the number of compute units):
 *                                 the 128-row kernel while every 128-row item
 *                                 has a compute unit and for cross-attention
 *                                 against few keys (320 per item on average;
 *                                 head_dim 64: 129 to 320); the ping-pong
 *                                 kernel where the 256-row items take no
 *                                 longer than the longest of them.  Past that,
 *                                 head_dim 64: the 128-row kernel, but not for
 *                                 self-attention whose short, well filled
 *                                 items are two rounds of the ping-pong kernel
 *                                 and more than one of this; head_dim 128: the
 *                                 ping-pong kernel unless its second round, or
 *                                 a third one of equal items, would be at most
 *                                 half full (a second one of self-attention
 *                                 with up to eleven tiles of 64 keys per item
 *                                 three sevenths, and not with 12 to 18), or
 *                                 (cross-attention) its items have at most
 *                                 eleven tiles on average
 *     DIT_ATTN_KERNEL_128     (0) 128 query rows per tile
 *     DIT_ATTN_KERNEL_PINGPONG(1) 256 rows per tile, two alternating groups
 * The kernels do the same arithmetic in the same order: their results agree
 * bit for bit.  A forced kernel applies to later calls on `ctx`; meant for
 * tests and measurements.
 * Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL or DIT_ATTN_ERR_KERNEL.
 */
#define DIT_ATTN_KERNEL_AUTO     (-1)
#define DIT_ATTN_KERNEL_128        0
#define DIT_ATTN_KERNEL_PINGPONG   1
int dit_attn_set_kernel(dit_attn_ctx* ctx, int kernel);

/*
 * Split-KV for small packs (paper Section 3 / Table 3: a low-resolution image step is far too small to fill a GPU).
 * With max_splits > 1, a pack whose work items leave at least half of the compute units idle has the keys of every
 * sequence cut into up to max_splits chunks: as many as fit one round of one item per compute unit and at most one per eight
 * tiles of 64 keys of the shortest sequence, where that is quicker on MI355X than the unsplit call.  Where two 128-row items
 * per compute unit fit, the chunks run on the 128-row kernel if the shortest sequence has under 64 tiles and the split takes
 * at least 12 of them (head_dim 64: 13) off every item, else on the ping-pong kernel, where it has to take 17.  Without that
 * room a pack is split only if its longest sequence has 128 tiles, on the ping-pong kernel.  (The partial results and their
 * merge cost about 8 us.)  The chunks of a sequence have equal numbers of tiles but for the last, which takes what is left
 * (65 tiles in eight chunks: seven of 9 tiles and one of 2).  They run as separate items that leave normalised fp32 partial
 * results and their log-sum-exp in a workspace owned by the context (grown with hipMalloc when a call needs more), and one
 * merge kernel on the same stream writes `out`.  Off (max_splits = 1) by default, because it changes the summation order: with it
 * a sequence's bits depend on what it is packed with (they stay within the same tolerance of the exact result).
 * Applies to every forward entry point but dit_attn_masked_varlen_fwd, which splits by itself.  Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL or DIT_ATTN_ERR_PARTS (outside 1..8).
 */
int dit_attn_set_split_kv(dit_attn_ctx* ctx, int max_splits);

/*
 * Clock sample of the last kernel launched through `ctx`: the first workgroup
 * of every launch reads the GPU's shader-cycle counter and its constant 100 MHz
 * counter when it starts and when it ends.  shader_mhz is the ratio (the clock
 * the chip sustained under that kernel; MI355X lowers it under matrix load, so
 * throughput at a fixed number of cycles per tile moves with it); kernel_ms is
 * how long that workgroup ran.  Either pointer may be NULL; both values are 0
 * before the first launch.  Synchronises the whole device.
 * Returns DIT_ATTN_OK, DIT_ATTN_ERR_NULL or DIT_ATTN_ERR_HIP.
 */
int dit_attn_last_launch_clock(dit_attn_ctx* ctx, double* shader_mhz, double* kernel_ms);

/*
 * Which attention kernel the last forward call on `ctx` launched:
 * DIT_ATTN_KERNEL_128 or DIT_ATTN_KERNEL_PINGPONG, or DIT_ATTN_KERNEL_AUTO (-1)
 * if no attention kernel has been launched yet.  For measurements that name
 * the kernel they timed.  Host state only; NULL returns DIT_ATTN_KERNEL_AUTO.
 */
int dit_attn_last_launch_kernel(const dit_attn_ctx* ctx);

/*
 * Text of the last error recorded in `ctx` (or of the last failed
 * dit_attn_create when ctx is NULL).  The string is owned by the library and
 * valid until the next call on the same context.
 */
const char* dit_attn_last_error(const dit_attn_ctx* ctx);

/*
 * Host-only: the work-list that dit_attn_varlen_fwd would run for this pack,
 * in execution order (paper Section 4.3: a batch mixes requests of different
 * lengths; the list balances their tiles over compute units by handing out the
 * costliest items first).  Needs no GPU and no context.
 *
 * Each item is one (sequence, head, query tile): 4 int32 values
 *     [0] q_start   first global query row of the tile
 *     [1] kv_start  first global key row (= start of the tile's sequence)
 *     [2] kv_len    number of keys (= length of the sequence)
 *     [3] (q_rows << 16) | head     q_rows in 1..block_m
 * Query tiles start at the sequence start (not at multiples of block_m of the
 * global row index), so a sequence's result does not depend on what it is
 * packed with.
 *
 *   items      HOST output buffer of capacity_items * 4 int32, may be NULL when
 *              capacity_items == 0 (to query the count).
 *   block_m    out: query rows per tile used for this head_dim.
 *   returns    the number of items (>= 0), or a negative error code;
 *              DIT_ATTN_ERR_CAPACITY if capacity_items > 0 is too small.
 */
int64_t dit_attn_plan(const int32_t* cu_seqlens, int32_t n_seqs,
                      int32_t n_heads, int32_t head_dim,
                      int32_t* items, int64_t capacity_items, int32_t* block_m);

/*
 * Host-only: the eviction policy of a context's cache of uploaded work-lists (at most 32 packs; paper Section 4.3:
 * dynamic batching produces many distinct packs over a serving run).  A forward call that is recorded into a HIP graph
 * pins its pack: the recorded launch reads the pack's device work-list (and, with split-KV, the context's workspace)
 * on every replay, so neither is freed before dit_attn_destroy; when every cached pack is pinned the cache grows
 * instead.  A call under capture for a pack that has no cached work-list yet (or whose split-KV workspace would have
 * to grow) returns DIT_ATTN_ERR_CAPTURE: call once outside the capture first.
 * Given last_use[i] (a use counter) and pinned[i] (non-zero: pinned) of n cached packs, returns the index the cache
 * evicts next: the least recently used unpinned one, or -1 if there is none (also for n < 0 or NULL arrays).
 */
int32_t dit_attn_plan_cache_victim(const uint64_t* last_use, const uint8_t* pinned, int32_t n);

/* Library version string, e.g. "dit_attn 0.1 gfx950". */
const char* dit_attn_version(void);

#ifdef __cplusplus
}
#endif
#endif /* DIT_ATTN_H_ */
