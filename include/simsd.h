/*
 * simsd.h -- C ABI of the SimSD verification step on AMD Instinct MI355X (gfx950).
 *
 * SimSD ("Simple Speculative Decoding in Diffusion Language Models") verifies
 * gamma drafted tokens of a block-diffusion LM in ONE target forward pass.
 * Each new sequence position appears twice: a block slot (the mask section,
 * where the target predicts) and, for drafted positions, a reference slot (the
 * data section, holding the drafted token).  A token-level temporal mask (Sec.
 * 3.1, eq. 1) lets the verification slot of draft r see the prompt and drafts
 * 1..r-1 only, so all gamma target distributions come out of one pass (Sec.
 * 3.2).  Acceptance keeps the longest prefix of drafts that pass eq. 2.
 *
 * This library computes the two data-parallel steps of that pass:
 *   simsd_verify_attention  attention of every new slot over [cached prefix |
 *                           new slots] under the temporal mask (generated on the
 *                           fly, never stored), GQA-packed, split over the prefix;
 *   simsd_verify_accept     vocabulary scan of the verification rows (argmax with
 *                           lowest-index ties, confidence, draft probability) and
 *                           the accepted-prefix length, i.e. eq. 2 at temperature 0;
 *   simsd_verify_accept_sampled  eq. 2 at temperature T: acceptance with
 *                           probability min(1, p_theta/p_phi) and the residual
 *                           draw at the first rejection.
 * and, for the passes around it:
 *   simsd_rotary            rotary positions of queries and keys, every layout and
 *                           scaling of the frequencies;
 *   simsd_rotary_append     the same, with the keys and values of a ragged batch
 *                           written to the cache;
 *   simsd_chunk_attention   block-causal attention of prompts, chunks and single
 *                           tokens over that cache (no drafts);
 *   simsd_sample            one token a row from filtered logits: what the drafter
 *                           proposes, or the target where nothing was drafted.
 * and, for long contexts in bounded memory:
 *   simsd_chunk_attention_window, simsd_verify_attention_window
 *                           both attentions under a sliding window whose first
 *                           tokens (sinks) stay visible;
 *   simsd_rotary_append_fp4, simsd_chunk_attention_fp4,
 *   simsd_verify_attention_fp4, simsd_fp4_values
 *                           a cache held in 4 bits: filled, attended over, read back.
 *
 * Conventions shared by all calls
 * --------------------------------
 *  - Sizes are element counts.  All tensors are row-major and densely packed
 *    unless a stride is given.  "b" = batch index.
 *  - New slots of a sequence: n_new = B + L, where B = block_size and
 *    L = max_ref.  Slot k < B is block slot k (the mask section).  Slot B + r
 *    is reference slot r, holding draft r+1 (the data section, Sec. 3.2).
 *  - step_map[b, k] (int32, one per block slot) extends the paper's step map
 *    (Sec. 3.1):
 *        1..gamma_b  block slot k is verified at draft step r (it is o_r);
 *        0           position committed before this step (visible to every
 *                    non-padded row, like the prompt);
 *        > gamma_b   position not drafted in this step (a mask placeholder at
 *                    every step);
 *        < 0         padding (its row outputs nothing, its column is unseen).
 *    num_ref[b] = gamma_b <= L; reference slots r >= gamma_b are padding.
 *    Each value 1..gamma_b must occur exactly once per sequence; the kernels
 *    do not check this (simsd_validate_step_map does, on the host).
 *  - Every pointer argument of a compute call is device memory owned by
 *    the caller.  The library allocates nothing, frees nothing and never
 *    synchronises: a call only enqueues work on `stream` (a hipStream_t
 *    passed as void*; NULL = the default stream) and return.
 *  - Errors: the host checks shapes, dtypes, null pointers, 16-byte alignment
 *    and workspace size before anything is enqueued and returns a status other
 *    than SIMSD_OK, with a message in simsd_last_error() (thread-local).  A
 *    failed launch returns SIMSD_ERR_HIP.  No C++ exception crosses the ABI.
 *    Data-dependent preconditions are not checked on the device and violating
 *    them is undefined: step maps as above, 0 <= prefix_lens[b] <=
 *    max_prefix_len, block_table ids inside the page pool, finite inputs.
 *  - Workspace: caller-owned device memory of at least the size the matching
 *    *_workspace_size() call returns (it may be 0, and then the pointer may
 *    be NULL).  It holds per-chunk partial results between the kernels of one
 *    call; its contents need no initialisation and are meaningless afterwards.
 *    Two calls in flight at the same time need two workspaces.  A
 *    call with less returns SIMSD_ERR_WORKSPACE, except that
 *    simsd_verify_attention takes a slower decomposition if one fits it (fp32,
 *    or more than 128 packed rows: Hq / Hkv * (B + L)).
 *  - Grid sizes follow the compute-unit count of the device a call's stream
 *    belongs to (queried once per device through the HIP device attributes
 *    and cached; a compute-partitioned MI355X reports its partition's units).
 *    The *_workspace_size() calls size for the current device (for an
 *    MI355X's 256 units when no device is visible); a call on a device with
 *    more units may need more and then returns SIMSD_ERR_WORKSPACE.  If the
 *    device query fails, argument errors are still reported first, then
 *    SIMSD_ERR_HIP.
 */
#ifndef SIMSD_H
#define SIMSD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define SIMSD_VERSION 100 /* 1.0.0 */

typedef enum {
  SIMSD_OK = 0,
  SIMSD_ERR_NULL_POINTER = 1,     /* a required pointer is NULL                       */
  SIMSD_ERR_BAD_SHAPE = 2,        /* inconsistent or out-of-range sizes/strides       */
  SIMSD_ERR_UNSUPPORTED = 3,      /* valid but not implemented (dtype, head_dim)      */
  SIMSD_ERR_ALIGNMENT = 4,        /* a pointer or stride is not 16-byte aligned       */
  SIMSD_ERR_WORKSPACE = 5,        /* workspace missing or smaller than required       */
  SIMSD_ERR_INVALID_STEP_MAP = 6, /* simsd_validate_step_map found a bad step map     */
  SIMSD_ERR_HIP = 7               /* the HIP runtime reported an error (device query
                                     or launch)                                       */
} simsd_status;

typedef enum {
  SIMSD_F32 = 0,  /* IEEE binary32                                      */
  SIMSD_BF16 = 1  /* bfloat16 (upper 16 bits of a binary32), RNE output  */
} simsd_dtype;

/* ------------------------------------------------------------------------ */
/* Verification attention                                                     */
/* ------------------------------------------------------------------------ */

/*
 * Shape of one verification-attention call.
 *
 * Query head h uses KV head h / (num_q_heads / num_kv_heads).  Scores are
 * scale * (q . k); scale == 0 selects 1/sqrt(head_dim).
 *
 * Cache layout.  page_size == 0: contiguous, element (b, t, h, i) of the
 * prefix at  cache[b*cache_stride_seq + t*cache_stride_token +
 * h*cache_stride_head + i]  for t < prefix_lens[b] <= max_prefix_len.
 * page_size > 0: paged, token t of sequence b lives in page
 * p = block_table[b*max_pages_per_seq + t/page_size] at row t % page_size:
 * cache[p*cache_stride_seq + (t%page_size)*cache_stride_token +
 * h*cache_stride_head + i]  (cache_stride_seq is then the page stride).
 * The same layout and strides apply to k_cache and v_cache.  Strides are in
 * elements, non-negative, at most 2^48, and must be multiples of 16 bytes.
 * The last index (head_dim) is contiguous.
 */
typedef struct {
  int32_t batch;              /* sequences, >= 1                                  */
  int32_t num_q_heads;        /* Hq >= 1                                          */
  int32_t num_kv_heads;       /* Hkv >= 1, Hq % Hkv == 0, Hq / Hkv <= 16          */
  int32_t head_dim;           /* 64 or 128                                        */
  int32_t block_size;         /* B >= 1                                           */
  int32_t max_ref;            /* L, 0 <= L <= B, B + L <= 64                      */
  int32_t max_prefix_len;     /* upper bound of prefix_lens[], >= 0               */
  int32_t page_size;          /* 0 = contiguous cache; else tokens per page       */
  int32_t max_pages_per_seq;  /* paged: block_table row length,
                                 >= ceil(max_prefix_len / page_size)              */
  int32_t kv_chunk;           /* prefix keys per work-group (multiple of 64);
                                 0 to let the library choose; -1 for the stream
                                 decomposition (equal tile ranges per resident
                                 work-group; bf16, Hq/Hkv*(B+L) <= 128 and
                                 batch <= 256 only, else SIMSD_ERR_UNSUPPORTED) */
  int64_t cache_stride_seq;   /* elements between sequences (contiguous) / pages  */
  int64_t cache_stride_token; /* elements between consecutive tokens              */
  int64_t cache_stride_head;  /* elements between consecutive KV heads            */
  float scale;                /* softmax scale; 0 = 1/sqrt(head_dim)              */
  simsd_dtype dtype;          /* of q, k_new, v_new, k_cache, v_cache and out     */
  float rope_theta;           /* 0: q and k_new arrive rotated.  > 0: they arrive
                                 unrotated and the kernels apply the rotary
                                 embedding with this base at the RoPE-copy
                                 positions (see simsd_verify_attention)          */
} simsd_attn_desc;

/* Bytes of workspace simsd_verify_attention needs for `desc` (host only; 0 for
 * an invalid descriptor, whose error simsd_verify_attention reports). */
size_t simsd_verify_attention_workspace_size(const simsd_attn_desc* desc);

/*
 * Attention of every new slot over its visible keys (Sec. 3.2, "Target Model
 * Verification"; mask: Sec. 3.1, eq. 1; the prompt is visible to every
 * non-padded response row, padding rows/columns are removed).
 *
 *   q       [batch, B+L, Hq,  head_dim]  queries of the new slots (after RoPE,
 *                                        or before it when rope_theta > 0)
 *   k_new   [batch, B+L, Hkv, head_dim]  keys of the new slots (likewise)
 *   v_new   [batch, B+L, Hkv, head_dim]  values of the new slots
 *   k_cache, v_cache                     cached prefix, layout above
 *   block_table [batch, max_pages_per_seq] int32, or NULL if page_size == 0
 *   prefix_lens [batch] int32            cached prefix length of each sequence
 *   step_map    [batch, B] int32         see the conventions above
 *   num_ref     [batch] int32            gamma_b
 *   out     [batch, B+L, Hq, head_dim]   softmax(scale q K^T) V over the visible
 *                                        keys, in `dtype` (bf16 rounded to
 *                                        nearest even); padding rows are 0
 *   lse     [batch, Hq, B+L] float32     natural-log log-sum-exp of the scaled
 *                                        scores of each row (-inf for padding
 *                                        rows), or NULL
 *   workspace, workspace_bytes           see the conventions above
 *   stream                               hipStream_t
 *
 * RoPE copy (Sec. 3.1, Sec. 3.2), when rope_theta > 0: dims i and i + d/2 of
 * each new slot's query and key are rotated by pos * rope_theta^(-2i/d), in
 * fp32, before the scores (the new keys are rounded back to the input dtype).
 * Block slot k sits at pos = prefix_lens[b] + k; reference slot r (draft r+1)
 * shares the index of its verification slot, prefix_lens[b] + k_{r+1}, where
 * step_map[b, k_{r+1}] = r + 1; padding reference slots take prefix_lens[b].
 * The cached prefix keys must already be rotated at indices 0..prefix_len-1.
 * rope_theta must be finite and >= 0 (SIMSD_ERR_BAD_SHAPE otherwise).
 */
simsd_status simsd_verify_attention(const simsd_attn_desc* desc, const void* q,
                                    const void* k_new, const void* v_new,
                                    const void* k_cache, const void* v_cache,
                                    const int32_t* block_table, const int32_t* prefix_lens,
                                    const int32_t* step_map, const int32_t* num_ref,
                                    void* out, float* lse, void* workspace,
                                    size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Vocabulary scan and acceptance                                            */
/* ------------------------------------------------------------------------ */

typedef struct {
  int32_t batch;             /* sequences, >= 1                                    */
  int32_t block_size;        /* B, 1 <= B <= 64                                    */
  int32_t max_ref;           /* L, 0 <= L <= B                                     */
  int32_t vocab;             /* V >= 1                                             */
  int32_t chunks_per_row;    /* work-groups per logits row, or 0 = library's choice */
  simsd_dtype logits_dtype;  /* of logits                                          */
} simsd_accept_desc;

size_t simsd_verify_accept_workspace_size(const simsd_accept_desc* desc);

/*
 * Greedy verification (eq. 2 at temperature 0, Sec. 3.2): draft r is accepted
 * while the target's argmax at its verification slot equals it; the longest
 * accepted prefix is kept.
 *
 *   logits      [batch, B, V]   row k = target logits at block slot k.  Only
 *                               rows with step_map >= 1 are read.
 *   draft_ids   [batch, L] int32  draft r at index r-1 (entries >= gamma_b unused)
 *   step_map, num_ref           as for simsd_verify_attention
 *   target_ids  [batch, B] int32   smallest index of the row maximum (stored
 *                                  values compared exactly, -0 == +0), or -1
 *                                  for rows that are not scanned
 *   confidence  [batch, B] float32 largest softmax probability of the row
 *                                  (0 for rows not scanned), or NULL
 *   draft_prob  [batch, L] float32 target softmax probability of draft r at
 *                                  its verification row; 0 for an id outside
 *                                  [0, V) and for r >= gamma_b; or NULL
 *   accept_len  [batch] int32      largest a <= gamma_b such that drafts
 *                                  1..a all equal their rows' target_ids.  A
 *                                  draft id outside [0, V) is a rejection.
 *                                  On rejection the correction token is
 *                                  target_ids at the row of draft a+1.
 */
simsd_status simsd_verify_accept(const simsd_accept_desc* desc, const void* logits,
                                 const int32_t* draft_ids, const int32_t* step_map,
                                 const int32_t* num_ref, int32_t* target_ids,
                                 float* confidence, float* draft_prob, int32_t* accept_len,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the greedy
 * verification of simsd_verify_accept with no workspace argument.  The scan
 * partials go to a fixed device array of SIMSD_NOALLOC_SCRATCH_BYTES inside the
 * library; each GPU the library runs on holds its own copy of it until the
 * process ends.
 *
 *   desc, logits, draft_ids, step_map, num_ref, target_ids, confidence,
 *   draft_prob, accept_len, stream     exactly as for simsd_verify_accept,
 *                                      and the outputs are the same bits
 *
 * Nothing is allocated, freed or synchronised by the call; its first call on a
 * device looks up that device's copy of the array (making the device current
 * for the lookup and restoring the previous one).  Shapes whose partials need
 * more than SIMSD_NOALLOC_SCRATCH_BYTES (16 bytes per scanned row and
 * vocabulary chunk, the size simsd_verify_accept_workspace_size reports)
 * return SIMSD_ERR_WORKSPACE with nothing enqueued: use simsd_verify_accept
 * with a workspace for those.  All calls on one GPU share its array, which
 * keeps the last call's contents (every entry is written before it is read, so
 * nothing needs clearing): calls that overlap on one GPU, on any streams, race
 * and must be serialised by the caller.  Other errors as simsd_verify_accept;
 * SIMSD_ERR_HIP also if the array's device address cannot be obtained.
 */
#define SIMSD_NOALLOC_SCRATCH_BYTES ((size_t)4 << 20) /* 4 MiB per device */
simsd_status simsd_verify_accept_noalloc(const simsd_accept_desc* desc, const void* logits,
                                         const int32_t* draft_ids, const int32_t* step_map,
                                         const int32_t* num_ref, int32_t* target_ids,
                                         float* confidence, float* draft_prob,
                                         int32_t* accept_len, void* stream);

/*
 * Stochastic verification (eq. 2 at temperature T > 0, Sec. 3.2; the paper's
 * experiments use T = 1, Sec. 4.1): the rule the greedy call is the T -> 0
 * limit of.  With p_theta(r) = softmax(logits[b, k_r] / T) at the
 * verification row k_r of draft r and p_phi(r) = softmax(draft_logits[b, r-1]
 * / T), draft r is accepted iff u_r * p_phi(r)(D_r) < p_theta(r)(D_r), which
 * for u_r ~ U[0, 1) happens with probability min(1, p_theta / p_phi).  The
 * longest accepted prefix is kept; at the first rejected draft a+1 the target's
 * token is drawn from the residual max(0, p_theta(a+1) - p_phi(a+1)) by
 * inverse CDF in vocabulary order: the smallest x whose running weight exceeds
 * w * (total weight), w = uniforms[b, L].  If the residual is zero everywhere
 * the draw uses p_theta(a+1).  The random numbers are the caller's.
 *
 *   temperature  T, finite and > 0 (else SIMSD_ERR_BAD_SHAPE)
 *   logits       [batch, B, V]  target logits; rows of steps 1..gamma_b are read
 *   draft_logits [batch, L, V]  row r-1 = the drafter's logits when it proposed
 *                               draft r (same dtype as logits, 16-byte aligned);
 *                               rows r-1 < gamma_b are read.  NULL only if L = 0
 *   draft_ids    [batch, L] int32
 *   step_map, num_ref           as for simsd_verify_attention
 *   uniforms     [batch, L + 1] float32 in [0, 1): u_1..u_L, then w
 *   p_target     [batch, L] float32  p_theta(r)(D_r), 0 for an id outside
 *                                    [0, V) and for r > gamma_b; or NULL
 *   p_draft      [batch, L] float32  p_phi(r)(D_r), likewise; or NULL
 *   accept_len   [batch] int32       accepted drafts, 0..gamma_b.  A draft id
 *                                    outside [0, V) is a rejection.
 *   correction   [batch] int32       token drawn at the first rejection, or -1
 *                                    when every draft was accepted
 * Probabilities and running sums are float32: the draw can differ from an
 * exact one only where w * total falls within rounding of a boundary.
 * The workspace must hold simsd_verify_accept_sampled_workspace_size() bytes.
 */
size_t simsd_verify_accept_sampled_workspace_size(const simsd_accept_desc* desc);
simsd_status simsd_verify_accept_sampled(const simsd_accept_desc* desc, float temperature,
                                         const void* logits, const void* draft_logits,
                                         const int32_t* draft_ids, const int32_t* step_map,
                                         const int32_t* num_ref, const float* uniforms,
                                         float* p_target, float* p_draft, int32_t* accept_len,
                                         int32_t* correction, void* workspace,
                                         size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* LM head fused with the scan                                                */
/* ------------------------------------------------------------------------ */

typedef struct {
  int32_t batch;             /* sequences, >= 1                                    */
  int32_t block_size;        /* B, 1 <= B <= 64                                    */
  int32_t max_ref;           /* L, 0 <= L <= B                                     */
  int32_t vocab;             /* V >= 1                                             */
  int32_t hidden;            /* H, a positive multiple of 64                       */
  simsd_dtype dtype;         /* of hidden and weight: SIMSD_BF16 only              */
} simsd_lmhead_desc;

size_t simsd_verify_accept_lmhead_workspace_size(const simsd_lmhead_desc* desc);

/*
 * Greedy verification as simsd_verify_accept, with the logits computed on
 * the fly from the verification rows' final hidden states and the LM-head
 * weight (the target model's prediction at each verification slot, Sec. 3.2):
 * logits[b, k, v] = hidden[b, k, :] . weight[v, :], accumulated in fp32 from
 * bf16 products, never stored.  Outputs and their meaning are those of
 * simsd_verify_accept (ties between exactly equal fp32 logits go to the lowest
 * index).
 *
 *   hidden  [batch, B, H] bf16, 16-byte aligned; row k = block slot k
 *   weight  [V, H] bf16, 16-byte aligned (a Linear layer's [out, in] layout)
 *   draft_ids, step_map, num_ref, target_ids, confidence, draft_prob,
 *   accept_len, workspace, workspace_bytes, stream   as for simsd_verify_accept
 *   (draft_ids may be NULL when max_ref == 0; confidence and draft_prob may be
 *   NULL)
 * The workspace must hold simsd_verify_accept_lmhead_workspace_size() bytes
 * (0 for an invalid descriptor), 16-byte aligned, no initialisation needed; it
 * is fully rewritten by each call, so calls on one stream may share it.  All
 * buffers belong to the caller; the library allocates nothing and does not
 * synchronise.  Three kernels are enqueued on the stream.  The fp32
 * accumulation order is fixed for a given shape, so repeated calls give the
 * same bits.
 * Errors (nothing is enqueued): SIMSD_ERR_NULL_POINTER, SIMSD_ERR_BAD_SHAPE
 * (descriptor out of range, H not a multiple of 64), SIMSD_ERR_UNSUPPORTED
 * (dtype other than SIMSD_BF16), SIMSD_ERR_ALIGNMENT (hidden, weight or
 * workspace), SIMSD_ERR_WORKSPACE; SIMSD_ERR_HIP if a launch fails.
 */
simsd_status simsd_verify_accept_lmhead(const simsd_lmhead_desc* desc, const void* hidden,
                                        const void* weight, const int32_t* draft_ids,
                                        const int32_t* step_map, const int32_t* num_ref,
                                        int32_t* target_ids, float* confidence, float* draft_prob,
                                        int32_t* accept_len, void* workspace,
                                        size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* Rotary positions, and the write into the cache                             */
/* ------------------------------------------------------------------------ */

/*
 * Shape of one rotary call on tokens packed back to back.  Element (i, h, c) of
 * x in {q, k, v, q_out, k_out} is x[i*x_stride_token + h*x_stride_head + c]: the
 * parts of a fused projection's output are passed as they lie.  Strides are in
 * elements, non-negative, at most 2^40 and multiples of 16 bytes; those of an
 * output must keep its rows apart.  The cache fields are those of
 * simsd_attn_desc; simsd_rotary ignores them.
 */
typedef struct {
  int32_t num_tokens;         /* rows of q, k, v and the outputs, 0..2^24          */
  int32_t num_q_heads;        /* Hq >= 0 (0: no queries, q and q_out NULL)         */
  int32_t num_kv_heads;       /* Hkv >= 0 (0: no keys; simsd_rotary only)          */
  int32_t head_dim;           /* a multiple of 8, 8..512                          */
  int32_t rotary_dim;         /* leading dims of a head that turn: even,
                                 2..head_dim; the rest is copied                  */
  int32_t interleaved;        /* 0: dims i and i + rotary_dim/2 pair;
                                 1: dims 2i and 2i + 1 pair                       */
  int32_t batch;              /* append: sequences, 1..65535                      */
  int32_t max_kv_len;         /* append: cache indices written are < this, >= 0    */
  int32_t page_size;          /* append: 0 = contiguous cache; else tokens per page */
  int32_t max_pages_per_seq;  /* append, paged: block_table row length,
                                 >= ceil(max_kv_len / page_size)                  */
  int32_t num_pages;          /* append, paged: pages in the pool, >= 0            */
  float attn_factor;          /* multiplies the rotated values; finite, > 0
                                 (1 unless the frequencies are scaled by "yarn")   */
  int64_t q_stride_token, q_stride_head;
  int64_t k_stride_token, k_stride_head;
  int64_t v_stride_token, v_stride_head;         /* append */
  int64_t q_out_stride_token, q_out_stride_head;
  int64_t k_out_stride_token, k_out_stride_head; /* simsd_rotary */
  int64_t cache_stride_seq, cache_stride_token, cache_stride_head;
  simsd_dtype dtype;          /* of q, k, v, the outputs and the cache            */
} simsd_rotary_desc;

/*
 * Rotary embedding: pair i < rotary_dim/2 of token t's heads,
 *   (x1, x2) -> attn_factor * (x1 cos a - x2 sin a, x2 cos a + x1 sin a),
 *   a = positions[t] * freq[i],
 * with the angle formed and reduced in fp64 and the rotation in fp32, rounded
 * once to `dtype`.  The verification step's new slots take their RoPE-copy
 * positions (simsd_verify_attention then gets rope_theta = 0); this call
 * serves the layouts and scaled frequencies that the fused rotation lacks.
 *
 *   q          [num_tokens, Hq, head_dim], or NULL if Hq == 0
 *   k          [num_tokens, Hkv, head_dim], or NULL if Hkv == 0
 *   positions  [num_tokens] int32 (any value)
 *   freq       [rotary_dim/2] float64, radians a position (device memory;
 *              simsd_rope_frequencies fills a host copy)
 *   q_out, k_out  like q and k; each may be its input itself, with the same
 *              strides (in place), and otherwise overlaps no input
 * All data pointers are 16-byte aligned.  One kernel; no workspace.
 */
simsd_status simsd_rotary(const simsd_rotary_desc* desc, const void* q, const void* k,
                          const int32_t* positions, const double* freq, void* q_out, void* k_out,
                          void* stream);

/*
 * The same rotation for the new tokens of a ragged batch, with the rotated keys
 * and the values written to the cache that simsd_verify_attention and
 * simsd_chunk_attention read.  Tokens q_starts[b] <= t < q_starts[b+1] belong to
 * sequence b and take the cache indices kv_lens[b] - n_b .. kv_lens[b] - 1 in
 * order (n_b of them: kv_lens counts the new tokens).
 *
 *   q_starts   [batch + 1] int32, not falling, at most num_tokens; rows of
 *              tokens before q_starts[0] or from q_starts[batch] on are left as
 *              they were
 *   kv_lens    [batch] int32 cached length of each sequence, new tokens included
 *   positions  [num_tokens] int32, or NULL: a token's position is its cache index
 *   v          [num_tokens, Hkv, head_dim], written to v_cache unchanged
 *   q, q_out   may both be NULL (Hq == 0) where only the cache is filled
 *   block_table [batch, max_pages_per_seq] int32, or NULL if page_size == 0
 * A token whose cache index is outside [0, max_kv_len), or whose page id is
 * outside [0, num_pages), is not written to the cache (its query still turns).
 * Two tokens that take one cache row leave either's values there.
 */
simsd_status simsd_rotary_append(const simsd_rotary_desc* desc, const void* q, const void* k,
                                 const void* v, const int32_t* positions, const double* freq,
                                 void* q_out, void* k_cache, void* v_cache,
                                 const int32_t* block_table, const int32_t* q_starts,
                                 const int32_t* kv_lens, void* stream);

/* ------------------------------------------------------------------------ */
/* Attention of a chunk of new tokens                                         */
/* ------------------------------------------------------------------------ */

/*
 * Shape of one chunk-attention call: the new tokens of a ragged batch, packed
 * back to back, over a cache that holds their own keys and values already
 * (simsd_rotary_append writes them).  Heads, scale and cache layout are those of
 * simsd_attn_desc.
 */
typedef struct {
  int32_t num_tokens;         /* rows of q and out, 0..2^23                       */
  int32_t batch;              /* sequences, 1..65535                              */
  int32_t num_q_heads;        /* Hq >= 1                                          */
  int32_t num_kv_heads;       /* Hkv >= 1, Hq % Hkv == 0, Hq / Hkv <= 16          */
  int32_t head_dim;           /* 64 or 128                                        */
  int32_t max_q_len;          /* most new tokens of a sequence, >= 0 (it chooses
                                 the kernel; longer sequences are served too)     */
  int32_t max_kv_len;         /* upper bound of kv_lens[], 0..2^30                */
  int32_t mask_block;         /* m: a token sees the keys up to the end of its
                                 block of m positions; 1: causal, 0: all keys     */
  int32_t page_size;          /* 0 = contiguous cache; else tokens per page       */
  int32_t max_pages_per_seq;  /* paged: block_table row length,
                                 >= ceil(max_kv_len / page_size)                  */
  int32_t kv_chunk;           /* keys per work-group (multiple of 64; fewer where
                                 a work-group's 2047 pages hold fewer), or 0 =
                                 library's choice                                 */
  int64_t cache_stride_seq;   /* elements between sequences (contiguous) / pages  */
  int64_t cache_stride_token; /* elements between consecutive tokens              */
  int64_t cache_stride_head;  /* elements between consecutive KV heads            */
  float scale;                /* softmax scale; 0 = 1/sqrt(head_dim)              */
  simsd_dtype dtype;          /* of q, the caches and out                         */
} simsd_chunk_desc;

size_t simsd_chunk_attention_workspace_size(const simsd_chunk_desc* desc);

/*
 * Block-causal attention of prompts, chunks of prompts and single tokens.  Token
 * i of the n_b = q_starts[b+1] - q_starts[b] new ones of sequence b sits at
 * position p = kv_lens[b] - n_b + i and sees the cached keys
 *   t < min(kv_lens[b], (p / m + 1) * m),   m = mask_block  (all for m = 0),
 * none if p < 0.  A row that sees no key gives 0 and a log-sum-exp of -inf.
 * Keys and values a row does not see have no part in it, whatever they hold.  An
 * infinite value that it sees makes that element of the row infinite, or NaN where
 * the key's weight is 0 in fp32 (as 0 times infinity is; which weights round to 0 on
 * the way may differ with kv_chunk and the shape).  Scores, weights and sums are fp32;
 * for bf16 the weights are rounded to bf16 for their product with the values, as in
 * simsd_verify_attention, which adds up to 2^-8 of sum w|v| / sum w to the output's
 * own rounding.
 *
 *   q           [num_tokens, Hq, head_dim]  (rotated)
 *   k_cache, v_cache, block_table           the cache, as in simsd_attn_desc
 *   q_starts    [batch + 1] int32, not falling, 0..num_tokens; rows of tokens
 *               before q_starts[0] or from q_starts[batch] on are left as they were
 *   kv_lens     [batch] int32, 0..max_kv_len, the new tokens included
 *   out         [num_tokens, Hq, head_dim]
 *   lse         [Hq, num_tokens] float32 natural-log log-sum-exp, or NULL
 * The workspace must hold simsd_chunk_attention_workspace_size() bytes (0 where
 * one work-group takes all keys of a row; a call with less returns
 * SIMSD_ERR_WORKSPACE).  One kernel, and a second that joins the parts of rows
 * whose keys were divided.  The order of additions is fixed for a given shape.
 * A call of more row blocks (16 to 256 rows of Hq / Hkv to a token) times KV heads
 * than 2^22, or of more than 65535 key ranges, returns SIMSD_ERR_BAD_SHAPE.
 */
simsd_status simsd_chunk_attention(const simsd_chunk_desc* desc, const void* q, const void* k_cache,
                                   const void* v_cache, const int32_t* block_table,
                                   const int32_t* q_starts, const int32_t* kv_lens, void* out,
                                   float* lse, void* workspace, size_t workspace_bytes,
                                   void* stream);

/* ------------------------------------------------------------------------ */
/* Sliding window with sinks                                                  */
/* ------------------------------------------------------------------------ */

/*
 * simsd_chunk_attention for layers whose tokens see a window of the latest keys and
 * a few first ones.  A token at position p, in the mask's block of m = mask_block
 * positions that starts at p0 = p / m * m, sees the cached keys
 *   t < min(kv_lens[b], p0 + m)  with  t > p0 - window  or  t < sinks:
 * its own block as before (m = 1: itself), the window - 1 keys before that, and the
 * first `sinks` keys.  All tokens of a block see the same keys.
 *
 *   window  >= 1, or 0: none (then sinks must be 0 too)
 *   sinks   >= 0
 * A window needs mask_block >= 1 (SIMSD_ERR_BAD_SHAPE otherwise).  Everything else is
 * as in simsd_chunk_attention, with its own workspace size; kv_chunk counts the keys
 * of the tiles of 64 that a row block's window and sinks lie in (fp32: 32).  Pages
 * none of whose keys a token of the call sees are not read, and neither are their
 * entries of block_table: both may have been given to other sequences.
 */
size_t simsd_chunk_attention_window_workspace_size(const simsd_chunk_desc* desc, int32_t window,
                                                   int32_t sinks);
simsd_status simsd_chunk_attention_window(const simsd_chunk_desc* desc, int32_t window, int32_t sinks,
                                          const void* q, const void* k_cache, const void* v_cache,
                                          const int32_t* block_table, const int32_t* q_starts,
                                          const int32_t* kv_lens, void* out, float* lse,
                                          void* workspace, size_t workspace_bytes, void* stream);

/*
 * simsd_verify_attention under the same window: the new slots are the block that
 * starts at position prefix_lens[b], so that each of them sees the cached keys
 *   t > prefix_lens[b] - window  or  t < sinks,
 * and the new slots that the temporal mask allows.  window 0: the whole prefix.
 * SIMSD_ERR_UNSUPPORTED: fp32, rope_theta > 0 (turn q and k_new with simsd_rotary),
 * kv_chunk < 0.  kv_chunk counts as in simsd_chunk_attention_window, the tile of the
 * new slots among them.  Keys and values a slot does not see have no part in its
 * row, whatever they hold.
 */
size_t simsd_verify_attention_window_workspace_size(const simsd_attn_desc* desc, int32_t window,
                                                    int32_t sinks);
simsd_status simsd_verify_attention_window(const simsd_attn_desc* desc, int32_t window, int32_t sinks,
                                           const void* q, const void* k_new, const void* v_new,
                                           const void* k_cache, const void* v_cache,
                                           const int32_t* block_table, const int32_t* prefix_lens,
                                           const int32_t* step_map, const int32_t* num_ref, void* out,
                                           float* lse, void* workspace, size_t workspace_bytes,
                                           void* stream);

/* ------------------------------------------------------------------------ */
/* A cache held in 4 bits                                                     */
/* ------------------------------------------------------------------------ */

/*
 * Keys and values in 4.25 bits an element.  32 dims of a head, from a multiple of 32
 * on, share a power of two 2^e; each is a code c of 4 bits: its sign, and the index of
 * its size in {0, 0.5, 1, 1.5, 2, 3, 4, 6}, times 2^e.
 *   codes   head_dim / 2 bytes a head, dims 2i and 2i + 1 in the low and high half of
 *           byte i
 *   scales  head_dim / 32 bytes a head, e + 127 each; 255: all 32 are NaN
 * Codes lie like the elements of a cache (see simsd_attn_desc), with the descriptor's
 * cache strides in bytes; scales with strides of their own.  A cache of zeros holds
 * zeros.  What a head's tokens take is least fetched where they lie next to each other
 * (strides of head outside token).
 */
typedef struct {
  void* k;                    /* codes, 16-byte aligned                           */
  void* v;
  void* k_scales;             /* scales, aligned to head_dim / 32 bytes
                                 (simsd_fp4_values: at any address)               */
  void* v_scales;
  int64_t scale_stride_seq;   /* bytes between sequences (contiguous) / pages; all
                                 three are multiples of head_dim / 32
                                 (simsd_fp4_values: any, >= 0)                    */
  int64_t scale_stride_token;
  int64_t scale_stride_head;
} simsd_fp4_cache;

/*
 * simsd_rotary_append to a 4-bit cache.  A turned key is rounded once to the nearest
 * code, ties to the even one, from the rotation in fp64, which is off by 1e-15 and, for
 * its angle, 4e-16 |position * freq| of the pair's length (1.3e-11 at position 32768 and
 * frequency 1); values likewise as they are.  e is the least exponent, from -125 to 125,
 * at which the largest of the 32 is below 7 * 2^e (it is held as 6 * 2^e at most);
 * larger ones than 6 * 2^125 are held as that.  32 of which one is infinite or NaN are
 * all held as NaN.  Queries are turned as in simsd_rotary_append.
 *   dtype SIMSD_BF16 and head_dim 64 or 128 only (SIMSD_ERR_UNSUPPORTED); cache
 *   strides in bytes, those of the codes multiples of 16; tokens' and heads' rows of
 *   codes and of scales apart.
 */
simsd_status simsd_rotary_append_fp4(const simsd_rotary_desc* desc, const void* q, const void* k,
                                     const void* v, const int32_t* positions, const double* freq,
                                     void* q_out, const simsd_fp4_cache* cache,
                                     const int32_t* block_table, const int32_t* q_starts,
                                     const int32_t* kv_lens, void* stream);

/*
 * simsd_chunk_attention_window over a 4-bit cache: its keys and values are the exact
 * values of their codes, past bf16's range (at scales of 253 and 254, which no append
 * writes) infinite, and the arithmetic is that of bf16.  dtype (of q and out)
 * SIMSD_BF16 only (SIMSD_ERR_UNSUPPORTED); cache_stride_* in bytes, multiples of 16.
 * kv_chunk counts tiles of 64 keys, or of 32 where a call has few rows a sequence.
 */
size_t simsd_chunk_attention_fp4_workspace_size(const simsd_chunk_desc* desc, int32_t window,
                                                int32_t sinks);
simsd_status simsd_chunk_attention_fp4(const simsd_chunk_desc* desc, int32_t window, int32_t sinks,
                                       const void* q, const simsd_fp4_cache* cache,
                                       const int32_t* block_table, const int32_t* q_starts,
                                       const int32_t* kv_lens, void* out, float* lse, void* workspace,
                                       size_t workspace_bytes, void* stream);

/*
 * simsd_verify_attention_window over a 4-bit prefix (k_new and v_new in bf16; the
 * accepted ones are appended with simsd_rotary_append_fp4).
 */
size_t simsd_verify_attention_fp4_workspace_size(const simsd_attn_desc* desc, int32_t window,
                                                 int32_t sinks);
simsd_status simsd_verify_attention_fp4(const simsd_attn_desc* desc, int32_t window, int32_t sinks,
                                        const void* q, const void* k_new, const void* v_new,
                                        const simsd_fp4_cache* cache, const int32_t* block_table,
                                        const int32_t* prefix_lens, const int32_t* step_map,
                                        const int32_t* num_ref, void* out, float* lse,
                                        void* workspace, size_t workspace_bytes, void* stream);

/* A 4-bit cache as a whole: [num, tokens, num_kv_heads] heads. */
typedef struct {
  int32_t num;                /* sequences or pages, >= 0                         */
  int32_t tokens;             /* of each, >= 0                                    */
  int32_t num_kv_heads;       /* >= 0; num * tokens * num_kv_heads <= 2^36, and
                                 times head_dim <= 2^37 - 8192                    */
  int32_t head_dim;           /* a multiple of 32, 32..512                        */
  int64_t cache_stride_seq;   /* of the codes, in bytes, multiples of 16          */
  int64_t cache_stride_token;
  int64_t cache_stride_head;
} simsd_fp4_values_desc;

/*
 * The values of a cache's keys and of its values: k_out and v_out [num, tokens,
 * num_kv_heads, head_dim] bf16, 16-byte aligned, not the same, each or NULL.  Exact; past bf16's
 * range infinite (no append writes such).  One kernel.
 */
simsd_status simsd_fp4_values(const simsd_fp4_values_desc* desc, const simsd_fp4_cache* cache,
                              void* k_out, void* v_out, void* stream);

/* ------------------------------------------------------------------------ */
/* Sampling                                                                   */
/* ------------------------------------------------------------------------ */

typedef struct {
  int32_t rows;              /* rows of logits, 0..2^21                            */
  int32_t vocab;             /* V, 1..2^22                                         */
  float temperature;         /* T, finite and >= 0 (0: the largest logit)          */
  int32_t top_k;             /* >= 0; 0 or >= V: off                               */
  float top_p;               /* 0..1; 1: off                                       */
  float min_p;               /* 0..1; 0: off                                       */
  simsd_dtype dtype;         /* of logits                                          */
} simsd_sample_desc;

/*
 * One token for each row of logits (the drafter's proposals, or the target's
 * own tokens where nothing was drafted).  With m the row's largest logit,
 * w_i = exp((x_i - m) / T), and tokens in the order of falling logits, the
 * lowest index first among equal ones (-0 == +0):
 *   top_k   keeps the first k tokens;
 *   top_p   of those, the fewest leading ones whose weights add up to top_p of
 *           all theirs or more (at least one);
 *   min_p   keeps the tokens with w_i >= min_p;
 * and the token is the first kept one, in that order, at which the running
 * weight exceeds u times the weight of all kept tokens, u = uniforms[row].
 * Logits of -inf or NaN, and those more than 700 T below m, are never kept.
 * If m is +inf, only the logits of +inf are.  T <= 0 (or NaN) selects the first
 * token of the order.  A row that keeps nothing gives token -1.  The random
 * numbers are the caller's, and the running sums are the same on every run and
 * exact to V * 2^-(63 - ceil(log2 V)) of the largest weight (weights are rounded
 * to as many binary places as V of them leave in 62 bits): 7.5e-9 at most up to
 * V = 2^18, 1.2e-7 at 2^20, 1.9e-6 at 2^22.
 *
 *   logits       [rows, V], aligned to their elements
 *   uniforms     [rows] float32 in [0, 1)
 *   temperatures, top_ks, top_ps, min_ps   [rows] float32 / int32, or NULL: the
 *                descriptor's value for every row.  In these, top_k <= 0,
 *                top_p >= 1 or NaN and min_p <= 0 or NaN are off, top_p <= 0
 *                keeps the first token, min_p >= 1 those equal to it, and an
 *                infinite temperature is the largest finite one
 *   token        [rows] int32
 *   prob         [rows] float32 the token's weight over that of all kept tokens
 *                (0 for token -1), or NULL
 *   kept         [rows] int32 number of kept tokens, or NULL
 * One kernel; no workspace.
 */
simsd_status simsd_sample(const simsd_sample_desc* desc, const void* logits, const float* uniforms,
                          const float* temperatures, const int32_t* top_ks, const float* top_ps,
                          const float* min_ps, int32_t* token, float* prob, int32_t* kept,
                          void* stream);

/* ------------------------------------------------------------------------ */
/* Host-only helpers (no GPU needed)                                          */
/* ------------------------------------------------------------------------ */

/* Checks host copies of step_map [batch, B] and num_ref [batch]: 0 <= gamma_b
 * <= L and every value 1..gamma_b exactly once per sequence.  Returns SIMSD_OK
 * or SIMSD_ERR_INVALID_STEP_MAP (SIMSD_ERR_NULL_POINTER / _BAD_SHAPE for bad
 * arguments: batch >= 1, 1 <= B <= 64, 0 <= L <= B), with the first offending
 * sequence in simsd_last_error(). */
simsd_status simsd_validate_step_map(const int32_t* step_map_host, const int32_t* num_ref_host,
                                     int32_t batch, int32_t block_size, int32_t max_ref);

/* Frequencies of the rotary pairs, and the factor on the rotated values, for a
 * context scaled to `factor` times the original one:
 *   NONE    f_i = theta^(-2i/rotary_dim)
 *   LINEAR  f_i / factor (positions interpolated)
 *   NTK     the base grown to theta * factor^(rotary_dim / (rotary_dim - 2))
 *   YARN    pairs that turn beta_fast times or more in the original context keep
 *           f_i, those that turn beta_slow times or less take f_i / factor, and
 *           those between are blended linearly in the pair index, between the
 *           indices of beta_fast (rounded down) and beta_slow (rounded up);
 *           *attn_factor = 0.1 ln(factor) + 1
 * `freq` [rotary_dim/2] and `attn_factor` are host memory; original_context and
 * the betas matter to YARN only. */
typedef enum {
  SIMSD_ROPE_NONE = 0,
  SIMSD_ROPE_LINEAR = 1,
  SIMSD_ROPE_NTK = 2,
  SIMSD_ROPE_YARN = 3
} simsd_rope_scaling;
simsd_status simsd_rope_frequencies(int32_t rotary_dim, double theta, simsd_rope_scaling scaling,
                                    double factor, int32_t original_context, double beta_fast,
                                    double beta_slow, double* freq, float* attn_factor);

const char* simsd_status_string(simsd_status status);
const char* simsd_last_error(void); /* message of this thread's last failed call */
int simsd_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SIMSD_H */
