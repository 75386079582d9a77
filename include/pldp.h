/*
 * pldp.h -- C ABI of the GB300 (sm_103a) PLD+ drafting and greedy
 * verification library.
 *
 * PLD+ (arXiv 2412.01447) speeds up decoding of input-guided tasks by
 * drafting a span copied from the context and verifying it with one forward
 * pass of the target model.  Per decode step and per sequence this library:
 *
 *   1. finds the earlier occurrences P of the last token (Eq. 1), narrowed to
 *      the longest suffix n-gram that occurs earlier     -> pldp_find_candidates
 *   2. ranks P with a model artifact: the cosine between hidden states
 *      H_{j-1} and H_{t-1} (Eq. 3)                        -> pldp_rank_hidden
 *      or the max attention of query t-1 over selected
 *      (layer, head) rows (Eq. 2)                         -> pldp_rank_attention
 *   3. drafts the K tokens after the best occurrence j*
 *      (Sec. 4.3)                                         -> pldp_extract_draft
 *   4. verifies the draft greedily against the target
 *      model's K+1 next-token distributions (Sec. 4.4)    -> pldp_verify_greedy
 *      or by sampling at temperature T                    -> pldp_verify_sample
 *
 * Fused forms: pldp_draft_step runs 1-3 in one call (scanning the contexts, or
 * with the incremental token index of pldp_index_build); pldp_verify_greedy_draft
 * and pldp_verify_sample_draft run 4 (greedy or by sampling) for the current step
 * and then 1-3 for the next step.  Offline:
 * pldp_rank_hidden_avg (App. B.2) and pldp_identify_heads / pldp_top_heads
 * (Sec. 4.2.1).  Around the target model's forward pass of a step, over a paged cache:
 * pldp_cache_append, pldp_attend_cache, pldp_rank_cache (2 from the cache), pldp_cache_read,
 * and pldp_token_logprobs on its logits.  Before the steps, and between them: prompts of
 * different lengths packed into the cache (pldp_cache_append_prompt, pldp_attend_prompt), and
 * its pages given out, shared and given back on the device (pldp_pages_reserve, pldp_pages_fork,
 * pldp_pages_free, pldp_pages_compact, pldp_cache_copy_pages).
 *
 * Conventions shared by every call
 *  - Every pointer argument is a DEVICE pointer owned by the caller (the
 *    attention rows A of the ranking calls may also be device-addressable
 *    page-locked host memory, read in place); the
 *    library allocates nothing and keeps no state between calls, except the
 *    caller-provided verification workspace described at pldp_verify_greedy
 *    (and that of pldp_attend_cache, which calls leave zeroed where that matters),
 *    the caller-provided token index that the indexed drafting calls keep up
 *    to date, and the fixed scratch area of pldp_verify_greedy_noalloc.
 *  - All work is enqueued asynchronously on `stream` (a cudaStream_t; NULL is
 *    the legacy default stream).  No call synchronises the device or reads
 *    device memory on the host, so every call may be captured in a CUDA graph.
 *  - Positions are 0-based int32.  Sequence b holds seq_len[b] tokens in
 *    ids[b*ids_stride + 0 .. seq_len[b]-1]; its last token is x_t with
 *    t = seq_len[b] - 1.  Model artifacts exist for positions 0..t-1 only.
 *  - Host-side argument checks run before anything is enqueued; a failed
 *    check returns PLDP_ERR_INVALID_ARG (or PLDP_ERR_UNSUPPORTED) and
 *    enqueues nothing.  A CUDA launch failure returns PLDP_ERR_CUDA.
 *    pldp_last_error() then gives a message (per host thread).
 *  - Data-dependent problems found on the device never trap: they set bits in
 *    the optional per-sequence status word (uint32 status[B], OR-ed in; the
 *    caller clears it) and the call produces the documented fallback.
 *  - dtype PLDP_BF16 data is raw bfloat16; PLDP_F32 is IEEE float.  Inputs
 *    must be finite (NaN is not supported).
 *  - Calls that overlap on the device must not share output buffers.
 */
#ifndef PLDP_H
#define PLDP_H

#include <stddef.h>
#include <stdint.h>

#if defined(_WIN32)
#define PLDP_API
#else
#define PLDP_API __attribute__((visibility("default")))
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PLDP_OK = 0,
    PLDP_ERR_INVALID_ARG = 1, /* null/misaligned pointer, bad size or stride  */
    PLDP_ERR_UNSUPPORTED = 2, /* dtype or size the kernels do not handle      */
    PLDP_ERR_CUDA = 3,        /* launch failed; see pldp_last_error()         */
    PLDP_ERR_TIMEOUT = 4      /* reserved: no call waits on the host          */
} pldp_status;

typedef enum { PLDP_F32 = 0, PLDP_BF16 = 1, PLDP_E4M3 = 2 /* caches only */ } pldp_dtype;

typedef enum { PLDP_AGG_MAX = 0, PLDP_AGG_SUM = 1 } pldp_agg;

/* Per-sequence device status bits. */
#define PLDP_ST_CAND_OVERFLOW 1u  /* |P| > C_cap: the first C_cap positions are listed   */
#define PLDP_ST_TOKEN_RANGE   2u  /* a draft token outside [0, V)                        */
#define PLDP_ST_CAPACITY      4u  /* the append would pass T_cap: nothing appended       */
#define PLDP_ST_SEQ_LEN       8u  /* seq_len outside its valid range: sequence skipped   */
#define PLDP_ST_DRAFT_LEN    16u  /* draft_len outside [0, K]: clamped into it           */
#define PLDP_ST_ROW_INDEX    32u  /* a row_idx entry outside [0, R): that row ignored    */
#define PLDP_ST_TIMEOUT      64u  /* an on-chip copy did not complete in time: no result */
#define PLDP_ST_PAGE        128u  /* a page table entry outside [0, n_pages): its positions skipped */

#define PLDP_MAX_NGRAM 8          /* largest ngram_max accepted                          */

/*
 * Candidate search -- Eq. 1 (Sec. 4.2):  P = { j | x_j = x_t, j < t },
 * narrowed by the longest-suffix n-gram rule of prompt lookup (Sec. 2, Fig. 2
 * caption): for n = ngram_max down to ngram_min, the first non-empty
 *   P_n = { j < t : j-n+1 >= 0 and x_{j-k} = x_{t-k} for k = 0..n-1 }
 * is P and n is match_len[b].  ngram_min = ngram_max = 1 is Eq. 1 itself.
 *
 *  ids        int32 [B, ids_stride]; row b holds the context of sequence b.
 *  ids_stride elements between rows (>= T_cap).
 *  seq_len    int32 [B]; valid range [0, T_cap] (else SEQ_LEN, nothing found).
 *  T_cap      row capacity: positions >= T_cap are never read.
 *  ngram_min, ngram_max   1 <= ngram_min <= ngram_max <= PLDP_MAX_NGRAM.
 *  cand_pos   int32 [B, C_cap] out: P in ascending order; slots past
 *             min(|P|, C_cap) are left untouched.
 *  C_cap      >= 0.  |P| > C_cap lists the first C_cap and sets CAND_OVERFLOW.
 *  cand_count int32 [B] out: the true |P| (even when it exceeds C_cap).
 *  match_len  int32 [B] out: the n of P, 0 when P is empty.
 *  status     uint32 [B] or NULL.
 * Fast path when ids is 16-byte aligned and ids_stride % 4 == 0.
 */
PLDP_API pldp_status pldp_find_candidates(const int32_t* ids, int64_t ids_stride,
                                          const int32_t* seq_len, int B, int64_t T_cap,
                                          int ngram_min, int ngram_max,
                                          int32_t* cand_pos, int C_cap,
                                          int32_t* cand_count, int32_t* match_len,
                                          uint32_t* status, void* stream);

/*
 * Ranking by hidden states -- Eq. 3 (Sec. 4.2.2):
 *   score_j = cos(H_{j-1}, H_{t-1}),  j* = argmax_{j in P} score_j,
 * with the optional threshold of App. B.3 (j kept only if score_j > threshold;
 * pass -INFINITY for none).  The caller passes the chosen layer l only.
 *
 *  H          [B, seq_stride] elements of dtype; row p of sequence b is
 *             H + b*seq_stride + p*d (rows are contiguous, d elements each).
 *  d          hidden width, 1 <= d and d * sizeof(dtype) <= 196608.
 *  seq_stride elements between sequences (>= T_cap * d).
 *  seq_len    int32 [B]; valid range [0, T_cap] (else SEQ_LEN, no result).
 *  T_cap      row capacity of H: rows >= T_cap are never read.
 *  cand_pos, cand_count, C_cap   as written by pldp_find_candidates; entries
 *             past min(cand_count, C_cap) are ignored.
 *  scores     float [B, C_cap] out or NULL: score of the i-th listed candidate.
 *             j = 0 (no H_{-1}) and positions outside [0, t) score -INFINITY
 *             and are never chosen.  A zero-norm row gives score 0.
 *  best_pos   int32 [B] out: j*, or -1 when no candidate is eligible.
 *  best_score float [B] out or NULL: score of j* (-INFINITY when none).
 *  status     uint32 [B] or NULL.
 * Scores are accumulated in fp32.  Ties go to the smaller position j; the
 * choice is deterministic for given inputs.  When H rows are 16-byte aligned
 * (H aligned, d*sizeof(dtype) and seq_stride*sizeof(dtype) multiples of 16)
 * the query row is staged in shared memory by a bulk asynchronous copy.
 */
PLDP_API pldp_status pldp_rank_hidden(const void* H, pldp_dtype dtype, int64_t d,
                                      int64_t seq_stride, const int32_t* seq_len, int B,
                                      int64_t T_cap, const int32_t* cand_pos,
                                      const int32_t* cand_count, int C_cap, float threshold,
                                      float* scores, int32_t* best_pos, float* best_score,
                                      uint32_t* status, void* stream);

/*
 * Ranking by averaged hidden states -- the variant of Eq. 3 studied in App. B.2
 * (the paper reports it does not help; it is here for completeness):
 *   Hbar_p  = mean(H_{max(0, p-m+1)}, ..., H_p)     (the m rows ending at p)
 *   score_j = cos(Hbar_{j-1}, Hbar_{t-1}),  j* = argmax_{j in P} score_j.
 * The printed formula averages H_1..H_m for every position; it is read as the
 * window of the m positions ending at the one averaged, cut at position 0.
 * m = 1 is Eq. 3.  Arguments, outputs and conventions as pldp_rank_hidden, plus
 *  m   window length, >= 1.
 * Limit: d * 4 <= 196608 (the query's window sum is held in fp32 in shared memory).
 */
PLDP_API pldp_status pldp_rank_hidden_avg(const void* H, pldp_dtype dtype, int64_t d,
                                          int64_t seq_stride, int m, const int32_t* seq_len, int B,
                                          int64_t T_cap, const int32_t* cand_pos,
                                          const int32_t* cand_count, int C_cap, float threshold,
                                          float* scores, int32_t* best_pos, float* best_score,
                                          uint32_t* status, void* stream);

/*
 * Ranking by attentions -- Eq. 2 (Sec. 4.2.1):
 *   score_j = max over the selected (layer, head) rows of A^{(l,g)}_{t-1}[j],
 *   j* = argmax_{j in P} score_j;  agg = PLDP_AGG_SUM sums the rows instead
 *   (the aggregation variant of Sec. 7.1).
 * The key index of Eq. 2 is read as the candidate j itself (the position an
 * induction head at query t-1 attends to is the token it copies).
 *
 *  A          dtype; for sequence b and row r the attention probabilities of
 *             query t-1 over keys:
 *               A + b*seq_stride + r*row_stride + key*key_stride.
 *             Rows with contiguous keys (key_stride = 1, row_stride >= T_cap) are
 *             the natural layout of one head's probabilities; the key-major layout
 *             (row_stride = 1, key_stride >= R) puts the R values of one key side
 *             by side, so each candidate's values are one contiguous read instead
 *             of R scattered 32-byte sectors.  A may also be page-locked host
 *             memory that device code can address (a cudaHostAlloc allocation
 *             under unified addressing): the kernels read only the selected rows'
 *             values at the candidate keys, so rows kept on the host need not be
 *             copied to the device whole.
 *  R          rows per sequence (>= 1).
 *  row_stride, key_stride   >= 1 (key_stride 0 is read as 1); the rows must not
 *             overlap: row_stride >= T_cap * key_stride or key_stride >= R *
 *             row_stride.  seq_stride >= (R-1)*row_stride + (T_cap-1)*key_stride + 1.
 *  row_idx    int32 [n_sel] device, or NULL for all R rows: the selected
 *             (layer, head) rows L* x G*.  Entries outside [0, R) are ignored
 *             and set ROW_INDEX.
 *  seq_len, T_cap, cand_pos, cand_count, C_cap, status   as pldp_rank_hidden.
 *  scores     float [B, C_cap] out or NULL.  Positions outside [0, t) score
 *             -INFINITY and are never chosen.
 *  best_pos, best_score   as pldp_rank_hidden.  Ties go to the smaller j.
 * MAX is exact; SUM accumulates in fp32 in a fixed order.
 */
PLDP_API pldp_status pldp_rank_attention(const void* A, pldp_dtype dtype, int R,
                                         int64_t row_stride, int64_t key_stride, int64_t seq_stride,
                                         const int32_t* row_idx, int n_sel, pldp_agg agg,
                                         const int32_t* seq_len, int B, int64_t T_cap,
                                         const int32_t* cand_pos, const int32_t* cand_count,
                                         int C_cap, float* scores, int32_t* best_pos,
                                         float* best_score, uint32_t* status, void* stream);

/*
 * Draft prediction -- Sec. 4.3:  xhat_i = x_{j*+i}, i = 1..K.
 * The span stops at the last token x_t: draft_len[b] = min(K, t - j*) tokens,
 * the rest of draft[b, :] is -1.  best_pos[b] = -1 (or outside [0, t), or an
 * invalid seq_len) gives draft_len 0.
 *
 *  ids, ids_stride, seq_len, T_cap   as pldp_find_candidates.
 *  best_pos   int32 [B].
 *  K          draft length, >= 1.
 *  draft      int32 [B, K] out;  draft_len  int32 [B] out.
 */
PLDP_API pldp_status pldp_extract_draft(const int32_t* ids, int64_t ids_stride,
                                        const int32_t* seq_len, int64_t T_cap,
                                        const int32_t* best_pos, int B, int K,
                                        int32_t* draft, int32_t* draft_len, void* stream);

/*
 * The drafting half of a step in one call: candidate search, ranking by hidden
 * states and/or attentions, and draft extraction, with the results of
 * pldp_find_candidates, pldp_rank_hidden, pldp_rank_attention and
 * pldp_extract_draft called in turn (same conventions, same status bits; the
 * fp32 score sums may be split differently, so scores can differ in the last
 * bits and a tie within rounding may be broken differently).  Eq. 1-3
 * (Sec. 4.2) and Sec. 4.3.
 *
 * A thread-block cluster per sequence: each CTA scans its chunk of the context once
 * and keeps the positions with the longest suffix match it met; the cluster then
 * knows the candidate list and deals the candidates out to its CTAs, which score
 * them (cosine and attention score), and its first CTA picks the best of each
 * ranking and writes the draft.  Sequences with many candidates are finished by a
 * second launch that spreads them over the whole GPU (through the workspace).
 *
 * Fields of the argument block (device pointers unless stated):
 *  ids .. match_len      as pldp_find_candidates (T_cap <= 2^27).
 *  H .. best_h_score     as pldp_rank_hidden (H = NULL skips hidden ranking;
 *                        H rows must be 16-byte aligned).  h_scores and
 *                        best_h_score may be NULL.
 *  A .. best_a_score     as pldp_rank_attention (A = NULL skips it; either
 *                        layout, a_key_stride as its key_stride; A may be
 *                        device-addressable page-locked host memory); a_scores
 *                        and best_a_score may be NULL.
 *  draft_from            0: draft after best_h, 1: after best_a (that ranking
 *                        must be given).
 *  K, draft, draft_len   as pldp_extract_draft.
 *  status                uint32 [B] or NULL.
 *  workspace             device scratch of pldp_draft_workspace_size(B) bytes,
 *                        16-byte aligned, ZEROED by the caller before its first
 *                        use; every call leaves it zeroed.  Calls that may
 *                        run concurrently need separate workspaces.  May be NULL
 *                        when an index is given.
 *  index, index_bytes, V optional incremental token index (NULL: scan the
 *                        contexts): device memory of pldp_index_size(B, V)
 *                        bytes, built by pldp_index_build, for token ids in
 *                        [0, V).  With it, a step looks up the occurrences of
 *                        x_t instead of scanning the context, and appends the
 *                        positions added since the last step; results are the
 *                        same as without it (a token with more than 15 earlier
 *                        occurrences, or a sequence whose index is unusable,
 *                        is scanned).  The index must only ever see the
 *                        contexts grow by appending: a sequence whose length
 *                        fell below what was indexed is marked unusable (and
 *                        scanned) until the index is rebuilt.
 * Layouts the fused path does not take return PLDP_ERR_UNSUPPORTED; the
 * separate calls accept them.
 */
typedef struct pldp_draft_step_args {
    const int32_t* ids;
    int64_t ids_stride;
    const int32_t* seq_len;
    int B;
    int64_t T_cap;
    int ngram_min;
    int ngram_max;
    int32_t* cand_pos;
    int C_cap;
    int32_t* cand_count;
    int32_t* match_len;
    const void* H;
    pldp_dtype h_dtype;
    int64_t d;
    int64_t h_seq_stride;
    float threshold;
    float* h_scores;
    int32_t* best_h;
    float* best_h_score;
    const void* A;
    pldp_dtype a_dtype;
    int R;
    int64_t a_row_stride;
    int64_t a_key_stride;   /* elements between keys of a row; 0 is read as 1 */
    int64_t a_seq_stride;
    const int32_t* row_idx;
    int n_sel;
    pldp_agg agg;
    float* a_scores;
    int32_t* best_a;
    float* best_a_score;
    int draft_from;
    int K;
    int32_t* draft;
    int32_t* draft_len;
    uint32_t* status;
    void* workspace;
    size_t workspace_bytes;
    void* index;
    size_t index_bytes;
    int V;
} pldp_draft_step_args;

/* `args` is a HOST pointer to the argument block, read before the call returns. */
PLDP_API pldp_status pldp_draft_step(const pldp_draft_step_args* args, void* stream);

/* Bytes of workspace pldp_draft_step needs for B sequences (0 if B < 0). */
PLDP_API size_t pldp_draft_workspace_size(int B);

/*
 * The incremental token index of pldp_draft_step (no counterpart in the paper:
 * it is a way to find the occurrences of Eq. 1 without rescanning the context).
 * Per sequence and token it holds the number of occurrences among the indexed
 * positions and up to 15 of them (one 64-byte entry); per sequence the number of
 * positions indexed.
 * pldp_index_build overwrites `index` and indexes positions 0 .. seq_len[b]-2 of
 * every sequence (all but the last token, which the next draft step looks up).
 * Token ids outside [0, V) mark that sequence's index unusable (TOKEN_RANGE);
 * seq_len outside [0, T_cap] too (SEQ_LEN).  Memory: about B * V * 64 bytes.
 * The last 32 (B + 1) bytes (rounded up to 256) are scratch of the drafting calls;
 * memory without them does too, with the same results and slower calls on contexts
 * that repeat their tokens much.
 */
PLDP_API size_t pldp_index_size(int B, int V);
PLDP_API pldp_status pldp_index_build(const int32_t* ids, int64_t ids_stride, const int32_t* seq_len,
                                      int B, int64_t T_cap, int V, void* index,
                                      size_t index_bytes, uint32_t* status, void* stream);

/*
 * Greedy verification -- Sec. 4.4 at temperature 0, with the K+1 next-token
 * distributions of one forward pass on the draft (Sec. 3):
 *   a_i   = argmax_v logits[b, i, v], i = 0..K   (smallest v among equal maxima;
 *           -0.0 equals +0.0)
 *   n     = first i < draft_len[b] with draft[b, i] != a_i, else draft_len[b]
 *   bonus = a_n
 * accept_len[b] = n and next_token[b] = bonus: the step emits
 * draft[b, 0..n-1] followed by bonus, exactly what greedy decoding emits.
 *
 *  logits     dtype [B, K+1, V], contiguous.  Fast path when logits is 16-byte
 *             aligned and V * sizeof(dtype) is a multiple of 16.
 *  draft      int32 [B, K];  draft_len  int32 [B] (outside [0, K]: clamped,
 *             DRAFT_LEN).  Draft tokens outside [0, V) never match (TOKEN_RANGE).
 *  argmax     int32 [B, K+1] out or NULL: every a_i.
 *  accept_len int32 [B] out;  next_token int32 [B] out.
 *  seq_len    int32 [B] in/out or NULL.  When given (valid range [1, T_cap],
 *             else SEQ_LEN and no bookkeeping for b), with L the old value:
 *               kv_keep_len[b] = L + n   (x_t and the n accepted tokens are the
 *                                         positions whose keys/values survive)
 *               if L + n + 1 <= T_cap: ids[b, L..L+n-1] = draft[b, 0..n-1],
 *                 ids[b, L+n] = bonus (ids may be NULL), seq_len[b] = L + n + 1;
 *               else CAPACITY and neither ids nor seq_len changes.
 *  ids, ids_stride, T_cap   the context rows to append to (ids may be NULL).
 *  kv_keep_len int32 [B] out or NULL (needs seq_len).
 *  status     uint32 [B] or NULL.
 *  workspace  device scratch of at least pldp_verify_workspace_size(B, K, V)
 *             bytes, 16-byte aligned, ZEROED by the caller before its first
 *             use.  Every call returns it to all-zero when it completes, so
 *             it can be reused by the next call on the same stream (or graph
 *             replay) without clearing.  Calls that may run concurrently need
 *             separate workspaces.
 */
PLDP_API pldp_status pldp_verify_greedy(const void* logits, pldp_dtype dtype, int B, int K,
                                        int V, const int32_t* draft, const int32_t* draft_len,
                                        int32_t* argmax, int32_t* accept_len,
                                        int32_t* next_token, int32_t* ids, int64_t ids_stride,
                                        int32_t* seq_len, int64_t T_cap, int32_t* kv_keep_len,
                                        uint32_t* status, void* workspace,
                                        size_t workspace_bytes, void* stream);

/*
 * Greedy verification of the current step followed by the drafting of the next
 * one, in one call -- pldp_verify_greedy then pldp_draft_step (with the token
 * index) on the context it has just extended, with the same results and status
 * bits as those two calls in turn.  The paper has no counterpart: in a decode
 * loop the next draft depends only on this step's verification (the accepted
 * tokens, the bonus token) and on the hidden states and attention rows of the
 * forward pass that produced this step's logits, so nothing runs between the
 * two.  The argmax pass is followed, one CTA per sequence, by the accept/bonus/
 * append of verification and then the candidate search, ranking and draft of
 * the next step.
 *
 *  logits, dtype, V   this step's logits [B, K+1, V], as pldp_verify_greedy.
 *  draft, draft_len   this step's draft [B, K] and lengths [B]; they may be the
 *                     same buffers as next.draft and next.draft_len (each
 *                     sequence's draft is read before it is replaced).
 *  argmax, accept_len, next_token, kv_keep_len, workspace, workspace_bytes
 *                     as pldp_verify_greedy (workspace zeroed before first use;
 *                     every call leaves it zero).
 *  next               the next step's pldp_draft_step arguments.  next.index is
 *                     required (built by pldp_index_build, with next.V == V).
 *                     next.B and next.K are the verification's B and K;
 *                     next.ids, next.ids_stride, next.seq_len and next.T_cap are
 *                     the context verification appends to (read and WRITTEN by
 *                     this call); next.status receives both calls' bits.
 *                     next.workspace is not used.
 */
typedef struct pldp_verify_draft_args {
    const void* logits;
    pldp_dtype dtype;
    int V;
    const int32_t* draft;
    const int32_t* draft_len;
    int32_t* argmax;
    int32_t* accept_len;
    int32_t* next_token;
    int32_t* kv_keep_len;
    void* workspace;
    size_t workspace_bytes;
    pldp_draft_step_args next;
} pldp_verify_draft_args;

/* `args` is a HOST pointer to the argument block, read before the call returns. */
PLDP_API pldp_status pldp_verify_greedy_draft(const pldp_verify_draft_args* args, void* stream);

/*
 * Sampling verification -- Sec. 4.4 at temperature T > 0 (the paper's sampled
 * runs use T = 1, Table 2).  Position i of sequence b draws
 *   y_i = the smallest v with sum_{v' <= v} p_v' > u[b, i],
 *         p = softmax(logits[b, i] / T)                  (inverse-CDF sampling)
 * from the caller's uniform u[b, i]; then, as for greedy verification,
 *   n = first i < draft_len[b] with draft[b, i] != y_i, else draft_len[b];
 *   bonus = y_n.
 * For a draft with one token per position (PLD+'s draft) this accepts draft_i
 * with probability p(draft_i) and on a rejection draws the bonus from p
 * restricted to the other tokens: the step emits exactly what sampling from the
 * target alone would.  The random numbers are inputs: the same uniforms give
 * the same draws.
 *
 *  logits        dtype [B, K+1, V], contiguous, finite.  Fast path when logits is
 *                16-byte aligned and V * sizeof(dtype) is a multiple of 16.
 *  temperature   T > 0, finite (else PLDP_ERR_INVALID_ARG).
 *  uniforms      float [B, K+1]; values outside [0, 1) are clamped into it.
 *  sampled       int32 [B, K+1] out or NULL: every y_i.
 *  draft, draft_len, accept_len, next_token, ids, ids_stride, seq_len, T_cap,
 *  kv_keep_len, status   as pldp_verify_greedy.
 *  workspace     device scratch of pldp_verify_sample_workspace_size(B, K, V, dtype)
 *                bytes, 16-byte aligned (no zeroing needed).
 * Probabilities are computed in fp32 (per-2 KB-piece maxima and sums of
 * exp2(log2(e) (l - max) / T)); a draw can differ from the exact draw only when
 * u lies within fp32 rounding (~1e-6) of a boundary of the cumulative
 * distribution.  K + 1 <= 12288.
 */
PLDP_API pldp_status pldp_verify_sample(const void* logits, pldp_dtype dtype, int B, int K, int V,
                                        float temperature, const float* uniforms,
                                        const int32_t* draft, const int32_t* draft_len,
                                        int32_t* sampled, int32_t* accept_len,
                                        int32_t* next_token, int32_t* ids, int64_t ids_stride,
                                        int32_t* seq_len, int64_t T_cap, int32_t* kv_keep_len,
                                        uint32_t* status, void* workspace,
                                        size_t workspace_bytes, void* stream);

/* Bytes of workspace pldp_verify_sample needs (0 if invalid). */
PLDP_API size_t pldp_verify_sample_workspace_size(int B, int K, int V, pldp_dtype dtype);

/*
 * Sampling verification of the current step followed by the drafting of the
 * next one, in one call -- pldp_verify_sample then pldp_draft_step (with the
 * token index) on the context it has just extended, with the same results and
 * status bits as those two calls in turn.  Sec. 4.4 at temperature T > 0 (the
 * paper's sampled runs use T = 1, Table 2), then Eq. 1-3 and Sec. 4.3; the paper
 * has no fused form.  Four launches: the per-piece stats pass over the logits,
 * one warp per row that draws, one CTA per sequence that accepts, appends and
 * drafts the next step, then the scoring of sequences with many candidates.
 *
 *  logits, dtype, V   this step's logits [B, K+1, V], as pldp_verify_sample.
 *  temperature        T > 0, finite (else PLDP_ERR_INVALID_ARG).
 *  uniforms           float [B, K+1], as pldp_verify_sample (clamped into [0, 1)).
 *  draft, draft_len   this step's draft [B, K] and lengths [B]; they may be the
 *                     same buffers as next.draft and next.draft_len.
 *  sampled            int32 [B, K+1] out or NULL: every draw y_i.
 *  accept_len, next_token, kv_keep_len   as pldp_verify_greedy.
 *  workspace          device scratch of pldp_verify_sample_draft_workspace_size(
 *                     B, K, V, dtype) bytes, 16-byte aligned (no zeroing needed).
 *                     Calls that may run concurrently need separate workspaces.
 *  next               the next step's pldp_draft_step arguments, as for
 *                     pldp_verify_greedy_draft (next.index required, next.V == V,
 *                     next.B and next.K are the verification's B and K, next.ids /
 *                     next.seq_len are appended to, next.status receives both
 *                     calls' bits, next.workspace is not used).
 * K + 1 <= 12288.  The draws are those of pldp_verify_sample on the same inputs.
 */
typedef struct pldp_verify_sample_draft_args {
    const void* logits;
    pldp_dtype dtype;
    int V;
    float temperature;
    const float* uniforms;
    const int32_t* draft;
    const int32_t* draft_len;
    int32_t* sampled;
    int32_t* accept_len;
    int32_t* next_token;
    int32_t* kv_keep_len;
    void* workspace;
    size_t workspace_bytes;
    pldp_draft_step_args next;
} pldp_verify_sample_draft_args;

/* `args` is a HOST pointer to the argument block, read before the call returns. */
PLDP_API pldp_status pldp_verify_sample_draft(const pldp_verify_sample_draft_args* args, void* stream);

/* Bytes of workspace pldp_verify_sample_draft needs (0 if invalid). */
PLDP_API size_t pldp_verify_sample_draft_workspace_size(int B, int K, int V, pldp_dtype dtype);

/*
 * Greedy verification without a caller workspace.  The paper has no counterpart:
 * this is a deployment convenience.  Same arguments, results and status bits as
 * pldp_verify_greedy, minus the workspace.
 *
 * Who needs it: callers that cannot allocate device memory for a workspace --
 * code embedded in a host program that owns every GPU allocation, and serving
 * loops that must not call cudaMalloc/cudaFree after start-up because those
 * calls can synchronise the whole device.
 *
 * The scratch lives in a fixed 1 MiB area compiled into the library; every GPU
 * that loads the library keeps it until the process exits.  Requests needing
 * more than that (pldp_verify_workspace_size(B, K, V) > 1048576, i.e. roughly
 * B*(K+1) > 130000 rows) are rejected with PLDP_ERR_INVALID_ARG.  The call
 * allocates nothing: it clears the part of the area it uses with
 * cudaMemsetAsync on `stream`, then launches the verification kernels.
 *
 * Every call looks up the area's device address in the CUDA context current on
 * the calling thread (cudaGetSymbolAddress, which allocates nothing), so a
 * switch of context or a device reset between calls never leaves it a stale
 * address.  The first call in a context also makes the runtime load the
 * library's device code there; make that first call before any stream capture.
 * All calls on a device share the one area, which keeps whatever the last call
 * left there: calls that can overlap on the GPU (different streams, or threads
 * without ordering between them) race on it and must be serialised by the
 * caller.
 */
PLDP_API pldp_status pldp_verify_greedy_noalloc(const void* logits, pldp_dtype dtype, int B,
                                                int K, int V, const int32_t* draft,
                                                const int32_t* draft_len, int32_t* argmax,
                                                int32_t* accept_len, int32_t* next_token,
                                                int32_t* ids, int64_t ids_stride,
                                                int32_t* seq_len, int64_t T_cap,
                                                int32_t* kv_keep_len, uint32_t* status,
                                                void* stream);

/* Bytes of workspace pldp_verify_greedy needs for these sizes (0 if invalid). */
PLDP_API size_t pldp_verify_workspace_size(int B, int K, int V);

/*
 * Induction-head identification -- Sec. 4.2.1, the offline step that picks the
 * (layer, head) rows Eq. 2 aggregates.  Each observation b is a generated token
 * x_p (p = pos[b]) with its context ids[b, 0..p] and the attention rows of query
 * p-1 over keys 0..p-1 for R candidate (layer, head) rows:
 *   P      = {j < p : x_j = x_p}
 *   ov(j)  = the largest k <= max_suffix with x_{j-i} = x_{p-i} for all i < k
 *   r*     = argmax_{j in P} ov(j)              (the smaller j on ties)
 *   counts[r] += 1 when row r's largest attention is at key r*
 *                                               (the smaller key on ties)
 * The paper's rule is read per row: a head counts when r* is where its own
 * attention peaks.  Run it over many observations, then keep the rows with the
 * most counts (pldp_top_heads).
 *
 *  B          observations, at most 65535 (else PLDP_ERR_UNSUPPORTED).
 *  ids, ids_stride, T_cap   int32 contexts [B, ids_stride], T_cap <= ids_stride.
 *  pos        int32 [B]; outside [1, T_cap - 1]: SEQ_LEN, nothing counted.
 *  max_suffix >= 1: cap on ov(j).
 *  A          dtype [B, seq_stride]: row r of observation b at
 *             A + b*seq_stride + r*row_stride, keys 0..p-1 (row_stride >= T_cap,
 *             seq_stride >= R*row_stride).
 *  counts     uint32 [R], ADDED to (initialise once, accumulate over calls).
 *  r_star     int32 [B] out or NULL: r*, -1 when x_p does not occur before p.
 *  status     uint32 [B] or NULL.
 * Atomic adds on counts: concurrent calls on one counts array accumulate
 * correctly.  Offline utility: not part of the decode step.
 */
PLDP_API pldp_status pldp_identify_heads(const int32_t* ids, int64_t ids_stride, const int32_t* pos,
                                         int B, int64_t T_cap, int max_suffix, const void* A,
                                         pldp_dtype dtype, int R, int64_t row_stride,
                                         int64_t seq_stride, uint32_t* counts, int32_t* r_star,
                                         uint32_t* status, void* stream);

/*
 * The k rows with the most counts (ties to the smaller row index), written in
 * that order to row_idx int32 [k] -- the row_idx argument of pldp_rank_attention.
 * 1 <= k <= R <= 8192.  counts: uint32 [R] (device).
 */
PLDP_API pldp_status pldp_top_heads(const uint32_t* counts, int R, int k, int32_t* row_idx, void* stream);

/* ---------------------------------------------------------------------------
 * The target model's cache around a step
 * ---------------------------------------------------------------------------
 * Verification's K+1 distributions come from one forward pass of the target model
 * over x_t and the draft (Sec. 4.4).  In each of its layers these calls norm and
 * rotate the new tokens' queries and keys and write keys and values to a paged
 * cache (pldp_cache_append), attend over the cache (pldp_attend_cache), and rank the
 * next step's candidates by that attention without its rows ever being written out
 * (pldp_rank_cache, Eq. 2); pldp_cache_read takes positions back out of the cache,
 * pldp_token_logprobs scores tokens under the logits.
 *
 * The step's tokens of sequence b are x_t and its draft: token i = 0..draft_len[b]
 * stands at position seq_len[b]-1+i, as verification numbers them.  (A prompt, or a
 * chunk of one that starts at position p, is the same with seq_len = p+1 and the
 * tokens after its first as the draft.)  The positions of tokens that verification
 * rejects are simply written again by the next step.
 *
 *  k, v       the pools of pages: the vector of position p, head h of sequence b is
 *               base + pages[b][p / page_size]*page_stride + (p % page_size)*pos_stride
 *                    + h*head_stride,  head_dim contiguous elements,
 *             the same strides for both; strides in elements, so either order of
 *             positions and heads within a page can be given.  Base 16-byte aligned,
 *             strides multiples of 16 bytes.
 *  dtype      PLDP_BF16, or PLDP_E4M3: 8-bit codes (4 exponent and 3 mantissa bits,
 *             largest 448) and one fp32 scale for each vector,
 *             value = code * scale, scales finite and 2^-80 (8.3e-25) or more.  A vector of
 *             zeros should have that smallest scale: attention's weights round relative to
 *             the largest of weight * scale.
 *  k_scale, v_scale   float [n_pages, heads, page_size], contiguous (PLDP_E4M3; else NULL).
 *  n_pages, page_size  >= 1, any size; max_pages * page_size < 2^31 (pldp_attend_cache:
 *             <= 2^31 - 4096).
 *  heads      key/value heads, 1..1024; head_dim a multiple of 16, 16..256.
 *  pages      int32 [B, pages_stride]: the page of each page_size positions, max_pages
 *             entries a sequence.  An entry outside [0, n_pages) sets PAGE: its
 *             positions are not written, read as zeros and attended to by nothing.
 */
typedef struct {
    void* k;
    void* v;
    pldp_dtype dtype;
    float* k_scale;
    float* v_scale;
    int n_pages, page_size, heads, head_dim;
    int64_t page_stride, pos_stride, head_stride;
    const int32_t* pages;
    int64_t pages_stride;
    int max_pages;
} pldp_cache;

/*
 * Appends a step's tokens to the cache.  For every token, in fp32:
 *   queries and keys   x <- x * rsqrt(mean(x^2) + eps) * norm     (q_norm / k_norm not NULL)
 *                      (a, b) <- (a cos - b sin, b cos + a sin)   (cos not NULL)
 *   q_out <- bf16(q);  the cache's keys and values <- k, v rounded to bf16, or in a
 *   PLDP_E4M3 cache scale = max(max|x| * (1/448), 2^-80), code = x / scale (in fp32,
 *   rounded to the nearest code).
 *
 *  q, k, v    dtype (PLDP_F32 or PLDP_BF16): [B, n, q_heads or cache.heads, head_dim]
 *             with strides of their own (sequence, token, head; elements), 16-byte
 *             aligned, strides multiples of 16 bytes: slices of one projection's output
 *             do.
 *  n          tokens a sequence has room for, >= 1 (K+1).
 *  q_heads    a multiple of cache.heads is needed by pldp_attend_cache only.
 *  q_norm, k_norm   dtype [head_dim], 16-byte aligned, or NULL; eps >= 0.
 *  cos, sin   float [rot_rows, rot/2], row p for position p, 16-byte aligned, or both
 *             NULL.  rot even, 2..head_dim: the first rot elements rotate, in pairs
 *             (e, e + rot/2), or (2e, 2e+1) when interleaved is not 0.
 *  seq_len    int32 [B], 1..capacity (0: nothing to do; else SEQ_LEN, skipped); the
 *             capacity is max_pages * page_size, and rot_rows where that is less.
 *  draft_len  int32 [B], or NULL for n-1; outside [0, n-1]: DRAFT_LEN, clamped.
 *  q_out      bf16 [B, n, q_heads, head_dim] with strides; may be q itself (bf16).
 *  status     uint32 [B] or NULL.
 * Tokens past draft_len leave q_out untouched, and so do tokens at or past the capacity
 * (CAPACITY).
 */
typedef struct {
    pldp_cache cache;
    const void* q;
    const void* k;
    const void* v;
    pldp_dtype dtype;
    int B, n, q_heads;
    int64_t q_strides[3], k_strides[3], v_strides[3]; /* sequence, token, head */
    const void* q_norm;
    const void* k_norm;
    float eps;
    const float* cos;
    const float* sin;
    int rot, interleaved;
    int64_t rot_rows;
    const int32_t* seq_len;
    const int32_t* draft_len;
    void* q_out;
    int64_t q_out_strides[3];
    uint32_t* status;
} pldp_cache_append_args;

PLDP_API pldp_status pldp_cache_append(const pldp_cache_append_args* args, void* stream);

/*
 * Reads positions start[b] .. start[b]+count[b]-1 of every sequence out of the cache into
 * dense rows 0..count[b]-1.
 *
 *  k_out, v_out   dtype (PLDP_F32 or PLDP_BF16) [B, n, cache.heads, head_dim] with the
 *             strides given (sequence, position, head; elements, the same for both),
 *             16-byte aligned, strides multiples of 16 bytes; v_out or k_out may be NULL.
 *  start      int32 [B], or NULL for 0.  count int32 [B], 0..n (else clamped,
 *             SEQ_LEN); a start outside the capacity, or a count that passes it, is cut
 *             there (CAPACITY).
 * Rows at and past count[b] are left untouched.
 */
typedef struct {
    pldp_cache cache;
    const int32_t* start;
    const int32_t* count;
    int B, n;
    pldp_dtype dtype;
    void* k_out;
    void* v_out;
    int64_t out_strides[3];
    uint32_t* status;
} pldp_cache_read_args;

PLDP_API pldp_status pldp_cache_read(const pldp_cache_read_args* args, void* stream);

/*
 * Attention of a step's tokens over the cache (their own keys and values included: append
 * first).  Token i of sequence b, query head h, with kv head h / (q_heads / cache.heads):
 *   s_j   = scale * q . k_j   for positions j = 0 .. seq_len[b]-1+i
 *   out   = sum_j exp(s_j - lse) v_j,   lse = ln sum_j exp(s_j)
 *
 *  q          bf16 [B, n, q_heads, head_dim] with strides (sequence, token, head),
 *             16-byte aligned, strides multiples of 16 bytes.
 *  q_heads    a multiple of cache.heads.
 *  seq_len, draft_len   as pldp_cache_append (the capacity is max_pages * page_size).
 *  scale      finite; 1/sqrt(head_dim) as a rule.
 *  out        bf16 [B, n, q_heads, head_dim] with strides, as q; it must not overlap q.
 *  lse        float [B, n, q_heads], contiguous, or NULL.
 *  workspace  pldp_attend_workspace_size bytes, 256-byte aligned, zeroed once before
 *             first use (every call leaves it zeroed where that matters; not one that
 *             sets TIMEOUT: zero it again).  Calls of different shapes may share one of the
 *             largest size; calls that may run concurrently need separate ones.
 *  status     uint32 [B] or NULL.  TIMEOUT: a wait inside the kernel ran out; the call's
 *             results are none.
 * Rows with nothing to attend to (tokens past draft_len, sequences skipped, positions
 * past the capacity) are written as zeros, their lse as -INFINITY.  Keys and values
 * past a sequence's last new token are never used, whatever they hold; those of its new
 * tokens must be finite for all of its rows, and a bf16 cache's values below 2^32 in size.
 * Sums and the running maximum are held in fp32; each weight exp(s_j - lse) is rounded on
 * its way into the products, by up to 2^-17 of it over a bf16 cache and 2^-11 over an e4m3
 * one; results are the same for the same inputs, however the work is scheduled.
 * A step's rows are what this is made for: of a prompt every 128 rows go through all of
 * their sequence's keys (pldp_attend_prompt: those that they see).
 */
typedef struct {
    pldp_cache cache;
    const void* q;
    int B, n, q_heads;
    int64_t q_strides[3];
    const int32_t* seq_len;
    const int32_t* draft_len;
    float scale;
    void* out;
    int64_t out_strides[3];
    float* lse;
    uint32_t* status;
    void* workspace;
    size_t workspace_bytes;
} pldp_attend_args;

PLDP_API pldp_status pldp_attend_cache(const pldp_attend_args* args, void* stream);

PLDP_API size_t pldp_attend_workspace_size(int B, int n, int q_heads, int heads, int head_dim);

/*
 * Ranking by attentions (Eq. 2, as pldp_rank_attention) straight from one layer's cache:
 * the attention of one query row a sequence at the candidates, from the row's queries, the
 * candidates' keys and the lse that pldp_attend_cache wrote,
 *   score_j = max (or sum) over the selected heads h of exp(scale * q_h . k_j - lse_h),
 * so no attention row is ever written out.  After verification the query t-1 of the new x_t
 * is row accept_len[b] of the step, and the positions before it are kv_keep_len[b].
 *
 *  q, q_heads, q_strides, scale, lse   of the step's pldp_attend_cache (lse [B, n, q_heads]).
 *  row        int32 [B] (accept_len), or NULL for row 0; outside [0, n): ROW_INDEX, no
 *             result (scores of -INFINITY, best_pos -1).
 *  kv_len     int32 [B] (kv_keep_len), 0..capacity (else SEQ_LEN, no result): candidates
 *             outside [0, kv_len) score -INFINITY and are never chosen, with accumulate too.
 *  heads      int32 [n_sel], or NULL for all q_heads (n_sel ignored): the selected query heads;
 *             entries outside [0, q_heads) are ignored and set ROW_INDEX.
 *             n_sel * head_dim <= 49152.
 *  accumulate not 0: scores holds those of other layers, and a candidate's score is
 *             the larger of both (MAX) or their sum (SUM): call layer by layer.  A
 *             candidate that this layer has no score for (PAGE, or no entry of heads is a
 *             head) keeps theirs; without accumulate it scores -INFINITY.
 *  cand_pos, cand_count, C_cap   as written by pldp_find_candidates.
 *  scores     float [B, C_cap] out, or NULL (not with accumulate).
 *  best_pos, best_score, status  as pldp_rank_attention; ties go to the smaller j.
 */
typedef struct {
    pldp_cache cache;
    const void* q;
    int B, n, q_heads;
    int64_t q_strides[3];
    const int32_t* row;
    const int32_t* kv_len;
    const float* lse;
    const int32_t* heads;
    int n_sel;
    pldp_agg agg;
    int accumulate;
    float scale;
    const int32_t* cand_pos;
    const int32_t* cand_count;
    int C_cap;
    float* scores;
    int32_t* best_pos;
    float* best_score;
    uint32_t* status;
} pldp_rank_cache_args;

PLDP_API pldp_status pldp_rank_cache(const pldp_rank_cache_args* args, void* stream);

/*
 * Log probabilities of given tokens, with the entropy and the likeliest alternatives, of
 * `rows` rows of logits (a step's B * (K+1), say) at temperature T: x = logits / T,
 *   lse = ln sum_v exp(x_v),  logprob = x_token - lse,  entropy = lse - sum_v p_v x_v.
 *
 *  logits     dtype [rows, V], contiguous, aligned to its elements, rows below 2^31 and
 *             V below 2^31 - 4096.
 *             -INFINITY is allowed (a masked token: p = 0).  A row with NaN or +INFINITY has no
 *             probabilities; its alternatives are tokens all the same.
 *  tokens     int32 [rows], or NULL (no logprob); outside [0, V): logprob -INFINITY.
 *  logprob, entropy   float [rows] out or NULL.
 *  top        alternatives wanted, 0..32 and <= V: top_id int32 [rows, top] and top_logprob
 *             float [rows, top], by descending logit, ties to the lower index (either
 *             may be NULL).
 *  workspace  pldp_token_logprobs_workspace_size bytes, 16-byte aligned; need not be
 *             cleared.  Calls that may run concurrently need separate ones.
 * A row of -INFINITY throughout: logprob -INFINITY, entropy 0, top_id 0, 1, ... with
 * -INFINITY.
 */
PLDP_API pldp_status pldp_token_logprobs(const void* logits, pldp_dtype dtype, int64_t rows, int V,
                                         float temperature, const int32_t* tokens, float* logprob,
                                         float* entropy, int top, int32_t* top_id,
                                         float* top_logprob, void* workspace,
                                         size_t workspace_bytes, void* stream);

PLDP_API size_t pldp_token_logprobs_workspace_size(int64_t rows, int V);

/* ---------------------------------------------------------------------------
 * Prompts: sequences of different lengths, packed
 * ---------------------------------------------------------------------------
 * The tokens of B prompts (or chunks of prompts) behind one another, without padding: those of
 * sequence b are rows rows[b] .. rows[b+1]-1, its row rows[b]+i stands at position start[b]+i.
 *
 *  R          rows of the tensors, >= 0 and below 2^31 - 256; rows behind rows[B] (or before
 *             rows[0]) belong to no sequence: nothing of them is used, nothing is written there.
 *  rows       int32 [B+1], ascending, 0 <= rows[b] <= rows[b+1] <= R; a sequence may have no
 *             rows.  Where a pair descends or leaves [0, R]: SEQ_LEN, that sequence is skipped, and
 *             no other one (rows that two sequences then claim hold what either gives them).
 *  start      int32 [B], or NULL for 0; outside [0, capacity]: SEQ_LEN, skipped.  Tokens at
 *             or past the capacity: CAPACITY, they take no part.
 */

/*
 * pldp_cache_append of packed tokens: the same arithmetic and results, and the same arguments,
 * without draft_len; q, k, v and q_out are [R, heads, head_dim] with strides (token, head).
 * The capacity is max_pages * page_size, and rot_rows where that is less.  B and R below 2^31.
 */
typedef struct {
    pldp_cache cache;
    const void* q;
    const void* k;
    const void* v;
    pldp_dtype dtype;
    int B, R, q_heads;
    int64_t q_strides[2], k_strides[2], v_strides[2]; /* token, head */
    const void* q_norm;
    const void* k_norm;
    float eps;
    const float* cos;
    const float* sin;
    int rot, interleaved;
    int64_t rot_rows;
    const int32_t* rows;
    const int32_t* start;
    void* q_out;
    int64_t q_out_strides[2];
    uint32_t* status;
} pldp_cache_append_prompt_args;

PLDP_API pldp_status pldp_cache_append_prompt(const pldp_cache_append_prompt_args* args, void* stream);

/*
 * Causal attention of packed prompts over the cache (their own keys and values included:
 * append first).  The row of sequence b at position p, query head h, with kv head
 * h / (q_heads / cache.heads):
 *   s_j   = scale * q . k_j   for positions j = 0 .. p
 *   out   = sum_j exp(s_j - lse) v_j,   lse = ln sum_j exp(s_j)
 * so a prompt's prefix may be in the cache already (a shared one, or earlier chunks).
 *
 *  q          bf16 [R, q_heads, head_dim] with strides (token, head), 16-byte aligned,
 *             strides multiples of 16 bytes.
 *  q_heads    a multiple of cache.heads.
 *  scale      finite; 1/sqrt(head_dim) as a rule.
 *  out        bf16 [R, q_heads, head_dim] with strides, as q; it must not overlap q.
 *  lse        float [R, q_heads], contiguous, or NULL (pldp_rank_cache takes that of one
 *             sequence's rows, the last of them its row).
 *  workspace  pldp_attend_prompt_workspace_size bytes, 256-byte aligned; need not be cleared.
 *             Calls of any shapes may share one of the largest size; calls that may run
 *             concurrently need separate ones.
 *  status     uint32 [B] or NULL.  TIMEOUT: a wait inside the kernel ran out; the call's
 *             results are none.
 * Rows of a sequence with nothing to attend to (skipped, past the capacity, no page holds any
 * of their positions) are written as zeros, their lse as -INFINITY; of the others those whose
 * query holds NaN as NaN.  Of a sequence whose rows are not within [0, R] nothing is written.
 * Keys and values past a sequence's last row are never used, whatever they hold; those before
 * it must be finite, a bf16 cache's values below 2^32 in size and an e4m3 one's scales below
 * 2^124.  Sums and the running maximum are held in fp32.  On the way into the product with the
 * values each weight exp(s_j - lse) is rounded, over a bf16 cache to bf16 (by up to 2^-8 of it), over
 * an e4m3 one to f16, as are the values' scales and the values (each by up to 2^-11; small ones by
 * up to 2^-32 of the row's largest weight, and 2^-21 of the largest value that the row sees);
 * pldp_attend_cache, which takes such rows as one long draft, holds weights over a bf16 cache to 2^-17.
 * Results are the same for the same inputs, however the work is scheduled.
 */
typedef struct {
    pldp_cache cache;
    const void* q;
    int B, R, q_heads;
    int64_t q_strides[2];
    const int32_t* rows;
    const int32_t* start;
    float scale;
    void* out;
    int64_t out_strides[2];
    float* lse;
    uint32_t* status;
    void* workspace;
    size_t workspace_bytes;
} pldp_attend_prompt_args;

PLDP_API pldp_status pldp_attend_prompt(const pldp_attend_prompt_args* args, void* stream);

/* Bytes of workspace pldp_attend_prompt needs on the current device, whatever B and R (0 if invalid). */
PLDP_API size_t pldp_attend_prompt_workspace_size(int q_heads, int heads, int head_dim);

/* ---------------------------------------------------------------------------
 * The pages of a cache
 * ---------------------------------------------------------------------------
 * Verification moves seq_len on the device, so the pages of the next step are given out there too:
 * these calls keep a page table (one for all layers: page p is page p of each layer's pool) and
 * the number of its entries that hold each page.  Pages that several sequences hold (a common
 * prompt) are shared until one of them writes.
 *
 *  pages      int32 [B, pages_stride], max_pages entries a row: the table that pldp_cache
 *             reads.  An entry outside [0, n_pages) holds no page; the calls write -1.
 *  refs       int32 [n_pages]: the entries that hold each page, 0 for a free one.  Start
 *             with a table of -1 and refs of 0, or with both as they belong together; a caller that
 *             adds 1 to a page's keeps it from being given out or written.
 *  B          rows, 0..65535 (else PLDP_ERR_UNSUPPORTED).  max_pages * page_size < 2^31,
 *             n_pages <= 2^31 - 4096.
 * Whatever refs holds, no call writes outside these arrays; results are the ones described
 * where refs is as described.  Calls on one table follow one another (one stream, or ordered ones).
 */
typedef struct {
    int32_t* pages;
    int64_t pages_stride;
    int B, max_pages, page_size;
    int32_t* refs;
    int n_pages;
} pldp_page_table;

/* Bytes of workspace pldp_pages_reserve and pldp_pages_compact need for a table (0 if invalid);
 * 16-byte aligned, need not be cleared. */
PLDP_API size_t pldp_pages_workspace_size(int B, int max_pages, int n_pages);

/*
 * Makes positions start[b] .. start[b]+count[b]-1 of every sequence ones that may be written:
 * entries in that range that hold no page, or one that others hold too (refs above 1 before the
 * call), get free pages, the lowest ones, in order of sequence and position.
 * A sequence gets all of the pages that it needs or, where it and those before it need more than
 * there are, none: CAPACITY, its entries stay as they are and it must not be written.
 *
 *  start      int32 [B] (kv_keep_len of a step: x_t's position).
 *  count      int32 [B], or NULL for n (K+1).  0: nothing to do.
 *  n          the largest count, >= 0.  A negative start, or a count outside [0, n]: SEQ_LEN, nothing done.
 *             A range that passes max_pages * page_size: CAPACITY, nothing done.
 *  copies     int32 [B, 2] out: the page that pldp_cache_copy_pages has to copy, and where to
 *             (the one in which start lies, if it was shared and start is not its first
 *             position), or -1, -1.
 *  status     uint32 [B] or NULL.
 */
PLDP_API pldp_status pldp_pages_reserve(const pldp_page_table* table, const int32_t* start, const int32_t* count, int n,
                                        int32_t* copies, uint32_t* status, void* workspace, size_t workspace_bytes,
                                        void* stream);

/*
 * Row b becomes the first entries of row parent[b], those that hold its positions 0..len[b]-1,
 * which both hold from then on; what row b held before is given back.
 *
 *  parent     int32 [B]; -1 or b itself: row b stays as it is.  Outside [-1, B), or a row
 *             that has another row as its parent itself: ROW_INDEX, row b stays as it is.
 *  len        int32 [B]; negative or past max_pages * page_size: SEQ_LEN, row b stays as it is.
 *  status     uint32 [B] or NULL.
 */
PLDP_API pldp_status pldp_pages_fork(const pldp_page_table* table, const int32_t* parent, const int32_t* len,
                                     uint32_t* status, void* stream);

/*
 * Gives back the entries past those that hold positions 0..keep_len[b]-1 (0: all of a sequence that
 * has ended); a negative keep_len[b] leaves row b as it is.
 */
PLDP_API pldp_status pldp_pages_free(const pldp_page_table* table, const int32_t* keep_len, void* stream);

/*
 * Moves the held pages to the front of the pool: the highest one to the lowest free one, and so
 * on, until the held ones are 0..U-1.  The table and refs are changed here, the contents follow with
 * pldp_cache_copy_pages (in every layer) before the next use.
 *
 *  copies     int32 [copies_cap, 2] out, copies_cap >= n_pages / 2: from, to.
 *  n_copies   int32 [1] out.
 *  used       int32 [1] out, or NULL: U.
 */
PLDP_API pldp_status pldp_pages_compact(const pldp_page_table* table, int32_t* copies, int copies_cap, int32_t* n_copies,
                                        int32_t* used, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Copies whole pages of one layer's keys and values (and scales): copies[i][0] to copies[i][1].
 *
 *  copies     int32 [n, 2]; a pair with an entry outside [0, n_pages), or with twice the same, is skipped.
 *  n_copies   int32 [1], or NULL for n: pairs 0..min(n, n_copies)-1.
 * No page may be written by one pair and read or written by another (in the lists of the calls above
 * none is): its contents are then those of any of them.
 */
PLDP_API pldp_status pldp_cache_copy_pages(const pldp_cache* cache, const int32_t* copies, int n, const int32_t* n_copies,
                                           void* stream);

/* Message describing the last failed call on this host thread ("" if none). */
PLDP_API const char* pldp_last_error(void);

/* Library version (major * 10000 + minor * 100 + patch). */
PLDP_API int pldp_version(void);

#ifdef __cplusplus
}
#endif

#endif /* PLDP_H */
