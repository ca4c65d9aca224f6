/*
 * ngc.h -- C ABI of the B200 (sm_100a) hot path of Neural Garbage Collection:
 * batched rollout decoding over a KV cache that the policy itself prunes.
 *
 * One eviction round is   ngc_score_evict -> ngc_sample_evict -> ngc_evict_logprob
 * -> ngc_compact_kv,   after which generation continues with
 * ngc_decode_attn_ragged over the surviving entries (paper Section 4.1: the
 * cache grows during generation and is pruned at each round).
 *
 * Conventions
 * -----------
 * - Plain C.  Host-side state: the last CUDA error code (per thread) and one
 *   flag per device recording that a kernel family has been configured there
 *   (the first call of a kernel family on each device sets its shared-memory
 *   limit, which CUDA stores per device; make that first call outside any
 *   stream capture).  Device-side state: none, except the built-in scratch
 *   array of ngc_decode_attn_ragged_static (see there).
 * - Every data pointer is a DEVICE pointer owned by the caller unless the
 *   comment says "host".  The library never allocates, frees or synchronises;
 *   scratch comes from a caller-supplied workspace sized by
 *   ngc_workspace_bytes() (ngc_decode_attn_ragged_static alone uses its own
 *   array instead).  Every call only enqueues work on `stream` (a
 *   cudaStream_t, which must belong to the current device) and returns.
 * - Return value: NGC_OK or a negative ngc_status.  Invalid host-visible
 *   arguments are refused before anything is launched.  Problems only visible
 *   on the device (a budget larger than the list, a NaN logit, a corrupt kept
 *   list, a full strip) are written to *dev_status (int32 in device memory,
 *   first error wins, 0 = none; may be NULL) and the offending list / strip /
 *   sequence is skipped.  Kernels never trap and every wait inside them is
 *   bounded.
 * - "Lists": a sequence has G eviction lists; G = 1 (one decision shared by all
 *   layers and heads), L (one per layer, the paper's setting: Section 4.1 has
 *   every layer evict an equal share of its entries but choose them on its
 *   own), or L*Hkv (one per layer and KV head).  List gi of sequence b is
 *   row b*G + gi of every [B][G][...] array.
 * - "Units": eviction acts on units of `block` consecutive tokens (Section 4.2,
 *   block-level evictions); the last unit of a sequence may be short.
 *
 * Cache layout
 * ------------
 *   k, v    : [L][Hkv][R][d] elements; R rows per (layer, KV head) plane.
 *   seq_off : int64 [B+1]; sequence b owns rows seq_off[b] .. seq_off[b+1] of
 *             every plane (its capacity); seq_off[0] = 0, seq_off[B] = R.
 *   lens    : int32 [B]; the first lens[b] rows of a strip are alive.  With
 *             lens_lists != 0 the cache holds one length per (sequence, list) instead:
 *             int32 [B][G] for that ngc_lists mode, and the strips of list gi of
 *             sequence b have lens[b*G + gi] alive rows.  The paper evicts per layer
 *             in units of several tokens, and a short last unit that one layer keeps
 *             and another evicts leaves the layers with different lengths.
 * A (layer, head, sequence) strip is therefore T x d contiguous rows, which
 * decode streams linearly and compaction moves row by row.  Rows at or beyond
 * lens[b] hold unspecified bytes.
 */
#ifndef NGC_H_
#define NGC_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct CUstream_st* ngc_stream;   /* == cudaStream_t */

typedef enum {
  NGC_OK = 0,
  NGC_ERR_INVALID_ARG = -1,   /* null pointer, negative size, inconsistent shape */
  NGC_ERR_UNSUPPORTED = -2,   /* shape / dtype combination not built */
  NGC_ERR_WORKSPACE = -3,     /* workspace missing or smaller than ngc_workspace_bytes() */
  NGC_ERR_CUDA = -4,          /* a CUDA call failed; code in ngc_last_cuda_error() */
  NGC_ERR_STATIC_SCRATCH = -5 /* launch needs more scratch than the built-in static array holds */
} ngc_status;

/* values written to *dev_status */
typedef enum {
  NGC_DEV_OK = 0,
  NGC_DEV_BAD_COUNTS = 1,     /* not 0 <= n_protect <= budget <= n <= n_max, or budget > k_max */
  NGC_DEV_NAN_LOGIT = 2,      /* a candidate logit is NaN */
  NGC_DEV_BAD_KEPT = 3,       /* kept list out of range, repeated or not ascending */
  NGC_DEV_STRIP_FULL = 4,     /* append would exceed the sequence's row capacity */
  NGC_DEV_LISTS_DISAGREE = 5, /* lists of one sequence keep different token counts */
  NGC_DEV_TIMEOUT = 6,        /* a bounded wait inside a kernel ran out */
  NGC_DEV_DEBUG_BOUNDS = 7,   /* bounds-checking build only: a kernel computed an index outside its array */
  NGC_DEV_BAD_TREE = 8,       /* a node count, parent link, drafted token or accepted path that is none */
  NGC_DEV_BAD_PROBS = 9,      /* numbers that are no probabilities, or have no finite positive sum */
  NGC_DEV_BAD_SOURCE = 10,    /* a fork's source is no sequence, or is itself a destination */
  NGC_DEV_BAD_PAGE = 11,      /* a page-table entry outside 0 .. pages_cap-1 (of a pool: 0 .. n_pages-1) */
  NGC_DEV_POOL_FULL = 12,     /* a pool has fewer free pages than a sequence needs */
  NGC_DEV_BAD_SLOT = 13       /* a slot outside the pool */
} ngc_dev_status;

typedef enum { NGC_F32 = 0, NGC_BF16 = 1 } ngc_dtype;
typedef enum { NGC_LISTS_SHARED = 0, NGC_LISTS_PER_LAYER = 1, NGC_LISTS_PER_LAYER_KVHEAD = 2 } ngc_lists;
typedef enum { NGC_OP_SCORE = 0, NGC_OP_SAMPLE = 1, NGC_OP_LOGPROB = 2, NGC_OP_COMPACT = 3, NGC_OP_DECODE = 4,
               NGC_OP_SCORE_BACKWARD = 5, NGC_OP_TREE_ATTN = 6 } ngc_op;

/* Describes the cache; owns nothing.  `rows` and `max_len` are host copies the
 * launch geometry needs: rows = seq_off[B]; max_len >= every length at the
 * time of the call (a loose bound such as the largest capacity is fine; it
 * only sizes grids and workspaces). */
typedef struct {
  void* k;
  void* v;
  const int64_t* seq_off;
  int32_t* lens;
  int64_t rows;
  int32_t L, B, Hq, Hkv, d;   /* Hq % Hkv == 0; d in {64, 128} */
  int32_t dtype;              /* ngc_dtype of k, v, queries and new rows */
  int32_t max_len;
  int32_t lens_lists;         /* 0: lens[B]; NGC_LISTS_PER_LAYER / _KVHEAD: lens[B][G] of that mode.  Calls that
                                 take an eviction `lists` mode need lens_lists == 0 or == lists. */
} ngc_cache;

/* Library version (major*10000 + minor*100 + patch). */
int ngc_version(void);
/* Text for an ngc_status (host string, never NULL). */
const char* ngc_strerror(int status);
/* cudaError_t of the most recent NGC_ERR_CUDA on this host thread (0 = none). */
int ngc_last_cuda_error(void);

/* Bytes of workspace `op` needs for this cache / list shape (0 = none).  For
 * NGC_OP_SAMPLE and NGC_OP_LOGPROB only c->B (sequences, times rounds for the
 * log-prob) is read from the cache descriptor; pass G, n_max, k_max as in the
 * call (NGC_OP_TREE_ATTN: n_max = nodes per tree; for a paged cache pass a
 * contiguous descriptor with rows = B * pages_cap * page and max_len =
 * pages_cap * page).  The workspace must be 256-byte aligned; its contents need not be
 * preserved between calls, and calls sharing a workspace must be stream-ordered. */
size_t ngc_workspace_bytes(int op, const ngc_cache* c, int G, int n_max, int k_max);

/* Number of token-range splits ngc_decode_attn_ragged uses for a call over
 * `layers` layers of this cache (1 = every strip is handled by one CTA and no
 * combine kernel runs).  Host-only planning query. */
int ngc_decode_splits(const ngc_cache* c, int layers);

/*
 * Eviction scores -- Section 4.2 ("Parameterizing eviction actions" and
 * "Coarsening the action space").  For every list: psi_t = mean, over the
 * query heads feeding the list and the w most recent queries, of the softmax
 * attention weight (scale 1/sqrt(d)) that query puts on alive key t; then
 * s_j = mean of psi over the tokens of unit j.
 *   q_recent [L][B][Hq][w][d], cache dtype.  Window query j sits at absolute
 *            position lens[b]-w+j and sees keys at positions <= its own; when
 *            lens[b] < w only the last lens[b] queries are used.
 *   lists    which heads are averaged: SHARED = all layers and heads,
 *            PER_LAYER = the Hq heads of the layer (the paper), PER_LAYER_KVHEAD
 *            = the Hq/Hkv heads of one KV group.
 *   logits   [B][G][n_max] fp32 out.  With one length per sequence, units >=
 *            ceil(lens[b]/block) are untouched.  With a length per list
 *            (lens_lists == lists) the sequence is scored on the units of its
 *            LONGEST list, n_b = max over its lists of ceil(len/block): a shorter
 *            list gets -inf in the units it lacks (never drawn by
 *            ngc_sample_evict, no mass in Eq. (1)); units >= n_b are untouched.
 *   n_units_out  int32 [B] out, may be NULL: n_b, the unit count per sequence to
 *            pass to ngc_sample_evict / ngc_evict_logprob as `n` (for one length
 *            per sequence simply ceil(lens[b]/block)).
 *   log_transform  0: logit = s_j (the paper's literal reading); 1: logit = log s_j.
 * Requires n_max >= ceil(max_len/block).  Reads K only.
 */
int ngc_score_evict(const ngc_cache* c, const void* q_recent, int w, int block, int lists,
                    int log_transform, float* logits, int n_max, int32_t* n_units_out,
                    void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/* Number of kernels one ngc_score_evict call enqueues for this cache and window (host-only planning query, for
 * launch counting). */
int ngc_score_evict_launches(const ngc_cache* c, int w);

/*
 * Gradient of the eviction scores with respect to the recent queries and the
 * keys -- Sections 4.4 and 4.5: the eviction loss reaches the model through
 * the scores, which the replay pass recomputes with gradients enabled.  The chain
 * rule through the block mean, the average over attention rows and the
 * softmax of ngc_score_evict:
 *   grad_logits   [B][G][n_max] fp32 upstream gradient (e.g. from ngc_evict_logprob_backward)
 *   logits        the forward output; read only when log_transform != 0 (else may be NULL)
 *   grad_q_recent [L][B][Hq][w][d] fp32 out (zero for window queries before the sequence start)
 *   grad_k        [L][Hkv][R][d] out, cache dtype; rows >= lens[b] are not written
 * Other arguments as in ngc_score_evict.  Built for bf16 caches with d = 128 and at most 40
 * (head, query) rows per KV head (Hq/Hkv * w <= 40); NGC_ERR_UNSUPPORTED otherwise.  K is read
 * twice and grad_k written once.  Workspace: ngc_workspace_bytes(NGC_OP_SCORE_BACKWARD, ...).
 */
int ngc_score_evict_backward(const ngc_cache* c, const void* q_recent, int w, int block, int lists, int log_transform,
                             const float* logits, const float* grad_logits, int n_max,
                             float* grad_q_recent, void* grad_k,
                             void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Sampling the keep set -- Section 4.3 (Gumbel-top-k): perturbed key =
 * logit + Gumbel noise; keep the budget largest.  The n_protect[b] leading
 * units are always kept and take no part in the draw; budget[b] counts them.
 * Noise: Philox4x32-10 with key = seed and counter = (i >> 2, list_base + b*G
 * + gi, round low, round high); unit i takes output word i & 3; the word
 * becomes an odd multiple of 2^-24 in (0,1) and then a Gumbel variate through a
 * fixed sequence of correctly rounded fp32 operations, so that the draw does
 * not depend on launch geometry, on the batch sharding or on the machine.
 * Ties (equal fp32 keys): smaller index first.  greedy != 0 drops the noise
 * (Section 5.1, evaluation uses deterministic top-k).
 *   logits      [B][G][n_max] fp32
 *   n, n_protect (may be NULL = 0), budget : int32 [B]
 *   kept_order  [B][G][k_max] out: the budget-n_protect drawn units, largest key
 *               first (the sequence sigma of Eq. (1)); -1 padded
 *   kept_sorted [B][G][k_max] out: all kept units ascending; -1 padded
 *   keep_mask   [B][G][n_max] out, 1 = kept (may be NULL)
 * A list with bad counts or a NaN candidate logit is reported in *dev_status
 * and gets all -1 / 0 outputs.
 */
int ngc_sample_evict(const float* logits, const int32_t* n, const int32_t* n_protect,
                     const int32_t* budget, int B, int G, int n_max, int k_max,
                     uint64_t seed, uint64_t round, uint32_t list_base, int greedy,
                     int32_t* kept_order, int32_t* kept_sorted, uint8_t* keep_mask,
                     void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Log-probability of the drawn sequence -- Eq. (1) of Section 4.3:
 *   log p(sigma | s) = sum_j [ s_sigma_j - log sum_{t not in sigma_1..sigma_{j-1}} exp s_t ],
 * over the non-protected units of each list, evaluated with the running
 * remaining-mass scan the paper mentions right after the equation, in fp64.
 * Rounds can be flattened into the leading dimension (the policy-gradient
 * recompute of Section 4.4 evaluates all rounds of a rollout at once).
 *   logits [n_batches][B][G][n_max] fp32; n, n_protect (NULL = 0), budget
 *   int32 [n_batches][B]; kept_order [n_batches][B][G][k_max];
 *   logp [n_batches][B][G] fp64 out (NaN for a list reported in *dev_status).
 */
int ngc_evict_logprob(const float* logits, const int32_t* n, const int32_t* n_protect,
                      const int32_t* budget, const int32_t* kept_order,
                      int n_batches, int B, int G, int n_max, int k_max, double* logp,
                      void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Gradient of that log-probability with respect to the logits -- what the
 * eviction half of the policy-gradient loss (Section 4.4, L_mem: the sum over
 * layers and rounds of -log pi(sigma) * advantage) sends back into the scores:
 *   d log p / d s_i = [i in sigma] - exp(s_i) * sum_{j : i not drawn before step j} 1 / rem_j ,
 * rem_j = the mass still present at step j (the same scan as the forward call).
 *   grad_logp   fp64 [n_batches][B][G] upstream gradient per list, or NULL (= 1)
 *   grad_logits fp32 [n_batches][B][G][n_max] out; every entry of a list is
 *               written: 0 for protected units and units >= n[b], NaN for a
 *               list reported in *dev_status.
 * Other arguments as in ngc_evict_logprob.  Lists with more than about 24 K
 * drawn units are refused with NGC_ERR_UNSUPPORTED.
 */
int ngc_evict_logprob_backward(const float* logits, const int32_t* n, const int32_t* n_protect,
                               const int32_t* budget, const int32_t* kept_order, const double* grad_logp,
                               int n_batches, int B, int G, int n_max, int k_max, float* grad_logits,
                               void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Replay visibility -- Appendix A.3 ("Reconstructing Replay Attention Masks
 * from Retention Decisions") and the replay-mask figure of Section 4.5.  The
 * training pass must show every token exactly the keys it saw at rollout time:
 * a query generated after round r sees kept_r (what round r left alive) plus,
 * causally, the tokens generated since.  This call turns the stored decisions
 * of all R rounds -- kept units in the coordinates of the cache at that round
 * -- into kept_r as ORIGINAL token positions, one ascending list per (round,
 * list), instead of the paper's dense B x T x T masks.
 *   kept_sorted  [R][B][G][k_max] as written by ngc_sample_evict at round r
 *   budget       [R][B] kept units;  alive_before [R][B] tokens alive when round
 *                r fired (lens[b] at that time), or [R][B][G] with per_list != 0 (caches
 *                with a length per list);  total_before [R][B] sequence
 *                length when round r fired (the tokens appended since the last
 *                round are the positions just below it)
 *   block        tokens per unit;  alive_max (host) >= every alive_before
 *   alive_pos    [R][B][G][k_max*block] out, ascending, -1 padded
 *   alive_count  [R][B][G] out (tokens), -1 for a list that failed
 * A list with inconsistent counts or a corrupt kept list is reported in
 * *dev_status and gets -1 from the failing round on.
 */
int ngc_replay_visibility(const int32_t* kept_sorted, const int32_t* budget, const int32_t* alive_before,
                          const int32_t* total_before, int R, int B, int G, int k_max, int block, int alive_max,
                          int per_list, int32_t* alive_pos, int32_t* alive_count, int32_t* dev_status, ngc_stream stream);

/*
 * Replay attention -- Section 4.5: one pass over ALL tokens of a rollout in
 * which every query sees exactly the keys it saw when it was generated, so
 * that token and eviction log-probabilities are recomputed on-policy.  The
 * masks of Appendix A.3 are not materialised: the query at position t attends
 * to kept_r (alive_pos of the last round that fired at or before t, from
 * ngc_replay_visibility) and, causally, to the tokens from that round's
 * boundary up to t itself; queries before the first round are plain causal.
 *   c            the FULL sequences: k, v [L][Hkv][R][d] hold every token in original
 *                order, lens[b] = T_b tokens (bf16, d = 128)
 *   q            [L][B][Hq][t_max][d] bf16; rows >= lens[b] are ignored
 *   alive_pos    [n_rounds][B][G][kt_max], alive_count [n_rounds][B][G], total_before
 *                [n_rounds][B] (ascending per sequence); n_rounds = 0: causal attention
 *   lists        how G maps to (layer, KV head), as everywhere
 *   out          [L][B][Hq][t_max][d] fp32 or bf16; rows >= lens[b] are not written
 * fp32 scores, softmax and accumulation; probabilities rounded to bf16 for P*V.
 * Needs no workspace.  Runs on the tcgen05 tensor cores with accumulators in
 * tensor memory; every wait inside is bounded (NGC_DEV_TIMEOUT).
 */
int ngc_replay_attn(const ngc_cache* c, const void* q, int t_max,
                    const int32_t* alive_pos, const int32_t* alive_count, const int32_t* total_before,
                    int n_rounds, int kt_max, int lists, float scale, void* out, int out_dtype,
                    int32_t* dev_status, ngc_stream stream);

/* ngc_replay_attn with the device path chosen by the caller (same arguments, same contract; for
 * measuring one path against the other).  AUTO is what ngc_replay_attn runs: the tcgen05 kernel
 * (S and O accumulators in tensor memory, one CTA per 128 query tokens of two heads).  MMA_SYNC is
 * the earlier warp-level kernel (64 query tokens of one head per CTA). */
typedef enum { NGC_REPLAY_ATTN_AUTO = 0, NGC_REPLAY_ATTN_MMA_SYNC = 1, NGC_REPLAY_ATTN_TCGEN05 = 2 } ngc_replay_attn_path;
int ngc_replay_attn_variant(const ngc_cache* c, const void* q, int t_max,
                            const int32_t* alive_pos, const int32_t* alive_count, const int32_t* total_before,
                            int n_rounds, int kt_max, int lists, float scale, void* out, int out_dtype, int variant,
                            int32_t* dev_status, ngc_stream stream);

/*
 * Physical eviction -- Section 4.1 (entries that are not kept are gone for good).  In place:
 * in every (layer, KV head, sequence) strip of K and V the tokens of the kept
 * units move to the front in ascending original order, and lens[b] becomes
 * the number of kept tokens.  Bit-exact row moves; rows beyond the new length
 * are unspecified afterwards.
 *   kept_sorted [B][G][k_max] ascending unit indices (as written by
 *   ngc_sample_evict); budget int32 [B]; lists says how G maps to (layer, head).
 * Errors leave whole sequences alone: with one length per sequence (lens_lists
 * == 0), a sequence that has a corrupt list (NGC_DEV_BAD_KEPT), or whose lists
 * would keep different token counts (NGC_DEV_LISTS_DISAGREE: units of several
 * tokens with a short last unit that some lists keep and others evict), is
 * reported and none of its strips moves; its lens[b] and every row are as
 * before the call.  With a length per list (lens_lists == lists) the lists are
 * independent: a corrupt list leaves its own strips and length untouched.
 * (While the call runs, lens[b] of such a sequence briefly holds a negative
 * marker; it is restored before the call's last kernel ends.)
 */
int ngc_compact_kv(ngc_cache* c, const int32_t* kept_sorted, const int32_t* budget, int k_max,
                   int lists, int block, int32_t* dev_status, ngc_stream stream);

/*
 * Decode attention over the surviving entries -- Section 4.1 (after a round,
 * generation goes on with only what was kept).  For layers
 * [layer_begin, layer_end): if new_k/new_v are given, the new token's K/V row
 * is first written at position lens[b] of each strip and is visible to its
 * own query; then out = softmax(scale * q K^T) V over the alive rows, one
 * pass, split along tokens.  lens[b] is incremented (once) by the call whose
 * layer_end == L when new rows were given.
 *   q      [L][B][Hq][d] cache dtype; new_k, new_v [L][B][Hkv][d] cache dtype or both NULL
 *   out    [L][B][Hq][d] of out_dtype (NGC_F32, or NGC_BF16 for a bf16 cache);
 *          only the layers of the range are written; an empty strip gives zeros.
 * bf16 caches: fp32 scores, softmax and accumulation; the probabilities are
 * rounded to bf16 for the P*V product.
 */
int ngc_decode_attn_ragged(ngc_cache* c, const void* q, const void* new_k, const void* new_v,
                           int layer_begin, int layer_end, float scale,
                           void* out, int out_dtype,
                           void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Paged variant -- Section 4.2 remarks that evicting whole blocks fits paged
 * KV caches: with one eviction unit = one page, evicting is
 * an edit of a page table and no K/V row moves.
 *
 *   k, v       : [L][Hkv][B * pages_cap][page][d] elements (bf16, d = 128)
 *   page_table : int32 [B][G][pages_cap]; the j-th page of tokens of list gi of
 *                sequence b lives in physical page  b * pages_cap + page_table[b][gi][j]
 *                of every (layer, KV head) plane the list covers.  Each row of the
 *                table is a permutation of 0 .. pages_cap-1: entries at and beyond
 *                ceil(lens[b] / page) name the sequence's free pages.
 *   lens       : int32 [B] alive tokens (same for every list of b), or int32 [B][G] with
 *                lens_per_list != 0 (a partly filled last page that one list keeps and
 *                another evicts leaves them with different lengths)
 *   lists      : ngc_lists, fixes G and which planes a list covers
 *   page       : tokens per page, 32 or 64
 */
typedef struct {
  void* k;
  void* v;
  int32_t* page_table;
  int32_t* lens;
  int32_t L, B, Hq, Hkv, d;
  int32_t dtype;
  int32_t page, pages_cap, lists;
  int32_t lens_per_list;
} ngc_paged_cache;

/*
 * ngc_score_evict over a paged cache: units are pages (block = page), the
 * lists are the cache's own (c->lists); K is read page by page through the
 * table.  logits [B][G][n_max], n_max >= pages_cap; n_units_out as in
 * ngc_score_evict (may be NULL).  Workspace as for
 * NGC_OP_SCORE of a contiguous cache with rows = B * pages_cap * page and
 * max_len = pages_cap * page.
 */
int ngc_score_evict_paged(const ngc_paged_cache* c, const void* q_recent, int w, int log_transform,
                          float* logits, int n_max, int32_t* n_units_out, void* ws, size_t ws_bytes,
                          int32_t* dev_status, ngc_stream stream);

/*
 * Eviction on a paged cache: for every list the pages named by kept_sorted
 * (ascending unit = page indices, as written by ngc_sample_evict) move to the
 * front of the list's page-table row in that order, the other pages follow as
 * free pages, and lens[b] becomes the number of kept tokens (a partly filled
 * last page stays last if it is kept).  No K/V row is touched.  A corrupt list
 * leaves its row and lens[b] unchanged and is reported in *dev_status.
 */
int ngc_evict_pages(ngc_paged_cache* c, const int32_t* kept_sorted, const int32_t* budget, int k_max,
                    int32_t* dev_status, ngc_stream stream);

/*
 * ngc_decode_attn_ragged over a paged cache: same arguments, results and
 * append semantics; the token tiles are fetched page by page through the
 * table.  The appended row goes to position lens[b] of the list's pages (a
 * sequence is full at pages_cap * page tokens).  Workspace as for
 * NGC_OP_DECODE of a cache with the same L, B, Hq, Hkv.
 */
int ngc_decode_attn_paged(ngc_paged_cache* c, const void* q, const void* new_k, const void* new_v,
                          int layer_begin, int layer_end, float scale,
                          void* out, int out_dtype,
                          void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * ngc_decode_attn_ragged without a caller-supplied workspace.  (The paper has
 * no counterpart: this entry exists for the library's users, not the method.)
 *
 * Some callers cannot hand the library device scratch memory: code embedded
 * in a host application that has already given every byte of device memory
 * to its own pool, plug-ins that are not allowed to call the CUDA allocator,
 * and latency-critical serving loops where a cudaMalloc (which synchronises
 * the whole device) must never happen.  For them the split partials of the
 * decode kernel live in a scratch array built into the library image
 * (NGC_STATIC_SCRATCH_BYTES of device memory, resident on every GPU that
 * loads the library until the process exits).  The call allocates nothing,
 * frees nothing and calls no allocating routine.
 *
 * Same arguments and results as ngc_decode_attn_ragged, minus ws/ws_bytes.
 * - A launch whose scratch need exceeds NGC_STATIC_SCRATCH_BYTES is refused
 *   with NGC_ERR_STATIC_SCRATCH before anything is enqueued (use the
 *   workspace variant, or narrow the layer range).
 * - The first call on each device looks up the device address of the array
 *   (a one-off host-side set-up on the current device, serialised by a
 *   mutex); make that first call before starting any stream capture.
 * - The array used is the CURRENT device's; a `stream` that belongs to another
 *   device is refused with NGC_ERR_INVALID_ARG.
 * - All calls on a device share the one array, which keeps whatever the last
 *   call left in it.  Nothing in it needs to start at zero (every slot is
 *   written before it is read within a call), but two calls that overlap on
 *   the GPU (different streams without an ordering between them) race on it:
 *   keep calls to this entry stream-ordered.
 */
#define NGC_STATIC_SCRATCH_BYTES (8u << 20)
int ngc_decode_attn_ragged_static(ngc_cache* c, const void* q, const void* new_k, const void* new_v,
                                  int layer_begin, int layer_end, float scale,
                                  void* out, int out_dtype, int32_t* dev_status, ngc_stream stream);

/*
 * Drafted tokens.  (The paper decodes one token per pass; these calls let a
 * rollout advance by several, and let the rollouts of one prompt -- Section 5.1
 * samples a group per prompt -- share its prefill.)  A draft is a TREE of up to
 * NGC_TREE_MAX_NODES tokens per sequence: node 0 is the pending token (the
 * last one sampled, whose K/V is not in the cache yet), every other node
 * continues its parent.  One step is
 *   ngc_tree_attn (per layer or for all) -> the model's output probabilities
 *   -> ngc_verify_draft -> ngc_commit_draft.
 * Nothing of the draft is in the cache before the commit, so there is nothing
 * to roll back.  Arguments shared by the calls:
 *   parent  [B][N] int32: parent[b][0] = -1, 0 <= parent[b][i] < i for i >= 1
 *   n_nodes [B] int32 or NULL (= N): nodes of each tree, 0 .. N; the others'
 *           entries are ignored wherever they appear
 * A sequence with a bad count or link is reported as NGC_DEV_BAD_TREE and
 * skipped.
 */
#define NGC_TREE_MAX_NODES 128

/*
 * Attention for a tree of drafted tokens over a cache: node i attends to every
 * alive cache row of its strip, to its ancestors and to itself,
 *   out_i = softmax_j(scale * q_i . k_j) V,  j over alive rows and ancestors-or-self.
 * For layers [layer_begin, layer_end); reads lens and the cache, changes neither.
 *   q       [L][B][Hq][N][d] cache dtype;  tree_k, tree_v [L][B][Hkv][N][d] cache dtype
 *   N       1 .. NGC_TREE_MAX_NODES (N = 1: the one-token decode without append)
 *   scale   positive, at most 2e38
 *   out     [L][B][Hq][N][d] of out_dtype (NGC_F32, or NGC_BF16 for a bf16
 *           cache); only the layers of the range and the nodes of each tree
 *           are written
 * Masked and dead rows take no part whatever they hold (infinities, NaN); a
 * row that sees a NaN or an infinite score is NaN, and so may be one with scores
 * of 2^30 and more.  fp32 scores, softmax and accumulation; on bf16 caches the
 * probabilities are rounded to bf16 for the P*V product.  Results are the same
 * in every run; where one lies in its last bits may depend on the lengths of
 * the call's other sequences (they decide how the work is cut).  A length
 * outside 0 .. capacity is reported (NGC_DEV_BAD_COUNTS) and the sequence
 * skipped.  A bf16 call is refused (NGC_ERR_UNSUPPORTED) if its layers, KV heads
 * and sequences make some 190 million strips or more.  The workspace is free
 * again when the call has run: calls that may run at the same time (other
 * streams, graphs) need one each.  q, tree_k, tree_v, out, k and v must be 16-byte
 * aligned.  Workspace: ngc_workspace_bytes(NGC_OP_TREE_ATTN, c, 1, N, 0), which
 * also serves calls that give a smaller max_len.
 */
int ngc_tree_attn(const ngc_cache* c, const void* q, const void* tree_k, const void* tree_v, const int32_t* parent,
                  const int32_t* n_nodes, int N, int layer_begin, int layer_end, float scale, void* out, int out_dtype,
                  void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/* Number of kernels one ngc_tree_attn call over `layers` layers of this cache enqueues (host-only planning query; 0: none, the
 * call would be refused). */
int ngc_tree_attn_launches(const ngc_cache* c, int layers, int N);

/* ngc_tree_attn over a paged cache.  A page-table entry outside 0 .. pages_cap-1 is reported as
 * NGC_DEV_BAD_PAGE; the outputs of that sequence are then unspecified. */
int ngc_tree_attn_paged(const ngc_paged_cache* c, const void* q, const void* tree_k, const void* tree_v, const int32_t* parent,
                        const int32_t* n_nodes, int N, int layer_begin, int layer_end, float scale, void* out, int out_dtype,
                        void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Verification of a drafted tree against the target's probabilities from given
 * random numbers (multi-round speculative sampling: the token sequence that
 * comes out is distributed as if sampled from the target).  The walk starts
 * at node 0 and tries the children of the current node in index order; at a
 * node with target row p and draft row q, starting from w = max(p, 0) and S = 1,
 * child i with token x = tokens[b][i] and u = uniforms[b][i]:
 *   draft_probs given (children drawn independently from q):
 *     accepted iff u * q(x) * S < w(x);  else w <- max(w - S q, 0), S <- sum w
 *   draft_probs NULL (children picked without chance, e.g. the likeliest tokens):
 *     accepted iff u * S < w(x);         else S <- S - w(x), w(x) <- 0
 *   greedy != 0 (uniforms and draft_probs unused): accepted iff x is the
 *     argmax of p (smallest index of equal ones)
 * (a rejection that would leave no mass leaves w and S as they were).  An
 * accepted child becomes the current node.  When no child is left the next
 * token is drawn from what remains: the first x whose running sum of w exceeds
 * uniforms[b][0] * sum w -- or the argmax, if greedy.
 *   tokens       [B][N] int32 in 0 .. vocab-1 (entry 0 unused)
 *   target_probs [B][N][vocab] fp32: row i follows node i.  Rows are taken as
 *                normalised; whole rows are read only where the walk comes.
 *                vocab <= 2^30
 *   draft_probs  [B][N][vocab] fp32 or NULL: row i is what node i's children were drawn from; no
 *                negative numbers (looked at for tested children only)
 *   uniforms     [B][N] fp32 in [0, 1) (may be NULL if greedy)
 *   path         [B][N] out: accepted nodes from node 0 on, -1 padded (ascending)
 *   n_path       [B] out: their number (>= 1; 0 for an empty tree)
 *   next_token   [B] out: the token that follows the path (-1 for an empty tree)
 * Decisions and sums in fp64: the outcome does not depend on launch geometry
 * beyond the last bits of an fp64 sum.  A bad tree or token (NGC_DEV_BAD_TREE)
 * or numbers that are no probabilities (NGC_DEV_BAD_PROBS) give path -1,
 * n_path 0, next_token -1.  The latter are looked for where the walk reads: a
 * tested child's p(x) or q(x) that is negative, infinite or NaN; a node where a
 * child drawn from q is rejected, if what is left has no finite sum; the last
 * node, if what is left has no finite positive sum; greedy: a NaN in any row that
 * the walk visits.
 */
int ngc_verify_draft(const int32_t* tokens, const int32_t* parent, const int32_t* n_nodes, const float* target_probs,
                     const float* draft_probs, const float* uniforms, int B, int N, int vocab, int greedy,
                     int32_t* path, int32_t* n_path, int32_t* next_token, int32_t* dev_status, ngc_stream stream);

/*
 * Appends the K/V rows of the accepted nodes: row path[b][j] of tree_k / tree_v
 * goes to position len + j of every strip, for j < n_path[b], and the lengths
 * grow by n_path[b].  Bit-exact row copies.
 *   tree_k, tree_v [L][B][Hkv][N][d] as given to ngc_tree_attn, 16-byte aligned
 *   path [B][N], n_path [B] as written by ngc_verify_draft
 * A path that is not ascending within 0 .. N-1 (NGC_DEV_BAD_TREE) or does not
 * fit the sequence's capacity in some list (NGC_DEV_STRIP_FULL) leaves the
 * sequence as it was.
 */
int ngc_commit_draft(ngc_cache* c, const void* tree_k, const void* tree_v, const int32_t* path, const int32_t* n_path,
                     int N, int32_t* dev_status, ngc_stream stream);

/* ngc_commit_draft on a paged cache: the rows go to the pages that positions len + j fall into.  A bad
 * page-table entry among them (NGC_DEV_BAD_PAGE) leaves the sequence as it was. */
int ngc_commit_draft_paged(ngc_paged_cache* c, const void* tree_k, const void* tree_v, const int32_t* path,
                           const int32_t* n_path, int N, int32_t* dev_status, ngc_stream stream);

/*
 * Forks sequences: sequence b becomes a copy of sequence src_of[b] (its alive
 * rows in every strip and its lengths; rows beyond them stay as they were).
 *   src_of [B] int32: -1 or b itself = sequence b is left alone.  A source must
 *          be left alone itself; otherwise, or with a source outside 0 .. B-1,
 *          b is reported (NGC_DEV_BAD_SOURCE) and left as it was, as is a b too
 *          small for its source in some list (NGC_DEV_STRIP_FULL) or one whose
 *          source has a length outside its capacity (NGC_DEV_BAD_COUNTS).
 *          B <= 65536
 */
int ngc_fork_kv(ngc_cache* c, const int32_t* src_of, int32_t* dev_status, ngc_stream stream);

/* ngc_fork_kv on a paged cache: rows are copied page by page, from the pages the source's table names to the
 * first pages of b's own table (the tables do not change).  A bad page-table entry among them (NGC_DEV_BAD_PAGE) leaves
 * b's lengths as they were; the rows of the lists whose entries are good may have been copied. */
int ngc_fork_pages(ngc_paged_cache* c, const int32_t* src_of, int32_t* dev_status, ngc_stream stream);

/*
 * Latent attention.  (The paper's models give every KV head rows of its own;
 * these calls serve models whose heads share ONE row per token and layer: a
 * latent vector c_j that every head's key and value are projections of, and a
 * rotary part r_j.)  With qn, qr the two parts of a head's query and U_h, W_h
 * its projections of the latent to a key and a value, the EXPANDED form is
 *   z_hj = scale * (qn_h . (U_h c_j) + qr_h . r_j),   out_h = sum_j softmax(z)_hj W_h c_j;
 * taking U_h into the query, ql_h = U_h^T qn_h, and W_h behind the sum gives
 * the ABSORBED form, which reads nothing but the shared rows:
 *   z_hj = scale * (ql_h . c_j + qr_h . r_j),         o_h = sum_j softmax(z)_hj c_j,   out_h = W_h o_h.
 * Generation uses the absorbed form over a pool of pages (ngc_pool_update ->
 * ngc_latent_write -> ngc_latent_decode per step), prompts and training the
 * expanded one over whole sequences (ngc_latent_replay_attn and its gradient).
 * The projections themselves are the caller's matrix products.  Built for bf16.
 */

/* Rows in pages of a COMMON pool: any page may serve any sequence, so pages that
 * eviction or a finished sequence frees go on to others.  As everywhere a
 * sequence has G eviction lists (`lists`, with one KV head: SHARED: G = 1,
 * otherwise G = L); list gi has its own free pages, the same n_pages in every
 * layer it covers.  Owns nothing. */
typedef struct {
  void* rows;            /* [L][n_pages][page][d_latent + d_rope] bf16, 16-byte aligned */
  int32_t* page_table;   /* [B][G][pages_cap]: page j of list gi of sequence b; entries at and beyond ceil(len / page) are -1 */
  uint8_t* page_used;    /* [G][n_pages]: 0 = free */
  int32_t* lens;         /* [B][G] alive tokens */
  int32_t L, B;
  int32_t d_latent;      /* 128, 256, 384 or 512 */
  int32_t d_rope;        /* 16, 32, 48 or 64 */
  int32_t dtype;         /* NGC_BF16 */
  int32_t page;          /* tokens per page, 32 or 64 */
  int32_t pages_cap, n_pages, lists;   /* L * n_pages * page < 2^31 */
} ngc_latent_pool;

/*
 * The pool's books for the next step, in one launch and for every list on its
 * own: what an eviction round keeps, what finished sequences give back, pages
 * for the new tokens and where each of them goes.  For sequence b:
 *   budget[b] >= 0:  only the units (= pages) kept_sorted[b][gi][0 .. budget[b]) stay: they move to the front of the table
 *                    row in that order, the others return to the pool, the length becomes what was kept (a short last page
 *                    stays last); budget[b] = -1, or kept_sorted NULL: no eviction
 *   n_new[b] >= 0:   the sequence grows by n_new[b] tokens;  n_new[b] = -1: it is finished, its pages return to the pool, its
 *                    length becomes 0
 * All returns come before all growth; growth takes the lowest free page numbers
 * in order of sequences.  Where they are too few, each sequence that still fits beside the ones before it grows: one that does
 * not keeps no pages from those after it.  Token t of sequence b's new ones is number first[b] + t.
 *   n_new [B];  kept_sorted [B][G][k_max] as written by ngc_sample_evict, budget [B], or both NULL
 *   slots [G][n_slots] out: page * (tokens per page) + place in the page of every new token; -1 from first[B] on
 *   first [B+1] out: new tokens of the sequences before (2^30 - 1 where there are more)
 * Per list, a sequence with counts that are none (NGC_DEV_BAD_COUNTS: also more
 * new tokens than n_slots holds), a bad kept list (NGC_DEV_BAD_KEPT) or page-table entry
 * (NGC_DEV_BAD_PAGE) is left as it was; one that outgrows pages_cap
 * (NGC_DEV_STRIP_FULL) or what is free when its turn comes (NGC_DEV_POOL_FULL) evicts but does
 * not grow.  Their new tokens get slot -1.  So after a report a sequence may have grown on some lists and not on others (its lens
 * differ by n_new[b]); calling again would grow the former twice.  n_new[b] = -1 takes it back on all lists, and it can be admitted anew.
 * B <= 8192, n_slots < 2^30.
 */
int ngc_pool_update(ngc_latent_pool* c, const int32_t* kept_sorted, const int32_t* budget, int k_max, const int32_t* n_new,
                    int32_t* slots, int n_slots, int32_t* first, int32_t* dev_status, ngc_stream stream);

/*
 * Writes the rows of new tokens to their slots, for layers [layer_begin, layer_end): bit-exact copies.
 *   latent [L][n_slots][d_latent], rope [L][n_slots][d_rope] bf16, 16-byte aligned; slots [G][n_slots] as written by ngc_pool_update
 * Slot -1: no row; a slot beyond the pool is reported (NGC_DEV_BAD_SLOT) and skipped.  A slot that occurs twice gets one of its
 * rows, or pieces of both.
 */
int ngc_latent_write(ngc_latent_pool* c, const int32_t* slots, int n_slots, const void* latent, const void* rope,
                     int layer_begin, int layer_end, int32_t* dev_status, ngc_stream stream);

/*
 * Absorbed form for one token per sequence, over the alive rows of the pool (the
 * token's own row among them: written before), for layers [layer_begin, layer_end):
 *   q_latent [L][B][H][d_latent], q_rope [L][B][H][d_rope] bf16, 16-byte aligned;  H 1 .. 128
 *   scale    positive, at most 2e38
 *   out      [L][B][H][d_latent] of out_dtype (NGC_F32 or NGC_BF16), 16-byte aligned; an empty sequence gives zeros
 * fp32 scores, softmax and sums; the probabilities are rounded to bf16 for the
 * second product.  Rows of a page behind the length take no part whatever they
 * hold; a head with a score that is NaN or plus infinity, or with none above
 * minus infinity, gets NaN.  A length outside 0 .. pages_cap * page is reported (NGC_DEV_BAD_COUNTS) and the
 * sequence skipped; a bad page-table entry is reported (NGC_DEV_BAD_PAGE) and the
 * outputs of its sequence are unspecified.  Results are the same in every run; where one lies in its
 * last bits may depend on the call's other lengths (they decide how the work is
 * cut).  Calls that may run at the same time need a workspace each.
 * Workspace: ngc_latent_decode_workspace_bytes (it depends on d_latent and H only).
 */
int ngc_latent_decode(const ngc_latent_pool* c, const void* q_latent, const void* q_rope, int H, int layer_begin, int layer_end,
                      float scale, void* out, int out_dtype, void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);
size_t ngc_latent_decode_workspace_bytes(const ngc_latent_pool* c, int H);

/* Whole sequences in token-major rows, as projections write them: sequence b owns rows seq_off[b] .. seq_off[b+1], the first
 * lens[b] of which are tokens.  Rows that are no tokens are neither read into results nor written. */
typedef struct {
  const int64_t* seq_off;    /* [B+1], seq_off[0] = 0, seq_off[B] = rows */
  const int32_t* lens;       /* [B] */
  int64_t rows;              /* host copy; L * rows < 2^31 */
  int32_t L, B, H;           /* L * B <= 65535 */
  int32_t d_nope, d_v;       /* 128 */
  int32_t d_rope;            /* 16, 32, 48 or 64 */
  int32_t dtype;             /* NGC_BF16 */
  int32_t max_len;           /* host bound on lens */
} ngc_latent_seqs;

/*
 * Expanded form for whole sequences under their history of evictions, the
 * counterpart of ngc_replay_attn: the query at position t sees key j iff j <= t
 * and no round at or before t has evicted j.
 *   q      [L][rows][H][d_nope + d_rope];  kv [L][rows][H][d_nope + d_v]: every head's key part and value;
 *   k_rope [L][rows][d_rope]: one rotary key part for all heads; all bf16, 16-byte aligned
 *   alive_pos [n_rounds][B][G][kt_max], alive_count [n_rounds][B][G], total_before [n_rounds][B] as for ngc_replay_attn
 *          (ascending per sequence; G by `lists` with one KV head); n_rounds = 0: causal attention (prompts).  A position that
 *          a round has evicted does not come back: a later round's list that names it again makes it count as never evicted
 *          in between.  A bad position is reported (NGC_DEV_BAD_KEPT) and passed over; a bad count is reported and counts as a
 *          round that keeps nothing.
 *   scale  positive, at most 2e38
 *   out    [L][rows][H][d_v] of out_dtype (NGC_F32 or NGC_BF16), 16-byte aligned
 *   lse    [L][H][rows] fp32 or NULL: log of the sum of exp(z) of every query, for the gradient (-inf for a query that sees nothing,
 *          whose output is zero)
 * fp32 scores, softmax and sums; probabilities rounded to bf16 for the second
 * product.  Infinities or NaN in a sequence's rows leave its results
 * unspecified, other sequences' untouched.  A length outside its sequence's rows or above max_len is
 * reported (NGC_DEV_BAD_COUNTS) and the sequence skipped.
 * Workspace: ngc_latent_replay_workspace_bytes(s, lists, n_rounds, 0); calls that may run at the same time need one each.
 */
int ngc_latent_replay_attn(const ngc_latent_seqs* s, const void* q, const void* kv, const void* k_rope,
                           const int32_t* alive_pos, const int32_t* alive_count, const int32_t* total_before, int n_rounds,
                           int kt_max, int lists, float scale, void* out, int out_dtype, float* lse,
                           void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);

/*
 * Gradient of ngc_latent_replay_attn with respect to q, kv and k_rope (for the latter summed over the heads that share it):
 *   P = exp(z - lse),  D = sum_c grad_out * out,  dV = P^T grad_out,  dz = scale P (grad_out V^T - D),
 *   dQ = dz K,  dK = dz^T Q.
 *   out, lse as the forward call wrote them; grad_out [L][rows][H][d_v] bf16
 *   grad_q, grad_kv, grad_k_rope: bf16 in the shapes of q, kv, k_rope; rows of tokens are written, no others
 * P and dz are rounded to bf16 for the products, every sum is held in fp32 and rounded once.  Results are the same in every run.
 * Workspace: ngc_latent_replay_workspace_bytes(s, lists, n_rounds, 1); its contents need not be those of the forward call.
 */
int ngc_latent_replay_attn_backward(const ngc_latent_seqs* s, const void* q, const void* kv, const void* k_rope,
                                    const int32_t* alive_pos, const int32_t* alive_count, const int32_t* total_before,
                                    int n_rounds, int kt_max, int lists, float scale, const void* out, int out_dtype,
                                    const float* lse, const void* grad_out, void* grad_q, void* grad_kv, void* grad_k_rope,
                                    void* ws, size_t ws_bytes, int32_t* dev_status, ngc_stream stream);
size_t ngc_latent_replay_workspace_bytes(const ngc_latent_seqs* s, int lists, int n_rounds, int backward);

/*
 * Self-test of the bounded wait.  (The paper has no counterpart: this is a
 * diagnostic of the library's own safety contract.)  The streaming kernels wait
 * for their TMA data on mbarriers with a time limit; when a wait runs out the
 * kernel records NGC_DEV_TIMEOUT in *dev_status and runs on to its end.  This
 * call launches one warp that waits, for at most limit_us microseconds
 * (1 .. 100000), on a barrier that nothing ever completes, so that the path
 * can be exercised on a healthy device: afterwards *dev_status is
 * NGC_DEV_TIMEOUT (if it was 0 before), *waited_ns (device uint64, may be
 * NULL) holds the time spent waiting, and the stream and context are usable as
 * before.  dev_status must not be NULL.
 */
int ngc_selftest_bounded_wait(uint32_t limit_us, int32_t* dev_status, uint64_t* waited_ns, ngc_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* NGC_H_ */
