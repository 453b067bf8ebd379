/*
 * pyr.h - C ABI of the MI355X (gfx950) prefill layer step of PyramidInfer
 * (arXiv 2405.12532, Algorithm 1 "One forward pass in PyramidInfer" and the
 * prefill paragraph of Section 4.1).
 *
 * One layer step, for every sequence of a packed batch:
 *   attention weights  ->  ensemble weights of the recent window  ->  TopP
 *   ->  Gather of K, V (and of the hidden rows that feed the next layer).
 *
 * Conventions that hold for every function below
 *   - returns PYR_OK (0) or a negative pyr_status; never throws;
 *   - arguments are checked on the host before anything is launched; a
 *     failed check launches nothing;
 *   - "dev" pointers are device (HBM) addresses, "host" pointers are ordinary
 *     host memory read during the call only; all buffers are caller-owned;
 *   - work is enqueued on `stream` (a hipStream_t passed as void*, NULL is the
 *     default stream); nothing synchronises the stream or the device and
 *     nothing allocates or frees device memory;
 *   - packed layouts, row-major, token-major, bfloat16 unless said otherwise:
 *       q, out : [T, Hq, d]      k, v : [T, Hkv, d]      hidden : [T, D]
 *     sequence b owns rows seq_offsets[b] .. seq_offsets[b+1]-1 (S_b rows);
 *     query head h reads key/value head h / (Hq / Hkv);
 *   - supported: d in {64, 128}, Hq % Hkv == 0, w >= 1, T < 2^31.
 */
#ifndef PYR_H
#define PYR_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define PYR_API __attribute__((visibility("default")))
#else
#define PYR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum pyr_status {
    PYR_OK = 0,
    PYR_ERR_NULL = -1,        /* a required pointer is NULL                               */
    PYR_ERR_SHAPE = -2,       /* negative / inconsistent sizes                            */
    PYR_ERR_UNSUPPORTED = -3, /* head_dim, head grouping or row size outside the set     */
    PYR_ERR_KEEP_LEN = -4,    /* keep_len[b] outside [min(w, S_b), S_b]                   */
    PYR_ERR_OFFSETS = -5,     /* seq_offsets not 0-based, not monotone, or != T at end    */
    PYR_ERR_WORKSPACE = -6,   /* workspace NULL, misaligned (256 B) or too small          */
    PYR_ERR_LAUNCH = -7,      /* the HIP runtime refused a launch (see hipGetLastError)   */
    PYR_ERR_TOO_LARGE = -8    /* needs more than PYR_STATIC_SCRATCH_BYTES of workspace     */
} pyr_status;

/* Size of the library's own workspace buffer (see pyr_prefill_layer_static). */
#define PYR_STATIC_SCRATCH_BYTES ((size_t)40 << 20)

typedef struct pyr_shape {
    int32_t n_seqs;       /* B                                   */
    int32_t total_tokens; /* T = sum of S_b                      */
    int32_t max_seqlen;   /* max S_b                             */
    int32_t n_q_heads;    /* Hq                                  */
    int32_t n_kv_heads;   /* Hkv                                 */
    int32_t head_dim;     /* d                                   */
} pyr_shape;

/* Text for a status code (static storage, never NULL). */
PYR_API const char* pyr_strerror(int status);

/* Library version, major*10000 + minor*100 + patch. */
PYR_API int pyr_version(void);

/*
 * Host only.  Bytes of device workspace pyr_prefill_layer needs for this
 * shape and window (row statistics of the softmax for the score pass, the
 * tile map of ragged batches, partial sums of the score pass).  Align the buffer to 256 bytes.
 */
PYR_API int pyr_workspace_bytes(const pyr_shape* shape, int32_t w, size_t* bytes_out);

/*
 * Host only.  Retention count for the next layer (Algorithm 1: the ratio p is
 * reduced layer by layer, and a layer whose length is at or below the minimum
 * PvC length N_l is left alone):
 *   k = max(floor((num*S + den/2)/den), floor_len, min(w, S)), capped at S.
 * Errors: PYR_ERR_NULL, PYR_ERR_SHAPE (S < 0, w < 1, den <= 0, num < 0, num > den).
 */
PYR_API int pyr_schedule_next(int32_t S, int32_t w, int32_t num, int32_t den, int32_t floor_len,
                      int32_t* keep_len_out);

/*
 * Host only.  Lengths of one sequence through n_layers layers, each with its own ratio
 * num[l]/den and minimum PvC length floor_len[l] (Algorithm 1: input N = {N_0, ...} and a p
 * that decays from layer to layer - the caller chooses the sequence p_l, e.g. geometric or
 * one of the patterns of the decay ablation in Section 5):
 *   context_relative == 0:  k = floor((num[l]*S + den/2)/den)                 (as pyr_schedule_next)
 *   context_relative != 0:  k = L' + floor((num[l]*(S-L') + den/2)/den), L' = min(w,S)
 *                           (Algorithm 1 ranks the columns :-L only: p as a fraction of the context)
 * then k = max(k, floor_len[l], L') capped at S, and S <- k.
 *   len_out            host int32 [n_layers+1], written: len_out[0] = S, len_out[l+1] after layer l
 * Errors: PYR_ERR_NULL, PYR_ERR_SHAPE (as pyr_schedule_next, per layer; len_out is then partly written).
 */
PYR_API int pyr_schedule_plan(int32_t S, int32_t w, int32_t n_layers, const int32_t* num, int32_t den,
                      const int32_t* floor_len, int32_t context_relative, int32_t* len_out);

/*
 * Step 1 - attention weights applied to V (Algorithm 1, "compute attention
 * weights of KV"): causal softmax attention inside each sequence,
 *   out[i,h,:] = sum_{j<=i} softmax_j(scale * q[i,h,:].k[j,h/g,:]) v[j,h/g,:].
 * bf16 MFMA products, fp32 accumulation and fp32 online softmax.
 *   q, k, v            dev, in
 *   seq_offsets_dev    dev int32 [B+1];  seq_offsets_host  host copy of the same
 *   softmax_scale      <= 0 selects 1/sqrt(d)
 *   out                dev bf16 [T,Hq,d], written
 *   lse                dev fp32 [T,Hq], written: log2 of the softmax denominator of
 *                      every row, in the scaled base-2 domain,
 *                      lse[i,h] = log2(sum_j 2^(scale*log2(e)*s_ij)); may be NULL.  A logit of -inf is a
 *                      key without weight; a row that has no other: -inf here, NaN in out
 *   tile_map           dev int32 [B+1] scratch, written (prefix sums of query
 *                      tiles per sequence); part of the workspace
 */
PYR_API int pyr_attention(const void* q, const void* k, const void* v,
                  const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                  const pyr_shape* shape, float softmax_scale,
                  void* out, float* lse, int32_t* tile_map, void* stream);

/*
 * Step 2 - ensemble attention weights (Algorithm 1, A_e = weighted_avg(A[-L:, :-L]);
 * Section 3.2.1): for every key position t of every sequence
 *   scores[t] = 1/(Hq*L') * sum_h sum_{i=S-L'}^{S-1} A_h[i,t],   L' = min(w, S),
 * uniform weights, all S columns written (the last L' too), fixed summation
 * order (bit-reproducible).  Needs `lse` from pyr_attention.
 *   scores             dev fp32 [T], written
 */
PYR_API int pyr_score(const void* q, const void* k, const float* lse,
              const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
              const pyr_shape* shape, int32_t w, float softmax_scale,
              float* scores, void* stream);

/*
 * Step 2 with averaging weights (Section 4.1, prefill phase: the ensemble is a weighted
 * average that may favour the more recent rows; the paper prints no weights, so they are
 * an argument):
 *   scores[t] = 1/Hq * sum_h sum_i omega_i A_h[i,t] / sum_i omega_i.
 *   row_weights_dev    dev fp32 [w], one weight per row of a full recent window in
 *                      position order (row_weights_dev[w-1]: the last token); a sequence
 *                      shorter than w uses the last S_b of them.  NULL = uniform, the
 *                      same as pyr_score.  The values are not checked (they live on the
 *                      device): they must be finite and >= 0, with a positive sum over
 *                      the rows in use, else the scores are undefined (NaN or inf).
 */
PYR_API int pyr_score_weighted(const void* q, const void* k, const float* lse,
                       const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                       const pyr_shape* shape, int32_t w, float softmax_scale,
                       const float* row_weights_dev, float* scores, void* stream);

/*
 * Step 3 - TopP (Algorithm 1, TopP(A_e, p) with a count: Section 3.1.1 calls p
 * a retention ratio): per sequence the keep_len[b]-L' context positions
 * (0 .. S_b-L'-1) with the largest score, ties to the lower position, plus the
 * last L' positions; ascending.  Exact on the fp32 values given.
 *   scores             dev fp32 [T], in, all values >= 0 and not NaN
 *   keep_len_dev       dev int32 [B];  keep_len_host  host copy, min(w,S_b) <= k_b <= S_b
 *   kept_idx           dev int32 [sum k_b], written: global packed row numbers
 *   out_offsets_dev    dev int32 [B+1], written: prefix sums of keep_len
 * A sequence of length 0 (keep_len 0) contributes nothing; with n_seqs == 0 nothing is launched
 * and nothing is written, out_offsets_dev[0] included.
 */
PYR_API int pyr_select(const float* scores,
               const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
               const int32_t* keep_len_dev, const int32_t* keep_len_host,
               int32_t n_seqs, int32_t w,
               int32_t* kept_idx, int32_t* out_offsets_dev, void* stream);

/*
 * Steps 4/5 - Gather (Algorithm 1, PvC <- Gather(KV, index); Figure 2(c): the
 * next layer only computes the kept tokens): dst[j,:] = src[kept_idx[j],:]
 * for j < n_kept, byte-exact.
 *   src, dst           dev, rows of row_bytes bytes (a multiple of 16, both
 *                      16-byte aligned), dst must not overlap src
 *   kept_idx           dev int32 [n_kept], every value a valid row of src
 *   n_kept == 0 is a no-op.
 */
PYR_API int pyr_compact(const void* src, size_t row_bytes, const int32_t* kept_idx, int64_t n_kept,
                void* dst, void* stream);

/* Same as two pyr_compact calls with one index list, in a single launch (K and V). */
PYR_API int pyr_compact2(const void* src0, void* dst0, const void* src1, void* dst1, size_t row_bytes,
                 const int32_t* kept_idx, int64_t n_kept, void* stream);

/*
 * Position ids of the kept tokens (Appendix A.2, the "gather" strategy of Table 5: the
 * survivors keep the position encodings they had instead of being renumbered):
 *   pos_out[j] = pos[kept_idx[j]]  for j < n_kept.
 *   pos                dev int32, indexed by packed row; pos_out dev int32 [n_kept], written
 *   kept_idx           dev int32 [n_kept], every value a valid row of pos
 * Carried through every layer, pos_out names each row's place in the original prompt.
 * n_kept == 0 is a no-op.
 */
PYR_API int pyr_gather_positions(const int32_t* pos, const int32_t* kept_idx, int64_t n_kept,
                         int32_t* pos_out, void* stream);

/*
 * The whole layer step (Algorithm 1, body of the loop, prefill phase): what
 * pyr_attention -> pyr_score -> pyr_select -> pyr_compact2 compute, on one stream
 * (see pyr_prefill_layer_fused for how the launches are merged).
 *   scores             dev fp32 [T], written (required: the selection reads it)
 *   k_out, v_out       dev bf16 [sum k_b, Hkv, d]; both NULL skips the gather
 *   workspace          dev, >= pyr_workspace_bytes(), 256-byte aligned
 */
PYR_API int pyr_prefill_layer(const void* q, const void* k, const void* v,
                      const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                      const pyr_shape* shape, int32_t w, float softmax_scale,
                      const int32_t* keep_len_dev, const int32_t* keep_len_host,
                      void* out, float* scores, int32_t* kept_idx, int32_t* out_offsets_dev,
                      void* k_out, void* v_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * pyr_prefill_layer for callers that cannot hand over a workspace they allocated: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments without
 * `workspace`; the workspace is a buffer inside the library's device image instead
 * (PYR_STATIC_SCRATCH_BYTES = 40 MiB per GPU the library runs on, held until the process ends;
 * enough for every shape with pyr_workspace_bytes() <= 40 MiB, i.e. T*Hq <= about 10.4 M rows x heads:
 * 64 x 2048 tokens x 32 heads uses 16 MiB, 4 x 32768 x 64 heads 32 MiB).  The call allocates
 * and frees nothing; the first call on a device looks the buffer's address up.
 *   - a larger step returns PYR_ERR_TOO_LARGE and launches nothing;
 *   - all calls on one GPU share the buffer: calls that overlap in time on one GPU (different
 *     streams or threads) race; serialise them or use pyr_prefill_layer with separate workspaces;
 *   - results are identical to pyr_prefill_layer's.
 */
PYR_API int pyr_prefill_layer_static(const void* q, const void* k, const void* v,
                      const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                      const pyr_shape* shape, int32_t w, float softmax_scale,
                      const int32_t* keep_len_dev, const int32_t* keep_len_host,
                      void* out, float* scores, int32_t* kept_idx, int32_t* out_offsets_dev,
                      void* k_out, void* v_out, void* stream);

/*
 * The same with the two optional extras: averaging weights for step 2 (see
 * pyr_score_weighted; NULL = uniform) and position ids gathered alongside K and V
 * (see pyr_gather_positions; pos and pos_out both NULL skips it).
 */
PYR_API int pyr_prefill_layer_ex(const void* q, const void* k, const void* v,
                      const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                      const pyr_shape* shape, int32_t w, float softmax_scale,
                      const int32_t* keep_len_dev, const int32_t* keep_len_host,
                      const float* row_weights_dev, const int32_t* pos,
                      void* out, float* scores, int32_t* kept_idx, int32_t* out_offsets_dev,
                      void* k_out, void* v_out, int32_t* pos_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * The whole layer step in as few launches as it takes (Appendix A.1 and the Limitations section: at small
 * batch the cost of selecting the PvC eats the gain - there every launch counts): attention; the score pass (a small
 * batch's in the attention's launch, by a walk that finds the denominators itself),
 * which, when the batch is too small to fill the chip otherwise, splits the heads over several workgroups that
 * write partial sums; the selection, which adds those in a fixed order; ONE gather for K, V, the hidden rows and the position ids
 * (in the selection's launch where there are only few rows).
 * pyr_prefill_layer and pyr_prefill_layer_ex are this call without the hidden rows.
 *   hidden             dev, rows of hidden_row_bytes bytes (a multiple of 16) indexed by packed row; hidden_out
 *                      dev [sum k_b rows], written; both NULL skips them
 *   everything else as in pyr_prefill_layer_ex; results are those of the separate calls (scores may differ in
 *   the last bits when the heads are split, as the partial sums are rounded once more, and where a walk finds the denominators itself).
 */
PYR_API int pyr_prefill_layer_fused(const void* q, const void* k, const void* v,
                      const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                      const pyr_shape* shape, int32_t w, float softmax_scale,
                      const int32_t* keep_len_dev, const int32_t* keep_len_host,
                      const float* row_weights_dev, const void* hidden, size_t hidden_row_bytes, const int32_t* pos,
                      void* out, float* scores, int32_t* kept_idx, int32_t* out_offsets_dev,
                      void* k_out, void* v_out, void* hidden_out, int32_t* pos_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Generation-phase update of one layer's compressed cache (Algorithm 1 with a non-empty
 * cache, KV = cat(PvC_past, KV); Section 4.1, generation phase: the recent window slides
 * over the generated tokens and the PvC is selected again with the prefill phase's
 * operation; with a constant keep_len the cache stays at a fixed size for any input length).
 *   k, v               dev bf16 [T,Hkv,d]: the packed caches with the new tokens' rows
 *                      already appended - per sequence its kept context rows, then its
 *                      recent rows, S_b rows in all (seq_offsets as elsewhere)
 *   q_win              dev bf16 [B,w,Hq,d]: the queries of the recent rows, right-aligned:
 *                      q_win[b,w-1] belongs to the newest token (cache row S_b-1); a
 *                      sequence with S_b < w uses the last S_b slots, the others are not read
 *   row_weights_dev    as in pyr_score_weighted, NULL = uniform;  pos / pos_out as in
 *                      pyr_prefill_layer_ex, both NULL skips them
 *   scores             dev fp32 [T], written: window row i (cache row S_b-L'+i) sees the
 *                      cache rows 0 .. S_b-L'+i; otherwise as pyr_score
 *   kept_idx, out_offsets_dev, k_out, v_out: as in pyr_prefill_layer (out of place: k_out
 *                      must not overlap k)
 *   workspace          dev, >= pyr_decode_workspace_bytes(), 256-byte aligned
 * Up to five launches on the stream: softmax statistics of the window rows per range of keys, their
 * fold into row denominators, the score pass, the selection, one gather for K, V and position ids (or fewer: short
 * sequences take one walk for the first three, few rows are gathered in the selection's launch).  The attention
 * output of the new token itself is not computed here.
 */
PYR_API int pyr_decode_workspace_bytes(const pyr_shape* shape, int32_t w, size_t* bytes_out);
PYR_API int pyr_decode_update(const void* q_win, const void* k, const void* v,
                      const int32_t* seq_offsets_dev, const int32_t* seq_offsets_host,
                      const pyr_shape* shape, int32_t w, float softmax_scale,
                      const int32_t* keep_len_dev, const int32_t* keep_len_host,
                      const float* row_weights_dev, const int32_t* pos,
                      float* scores, int32_t* kept_idx, int32_t* out_offsets_dev,
                      void* k_out, void* v_out, int32_t* pos_out,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * A cache held in 4 bits, for the generation phase of many sequences: pages in device memory that the slots of a table share.
 * K and V of a token are stored as 4-bit floating-point numbers (e2m1: a sign and 0, 0.5, 1, 1.5, 2, 3, 4 or 6) times a power of two per 32
 * channels of a head (one byte from 1 to 252, 2^(byte - 127), or 255: not a number) - 34 bytes for 32 channels of K and V, 4.25 bits a number against
 * bf16's 16.  A block's power of two is the smallest that brings its largest magnitude to 7 or less (7 is rounded to 6), between 2^-126 and 2^125; numbers are
 * rounded to the nearest, ties to the even code; a block with an infinity or a NaN is stored as NaN as a whole.
 *
 * A slot is a sequence: lens[slot] tokens, in pages table[slot][0 .. ceil(lens / page_tokens) - 1], the last one filled in part.  refs[page] says how
 * many slots hold a page; 0 is a free one.  Full pages may be shared (pyr_cache_fork), a page filled in part never is, so storing behind the last
 * token touches no other slot.  An empty cache: refs and lens 0 (the table and the pages may hold anything).
 * All of it lives in device memory that the caller owns and may be read between calls; no call waits for the device, and every call
 * can be captured into a graph and replayed, the sequences growing from replay to replay.  Calls that change one cache, and calls that read it,
 * are ordered by the caller (one stream, or events).
 *
 * What is on the device is checked there: a slot of -1 is a row of a padded batch and skipped; pages outside the pool and slots outside the table are never
 * followed (what each call does then is said there).  The calls that hand out or share pages write a status to device memory:
 *   0   done
 *   n > 0   n pages are lacking: nothing was changed
 *   PYR_CACHE_BAD_SLOT    a slot outside the table (other than -1) or named twice, a child that holds tokens or is a parent: nothing was changed
 *   PYR_CACHE_BAD_COUNT   a count below 0, or more tokens than a row of the table or the call's limit holds: nothing was changed
 * (the lower one if both apply).  Pages are handed out from the lowest, in the order of the rows.
 *
 * Layout, for programs that read or write pages themselves: a page is [n_kv_heads][page_tokens / 32] tiles of 34 * d bytes, a tile
 * being 32 tokens of one head; with nb = d / 32, in this order
 *   16 d bytes  K's codes   [half 2][block nb][token 16][byte 16]: token 16 * half + token, channel 32 * block + 2 * byte (low four bits) and the next
 *   16 d bytes  V's codes   [h d/64][j 4][r 16][p 2][q 2][byte 4]: channel 64 h + 32 p + 2 r + q, token 16 * (byte / 2) + 4 j + 2 * (byte % 2) and the next
 *      d bytes  K's scales  [block nb][token 16][half 2]
 *      d bytes  V's scales  [j 4][block nb][half 2][s 4]: token 16 * half + 4 j + s
 *
 * Host checks of every call: PYR_ERR_NULL; PYR_ERR_SHAPE (negative sizes; n_slots > PYR_CACHE_MAX_SLOTS; n > PYR_CACHE_MAX_ROWS where pages are handed out or shared);
 * PYR_ERR_UNSUPPORTED (head_dim not 64 or 128, page_tokens not a power of two from 32 to 1024, pages not 256-byte aligned, rows not 16-byte aligned,
 * 2^31 or more tokens in the pool, a row of the table or a batch, or entries of the table; 2^24 or more workgroups, which take a KV head of a sequence in
 * the attention, a sequence's 32 tokens of up to four heads where rows go in or out, and 32 kept tokens where slots are cut); PYR_ERR_WORKSPACE;
 * PYR_ERR_LAUNCH.  Limits that only cut up the work (max_keep, max_new, max_len) may be as large as an int32.
 */
#define PYR_CACHE_MAX_ROWS 4096
#define PYR_CACHE_MAX_SLOTS 262144
#define PYR_CACHE_BAD_SLOT (-1)
#define PYR_CACHE_BAD_COUNT (-2)

typedef struct pyr_cache {
    void* pages;          /* dev [n_pages] pages of pyr_cache_page_bytes() bytes, 256-byte aligned   */
    int32_t* refs;        /* dev int32 [n_pages]                                                     */
    int32_t* table;       /* dev int32 [n_slots, max_pages]                                          */
    int32_t* lens;        /* dev int32 [n_slots]                                                     */
    int32_t n_pages;
    int32_t page_tokens;  /* 32, 64, ... 1024                                                        */
    int32_t n_slots;
    int32_t max_pages;    /* of a slot                                                               */
    int32_t n_kv_heads;
    int32_t head_dim;
} pyr_cache;

/* Host only.  Bytes of a page; reads page_tokens, n_kv_heads and head_dim of the cache. */
PYR_API int pyr_cache_page_bytes(const pyr_cache* cache, size_t* bytes_out);

/*
 * Room for n_new[i] more tokens in slots[i] (i < n), and their place: start[i] = lens[slots[i]], lens[slots[i]] += n_new[i], pages as needed.
 *   slots, n_new       dev int32 [n]
 *   start              dev int32 [n], written: the place of the first new token, what pyr_cache_store takes; -1 for a
 *                      skipped row, and for all rows if the status is not 0
 *   status             dev int32 [1], written
 */
PYR_API int pyr_cache_reserve(const pyr_cache* cache, const int32_t* slots, const int32_t* n_new, int32_t n,
                      int32_t* start, int32_t* status, void* stream);

/*
 * children[i] becomes a copy of parents[i]: full pages are shared, of a page filled in part the tokens are copied into a fresh one.  Several children
 * may have one parent.  A row is skipped if both are -1.  A parent's page outside the pool is passed on as it is; where that is the page filled in
 * part, the child's fresh one keeps what lay in it.
 *   parents, children  dev int32 [n]; children are empty slots
 *   status             dev int32 [1], written
 */
PYR_API int pyr_cache_fork(const pyr_cache* cache, const int32_t* parents, const int32_t* children, int32_t n,
                   int32_t* status, void* stream);

/*
 * Slots are emptied: their pages' counts go down (0: free), their entries of the table become -1, lens 0.  A slot named twice is
 * emptied once; slots outside the table are skipped, pages outside the pool have no count that goes down.
 *   slots              dev int32 [n]
 */
PYR_API int pyr_cache_release(const pyr_cache* cache, const int32_t* slots, int32_t n, void* stream);

/*
 * Slots are cut to the tokens that a selection kept (Gather(KV, index) without leaving 4 bits): token j of slots[i] becomes its token
 * kept_idx[out_offsets[i] + j] - seq_offsets[i], j < out_offsets[i+1] - out_offsets[i], its bits unchanged.  Indexes as pyr_select and pyr_decode_update write
 * them, seq_offsets as the batch they ran on (lens[slots[i]] rows each); any order and repetitions are fine.
 * The tokens go into fresh pages, then the old ones are given back: the pool needs room for both.  A slot that shares pages leaves the others as they are.
 *   slots              dev int32 [n]
 *   kept_idx           dev int32 [n_kept]; an index outside the slot's tokens, or a token on a page outside the pool, gives a token of NaN
 *   seq_offsets        dev int32 [n] or more;  out_offsets  dev int32 [n+1], within 0 .. n_kept
 *   max_keep           no out_offsets[i+1] - out_offsets[i] is larger
 *   status             dev int32 [1], written
 *   workspace          dev, >= pyr_cache_compact_workspace_bytes(), 256-byte aligned
 */
PYR_API int pyr_cache_compact_workspace_bytes(const pyr_cache* cache, int32_t n, size_t* bytes_out);
PYR_API int pyr_cache_compact(const pyr_cache* cache, const int32_t* slots, int32_t n, const int32_t* kept_idx, int32_t n_kept,
                      const int32_t* seq_offsets, const int32_t* out_offsets, int32_t max_keep, int32_t* status,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Rows of K and V into the cache: token start[i] + j of slots[i] becomes row offsets[i] + j, or row row_idx[offsets[i] + j],
 * j < offsets[i+1] - offsets[i].  Rows of a prompt's selection go in straight from the layer's K and V: row_idx = kept_idx, offsets = out_offsets.
 *   k, v               dev bf16 [n_rows, Hkv, d]
 *   row_idx            dev int32 [n_list] or NULL (then n_list = n_rows)
 *   offsets            dev int32 [n+1];  slots, start  dev int32 [n]
 *   max_new            no offsets[i+1] - offsets[i] is larger (tokens beyond it are not stored, or some of them)
 * Tokens from lens[slots[i]] on (they were not reserved), tokens that have no page, a start of -1 (pyr_cache_reserve found no room) and rows outside
 * k and v or the list (an offset may be below 0) are not stored; nothing else in the pages changes.  Of rows that name the same slot the first is stored.
 */
PYR_API int pyr_cache_store(const pyr_cache* cache, const void* k, const void* v, int32_t n_rows, const int32_t* row_idx, int32_t n_list,
                    const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n, int32_t max_new, void* stream);

/*
 * The cache as bf16 rows (exactly: every number of the cache is one of bf16's), packed as pyr_decode_update and pyr_score read them: row
 * offsets[i] + j is token j of slots[i], j < min(lens[slots[i]], offsets[i+1] - offsets[i], max_len).  Rows that no token goes to stay as they were,
 * those of tokens on a page outside the pool among them; a sequence whose offset is below 0 is skipped.
 *   offsets            dev int32 [n+1];  slots  dev int32 [n]
 *   k_out, v_out       dev bf16 [n_rows, Hkv, d]; one of them may be NULL; rows from n_rows on are not written
 */
PYR_API int pyr_cache_load(const pyr_cache* cache, const int32_t* slots, const int32_t* offsets, int32_t n, int32_t max_len,
                   void* k_out, void* v_out, int32_t n_rows, void* stream);

/*
 * Attention of each sequence's newest n_tokens tokens over its cache, theirs included (store them first): token i of slots[b] sees the tokens
 * 0 .. lens[slots[b]] - n_tokens + i.
 *   out[b,i,h,:] = sum_t softmax_t(scale * q[b,i,h,:].k[t,h/g,:]) v[t,h/g,:]
 * bf16 MFMA products on the cache's exact values (P times V's power of two is rounded to bf16), fp32 accumulation and softmax.  Sums of P V stay in fp32's
 * range as long as V's largest power of two times the sequence's tokens is below 2^114 (a number whose sum leaves it is NaN).  What of P times a power of two
 * lies below 2^-126 may lose its bits: an output is off by another 2^-123 for every token and one, at most.
 *   q                  dev bf16 [n, n_tokens, Hq, d]
 *   slots              dev int32 [n]
 *   max_len            about the longest sequence (it decides how the work is cut up and how large the workspace is, not the result: longer
 *                      ones are right as well); a captured graph takes one for the lengths to come
 *   softmax_scale      <= 0 selects 1/sqrt(d)
 *   out                dev bf16 [n, n_tokens, Hq, d], written
 *   lse                dev fp32 [n, n_tokens, Hq], written, as pyr_attention's; may be NULL
 *   workspace          dev, >= pyr_cache_attention_workspace_bytes(), 256-byte aligned; not read where that is 0
 * A row that sees nothing (an empty slot, a skipped row, fewer tokens in the cache than n_tokens): zeros in out, -inf in lse.  A token of NaN makes
 * the rows that see it NaN, unless its K is a number and its weight 0 in fp32 already when its tile was taken; what a row does not see never reaches it.  A page outside the pool
 * among those of a sequence: NaN in all of its rows, in out and lse.
 * One launch, and one that adds up partial results where few long sequences are split.
 */
PYR_API int pyr_cache_attention_workspace_bytes(const pyr_cache* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                                        size_t* bytes_out);
PYR_API int pyr_cache_attention(const pyr_cache* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads,
                        int32_t max_len, float softmax_scale, void* out, float* lse,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * A cache held in 8 bits, in pages that the slots of a table share as those of the cache in 4 bits are: twice the bytes, two more bits of every number.  Pages
 * are handed out and given back by pyr_cache_reserve and pyr_cache_release on `pool`, whose pages have pyr_cache8_page_bytes() bytes; all other calls on
 * it are the pyr_cache8_* below.  What is said above of slots, pages, counts, statuses, graphs and host checks holds here as well.
 *
 * 32 tokens of a KV head are a block.  K and V of a block are 8-bit floating-point numbers (e4m3: a sign, four exponent bits and three mantissa bits, up to
 * 448, no infinities) times a power of two, one for K and one for V: the smallest that brings the largest magnitude of what has been stored to 448 or
 * less, from 2^-100 to 2^119.  Numbers are rounded to the nearest, ties to the even code; an infinity, a NaN, and what would be rounded to more than
 * 448 * 2^119 is stored as NaN, by itself.  A block that gets tokens behind others keeps its power or takes a larger one, which its older numbers are
 * rounded to (exact, but for those that leave four significant bits: below 2^-6 of a unit).  Storing a block's first token starts it
 * anew: what lay behind the new tokens in it holds nothing then.  So a block is filled from its first token on: the power that lies in front of tokens
 * whose predecessors were never stored counts as theirs, whatever it is (zeroed pages: as the smallest).
 * A block keeps bounds of its K, for pyr_cache8_select: the largest and the smallest number that a channel has held since then, rounded outward to whole
 * multiples of 4 times the power, from -112 to 112; +-127 where one of them was NaN.  When the power grows they are divided and rounded outward.
 *
 * Layout, for programs that read or write pages themselves: for H = n_kv_heads and T = page_tokens / 32, one behind the other, up to a multiple of 256 bytes
 *   [H][T] 64 d bytes   K's codes [half 2][s d/64][j 4][t 16][byte 16]: token 16 * half + t, channel 64 s + 16 j + byte;
 *                       V's codes [g d/32][j 4][r 16][p 2][e 8]: token 16 * (e / 4) + 4 j + e % 4, channel 32 g + 16 p + r
 *   [H][T]  2 d bytes   bounds: the largest [d], the smallest [d], int8
 *   [H][T]  2 bytes     powers of K and of V: 2^(byte - 127)
 *
 * Host checks as above, and PYR_ERR_UNSUPPORTED for pages of 2^31 bytes or more and for lists of more than 2^26 blocks; a workgroup takes a sequence's 32
 * tokens of up to four heads of K, V and Q where rows go in, a token's KV head where blocks are chosen or listed (among more than 256 blocks, 2^23 are too many already).
 */
typedef struct pyr_cache8 {
    pyr_cache pool;       /* pages of pyr_cache8_page_bytes() bytes                                  */
} pyr_cache8;

/* Host only.  Bytes of a page; reads page_tokens, n_kv_heads and head_dim of the pool. */
PYR_API int pyr_cache8_page_bytes(const pyr_cache8* cache, size_t* bytes_out);

/* As pyr_cache_fork; of a page filled in part all bytes are copied. */
PYR_API int pyr_cache8_fork(const pyr_cache8* cache, const int32_t* parents, const int32_t* children, int32_t n, int32_t* status, void* stream);

/* Position encodings by rotation: channels a and b of pair i become a cos(p f_i) - b sin(p f_i) and b cos(p f_i) + a sin(p f_i) at position p. */
typedef struct pyr_rotation {
    const float* freqs;        /* dev fp32 [dims / 2]: f_i, radians a position; finite                                 */
    const int32_t* positions;  /* dev int32 [n_rows]: p of every row, also of rows that a list leaves out             */
    int32_t dims;              /* channels that turn, the first ones of a head: a multiple of 16, at most head_dim    */
    int32_t interleaved;       /* pair i is channels i and i + dims / 2 (0) or 2 i and 2 i + 1 (else)                  */
} pyr_rotation;

/*
 * Rows of K and V into the cache, turned by their positions on the way: token start[i] + j of slots[i] becomes row offsets[i] + j, or row
 * row_idx[offsets[i] + j], j < min(offsets[i+1] - offsets[i], max_new).  The rows of a prompt's selection go in as they are (rotation NULL): row_idx = kept_idx.
 * A new token's go in as the projections leave them; its position is an argument, as a cache that was cut holds fewer tokens than the text has.
 *   k, v               dev bf16 [n_rows, Hkv, d], rows k_stride and v_stride elements apart (a multiple of 8; 0: Hkv * d)
 *   row_idx            dev int32 [n_list] or NULL (then n_list = n_rows)
 *   offsets            dev int32 [n+1];  slots, start  dev int32 [n]
 *   rotation           host, its pointers dev; NULL or dims 0: nothing turns.  Sine and cosine of p f_i are worked out in 64 bits (by less than 2^-32 off for |p f_i| up to
 *                      2^47, those of some angle beyond it) and rounded to fp32, the turn itself is fp32, and K is rounded once, to its code (again in 64 bits where fp32 leaves it next to a border between two)
 *   q                  dev bf16 [n_rows, Hq, d], rows q_stride elements apart, or NULL
 *   q_out              dev bf16 [n_rows, Hq, d], written: the rows of q whose tokens are stored, turned; the others stay as they were
 * Tokens from lens[slots[i]] on (they were not reserved), tokens that have no page and a start of -1 are not stored; a row outside k and v or the list is
 * stored as NaN; nothing else in the pages changes, but for what a larger power does to its block.  Of rows that name the same slot the first is stored.
 * q_out must not overlap k, v or q - but it may be q itself, packed, if no row is named twice.  No rows, no list, max_new 0: nothing is done.
 */
PYR_API int pyr_cache8_append(const pyr_cache8* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride, int32_t n_rows,
                      const int32_t* row_idx, int32_t n_list, const int32_t* offsets, const int32_t* slots, const int32_t* start, int32_t n, int32_t max_new,
                      const pyr_rotation* rotation, const void* q, int64_t q_stride, int32_t n_q_heads, void* q_out, void* stream);

/*
 * The cache as bf16 rows (exactly), packed as pyr_decode_update and pyr_score read them: row offsets[i] + j is token first[i] + j of slots[i],
 * j < min(lens[slots[i]] - first[i], offsets[i+1] - offsets[i], max_len).  Rows that no token goes to stay as they were, those of tokens on a
 * page outside the pool among them; a sequence whose offset or first token is below 0 is skipped.
 *   first              dev int32 [n] or NULL: 0
 *   offsets            dev int32 [n+1];  slots  dev int32 [n]
 *   k_out, v_out       dev bf16 [n_rows, Hkv, d]; one of them may be NULL; rows from n_rows on are not written
 */
PYR_API int pyr_cache8_load(const pyr_cache8* cache, const int32_t* slots, const int32_t* first, const int32_t* offsets, int32_t n, int32_t max_len,
                    void* k_out, void* v_out, int32_t n_rows, void* stream);

/*
 * The blocks that each of a sequence's newest n_tokens tokens attends to, for every KV head.  Token i of slots[b] sees the tokens 0 .. s - 1,
 * s = lens[slots[b]] - n_tokens + i + 1, and so the blocks 0 .. c - 1, c = ceil(s / 32).  It takes the first n_first of them, the last n_recent and, of
 * those in between, the n_best with the highest scores (ties: the lower number):
 *   score = max over the group's query heads h of 2^x sum_c max(u_c hi_c, u_c lo_c)
 * with the block's bounds hi and lo, u_c = q_c / 2^e rounded to the nearest whole number (ties to even, from -127 to 127, 0 for NaN), 2^e the smallest power of two
 * that brings the head's largest finite |q_c| to 127 or less (2^-100 at least), x = min(max(e + 2 + the power of the block's K, -120), 100).  Sums of whole numbers
 * below 2^22: a score is exact in fp32, and the choice the same wherever it is made.
 *   q                  dev bf16 [n, n_tokens, Hq, d];  slots  dev int32 [n]
 *   max_len            at least the longest sequence; of a longer one the blocks from ceil(max_len / 32) on are not among those that are scored
 *   n_first, n_best    0 or more;  n_recent  1 or more
 *   blocks             dev int32 [n, n_tokens, Hkv, n_first + n_recent + n_best], written: ascending, -1 behind the last
 *   workspace          dev, >= pyr_cache8_select_workspace_bytes(), 256-byte aligned; not read where that is 0
 * One launch, or two: where few rows score many blocks, or any score more than 4096.
 */
PYR_API int pyr_cache8_select_workspace_bytes(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, size_t* bytes_out);
PYR_API int pyr_cache8_select(const pyr_cache8* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads,
                      int32_t max_len, int32_t n_first, int32_t n_recent, int32_t n_best, int32_t* blocks, void* workspace, size_t workspace_bytes,
                      void* stream);

/*
 * Attention of each sequence's newest n_tokens tokens over its cache, theirs included, as pyr_cache_attention; or over the blocks of a list for every token and
 * KV head, of which a token sees what it sees without one.
 *   blocks             dev int32 [n, n_tokens, Hkv, n_blocks], as pyr_cache8_select writes it or any other; NULL with n_blocks 0: all blocks.
 *                      An entry that is no block which the token sees is left out, one that is there twice counts twice.
 *   max_len            as in pyr_cache_attention; not looked at where there are lists
 *   q, slots, softmax_scale, out, lse, workspace  as in pyr_cache_attention
 * bf16 MFMA products on the cache's exact values (P as the sum of two bf16 numbers, sixteen bits), fp32 accumulation and softmax.  Sums of P V stay in fp32's range as long as V's
 * largest power of two times the sequence's tokens is below 2^108 (a number whose sum leaves it is NaN).
 * A row that sees nothing (an empty slot, a skipped row, a list without blocks): zeros in out, -inf in lse.  A K that is NaN makes the rows that see it NaN, a V
 * the channel of those rows; what a row does not see never reaches it.  A page outside the pool among those that it takes: NaN in the sequence's rows, or the list's.
 */
PYR_API int pyr_cache8_attention_workspace_bytes(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                                         int32_t n_blocks, size_t* bytes_out);
PYR_API int pyr_cache8_attention(const pyr_cache8* cache, const void* q, const int32_t* slots, int32_t n, int32_t n_tokens, int32_t n_q_heads,
                         int32_t max_len, float softmax_scale, const int32_t* blocks, int32_t n_blocks, void* out, float* lse,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * Diagnostic for the benchmark report, not part of the method: a launch of nothing but bf16 MFMAs
 * (v_mfma_f32_32x32x16_bf16 back to back, two wavefronts per SIMD, every compute unit), so that the
 * rate this very GPU sustains can be printed beside the published peak.
 *   iters              loop trips per wavefront (16 MFMAs each)
 *   sink_dev           dev, one float (never written in practice)
 *   flops_out          host, written: floating-point operations of the launch
 */
PYR_API int pyr_diag_mfma_only(int32_t iters, float* sink_dev, void* stream, double* flops_out);

/*
 * Diagnostic for the benchmark report, not part of the method: a launch that only reads `bytes` of device
 * memory with LDS-direct loads, as the score pass reads K (16 KB tiles here, one in flight per wavefront, six
 * wavefronts per compute unit) and discards them, so that the read rate this very GPU sustains can be printed
 * beside the published HBM peak.
 *   data_dev           dev, `bytes` readable bytes, 16-byte aligned
 *   bytes              a positive multiple of 524288, below 2^50
 *   k_layout           0: consecutive tiles; != 0: tiles of 64 rows x 256 bytes, rows 8192 bytes apart (one head of
 *                      64 tokens of a [T, 32, 128] bf16 K)
 *   sink_dev           dev, one int32 (never written in practice)
 * Errors: PYR_ERR_NULL, PYR_ERR_SHAPE (bytes), PYR_ERR_LAUNCH.
 */
PYR_API int pyr_diag_read_stream(const void* data_dev, size_t bytes, int32_t k_layout, int32_t* sink_dev, void* stream);

/*
 * Diagnostic, not part of the method: which kernels and which cut of the work the entry points above take for a batch,
 * so that a test can assert that it reaches the path it is written for.  Host only; launches nothing.
 *   compute_units, xcds  of the device to answer for; both 0: the current device
 *   route_out            host, written:
 */
typedef struct pyr_route {
    int32_t attention;          /* 0: lists of 256-row tiles; 1, 2: one 128-row tile per workgroup, keys in one or two groups */
    int32_t attention_items;    /* attention == 0: most items (pairs of tiles) in one workgroup's list, else 0 */
    int32_t attention_listed;   /* attention != 0: 1 if the grid is a list of the tiles that exist, else 0 */
    int32_t score_tiles, score_waves, score_groups;     /* prefill score pass: 32-key tiles of a range, wavefronts, split */
    int32_t score_order;        /* 0: a sequence per XCD, 1: equally many ranges, 2: counted, 3: places for the longest sequence */
    int32_t stats_tiles, stats_waves, stats_groups;     /* the same of the generation phase's statistics (all 0: one pass does both) ... */
    int32_t window_tiles, window_waves, window_groups;  /* ... and of its score pass (or of the one pass: tiles per wavefront) */
} pyr_route;
PYR_API int pyr_diag_route(const pyr_shape* shape, const int32_t* seq_offsets_host, int32_t w, int32_t compute_units,
                           int32_t xcds, pyr_route* route_out);

/*
 * Diagnostic, not part of the method: what pyr_diag_route leaves out, for the same purpose.  Host only; launches nothing.
 *   generation         0: of pyr_prefill_layer_fused, else of pyr_decode_update
 *   keep_len_host      as in those; NULL: the selection and the gather are left out
 *   row_bytes          bytes gathered per kept row from all sources together, position ids aside (K and V: 2 * n_kv_heads * head_dim * 2)
 *   compute_units, xcds  as in pyr_diag_route
 *   launches_out       host, written
 */
typedef struct pyr_launches {
    int32_t attention_chunk;    /* one 128-row tile per workgroup, not listed: KV heads of a sequence that an XCD works on at a time ... */
    int32_t attention_units;    /* ... of so many that it has; else both 0 */
    int32_t stats_order, window_order;  /* generation phase, two walks: score_order of the statistics and of the score pass; else -1 */
    int32_t sums;               /* 1: rows of partial sums are added by a launch of their own */
    int32_t select_split;       /* selection and gather in one launch: workgroups per sequence; in two: 0 */
} pyr_launches;
PYR_API int pyr_diag_launches(const pyr_shape* shape, const int32_t* seq_offsets_host, int32_t w, int32_t generation,
                              const int32_t* keep_len_host, int64_t row_bytes, int32_t compute_units, int32_t xcds,
                              pyr_launches* launches_out);

/*
 * Diagnostic, not part of the method: whether pyr_prefill_layer_fused takes a batch's attention and scores in one launch.  Host only; launches nothing.
 *   compute_units, xcds  as in pyr_diag_route
 *   groups_out           host, written: rows of partial scores of that launch; 0: attention and scores have a launch each
 */
PYR_API int pyr_diag_layer(const pyr_shape* shape, const int32_t* seq_offsets_host, int32_t w, int32_t compute_units, int32_t xcds,
                           int32_t* groups_out);

/*
 * Diagnostic, not part of the method: in which order the one walk of pyr_decode_update takes its tasks (a row block of a query head each).  Host
 * only; launches nothing.
 *   compute_units, xcds  as in pyr_diag_route
 *   order_out            host, written: 0 query head after query head, 1 in turn over the KV heads; -1: a batch of two walks, or without tokens
 */
PYR_API int pyr_diag_update(const pyr_shape* shape, const int32_t* seq_offsets_host, int32_t w, int32_t compute_units, int32_t xcds,
                            int32_t* order_out);

/*
 * Diagnostic, not part of the method: how pyr_cache_attention cuts up a call, so that a test can assert that it reaches the path it is written for.
 * Host only; launches nothing.
 *   route_out          host, written:
 */
typedef struct pyr_cache_route {
    int32_t col_tiles;          /* 16-row tiles of query rows in a workgroup ...                                     */
    int32_t repeats;            /* ... and how many times the rows stand in one                                      */
    int32_t waves;              /* wavefronts of a workgroup                                                         */
    int32_t col_groups;         /* workgroups per KV head and split                                                  */
    int32_t chunk, splits;      /* 32-token tiles of a split; splits along the cache: more than one take a second launch */
} pyr_cache_route;
PYR_API int pyr_diag_cache_attention(const pyr_cache* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len,
                                     pyr_cache_route* route_out);

/* The same of pyr_cache8_attention (repeats: always 1). */
PYR_API int pyr_diag_cache8_attention(const pyr_cache8* cache, int32_t n, int32_t n_tokens, int32_t n_q_heads, int32_t max_len, int32_t n_blocks,
                                      pyr_cache_route* route_out);

#ifdef __cplusplus
}
#endif
#endif /* PYR_H */
