/*
 * climber.h -- C ABI of the MI355X-native Climber serving hot path.
 *
 * The library implements the serving flow of Climber (arXiv 2502.09888, Sec. 3.2
 * "Deployment"): a user's behaviour history is encoded once, its per-layer keys
 * and values are kept in a cache in device memory, and M candidate items are then
 * scored in one batch ("single user, multiple items"): every candidate attends to
 * the whole cached history plus itself and never to another candidate.  The
 * attention is the Adaptive Transformer Layer of Sec. 3.1.3, Eq. (3): logits
 * R = qk_scale * Q K^T are divided by a temperature looked up per query row from a
 * (scenario, behaviour) table before the softmax.  History tokens only attend
 * inside their own subsequence (multi-scale sequence extraction, Sec. 3.1.2), i.e.
 * block-diagonal attention over equal subsequences of `sub_len` tokens.
 *
 * General rules
 *  - Every function returns 0 (CLIMBER_OK) or a negative CLIMBER_ERR_* code;
 *    climber_strerror() names it.  No exceptions, no output on stderr.
 *  - "dev" pointers are device (HBM) addresses owned by the caller; the library
 *    never allocates, frees or keeps them beyond what is documented for the KV
 *    cache handle.  "host" pointers are ordinary host memory, read during the call.
 *  - All device work is enqueued on the caller's stream (`stream` is a hipStream_t
 *    passed as void*; NULL is the default stream).  Compute calls do not
 *    synchronise; they return after the launches are enqueued.
 *  - Arguments are validated on the host before anything is launched; a failed
 *    call has launched nothing.  Device-resident ids cannot be checked on the
 *    host: scenario / behaviour ids outside the table are clamped into range by
 *    the kernels (results for such rows are then those of the clamped id).
 *    Temperatures must be finite and > 0; this is the caller's contract (a
 *    non-positive entry gives unspecified values for the rows that use it, never
 *    an out-of-bounds access).  climber_check_inputs() checks both on the device
 *    and reports into a caller-owned status word.
 *  - Packed batches: the histories of the B users of a batch are stored back to
 *    back with per-user padded lengths; user b owns rows
 *    tok_off[b] .. tok_off[b] + hist_len_padded[b] - 1 of every per-token array,
 *    of which the first hist_len[b] are valid.  Padded rows are never read as
 *    keys/values (they may hold anything, NaN included) and produce zeros as
 *    query rows.  Candidates are packed with device offsets cand_off[B+1].
 *  - An array of zero length may be passed as NULL: with m_total == 0 the per-candidate pointers
 *    (rows, ids, outputs) are not looked at and nothing is launched for the candidates.
 *  - Activations are token-major: q/k/v are [rows][n_heads][d_head], attention
 *    outputs and hidden states are [rows][d_model], d_model = n_heads * d_head.
 *
 * Precision paths
 *  - CLIMBER_F32 : everything fp32 (reference path; any d_head <= 256).
 *  - CLIMBER_BF16: bf16 storage, bf16 MFMA products with fp32 accumulation, fp32
 *    softmax statistics, probabilities rounded to bf16 before the P V product;
 *    requires d_head == 64, padded history lengths that are multiples of 64 and
 *    sub_len == 0 or a multiple of 128.
 *    A candidate's result does not depend on which other candidates are scored with it (the
 *    mask of Sec. 3.2); on this path it is bitwise the same however the candidates are chunked or
 *    ordered as long as its logits are of ordinary size.  With large logits the kernel picks the
 *    form of its softmax (scale folded into the query / applied in fp32 / running maximum) per
 *    wavefront or workgroup from the rows it holds, so a candidate's rounding can then differ
 *    with its neighbours in the tile; every form is within the path's tolerance.
 */
#ifndef CLIMBER_H
#define CLIMBER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define CLIMBER_OK 0
#define CLIMBER_ERR_NULL (-1)        /* a required pointer is NULL */
#define CLIMBER_ERR_SHAPE (-2)       /* a size is <= 0 or inconsistent (d_model != H*d_head ...) */
#define CLIMBER_ERR_ALIGN (-3)       /* padding / multiple-of / pointer alignment rule violated */
#define CLIMBER_ERR_RANGE (-4)       /* layer index, length or offset out of range */
#define CLIMBER_ERR_TAU (-5)         /* qk_scale / rms_eps not finite or not positive */
#define CLIMBER_ERR_BUFSIZE (-6)     /* caller buffer (cache, workspace) too small */
#define CLIMBER_ERR_UNSUPPORTED (-7) /* valid request the selected precision path cannot run */
#define CLIMBER_ERR_RUNTIME (-8)     /* a HIP runtime call failed (no device, bad stream ...) */

#define CLIMBER_F32 0
#define CLIMBER_BF16 1

#define CLIMBER_HIST_CAUSAL 1 /* flags bit 0: history token i only sees j <= i of its subsequence */
/* Path selection, results equal to within rounding.  The bf16 history pass has two routes: one launch that stores the
 * cache blocks and attends, where it is the faster way and the outputs allow it (default), or cache writer + attention
 * from the cache. */
#define CLIMBER_HIST_TWO_KERNEL 2 /* flags bit 1: always take the cache writer + attention route */
/* The stack's fused QKV projection writes history keys / values into the cache from its epilogue
 * (default), or stores them as rows that the history pass then copies into the cache. */
#define CLIMBER_QKV_VIA_ROWS 4    /* flags bit 2: keys / values go through rows */

#define CLIMBER_MODE_HISTORY 0
#define CLIMBER_MODE_CANDIDATE 1

/* Hyper-parameters.  Plain data, passed by pointer, copied where kept. */
typedef struct climber_config {
    int32_t n_layers; /* layers of the stack (>= 1); attention-only use: number of cache layers */
    int32_t d_model;  /* = n_heads * d_head */
    int32_t n_heads;
    int32_t d_head;
    int32_t d_ffn;    /* feed-forward hidden width; ignored by the attention-only calls */
    int32_t n_scen;   /* temperature table rows (scenarios) */
    int32_t n_beh;    /* temperature table columns (behaviours / extraction strategies) */
    int32_t sub_len;  /* subsequence length n_k of Sec. 3.1.2; 0 = one subsequence */
    int32_t dtype;    /* CLIMBER_F32 | CLIMBER_BF16 */
    int32_t flags;    /* CLIMBER_HIST_CAUSAL | CLIMBER_HIST_TWO_KERNEL | CLIMBER_QKV_VIA_ROWS */
    float qk_scale;   /* multiplies Q K^T before the temperature divide; Eq. (3) literally = 1 */
    float rms_eps;    /* epsilon of the RMSNorm in the layer stack */
} climber_config;

/* One layer's weights: device pointers, row-major, element type = config dtype (bf16 / fp32).
 *   g1 [d]   gain of the pre-attention RMSNorm      wqkv [d][3d]  columns Q heads | K heads | V heads
 *   wo [d][d]                                       g2 [d]   gain of the pre-FFN RMSNorm
 *   w1 [d][d_ffn]                                   w2 [d_ffn][d]
 * Layer (f_QKV and f_FFN of Eq. (3) made concrete; the paper does not fix these details):
 *   qkv = RMSNorm(x; g1) wqkv;  o = attention;  h = x + o wo;  y = h + GELU_erf(RMSNorm(h; g2) w1) w2 */
typedef struct climber_layer_weights {
    const void *g1, *wqkv, *wo, *g2, *w1, *w2;
} climber_layer_weights;

typedef struct climber_weights {
    int32_t n_layers;                    /* must equal config.n_layers */
    const climber_layer_weights *layers; /* host array of n_layers entries */
    const void *packed;                  /* dev, or NULL.  The buffer climber_pack_weights filled from
                                            these weights: climber_history_encode / climber_sumi_score
                                            then read it (and never `layers`, which may be NULL)
                                            instead of repacking the weights on every call. */
} climber_weights;

/* Opaque host-side handle describing a KV cache that lives in a caller-owned device buffer. */
typedef struct climber_kv_cache climber_kv_cache;

const char *climber_strerror(int code);

/* ---- KV cache (Sec. 3.2: "multi-layered key-value cache vectors from user features") ----------
 * The cache holds, for each of config.n_layers layers, the keys and values of every (padded)
 * history token of the batch, in a layout private to the library (for bf16: MFMA operand
 * fragments of 32-key blocks, so that the candidate pass streams it with linear 16-byte
 * accesses; padded slots are stored as zeros).  It is immutable between encodes, so any
 * number of scoring calls, on any streams, may read it concurrently.
 */

/* Bytes the device buffer of a cache must have.  hist_len_padded: host [B].  Returns 0 on any
 * invalid argument. */
size_t climber_kv_cache_bytes(const climber_config *cfg, int32_t B, const int32_t *hist_len_padded);

/* Create the handle.  hist_len, hist_len_padded: host [B], copied.  dev_buf: dev, `bytes` long,
 * 256-byte aligned, owned by the caller and must outlive the handle's use.  A small descriptor
 * (lengths, offsets, schedule) is copied into the head of dev_buf with a synchronous copy; this
 * is the only call of the library that synchronises.  0 <= hist_len[b] <= hist_len_padded[b];
 * B >= 1; sum of padded lengths < 2^31 / d_model.
 * Errors: NULL, SHAPE, ALIGN (padding rule of the dtype), RANGE, BUFSIZE, UNSUPPORTED, RUNTIME. */
int climber_kv_cache_create(const climber_config *cfg, int32_t B, const int32_t *hist_len,
                            const int32_t *hist_len_padded, void *dev_buf, size_t bytes,
                            climber_kv_cache **out);

/* Frees the host handle only; the device buffer stays with the caller.  NULL is accepted. */
int climber_kv_cache_destroy(climber_kv_cache *cache);

/* Total padded history rows of the batch (= tok_off[B]); negative error code on NULL. */
int64_t climber_kv_cache_rows(const climber_kv_cache *cache);

/* ---- attention-only entry points (caller supplies Q/K/V of one layer) ------------------------- */

/* History side of one layer (Eq. (3) restricted to a subsequence, Sec. 3.1.2):
 *  1. stores k, v of all history tokens into cache layer `layer`;
 *  2. if o_hist != NULL, block-diagonal attention of the history tokens:
 *       o_i = sum_j softmax_j( qk_scale <q_i,k_j> / tau[scen_i][beh_i] ) v_j
 *     over the valid tokens j of i's subsequence (j <= i as well under CLIMBER_HIST_CAUSAL).
 * tau_layer: dev [n_scen][n_beh] fp32.  q (may be NULL iff o_hist is NULL), k, v: dev
 * [rows][H][d_head] of the config dtype, rows = climber_kv_cache_rows().  scen, beh: dev int32
 * [rows] (only read when o_hist != NULL).  o_hist: dev [rows][d_model] of the config dtype;
 * padded rows receive zeros. */
int climber_attn_history(const climber_config *cfg, const float *tau_layer, const void *q,
                         const void *k, const void *v, const int32_t *scen, const int32_t *beh,
                         climber_kv_cache *cache, int32_t layer, void *o_hist, void *stream);

/* SUMI attention of one layer (mask of Sec. 3.2, temperature of Eq. (3)): for candidate c of
 * user b
 *     o_c = softmax over { all hist_len[b] cached history keys of b, c's own key } of
 *           qk_scale <q_c, k> / tau[cscen_c][cbeh_c],   applied to the matching values.
 * q_c, k_c, v_c: dev [m_total][H][d_head]; cand_off: dev int32 [B+1], cand_off[0] = 0,
 * non-decreasing, cand_off[B] = m_total; m_max: host value, must be >= max_b (cand_off[b+1] -
 * cand_off[b]): it sizes the launch, and m_max * B == m_total tells the library that every user
 * has exactly m_max candidates.  A smaller m_max breaks the contract (rows may then be left
 * unwritten or scored against the wrong user's history, never an out-of-bounds access);
 * climber_check_inputs reports it.
 * cand_scen, cand_beh: dev int32 [m_total].  o_c: dev [m_total][d_model].
 * Scoring a candidate set in chunks = calling this repeatedly on the same (const) cache. */
int climber_attn_sumi(const climber_config *cfg, const float *tau_layer,
                      const climber_kv_cache *cache, int32_t layer, const void *q_c,
                      const void *k_c, const void *v_c, const int32_t *cand_off, int32_t m_total,
                      int32_t m_max, const int32_t *cand_scen, const int32_t *cand_beh, void *o_c,
                      void *stream);

/* ---- relative attention bias (Eq. (3): R = Q K^T + f_b, divided by the temperature) -----------
 * Sec. 3.1.3 names what the bias depends on (relative position and relative time, per extraction
 * strategy and scenario) and not its form.  The form of this library:
 *     bias(i, j; h) = pos_table[scen_i][beh_i][h][bp(pos_i - pos_j)]
 *                   + time_table[scen_i][beh_i][h][bt(ts_i - ts_j)]
 *     bp(d) = clip(d, -(n_pos-1)/2, (n_pos-1)/2) + (n_pos-1)/2          (n_pos odd, >= 1)
 *     bt(d) = min( floor(log2(max(|d|, 1))), n_time - 1 )               (n_time >= 1)
 * i = query row (its scenario / behaviour ids select the table row, as they select its temperature),
 * j = key; pos / ts are caller-defined integers per history row and per candidate (e.g. index in the
 * history and seconds); a candidate's own key has distance 0 in both.  The bias is added to
 * qk_scale <q_i, k_j> and the sum is divided by the row's temperature.
 * All pointers dev; tables fp32 (both precision paths); hist_pos / hist_ts: int32 [rows], 16-byte
 * aligned, padded rows may hold anything; cand_pos / cand_ts: int32 [m_total]. */
typedef struct climber_rel_bias {
    const float *pos_table;  /* [n_scen][n_beh][n_heads][n_pos] */
    const float *time_table; /* [n_scen][n_beh][n_heads][n_time] */
    int32_t n_pos, n_time;
    const int32_t *hist_pos, *hist_ts;
    const int32_t *cand_pos, *cand_ts; /* only read by climber_attn_sumi_bias */
} climber_rel_bias;

/* climber_attn_history / climber_attn_sumi with the bias term (bias != NULL; everything else as
 * documented there).
 * Additional errors: CLIMBER_ERR_NULL (bias or a pointer it needs), _SHAPE (n_pos even or < 1,
 * n_time < 1), _ALIGN (hist_pos / hist_ts). */
int climber_attn_history_bias(const climber_config *cfg, const float *tau_layer, const void *q,
                              const void *k, const void *v, const int32_t *scen, const int32_t *beh,
                              climber_kv_cache *cache, int32_t layer, void *o_hist,
                              const climber_rel_bias *bias, void *stream);
int climber_attn_sumi_bias(const climber_config *cfg, const float *tau_layer,
                           const climber_kv_cache *cache, int32_t layer, const void *q_c,
                           const void *k_c, const void *v_c, const int32_t *cand_off,
                           int32_t m_total, int32_t m_max, const int32_t *cand_scen,
                           const int32_t *cand_beh, void *o_c, const climber_rel_bias *bias,
                           void *stream);

/* ---- paged history cache ----------------------------------------------------------------------
 * climber_kv_cache holds histories that are encoded once.  A history that grows -- a behaviour, a
 * session at a time -- or that is too long to keep whole lives in pages instead: one layer's keys and
 * values in a pool of pages, and for every sequence (user) the list of its pages.  Three calls work on it:
 *   climber_attn_history_paged  stores a chunk of new behaviours per sequence and attends from them
 *   climber_attn_sumi_paged     candidates against the stored history (the mask of Sec. 3.2)
 *   climber_paged_evict         cuts every sequence to a budget, the tokens with the least weight first
 * All memory belongs to the caller; there is no handle, and a layout that the caller may read and write:
 *   k, v        dev [n_pages][n_kv_heads][page_size][d_head], config dtype, 16-byte aligned
 *   page_table  dev int32 [n_seqs][table_ld]: token `slot` of sequence b is row slot % page_size of page
 *               page_table[b][slot / page_size].  Entries behind the pages in use may hold anything.
 *   len         dev int32 [n_seqs]: tokens in the cache before the call.  No call but climber_paged_evict
 *               and climber_pages_fork changes a length: after an append the caller adds the chunk's rows.
 *   max_len     host: no sequence has more tokens than this after the call.  It sizes the launches (a
 *               HIP graph keeps working while lengths grow up to it) and is at most table_ld * page_size.
 *   mass        dev fp32 [n_pages][page_size] or NULL: accumulated attention weight per token.  Where it is
 *               not NULL, both attention calls add to a token's entry its softmax weights in all of the call's
 *               rows and heads (not a candidate's weight on itself); an appended token starts from 0.  Sums are
 *               made in fp32 in an order that only depends on the sizes of the call.  Two calls that add to
 *               the same tokens must not overlap, and no two sequences of a call may list the same page then.
 *   stamp       dev int32 [n_pages][page_size] or NULL: a number of the caller's per token (its time, its
 *               position), stored by climber_attn_history_paged and kept with its token by climber_paged_evict.
 *   d_head, elem_bytes  host: elements of a head's key or value in the pages, and bytes of one.  A call whose cfg has others is refused
 *               (CLIMBER_ERR_SHAPE): it would read and write beyond the pool.  0: not stated, and not checked.
 * page_size: a power of two, 16 .. 4096.  n_kv_heads divides cfg->n_heads: query head h reads cache head
 * h / (n_heads / n_kv_heads).  CLIMBER_BF16: d_head 64 or 128; CLIMBER_F32: d_head <= 128, a multiple of 4.
 * A page may be listed by several sequences (a shared prefix) as long as no call writes into it: an append
 * writes the pages of slots len[b] .. len[b] + rows - 1, an eviction those of slots below the budget, and with
 * mass every call its entries of all tokens.
 * Contents of slots from len[b] on are never used: they may hold anything, NaN included.
 * Lengths, offsets and page numbers are device memory and cannot be checked on the host: lengths are clamped to
 * max_len, offsets to m_total, page numbers that are read to the pool, and a token whose page number lies outside the
 * pool is not stored.  Nor are new tokens from slot max_len on: no row sees them, theirs attend to what the cache then holds, and cached tokens
 * stay.  climber_check_paged reports such values.
 * Values are added up before they are divided by the sum of their weights: |v| times the tokens that a row sees has to stay below
 * 2^119, or outputs may be infinite.  Logits (qk_scale <q, k> / tau) have to stay below 10^7 in magnitude, where a step of fp32 is 1, or
 * rows may be no numbers; <q, k> itself may be any finite fp32 number.
 * A workspace belongs to one call at a time: two calls, or two captured graphs, that may run at once need one each.
 * Rows (q, k, v, o): row r starts r * ld elements behind the pointer and holds its heads one after the other;
 * pointers and row pitches are multiples of 16 bytes; o must not share an element with q, k or v.  Rows of no
 * sequence (behind off[n_seqs]) stay as they are. */
typedef struct climber_paged_kv {
    void *k, *v;
    float *mass;
    int32_t *stamp;
    const int32_t *page_table, *len;
    int32_t n_pages, page_size, n_kv_heads, n_seqs, table_ld, max_len;
    int32_t d_head, elem_bytes;
} climber_paged_kv;

/* Bytes of scratch that any call on this cache needs for up to m_total rows, at most m_max per sequence (0, 0: eviction only).
 * Reads the sizes, and whether mass is NULL.  0 on an invalid argument. */
size_t climber_paged_workspace_bytes(const climber_config *cfg, const climber_paged_kv *kv, int32_t m_total, int32_t m_max);

/* A chunk of new behaviours.  off: dev int32 [n_seqs + 1], rows off[b] .. off[b + 1] - 1 are sequence b's next tokens (m_total, m_max
 * as in climber_attn_sumi; a sequence may have none).  Their k, v (and stamp: dev int32 [m_total], needed if kv->stamp) are stored as
 * slots len[b] + i, and
 *     o_i = softmax over { cached tokens of b, new tokens j <= i of b } of qk_scale <q_i, k_j> / tau[scen_i][beh_i], applied to v
 * (CLIMBER_HIST_CAUSAL; without it, all new tokens of b).  With len = 0 this is the attention of whole histories.  A token that a row
 * does not see has no influence on it, whatever it holds.  cfg->sub_len must be 0: a sequence is one subsequence.
 * q, o: [m_total][ld] of n_heads * d_head; k, v: [m_total][ld_kv] of n_kv_heads * d_head.
 * Errors: CLIMBER_ERR_NULL, _SHAPE, _ALIGN, _RANGE, _TAU, _BUFSIZE, _UNSUPPORTED (d_head, sub_len, o on q, k or v), _RUNTIME. */
int climber_attn_history_paged(const climber_config *cfg, const float *tau_layer, const climber_paged_kv *kv, const void *q,
                               int64_t ld_q, const void *k, const void *v, int64_t ld_kv, const int32_t *off, int32_t m_total,
                               int32_t m_max, const int32_t *scen, const int32_t *beh, const int32_t *stamp, void *o,
                               int64_t ld_o, void *workspace, size_t ws_bytes, void *stream);

/* Candidates: climber_attn_sumi over the paged history.  Every candidate sees all cached tokens of its sequence and itself; nothing
 * is stored.  cfg->sub_len and CLIMBER_HIST_CAUSAL do not concern it.  Errors as above. */
int climber_attn_sumi_paged(const climber_config *cfg, const float *tau_layer, const climber_paged_kv *kv, const void *q_c,
                            int64_t ld_q, const void *k_c, const void *v_c, int64_t ld_kv, const int32_t *cand_off,
                            int32_t m_total, int32_t m_max, const int32_t *cand_scen, const int32_t *cand_beh, void *o_c,
                            int64_t ld_o, void *workspace, size_t ws_bytes, void *stream);

/* Sequence b keeps min(budget[b], len[b]) tokens (budget: dev int32 [n_seqs]; below 0 counts as 0).  Tokens rank by
 *     stamp >= keep_from[b] before all others (keep_from: dev int32 [n_seqs], or NULL: no such rule; needs kv->stamp),
 *     then rank descending (rank: dev fp32 laid out as kv->mass, or NULL: kv->mass; NaN ranks below everything),
 *     then slot ascending.
 * The cache of a sequence is a set: kept tokens of slots below the new length stay where they are, and the places of evicted tokens
 * among them are filled, in ascending order, with the kept tokens of the slots behind.  k, v, and mass and stamp where they are
 * not NULL, move with their token; `rank` is only read.  Slots from the new length on keep what they held.
 * len_out: dev int32 [n_seqs], the new lengths (may be kv->len, or budget).  src: dev int32 [n_seqs][table_ld * page_size] or NULL: for each slot below
 * the new length the slot that its token had before, -1 from there on.  A caller with more data per token moves it by src.
 * Errors: CLIMBER_ERR_NULL, _SHAPE, _ALIGN, _RANGE, _BUFSIZE, _UNSUPPORTED (d_head; max_len over 2^22), _RUNTIME. */
int climber_paged_evict(const climber_config *cfg, const climber_paged_kv *kv, const float *rank, const int32_t *budget,
                        const int32_t *keep_from, int32_t *len_out, int32_t *src, void *workspace, size_t ws_bytes, void *stream);

/* climber_check_inputs for a paged cache: one small kernel that reads page_table, len and, if not NULL, off against the rules
 * above for a call of m_total rows that stores them (appends != 0) or does not, and ORs CLIMBER_BAD_* bits into *status.  Offsets
 * that end before m_total are in order: the rows behind belong to no sequence. */
#define CLIMBER_BAD_PAGE 32 /* a page number of a token outside [0, n_pages) */
#define CLIMBER_BAD_LEN 64  /* a length below 0, or over max_len after the call */
int climber_check_paged(const climber_config *cfg, const climber_paged_kv *kv, const int32_t *off, int32_t m_total, int32_t m_max,
                        int32_t appends, int32_t *status, void *stream);

/* ---- paged history cache in 8 bits --------------------------------------------------------------
 * The same cache at half the memory and half the traffic: keys and values are held as e4m3 numbers (4 exponent bits, 3 mantissa bits,
 * largest 448) with a power of two for each block of 16 tokens and cache head:
 *   kv.k, kv.v        dev [n_pages][n_kv_heads][page_size][d_head], one byte each (kv.elem_bytes 1, or 0: not stated), 16-byte aligned
 *   k_scale, v_scale  dev [n_pages][n_kv_heads][page_size / 16], one byte s each: the block's elements stand for e4m3 * 2^(s - 127)
 * and everything else as in climber_paged_kv.  CLIMBER_BF16 with d_head 64 or 128 (rows of a call are bf16); kv.mass must be NULL.
 * A block's scale is the least s >= 10 with which every finite element of its tokens is at most 448 * 2^(s - 127) in magnitude; elements
 * are rounded to the nearest e4m3 number, ties to even, and infinities and NaN become NaN.  A token that joins a block raises the scale
 * where it has to: the block's older elements are then rounded once more.  A scale never falls while its block has tokens (where some of them were cut
 * off, or copied without the others, it stays as well); the first token of a block (slot a multiple of 16) starts it anew.  Elements of keys and values have to stay below 2^127 in magnitude, and scales that the caller
 * writes between 10 and 247.
 * Two sequences of a call may list the same page as long as no call writes it; the append writes to the blocks of slots len[b] .. len[b] + rows - 1
 * whole, the older tokens of the first one among them.  Eviction does not take this cache; climber_check_paged takes &kv8->kv. */
typedef struct climber_paged_kv8 {
    climber_paged_kv kv;
    uint8_t *k_scale, *v_scale;
} climber_paged_kv8;

/* Bytes of scratch for up to m_total rows, at most m_max per sequence.  0 on an invalid argument. */
size_t climber_paged8_workspace_bytes(const climber_config *cfg, const climber_paged_kv8 *kv8, int32_t m_total, int32_t m_max);

/* climber_attn_history_paged: cached tokens as the cache holds them before the call, the chunk's own as they are brought; then the
 * chunk is rounded and stored.  Errors as there (_UNSUPPORTED also: not CLIMBER_BF16, mass). */
int climber_attn_history_paged8(const climber_config *cfg, const float *tau_layer, const climber_paged_kv8 *kv8, const void *q,
                                int64_t ld_q, const void *k, const void *v, int64_t ld_kv, const int32_t *off, int32_t m_total,
                                int32_t m_max, const int32_t *scen, const int32_t *beh, const int32_t *stamp, void *o,
                                int64_t ld_o, void *workspace, size_t ws_bytes, void *stream);

/* climber_attn_sumi_paged over the cache in 8 bits. */
int climber_attn_sumi_paged8(const climber_config *cfg, const float *tau_layer, const climber_paged_kv8 *kv8, const void *q_c,
                             int64_t ld_q, const void *k_c, const void *v_c, int64_t ld_kv, const int32_t *cand_off,
                             int32_t m_total, int32_t m_max, const int32_t *cand_scen, const int32_t *cand_beh, void *o_c,
                             int64_t ld_o, void *workspace, size_t ws_bytes, void *stream);

/* ---- pages -------------------------------------------------------------------------------------
 * Who holds which pages of a paged cache.  One pool of page numbers serves any number of caches of the same page_size (the layers of a
 * stack): the three calls below change the page table, and climber_paged_copy / climber_paged8_copy then do what has to be done in each cache.
 *   refs        dev int32 [n_pages]: how many entries of the table hold a page, and whatever else the caller counts (a prefix that is
 *               to stay adds 1); 0: the page is free
 *   page_table  dev int32 [n_seqs][table_ld], as a climber_paged_kv's
 *   held        dev int32 [n_seqs]: pages that a sequence holds, its row's first entries
 *   len         dev int32 [n_seqs]: its tokens, as a climber_paged_kv's: at most held * page_size
 * Empty: all zeros.  page_size, and the limits of the sizes, as in climber_paged_kv; n_seqs * table_ld below 2^31, n_seqs below 2^24.
 * A cache whose pages are shared has no mass (see climber_paged_kv), and eviction writes pages: of a sequence that shares none.
 * Results do not depend on the order in which the device works.  Values are device memory and cannot be checked on the host: whatever
 * they hold, nothing is read or written outside the arrays, and calls OR what they find into *status (dev int32, not cleared):
 *   CLIMBER_BAD_PAGE  a page number that is held lies outside the pool (fork: one that a row takes or gives up; extend: one that new tokens go into;
 *                     compact: any), or, compact, is of a page with refs 0: it counts as free, and a page may have been moved into it
 *   CLIMBER_BAD_SEQ   fork: a parent from n_seqs on (the row stays as it is)
 *   CLIMBER_POOL_FULL extend: not enough free pages, or more than a row of the table has room for
 * A workspace belongs to one call at a time, and so does a pool.  workspace: climber_pages_workspace_bytes(), 256-byte aligned.
 * Errors: CLIMBER_ERR_NULL, _SHAPE, _ALIGN, _RANGE, _BUFSIZE, _RUNTIME. */
#define CLIMBER_POOL_FULL 128
#define CLIMBER_BAD_SEQ 256
typedef struct climber_page_pool {
    int32_t *refs, *page_table, *held, *len;
    int32_t n_pages, page_size, n_seqs, table_ld;
} climber_page_pool;

size_t climber_pages_workspace_bytes(const climber_page_pool *pool); /* 0 on an invalid argument */

/* All rows at once: sequence b becomes what sequence parent[b] was before the call, up to its first keep[b] tokens (parent, keep: dev int32
 * [n_seqs]; keep NULL: all of them; below 0 counts as 0).  parent[b] = b with keep NULL: the row stays as it is, with the pages
 * that it holds beyond its tokens.  parent[b] < 0: the sequence becomes empty.  Otherwise the pages that hold the tokens are shared
 * (held: as many), what the row held before is given up, and entries of it that are held no more become -1.  Branches of a history, beams that take
 * each other's place, a shared prefix, tokens taken back, users that leave are each one call; after an eviction one with parent[b] = b and keep = len gives
 * the pages back that hold no token any more. */
int climber_pages_fork(const climber_page_pool *pool, const int32_t *parent, const int32_t *keep, int32_t *status, void *workspace,
                       size_t ws_bytes, void *stream);

/* Room for rows[b] more tokens of each sequence (dev int32 [n_seqs]; below 1: none), to be called before the append: then the pages of slots
 * len[b] .. len[b] + rows[b] - 1 are held, and by nobody else.  Free pages are handed out in ascending order, to the sequences
 * in ascending order: first in the places of shared pages that the new tokens go into, then for new ones.  A shared page that all who hold
 * it write to in this call (as many sequences as its refs) stays with the last of them.  Where a page was replaced and holds tokens of
 * the sequence, copies gets (page, its replacement, tokens).  A call that cannot be served whole (CLIMBER_POOL_FULL, CLIMBER_BAD_PAGE) changes nothing.
 * copies: dev int32 [n_seqs][3]; counts: dev int32 [2]: how many of them there are (those behind stay as they are), and pages in use after the call.
 * A page that was given up may be handed out again by the next extend: copy before it. */
int climber_pages_extend(const climber_page_pool *pool, const int32_t *rows, int32_t *copies, int32_t *counts, int32_t *status,
                         void *workspace, size_t ws_bytes, void *stream);

/* Moves pages so that the pages in use are 0 .. counts[1] - 1: those behind go, in ascending order, to the free ones before.  Table and refs
 * follow; copies (dev int32 [n_pages / 2][3]; a pool of one page needs none, and takes NULL) gets (old number, new number, page_size) of each,
 * counts[0] of them. */
int climber_pages_compact(const climber_page_pool *pool, int32_t *copies, int32_t *counts, int32_t *status, void *workspace,
                          size_t ws_bytes, void *stream);

/* In a cache: the first copies[i][2] tokens of page copies[i][0] to page copies[i][1], i < min(counts[0], max_copies): keys, values, and
 * mass, stamp and scales where there are any.  max_copies (host) sizes the launch.  No page may be both read and written, or written twice.
 * Pages outside the pool are left out.  Errors: CLIMBER_ERR_NULL, _SHAPE, _ALIGN, _RANGE, _TAU, _UNSUPPORTED, _RUNTIME. */
int climber_paged_copy(const climber_config *cfg, const climber_paged_kv *kv, const int32_t *copies, const int32_t *counts,
                       int32_t max_copies, void *stream);
int climber_paged8_copy(const climber_config *cfg, const climber_paged_kv8 *kv8, const int32_t *copies, const int32_t *counts,
                        int32_t max_copies, void *stream);

/* ---- rotary positions ---------------------------------------------------------------------------
 * Query and key rows are turned by their positions before they are appended or scored: the products of a query and a key, and with them
 * the logits of Eq. (3), then depend on the distance of the two.  Pair i of a head's first rot_dims elements, (a, b), becomes
 *     scale * (a cos t - b sin t, a sin t + b cos t),  t = pos * freq[i]
 * b: the element behind a (interleaved != 0), or rot_dims / 2 behind it.  Elements from rot_dims on stay as they are.  inverse != 0 turns the other way: with
 * rows of gradients this is the gradient of the call.  Angles are made in 64 bits, products and sums in 32, rounded once.
 *   freq  dev fp64 [rot_dims / 2], radians per position; climber_rotary_frequencies makes them on the host. */
typedef struct climber_rotary_plan {
    const double *freq;
    int32_t rot_dims, interleaved, inverse;
    float scale;
} climber_rotary_plan;

/* freq[i] (host, rot_dims / 2 of them) = base^(-2 i / rot_dims), for contexts longer than those that a model was made for by a factor:
 *   CLIMBER_ROTARY_LINEAR  divided by factor
 *   CLIMBER_ROTARY_BASE    with base * factor^(rot_dims / (rot_dims - 2)): the slowest pair is divided by factor, the fastest stays
 *   CLIMBER_ROTARY_PARTS   with r = made_for * freq / (2 pi) turns within the length made_for (arXiv 2309.00071, Sec. 3.2): pairs of at least `fast`
 *                          turns stay, those of at most `slow` are divided by factor, and between them linearly in r; *scale = 0.1 ln(factor) + 1
 * *scale is 1 otherwise.  What a kind does not use is not looked at.  Errors: CLIMBER_ERR_NULL, _SHAPE, _RANGE, _UNSUPPORTED (kind). */
#define CLIMBER_ROTARY_PLAIN 0
#define CLIMBER_ROTARY_LINEAR 1
#define CLIMBER_ROTARY_BASE 2
#define CLIMBER_ROTARY_PARTS 3
int climber_rotary_frequencies(int32_t rot_dims, double base, int32_t kind, double factor, double made_for, double fast,
                               double slow, double *freq, float *scale);

/* q [m][ld_q] of cfg->n_heads * d_head, k [m][ld_k] of n_kv_heads * d_head (n_kv_heads 0: no k), elements of the config's dtype; pos: dev int32 [m].
 * Row pitches are free, and so is the alignment; heads whose turned halves and rest are whole 16 bytes are faster.  q_out, k_out: of the same widths; q_out may be q
 * with the same pitch (turned in place), and k_out k; otherwise what is written must not share an element with anything else.  Uses d_model,
 * n_heads, d_head and dtype of cfg; any d_head, rot_dims even, 2 .. min(d_head, 512).
 * Errors: CLIMBER_ERR_NULL, _SHAPE, _ALIGN, _RANGE, _UNSUPPORTED, _RUNTIME. */
int climber_rotary(const climber_config *cfg, const climber_rotary_plan *rot, const int32_t *pos, int64_t m, int32_t n_kv_heads,
                   const void *q, int64_t ld_q, const void *k, int64_t ld_k, void *q_out, int64_t ld_qo, void *k_out, int64_t ld_ko,
                   void *stream);

/* ---- debug check of device-resident inputs -----------------------------------------------------
 * Eq. (3) divides a row's logits by tau[scen][beh]: the ids must lie inside the table and the entry
 * must be finite and > 0.  Ids, offsets and the table live in device memory, so the compute calls
 * cannot validate them on the host (they clamp ids and leave the rest to the caller's contract).
 * This call launches one small kernel on `stream` that reads, inside the given bounds only,
 *   - history rows (cache != NULL): scen / beh of the valid rows of every user of the cache
 *     (padding rows may hold anything); cand_off, B_cand, m_max are ignored;
 *   - candidate rows (cache == NULL): scen / beh [m_total], and, if cand_off != NULL, cand_off
 *     [B_cand + 1] against the rules of climber_attn_sumi (starts at 0, non-decreasing, ends at
 *     m_total, every count <= m_max);
 *   - the entries of tau_layer that the checked rows select;
 * and ORs CLIMBER_BAD_* bits into *status (dev int32; the caller zeroes it before, and reads it after
 * synchronising the stream: 0 = nothing found).  The kernel always runs to completion.
 * Errors: CLIMBER_ERR_NULL, _SHAPE (m_total < 0, B_cand < 1 with cand_off), _RUNTIME. */
#define CLIMBER_BAD_SCEN 1    /* a scenario id outside [0, n_scen) */
#define CLIMBER_BAD_BEH 2     /* a behaviour id outside [0, n_beh) */
#define CLIMBER_BAD_TAU 4     /* a selected temperature is not finite or not > 0 */
#define CLIMBER_BAD_OFFSETS 8 /* cand_off not 0-based, decreasing somewhere, or not ending at m_total */
#define CLIMBER_BAD_M_MAX 16  /* a user has more candidates than m_max */
int climber_check_inputs(const climber_config *cfg, const float *tau_layer, const int32_t *scen,
                         const int32_t *beh, const climber_kv_cache *cache, int32_t m_total,
                         const int32_t *cand_off, int32_t B_cand, int32_t m_max, int32_t *status,
                         void *stream);

/* ---- layer stack (CLIMBER_BF16 only) ---------------------------------------------------------- */

/* Bytes of scratch the stack calls need for up to max_rows rows (history rows or candidates). */
size_t climber_workspace_bytes(const climber_config *cfg, int64_t max_rows);

/* One layer of the stack on the history rows (mode HISTORY: writes cache layer `layer`, attends
 * block-diagonally) or on candidate rows (mode CANDIDATE: SUMI attention against cache layer
 * `layer`).  x_in, x_out: dev fp32 [rows][d_model] residual stream (x_out may be NULL in HISTORY
 * mode: then only the layer's K/V are produced, which is all the last layer of an encode needs;
 * x_out may alias x_in).  ids: per-row scenario / behaviour ids of the rows being processed.
 * cand_off / m_total / m_max as in climber_attn_sumi (ignored in HISTORY mode).
 * workspace: dev, >= climber_workspace_bytes(cfg, rows), 256-byte aligned. */
int climber_layer_forward(const climber_config *cfg, const climber_layer_weights *w,
                          const float *tau_layer, int32_t layer, int32_t mode,
                          climber_kv_cache *cache, const float *x_in, float *x_out,
                          const int32_t *scen, const int32_t *beh, const int32_t *cand_off,
                          int32_t m_total, int32_t m_max, void *workspace, size_t ws_bytes,
                          void *stream);

/* The projections read their weights as MFMA operand fragments with the RMSNorm gains multiplied
 * in (f_QKV / f_FFN of Eq. (3)); the stack calls bring `layers` into that form in their workspace
 * on every call (~1 % of a step).  A caller whose weights do not change can do it once:
 * climber_pack_weights fills `packed` (dev, 256-byte aligned, >= climber_packed_weights_bytes(cfg),
 * 0 on an invalid config) from weights->layers on `stream`; the caller then sets weights->packed
 * to that buffer, which must stay unchanged while calls that were given it are running.  Results
 * are bitwise the same either way.  Errors: CLIMBER_ERR_NULL, _SHAPE (n_layers), _ALIGN,
 * _BUFSIZE, _UNSUPPORTED (not the bf16 stack), _RUNTIME. */
size_t climber_packed_weights_bytes(const climber_config *cfg);
int climber_pack_weights(const climber_config *cfg, const climber_weights *weights, void *packed,
                         size_t bytes, void *stream);

/* History encode (first phase of the serving flow, Sec. 3.2): runs the packed history embeddings
 * x_hist (dev bf16 [rows][d_model]) through all layers and fills every layer of the cache.  The
 * last layer stops after its K/V are stored.  tau: dev fp32 [n_layers][n_scen][n_beh].
 * workspace must hold climber_workspace_bytes(cfg, rows). */
int climber_history_encode(const climber_config *cfg, const climber_weights *weights,
                           const float *tau, const void *x_hist, const int32_t *scen,
                           const int32_t *beh, climber_kv_cache *cache, void *workspace,
                           size_t ws_bytes, void *stream);

/* Candidate scoring (second phase): x_cand dev bf16 [m_total][d_model] -> y_cand dev fp32
 * [m_total][d_model], the candidates' final-layer hidden states (the paper's scalar score needs
 * its fusion module and an unspecified head on top of these).  workspace must hold
 * climber_workspace_bytes(cfg, m_total). */
int climber_sumi_score(const climber_config *cfg, const climber_weights *weights, const float *tau,
                       const climber_kv_cache *cache, const void *x_cand, const int32_t *cand_off,
                       int32_t m_total, int32_t m_max, const int32_t *cand_scen,
                       const int32_t *cand_beh, float *y_cand, void *workspace, size_t ws_bytes,
                       void *stream);

/* Training-side form of the "single user, multiple items" pattern (Sec. 3.2): the histories and the
 * candidates of a batch run through all layers TOGETHER as one packed set of rows under the mask of
 * that section (history rows: own subsequence; a candidate: its user's whole history and itself,
 * never another candidate) and nothing is cached across calls -- the forward pass behind the
 * paper's training-throughput figure.  Same result as climber_history_encode followed by
 * climber_sumi_score (bitwise for y_cand under the default flags); the output projection and
 * feed-forward launches of a layer cover both kinds of rows, and the history keys / values of the
 * layer being computed live in layer 0 of `scratch_cache` (a cache handle
 * created for this batch's histories with any number of layers; its layer 0 is overwritten).
 * y_hist: dev fp32 [rows][d_model] or NULL (then the last layer skips the history rows' attention
 * and feed-forward); y_cand: dev fp32 [m_total][d_model].  workspace must hold
 * climber_workspace_bytes(cfg, rows + m_total).  Candidate counts may differ per user (cand_off).
 * Errors as climber_history_encode / climber_sumi_score. */
int climber_sumi_forward(const climber_config *cfg, const climber_weights *weights, const float *tau,
                         const void *x_hist, const int32_t *scen, const int32_t *beh,
                         const void *x_cand, const int32_t *cand_off, int32_t m_total, int32_t m_max,
                         const int32_t *cand_scen, const int32_t *cand_beh,
                         climber_kv_cache *scratch_cache, float *y_hist, float *y_cand,
                         void *workspace, size_t ws_bytes, void *stream);

/* ---- bit-wise gating fusion (Sec. 3.1.4, Eq. (4)) and score ------------------------------------
 * The paper runs one Transformer block per subsequence ("corresponding block", Sec. 3.1.2); block k
 * turns a candidate into an output vector E(S_k), and the fusion module turns the N_b vectors of a
 * candidate into its score:
 *     G = ATL(E)                     one attention layer over the N_b rows of the candidate, every row
 *                                    seeing every row, no relative attention bias, temperature from the
 *                                    candidate's scenario only (tau_scen[scen])
 *     Y = G (.) sigmoid(f_gate(G))   f_gate: squeeze-and-excitation with equal input / output size
 *     score = head(Y)
 * As fixed by this library where the paper is silent: the fusion ATL is a layer of the stack's
 * composition (see climber_layer_weights) with weights of its own; f_gate maps the N_b * d_model
 * values of G, flattened row by row, down to d_gate, applies ReLU, and maps back (no bias vectors);
 * the head is <w_head, vec(Y)> + b_head.  Block k's E(S_k) is produced with the calls above: a
 * cache over subsequence k only (sub_len = 0), block k's weights, climber_history_encode, then
 * climber_sumi_score or climber_sumi_forward: its y_cand rows are E(S_k).
 * e: dev fp32 [m_total][n_blocks][d_model]; cand_scen: dev int32 [m_total]; y: dev fp32 like e, or
 * NULL; score: dev fp32 [m_total].  CLIMBER_BF16, d_head = 64, 1 <= n_blocks <= 16, d_gate a
 * multiple of 128 and <= n_blocks * d_model.  e, y, w_down, w_up, w_head: 16-byte aligned.
 * workspace: climber_bgf_workspace_bytes(), 256-byte aligned.  Errors: CLIMBER_ERR_NULL, _SHAPE, _UNSUPPORTED, _ALIGN, _RANGE, _BUFSIZE, _RUNTIME. */
typedef struct climber_bgf_weights {
    climber_layer_weights atl; /* fusion layer, bf16, shapes of a stack layer */
    const void *w_down;        /* dev bf16 [n_blocks * d_model][d_gate] */
    const void *w_up;          /* dev bf16 [d_gate][n_blocks * d_model] */
    const float *w_head;       /* dev fp32 [n_blocks * d_model] */
    const float *tau_scen;     /* dev fp32 [n_scen] */
    float b_head;
    int32_t n_blocks, d_gate;
} climber_bgf_weights;
size_t climber_bgf_workspace_bytes(const climber_config *cfg, int32_t n_blocks, int32_t d_gate,
                                   int64_t m_total);
int climber_bgf_score(const climber_config *cfg, const climber_bgf_weights *w, const float *e,
                      const int32_t *cand_scen, int32_t m_total, float *y, float *score,
                      void *workspace, size_t ws_bytes, void *stream);

/* climber_sumi_score for callers that cannot allocate or hand over device memory for scratch: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments,
 * same kernels and bitwise the same y_cand as climber_sumi_score, but the scratch lives in a fixed
 * array of CLIMBER_STATIC_SCRATCH_BYTES inside the library (one per GPU, held until the process
 * ends) instead of a caller's workspace, and the call allocates and frees nothing.
 *  - weights->packed must be set (climber_pack_weights): CLIMBER_ERR_NULL otherwise.
 *  - m_total is limited by the array: climber_workspace_bytes(cfg, m_total) minus
 *    climber_packed_weights_bytes(cfg) must not exceed CLIMBER_STATIC_SCRATCH_BYTES
 *    (2512 candidates at d_model 512, d_ffn 2048); beyond that CLIMBER_ERR_BUFSIZE and nothing is
 *    launched.
 *  - All calls on one GPU share that GPU's array: calls that may overlap on one GPU (different
 *    streams, different threads) race; serialise them.  The first call on a GPU looks the array's
 *    address up (no allocation); make that call outside a graph capture.
 * Other errors as climber_sumi_score. */
#define CLIMBER_STATIC_SCRATCH_BYTES (32u << 20)
int climber_sumi_score_static(const climber_config *cfg, const climber_weights *weights,
                              const float *tau, const climber_kv_cache *cache, const void *x_cand,
                              const int32_t *cand_off, int32_t m_total, int32_t m_max,
                              const int32_t *cand_scen, const int32_t *cand_beh, float *y_cand,
                              void *stream);

#ifdef __cplusplus
}
#endif
#endif /* CLIMBER_H */
