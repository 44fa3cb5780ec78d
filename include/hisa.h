/*
 * hisa.h -- C ABI of the HISA hierarchical indexer for AMD MI355X (gfx950).
 *
 * The library computes, per query t, the token-index set that Sparse MLA consumes, by the
 * two-stage search of the HISA paper (Section 4.1, Algorithm 1), and the flat DSA indexer
 * (Section 3, Eqs. 1-2) as the baseline at the same shapes.
 *
 * Conventions for every call
 *   - Every tensor pointer is a DEVICE pointer owned by the caller, row-major, densely packed.
 *     The descriptor structs themselves live in HOST memory.
 *   - The library allocates nothing and keeps no state.  Scratch memory is a caller-provided
 *     device workspace `ws` of `ws_bytes` bytes (256-byte aligned); hisa_workspace_bytes() gives
 *     the size a call wants.  A call may be given more; it never touches bytes past ws_bytes.
 *   - A call only enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = the null
 *     stream) and returns without synchronising.  Calls sharing one workspace must be ordered on
 *     one stream.
 *   - Return value: HISA_OK, or an error code.  Validation is done on the host BEFORE anything is
 *     launched: on an error other than HISA_ERR_LAUNCH nothing was enqueued and outputs are
 *     untouched.  Device-resident arrays (seq_len, q_seq, q_pos, block_idx) cannot be validated
 *     on the host; kernels clamp positions to the sequence length so a bad value cannot cause an
 *     out-of-bounds access, but the result for that query is then unspecified.
 *   - Positions are 0-based.  The query at position p sees keys s <= p of its own sequence
 *     (Section 4.1, boundary behaviour: a prefix no longer than k is selected whole).
 *   - Top-k / top-m order candidates by score descending, ties by lower index.  Index outputs
 *     hold the selected ids in ASCENDING order, then -1 padding when fewer than k (m) exist.
 *
 * Supported shapes
 *   - q F32  + k F32  (+ pooled F32):  any H <= 128, d % 4 == 0, d <= 512  (plain fp32 ALU path)
 *   - q BF16 + k BF16 or FP8_E4M3 (+ pooled BF16):  d == 128, H in {32, 64}, B % 32 == 0
 *     (MFMA path, fp32 accumulation.  bf16 keys: bf16 MFMA.  fp8 keys: the stored codes go into
 *     the fp8 MFMA against the bf16 query written as the sum of two e4m3 numbers per element,
 *     after a power-of-two scaling per head; that sum is the query exactly except for elements
 *     2^9 below their head's largest, which keep 2^-17 of that largest; the per-token scale
 *     multiplies the finished score, which equals Eq. 1 on the dequantised key because the scale
 *     is positive.  Scores agree with a double-precision evaluation of the same stored bits to
 *     about 2e-7 relative with bf16 keys and 2e-5 (6e-5 worst observed) with fp8 keys, the fp8 MFMA's
 *     own accumulation.)
 *   - top-k / candidate limits: k <= 8192, m <= 1024, m * B <= 65536; one sequence's key array
 *     (s_max * d elements) must stay below 2 GiB.
 *   - T <= 4194304 queries per call and n_seq <= 65535 sequences per key array (launch-grid limits;
 *     more queries: split the call); anything beyond returns HISA_ERR_SHAPE before a launch.
 */
#ifndef HISA_H_
#define HISA_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HISA_OK = 0,
  HISA_ERR_NULL = 1,        /* a required pointer is NULL                                        */
  HISA_ERR_SHAPE = 2,       /* H, d, B, m, k, T, s_max outside the supported set                 */
  HISA_ERR_DTYPE = 3,       /* unsupported dtype or dtype combination                            */
  HISA_ERR_INFEASIBLE = 4,  /* m * B < k (Section 4.1, feasibility constraint) or m < 2          */
  HISA_ERR_WORKSPACE = 5,   /* ws is NULL or smaller than the call's minimum                     */
  HISA_ERR_ALIGN = 6,       /* a tensor pointer is not 16-byte aligned                           */
  HISA_ERR_LAUNCH = 7       /* the HIP runtime refused a launch (hipGetLastError was non-zero)   */
} hisa_status;

typedef enum {
  HISA_F32 = 0,
  HISA_BF16 = 1,
  HISA_FP8_E4M3 = 2         /* OCP e4m3fn codes + one fp32 scale per token                       */
} hisa_dtype;

/* Token-level indexing keys k_s (Section 3): n_seq sequences padded to s_max rows each. */
typedef struct {
  const void*    k;         /* [n_seq, s_max, d] of k_dtype (device)                             */
  const float*   k_scale;   /* [n_seq, s_max] fp32, required iff k_dtype == FP8: key = scale*code */
  const int32_t* seq_len;   /* [n_seq] valid keys per sequence (device)                          */
  int32_t        n_seq;
  int32_t        s_max;
  int32_t        d;
  int32_t        k_dtype;   /* hisa_dtype */
} hisa_keys;

/* Indexing queries q_{t,j} and gates w_{t,j} (Section 3) for T packed queries. */
typedef struct {
  const void*    q;         /* [T, H, d] of q_dtype (device)                                     */
  const float*   w;         /* [T, H] fp32 gates, any sign (device)                              */
  const int32_t* q_seq;     /* [T] sequence id of each query, or NULL: all queries in sequence 0 */
  const int32_t* q_pos;     /* [T] position of each query, or NULL: q_pos[t] = q_pos0 + t        */
  const int32_t* q_lo;      /* [T] first visible position of each query, or NULL: 0.  For sequences
                               packed into one key stream without padding (Section 4.1: a block may
                               then straddle two sequences): q_lo[t] = first token of the query's
                               sequence in the stream, q_pos[t] its own position there; the query
                               sees the keys q_lo[t] .. q_pos[t].  Blocks stay multiples of B of the
                               stream and are pooled over everything they hold; the visible blocks
                               are q_lo/B .. q_pos/B, the first and the last of them forced.  (device) */
  int32_t        T;
  int32_t        H;
  int32_t        q_pos0;
  int32_t        q_dtype;   /* hisa_dtype: F32 or BF16 */
} hisa_queries;

/* Operation selector for hisa_workspace_bytes. */
enum { HISA_OP_POOL = 0, HISA_OP_BLOCK_SCORE_TOPK = 1, HISA_OP_TOKEN_REFINE_TOPK = 2,
       HISA_OP_FLAT_TOPK = 3 };

/*
 * Block pooling (Eq. 4; Algorithm 1, pooling loop): pooled[n, b, :] = mean of the keys of block
 * b of sequence n, for b in [blk_begin, blk_end) (blk_end <= s_max / B; pass 0, s_max / B for all).
 * A block holds tokens bB .. min((b+1)B, seq_len[n]) - 1 and is averaged over the tokens present;
 * a block with no token is written as zeros.  Accumulation in fp32, one rounding to pooled_dtype
 * (F32, or BF16 for BF16/FP8 keys).  pooled: [n_seq, s_max / B, d] device, written in the given
 * block range only.  Needs no workspace.
 */
int hisa_pool_blocks(const hisa_keys* keys, int32_t B, int32_t blk_begin, int32_t blk_end,
                     void* pooled, int32_t pooled_dtype, void* stream);

/*
 * The same call with the per-dimension MAXIMUM over the tokens present in a block instead of their
 * mean: Eq. 4 is written for a generic Pool, the paper uses the mean and names max-pooling as a
 * variant to explore.  Everything else as hisa_pool_blocks (a block with no token is zeros); the
 * later stages take either pooled array.  hisa_pool_append maintains the mean only.
 */
int hisa_pool_blocks_max(const hisa_keys* keys, int32_t B, int32_t blk_begin, int32_t blk_end,
                         void* pooled, int32_t pooled_dtype, void* stream);

/*
 * Stage 1 (Eqs. 5-6; Algorithm 1, block-level coarse filter).  For each query, scores the pooled
 * keys of the visible blocks 0 .. b_t (b_t = q_pos / B) and keeps min(m, b_t + 1) blocks: block 0
 * and block b_t always (Section 4.1: first and last block forced, counted inside the budget m),
 * the rest by score.  `keys` supplies shapes and seq_len only (keys->k may be NULL).
 *   pooled       [n_seq, s_max / B, d] of pooled_dtype (device, in)
 *   block_idx    [T, m] int32 (device, out): kept block ids ascending, then -1
 *   block_scores [T, s_max / B] fp32 (device, out) or NULL: J_{t,b} for b <= b_t, -inf beyond
 * Workspace: T * (s_max / B) floats when block_scores is NULL, else none.  (A batch of at most 256
 * queries with bf16 pooled keys and at most 8192 blocks per sequence -- a decode step -- is scored
 * and selected in one launch that keeps the block scores on chip; the workspace must still be
 * passed, and is then left untouched.)
 */
int hisa_block_score_topk(const hisa_queries* queries, const hisa_keys* keys, const void* pooled,
                          int32_t pooled_dtype, int32_t B, int32_t m, int32_t* block_idx,
                          float* block_scores, void* ws, size_t ws_bytes, void* stream);

/*
 * Stage 2 (Eqs. 7-9; Algorithm 1, token-level refinement).  Scores, with Eq. 1, the visible
 * tokens of the kept blocks and selects the k best.
 *   block_idx   [T, m] int32 (device, in): ascending block ids then -1, as Stage 1 writes them
 *   topk_idx    [T, k] int32 (device, out): selected token positions (within the query's
 *               sequence) ascending, then -1
 *   topk_scores [T, k] fp32 (device, out) or NULL: scores aligned with topk_idx (padding: -inf)
 *   cand_scores [T, m * B] fp32 (device, out) or NULL: every candidate score, slot c = kept block
 *               c / B, offset c % B; -inf where masked.  Requesting it selects the two-kernel path.
 * Workspace: none for the fused path (cand_scores NULL, T >= 256, m * B <= 16384), otherwise
 * T * m * B floats unless cand_scores is given.
 */
int hisa_token_refine_topk(const hisa_queries* queries, const hisa_keys* keys, int32_t B, int32_t m,
                           const int32_t* block_idx, int32_t k, int32_t* topk_idx,
                           float* topk_scores, float* cand_scores, void* ws, size_t ws_bytes,
                           void* stream);

/*
 * hisa_token_refine_topk for callers that cannot allocate device memory and have no workspace to
 * hand over: code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * Same inputs, outputs and results as hisa_token_refine_topk with cand_scores == NULL; the
 * candidate scores of the two-kernel path (T < 256, or m * B > 16384) go through a static device
 * array of HISA_STATIC_SCRATCH_BYTES inside the library instead of a workspace.  The call
 * allocates and frees nothing and, like every other call, only enqueues kernels on `stream`.
 *   - Limit: T * m * B * 4 <= HISA_STATIC_SCRATCH_BYTES on that path (a decode batch of 512
 *     queries at m * B = 8192); beyond it the call returns HISA_ERR_WORKSPACE and launches nothing.
 *   - Every GPU the process uses holds its own copy of the array until the process ends.  The
 *     first call on a device looks its address up (make that call outside a graph capture).
 *   - All calls on one GPU share the array: calls that may overlap in time (different streams
 *     without an ordering between them) race on it.  Nothing in it has to be cleared between calls:
 *     the scoring kernel rewrites every slot the select reads.
 */
#define HISA_STATIC_SCRATCH_BYTES (16u << 20)
int hisa_token_refine_topk_static(const hisa_queries* queries, const hisa_keys* keys, int32_t B, int32_t m,
                                  const int32_t* block_idx, int32_t k, int32_t* topk_idx,
                                  float* topk_scores, void* stream);

/*
 * Flat DSA indexer (Eqs. 1-2): scores every visible key s <= q_pos and selects the k best.
 * Same outputs as Stage 2.  The scores of a chunk of queries go through the workspace (one row of
 * round_up(s_max, 64) floats per query) and are selected row by row; the library loops over
 * chunks sized to the workspace: minimum 8 rows (plus, only for k > 2048 with s_max > 65536,
 * 8 * k bytes per 65536-entry segment and query; hisa_workspace_bytes gives the size to pass).
 */
int dsa_flat_indexer_topk(const hisa_queries* queries, const hisa_keys* keys, int32_t k,
                          int32_t* topk_idx, float* topk_scores, void* ws, size_t ws_bytes,
                          void* stream);

/*
 * Algorithm 1 whole in one launch: Stage 1 (Eqs. 5-6) and Stage 2 (Eqs. 7-9) of each query run
 * back to back in one workgroup, the query is read once, the block scores and the kept block ids
 * never leave the CU.  Same results as hisa_block_score_topk followed by hisa_token_refine_topk.
 * A convenience for callers that want one call and no workspace, NOT the fast path: on MI355X the
 * two calls are quicker at every shape measured (prefill: the separate Stage 1 kernel shares each
 * pooled-key tile between 8 queries or keeps the tiles resident; decode: the two calls spread a
 * query's tiles over many compute units, one workgroup per query cannot), by 1 % (decode batch) to
 * 18 % (1M-context chunk).
 *   pooled     [n_seq, s_max / B, d] BF16 (device, in), as hisa_pool_blocks writes it
 *   block_idx  [T, m] int32 (device, out) or NULL: the kept block ids, ascending then -1
 *   topk_idx / topk_scores: as hisa_token_refine_topk
 * Supported: q BF16, k BF16 or FP8_E4M3, pooled BF16, d == 128, H in {32, 64}, B % 32 == 0,
 * m * B <= 16384, s_max / B <= 8192; anything else returns HISA_ERR_SHAPE / HISA_ERR_DTYPE (use the
 * two calls).  Needs no workspace.
 */
int hisa_indexer_topk(const hisa_queries* queries, const hisa_keys* keys, const void* pooled,
                      int32_t pooled_dtype, int32_t B, int32_t m, int32_t k, int32_t* block_idx,
                      int32_t* topk_idx, float* topk_scores, void* stream);

/*
 * Incremental maintenance of the pooled-key cache (Section 4.1, block pooling: the pooled keys are
 * a cache kept up to date next to the KV cache; Section 4.2 assumes it).  After sequence n grew
 * from prev_len[n] to keys->seq_len[n] tokens (appended at the end), recomputes exactly the pooled
 * keys of the blocks that received tokens: blocks prev_len[n] / B .. (seq_len[n] - 1) / B.  The
 * result is bit-identical to hisa_pool_blocks over the whole sequence.
 *   prev_len       [n_seq] int32 (device): lengths at the previous update (0 for a new sequence)
 *   max_new_tokens host bound on seq_len[n] - prev_len[n] over all sequences (sizes the launch);
 *                  growth beyond it is NOT pooled
 *   pooled         [n_seq, s_max / B, d] (device, in/out)
 */
int hisa_pool_append(const hisa_keys* keys, int32_t B, const int32_t* prev_len, int32_t max_new_tokens,
                     void* pooled, int32_t pooled_dtype, void* stream);

/*
 * Block-Sparse baseline of the paper's evaluation (Section 5: Stage 1 only, every token of the kept
 * blocks is attended): expands block_idx into token positions.
 *   tokens [T, m * B] int32 (device, out): slot c = block_idx[t, c / B] * B + c % B if that token
 *   is visible to the query (<= q_pos), else -1.  With block_idx as Stage 1 writes it (ascending,
 *   own block last) the valid entries are ascending and the -1 entries form the tail.
 */
int hisa_block_sparse_tokens(const hisa_queries* queries, const hisa_keys* keys, int32_t B, int32_t m,
                             const int32_t* block_idx, int32_t* tokens, void* stream);

/*
 * Selection-consistency diagnostic (Eq. 12): iou[t] = |A_t & B_t| / |A_t | B_t| for two index
 * tensors [T, k] whose rows are ascending with -1 padding at the end (as this library writes
 * them); two empty rows give 1.  iou: [T] fp32 (device, out).
 */
int hisa_index_iou(const int32_t* a_idx, const int32_t* b_idx, int32_t T, int32_t k, float* iou,
                   void* stream);

/* ------------------------------------------------------------------------------------------------
 * Around the indexer: a paged key/value cache, what fills it, and the attention that reads it.
 * ---------------------------------------------------------------------------------------------- */

/*
 * What the attention over a BF16 or FP8 cache multiplies with its values (the sums of weights are fp32 either way):
 *   HISA_WEIGHTS_16BIT  (0) two bf16 parts of each weight, 16 bits together: a result is off by little more than its
 *                       own rounding to bf16
 *   HISA_WEIGHTS_8BIT   one bf16, 8 bits: a result of many keys is off by up to 1.45 times that in the mean square.
 *                       For prompts, where the second part is a sixth to a quarter of the call; single tokens wait
 *                       for memory and gain nothing
 */
typedef enum { HISA_WEIGHTS_16BIT = 0, HISA_WEIGHTS_8BIT = 1 } hisa_weights;

/*
 * A cache of n_pages pages of `page` token rows each, H_kv heads of d elements per row.  Row (page p,
 * offset o, head h) begins page_stride * p + token_stride * o + head_stride * h elements behind k and
 * behind v (one set of strides for both, so [n_pages, page, H_kv, d], [n_pages, H_kv, page, d] and
 * arrays that interleave keys and values all fit); its d elements are contiguous.  Slot p * page + o
 * names a row of all heads.  Rows that no slot or table names are never touched.
 */
typedef struct {
  void*          k;           /* first key row, of `dtype` (device)                                    */
  void*          v;           /* first value row; NULL for a cache of keys alone (hisa_cache_append)   */
  float*         k_scale;     /* [n_pages, page, H_kv] fp32, required iff dtype == FP8: row = scale*code */
  float*         v_scale;     /* the same for the values                                               */
  const int32_t* block_table; /* [n_seq, max_pages]: page of tokens j*page .. of sequence n (device)   */
  const int32_t* seq_len;     /* [n_seq] tokens of each sequence, the new ones included (device)       */
  int64_t        page_stride, token_stride, head_stride;   /* in elements                              */
  int32_t        n_pages;
  int32_t        page;
  int32_t        n_seq;
  int32_t        max_pages;
  int32_t        H_kv;
  int32_t        d;
  int32_t        dtype;       /* hisa_dtype                                                            */
  int32_t        weights;     /* hisa_weights: of the attention over a BF16 or FP8 cache                */
} hisa_cache;

/*
 * Block tables and slot maps of a batch from the lengths of its requests.  Sequence n holds ctx_len[n]
 * tokens and receives new_len[n] more (negative lengths count as 0); the new tokens of all sequences
 * stand in `rows` token rows, sequence after sequence.  All arrays are device arrays.
 *   block_table [n_seq, max_pages] in/out: the entries ceil(ctx_len/page) .. ceil((ctx_len+new_len)/page)
 *               - 1 of each sequence are taken from free_pages, in the order of the sequences; every
 *               other entry is left as it was.  New tokens beyond the last of `rows` get their pages all
 *               the same (and count in seq_len), only no row and no slot
 *   free_pages  [n_free] page ids; the first page_start[n_seq] of them are in use afterwards.  If that
 *               number exceeds n_free, the entries beyond are written as -1 and their tokens get no slot
 *   seq_len     [n_seq] out: ctx_len + new_len, at most max_pages * page
 *   q_start     [n_seq + 1] out: first token row of each sequence, and their number (at most rows)
 *   page_start  [n_seq + 1] out: how many free pages the sequences before took, and all of them
 *   q_seq, q_pos [rows] out: sequence and position of each token row, as hisa_queries takes them; rows
 *               behind the last token (a padded batch): 0 and -1, a query that sees nothing
 *   slots       [rows] out: slot of each token row in the pages, -1: none (padding, no page left, or
 *               beyond max_pages * page)
 *   key_rows    [rows] out or NULL: q_seq * s_max + q_pos, the row of the token in a padded key array
 *               [n_seq, s_max, d] as hisa_keys describes it (-1: padding, or a position >= s_max)
 * Positions stop at 2^31 - 1, a slot from 2^31 on is none.  Arrays must not overlap (seq_len == ctx_len,
 * say, is refused).  Limits: n_seq <= 65535, rows <= 4194304, n_seq * max_pages and max_pages * page below
 * 2^31, n_seq * s_max below 2^31 (with key_rows).  Needs no workspace.
 */
int hisa_page_tables(const int32_t* ctx_len, const int32_t* new_len, int32_t n_seq, int32_t* block_table,
                     int32_t max_pages, int32_t page, const int32_t* free_pages, int32_t n_free, int32_t rows,
                     int32_t s_max, int32_t* seq_len, int32_t* q_start, int32_t* page_start, int32_t* q_seq,
                     int32_t* q_pos, int32_t* slots, int32_t* key_rows, void* stream);

/*
 * Writes T new rows (0: nothing to do) into the cache: row t of k_new (and of v_new, unless both it and cache->v are NULL)
 * goes to slot slots[t]; a slot outside [0, n_pages * page) is skipped.  k_new, v_new: H_kv heads of d
 * contiguous elements per row, rows src_stride elements apart (>= H_kv * d), of src_dtype (F32 or
 * BF16).  Converted to cache->dtype: F32 (from F32), BF16 (rounded to nearest even), or FP8_E4M3 with
 * one scale per row and head: scale = largest finite |element| / 448 (1 for a row of zeros, never
 * below 2^-126), code = e4m3fn(element / scale) to nearest even; an element that is not finite becomes
 * the NaN code.  Slots must differ from each other: which of two rows a slot named twice holds (or
 * which part of each) is unspecified.  The indexer's padded key array is a cache of n_seq pages of
 * s_max rows with one head and no values, and hisa_page_tables gives its slots as key_rows.
 * block_table and seq_len are not read (may be NULL).  d % 8 == 0, d <= 512, strides multiples of 8;
 * n_pages * page below 2^31; k, v, k_new, v_new 16-byte aligned, src_stride a multiple of 8; T * H_kv *
 * d (rounded up to a power of two) below 2^35.
 * Needs no workspace.
 */
int hisa_cache_append(const hisa_cache* cache, const int32_t* slots, const void* k_new, const void* v_new,
                      int32_t src_dtype, int64_t src_stride, int32_t T, void* stream);

/*
 * Attention of new tokens over the paged cache: for every query t (one of `T` token rows) and head h,
 * over the positions s that it sees, q_lo[t] <= s <= q_pos[t] and s < seq_len of its sequence,
 *   out[t, h, :] = sum_s p_s v_s / sum_s p_s,  p_s = exp(scale * q_{t,h} . k_s),  lse[t, h] = log sum_s p_s,
 * where k_s, v_s are the rows of KV head h / (H / H_kv).  Nothing at a position that a query does not
 * see affects its result, infinities and NaN included.  A query that sees no key gives zeros and -inf.
 *   queries     q [T, H, d], T, H, q_dtype; q_pos (NULL: the new tokens are the last q_start[n+1] -
 *               q_start[n] positions of their sequence, which is not so where hisa_page_tables had more new
 *               tokens than rows: its q_pos is right there too) and q_lo (NULL: 0) as everywhere.  A document
 *               or sliding-window mask is a q_lo, a prefix that sees itself whole a q_pos beyond the
 *               own position.  w, q_seq and q_pos0 are not read
 *   q_start     [n_seq + 1] first token row of each sequence, ascending, T at most (device, in), as
 *               hisa_page_tables writes it.  Rows before q_start[0] and from q_start[n_seq] on belong to
 *               nobody: their out and lse are left as they were
 *   out         [T, H, d] of q_dtype (device, out)
 *   lse         [T, H] fp32 (device, out) or NULL
 * A block_table entry outside [0, n_pages) holds no key that anybody sees.
 * Supported: 1 <= T <= 4194304; q BF16 with a BF16 or FP8_E4M3 cache, d in {64, 128}; q F32 with an F32 cache, d % 4 == 0,
 * d <= 256.  H <= 256, H_kv divides H; page a power of two; k, v and q 16-byte aligned, strides times
 * the element size multiples of 16 bytes; max_pages * page and n_pages * page below 2^31;
 * scale positive and finite (below 2^127).  A launch holds fewer than 2^23 workgroups: split larger calls.  What always
 * fits: T * H_kv * ceil(H / H_kv / 32) below that (lists), T * H / 32 + 4 * n_seq * H_kv (ranges).
 * Scores, the running maximum and sum and the output are held in fp32; for the second product (bf16 and
 * fp8 caches) the weights p_s are rounded as cache->weights says.  Weights are kept below 2^8 until the division by their
 * sum, so finite values (scale * code) of 2^88 and less never overflow, whatever their number.  All sums have a fixed order: the same
 * call gives the same bits.
 * How a call is cut up goes by T, n_seq and max_pages, since the lengths are on the device: T <= 2 * n_seq (FP8:
 * 4 * n_seq) is taken for a batch of single tokens, each of which reads its keys by itself.  So
 * pass no idle sequences, little padding and a table of the width in use, and give a long chunk beside single tokens a
 * call of its own: the same queries and out, and the sequence's part of block_table, seq_len (n_seq = 1) and q_start.
 * Workspace: hisa_attention_workspace_bytes(queries, cache, 0), which depends on shapes and types only and
 * not always grows with T.
 */
int hisa_paged_attention(const hisa_queries* queries, const hisa_cache* cache, const int32_t* q_start,
                         float scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * The same attention over a list of positions per query, such as the indexer's output, for heads with plain keys and
 * values of one width d (not over latent rows, whose scores and values have widths of their own: those are refused
 * as any other d is).  Query t of sequence q_seq[t] (NULL: 0) attends to the positions topk_idx[t, :]
 * (order does not matter; a position named twice counts twice), entries outside [0, seq_len) are
 * skipped, so both hisa_token_refine_topk's lists and hisa_block_sparse_tokens' fit; a query whose
 * sequence is outside [0, n_seq) sees nothing.  Whether a position is visible is the list's business:
 * q_pos and q_lo are not read.
 *   topk_idx    [T, k] int32 (device, in), k <= 65536
 * Everything else, the workspace rule (hisa_attention_workspace_bytes(queries, cache, k)) included, as
 * hisa_paged_attention.
 */
int hisa_sparse_attention(const hisa_queries* queries, const hisa_cache* cache, const int32_t* topk_idx,
                          int32_t k, float scale, void* out, float* lse, void* ws, size_t ws_bytes,
                          void* stream);

/* Workspace in bytes for hisa_paged_attention (k == 0) or hisa_sparse_attention (k >= 1) at these shapes and
 * types; 0 if none is needed or the call would refuse the descriptors.  They are checked as the call checks them, so
 * the pointers have to be there and aligned; they are not read, and any aligned address gives the size before
 * the arrays exist.  More queries do not always need more: with enough of them the keys are not split (H = 64, H_kv = 8,
 * d = 128, one sequence of up to 131072: 34078720 bytes at T = 64 and at T = 256, none at T = 1024).  A workspace for batches
 * of several sizes is the largest of what each of them asks for. */
size_t hisa_attention_workspace_bytes(const hisa_queries* queries, const hisa_cache* cache, int32_t k);

/*
 * Attainable-peak probes for benchmarks (measurement aids; nothing of the paper's method).
 * hisa_probe_copy: one streaming device-to-device copy of `bytes` (a multiple of 16; both pointers
 * device, 16-byte aligned) with a 4096-workgroup grid: bytes read + bytes written over its time is
 * the HBM rate this chip sustains.  hisa_probe_mfma: 512 workgroups of 4 waves each issue
 * iters * 16 v_mfma_f32_32x32x16_bf16 and nothing else; *flop (host) receives the flop count of the
 * launch, out (device, 512 * 256 floats) receives values that only keep the loop alive.
 * hisa_probe_mfma_fp8: the same with iters * 8 v_mfma_f32_32x32x64_f8f6f4 (e4m3 x e4m3), the
 * instruction the fp8-key scoring runs on.  hisa_probe_mfma_toggling: either loop (fp8 = 0 / 1) on
 * operands that differ per lane and per instruction (pseudo-random signs and mantissas): the rate
 * the matrix cores sustain once their inputs toggle as real data does, which on this chip is below
 * the rate of the two constant-operand probes because the clock drops under that load.
 */
int hisa_probe_copy(const void* src, void* dst, size_t bytes, void* stream);
int hisa_probe_mfma(float* out, int32_t iters, double* flop, void* stream);
int hisa_probe_mfma_fp8(float* out, int32_t iters, double* flop, void* stream);
int hisa_probe_mfma_toggling(float* out, int32_t iters, int32_t fp8, double* flop, void* stream);

/* Recommended workspace size in bytes for `op` (HISA_OP_*) at these shapes; 0 if none is needed
 * or the shapes are invalid.  `want_scores` != 0: the optional full score output of Stage 1 / 2
 * is requested (which then replaces the workspace). */
size_t hisa_workspace_bytes(int op, const hisa_queries* queries, const hisa_keys* keys, int32_t B,
                            int32_t m, int32_t k, int32_t want_scores);

/* Static description of a status code. */
const char* hisa_status_string(int status);

/* Library version, "major.minor". */
const char* hisa_version(void);

#ifdef __cplusplus
}
#endif
#endif /* HISA_H_ */
