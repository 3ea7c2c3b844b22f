/*
 * rsa.h -- C-ABI of librsa.so: rectified block-sparse self-attention of a video DiT
 * (Rectified SpaAttn, arXiv 2511.19835) for one AMD MI355X (gfx950).
 *
 * One attention layer is three calls on one HIP stream, with no host synchronisation
 * in between (paper Alg. 1):
 *
 *   rsa_pool                   steps 1-11   pooling, implicit full attention (IPAR),
 *                                           compensation mask (GAPR)
 *   rsa_select_blocks          steps 13-14, 19   sparse mask, block lists, factor R
 *   rsa_sparse_attn_rectified  steps 16-23  block-sparse attention + rectification
 *
 * Conventions for every entry point
 *   - All tensor pointers are DEVICE pointers owned by the caller. The library never
 *     allocates, frees or synchronises; all work is enqueued on `stream` (a hipStream_t
 *     passed as void*; NULL is the default stream). Outputs are fully overwritten.
 *   - Q, K, V, O are bf16, token order [video | text] (Alg. 1 steps 1-2, 23), addressed as
 *     ptr[b*stride_b + h*stride_h + t*stride_t + c], c < head_dim contiguous. Strides are
 *     in elements and must be multiples of 8 (16-byte rows).
 *   - Blocks (Sec. 3.1): B = B^q = B^k = `block`. Video block m < N covers tokens
 *     [m*B, min((m+1)*B, T_v)); text block N+i covers [T_v + i*B, min(T_v + (i+1)*B, T)).
 *     N = ceil(T_v/B), M = N + ceil(T_t/B). Text always starts a block of its own (isolated
 *     pooling, Sec. 4.1); the last video and last text block may be ragged. Query blocks use
 *     the same partition: blocks n < N are the sparse rows, text query blocks run dense.
 *   - Pooled/score tensors are fp32, contiguous, batch-major then head-major:
 *     [batch][heads][...].  W = ceil(M/32) 32-bit words per bit-mask row, bit (m % 32) of
 *     word (m / 32) is block m; bits at m >= M are zero.
 *   - Return value: RSA_OK or a negative RSA_E_* code. Arguments are validated on the host
 *     before anything is launched: with any code but RSA_E_LAUNCH nothing has been enqueued.
 *     RSA_E_LAUNCH (the HIP runtime refused a kernel launch) may leave the kernels launched
 *     before the refused one enqueued; the outputs are then unspecified. No exceptions, no exit.
 *   - Results are deterministic (no atomics on any output path).
 */
#ifndef RSA_H
#define RSA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  RSA_OK = 0,
  RSA_E_NULL = -1,        /* a required pointer is NULL */
  RSA_E_SHAPE = -2,       /* non-positive sizes, misaligned strides */
  RSA_E_UNSUPPORTED = -3, /* head_dim or block outside {64,128}, M > RSA_MAX_BLOCKS,
                             block * stride_t * 2 bytes >= 2^31 */
  RSA_E_WORKSPACE = -4,   /* workspace smaller than rsa_workspace_bytes says */
  RSA_E_RANGE = -5,       /* sparsity / p / mode / flags out of range */
  RSA_E_LAUNCH = -6       /* the HIP runtime refused a launch */
};

#define RSA_MAX_BLOCKS 4096 /* largest M = key blocks per (batch, head) */
#define RSA_STATIC_SCRATCH_BYTES (16u << 20) /* scratch held per GPU for rsa_sparse_attn_rectified_static */

/* Problem statement of Alg. 1 ("Require": Q, K, V, T_v, T_t) plus the block size of Sec. 3.1. */
typedef struct rsa_shape {
  int32_t batch;     /* >= 1 */
  int32_t heads;     /* >= 1 */
  int32_t head_dim;  /* d: 64 or 128 */
  int32_t block;     /* B: 64 or 128 */
  int64_t t_video;   /* T_v >= 1 */
  int64_t t_text;    /* T_t >= 0 */
  int64_t stride_b, stride_h, stride_t; /* element strides of Q, K, V and O */
  float scale;       /* softmax scale; 0 selects 1/sqrt(d) (Sec. 3.1) */
} rsa_shape;

/* rsa_sparse_attn_rectified flags */
#define RSA_RECTIFY_CRITICAL 1 /* multiply video rows by R_n      (Alg. 1 step 20) */
#define RSA_COMPENSATE 2       /* add the pooled non-critical term (Alg. 1 steps 21-22) */
#define RSA_DENSE 4            /* ignore lists: every query block attends to all M blocks,
                                  no rectification (full attention, Sec. 3.1) */

/* Host only. N (video blocks), M (all key blocks) and W (mask words per row) for a shape. */
int rsa_block_counts(const rsa_shape* shape, int64_t* n_video_blocks, int64_t* n_blocks,
                     int64_t* mask_words);

/* Host only. Bytes of device scratch rsa_pool and rsa_sparse_attn_rectified need. */
int rsa_workspace_bytes(const rsa_shape* shape, size_t* pool_ws_bytes, size_t* attn_ws_bytes);

/*
 * Alg. 1 steps 1-11.
 *   Qp  [b][h][N][d]  block means of the video queries      (Sec. 3.2 pooled equations)
 *   Kp  [b][h][M][d]  block means of all key blocks; a text block's mean is only used by
 *                     the gain/error gate, never by the implicit attention
 *   Vp  [b][h][M][d]  block means of V                      (Alg. 1 step 3)
 *   Vt  [b][h][M][d][B] bf16: V of each key block stored channel-major so the P.V product
 *                     reads it like K; tokens past the end of a ragged block are zero.
 *                     Within every run of 16 tokens the two middle groups of four are
 *                     swapped (order 0-3, 8-11, 4-7, 12-15). Opaque to callers: pass it on
 *                     to rsa_sparse_attn_rectified.
 *   Spool [b][h][N][M] raw pooled scores  s^pool = q^pool . k^pool * scale   (Sec. 3.2)
 *   Lmass [b][h][N][M] block log-mass: s^pool + ln(c_m) for a video block (c_m = tokens in
 *                     the block), log-sum-exp over the block's individual token scores
 *                     q^pool . k_t * scale for a text block (Sec. 4.1, isolated pooling)
 *   Apool [b][h][N][M] implicit full attention A^pool = row-softmax(Lmass); equal to the
 *                     paper's reallocation: video block weights times block size, text
 *                     token weights summed per block, renormalised (Sec. 4.1)
 *   Mc_bits [b][h][N][W] compensation mask M_c (Sec. 4.2). gapr_mode 0: all zero;
 *                     2: all ones; 1: bit set iff  |s^pool| > DA + DB  with
 *                     DA = mean_i |(q_i - q^pool_n).k^pool_m| * scale and
 *                     DB = mean_j |q^pool_n.(k_j - k^pool_m)| * scale, i.e. the gain
 *                     |sum_ij s^pool| exceeds the first-order pooling error with the
 *                     absolute value taken per term (the printed signed sum vanishes).
 *   ws / ws_bytes     device scratch, at least pool_ws_bytes, 256-byte aligned.
 */
int rsa_pool(const rsa_shape* shape, const void* Q, const void* K, const void* V,
             float* Qp, float* Kp, float* Vp, void* Vt,
             float* Spool, float* Apool, float* Lmass, uint32_t* Mc_bits, int gapr_mode,
             void* ws, size_t ws_bytes, void* stream);

/*
 * The value part of rsa_pool alone (Alg. 1 step 3 for V): Vp and the channel-major copy Vt of a
 * new V, nothing else. For callers that keep the masks, lists, factors and A^pool of an earlier
 * call (the paper combines the method with caches across diffusion steps, Sec. 5 and appendix
 * "Implementations") and only
 * attend again with new tensors: rsa_pool_values(V') then rsa_sparse_attn_rectified(Q', K', Vt', ...).
 * Same layouts and ownership as in rsa_pool; Vp and Vt are fully overwritten.
 */
int rsa_pool_values(const rsa_shape* shape, const void* V, float* Vp, void* Vt, void* stream);

/*
 * Alg. 1 steps 5-7 alone (Sec. 3.2, Sec. 4.1): the implicit full attention from pooled vectors that
 * an earlier rsa_pool call left in Qp and Kp, together with the text keys of K -- Spool, Lmass and
 * Apool exactly as rsa_pool writes them, nothing else. For callers that re-derive A^pool from stored
 * pooled vectors, and the unit this stage is timed in. Same layouts and ownership as in rsa_pool; the
 * three outputs are fully overwritten.
 */
int rsa_implicit_attention(const rsa_shape* shape, const void* K, const float* Qp, const float* Kp,
                           float* Spool, float* Lmass, float* Apool, void* stream);

/*
 * Alg. 1 steps 13-14 and 19, per video query block n:
 *   keep the k = clamp(M - floor(sparsity*M + 1e-6), 1, M) blocks of largest Lmass (equal
 *   keys: lower block index first); if p > 0 extend, in the same descending order, until
 *   the kept A^pool weight exceeds p; OR with forced_bits (the adjacency mask M_adja,
 *   [b][h][N][W], may be NULL).
 *   mask_bits [b][h][N][W]  the sparse mask
 *   block_idx [b][h][N][M]  kept block indices, ascending, first count[n] entries valid
 *   count     [b][h][N]
 *   R         [b][h][N]     rectification factor: sum of A^pool over kept blocks (Sec. 4.1)
 * sparsity in [0,1], p in [0,1].
 */
int rsa_select_blocks(const rsa_shape* shape, const float* Lmass, const float* Apool,
                      double sparsity, double p, const uint32_t* forced_bits,
                      uint32_t* mask_bits, int32_t* block_idx, int32_t* count, float* R,
                      void* stream);

/*
 * Appendix "Implementations" (the token sequence is reordered before inference so that blocks
 * hold spatially close tokens): moves the rows of one [b][h][T][d] bf16 tensor between raster
 * order (token index (t*H + h)*W + w) and the tile order the other entry points expect (tiles of
 * `tile` in raster order over the (T, H, W) grid, tokens in raster order inside a tile). Text
 * rows [t_video, T) keep their place.
 *   direction 0: dst[tile-order position] = src[raster index]   (before the layer: Q, K, V)
 *   direction 1: dst[raster index] = src[tile-order position]   (after the layer: O)
 *   grid [3], tile [3]: HOST arrays; T*H*W must equal t_video. src and dst: device, both with the
 *   strides of `shape`, must not alias (RSA_E_RANGE). dst is fully overwritten.
 */
int rsa_reorder_tokens(const rsa_shape* shape, const int32_t* grid, const int32_t* tile, int direction,
                       const void* src, void* dst, void* stream);

/*
 * Alg. 1 "Require" and step 14, Sec. 4.3 (spatial-temporal neighbour blocks are always kept):
 * the adjacency mask M_adja for a video latent grid whose tokens are stored tile by tile
 * (tiles in raster order over (T, H, W), tokens in raster order inside a tile, partial tiles
 * at the upper faces of the grid). A video query block n and a video key block m are
 * neighbours when some tile touched by n and some tile touched by m differ by at most
 * `radius` in every tile coordinate (radius 1: the block itself and the surrounding 26 tiles
 * where blocks and tiles coincide). Text key blocks are never set.
 *   grid [3], tile [3]   HOST arrays (T, H, W) and (tile_t, tile_h, tile_w); T*H*W must equal
 *                        t_video (RSA_E_SHAPE otherwise); radius in [0, 64]
 *   forced_bits          device, [b][h][N][W] u32, fully overwritten (same rows for every b, h);
 *                        pass it to rsa_select_blocks
 */
int rsa_adjacency_mask(const rsa_shape* shape, const int32_t* grid, const int32_t* tile, int radius,
                       uint32_t* forced_bits, void* stream);

/*
 * Alg. 1 steps 16-23. For video query block n: online-softmax attention of its tokens over
 * the tokens of the blocks in block_idx[n][0..count[n]) only (masked keys are excluded from
 * the softmax, Sec. 3.1), times R[n] (RSA_RECTIFY_CRITICAL), plus
 * sum_{m: not mask and M_c} Apool[n][m] * Vp[m] (RSA_COMPENSATE). Text query blocks: full
 * attention over all tokens. O has the layout of Q. `lse` (nullable, [b][h][T] fp32)
 * receives the natural-log softmax denominator (including the row maximum) of the
 * un-rectified sparse/dense attention of every row.
 * With RSA_DENSE every list/mask/R/Apool/Mc/Vp pointer may be NULL.
 * ws / ws_bytes: device scratch of at least attn_ws_bytes, 256-byte aligned (RSA_E_WORKSPACE
 * otherwise). It receives the pooled compensation term C_n (fp32 [b][h][N][d], Alg. 1 step 21),
 * an order of the video query blocks (rows with similar lists next to each other, so that they
 * share K/V tiles in the L2 of their XCD), the schedule that deals the query blocks, in that
 * order and balanced by the length of their lists, to the resident workgroups of the attention
 * kernel, and fp32 buffers for the query blocks that the schedule cuts into pieces (where a few long rows
 * or an uneven last round would leave part of the chip idle). A query block that is cut adds the same terms in
 * another order, and each piece rounds its probabilities to bf16 against its own reference where the scores ask for one
 * other than 0, so that with and without a workspace the last bits may differ; for the same arguments and
 * workspace size the results are always the same. Required with RSA_COMPENSATE
 * (RSA_E_NULL); without that flag it may be NULL, and the query blocks are then dealt whole in index
 * order. With RSA_DENSE a workspace that is too small or misaligned is ignored (index order).
 * The caller owns it; its contents afterwards are unspecified.
 */
int rsa_sparse_attn_rectified(const rsa_shape* shape, const void* Q, const void* K, const void* Vt,
                              const int32_t* block_idx, const int32_t* count,
                              const uint32_t* mask_bits, const float* R, const float* Apool,
                              const uint32_t* Mc_bits, const float* Vp, int flags,
                              void* O, float* lse, void* ws, size_t ws_bytes, void* stream);

/*
 * For callers that cannot allocate device memory or hand over a workspace: code running under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc. Same computation, arguments and
 * error codes as rsa_sparse_attn_rectified, without ws / ws_bytes: the scratch (C_n, the
 * order of the query blocks and their schedule) lives in a device array of RSA_STATIC_SCRATCH_BYTES (16 MiB) that is part of the
 * library image, one copy per GPU, held until the process ends. The call allocates and frees nothing.
 * Its first call on a device looks up that device's copy (hipGetSymbolAddress; RSA_E_LAUNCH if that
 * fails). Results are those of rsa_sparse_attn_rectified, to the last bit where both cut the same query
 * blocks. Here none is cut where rsa_workspace_bytes asks for more than RSA_STATIC_SCRATCH_BYTES (the buffers of
 * the pieces do not fit then) nor under RSA_DENSE; the last bits may differ there.
 * Shapes are refused with RSA_E_WORKSPACE, before anything is enqueued, when C_n and the query block order,
 * 4 * batch * heads * N * (head_dim + 1) bytes, and 50 to 570 KB for the schedule (a word for each of twice the average
 * number of query blocks of a group of waves, and 32 KiB) exceed RSA_STATIC_SCRATCH_BYTES; 24 heads of 118 800 + 256
 * tokens at block 128, head_dim 128 take 11.7 MB.
 * Every call on a GPU uses that GPU's one array and overwrites all of it that it reads (nothing has
 * to start at zero); two calls that overlap in time on one GPU (different streams) race on it.
 * With RSA_DENSE the scratch is not touched (the query blocks are dealt in index order).
 */
int rsa_sparse_attn_rectified_static(const rsa_shape* shape, const void* Q, const void* K, const void* Vt,
                                     const int32_t* block_idx, const int32_t* count,
                                     const uint32_t* mask_bits, const float* R, const float* Apool,
                                     const uint32_t* Mc_bits, const float* Vp, int flags,
                                     void* O, float* lse, void* stream);

/*
 * The 8-bit key/value cache: keys and values of earlier frames or tokens, kept for queries that arrive
 * later (frame by frame, token by token). Four calls work on it:
 *
 *   rsa_cache_write    new keys and values into their pages
 *   rsa_cache_read     a range of tokens back in bf16
 *   rsa_cache_select   which blocks a group of query tokens reads, by a cheap score
 *   rsa_cache_attn     attention of new queries over all blocks, or over those lists
 *
 * A page holds one block of `block` tokens of all key/value heads; `table` says which page each block of
 * a sequence is. Entries that are no page (negative, or >= pages) hold no tokens: what is written there
 * is dropped, attention and selection pass over them, reading leaves those rows as they were. A page may stand in several places of
 * the table (a shared prefix) as long as no call writes it through two of them.
 *
 * Codes are e4m3 with one power-of-two scale for each (page, key/value head) of K and of V:
 *   value = code * 2^e,  e the least >= -126 with max |value| <= 448 * 2^e,  rounded to nearest even.
 * A token that joins a block that was begun earlier can only raise e; the older codes are then rounded
 * to the new scale. A block begun by the call (its first token among the new ones) takes its e
 * from the new tokens alone. Infinities and NaN are stored as NaN and count neither for e nor for the mean.
 * The mean of a page's keys (of the stored values of the tokens that it holds) is kept in 8 bits too:
 *   mean = int8 * 2^em,  em the least >= -100 with max |mean| <= 127 * 2^em.
 * Everything but the rounding to 4 (8) bits is exact, so that pages are the same bits however calls are cut,
 * up to values below 2^-6 of a block's scale that were rounded twice. (Values from 1.9375 * 2^127 on round to 2^128, which
 * bf16 does not hold: they are read back as infinity.)
 *
 * A page of the codes is opaque but for its size; `scales` is {2^eK, 2^eV, 2^em, 0}. Codes, scales and means need no initial
 * values, but a page is to be written before it is used: those that the table gives for the first kv_len[b] tokens by selection and
 * attention, those of a range by reading it, and by a write that begins inside a block the block's earlier tokens. Of a page
 * that was not, calls read whatever it holds: their results say nothing then, but stay within their buffers.
 */
typedef struct rsa_cache {
  int32_t batch;       /* sequences, >= 1 */
  int32_t heads_kv;    /* >= 1; batch * heads_kv <= 65535 */
  int32_t head_dim;    /* 64 or 128 */
  int32_t block;       /* tokens of a page: 64 or 128 */
  int32_t max_blocks;  /* entries of a row of the table, >= 1 */
  int64_t pages;       /* 1 .. 2^31 - 1 */
  void* k_codes;       /* device, [pages][heads_kv][block * head_dim] bytes, 16-byte aligned */
  void* v_codes;       /* the same */
  float* scales;       /* device, [pages][heads_kv][4], 16-byte aligned */
  int8_t* k_mean;      /* device, [pages][heads_kv][head_dim], 16-byte aligned */
  const int32_t* table;/* device, [batch][max_blocks] */
} rsa_cache;

/* Rows of new keys and values, or of queries and outputs: bf16 at ptr[b*stride_b + h*stride_h + t*stride_t + c],
 * strides in elements, multiples of 8; pointers 16-byte aligned. */
typedef struct rsa_rows {
  int32_t heads;       /* K, V: heads_kv. Q, O: a multiple of heads_kv; head h reads key/value head h / (heads / heads_kv) */
  int32_t t;           /* rows of a sequence, >= 1 (shorter sequences of a batch say so in `count` or `q_len`);
                          batch * heads * t < 2^28 and no more than 2^23 workgroups (RSA_E_UNSUPPORTED) */
  int64_t stride_b, stride_h, stride_t;
} rsa_rows;

#define RSA_CACHE_CAUSAL 1           /* a query sees the keys up to its own position */
#define RSA_CACHE_MAX_SELECT 16384   /* largest max_blocks of rsa_cache_select */

/* Host only. Bytes of k_codes (and of v_codes), of scales and of k_mean; the pointers in `cache` may be NULL here. */
int rsa_cache_bytes(const rsa_cache* cache, size_t* code_bytes, size_t* scale_bytes, size_t* mean_bytes);

/* Host only. Bytes of device scratch of rsa_cache_select and rsa_cache_attn for queries `rows` in groups of `group`
 * (0: no lists), whatever list_len. The pointers in `cache` may be NULL. */
int rsa_cache_workspace_bytes(const rsa_cache* cache, const rsa_rows* rows, int group, size_t* select_ws_bytes,
                              size_t* attn_ws_bytes);

/*
 * Tokens start[b] .. start[b] + count[b] - 1 of every sequence b (device int32 [batch]; count NULL: all rows->t,
 * more than rows->t counts as rows->t, less than 1 as none, a negative start as none) take rows 0 .. count[b] - 1 of K and V.
 * Tokens behind the table are dropped. Of the blocks that are touched, pages, scales and mean are renewed: tokens
 * before start[b] stay, what the block held from start[b] + count[b] on is gone (so a sequence may be taken
 * back to an earlier length by writing there).
 */
int rsa_cache_write(const rsa_cache* cache, const rsa_rows* rows, const void* K, const void* V, const int32_t* start,
                    const int32_t* count, void* stream);

/* The same range of tokens back into rows 0 .. count[b] - 1 of K and V (exact: a code has 4 significant bits).
 * Rows behind count[b], or of tokens without a page, are left as they were. */
int rsa_cache_read(const rsa_cache* cache, const rsa_rows* rows, const int32_t* start, const int32_t* count, void* K,
                   void* V, void* stream);

/*
 * Query token i < q_len[b] of sequence b stands at position kv_len[b] - q_len[b] + i; its own key is in the cache
 * by then (kv_len: device int32 [batch], tokens in the cache, less than 0 as 0; q_len NULL: all rows->t, more than rows->t
 * counts as rows->t). A query before position 0 sees no key under RSA_CACHE_CAUSAL. Tokens are taken in groups of `group` >= 1
 * from i = 0 on; a group and a key/value head have one list, for all query heads that share it.
 *   visible   the blocks of the first kv_len[b] tokens; with RSA_CACHE_CAUSAL up to the block of the group's last position
 *   score     q8 . mean * 2^em, q8 the sum of the group's queries over its tokens and heads (finite values), rounded
 *             to 8 bits as the means are; exact, so that equal scores are equal: the lower block goes first
 *   forced    blocks below `first`; and, where last >= 1, from `last` - 1 before the block of the group's first
 *             position to the block of its last one
 * Kept are the visible forced blocks and, by score, as many others as make `keep` in all.
 *   block_idx [batch][heads_kv][groups][list_len]  kept blocks, ascending, then -1;  groups = ceil(rows->t / group)
 *   kept      [batch][heads_kv][groups]            how many
 * list_len must be at least min(max_blocks, max(keep, first + last + ceil(group / block) + 1)) (RSA_E_RANGE).
 * max_blocks <= RSA_CACHE_MAX_SELECT (RSA_E_UNSUPPORTED). ws: select_ws_bytes, 256-byte aligned; may be NULL (slower where few groups score many blocks).
 */
int rsa_cache_select(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len,
                     const int32_t* q_len, int group, int keep, int first, int last, int flags, int32_t* block_idx,
                     int32_t* kept, int list_len, void* ws, size_t ws_bytes, void* stream);

/*
 * O = softmax(scale * Q K^T) V over the cached tokens that a query sees: the first kv_len[b], with RSA_CACHE_CAUSAL
 * those up to its own position; with lists (block_idx and kept not NULL, as rsa_cache_select leaves them, `group`
 * as there) of the listed blocks only. Entries of a list that are negative or behind the last visible block are passed over; a block
 * listed twice counts twice. scale 0 selects 1/sqrt(head_dim); scale * log2(e) is to be finite in fp32 (RSA_E_RANGE). A query
 * that sees no key gets 0 and a log-sum-exp of -inf. A NaN among the stored keys or values reaches the queries that see its token
 * and no others. Scores and sums are fp32 (queries times codes, that times 2^eK * scale, have to stay in its range), weights
 * are rounded to fp16: beside the rounding of O to bf16 and those of the fp32 steps an output is off by at most
 * sum max(2^-11 p, 2^-25) |v| / sum p, the largest p being 1, where the blocks that a row gives weight to are over scales within 2^60 of each other
 * (weights below 2^-25 may vanish, however large their values).
 * Without lists both pointers are NULL and `group` and `list_len` are ignored.
 *   O    as Q (may be Q). Rows behind q_len[b] are left as they were
 *   lse  (nullable) [batch][heads][t] fp32, natural log of the softmax denominator including the maximum
 *   ws   attn_ws_bytes, 256-byte aligned (RSA_E_WORKSPACE); NULL: the key axis is not split over workgroups (slower
 *        where there are few query rows; the last bits differ). A workspace belongs to one call at a time.
 */
int rsa_cache_attn(const rsa_cache* cache, const rsa_rows* rows, const void* Q, const int32_t* kv_len,
                   const int32_t* q_len, float scale, int flags, const int32_t* block_idx, const int32_t* kept, int group,
                   int list_len, void* O, float* lse, void* ws, size_t ws_bytes, void* stream);

/* Static string for a return code. */
const char* rsa_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* RSA_H */
