/*
 * mars_cache.h -- C ABI of the paged 4-bit key/value cache around the verification pass (AMD MI355X, gfx950).
 *
 * What a step of speculative decoding does with the cache, layer by layer: the keys and values of the drafted nodes
 * are put behind the committed tokens (mars_kv_append), every node attends the committed tokens and its own ancestors
 * (mars_tree_mask once per step, mars_kv_attention per layer); when mars_verify has chosen a path, the accepted nodes' rows
 * move up behind the committed ones and the rest is dropped (mars_kv_commit: the rollback of Sec. 3.4).
 * Sequences that branch share their pages until one of them writes (mars_kv_fork, mars_kv_reserve) and give
 * them back (mars_kv_release).
 *
 * The format.  A token's key (or value) of a head, dim channels, is dim/32 blocks of 32 channels.  A block is one byte e (its
 * scale is 2^(e - 127)) and 32 codes of 4 bits: sign, two bits of exponent, one of mantissa, standing for
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.  e is the least exponent at which the largest magnitude of the block is below
 * 7 scales (so that nothing is off by more than half a step), within 1 .. 252; codes are rounded to nearest, ties
 * to the even code.  A token whose key or value (of one head) holds a NaN or an infinity is stored with e = 255 in all
 * blocks of its key: it reads back as NaN, and the rows that see it become NaN; rows that do not see it are as they would be
 * without it.
 *
 * The pool.  [layers][pages][heads][page * (dim + dim/16)] bytes, 16-byte aligned; of a head in a page:
 *   keys' codes    [page][dim/2]            the even channel in the low half of a byte
 *   values' codes  [page/8][dim/8][8][4]    eight tokens' codes of the same eight channels beside each other
 *   keys' scales   [page][dim/32]
 *   values' scales [page/8][dim/32][8]
 *
 * The tables.  page_table [sequences][width]: the pages of a sequence, then -1.  lens [sequences]: committed tokens; the caller may lower it
 * between calls (the sequence goes on from an earlier token; its pages stay).
 * held [sequences]: pages in the table's row.  refs [pages]: how many sequences hold a page; a page is free exactly when that is
 * 0, there is no other list, and free pages are given out lowest first.  An empty cache is page_table = -1 and zeros in the other three.
 *
 * All pointers are DEVICE pointers unless stated.  The library keeps no state and allocates nothing; calls only enqueue work on the
 * given HIP stream.  No exceptions and no C++ types cross this boundary.
 */
#ifndef MARS_CACHE_H_
#define MARS_CACHE_H_

#include "mars.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Per-request status written by the device. */
enum {
  MARS_KV_OK           = 0,
  MARS_KV_NO_PAGES     = 1, /* not enough free pages (reserve); a token's page is missing (append): it was not written */
  MARS_KV_TOO_LONG     = 2, /* the sequence would need more pages than the table is wide */
  MARS_KV_BAD_SEQUENCE = 3, /* sequence number outside [0, sequences) */
  MARS_KV_BAD_PATH     = 4, /* accept_len outside [0, N), or path_idx not increasing within [1, N) */
  MARS_KV_NOT_EMPTY    = 5  /* the target of a fork holds pages */
};

/* Most requests per call. */
#define MARS_KV_MAX_REQUESTS 4096

/* The cache (a HOST struct; the pointers in it are device pointers).  A call that does not name a table may be given NULL for it. */
typedef struct mars_kv_cache {
  void*    pool;
  int32_t* page_table;
  int32_t* lens;
  int32_t* held;
  int32_t* refs;
  int32_t  layers, pages, heads;
  int32_t  dim;       /* 64, 128 or 256 */
  int32_t  page;      /* tokens: a power of two, 8 .. 256 */
  int32_t  sequences, width;
} mars_kv_cache;

/* Rows [B][N][heads][dim] (a HOST struct): element [b][i][h][c] is data[b*request + i*node + h*head + c].  Strides in elements, multiples of
 * 16 bytes; data 16-byte aligned. */
typedef struct mars_kv_rows {
  void*   data;
  int64_t request, node, head;
} mars_kv_rows;

/* Bytes of a head in a page (times heads: of a page in a layer); 0 if dim or page is not supported. */
size_t mars_kv_head_bytes(int dim, int page);

/*
 * The rows k, v of N new tokens per request into `layer`, at positions lens[s] .. lens[s] + n_new[b] - 1 of sequence s = seqs[b].
 * lens is not changed: the rows of a drafted tree lie behind the committed tokens until mars_kv_commit.
 *   seqs      [B], or NULL: request b is sequence b.  Sequences of a call differ from each other.
 *   dtype     MARS_F32 or MARS_BF16, of k and v.
 *   n_new     [B], 0 <= n_new[b] <= N, or NULL: N for all.
 *   status    out, optional, [B]: MARS_KV_OK, MARS_KV_BAD_SEQUENCE, or MARS_KV_NO_PAGES where a row's page is missing (the others
 *             are written).
 * Reads page_table, lens.  The pages written must not be shared (mars_kv_reserve sees to that).
 */
int mars_kv_append(const mars_kv_cache* cache, int layer, const int32_t* seqs, const mars_kv_rows* k, const mars_kv_rows* v,
                   int dtype, const int32_t* n_new, int B, int N, int32_t* status, void* hip_stream);

/*
 * Keys and values of positions first[b] .. first[b] + N - 1 (NULL: from 0 on) as rows of `dtype`; both types hold them exactly.
 * Positions without a page -- in front of 0, past the table or past held (if given) -- read as zero.  Reads page_table.
 */
int mars_kv_read(const mars_kv_cache* cache, int layer, const int32_t* seqs, const int32_t* first, const mars_kv_rows* k,
                 const mars_kv_rows* v, int dtype, int B, int N, void* hip_stream);

/*
 * What the nodes of drafted trees see of each other: bit j of mask[b][i] (word j/64) is set iff node j is node i or one of its ancestors.
 *   tree_parent  [B][N] as for mars_verify; N <= MARS_MAX_NODES.
 *   n_new        [B], or NULL: N for all.  Nodes from n_new[b] on see nothing and are seen by none.
 *   mask         out, [B][N][(N + 63)/64] uint64.
 *   status       out, optional, [B]: MARS_REQ_OK or MARS_REQ_BAD_TREE (parent[0] != -1, or parent[i] not in [0, i)): then no node but the
 *                root sees any.
 */
int mars_tree_mask(const int32_t* tree_parent, const int32_t* n_new, int B, int N, uint64_t* mask, int32_t* status, void* hip_stream);

/*
 * Attention of N query rows per request (the nodes that mars_kv_append put behind the committed tokens) over the cache:
 *   out[b][i][h] = sum_j p_j v_j,  p = softmax_j(scale * q[b][i][h] . k_j),  keys and values of cache head h / (q_heads / heads),
 * over the committed tokens j < lens[s] and the nodes that row i sees.  A row that sees nothing gets zeros.
 *   q, out     rows [B][N][q_heads][dim] of `dtype` (MARS_F32 or MARS_BF16); q_heads a multiple of heads, at most 64 times it.
 *   lse        out, optional, [B][N][q_heads] fp32: log sum_j exp(scale * q.k_j); -inf for a row that sees nothing.
 *   n_new      [B], or NULL: N for all.  Rows from n_new[b] on see nothing, not even committed tokens.
 *   mask       [B][N][(N + 63)/64] uint64, bit j of row i: row i sees node j (any mask; mars_tree_mask makes a tree's); N <= MARS_MAX_NODES.
 *              NULL: a chain, row i sees nodes 0 .. i; any N.
 *   scale      > 0, and scale * log2(e) finite in fp32.
 *   max_len    HOST: what the lens are expected not to exceed; 0: the table's width times page.  It only guides how the work is split:
 *              longer sequences are attended in full.
 *   workspace  256-byte aligned, >= mars_kv_attention_workspace_bytes(...); scratch, calls that share it must not overlap.
 * Scores, softmax statistics and sums are held in fp32.  For bf16 rows the probabilities are rounded to bf16 in front of the
 * product with the values (a relative error of at most 2^-8 per key; equal ones are rounded the same way); for fp32 rows they and the queries go through the
 * matrix cores as three bf16 terms each (a query beyond bf16's largest number, 3.39e38, makes its row NaN).  Scores are those of fp32: q.k beyond its range is
 * infinite, whatever scale makes of it.  Results are reproducible bit for bit.
 * A sequence number outside the cache gives rows of zeros (without seqs: requests from `sequences` on); a page number outside it among a row's keys gives NaN.
 * Reads page_table, lens.
 */
size_t mars_kv_attention_workspace_bytes(int B, int N, int q_heads, int heads, int dim, int dtype);
int mars_kv_attention(const mars_kv_cache* cache, int layer, const int32_t* seqs, const mars_kv_rows* q, int dtype, int q_heads,
                      const int32_t* n_new, const uint64_t* mask, float scale, int max_len, const mars_kv_rows* out, float* lse,
                      int B, int N, void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * After verification: in every layer the row of the i-th accepted node (behind the committed tokens at path_idx[b][i]) moves to position
 * lens[s] + 1 + i, behind the root's; new_lens[s] = lens[s] + 1 + accept_len[b].
 *   accept_len, path_idx   [B], [B][N] as mars_verify writes them.
 *   new_lens   out, [sequences]; only the sequences of the call are written.  May be lens itself.
 *   status     out, optional, [B]: MARS_KV_OK, MARS_KV_BAD_SEQUENCE, MARS_KV_BAD_PATH or MARS_KV_NO_PAGES (a row's page, or the
 *              root's, is missing).  With one of the last two nothing is moved and new_lens[s] = lens[s].
 * The pages behind the new length stay with the sequence (the next step's nodes go there).  Reads page_table, lens.
 */
int mars_kv_commit(const mars_kv_cache* cache, const int32_t* seqs, const int32_t* accept_len, const int32_t* path_idx, int B, int N,
                   int32_t* new_lens, int32_t* status, void* hip_stream);

/*
 * Room for n_new[b] (NULL: N) tokens behind lens[s], in pages that are the sequence's own: pages are added to its row, and a page in the row that these
 * tokens go into and that others hold too is replaced by a free one -- the first of them, if committed tokens are in it, by a copy in all
 * layers.  Where all holders of a page write it in one call, the last of them keeps the page.  Free pages are given out lowest first, request by
 * request: in place of shared ones in the order of the row, then the added ones.
 *   status     out, optional, [B]: MARS_KV_OK, MARS_KV_BAD_SEQUENCE, MARS_KV_TOO_LONG, or MARS_KV_NO_PAGES; other than OK:
 *              nothing was changed for this request.  When the pages run out, every later request that needs one goes without, and so
 *              does the last holder of a page of which an earlier one did not get its own.
 *   workspace  256-byte aligned, >= mars_kv_reserve_workspace_bytes(pages, B).
 * Sequences of a call differ from each other.  Reads and writes all tables.
 */
size_t mars_kv_reserve_workspace_bytes(int pages, int B);
int mars_kv_reserve(const mars_kv_cache* cache, const int32_t* seqs, const int32_t* n_new, int B, int N, int32_t* status, void* workspace,
                    size_t workspace_bytes, void* hip_stream);

/*
 * Sequence dst[b] becomes a copy of src[b]: it holds the pages of its committed tokens too.  No row is copied.
 * dst sequences are empty (held = 0), differ from each other, and none of them is among the src.
 *   status     out, optional, [B]: MARS_KV_OK, MARS_KV_BAD_SEQUENCE, MARS_KV_NOT_EMPTY.
 */
int mars_kv_fork(const mars_kv_cache* cache, const int32_t* src, const int32_t* dst, int B, int32_t* status, void* hip_stream);

/* The sequences give their pages back and are empty.  status out, optional, [B]: MARS_KV_OK, MARS_KV_BAD_SEQUENCE. */
int mars_kv_release(const mars_kv_cache* cache, const int32_t* seqs, int B, int32_t* status, void* hip_stream);

/* Page dst[i] becomes a copy of page src[i] in all layers; pairs with a number outside [0, pages) are skipped.  dst pages differ from each other
 * and from the src.  Reads and writes the pool only. */
int mars_kv_copy_pages(const mars_kv_cache* cache, const int32_t* src, const int32_t* dst, int n, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* MARS_CACHE_H_ */
