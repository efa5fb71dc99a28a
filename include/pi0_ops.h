/*
 * pi0_ops.h - operators on a paged key/value cache (same shared library as pi0.h).
 *
 * pi0_prefill leaves the prefix's keys and values inside a ctx, where only the action expert reads them.  These entry
 * points are what the language half needs to go on from there: a cache of many sequences in pages that the caller owns
 * (pi0_pages_reserve, _fork, _compact), the way between it and a ctx (pi0_pages_store, pi0_pages_load), norm and
 * rotation of new tokens' queries and keys together with their place in the cache (pi0_qk_norm_rope), and the attention
 * of a tree of drafted tokens - one token, in the simplest case - over it (pi0_tree_attention).
 *
 * One step of drafting over it, for every layer l:     reserve -> { qk_norm_rope(l) -> tree_attention(l) } -> compact
 *
 * Conventions are those of pi0.h: d_* are device pointers that the caller owns, calls only enqueue work on hip_stream
 * and allocate nothing, argument checks come before any GPU call, nothing throws or aborts.  The pointers and the stream belong to the
 * device that is current.  No call needs a ctx except store and load.  The caller may capture any of them into a HIP graph, except
 * pi0_pages_status, which waits, and store and load, which go by what the ctx holds at the time of the call and refuse a stream that is
 * being captured (PI0_EHIP, hipErrorIllegalState).  Calls that overlap in time must not share a workspace, nor may one change a cache that
 * another reads; a graph keeps the addresses it was captured with, its workspace included.
 * PI0_EHIP is a failure of the call's own launches, whatever error an earlier call of the caller's has left; a part of the work may
 * have run by then, and a cache that pi0_pages_reserve or _compact was to change is no longer to be used.
 * Results do not depend on what else runs: no sums by atomics, pages are handed out in one fixed order.
 */
#ifndef PI0_OPS_H
#define PI0_OPS_H

#include "pi0.h"

#ifdef __cplusplus
extern "C" {
#endif

enum pi0_dtype { PI0_BF16 = 0, PI0_F16 = 1, PI0_F32 = 2 };

/*
 * A paged cache: n_seqs sequences, each a list of pages out of one pool, the same list for every layer.
 * Position p of sequence s is row p % page_tokens of page table[s][p / page_tokens].
 *   - table[s] holds the sequence's pages in front and -1 behind them.  Entries outside [0, n_pages) end the list where
 *     pages are counted, and are positions that nobody sees or writes everywhere else.
 *   - length[s] counts the positions that are there for good ("committed").  New tokens stand behind them, in pages that
 *     pi0_pages_reserve has taken, until pi0_pages_compact commits those that stay.
 *   - refs[p] counts the sequences that hold page p; 0: free.  Free pages are taken in ascending order.
 * An empty cache: table all -1, length and refs all 0.
 * Strides are in elements, multiples of 8, of the same layout for keys and values; the head_dim elements of a row are
 * contiguous.  The rows must not overlap; token_stride is below 2^27.
 */
typedef struct pi0_pages {
  void* d_k;             /* keys; 16-byte aligned                                                     */
  void* d_v;             /* values; 16-byte aligned                                                   */
  int32_t* d_table;      /* [n_seqs][max_pages]                                                       */
  int32_t* d_length;     /* [n_seqs]                                                                  */
  int32_t* d_refs;       /* [n_pages]                                                                 */
  int32_t* d_status;     /* [1], 0 at first: what pi0_pages_status reports                            */
  int64_t layer_stride, page_stride, token_stride, head_stride;
  int32_t dtype;         /* PI0_BF16 or PI0_F16                                                       */
  int32_t layers;        /* 1 .. 65536, layers * kv_heads * head_dim <= 2^29                          */
  int32_t n_pages;       /* 1 .. 2^24                                                                 */
  int32_t page_tokens;   /* 16, 32, 64, 128 or 256                                                    */
  int32_t kv_heads;      /* 1 .. 256                                                                  */
  int32_t head_dim;      /* 64, 128 or 256                                                            */
  int32_t n_seqs;        /* 1 .. 1024                                                                 */
  int32_t max_pages;     /* >= 1, max_pages * page_tokens <= 2^24                                     */
} pi0_pages;

/*
 * Rows of heads: element e of head h of row r at d_x[r * row_stride + h * head_stride + e], strides in elements.
 * The new tokens of all sequences lie behind each other, those of sequence s in rows row_start[s] .. row_start[s + 1] - 1
 * (d_row_start int32 [n_seqs + 1], ascending); at most max_rows of a sequence are taken.  Rows that belong to no sequence, or
 * lie outside [0, n_rows), are neither read nor written.  n_rows is 1 .. 2^24, max_rows 1 .. n_rows: a call without a new token is none.
 */
typedef struct pi0_rows {
  void* d_x;             /* 16-byte aligned                                                           */
  int64_t row_stride, head_stride;   /* multiples of 8, at least head_dim                             */
  int32_t heads;
  int32_t dtype;         /* pi0_dtype                                                                 */
} pi0_rows;

/* Bytes of device workspace (16-byte aligned) of pi0_pages_reserve and pi0_pages_compact; 0 if *pages is invalid. */
size_t pi0_pages_workspace_bytes(const pi0_pages* pages);

/*
 * Room for d_extra[s] (int32 [n_seqs], device) more positions behind length[s]; a negative entry leaves the sequence
 * as it is.  Takes free pages where the sequence holds too few, and gives it its own copy of a page that others hold as
 * well and that the new positions will be written to (all layers, the committed rows).  Pages that become free do so for
 * the next call.
 * Failing on the device - reported by pi0_pages_status, and nothing is changed then, for no sequence: PI0_ENOMEM (not
 * enough free pages), PI0_EINVAL (more positions than max_pages hold, a length beyond the pages that are held).
 * Errors: EINVAL, ENOMEM (workspace), EHIP.
 */
int pi0_pages_reserve(const pi0_pages* pages, const int32_t* d_extra, void* d_workspace, size_t ws_bytes, void* hip_stream);

/*
 * Sequence d_dst[i] becomes a continuation of sequence d_src[i], i < n (int32 [n], device; 1 <= n <= n_seqs): it holds the
 * same pages up to the committed length and lets go of those it held.  Nothing is copied before one of the two is
 * written to (see pi0_pages_reserve).
 * Failing on the device, nothing changed: PI0_EINVAL (an index outside [0, n_seqs), a dst that occurs twice or is a src
 * of the same call, a source whose length goes beyond its pages).  Errors: EINVAL, EHIP.
 */
int pi0_pages_fork(const pi0_pages* pages, const int32_t* d_src, const int32_t* d_dst, int n, void* hip_stream);

/*
 * Keeps, of what sequence s holds from position start on, the positions start + keep[s][0], start + keep[s][1], ... of
 * d_n_keep[s] entries, moves them up to start, start + 1, ... in every layer, sets length[s] = start + n_keep[s] and
 * lets go of the pages behind.  start = d_start[s], or length[s] where d_start is NULL.
 *   accept drafts           start = length, keep = the accepted nodes
 *   drop tokens             start < length, keep = what stays
 *   cut to t, free all      start = t (0), n_keep = 0
 *   d_keep    int32 [n_seqs][keep_stride], strictly ascending from 0 on in each row; may be NULL iff keep_stride == 0
 *   d_n_keep  int32 [n_seqs]; negative: the sequence stays as it is
 * Pages that others hold too are not written: rows that move into one get a free page of their own.
 * Failing on the device, nothing changed: PI0_ENOMEM (free pages), PI0_EINVAL (n_keep > keep_stride, start outside
 * [0, length], entries not ascending or beyond the pages that are held).
 * Errors: EINVAL, ENOMEM (workspace), EHIP.
 */
int pi0_pages_compact(const pi0_pages* pages, const int32_t* d_start, const int32_t* d_keep, int keep_stride, const int32_t* d_n_keep,
                      void* d_workspace, size_t ws_bytes, void* hip_stream);

/*
 * The prefix that the last pi0_prefill / pi0_infer / pi0_stream_frame / pi0_pages_load left in ctx, as the contents of sequence seq: its keys
 * (rotated) and values of all layers into the sequence's pages, length[seq] = its tokens.  The pages must be there (pi0_pages_reserve on
 * the emptied sequence) and be the sequence's own.  Store and load are ordered by their stream alone, as pi0_prefill is: between
 * frames, and in front of the first, both belong on stream_prefill.
 * Needs kv_heads 1, head_dim 256, PI0_BF16 and layers = llm_layers.  Failing on the device, nothing changed: PI0_ENOMEM
 * (too few pages), PI0_EINVAL (a page that others hold too).  Errors: EINVAL, ESTATE (no valid prefill, or
 * another device than that of pi0_load_weights is current), EHIP.
 */
int pi0_pages_store(pi0_ctx* ctx, const pi0_pages* pages, int seq, void* hip_stream);

/*
 * The way back: the first n_tokens positions of sequence seq become the ctx's prefix, as if pi0_prefill had left them
 * there; pi0_denoise (and the denoise half of the next pi0_stream_frame, if the load was on its stream_prefill) then runs against them, its
 * suffix at position n_tokens.  Any number from one view's tokens up to max_views * tokens per view + max_prompt, for instance a prefix
 * stored earlier, or one with decoded tokens behind it.  Positions without a page are zero.
 * Errors: EINVAL (also: another geometry than pi0_pages_store takes), ESTATE (weights not loaded, or another device is current), EHIP.
 */
int pi0_pages_load(pi0_ctx* ctx, const pi0_pages* pages, int seq, int n_tokens, void* hip_stream);

/*
 * Synchronises hip_stream and returns what the last operation that failed on the device reported (PI0_OK: none did
 * since the last call), and clears it.  Errors: EINVAL, EHIP.
 */
int pi0_pages_status(const pi0_pages* pages, void* hip_stream);

/*
 * Norms of queries and keys for each head, with the position rotation in the same pass; keys and values go to their
 * place in the cache.  For token j of sequence s (row row_start[s] + j), x a head of q or k:
 *     y = x / sqrt(mean(x^2) + eps) * (gain_offset + gain)                         (gain NULL: y = x)
 *     (y[a], y[b]) <- (y[a] cos t - y[b] sin t, y[a] sin t + y[b] cos t),          t = position * rope_base^(-2 i / rope_dim)
 * for i < rope_dim / 2 with (a, b) = (i, i + rope_dim / 2), or (2 i, 2 i + 1) if interleaved.  Rotated queries go to
 * `out`, rotated keys and the values (as they are) to position length[s] + j of layer `layer`; where the sequence has no
 * page for it, key and value are dropped.  Arithmetic in fp32, angles in fp64 turns, one rounding at the end.
 *   q, out      n_rows rows of q->heads heads; out of the cache's type, and may be q itself
 *   k, v        n_rows rows of kv_heads heads.  q, k, v: all of one type, the cache's or PI0_F32; they may be slices of one row
 *   d_position  int32 [n_rows] (drafts of a tree: length + depth), or NULL: the position in the cache
 *   d_q_gain, d_k_gain   float32 [head_dim], 16-byte aligned, or NULL
 *   rope_dim    0 .. head_dim, a multiple of 8; 0: no rotation
 * Errors: EINVAL, EHIP.
 */
int pi0_qk_norm_rope(const pi0_pages* pages, int layer, const pi0_rows* q, const pi0_rows* k, const pi0_rows* v, const pi0_rows* out,
                     const int32_t* d_row_start, int n_rows, int max_rows, const int32_t* d_position, const float* d_q_gain,
                     const float* d_k_gain, float gain_offset, float eps, int rope_dim, double rope_base, int interleaved, void* hip_stream);

/*
 * Attention of each sequence's new tokens over its committed positions and each other.  Token i of sequence s sees all
 * positions below length[s], and of the tokens j < min(number of tokens, max_rows) whose keys and values stand at
 * length[s] + j those with bit j % 32 of mask[row of i][j / 32] set - its ancestors in the tree of drafts and itself -, or all
 * j <= i without a mask.  Heads h of q share key/value head h / (heads / kv_heads).
 *     out = sum_j softmax_j(scale * q . k_j) v_j        over what the token sees; 0 if that is nothing
 * What a token does not see does not reach it, whatever is stored there (a NaN, an unwritten page).
 *   q, out    n_rows rows of `heads` heads, a multiple of kv_heads; both of the cache's type; out may be q itself
 *   max_rows  most new tokens of a sequence, 1024 at most; n_seqs * kv_heads * ceil(max_rows * heads / kv_heads / 16) *
 *             (max_pages * page_tokens / 32 + 7) below 2^30
 *   d_mask    uint32 [n_rows][mask_words], 1 .. 32 words, or NULL (mask_words 0); bits behind the last word are clear
 *   scale     any number of magnitude below 2^127
 * Products on matrix cores with fp32 sums, softmax in fp32, its weights rounded to the cache's type in front of the second
 * product.  The workspace is scratch of this call: 16-byte aligned, pi0_tree_attention_workspace_bytes
 * of the same arguments (0: invalid arguments).  Errors: EINVAL, ENOMEM (workspace), EHIP.
 */
size_t pi0_tree_attention_workspace_bytes(const pi0_pages* pages, int heads, int n_rows, int max_rows);
int pi0_tree_attention(const pi0_pages* pages, int layer, const pi0_rows* q, const pi0_rows* out, const int32_t* d_row_start, int n_rows,
                       int max_rows, const uint32_t* d_mask, int mask_words, float scale, void* d_workspace, size_t ws_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* PI0_OPS_H */
