/*
 * qwen3_decode.h - what answers are generated with (qwen3.h's conventions hold
 * here): a paged cache of keys and values, attention of new tokens over it, and
 * the adjustment of logits before a token is chosen; the calls that a program
 * makes by itself, and those that put the cache into the Qwen3-shaped model's
 * forward. Calls without a model take the stream to enqueue on; it belongs to
 * the current device, and so do the pointers. Nothing here synchronises:
 * lengths, page tables and counts are read on the device, so that a captured
 * call goes on with what they hold when it is replayed.
 * qwen3_last_error(NULL) says why a call failed.
 */
#ifndef QWEN3_DECODE_MI355X_H
#define QWEN3_DECODE_MI355X_H

#include "qwen3.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A cache of the keys and values of n_seq sequences in n_layer layers. A page
 * holds page_size tokens in every layer; a sequence's tokens are on the pages
 * of its row of the table, in order. Sequences may share pages. All buffers are
 * the caller's; the calls keep these rules, and so must whoever fills them:
 *  - d_table[s][i] is a page below n_pages for i < ceil(d_lens[s] / page_size),
 *    and -1 behind;
 *  - d_refs[p] is how many places of the table hold page p; 0: it is free.
 * An empty cache has -1, 0 and 0 there; d_pages needs no initial value. What a
 * table holds outside [0, n_pages) is read as a page whose tokens nobody sees.
 * Calls on one cache run one after another. Forking, appending and compacting
 * change it (attention does not). */
typedef struct qwen3_cache {
  int32_t n_layer, n_kv_head, head_dim;   /* 65535 and 4096 at most; head_dim 64 or 128 */
  int32_t page_size;                      /* 16, 32, 64, 128 or 256 */
  int32_t n_pages, n_seq, max_pages;      /* pages, below 2^28; sequences, 4096 at most; pages of a sequence,
                                             max_pages * page_size below 2^30 */
  void* d_pages;      /* bf16 [n_layer][n_pages][2: keys, values][n_kv_head][page_size][head_dim], 16-byte aligned */
  int32_t* d_table;   /* [n_seq][max_pages] */
  int32_t* d_lens;    /* [n_seq], tokens of each sequence */
  int32_t* d_refs;    /* [n_pages] */
  int32_t* d_short;   /* [1], see qwen3_cache_append */
  void* d_scratch;    /* qwen3_cache_scratch bytes, 16-byte aligned, scratch of the calls that change the cache */
} qwen3_cache;
gpt2_status qwen3_cache_scratch(const qwen3_cache* c, size_t* bytes_out);

/* Every sequence s becomes the first min(d_keep[s], length) tokens of what
 * sequence d_src[s] was before the call: forking, reordering, truncating. A
 * d_src[s] outside [0, n_seq) frees s. d_keep NULL: all tokens; negative: none.
 * No tokens are copied: pages are shared, and free once nobody has them. */
gpt2_status qwen3_cache_fork(const qwen3_cache* c, const int32_t* d_src,
                             const int32_t* d_keep, void* hip_stream);

/* New tokens' keys and values, of every layer, behind those of their sequences.
 * d_qkv: bf16 [n_layer][n_rows] rows q [n_head * head_dim] | k [n_kv_head *
 * head_dim] | v likewise, layers layer_stride elements apart (a multiple of 8,
 * 2^40 at most), 16-byte aligned, n_head a positive multiple of n_kv_head, 4096
 * at most, n_rows below 2^28. Sequence s has rows
 * d_starts[s]..d_starts[s+1]-1 (d_starts int32 [n_seq + 1], within 0..n_rows,
 * not falling). It takes the first d_counts[s] of them (NULL: all), or, with
 * d_path int32 [n_seq][max_new], rows d_starts[s] + d_path[s][i], i <
 * d_counts[s] (a tree's accepted tokens); a path entry that is not among the
 * sequence's rows leaves its token's place in the cache as it was. No sequence
 * takes more than max_new, which is below 2^22, or small enough that n_seq *
 * max_new is below 2^25; with d_path the latter in any case.
 * Pages are taken from the free ones, the lowest numbers first, for the
 * sequences in their order. Tokens on a last page that others have too are
 * copied to one of its own first. d_short receives the number of pages that
 * were missing (in the pool, or in the rows of the table); unless it is 0, the
 * call changes nothing else. */
gpt2_status qwen3_cache_append(const qwen3_cache* c, const void* d_qkv,
                               int32_t n_head, int32_t n_rows,
                               size_t layer_stride, const int32_t* d_starts,
                               const int32_t* d_counts, const int32_t* d_path,
                               int32_t max_new, void* hip_stream);

/* With U pages in use, those numbered U and above move to the free numbers
 * below U, the lowest to the lowest, in every layer, and the table and the
 * counts follow: afterwards pages 0..U-1 are in use. */
gpt2_status qwen3_cache_compact(const qwen3_cache* c, void* hip_stream);

/* Attention of new tokens over one layer of the cache and among themselves.
 * Rows as above (one layer's, d_qkv bf16 [n_rows][(n_head + 2 n_kv_head)
 * head_dim], already turned by their positions); their own keys and values are
 * read from the rows, not from the cache. A token sees all of its sequence's
 * tokens in the cache, and of the new tokens of its sequence
 *   without d_mask those up to itself (one token, a piece of a prompt),
 *   with d_mask, int32 [n_rows][mask_words], token j where bit j % 32 of word
 *     j / 32 of its row is set (a tree of drafts: a token and its ancestors).
 * What it does not see does not reach it, whatever it holds; a row that sees
 * nothing gets 0 and an lse of -infinity. Query head h reads key/value head h /
 * (n_head / n_kv_head); scores are scaled by 1/sqrt(head_dim).
 * d_out bf16 [n_rows][n_head * head_dim], 16-byte aligned; d_lse fp32
 * [n_head][n_rows], the log-sum-exp of the scaled scores, or NULL. Neither
 * overlaps an input or the other. Of every sequence's rows the first max_new
 * are computed; other rows are left as they were. d_workspace:
 * qwen3_tree_size bytes, 256-byte aligned, scratch until the call's kernels have
 * run: calls that may run at the same time take one each.
 * The work that the capacities allow is counted in 32 bits: (max_pages *
 * page_size + max_new + 64) / 32 * (n_head * n_rows / 32 + n_kv_head * n_seq) up
 * to 2 * 10^9 is taken, what is much beyond is INVALID_ARG. */
typedef struct qwen3_tree {
  int32_t n_head, n_rows;   /* n_head * n_rows below 2^26 */
  int32_t max_new;       /* no sequence has more new tokens; below 2^28 */
  int32_t layer;         /* of the cache */
  int32_t mask_words;    /* 2^20 at most; not looked at without d_mask */
} qwen3_tree;
gpt2_status qwen3_tree_size(const qwen3_cache* c, const qwen3_tree* t,
                            size_t* bytes_out);
gpt2_status qwen3_tree_attention(const qwen3_cache* c, const qwen3_tree* t,
                                 const void* d_qkv, const int32_t* d_starts,
                                 const int32_t* d_mask, void* d_out,
                                 float* d_lse, void* d_workspace,
                                 size_t workspace_bytes, void* hip_stream);

/* The rows' positions, int32 [n_rows]: a sequence's tokens in the cache, plus the
 * new tokens that the row sees besides itself (in order: those before it; with
 * a mask: its set bits less one); 0 for rows of no sequence. For
 * qwen3_rotary_forward, before the rows go into the attention. */
gpt2_status qwen3_tree_positions(const qwen3_cache* c, const qwen3_tree* t,
                                 const int32_t* d_starts,
                                 const int32_t* d_mask, int32_t* d_positions,
                                 void* hip_stream);

/* The cache in the model's forward, from the next qwen3_forward on: its B*T
 * tokens are the rows of qwen3_tree_attention (c's sequences; n_layer, n_kv_head
 * and head_dim the model's), rows of no sequence are padding whose results mean
 * nothing. Attention of layer l is over the cache's layer l. Positions are those
 * of qwen3_tree_positions, worked out by every forward, unless
 * qwen3_set_positions gives others. The forward takes no targets and no
 * backward follows it; with a config whose loss_from is 0, qwen3_logits_info has
 * the logits of every row. d_starts and d_mask (or NULL) are read by every
 * forward, the caller's to keep, like the cache's buffers; c itself is copied.
 * d_workspace: qwen3_set_cache_size bytes, 256-byte aligned, the caller's to
 * keep while the cache is in use, by graphs too. c NULL goes back to the
 * forward without a cache. INVALID_ARG for what is not as said here, and while a
 * layout is set (qwen3_set_layout). */
gpt2_status qwen3_set_cache_size(const qwen3_model* m, const qwen3_cache* c,
                                 int32_t max_new, size_t* bytes_out);
gpt2_status qwen3_set_cache(qwen3_model* m, const qwen3_cache* c,
                            const int32_t* d_starts, const int32_t* d_mask,
                            int32_t mask_words, int32_t max_new,
                            void* d_workspace, size_t workspace_bytes);
/* qwen3_cache_append of the last forward's rows to the cache that it read, on
 * the model's stream. STATE without such a forward. Of every sequence's rows
 * that forward computed the first max_new that qwen3_set_cache was given:
 * without d_path a larger max_new is INVALID_ARG, and a path entry that names a
 * row behind them is one that is not among the sequence's rows. */
gpt2_status qwen3_keep_tokens(qwen3_model* m, const int32_t* d_counts,
                              const int32_t* d_path, int32_t max_new);
/* Where the last forward's logits are: bf16 [rows][vocab] at *offset_bytes of
 * the activations, the positions with loss in order. STATE unless the last
 * forward had no targets (with targets their gradients are there). */
gpt2_status qwen3_logits_info(const qwen3_model* m, size_t* offset_bytes,
                              int32_t* rows);

/* Logits as the choice of a token wants them. For every row r with history row
 * h = d_row_seq[r] (NULL: r), x its logits and, of token v,
 *   seen:  v is among the first d_lens[h] tokens of d_history[h], or in d_path[r];
 *   count: how often it is there from place d_prompt_lens[h] on, or in d_path[r]:
 *   x_v <- x_v > 0 ? x_v / repetition : x_v repetition     where seen
 *   x_v <- x_v - frequency count - presence                where count > 0
 *   x_v <- x_v + bias                                      of the last entry that names v
 *   x_v <- -infinity                                       where mask d_row_mask[r] lacks bit v
 * in fp32, rounded once. Entries outside [0, vocab) name no token. Penalties are
 * a value a row, each array or NULL for none (1, 0, 0). A d_row_seq outside
 * [0, n_seq) is a row without a history; a d_row_mask outside [0, n_masks) a row
 * without a mask. d_logits and d_out: bf16 (dtype 1) or fp32 (dtype 0) [rows],
 * rows logits_stride and out_stride elements apart (vocab at least); d_out may
 * be d_logits, with the same stride, and overlaps it in no other way. Columns
 * from vocab on are neither read nor written. */
typedef struct qwen3_logits {
  int32_t rows, vocab, dtype;      /* 65535 rows and a vocab of 2^26 at most */
  int64_t logits_stride, out_stride;   /* 2^40 at most */
  int32_t n_seq, history_stride;   /* d_history int32 [n_seq][history_stride], 2^28 at most */
  int32_t path_len;                /* d_path int32 [rows][path_len], 2^20 at most */
  int32_t n_bias;                  /* d_bias_ids int32, d_bias fp32 [rows][n_bias], 1024 at most */
  int32_t n_masks;                 /* d_masks int32 [n_masks][ceil(vocab / 32)] */
  const int32_t *d_history, *d_prompt_lens, *d_lens, *d_row_seq, *d_path;
  const float *d_repetition, *d_frequency, *d_presence;   /* [rows] */
  const int32_t* d_bias_ids;
  const float* d_bias;
  const int32_t *d_masks, *d_row_mask;                    /* d_row_mask [rows], NULL: row r has mask r */
} qwen3_logits;
gpt2_status qwen3_adjust_logits(const qwen3_logits* l, const void* d_logits,
                                void* d_out, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif
