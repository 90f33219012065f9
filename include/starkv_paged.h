/*
 * starkv_paged.h -- C ABI of generation over a paged KV cache on MI355X.
 *
 * After the compression stage an agent generates: several sequences of
 * different lengths grow token by token, share prefixes, are compressed by
 * the stage's selection, and attend to what is left.  Their K and V rows lie
 * in the pages of one pool:
 *   starkv_pages_init     an empty pool
 *   starkv_pages_grow     pages for new tokens (shared pages copied on write)
 *   starkv_pages_write    K and V of the new tokens into their pages
 *     ..._write_grown     the same behind a grow that may have found no pages
 *   starkv_pages_fork     a sequence that shares another's pages
 *   starkv_pages_free     pages of dropped tokens back to the pool
 *   starkv_pages_compact  the kept tokens into fresh pages (a selection of
 *                         starkv_select, or the accepted path of a tree)
 *     ..._compact_grown   the same behind a grow that may have found no pages
 *   starkv_attend_tree    attention of a tree of drafted tokens
 *   starkv_attend_window  attention with a sliding window and sink tokens
 *
 * The conventions of starkv.h hold: asynchronous on `stream`, no allocation,
 * no copy to the host, arguments validated on the host before any GPU work
 * (on an error code nothing is written), bitwise deterministic, no pointer
 * kept.  Host arrays (slots, rows, ...) are read only during the call, so a
 * captured call keeps the lists that it was captured with; lengths and page
 * tables are read on the device, so a replay sees their current values.
 * Calls that may overlap on a GPU need workspaces of their own, and calls
 * that change one cache (grow, write, fork, free, compact) must be ordered.
 */
#ifndef STARKV_PAGED_H
#define STARKV_PAGED_H

#include "starkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define STARKV_MAX_SEQS 256        /* sequences per call */
#define STARKV_MAX_DRAFT_WORDS 4   /* 64-bit mask words per drafted token */

/* A paged cache.  Token t of the sequence in slot b lies in page
 * table[b][t / page_tokens], row t % page_tokens; element (layer, page,
 * group, row, j) of K (and of V) at base + layer*layer_stride +
 * page*page_stride + group*group_stride + row*token_stride + j.  A table
 * entry that is not in [0, n_pages) (normally -1) is no page: its tokens are
 * dropped, and no call reads or writes memory for them.
 *   n_layers in [1, 4096], G in [1, STARKV_MAX_GROUPS], H % G == 0, H <= 4096,
 *   d in {64, 128}, dtype STARKV_F32 or STARKV_BF16,
 *   page_tokens a power of two in [16, 1024], n_pages in [1, 2^26],
 *   n_slots in [1, 2^20], max_pages*page_tokens <= 2^26,
 *   strides times the element size multiples of 16 bytes, not negative,
 *   token_stride >= d and under 2^28 bytes; k and v 16-byte aligned, the int32 arrays 4-byte.
 * refs[p] is how many table entries name page p; a page is free when refs[p]
 * is 0.  Calls that allocate take the lowest-numbered pages that were free
 * when the call began, in the order of the call's sequences; they look for
 * them from page 0 up, 4 us for every 8,192 pages before the last that they
 * take.  To write or attend to one layer of a cache, pass n_layers = 1 and k, v
 * moved on by the layer's offset; grow and compact move rows of the layers that
 * they are given and change the table once, so they take all layers. */
typedef struct starkv_paged {
  int32_t n_layers;
  int32_t H;
  int32_t G;
  int32_t d;
  int32_t dtype;
  int32_t page_tokens;
  int32_t n_pages;
  int32_t n_slots;
  int32_t max_pages;     /* entries of a table row */
  int32_t reserved;      /* 0 */
  int64_t layer_stride;  /* element strides */
  int64_t page_stride;
  int64_t group_stride;
  int64_t token_stride;
  void* k;               /* device */
  void* v;               /* device */
  int32_t* table;        /* device, [n_slots][max_pages] */
  int32_t* len;          /* device, [n_slots]: tokens of each sequence */
  int32_t* refs;         /* device, [n_pages] */
} starkv_paged;

/* What grow and compact report per sequence of the call (int32, device). */
#define STARKV_SEQ_OK 0
#define STARKV_SEQ_NO_PAGES 1  /* the pool had too few free pages: unchanged */
#define STARKV_SEQ_RANGE 2     /* past the table row, tail past the sequence or of dropped tokens,
                                  or it would go on within a page that was dropped: unchanged */

/* ------------------------------------------------------------------ */
/* pages                                                               */
/* ------------------------------------------------------------------ */
/* Slot lists: host, n in [0, STARKV_MAX_SEQS] entries in [0, n_slots), no
 * slot twice in a list of sequences that the call changes (E_PARAM).  n = 0
 * does nothing. */

/* An empty pool: refs 0, lengths 0, table entries -1.  k and v are not
 * touched.  Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_HIP. */
starkv_status starkv_pages_init(const starkv_paged* cache, void* stream);

/* Bytes of device workspace that grow and compact need for n sequences, with
 * at most `most` tokens added to (grow), or moved within (compact: B + tail),
 * a sequence.  0 if the arguments are invalid. */
size_t starkv_pages_workspace_bytes(const starkv_paged* cache, int32_t n, int32_t most);

/* Lengthen each sequence by add[b] >= 0 tokens (host), with pages for them.
 * Where the old last page is partly filled and another sequence shares it,
 * its filled rows are copied to a fresh page first (all layers and groups of
 * `cache`), so that the new tokens can be written.  Every sequence that
 * shared its page when the call began gets a copy.  If the free pages do not
 * suffice, the sequences are served in order while they do.
 * status: device out, int32 [n] (STARKV_SEQ_*).
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_WORKSPACE, E_HIP. */
starkv_status starkv_pages_grow(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                const int32_t* add, int32_t* status, void* ws, size_t ws_bytes,
                                void* stream);

/* Write K and V of the last rows[b] >= 0 tokens (host) of each sequence: row
 * r of k and v, layout *rows_layout with "token" the row number over all
 * sequences of the call in order, group the KV group.  Tokens without a page,
 * of a page that another sequence shares, or before the sequence's first are
 * not written.  After a grow that left a sequence unchanged its last tokens are
 * older ones, and this call writes over them: behind a grow whose status the
 * host has not read, the call below is the one.  k, v: device, the cache's
 * dtype.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_HIP. */
starkv_status starkv_pages_write(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 const int32_t* rows, const void* k, const void* v,
                                 const starkv_kv_layout* rows_layout, void* stream);

/* The same for the tokens of a grow: sequence b is written where grown[b] is
 * STARKV_SEQ_OK, and stays as it is otherwise.  grown: device, int32 [n], the
 * status of the starkv_pages_grow that made the tokens, of the same slots in
 * the same order.  Errors: as above. */
starkv_status starkv_pages_write_grown(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                       const int32_t* rows, const void* k, const void* v,
                                       const starkv_kv_layout* rows_layout, const int32_t* grown,
                                       void* stream);

/* Make the sequence in dst[i] a fork of the one in src[i]: the same pages and
 * length, no row copied.  What dst held is freed first.  dst: no slot twice,
 * none that is also in src (E_PARAM); a src may repeat.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_HIP. */
starkv_status starkv_pages_fork(const starkv_paged* cache, const int32_t* src,
                                const int32_t* dst, int32_t n, void* stream);

/* Drop tokens of each sequence, and free the pages that hold none of those
 * kept.  keep_last = 0: the first keep_first tokens stay, and the length
 * becomes min(length, keep_first) (0: the sequence ends).  keep_last > 0: the
 * first keep_first and the last keep_last tokens stay where they are; the
 * length does not change (what a window with sinks no longer sees).
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_HIP. */
starkv_status starkv_pages_free(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                int32_t keep_first, int32_t keep_last, void* stream);

/* Compact each sequence b of length L: of its last `span` tokens (span[b],
 * host; NULL: all of them), a = L - span, the tokens a + idx[layer][b][j], j <
 * count, then the sequence's last `tail` tokens are kept behind the a first
 * ones: the new length is a + count + tail.  With span NULL, idx of
 * starkv_select and tail = W this is starkv_compact within the pool; with
 * span the drafted tokens, idx the accepted path, tail 0, it ends a
 * speculative step.  The kept rows go to fresh pages (bit copies, from the
 * page of token a on); the pages that they came from are let go, and are free
 * afterwards unless other sequences share them.  Rows may be picked in any
 * order and more than once.  A tail of which a token was dropped has no rows to
 * keep: STARKV_SEQ_RANGE.
 * idx:    device, int32 [n][B] per layer, layer l at idx + l*idx_layer_stride
 *         (0: all layers keep the same tokens).  An entry outside [0, span -
 *         tail), or whose token was dropped, gives an all-zero row.
 * counts: device, int32 [n], clamped to [0, B]; NULL: B for all.
 * status: device out, int32 [n] (STARKV_SEQ_*).
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_BUDGET (B or tail negative, or
 * B + tail > 2^26), E_PARAM, E_WORKSPACE, E_HIP. */
starkv_status starkv_pages_compact(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                   const int32_t* span, const int32_t* idx,
                                   int64_t idx_layer_stride, int32_t B, const int32_t* counts,
                                   int32_t tail, int32_t* status, void* ws, size_t ws_bytes,
                                   void* stream);

/* The same for tokens that a grow made, as the drafted ones are: where grown[b]
 * is not STARKV_SEQ_OK the last `span` tokens are older ones, which the call
 * keeps: the sequence stays as it is, and status[b] becomes grown[b].  grown:
 * as for starkv_pages_write_grown; it may be `status` itself.  Errors: as above. */
starkv_status starkv_pages_compact_grown(const starkv_paged* cache, const int32_t* slots,
                                         int32_t n, const int32_t* span, const int32_t* idx,
                                         int64_t idx_layer_stride, int32_t B,
                                         const int32_t* counts, int32_t tail,
                                         const int32_t* grown, int32_t* status, void* ws,
                                         size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ */
/* attention over the pages                                            */
/* ------------------------------------------------------------------ */
/* Both calls take rows[b] >= 0 query tokens (host) of each sequence (a slot
 * may repeat): those of its last rows[b] cached tokens, whose K and V are in
 * the cache already.  rows[b] is at most what a table row holds, their sum at
 * most 2^26, and n_layers * G * sum of ceil(rows[b]*H/G / 16) at most 2^23
 * (E_PARAM; bf16 calls of many rows take eight times as many).  With V(i) the
 * cached tokens that query token i sees,
 *   x[h,t] = q[h] . K[g(h),t] / sqrt(d),
 *   out[h] = sum_{t in V(i)} softmax_t(x[h,t]) V[g(h),t],
 *   lse[h] = ln sum_{t in V(i)} exp(x[h,t]).
 * A row that sees nothing gets out = 0 and lse = -infinity, and so does one
 * whose logits are all -infinity (from K or q themselves).  Tokens outside
 * V(i), and dropped ones, do not touch row i, whatever their K and V hold
 * (infinities and NaN included).  Softmax, sums and lse are float32 (bf16
 * caches: the weights are rounded to bf16 for the product with V).
 * q:   device, the cache's dtype, [n_layers][sum rows][H][d] contiguous, rows
 *      of the call's sequences in order; 16-byte aligned.
 * out: device out, as q.   lse: device out, float32 [n_layers][sum rows][H],
 *      or NULL.
 * max_len: a bound on the lengths of the call's sequences, by which the work
 *      is split (1 to 2^26; the table row's tokens where it is larger).  A
 *      sequence that is longer is still read whole, only less evenly.
 * ws:  device workspace of ws_bytes >= starkv_attend_workspace_bytes().
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_WORKSPACE, E_HIP. */

/* Bytes of device workspace of an attention call with these arguments.  0 if
 * they are invalid, or none is needed (ws may then be NULL).  Calls of fewer
 * rows, or on fewer layers, are split further and may need more: a workspace
 * for several kinds of calls has the size of the one that needs most. */
size_t starkv_attend_workspace_bytes(const starkv_paged* cache, const int32_t* rows, int32_t n,
                                     int32_t max_len);

/* A tree of drafted tokens per sequence: V(i) is every token before the
 * drafted ones, and drafted token j where bit j of row i's mask is set (bit j
 * % 64 of word j / 64; the row's own bit is not implied, bits from rows[b] on
 * are ignored).
 * mask: device, uint64 [sum rows][words], words in [1, STARKV_MAX_DRAFT_WORDS],
 *       rows[b] <= 64*words (E_PARAM); 8-byte aligned. */
starkv_status starkv_attend_tree(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 const int32_t* rows, const void* q, const uint64_t* mask,
                                 int32_t words, int32_t max_len, void* out, float* lse, void* ws,
                                 size_t ws_bytes, void* stream);

/* A sliding window with sinks: query token i of sequence b is the token at
 * p = length - rows[b] + i, and sees t <= p with t > p - window or t < sinks.
 * window = 0: every t <= p.  window and sinks in [0, 2^26] (E_PARAM). */
starkv_status starkv_attend_window(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                   const int32_t* rows, const void* q, int32_t window,
                                   int32_t sinks, int32_t max_len, void* out, float* lse,
                                   void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* STARKV_PAGED_H */
