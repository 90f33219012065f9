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
 *   starkv_pages_read     K and V of a sequence's last tokens out of their pages
 *   starkv_pages_fork     a sequence that shares another's pages
 *   starkv_pages_free     pages of dropped tokens back to the pool
 *   starkv_pages_compact  the kept tokens into fresh pages (a selection of
 *                         starkv_select, or the accepted path of a tree)
 *     ..._compact_grown   the same behind a grow that may have found no pages
 *   starkv_attend_tree    attention of a tree of drafted tokens
 *   starkv_attend_window  attention with a sliding window and sink tokens
 *   starkv_mass_add       attention weights added up per cached token
 *     ..._add_grown       the same behind a grow that may have found no pages
 *   starkv_mass_fork      a fork's copy of them
 *   starkv_pages_evict    the tokens of the least accumulated weight evicted
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

/* A cache held in 4 bits, a dtype of starkv_paged alone: 32 elements of a K or
 * V row share a power of two.  An element is 4 bits, e2m1: a sign (bit 3) and
 * one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0 to 2); element 2i lies in the low half
 * of byte i.  Scale byte b stands for 2^(b - 127); 255 makes its block NaN.  A
 * (layer, page, group)'s page_tokens rows of d/2 bytes lie one behind the other,
 * token_stride = d/2, and behind them, from byte page_tokens*d/2 on, their
 * scales, d/32 bytes a row: page_tokens*(d/2 + d/32) bytes in all.  Strides count
 * bytes.  q, out, and the rows given and read are bf16.
 *   starkv_pages_write quantises: with a the largest magnitude of 32 elements,
 * the scale is the 2^e for which a is in (3.5, 7] * 2^e (b clamped to [2, 252]), and
 * an element becomes the nearest of the above times 2^e, ties to the even code,
 * beyond 6 to 6.  A block that holds an infinity or NaN becomes NaN.  Every other
 * block stands for finite bf16 numbers, and the attentions are those over them.  In a
 * pool filled otherwise (bytes 253 and 254) what is 2^128 or more is an infinity. */
#define STARKV_FP4 4

/* A paged cache.  Token t of the sequence in slot b lies in page
 * table[b][t / page_tokens], row t % page_tokens; element (layer, page,
 * group, row, j) of K (and of V) at base + layer*layer_stride +
 * page*page_stride + group*group_stride + row*token_stride + j.  A table
 * entry that is not in [0, n_pages) (normally -1) is no page: its tokens are
 * dropped, and no call reads or writes memory for them.
 *   n_layers in [1, 4096], G in [1, STARKV_MAX_GROUPS], H % G == 0, H <= 4096,
 *   d in {64, 128}, dtype STARKV_F32, STARKV_BF16 or STARKV_FP4,
 *   page_tokens a power of two in [16, 1024], n_pages in [1, 2^26],
 *   n_slots in [1, 2^20], max_pages*page_tokens <= 2^26,
 *   strides times the element size multiples of 16 bytes, not negative,
 *   token_stride >= d (STARKV_FP4: d/2) and under 2^28 bytes; k and v 16-byte aligned, the int32 arrays 4-byte.
 * refs[p] is how many table entries name page p; a page is free when refs[p]
 * is 0.  Calls that allocate take the lowest-numbered pages that were free
 * when the call began, in the order of the call's sequences; they look for
 * them from page 0 up, 4 us for every 8,192 pages before the last that they
 * take.  To write or attend to one layer of a cache, pass n_layers = 1 and k, v
 * moved on by the layer's offset; grow, compact and evict move rows of the layers
 * that they are given and change the table once, so they take all layers. */
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
#define STARKV_SEQ_SHORT 3     /* evict: no longer than what is kept: unchanged */

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
 * dtype (STARKV_FP4: bf16).
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

/* Read K and V of the last rows[b] >= 0 tokens (host) of each sequence into k
 * and v (device out, dtype and layout as for starkv_pages_write; a slot may
 * repeat).  A token without a page, or before the sequence's first, gives an
 * all-zero row.  STARKV_FP4: the bf16 numbers that the rows stand for.
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_HIP. */
starkv_status starkv_pages_read(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                const int32_t* rows, void* k, void* v,
                                const starkv_kv_layout* rows_layout, void* stream);

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
 * (infinities and NaN included).  Softmax, sums and lse are float32 (bf16 and
 * 4-bit caches: the weights are rounded to bf16 for the product with V).  The sums are
 * of weights relative to the largest so far, 2^8 at most: where 2^8 sum_t |v_t| is 2^128
 * or more, an output that is finite may overflow on the way.
 * q:   device, the cache's dtype (STARKV_FP4: bf16), [n_layers][sum rows][H][d] contiguous, rows
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

/* ------------------------------------------------------------------ */
/* eviction by accumulated attention weight                            */
/* ------------------------------------------------------------------ */
/* A mass is what the attention has weighted a cached token with, summed over
 * the query tokens and heads of a layer: float32 [n_layers][n_slots][max_pages *
 * page_tokens], device, contiguous, beside the cache.  starkv_mass_add follows
 * each attention, starkv_mass_fork each fork, and starkv_pages_evict takes the
 * lightest tokens away, their masses with them.  A token has a mass from the call
 * on whose rows it is one of: it needs no start, and what lies behind a sequence
 * or in a slot in no use is not looked at.  starkv_pages_compact moves no masses.
 * After the compaction of a drafted tree's path, weigh the accepted tokens with their
 * rows of q and lse of the starkv_attend_tree call, gathered, and no window: where
 * an accepted row saw its ancestors, they and the prefix are what is before it now. */

/* Add the weights of the last rows[b] >= 0 tokens (host) of each sequence: with
 * x, window, sinks and the tokens V(i) that query token i sees as for
 * starkv_attend_window, and lse what that call gave for these rows,
 *   out[t] = old[t] + sum_{i, h: t in V(i)} exp(x[h,t] - lse[i,h]),
 * old[t] = mass[t] for the tokens before the rows', 0 for the rows' own.  A row
 * whose lse is -infinity or NaN adds nothing.  All tokens of the sequence are written
 * (dropped ones keep old[t]), none behind it; sequences without rows are left as
 * they are.  Logits, weights and sums are float32.  After a grow that left a
 * sequence unchanged its last tokens are older ones, whose masses this call loses:
 * behind a grow whose status the host has not read, the call below is the one.
 * slots: no slot twice (E_PARAM).   rows: each at most what a table row holds,
 *      their sum at most 2^26 (E_PARAM).
 * q:   as for the attentions.   lse: device, float32 [n_layers][sum rows][H].
 * mass: device, as above.   out: device out, as mass; it may be mass.
 * max_len, ws: as for the attentions, with starkv_mass_workspace_bytes() (calls of
 *      fewer rows or layers may need more: size it for each that is made).
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_PARAM, E_WORKSPACE, E_HIP. */
starkv_status starkv_mass_add(const starkv_paged* cache, const int32_t* slots, int32_t n,
                              const int32_t* rows, const void* q, const float* lse,
                              int32_t window, int32_t sinks, int32_t max_len, const float* mass,
                              float* out, void* ws, size_t ws_bytes, void* stream);

/* The same behind the grow that made the rows: where grown[b] is not
 * STARKV_SEQ_OK nothing is added and no token is the rows' own, out[t] = mass[t] for
 * all tokens of the sequence.  grown: as for starkv_pages_write_grown, or the status of
 * the compaction behind that grow.  Errors: as above. */
starkv_status starkv_mass_add_grown(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                    const int32_t* rows, const void* q, const float* lse,
                                    int32_t window, int32_t sinks, int32_t max_len,
                                    const float* mass, float* out, const int32_t* grown, void* ws,
                                    size_t ws_bytes, void* stream);

/* Bytes of device workspace of both with these arguments.  0 if they
 * are invalid, or none is needed (ws may then be NULL). */
size_t starkv_mass_workspace_bytes(const starkv_paged* cache, const int32_t* rows, int32_t n,
                                   int32_t max_len);

/* Copy the masses of the sequences in src to dst, after (or before)
 * starkv_pages_fork of the same slots: the first length(src) of each.
 * Errors: as for starkv_pages_fork. */
starkv_status starkv_mass_fork(const starkv_paged* cache, const int32_t* src, const int32_t* dst,
                               int32_t n, float* mass, void* stream);

/* Cut each sequence longer than sinks + keep + recent down to its first `sinks`
 * tokens, its last `recent` ones, and of those between the `keep` of the largest
 * mass, by layer, in their order (equal masses: the lower token; NaN counts as
 * the largest).  Dropped tokens are not kept; where that leaves fewer than asked
 * for, the sequence ends up shorter.  Rows move as with starkv_pages_compact and
 * tail = recent, and the masses with them.  Other sequences stay as they are,
 * STARKV_SEQ_SHORT.
 * The rows move to pages that were free when the call began, and their own are let
 * go afterwards: a call takes ceil((sinks + keep + recent) / page_tokens) free pages for
 * each long sequence (fewer where dropped tokens leave fewer to keep), in order while
 * they last, and the others get STARKV_SEQ_NO_PAGES.  A full pool evicts nothing, so keep
 * the pages of one sequence aside: with these, calls of one sequence each can evict all,
 * as each lets go of no fewer than it took (unless forks share them).
 * slots: no slot twice (E_PARAM).   mass: device, in and out.
 * idx:    device out, int32 [n_layers][n][sinks + keep]: the kept tokens but for
 *         the recent ones, ascending; -1 behind the last, and for short sequences.
 * status: device out, int32 [n] (STARKV_SEQ_*): where it is not STARKV_SEQ_OK the
 *         sequence and its masses are as before.
 * ws: device workspace of ws_bytes >= starkv_evict_workspace_bytes().
 * Errors: E_NULL, E_SHAPE, E_DTYPE, E_ALIGN, E_BUDGET (keep, sinks or recent
 * negative, or their sum over 2^26), E_PARAM, E_WORKSPACE, E_HIP. */
starkv_status starkv_pages_evict(const starkv_paged* cache, const int32_t* slots, int32_t n,
                                 float* mass, int32_t keep, int32_t sinks, int32_t recent,
                                 int32_t* idx, int32_t* status, void* ws, size_t ws_bytes,
                                 void* stream);

/* Bytes of device workspace that starkv_pages_evict needs for n sequences.  0 if
 * the arguments are invalid. */
size_t starkv_evict_workspace_bytes(const starkv_paged* cache, int32_t n, int32_t keep,
                                    int32_t sinks, int32_t recent);

#ifdef __cplusplus
}
#endif

#endif /* STARKV_PAGED_H */
