/*
 * libarkv, operators around a paged cache - for servers that keep many requests' rows in pages of one pool: rotary
 * positions on the way into the pages, attention of the requests' new tokens over them, the attention weight that every
 * cached row collected, and eviction by that weight.  Pages may hold rows of 16 bits, or packed ones of 8 or 4 bits a channel
 * (arkv_packed_*); tokens may see all rows up to their own, or those that a window or a tree of drafted tokens leaves (arkv_sight).
 *
 * C ABI, the conventions of arkv.h: every call returns 0 or a negative ARKV_E* code, nothing throws, every call is
 * asynchronous on hip_stream (a hipStream_t as void*, NULL = the default stream).  Here the caller owns all memory: no
 * call allocates, synchronises or keeps anything, so every one of them can be captured into a graph, and replayed with
 * other lengths, tables and rows in the same arrays.
 *
 * Notation: B sequences, H_q query heads, H_kv KV heads, G = H_q / H_kv, d head dimension.  A page holds page_size slots
 * of every kv-head.  Slot j of sequence b lies in page table[b][j / page_size], offset j % page_size.  kv_len[b] slots
 * are in use; the last q_len[b] = cu_q[b+1] - cu_q[b] of them are the new tokens, whose query rows are the rows
 * cu_q[b] .. cu_q[b+1] - 1 of the token-major arrays, in slot order.  ctx_b = kv_len[b] - q_len[b].
 *
 * What lies on the device cannot be checked by the host; the kernels check it.  Lengths are cut to what the caller
 * announced (n_tokens, max_q, max_kv, table_width).  A page id outside [0, n_pages) makes its slots absent: nobody sees
 * them, nothing is written there.  A new token whose slot would be negative (kv_len < q_len) has no slot and sees
 * nothing but a prefix.  Rows of the token-major arrays that belong to no sequence are left alone.  With n_tokens = 0 the
 * addresses of token-major arrays may be NULL.
 */
#ifndef ARKV_PAGED_H
#define ARKV_PAGED_H

#include <stddef.h>
#include <stdint.h>

#include "arkv.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ARKV_DTYPE_BF16 0
#define ARKV_DTYPE_FP16 1

/* One layer's pages.  k, v DEVICE [n_pages][H_kv][page_size][d] of dtype; pos DEVICE int32, weight DEVICE float
 * [n_pages][H_kv][page_size]: a row's position and the attention weight it collected (weight may be NULL where no
 * weights are kept).  page_size: a power of two from 16 to 1024.  head_dim 64 or 128.  n_pages H_kv page_size < 2^31.  All four 16-byte aligned. */
typedef struct {
  int32_t dtype, n_pages, page_size, n_kv_heads, head_dim;
  void* k;
  void* v;
  int32_t* pos;
  float* weight;
} arkv_pages;

/* One step's sequences.  cu_q DEVICE int32 [B+1] (not decreasing), kv_len DEVICE int32 [B], table DEVICE int32
 * [B][table_width] (entries behind a sequence's last page are not read).  n_tokens: rows of the token-major arrays;
 * max_q, max_kv: bounds of q_len and kv_len (they shape the launches; tight ones are faster).  B H_kv <= 2^20, B H_kv max_kv <= 2^40,
 * n_tokens H_q < 2^31. */
typedef struct {
  int32_t batch, n_tokens, max_q, max_kv, table_width;
  const int32_t* cu_q;
  const int32_t* kv_len;
  const int32_t* table;
} arkv_page_batch;

/* Token-major rows [n_tokens][heads][d] DEVICE: strides in elements (multiples of 8, not negative), 16-byte aligned, channels adjacent. */
typedef struct {
  const void* p;
  int64_t token_stride, head_stride;
} arkv_rows;

/* Rotary positions with up to 4 axes (text: one; images: height, width; video: time too).  Pair i of rot_dim / 2 pairs
 * turns by position[axis[i]] * freq[i] radians.  adjacent = 0: pair i is channels (i, i + rot_dim / 2); 1: (2i, 2i + 1).
 * Channels from rot_dim on are copied.  rot_dim: multiple of 16, 0 (nothing turns) to head_dim.  axis HOST (in this struct),
 * freq DEVICE double [rot_dim / 2]. */
typedef struct {
  int32_t rot_dim, n_axes, adjacent;
  uint8_t axis[64];
  const double* freq;
} arkv_rotary;

/* How a logit comes about: x = scale q.k; with cap > 0: x = cap tanh(x / cap); with slopes (DEVICE float [H_q]):
 * x -= slopes[h] |q_pos - pos|, q_pos DEVICE int32 [n_tokens], pos the cached row's (less than 2^31 apart).  New token i of sequence b sees the
 * slots up to its own, j <= ctx_b + i, and with prefix (DEVICE int32 [B]) every slot j < prefix[b]; all of them < kv_len[b].
 * The cap puts x off by 2^-22 cap at most; one above 256 by 2^-19 of x. */
typedef struct {
  float scale, cap;
  const float* slopes;
  const int32_t* q_pos;
  const int32_t* prefix;
} arkv_scores;

/* Which slots new token i of sequence b sees, where that is not all up to its own, p = ctx_b + i.  window w > 0: the slots j <= p with
 * j > p - w or j < sink.  tree (DEVICE uint64 [n_tokens][tree_words], 8-byte aligned, 64 tree_words >= max_q): bit t of the token's words says
 * whether it sees new token t, itself among them; the slots below ctx_b it sees all, or with a window as a token at p = ctx_b + (new tokens it
 * sees) - 1, at ctx_b where it sees none.  The window takes no new token away: a draft that w or more others come before sees first ones that it
 * would not see once they are accepted, so trees should be less deep than the window.  Bits from q_len[b] on count for nothing.  A prefix of the scores is
 * seen besides.  All zero: no limits. */
typedef struct {
  int32_t window, sink, tree_words;
  const uint64_t* tree;
} arkv_sight;

/* One layer's packed pages: k, v DEVICE [n_pages][H_kv][page_size][d bits / 8], k_scale, v_scale DEVICE uint8 [n_pages][H_kv][page_size][d / 32],
 * pos as in arkv_pages.  A row's channels lie in blocks of 32, each with a scale byte s; a channel is its code's value times 2^(s - 127).
 * bits = 8: a code is a byte: sign, 4 bits of exponent (bias 7), 3 of mantissa, 127 and 255 NaN, the largest value 448; 4: half a byte (an even
 * channel's the low half): sign, 2 bits of exponent (bias 1), 1 of mantissa, the largest value 6.  s = 255: NaN, the whole block.
 * dtype: of the rows that go in and come out, and of q.  All five 16-byte aligned; sizes as in arkv_pages.  Other bits: ARKV_EUNSUPPORTED. */
typedef struct {
  int32_t dtype, bits, n_pages, page_size, n_kv_heads, head_dim;
  void* k;
  void* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int32_t* pos;
} arkv_packed_pages;

/* Turns q and k of the new tokens and stores k, v into their slots: q_out [n_tokens][H_q][d] (dense, DEVICE), rows k and v of
 * the pages, pos = positions[0][token], weight = 0.  positions DEVICE int32 [n_axes][n_tokens].  Angles are formed in 64
 * bits, products in 32, each result rounded once.  q.p may equal q_out (in place) if it is dense too.  q = NULL and q_out = NULL: keys and values only.
 * ARKV_EINVAL: null pointers, sizes, alignment, an axis >= n_axes, q.p = q_out with other strides.  ARKV_EUNSUPPORTED: head_dim, dtype, n_pages H_kv page_size >= 2^31,
 * n_tokens > 2^26 - 4. */
int arkv_paged_append(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_rotary* rotary, int32_t n_q_heads,
                      const arkv_rows* q, const arkv_rows* k, const arkv_rows* v, const int32_t* positions, void* q_out,
                      void* hip_stream);

/* Bytes of DEVICE workspace that the calls below need for this batch and any of their options (64 KiB or more).  HOST, pure.
 * The first 64 KiB must be zero before the workspace's first use; every call leaves them zero, so one workspace serves calls one
 * after the other.  It is large enough for every batch of the same head_dim, H_kv and H_q whose batch, n_tokens, max_q and max_kv are none of
 * them larger than here: at most 136 MB for chunks (fewer rows are cut finer), and 8 KB for each 2048 rows of a kv-head for single tokens.
 * Calls that may overlap in time need workspaces of their own. */
int arkv_paged_workspace(const arkv_pages* pages, const arkv_page_batch* batch, int32_t n_q_heads, size_t* bytes);

/* out [n_tokens][H_q][d] (dense, DEVICE, of the pages' dtype) = softmax over the visible slots of x, times v.  lse DEVICE float
 * [n_tokens][H_q] or NULL: natural logarithm of the sum of exp(x).  A token that sees nothing gets zeros and
 * -infinity.  What lies in slots that a token does not see has no influence on its row, whatever bits it holds.
 * The new tokens' own rows must be in the pages already (arkv_paged_append).  G <= 16.
 * Probabilities are rounded to the pages' dtype in front of the product with v; sums, maxima and the denominator are fp32.  workspace 16-byte
 * aligned, as arkv_paged_workspace says.  ARKV_EUNSUPPORTED, besides the above: 2^24 workgroups or more (about n_tokens H_q / 128 +
 * B H_kv max_kv / 2048; a sequence's last 128 rows may be a short block). */
int arkv_paged_attention(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                         int32_t n_q_heads, const arkv_rows* q, void* out, float* lse, void* workspace, size_t bytes,
                         void* hip_stream);

/* The same, a token seeing the slots that sight says (NULL: arkv_paged_attention).  What no token of a workgroup sees in front of its window is not
 * read, nor its table entries, whole granules of 16 slots at a time.  The lengths choose how long sequences are cut: a row's last bits may differ with
 * the batch that it is in.  lse is no input for arkv_paged_weights, which knows of no sight.  After drafting, the accepted tokens' rows are appended once
 * more, kv_len cut to them: their slots are the first drafts'.  ARKV_EINVAL, besides: window or sink negative, tree_words too small, tree not aligned. */
int arkv_paged_attention_sight(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                               const arkv_sight* sight, int32_t n_q_heads, const arkv_rows* q, void* out, float* lse,
                               void* workspace, size_t bytes, void* hip_stream);

/* arkv_paged_append into packed pages.  k is turned in 64 bits, by an angle that is off by 2^-51 of position * freq and a few 2^-53 at most: a code or a
 * scale is the next one only where the turned key lies that close to a border between them; q_out is what arkv_paged_append gives.  A block's s is the
 * smallest from 1 on with max|x| <= 448 (6) times 2^(s - 127); codes are the nearest ones, ties to the even one.  Channels that are not finite, or beyond
 * the type's range once turned, count for nothing in max|x|; with 8 bits they are stored as NaN, with 4 their block is.  Where the nearest code's value
 * would be beyond the type's range, the largest one that is not is stored. */
int arkv_packed_append(const arkv_packed_pages* pages, const arkv_page_batch* batch, const arkv_rotary* rotary, int32_t n_q_heads,
                       const arkv_rows* q, const arkv_rows* k, const arkv_rows* v, const int32_t* positions, void* q_out,
                       void* hip_stream);

/* The rows of the batch's new tokens (the last q_len[b] slots of each sequence: all of them, where q_len = kv_len) as their values:
 * k, v [n_tokens][H_kv][d] (dense, DEVICE, of dtype, 16-byte aligned; either may be NULL).  Nothing is rounded, but values below the type's
 * normal range.  A row without a slot, or in an absent page, is zeros. */
int arkv_packed_read(const arkv_packed_pages* pages, const arkv_page_batch* batch, void* k, void* v, void* hip_stream);

/* arkv_paged_workspace for arkv_packed_attention. */
int arkv_packed_workspace(const arkv_packed_pages* pages, const arkv_page_batch* batch, int32_t n_q_heads, size_t* bytes);

/* arkv_paged_attention over the values of packed rows; sight as in arkv_paged_attention_sight, or NULL. */
int arkv_packed_attention(const arkv_packed_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                          const arkv_sight* sight, int32_t n_q_heads, const arkv_rows* q, void* out, float* lse,
                          void* workspace, size_t bytes, void* hip_stream);

/* weight = decay * carried + sum of exp(x - lse) over the G heads of the row's group and the new tokens that see it, for every slot in
 * use (slots of no sequence are left alone).  carried: DEVICE, laid out as weight; NULL or weight itself: in place; another
 * array: e.g. the weights before drafted tokens that may be rejected.  With decay = 0 carried is not read.  lse DEVICE float [n_tokens][H_q], what
 * arkv_paged_attention returned for the same batch, scores and q (one of a call with a sight is accepted, but then rows that the sight hid collect
 * weight; packed pages keep none).  Pages that several sequences of the batch share would be updated
 * by each: their weight is the last writer's.  Sums are fp32, in an order that the sizes alone fix;
 * terms below 2^-126 count as zero. */
int arkv_paged_weights(const arkv_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores,
                       int32_t n_q_heads, const arkv_rows* q, const float* lse, float decay, const float* carried,
                       void* workspace, size_t bytes, void* hip_stream);

/* Every kv-head of sequence b keeps m = min(kv_len[b], keep[b]) of its rows: the first min(sink, m), the last
 * min(recent, m - that), and of the others those of the largest weight (equal weights: the lower slot; -0 = +0; NaN
 * and rows in absent pages, alike: below every number, the lower slot first).  The survivors' k, v, pos and weight are copied, in slot order, to the slots 0 .. m - 1 of the pages dst_table[b]
 * ([B][dst_width] DEVICE int32), which must be pages that no table of the batch names: the sources stay as they are, so
 * pages that other sequences share can be evicted from.  kept DEVICE int32 [B][H_kv][max_keep]: the survivors' former
 * slots, -1 behind them.  new_len DEVICE int32 [B] = m.  keep DEVICE int32 [B], cut to [0, max_keep].  cu_q and the new tokens play no
 * part.  kept and new_len must not overlap kv_len, keep, the tables or each other (lengths are read until the end of the call: copy new_len
 * over kv_len behind it).  For a survivor in an absent page nothing is copied: its new slot holds what it held before.  workspace as arkv_paged_workspace says; NULL will do
 * where max_keep head_dim <= 32768 and max_kv <= 36864 (with one, few units of many rows are counted faster).
 * ARKV_EINVAL: as above, weight NULL, arrays that overlap, max_keep outside [1, dst_width * page_size], sink or recent negative, a workspace
 * that is too small, not aligned to 16 bytes, or missing. */
int arkv_paged_evict(const arkv_pages* pages, const arkv_page_batch* batch, const int32_t* keep, int32_t max_keep,
                     int32_t sink, int32_t recent, const int32_t* dst_table, int32_t dst_width, int32_t* kept,
                     int32_t* new_len, void* workspace, size_t bytes, void* hip_stream);

/* Parity hook, HOST, pure: where the kernels look for slot `slot` of a sequence: the row of [n_pages][H_kv][page_size], or -1 where
 * there is none (a slot outside [0, len), a page id outside [0, n_pages)).  table_row HOST int32 [table_width]; *row gets it.
 * ARKV_EINVAL: null pointers, sizes, kv_head outside [0, H_kv). */
int arkv_debug_paged_row(const int32_t* table_row, int32_t table_width, int32_t n_pages, int32_t page_size,
                         int32_t n_kv_heads, int32_t kv_head, int32_t len, int32_t slot, int64_t* row);

/* Parity hook, HOST, pure: how arkv_packed_attention, or with bits = 16 arkv_paged_attention_sight, divides a batch.  HOST arrays here: the batch's cu_q and
 * kv_len, the scores' prefix; no other address is followed.  cut HOST int32 [9]: [0] bit 0: blocks of 128 rows (a row: a new token and a query
 * head of the group) are launched, bit 1: groups of up to 16; [1] groups that sequences of more rows are divided into, at most (0: into blocks); [2] keys
 * of a group's piece; [3] pieces of a group, the most; [4] keys of a block's piece; [5] pieces of a block, the most; [6] where a block has more than
 * one, they are joined by 1: the last workgroup to finish, 2: a launch of blocks, 3: a launch of rows; [7] pieces of all blocks and kv-heads;
 * [8] workgroups that the chip holds at once, which [4] is chosen for (0: by the batch's bounds alone).  ARKV_EINVAL, ARKV_EUNSUPPORTED: as those calls. */
int arkv_debug_attention_cut(const arkv_packed_pages* pages, const arkv_page_batch* batch, const arkv_scores* scores, const arkv_sight* sight,
                             int32_t n_q_heads, int32_t* cut);

#ifdef __cplusplus
}
#endif
#endif /* ARKV_PAGED_H */
