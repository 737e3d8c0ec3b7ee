/*
 * ecokv_decode.h - C ABI of libecokv.so, the decode step over an evicted cache.
 *
 * The eviction pass (ecokv.h) turns a prompt's cache into a compact one.  What
 * follows it is a batch of sequences that share this cache as their prefix
 * (several questions about the same video) and grow caches of their own:
 *
 *   ecokv_rotate   norm of each head's row (optional) and rotary positions, for
 *                  queries and keys; before the eviction pass too
 *   ecokv_append   the same on the way of new keys and values into a paged cache
 *   ecokv_attend   attention of the batch's new tokens over the shared prefix and
 *                  each sequence's own pages
 *
 * Drafted tokens (speculative decoding) go through the same cache as a tree a sequence:
 *
 *   ecokv_tree_mask    which drafts each one sees: itself and its ancestors
 *   ecokv_attend_tree  ecokv_attend with that mask in place of the causal one
 *   ecokv_commit       the rows of the accepted drafts move to the front, the others are given up
 *
 * and a cache that has grown is made smaller again:
 *
 *   ecokv_weigh    adds the attention weight that each key gets to what it has had so far
 *   ecokv_prune    keeps the heaviest slots of each head, the first ones and the last ones
 *
 * The paper has no counterpart: they are the operators next to its pass.
 *
 * Conventions as in ecokv.h: device pointers of the caller's, no allocation,
 * argument errors returned before anything is launched, calls asynchronous on
 * `stream`, device-side errors in the workspace's status word
 * (ecokv_device_status), calls that share a workspace ordered on one stream.
 * Rows are d = 128 contiguous elements at 16-byte aligned addresses; strides
 * count elements and are positive multiples of 16 bytes (those of ecokv_rows' x, which
 * is only read, may be zero or negative too).  An output's rows do not overlap.  Data on the device
 * (positions, lengths, page numbers) is read on the device, so a call can be captured
 * in a graph and replayed as they change.  A call of no tokens does nothing, whatever
 * its pointers (ecokv_commit apart, whose sequences have lengths all the same).
 */
#ifndef ECOKV_DECODE_H
#define ECOKV_DECODE_H

#include "ecokv.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ rotary positions
 * Element pair f of a row (f < rot_dim / 2) is turned by the angle
 * position * inv_freq[f]:
 *     y_a = m (x_a cos - x_b sin),  y_b = m (x_b cos + x_a sin)
 * with (a, b) = (f, f + rot_dim / 2) or (2f, 2f + 1).  The other elements stay. */
typedef enum { ECOKV_ROTARY_HALF = 0, ECOKV_ROTARY_INTERLEAVED = 1 } ecokv_rotary_layout;
typedef enum {
  ECOKV_ROTARY_NONE = 0,   /* inv_freq[f] = base^(-2f / rot_dim)                                        */
  ECOKV_ROTARY_LINEAR = 1, /* all of them / factor                                                      */
  ECOKV_ROTARY_NTK = 2,    /* base * factor^(rot_dim / (rot_dim - 2)) in place of base                  */
  ECOKV_ROTARY_YARN = 3    /* YaRN (Peng et al. 2023): those that turn more than 32 times in `original`
                              positions stay, those that turn less than once are / factor, a linear ramp
                              over f between the two; m = 0.1 ln(factor) + 1                            */
} ecokv_rotary_scaling;

#define ECOKV_ROTARY_AXES 4
typedef struct {
  int32_t rot_dim;     /* rotated elements, the row's first: a multiple of 16, 16 .. 128           */
  int32_t layout;      /* ecokv_rotary_layout                                                      */
  int32_t axes;        /* positions a token has, 1 .. ECOKV_ROTARY_AXES                            */
  float magnitude;     /* m above                                                                  */
  uint64_t turns[64];  /* inv_freq[f] / (2 pi) mod 1, in units of 2^-64: position * turns mod 2^64
                          is the angle in turns, without a rounding however large the position     */
  uint8_t axis[64];    /* which of the token's positions turns pair f                              */
} ecokv_rotary;

/* Fill *r for one position axis.  `original` (positions the model was made
 * for) matters to ECOKV_ROTARY_YARN only, `factor` (> 0) to every scaling.
 * Host only.  ECOKV_ERR_INVALID_ARG for sizes, bases (> 0, not 1) or codes out of range. */
ecokv_status ecokv_rotary_init(ecokv_rotary* r, int32_t rot_dim, int32_t layout, double base, int32_t scaling,
                               double factor, int32_t original);
/* The caller's own frequencies: inv_freq [rot_dim / 2] in radians a position. */
ecokv_status ecokv_rotary_set(ecokv_rotary* r, int32_t rot_dim, int32_t layout, const double* inv_freq,
                              float magnitude);
/* Several position axes (time, height, width): counts[a] consecutive pairs
 * turn with axis a; they add up to rot_dim / 2. */
ecokv_status ecokv_rotary_sections(ecokv_rotary* r, const int32_t* counts, int32_t axes);

/* Rows of one tensor [tokens][heads][d] and where its result goes.  x and y
 * may be the same rows (equal pointers and strides), else they do not overlap. */
typedef struct {
  const void* x;
  void* y;
  int64_t x_token, x_head; /* strides of x; 0: one row for all */
  int64_t y_token, y_head; /* strides of y */
  const void* norm;        /* [d] weights (dtype) of x / sqrt(mean(x^2) + eps) * weight, or NULL: no norm */
  int32_t heads;
} ecokv_rows;

/* q and k (either may be NULL), normed and rotated.
 *   r         : NULL = no rotation (norms alone)
 *   positions : int32 [axes][tokens], any sign; may be NULL when r is
 *   eps       : of the norms, >= 0
 * Each row is widened to fp32 and rounded once. */
ecokv_status ecokv_rotate(const ecokv_rotary* r, ecokv_dtype dtype, const ecokv_rows* q, const ecokv_rows* k,
                          const int32_t* positions, int32_t tokens, float eps, void* stream);

/* ------------------------------------------------------------------ paged cache
 * Slot s of sequence b lies in page table[b][s / page_size] at row s %
 * page_size.  Row (page, head, row) of K and of V is at
 * page * page_stride + head * head_stride + row * slot_stride of k and v: any
 * order of the three.  Slots from lengths[b] on hold anything, NaN too. */
typedef struct {
  void* k;
  void* v;
  int64_t page_stride, head_stride, slot_stride;
  int32_t n_pages;
  int32_t page_size;      /* a power of two, 8 .. 4096                                     */
  const int32_t* table;   /* [batch][table_stride] page numbers; entries past a sequence's
                             last page are not read                                        */
  int32_t table_stride;   /* page_size * table_stride <= 2^24                              */
  const int32_t* lengths; /* [batch] slots in use, the call's new tokens included          */
} ecokv_pages;

/* Tokens of a call: those of sequence b are starts[b] .. starts[b + 1] - 1
 * (int32 [batch + 1], from 0, not descending, the last = tokens); starts NULL:
 * token b is sequence b's only one (tokens = batch).  Token i of the T_b of
 * sequence b has slot lengths[b] - T_b + i. */

/* New tokens' rows: k (normed and rotated) and v (copied) to their slots,
 * q (may be NULL; normed and rotated) to q->y.  k->y and v->y are not used.
 * r, positions, eps as for ecokv_rotate.  A token whose slot or page number is
 * out of range is not written to the cache and, when ws is given, sets
 * ECOKV_ERR_DEVICE_INDEX in its status word; ws may be NULL, else at least
 * 256 bytes. */
ecokv_status ecokv_append(const ecokv_rotary* r, ecokv_dtype dtype, const ecokv_rows* q, const ecokv_rows* k,
                          const ecokv_rows* v, const ecokv_pages* cache, const int32_t* positions,
                          const int32_t* starts, int32_t tokens, int32_t batch, float eps, void* ws,
                          size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ attention
 * The shared prefix, as the eviction pass leaves one layer: row r < rows of
 * head h at h * head_stride + r * row_stride of k and v; or, with head_off
 * (ecokv_evict_adaptive), head h's rows head_off[h] .. head_off[h + 1] - 1 of the
 * `rows` rows at r * row_stride (head_stride is not used). */
typedef struct {
  const void* k;
  const void* v;
  int64_t head_stride, row_stride;
  int32_t rows;            /* rows a head, or of all heads with head_off; 0 <= rows <= 2^24 */
  const int32_t* head_off; /* device int32 [h_kv + 1] or NULL                               */
} ecokv_prefix;

typedef struct {
  int32_t h_q, h_kv;   /* query head q belongs to KV head q / (h_q / h_kv); h_q / h_kv <= 64 */
  int32_t d;           /* 128                                                                */
  int32_t tokens;      /* new tokens of the call                                             */
  int32_t batch;
  float scale;         /* of q . k; <= 0 selects 1 / sqrt(d)                                 */
  int64_t q_token, q_head, out_token, out_head; /* strides of q and out                      */
  uint32_t flags;      /* ECOKV_FLAG_FORCE_SIMT (bf16 on CUDA cores) or ECOKV_FLAG_TEST_STALL
                          (bf16 on tensor cores, else ECOKV_ERR_UNSUPPORTED: no tile of the cache
                          ever comes, the waits run out, ECOKV_ERR_TIMEOUT is recorded)            */
  uint32_t timeout_us; /* as in ecokv_params                                                 */
} ecokv_attend_params;

/* Bytes of workspace for `tokens` tokens of `batch` sequences (0: invalid). */
size_t ecokv_attend_workspace_size(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, ecokv_dtype dtype);

/* out[t][h] = sum_j softmax_j(scale q_t,h . k_j) v_j over every row of the
 * head's prefix and the slots j <= lengths[b] - T_b + i of the token's own
 * sequence: position enters through the rotation only.
 *   q, out : [tokens][h_q][d] (dtype), strides as in *p
 *   prefix : NULL = none.  One for all sequences of a call: sequences with prompts
 *            of their own take a call each
 *   cache  : NULL = none (then starts is not used)
 *   lse    : out, float32 [tokens][h_q], ln of the sum of exponentials; may be NULL
 * A row that sees no key: out = 0, lse = -inf; a token of no sequence (starts that do
 * not reach it) sees the prefix alone.  Scores, maxima, sums and the output are fp32;
 * for bf16 (but with ECOKV_FLAG_FORCE_SIMT) the softmax weights are rounded to bf16 for
 * the second product, as their factor V is: 2^-9 of a weight.  q, the prefix and the
 * slots in use must be finite, and V below 2^86 in magnitude (fp32, and bf16 on CUDA
 * cores: 2^102): the sums before the division are fp32, of weights up to 2^16 (there: 1).
 * The result is deterministic.  A page number out of range reads as zeros, a length
 * out of range is clamped, offsets out of order are clamped; each sets
 * ECOKV_ERR_DEVICE_INDEX in the workspace's status word.
 * ECOKV_ERR_UNSUPPORTED: d != 128, h_q / h_kv > 64, or more work than 31 bits count:
 *   h_kv (n u(rows) + (n + batch) u(page_size * table_stride)) >= 2^31, where
 *   n = ceil(tokens / (2 floor(128 / group))) and u(keys) = 2 ceil(keys / 128) + 4
 *   (fp32, and bf16 on CUDA cores: ceil(tokens / floor(64 / group)) and
 *   ceil(keys / 128)); u(0) = 0, group = h_q / h_kv.  The room of the table counts,
 *   not the lengths, which the host does not see. */
ecokv_status ecokv_attend(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q, const ecokv_prefix* prefix,
                          const ecokv_pages* cache, const int32_t* starts, void* out, float* lse, void* ws,
                          size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ drafted tokens
 * A sequence's new tokens i < T_b are drafts that follow each other as a tree: draft i
 * goes on from draft parents[t] < i of its sequence, or, at -1, from the last token
 * before them.  Its position is its parent's and one; its slot lengths[b] - T_b + i as
 * for any new token, so ecokv_append puts it into the cache. */

/* mask[t][words]: bit j % 64 of word j / 64 is set where draft t sees draft j of its
 * sequence: j is t itself or an ancestor.
 *   parents : int32 [tokens]
 *   mask    : out, uint64 [tokens][words], 1 <= words <= 64
 * Rows of tokens of no sequence are left as they were.  A parent out of range (not -1 ..
 * i - 1) counts as -1, a draft from 64 * words on gets a row of zeros, and each sets
 * ECOKV_ERR_DEVICE_INDEX in the status word of ws (may be NULL, else at least 256
 * bytes). */
ecokv_status ecokv_tree_mask(const int32_t* parents, const int32_t* starts, int32_t tokens, int32_t batch,
                             uint64_t* mask, int32_t words, void* ws, size_t ws_bytes, void* stream);

/* As ecokv_attend (its arguments, workspace and limits), where token i of sequence b sees
 * the prefix, the slots below lengths[b] - T_b and those of the tokens j of its
 * sequence whose bit is set in mask[t] (uint64 [tokens][words]): any bits, those of
 * later tokens too.  Bits of j >= T_b are not read, tokens j >= 64 * words are not seen.
 * cache and mask are wanted.  ECOKV_ERR_UNSUPPORTED: words > 64 too. */
ecokv_status ecokv_attend_tree(const ecokv_attend_params* p, ecokv_dtype dtype, const void* q,
                               const ecokv_prefix* prefix, const ecokv_pages* cache, const int32_t* starts,
                               const uint64_t* mask, int32_t words, void* out, float* lse, void* ws, size_t ws_bytes,
                               void* stream);

/* A float32 number of each row of a cache or a prefix (the attention weight that its key
 * has had): of row (page, head, row) at page * page_stride + head * head_stride + row *
 * slot_stride of w, of a prefix's row r of head h at h * head_stride + r * slot_stride (with
 * head_off r * slot_stride).  Strides count elements and are positive. */
typedef struct {
  float* w;
  int64_t page_stride, head_stride, slot_stride;
} ecokv_weights;

/* Accepted drafts: row lengths[b] - T_b + accepted[b][i] of K, V and, where given, the
 * weights moves to row lengths[b] - T_b + i, i < counts[b], and lengths_out[b] = lengths[b]
 * - T_b + counts[b].
 *   accepted    : int32 [batch][stride], the drafts' numbers in their sequence, ascending
 *                 (a path from the root does)
 *   counts      : int32 [batch], 0 <= counts[b] <= T_b, stride
 *   weights     : of the cache, or NULL
 *   lengths_out : int32 [batch]; may be the cache's lengths, else it overlaps no input
 * A sequence's pages with new tokens are its own.  A sequence with numbers out of
 * range or out of order keeps none of its drafts (as with counts[b] = 0), a row whose
 * page number is out of range is not moved, and each sets ECOKV_ERR_DEVICE_INDEX in the
 * status word of ws (may be NULL, else at least 256 bytes).
 * ECOKV_ERR_UNSUPPORTED: batch * h_kv > 2^29. */
ecokv_status ecokv_commit(ecokv_dtype dtype, const ecokv_pages* cache, int32_t h_kv, const int32_t* accepted,
                          int32_t stride, const int32_t* counts, const int32_t* starts, int32_t tokens, int32_t batch,
                          const ecokv_weights* weights, int32_t* lengths_out, void* ws, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ attention weights of keys */
typedef struct {
  int32_t h_q, h_kv, d, tokens, batch;  /* as in ecokv_attend_params */
  float scale;
  float decay;                          /* of the weights so far, finite, >= 0 (0: they do not count) */
  int64_t q_token, q_head;
  uint32_t flags;                       /* as in ecokv_attend_params */
  uint32_t timeout_us;
} ecokv_weigh_params;

/* Bytes of workspace for `tokens` tokens of `batch` sequences (0: invalid). */
size_t ecokv_weigh_workspace_size(int32_t tokens, int32_t batch, int32_t h_q, int32_t h_kv, ecokv_dtype dtype);

/* What every key is given by the new tokens' attention, added over the query heads of
 * its KV head and the tokens that see it as in ecokv_attend:
 *   A = decay * A + sum_{t,h} exp(scale q_t,h . k - lse[t][h])
 * for every row of the prefix (over the tokens of all sequences) and every slot in
 * use, where a new token's own slot starts at 0.  lse is what ecokv_attend has left; for
 * drafts, once they are committed, that of the accepted ones (their ancestors are
 * the tokens before them).  A row whose lse is -inf gives nothing, nor does a token of no
 * sequence (without a cache: every token counts).
 *   prefix, cache                    : either may be NULL; v is not read
 *   prefix_weights, weights          : theirs, wanted where the prefix (cache) is; weights of slots
 *                                      from lengths[b] on are left as they were
 * Slots in use belong to one sequence each.  Sums are fp32 and in a fixed order: the
 * result is deterministic.  q, lse and the keys in use must be finite (lse: or -inf).
 * A call of no tokens changes nothing.  One that ends with ECOKV_ERR_TIMEOUT in the status
 * word has weighed some keys, others by a part of their rows or not at all: the weights
 * are lost.
 * Page numbers, lengths and offsets out of range: as for ecokv_attend; a slot without a
 * page has no weight.  ECOKV_ERR_UNSUPPORTED: d, h_q / h_kv as for ecokv_attend, and
 * more work than 31 bits count, which it is not while
 *   h_kv (k(rows) (32 + n) + k(page_size * table_stride) (40 batch + n + 48)) < 2^31,
 * n = tokens h_q / h_kv, k(keys) = ceil(keys / 128). */
ecokv_status ecokv_weigh(const ecokv_weigh_params* p, ecokv_dtype dtype, const void* q, const float* lse,
                         const ecokv_prefix* prefix, const ecokv_pages* cache, const int32_t* starts,
                         const ecokv_weights* prefix_weights, const ecokv_weights* weights, void* ws, size_t ws_bytes,
                         void* stream);

/* ------------------------------------------------------------------ pruning
 * A sequence of more than `limit` slots keeps `budget` of them in each head: the
 * `first` first ones, the `recent` last ones and between them the ones of the
 * largest weights (of equal ones the lower slot; NaN counts below every number), each
 * head for itself.  The rows kept, in their order, take slots 0 ..
 * of the same cache, or of another one.
 *   0 <= first, 0 <= recent, first + recent <= budget, 1 <= budget <= limit
 *   to          : NULL = the same cache; else one of the same dtype whose pages in use are no
 *                 pages in use of `cache`; its table has entries for the rows kept, its
 *                 lengths are not read.  Sequences of up to `limit` slots are copied whole.
 *   to_weights  : where the kept rows' weights go (in the same cache: `weights` itself),
 *                 NULL = they are not moved
 *   idx         : out, int32 [batch][h_kv][limit], the kept slots, then -1
 *   lengths_out : int32 [batch], budget or, up to limit, lengths[b]; may be the lengths of
 *                 either cache, else it overlaps no input
 * Slots in use belong to one sequence each.  A slot whose page number is out of range has
 * weight -inf and its row is not moved; a length out of range is clamped; each sets
 * ECOKV_ERR_DEVICE_INDEX in the status word of ws (may be NULL, else at least 256
 * bytes).  The result is deterministic.
 * ECOKV_ERR_UNSUPPORTED: batch * h_kv > 2^29. */
typedef struct {
  int32_t h_kv, batch;
  int32_t budget, limit, first, recent;
} ecokv_prune_params;

ecokv_status ecokv_prune(const ecokv_prune_params* p, ecokv_dtype dtype, const ecokv_pages* cache,
                         const ecokv_weights* weights, const ecokv_pages* to, const ecokv_weights* to_weights,
                         int32_t* idx, int32_t* lengths_out, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* ECOKV_DECODE_H */
