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
 * its pointers.
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

#ifdef __cplusplus
}
#endif

#endif /* ECOKV_DECODE_H */
