/*
 * eb_attention.h -- the steps of a decoder layer between its QKV and its O
 * projection, for serving: a paged cache of keys and values, the norm and
 * rotation of query and key heads with the write into that cache, and
 * attention over it (paper section 2.1: the backbones are decoder stacks;
 * section 3.2: the backbone's keys and values are state that the action expert
 * reads on every tick while the backbone is refreshed less often).
 *
 * One step of a batch: eb_kv_extend once, then for every layer the QKV
 * projection (eb_qlinear_fused), eb_rope_append, eb_attention and the O
 * projection.  Lengths, block tables and slots stay on the GPU: no call reads
 * them back, so a step with fixed row and sequence counts can be captured into
 * a HIP graph and replayed as the lengths grow.
 *
 * Conventions beyond those of eb.h:
 *   - Rows.  The new tokens of all sequences are packed: sequence b has rows
 *     q_start[b] .. q_start[b + 1] - 1.  Rows behind the last sequence are
 *     padding: they are read by nothing and their outputs left as they were.
 *   - Device integers cannot be checked on the host.  A page outside
 *     0 .. pages - 1 is a missing page and a slot outside 0 .. pages * page - 1
 *     is no slot; lengths and offsets are clamped to their arrays.  No value of
 *     them makes a kernel read or write out of bounds.
 *   - What a mask hides may hold anything, infinities and NaN included, and so
 *     may cache rows that no visible key lives in.
 *   - Calls on one stream run in order; a workspace is used in stream order,
 *     so calls that share one must be ordered (two graphs that may run at the
 *     same time need one each, and so do two host threads on one stream: a call
 *     is up to three launches).
 */
#ifndef EB_ATTENTION_H
#define EB_ATTENTION_H

#include "eb.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The keys and values of one layer: k and v are [pages][heads][page][dim],
 * device, 16-byte aligned.  One page of >= n tokens is a plain cache of one
 * sequence. */
typedef struct {
  void *k;
  void *v;
  int32_t type;     /* EB_F16 or EB_BF16 */
  int32_t heads;    /* key/value heads, 1 .. 1024 */
  int32_t dim;      /* 64, 128 or 256 */
  int32_t page;     /* tokens per page: a power of two, 16 .. 65536 */
  int32_t pages;    /* >= 1, pages * page <= 2^31 - 1 */
  int32_t reserved; /* must be 0 */
} eb_kv_cache;

/* New tokens join the sequences of a batch.  Sequence b holds cached[b] tokens
 * and gets added[b] more (negative values count as 0), as far as the step's rows
 * go: the new tokens of all sequences behind the first `rows` do not join, take no
 * page and are counted in short_rows.  total_b is cached[b] and those of
 * sequence b that join.  Its table row holds a page for each
 * `page` tokens; the ceil(total_b / page) - ceil(cached[b] / page) pages it
 * lacks are taken from the top of the stack free_pages[0 .. n_free - 1]:
 * sequence 0 first, then sequence 1, and so on, each in ascending order, the
 * first page being free_pages[n_free - 1].  Written:
 *   table      the new pages' entries (-1 where the stack is empty or its entry
 *              is no page); all others stay
 *   q_start    [batch + 1]: exclusive prefix sums of the tokens that join: of
 *              added, at most `rows`
 *   kv_len     [batch]: total_b, at most table_stride * page
 *   positions  [rows]: the place in its sequence of each row's token
 *   slots      [rows]: page * tokens per page + place in the page, where
 *              eb_rope_append writes the token; -1 where it has no page
 *   n_free_out [1]: pages left (another integer than n_free)
 *   short_rows [1]: new tokens that did not join or have no page (0: all went
 *              well); a sequence that ran past its table row has its rows' places
 *              counted from the end of that row, so their attention is void
 * Rows behind the last sequence get slot -1 and position 0.  Pages of finished
 * sequences go back by pushing them onto the stack. */
typedef struct {
  const int32_t *cached;     /* [batch] */
  const int32_t *added;      /* [batch] */
  int32_t *table;            /* [batch][table_stride], in and out */
  const int32_t *free_pages; /* [free_capacity] */
  const int32_t *n_free;     /* [1], clamped to 0 .. free_capacity */
  int32_t *n_free_out;       /* [1] */
  int32_t *q_start;          /* [batch + 1] */
  int32_t *kv_len;           /* [batch] */
  int32_t *slots;            /* [rows] */
  int32_t *positions;        /* [rows] */
  int32_t *short_rows;       /* [1] */
  int32_t batch;             /* 1 .. 4096 */
  int32_t rows;              /* 0 .. 2^24: the rows that the step runs with */
  int32_t page;              /* as in eb_kv_cache */
  int32_t pages;
  int32_t table_stride;      /* >= 1, table_stride * page <= 2^30 */
  int32_t free_capacity;     /* 0 .. 2^27 */
} eb_kv_extend_op;

/* EB_ERR_INVALID: null pointer (free_pages may be null with free_capacity 0,
 * slots and positions with rows 0), a size out of range, an output that
 * overlaps an input or another output.  EB_ERR_ALIGN: a pointer that is not
 * 4-byte aligned. */
eb_status eb_kv_extend(const eb_kv_extend_op *op, hipStream_t stream);

/* Rotated pairs of a head: (j, j + rot / 2), or (2 j, 2 j + 1), for
 * 0 <= j < rot / 2; elements from rot on stay. */
#define EB_ROT_HALF 0
#define EB_ROT_ADJACENT 1

/* From the rows of a QKV projection (q_heads query heads, then the cache's
 * heads of keys, then as many of values, each of dim elements): queries and
 * keys are normalised where a norm weight is given,
 *   x <- x * g / sqrt(eps + mean x^2)        (over the head's dim elements)
 * and rotated: pair j = (a, b) of a head turns by t = positions[axis][row] *
 * freqs[j] radians to (a cos t - b sin t, b cos t + a sin t), pair j belonging
 * to the axis whose section holds it (sections[0] pairs for axis 0, then
 * sections[1] for axis 1, ...: e.g. time, height and width).  Queries go to
 * q_out, keys and values to the cache at the row's slot.  A row without a slot
 * writes nothing.  Two rows with one slot leave either's values there, element
 * by element.
 * All arithmetic is fp32, the angle's in fp64 (so that far positions keep
 * their phase); each output is rounded once, to nearest even, in the cache's
 * type.  Angles are exact to 2^-21 of a turn for |position * freq| < 2^31. */
typedef struct {
  eb_kv_cache cache;
  const void *qkv;          /* [rows][qkv_stride] of qkv_type, 16-byte aligned */
  void *q_out;              /* [rows][q_stride] of the cache's type, 16-byte aligned */
  const int32_t *slots;     /* [rows] */
  const int32_t *positions; /* [n_axes][pos_stride]; null with rot 0 */
  const float *freqs;       /* [rot / 2]; null with rot 0 */
  const float *q_norm;      /* [dim], 16-byte aligned, or null: no norm of queries */
  const float *k_norm;      /* [dim], 16-byte aligned, or null: no norm of keys */
  int64_t qkv_stride;       /* elements, >= (q_heads + 2 heads) * dim, a multiple of 8 */
  int64_t q_stride;         /* elements, >= q_heads * dim, a multiple of 8 */
  int64_t pos_stride;       /* elements, >= rows */
  int32_t qkv_type;         /* EB_F32, EB_F16 or EB_BF16 */
  int32_t q_heads;          /* 1 .. 4096 */
  int32_t rows;             /* 0 .. 2^24 */
  int32_t rot;              /* rotated elements of a head: a multiple of 8, 0 .. dim */
  int32_t style;            /* EB_ROT_HALF or EB_ROT_ADJACENT */
  int32_t n_axes;           /* 1 .. 3 */
  int32_t sections[3];      /* each >= 0, those of the axes adding up to rot / 2 */
  float norm_eps;           /* finite, >= 0 (a zero head needs eps > 0; eps + the mean of squares,
                               in fp32, is taken as 2^-126 at least) */
} eb_rope_append_op;

/* EB_ERR_INVALID: null pointer, a size, stride or enum out of range, an output
 * that overlaps an input or another output.  EB_ERR_ALIGN: a pointer or stride
 * not aligned as stated.  EB_ERR_UNSUPPORTED: a head size or cache type other
 * than those above. */
eb_status eb_rope_append(const eb_rope_append_op *op, hipStream_t stream);

/* Which keys a token sees.  Token i of the new tokens of sequence b is at place
 * p = kv_len[b] - (q_start[b + 1] - q_start[b]) + i; key j of its kv_len[b]
 * keys is seen if (j <= p, or j < prefix[b], or the mask is EB_MASK_FULL) and
 * (window is 0, or p - j < window). */
#define EB_MASK_CAUSAL 0
#define EB_MASK_FULL 1

/* Attention of the new tokens of a batch over the cache, which holds their own
 * keys and values already: with t_j = scale * q . k_j, capped to
 * softcap * tanh(t_j / softcap) where softcap > 0,
 *   out = sum_j e^{t_j} v_j / sum_j e^{t_j}      over the keys j that are seen.
 * A row that sees no key is 0, and so is one whose scores are all -infinity, over
 * finite values; a key on a missing page is not seen.  Query head
 * h reads key/value head h / (q_heads / heads).
 * max_new and max_kv are the host's bounds on any sequence's new tokens and
 * kv_len: they decide the launch; tokens past max_new are not computed (their
 * rows stay), keys past max_kv are still seen.
 * Products take the 16-bit values on the matrix cores with fp32 sums; running
 * maxima and sums of the softmax are fp32; capped scores are off by at most
 * softcap * 2^-20, which is why caps past 2^10 are not taken.  The weights e^{t - max} are rounded
 * once to the cache's type for the second product (each off by at most 2^-8 of
 * itself for EB_BF16, 2^-11 for EB_F16, or 2^-36 of the row's largest weight, where
 * that is more), as is the output.
 * With several sequences, or few rows, the keys of a row are split over
 * workgroups and joined in a fixed order by a second launch: results are
 * deterministic. */
typedef struct {
  eb_kv_cache cache;
  const void *q;          /* [rows][q_stride] of the cache's type, 16-byte aligned */
  void *out;              /* [rows][out_stride] of the cache's type, 16-byte aligned */
  const int32_t *table;   /* [batch][table_stride] */
  const int32_t *q_start; /* [batch + 1] */
  const int32_t *kv_len;  /* [batch], clamped to 0 .. table_stride * page */
  const int32_t *prefix;  /* [batch], or null: no prefix */
  int64_t q_stride;       /* elements, >= q_heads * dim, a multiple of 8 */
  int64_t out_stride;     /* elements, >= q_heads * dim, a multiple of 8 */
  int32_t rows;           /* 0 .. 2^24, rows * q_heads / heads <= 2^30 */
  int32_t batch;          /* 1 .. 4096 */
  int32_t q_heads;        /* a multiple of the cache's heads, at most 4096 */
  int32_t table_stride;   /* >= 1, table_stride * page <= 2^30 */
  int32_t max_new;        /* >= 1 */
  int32_t max_kv;         /* >= 1 */
  int32_t mask;           /* EB_MASK_CAUSAL or EB_MASK_FULL */
  int32_t window;         /* >= 0; 0: none */
  float scale;            /* |scale| <= 65536 */
  float softcap;          /* 0: none, or 2^-10 .. 2^10 */
} eb_attention_op;

/* Bytes of workspace eb_attention needs for *op: the fp32 sums of rows whose
 * keys are split over workgroups.  0 when it needs none or *op is invalid.
 * Depends on sizes, types, mask, window and whether there is a prefix, not on
 * device contents. Host-only
 * but for the current device's CU count. */
size_t eb_attention_workspace_bytes(const eb_attention_op *op);

/* workspace: device, 256-byte aligned, at least eb_attention_workspace_bytes
 * bytes, or null with 0 bytes where none is needed.
 * EB_ERR_INVALID: null pointer, a size, stride or enum out of range, a
 * workspace too small, `out` or the workspace overlapping another operand.
 * EB_ERR_ALIGN and EB_ERR_UNSUPPORTED as for eb_rope_append. */
eb_status eb_attention(const eb_attention_op *op, void *workspace, size_t workspace_bytes,
                       hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* EB_ATTENTION_H */
