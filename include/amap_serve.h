/*
 * amap_serve.h -- what a transformer does with the heads a composed map has
 * split: rotary positions, a paged key/value cache, the attention of one new
 * token per request that reads it, and the choice of the next token.  Their
 * addresses depend on data that
 * lives on the device (positions, slots, block tables, lengths), so they are
 * operators of their own beside amap_execute.
 *
 * Conventions (those of amap.h, and)
 *  - Every pointer in an argument struct is a DEVICE pointer unless marked
 *    host.  Strides and offsets count ELEMENTS; the innermost dimension (the
 *    elements of a head) is always contiguous.
 *  - Every call checks its arguments, enqueues its one kernel on `cuda_stream`
 *    of the current device and returns without synchronising or allocating.
 *    A refused call enqueues nothing; amap_serve_error() says why.
 *  - Kernels are launched with programmatic stream serialisation and touch no
 *    buffer before the kernel ahead of them on the stream has completed.
 *  - What a kernel reads from device memory as an index (page numbers, slots,
 *    lengths, counts) is bounds-checked there: a bad one is skipped as stated
 *    at each operator and never used as an address.
 */
#ifndef AMAP_SERVE_H_
#define AMAP_SERVE_H_

#include <stdint.h>

#include "amap.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum amap_dtype {
  AMAP_BF16 = 1,
  AMAP_FP16 = 2,
  AMAP_FP32 = 3,
  AMAP_E4M3 = 4 /* 8 bits: 4 exponent, 3 mantissa, no infinity, largest value 448; caches only */
} amap_dtype;

/* why the last amap_pages_* / amap_rope_* / amap_attend* call of this thread did not return AMAP_OK ("" if none) */
const char *amap_serve_error(void);

/* ---------------------------------------------------------------------------
 * Pages.  A cache is a pool of n_pages pages of page_size tokens; row r of the
 * block table lists the pages of request r in the order of its tokens; pages
 * in no row are stacked in free_pages[0 .. *free_count).
 *
 * amap_pages_extend: one step.  Request r = 0 .. n_requests-1 holds seq_lens[r]
 * tokens and wants new_lens[r] more.  In the order of the requests, with
 *   need(r) = ceil((seq+new)/page_size) - ceil(seq/page_size),
 * the pages needed are popped off the stack and entered in the block table (in
 * place), and the step's tokens, all requests' one after another, get
 *   slots[i]     = page * page_size + offset   of the place token i belongs in
 *   positions[i] = its position in its request
 *   requests[i]  = its request
 * (-1, 0, -1 for i beyond the last token, up to max_tokens, so that a captured
 * graph of fixed size skips them).  status[r]: 0 granted, else the request gets
 * nothing in this step:
 *   1  a negative length, or more tokens than its table row has room for
 *   2  the pool: the needs of the requests up to r add up to more than *free_count
 *   3  the tokens of the requests up to r add up to more than max_tokens
 * (sums run over all requests that status 1 does not concern, granted or not,
 * so the answer does not depend on timing.)  A request that wants nothing and
 * a request whose last page has room need no page and are not refused for 2.
 *   query_start[r]   first token of request r in the step (n_requests + 1 entries)
 *   seq_lens_out[r]  seq_lens[r] + granted tokens;  free_count_out: pages left
 * The inputs seq_lens and free_count are not changed and must not overlap the
 * outputs: calling again gives the same answer.  *free_count is clamped to
 * [0, free_capacity]; a token whose page number is outside [0, n_pages) gets
 * slot -1.
 * ------------------------------------------------------------------------- */
typedef struct amap_pages_extend_args {
  int32_t n_requests;    /* R >= 1 */
  int32_t max_pages;     /* entries of a table row */
  int32_t page_size;     /* >= 1; n_pages * page_size and max_pages * page_size below 2^31 */
  int32_t n_pages;       /* page numbers are 0 .. n_pages-1 */
  int32_t free_capacity; /* entries of free_pages */
  int32_t max_tokens;    /* entries of slots, positions, requests; >= 1 */
  int64_t table_stride;  /* between table rows, >= max_pages */
  const int32_t *new_lens;
  const int32_t *seq_lens;
  int32_t *block_table;
  const int32_t *free_pages;
  const int32_t *free_count;
  int32_t *query_start;
  int32_t *slots;
  int32_t *positions;
  int32_t *requests;
  int32_t *seq_lens_out;
  int32_t *free_count_out;
  int32_t *status;
} amap_pages_extend_args;
int amap_pages_extend(const amap_pages_extend_args *args /* host */, void *cuda_stream);

/* amap_pages_release: the pages of the requests with done[r] != 0 go back on
 * the stack, request by request in the order of their tokens, on top of what
 * is there; seq_lens_out[r] is 0 for them and seq_lens[r] for the others.
 * A negative table entry is a hole (a page given back earlier, behind a window)
 * and is passed over; amap_pages_release_within passes over every entry outside
 * [0, n_pages).
 * free_pages changes only at and above *free_count; what does not fit
 * free_capacity is dropped and not counted.  Table rows keep their entries. */
typedef struct amap_pages_release_args {
  int32_t n_requests;
  int32_t max_pages;
  int32_t page_size;
  int32_t free_capacity;
  int64_t table_stride;
  const uint8_t *done; /* n_requests bytes */
  const int32_t *seq_lens;
  const int32_t *block_table;
  int32_t *free_pages;
  const int32_t *free_count;
  int32_t *seq_lens_out;
  int32_t *free_count_out;
} amap_pages_release_args;
int amap_pages_release(const amap_pages_release_args *args /* host */, void *cuda_stream);
int amap_pages_release_within(const amap_pages_release_args *args /* host */, int32_t n_pages, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Rotary positions with several axes.  The first rotary_dim elements of a head
 * are rotary_dim/2 pairs; pair i belongs to one position axis (text: one axis;
 * images and video: time, height, width) and turns by the angle
 *     th = positions[axis(i)][token] * inv_freq[i]:
 *     (a, b) -> scale * (a cos th - b sin th,  a sin th + b cos th);
 * elements behind rotary_dim pass through.  The gradient of the inputs is the
 * same operator with th negated (`inverse`).  AMAP_PAIRS_HALF: pair i is
 * (x[i], x[i + rotary_dim/2]); AMAP_PAIRS_ADJACENT: (x[2i], x[2i+1]).
 *
 * Positions are whole numbers of any sign and size: the angle is reduced modulo
 * a full turn in 64-bit fixed point (inv_freq/2pi as a fraction of 2^64, times
 * the position, wraps exactly), so it is as exact at position 2^31 as at 1.
 * Arithmetic in 32 bits, rounded once.
 *
 * The plan is host memory only and may be used on any device and stream.
 * ------------------------------------------------------------------------- */
#define AMAP_PAIRS_HALF 0
#define AMAP_PAIRS_ADJACENT 1
#define AMAP_ROPE_MAX_DIM 256
#define AMAP_ROPE_MAX_AXES 4
typedef struct amap_rope_t amap_rope_t;
int amap_rope_plan(int32_t head_dim,       /* 1 .. AMAP_ROPE_MAX_DIM */
                   int32_t rotary_dim,     /* even, 0 .. head_dim */
                   const double *inv_freq, /* host, rotary_dim/2 finite values */
                   const int32_t *axis,    /* host, rotary_dim/2 values in [0, n_axes); NULL: all 0 */
                   int32_t n_axes,         /* 1 .. AMAP_ROPE_MAX_AXES */
                   int32_t pairs, float scale, amap_rope_t **out);
void amap_rope_destroy(amap_rope_t *plan);

/* rows x heads x head_dim elements: x is read, y written (y may be x itself with x's strides; else y must not overlap
 * any part's x).  No element of a y may be one of another part's x or y: parts turned in place may lie side by side in
 * one buffer, with the same row stride where their bytes interleave. */
typedef struct amap_rope_part {
  const void *x;
  void *y;
  int64_t x_row, x_head, y_row, y_head; /* strides */
  int32_t heads;
  int32_t reserved; /* 0 */
} amap_rope_part;

typedef struct amap_rope_args {
  int32_t n_parts; /* 1 .. 4 tensors turned by the same positions in one launch (q and k, or their gradients) */
  int32_t dtype;   /* AMAP_BF16, AMAP_FP16 or AMAP_FP32 */
  int64_t rows;    /* tokens, below 2^31 */
  const void *positions;
  int64_t position_axis, position_row; /* strides of positions[axis][row] */
  int32_t position_bits;               /* 32 or 64: signed whole numbers */
  int32_t inverse;                     /* 1: turn backwards (the gradient) */
  amap_rope_part part[4];
} amap_rope_args;
int amap_rope_rotate(const amap_rope_t *plan, const amap_rope_args *args /* host */, void *cuda_stream);

/* A paged cache: K and V as [page][token in page][head][element] with any strides over the first three. */
typedef struct amap_cache {
  void *k, *v;
  int64_t k_page, k_token, k_head, v_page, v_token, v_head; /* strides */
  int32_t n_pages, page_size, heads, head_dim;              /* n_pages * page_size below 2^31 */
  int32_t dtype;                                            /* AMAP_BF16, AMAP_FP16 or AMAP_E4M3 */
  float k_scale, v_scale; /* an element stands for its value times the scale (1 for 16-bit caches) */
} amap_cache;

/* What amap_attend's copies need to know of a cache, encoded once where the cache is set up (host memory, any alignment;
 * to be encoded anew when the cache's description changes). */
typedef struct amap_cache_maps {
  uint64_t k_map[16], v_map[16];
  int32_t box_shift, usable;
} amap_cache_maps;
int amap_cache_encode(const amap_cache *cache /* host */, amap_cache_maps *out /* host */);

/* amap_rope_append: a step's q, k, v [rows][heads][head_dim] in one launch.
 *   q_out = rotated q;  K[slots[i]] = rotated k of row i;  V[slots[i]] = v of row i.
 * A slot outside [0, n_pages*page_size) writes nothing to the cache (its q is rotated all the same).  Slots must be
 * distinct.  A 16-bit cache has the type of q, k, v; an e4m3 cache takes value/scale, a division in 32
 * bits, rounded to nearest even and clamped to +-448 (NaN stays NaN). */
typedef struct amap_append_args {
  int64_t rows;
  int32_t dtype;   /* AMAP_BF16 or AMAP_FP16 */
  int32_t q_heads; /* 0: k and v only */
  const void *q, *k, *v;
  void *q_out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, q_out_row, q_out_head;
  const void *positions;
  int64_t position_axis, position_row;
  int32_t position_bits;
  int32_t reserved; /* 0 */
  const int32_t *slots;
  amap_cache cache;
} amap_append_args;
int amap_rope_append(const amap_rope_t *plan, const amap_append_args *args /* host */, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Attention of one new token per request over the paged cache.  For request r
 * with n = seq_lens[r] tokens in the cache (the new one included) and q head h,
 * which reads cache head h * heads / q_heads:
 *   s_t = scale * <q[r][h], K[t]>        t = max(0, n - window) .. n-1  (window 0: from 0)
 *   s_t = softcap * tanh(s_t / softcap)  if softcap > 0
 *   out = sum_t exp(s_t - lse) V[t],     lse = log sum_t exp(s_t)
 * A request with no token (n <= 0) gets zeros and lse = -inf.  n is clamped to
 * max_pages * page_size; a table entry outside [0, n_pages) is a hole whose
 * tokens take no part.  Only tokens that take part count: of the pages in a
 * request's row, whole runs of up to 64 tokens may be read, so what lies behind
 * its end there may be anything, NaN included.  Pages in no row are not read.
 * Scores, maximum, sum and output are kept in 32 bits.
 *
 * Every wait inside the kernel ends: one that has lasted two seconds is given up, and the int32 at byte
 * amap_attend_workspace()'s *failed of the workspace becomes 1 (the outputs of this call and of later ones are then worth
 * nothing until the workspace has been zeroed; before it ends, a block lets its copies land, with the same limit).
 *
 * workspace: amap_attend_workspace() bytes, 256-byte aligned, ZEROED before its first use; every call leaves
 * it ready for the next.  Calls that share a workspace must have the same q_heads, cache.heads and cache.head_dim and be
 * ordered (one stream, or events); n_requests may be anything up to what the workspace was sized for.
 * ------------------------------------------------------------------------- */
typedef struct amap_attend_args {
  int32_t n_requests;
  int32_t q_heads;   /* a multiple of cache.heads */
  int32_t dtype;     /* of q and out: AMAP_BF16 or AMAP_FP16; a 16-bit cache has the same */
  int32_t max_pages; /* entries of a table row; max_pages * page_size below 2^31 */
  const void *q;
  void *out;
  float *lse; /* [n_requests][q_heads], may be NULL */
  int64_t q_row, q_head, out_row, out_head, lse_row;
  const int32_t *block_table;
  int64_t table_stride;
  const int32_t *seq_lens;
  float scale;
  float softcap;  /* 0: none */
  int32_t window; /* 0: none */
  int32_t reserved; /* 0 */
  void *workspace;
  int64_t workspace_bytes;
  const amap_cache_maps *maps; /* host; of `cache`; NULL: encoded in the call */
  amap_cache cache; /* head_dim a multiple of 8 (e4m3: 16), up to 256; rows aligned to 16 bytes */
} amap_attend_args;
int amap_attend(const amap_attend_args *args /* host */, void *cuda_stream);
/* bytes of workspace for up to n_requests requests on the current device, and where in it the mark of a failure is */
int amap_attend_workspace(int32_t n_requests, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int64_t *bytes,
                          int64_t *failed /* may be NULL */);

/* ---------------------------------------------------------------------------
 * A paged cache of 4 bits.  A head's elements are held in groups of 32 or 64:
 *   low  = the group's smallest element, rounded down to bf16;
 *   step = (its largest element - low) / 15, rounded to fp32 and that to bf16;
 *   code = (element - low) / step, rounded to nearest even, within 0 .. 15 (0
 *          where step is 0), and stands for low + step * code.
 * A group that holds a NaN or an infinity, or whose low or step is none of
 * bf16's finite numbers, reads as NaN throughout.
 *
 * A page of a head is one run of page_size / 16 cells of 16 tokens, codes and
 * groups' numbers of K and V together (amap_packed_bytes() in all); what lies
 * where inside a cell is the library's own.  Memory that no token has been
 * written to may hold anything.
 * ------------------------------------------------------------------------- */
typedef struct amap_packed {
  void *data;                                  /* aligned to 16 bytes */
  int64_t page, head;                          /* strides in BYTES between pages and between a page's heads: multiples of 16 */
  int32_t n_pages, page_size, heads, head_dim; /* page_size a multiple of 16, n_pages * page_size below 2^31; head_dim 64, 96, 128 or 256 */
  int32_t group;                               /* 32, or 64 where it divides head_dim */
  int32_t reserved;                            /* 0 */
} amap_packed;
/* bytes of a page of a head; 0, with the reason, where there is no such cache */
int64_t amap_packed_bytes(int32_t page_size, int32_t head_dim, int32_t group);

/* amap_packed_append: a step's q, k, v [rows][heads][head_dim] in one launch, as amap_rope_append: q_out = rotated q, and
 * the rotated k and the v of row i go to slots[i].  k is quantised as the exact rotation gives it (64 bits).
 * plan NULL: nothing turns, and positions are not read.  A slot outside [0, n_pages*page_size) writes nothing to the
 * cache.  Slots must be distinct. */
typedef struct amap_packed_append_args {
  int64_t rows;
  int32_t dtype;   /* AMAP_BF16 or AMAP_FP16 */
  int32_t q_heads; /* 0: k and v only */
  const void *q, *k, *v;
  void *q_out;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, q_out_row, q_out_head;
  const void *positions;
  int64_t position_axis, position_row;
  int32_t position_bits;
  int32_t reserved; /* 0 */
  const int32_t *slots;
  amap_packed cache;
} amap_packed_append_args;
int amap_packed_append(const amap_rope_t *plan, const amap_packed_append_args *args /* host */, void *cuda_stream);

/* amap_packed_read: k[i], v[i] [heads][head_dim] = what the cache holds at slots[i], in 32 bits and rounded once; zeros for a
 * slot outside [0, n_pages*page_size). */
typedef struct amap_packed_read_args {
  int64_t rows;
  int32_t dtype;    /* AMAP_BF16, AMAP_FP16 or AMAP_FP32 */
  int32_t reserved; /* 0 */
  const int32_t *slots;
  void *k, *v;
  int64_t k_row, k_head, v_row, v_head; /* strides */
  amap_packed cache;
} amap_packed_read_args;
int amap_packed_read(const amap_packed_read_args *args /* host */, void *cuda_stream);

/* amap_packed_attend: amap_attend over such a cache; `maps` and `cache` of the arguments are not looked at.  The workspace is
 * amap_attend's, and may be shared with its calls as those may share it. */
int amap_packed_attend(const amap_attend_args *args /* host */, const amap_packed *cache /* host */, void *cuda_stream);

/* ---------------------------------------------------------------------------
 * Sampling: a token for every row of logits, from one uniform number in [0, 1).
 * With x_i the row's logits, w_i = exp((x_i - max x) / temperature), and tokens
 * ordered by their logits, ties by their index:
 *   top_k  keeps the first top_k tokens (0 or less: all);
 *   min_p  keeps those with w_i >= min_p;
 *   top_p  keeps, of what these leave, the shortest beginning of the order whose
 *          sum of w is at least top_p of their sum, one token at least;
 * the token drawn is the first, by index, whose sum of w over the kept tokens up
 * to it is above uniform times the sum over all kept ones.  temperature 0 or
 * less: the largest logit, the first of them.  A NaN counts as -infinity; a row
 * with no logit above -infinity gives -1; where the largest is +infinity, the
 * tokens that have it share the weight.  A temperature above 1e30 counts as 1e30.
 * A uniform number outside counts as the nearest inside, NaN as 0; so do min_p
 * and top_p of a row; those of a row that are NaN count as not given, a
 * temperature that is as 0.
 * logprob[r] = log of the probability with which the token was drawn (0 for
 * temperature 0, -infinity with token -1).
 * Sums are whole numbers, in no order: w is rounded to units of 2^-44 of the
 * largest, so that a token with less than 2^-45 of it is never drawn, and the
 * answer is the definition's in 64 bits but where uniform times the sum is
 * within vocab * 2^-45 of a border between two tokens.  logprob is not rounded
 * to these units.
 * ------------------------------------------------------------------------- */
typedef struct amap_sample_args {
  int32_t rows;    /* 1 .. 65535 */
  int32_t vocab;   /* 1 .. 2^19 */
  int32_t dtype;   /* AMAP_BF16, AMAP_FP16 or AMAP_FP32 */
  int32_t by_row;  /* bits 0 .. 3: temperature, top_k, top_p, min_p are arrays of `rows` numbers, not one */
  const void *logits;
  int64_t row;     /* stride between rows */
  const float *uniform;
  const float *temperatures; /* with bit 0, else `temperature` counts */
  const int32_t *top_ks;
  const float *top_ps, *min_ps;
  float temperature;
  int32_t top_k;
  float top_p, min_p;
  int32_t *tokens;
  float *logprobs; /* may be NULL */
} amap_sample_args;
int amap_sample(const amap_sample_args *args /* host */, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* AMAP_SERVE_H_ */
