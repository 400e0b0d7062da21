/*
 * preba_tokens.h — C ABI of the serving step behind the preprocessing front-end, for models that
 * answer in tokens: the pages of a paged key/value cache, three-axis rotary positions of text,
 * images and video, the rotation of queries and keys with the write into the cache, and the
 * attention of the new tokens over the cache.
 *
 * One step of a batch of requests runs the four device calls in this order on one stream:
 *   preba_pages_plan      lengths -> block table, row starts, slots, plain positions
 *   preba_rope_positions  spans of the prompts -> positions on three axes
 *   preba_rope_append     (per layer) rotate queries and keys, write keys and values to the cache
 *   preba_pages_attend    (per layer) attention of the step's tokens over the cache
 * A step may mix whole prompts, chunks of prompts and single tokens.  The token axis is ragged and
 * packed: request r owns rows cu_q[r] .. cu_q[r+1]-1 of every per-token array.
 *
 * The conventions are those of preba.h: plain C, no exceptions, no allocation, no synchronisation,
 * 0 or a negative PREBA_ERR_*, every buffer the caller's, no state between calls.  All calls can be
 * captured in a CUDA graph: what they read of lengths and tables is read on the device.  Strides
 * are in elements.  Lengths and tables are checked on the device where they are used; an entry that
 * is out of range is never followed, the first such PREBA_ERR_* is stored in `status`.
 *
 * The kernels of these calls let the next kernel on the stream be set up while they run.  That changes
 * nothing for an ordinary launch, but a launch that asks not to wait (PREBA_OVERLAP_PREVIOUS,
 * PREBA_AUDIO_OVERLAP_PREVIOUS) may run beside the call directly before it, and must share no buffer
 * with that call.
 */
#ifndef PREBA_TOKENS_H_
#define PREBA_TOKENS_H_

#include "preba.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PREBA_PAGES_MAX_REQUESTS 16384u /* requests in one call */
#define PREBA_PAGES_MAX_PAGE 256u       /* page sizes: powers of two from 8 to this */
#define PREBA_PAGES_MAX_HEAD_DIM 128u   /* head sizes: multiples of 8 up to this */
#define PREBA_PAGES_MAX_KEYS 0x7ffff000u /* tokens of one request, cached and fresh (2^31 - 4096) */
#define PREBA_ROPE_MAX_POSITION (1 << 24)

/*
 * preba_pages_plan — the block table and the slot of every new token, from the requests' lengths.
 * A request with `cached` tokens holds ceil(cached/page_size) pages; the call gives it the pages
 * that `fresh` more tokens need, from the top of the stack of free pages (the k-th new page of the
 * step, in request order, is free_pages[*free_count - 1 - k]), and appends them to its row of the
 * table.  Slot = page * page_size + position mod page_size.  The call reads *free_count and writes
 * *free_left, and nothing that it reads: run twice on the same inputs it writes the same again.
 * A request is refused if its lengths are negative or add up to more than PREBA_PAGES_MAX_KEYS, if its
 * row of the table is too short, if its rows end beyond `tokens` (status PREBA_ERR_BAD_TABLE) or if the
 * free pages do not suffice for it and those before it (PREBA_ERR_BUFFER_TOO_SMALL): it gets no page,
 * its slots are -1 and its kv_len is 0.  What it held it still holds: a caller that takes kv_len over as the
 * next step's `cached` leaves out the zeros, and may ask for the same tokens again.
 * Tokens behind the last request's get slot -1 and position 0, so that a step can be padded.
 * All buffers are distinct; one kernel launch.
 * Errors: PREBA_ERR_INVALID_ARG (NULL, n == 0 or above PREBA_PAGES_MAX_REQUESTS, page_size not a power
 * of two in 8 .. PREBA_PAGES_MAX_PAGE, pages * page_size above 2^31 - 1), PREBA_ERR_CUDA.
 */
typedef struct {
  const int32_t* cached;      /* DEVICE, n: tokens in the cache before the step */
  const int32_t* fresh;       /* DEVICE, n: tokens of the step (0: the request sits it out) */
  int32_t* block_table;       /* DEVICE, n rows of table_width page numbers, in and out */
  const int32_t* free_pages;  /* DEVICE, free_capacity page numbers, the stack of free pages */
  const int32_t* free_count;  /* DEVICE word: pages on the stack */
  int32_t* cu_q;              /* DEVICE, n + 1, written: first row of each request, rows in all */
  int32_t* kv_len;            /* DEVICE, n, written: cached + fresh, or 0 for a refused request */
  int32_t* slots;             /* DEVICE, tokens, written */
  int32_t* positions;         /* DEVICE, tokens, written, or NULL: place within the request */
  int32_t* free_left;         /* DEVICE word, written: pages left on the stack */
  int32_t* status;            /* DEVICE word or NULL, as preba_batch_t.status */
  uint64_t table_stride;      /* from row to row of the table */
  uint32_t table_width;
  uint32_t free_capacity;
  uint32_t n;
  uint32_t tokens;            /* capacity of slots and positions */
  uint32_t page_size;
  uint32_t pages;             /* pages of the cache: page numbers are below this */
} preba_pages_plan_t;
int preba_pages_plan(const preba_pages_plan_t* plan, void* stream);

/*
 * preba_rope_positions — the positions of the step's tokens on three axes (time, height, width).
 * A request's prompt is a sequence of spans {t, h, w, step}.  h == 0: t tokens of text, which have
 * the same position on all axes and count on from the span before.  h > 0: the t*h*w patches of an
 * image (t == 1) or a video, in that order; patch (a, y, x) of a span that begins at position B has
 * the positions (B + a*step, B + y, B + x), and the next span begins at
 * B + max((t-1)*step + 1, h, w).  A request's tokens past its spans are text.  The call writes the
 * positions of tokens cached[r] .. cached[r] + cu_q[r+1] - cu_q[r] - 1 of every request, so that it
 * serves whole prompts, chunks that begin inside an image, and single tokens alike.
 * A span with a negative member, with w == 0 or step == 0 where h > 0, or whose tokens or step exceed 2^24
 * counts as empty (status PREBA_ERR_BAD_TABLE); a request whose rows or spans are out of range is skipped (the
 * same).  Positions are formed modulo 2^32: steps and extents that add up to more than 2^31 - 1 wrap.
 * Rows behind the last request's are written as 0.  One kernel launch.
 * Errors: PREBA_ERR_INVALID_ARG, PREBA_ERR_CUDA.
 */
typedef struct {
  const int32_t* spans;       /* DEVICE, n_spans x 4, 16-byte aligned (NULL if n_spans == 0) */
  const int32_t* span_begin;  /* DEVICE, n + 1: request r owns spans span_begin[r] .. [r+1]-1 */
  const int32_t* cached;      /* DEVICE, n: the request's tokens before the step */
  const int32_t* cu_q;        /* DEVICE, n + 1: first row of each request (preba_pages_plan) */
  int32_t* positions;         /* DEVICE, three rows of `tokens`, written */
  int32_t* status;            /* DEVICE word or NULL */
  uint64_t axis_stride;       /* from axis to axis of positions, >= tokens */
  uint32_t n_spans;
  uint32_t n;
  uint32_t tokens;
  uint32_t reserved;
} preba_rope_positions_t;
int preba_rope_positions(const preba_rope_positions_t* req, void* stream);

/* preba_rope_append_t.flags */
#define PREBA_ROPE_INTERLEAVED 1u  /* pair j is elements 2j, 2j+1; else j and j + rotary_dim/2 */
#define PREBA_ROPE_AXES_IN_TURN 2u /* axis of pair j: a = j mod 3 if a > 0 and j/3 < sections[a],
                                      else 0; without it the first sections[0] pairs turn with time,
                                      the next sections[1] with height, the last with width */

/*
 * preba_rope_append — rotates the step's queries and keys by their positions and writes keys and
 * values into the paged cache.  Pair j = (x, y) of a head of token t becomes
 * (x cos a - y sin a, y cos a + x sin a), a = positions[axis(j)][t] * inv_freq[j]; elements from
 * rotary_dim on are copied.  The angle is reduced in 64 bits, so it is as exact at position 2^24 as
 * at 1; the rotation is fp32, rounded once.  Keys and values of token t go to slots[t]; a negative
 * slot leaves them out (the queries are rotated all the same), one beyond the cache too, with status
 * PREBA_ERR_BAD_TABLE.  q_out may be q itself.  Positions beyond +-PREBA_ROPE_MAX_POSITION lose
 * exactness.  One kernel launch.
 * Errors: PREBA_ERR_INVALID_ARG (also: a base that is not 16-byte aligned, a stride that is not a
 * multiple of 8; head_dim not a multiple of 8 in 8 .. PREBA_PAGES_MAX_HEAD_DIM; rotary_dim above it or not
 * a multiple of 16; sections that do not add up to rotary_dim/2 or, in turn, find no room),
 * PREBA_ERR_CUDA.
 */
typedef struct {
  const void* q;              /* DEVICE, [tokens, heads_q, head_dim]; NULL if heads_q == 0 */
  const void* k;              /* DEVICE, [tokens, heads_kv, head_dim]; NULL if heads_kv == 0 */
  const void* v;              /* DEVICE, [tokens, heads_kv, head_dim] */
  void* q_out;                /* DEVICE, [tokens, heads_q, head_dim] */
  void* k_cache;              /* DEVICE, [pages, page_size, heads_kv, head_dim] by strides */
  void* v_cache;              /* DEVICE, likewise, the same strides */
  const int32_t* positions;   /* DEVICE, three rows of `tokens` */
  const int32_t* slots;       /* DEVICE, tokens */
  const double* inv_freq;     /* DEVICE, rotary_dim/2 angular frequencies per position */
  int32_t* status;            /* DEVICE word or NULL */
  uint64_t q_stride[2];       /* token, head */
  uint64_t k_stride[2];
  uint64_t v_stride[2];
  uint64_t q_out_stride[2];
  uint64_t cache_stride[3];   /* page, slot in page, head */
  uint64_t axis_stride;       /* from axis to axis of positions; 0: one row for all axes */
  uint32_t sections[3];       /* pairs that turn with time, height, width */
  uint32_t tokens;
  uint32_t heads_q;
  uint32_t heads_kv;
  uint32_t head_dim;
  uint32_t rotary_dim;        /* <= head_dim */
  uint32_t pages;
  uint32_t page_size;
  int32_t dtype;              /* PREBA_F16 or PREBA_BF16 */
  uint32_t flags;
} preba_rope_append_t;
int preba_rope_append(const preba_rope_append_t* req, void* stream);

/* preba_pages_attend_t.flags */
#define PREBA_ATTEND_CAUSAL 1u /* a token sees the keys up to its own place only */

/*
 * preba_pages_attend — attention of the step's tokens over the paged cache, which holds their own
 * keys and values already.  Row i of request r stands at place c = kv_len[r] - q_len + i of the
 * request's keys (q_len = cu_q[r+1] - cu_q[r]) and sees key k if 0 <= k < kv_len[r], and k <= c
 * with PREBA_ATTEND_CAUSAL, and k > c - window where window > 0.  Per query head h, with the key
 * head h / (heads_q / heads_kv):
 *   out = sum_k p_k v_k / sum_k p_k,   p_k = exp(scale q.k_k - m),   m = max_k scale q.k_k
 *   lse = m + ln sum_k p_k
 * A row that sees no key is 0, its lse -inf (kv_len may be 0, or below q_len); so is one whose scores
 * are all -inf.  A row with a score that is not a number is not a number, nor is its lse.  Products and sums
 * are fp32; p is rounded to the cache's type for the product with v, as the matrix instructions
 * take it, and out is rounded once.  Cache slots that no row of the request sees may hold anything,
 * infinities and NaN included, and table entries whose pages no row sees are not followed; a key or
 * value that is not finite and that some row sees may show in other rows of its request.  Rows behind
 * cu_q[n] are not written.  Results do not depend on timing: the same call gives the same bits.
 *   preba_pages_attend_query  bytes of workspace that a call with these sizes needs (host only);
 *                             the caller zeroes the workspace once, every call leaves its counters
 *                             zeroed again; calls that may overlap on the device need one each.
 * A request is skipped (its rows are not written) and PREBA_ERR_BAD_TABLE stored if its rows are out of range or
 * more than max_q, or if kv_len is negative, beyond its row of the table or above PREBA_PAGES_MAX_KEYS; a
 * seen page number that is out of range reads as zeros and stores PREBA_ERR_BAD_TABLE.
 * Every wait of the kernels has a limit.  If one runs out, PREBA_ERR_TIMEOUT is stored and the rows that the
 * call would have written hold anything; nothing else does, and the workspace is left as by any call.
 * Errors: PREBA_ERR_INVALID_ARG (also: a base that is not 16-byte aligned, a stride that is not a
 * multiple of 8, heads_q not a multiple of heads_kv, more than 128 query heads on one key head,
 * page_size as for preba_pages_plan, tokens above PREBA_PAGES_MAX_KEYS, head_dim not a multiple of 8 in 8 .. PREBA_PAGES_MAX_HEAD_DIM, a
 * stride of 0 on an axis of q or a cache that has more than one entry, tables so wide that
 * n * heads_kv * (table_width * page_size / 64 + 2) passes 2e9, or, with more than 16 rows on a key head
 * (max_q * heads_q / heads_kv), so many rows that heads_kv * (n + tokens / (2 * g)) passes 2^31 - 1, where
 * g = 128 * heads_kv / heads_q rounded down), PREBA_ERR_BUFFER_TOO_SMALL (workspace), PREBA_ERR_CUDA.
 */
typedef struct {
  const void* q;              /* DEVICE, [tokens, heads_q, head_dim] */
  const void* k_cache;        /* DEVICE, [pages, page_size, heads_kv, head_dim] by strides */
  const void* v_cache;        /* DEVICE, likewise */
  const int32_t* block_table; /* DEVICE, n rows of table_width page numbers */
  const int32_t* cu_q;        /* DEVICE, n + 1 */
  const int32_t* kv_len;      /* DEVICE, n: keys of each request, the step's own included */
  void* out;                  /* DEVICE, [tokens, heads_q, head_dim] */
  float* lse;                 /* DEVICE, [tokens, heads_q] contiguous, or NULL */
  void* workspace;            /* DEVICE, 16-byte aligned */
  uint64_t workspace_bytes;
  int32_t* status;            /* DEVICE word or NULL */
  uint64_t q_stride[2];       /* token, head */
  uint64_t out_stride[2];
  uint64_t k_stride[3];       /* page, slot in page, head */
  uint64_t v_stride[3];
  uint64_t table_stride;
  uint32_t table_width;
  uint32_t n;
  uint32_t tokens;
  uint32_t max_q;             /* no request has more rows than this */
  uint32_t heads_q;
  uint32_t heads_kv;
  uint32_t head_dim;
  uint32_t pages;
  uint32_t page_size;
  uint32_t window;            /* 0: no limit */
  int32_t dtype;              /* PREBA_F16 or PREBA_BF16: q, caches and out */
  uint32_t flags;
  float scale;
  uint32_t reserved;
} preba_pages_attend_t;
int preba_pages_attend_query(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv,
                             uint32_t head_dim, uint64_t* workspace_bytes);
int preba_pages_attend(const preba_pages_attend_t* req, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PREBA_TOKENS_H_ */
