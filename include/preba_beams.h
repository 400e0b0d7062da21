/*
 * preba_beams.h — C ABI of a beam search over an encoder's states: attention of the decoder's rows to
 * the states of their request, the selection of the next beams over beams and vocabulary, and the
 * paged cache's part of it, block tables that follow the beams and copies of the open pages.
 *
 * n requests have `beams` rows each; row r * beams + b is beam b of request r, in every array here
 * and as a request of its own in the calls of preba_tokens.h.  One step of the search:
 *   preba_pages_plan, preba_rope_append, preba_pages_attend   (every row has one new token)
 *   preba_cross_attend    (per layer) the rows of a request see its encoder's states
 *   preba_beam_select     logits -> parents, tokens and scores of the next beams
 *   preba_beam_pages      parents -> block table of the next beams, pages released, open pages to copy
 *   preba_pages_copy      those pages, in all layers
 *
 * The conventions are those of preba_tokens.h: plain C, no exceptions, no allocation, no
 * synchronisation, 0 or a negative PREBA_ERR_*, every buffer the caller's, no state between calls, all
 * calls can be captured; strides are in elements; what lengths and tables hold is checked on the device where
 * it is used, the first fault found is stored in `status`; the kernels let the next one be set up early.
 */
#ifndef PREBA_BEAMS_H_
#define PREBA_BEAMS_H_

#include "preba_tokens.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PREBA_BEAMS_MAX 32u             /* beams of a request */
#define PREBA_BEAMS_MAX_WIDTH 64u       /* candidates chosen for a request */
#define PREBA_BEAMS_MAX_VOCAB (1u << 20)
#define PREBA_COPY_MAX_LAYERS 128u

/*
 * preba_cross_attend — attention of the decoder's rows to the states of an encoder, which lie packed
 * one request after the other and belong to all rows of theirs: request r owns rows cu_q[r] .. cu_q[r+1]-1 (its
 * beams' single tokens, or a whole prompt) and states cu_k[r] .. cu_k[r+1]-1.  Row i sees the first seen[i]
 * states of its request, all of them without `seen` (a row of a prompt with images sees those of the images before
 * it, a row of a stream what has arrived).  Per query head h, with the key head h / (heads_q / heads_kv):
 *   out = sum_k p_k v_k / sum_k p_k,   p_k = exp(scale q.k_k - m),   m = max_k scale q.k_k
 *   lse = m + ln sum_k p_k
 * A row that sees no state is 0, its lse -inf; so is one whose scores are all -inf.  A row with a score that is not a
 * number is not a number, nor is its lse.  Products and sums are fp32; p is rounded to the type of the states for the product
 * with v, as the matrix instructions take it, and out is rounded once.  States that no row of the request sees may
 * hold anything, infinities and NaN included; a state that is not finite and that some row sees may show
 * in other rows of its request.  Rows behind cu_q[n] are not written.  Results do not depend on timing.
 *   preba_cross_attend_query  bytes of workspace that a call with these sizes needs (host only);
 *                             the caller zeroes the workspace once, every call leaves its counters
 *                             zeroed again; calls that may overlap on the device need one each.
 * A request is skipped (its rows are not written) and PREBA_ERR_BAD_TABLE stored if its rows or states are out of range or
 * its rows more than max_q.  Requests whose states or rows overlap (only with others skipped between them can they) may
 * come to more work than n, tokens and states allow for: then PREBA_ERR_BAD_TABLE is stored and any rows may be left unwritten.
 * Every wait of the kernels has a limit.  If one runs out, PREBA_ERR_TIMEOUT is stored and the rows that the
 * call would have written hold anything; nothing else does, and the workspace is left as by any call.
 * Errors: PREBA_ERR_INVALID_ARG (NULL, sizes of 0, n above PREBA_PAGES_MAX_REQUESTS, tokens or states above
 * PREBA_PAGES_MAX_KEYS, a base that is not 16-byte aligned, a stride that is not a multiple of 8, heads_q not a multiple of
 * heads_kv, heads_q above 65535, more than 128 query heads on one key head, head_dim not a multiple of 8 in
 * 8 .. PREBA_PAGES_MAX_HEAD_DIM, another dtype than the two, a scale that is not positive and finite, a stride of 2^38 or more,
 * a stride of 0 on an axis of q, k or v that has more than one entry, so many states that
 * heads_kv * (2 * n + states / 128) passes 2e9, or so many rows that heads_kv * (n + tokens / (2 * g)) passes 2^31 - 1, where
 * g = 128 * heads_kv / heads_q rounded down), PREBA_ERR_BUFFER_TOO_SMALL (workspace), PREBA_ERR_CUDA.
 */
typedef struct {
  const void* q;              /* DEVICE, [tokens, heads_q, head_dim] */
  const void* k;              /* DEVICE, [states, heads_kv, head_dim] */
  const void* v;              /* DEVICE, likewise */
  const int32_t* cu_q;        /* DEVICE, n + 1 */
  const int32_t* cu_k;        /* DEVICE, n + 1 */
  const int32_t* seen;        /* DEVICE, tokens, or NULL */
  void* out;                  /* DEVICE, [tokens, heads_q, head_dim] */
  float* lse;                 /* DEVICE, [tokens, heads_q] contiguous, or NULL */
  void* workspace;            /* DEVICE, 16-byte aligned */
  uint64_t workspace_bytes;
  int32_t* status;            /* DEVICE word or NULL */
  uint64_t q_stride[2];       /* token, head */
  uint64_t out_stride[2];
  uint64_t k_stride[2];       /* state, head */
  uint64_t v_stride[2];
  uint32_t n;
  uint32_t tokens;
  uint32_t states;
  uint32_t max_q;             /* no request has more rows than this */
  uint32_t heads_q;
  uint32_t heads_kv;
  uint32_t head_dim;
  int32_t dtype;              /* PREBA_F16 or PREBA_BF16: q, k, v and out */
  float scale;
  uint32_t reserved;
} preba_cross_attend_t;
int preba_cross_attend_query(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv,
                             uint32_t head_dim, uint64_t* workspace_bytes);
int preba_cross_attend(const preba_cross_attend_t* req, void* stream);

/*
 * preba_beam_select — the best `width` continuations of every request over its beams and the vocabulary.
 * Row i = r * beams + b offers every token v that `allowed` leaves it, at
 *   value = scores[i] + x_v - ln sum_u exp x_u   (u over the allowed tokens),   rank = weights[i] * value,
 * or, where done[i] is not 0, its end token alone at value = scores[i].  Candidates are ordered by rank,
 * equal ranks by beam, then by logit, then by token (the lowest first), and the first `width` are
 * written in this order: the beam that is continued, the token, the value.  What is missing (rows that offer
 * nothing) has token and parent -1, value -inf and is not done.  Only finite ranks are offered: nothing by a row whose
 * score is -inf, and no token whose logit is -inf.  A row with an allowed logit that is NaN or +inf, a score that is, or
 * a weight that is not positive and finite offers nothing either, and PREBA_ERR_BAD_TABLE is stored.  Logits of tokens
 * that are not allowed, and of rows that are done or have the score -inf, may hold anything.
 * Exponentials and partial sums are fp32, sums of those, logarithms, values and ranks 64-bit; values are rounded
 * once.  Results do not depend on timing, and rows with equal logits have equal sums.
 *   preba_beam_select_query  bytes of workspace (host only); its contents mean nothing before and after a call;
 *                            calls that may overlap on the device need one each.
 * Outputs are distinct from inputs (scores_out == scores and done_out == done are refused).  Two kernel launches.
 * Errors: PREBA_ERR_INVALID_ARG (NULL, sizes of 0 or above the limits here, n * beams above
 * PREBA_PAGES_MAX_REQUESTS, a base that is not aligned to its elements, the workspace to 16 bytes, row_stride below vocab
 * or allowed_stride not 0 and below a row's words with more than one row, either of 2^38 or more, end_token below -1 or not below
 * vocab, or -1 where `done` is given, another dtype than the three),
 * PREBA_ERR_BUFFER_TOO_SMALL (workspace), PREBA_ERR_CUDA.
 */
typedef struct {
  const void* logits;        /* DEVICE, [n * beams, vocab] by row_stride */
  const float* scores;       /* DEVICE, n * beams: the beams' sums of log-probabilities */
  const uint8_t* done;       /* DEVICE, n * beams, or NULL: beams that have ended */
  const uint32_t* allowed;   /* DEVICE or NULL: a row of (vocab + 31) / 32 words for each beam; token v may
                                follow if bit v % 32 of word v / 32 is set */
  const float* weights;      /* DEVICE, n * beams, or NULL (1): what values are multiplied with for the order */
  int32_t* tokens;           /* DEVICE, [n, width], written */
  int32_t* parents;          /* DEVICE, [n, width], written: beams of the same request */
  float* scores_out;         /* DEVICE, [n, width], written */
  uint8_t* done_out;         /* DEVICE, [n, width], written, or NULL: the parent is done or the token is end_token */
  void* workspace;           /* DEVICE, 16-byte aligned */
  uint64_t workspace_bytes;
  int32_t* status;           /* DEVICE word or NULL */
  uint64_t row_stride;       /* of logits */
  uint64_t allowed_stride;   /* words from row to row; 0: one row for all */
  uint32_t n;
  uint32_t beams;
  uint32_t width;
  uint32_t vocab;
  int32_t end_token;         /* or -1 */
  int32_t dtype;             /* of logits: PREBA_F32, PREBA_F16 or PREBA_BF16 */
} preba_beam_select_t;
int preba_beam_select_query(uint32_t n, uint32_t beams, uint32_t width, uint32_t vocab, int32_t dtype,
                            uint64_t* workspace_bytes);
int preba_beam_select(const preba_beam_select_t* req, void* stream);

/*
 * preba_beam_pages — the block table of the next beams.  New row i of request r takes over the pages and the
 * length of row parents[i] of r (negative: the row is empty, its length 0).  Full pages are shared: beams of one
 * request may hold the same page at the same place of their rows, and only there.  The last page of a
 * length that does not fill it is open, the next token is written there, so it belongs to one beam (a search that begins with
 * one prompt begins with one beam that has it): the first child of a beam keeps it,
 * every other child gets a page of its own, and copies[i] = {from, to, tokens, 0} says what preba_pages_copy has to
 * bring there (all zeros where nothing has).  A page that no new row holds is released, unless it lies at one of the first
 * kept[r] places of its row (pages that the request shares with others).
 * Released pages, in the order of requests, places and beams, are given to the copies in the order of their
 * rows.  Copies beyond them take the k-th page from the top of the stack, free_pages[*free_count - 1 - k];
 * pages beyond the copies are put on top of it, at free_pages[*free_count + k].  *free_left is the count afterwards.
 * The call writes nothing that it reads: run twice on the same inputs it writes the same again.
 * A request is refused if a length is negative or longer than its row of the table, or a parent is not below `beams`
 * (PREBA_ERR_BAD_TABLE), or if the free pages, what the requests before it that were not refused left of them, and its
 * own released pages do not suffice (PREBA_ERR_BUFFER_TOO_SMALL): its rows of table_out are as in `table`, their lengths
 * 0, nothing is copied or released; a caller that takes lengths_out over leaves out the refused requests' zeros.
 * Every request is refused if *free_count is negative or above free_capacity (PREBA_ERR_BAD_TABLE); the stack stays as it is, and
 * *free_left is 0.
 * A released page that is not a page number is dropped, as is one for which the stack has no room (PREBA_ERR_BAD_TABLE);
 * a page from the stack that is not one is not copied to (the same).  Entries of table_out behind the last page
 * of a row are left as they were.
 *   preba_beam_pages_query  bytes of workspace (host only), as for preba_beam_select.
 * Errors: PREBA_ERR_INVALID_ARG (NULL, n, beams or table_width 0, n * beams above PREBA_PAGES_MAX_REQUESTS, beams above
 * PREBA_BEAMS_MAX, page_size not a power of two in 8 .. PREBA_PAGES_MAX_PAGE, pages * page_size above 2^31 - 1, a stride
 * below table_width, table_width * page_size above 2^31 - 1, n * beams * table_width above 2^32 - 1,
 * table_out == table, lengths_out == lengths, free_left == free_count, free_capacity above 2^31 - 1, copies or the workspace not
 * 16-byte aligned), PREBA_ERR_BUFFER_TOO_SMALL (workspace), PREBA_ERR_CUDA.
 */
typedef struct {
  const int32_t* parents;     /* DEVICE, n * beams */
  const int32_t* lengths;     /* DEVICE, n * beams: tokens in the cache */
  const int32_t* kept;        /* DEVICE, n, or NULL (0) */
  const int32_t* table;       /* DEVICE, n * beams rows of table_width page numbers */
  int32_t* table_out;         /* DEVICE, likewise, written */
  int32_t* lengths_out;       /* DEVICE, n * beams, written */
  int32_t* copies;            /* DEVICE, [n * beams, 4], 16-byte aligned, written */
  int32_t* free_pages;        /* DEVICE, free_capacity page numbers: read below *free_count, written from there */
  const int32_t* free_count;  /* DEVICE word: pages on the stack */
  int32_t* free_left;         /* DEVICE word, written */
  int32_t* status;            /* DEVICE word or NULL */
  void* workspace;            /* DEVICE, 16-byte aligned */
  uint64_t workspace_bytes;
  uint64_t table_stride;      /* from row to row, of both tables */
  uint64_t table_out_stride;
  uint32_t table_width;
  uint32_t free_capacity;
  uint32_t n;
  uint32_t beams;
  uint32_t page_size;
  uint32_t pages;             /* page numbers are below this */
} preba_beam_pages_t;
int preba_beam_pages_query(uint32_t n, uint32_t beams, uint32_t table_width, uint64_t* workspace_bytes);
int preba_beam_pages(const preba_beam_pages_t* req, void* stream);

/*
 * preba_pages_copy — copies[i] = {from, to, tokens, 0}: the first `tokens` slots of page `from` go to page `to`, keys
 * and values, in every layer; tokens == 0: nothing.  No page is written twice, and none that is written is read (the
 * copies of preba_beam_pages are so).  An entry whose pages or tokens are out of range is left out (status
 * PREBA_ERR_BAD_TABLE).  One kernel launch for all layers.
 * Errors: PREBA_ERR_INVALID_ARG (NULL, layers of 0 or above PREBA_COPY_MAX_LAYERS, rows of 0 or above
 * PREBA_PAGES_MAX_REQUESTS, a cache or copies that is not 16-byte aligned, strides that are not multiples of 8
 * or 2^38 or more, head_dim and page_size as for preba_pages_attend, pages * page_size above 2^31 - 1, another dtype than the two,
 * heads_kv of 0 or above 65535), PREBA_ERR_CUDA.
 */
typedef struct {
  const int32_t* copies;      /* DEVICE, [rows, 4] */
  void* const* k_caches;      /* HOST, `layers` DEVICE pointers, read during the call */
  void* const* v_caches;      /* HOST, likewise */
  int32_t* status;            /* DEVICE word or NULL */
  uint64_t cache_stride[3];   /* page, slot in page, head; the same for all caches */
  uint32_t rows;
  uint32_t layers;
  uint32_t heads_kv;
  uint32_t head_dim;
  uint32_t pages;
  uint32_t page_size;
  int32_t dtype;              /* PREBA_F16 or PREBA_BF16 */
  uint32_t reserved;
} preba_pages_copy_t;
int preba_pages_copy(const preba_pages_copy_t* req, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PREBA_BEAMS_H_ */
