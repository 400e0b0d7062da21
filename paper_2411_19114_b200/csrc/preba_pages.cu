// Pages, positions and rotation of a serving step (preba_tokens.h): preba_pages_plan,
// preba_rope_positions, preba_rope_append.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "preba_internal.h"
#include "preba_tokens.h"

namespace preba {
namespace {

constexpr uint32_t kFull = 0xffffffffu;

__device__ __forceinline__ void report(int32_t* status, int32_t code) {
  if (status) atomicCAS(status, 0, code);
}

// ---- preba_pages_plan -----------------------------------------------------------------------------
//
// Two sums run over the requests, of rows and of new pages; a token then needs its request's two
// sums only.  A step has hundreds of requests and up to hundreds of thousands of tokens, so every CTA
// adds the lengths up for itself (they come from L2 after the first) instead of waiting for
// another to do it: one launch, no flag between CTAs.  Bound by latency: two loads, a sum over the block, a
// search, two loads, a store.  4.0 us a call for 64 single tokens, 6.0 us for 145 K tokens of 1500 requests
// (1.2 MB) in a sequence of calls.

constexpr int kPlanThreads = 512;
constexpr uint32_t kPlanTokensPerCta = 4 * kPlanThreads;

// Exclusive sums over the block's threads of two numbers at once; the totals come back too.
struct sums_t {
  int64_t rows, pages;
};
__device__ __forceinline__ sums_t block_exclusive(sums_t v, sums_t* warp_sums, sums_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  sums_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t rows = __shfl_up_sync(kFull, incl.rows, o), pages = __shfl_up_sync(kFull, incl.pages, o);
    if (lane >= o) incl.rows += rows, incl.pages += pages;
  }
  __syncthreads();  // what an earlier call left has been read
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  static_assert(kPlanThreads / 32 <= 32, "one lane per warp");
  sums_t all = lane < kPlanThreads / 32 ? warp_sums[lane] : sums_t{0, 0};
  sums_t before = lane < warp ? all : sums_t{0, 0};
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    all.rows += __shfl_xor_sync(kFull, all.rows, o), all.pages += __shfl_xor_sync(kFull, all.pages, o);
    before.rows += __shfl_xor_sync(kFull, before.rows, o), before.pages += __shfl_xor_sync(kFull, before.pages, o);
  }
  total = all;
  return {before.rows + incl.rows - v.rows, before.pages + incl.pages - v.pages};
}

// The last i in [0, n) with a[i] <= x, for ascending a with a[0] <= x.
__device__ __forceinline__ uint32_t last_not_above(const int32_t* a, uint32_t n, int32_t x) {
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (a[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads)
plan_kernel(const preba_pages_plan_t p, const uint32_t page_shift) {
  extern __shared__ int32_t plan_smem[];
  chained_begin();
  int32_t* cu = plan_smem;               // n + 1: first row of each request
  int32_t* first = plan_smem + p.n + 1;  // n: new pages before the request's, or -1: refused
  __shared__ sums_t warp_sums[kPlanThreads / 32];
  const bool writer = blockIdx.x == 0;   // one CTA writes what belongs to requests
  const uint32_t per = (p.n + kPlanThreads - 1) / kPlanThreads;
  const uint32_t r0 = min(threadIdx.x * per, p.n), r1 = min(r0 + per, p.n);
  const int64_t page_mask = (1ll << page_shift) - 1;
  int32_t count = *p.free_count;
  if (count < 0 || static_cast<uint32_t>(count) > p.free_capacity) {
    if (writer && threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
    count = 0;
  }

  // new pages of a request whose last row is `end`; -1: its lengths, its row of the table or its rows are
  // out of range
  auto need_of = [&](int64_t cached, int64_t fresh, int64_t end) -> int64_t {
    const int64_t pages = (cached + fresh + page_mask) >> page_shift;
    if (cached < 0 || fresh < 0 || end > p.tokens || pages > p.table_width || cached + fresh > PREBA_PAGES_MAX_KEYS)
      return -1;  // places within a request and numbers of keys are 32-bit, here and in the calls that follow
    return pages - ((cached + page_mask) >> page_shift);
  };
  sums_t mine{0, 0}, total;
  for (uint32_t r = r0; r < r1; ++r) {
    const int64_t c = p.cached[r], f = p.fresh[r];
    mine.rows += max(f, static_cast<int64_t>(0));
    mine.pages += max(need_of(c, f, 0), static_cast<int64_t>(0));
  }
  sums_t at = block_exclusive(mine, warp_sums, total);
  if (total.rows > p.tokens) {
    // some requests' rows do not fit: they take no pages, which only shows now
    mine.pages = 0;
    int64_t end = at.rows;
    for (uint32_t r = r0; r < r1; ++r) {
      const int64_t c = p.cached[r], f = p.fresh[r];
      end += max(f, static_cast<int64_t>(0));
      mine.pages += max(need_of(c, f, end), static_cast<int64_t>(0));
    }
    at = block_exclusive(mine, warp_sums, total);
  }
  if (threadIdx.x == 0) cu[p.n] = static_cast<int32_t>(min(total.rows, static_cast<int64_t>(p.tokens)));
  int64_t left = count;  // what this thread's last served request leaves
  int64_t end = at.rows, taken = at.pages;
  for (uint32_t r = r0; r < r1; ++r) {
    const int64_t c = p.cached[r], f = p.fresh[r];
    cu[r] = static_cast<int32_t>(min(end, static_cast<int64_t>(p.tokens)));
    end += max(f, static_cast<int64_t>(0));
    const int64_t k = need_of(c, f, end);
    taken += max(k, static_cast<int64_t>(0));
    // sums never shrink: once the stack is short, every later request that needs a page is refused
    const bool served = k == 0 || (k > 0 && taken <= count);
    first[r] = served ? static_cast<int32_t>(taken - k) : -1;
    if (k > 0 && served) left = count - taken;
    if (writer) {
      p.cu_q[r] = cu[r];
      p.kv_len[r] = served ? static_cast<int32_t>(c + f) : 0;
      if (!served) report(p.status, k < 0 ? PREBA_ERR_BAD_TABLE : PREBA_ERR_BUFFER_TOO_SMALL);
    }
  }
  if (writer) {
    if (threadIdx.x == 0) p.cu_q[p.n] = cu[p.n];
    // the smallest `left` is that of the last request that was given a page
    __shared__ int32_t least[kPlanThreads / 32];
    const int32_t of_warp = __reduce_min_sync(kFull, static_cast<int32_t>(left));
    if ((threadIdx.x & 31) == 0) least[threadIdx.x >> 5] = of_warp;
    __syncthreads();
    if (threadIdx.x < 32) {
      const int32_t v = __reduce_min_sync(kFull, threadIdx.x < kPlanThreads / 32 ? least[threadIdx.x] : count);
      if (threadIdx.x == 0) *p.free_left = v;
    }
  }
  __syncthreads();

  // four tokens in a row per thread: one search, one vector store
  const uint32_t t0 = blockIdx.x * kPlanTokensPerCta + 4 * threadIdx.x;
  if (t0 >= p.tokens) return;
  const uint32_t live = cu[p.n];
  int32_t slot[4], pos[4];
  uint32_t r = t0 < live ? last_not_above(cu, p.n, static_cast<int32_t>(t0)) : p.n;
  int32_t cached = 0, begin = 0, end_row = 0, base = 0, held = 0;
  bool loaded = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t t = t0 + i;
    slot[i] = -1;
    pos[i] = 0;
    if (t >= live) continue;
    if (!loaded || t >= static_cast<uint32_t>(end_row)) {
      while (static_cast<uint32_t>(cu[r + 1]) <= t) ++r;  // ends: t < cu[n]
      cached = p.cached[r];
      begin = cu[r];
      end_row = cu[r + 1];
      base = first[r];
      held = static_cast<int32_t>((cached + page_mask) >> page_shift);
      loaded = true;
    }
    if (base < 0) continue;  // refused
    const int32_t at_pos = cached + static_cast<int32_t>(t) - begin;
    const int32_t col = at_pos >> page_shift;
    int32_t* entry = p.block_table + static_cast<uint64_t>(r) * p.table_stride + col;
    int32_t page;
    if (col < held) {
      page = *entry;
    } else {
      const int32_t k = count - 1 - (base + col - held);
      if (!PREBA_IN_RANGE(p.status, k >= 0 && static_cast<uint32_t>(k) < p.free_capacity)) continue;
      page = p.free_pages[k];
      // the page's first slot belongs to a token of the step: that token enters the page
      if ((at_pos & page_mask) == 0) *entry = page;
    }
    pos[i] = at_pos;
    if (page < 0 || static_cast<uint32_t>(page) >= p.pages) {
      report(p.status, PREBA_ERR_BAD_TABLE);
      continue;
    }
    slot[i] = (page << page_shift) + static_cast<int32_t>(at_pos & page_mask);
  }
  auto put = [&](int32_t* to, const int32_t (&v)[4]) {
    if (t0 + 4 <= p.tokens && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
      *reinterpret_cast<int4*>(to + t0) = make_int4(v[0], v[1], v[2], v[3]);
    } else {
      for (int i = 0; i < 4; ++i)
        if (t0 + i < p.tokens) to[t0 + i] = v[i];
    }
  };
  put(p.slots, slot);
  if (p.positions) put(p.positions, pos);
}

// ---- preba_rope_positions -------------------------------------------------------------------------
//
// Requests are independent, so no sum crosses them: a warp takes a run of consecutive rows, adds up
// the spans of the requests it meets 32 at a time, and writes the rows of every span that lie in
// its run.  No shared memory, no limit on spans or requests.  Bound by latency (the search, the lengths, the
// spans, the store): 4.1 us a call for 76 K rows of prompts with images, 3.1 us for 256 single tokens.

constexpr int kPosThreads = 128;
constexpr uint32_t kPosMaxTokens = 1u << 24;  // of one span

// The last i in [0, n) with a[i] <= x, or 0; the whole warp probes 32 places at a time.
__device__ __forceinline__ uint32_t warp_last_not_above(const int32_t* a, uint32_t n, int64_t x) {
  const uint32_t lane = threadIdx.x & 31;
  uint32_t lo = 0, len = n;
  while (len > 1) {
    const uint32_t step = (len + 31) / 32;
    const uint32_t i = lo + lane * step;
    const bool below = lane * step < len && a[i] <= x;
    const uint32_t hits = __popc(__ballot_sync(kFull, below));
    if (hits == 0) return 0;
    lo += (hits - 1) * step;
    len = min(step, n - lo);
  }
  return lo;
}

struct span_t {
  int32_t t, h, w, step;
  int64_t tokens, extent;  // how many tokens, how many positions
};

__device__ __forceinline__ span_t load_span(const int32_t* spans, uint32_t i, int32_t* status) {
  const int4 v = reinterpret_cast<const int4*>(spans)[i];
  span_t s{v.x, v.y, v.z, v.w, 0, 0};
  const bool text = s.h == 0;
  bool ok = s.t >= 0 && s.h >= 0 && s.w >= 0 && s.step >= 0;
  if (ok && !text) ok = s.w > 0 && s.step > 0;
  if (ok && !text) {
    const int64_t hw = static_cast<int64_t>(s.h) * s.w;  // below 2^62
    ok = hw <= kPosMaxTokens && hw * s.t <= kPosMaxTokens && s.step <= (1 << 24);
    if (ok && s.t > 0) {
      s.tokens = hw * s.t;
      s.extent = max(static_cast<int64_t>(s.t - 1) * s.step + 1,
                     static_cast<int64_t>(max(s.h, s.w)));
    }
  } else if (ok) {
    ok = static_cast<uint32_t>(s.t) <= kPosMaxTokens;
    if (ok) s.tokens = s.extent = s.t;
  }
  if (!ok) report(status, PREBA_ERR_BAD_TABLE);
  return s;
}

__global__ void __launch_bounds__(kPosThreads)
positions_kernel(const preba_rope_positions_t p, const uint32_t run) {
  chained_begin();
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t warp = (static_cast<uint64_t>(blockIdx.x) * kPosThreads + threadIdx.x) >> 5;
  const uint64_t first = warp * run;
  if (first >= p.tokens) return;
  const uint32_t t0 = static_cast<uint32_t>(first);
  const uint32_t t1 = static_cast<uint32_t>(min(first + run, static_cast<uint64_t>(p.tokens)));
  int32_t* out = p.positions;
  auto put = [&](uint32_t t, int64_t a, int64_t b, int64_t c) {
    out[t] = static_cast<int32_t>(a);
    out[p.axis_stride + t] = static_cast<int32_t>(b);
    out[2 * p.axis_stride + t] = static_cast<int32_t>(c);
  };
  uint32_t r = warp_last_not_above(p.cu_q, p.n, t0);
  uint32_t done = t0;  // rows below this are written
  while (done < t1 && r < p.n) {
    const int64_t begin = p.cu_q[r], end = p.cu_q[r + 1];
    if (begin < 0 || end < begin || end > p.tokens) {
      if (lane == 0) report(p.status, PREBA_ERR_BAD_TABLE);
      ++r;
      continue;
    }
    const int64_t row0 = max(begin, static_cast<int64_t>(done));
    const int64_t row1 = min(end, static_cast<int64_t>(t1));
    if (row0 >= row1) {
      if (begin >= t1) break;
      ++r;
      continue;
    }
    // rows between two requests (their starts need not meet) belong to nobody
    for (uint32_t t = done + lane; t < row0; t += 32) put(t, 0, 0, 0);
    const int64_t cached = p.cached[r];
    int64_t s0 = p.span_begin[r], s1 = p.span_begin[r + 1];
    done = static_cast<uint32_t>(row1);
    if (s0 < 0 || s1 < s0 || s1 > p.n_spans || cached < 0) {
      if (lane == 0) report(p.status, PREBA_ERR_BAD_TABLE);
      for (uint32_t t = static_cast<uint32_t>(row0) + lane; t < row1; t += 32) put(t, 0, 0, 0);
      ++r;
      continue;
    }
    // the rows as token numbers of the request
    const int64_t i0 = cached + row0 - begin, i1 = cached + row1 - begin;
    int64_t at = 0, place = 0;  // tokens and positions before the next 32 spans
    for (; s0 < s1 && at < i1; s0 += 32) {
      span_t s{0, 0, 0, 0, 0, 0};
      if (s0 + lane < s1) s = load_span(p.spans, static_cast<uint32_t>(s0) + lane, p.status);
      int64_t tok = s.tokens, ext = s.extent;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t a = __shfl_up_sync(kFull, tok, o), b = __shfl_up_sync(kFull, ext, o);
        if (lane >= static_cast<uint32_t>(o)) tok += a, ext += b;
      }
      const int64_t my_at = at + tok - s.tokens, my_place = place + ext - s.extent;
      uint32_t hit = __ballot_sync(kFull, s.tokens > 0 && my_at < i1 && my_at + s.tokens > i0);
      while (hit) {
        const int src = __ffs(hit) - 1;
        hit &= hit - 1;
        const int64_t b_at = __shfl_sync(kFull, my_at, src);
        const int64_t base = __shfl_sync(kFull, my_place, src);
        const int64_t n_tok = __shfl_sync(kFull, s.tokens, src);
        const int32_t h = __shfl_sync(kFull, s.h, src), w = __shfl_sync(kFull, s.w, src);
        const int32_t step = __shfl_sync(kFull, s.step, src);
        const int64_t a0 = max(i0, b_at), a1 = min(i1, b_at + n_tok);
        const uint32_t hw = h == 0 ? 1u : static_cast<uint32_t>(h) * w;
        for (int64_t i = a0 + lane; i < a1; i += 32) {
          const uint32_t rel = static_cast<uint32_t>(i - b_at);
          const uint32_t t = static_cast<uint32_t>(begin + i - cached);
          if (h == 0) {
            put(t, base + rel, base + rel, base + rel);
          } else {
            const uint32_t frame = rel / hw, in = rel - frame * hw, y = in / w;
            put(t, base + static_cast<int64_t>(frame) * step, base + y, base + in - y * w);
          }
        }
      }
      at += __shfl_sync(kFull, tok, 31);
      place += __shfl_sync(kFull, ext, 31);
    }
    // text behind the spans
    for (int64_t i = max(i0, at) + lane; i < i1; i += 32) {
      const int64_t v = place + i - at;
      put(static_cast<uint32_t>(begin + i - cached), v, v, v);
    }
    ++r;
  }
  for (uint32_t t = done + lane; t < t1; t += 32) put(t, 0, 0, 0);
}

// ---- preba_rope_append ----------------------------------------------------------------------------
//
// A CTA takes a few tokens: it works out their cosines and sines once (one per pair, in 64 bits up to
// the reduced angle; all heads of a token share them) and then moves the heads, eight pairs or sixteen
// copied elements to a thread, in 16-byte loads and stores.  Where there are few tokens, several CTAs share
// one and each takes a part of its heads, so that no thread moves more than one job.  Bound by bytes: 54 to
// 57 us for 16 K rows of 32 + 8 + 8 heads of 128 (327 MB, 5.8 TB/s), 5.6 us for 20 MB, 3.3 us for 32 rows.

constexpr int kRopeThreads = 256;
constexpr uint32_t kRopeTokens = 4;
constexpr uint32_t kRopePlaces = 148 * 4;  // blocks that are resident at a time, about

template <typename T> struct pair_of;
template <> struct pair_of<__half> {
  static __device__ __forceinline__ float2 open(uint32_t v) {
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
  }
  static __device__ __forceinline__ uint32_t close(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};
template <> struct pair_of<__nv_bfloat16> {
  static __device__ __forceinline__ float2 open(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t close(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
};

__device__ __forceinline__ uint32_t axis_of(uint32_t j, const uint32_t (&sections)[3], bool in_turn) {
  if (!in_turn) return (j >= sections[0]) + (j >= sections[0] + sections[1]);
  const uint32_t third = j / 3, a = j - 3 * third;
  return a == 1 ? (third < sections[1] ? 1u : 0u) : a == 2 ? (third < sections[2] ? 2u : 0u) : 0u;
}

template <typename T, bool kShared>
__global__ void __launch_bounds__(kRopeThreads)
append_kernel(const preba_rope_append_t p, const uint32_t page_shift, const uint32_t blocks) {
  chained_begin();
  constexpr uint32_t kTokens = kShared ? 1 : kRopeTokens;  // of a block, or of `blocks` blocks
  __shared__ float2 turn[kTokens][PREBA_PAGES_MAX_HEAD_DIM / 2];
  const uint32_t group = kShared ? blockIdx.x / blocks : blockIdx.x;
  const uint32_t t0 = group * kTokens;
  const uint32_t n_tok = min(kTokens, p.tokens - t0);
  const uint32_t first = kShared ? (blockIdx.x - group * blocks) * kRopeThreads : 0;
  const uint32_t stride = kShared ? blocks * kRopeThreads : kRopeThreads;
  const uint32_t pairs = p.rotary_dim / 2;
  const bool in_turn = p.flags & PREBA_ROPE_AXES_IN_TURN;
  const bool inter = p.flags & PREBA_ROPE_INTERLEAVED;
  for (uint32_t i = threadIdx.x; i < n_tok * pairs; i += kRopeThreads) {
    const uint32_t tok = i / pairs, j = i - tok * pairs;
    const int32_t pos = p.positions[axis_of(j, p.sections, in_turn) * p.axis_stride + t0 + tok];
    // the angle in half turns, reduced to [-1, 1] in 64 bits: what is left is exact to fp32
    const double half = pos * p.inv_freq[j] * 0.31830988618379067154;
    float s, c;
    sincospif(static_cast<float>(half - 2.0 * rint(0.5 * half)), &s, &c);
    turn[tok][j] = make_float2(c, s);
  }
  __syncthreads();
  // jobs of a token: heads_q + heads_kv heads of pairs/8 rotations and (head_dim - rotary_dim)/16
  // copies, then heads_kv heads of values of head_dim/16 copies (rounded up)
  const uint32_t rot_jobs = pairs / 8, rest_jobs = (p.head_dim - p.rotary_dim + 15) / 16;
  const uint32_t head_jobs = rot_jobs + rest_jobs, v_jobs = (p.head_dim + 15) / 16;
  const uint32_t qk_jobs = (p.heads_q + p.heads_kv) * head_jobs;
  const uint32_t jobs = qk_jobs + p.heads_kv * v_jobs;
  const uint64_t slots = static_cast<uint64_t>(p.pages) << page_shift;
  for (uint32_t i = first + threadIdx.x; i < n_tok * jobs; i += stride) {
    const uint32_t tok = i / jobs;
    uint32_t job = i - tok * jobs;
    const uint32_t t = t0 + tok;
    const bool values = job >= qk_jobs;
    if (values) job -= qk_jobs;
    const uint32_t per = values ? v_jobs : head_jobs;
    uint32_t head = job / per;
    job -= head * per;
    const T* from;
    T* to;
    if (!values && head < p.heads_q) {
      from = static_cast<const T*>(p.q) + t * p.q_stride[0] + head * p.q_stride[1];
      to = static_cast<T*>(p.q_out) + t * p.q_out_stride[0] + head * p.q_out_stride[1];
    } else {
      if (!values) head -= p.heads_q;
      const int32_t slot = p.slots[t];
      if (slot < 0) continue;
      if (static_cast<uint64_t>(slot) >= slots) {
        report(p.status, PREBA_ERR_BAD_TABLE);
        continue;
      }
      const uint64_t at = (static_cast<uint32_t>(slot) >> page_shift) * p.cache_stride[0] +
                          (static_cast<uint32_t>(slot) & ((1u << page_shift) - 1)) * p.cache_stride[1] +
                          head * p.cache_stride[2];
      if (values) {
        from = static_cast<const T*>(p.v) + t * p.v_stride[0] + head * p.v_stride[1];
        to = static_cast<T*>(p.v_cache) + at;
      } else {
        from = static_cast<const T*>(p.k) + t * p.k_stride[0] + head * p.k_stride[1];
        to = static_cast<T*>(p.k_cache) + at;
      }
    }
    if (values || job >= rot_jobs) {
      const uint32_t e = values ? 16 * job : p.rotary_dim + 16 * (job - rot_jobs);
      *reinterpret_cast<uint4*>(to + e) = *reinterpret_cast<const uint4*>(from + e);
      if (e + 8 < p.head_dim)
        *reinterpret_cast<uint4*>(to + e + 8) = *reinterpret_cast<const uint4*>(from + e + 8);
      continue;
    }
    const uint32_t ea = inter ? 16 * job : 8 * job;
    const uint32_t eb = inter ? 16 * job + 8 : 8 * job + pairs;
    union { uint4 v; uint32_t u[4]; } a, b;
    a.v = *reinterpret_cast<const uint4*>(from + ea);
    b.v = *reinterpret_cast<const uint4*>(from + eb);
    const float2* cs = &turn[tok][8 * job];
    if (inter) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 x = pair_of<T>::open(a.u[k]), y = pair_of<T>::open(b.u[k]);
        const float2 ca = cs[k], cb = cs[4 + k];
        a.u[k] = pair_of<T>::close(x.x * ca.x - x.y * ca.y, x.y * ca.x + x.x * ca.y);
        b.u[k] = pair_of<T>::close(y.x * cb.x - y.y * cb.y, y.y * cb.x + y.x * cb.y);
      }
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 x = pair_of<T>::open(a.u[k]), y = pair_of<T>::open(b.u[k]);
        const float2 c0 = cs[2 * k], c1 = cs[2 * k + 1];
        a.u[k] = pair_of<T>::close(x.x * c0.x - y.x * c0.y, x.y * c1.x - y.y * c1.y);
        b.u[k] = pair_of<T>::close(y.x * c0.x + x.x * c0.y, y.y * c1.x + x.y * c1.y);
      }
    }
    *reinterpret_cast<uint4*>(to + ea) = a.v;
    *reinterpret_cast<uint4*>(to + eb) = b.v;
  }
}

bool power_of_two_page(uint32_t page) {
  return page >= 8 && page <= PREBA_PAGES_MAX_PAGE && (page & (page - 1)) == 0;
}

uint32_t log2_of(uint32_t v) { return 31 - __builtin_clz(v); }

int finish(cudaError_t err) {
  if (err == cudaSuccess) return PREBA_OK;
  g_last_cuda_error = static_cast<int>(err);
  return PREBA_ERR_CUDA;
}

bool aligned(const void* ptr, uint64_t to) { return (reinterpret_cast<uintptr_t>(ptr) & (to - 1)) == 0; }

}  // namespace
}  // namespace preba

extern "C" int preba_pages_plan(const preba_pages_plan_t* plan, void* stream) {
  using namespace preba;
  if (!plan) return PREBA_ERR_INVALID_ARG;
  const preba_pages_plan_t& p = *plan;
  if (!p.cached || !p.fresh || !p.block_table || !p.free_count || !p.cu_q || !p.kv_len || !p.free_left ||
      (!p.free_pages && p.free_capacity) || (!p.slots && p.tokens) || p.n == 0 ||
      p.n > PREBA_PAGES_MAX_REQUESTS || !power_of_two_page(p.page_size) || p.tokens > INT32_MAX ||
      static_cast<uint64_t>(p.pages) * p.page_size > INT32_MAX || p.table_stride < p.table_width ||
      p.free_left == p.free_count)
    return PREBA_ERR_INVALID_ARG;
  const size_t smem = (2ull * p.n + 1) * sizeof(int32_t);
  if (smem > 48 * 1024) {
    const int rc = finish(cudaFuncSetAttribute(
        plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
        static_cast<int>((2 * PREBA_PAGES_MAX_REQUESTS + 1) * sizeof(int32_t))));
    if (rc != PREBA_OK) return rc;
  }
  const uint32_t grid = std::max(1u, (p.tokens + kPlanTokensPerCta - 1) / kPlanTokensPerCta);
  return finish(launch_chained(plan_kernel, grid, kPlanThreads, smem, static_cast<cudaStream_t>(stream), p,
                               log2_of(p.page_size)));
}

extern "C" int preba_rope_positions(const preba_rope_positions_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_rope_positions_t& p = *req;
  if ((!p.spans && p.n_spans) || !p.span_begin || !p.cached || !p.cu_q || !p.positions || p.n == 0 ||
      p.n > INT32_MAX || p.tokens == 0 || p.tokens > INT32_MAX || p.n_spans > INT32_MAX ||
      p.axis_stride < p.tokens || !aligned(p.spans, 16))
    return PREBA_ERR_INVALID_ARG;
  // about 2400 warps fill the GPU once; a warp has at least one row and, in large steps, many
  const uint32_t run = std::min(256u, (p.tokens + 2367) / 2368);
  const uint64_t warps = (p.tokens + run - 1) / run;
  const uint32_t grid = static_cast<uint32_t>((warps * 32 + kPosThreads - 1) / kPosThreads);
  return finish(launch_chained(positions_kernel, grid, kPosThreads, 0, static_cast<cudaStream_t>(stream), p, run));
}

extern "C" int preba_rope_append(const preba_rope_append_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_rope_append_t& p = *req;
  if (p.tokens == 0 || p.tokens > INT32_MAX || p.heads_q + static_cast<uint64_t>(p.heads_kv) == 0 ||
      p.heads_q > 65535 || p.heads_kv > 65535 || !p.positions ||
      (p.dtype != PREBA_F16 && p.dtype != PREBA_BF16) ||
      (p.flags & ~(PREBA_ROPE_INTERLEAVED | PREBA_ROPE_AXES_IN_TURN)))
    return PREBA_ERR_INVALID_ARG;
  if (p.head_dim == 0 || p.head_dim % 8 || p.head_dim > PREBA_PAGES_MAX_HEAD_DIM || p.rotary_dim > p.head_dim ||
      p.rotary_dim % 16 || (p.rotary_dim && (!p.inv_freq || !aligned(p.inv_freq, 8))))
    return PREBA_ERR_INVALID_ARG;
  const uint64_t pairs = p.rotary_dim / 2;
  if (static_cast<uint64_t>(p.sections[0]) + p.sections[1] + p.sections[2] != pairs)
    return PREBA_ERR_INVALID_ARG;
  if ((p.flags & PREBA_ROPE_AXES_IN_TURN) &&
      (p.sections[1] > (pairs + 1) / 3 || p.sections[2] > pairs / 3))
    return PREBA_ERR_INVALID_ARG;
  auto strides_ok = [](const uint64_t* s, int count) {
    for (int i = 0; i < count; ++i)
      if (s[i] % 8) return false;
    return true;
  };
  if (p.heads_q && (!p.q || !p.q_out || !aligned(p.q, 16) || !aligned(p.q_out, 16) ||
                    !strides_ok(p.q_stride, 2) || !strides_ok(p.q_out_stride, 2)))
    return PREBA_ERR_INVALID_ARG;
  if (p.heads_kv &&
      (!p.k || !p.v || !p.k_cache || !p.v_cache || !p.slots || !aligned(p.k, 16) || !aligned(p.v, 16) ||
       !aligned(p.k_cache, 16) || !aligned(p.v_cache, 16) || !strides_ok(p.k_stride, 2) ||
       !strides_ok(p.v_stride, 2) || !strides_ok(p.cache_stride, 3) || !power_of_two_page(p.page_size) ||
       static_cast<uint64_t>(p.pages) * p.page_size > INT32_MAX))
    return PREBA_ERR_INVALID_ARG;
  // where blocks of several tokens would leave places on the GPU empty, every token gets as many blocks as
  // it has jobs for: 32 tokens of 40 heads 5.3 -> 3.3 us, 4000 tokens of 18 heads 5.5 us (single: 9.0)
  const uint32_t jobs = (p.heads_q + p.heads_kv) * (p.rotary_dim / 16 + (p.head_dim - p.rotary_dim + 15) / 16) +
                        p.heads_kv * ((p.head_dim + 15) / 16);
  const bool shared = p.tokens < kRopePlaces;
  const uint32_t blocks = shared ? (jobs + kRopeThreads - 1) / kRopeThreads : 1;
  const uint32_t grid = shared ? p.tokens * blocks : (p.tokens + kRopeTokens - 1) / kRopeTokens;
  const uint32_t shift = p.heads_kv ? log2_of(p.page_size) : 3;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto kernel = p.dtype == PREBA_F16
                    ? (shared ? append_kernel<__half, true> : append_kernel<__half, false>)
                    : (shared ? append_kernel<__nv_bfloat16, true> : append_kernel<__nv_bfloat16, false>);
  return finish(launch_chained(kernel, grid, kRopeThreads, 0, s, p, shift, blocks));
}
