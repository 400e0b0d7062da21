// A beam search over the paged cache (preba_beams.h): preba_beam_select, preba_beam_pages, preba_pages_copy.
#include <algorithm>

#include "preba_attend.h"
#include "preba_beams.h"

namespace preba {
namespace {

using attend::exp2_approx;
using attend::kFull;
using attend::kLog2e;
using attend::report;

// ---- preba_beam_select ------------------------------------------------------------------------------
//
// The logits have to be read once and the answer is a few numbers, so bytes bound it, and latency where they are
// few.  A first kernel reads them in segments of 2 KB, a warp each, and leaves of every segment its maximum
// and the sum of its exponentials beside that maximum.  No lists are kept on the way: the best `width` tokens of a
// request lie in the `width` segments with the best maxima (in the order of rank, beam, segment), because
// every other segment has `width` maxima before all that it holds.  The second kernel, a block per request, adds the
// sums up in 64 bits, orders the maxima, reads those few segments again and orders what they hold.

constexpr int kSegmentWords = 512;  // of 32 bits
constexpr int kLaneWords = kSegmentWords / 32;
constexpr int kScanThreads = 256, kChooseThreads = 512;
constexpr int kChooseWarps = kChooseThreads / 32;

template <typename T> constexpr int kPerWord = 4 / sizeof(T);
template <typename T> constexpr int kSegment = kSegmentWords * kPerWord<T>;  // elements
template <typename T> constexpr int kLane = kLaneWords * kPerWord<T>;        // elements of a lane

struct select_args {
  preba_beam_select_t p;
  uint32_t segments;  // of a row
  float2* parts;      // of every segment: maximum, sum of exponentials
};

// The place in its segment of a lane's i-th element, ascending in i.  Vectors of 16 bytes where every row begins at a
// multiple of 16; else words, lane by lane.  All rows of a call are read alike, so that equal rows have equal sums.
template <typename T, bool Vec> __device__ __forceinline__ uint32_t place(int i) {
  constexpr int per = kPerWord<T>;
  const uint32_t lane = threadIdx.x & 31, w = i / per;
  const uint32_t word = Vec ? (w / 4) * 128 + lane * 4 + w % 4 : w * 32 + lane;
  return word * per + i % per;
}

__device__ __forceinline__ float number(float v) { return v; }
__device__ __forceinline__ float number(__half v) { return __half2float(v); }
__device__ __forceinline__ float number(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ void unpack(uint32_t w, float* x);
template <> __device__ __forceinline__ void unpack<float>(uint32_t w, float* x) { x[0] = __uint_as_float(w); }
template <> __device__ __forceinline__ void unpack<__half>(uint32_t w, float* x) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  x[0] = f.x, x[1] = f.y;
}
template <> __device__ __forceinline__ void unpack<__nv_bfloat16>(uint32_t w, float* x) {
  x[0] = __uint_as_float(w << 16), x[1] = __uint_as_float(w & 0xffff0000u);
}

// A lane's elements of segment s of a row; what is behind the vocabulary or not allowed is -inf.
template <typename T, bool Vec>
__device__ __forceinline__ void load_segment(const select_args& a, uint32_t row, uint32_t s, float (&x)[kLane<T>]) {
  const preba_beam_select_t& p = a.p;
  constexpr int per = kPerWord<T>;
  const uint32_t first = s * kSegment<T>;
  const T* from = static_cast<const T*>(p.logits) + row * p.row_stride + first;
  const uint32_t left = p.vocab - first;  // at least 1
  if (left >= kSegment<T>) {
    if (Vec) {
#pragma unroll
      for (int w = 0; w < kLaneWords; w += 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(from + place<T, Vec>(w * per)));
        unpack<T>(v.x, x + w * per), unpack<T>(v.y, x + (w + 1) * per);
        unpack<T>(v.z, x + (w + 2) * per), unpack<T>(v.w, x + (w + 3) * per);
      }
    } else if (per == 1 || !(reinterpret_cast<uintptr_t>(from) & 2)) {
#pragma unroll
      for (int w = 0; w < kLaneWords; ++w)
        unpack<T>(__ldg(reinterpret_cast<const uint32_t*>(from + place<T, Vec>(w * per))), x + w * per);
    } else {
#pragma unroll
      for (int i = 0; i < kLane<T>; ++i) x[i] = number(from[place<T, Vec>(i)]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kLane<T>; ++i) {
      const uint32_t e = place<T, Vec>(i);
      x[i] = e < left ? number(from[e]) : -INFINITY;
    }
  }
  if (p.allowed) {
    // elements of a word lie in the same word of bits, and so do those of a vector
    const uint32_t* bits = p.allowed + row * p.allowed_stride + first / 32;
    constexpr int step = Vec ? 4 * per : per;
#pragma unroll
    for (int i = 0; i < kLane<T>; i += step) {
      const uint32_t e = place<T, Vec>(i);
      const uint32_t word = e < left ? __ldg(bits + e / 32) >> (e % 32) : 0;
#pragma unroll
      for (int k = 0; k < step; ++k)
        if (!(word >> k & 1)) x[i + k] = -INFINITY;
    }
  }
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
  return v;
}
template <typename N> __device__ __forceinline__ N warp_sum(N v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}

// Whether a row offers what its logits say: it is there and has not ended.
__device__ __forceinline__ bool row_live(const preba_beam_select_t& p, uint32_t row) {
  return !(p.done && p.done[row]) && p.scores[row] != -INFINITY;
}

template <typename T, bool Vec>
__global__ void __launch_bounds__(kScanThreads) scan_kernel(const select_args a) {
  const preba_beam_select_t& p = a.p;
  chained_begin();
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t total = p.n * p.beams * a.segments;
  const uint32_t stride = gridDim.x * (kScanThreads / 32);
  for (uint32_t unit = blockIdx.x * (kScanThreads / 32) + threadIdx.x / 32; unit < total; unit += stride) {
    const uint32_t row = unit / a.segments, s = unit - row * a.segments;
    if (!row_live(p, row)) continue;
    float x[kLane<T>];
    load_segment<T, Vec>(a, row, s, x);
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kLane<T>; ++i) top = fmaxf(top, x[i]);
    top = warp_max(top);
    const float from = top == -INFINITY ? 0.f : top;  // then all of it is -inf, or not a number
    float sum = 0.f;
    // the difference is rounded before it is scaled: what is near the maximum, and counts, is exact
#pragma unroll
    for (int i = 0; i < kLane<T>; ++i) sum += exp2_approx((x[i] - from) * kLog2e);
    sum = warp_sum(sum);
    if (lane == 0) a.parts[unit] = make_float2(top, sum);
  }
}

// A candidate: a segment by its maximum, or a token.  `at` is the segment or the token.
struct candidate_t {
  double rank;
  float x;       // the logit (of a row that is done: 0)
  uint32_t row;  // the beam
  uint32_t at;
};
__device__ __forceinline__ bool before(const candidate_t& a, const candidate_t& b) {
  if (a.rank != b.rank) return a.rank > b.rank;
  if (a.row != b.row) return a.row < b.row;
  if (a.x != b.x) return a.x > b.x;
  return a.at < b.at;
}

struct choose_shared {
  double lse[PREBA_BEAMS_MAX], score[PREBA_BEAMS_MAX], weight[PREBA_BEAMS_MAX];
  uint32_t live[PREBA_BEAMS_MAX];     // 0: offers nothing, 1: its logits, 2: its end token
  uint32_t listed, chosen, found;
  candidate_t best[PREBA_BEAMS_MAX_WIDTH];  // segments
};

// Candidates of a request at most: segments, the first `width` of each row, or tokens, where the k-th segment can
// give no more than width - k.
__host__ __device__ inline uint32_t candidates_of(uint32_t beams, uint32_t width) {
  const uint32_t tokens = width * (width + 1) / 2;
  return beams * width > tokens ? beams * width : tokens;
}

// One more candidate; their order in the list is that of whoever came first and means nothing.
__device__ __forceinline__ void add(const preba_beam_select_t& p, candidate_t* list, uint32_t* count, uint32_t room,
                                    const candidate_t& c) {
  const uint32_t at = atomicAdd(count, 1);
  if (PREBA_IN_RANGE(p.status, at < room)) list[at] = c;
}

__device__ __forceinline__ double value_of(const choose_shared& c, uint32_t row, float x) {
  return (static_cast<double>(x) - c.lse[row]) + c.score[row];
}

// The best candidate of the warp's lanes, `none` lanes taking no part; false if there is none.  In one row: by
// logit, then place.
__device__ __forceinline__ bool warp_best(float& x, uint32_t& at) {
  const float top = warp_max(x);
  if (top == -INFINITY) return false;
  at = __reduce_min_sync(kFull, x == top ? at : UINT32_MAX);
  x = top;
  return true;
}

template <typename T, bool Vec>
__global__ void __launch_bounds__(kChooseThreads) choose_kernel(const select_args a) {
  extern __shared__ __align__(16) uint8_t choose_smem[];
  candidate_t* list = reinterpret_cast<candidate_t*>(choose_smem);
  __shared__ choose_shared c;
  const preba_beam_select_t& p = a.p;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t r = blockIdx.x, row0 = r * p.beams, room = candidates_of(p.beams, p.width);
  if (threadIdx.x == 0) c.listed = c.chosen = c.found = 0;
  __syncthreads();
  chained_begin();

  // a warp per beam: the sum of its exponentials, then its best segments
  for (uint32_t b = warp; b < p.beams; b += kChooseWarps) {
    const uint32_t row = row0 + b;
    const float score = p.scores[row], weight = p.weights ? p.weights[row] : 1.f;
    const bool done = p.done && p.done[row];
    if (score == -INFINITY) {
      if (lane == 0) c.live[b] = 0;
      continue;
    }
    bool good = score < INFINITY && weight > 0.f && weight < INFINITY;
    const float2* parts = a.parts + static_cast<uint64_t>(row) * a.segments;
    float top = -INFINITY;
    double sum = 0, lse = 0;
    if (!done) {
      for (uint32_t s = lane; s < a.segments; s += 32) top = fmaxf(top, parts[s].x);
      top = warp_max(top);
      for (uint32_t s = lane; s < a.segments; s += 32) {
        const float2 part = parts[s];
        // a segment of nothing has the sum 0; one of -inf and NaN has a sum that is not a number
        sum += part.x == -INFINITY ? static_cast<double>(part.y) : static_cast<double>(part.y) * exp(static_cast<double>(part.x) - top);
      }
      sum = warp_sum(sum);
      lse = top + log(sum);
      good = good && (top == -INFINITY ? sum == 0 : lse < INFINITY);  // not a number: false
    }
    if (lane == 0) {
      if (!good) report(p.status, PREBA_ERR_BAD_TABLE);
      c.live[b] = !good ? 0 : done ? 2 : top > -INFINITY;
      c.lse[b] = lse;
      c.score[b] = score;
      c.weight[b] = weight;
    }
    __syncwarp();
    if (!good) continue;
    if (done) {
      if (lane == 0) add(p, list, &c.listed, room, {static_cast<double>(weight) * score, 0.f, b, UINT32_MAX});
      continue;
    }
    // the segments in order, one by one: what follows the one before
    float last_x = INFINITY;
    uint32_t last_s = 0;
    for (uint32_t k = 0; k < p.width; ++k) {
      float x = -INFINITY;
      uint32_t at = UINT32_MAX;
      for (uint32_t s = lane; s < a.segments; s += 32) {
        const float m = parts[s].x;
        const bool after = m < last_x || (m == last_x && s > last_s);
        if (after && m > x) x = m, at = s;
      }
      if (!warp_best(x, at)) break;
      last_x = x, last_s = at;
      if (lane == 0) add(p, list, &c.listed, room, {c.weight[b] * value_of(c, b, x), x, b, at});
    }
  }
  __syncthreads();

  // the order of the segments: everyone counts who comes before
  const uint32_t listed = min(c.listed, room);
  for (uint32_t i = threadIdx.x; i < listed; i += kChooseThreads) {
    const candidate_t mine = list[i];
    uint32_t ahead = 0;
    for (uint32_t k = 0; k < listed; ++k) ahead += before(list[k], mine);
    if (ahead < p.width) c.best[ahead] = mine;
  }
  if (threadIdx.x == 0) c.chosen = min(listed, p.width);
  __syncthreads();

  // what the best segments hold, as far as it can be among the first: a warp per segment
  const uint32_t chosen = c.chosen;
  const bool full = chosen == p.width;  // nothing after the last segment's maximum is among the first
  for (uint32_t k = warp; k < chosen; k += kChooseWarps) {
    const candidate_t seg = c.best[k];
    if (seg.at == UINT32_MAX) {
      if (lane == 0) add(p, list, &c.found, room, {seg.rank, 0.f, seg.row, static_cast<uint32_t>(p.end_token)});
      continue;
    }
    float x[kLane<T>];
    load_segment<T, Vec>(a, row0 + seg.row, seg.at, x);
    const double floor = c.best[chosen - 1].rank;
    for (uint32_t j = k; j < p.width; ++j) {
      float best = -INFINITY;
      uint32_t at = UINT32_MAX;
#pragma unroll
      for (int i = 0; i < kLane<T>; ++i)
        if (x[i] > best) best = x[i], at = place<T, Vec>(i);
      if (!warp_best(best, at)) break;
      const double rank = c.weight[seg.row] * value_of(c, seg.row, best);
      if (full && rank < floor) break;
#pragma unroll
      for (int i = 0; i < kLane<T>; ++i)
        if (place<T, Vec>(i) == at) x[i] = -INFINITY;
      if (lane == 0) add(p, list, &c.found, room, {rank, best, seg.row, seg.at * kSegment<T> + at});
    }
  }
  __syncthreads();

  const uint32_t found = min(c.found, room);
  const uint64_t out = static_cast<uint64_t>(r) * p.width;
  for (uint32_t i = threadIdx.x; i < found; i += kChooseThreads) {
    const candidate_t mine = list[i];
    uint32_t ahead = 0;
    for (uint32_t k = 0; k < found; ++k) ahead += before(list[k], mine);
    if (ahead >= p.width) continue;
    const bool done = c.live[mine.row] == 2;
    p.tokens[out + ahead] = static_cast<int32_t>(mine.at);
    p.parents[out + ahead] = static_cast<int32_t>(mine.row);
    p.scores_out[out + ahead] = static_cast<float>(done ? c.score[mine.row] : value_of(c, mine.row, mine.x));
    if (p.done_out) p.done_out[out + ahead] = done || static_cast<int32_t>(mine.at) == p.end_token;
  }
  for (uint32_t i = found + threadIdx.x; i < p.width; i += kChooseThreads) {
    p.tokens[out + i] = p.parents[out + i] = -1;
    p.scores_out[out + i] = -INFINITY;
    if (p.done_out) p.done_out[out + i] = 0;
  }
}

int finish(cudaError_t err) {
  if (err == cudaSuccess) return PREBA_OK;
  g_last_cuda_error = static_cast<int>(err);
  return PREBA_ERR_CUDA;
}

bool aligned(const void* p, uintptr_t a) { return !(reinterpret_cast<uintptr_t>(p) & (a - 1)); }

bool select_sizes_ok(uint32_t n, uint32_t beams, uint32_t width, uint32_t vocab, int32_t dtype) {
  return n >= 1 && beams >= 1 && beams <= PREBA_BEAMS_MAX && static_cast<uint64_t>(n) * beams <= PREBA_PAGES_MAX_REQUESTS &&
         width >= 1 && width <= PREBA_BEAMS_MAX_WIDTH && vocab >= 1 && vocab <= PREBA_BEAMS_MAX_VOCAB &&
         (dtype == PREBA_F32 || dtype == PREBA_F16 || dtype == PREBA_BF16);
}
uint32_t segments_of(uint32_t vocab, int32_t dtype) {
  const uint32_t segment = dtype == PREBA_F32 ? kSegment<float> : kSegment<__half>;
  return (vocab + segment - 1) / segment;
}

template <typename T, bool Vec> cudaError_t launch_select(const select_args& a, int sms, cudaStream_t stream) {
  const preba_beam_select_t& p = a.p;
  const uint64_t units = static_cast<uint64_t>(p.n) * p.beams * a.segments;
  const uint32_t grid = static_cast<uint32_t>(std::min<uint64_t>((units + kScanThreads / 32 - 1) / (kScanThreads / 32), 8ull * sms));
  cudaError_t err = launch_chained(scan_kernel<T, Vec>, grid, kScanThreads, 0, stream, a);
  if (err != cudaSuccess) return err;
  const size_t smem = candidates_of(p.beams, p.width) * sizeof(candidate_t);
  if (smem > 40 * 1024) {  // beside 3 KB of its own
    err = cudaFuncSetAttribute(choose_kernel<T, Vec>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(candidates_of(PREBA_BEAMS_MAX, PREBA_BEAMS_MAX_WIDTH) * sizeof(candidate_t)));
    if (err != cudaSuccess) return err;
  }
  return launch_chained(choose_kernel<T, Vec>, p.n, kChooseThreads, smem, stream, a);
}

// ---- preba_beam_pages -------------------------------------------------------------------------------
//
// The tables have to be read and written once; with a few hundred columns that is little, and latency bounds it.
// Beams share pages only at the same place of their rows, so what is released shows column by column, without
// counts of holders: a page of a beam that has no child, that no beam with a child has in that column, and that no
// childless beam before it has.  A first kernel, a block per 256 columns of a request, writes the new rows and
// lists what is released; a second, one block, numbers all of it and hands it out.

constexpr int kColumns = 256;
constexpr int kHandThreads = 1024;

struct pages_args {
  preba_beam_pages_t p;
  uint32_t page_shift, chunks;  // chunks of columns of a row
  int32_t* need;      // n: copies of a request, or below 0: refused
  uint32_t* copies_before;  // n
  uint32_t* counts;   // n * chunks: pages released
  int64_t* before;    // n * chunks: pages released before
  int32_t* given;     // n * beams: the first released pages
  int32_t* lists;     // n * chunks lists of kColumns * beams pages
};

__device__ __forceinline__ uint32_t held_pages(const pages_args& a, int32_t length) {
  return (static_cast<uint32_t>(length) + (1u << a.page_shift) - 1) >> a.page_shift;
}

__global__ void __launch_bounds__(kColumns) follow_kernel(const pages_args a) {
  extern __shared__ int32_t tile[];  // beams x kColumns
  __shared__ int32_t parent[PREBA_BEAMS_MAX], length[PREBA_BEAMS_MAX];
  __shared__ uint32_t held[PREBA_BEAMS_MAX], warp_sums[kColumns / 32];
  const preba_beam_pages_t& p = a.p;
  const uint32_t r = blockIdx.x / a.chunks, chunk = blockIdx.x - r * a.chunks, row0 = r * p.beams;
  const uint32_t c = chunk * kColumns + threadIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  chained_begin();
  bool bad = false;
  if (threadIdx.x < p.beams) {
    const int32_t len = p.lengths[row0 + threadIdx.x], par = p.parents[row0 + threadIdx.x];
    const uint32_t h = len < 0 ? 0 : held_pages(a, len);
    bad = len < 0 || h > p.table_width || par >= static_cast<int32_t>(p.beams);
    parent[threadIdx.x] = par < 0 ? -1 : par;
    length[threadIdx.x] = len;
    held[threadIdx.x] = min(h, p.table_width);
  }
  const bool refused = __syncthreads_or(bad);
  uint32_t parents = 0;  // a bit per beam that has a child
  for (uint32_t b = 0; b < p.beams; ++b)
    if (parent[b] >= 0 && !refused) parents |= 1u << parent[b];
  for (uint32_t b = 0; b < p.beams; ++b)
    if (c < held[b]) tile[b * kColumns + threadIdx.x] = p.table[(row0 + b) * p.table_stride + c];
  // the new rows; every thread reads its own column only
  for (uint32_t i = 0; i < p.beams; ++i) {
    const int32_t from = refused ? static_cast<int32_t>(i) : parent[i];
    if (from >= 0 && c < held[from]) p.table_out[(row0 + i) * p.table_out_stride + c] = tile[from * kColumns + threadIdx.x];
  }
  // what this column releases, a bit per beam
  uint32_t gone = 0;
  const int64_t kept = p.kept ? p.kept[r] : 0;
  if (!refused && c >= kept)
    for (uint32_t b = 0; b < p.beams; ++b) {
      if (parents >> b & 1 || c >= held[b]) continue;
      const int32_t page = tile[b * kColumns + threadIdx.x];
      bool alone = true;
      for (uint32_t o = 0; o < p.beams; ++o)
        if ((parents >> o & 1 || o < b) && c < held[o] && tile[o * kColumns + threadIdx.x] == page) alone = false;
      if (!alone) continue;
      if (page < 0 || static_cast<uint32_t>(page) >= p.pages) report(p.status, PREBA_ERR_BAD_TABLE);
      else gone |= 1u << b;
    }
  const uint32_t mine = __popc(gone);
  uint32_t incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  uint32_t at = incl - mine, total = 0;
  for (int w = 0; w < kColumns / 32; ++w) {
    if (w < warp) at += warp_sums[w];
    total += warp_sums[w];
  }
  int32_t* to = a.lists + static_cast<uint64_t>(blockIdx.x) * kColumns * p.beams;
  for (; gone; gone &= gone - 1)
    if (PREBA_IN_RANGE(p.status, at < kColumns * p.beams)) to[at++] = tile[(__ffs(gone) - 1) * kColumns + threadIdx.x];
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;

  if (chunk) return;
  // lengths, and which children need an open page: a row's number among those of its request in place of the page
  uint32_t copied = 0;
  int4 copy = make_int4(0, 0, 0, 0);
  if (warp == 0) {
    bool needs = false;
    if (lane < static_cast<int>(p.beams)) {
      const int32_t from = parent[lane];
      const bool there = !refused && from >= 0;
      const uint32_t open = there ? length[from] & ((1u << a.page_shift) - 1) : 0;
      p.lengths_out[row0 + lane] = there ? length[from] : 0;
      bool first = true;
      for (int i = 0; i < lane; ++i) first = first && parent[i] != from;
      needs = there && open && !first;
      if (needs) copy = make_int4(p.table[(row0 + from) * p.table_stride + held[from] - 1], 0, open, 0);
    }
    copied = __ballot_sync(kFull, needs);
    copy.y = needs ? __popc(copied & ((1u << lane) - 1)) : 0;
    if (lane < static_cast<int>(p.beams)) reinterpret_cast<int4*>(p.copies)[row0 + lane] = copy;
    if (lane == 0) {
      a.need[r] = refused ? -1 : __popc(copied);
      if (refused) report(p.status, PREBA_ERR_BAD_TABLE);
    }
  }
}

struct both_t {
  int64_t copies, released;
};
__device__ __forceinline__ both_t hand_exclusive(both_t v, both_t* warp_sums, both_t& total) {
  static_assert(kHandThreads == 1024, "a lane per warp");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  both_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(kFull, incl.copies, o), y = __shfl_up_sync(kFull, incl.released, o);
    if (lane >= o) incl.copies += x, incl.released += y;
  }
  __syncthreads();  // what an earlier call left has been read
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  const both_t of = warp_sums[lane];
  total = {warp_sum(of.copies), warp_sum(of.released)};
  return {warp_sum(lane < warp ? of.copies : 0) + incl.copies - v.copies,
          warp_sum(lane < warp ? of.released : 0) + incl.released - v.released};
}

__global__ void __launch_bounds__(kHandThreads) hand_out_kernel(const pages_args a) {
  __shared__ both_t warp_sums[32];
  const preba_beam_pages_t& p = a.p;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  chained_begin();
  int64_t count = *p.free_count;
  if (count < 0 || count > p.free_capacity) {
    if (threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
    count = 0;
  }
  const uint32_t per = (p.n + kHandThreads - 1) / kHandThreads;
  const uint32_t r0 = min(threadIdx.x * per, p.n), r1 = min(r0 + per, p.n);
  auto released_of = [&](uint32_t r) {
    int64_t sum = 0;
    for (uint32_t k = 0; k < a.chunks; ++k) sum += a.counts[r * a.chunks + k];
    return sum;
  };
  both_t before, total;
  bool any_refused = false;
  for (int round = 0; round < 2; ++round) {
    both_t mine{0, 0};
    bool refused = false, short_of = false;
    for (uint32_t r = r0; r < r1; ++r) {
      const int32_t need = a.need[r];
      refused |= need < 0;
      if (need >= 0) mine.copies += need, mine.released += released_of(r);
    }
    before = hand_exclusive(mine, warp_sums, total);
    both_t at = before;
    for (uint32_t r = r0; r < r1; ++r) {
      if (a.need[r] < 0) continue;
      at.copies += a.need[r], at.released += released_of(r);
      short_of |= count + at.released < at.copies;
    }
    any_refused = __syncthreads_or(refused);
    if (!__syncthreads_or(short_of)) break;
    // the pages do not suffice for all: one by one, in order.  The next round finds that they suffice
    if (threadIdx.x == 0) {
      int64_t left = count;
      for (uint32_t r = 0; r < p.n; ++r) {
        if (a.need[r] < 0) continue;
        const int64_t then = left + released_of(r) - a.need[r];
        if (then < 0) {
          a.need[r] = -2;
          report(p.status, PREBA_ERR_BUFFER_TOO_SMALL);
        } else {
          left = then;
        }
      }
    }
    __syncthreads();
  }
  both_t at = before;
  for (uint32_t r = r0; r < r1; ++r) {
    const bool served = a.need[r] >= 0;
    a.copies_before[r] = static_cast<uint32_t>(at.copies);
    if (served) at.copies += a.need[r];
    for (uint32_t k = 0; k < a.chunks; ++k) {
      const uint32_t unit = r * a.chunks + k;
      a.before[unit] = at.released;
      if (served) at.released += a.counts[unit];
      else a.counts[unit] = 0;
    }
  }
  __syncthreads();
  // what is released: to the copies first, then onto the stack
  for (uint32_t unit = warp; unit < p.n * a.chunks; unit += kHandThreads / 32) {
    const uint32_t pages = a.counts[unit];
    const int64_t first = a.before[unit];
    const int32_t* from = a.lists + static_cast<uint64_t>(unit) * kColumns * p.beams;
    for (uint32_t i = lane; i < pages; i += 32) {
      const int64_t k = first + i;
      if (k < total.copies) {
        if (PREBA_IN_RANGE(p.status, k < static_cast<int64_t>(p.n) * p.beams)) a.given[k] = from[i];
      } else if (count + k - total.copies < p.free_capacity) {
        p.free_pages[count + k - total.copies] = from[i];
      } else {
        report(p.status, PREBA_ERR_BAD_TABLE);
      }
    }
  }
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < p.n * p.beams; i += kHandThreads) {
    int4 copy = reinterpret_cast<const int4*>(p.copies)[i];
    if (copy.z == 0) continue;
    const uint32_t r = i / p.beams;
    if (a.need[r] < 0) {
      reinterpret_cast<int4*>(p.copies)[i] = make_int4(0, 0, 0, 0);
      continue;
    }
    const int64_t k = static_cast<int64_t>(a.copies_before[r]) + copy.y;
    copy.y = k < total.released ? a.given[k] : p.free_pages[count - 1 - (k - total.released)];
    const uint32_t last = held_pages(a, p.lengths_out[i]) - 1;
    if (PREBA_IN_RANGE(p.status, last < p.table_width)) p.table_out[i * p.table_out_stride + last] = copy.y;
    if (copy.y < 0 || static_cast<uint32_t>(copy.y) >= p.pages) {
      report(p.status, PREBA_ERR_BAD_TABLE);
      copy = make_int4(0, 0, 0, 0);
    }
    reinterpret_cast<int4*>(p.copies)[i] = copy;
  }
  if (threadIdx.x == 0)
    *p.free_left = static_cast<int32_t>(min(count + total.released - total.copies, static_cast<int64_t>(p.free_capacity)));
  if (!any_refused) return;
  // requests that were refused for want of pages: their rows as they were
  __syncthreads();
  for (uint32_t i = warp; i < p.n * p.beams; i += kHandThreads / 32) {
    if (a.need[i / p.beams] != -2) continue;
    const uint32_t held = held_pages(a, p.lengths[i]);
    for (uint32_t c = lane; c < held; c += 32) p.table_out[i * p.table_out_stride + c] = p.table[i * p.table_stride + c];
    if (lane == 0) p.lengths_out[i] = 0;
  }
}

uint64_t up16(uint64_t v) { return (v + 15) / 16 * 16; }

bool beam_sizes_ok(uint32_t n, uint32_t beams, uint32_t table_width) {
  return n >= 1 && beams >= 1 && beams <= PREBA_BEAMS_MAX && static_cast<uint64_t>(n) * beams <= PREBA_PAGES_MAX_REQUESTS &&
         table_width >= 1 && table_width <= INT32_MAX / 8;
}
uint64_t pages_workspace(uint32_t n, uint32_t beams, uint32_t table_width) {
  const uint64_t units = static_cast<uint64_t>(n) * ((table_width + kColumns - 1) / kColumns);
  return 2 * up16(4ull * n) + up16(4 * units) + up16(8 * units) + up16(4ull * n * beams) + 4 * units * kColumns * beams;
}

// ---- preba_pages_copy -------------------------------------------------------------------------------
//
// Bytes bound it: what is copied, in and out once.  The rows that have a copy are found by every block for itself, a
// job is a row's page in one cache, keys or values, and blocks take jobs in turn.

constexpr int kCopyThreads = 256;
constexpr uint32_t kCopyRows = 1024;  // looked at in one go
constexpr int kCopyDeep = 4;          // 16-byte loads of a thread on the way together

struct copy_args {
  preba_pages_copy_t p;
  uint32_t heads_first;  // heads are outside the slots in memory
  void* caches[2 * PREBA_COPY_MAX_LAYERS];
};

__global__ void __launch_bounds__(kCopyThreads) copy_kernel(const __grid_constant__ copy_args a) {
  __shared__ int4 jobs[kCopyRows];
  __shared__ uint32_t n_jobs;
  const preba_pages_copy_t& p = a.p;
  chained_begin();
  const uint32_t vectors = p.head_dim / 8;
  uint32_t turn = blockIdx.x;  // the block's next job, among all of them
  for (uint32_t row0 = 0; row0 < p.rows; row0 += kCopyRows) {
    __syncthreads();  // the jobs before have been read
    if (threadIdx.x < 32) {
      // in the order of the rows, for all blocks alike
      uint32_t found = 0;
      for (uint32_t i = row0 + threadIdx.x; i - threadIdx.x < min(p.rows, row0 + kCopyRows); i += 32) {
        int4 c = make_int4(0, 0, 0, 0);
        if (i < p.rows) c = __ldg(reinterpret_cast<const int4*>(p.copies) + i);
        const bool any = c.z != 0;
        const bool good = any && c.x >= 0 && static_cast<uint32_t>(c.x) < p.pages && c.y >= 0 &&
                          static_cast<uint32_t>(c.y) < p.pages && c.z > 0 && static_cast<uint32_t>(c.z) <= p.page_size;
        if (any && !good && blockIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
        const uint32_t mask = __ballot_sync(kFull, good);
        if (good) jobs[found + __popc(mask & ((1u << threadIdx.x) - 1))] = c;
        found += __popc(mask);
      }
      if (threadIdx.x == 0) n_jobs = found;
    }
    __syncthreads();
    const uint32_t caches = 2 * p.layers, all = n_jobs * caches;
    for (; turn < all; turn += gridDim.x) {
      const int4 c = jobs[turn / caches];
      uint8_t* base = static_cast<uint8_t*>(a.caches[turn % caches]);
      const uint8_t* from = base + 2 * c.x * p.cache_stride[0];
      uint8_t* to = base + 2 * c.y * p.cache_stride[0];
      const uint32_t total = c.z * p.heads_kv * vectors;
      const uint32_t inner = a.heads_first ? c.z : p.heads_kv;
      auto offset = [&](uint32_t i) -> uint64_t {
        const uint32_t v = i % vectors, k = i / vectors, in = k % inner, out = k / inner;
        const uint32_t slot = a.heads_first ? in : out, head = a.heads_first ? out : in;
        return 2 * (slot * p.cache_stride[1] + head * p.cache_stride[2] + 8 * v);
      };
      for (uint32_t i = threadIdx.x; i < total; i += kCopyDeep * kCopyThreads) {
        uint4 got[kCopyDeep];
        uint64_t at[kCopyDeep];
#pragma unroll
        for (int k = 0; k < kCopyDeep; ++k)
          if (i + k * kCopyThreads < total) {
            at[k] = offset(i + k * kCopyThreads);
            got[k] = *reinterpret_cast<const uint4*>(from + at[k]);
          }
#pragma unroll
        for (int k = 0; k < kCopyDeep; ++k)
          if (i + k * kCopyThreads < total) *reinterpret_cast<uint4*>(to + at[k]) = got[k];
      }
    }
    turn -= all;
  }
}

int device_sms(int* sms) {
  int device = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device);
  return finish(err);
}

}  // namespace
}  // namespace preba

extern "C" int preba_beam_select_query(uint32_t n, uint32_t beams, uint32_t width, uint32_t vocab, int32_t dtype,
                                       uint64_t* workspace_bytes) {
  using namespace preba;
  if (!workspace_bytes || !select_sizes_ok(n, beams, width, vocab, dtype)) return PREBA_ERR_INVALID_ARG;
  *workspace_bytes = up16(static_cast<uint64_t>(n) * beams * segments_of(vocab, dtype) * sizeof(float2));
  return PREBA_OK;
}

extern "C" int preba_beam_select(const preba_beam_select_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_beam_select_t& p = *req;
  uint64_t need = 0;
  if (preba_beam_select_query(p.n, p.beams, p.width, p.vocab, p.dtype, &need) != PREBA_OK) return PREBA_ERR_INVALID_ARG;
  const uint32_t wide = p.dtype == PREBA_F32 ? 4 : 2;
  const uint32_t rows = p.n * p.beams;
  if (!p.logits || !aligned(p.logits, wide) || !p.scores || !aligned(p.scores, 4) || !aligned(p.allowed, 4) ||
      !aligned(p.weights, 4) || !p.tokens || !aligned(p.tokens, 4) || !p.parents || !aligned(p.parents, 4) ||
      !p.scores_out || !aligned(p.scores_out, 4) || !p.workspace || !aligned(p.workspace, 16) ||
      (rows > 1 && p.row_stride < p.vocab) || p.row_stride >= (1ull << 38) || p.allowed_stride >= (1ull << 38) ||
      (rows > 1 && p.allowed && p.allowed_stride && p.allowed_stride < (p.vocab + 31) / 32) ||
      p.end_token < -1 || p.end_token >= static_cast<int64_t>(p.vocab) || (p.done && p.end_token < 0) ||
      p.scores_out == p.scores || (p.done && p.done_out == p.done))
    return PREBA_ERR_INVALID_ARG;
  if (p.workspace_bytes < need) return PREBA_ERR_BUFFER_TOO_SMALL;
  int sms = 0;
  const int rc = device_sms(&sms);
  if (rc != PREBA_OK) return rc;
  select_args a{p, segments_of(p.vocab, p.dtype), static_cast<float2*>(p.workspace)};
  const bool vec = aligned(p.logits, 16) && (rows == 1 || p.row_stride * wide % 16 == 0);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (p.dtype == PREBA_F32) return finish(vec ? launch_select<float, true>(a, sms, s) : launch_select<float, false>(a, sms, s));
  if (p.dtype == PREBA_F16) return finish(vec ? launch_select<__half, true>(a, sms, s) : launch_select<__half, false>(a, sms, s));
  return finish(vec ? launch_select<__nv_bfloat16, true>(a, sms, s) : launch_select<__nv_bfloat16, false>(a, sms, s));
}

extern "C" int preba_beam_pages_query(uint32_t n, uint32_t beams, uint32_t table_width, uint64_t* workspace_bytes) {
  using namespace preba;
  if (!workspace_bytes || !beam_sizes_ok(n, beams, table_width)) return PREBA_ERR_INVALID_ARG;
  *workspace_bytes = pages_workspace(n, beams, table_width);
  return PREBA_OK;
}

extern "C" int preba_beam_pages(const preba_beam_pages_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_beam_pages_t& p = *req;
  if (!beam_sizes_ok(p.n, p.beams, p.table_width) || !p.parents || !p.lengths || !p.table || !p.table_out ||
      !p.lengths_out || !p.copies || !aligned(p.copies, 16) || (!p.free_pages && p.free_capacity) || !p.free_count ||
      !p.free_left || !p.workspace || !aligned(p.workspace, 16) || p.page_size < 8 || p.page_size > PREBA_PAGES_MAX_PAGE ||
      (p.page_size & (p.page_size - 1)) || static_cast<uint64_t>(p.pages) * p.page_size > INT32_MAX ||
      static_cast<uint64_t>(p.table_width) * p.page_size > INT32_MAX || p.table_stride < p.table_width ||
      p.table_out_stride < p.table_width || p.table_out == p.table || p.free_left == p.free_count ||
      p.lengths_out == p.lengths || p.free_capacity > INT32_MAX ||
      static_cast<uint64_t>(p.n) * ((p.table_width + kColumns - 1) / kColumns) > INT32_MAX)
    return PREBA_ERR_INVALID_ARG;
  if (p.workspace_bytes < pages_workspace(p.n, p.beams, p.table_width)) return PREBA_ERR_BUFFER_TOO_SMALL;
  pages_args a{};
  a.p = p;
  a.page_shift = 31 - __builtin_clz(p.page_size);
  a.chunks = (p.table_width + kColumns - 1) / kColumns;
  const uint64_t units = static_cast<uint64_t>(p.n) * a.chunks;
  uint8_t* at = static_cast<uint8_t*>(p.workspace);
  auto take = [&](uint64_t bytes) {
    uint8_t* got = at;
    at += up16(bytes);
    return got;
  };
  a.need = reinterpret_cast<int32_t*>(take(4ull * p.n));
  a.copies_before = reinterpret_cast<uint32_t*>(take(4ull * p.n));
  a.counts = reinterpret_cast<uint32_t*>(take(4 * units));
  a.before = reinterpret_cast<int64_t*>(take(8 * units));
  a.given = reinterpret_cast<int32_t*>(take(4ull * p.n * p.beams));
  a.lists = reinterpret_cast<int32_t*>(at);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t err = launch_chained(follow_kernel, static_cast<uint32_t>(units), kColumns,
                                         sizeof(int32_t) * kColumns * p.beams, s, a);
  if (err != cudaSuccess) return finish(err);
  return finish(launch_chained(hand_out_kernel, 1, kHandThreads, 0, s, a));
}

extern "C" int preba_pages_copy(const preba_pages_copy_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_pages_copy_t& p = *req;
  if (!p.copies || !aligned(p.copies, 16) || !p.k_caches || !p.v_caches || p.rows == 0 ||
      p.rows > PREBA_PAGES_MAX_REQUESTS || p.layers == 0 || p.layers > PREBA_COPY_MAX_LAYERS || p.heads_kv == 0 ||
      p.heads_kv > 65535 || p.head_dim < 8 || p.head_dim % 8 || p.head_dim > PREBA_PAGES_MAX_HEAD_DIM ||
      p.page_size < 8 || p.page_size > PREBA_PAGES_MAX_PAGE || (p.page_size & (p.page_size - 1)) ||
      static_cast<uint64_t>(p.pages) * p.page_size > INT32_MAX || (p.dtype != PREBA_F16 && p.dtype != PREBA_BF16))
    return PREBA_ERR_INVALID_ARG;
  for (uint64_t stride : p.cache_stride)
    if (stride % 8 || stride >= (1ull << 38)) return PREBA_ERR_INVALID_ARG;
  copy_args a{};
  a.p = p;
  a.heads_first = p.cache_stride[2] > p.cache_stride[1];
  for (uint32_t l = 0; l < p.layers; ++l) {
    a.caches[2 * l] = p.k_caches[l];
    a.caches[2 * l + 1] = p.v_caches[l];
    if (!a.caches[2 * l] || !aligned(a.caches[2 * l], 16) || !a.caches[2 * l + 1] || !aligned(a.caches[2 * l + 1], 16))
      return PREBA_ERR_INVALID_ARG;
  }
  int sms = 0;
  const int rc = device_sms(&sms);
  if (rc != PREBA_OK) return rc;
  const uint64_t most = 2ull * p.layers * p.rows;
  const uint32_t grid = static_cast<uint32_t>(std::min<uint64_t>(most, 8ull * sms));
  return finish(launch_chained(copy_kernel, grid, kCopyThreads, 0, static_cast<cudaStream_t>(stream), a));
}
