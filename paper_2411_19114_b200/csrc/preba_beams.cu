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
//
// 64 requests of 8 beams, 128000 tokens in bf16: 31 to 32 us a call, of which 20 are the bytes at the measured copy rate; the scan
// takes 26 under the profiler (exponentials 65 % of their rate, issue slots 59 %), the choice 8.5.  4 beams of 32000 tokens: 6.6 to
// 7.0 us, two launches.

constexpr int kSegmentWords = 512;  // of 32 bits
constexpr int kLaneWords = kSegmentWords / 32;
constexpr int kScanThreads = 256, kChooseThreads = 512;
constexpr int kScanBlocks = 4;      // on an SM
constexpr int kChooseWarps = kChooseThreads / 32;

template <typename T> constexpr int kPerWord = 4 / sizeof(T);
template <typename T> constexpr int kSegment = kSegmentWords * kPerWord<T>;  // elements
template <typename T> constexpr int kLane = kLaneWords * kPerWord<T>;        // elements of a lane
constexpr float kFar = 65536.f;      // numbers beyond this have less exact exponents
template <typename T> constexpr uint32_t kNothing = 0xff800000u;             // -inf in every element of a word
template <> constexpr uint32_t kNothing<__half> = 0xfc00fc00u;
template <> constexpr uint32_t kNothing<__nv_bfloat16> = 0xff80ff80u;

struct select_args {
  preba_beam_select_t p;
  uint32_t segments;  // of a row
  float2* parts;      // of every segment: maximum, sum of the exponentials beside it
};

// The place in its segment of a lane's i-th element, ascending in i.  Vectors of 16 bytes (Vec) where every row begins at a
// multiple of 16; else words, lane by lane.  All rows of a call are read alike, so that equal rows have equal sums.
template <typename T, bool Vec> __device__ __forceinline__ uint32_t place(int i) {
  constexpr int per = kPerWord<T>;
  const uint32_t lane = threadIdx.x & 31, w = i / per;
  return (Vec ? w / 4 * 128 + lane * 4 + w % 4 : w * 32 + lane) * per + i % per;
}

template <typename T> __device__ __forceinline__ float element(uint32_t w, int i);
template <> __device__ __forceinline__ float element<float>(uint32_t w, int) { return __uint_as_float(w); }
template <> __device__ __forceinline__ float element<__half>(uint32_t w, int i) {
  const __half2 h = *reinterpret_cast<const __half2*>(&w);
  return i ? __high2float(h) : __low2float(h);
}
template <> __device__ __forceinline__ float element<__nv_bfloat16>(uint32_t w, int i) {
  return __uint_as_float(i ? w & 0xffff0000u : w << 16);
}
// The larger elements of two words; what is not a number is left out.
template <typename T> __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b);
template <> __device__ __forceinline__ uint32_t larger<float>(uint32_t a, uint32_t b) {
  return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
}
template <> __device__ __forceinline__ uint32_t larger<__half>(uint32_t a, uint32_t b) {
  const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}
template <> __device__ __forceinline__ uint32_t larger<__nv_bfloat16>(uint32_t a, uint32_t b) {
  const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&m);
}

// Puts -inf in the place of what is behind the vocabulary (from the `left`-th element on) or not allowed: a lane holds 32 of the
// segment's bits, and the elements of a word, or of a vector, lie in the same ones.
template <typename T, bool Vec>
__device__ __forceinline__ void drop(uint32_t (&w)[kLaneWords], uint32_t left, bool masked, uint32_t bits) {
  constexpr int per = kPerWord<T>;
  if (left >= kSegment<T> && !masked) return;
#pragma unroll
  for (int i = 0; i < kLaneWords; ++i) {
    const uint32_t e = place<T, Vec>(i * per);
    uint32_t keep = ~0u;
    if (masked) keep = __shfl_sync(kFull, bits, e / 32) >> (e % 32);
    if (!(keep & 1) || e >= left) w[i] = per == 1 ? kNothing<T> : (w[i] & 0xffff0000u) | (kNothing<T> & 0xffffu);
    if (per == 2 && (!(keep & 2) || e + 1 >= left)) w[i] = (w[i] & 0xffffu) | (kNothing<T> & 0xffff0000u);
  }
}
// A lane's words of segment s of a row.  fetch() has the loads on the way, finish() makes of them what they stand for.
template <typename T, bool Vec> struct segment_t {
  uint32_t w[kLaneWords], extra, bits;
  bool odd;  // words as they lie in memory, of a row of 16-bit elements that begins in the middle of one

  __device__ __forceinline__ void fetch(const select_args& a, uint32_t row, uint32_t s) {
    const preba_beam_select_t& p = a.p;
    constexpr int per = kPerWord<T>;
    const uint32_t lane = threadIdx.x & 31, first = s * kSegment<T>, left = p.vocab - first;  // left: at least 1
    const T* from = static_cast<const T*>(p.logits) + row * p.row_stride + first;
    const bool middle = !Vec && per == 2 && (reinterpret_cast<uintptr_t>(from) & 2);
    // such a row's first and last words have a neighbour's element in them, or nobody's
    const bool edge = left < kSegment<T> || (middle && (s == 0 || left == kSegment<T>));
    odd = middle && !edge;
    if (edge) {
#pragma unroll
      for (int i = 0; i < kLaneWords; ++i) {
        const uint32_t e = place<T, Vec>(i * per);
        w[i] = 0;
        if (per == 1) {
          if (e < left) w[i] = __ldg(reinterpret_cast<const uint32_t*>(from) + e);
        } else {
          const uint16_t* half = reinterpret_cast<const uint16_t*>(from) + e;
          if (e < left) w[i] = __ldg(half);
          if (e + 1 < left) w[i] |= static_cast<uint32_t>(__ldg(half + 1)) << 16;
        }
      }
    } else if (Vec) {
#pragma unroll
      for (int i = 0; i < kLaneWords; i += 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(from) + 8 * i + lane);
        w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
      }
    } else {
      const uint32_t* words = reinterpret_cast<const uint32_t*>(from - (odd ? 1 : 0));
#pragma unroll
      for (int i = 0; i < kLaneWords; ++i) w[i] = __ldg(words + i * 32 + lane);
      if (odd) extra = __ldg(words + kSegmentWords);
    }
    bits = bits_of(p, row, first);
  }

  // What of a row's bits belongs to a lane in the segment that begins with element `first`.
  static __device__ __forceinline__ uint32_t bits_of(const preba_beam_select_t& p, uint32_t row, uint32_t first) {
    const uint32_t lane = threadIdx.x & 31;
    if (!p.allowed || lane >= kSegment<T> / 32 || first + lane * 32 >= p.vocab) return 0;
    return __ldg(p.allowed + row * p.allowed_stride + first / 32 + lane);
  }

  __device__ __forceinline__ void finish(const select_args& a, uint32_t s) {
    if (odd) {
      // the second half of a word and the first half of the next, which is the next lane's
      const uint32_t lane = threadIdx.x & 31;
      uint32_t next = __shfl_sync(kFull, w[0], (lane + 1) & 31);
#pragma unroll
      for (int i = 0; i < kLaneWords; ++i) {
        const uint32_t after = i + 1 < kLaneWords ? __shfl_sync(kFull, w[i + 1], (lane + 1) & 31) : extra;
        w[i] = __funnelshift_r(w[i], lane == 31 ? after : next, 16);
        next = after;
      }
    }
    drop<T, Vec>(w, a.p.vocab - s * kSegment<T>, a.p.allowed, bits);
  }
};

// The largest number of the warp; what is not a number is left out.
__device__ __forceinline__ float warp_max(float v) {
  float top;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(v));
  return top;
}
template <typename N> __device__ __forceinline__ N warp_sum(N v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
  return v;
}
// Arithmetic on two fp32 numbers at once.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ void apart(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}

// What a word's elements are above a maximum: not above 0, so that its type holds it, rounded where that no longer matters.
template <typename T> __device__ __forceinline__ uint32_t below(uint32_t w, float top) { return __float_as_uint(__uint_as_float(w) - top); }
template <> __device__ __forceinline__ uint32_t below<__half>(uint32_t w, float) { return w; }  // never as large
template <> __device__ __forceinline__ uint32_t below<__nv_bfloat16>(uint32_t w, float top) {
  const __nv_bfloat162 d = __floats2bfloat162_rn(element<__nv_bfloat16>(w, 0) - top, element<__nv_bfloat16>(w, 1) - top);
  return *reinterpret_cast<const uint32_t*>(&d);
}

// Whether a row offers what its logits say: it is there and has not ended.
__device__ __forceinline__ bool row_live(const preba_beam_select_t& p, uint32_t row) {
  return !(p.done && p.done[row]) && p.scores[row] != -INFINITY;
}

// The warps take segments in turn, so that together they read what lies together; the next one is on the way while one is looked
// at.
template <typename T, bool Vec>
__global__ void __launch_bounds__(kScanThreads, kScanBlocks) scan_kernel(const __grid_constant__ select_args a) {
  const preba_beam_select_t& p = a.p;
  const uint32_t rows = p.n * p.beams, warps = gridDim.x * (kScanThreads / 32);
  const uint32_t step_rows = warps / a.segments, step = warps - step_rows * a.segments;
  const uint32_t unit = blockIdx.x * (kScanThreads / 32) + threadIdx.x / 32;
  uint32_t row = unit / a.segments, s = unit - row * a.segments;
  chained_begin();
  segment_t<T, Vec> next;
  if (row < rows) next.fetch(a, row, s);  // the first one before it is known whether it is wanted
  bool live = row < rows && row_live(p, row);
#pragma unroll 1
  while (row < rows) {
    segment_t<T, Vec> seg = next;
    const uint64_t at = static_cast<uint64_t>(row) * a.segments + s;
    const uint32_t here = s;
    const bool wanted = live;
    row += step_rows;
    s += step;
    if (s >= a.segments) s -= a.segments, ++row;
    live = row < rows && row_live(p, row);
    if (live) next.fetch(a, row, s);
    if (!wanted) continue;
    seg.finish(a, here);
    uint32_t most[4] = {seg.w[0], seg.w[1], seg.w[2], seg.w[3]};
#pragma unroll
    for (int i = 4; i < kLaneWords; ++i) most[i % 4] = larger<T>(most[i % 4], seg.w[i]);
    const uint32_t most1 = larger<T>(larger<T>(most[0], most[1]), larger<T>(most[2], most[3]));
    float top = element<T>(most1, 0);
    if (kPerWord<T> == 2) top = fmaxf(top, element<T>(most1, 1));
    top = warp_max(top);
    // Exponents are x log2(e) - top log2(e), rounded once, beside a rounded product with the maximum whose error is the
    // same for all and is taken out of the sum.  Where all is -inf, or not a number, beside 0; where that error would be more
    // than 2^-7, (x - top) log2(e)
    const bool far = fabsf(top) > kFar;
    const float beside = far ? 0.f : top * kLog2e, off = far ? 0.f : fmaf(-top, kLog2e, beside);
    if (far && top > -INFINITY) {
#pragma unroll
      for (int i = 0; i < kLaneWords; ++i) seg.w[i] = below<T>(seg.w[i], top);
    }
    const uint64_t scale = two(kLog2e, kLog2e), less = two(-beside, -beside);
    uint64_t sums[2] = {0, 0};
    constexpr int kStep = 2 / kPerWord<T>;  // words of two elements
#pragma unroll
    for (int i = 0; i < kLaneWords; i += kStep) {
      float z0, z1;
      apart(fma_two(two(element<T>(seg.w[i], 0), element<T>(seg.w[i + kStep - 1], 1)), scale, less), z0, z1);
      sums[i / kStep & 1] = add_two(sums[i / kStep & 1], two(exp2_approx(z0), exp2_approx(z1)));
    }
    float sum0, sum1;
    apart(add_two(sums[0], sums[1]), sum0, sum1);
    const float sum = warp_sum(sum0 + sum1) * exp2_approx(off);
    if ((threadIdx.x & 31) == 0) a.parts[at] = make_float2(top, sum);
  }
}

// Candidates: segments by their maxima, or tokens.  `at` is the segment or the token.
struct candidate_t {
  double rank;
  float x;       // the logit (of a row that is done: 0)
  uint32_t row;  // the beam
  uint32_t at;
};
constexpr uint32_t kCandidateBytes = 8 + 4 + 4 + 4;
constexpr uint32_t kTeam = 8, kGroups = kChooseThreads / kTeam;  // threads in groups of eight
static_assert(kGroups >= PREBA_BEAMS_MAX_WIDTH, "the width-th of them has to exist");

// A list of them in shared memory, member by member: ranks decide, the others are looked at where two are equal.
struct list_t {
  double* rank;
  float* x;
  uint32_t* row;
  uint32_t* at;
  __device__ __forceinline__ list_t(uint8_t* base, uint32_t room)
      : rank(reinterpret_cast<double*>(base)), x(reinterpret_cast<float*>(rank + room)),
        row(reinterpret_cast<uint32_t*>(x + room)), at(row + room) {}
  __device__ __forceinline__ void put(uint32_t i, const candidate_t& c) const { rank[i] = c.rank, x[i] = c.x, row[i] = c.row, at[i] = c.at; }
  __device__ __forceinline__ candidate_t get(uint32_t i) const { return {rank[i], x[i], row[i], at[i]}; }
  __device__ __forceinline__ bool before(uint32_t i, const candidate_t& c) const {
    const double r = rank[i];
    if (r != c.rank) return r > c.rank;
    if (row[i] != c.row) return row[i] < c.row;
    if (x[i] != c.x) return x[i] > c.x;
    return at[i] < c.at;
  }
};

struct choose_shared {
  double lse[PREBA_BEAMS_MAX], score[PREBA_BEAMS_MAX], weight[PREBA_BEAMS_MAX];
  uint32_t live[PREBA_BEAMS_MAX];      // 0: offers nothing, 1: its logits, 2: its end token
  uint32_t segments[PREBA_BEAMS_MAX];  // of the row's that are listed
  uint32_t listed, found;
  double groups[kGroups], floor;       // the best ranks of groups of threads, and the `width`-th of them
  candidate_t best[PREBA_BEAMS_MAX_WIDTH];  // segments
};

// Candidates of a request at most: segments, as many as pass a threshold that is close to the `width`-th, or, where more do,
// `width` of each row; then tokens, where the k-th segment can give no more than width - k.
__host__ __device__ inline uint32_t candidates_of(uint32_t beams, uint32_t width) {
  const uint32_t tokens = width * (width + 1) / 2, rows = beams * width, passed = 16 * width;
  const uint32_t segments = rows > passed ? rows : passed;
  return segments > tokens ? segments : tokens;
}

__device__ __forceinline__ double value_of(const choose_shared& c, uint32_t row, float x) {
  return (static_cast<double>(x) - c.lse[row]) + c.score[row];
}

// The best of the lanes' numbers, and where it is; of equals the lowest place.  False if there is none.
__device__ __forceinline__ bool warp_best(float& x, uint32_t& at) {
  const float top = warp_max(x);
  if (top == -INFINITY) return false;
  at = __reduce_min_sync(kFull, x == top ? at : UINT32_MAX);
  x = top;
  return true;
}

// How many of a list come before one of its entries, by eight threads for each; `take` gets the entry and its place.
template <typename Take> __device__ __forceinline__ void in_order(const list_t& list, uint32_t count, const Take& take) {
  const uint32_t member = threadIdx.x % kTeam;
  for (uint32_t i0 = 0; i0 < count; i0 += kChooseThreads / kTeam) {  // the same for the whole block
    const uint32_t i = i0 + threadIdx.x / kTeam;
    const candidate_t mine = list.get(min(i, count - 1));
    uint32_t ahead = 0;
#pragma unroll 4
    for (uint32_t k = member; k < count; k += kTeam) ahead += list.before(k, mine);
#pragma unroll
    for (uint32_t o = 1; o < kTeam; o *= 2) ahead += __shfl_xor_sync(kFull, ahead, o);
    if (member == 0 && i < count) take(mine, ahead);
  }
}

constexpr uint32_t kHeld = 8;  // segments of a row that a lane keeps; rows of more are read again each time
constexpr uint32_t kItems = 4;  // segments of all rows that a thread keeps, likewise

template <typename T, bool Vec>
__global__ void __launch_bounds__(kChooseThreads) choose_kernel(const __grid_constant__ select_args a) {
  extern __shared__ __align__(16) uint8_t choose_smem[];
  __shared__ choose_shared c;
  const preba_beam_select_t& p = a.p;
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t r = blockIdx.x, row0 = r * p.beams, room = candidates_of(p.beams, p.width);
  const list_t list(choose_smem, room);
  if (threadIdx.x == 0) c.listed = c.found = 0;
  chained_begin();

  // a warp per beam: the logarithm of its sum
  const float2* all_parts = a.parts + static_cast<uint64_t>(row0) * a.segments;
  for (uint32_t b = warp; b < p.beams; b += kChooseWarps) {
    const uint32_t row = row0 + b;
    const float2* parts = all_parts + b * a.segments;
    float2 held[kHeld];
#pragma unroll
    for (uint32_t k = 0; k < kHeld; ++k)  // of a row that is not live they mean nothing
      held[k] = lane + 32 * k < a.segments ? __ldcg(parts + lane + 32 * k) : make_float2(-INFINITY, 0.f);
    const bool done = p.done && p.done[row];
    const float score = p.scores[row], weight = p.weights ? p.weights[row] : 1.f;
    bool good = score < INFINITY && weight > 0.f && weight < INFINITY;
    float top = -INFINITY;
    double lse = 0;
    if (!done && score != -INFINITY) {
#pragma unroll
      for (uint32_t k = 0; k < kHeld; ++k) top = fmaxf(top, held[k].x);
      for (uint32_t s = lane + 32 * kHeld; s < a.segments; s += 32) top = fmaxf(top, __ldcg(parts + s).x);
      top = warp_max(top);
      // a segment of nothing has the sum 0; one of -inf and NaN has a sum that is not a number
      auto beside = [&](float2 v) {
        return static_cast<double>(v.x == -INFINITY ? v.y : v.y * exp2_approx((v.x - top) * kLog2e));
      };
      double sum = 0;
#pragma unroll
      for (uint32_t k = 0; k < kHeld; ++k)
        if (32 * k < a.segments) sum += beside(held[k]);
      for (uint32_t s = lane + 32 * kHeld; s < a.segments; s += 32) sum += beside(__ldcg(parts + s));
      sum = warp_sum(sum);
      lse = top + log(sum);
      good = good && (top == -INFINITY ? sum == 0 : lse < INFINITY);  // not a number: false
    }
    if (lane == 0) {
      if (!good) report(p.status, PREBA_ERR_BAD_TABLE);
      c.live[b] = !good || score == -INFINITY ? 0 : done ? 2 : top > -INFINITY;
      c.lse[b] = lse;
      c.score[b] = score;
      c.weight[b] = weight;
    }
  }
  // the rows' segments, and behind them an end token for each, thread by thread
  const uint32_t segments = p.beams * a.segments, items = segments + p.beams;
  float kept[kItems];
#pragma unroll
  for (uint32_t k = 0; k < kItems; ++k) {
    const uint32_t i = threadIdx.x + k * kChooseThreads;
    kept[k] = i < segments ? __ldcg(&all_parts[i].x) : 0.f;
  }
  __syncthreads();
  auto item = [&](uint32_t i, float x) -> candidate_t {
    const uint32_t b = i < segments ? i / a.segments : i - segments;
    const bool there = i < segments ? c.live[b] == 1 && x > -INFINITY : i < items && c.live[b] == 2;
    if (!there) return {-INFINITY, 0.f, 0, 0};
    if (i >= segments) return {c.weight[b] * c.score[b], 0.f, b, UINT32_MAX};
    return {c.weight[b] * value_of(c, b, x), x, b, i - b * a.segments};
  };
  auto every_item = [&](const auto& take) {
#pragma unroll
    for (uint32_t k = 0; k < kItems; ++k)
      if (k * kChooseThreads < items) take(item(threadIdx.x + k * kChooseThreads, kept[k]));
    for (uint32_t i = threadIdx.x + kItems * kChooseThreads; i < items; i += kChooseThreads)
      take(item(i, i < segments ? __ldcg(&all_parts[i].x) : 0.f));
  };
  // As many groups of threads as are wanted have a candidate of the rank of the `width`-th best group, or a better one: the
  // others need not be looked at
  double best_rank = -INFINITY;
  every_item([&](const candidate_t& x) { best_rank = fmax(best_rank, x.rank); });
#pragma unroll
  for (uint32_t o = 1; o < kTeam; o *= 2) best_rank = fmax(best_rank, __shfl_xor_sync(kFull, best_rank, o));
  if (threadIdx.x % kTeam == 0) c.groups[threadIdx.x / kTeam] = best_rank;
  __syncthreads();
  {
    const uint32_t g = threadIdx.x / kTeam;
    uint32_t ahead = 0;
#pragma unroll
    for (uint32_t k = threadIdx.x % kTeam; k < kGroups; k += kTeam) ahead += c.groups[k] > best_rank || (c.groups[k] == best_rank && k < g);
#pragma unroll
    for (uint32_t o = 1; o < kTeam; o *= 2) ahead += __shfl_xor_sync(kFull, ahead, o);
    if (threadIdx.x % kTeam == 0 && ahead == p.width - 1) c.floor = best_rank;
  }
  __syncthreads();
  const double floor = c.floor;
  every_item([&](const candidate_t& x) {
    if (!(x.rank >= floor) || x.rank == -INFINITY) return;
    const uint32_t at = atomicAdd(&c.listed, 1);
    if (at < room) list.put(at, x);
  });
  __syncthreads();
  uint32_t slots = c.listed;
  if (slots > room) {
    // Too many are equal to it.  A row's segments in order, one by one: what follows the one before
    for (uint32_t b = warp; b < p.beams; b += kChooseWarps) {
      float last_x = INFINITY;
      uint32_t last_s = 0, n = 0;
      for (; n < p.width && c.live[b] == 1; ++n) {
        float x = -INFINITY;
        uint32_t at = UINT32_MAX;
        for (uint32_t s = lane; s < a.segments; s += 32) {
          const float m = __ldcg(&all_parts[b * a.segments + s].x);
          const bool after = m < last_x || (m == last_x && s > last_s);
          if (after && m > x) x = m, at = s;
        }
        if (!warp_best(x, at)) break;
        last_x = x, last_s = at;
        if (lane == 0 && PREBA_IN_RANGE(p.status, b * p.width + n < room))
          list.put(b * p.width + n, {c.weight[b] * value_of(c, b, x), x, b, at});
      }
      if (c.live[b] == 2) {
        if (lane == 0) list.put(b * p.width, {c.weight[b] * c.score[b], 0.f, b, UINT32_MAX});
        n = 1;
      }
      for (uint32_t k = n + lane; k < p.width; k += 32) list.put(b * p.width + k, {-INFINITY, 0.f, UINT32_MAX, b * p.width + k});
    }
    slots = p.beams * p.width;
    __syncthreads();
  }
  in_order(list, slots, [&](const candidate_t& mine, uint32_t ahead) {
    if (ahead < p.width) c.best[ahead] = mine;
  });
  __syncthreads();
  const uint32_t listed = __syncthreads_count(threadIdx.x < min(slots, p.width) && c.best[threadIdx.x].rank > -INFINITY);

  // what the best segments hold, as far as it can be among the first: a warp per segment
  const uint32_t chosen = min(listed, p.width);
  const bool full = chosen == p.width;  // nothing after the last segment's maximum is among the first
  auto add = [&](const candidate_t& x) {  // their order in the list is that of whoever came first and means nothing
    const uint32_t at = atomicAdd(&c.found, 1);
    if (PREBA_IN_RANGE(p.status, at < room)) list.put(at, x);
  };
  for (uint32_t k = warp; k < chosen; k += kChooseWarps) {
    const candidate_t seg = c.best[k];
    if (seg.at == UINT32_MAX) {
      if (lane == 0) add({seg.rank, 0.f, seg.row, static_cast<uint32_t>(p.end_token)});
      continue;
    }
    segment_t<T, Vec> words;
    words.fetch(a, row0 + seg.row, seg.at);
    const double last = c.best[chosen - 1].rank, weight = c.weight[seg.row];
    // the least logit that may do, less what it may be off by; where a weight has no reciprocal, all may
    const double level = last * (1.f / static_cast<float>(weight)), least = level - c.score[seg.row] + c.lse[seg.row];
    const float least_x =
        full && isfinite(level) ? static_cast<float>(least - 1e-6 * (1 + fabs(level) + fabs(c.score[seg.row]) + fabs(c.lse[seg.row]))) : -INFINITY;
    words.finish(a, seg.at);
    uint32_t enough = 0;  // a bit for each of the lane's elements
#pragma unroll
    for (int i = 0; i < kLane<T>; ++i)
      if (element<T>(words.w[i / kPerWord<T>], i % kPerWord<T>) >= least_x) enough |= 1u << i;
    if (__reduce_add_sync(kFull, __popc(enough)) <= p.width - k) {
      // few enough to be listed as they are
      for (; enough; enough &= enough - 1) {
        const int which = __ffs(enough) - 1;
        float x = 0.f;
        uint32_t at = 0;
#pragma unroll
        for (int u = 0; u < kLane<T>; ++u)
          if (u == which) x = element<T>(words.w[u / kPerWord<T>], u % kPerWord<T>), at = place<T, Vec>(u);
        if (x > -INFINITY) add({weight * value_of(c, seg.row, x), x, seg.row, seg.at * kSegment<T> + at});
      }
      continue;
    }
    uint32_t taken = 0;  // a bit for each of the lane's elements
    for (uint32_t j = k; j < p.width; ++j) {
      float best = -INFINITY;
      uint32_t at = UINT32_MAX, which = 0;
#pragma unroll
      for (int i = 0; i < kLane<T>; ++i) {
        const float x = element<T>(words.w[i / kPerWord<T>], i % kPerWord<T>);
        if (x > best && !(taken >> i & 1)) best = x, at = place<T, Vec>(i), which = i;
      }
      const uint32_t own = at;
      if (!warp_best(best, at)) break;
      const double rank = weight * value_of(c, seg.row, best);
      if (full && rank < last) break;
      if (own == at) taken |= 1u << which;
      if (lane == 0) add({rank, best, seg.row, seg.at * kSegment<T> + at});
    }
  }
  __syncthreads();

  const uint32_t found = min(c.found, room);
  const uint64_t out = static_cast<uint64_t>(r) * p.width;
  in_order(list, found, [&](const candidate_t& mine, uint32_t ahead) {
    if (ahead >= p.width) return;
    const bool done = c.live[mine.row] == 2;
    p.tokens[out + ahead] = static_cast<int32_t>(mine.at);
    p.parents[out + ahead] = static_cast<int32_t>(mine.row);
    p.scores_out[out + ahead] = static_cast<float>(done ? c.score[mine.row] : value_of(c, mine.row, mine.x));
    if (p.done_out) p.done_out[out + ahead] = done || static_cast<int32_t>(mine.at) == p.end_token;
  });
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

int device_sms(int* sms) {
  int device = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device);
  return finish(err);
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
  const uint64_t blocks = (static_cast<uint64_t>(p.n) * p.beams * a.segments + kScanThreads / 32 - 1) / (kScanThreads / 32);
  cudaError_t err = launch_chained(scan_kernel<T, Vec>, static_cast<uint32_t>(std::min(blocks, static_cast<uint64_t>(kScanBlocks) * sms)),
                                   kScanThreads, 0, stream, a);
  if (err != cudaSuccess) return err;
  const size_t smem = candidates_of(p.beams, p.width) * kCandidateBytes;
  if (smem > 40 * 1024) {  // beside 3 KB of its own
    err = cudaFuncSetAttribute(choose_kernel<T, Vec>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               static_cast<int>(candidates_of(PREBA_BEAMS_MAX, PREBA_BEAMS_MAX_WIDTH) * kCandidateBytes));
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
// lists what is released.  In a second every block adds all requests' numbers up for itself (they are few and come from
// L2), so that it knows where its own requests' copies and pages stand among all, and hands out without asking another.
// Only then it is known who is refused for want of pages, and a refused row keeps what lies behind its last page: so where the
// stack may not suffice, the first kernel leaves the places of a row behind its own last page to the second (which then takes 0.3
// to 0.5 us more; where a search begins and all rows come from one of 8192 tokens, 10 us more for 128 requests, 3 for 4).
// 128 requests of 8 beams over 8192 tokens: 10.6 to 11.2 us (one block that hands out for all: 35); 2 of 4: 6.5 to 7.0 us, two launches.

constexpr int kColumns = 256;
constexpr int kHandThreads = 256;
constexpr uint32_t kAtOnce = 8;  // beams whose entries of a column are on the way together

struct pages_args {
  preba_beam_pages_t p;
  uint32_t page_shift, chunks;  // chunks of columns of a row
  int32_t* need;      // n: copies of a request, or -1: it is at fault
  uint32_t* counts;   // n * chunks: pages released
  int32_t* lists;     // n * chunks lists of kColumns * beams pages
};

__device__ __forceinline__ uint32_t held_pages(const pages_args& a, int32_t length) {
  return (static_cast<uint32_t>(length) + (1u << a.page_shift) - 1) >> a.page_shift;
}

// Pages on the stack, or -1 where that cannot be: what lies there is then not known, and no request is served.
__device__ __forceinline__ int64_t on_stack(const preba_beam_pages_t& p) {
  const int64_t count = *p.free_count;
  return count < 0 || count > p.free_capacity ? -1 : count;
}
// Whether the stack alone has a page for every row that can need one: then nobody is refused for want of pages.
__device__ __forceinline__ bool plenty(const preba_beam_pages_t& p, int64_t count) {
  return count >= static_cast<int64_t>(p.n) * (p.beams - 1);
}

// Few: at most kAtOnce beams, whose entries of a column a thread then keeps in registers; else they lie in shared memory.
template <bool Few> __global__ void __launch_bounds__(kColumns) follow_kernel(const __grid_constant__ pages_args a) {
  extern __shared__ int32_t tile[];  // beams x kColumns
  __shared__ __align__(16) int32_t parent[PREBA_BEAMS_MAX], length[PREBA_BEAMS_MAX];
  __shared__ __align__(16) uint32_t held[PREBA_BEAMS_MAX];
  __shared__ uint32_t warp_sums[kColumns / 32], parents_of;
  const preba_beam_pages_t& p = a.p;
  const uint32_t r = blockIdx.x / a.chunks, chunk = blockIdx.x - r * a.chunks, row0 = r * p.beams;
  const uint32_t c = chunk * kColumns + threadIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  chained_begin();
  const int64_t kept = p.kept ? p.kept[r] : 0;
  const bool sure = plenty(p, on_stack(p));
  bool bad = false;
  if (warp == 0) {
    uint32_t child_of = 0;
    parent[lane] = -1, held[lane] = 0;
    if (lane < static_cast<int>(p.beams)) {
      const int32_t len = p.lengths[row0 + lane], par = p.parents[row0 + lane];
      const uint32_t h = len < 0 ? 0 : held_pages(a, len);
      bad = len < 0 || h > p.table_width || par >= static_cast<int32_t>(p.beams);
      parent[lane] = par < 0 ? -1 : par;
      length[lane] = len;
      held[lane] = min(h, p.table_width);
      if (par >= 0 && !bad) child_of = 1u << par;
    }
    child_of = __reduce_or_sync(kFull, child_of);
    if (lane == 0) parents_of = child_of;
  }
  const bool refused = __syncthreads_or(bad);
  const uint32_t parents = refused ? 0 : parents_of;  // a bit per beam that has a child
  // the page that a row's copy comes from is looked up beside the columns
  int32_t source = 0;
  if (chunk == 0 && warp == 0 && lane < static_cast<int>(p.beams) && !refused && parent[lane] >= 0 && held[parent[lane]])
    source = p.table[(row0 + parent[lane]) * p.table_stride + held[parent[lane]] - 1];
  // every thread has a column, and reads no other's
  int32_t page[kAtOnce];
  uint32_t have = 0;  // beams with a page here, of the first kAtOnce
  auto follow = [&](uint32_t i) {
    const int32_t from = refused ? static_cast<int32_t>(i) : parent[i];
    if (from >= 0 && c < held[from] && (sure || c < held[i])) p.table_out[(row0 + i) * p.table_out_stride + c] = tile[from * kColumns + threadIdx.x];
  };
  if (Few) {
    const int32_t* from = p.table + row0 * p.table_stride + c;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k) have |= (c < held[k] ? 1u : 0u) << k;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k, from += p.table_stride) page[k] = have >> k & 1 ? *from : 0;
#pragma unroll
    for (uint32_t k = 0; k < kAtOnce; ++k)
      if (have >> k & 1) tile[k * kColumns + threadIdx.x] = page[k];
#pragma unroll
    for (uint32_t i = 0; i < kAtOnce; ++i)
      if (i < p.beams) follow(i);
  } else {
    for (uint32_t b0 = 0; b0 < p.beams; b0 += kAtOnce) {
#pragma unroll
      for (uint32_t k = 0; k < kAtOnce; ++k)
        page[k] = b0 + k < p.beams && c < held[b0 + k] ? p.table[(row0 + b0 + k) * p.table_stride + c] : 0;
#pragma unroll
      for (uint32_t k = 0; k < kAtOnce; ++k)
        if (b0 + k < p.beams) tile[(b0 + k) * kColumns + threadIdx.x] = page[k];
    }
    for (uint32_t i = 0; i < p.beams; ++i) follow(i);
  }
  // what this column releases, a bit per beam
  uint32_t gone = 0;
  if (!refused && c >= kept) {
    if (Few) {
      gone = have & ~parents;
      if (gone) {
#pragma unroll
        for (uint32_t b = 0; b < kAtOnce; ++b) {
          uint32_t same = 0;
#pragma unroll
          for (uint32_t o = 0; o < kAtOnce; ++o)
            if (o != b) same |= (page[o] == page[b] ? 1u : 0u) << o;
          if (same & have & (parents | ((1u << b) - 1))) gone &= ~(1u << b);
        }
      }
    } else {
      for (uint32_t b = 0; b < p.beams; ++b) {
        if (parents >> b & 1 || c >= held[b]) continue;
        const int32_t mine = tile[b * kColumns + threadIdx.x];
        bool alone = true;
        for (uint32_t o = 0; o < p.beams; ++o)
          if ((parents >> o & 1 || o < b) && c < held[o] && tile[o * kColumns + threadIdx.x] == mine) alone = false;
        if (alone) gone |= 1u << b;
      }
    }
    for (uint32_t left = gone; left; left &= left - 1) {
      const int b = __ffs(left) - 1;
      const int32_t number = tile[b * kColumns + threadIdx.x];
      if (number >= 0 && static_cast<uint32_t>(number) < p.pages) continue;
      report(p.status, PREBA_ERR_BAD_TABLE);
      gone &= ~(1u << b);
    }
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
#pragma unroll
  for (int w = 0; w < kColumns / 32; ++w) {
    if (w < warp) at += warp_sums[w];
    total += warp_sums[w];
  }
  int32_t* to = a.lists + static_cast<uint64_t>(blockIdx.x) * kColumns * p.beams;
  for (; gone; gone &= gone - 1)
    if (PREBA_IN_RANGE(p.status, at < kColumns * p.beams)) to[at++] = tile[(__ffs(gone) - 1) * kColumns + threadIdx.x];
  if (threadIdx.x == 0) a.counts[blockIdx.x] = total;

  if (chunk || warp) return;
  // lengths, and which children need an open page: a row's number among those of its request in place of the page
  bool needs = false;
  int4 copy = make_int4(0, 0, 0, 0);
  if (lane < static_cast<int>(p.beams)) {
    const int32_t from = parent[lane];
    const bool there = !refused && from >= 0;
    const uint32_t open = there ? length[from] & ((1u << a.page_shift) - 1) : 0;
    p.lengths_out[row0 + lane] = there ? length[from] : 0;
    bool first = true;
    for (int i = 0; i < lane; ++i) first = first && parent[i] != from;
    needs = there && open && !first;
    if (needs) copy = make_int4(source, 0, open, 0);
  }
  const uint32_t copied = __ballot_sync(kFull, needs);
  copy.y = needs ? __popc(copied & ((1u << lane) - 1)) : 0;
  if (lane < static_cast<int>(p.beams)) reinterpret_cast<int4*>(p.copies)[row0 + lane] = copy;
  if (lane == 0) {
    a.need[r] = refused ? -1 : __popc(copied);
    if (refused) report(p.status, PREBA_ERR_BAD_TABLE);
  }
}

struct both_t {
  int64_t copies, released;
};
struct sums_t {  // 32 bits do: the table has no more entries
  uint32_t copies, released;
};
constexpr uint32_t kHandBytes = sizeof(sums_t) + 1;  // shared, of a request
__device__ __forceinline__ both_t hand_exclusive(both_t v, both_t* warp_sums, both_t& total) {
  constexpr int kWarps = kHandThreads / 32;
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
  total = {0, 0};
  both_t before = {incl.copies - v.copies, incl.released - v.released};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const both_t of = warp_sums[w];
    total.copies += of.copies, total.released += of.released;
    if (w < warp) before.copies += of.copies, before.released += of.released;
  }
  return before;
}

__global__ void __launch_bounds__(kHandThreads) hand_out_kernel(const __grid_constant__ pages_args a) {
  extern __shared__ __align__(16) uint8_t hand_smem[];
  const preba_beam_pages_t& p = a.p;
  sums_t* sums = reinterpret_cast<sums_t*>(hand_smem);  // n: copies and pages, then those of the requests before
  uint8_t* served = hand_smem + p.n * sizeof(sums_t);    // n
  __shared__ both_t warp_sums[kHandThreads / 32];
  chained_begin();
  int64_t count = on_stack(p);
  const bool stack = count >= 0;
  if (!stack) {
    if (blockIdx.x == 0 && threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
    count = 0;
  }
  // what every request asks for and releases
  for (uint32_t r = threadIdx.x; r < p.n; r += kHandThreads) {
    const int32_t need = a.need[r];
    uint32_t released = 0;
#pragma unroll 4
    for (uint32_t k = 0; k < a.chunks; ++k) released += a.counts[r * a.chunks + k];
    served[r] = need >= 0 && stack;
    sums[r] = {static_cast<uint32_t>(max(need, 0)), released};  // one at fault releases nothing
  }
  __syncthreads();
  const uint32_t per = (p.n + kHandThreads - 1) / kHandThreads;
  const uint32_t r0 = min(threadIdx.x * per, p.n), r1 = min(r0 + per, p.n);
  both_t total;
  for (int round = 0;; ++round) {
    both_t mine{0, 0};
    for (uint32_t r = r0; r < r1; ++r)
      if (served[r]) mine.copies += sums[r].copies, mine.released += sums[r].released;
    const both_t before = hand_exclusive(mine, warp_sums, total);
    both_t at = before;
    bool short_of = false;
    for (uint32_t r = r0; r < r1; ++r) {
      if (!served[r]) continue;
      at.copies += sums[r].copies, at.released += sums[r].released;
      short_of |= count + at.released < at.copies;
    }
    if (!__syncthreads_or(short_of)) {
      at = before;
      for (uint32_t r = r0; r < r1; ++r) {
        const sums_t here = sums[r];
        sums[r] = {static_cast<uint32_t>(at.copies), static_cast<uint32_t>(at.released)};
        if (served[r]) at.copies += here.copies, at.released += here.released;
      }
      break;
    }
    // The pages do not suffice for all: one by one, in order.  The next round finds that they suffice
    if (threadIdx.x == 0) {
      int64_t left = count;
      for (uint32_t r = 0; r < p.n; ++r) {
        if (!served[r]) continue;
        const int64_t then = left + sums[r].released - static_cast<int64_t>(sums[r].copies);
        if (then < 0) {
          served[r] = 2;  // for a moment: refused
          if (blockIdx.x == 0) report(p.status, PREBA_ERR_BUFFER_TOO_SMALL);
        } else {
          left = then;
        }
      }
    }
    __syncthreads();
    for (uint32_t r = threadIdx.x; r < p.n; r += kHandThreads)
      if (served[r] == 2) served[r] = 0;
    __syncthreads();
  }
  __syncthreads();

  // this block's requests
  const uint32_t each = (p.n + gridDim.x - 1) / gridDim.x;
  const uint32_t b0 = min(blockIdx.x * each, p.n), b1 = min(b0 + each, p.n);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr int kCopyWarps = 2;
  if (warp < kCopyWarps) {
    // copies: a thread per row.  The k-th takes the k-th of the released pages, or one from the stack
    for (uint32_t i = b0 * p.beams + threadIdx.x; i < b1 * p.beams; i += 32 * kCopyWarps) {
      int4 copy = reinterpret_cast<const int4*>(p.copies)[i];
      const int32_t length = p.lengths_out[i];
      if (copy.z == 0) continue;
      const uint32_t r = i / p.beams;
      if (!served[r]) {
        reinterpret_cast<int4*>(p.copies)[i] = make_int4(0, 0, 0, 0);
        continue;
      }
      int64_t k = static_cast<int64_t>(sums[r].copies) + copy.y;
      if (k < total.released) {
        uint32_t lo = 0, hi = p.n;  // the last request with no more released before it than k
        while (hi - lo > 1) {
          const uint32_t mid = (lo + hi) / 2;
          if (sums[mid].released <= k) lo = mid; else hi = mid;
        }
        k -= sums[lo].released;
        uint32_t unit = lo * a.chunks;
        for (const uint32_t last = unit + a.chunks - 1; unit < last; ++unit) {
          const uint32_t pages = a.counts[unit];
          if (k < pages) break;
          k -= pages;
        }
        copy.y = PREBA_IN_RANGE(p.status, k < kColumns * p.beams) ? a.lists[static_cast<uint64_t>(unit) * kColumns * p.beams + k] : -1;
      } else {
        copy.y = p.free_pages[count - 1 - (k - total.released)];
      }
      const uint32_t last = held_pages(a, length) - 1;
      if (PREBA_IN_RANGE(p.status, last < p.table_width)) p.table_out[i * p.table_out_stride + last] = copy.y;
      if (copy.y < 0 || static_cast<uint32_t>(copy.y) >= p.pages) {
        report(p.status, PREBA_ERR_BAD_TABLE);
        copy = make_int4(0, 0, 0, 0);
      }
      reinterpret_cast<int4*>(p.copies)[i] = copy;
    }
  } else {
    // What is released and not given to a copy goes onto the stack: a warp per request, or all of these where there is one
    const uint32_t threads = kHandThreads - 32 * kCopyWarps, team = each == 1 ? threads : 32;
    const uint32_t place = threadIdx.x - 32 * kCopyWarps, member = place % team;
    for (uint32_t r = b0 + place / team; r < b1; r += threads / team) {
      if (!served[r]) continue;
      int64_t first = static_cast<int64_t>(sums[r].released) - total.copies;  // its place above the old top
      for (uint32_t k = 0; k < a.chunks; ++k) {
        const uint32_t unit = r * a.chunks + k, pages = a.counts[unit];
        const int32_t* from = a.lists + static_cast<uint64_t>(unit) * kColumns * p.beams;
#pragma unroll 4
        for (uint32_t i = member; i < pages; i += team) {
          if (first + i < 0) continue;
          if (count + first + i < p.free_capacity) p.free_pages[count + first + i] = from[i];
          else report(p.status, PREBA_ERR_BAD_TABLE);
        }
        first += pages;
      }
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0)
    *p.free_left = static_cast<int32_t>(min(count + total.released - total.copies, static_cast<int64_t>(p.free_capacity)));
  if (stack && plenty(p, count)) return;
  // rows of requests that were refused for want of pages, or of a stack, as they were; of the others, what was left to this kernel
  for (uint32_t i = b0 * p.beams + warp; i < b1 * p.beams; i += kHandThreads / 32) {
    const uint32_t r = i / p.beams, row0 = r * p.beams;
    if (a.need[r] < 0) continue;
    const uint32_t own = held_pages(a, p.lengths[i]);
    uint32_t from = i, first = 0, last = own;
    if (served[r]) {
      const int32_t parent = p.parents[i];
      if (parent < 0) continue;
      from = row0 + parent;
      const int32_t length = p.lengths[from];
      first = own, last = held_pages(a, length);
      // the last page of all children but the first is another one, and written above
      const bool before = lane < static_cast<int>(i - row0);
      const bool again = __any_sync(kFull, before && p.parents[row0 + lane] == parent);
      if (again && (length & ((1u << a.page_shift) - 1))) --last;
    } else if (lane == 0) {
      p.lengths_out[i] = 0;
    }
    for (uint32_t c = first + lane; c < last; c += 32) p.table_out[i * p.table_out_stride + c] = p.table[from * p.table_stride + c];
  }
}

uint64_t up16(uint64_t v) { return (v + 15) / 16 * 16; }

bool beam_sizes_ok(uint32_t n, uint32_t beams, uint32_t table_width) {
  return n >= 1 && beams >= 1 && beams <= PREBA_BEAMS_MAX && static_cast<uint64_t>(n) * beams <= PREBA_PAGES_MAX_REQUESTS &&
         table_width >= 1 && table_width <= INT32_MAX / 8 && static_cast<uint64_t>(n) * beams * table_width <= UINT32_MAX;
}
uint64_t pages_workspace(uint32_t n, uint32_t beams, uint32_t table_width) {
  const uint64_t units = static_cast<uint64_t>(n) * ((table_width + kColumns - 1) / kColumns);
  return up16(4ull * n) + up16(4 * units) + 4 * units * kColumns * beams;
}

// ---- preba_pages_copy -------------------------------------------------------------------------------
//
// Bytes bound it: what is copied, in and out once.  The rows that have a copy are found by every block for itself, a
// job is a row's page in one cache, keys or values, and blocks take jobs in turn.  64 requests of 8 beams, 12 layers, 304 MB in
// and out: 49 to 52 us, 90 to 94 % of the measured copy rate; 4 requests of 4 beams: 3.0 to 3.6 us, a launch.

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
  __shared__ uint32_t warp_jobs[kCopyThreads / 32];
  const preba_pages_copy_t& p = a.p;
  chained_begin();
  const uint32_t vectors = p.head_dim / 8;
  uint32_t turn = blockIdx.x;  // the block's next job, among all of them
  for (uint32_t row0 = 0; row0 < p.rows; row0 += kCopyRows) {
    // in the order of the rows, for all blocks alike: four rows of a thread, 32 apart, 128 of a warp
    constexpr int kEach = kCopyRows / kCopyThreads;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int4 c[kEach];
    uint32_t masks[kEach], found = 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const uint32_t i = row0 + warp * 32 * kEach + 32 * k + lane;
      c[k] = i < p.rows ? __ldg(reinterpret_cast<const int4*>(p.copies) + i) : make_int4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      const bool good = c[k].x >= 0 && static_cast<uint32_t>(c[k].x) < p.pages && c[k].y >= 0 &&
                        static_cast<uint32_t>(c[k].y) < p.pages && c[k].z > 0 && static_cast<uint32_t>(c[k].z) <= p.page_size;
      if (c[k].z != 0 && !good && blockIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
      masks[k] = __ballot_sync(kFull, good);
      found += __popc(masks[k]);
    }
    __syncthreads();  // the jobs before have been read
    if (lane == 0) warp_jobs[warp] = found;
    __syncthreads();
    uint32_t at = 0, n_jobs = 0;
#pragma unroll
    for (int w = 0; w < kCopyThreads / 32; ++w) {
      if (w < static_cast<int>(warp)) at += warp_jobs[w];
      n_jobs += warp_jobs[w];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (masks[k] >> lane & 1) jobs[at + __popc(masks[k] & ((1u << lane) - 1))] = c[k];
      at += __popc(masks[k]);
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
  const select_args a{p, segments_of(p.vocab, p.dtype), static_cast<float2*>(p.workspace)};
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool vec = aligned(p.logits, 16) && (rows == 1 || p.row_stride * wide % 16 == 0);
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
  int sms = 0;
  const int rc = device_sms(&sms);
  if (rc != PREBA_OK) return rc;
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
  a.counts = reinterpret_cast<uint32_t*>(take(4 * units));
  a.lists = reinterpret_cast<int32_t*>(at);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  cudaError_t err = launch_chained(p.beams <= kAtOnce ? follow_kernel<true> : follow_kernel<false>, static_cast<uint32_t>(units),
                                   kColumns, sizeof(int32_t) * kColumns * p.beams, s, a);
  if (err != cudaSuccess) return finish(err);
  const size_t smem = static_cast<size_t>(p.n) * kHandBytes;
  if (smem > 40 * 1024)  // 48 KB need no leave
    err = cudaFuncSetAttribute(hand_out_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, PREBA_PAGES_MAX_REQUESTS * kHandBytes);
  if (err != cudaSuccess) return finish(err);
  return finish(launch_chained(hand_out_kernel, std::min<uint32_t>(p.n, sms), kHandThreads, smem, s, a));
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
