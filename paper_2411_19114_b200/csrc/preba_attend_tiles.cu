// Attention of many rows over the paged cache on the 5th-generation tensor cores: the second kernel
// of preba_pages_attend (the first, for few rows, is in preba_attend.cu).
//
// Rows are (token, query head) pairs of one key head: all heads of a group share the keys, so a tile of
// 128 rows holds floor(128 / group) tokens.  A CTA works on two such tiles, A and B, and streams the
// keys and values they see through a ring of 128-key slots:
//   S = Q K^T  (tcgen05, both operands in shared memory, S in tensor memory)
//   P = exp2(scale log2(e) S - m), written over S in the 16-bit type, row sums in fp32 registers
//   O += P V   (tcgen05, P from tensor memory, V from shared memory as it lies: rows are keys)
// Two groups of four warps, a thread per row, do the exponentials of A and B while the tensor cores work
// on the other tile.  The accumulator O stays in tensor memory; it is multiplied only when a row's
// maximum has grown by more than 2^8 since the last time (until then P is at most 2^8 and the sums
// simply carry the old reference; the result is the same quotient).
//
// The work is a list of (request, pair of tiles, key head) with their numbers of key tiles.  If the
// longest is short beside a CTA's share, CTAs claim them one by one, longest first.  Otherwise the
// key tiles of all of them form one line, every CTA takes an equal run of it, and pieces that are not
// whole leave partial sums which a last kernel joins in the order of the keys.  Which, and the list, is
// decided on the device, as the lengths are there: by a planning kernel, or, where there are too few pairs
// to be claimed, by every CTA for its own run.
//
// P is rounded to 16 bits because the matrix instructions take it so; its row sums are not.  With the one
// rounding of the result the error against 64 bits is 1.3 to 1.4 times that of the one rounding alone.
//
// Bound by the chain of a row tile, not by a unit: a pair of row tiles and 128 keys takes 2048 clocks of the
// tensor pipe and 2048 of MUFU and 3050 altogether, because a tile's softmax (1845 clocks of its threads), the
// second half of P V (256), Q K^T of the next keys (512) and the hand-overs between them follow one another; the
// softmax of both tiles without products takes 2480.  4 prompts of up to 4096 tokens, 32 query heads of 128:
// 325 us at the full clock, 372 to 381 at the 1.57 GHz that the GPU holds under it (1.20 and 1.03 PFLOP/s);
// 512 tokens over 30000 keys: 211 us, and 245 to 250 at 1.47 GHz; a step of 9 chunks and 28 single tokens with
// a window of 1000: 40 to 42 us.
#include <algorithm>

#include <type_traits>

#include "preba_attend.h"
#include "preba_attend_plan.h"

namespace preba {
namespace {

using namespace attend;

constexpr int kTile = kTileRows;       // rows of a tile, keys of a slot
constexpr int kSoftWarps = 8;          // four per tile
constexpr int kCopyWarp = 8, kMmaWarp = 9;
constexpr int kThreads = 32 * 12;       // the last two warps only complete the third warpgroup
// Registers: launched with 168 a thread, 64512 in all; the softmax threads hold a row of S each.
constexpr int kSoftRegisters = 208, kOtherRegisters = 88;
static_assert(256 * kSoftRegisters + 128 * kOtherRegisters <= 168 * kThreads, "register split");
constexpr uint32_t kTmemColumns = 512;
constexpr float kGrowth = 8.f;         // log2 of what a row may outgrow its reference by

template <int DP> struct layout {      // DP: head_dim rounded up to 64 or 128
  static constexpr int kHalves = DP / 64;
  static constexpr uint32_t kHalf = kTile * 128;            // 64 elements of 128 rows
  static constexpr uint32_t kQ = kHalves * kHalf;           // a tile of queries
  static constexpr uint32_t kSlot = kHalves * kHalf;        // a tile of keys, or of values
  static constexpr int kSlots = DP == 128 ? 5 : 10;
  static constexpr uint32_t kRing = 2 * kQ;
  static constexpr uint32_t kBars = kRing + kSlots * kSlot;
  static constexpr uint32_t kItems = kBars + 512;
  static constexpr uint32_t kPlan = kItems + 256;      // own_plan_t
  static constexpr uint32_t kBytes = kPlan + 2048;
  // tensor memory columns: S of A and B (P lies over them), O of A and B
  static constexpr uint32_t kS = 0, kO = 256;
};

// Partial sums of a piece in groups of four floats: 256 rows of O, then a maximum and a sum for each.
template <int DP> constexpr uint32_t kPartial = 2 * kTile * DP / 4 + kTile;

// A piece of work: key tiles [tile, tile + count) of a pair of row tiles on one key head.
struct item_t {
  int32_t count;                 // 0: no more
  uint32_t request, head;
  int32_t row, rows, keys;       // the request: first row, rows, keys
  int32_t token;                 // first token of tile A within the request
  int32_t lo, hi;                // keys that any row of the pair sees
  int32_t tile;
  int32_t first[2], last[2];     // key tiles of A and B within the piece: [first, last)
  int32_t whole;                 // the piece is all of the pair's keys
  uint32_t slot;                 // else: where its partial sums go
};
static_assert(2 * sizeof(item_t) <= 256, "layout::kBytes");

// What the planning kernel leaves for the CTAs.
struct tiles_head {
  uint32_t next;      // claims
  uint32_t n_pairs, units, claim, per;
};

// Two row tiles of a request.
struct pair_t {
  uint32_t request, pair;   // and which pair of it
  uint32_t before, tiles;   // key tiles of the pairs before, key tiles
  int32_t row, rows, keys;  // the request
  uint32_t reserved;
};
static_assert(sizeof(pair_t) == 32, "two vector loads");

// Where a CTA's run of the line begins, and what that beginning cuts in two.
struct run_t {
  pair_t pair;            // the pair of the run's first key tile
  uint32_t which, head;   // its number, and the key head
  uint32_t first, last;   // the CTAs with pieces of it, if this is the first run that begins inside it;
                          // else the same twice
};
static_assert(sizeof(run_t) == 48, "three vector loads");

struct tiles_args {
  preba_pages_attend_t p;
  uint32_t page_shift, group, tokens_per_tile, box_rows, box_shift, grid, max_pairs;
  uint32_t own_plan;  // every CTA makes the plan for itself: it is small and sure to be a line
  tiles_head* head;
  pair_t* pairs;
  run_t* runs;        // one per CTA
  uint32_t* order;    // pairs, longest first
  float4* partials;   // two per CTA
#if defined(PREBA_CHECKED)
  wait_limits_t limits = wait_limits();
#endif
};

struct pair_range {
  int32_t lo, hi;                // keys
  int32_t first[2], last[2];     // key tiles of A and B
  int32_t begin, end;            // of both
};
__device__ __forceinline__ pair_range range_of(const tiles_args& a, const request_t& q, uint32_t pair) {
  pair_range r;
  r.lo = r.hi = 0;
  r.begin = r.end = 0;
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int32_t j0 = (2 * pair + x) * a.tokens_per_tile;
    const int32_t j1 = min(j0 + static_cast<int32_t>(a.tokens_per_tile), q.rows);
    r.first[x] = r.last[x] = 0;
    if (j0 >= j1) continue;  // only B
    int32_t lo, hi;
    seen_by(a.p, q, j0, j1, lo, hi);
    lo = min(lo, max(0, q.keys - 1));  // rows behind all keys see nothing: one empty tile
    r.first[x] = lo / kTile;
    r.last[x] = max(r.first[x] + 1, (hi + kTile - 1) / kTile);
    if (x == 0 || lo < r.lo) r.lo = lo;
    r.hi = max(r.hi, hi);
    if (x == 0 || r.first[x] < r.begin) r.begin = r.first[x];
    r.end = max(r.end, r.last[x]);
  }
  return r;
}

// ---- the plan -------------------------------------------------------------------------------------

constexpr int kPlanThreads = 1024;
constexpr int kBins = 1024;

// In 64 bits: 2^30 pairs of up to 2^24 key tiles are possible.
__device__ __forceinline__ uint64_t block_exclusive(uint64_t v, uint64_t* warp_sums, uint64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint64_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t up = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  const uint64_t s = warp_sums[lane];
  uint64_t up_to = s;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t up = __shfl_up_sync(kFull, up_to, o);
    if (lane >= o) up_to += up;
  }
  total = __shfl_sync(kFull, up_to, 31);
  const uint64_t before = __shfl_sync(kFull, up_to - s, warp);
  __syncthreads();
  return before + incl - v;
}

__global__ void __launch_bounds__(kPlanThreads) tiles_plan_kernel(const tiles_args a) {
  extern __shared__ __align__(16) uint8_t plan_smem[];
  pair_t* near = reinterpret_cast<pair_t*>(plan_smem);  // the first kPlanThreads pairs
  uint32_t* pairs_before = reinterpret_cast<uint32_t*>(near + kPlanThreads);  // n + 1: pairs of the requests before
  __shared__ uint64_t warp_sums[32];
  __shared__ uint32_t bins[kBins], longest;
  const preba_pages_attend_t& p = a.p;
  if (threadIdx.x == 0) longest = 0;
  for (uint32_t b = threadIdx.x; b < kBins; b += kPlanThreads) bins[b] = 0;
  chained_begin();

  const uint32_t each = (p.n + kPlanThreads - 1) / kPlanThreads;
  const uint32_t r0 = min(threadIdx.x * each, p.n), r1 = min(r0 + each, p.n);
  auto pairs_of = [&](uint32_t r) -> uint32_t {
    request_t q;
    if (!load_request(p, r, q)) {
      report(p.status, PREBA_ERR_BAD_TABLE);
      return 0;
    }
    return (q.rows + 2 * a.tokens_per_tile - 1) / (2 * a.tokens_per_tile);
  };
  uint64_t mine = 0, all_pairs;
  for (uint32_t r = r0; r < r1; ++r) mine += pairs_of(r);
  uint64_t at = block_exclusive(mine, warp_sums, all_pairs);
  // rows of different requests do not overlap in a valid step; if they do, the list ends early
  const uint64_t listed = min(all_pairs, static_cast<uint64_t>(a.max_pairs));
  const uint32_t n_pairs = static_cast<uint32_t>(listed);
  if (all_pairs > listed && threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
  for (uint32_t r = r0; r < r1; ++r) {
    pairs_before[r] = static_cast<uint32_t>(min(at, listed));
    at += pairs_of(r);
  }
  if (threadIdx.x == 0) pairs_before[p.n] = n_pairs;
  __syncthreads();
  uint64_t total = 0;
  for (uint32_t base = 0; base < n_pairs; base += kPlanThreads) {
    const uint32_t i = base + threadIdx.x;
    uint32_t tiles = 0, r = 0;
    request_t q;
    if (i < n_pairs) {
      uint32_t lo = 0, hi = p.n;  // the last request with no more pairs before it than i
      while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (pairs_before[mid] <= i) lo = mid; else hi = mid;
      }
      r = lo;
      load_request(p, r, q);
      const pair_range range = range_of(a, q, i - pairs_before[r]);
      tiles = range.end - range.begin;
    }
    uint64_t sum;
    const uint64_t before = total + block_exclusive(tiles, warp_sums, sum);
    if (i < n_pairs) {  // `before` means something in a line only, where it is below 2^31
      const pair_t pair{r, i - pairs_before[r], static_cast<uint32_t>(before), tiles, q.row, q.rows, q.keys, 0};
      a.pairs[i] = pair;
      if (i < kPlanThreads) near[i] = pair;
      atomicMax(&longest, tiles);
    }
    total += sum;
  }
  __syncthreads();
  const share_t share = share_out(total, p.heads_kv, longest, a.grid);
  const uint32_t per = share.per;
  for (uint32_t c = threadIdx.x; c < a.grid; c += kPlanThreads) a.runs[c].first = a.runs[c].last = 0;
  __syncthreads();
  if (!share.claim) {
    // a pair writes down the runs that begin in it, with as many threads as there are for each
    uint32_t lanes = 32;
    while (lanes > 1 && n_pairs * lanes > kPlanThreads) lanes /= 2;
    for (uint32_t i = threadIdx.x / lanes; i < n_pairs; i += kPlanThreads / lanes) {
      const pair_t pair = i < kPlanThreads ? near[i] : a.pairs[i];
      const uint32_t from = pair.before * p.heads_kv, to = from + pair.tiles * p.heads_kv;
      for (uint32_t c = (from + per - 1) / per + threadIdx.x % lanes; c < a.grid && c * per < to; c += lanes) {
        const uint32_t head = (c * per - from) / pair.tiles, start = from + head * pair.tiles;
        const bool cuts = c * per > start && (c - 1) * per <= start;
        a.runs[c] = {pair, i, head, cuts ? c - 1 : 0, cuts ? (start + pair.tiles - 1) / per : 0};
      }
    }
  } else {
    const uint32_t top = max(longest, 1u);
    auto bin_of = [&](uint32_t tiles) {  // longest first
      return kBins - 1 - static_cast<uint32_t>(static_cast<uint64_t>(tiles) * (kBins - 1) / top);
    };
    for (uint32_t i = threadIdx.x; i < n_pairs; i += kPlanThreads) atomicAdd(&bins[bin_of(i < kPlanThreads ? near[i].tiles : a.pairs[i].tiles)], 1);
    __syncthreads();
    uint64_t sum;
    const uint64_t before = block_exclusive(bins[threadIdx.x], warp_sums, sum);
    bins[threadIdx.x] = static_cast<uint32_t>(before);
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n_pairs; i += kPlanThreads)
      a.order[atomicAdd(&bins[bin_of(i < kPlanThreads ? near[i].tiles : a.pairs[i].tiles)], 1)] = i;
  }
  if (threadIdx.x == 0) {
    tiles_head h;
    h.next = 0;
    h.n_pairs = n_pairs;
    h.units = share.units;
    h.claim = share.claim;
    h.per = per;
    *a.head = h;
  }
}
static_assert(kBins == kPlanThreads, "one bin per thread in the sum");

// The same by a CTA of the kernel itself, for itself: where there are few pairs, all of them are certain to
// form one line, and a CTA needs its own run of it only.  One launch and 1.6 to 5 us less per call (4 chunks of 32
// tokens over 500 keys 16.5 -> 14.9 us, 512 tokens over 30000 keys 247 -> 241 us).
static_assert(kOwnPairs == 3 * kMaxTileCtas, "fewer than this, and they cannot be claimed one by one");

struct own_plan_t {
  run_t run;
  uint32_t units, per;
  uint32_t sums[12];                 // of the warps
  uint32_t pairs_before[kOwnPairs];  // n + 1
};
static_assert(sizeof(own_plan_t) <= 2048, "layout::kBytes");

template <int kThreads>
__device__ __forceinline__ uint32_t cta_exclusive(uint32_t v, uint32_t* sums, uint32_t& total) {
  static_assert(kThreads == 12 * 32, "own_plan_t::sums");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t incl = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += up;
  }
  __syncthreads();  // what an earlier call left has been read
  if (lane == 31) sums[warp] = incl;
  __syncthreads();
  const uint32_t of_warp = lane < kThreads / 32 ? sums[lane] : 0;
  total = __reduce_add_sync(kFull, of_warp);
  return __reduce_add_sync(kFull, lane < warp ? of_warp : 0) + incl - v;
}

__device__ __forceinline__ void plan_own(const tiles_args& a, own_plan_t& plan) {
  const preba_pages_attend_t& p = a.p;
  auto pairs_of = [&](uint32_t r) -> uint32_t {
    request_t q;
    if (!load_request(p, r, q)) {
      if (blockIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
      return 0;
    }
    return (q.rows + 2 * a.tokens_per_tile - 1) / (2 * a.tokens_per_tile);
  };
  const uint32_t share = (p.n + kThreads - 1) / kThreads;
  const uint32_t r0 = min(threadIdx.x * share, p.n), r1 = min(r0 + share, p.n);
  uint32_t mine = 0, n_pairs;
  for (uint32_t r = r0; r < r1; ++r) mine += pairs_of(r);
  uint32_t at = cta_exclusive<kThreads>(mine, plan.sums, n_pairs);
  for (uint32_t r = r0; r < r1; ++r) {
    plan.pairs_before[r] = at;
    at += pairs_of(r);
  }
  if (threadIdx.x == 0) plan.pairs_before[p.n] = n_pairs;
  __syncthreads();
  if (n_pairs > a.max_pairs) {  // rows of different requests overlap: the list ends early
    if (threadIdx.x == 0 && blockIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
    n_pairs = a.max_pairs;
  }
  constexpr int kEach = (kOwnPairs + kThreads - 1) / kThreads;
  pair_t pair[kEach];
  uint32_t tiles = 0;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint32_t i = kEach * threadIdx.x + k;
    pair[k].tiles = 0;
    if (i >= n_pairs) continue;
    uint32_t lo = 0, hi = p.n;  // the last request with no more pairs before it than i
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (plan.pairs_before[mid] <= i) lo = mid; else hi = mid;
    }
    request_t q;
    load_request(p, lo, q);
    const pair_range range = range_of(a, q, i - plan.pairs_before[lo]);
    pair[k] = {lo, i - plan.pairs_before[lo], 0, static_cast<uint32_t>(range.end - range.begin), q.row, q.rows, q.keys, 0};
    tiles += pair[k].tiles;
  }
  uint32_t total;
  uint32_t before = cta_exclusive<kThreads>(tiles, plan.sums, total);
  const uint32_t units = total * p.heads_kv;
  const uint32_t per = max(kMinRun, (units + a.grid - 1) / a.grid), unit = blockIdx.x * per;
  if (threadIdx.x == 0) {
    plan.units = units;
    plan.per = per;
    if (unit >= units) a.runs[blockIdx.x].first = a.runs[blockIdx.x].last = 0;
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const uint32_t from = before * p.heads_kv, to = from + pair[k].tiles * p.heads_kv;
    if (unit >= from && unit < to) {  // one thread's pair
      pair[k].before = before;
      const uint32_t head = (unit - from) / pair[k].tiles, start = from + head * pair[k].tiles;
      const bool cuts = unit > start && unit - per <= start;
      plan.run = {pair[k], kEach * threadIdx.x + k, head, cuts ? blockIdx.x - 1 : 0,
                  cuts ? (start + pair[k].tiles - 1) / per : 0};
      a.runs[blockIdx.x] = plan.run;  // for the joining kernel
    }
    before += pair[k].tiles;
  }
  __syncthreads();
}

// ---- tensor core instructions (PTX) ---------------------------------------------------------------

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory operand: rows of 128 bytes in the 128-byte swizzle, eight rows (1024 bytes) to a group.
// `leading` is the distance between 64-element columns of an operand whose rows are its contraction
// axis.  The low word of the descriptor; the high one is the same for all.
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t leading) {
  return (addr & 0x3ffff) >> 4 | (leading >> 4) << 16;
}
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// fp32 accumulator, 128 rows, `columns` columns; values: the second operand's rows are contracted.
template <typename T> __device__ __forceinline__ constexpr uint32_t shape(uint32_t columns, bool values) {
  const uint32_t kind = sizeof(T) == 2 && !std::is_same<T, __half>::value ? 1 : 0;  // bfloat16 : binary16
  return 1u << 4 | kind << 7 | kind << 10 | (values ? 1u << 16 : 0u) | (columns / 8) << 17 | (kTile / 16) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc),
      "r"(add), "n"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.u32 p, %4, 0;\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc),
      "r"(add), "n"(kOperandHigh)
      : "memory");
}
// One lane of the (converged) warp, always the same.
__device__ __forceinline__ bool elected() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
// Arrives at the barrier when all matrix products issued before have finished.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar)
               : "memory");
}

// Arithmetic on two fp32 numbers at once, and a maximum of three.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b));
  return v;
}
__device__ __forceinline__ uint64_t pair(uint32_t a, uint32_t b) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(a), "r"(b));
  return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v));
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ float max3(float a, uint32_t b, uint32_t c) {
  float v;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(v) : "f"(a), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
  return v;
}
__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c) {
  return max3(__uint_as_float(a), b, c);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  return max3(a, __float_as_uint(b), __float_as_uint(c));
}

#define PREBA_R8(v, i) "+r"(v[i]), "+r"(v[i + 1]), "+r"(v[i + 2]), "+r"(v[i + 3]), "+r"(v[i + 4]), \
    "+r"(v[i + 5]), "+r"(v[i + 6]), "+r"(v[i + 7])
#define PREBA_I8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), \
    "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
#define PREBA_L32 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24," \
    "%25,%26,%27,%28,%29,%30,%31}"
// 32 columns of the thread's row.  The registers hold them once tmem_loaded() has returned.
__device__ __forceinline__ void tmem_load32(uint32_t* v, uint32_t addr) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 " PREBA_L32 ", [%32];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]),
                 "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]),
                 "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
                 "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
                 "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
               : "r"(addr)
               : "memory");
}
// Nothing that uses the 32 registers moves above it.
__device__ __forceinline__ void tmem_loaded(uint32_t* v) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : PREBA_R8(v, 0), PREBA_R8(v, 8), PREBA_R8(v, 16), PREBA_R8(v, 24)::"memory");
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t* v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], " PREBA_L32 ";" ::PREBA_I8(v, 0), PREBA_I8(v, 8),
               PREBA_I8(v, 16), PREBA_I8(v, 24), "r"(addr)
               : "memory");
}
__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::
          PREBA_I8(v, 0), PREBA_I8(v, 8), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- the kernel -----------------------------------------------------------------------------------

// Four neighbouring threads hold four blocks of four words each, one row per thread; afterwards thread q of
// them holds block q of all four rows, in the order of the rows.
__device__ __forceinline__ void turn_four(uint32_t (&w)[16]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int bit = 2; bit; bit >>= 1) {
    const bool up = lane & bit;
#pragma unroll
    for (int block = 0; block < 4; ++block) {
      if (block & bit) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t &lo = w[4 * block + i], &hi = w[4 * (block | bit) + i];
        const uint32_t got = __shfl_xor_sync(kFull, up ? lo : hi, bit);
        lo = up ? got : lo;
        hi = up ? hi : got;
      }
    }
  }
}

// The lowest n bits, of 32.
__device__ __forceinline__ uint32_t below(int32_t n) {
  return n <= 0 ? 0u : n >= 32 ? kFull : (1u << n) - 1;
}

// A counter of ring slots with the parity that a wait for its next use takes.
template <int N> struct ring {
  uint32_t slot = 0, phase = 0;
  __device__ __forceinline__ void step() {
    if (++slot == N) slot = 0, phase ^= 1;
  }
};

template <typename T, int DP>
__global__ void __launch_bounds__(kThreads, 1)
tiles_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
             const __grid_constant__ CUtensorMap map_v, const __grid_constant__ tiles_args a) {
  using L = layout<DP>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const preba_pages_attend_t& p = a.p;
  const int lane = threadIdx.x & 31;
  const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0);
  const uint32_t base = smem_addr(smem);
  const uint32_t kv_full = base + L::kBars, kv_empty = kv_full + 8 * L::kSlots;
  const uint32_t q_full = kv_empty + 8 * L::kSlots, q_empty = q_full + 8;
  const uint32_t s_full = q_empty + 8, p_full = s_full + 16, o_full = p_full + 16;  // A, B each
  const uint32_t item_full = o_full + 16, item_empty = item_full + 16;             // two slots each
  const uint32_t drained = item_empty + 16, h_full = drained + 8;
  static_assert(8 * (2 * L::kSlots + 15) + 8 <= 504, "layout::kItems");
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kBars + 504);
  item_t* items = reinterpret_cast<item_t*>(smem + L::kItems);

  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kSlots; ++s) {
      mbar_init(kv_full + 8 * s, 1);
      mbar_init(kv_empty + 8 * s, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full + 8 * x, 1);
      mbar_init(p_full + 8 * x, kSoftWarps / 2);
      mbar_init(h_full + 8 * x, kSoftWarps / 2);
      mbar_init(o_full + 8 * x, 1);
      mbar_init(item_full + 8 * x, 1);
      mbar_init(item_empty + 8 * x, kSoftWarps + 1);
    }
    mbar_init(drained, 1);
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  chained_begin();
  // Only now: a kernel before this one that has let it in may still have its tensor memory to allocate, and
  // would wait for this CTA as this CTA waits for it.
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(tmem_slot)),
                 "n"(kTmemColumns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = *tmem_slot;
  own_plan_t& own = *reinterpret_cast<own_plan_t*>(smem + L::kPlan);
  if (a.own_plan) plan_own(a, own);
  waits_t wait(a);
  bool ok = true;

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegisters));
    if (warp == kCopyWarp) {
      // ---- work and copies
      tiles_head plan;
      run_t run;  // means something only if the run has a key tile
      if (a.own_plan) {
        plan = {0, 0, own.units, 0, own.per};
        run = own.run;
      } else {
        plan = *a.head;
        run = a.runs[blockIdx.x];
      }
      const uint32_t boxes = kTile >> a.box_shift;
      const uint32_t chunk = lane & (boxes - 1), half = lane / boxes;
      const bool mine = half < L::kHalves;
      const uint32_t dst = half * L::kHalf + (chunk << a.box_shift) * 128;
      ring<L::kSlots> kv;
      ring<1> q_ring;
      ring<2> out;
      uint32_t issued = 0, q_issued = 0;
      uint32_t unit = min(static_cast<uint64_t>(blockIdx.x) * plan.per, static_cast<uint64_t>(plan.units));
      const uint32_t unit_end = min(unit + plan.per, plan.units);
      uint32_t pair = run.which;
      pair_t of = run.pair;  // of the run's first piece
      bool next_pair = false;
      while (ok) {
        // the next piece
        item_t item;
        item.count = 0;
        if (next_pair && unit < unit_end) {
          ++pair;
          next_pair = false;
          if (a.own_plan) {
            of.before += of.tiles;
            while (own.pairs_before[of.request + 1] <= pair) ++of.request;  // ends: the run has a key tile left
            of.pair = pair - own.pairs_before[of.request];
            request_t q;
            load_request(p, of.request, q);
            of.row = q.row;
            of.rows = q.rows;
            of.keys = q.keys;
            const pair_range range = range_of(a, q, of.pair);
            of.tiles = range.end - range.begin;
          } else {
            if (!PREBA_IN_RANGE(p.status, pair < plan.n_pairs)) pair = 0;
            of = a.pairs[pair];
          }
        }
        if (plan.claim) {
          uint32_t k = 0;
          if (lane == 0) k = atomicAdd(&a.head->next, 1);
          k = __shfl_sync(kFull, k, 0);
          if (k < plan.n_pairs * p.heads_kv) {
            of = a.pairs[a.order[k / p.heads_kv]];
            item.head = k % p.heads_kv;
            item.count = of.tiles;
            item.tile = 0;
            item.whole = 1;
            item.slot = 0;
          }
        } else if (unit < unit_end) {
          const uint32_t offset = unit - of.before * p.heads_kv;
          item.head = offset / of.tiles;
          item.tile = offset - item.head * of.tiles;
          item.count = min(of.tiles - item.tile, unit_end - unit);
          item.whole = item.count == static_cast<int32_t>(of.tiles);
          item.slot = 2 * blockIdx.x + (item.tile == 0);
          unit += item.count;
          next_pair = offset + item.count == of.tiles * p.heads_kv;
        }
        const bool done = item.count == 0;
        if (!done) {
          const request_t q{of.row, of.rows, of.keys};
          const pair_range range = range_of(a, q, of.pair);
          item.request = of.request;
          item.row = q.row;
          item.rows = q.rows;
          item.keys = q.keys;
          item.token = 2 * of.pair * a.tokens_per_tile;
          item.lo = range.lo;
          item.hi = range.hi;
          item.tile += range.begin;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            item.first[x] = max(range.first[x], item.tile);
            item.last[x] = max(item.first[x], min(range.last[x], item.tile + item.count));
          }
        }
        ok = wait(item_empty + 8 * out.slot, out.phase ^ 1);
        if (!ok) break;
        if (lane == 0) {
          items[out.slot] = item;
          mbar_arrive(item_full + 8 * out.slot);
        }
        out.step();
        if (done) break;
        // queries
        ok = wait(q_empty, q_ring.phase ^ 1);
        if (!ok) break;
        if (lane == 0) {
          const uint32_t bytes = a.tokens_per_tile * a.group * 128 * L::kHalves;
          const bool two = item.token + static_cast<int32_t>(a.tokens_per_tile) < item.rows;
          mbar_arrive_expect_tx(q_full, two ? 2 * bytes : bytes);
          for (int x = 0; x < (two ? 2 : 1); ++x)
            for (int h = 0; h < L::kHalves; ++h)
              tensor_copy(base + x * L::kQ + h * L::kHalf, &map_q, 64 * h, item.head * a.group,
                          item.row + item.token + x * a.tokens_per_tile, 0, q_full);
        }
        ++q_issued;
        q_ring.step();
        // keys and values, tile by tile
        const int32_t* row = p.block_table + static_cast<uint64_t>(item.request) * p.table_stride;
        int32_t key = item.tile * kTile + (chunk << a.box_shift);
        auto wanted = [&](int32_t k) {
          return mine && k < item.hi && k + static_cast<int32_t>(a.box_rows) > item.lo;
        };
        int32_t entry = wanted(key) ? row[key >> a.page_shift] : 0;
        for (int32_t t = 0; t < item.count && ok; ++t, key += kTile) {
          int32_t page = entry;
          const bool want = wanted(key);
          if (t + 1 < item.count) entry = wanted(key + kTile) ? row[(key + kTile) >> a.page_shift] : 0;
          if (want && (page < 0 || static_cast<uint32_t>(page) >= p.pages)) {
            report(p.status, PREBA_ERR_BAD_TABLE);
            page = p.pages;  // beyond the tensor: the box is filled with zeros
          }
          const uint32_t bytes = __popc(__ballot_sync(kFull, want)) * a.box_rows * 128;
#pragma unroll
          for (int v = 0; v < 2; ++v) {
            ok = ok && wait(kv_empty + 8 * kv.slot, kv.phase ^ 1);
            if (!ok) break;
            if (lane == 0) mbar_arrive_expect_tx(kv_full + 8 * kv.slot, bytes);
            __syncwarp();
            if (want)
              tensor_copy(base + L::kRing + kv.slot * L::kSlot + dst, v ? &map_v : &map_k, half * 64,
                          key & (p.page_size - 1), item.head, page, kv_full + 8 * kv.slot);
            ++issued;
            kv.step();
          }
        }
      }
      if (!ok) {  // what is in flight lands before the memory goes to another
        report(p.status, PREBA_ERR_TIMEOUT);
        for (uint32_t i = issued - min(issued, static_cast<uint32_t>(L::kSlots)); i < issued; ++i)
          mbar_wait(kv_full + 8 * (i % L::kSlots), (i / L::kSlots) & 1);
        if (q_issued) mbar_wait(q_full, (q_issued - 1) & 1);
      }
    } else if (warp == kMmaWarp) {
      // ---- matrix products: one lane issues, the warp clears values that nobody sees
      constexpr uint32_t kQkShape = shape<T>(kTile, false), kPvShape = shape<T>(DP, true);
      ring<L::kSlots> kv;  // next slot to be waited for
      ring<1> q_ring, p_ring[2];
      ring<2> in;
      while (ok) {
        ok = wait(item_full + 8 * in.slot, in.phase);
        if (!ok) break;
        const item_t item = items[in.slot];
        __syncwarp();
        if (lane == 0) mbar_arrive(item_empty + 8 * in.slot);
        in.step();
        if (item.count == 0) break;
        ok = wait(q_full, q_ring.phase);
        if (!ok) break;
        q_ring.step();
        const int32_t end = item.tile + item.count;
        uint32_t k_slot = 0, v_slot = 0;
        auto qk = [&](int x) {
          const uint32_t q_op = __shfl_sync(kFull, operand(base + x * L::kQ, 16), 0);
          const uint32_t k_op = __shfl_sync(kFull, operand(base + L::kRing + k_slot * L::kSlot, 16), 0);
          const uint32_t d = __shfl_sync(kFull, tmem + L::kS + x * kTile, 0);
          if (elected()) {
#pragma unroll
            for (int ks = 0; ks < DP / 16; ++ks) {
              const uint32_t off = (ks / 4) * L::kHalf + (ks % 4) * 32;
              mma_ss(d, q_op + (off >> 4), k_op + (off >> 4), kQkShape, ks > 0);
            }
            mma_commit(s_full + 8 * x);
          }
          __syncwarp();
        };
        auto pv = [&](int x, bool add, int from, int to) {
          const uint32_t v_op = __shfl_sync(kFull, operand(base + L::kRing + v_slot * L::kSlot, L::kHalf), 0);
          const uint32_t d = __shfl_sync(kFull, tmem + L::kO + x * DP, 0);
          const uint32_t a_op = __shfl_sync(kFull, tmem + L::kS + x * kTile, 0);
          if (elected()) {
#pragma unroll
            for (int ks = from; ks < to; ++ks)
              mma_ts(d, a_op + 8 * ks, v_op + (ks * 2048 >> 4), kPvShape, add || ks > 0);
          }
          __syncwarp();
        };
        // keys of the first tile
        ok = wait(kv_full + 8 * kv.slot, kv.phase);
        if (!ok) break;
        fence_after();
        k_slot = kv.slot;
        kv.step();
#pragma unroll
        for (int x = 0; x < 2; ++x)
          if (item.first[x] == item.tile && item.first[x] < item.last[x]) qk(x);
        if (elected()) {
          mma_commit(kv_empty + 8 * k_slot);
          if (item.count == 1) mma_commit(q_empty);
        }
        for (int32_t t = item.tile; t < end && ok; ++t) {
          ok = wait(kv_full + 8 * kv.slot, kv.phase);
          if (!ok) break;
          v_slot = kv.slot;
          kv.step();
          const int32_t key = t * kTile;
          if (key < item.lo || key + kTile > item.hi) {
            // values outside the seen keys may be anything, and 0 times NaN is NaN: clear them
            const int32_t c0 = min(max(item.lo - key, 0), kTile), c1 = min(max(item.hi - key, 0), kTile);
            uint8_t* at = smem + L::kRing + v_slot * L::kSlot;
            for (int32_t i = lane; i < kTile * 8; i += 32) {
              const int32_t k = i >> 3;
              if (k < c0 || k >= c1)
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h)
                  *reinterpret_cast<uint4*>(at + h * L::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
          bool k_waited = false;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (t >= item.first[x] && t < item.last[x]) {
              // the product with the first half of P while the second is being made
              ok = ok && wait(h_full + 8 * x, p_ring[x].phase);
              if (!ok) break;
              fence_after();
              pv(x, t > item.first[x], 0, kTile / 32);
              ok = ok && wait(p_full + 8 * x, p_ring[x].phase);
              if (!ok) break;
              p_ring[x].step();
              fence_after();
              pv(x, true, kTile / 32, kTile / 16);
              if (t + 1 == item.last[x] && elected()) mma_commit(o_full + 8 * x);
            }
            if (t + 1 >= item.first[x] && t + 1 < item.last[x]) {
              if (!k_waited) {
                ok = ok && wait(kv_full + 8 * kv.slot, kv.phase);
                if (!ok) break;
                fence_after();
                k_slot = kv.slot;
                k_waited = true;
              }
              qk(x);
            }
          }
          if (!ok) break;
          if (elected()) mma_commit(kv_empty + 8 * v_slot);
          if (t + 1 < end) {  // A or B sees every key tile of the piece, so its keys were waited for
            kv.step();
            if (elected()) {
              mma_commit(kv_empty + 8 * k_slot);
              if (t + 2 == end) mma_commit(q_empty);
            }
          }
        }
      }
      if (!ok) {
        report(p.status, PREBA_ERR_TIMEOUT);
        // what was issued ends before the memory goes to another; a commit counts its own thread's products
        if (elected()) mma_commit(drained);
        __syncwarp();
        mbar_wait(drained, 0);
      }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kMmaWarp)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(kTmemColumns)
                   : "memory");
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegisters));
    // ---- softmax: group x has row tile x, a thread a row
    const int x = warp >> 2, r = threadIdx.x & (kTile - 1);
    const uint32_t lanes = static_cast<uint32_t>(warp & 3) << 21;  // 32 rows of tensor memory each
    const uint32_t s_at = tmem + lanes + L::kS + x * kTile, o_at = tmem + lanes + L::kO + x * DP;
    const float scale = p.scale * kLog2e;
    const int32_t j = r / static_cast<int32_t>(a.group), g = r - j * static_cast<int32_t>(a.group);
    ring<1> s_ring, o_ring;
    ring<2> in;
    while (ok) {
      ok = wait(item_full + 8 * in.slot, in.phase);
      if (!ok) break;
      const item_t item = items[in.slot];
      const int32_t first = items[in.slot].first[x], last = items[in.slot].last[x];
      __syncwarp();
      if (lane == 0) mbar_arrive(item_empty + 8 * in.slot);
      in.step();
      if (item.count == 0) break;
      const int32_t token = item.token + x * static_cast<int32_t>(a.tokens_per_tile);
      if (token >= item.rows) continue;  // B has no rows
      const int32_t tokens = min(static_cast<int32_t>(a.tokens_per_tile), item.rows - token);
      const bool live = j < tokens;
      request_t q{item.row, item.rows, item.keys};
      int32_t row_lo = 0, row_hi = 0, low, high;
      if (live) seen_by(p, q, token + j, token + j + 1, row_lo, row_hi);
      int32_t all_lo, all_hi;  // keys that every row of the tile sees
      seen_by(p, q, token, token + 1, low, all_hi);
      seen_by(p, q, token + tokens - 1, token + tokens, all_lo, high);
      float m = -INFINITY, l = 0.f;
      for (int32_t t = first; t < last && ok; ++t) {
        ok = wait(s_full + 8 * x, s_ring.phase);
        if (!ok) break;
        s_ring.step();
        fence_after();
        uint32_t s[kTile];
#pragma unroll
        for (int c = 0; c < kTile; c += 32) tmem_load32(s + c, s_at + c);
#pragma unroll
        for (int c = 0; c < kTile; c += 32) tmem_loaded(s + c);
        const int32_t key = t * kTile;
        if (key < all_lo || key + kTile > all_hi) {
          // a bit per key of 32: constant bit tests come out as predicates, eight at a time
#pragma unroll
          for (int c = 0; c < kTile; c += 32) {
            const uint32_t seen = below(row_hi - key - c) & ~below(row_lo - key - c);
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (!(seen >> i & 1)) s[c + i] = 0xff800000u;
          }
        }
        float tops[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) tops[c] = max3(s[3 * c], s[3 * c + 1], s[3 * c + 2]);
#pragma unroll
        for (int c = 12; c < 124; c += 8)
#pragma unroll
          for (int k = 0; k < 4; ++k) tops[k] = max3(tops[k], s[c + 2 * k], s[c + 2 * k + 1]);
        float top = fmaxf(max3(tops[0], s[124], s[125]), max3(tops[1], s[126], s[127]));
        top = max3(top, tops[2], tops[3]);
        top *= scale;
        const bool grown = top > m + kGrowth;  // true for the first key seen: m is -inf
        if (__any_sync(kFull, grown)) {
          const float to = fmaxf(m, top);
          const float keep = to == -INFINITY ? 0.f : exp2_approx(m - to);
          m = to;
          l *= keep;
          if (t > first) {  // the product before has finished: S could not be there otherwise
            for (int c = 0; c < DP; c += 32) {
              uint32_t o[32];
              tmem_load32(o, o_at + c);
              tmem_loaded(o);
#pragma unroll
              for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep);
              tmem_store32(o_at + c, o);
            }
          }
        }
        const float shift = m == -INFINITY ? 0.f : m;
        const uint64_t scale2 = pair(scale, scale), shift2 = pair(-shift, -shift);
        uint64_t sums[2] = {0, 0};
#pragma unroll
        for (int c = 0; c < kTile; c += 32) {
          uint32_t e[16];
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            float z0, z1;
            unpair(fma2(pair(s[c + i], s[c + i + 1]), scale2, shift2), z0, z1);
            z0 = exp2_approx(z0);
            z1 = exp2_approx(z1);
            sums[(i / 2) & 1] = add2(sums[(i / 2) & 1], pair(z0, z1));
            e[i / 2] = pack2<T>(z0, z1);
          }
          tmem_store16(s_at + c / 2, e);
          if (c == 32) {  // the first half is there: its product may start
            tmem_stored();
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(h_full + 8 * x);
          }
        }
        float l0, l1;
        unpair(add2(sums[0], sums[1]), l0, l1);
        l += l0 + l1;
        tmem_stored();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(p_full + 8 * x);
      }
      if (!ok) break;
      const bool any = first < last;
      if (any) {
        ok = wait(o_full + 8 * x, o_ring.phase);
        if (!ok) break;
        o_ring.step();
        fence_after();
      }
      if (item.whole) {
        const uint32_t h = item.head * a.group + g, tok = item.row + token + j;
        const bool write = live && PREBA_IN_RANGE(p.status, tok < p.tokens && h < p.heads_q);
        const float inv = l > 0.f ? 1.f / l : 0.f;
        // Four threads turn 64 bytes of their four rows around, so that a store writes 64 bytes of eight
        // rows and not 16 bytes of 32: the stores of a tile were bound by the lines they touch (3850 clocks).
        T* rows[4];
        uint32_t writes = __ballot_sync(kFull, write) >> (lane & ~3);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          rows[k] = reinterpret_cast<T*>(__shfl_sync(
              kFull, reinterpret_cast<uint64_t>(static_cast<T*>(p.out) + tok * p.out_stride[0] + h * p.out_stride[1]),
              (lane & ~3) + k)) + 8 * (lane & 3);
#pragma unroll 1
        for (int c = 0; c < DP; c += 32) {
          uint32_t o[32], w[16];
          tmem_load32(o, o_at + c);
          tmem_loaded(o);
#pragma unroll
          for (int i = 0; i < 32; i += 2) w[i / 2] = pack2<T>(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
          turn_four(w);
          if (c + 8 * (lane & 3) < static_cast<int32_t>(p.head_dim)) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (writes >> k & 1)
                *reinterpret_cast<uint4*>(rows[k] + c) = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
        if (p.lse && write)
          p.lse[static_cast<uint64_t>(tok) * p.heads_q + h] = row_lse(m, l);
      } else {
        // partial sums, four columns of 256 rows after the other, then maxima and sums
        float4* to = a.partials + static_cast<uint64_t>(item.slot) * kPartial<DP> + x * kTile + r;
        if (any)
#pragma unroll 1
          for (int c = 0; c < DP; c += 32) {
            uint32_t o[32];
            tmem_load32(o, o_at + c);
            tmem_loaded(o);
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              to[(c + i) / 4 * 2 * kTile] = make_float4(__uint_as_float(o[i]), __uint_as_float(o[i + 1]),
                                                        __uint_as_float(o[i + 2]), __uint_as_float(o[i + 3]));
          }
        reinterpret_cast<float2*>(to - (x * kTile + r) + DP / 4 * 2 * kTile)[x * kTile + r] = make_float2(marked(m, l), l);
      }
      fence_before();
    }
    if (!ok) report(p.status, PREBA_ERR_TIMEOUT);

    fence_before();
    __syncthreads();
  }
}

// ---- joining ----------------------------------------------------------------------------------------
//
// Pairs of which several CTAs had a piece: a block adds up 16 columns of one, a thread a row.  All SMs
// take part, which is why this is a kernel of its own (the last CTA of each pair doing it by itself kept
// a third of the SMs busy for 10 to 20 us).

constexpr int kJoinColumns = 16;

template <typename T, int DP>
__global__ void __launch_bounds__(2 * kTile, 2) tiles_join_kernel(const __grid_constant__ tiles_args a) {
  chained_begin();
  const preba_pages_attend_t& p = a.p;
  constexpr uint32_t kParts = DP / kJoinColumns;
  const uint32_t e = blockIdx.x % kParts * kJoinColumns;
  const run_t run = a.runs[blockIdx.x / kParts];
  const uint32_t first = run.first, last = run.last, head = run.head;
  if (first == last || e >= p.head_dim) return;
  const int x = threadIdx.x / kTile, r = threadIdx.x % kTile;
  const int32_t j = r / static_cast<int32_t>(a.group), g = r - j * static_cast<int32_t>(a.group);
  // Pieces in the order of the keys, four at a time so that their loads are on the way together; the
  // first CTA's piece begins the pair and lies in its second slot, the others in their first.
  float m = -INFINITY, l = 0.f, acc[kJoinColumns] = {};
#pragma unroll 1
  for (uint32_t c = first; c <= last; c += 4) {
    float2 v[4];
    float4 part[4][kJoinColumns / 4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint32_t cta = min(c + k, last);  // the last one again: it is not counted
      const float4* from = a.partials + static_cast<uint64_t>(2 * cta + (cta == first)) * kPartial<DP>;
      v[k] = __ldcg(reinterpret_cast<const float2*>(from + DP / 4 * 2 * kTile) + threadIdx.x);
#pragma unroll
      for (int i = 0; i < kJoinColumns / 4; ++i)
        part[k][i] = __ldcg(from + (e / 4 + i) * 2 * kTile + threadIdx.x);
    }
    const float to = fmaxf(m, fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x)));
    const float keep = to == -INFINITY ? 0.f : exp2_approx(m - to);
    m = to;
    l *= keep;
#pragma unroll
    for (int i = 0; i < kJoinColumns; ++i) acc[i] *= keep;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // a piece that saw nothing left no sums: what lies in their place may be anything
      if (c + k > last || v[k].x == -INFINITY) continue;
      const float w = exp2_approx(v[k].x - m);
      l = fmaf(w, v[k].y, l);
#pragma unroll
      for (int i = 0; i < kJoinColumns / 4; ++i) {
        acc[4 * i] = fmaf(w, part[k][i].x, acc[4 * i]);
        acc[4 * i + 1] = fmaf(w, part[k][i].y, acc[4 * i + 1]);
        acc[4 * i + 2] = fmaf(w, part[k][i].z, acc[4 * i + 2]);
        acc[4 * i + 3] = fmaf(w, part[k][i].w, acc[4 * i + 3]);
      }
    }
  }
  const int32_t token = (2 * run.pair.pair + x) * a.tokens_per_tile + j;
  if (j >= static_cast<int32_t>(a.tokens_per_tile) || token >= run.pair.rows) return;
  const uint32_t h = head * a.group + g, tok = run.pair.row + token;
  const float inv = l > 0.f ? 1.f / l : 0.f;
  T* to = static_cast<T*>(p.out) + tok * p.out_stride[0] + h * p.out_stride[1] + e;
#pragma unroll
  for (int i = 0; i < kJoinColumns; i += 8)
    if (e + i < p.head_dim) {
      uint4 v;
      v.x = pack2<T>(acc[i] * inv, acc[i + 1] * inv);
      v.y = pack2<T>(acc[i + 2] * inv, acc[i + 3] * inv);
      v.z = pack2<T>(acc[i + 4] * inv, acc[i + 5] * inv);
      v.w = pack2<T>(acc[i + 6] * inv, acc[i + 7] * inv);
      *reinterpret_cast<uint4*>(to + i) = v;
    }
  if (p.lse && e == 0)
    p.lse[static_cast<uint64_t>(tok) * p.heads_q + h] = row_lse(m, l);
}

template <typename T, int DP>
cudaError_t launch(const tiles_args& a, cudaStream_t stream) {
  using L = layout<DP>;
  const preba_pages_attend_t& p = a.p;
  CUtensorMap map_q, map_k, map_v;
  const uint64_t dims_q[4] = {p.head_dim, p.heads_q, p.tokens, 1};
  const uint64_t strides_q[3] = {p.q_stride[1], p.q_stride[0], 0};
  const uint32_t box_q[2] = {a.group, a.tokens_per_tile};
  cudaError_t err = tensor_map(&map_q, p.dtype, p.q, dims_q, strides_q, box_q);
  if (err == cudaSuccess) err = cache_map(&map_k, p, p.k_cache, p.k_stride, a.box_rows);
  if (err == cudaSuccess) err = cache_map(&map_v, p, p.v_cache, p.v_stride, a.box_rows);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(tiles_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (err != cudaSuccess) return err;
  err = launch_chained(tiles_kernel<T, DP>, a.grid, kThreads, L::kBytes, stream, map_q, map_k, map_v, a);
  if (err != cudaSuccess) return err;
  return launch_chained(tiles_join_kernel<T, DP>, a.grid * (DP / kJoinColumns), 2 * kTile, 0,
                        stream, a);
}

uint64_t up16(uint64_t v) { return (v + 15) / 16 * 16; }

}  // namespace

namespace attend {

uint64_t tiles_workspace(uint32_t n, uint32_t tokens, uint32_t group, uint32_t head_dim) {
  const uint64_t pairs = pairs_at_most(n, tokens, group);
  return up16(sizeof(tiles_head)) + sizeof(run_t) * kMaxTileCtas + sizeof(pair_t) * pairs + up16(4 * pairs) +
         2ull * kMaxTileCtas * (head_dim <= 64 ? kPartial<64> : kPartial<128>) * sizeof(float4);
}

cudaError_t launch_tiles(const preba_pages_attend_t& p, uint32_t page_shift, int sms, void* workspace,
                         cudaStream_t stream) {
  tiles_args a{};
  a.p = p;
  a.page_shift = page_shift;
  a.group = p.heads_q / p.heads_kv;
  a.tokens_per_tile = kTile / a.group;
  a.box_rows = std::min<uint32_t>(p.page_size, kTile);
  a.box_shift = 31 - __builtin_clz(a.box_rows);
  a.grid = std::min(sms, kMaxTileCtas);
  const uint64_t pairs = pairs_at_most(p.n, p.tokens, a.group);
  a.max_pairs = static_cast<uint32_t>(pairs);
  uint8_t* at = static_cast<uint8_t*>(workspace);
  a.head = reinterpret_cast<tiles_head*>(at);
  at += up16(sizeof(tiles_head));
  a.runs = reinterpret_cast<run_t*>(at);
  at += sizeof(run_t) * kMaxTileCtas;
  a.pairs = reinterpret_cast<pair_t*>(at);
  at += sizeof(pair_t) * pairs;
  a.order = reinterpret_cast<uint32_t*>(at);
  at += up16(4 * pairs);
  a.partials = reinterpret_cast<float4*>(at);
  a.own_plan = plans_own(pairs, p.heads_kv, a.grid,
                         std::min<uint64_t>(static_cast<uint64_t>(p.table_width) * p.page_size, PREBA_PAGES_MAX_KEYS));
  const size_t smem = kPlanThreads * sizeof(pair_t) + 4 * (static_cast<size_t>(p.n) + 1);
  if (smem > 40 * 1024) {  // beside 5 KB of its own; 48 KB need no leave
    const cudaError_t err = cudaFuncSetAttribute(tiles_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 kPlanThreads * sizeof(pair_t) + 4 * (PREBA_PAGES_MAX_REQUESTS + 1));
    if (err != cudaSuccess) return err;
  }
  if (!a.own_plan) {
    const cudaError_t err = launch_chained(tiles_plan_kernel, 1, kPlanThreads, smem, stream, a);
    if (err != cudaSuccess) return err;
  }
  if (p.dtype == PREBA_F16)
    return p.head_dim <= 64 ? launch<__half, 64>(a, stream) : launch<__half, 128>(a, stream);
  return p.head_dim <= 64 ? launch<__nv_bfloat16, 64>(a, stream) : launch<__nv_bfloat16, 128>(a, stream);
}

}  // namespace attend
}  // namespace preba
