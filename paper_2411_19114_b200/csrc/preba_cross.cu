// Attention of a decoder's rows to an encoder's packed states (preba_beams.h): preba_cross_attend.
//
// Where few rows share a key head (the beams of a request, times the query heads of a group) the states have to
// be read once and bytes bound the call; rows are too few to fill the 128 of a matrix product, but states are
// not.  So states take the rows' place:
//   S^T = K Q^T        128 states x rows   (tcgen05, both operands in shared memory as they lie)
//   P^T = exp2(scale log2(e) S^T - m)      a thread per state, a register per row; written to shared memory in 16 bits
//   O^T += V^T P^T     head_dim x rows     (tcgen05, V as it lies: its rows are the contraction)
// A thread adds up its own states' probabilities, row by row, and the threads are joined once per piece.  All
// that crosses threads in a tile is a vote: only if some score outgrows its row's reference by more than 2^8 (and for the
// first tile) the maxima are taken over the threads and the accumulator is rescaled; until then P is at
// most 2^8 and the sums carry the old reference, which leaves the quotient as it is.
//
// The work is one line of tiles, request by request and key head by key head, of which every CTA takes an equal run,
// whatever the lengths are; a (request, key head) that crosses CTAs is left as partial sums, which the last of them
// to finish joins in the order of the states, so that timing does not change a bit.
//
// P is rounded to the states' type because the matrix instructions take it so; its sums are not.
//
// Bound by bytes, less a start and an end: 64 requests of 5 beams over 1500 states of 20 heads of 64 59 to 60 us, 48 of 8 beams
// over 2000 states of 8 heads of 128 51 to 53 us (floors 50 and 41; 6.1 TB/s while it streams); 2 requests of 4 beams over
// 375 states 7.9 us, a chain of latencies.
//
// More rows go to the kernels for many rows (preba_attend_tiles.cu).
#include <algorithm>
#include <type_traits>

#include "preba_attend.h"
#include "preba_attend_plan.h"
#include "preba_beams.h"
#include "preba_tensor.h"

namespace preba {
namespace {

using namespace attend;

constexpr int kTile = 128;            // states of a tile
constexpr int kColumns = 64;          // rows on a key head, or a pair of them, that this kernel takes

// Rows on a key head that this kernel takes.  Measured, here and by the kernels for many rows: 48 requests of up to 2000 states on
// 8 heads of 128, 16 rows 59 and 79 us, 64 rows 67 and 87; two of up to 400, 64 rows 11 and 15.  64 requests of up
// to 1500 on 20 heads of 64, 32 rows 80 and 120 us; 4 of them, 16 rows 18.5 and 20, 32 rows 26 and 20.  More than 32 rows of
// two heads do not fit the columns, and one such head at a time took 134 and 122 us.
constexpr uint32_t few_rows(uint32_t head_dim) { return head_dim <= 64 ? kColumns / 2 : kColumns; }
constexpr int kSoftWarps = 4, kSoftThreads = 32 * kSoftWarps;
constexpr int kCopyWarp = 4, kMmaWarp = 5;
constexpr int kThreads = 192;
constexpr uint32_t kMinUnits = 3;     // a CTA's run is not shorter than this
constexpr uint32_t kWholeTiles = 8;   // tiles of a (request, key head) that is not split where there is a CTA for each
constexpr uint64_t kMostUnits = 2000000000;  // of the line
constexpr uint64_t kNowhere = ~0ull;  // of a column without a row
constexpr float kGrowth = 8.f;        // log2 of what a row may outgrow its reference by
constexpr uint64_t kCounterBytes = kMaxTileCtas * 4;  // at the workspace's start

// D: head_dim rounded up to 64 or 128.  H: key heads of a piece.  Heads of up to 64 are taken in pairs, whose rows in memory
// lie side by side more often than not: 64 requests of 5 beams over 1500 states of 20 heads of 64, single heads 76 us (61 if
// each head's states lay together), pairs 68 to 70 either way, and 60 by what came after.  The product with the values then has the elements of both heads as its 128
// rows, and of its columns each half belongs to one of them.  N: columns, R rows of each head.
template <int D, int H, int R> struct layout {
  static constexpr int N = H * R;
  static_assert(H * D == 128, "a head of 128 or two of 64");
  static constexpr int kHalves = 2;                         // of 64 elements: of one head, or of a pair
  static constexpr uint32_t kHalf = kTile * 128;            // 64 elements of 128 states
  static constexpr uint32_t kSlot = kHalves * kHalf;        // a tile of keys, or of values
  static constexpr int kSlots = N <= 32 ? 6 : 5;
  // Two tiles of P^T, 128 states of N rows each in lines of 128 bytes: side by side if they fit, else one after the other
  static constexpr uint32_t kP = kSlots * kSlot;
  static constexpr uint32_t kPNext = N <= 32 ? N * 2 : kTile * 128;
  static constexpr uint32_t kQ = kP + (N <= 32 ? 1 : 2) * kTile * 128;  // two sets of queries: 64 elements of R rows, twice
  static constexpr uint32_t kQSize = kHalves * R * 128;
  static constexpr uint32_t kStats = kQ + 2 * kQSize;
  static constexpr uint32_t kBars = kStats + 8 * N * 4 + N * 8;
  static constexpr uint32_t kControl = kBars + 8 * (2 * kSlots + 12);
  static constexpr uint32_t kBytes = kControl + 256;
  // Tensor memory columns.
  static constexpr uint32_t kS = 0, kO = 2 * N;
  static constexpr uint32_t kTmem = N == 64 ? 256 : N == 32 ? 128 : 64;
  static_assert(kBars % 8 == 0 && kBytes <= 227 * 1024 && kP >= kTile * 128, "shared memory");
};
// Floats of a partial sum: O^T column by column, then a maximum and a sum for each.
template <int D> constexpr uint32_t kPartial = kColumns * D + 2 * kColumns;
constexpr uint32_t kDirect = 4;  // pieces of a (request, head) that the CTA with the first of them joins on the spot, at most

// What a call is about beside the sizes it shares with the paged attention.
struct cross_args {
  preba_pages_attend_t p;
  const int32_t* cu_k;
  const int32_t* seen;
  uint32_t states, group, grid, q_rows;  // q_rows: tokens of a request, at most
  uint32_t heads;                        // key heads, or pairs of them
#if defined(PREBA_CHECKED)
  wait_limits_t limits = wait_limits();
#endif
};

struct piece_t {
  uint32_t request, head;
  uint32_t first, last;  // CTAs that hold pieces of the same (request, key head)
};
// A request as the walk needs it.
struct entry_t {
  request_t q;
  int32_t state0, hi;  // its first state, and how many of them some row sees
  uint32_t tiles;      // on one key head (or pair); 0: it has no rows or is at fault
};
struct run_t {
  uint32_t begin, end, per;  // units; units per CTA
  uint32_t request, offset;  // of the first unit
  entry_t entry;
};
struct control_t {
  run_t run;
  piece_t pieces[2];
  uint64_t warp_sums[kThreads / 32];
  uint32_t warp_pieces[kThreads / 32], warp_longest[kThreads / 32], joins[2], alone, tmem;
};
static_assert(sizeof(control_t) <= 256, "layout::kBytes");

__device__ __forceinline__ bool load_entry(const cross_args& a, uint32_t r, entry_t& e) {
  e.tiles = 0;
  if (!load_packed(a.p, a.cu_k, a.states, r, e.q)) return false;
  e.state0 = a.cu_k[r];
  e.hi = packed_seen(a.seen, e.q, 0, e.q.rows);
  if (e.q.rows) e.tiles = max(1, (e.hi + kTile - 1) / kTile);  // one that sees nothing still has its zeros to write
  return true;
}

// Where a CTA's run begins: the block adds up the units of all requests, each thread of a run of them.  The units of a (request,
// key head) are one for its beginning and end, which cost about what a tile does, and one for each tile.  Where there is a CTA
// for every (request, key head), and none of them is long, each takes one and nothing has to be joined (two
// requests of up to 3 tiles on 8 heads: 7.9 us, in equal runs 11.3).
__device__ __forceinline__ void find_run(const cross_args& a, control_t& ctl) {
  const preba_pages_attend_t& p = a.p;
  const uint32_t chunk = (p.n + kThreads - 1) / kThreads;
  const uint32_t r0 = min(threadIdx.x * chunk, p.n), r1 = min(r0 + chunk, p.n);
  uint64_t mine = 0;
  uint32_t my_pieces = 0, longest = 0;
  entry_t e{};
  for (uint32_t r = r0; r < r1; ++r) {
    if (!load_entry(a, r, e) && blockIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
    if (e.tiles) mine += static_cast<uint64_t>(e.tiles + 1) * a.heads, my_pieces += a.heads;
    longest = max(longest, e.tiles);
  }
  uint64_t incl = mine;
  uint32_t pieces_incl = my_pieces;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t up = __shfl_up_sync(kFull, incl, o);
    const uint32_t pieces_up = __shfl_up_sync(kFull, pieces_incl, o);
    if (lane >= o) incl += up, pieces_incl += pieces_up;
  }
  longest = __reduce_max_sync(kFull, longest);
  if (lane == 31) ctl.warp_sums[warp] = incl, ctl.warp_pieces[warp] = pieces_incl, ctl.warp_longest[warp] = longest;
  __syncthreads();
  uint64_t sum = 0, before = 0;
  uint32_t pieces = 0, pieces_before = 0;  // at most 16384 * 65535
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += ctl.warp_sums[w], pieces_before += ctl.warp_pieces[w];
    sum += ctl.warp_sums[w];
    pieces += ctl.warp_pieces[w];
    longest = max(longest, ctl.warp_longest[w]);
  }
  // requests that do not overlap never come to more (the host has seen to it); if they do, nothing is done
  if (sum > kMostUnits && blockIdx.x == 0 && threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
  const uint32_t total = sum > kMostUnits ? 0 : static_cast<uint32_t>(sum);
  const bool whole = pieces <= gridDim.x && longest <= kWholeTiles;
  const uint32_t per = whole ? 1 : max(kMinUnits, (total + gridDim.x - 1) / gridDim.x);
  const uint32_t all = whole ? pieces : total;  // in pieces, or in units
  const uint32_t begin = min(static_cast<uint64_t>(blockIdx.x) * per, static_cast<uint64_t>(all));
  uint64_t at = whole ? pieces_before + pieces_incl - my_pieces : before + incl - mine;
  if (begin >= all) {
    if (threadIdx.x == 0) ctl.run.begin = ctl.run.end = 0;
  } else if (begin >= at && begin < at + (whole ? my_pieces : mine)) {  // one thread
    uint32_t r = r0;
    for (;; ++r) {
      if (r1 - r0 > 1) load_entry(a, r, e);
      const uint32_t here = e.tiles == 0 ? 0 : whole ? a.heads : (e.tiles + 1) * a.heads;
      if (begin < at + here) break;
      at += here;
    }
    const uint32_t from = static_cast<uint32_t>(begin - at);
    if (whole) ctl.run = {0, e.tiles + 1, e.tiles + 1, r, from * (e.tiles + 1), e};
    else ctl.run = {begin, min(begin + per, all), per, r, from, e};
  }
  __syncthreads();
}

// Walks a CTA's run piece by piece; every warp does so for itself.
struct walk_t {
  uint32_t unit, end, per, request, offset;  // next unit; offset within the request
  entry_t of;
  uint32_t start, head, tile, count;         // the current piece; start: of the (request, key head)
  __device__ __forceinline__ explicit walk_t(const run_t& run)
      : unit(run.begin), end(run.end), per(run.per), request(run.request), offset(run.offset), of(run.entry) {}
  __device__ __forceinline__ bool next(const cross_args& a) {
    while (unit < end) {
      while (offset >= (of.tiles + 1) * a.heads || of.tiles == 0) {  // ends: unit < end, so a later request has tiles
        offset = 0;
        load_entry(a, ++request, of);
      }
      const uint32_t units = of.tiles + 1;
      head = offset / units;
      const uint32_t at = offset - head * units, take = min(units - at, end - unit);
      start = unit - at;
      unit += take;
      offset += take;
      tile = at ? at - 1 : 0;
      count = at ? take : take - 1;
      if (count) return true;
    }
    return false;
  }
  __device__ __forceinline__ bool whole() const { return count == of.tiles; }
  __device__ __forceinline__ uint32_t first_cta() const { return (start + 1) / per; }
  __device__ __forceinline__ uint32_t last_cta() const { return (start + of.tiles) / per; }
};

// 128 rows; the first operand's rows or columns are contracted, as the second's are.
template <typename T> __device__ __forceinline__ constexpr uint32_t shape(uint32_t columns, bool rows_contracted) {
  const uint32_t kind = std::is_same<T, __half>::value ? 0 : 1;  // binary16 : bfloat16
  return 1u << 4 | kind << 7 | kind << 10 | (rows_contracted ? 3u << 15 : 0u) | (columns / 8) << 17 | (kTile / 16) << 24;
}

template <int N> __device__ __forceinline__ void tmem_load(uint32_t (&v)[N], uint32_t addr) {
  if constexpr (N == 16) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
                   "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
                 : "r"(addr)
                 : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" : PREBA_R8(v, 0), PREBA_R8(v, 8)::"memory");
  } else {
#pragma unroll
    for (int c = 0; c < N; c += 32) tmem_load32(v + c, addr + c);
#pragma unroll
    for (int c = 0; c < N; c += 32) tmem_loaded(v + c);
  }
}
// The softmax threads: all of them, whatever became of their waits.
__device__ __forceinline__ void soft_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kSoftThreads) : "memory"); }
__device__ __forceinline__ bool soft_any(bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(static_cast<uint32_t>(mine)), "n"(kSoftThreads)
      : "memory");
  return any != 0;
}
// The largest number of the warp; what is not a number is left out.
__device__ __forceinline__ float warp_max_of(uint32_t v) {
  float top;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(top) : "f"(__uint_as_float(v)));
  return top;
}
// The result: a row's sum of products times one over its sum of probabilities, 0 where that is 0.
template <typename T> __device__ __forceinline__ T result_of(float v, float inverse) {
  const float x = inverse == 0.f ? 0.f : v * inverse;
  if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
  else return __float2bfloat16_rn(x);
}
__device__ __forceinline__ float inverse_of(float sum) { return sum == 0.f ? 0.f : 1.f / sum; }

// Sums over the warp's lanes of N numbers each; afterwards lane l holds those of the columns that column_of() names.
template <int N, int O = 16, int Half = N / 2> __device__ __forceinline__ void sum_columns(float (&v)[N]) {
  if constexpr (O > 0) {
    if constexpr (Half > 0) {
      const bool up = threadIdx.x & O;
#pragma unroll
      for (int i = 0; i < Half; ++i) {
        const float send = up ? v[i] : v[i + Half], keep = up ? v[i + Half] : v[i];
        v[i] = keep + __shfl_xor_sync(kFull, send, O);
      }
    } else {  // 16 columns: two lanes have the same one
      v[0] += __shfl_xor_sync(kFull, v[0], O);
    }
    sum_columns<N, O / 2, Half / 2>(v);
  }
}
template <int N> __device__ __forceinline__ int column_of(int i) {
  const int lane = threadIdx.x & 31;
  return N == 16 ? lane >> 1 : N == 32 ? lane : 2 * lane + i;
}

template <int D> __device__ __forceinline__ float* partial_of(const cross_args& a, uint32_t cta, uint32_t slot) {
  if (!PREBA_IN_RANGE(a.p.status, 2 * cta + slot < 2 * a.grid)) cta = slot = 0;
  return reinterpret_cast<float*>(static_cast<uint8_t*>(a.p.workspace) + kCounterBytes) +
         static_cast<uint64_t>(2 * cta + slot) * kPartial<D>;
}

template <typename T, int D, int H, int R>
__global__ void __launch_bounds__(kThreads, 1)
cross_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
             const __grid_constant__ CUtensorMap map_v, const __grid_constant__ cross_args a) {
  using L = layout<D, H, R>;
  constexpr int N = L::N;
  extern __shared__ __align__(1024) uint8_t smem[];
  const preba_pages_attend_t& p = a.p;
  const int lane = threadIdx.x & 31;
  const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0);
  const uint32_t base = smem_addr(smem);
  const uint32_t kv_full = base + L::kBars, kv_empty = kv_full + 8 * L::kSlots;
  const uint32_t drained = kv_empty + 8 * L::kSlots;
  const uint32_t s_full = drained + 8, p_full = s_full + 16, o_done = p_full + 16, q_full = o_done + 16,
                 q_empty = q_full + 16;  // two each
  control_t& ctl = *reinterpret_cast<control_t*>(smem + L::kControl);

  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kSlots; ++s) {
      mbar_init(kv_full + 8 * s, 1);
      mbar_init(kv_empty + 8 * s, 1);
    }
    mbar_init(drained, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(q_full + 8 * x, 1);
      mbar_init(q_empty + 8 * x, 1);
      mbar_init(s_full + 8 * x, 1);
      mbar_init(p_full + 8 * x, kSoftWarps);
      mbar_init(o_done + 8 * x, 1);
    }
    ctl.joins[0] = ctl.joins[1] = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  chained_begin();
  // Only now: a kernel before this one that has let it in may still have its tensor memory to allocate, and
  // would wait for this CTA as this CTA waits for it.
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)),
                 "n"(L::kTmem)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  find_run(a, ctl);  // synchronises
  fence_after();
  const uint32_t tmem = ctl.tmem;
  const run_t run = ctl.run;
  waits_t wait(a);
  bool ok = true;

  if (run.begin >= run.end) {
    // nothing to do but to give the tensor memory back
  } else if (warp == kCopyWarp) {
    // ---- copies: a lane per box of 32 states, 64 elements wide
    constexpr uint32_t kBoxes = kTile / kStateRows;
    const uint32_t chunk = lane % kBoxes, half = lane / kBoxes;
    const uint32_t dst = half * L::kHalf + chunk * kStateRows * 128;
    const uint32_t x = H == 2 ? 0 : half * 64, of_pair = H == 2 ? half : 0;  // a half is elements of the head, or a head of the pair
    walk_t w(run);
    uint32_t slot = 0, phase = 1, issued = 0, pieces = 0;  // a fresh barrier counts as emptied
    while (ok && w.next(a)) {
      const int32_t state0 = w.of.state0;
      // the piece's queries, and whatever lies behind them up to q_rows tokens
      const uint32_t qb = pieces & 1;
      ok = wait(q_empty + 8 * qb, (pieces >> 1 & 1) ^ 1);
      if (!ok) break;
      ++pieces;
      if (lane == 0) {
        mbar_arrive_expect_tx(q_full + 8 * qb, a.q_rows * a.group * 128 * L::kHalves);
        for (int h = 0; h < L::kHalves; ++h)  // a head behind the last reads as 0
          tensor_copy(base + L::kQ + qb * L::kQSize + h * R * 128, &map_q, H == 2 ? 0 : 64 * h,
                      (H * w.head + (H == 2 ? h : 0)) * a.group, w.of.q.row, 0, q_full + 8 * qb);
      }
      const bool mine = half < L::kHalves && H * w.head + of_pair < p.heads_kv;
      int32_t key = w.tile * kTile + chunk * kStateRows;
      for (uint32_t t = 0; t < w.count && ok; ++t, key += kTile) {
        const bool want = mine && key < w.of.hi;
        const uint32_t bytes = __popc(__ballot_sync(kFull, want)) * kStateRows * 128;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          ok = ok && wait(kv_empty + 8 * slot, phase);
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(kv_full + 8 * slot, bytes);
          __syncwarp();
          if (want)
            tensor_copy(base + slot * L::kSlot + dst, v ? &map_v : &map_k, x, state0 + key, H * w.head + of_pair, 0,
                        kv_full + 8 * slot);
          ++issued;
          if (++slot == L::kSlots) slot = 0, phase ^= 1;
        }
      }
    }
    if (!ok) {  // what is in flight lands before the memory goes to another
      report(p.status, PREBA_ERR_TIMEOUT);
      for (uint32_t i = issued - min(issued, static_cast<uint32_t>(L::kSlots)); i < issued; ++i)
        mbar_wait(kv_full + 8 * (i % L::kSlots), (i / L::kSlots) & 1);
      for (uint32_t i = pieces - min(pieces, 2u); i < pieces; ++i) mbar_wait(q_full + 8 * (i & 1), (i >> 1) & 1);
    }
  } else if (warp == kMmaWarp) {
    // ---- matrix products: one lane issues, the warp clears values that nobody sees
    constexpr uint32_t kQkShape = shape<T>(R, false), kPvShape = shape<T>(N, true);
    walk_t w(run);
    uint32_t slot = 0, phase = 0;
    uint32_t n_s = 0, n_p = 0, pieces = 0;  // tiles and pieces so far
    auto step = [&]() {
      const uint32_t s = slot;
      if (++slot == L::kSlots) slot = 0, phase ^= 1;
      return s;
    };
    auto qk = [&](bool last) {
      ok = ok && wait(kv_full + 8 * slot, phase);
      if (!ok) return;
      fence_after();
      const uint32_t k_slot = step();
      const uint32_t k_op = __shfl_sync(kFull, operand(base + k_slot * L::kSlot, 16), 0);
      const uint32_t qb = pieces & 1;
      const uint32_t q_op = __shfl_sync(kFull, operand(base + L::kQ + qb * L::kQSize, 16), 0);
      const uint32_t d = __shfl_sync(kFull, tmem + L::kS + (n_s & 1) * N, 0);
      if (elected()) {
#pragma unroll
        for (int ks = 0; ks < H * D / 16; ++ks)  // of the head, or of one head of the pair after the other
          mma_ss(H == 2 ? d + ks / 4 * R : d, k_op + (((ks / 4) * L::kHalf + (ks % 4) * 32) >> 4),
                 q_op + (((ks / 4) * R * 128 + (ks % 4) * 32) >> 4), kQkShape, H == 2 ? ks % 4 > 0 : ks > 0);
        mma_commit(s_full + 8 * (n_s & 1));
        mma_commit(kv_empty + 8 * k_slot);
        if (last) mma_commit(q_empty + 8 * qb);
      }
      __syncwarp();
      ++n_s;
    };
    for (; ok && w.next(a); ++pieces) {
      ok = wait(q_full + 8 * (pieces & 1), (pieces >> 1) & 1);
      if (!ok) break;
      fence_after();
      qk(w.count == 1);
      for (uint32_t t = 0; t < w.count && ok; ++t) {
        // values come before the next keys; the scores of the next tile are made while this one's are looked at
        const uint32_t v_slot = slot, v_phase = phase;
        step();
        if (t + 1 < w.count) qk(t + 2 == w.count);
        ok = ok && wait(kv_full + 8 * v_slot, v_phase);
        if (!ok) break;
        const int32_t seen = w.of.hi - static_cast<int32_t>((w.tile + t) * kTile);
        if (seen < kTile) {
          // values outside the seen states may be anything, and 0 times NaN is NaN: clear them
          uint8_t* at = smem + v_slot * L::kSlot;
          for (int32_t i = max(seen, 0) * 8 + lane; i < kTile * 8; i += 32)
#pragma unroll
            for (int h = 0; h < L::kHalves; ++h) *reinterpret_cast<uint4*>(at + h * L::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
        }
        const uint32_t b = n_p & 1;
        ok = wait(p_full + 8 * b, (n_p >> 1) & 1);
        if (!ok) break;
        fence_after();
        const uint32_t v_op = __shfl_sync(kFull, operand(base + v_slot * L::kSlot, L::kHalf), 0);
        const uint32_t p_op = __shfl_sync(kFull, operand(base + L::kP + b * L::kPNext, 16), 0);
        const uint32_t d = __shfl_sync(kFull, tmem + L::kO, 0);
        if (elected()) {
#pragma unroll
          for (int ks = 0; ks < kTile / 16; ++ks) mma_ss(d, v_op + (ks * 2048 >> 4), p_op + (ks * 2048 >> 4), kPvShape, t > 0 || ks > 0);
          mma_commit(o_done + 8 * b);
          mma_commit(kv_empty + 8 * v_slot);
        }
        __syncwarp();
        ++n_p;
      }
    }
    if (!ok) {
      report(p.status, PREBA_ERR_TIMEOUT);
      // what was issued ends before the memory goes to another; a commit counts its own thread's products
      if (elected()) mma_commit(drained);
      __syncwarp();
      mbar_wait(drained, 0);
    }
  } else {
    // ---- softmax: a thread per state of the tile, then per element of the result
    const int r = threadIdx.x;
    const uint32_t lanes = static_cast<uint32_t>(warp) << 21;  // 32 rows of tensor memory each
    const float scale = p.scale * kLog2e;
    float* stats = reinterpret_cast<float*>(smem + L::kStats);      // of four warps, N columns each
    float* ref = stats + 4 * N;                                     // what a row's exponents are taken beside
    float* keep = ref + N;                                          // and what is left of its sums when that grows
    int32_t* row_hi = reinterpret_cast<int32_t*>(keep + N);         // states that a row sees
    uint64_t* row_at = reinterpret_cast<uint64_t*>(row_hi + 2 * N); // where a row's result goes
    walk_t w(run);
    uint32_t n = 0;  // tiles so far
    // A piece whose partial sums are on their way is counted a tile later, when they have arrived: a fence behind them
    // waits for 2 to 4 us while all SMs read
    bool pending = false;
    piece_t pending_piece{};
    uint32_t before_pending = 0;  // counted before it, known to thread 0 when it is needed
    auto count_piece = [&]() {  // behind a barrier behind everybody's fence
      if (r == 0) before_pending = atomicAdd(static_cast<uint32_t*>(p.workspace) + pending_piece.first, 1);
      pending = false;
    };
    auto counted = [&](int which) {
      if (r != 0) return;
      const bool last = before_pending == pending_piece.last - pending_piece.first;
      if (last) static_cast<uint32_t*>(p.workspace)[pending_piece.first] = 0;  // as the next call wants it
      ctl.pieces[which] = pending_piece;
      ctl.joins[which] = last;
    };
    bool first_counted = false;
    while (w.next(a)) {
      const request_t q = w.of.q;
      const int32_t rows = q.rows * a.group;
      const bool go = !soft_any(!ok);
      ok = go;
      float m = -INFINITY;  // of row r, where there is one: the largest score of those looked at when it grew last
      int32_t hi = 0;
      // the row of column r: query row j, query head h
      const uint32_t kv_head = H * w.head + r / R, in_head = r % R;
      const bool row_there = r < N && in_head < static_cast<uint32_t>(rows) && kv_head < p.heads_kv;
      const uint32_t j = in_head / a.group, h = kv_head * a.group + in_head - j * a.group;
      if (r < N) {
        if (row_there) hi = packed_seen(a.seen, q, j, j + 1);
        row_hi[r] = hi;
        row_at[r] = row_there ? (q.row + j) * p.out_stride[0] + h * p.out_stride[1] : kNowhere;
        ref[r] = row_there ? 0.f : INFINITY;  // columns without a row hold whatever lay behind the queries: they outgrow nothing
      }
      soft_sync();  // what every row sees is there
      int32_t all = w.of.hi;  // states that every row sees
      if (a.seen)
        for (int c = 0; c < N; ++c)
          if (row_at[c] != kNowhere) all = min(all, row_hi[c]);
      float l[N];
#pragma unroll
      for (int c = 0; c < N; ++c) l[c] = 0.f;
      for (uint32_t t = 0; go && t < w.count; ++t, ++n) {
        const uint32_t b = n & 1;
        const int32_t key = (w.tile + t) * kTile + r;
        uint32_t s[N];
        auto scores = [&]() {
          tmem_load<N>(s, tmem + lanes + L::kS + b * N);
          if (key - r + kTile > all) {
#pragma unroll
            for (int c = 0; c < N; ++c)
              if (key >= row_hi[c]) s[c] = 0xff800000u;
          }
        };
        auto exponents = [&]() {
          float top = -INFINITY;
#pragma unroll
          for (int c = 0; c < N; c += 4) {
            const float4 of = *reinterpret_cast<const float4*>(ref + c);
            const float z[4] = {fmaf(__uint_as_float(s[c]), scale, -of.x), fmaf(__uint_as_float(s[c + 1]), scale, -of.y),
                                fmaf(__uint_as_float(s[c + 2]), scale, -of.z), fmaf(__uint_as_float(s[c + 3]), scale, -of.w)};
#pragma unroll
            for (int i = 0; i < 4; ++i) s[c + i] = __float_as_uint(z[i]), top = fmaxf(top, z[i]);
          }
          return top;
        };
        const bool count_now = pending && t == 1;
        if (count_now) __threadfence();
        ok = ok && wait(s_full + 8 * b, (n >> 1) & 1);
        fence_after();
        scores();
        // a row that sees a state and has no reference yet gets one
        const bool slow = soft_any(exponents() > kGrowth || (m == -INFINITY && hi > 0) || !ok);
        if (count_now) count_piece();
        if (slow) {
          if (soft_any(!ok)) {
            ok = false;
            break;
          }
          scores();
#pragma unroll
          for (int c = 0; c < N; ++c) {
            const float top = warp_max_of(s[c]);
            if (lane == 0) stats[warp * N + c] = top;
          }
          soft_sync();
          if (r < N) {
            const float top = fmaxf(fmaxf(stats[r], stats[N + r]), fmaxf(stats[2 * N + r], stats[3 * N + r])) * scale;
            const float to = fmaxf(m, top);
            keep[r] = to == -INFINITY ? 0.f : exp2_approx(m - to);
            if (row_there) ref[r] = to == -INFINITY ? 0.f : to;
            m = to;
          }
          soft_sync();
#pragma unroll
          for (int c = 0; c < N; ++c) l[c] *= keep[c];
          if (t > 0) {
            ok = wait(o_done + 8 * (b ^ 1), ((n - 1) >> 1) & 1);  // of the tile before
            fence_after();
#pragma unroll
            for (int c = 0; c < N; c += 16) {
              uint32_t o[16];
              tmem_load<16>(o, tmem + lanes + L::kO + c);
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * keep[c + i]);
              tmem_store16(tmem + lanes + L::kO + c, o);
            }
            tmem_stored();
          }
          scores();  // again: nobody holds them meanwhile
          exponents();
        }
        if (t > 1) ok = ok && wait(o_done + 8 * b, ((n - 2) >> 1) & 1);  // that product has read its P
        uint8_t* to = smem + L::kP + (N <= 32 ? 0 : b * L::kPNext) + r * 128;
        const uint32_t chunk0 = N <= 32 ? b * (N / 8) : 0;
#pragma unroll
        for (int c = 0; c < N; c += 8) {
          uint32_t e[4];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float z0 = exp2_approx(__uint_as_float(s[c + i])), z1 = exp2_approx(__uint_as_float(s[c + i + 1]));
            l[c + i] += z0, l[c + i + 1] += z1;
            e[i / 2] = pack2<T>(z0, z1);
          }
          if (ok) *reinterpret_cast<uint4*>(to + (((chunk0 + c / 8) ^ (r & 7)) << 4)) = make_uint4(e[0], e[1], e[2], e[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        __syncwarp();
        if (ok && lane == 0) mbar_arrive(p_full + 8 * b);
      }
      // ---- the piece is over: the threads' sums are joined
      const bool whole = w.whole(), begins = w.tile == 0;
      const piece_t x{w.request, w.head, w.first_cta(), w.last_cta()};
      uint32_t* counter = static_cast<uint32_t*>(p.workspace) + x.first;
      uint32_t arrived = 0;
      if (r == 0 && begins && !whole) arrived = *static_cast<volatile uint32_t*>(counter);
      ok = ok && wait(o_done + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
      fence_after();
      // a thread has an element of one head, and the columns of that head
      constexpr int kMine = H == 2 ? R : N;
      const int e = r % (H == 2 ? 64 : 128), col0 = H == 2 ? r / 64 * R : 0;
      uint32_t o[kMine];
      tmem_load<kMine>(o, tmem + lanes + L::kO + col0);
      fence_before();
      sum_columns<N>(l);
#pragma unroll
      for (int i = 0; i < (N + 31) / 32; ++i) stats[warp * N + column_of<N>(i)] = l[i];
      // The others' pieces were counted when they were over, which for a run's first piece is early: if they are all there
      // the CTA with the first piece joins them on the spot, and its own is never written down
      if (r == 0) {
        ctl.alone = begins && !whole && arrived == x.last - x.first && x.last - x.first < kDirect;
        if (ctl.alone) {
          *counter = 0;  // as the next call wants it
          __threadfence();
        }
      }
      if (pending) __threadfence();
      soft_sync();
      if (pending) count_piece();  // the piece after it had one tile
      const bool here = ctl.alone;
      float sum = 0.f;
      if (row_there) sum = (stats[r] + stats[N + r]) + (stats[2 * N + r] + stats[3 * N + r]);
      if (whole || here) {
        if (here) {
          // weights of the pieces in the order of the states, as below; nobody reads P now
          float* weights = reinterpret_cast<float*>(smem + L::kP);
          if (row_there) {
            float2 stat[kDirect];
            stat[0] = make_float2(marked(m, sum), sum);
#pragma unroll
            for (uint32_t k = 1; k < kDirect; ++k)
              stat[k] = x.first + k <= x.last ? __ldcg(reinterpret_cast<const float2*>(partial_of<D>(a, x.first + k, 0) + kColumns * D) + r)
                                              : make_float2(-INFINITY, 0.f);
            float top = -INFINITY;
#pragma unroll
            for (uint32_t k = 0; k < kDirect; ++k) top = fmaxf(top, stat[k].x);
            sum = 0.f;
#pragma unroll
            for (uint32_t k = 0; k < kDirect; ++k) {
              const float weight = stat[k].x == -INFINITY ? 0.f : exp2_approx(stat[k].x - top);
              if (weight != 0.f) sum = fmaf(weight, stat[k].y, sum);
              weights[k * N + r] = weight;
            }
            m = top;
          }
          soft_sync();
#pragma unroll
          for (int c = 0; c < kMine; ++c) {
            const float weight = weights[col0 + c];
            o[c] = weight == 0.f ? 0u : __float_as_uint(fmaf(weight, __uint_as_float(o[c]), 0.f));
          }
          for (uint32_t k = 1; x.first + k <= x.last; ++k) {
            const float* from = partial_of<D>(a, x.first + k, 0) + col0 * D + e;
            float part[kMine];
#pragma unroll
            for (int c = 0; c < kMine; ++c) part[c] = row_at[col0 + c] != kNowhere && e < D ? __ldcg(from + c * D) : 0.f;
#pragma unroll
            for (int c = 0; c < kMine; ++c) {
              const float weight = weights[k * N + col0 + c];
              if (weight != 0.f) o[c] = __float_as_uint(fmaf(weight, part[c], __uint_as_float(o[c])));
            }
          }
          soft_sync();  // the weights have been read
        }
        if (row_there) {
          keep[r] = inverse_of(sum);
          if (p.lse && PREBA_IN_RANGE(p.status, q.row + j < p.tokens && h < p.heads_q))
            p.lse[static_cast<uint64_t>(q.row + j) * p.heads_q + h] = row_lse(m, sum);
        }
        soft_sync();
        // turned around in shared memory (nobody reads P now), so that 16 bytes of a row are stored at a time
        T* turned = reinterpret_cast<T*>(smem + L::kP);
        if (e < D) {
#pragma unroll
          for (int c = 0; c < kMine; ++c) turned[(col0 + c) * D + e] = result_of<T>(__uint_as_float(o[c]), keep[col0 + c]);
        }
        soft_sync();
#pragma unroll
        for (int i = 0; i < N * D / 8; i += kSoftThreads) {
          const int c = (i + r) / (D / 8), at = (i + r) % (D / 8) * 8;
          if (row_at[c] != kNowhere && at < static_cast<int>(p.head_dim))
            *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + row_at[c] + at) = *reinterpret_cast<const uint4*>(turned + c * D + at);
        }
      } else {
        float* part = partial_of<D>(a, blockIdx.x, begins);
        if (row_there) reinterpret_cast<float2*>(part + kColumns * D)[r] = make_float2(marked(m, sum), sum);
        if (e < D) {
#pragma unroll
          for (int c = 0; c < kMine; ++c)
            if (row_at[col0 + c] != kNowhere) part[(col0 + c) * D + e] = __uint_as_float(o[c]);
        }
        if (w.unit < w.end) {
          pending = first_counted = true;
          pending_piece = x;
        } else {
          if (first_counted) counted(0);
          first_counted = false;
          __threadfence();
          soft_sync();
          pending_piece = x;
          count_piece();
          counted(1);
        }
      }
      soft_sync();  // what lies in shared memory has been read
    }
    if (!ok) report(p.status, PREBA_ERR_TIMEOUT);
    if (pending) {  // the run ended with the beginning of a piece, but no tile of it
      __threadfence();
      soft_sync();
      count_piece();
    }
    if (first_counted) {
      counted(0);
      soft_sync();
    }

    // ---- join the CTAs: whoever finishes a (request, key head) last adds its pieces up
    if (ctl.joins[0] || ctl.joins[1]) {
      __threadfence();
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        if (!ctl.joins[i]) continue;
        const piece_t x = ctl.pieces[i];
        request_t q;
        load_packed(p, a.cu_k, a.states, x.request, q);
        const uint32_t rows = q.rows * a.group, count = x.last - x.first + 1;
        // The first CTA's piece begins the (request, key head) and lies in its slot 1, the others in slot 0.  A thread per row
        // makes weights of the pieces' maxima and sums, in the order of the states; they lie where the tiles were
        float2* stat = reinterpret_cast<float2*>(smem);  // of piece and column: maximum and sum, then weight
        static_assert(kMaxTileCtas * N * sizeof(float2) <= L::kP, "room for the weights");
        if (r < N) {
          const uint32_t kv_head = H * x.head + r / R, in_head = r % R;
          const uint32_t j = in_head / a.group, h = kv_head * a.group + in_head - j * a.group;
          row_at[r] = kNowhere;
          if (in_head < rows && kv_head < p.heads_kv && PREBA_IN_RANGE(p.status, q.row + j < p.tokens && h < p.heads_q)) {
            float top = -INFINITY, sum = 0.f;
#pragma unroll 8
            for (uint32_t k = 0; k < count; ++k) {
              const float2 v = __ldcg(reinterpret_cast<const float2*>(partial_of<D>(a, x.first + k, k == 0) + kColumns * D) + r);
              stat[k * N + r] = v;
              top = fmaxf(top, v.x);
            }
            for (uint32_t k = 0; k < count; ++k) {
              const float2 v = stat[k * N + r];
              const float weight = v.x == -INFINITY ? 0.f : exp2_approx(v.x - top);
              if (weight != 0.f) sum = fmaf(weight, v.y, sum);
              stat[k * N + r].x = weight;
            }
            keep[r] = inverse_of(sum);
            row_at[r] = (q.row + j) * p.out_stride[0] + h * p.out_stride[1];
            if (p.lse) p.lse[static_cast<uint64_t>(q.row + j) * p.heads_q + h] = row_lse(top, sum);
          }
        }
        soft_sync();
        // four elements of a row each, several rows and pieces on the way together
        constexpr int kEach = N * D / 4 / kSoftThreads, kGo = kEach < 4 ? kEach : 4;
#pragma unroll 1
        for (int i0 = 0; i0 < kEach; i0 += kGo) {
          float4 acc[kGo];
#pragma unroll
          for (int i = 0; i < kGo; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
          for (uint32_t k = 0; k < count; ++k) {
            const float* from = partial_of<D>(a, x.first + k, k == 0);
            float4 v[kGo];
#pragma unroll
            for (int i = 0; i < kGo; ++i) {
              const int at = (i0 + i) * kSoftThreads + r, c = at / (D / 4);
              v[i] = row_at[c] != kNowhere ? __ldcg(reinterpret_cast<const float4*>(from) + at) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int i = 0; i < kGo; ++i) {
              const int c = ((i0 + i) * kSoftThreads + r) / (D / 4);
              const float weight = row_at[c] != kNowhere ? stat[k * N + c].x : 0.f;
              if (weight == 0.f) continue;  // a piece that saw nothing left no sums
              acc[i].x = fmaf(weight, v[i].x, acc[i].x);
              acc[i].y = fmaf(weight, v[i].y, acc[i].y);
              acc[i].z = fmaf(weight, v[i].z, acc[i].z);
              acc[i].w = fmaf(weight, v[i].w, acc[i].w);
            }
          }
#pragma unroll
          for (int i = 0; i < kGo; ++i) {
            const int at = (i0 + i) * kSoftThreads + r, c = at / (D / 4), e = at % (D / 4) * 4;
            if (row_at[c] == kNowhere || e >= static_cast<int>(p.head_dim)) continue;
            alignas(8) T v[4] = {result_of<T>(acc[i].x, keep[c]), result_of<T>(acc[i].y, keep[c]), result_of<T>(acc[i].z, keep[c]),
                                 result_of<T>(acc[i].w, keep[c])};
            *reinterpret_cast<uint2*>(static_cast<T*>(p.out) + row_at[c] + e) = *reinterpret_cast<const uint2*>(v);
          }
        }
        soft_sync();  // the other (request, key head) has weights of its own
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kTmem) : "memory");
}

bool cross_sizes_ok(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv, uint32_t head_dim) {
  return n >= 1 && n <= PREBA_PAGES_MAX_REQUESTS && tokens >= 1 && tokens <= PREBA_PAGES_MAX_KEYS && heads_q >= 1 &&
         heads_q <= 65535 && heads_kv >= 1 && heads_q % heads_kv == 0 && heads_q / heads_kv <= 128 &&
         head_dim >= 8 && head_dim % 8 == 0 && head_dim <= PREBA_PAGES_MAX_HEAD_DIM;
}

// A counter per CTA, which every call leaves zeroed; then what one call needs, partial sums of this kernel or the list and
// the partial sums of the other.
uint64_t cross_workspace(uint32_t n, uint32_t tokens, uint32_t group, uint32_t head_dim) {
  const uint64_t few = 2ull * kMaxTileCtas * 4 * (head_dim <= 64 ? kPartial<64> : kPartial<128>);
  return kCounterBytes + std::max(few, tiles_workspace(n, tokens, group, head_dim));
}

template <typename T, int D, int H, int R> cudaError_t launch_cross(cross_args& a, cudaStream_t stream) {
  using L = layout<D, H, R>;
  a.heads = (a.p.heads_kv + H - 1) / H;
  CUtensorMap map_q, map_k, map_v;
  const uint64_t dims_q[4] = {a.p.head_dim, a.p.heads_q, a.p.tokens, 1};
  const uint64_t strides_q[3] = {a.p.q_stride[1], a.p.q_stride[0], 0};
  const uint32_t box_q[2] = {a.group, a.q_rows};
  cudaError_t err = tensor_map(&map_q, a.p.dtype, a.p.q, dims_q, strides_q, box_q);
  if (err == cudaSuccess) err = states_map(&map_k, a.p, a.states, a.p.k_cache, a.p.k_stride, kStateRows);
  if (err == cudaSuccess) err = states_map(&map_v, a.p, a.states, a.p.v_cache, a.p.v_stride, kStateRows);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(cross_kernel<T, D, H, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (err != cudaSuccess) return err;
  return launch_chained(cross_kernel<T, D, H, R>, a.grid, kThreads, L::kBytes, stream, map_q, map_k, map_v, a);
}
template <typename T> cudaError_t launch_few(cross_args& a, uint32_t rows, cudaStream_t stream) {
  if (a.p.head_dim <= 64) return rows <= 16 ? launch_cross<T, 64, 2, 16>(a, stream) : launch_cross<T, 64, 2, 32>(a, stream);
  return rows <= 16 ? launch_cross<T, 128, 1, 16>(a, stream) : rows <= 32 ? launch_cross<T, 128, 1, 32>(a, stream)
                                                                          : launch_cross<T, 128, 1, 64>(a, stream);
}

bool base_ok(const void* base, const uint64_t* strides) {
  return base && !(reinterpret_cast<uintptr_t>(base) & 15) && strides[0] % 8 == 0 && strides[1] % 8 == 0 &&
         std::max(strides[0], strides[1]) < (1ull << 38);
}
// An axis with more than one entry has a stride.
bool strides_used(const uint64_t* strides, uint32_t outer, uint32_t inner) {
  return (outer == 1 || strides[0]) && (inner == 1 || strides[1]);
}

}  // namespace
}  // namespace preba

extern "C" int preba_cross_attend_query(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv,
                                        uint32_t head_dim, uint64_t* workspace_bytes) {
  using namespace preba;
  if (!workspace_bytes || !cross_sizes_ok(n, tokens, heads_q, heads_kv, head_dim)) return PREBA_ERR_INVALID_ARG;
  *workspace_bytes = cross_workspace(n, tokens, heads_q / heads_kv, head_dim);
  return PREBA_OK;
}

extern "C" int preba_cross_attend(const preba_cross_attend_t* req, void* stream) {
  using namespace preba;
  using attend::finish;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_cross_attend_t& c = *req;
  if (!cross_sizes_ok(c.n, c.tokens, c.heads_q, c.heads_kv, c.head_dim) || !base_ok(c.q, c.q_stride) ||
      !base_ok(c.out, c.out_stride) || !base_ok(c.k, c.k_stride) || !base_ok(c.v, c.v_stride) ||
      !strides_used(c.q_stride, c.tokens, c.heads_q) || !strides_used(c.k_stride, c.states, c.heads_kv) ||
      !strides_used(c.v_stride, c.states, c.heads_kv) || !c.cu_q || !c.cu_k || c.max_q == 0 || c.states == 0 ||
      c.states > PREBA_PAGES_MAX_KEYS || (c.dtype != PREBA_F16 && c.dtype != PREBA_BF16) ||
      static_cast<double>(c.heads_kv) * (2.0 * c.n + c.states / 128.0) > kMostUnits || !(c.scale > 0.f) || !(c.scale < INFINITY) ||
      pairs_at_most(c.n, c.tokens, c.heads_q / c.heads_kv) * c.heads_kv > INT32_MAX || !c.workspace ||
      (reinterpret_cast<uintptr_t>(c.workspace) & 15))
    return PREBA_ERR_INVALID_ARG;
  const uint32_t group = c.heads_q / c.heads_kv;
  if (c.workspace_bytes < cross_workspace(c.n, c.tokens, group, c.head_dim)) return PREBA_ERR_BUFFER_TOO_SMALL;
  preba_pages_attend_t p{};
  p.q = c.q;
  p.k_cache = c.k;
  p.v_cache = c.v;
  p.cu_q = c.cu_q;
  p.out = c.out;
  p.lse = c.lse;
  p.workspace = c.workspace;
  p.workspace_bytes = c.workspace_bytes;
  p.status = c.status;
  for (int i = 0; i < 2; ++i) {
    p.q_stride[i] = c.q_stride[i];
    p.out_stride[i] = c.out_stride[i];
    p.k_stride[1 + i] = c.k_stride[i];
    p.v_stride[1 + i] = c.v_stride[i];
  }
  p.n = c.n;
  p.tokens = c.tokens;
  p.max_q = std::min(c.max_q, c.tokens);
  p.heads_q = c.heads_q;
  p.heads_kv = c.heads_kv;
  p.head_dim = c.head_dim;
  p.dtype = c.dtype;
  p.scale = c.scale;
  int device = 0, sms = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (err != cudaSuccess) return finish(err);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const uint64_t rows = static_cast<uint64_t>(group) * p.max_q;
  if (rows > few_rows(c.head_dim))
    return finish(launch_packed_tiles(p, c.cu_k, c.seen, c.states, sms, static_cast<uint8_t*>(c.workspace) + kCounterBytes, s));
  cross_args a{p, c.cu_k, c.seen, c.states, group, static_cast<uint32_t>(std::min(sms, kMaxTileCtas)), p.max_q, 0};
  return finish(c.dtype == PREBA_F16 ? launch_few<__half>(a, static_cast<uint32_t>(rows), s)
                                     : launch_few<__nv_bfloat16>(a, static_cast<uint32_t>(rows), s));
}
