// Attention of a decoder's rows to an encoder's packed states (preba_beams.h): preba_cross_attend.
//
// Where few rows share a key head (the beams of a request, times the query heads of a group, up to 64) the states have to
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
constexpr int kFewRows = 64;          // rows on a key head that this kernel takes
constexpr int kSoftWarps = 4, kSoftThreads = 32 * kSoftWarps;
constexpr int kCopyWarp = 4, kMmaWarp = 5;
constexpr int kThreads = 192;
constexpr uint32_t kMinTiles = 2;     // a CTA's run is not shorter than this
constexpr uint64_t kMostUnits = 2000000000;  // of the line
constexpr float kGrowth = 8.f;        // log2 of what a row may outgrow its reference by
constexpr uint64_t kCounterBytes = kMaxTileCtas * 4;  // at the workspace's start

// DP: head_dim rounded up to 64 or 128; N: rows rounded up to 16, 32 or 64.
template <int DP, int N> struct layout {
  static constexpr int kHalves = DP / 64;
  static constexpr uint32_t kHalf = kTile * 128;            // 64 elements of 128 states
  static constexpr uint32_t kSlot = kHalves * kHalf;        // a tile of keys, or of values
  static constexpr int kSlots = DP == 128 ? 5 : 10;
  static constexpr uint32_t kP = kSlots * kSlot;            // two tiles of P^T: 128 states of 128 bytes
  static constexpr uint32_t kQ = kP + 2 * kTile * 128;      // 64 elements of N rows, twice where DP is 128
  static constexpr uint32_t kStats = kQ + kHalves * N * 128;
  static constexpr uint32_t kBars = kStats + 8 * N * 4 + N * 8;
  static constexpr uint32_t kControl = kBars + 8 * (2 * kSlots + 8);
  static constexpr uint32_t kBytes = kControl + 256;
  // Tensor memory columns.  P^T of 64 rows fills a line of 128 bytes, that of fewer leaves the rest of it unused.
  static constexpr uint32_t kS = 0, kO = 2 * N;
  static constexpr uint32_t kColumns = N == 64 ? 256 : N == 32 ? 128 : 64;
  // With head_dim 64 the product has 128 rows all the same; what the upper 64 hold is read from behind the tile (there is
  // always something of this CTA's there) and never looked at.
  static constexpr uint32_t kLeading = kHalf;
  static_assert(kBars % 8 == 0 && kBytes <= 227 * 1024, "shared memory");
};
// Floats of a partial sum: O^T row by row, then a maximum and a sum for each.
template <int DP> constexpr uint32_t kPartial = kFewRows * DP + 2 * kFewRows;

// What a call is about beside the sizes it shares with the paged attention.
struct cross_args {
  preba_pages_attend_t p;
  const int32_t* cu_k;
  const int32_t* seen;
  uint32_t states, group, grid;
#if defined(PREBA_CHECKED)
  wait_limits_t limits = wait_limits();
#endif
};

struct piece_t {
  int32_t live;          // 0: none
  uint32_t request, head;
  uint32_t first, last;  // CTAs that hold pieces of the same (request, key head)
};
struct run_t {
  uint32_t begin, end, per;  // units of one tile of one key head; units per CTA
  uint32_t request, offset;  // of the first unit
};
struct control_t {
  run_t run;
  piece_t pieces[2];
  uint64_t warp_sums[kThreads / 32];
  uint32_t joins[2], tmem;
};
static_assert(sizeof(control_t) <= 256, "layout::kBytes");

__device__ __forceinline__ uint32_t tiles_of(const cross_args& a, const request_t& q, int32_t& hi) {
  if (q.rows == 0) return 0;
  hi = packed_seen(a.p.tokens, a.seen, q, 0, q.rows);
  return max(1, (hi + kTile - 1) / kTile);  // a request whose rows see nothing still has its zeros to write
}
__device__ __forceinline__ uint32_t units_of(const cross_args& a, uint32_t r) {
  request_t q;
  int32_t hi;
  return load_packed(a.p, a.cu_k, a.states, r, q) ? tiles_of(a, q, hi) * a.p.heads_kv : 0;
}

// Where a CTA's run begins: the block adds up the tiles of all requests, each thread of a run of them.
__device__ __forceinline__ void find_run(const cross_args& a, control_t& ctl) {
  const preba_pages_attend_t& p = a.p;
  const uint32_t chunk = (p.n + kThreads - 1) / kThreads;
  const uint32_t r0 = min(threadIdx.x * chunk, p.n), r1 = min(r0 + chunk, p.n);
  uint64_t mine = 0;
  for (uint32_t r = r0; r < r1; ++r) {
    mine += units_of(a, r);
    request_t q;
    if (blockIdx.x == 0 && !load_packed(p, a.cu_k, a.states, r, q)) report(p.status, PREBA_ERR_BAD_TABLE);
  }
  uint64_t incl = mine;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t up = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) ctl.warp_sums[warp] = incl;
  __syncthreads();
  uint64_t sum = 0, before = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += ctl.warp_sums[w];
    sum += ctl.warp_sums[w];
  }
  // requests that do not overlap never come to more (the host has seen to it); if they do, nothing is done
  if (sum > kMostUnits && blockIdx.x == 0 && threadIdx.x == 0) report(p.status, PREBA_ERR_BAD_TABLE);
  const uint32_t total = sum > kMostUnits ? 0 : static_cast<uint32_t>(sum);
  const uint32_t per = max(kMinTiles, (total + gridDim.x - 1) / gridDim.x);
  const uint32_t begin = min(static_cast<uint64_t>(blockIdx.x) * per, static_cast<uint64_t>(total));
  uint64_t at = before + incl - mine;
  if (threadIdx.x == 0) {
    ctl.run.begin = begin;
    ctl.run.end = min(begin + per, total);
    ctl.run.per = per;
  }
  if (begin < total && begin >= at && begin < at + mine) {
    uint32_t r = r0;
    for (;; ++r) {
      const uint32_t units = units_of(a, r);
      if (begin < at + units) break;
      at += units;
    }
    ctl.run.request = r;
    ctl.run.offset = static_cast<uint32_t>(begin - at);
  }
  __syncthreads();
}

// Walks a CTA's run piece by piece; every warp does so for itself.
struct walk_t {
  uint32_t unit, end, request, offset;  // next unit; offset within the request
  request_t q;
  int32_t hi;                           // states that some row sees
  uint32_t tiles, head, tile, count;    // of the current piece
  __device__ __forceinline__ explicit walk_t(const run_t& run)
      : unit(run.begin), end(run.end), request(run.request), offset(run.offset) {}
  __device__ __forceinline__ bool next(const cross_args& a) {
    if (unit >= end) return false;
    for (;; ++request, offset = 0) {    // ends: unit < end, so a later request has tiles
      if (!load_packed(a.p, a.cu_k, a.states, request, q)) continue;
      tiles = tiles_of(a, q, hi);
      if (offset < tiles * a.p.heads_kv) break;
    }
    head = offset / tiles;
    tile = offset - head * tiles;
    count = min(tiles - tile, end - unit);
    unit += count;
    offset += count;
    return true;
  }
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

template <int DP> __device__ __forceinline__ float* partial_of(const cross_args& a, uint32_t cta, uint32_t slot) {
  if (!PREBA_IN_RANGE(a.p.status, 2 * cta + slot < 2 * kMaxTileCtas)) cta = slot = 0;
  return reinterpret_cast<float*>(static_cast<uint8_t*>(a.p.workspace) + kCounterBytes) +
         static_cast<uint64_t>(2 * cta + slot) * kPartial<DP>;
}

template <typename T, int DP, int N>
__global__ void __launch_bounds__(kThreads, 1)
cross_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
             const __grid_constant__ cross_args a) {
  using L = layout<DP, N>;
  extern __shared__ __align__(1024) uint8_t smem[];
  const preba_pages_attend_t& p = a.p;
  const int lane = threadIdx.x & 31;
  const int warp = __shfl_sync(kFull, threadIdx.x >> 5, 0);
  const uint32_t base = smem_addr(smem);
  const uint32_t kv_full = base + L::kBars, kv_empty = kv_full + 8 * L::kSlots;
  const uint32_t q_full = kv_empty + 8 * L::kSlots, drained = q_full + 8;
  const uint32_t s_full = drained + 8, p_full = s_full + 16, o_done = p_full + 16;  // two each
  control_t& ctl = *reinterpret_cast<control_t*>(smem + L::kControl);

  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kSlots; ++s) {
      mbar_init(kv_full + 8 * s, 1);
      mbar_init(kv_empty + 8 * s, 1);
    }
    mbar_init(q_full, kSoftWarps);
    mbar_init(drained, 1);
    for (int x = 0; x < 2; ++x) {
      mbar_init(s_full + 8 * x, 1);
      mbar_init(p_full + 8 * x, kSoftWarps);
      mbar_init(o_done + 8 * x, 1);
    }
    ctl.pieces[0].live = ctl.pieces[1].live = 0;
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  chained_begin();
  // Only now: a kernel before this one that has let it in may still have its tensor memory to allocate, and
  // would wait for this CTA as this CTA waits for it.
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&ctl.tmem)),
                 "n"(L::kColumns)
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
    const bool mine = half < L::kHalves;
    const uint32_t dst = half * L::kHalf + chunk * kStateRows * 128;
    walk_t w(run);
    uint32_t slot = 0, phase = 1, issued = 0;  // a fresh barrier counts as emptied
    while (ok && w.next(a)) {
      const int32_t state0 = a.cu_k[w.request];
      int32_t key = w.tile * kTile + chunk * kStateRows;
      for (uint32_t t = 0; t < w.count && ok; ++t, key += kTile) {
        const bool want = mine && key < w.hi;
        const uint32_t bytes = __popc(__ballot_sync(kFull, want)) * kStateRows * 128;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          ok = ok && wait(kv_empty + 8 * slot, phase);
          if (!ok) break;
          if (lane == 0) mbar_arrive_expect_tx(kv_full + 8 * slot, bytes);
          __syncwarp();
          if (want)
            tensor_copy(base + slot * L::kSlot + dst, v ? &map_v : &map_k, half * 64, state0 + key, w.head, 0,
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
    }
  } else if (warp == kMmaWarp) {
    // ---- matrix products: one lane issues, the warp clears values that nobody sees
    constexpr uint32_t kQkShape = shape<T>(N, false), kPvShape = shape<T>(N, true);
    walk_t w(run);
    uint32_t slot = 0, phase = 0, q_phase = 0;
    uint32_t n_s = 0, n_p = 0;  // tiles so far
    auto step = [&]() {
      const uint32_t s = slot;
      if (++slot == L::kSlots) slot = 0, phase ^= 1;
      return s;
    };
    auto qk = [&]() {
      ok = ok && wait(kv_full + 8 * slot, phase);
      if (!ok) return;
      fence_after();
      const uint32_t k_slot = step();
      const uint32_t k_op = __shfl_sync(kFull, operand(base + k_slot * L::kSlot, 16), 0);
      const uint32_t q_op = __shfl_sync(kFull, operand(base + L::kQ, 16), 0);
      const uint32_t d = __shfl_sync(kFull, tmem + L::kS + (n_s & 1) * N, 0);
      if (elected()) {
#pragma unroll
        for (int ks = 0; ks < DP / 16; ++ks)
          mma_ss(d, k_op + (((ks / 4) * L::kHalf + (ks % 4) * 32) >> 4), q_op + (((ks / 4) * N * 128 + (ks % 4) * 32) >> 4),
                 kQkShape, ks > 0);
        mma_commit(s_full + 8 * (n_s & 1));
        mma_commit(kv_empty + 8 * k_slot);
      }
      __syncwarp();
      ++n_s;
    };
    while (ok && w.next(a)) {
      ok = wait(q_full, q_phase);
      if (!ok) break;
      q_phase ^= 1;
      fence_after();
      qk();
      for (uint32_t t = 0; t < w.count && ok; ++t) {
        // values come before the next keys; the scores of the next tile are made while this one's are looked at
        const uint32_t v_slot = slot, v_phase = phase;
        step();
        if (t + 1 < w.count) qk();
        ok = ok && wait(kv_full + 8 * v_slot, v_phase);
        if (!ok) break;
        const int32_t seen = w.hi - static_cast<int32_t>((w.tile + t) * kTile);
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
        const uint32_t v_op = __shfl_sync(kFull, operand(base + v_slot * L::kSlot, L::kLeading), 0);
        const uint32_t p_op = __shfl_sync(kFull, operand(base + L::kP + b * kTile * 128, 16), 0);
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
    while (w.next(a)) {
      const int32_t rows = w.q.rows * a.group;
      const bool go = !soft_any(!ok);
      ok = go;
      // queries, 16 bytes at a time; rows that are not there are 0 and take part in nothing
      for (int i = r; i < N * (DP / 8); i += kSoftThreads) {
        const int row = i / (DP / 8), e = i % (DP / 8) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < rows && e < static_cast<int>(p.head_dim)) {
          const uint32_t j = row / a.group, h = w.head * a.group + row - j * a.group;
          v = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + (w.q.row + j) * p.q_stride[0] + h * p.q_stride[1] + e);
        }
        *reinterpret_cast<uint4*>(smem + L::kQ + e / 64 * N * 128 + row * 128 + ((e / 8 % 8 ^ (row & 7)) << 4)) = v;
      }
      float m = -INFINITY;  // of row r, where there is one: the largest score of those looked at when it grew last
      int32_t hi = 0;
      if (r < N) {
        const uint32_t j = r / a.group, h = w.head * a.group + r - j * a.group;
        if (r < rows) hi = packed_seen(p.tokens, a.seen, w.q, j, j + 1);
        row_hi[r] = hi;
        row_at[r] = r < rows ? (w.q.row + j) * p.out_stride[0] + h * p.out_stride[1] : 0;
        ref[r] = 0.f;
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      fence_before();
      if (lane == 0) mbar_arrive(q_full);
      soft_sync();  // what every row sees is there
      int32_t all = w.hi;  // states that every row sees
      if (a.seen)
        for (int c = 0; c < rows; ++c) all = min(all, row_hi[c]);
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
        ok = ok && wait(s_full + 8 * b, (n >> 1) & 1);
        fence_after();
        scores();
        // a row that sees a state and has no reference yet gets one
        if (soft_any(exponents() > kGrowth || (m == -INFINITY && hi > 0) || !ok)) {
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
            ref[r] = to == -INFINITY ? 0.f : to;
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
        uint8_t* to = smem + L::kP + b * kTile * 128 + r * 128;
#pragma unroll
        for (int c = 0; c < N; c += 8) {
          uint32_t e[4];
#pragma unroll
          for (int i = 0; i < 8; i += 2) {
            const float z0 = exp2_approx(__uint_as_float(s[c + i])), z1 = exp2_approx(__uint_as_float(s[c + i + 1]));
            l[c + i] += z0, l[c + i + 1] += z1;
            e[i / 2] = pack2<T>(z0, z1);
          }
          if (ok) *reinterpret_cast<uint4*>(to + ((c / 8 ^ (r & 7)) << 4)) = make_uint4(e[0], e[1], e[2], e[3]);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        fence_before();
        __syncwarp();
        if (ok && lane == 0) mbar_arrive(p_full + 8 * b);
      }
      // ---- the piece is over: the threads' sums are joined
      ok = ok && wait(o_done + 8 * ((n - 1) & 1), ((n - 1) >> 1) & 1);
      fence_after();
      uint32_t o[N];
      tmem_load<N>(o, tmem + lanes + L::kO);
      fence_before();
      sum_columns<N>(l);
#pragma unroll
      for (int i = 0; i < (N + 31) / 32; ++i) stats[warp * N + column_of<N>(i)] = l[i];
      soft_sync();
      const bool whole = w.count == w.tiles;
      const uint32_t piece = w.tile == 0;
      float* part = partial_of<DP>(a, blockIdx.x, piece);
      if (r < rows) {
        const float sum = (stats[r] + stats[N + r]) + (stats[2 * N + r] + stats[3 * N + r]);
        if (whole) {
          keep[r] = inverse_of(sum);
          const uint32_t j = r / a.group, h = w.head * a.group + r - j * a.group;
          if (p.lse && PREBA_IN_RANGE(p.status, w.q.row + j < p.tokens))
            p.lse[static_cast<uint64_t>(w.q.row + j) * p.heads_q + h] = row_lse(m, sum);
        } else {
          reinterpret_cast<float2*>(part + kFewRows * DP)[r] = make_float2(marked(m, sum), sum);
        }
      }
      soft_sync();
      if (whole) {
        if (r < static_cast<int>(p.head_dim)) {
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (c < rows) static_cast<T*>(p.out)[row_at[c] + r] = result_of<T>(__uint_as_float(o[c]), keep[c]);
        }
      } else {
        if (r < DP) {
#pragma unroll
          for (int c = 0; c < N; ++c)
            if (c < rows) part[c * DP + r] = __uint_as_float(o[c]);
        }
        if (r == 0) {
          const uint32_t start = w.unit - w.count - w.tile;  // of the (request, key head)
          ctl.pieces[piece] = {1, w.request, w.head, start / run.per, (start + w.tiles - 1) / run.per};
        }
      }
      soft_sync();  // what lies in shared memory has been read
    }
    if (!ok) report(p.status, PREBA_ERR_TIMEOUT);

    // ---- join the CTAs: whoever finishes a (request, key head) last adds its pieces up
    if (ctl.pieces[0].live || ctl.pieces[1].live) {
      __threadfence();
      soft_sync();
      uint32_t* counters = static_cast<uint32_t*>(p.workspace);
      if (r < 2) {
        const piece_t& x = ctl.pieces[r];
        uint32_t last = 0;
        if (x.live) {
          last = atomicAdd(&counters[x.first], 1) == x.last - x.first;
          if (last) counters[x.first] = 0;  // as the next call wants it
          __threadfence();
        }
        ctl.joins[r] = last;
      }
      soft_sync();
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        if (!ctl.joins[i]) continue;
        const piece_t x = ctl.pieces[i];
        request_t q;
        load_packed(p, a.cu_k, a.states, x.request, q);
        const int32_t rows = q.rows * a.group;
        // a thread per element, rows in turn; pieces in the order of the states.  The first CTA's piece begins the
        // (request, key head) and lies in its slot 1, the others in slot 0
#pragma unroll 1
        for (int c = DP == 64 ? r / 64 : 0; c < rows; c += DP == 64 ? 2 : 1) {
          const int e = r % DP;
          float top = -INFINITY, sum = 0.f, acc = 0.f;
#pragma unroll 1
          for (uint32_t k = x.first; k <= x.last; k += 8) {
            float2 stat[8];
            float part[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const uint32_t cta = min(k + u, x.last);  // the last one again: it is not counted
              const float* from = partial_of<DP>(a, cta, cta == x.first);
              stat[u] = __ldcg(reinterpret_cast<const float2*>(from + kFewRows * DP) + c);
              part[u] = __ldcg(from + c * DP + e);
            }
            float to = top;
#pragma unroll
            for (int u = 0; u < 8; ++u) to = fmaxf(to, stat[u].x);
            const float keep = to == -INFINITY ? 0.f : exp2_approx(top - to);
            top = to;
            sum *= keep, acc *= keep;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const float weight = k + u > x.last || stat[u].x == -INFINITY ? 0.f : exp2_approx(stat[u].x - to);
              if (weight != 0.f) {  // a piece that saw nothing left no sums
                sum = fmaf(weight, stat[u].y, sum);
                acc = fmaf(weight, part[u], acc);
              }
            }
          }
          const uint32_t j = c / a.group, h = x.head * a.group + c - j * a.group, tok = q.row + j;
          if (!PREBA_IN_RANGE(p.status, tok < p.tokens)) continue;
          if (e < static_cast<int>(p.head_dim))
            static_cast<T*>(p.out)[tok * p.out_stride[0] + h * p.out_stride[1] + e] = result_of<T>(acc, inverse_of(sum));
          if (p.lse && e == 0) p.lse[static_cast<uint64_t>(tok) * p.heads_q + h] = row_lse(top, sum);
        }
      }
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (warp == kMmaWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(L::kColumns) : "memory");
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

template <typename T, int DP, int N> cudaError_t launch_cross(const cross_args& a, cudaStream_t stream) {
  using L = layout<DP, N>;
  CUtensorMap map_k, map_v;
  cudaError_t err = states_map(&map_k, a.p, a.states, a.p.k_cache, a.p.k_stride, kStateRows);
  if (err == cudaSuccess) err = states_map(&map_v, a.p, a.states, a.p.v_cache, a.p.v_stride, kStateRows);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(cross_kernel<T, DP, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kBytes);
  if (err != cudaSuccess) return err;
  return launch_chained(cross_kernel<T, DP, N>, a.grid, kThreads, L::kBytes, stream, map_k, map_v, a);
}
template <typename T, int DP> cudaError_t launch_cross(const cross_args& a, uint32_t rows, cudaStream_t stream) {
  return rows <= 16 ? launch_cross<T, DP, 16>(a, stream) : rows <= 32 ? launch_cross<T, DP, 32>(a, stream)
                                                                      : launch_cross<T, DP, 64>(a, stream);
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
      static_cast<double>(c.heads_kv) * (c.n + c.states / 128.0) > kMostUnits || !(c.scale > 0.f) || !(c.scale < INFINITY) ||
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
  if (rows > kFewRows)
    return finish(launch_packed_tiles(p, c.cu_k, c.seen, c.states, sms, static_cast<uint8_t*>(c.workspace) + kCounterBytes, s));
  const cross_args a{p, c.cu_k, c.seen, c.states, group, static_cast<uint32_t>(std::min(sms, kMaxTileCtas))};
  const uint32_t few = static_cast<uint32_t>(rows);
  if (c.dtype == PREBA_F16)
    return finish(c.head_dim <= 64 ? launch_cross<__half, 64>(a, few, s) : launch_cross<__half, 128>(a, few, s));
  return finish(c.head_dim <= 64 ? launch_cross<__nv_bfloat16, 64>(a, few, s) : launch_cross<__nv_bfloat16, 128>(a, few, s));
}
