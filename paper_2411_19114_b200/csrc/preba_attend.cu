// Attention of a step's tokens over the paged cache (preba_tokens.h): preba_pages_attend.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "preba_attend.h"
#include "preba_attend_plan.h"

namespace preba {
namespace {

using namespace attend;

// ---- few rows: at most 16 (token, head) rows on a key head -----------------------------------------
//
// Such a step has to read the keys and values once and does 4 flops per byte and row with them, far
// below what the matrix instructions give: bytes bound it.  So all rows of a key head share one 16-row
// fragment and every CTA streams tiles of 64 keys through a ring of tensor copies, 64 KB or more on the
// way per SM at any time.  The work is one line of tiles, request by request and key head by key head;
// the CTAs take equal runs of it, whatever the lengths are, and a (request, key head) that crosses
// CTAs is left as partial sums that the last of them to finish joins, in the order of the keys, so that
// timing does not change a bit.  Within a tile each of the four warps takes 16 keys with a running maximum
// and sum of its own; the warps are joined once per (request, key head).  128 single tokens over up to 8192
// keys of 8 heads of 128: 277 to 281 us (1762 MB, 6.3 TB/s; a copy reaches 6.56); 4 of them over up to 2048
// keys: 13 us, which the launch, the first loads (2.7 us), the partial sums' fence and count (1.5 us) and
// their join (2 to 3 us) take the most of.  Probabilities are rounded to 16 bits for the product, as the
// matrix instructions take them, their sums are not: with the one rounding of the result the error against
// 64 bits is up to 1.04 times that of the one rounding alone.

constexpr uint64_t kCounterBytes = kMaxSplitCtas * 4;  // at the workspace's start
constexpr int kRowsMax = 16;
constexpr int kTileKeys = 64;
constexpr int kWarps = 4;                      // of consumers; one more warp issues the copies
constexpr int kFewThreads = 32 * (kWarps + 1);
constexpr uint32_t kMinTiles = 2;              // a CTA's run is not shorter than this

template <int DP> struct few_layout {          // DP: head_dim rounded up to 64 or 128
  static constexpr int kHalves = DP / 64;
  static constexpr uint32_t kOperand = kTileKeys * DP * 2;  // bytes of a tile's keys (or values)
  static constexpr uint32_t kStage = 2 * kOperand;
  static constexpr int kStages = 3 * 128 / DP;
  static constexpr uint32_t kJoin = kStages * kStage;             // eight rows of each warp's sums
  static constexpr uint32_t kStats = kJoin + kWarps * 8 * DP * 4;  // the warps' maxima and sums
  static constexpr uint32_t kBars = kStats + kWarps * 2 * kRowsMax * 4;
  static constexpr uint32_t kControl = kBars + 2 * kStages * 8;
  static constexpr uint32_t kBytes = kControl + 128;
  static constexpr uint32_t kPartial = kRowsMax * DP * 4 + 2 * kRowsMax * 4;  // of one partial sum
};

// A piece of a CTA's run that is left as a partial sum.
struct piece_t {
  int32_t live;       // 0: none
  uint32_t request, head;
  uint32_t first, last;  // CTAs that hold pieces of the same (request, key head)
};

// What the CTA's threads share beside the ring (in the dynamic memory: two CTAs fill an SM's).
struct run_t {
  uint32_t begin, end, per;  // units of one tile of one key head; units per CTA
  uint32_t request, offset;  // of the first unit
};
struct control_t {
  run_t run;
  piece_t pieces[2];
  uint32_t warp_sums[kWarps + 1], joins[2];
};
static_assert(sizeof(control_t) <= 128, "few_layout::kBytes");

struct few_args {
  preba_pages_attend_t p;
  uint32_t page_shift, group, box_rows, box_shift;
#if defined(PREBA_CHECKED)
  wait_limits_t limits = wait_limits();
#endif
};

__device__ __forceinline__ uint32_t few_tiles(const preba_pages_attend_t& p, const request_t& q,
                                              int32_t& lo, int32_t& hi) {
  if (q.rows == 0) return 0;
  seen_by(p, q, 0, q.rows, lo, hi);
  // a request whose rows see nothing still has its zeros to write
  return max(1, (hi + kTileKeys - 1) / kTileKeys - lo / kTileKeys);
}

__device__ __forceinline__ uint32_t few_tiles_of(const preba_pages_attend_t& p, uint32_t r) {
  request_t q;
  int32_t lo, hi;
  if (!load_request(p, r, q)) return 0;
  return few_tiles(p, q, lo, hi);
}

// Where a CTA's run begins: the block adds up the tiles of all requests, each thread of a run of them.
__device__ __forceinline__ void find_run(const few_args& a, run_t* run, uint32_t* warp_sums) {
  const preba_pages_attend_t& p = a.p;
  const uint32_t chunk = (p.n + kFewThreads - 1) / kFewThreads;
  const uint32_t r0 = min(threadIdx.x * chunk, p.n), r1 = min(r0 + chunk, p.n);
  uint32_t mine = 0;
  for (uint32_t r = r0; r < r1; ++r) {
    mine += few_tiles_of(p, r) * p.heads_kv;
    if (blockIdx.x == 0) {
      request_t q;
      if (!load_request(p, r, q)) report(p.status, PREBA_ERR_BAD_TABLE);
    }
  }
  uint32_t incl = mine;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t up = __shfl_up_sync(kFull, incl, o);
    if (lane >= o) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  uint32_t total = 0, before = 0;
#pragma unroll
  for (int w = 0; w <= kWarps; ++w) {
    if (w < warp) before += warp_sums[w];
    total += warp_sums[w];
  }
  const uint32_t per = max(kMinTiles, (total + gridDim.x - 1) / gridDim.x);
  const uint32_t begin = min(static_cast<uint64_t>(blockIdx.x) * per, static_cast<uint64_t>(total));
  uint32_t at = before + incl - mine;
  if (threadIdx.x == 0) {
    run->begin = begin;
    run->end = min(begin + per, total);
    run->per = per;
  }
  if (begin < total && begin >= at && begin < at + mine) {
    uint32_t r = r0;
    for (;; ++r) {
      const uint32_t units = few_tiles_of(p, r) * p.heads_kv;
      if (begin < at + units) break;
      at += units;
    }
    run->request = r;
    run->offset = begin - at;
  }
  __syncthreads();
}

// Walks a CTA's run piece by piece; every warp does so for itself.
struct walk_t {
  uint32_t unit, end, request, offset;  // next unit; offset within the request
  request_t q;
  int32_t lo, hi;
  uint32_t tiles, head, tile, count;    // of the current piece
  __device__ __forceinline__ bool next(const few_args& a) {
    if (unit >= end) return false;
    for (;; ++request, offset = 0) {    // ends: unit < end, so a later request has tiles
      if (!load_request(a.p, request, q)) continue;
      tiles = few_tiles(a.p, q, lo, hi);
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

template <typename T>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<__half>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                              uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<__nv_bfloat16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0,
                                                     uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void consumers_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(32 * kWarps) : "memory");
}

// The result of rows lane/4 and lane/4 + 8 from sums over eight columns each (the fragment layout of
// the matrix instruction), with their sums l and maxima m in units of log2.
template <typename T, int TILES>
__device__ __forceinline__ void store_rows(const few_args& a, const request_t& q, uint32_t head,
                                           const float (&o)[TILES][4], const float (&l)[2],
                                           const float (&m)[2], int first_tile) {
  const preba_pages_attend_t& p = a.p;
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t row = (lane >> 2) + 8 * i;
    if (row >= q.rows * a.group) continue;
    if (!PREBA_IN_RANGE(p.status, static_cast<uint32_t>(q.row) + row / a.group < p.tokens)) continue;
    const uint32_t j = row / a.group, h = head * a.group + row - j * a.group, t = q.row + j;
    const float inv = l[i] > 0.f ? 1.f / l[i] : 0.f;
    T* to = static_cast<T*>(p.out) + t * p.out_stride[0] + h * p.out_stride[1];
#pragma unroll
    for (int n = 0; n < TILES; ++n) {
      const uint32_t e = 8 * (first_tile + n) + 2 * (lane & 3);
      if (e < p.head_dim)
        *reinterpret_cast<uint32_t*>(to + e) = pack2<T>(o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
    }
    if (p.lse && first_tile == 0 && (lane & 3) == 0)
      p.lse[static_cast<uint64_t>(t) * p.heads_q + h] = row_lse(m[i], l[i]);
  }
}

// Partial sums of a CTA's first (slot 0) or last piece: pairs of columns in the fragment layout, rows 0 to
// 7, then rows 8 to 15, then a maximum and a sum for each row.
template <int DP> __device__ __forceinline__ float2* partial_of(const preba_pages_attend_t& p, uint32_t cta, uint32_t slot) {
  if (!PREBA_IN_RANGE(p.status, 2 * cta + slot < 2 * kMaxSplitCtas)) cta = slot = 0;
  return reinterpret_cast<float2*>(static_cast<uint8_t*>(p.workspace) + kCounterBytes +
                                   static_cast<uint64_t>(2 * cta + slot) * few_layout<DP>::kPartial);
}

template <typename T, int DP>
__global__ void __launch_bounds__(kFewThreads, 2)
few_rows_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                const __grid_constant__ few_args a) {
  using L = few_layout<DP>;
  constexpr int kTiles = DP / 8 / kWarps;  // column groups of a warp where the work is split by columns
  extern __shared__ __align__(1024) uint8_t smem[];
  const preba_pages_attend_t& p = a.p;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t base = smem_addr(smem), bars = base + L::kBars;
  const uint32_t full = bars, empty = bars + 8 * L::kStages;
  control_t& ctl = *reinterpret_cast<control_t*>(smem + L::kControl);
  if (threadIdx.x == 0) {
    for (int s = 0; s < L::kStages; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(empty + 8 * s, kWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    ctl.pieces[0].live = ctl.pieces[1].live = 0;
  }
  chained_begin();
  find_run(a, &ctl.run, ctl.warp_sums);  // synchronises
  const run_t run = ctl.run;
  waits_t wait(a);
  if (run.begin >= run.end) return;
  walk_t w;
  w.unit = run.begin;
  w.end = run.end;
  w.request = run.request;
  w.offset = run.offset;

  if (warp == kWarps) {
    // ---- copies: a lane per box (a page's keys or values, 64 elements wide)
    const uint32_t boxes = kTileKeys >> a.box_shift;  // of a tile, along the keys
    const uint32_t chunk = lane & (boxes - 1), part = lane / boxes;
    const uint32_t half = part % L::kHalves, values = part / L::kHalves;
    const bool mine = values < 2;
    const uint32_t dst = values * L::kOperand + half * (kTileKeys * 128) + (chunk << a.box_shift) * 128;
    uint32_t stage = 0, phase = 1;  // a fresh barrier counts as emptied
    uint32_t issued = 0;
    bool ok = true;
    while (ok && w.next(a)) {
      const int32_t* row = p.block_table + static_cast<uint64_t>(w.request) * p.table_stride;
      const int32_t tile0 = w.lo / kTileKeys + w.tile;
      int32_t key = tile0 * kTileKeys + (chunk << a.box_shift);
      auto entry = [&](int32_t k) {
        return mine && k < w.hi && k + static_cast<int32_t>(a.box_rows) > w.lo ? row[k >> a.page_shift] : 0;
      };
      int32_t page = entry(key);
      for (uint32_t t = 0; t < w.count; ++t, key += kTileKeys) {
        const bool wanted = mine && key < w.hi && key + static_cast<int32_t>(a.box_rows) > w.lo;
        int32_t from = page;
        if (t + 1 < w.count) page = entry(key + kTileKeys);
        ok = wait(empty + 8 * stage, phase);
        if (!ok) break;
        const uint32_t count = __popc(__ballot_sync(kFull, wanted));
        if (lane == 0) mbar_arrive_expect_tx(full + 8 * stage, count * a.box_rows * 128);
        __syncwarp();
        if (wanted) {
          if (from < 0 || static_cast<uint32_t>(from) >= p.pages) {
            report(p.status, PREBA_ERR_BAD_TABLE);
            from = p.pages;  // beyond the tensor: the box is filled with zeros
          }
          tensor_copy(base + stage * L::kStage + dst, values ? &map_v : &map_k, half * 64,
                      key & (p.page_size - 1), w.head, from, full + 8 * stage);
        }
        ++issued;
        if (++stage == L::kStages) stage = 0, phase ^= 1;
      }
    }
    if (!ok) {
      report(p.status, PREBA_ERR_TIMEOUT);
      // the copies in flight land before the CTA's memory goes to another: wait for those not
      // known to have been read, oldest first
      const uint32_t pending = min(issued, static_cast<uint32_t>(L::kStages));
      for (uint32_t i = issued - pending; i < issued; ++i)
        mbar_wait(full + 8 * (i % L::kStages), (i / L::kStages) & 1);
    }
    return;
  }

  // ---- consumers
  const float scale = p.scale * kLog2e;
  uint32_t stage = 0, phase = 0;
  bool ok = true;
  float o[DP / 8][4], m[2], l[2];
  const uint32_t k_lane = (16 * warp + (lane >> 4) * 8 + (lane & 7)) * 128;
  const uint32_t v_lane = (16 * warp + ((lane >> 3) & 1) * 8 + (lane & 7)) * 128;
  while (w.next(a)) {
    const int32_t rows = w.q.rows * a.group;
    uint32_t qf[DP / 16][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t row = (lane >> 2) + 8 * i;
      const bool in = row < rows;
      const uint32_t j = in ? row / a.group : 0, h = in ? row - j * a.group : 0;
      const T* from = static_cast<const T*>(p.q) + (w.q.row + j) * p.q_stride[0] +
                      (w.head * a.group + h) * p.q_stride[1];
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        const uint32_t e = 16 * ks + 2 * (lane & 3);
        qf[ks][i] = in && e < p.head_dim ? *reinterpret_cast<const uint32_t*>(from + e) : 0;
        qf[ks][2 + i] = in && e + 8 < p.head_dim ? *reinterpret_cast<const uint32_t*>(from + e + 8) : 0;
      }
    }
    int32_t row_lo[2], row_hi[2];
    const int32_t at0 = w.q.keys - w.q.rows;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int32_t row = (lane >> 2) + 8 * i;
      row_lo[i] = row_hi[i] = 0;
      if (row < rows) seen_by(p, w.q, row / a.group, row / a.group + 1, row_lo[i], row_hi[i]);
    }
    // keys in [all_lo, all_hi) are seen by every row
    const int32_t all_hi = (p.flags & PREBA_ATTEND_CAUSAL) ? min(w.q.keys, at0 + 1) : w.q.keys;
    const int32_t all_lo = p.window ? static_cast<int32_t>(max(static_cast<int64_t>(0),
                                          static_cast<int64_t>(w.q.keys) - p.window)) : 0;
#pragma unroll
    for (int n = 0; n < DP / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
    int32_t key0 = (w.lo / kTileKeys + w.tile) * kTileKeys + 16 * warp;
    for (uint32_t t = 0; t < w.count && ok; ++t, key0 += kTileKeys) {
      ok = wait(full + 8 * stage, phase);
      if (!ok) break;
      const uint32_t ks_base = base + stage * L::kStage, vs_base = ks_base + L::kOperand;
      float s[2][4] = {};
#pragma unroll
      for (int ks = 0; ks < DP / 16; ++ks) {
        uint32_t b[4];
        const uint32_t chunk = (ks & 3) * 2 + ((lane >> 3) & 1);
        ldm4(b, ks_base + (ks >> 2) * (kTileKeys * 128) + k_lane + ((chunk ^ (lane & 7)) << 4));
        mma16<T>(s[0], qf[ks], b[0], b[1]);
        mma16<T>(s[1], qf[ks], b[2], b[3]);
      }
      const bool whole = key0 >= all_lo && key0 + 16 <= all_hi;  // the same for the whole warp
      uint32_t keep0 = kFull, keep1 = kFull;
      if (!whole) {
        const int32_t k = key0 + 2 * (lane & 3);
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int32_t key = k + 8 * n + (c & 1);
            if (key < row_lo[c >> 1] || key >= row_hi[c >> 1]) s[n][c] = -INFINITY;
          }
        // values that no row sees may be anything: they are cleared, 0 times NaN would be NaN
        auto seen = [&](int32_t key) { return key >= w.lo && key < w.hi; };
        keep0 = (seen(k) ? 0xffffu : 0u) | (seen(k + 1) ? 0xffff0000u : 0u);
        keep1 = (seen(k + 8) ? 0xffffu : 0u) | (seen(k + 9) ? 0xffff0000u : 0u);
      }
      uint32_t pf[4];
      float top[2], shift[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float x = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
        x = fmaxf(x, __shfl_xor_sync(kFull, x, 1));
        x = fmaxf(x, __shfl_xor_sync(kFull, x, 2));
        top[i] = fmaxf(m[i], x * scale);
      }
      if (__any_sync(kFull, top[0] > m[0] || top[1] > m[1])) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          // nothing seen yet: both are -inf, and so are the sums 0
          const float keep = top[i] == -INFINITY ? 0.f : exp2_approx(m[i] - top[i]);
          m[i] = top[i];
          l[i] *= keep;
#pragma unroll
          for (int n = 0; n < DP / 8; ++n) o[n][2 * i] *= keep, o[n][2 * i + 1] *= keep;
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        shift[i] = m[i] == -INFINITY ? 0.f : m[i];
        float e[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) e[c] = exp2_approx(fmaf(s[c >> 1][2 * i + (c & 1)], scale, -shift[i]));
        l[i] += (e[0] + e[1]) + (e[2] + e[3]);
        pf[i] = pack2<T>(e[0], e[1]);
        pf[2 + i] = pack2<T>(e[2], e[3]);
      }
#pragma unroll
      for (int n = 0; n < DP / 16; ++n) {
        uint32_t b[4];
        const uint32_t chunk = (n & 3) * 2 + (lane >> 4);
        ldm4t(b, vs_base + (n >> 2) * (kTileKeys * 128) + v_lane + ((chunk ^ (lane & 7)) << 4));
        if (!whole) b[0] &= keep0, b[1] &= keep1, b[2] &= keep0, b[3] &= keep1;
        mma16<T>(o[2 * n], pf, b[0], b[1]);
        mma16<T>(o[2 * n + 1], pf, b[2], b[3]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty + 8 * stage);
      if (++stage == L::kStages) stage = 0, phase ^= 1;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(kFull, l[i], 1);
      l[i] += __shfl_xor_sync(kFull, l[i], 2);
    }
    // ---- join the warps: every warp lays its sums down, scaled to the common maximum, eight rows at a
    // time, and adds up a quarter of the columns of all four
    float* join = reinterpret_cast<float*>(smem + L::kJoin);
    float* stats = reinterpret_cast<float*>(smem + L::kStats);
    if ((lane & 3) == 0)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        stats[(2 * warp + 0) * kRowsMax + (lane >> 2) + 8 * i] = marked(m[i], l[i]);
        stats[(2 * warp + 1) * kRowsMax + (lane >> 2) + 8 * i] = l[i];
      }
    consumers_sync();
    float mine[2] = {m[0], m[1]};
    float r[kTiles][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float part[kWarps];
#pragma unroll
      for (int k = 0; k < kWarps; ++k) part[k] = stats[2 * k * kRowsMax + (lane >> 2) + 8 * i];
      m[i] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
      l[i] = 0.f;
#pragma unroll
      for (int k = 0; k < kWarps; ++k)
        if (part[k] != -INFINITY)
          l[i] += exp2_approx(part[k] - m[i]) * stats[(2 * k + 1) * kRowsMax + (lane >> 2) + 8 * i];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int n = 0; n < kTiles; ++n) r[n][2 * i] = r[n][2 * i + 1] = 0.f;
      if (i == 1 && rows <= 8) break;
      const float keep = mine[i] == -INFINITY ? 0.f : exp2_approx(mine[i] - m[i]);
      float2* to = reinterpret_cast<float2*>(join) + warp * (DP / 8) * 32 + lane;
      if (i) consumers_sync();  // the first eight rows have been added up
#pragma unroll
      for (int n = 0; n < DP / 8; ++n) to[n * 32] = make_float2(o[n][2 * i] * keep, o[n][2 * i + 1] * keep);
      consumers_sync();
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float2 v = (reinterpret_cast<const float2*>(join) + lane)[(k * (DP / 8) + kTiles * warp + n) * 32];
          r[n][2 * i] += v.x;
          r[n][2 * i + 1] += v.y;
        }
    }
    if (w.count == w.tiles) {
      store_rows<T, kTiles>(a, w.q, w.head, r, l, m, kTiles * warp);
    } else {
      const uint32_t slot = w.tile == 0;
      float2* to = partial_of<DP>(p, blockIdx.x, slot) + lane;
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
        to[(kTiles * warp + n) * 32] = make_float2(r[n][0], r[n][1]);
        if (rows > 8) to[(DP / 8 + kTiles * warp + n) * 32] = make_float2(r[n][2], r[n][3]);
      }
      if (warp == 0 && (lane & 3) == 0)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          (to - lane)[kRowsMax * DP / 2 + (lane >> 2) + 8 * i] = make_float2(marked(m[i], l[i]), l[i]);
      if (threadIdx.x == 0) {
        const uint32_t start = w.unit - w.count - w.tile;  // of the (request, key head)
        ctl.pieces[slot] = {1, w.request, w.head, start / run.per, (start + w.tiles - 1) / run.per};
      }
    }
    consumers_sync();  // what the warps laid down has been read
  }
  if (!ok) report(p.status, PREBA_ERR_TIMEOUT);

  // ---- join the CTAs: whoever finishes a (request, key head) last adds its pieces up
  if (!ctl.pieces[0].live && !ctl.pieces[1].live) return;
  __threadfence();
  consumers_sync();
  uint32_t* counters = static_cast<uint32_t*>(p.workspace);
  if (threadIdx.x < 2) {
    const piece_t& x = ctl.pieces[threadIdx.x];
    uint32_t last = 0;
    if (x.live) {
      last = atomicAdd(&counters[x.first], 1) == x.last - x.first;
      if (last) counters[x.first] = 0;  // as the next call wants it
      __threadfence();
    }
    ctl.joins[threadIdx.x] = last;
  }
  consumers_sync();
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    if (!ctl.joins[i]) continue;
    const piece_t x = ctl.pieces[i];
    request_t q;
    load_request(p, x.request, q);
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f}, acc[kTiles][4] = {};
    // in the order of the keys, a few pieces at a time so that their loads are on the way together
    auto add = [&](auto count, auto first_row) {
      constexpr int N = decltype(count)::value, h = decltype(first_row)::value;
#pragma unroll 1
      for (uint32_t c = x.first; c <= x.last; c += N) {
        float2 stat[N], part[N][kTiles];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const uint32_t cta = min(c + k, x.last);  // the last one again: it is not counted
          // the first CTA's piece begins the (request, key head): slot 1; the others lie in slot 0
          const float2* from = partial_of<DP>(p, cta, cta == x.first);
          stat[k] = __ldcg(from + kRowsMax * DP / 2 + (lane >> 2) + 8 * h);
#pragma unroll
          for (int n = 0; n < kTiles; ++n) part[k][n] = __ldcg(from + (h * (DP / 8) + kTiles * warp + n) * 32 + lane);
        }
        float to = top[h];
#pragma unroll
        for (int k = 0; k < N; ++k) to = fmaxf(to, stat[k].x);
        const float keep = to == -INFINITY ? 0.f : exp2_approx(top[h] - to);
        top[h] = to;
        sum[h] *= keep;
#pragma unroll
        for (int n = 0; n < kTiles; ++n) acc[n][2 * h] *= keep, acc[n][2 * h + 1] *= keep;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float e = c + k > x.last || stat[k].x == -INFINITY ? 0.f : exp2_approx(stat[k].x - to);
          sum[h] = fmaf(e, stat[k].y, sum[h]);
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            acc[n][2 * h] = fmaf(e, part[k][n].x, acc[n][2 * h]);
            acc[n][2 * h + 1] = fmaf(e, part[k][n].y, acc[n][2 * h + 1]);
          }
        }
      }
    };
    using std::integral_constant;
    add(integral_constant<int, 8>(), integral_constant<int, 0>());
    if (q.rows * a.group > 8) add(integral_constant<int, 8>(), integral_constant<int, 1>());
    store_rows<T, kTiles>(a, q, x.head, acc, sum, top, kTiles * warp);
  }
}

bool sizes_ok(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv, uint32_t head_dim) {
  return n >= 1 && n <= PREBA_PAGES_MAX_REQUESTS && tokens >= 1 && tokens <= PREBA_PAGES_MAX_KEYS && heads_q >= 1 &&
         heads_q <= 65535 && heads_kv >= 1 && heads_q % heads_kv == 0 && heads_q / heads_kv <= 128 &&
         head_dim >= 8 && head_dim % 8 == 0 && head_dim <= PREBA_PAGES_MAX_HEAD_DIM;
}

// The workspace: a counter per CTA of the kernel for few rows, which every call leaves zeroed; then what
// one call needs, partial sums of that kernel or the list and the partial sums of the other.
uint64_t workspace_of(uint32_t n, uint32_t tokens, uint32_t group, uint32_t head_dim) {
  const uint64_t few = 2ull * kMaxSplitCtas * (head_dim <= 64 ? few_layout<64>::kPartial
                                                              : few_layout<128>::kPartial);
  return kCounterBytes + std::max(few, tiles_workspace(n, tokens, group, head_dim));
}

// cuTensorMapEncodeTiled, found through the runtime so that the library needs no libcuda to load.
using encode_fn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                               const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                               CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                               CUtensorMapFloatOOBfill);
cudaError_t encoder(encode_fn* fn) {
  static std::atomic<void*> found{nullptr};
  void* f = found.load(std::memory_order_relaxed);
  if (!f) {
    cudaDriverEntryPointQueryResult result;
    const cudaError_t err =
        cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &result);
    if (err != cudaSuccess) return err;
    if (result != cudaDriverEntryPointSuccess || !f) return cudaErrorNotSupported;
    found.store(f, std::memory_order_relaxed);
  }
  *fn = reinterpret_cast<encode_fn>(f);
  return cudaSuccess;
}

}  // namespace

namespace attend {

int finish(cudaError_t err) {
  if (err == cudaSuccess) return PREBA_OK;
  g_last_cuda_error = static_cast<int>(err);
  return PREBA_ERR_CUDA;
}

cudaError_t tensor_map(CUtensorMap* map, int dtype, const void* base, const uint64_t* dims,
                       const uint64_t* strides, const uint32_t* box) {
  encode_fn encode;
  const cudaError_t err = encoder(&encode);
  if (err != cudaSuccess) return err;
  const cuuint64_t extent[4] = {dims[0], dims[1], dims[2], dims[3]};
  cuuint64_t bytes[3];
  // the stride of an axis of one entry is never used: any valid one will do
  for (int i = 0; i < 3; ++i) bytes[i] = dims[i + 1] > 1 ? 2 * strides[i] : 16;
  const cuuint32_t boxes[4] = {64, box[0], box[1], 1}, step[4] = {1, 1, 1, 1};
  const CUresult rc = encode(
      map, dtype == PREBA_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
      const_cast<void*>(base), extent, bytes, boxes, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return rc == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t cache_map(CUtensorMap* map, const preba_pages_attend_t& p, const void* cache,
                      const uint64_t* strides, uint32_t box_rows) {
  const uint64_t dims[4] = {p.head_dim, p.page_size, p.heads_kv, p.pages};
  const uint64_t order[3] = {strides[1], strides[2], strides[0]};
  const uint32_t box[2] = {box_rows, 1};
  return tensor_map(map, p.dtype, cache, dims, order, box);
}

cudaError_t states_map(CUtensorMap* map, const preba_pages_attend_t& p, uint32_t states, const void* base,
                       const uint64_t* strides, uint32_t box_rows) {
  const uint64_t dims[4] = {p.head_dim, states, p.heads_kv, 1};
  const uint64_t order[3] = {strides[1], strides[2], 0};
  const uint32_t box[2] = {box_rows, 1};
  return tensor_map(map, p.dtype, base, dims, order, box);
}

}  // namespace attend

namespace {

template <typename T, int DP>
cudaError_t launch_few(const few_args& a, int sms, cudaStream_t stream) {
  CUtensorMap map_k, map_v;
  cudaError_t err = cache_map(&map_k, a.p, a.p.k_cache, a.p.k_stride, a.box_rows);
  if (err == cudaSuccess) err = cache_map(&map_v, a.p, a.p.v_cache, a.p.v_stride, a.box_rows);
  if (err == cudaSuccess)
    err = cudaFuncSetAttribute(few_rows_kernel<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                               few_layout<DP>::kBytes);
  if (err != cudaSuccess) return err;
  const int grid = std::min(2 * sms, kMaxSplitCtas);
  return launch_chained(few_rows_kernel<T, DP>, grid, kFewThreads, few_layout<DP>::kBytes, stream, map_k, map_v, a);
}

bool operand_ok(const void* base, const uint64_t* strides, int count) {
  if (!base || (reinterpret_cast<uintptr_t>(base) & 15)) return false;
  for (int i = 0; i < count; ++i)
    if (strides[i] % 8) return false;
  return true;
}

// An axis of the queries and caches with more than one entry has a stride (tensor copies know no other kind).
bool strides_used(const preba_pages_attend_t& p) {
  for (const uint64_t* s : {p.k_stride, p.v_stride})
    if (s[1] == 0 || (p.heads_kv > 1 && s[2] == 0) || (p.pages > 1 && s[0] == 0) ||
        std::max({s[0], s[1], s[2]}) >= (1ull << 38))
      return false;
  return (p.heads_q == 1 || p.q_stride[1]) && (p.tokens == 1 || p.q_stride[0]) &&
         std::max(p.q_stride[0], p.q_stride[1]) < (1ull << 38);
}

}  // namespace
}  // namespace preba

extern "C" int preba_pages_attend_query(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv,
                                        uint32_t head_dim, uint64_t* workspace_bytes) {
  using namespace preba;
  if (!workspace_bytes || !sizes_ok(n, tokens, heads_q, heads_kv, head_dim)) return PREBA_ERR_INVALID_ARG;
  *workspace_bytes = workspace_of(n, tokens, heads_q / heads_kv, head_dim);
  return PREBA_OK;
}

#if defined(PREBA_CHECKED)
// For tests of the checked build: from the next call on, a warp's wait runs out after `waits` that did not, or
// when it has polled `polls` times.  0, 0: as ever.
static std::atomic<uint32_t> g_checked_waits{UINT32_MAX}, g_checked_polls{preba::attend::kSpinLimit};
extern "C" void preba_checked_waits(uint32_t waits, uint32_t polls) {
  g_checked_waits = polls ? waits : UINT32_MAX;
  g_checked_polls = polls ? polls : preba::attend::kSpinLimit;
}
preba::attend::wait_limits_t preba::attend::wait_limits() { return {g_checked_waits, g_checked_polls}; }
#endif

extern "C" int preba_pages_attend(const preba_pages_attend_t* req, void* stream) {
  using namespace preba;
  using attend::finish;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_pages_attend_t& p = *req;
  if (!sizes_ok(p.n, p.tokens, p.heads_q, p.heads_kv, p.head_dim) || !operand_ok(p.q, p.q_stride, 2) ||
      !operand_ok(p.out, p.out_stride, 2) || !operand_ok(p.k_cache, p.k_stride, 3) ||
      !operand_ok(p.v_cache, p.v_stride, 3) || !p.block_table || !p.cu_q || !p.kv_len || p.max_q == 0 ||
      p.pages == 0 || p.page_size < 8 || p.page_size > PREBA_PAGES_MAX_PAGE ||
      (p.page_size & (p.page_size - 1)) || p.table_stride < p.table_width ||
      (p.dtype != PREBA_F16 && p.dtype != PREBA_BF16) || (p.flags & ~PREBA_ATTEND_CAUSAL) ||
      p.window > INT32_MAX || p.pages > INT32_MAX / p.page_size || !strides_used(p) ||
      static_cast<double>(p.n) * p.heads_kv * (static_cast<double>(p.table_width) * p.page_size / 64 + 2) > 2e9 ||
      !(p.scale > 0.f) || !(p.scale < INFINITY))
    return PREBA_ERR_INVALID_ARG;
  if (!p.workspace || (reinterpret_cast<uintptr_t>(p.workspace) & 15)) return PREBA_ERR_INVALID_ARG;
  const uint32_t group = p.heads_q / p.heads_kv;
  if (p.workspace_bytes < workspace_of(p.n, p.tokens, group, p.head_dim)) return PREBA_ERR_BUFFER_TOO_SMALL;
  // One 16-row fragment holds the rows of a key head, or the other kernel takes them.  64 requests of up to 8192
  // keys of 8 heads of 128 (floor by bytes 133 us), rows on a key head: 4 and 8: 144 us here, 177 there; 16: 149
  // and 183; 17 to 128 there only, 178 to 213.  4 requests of up to 2048 keys, 8 rows: 13.5 and 20.2, 16: 17.3
  // and 20.1.  The longest request of a step decides, so that one chunk takes its single tokens along.
  const bool few = static_cast<uint64_t>(group) * p.max_q <= kRowsMax;
  // claims of the kernel for many rows are numbered in 32 bits
  if (!few && pairs_at_most(p.n, p.tokens, group) * p.heads_kv > INT32_MAX) return PREBA_ERR_INVALID_ARG;
  const uint32_t shift = 31 - __builtin_clz(p.page_size);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int device = 0, sms = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
  if (err != cudaSuccess) return finish(err);
  if (few) {
    const uint32_t box_rows = std::min<uint32_t>(p.page_size, kTileKeys);
    const few_args a{p, shift, group, box_rows, 31u - __builtin_clz(box_rows)};
    if (p.dtype == PREBA_F16)
      return finish(p.head_dim <= 64 ? launch_few<__half, 64>(a, sms, s) : launch_few<__half, 128>(a, sms, s));
    return finish(p.head_dim <= 64 ? launch_few<__nv_bfloat16, 64>(a, sms, s)
                                   : launch_few<__nv_bfloat16, 128>(a, sms, s));
  }
  return finish(launch_tiles(p, shift, sms, static_cast<uint8_t*>(p.workspace) + kCounterBytes, s));
}
