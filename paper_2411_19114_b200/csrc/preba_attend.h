// Shared by the two attention kernels (preba_attend.cu): requests, barriers, tensor copies.
#ifndef PREBA_ATTEND_H_
#define PREBA_ATTEND_H_

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "preba_internal.h"
#include "preba_tokens.h"

namespace preba {
namespace attend {

constexpr uint32_t kFull = 0xffffffffu;
constexpr uint32_t kSpinLimit = 1u << 20;  // polls of one wait
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxTileCtas = 160;                // of the kernel for many rows: one per SM
constexpr int kMaxSplitCtas = 2 * kMaxTileCtas;  // of the kernel for few rows: two per SM

// Tensor maps of four axes, 16-bit elements, boxes of 64 elements x box[0] x box[1] x 1 in the 128-byte
// swizzle; what lies outside the tensor reads as 0.  Strides in elements, of axes 1 to 3.
cudaError_t tensor_map(CUtensorMap* map, int dtype, const void* base, const uint64_t* dims,
                       const uint64_t* strides, const uint32_t* box);
// The cache: boxes of box_rows slots of one head of one page.
cudaError_t cache_map(CUtensorMap* map, const preba_pages_attend_t& p, const void* cache,
                      const uint64_t* strides, uint32_t box_rows);

// The kernel for many rows (preba_attend_tiles.cu): its workspace and its launches.
uint64_t tiles_workspace(uint32_t n, uint32_t tokens, uint32_t group, uint32_t head_dim);
cudaError_t launch_tiles(const preba_pages_attend_t& p, uint32_t page_shift, int sms, void* workspace,
                         cudaStream_t stream);

__device__ __forceinline__ void report(int32_t* status, int32_t code) {
  if (status) atomicCAS(status, 0, code);
}

// What a request's rows and keys are, checked.  False: the request is skipped.
struct request_t {
  int32_t row, rows, keys;  // first row, rows, keys
};
__device__ __forceinline__ bool load_request(const preba_pages_attend_t& p, uint32_t r, request_t& q) {
  const int32_t a = p.cu_q[r], b = p.cu_q[r + 1], kv = p.kv_len[r];
  q.row = a;
  q.rows = b - a;
  q.keys = kv;
  return !(a < 0 || b < a || static_cast<uint32_t>(b) > p.tokens || static_cast<uint32_t>(b - a) > p.max_q ||
           kv < 0 || static_cast<uint32_t>(kv) > PREBA_PAGES_MAX_KEYS ||  // key numbers stay 32-bit past a tile's end
           static_cast<uint64_t>(kv) > static_cast<uint64_t>(p.table_width) * p.page_size);
}

// Rows j0 .. j1-1 of a request see keys in [lo, hi) and no others (each row its own part of them).
__device__ __forceinline__ void seen_by(const preba_pages_attend_t& p, const request_t& q, int32_t j0,
                                        int32_t j1, int32_t& lo, int32_t& hi) {
  const int32_t at0 = q.keys - q.rows;  // place of row 0; may be negative
  hi = (p.flags & PREBA_ATTEND_CAUSAL) ? max(0, min(q.keys, at0 + j1)) : q.keys;
  lo = p.window ? static_cast<int32_t>(max(static_cast<int64_t>(0),
                                           static_cast<int64_t>(at0) + j0 + 1 - p.window)) : 0;
}

// ---- shared-memory barriers and tensor copies (PTX) ------------------------------------------

__device__ __forceinline__ uint32_t smem_addr(const void* ptr) {
  return static_cast<uint32_t>(__cvta_generic_to_shared(ptr));
}
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
// A whole warp waits for the phase with the given parity to complete; false if the limit ran out.  The lanes
// agree on it: what follows are instructions that the whole warp has to take part in.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, uint32_t limit = kSpinLimit) {
  for (uint32_t it = 0; it < limit; ++it)
    if (__all_sync(kFull, mbar_try_wait(bar, parity))) return true;
  return false;
}

// The waits of a warp.  The checked build can have them run out early (preba_checked_waits), so that tests
// see what the kernels leave then; what a kernel waits for after that, before it returns, has the full limit.
#if defined(PREBA_CHECKED)
struct wait_limits_t {
  uint32_t waits, polls;  // waits of a warp before one runs out; polls of one wait
};
wait_limits_t wait_limits();
struct waits_t {
  wait_limits_t left;
  template <typename A> __device__ __forceinline__ explicit waits_t(const A& a) : left(a.limits) {}
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) {
    if (left.waits == 0) return false;
    --left.waits;
    return mbar_wait(bar, parity, left.polls);
  }
};
#else
struct waits_t {
  template <typename A> __device__ __forceinline__ explicit waits_t(const A&) {}
  __device__ __forceinline__ bool operator()(uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity); }
};
#endif

// One box of a four-dimensional tensor into shared memory.
__device__ __forceinline__ void tensor_copy(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y,
                                            int32_t z, int32_t w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Maxima leave out what is not a number, sums do not.  A partial sum whose row saw such a score carries that
// in its maximum too, so that -inf there means nothing but "no key seen".
__device__ __forceinline__ float marked(float m, float l) { return l != l ? l : m; }
// The log-sum-exp of a row from its sum and maximum in units of log2.
__device__ __forceinline__ float row_lse(float m, float l) {
  return l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

}  // namespace attend
}  // namespace preba

#endif  // PREBA_ATTEND_H_
