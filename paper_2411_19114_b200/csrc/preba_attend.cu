// Attention of a step's tokens over the paged cache (preba_tokens.h): preba_pages_attend.
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

template <typename T> __device__ __forceinline__ float2 open2(uint32_t v);
template <> __device__ __forceinline__ float2 open2<__half>(uint32_t v) {
  return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
template <> __device__ __forceinline__ float2 open2<__nv_bfloat16>(uint32_t v) {
  return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}

// What a request's rows and keys are, checked.  False: the request is skipped.
struct request_t {
  int32_t row, rows, keys;
};
__device__ __forceinline__ bool load_request(const preba_pages_attend_t& p, uint32_t r, request_t& q) {
  const int32_t a = p.cu_q[r], b = p.cu_q[r + 1], kv = p.kv_len[r];
  q = {a, b - a, kv};
  if (a < 0 || b < a || static_cast<uint32_t>(b) > p.tokens || static_cast<uint32_t>(b - a) > p.max_q ||
      kv < 0 || static_cast<uint64_t>(kv) > static_cast<uint64_t>(p.table_width) * p.page_size) {
    report(p.status, PREBA_ERR_BAD_TABLE);
    return false;
  }
  return true;
}

// One warp per (request, row, query head): 32 keys at a time, one per lane, then the values with an
// element per lane.
template <typename T>
__global__ void __launch_bounds__(128)
attend_kernel(const preba_pages_attend_t p, const uint32_t page_shift) {
  const uint32_t lane = threadIdx.x & 31;
  const uint64_t unit = (static_cast<uint64_t>(blockIdx.x) * 128 + threadIdx.x) >> 5;
  if (unit >= static_cast<uint64_t>(p.tokens) * p.heads_q) return;
  const uint32_t token = static_cast<uint32_t>(unit / p.heads_q), head = unit % p.heads_q;
  // the request that owns the token
  uint32_t r = 0;
  for (; r < p.n; ++r)
    if (p.cu_q[r + 1] > static_cast<int64_t>(token)) break;
  request_t q;
  if (r == p.n || !load_request(p, r, q) || static_cast<uint32_t>(q.row) > token) return;
  const int64_t at = static_cast<int64_t>(q.keys) - q.rows + (token - q.row);
  int64_t k1 = q.keys, k0 = 0;
  if (p.flags & PREBA_ATTEND_CAUSAL) k1 = min(k1, at + 1);
  if (p.window) k0 = max(k0, at - p.window + 1);
  const uint32_t head_kv = head / (p.heads_q / p.heads_kv);
  const T* qp = static_cast<const T*>(p.q) + token * p.q_stride[0] + head * p.q_stride[1];
  float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int64_t k = k0; k < k1; k += 32) {
    const int64_t mine = k + lane;
    float s = -INFINITY;
    uint64_t v_at = 0;
    if (mine < k1) {
      const int32_t page = p.block_table[r * p.table_stride + (mine >> page_shift)];
      const uint32_t in = static_cast<uint32_t>(mine) & (p.page_size - 1);
      if (page < 0 || static_cast<uint32_t>(page) >= p.pages) {
        report(p.status, PREBA_ERR_BAD_TABLE);
        v_at = ~0ull;
        s = 0.f;
      } else {
        const T* kp = static_cast<const T*>(p.k_cache) + page * p.k_stride[0] + in * p.k_stride[1] +
                      head_kv * p.k_stride[2];
        v_at = page * p.v_stride[0] + in * p.v_stride[1] + head_kv * p.v_stride[2];
        float sum = 0.f;
        for (uint32_t e = 0; e < p.head_dim; e += 8) {
          const uint4 x = *reinterpret_cast<const uint4*>(qp + e);
          const uint4 y = *reinterpret_cast<const uint4*>(kp + e);
          const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 a = open2<T>(xs[i]), b = open2<T>(ys[i]);
            sum = fmaf(a.x, b.x, fmaf(a.y, b.y, sum));
          }
        }
        s = sum * p.scale;
      }
    }
    float top = s;
#pragma unroll
    for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, d));
    top = fmaxf(top, m);
    const float keep = expf(m - top), e = mine < k1 ? expf(s - top) : 0.f;
    m = top;
    float sum = e;
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
    l = l * keep + sum;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= keep;
    for (int j = 0; j < 32 && k + j < k1; ++j) {
      const float w = __shfl_sync(kFull, e, j);
      const uint64_t base = __shfl_sync(kFull, v_at, j);
      if (base == ~0ull) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < p.head_dim)
          o[i] = fmaf(w, static_cast<float>(static_cast<const T*>(p.v_cache)[base + lane + 32 * i]), o[i]);
    }
  }
  T* to = static_cast<T*>(p.out) + token * p.out_stride[0] + head * p.out_stride[1];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (lane + 32 * i < p.head_dim) to[lane + 32 * i] = static_cast<T>(l > 0.f ? o[i] / l : 0.f);
  if (p.lse && lane == 0)
    p.lse[static_cast<uint64_t>(token) * p.heads_q + head] = l > 0.f ? m + logf(l) : -INFINITY;
}

int finish(cudaError_t err) {
  if (err == cudaSuccess) return PREBA_OK;
  g_last_cuda_error = static_cast<int>(err);
  return PREBA_ERR_CUDA;
}

bool sizes_ok(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv, uint32_t head_dim) {
  return n >= 1 && n <= PREBA_PAGES_MAX_REQUESTS && tokens >= 1 && tokens <= INT32_MAX && heads_q >= 1 &&
         heads_q <= 65535 && heads_kv >= 1 && heads_q % heads_kv == 0 && heads_q / heads_kv <= 128 &&
         head_dim >= 8 && head_dim % 8 == 0 && head_dim <= PREBA_PAGES_MAX_HEAD_DIM;
}

uint64_t workspace_of() { return 16; }

bool operand_ok(const void* base, const uint64_t* strides, int count) {
  if (!base || (reinterpret_cast<uintptr_t>(base) & 15)) return false;
  for (int i = 0; i < count; ++i)
    if (strides[i] % 8) return false;
  return true;
}

}  // namespace
}  // namespace preba

extern "C" int preba_pages_attend_query(uint32_t n, uint32_t tokens, uint32_t heads_q, uint32_t heads_kv,
                                        uint32_t head_dim, uint64_t* workspace_bytes) {
  using namespace preba;
  if (!workspace_bytes || !sizes_ok(n, tokens, heads_q, heads_kv, head_dim)) return PREBA_ERR_INVALID_ARG;
  *workspace_bytes = workspace_of();
  return PREBA_OK;
}

extern "C" int preba_pages_attend(const preba_pages_attend_t* req, void* stream) {
  using namespace preba;
  if (!req) return PREBA_ERR_INVALID_ARG;
  const preba_pages_attend_t& p = *req;
  if (!sizes_ok(p.n, p.tokens, p.heads_q, p.heads_kv, p.head_dim) || !operand_ok(p.q, p.q_stride, 2) ||
      !operand_ok(p.out, p.out_stride, 2) || !operand_ok(p.k_cache, p.k_stride, 3) ||
      !operand_ok(p.v_cache, p.v_stride, 3) || !p.block_table || !p.cu_q || !p.kv_len || p.max_q == 0 ||
      p.pages == 0 || p.page_size < 8 || p.page_size > PREBA_PAGES_MAX_PAGE ||
      (p.page_size & (p.page_size - 1)) || p.table_stride < p.table_width ||
      (p.dtype != PREBA_F16 && p.dtype != PREBA_BF16) || (p.flags & ~PREBA_ATTEND_CAUSAL) ||
      p.window > INT32_MAX || !(p.scale > 0.f) || !(p.scale < INFINITY))
    return PREBA_ERR_INVALID_ARG;
  if (!p.workspace || (reinterpret_cast<uintptr_t>(p.workspace) & 15)) return PREBA_ERR_INVALID_ARG;
  if (p.workspace_bytes < workspace_of()) return PREBA_ERR_BUFFER_TOO_SMALL;
  const uint64_t units = static_cast<uint64_t>(p.tokens) * p.heads_q;
  const uint32_t shift = 31 - __builtin_clz(p.page_size);
  const uint32_t grid = static_cast<uint32_t>((units + 3) / 4);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (p.dtype == PREBA_F16)
    attend_kernel<__half><<<grid, 128, 0, s>>>(p, shift);
  else
    attend_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(p, shift);
  return finish(cudaGetLastError());
}
