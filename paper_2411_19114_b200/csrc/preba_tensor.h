// Instructions of the 5th-generation tensor cores and of tensor memory (PTX), for the attention kernels that use them
// (preba_attend_tiles.cu, preba_cross.cu).
#ifndef PREBA_TENSOR_H_
#define PREBA_TENSOR_H_

#include "preba_attend.h"

namespace preba {
namespace attend {

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Shared-memory operand: rows of 128 bytes in the 128-byte swizzle, eight rows (1024 bytes) to a group.
// `leading` is the distance between 64-element columns of an operand whose rows are its contraction
// axis.  The low word of the descriptor; the high one is the same for all.
__device__ __forceinline__ uint32_t operand(uint32_t addr, uint32_t leading) {
  return (addr & 0x3ffff) >> 4 | (leading >> 4) << 16;
}
constexpr uint32_t kOperandHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
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

}  // namespace attend
}  // namespace preba

#endif  // PREBA_TENSOR_H_
