// The tensor cores of sm_100a: operand descriptors, products with their sums in tensor memory, and that memory.
#pragma once
#include <cuda_runtime.h>

namespace umma {

__device__ __forceinline__ unsigned smem_addr(const void *p) { return (unsigned)__cvta_generic_to_shared(p); }

// Operand descriptor in two words: start and leading byte offset, stride byte offset and layout (0 = none, 2 = 128-byte
// swizzle), in 16-byte units.  Starts move by adding to the first word.
__host__ __device__ constexpr unsigned operand_lo(unsigned lead) { return (lead >> 4) << 16; }
__host__ __device__ constexpr unsigned operand_hi(unsigned stride, unsigned layout) { return (stride >> 4) | (1u << 14) | (layout << 29); }
// fp32 sums of 16-bit products; A 128 x 16, B 16 x n, B and (unless a_by_rows) A with consecutive depth.
__host__ __device__ constexpr unsigned instruction(bool f16, bool a_by_rows, int n) {
  return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((a_by_rows ? 1u : 0u) << 15) |
         ((unsigned)(n >> 3) << 17) | ((unsigned)(128 >> 4) << 24);
}
// The warp that issues runs as a whole, and one lane of it issues: descriptors are then computed once per warp, in uniform
// registers.  (A single lane in a branch of its own took 115..134 cycles per product, several times what a product takes.)
__device__ __forceinline__ unsigned elect() {
  unsigned e;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(e));
  return e;
}
__device__ __forceinline__ void mma(unsigned lead, unsigned d, unsigned alo, unsigned ahi, unsigned blo, unsigned bhi,
                                    unsigned idesc, unsigned add) {
  asm volatile("{\n .reg .pred p, q;\n .reg .b64 a, b;\n setp.ne.u32 q, %0, 0;\n setp.ne.u32 p, %7, 0;\n"
               " mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n"
               " @q tcgen05.mma.cta_group::1.kind::f16 [%1], a, b, %6, p;\n}\n"
               ::"r"(lead), "r"(d), "r"(alo), "r"(ahi), "r"(blo), "r"(bhi), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void commit(unsigned lead, unsigned long long *bar) {  // arrives once all products so far are done
  asm volatile("{\n .reg .pred q;\n setp.ne.u32 q, %0, 0;\n"
               " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n}\n"
               ::"r"(lead), "r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ void tmem_alloc(unsigned *slot, unsigned cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_addr(slot)), "r"(cols) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
}
__device__ __forceinline__ void tmem_free(unsigned base, unsigned cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(base), "r"(cols) : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
// The wait names the registers it is for, so that nothing that uses them is moved in front of it.
__device__ __forceinline__ void tmem_wait(float (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n"
               : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                 "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
               :: "memory");
}
// this lane's row, 16 columns
__device__ __forceinline__ void tmem_ld16(unsigned addr, float (&v)[16]) {
  unsigned *r = reinterpret_cast<unsigned *>(v);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                 "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr));
}

}  // namespace umma
