// tcgen05.cuh -- the fifth-generation tensor cores: tensor memory, its matrix instruction and their barriers.
#pragma once

#include "mma.cuh"

namespace kvx {
namespace {

// ---- barriers in shared memory

__device__ __forceinline__ void bar_init(uint32_t bar) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
// Waits for a phase, for at most `cycles`; false if it did not come.
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, long long cycles) {
  if (bar_try(bar, parity)) return true;
  const long long start = clock64();
  do {
    if (bar_try(bar, parity)) return true;
  } while (clock64() - start < cycles);
  return false;
}
// Makes this thread's writes to shared memory visible to the matrix instructions issued after a barrier.
__device__ __forceinline__ void fence_operands() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ---- tensor memory: 128 lanes of 512 32-bit columns; an address is lane << 16 | column

__device__ __forceinline__ void tmem_alloc(uint32_t to, int columns) {  // one warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void tmem_free(uint32_t at, int columns) {  // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
// A group of four warps gives up registers of its threads, or takes what others of the CTA have given up (and waits
// until it is there).
template <int kRegs>
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs)); }
template <int kRegs>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs)); }
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16 neighbouring columns of a warp's 32 lanes, a lane each.
__device__ __forceinline__ void tmem_load16(float (&r)[16], uint32_t at) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
                 "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]) : "r"(at));
}
__device__ __forceinline__ void tmem_load1(uint32_t& r, uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(at));
}
__device__ __forceinline__ void tmem_store8(uint32_t at, const uint32_t (&u)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(at), "r"(u[0]), "r"(u[1]),
               "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]) : "memory");
}

// ---- matrix instruction: D (128 x n, fp32, tensor memory) = [D +] A (128 x 16) B (16 x n), one thread

// Operands in shared memory are panels of rows of 64 16-bit elements (128 bytes), 128 rows one after another, with the
// row's 16-byte vectors permuted by its number (128-byte swizzle): vector c of row r at r * 128 + ((c ^ r % 8) << 4).
// Rows are an operand's outer dimension (its elements lie along k) or k itself (its elements lie along the outer one);
// a matrix wider than 64 has its next panel kPanel bytes further on.
constexpr int kPanel = 128 * 128;
__device__ __forceinline__ uint32_t panel_at(int row, int vec) {  // vec: of the whole row, over the panels
  return (vec >> 3) * kPanel + row * 128 + (((vec & 7) ^ (row & 7)) << 4);
}
constexpr uint64_t kOperand = (uint64_t)(1024 >> 4) << 32 /* bytes between groups of 8 rows */ | 1ull << 46 | 2ull << 61;
// Step k (16 elements along k) of an operand whose elements lie along k, and of one whose rows are k.
__device__ __forceinline__ uint64_t operand_k(uint32_t at, int k) {
  return kOperand | 1ull << 16 | ((at + (k >> 2) * kPanel + (k & 3) * 32) >> 4 & 0x3FFF);
}
__device__ __forceinline__ uint64_t operand_rows(uint32_t at, int k) {
  return kOperand | (uint64_t)(kPanel >> 4) << 16 | ((at + k * 16 * 128) >> 4 & 0x3FFF);
}
// Types (E: Bf16, or fp16 otherwise), which of A and B have rows of k, and n.
template <class E>
__host__ __device__ constexpr uint32_t instruction(bool a_rows, bool b_rows, int n) {
  const uint32_t type = std::is_same<E, Bf16>::value ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (uint32_t)a_rows << 15 | (uint32_t)b_rows << 16 | (uint32_t)(n >> 3) << 17 |
         (128u >> 4) << 24;
}
__device__ __forceinline__ void matrix_product(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
               "l"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void matrix_product_t(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {  // A in tensor memory
  asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
               "r"(a), "l"(b), "r"(what), "r"((uint32_t)add) : "memory");
}
// One lane of a converged warp: in a branch on it the compiler keeps what the warp shares in uniform registers, which
// is where matrix instructions want their operands (issued by a thread picked by its number, one took 60 cycles).
__device__ __forceinline__ bool elected() {
  uint32_t one;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(one));
  return one != 0;
}
// The barrier's phase ends when the instructions issued so far are done.
__device__ __forceinline__ void products_done(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

}  // namespace
}  // namespace kvx
