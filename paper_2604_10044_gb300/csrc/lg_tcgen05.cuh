// The tcgen05 instructions the chunk attention uses: tensor memory, matrix products of one CTA
// issued by one thread, and their descriptors.
#pragma once
#include <cuda.h>
#include <cudaTypedefs.h>
#include <stdint.h>

#include "lg_common.cuh"

namespace lg {

// tensor maps (lg_attend_mma.cu)
PFN_cuTensorMapEncodeTiled_v12000 encode_fn();
bool make_kv_map(CUtensorMap *m, const void *base, int dtype, int d, int64_t rows, int box_rows);

// whole warp; *smem_out receives the address of `cols` columns of tensor memory
__device__ __forceinline__ void tmem_alloc(uint32_t *smem_out, uint32_t cols) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_addr(smem_out)),
               "r"(cols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols)
               : "memory");
}

__device__ __forceinline__ void tc_fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void tc_fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}

// arrives on `bar` once every product this thread has issued so far is done
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(
                   smem_addr(bar))
               : "memory");
}

// Descriptor of a bf16 operand in shared memory in 128-byte-swizzled rows, as its two halves (the
// upper one is the same for every operand here, and moving along an operand adds to the lower one).
// For rows of 64 consecutive contraction elements (K-major): 1024 bytes from 8 rows to the next 8.
// For rows of 64 consecutive row/column elements (MN-major): `lbo` bytes from one 64 of them to the
// next, 1024 bytes from 8 contraction steps to the next 8.
constexpr uint32_t kDescHi = 1024u >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) {
  return ((addr & 0x3ffff) >> 4) | (lbo >> 4) << 16;
}

// One lane of a converged warp, always the same.  The products are issued by a whole warp's code of
// which one lane executes the instructions: their operands live in uniform registers, and only for
// code that all lanes run does the compiler keep them there (issued from a branch of one lane, 16
// products took 1600 to 2400 cycles to issue; they run for 1024).
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(r));
  return r != 0;
}

// Instruction descriptor: bf16 x bf16 -> fp32, each operand K-major or MN-major
__host__ __device__ constexpr uint32_t mma_idesc(int m, int n, bool a_mn_major, bool b_mn_major) {
  return 1u << 4 | 1u << 7 | 1u << 10 | (a_mn_major ? 1u << 15 : 0u) |
         (b_mn_major ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 |
         (uint32_t)(m >> 4) << 24;
}

// d (tensor memory) = [d +] A B, A in shared memory (lower halves of the descriptors)
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                          bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 da, db;\n setp.ne.u32 p, %4, 0;\n mov.b64 da, {%1, %5};\n"
      " mov.b64 db, {%2, %5};\n tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kDescHi)
      : "memory");
}

// the same with A in tensor memory (two bf16 a column)
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc,
                                          bool add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 db;\n setp.ne.u32 p, %4, 0;\n mov.b64 db, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n}\n" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kDescHi)
      : "memory");
}

#define LG_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), \
                    "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define LG_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), \
                    "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])

// 32 columns of this thread's lane (warp w of four: lanes 32 w ..)
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t *v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];"
      : LG_R8(v, 0), LG_R8(v, 8), LG_R8(v, 16), LG_R8(v, 24)
      : "r"(addr)
      : "memory");
}

__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, "
      "%11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, "
      "%29, %30, %31};" ::LG_W8(v, 0),
      LG_W8(v, 8), LG_W8(v, 16), LG_W8(v, 24), "r"(addr)
      : "memory");
}

__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t *v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, "
      "%12, %13, %14, %15}, [%16];"
      : LG_R8(v, 0), LG_R8(v, 8)
      : "r"(addr)
      : "memory");
}

__device__ __forceinline__ void tmem_store16(uint32_t addr, const uint32_t *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, "
      "%10, %11, %12, %13, %14, %15};" ::LG_W8(v, 0),
      LG_W8(v, 8), "r"(addr)
      : "memory");
}

__device__ __forceinline__ void tmem_wait_load() {
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_wait_store() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

// tensor copies of one box, completing on `bar`
__device__ __forceinline__ void tma_box_2d(void *dst, const CUtensorMap *map, int x, int y,
                                           uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%2, %3}], [%4];" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(smem_addr(bar))
      : "memory");
}
__device__ __forceinline__ void tma_box_3d(void *dst, const CUtensorMap *map, int x, int y, int z,
                                           uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], "
      "[%1, {%2, %3, %4}], [%5];" ::"r"(smem_addr(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(smem_addr(bar))
      : "memory");
}

}  // namespace lg
