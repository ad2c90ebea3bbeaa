// Thin inline-PTX wrappers for the 5th-generation tensor cores: tensor memory, matrix instructions of bf16 operands
// with fp32 sums, and their descriptors.
#pragma once

#include <stdint.h>

#include "ptx.cuh"

namespace voxzip {
namespace tc {

// ---------------------------------------------------------------- tensor memory
// A column of it is 128 lanes of 32 bits. An address is lane << 16 | column; a warp of a warpgroup reads and writes the
// 32 lanes of its own rank.
__device__ __forceinline__ void alloc(uint32_t *smem_dst, uint32_t columns) {  // one warp
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(ptx::smem_u32(smem_dst)),
                 "r"(columns)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
__device__ __forceinline__ void dealloc(uint32_t tmem, uint32_t columns) {  // the warp that allocated
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns));
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of this warp's lanes: register i of a lane is column i of its row.
__device__ __forceinline__ void ld32(uint32_t addr, float (&r)[32]) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
          "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
          "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
          "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
// Half of a warp's lanes (16 rows; the address names the first), 64 columns, four threads to a row: thread i has, of each
// block b of 8 columns, columns 2 (i % 4) and the next of row i / 4 in r[4 b] and r[4 b + 1], and of row i / 4 + 8 in the
// other two.
__device__ __forceinline__ void ld_rows(uint32_t addr, float (&r)[32]) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]),
          "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]),
          "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]),
          "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
        : "r"(addr));
}
// The same rows and threads, 32 columns of one word each: of each block b of 4, column i % 4 of row i / 4 from u[2 b], of
// row i / 4 + 8 from u[2 b + 1]. Pairs of the logits that ld_rows gave lie where their columns' halves are.
__device__ __forceinline__ void st_rows(uint32_t addr, const uint32_t (&u)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
        "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]),
        "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15])
        : "memory");
}
// 16 columns in ld_rows' layout, both ways (an output's).
__device__ __forceinline__ void ld_rows16(uint32_t addr, float (&r)[8]) {
    uint32_t *u = reinterpret_cast<uint32_t *>(r);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
                 : "r"(addr));
}
__device__ __forceinline__ void st_rows16(uint32_t addr, const float (&r)[8]) {
    const uint32_t *u = reinterpret_cast<const uint32_t *>(r);
    asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(u[0]),
                 "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
}

// ---------------------------------------------------------------- descriptors
// Operand tiles as the tiled copies leave them with the 128-byte swizzle: rows of 64 bf16 (128 bytes), 8 rows to a
// swizzle atom of 1024 bytes; the tile starts on a multiple of 1024.
//   rows along M or N, the 64 along K ("K-major"): 8-row groups 1024 bytes apart.
//   rows along K, the 64 along N ("N-major"): 8-row groups 1024 bytes apart, the next 64 of N `next` bytes on.
__device__ __forceinline__ uint64_t operand(uint32_t smem_addr, uint32_t next) {
    constexpr uint64_t kVersion = 1ull << 46, kSwizzle128 = 2ull << 61;
    return (uint64_t)((smem_addr >> 4) & 0x3fff) | (uint64_t)((next >> 4) & 0x3fff) << 16 | (uint64_t)(1024 >> 4) << 32 |
           kVersion | kSwizzle128;
}
// bf16 x bf16 -> fp32 of M = 128 rows; A K-major.
__host__ __device__ constexpr uint32_t instruction(int n, bool b_n_major) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_n_major ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (128u / 16) << 24;
}

// ---------------------------------------------------------------- matrix instructions
// Called by a whole warp, whose elected lane issues them (the same one each time). Operands of a warp-uniform call live
// in uniform registers; under a branch on the lane each of them would be moved there first, at 20 cycles an instruction.
// d (128 x n, tensor memory) = a (128 x 16, shared memory) b (16 x n) + (add ? d : 0).
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t inst, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(inst), "r"((uint32_t)add)
        : "memory");
}
// The same with a in tensor memory: column i of it holds elements 2 i and 2 i + 1 of each lane's row.
__device__ __forceinline__ void mma_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t inst, bool add) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(inst), "r"((uint32_t)add)
        : "memory");
}
// `bar` gets an arrival when every matrix instruction that the elected lane has issued is done.
__device__ __forceinline__ void commit(uint64_t *bar) {
    asm volatile(
        "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(ptx::smem_u32(bar))
        : "memory");
}

}  // namespace tc
}  // namespace voxzip
