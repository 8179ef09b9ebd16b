// Products of few rows with a large matrix on tcgen05 (up to 256 rows of 16-bit operands: serving): reading the matrix is all that costs, so it is the operand with many rows (128 of a tile, M of the
// instruction) and the few rows are the narrow one (N of the instruction, 16 to 256 in steps of 16).  Each CTA by itself (cta_group::1) streams stages of 64 values of the reduction through a ring as
// deep as shared memory allows (16 rows: 11 stages of 18 KB, so that an SM has 180 KB on their way).  What gated_skinny.cuh and class_loss.cu share of it.
#pragma once

#include "class_gemm.cuh"

namespace gad {

namespace {

constexpr int SK_M = 128, SK_MOST_ROWS = 256;
constexpr int SK_GROUPS = 4;                                // of four draining warps (a quarter of the accumulator's rows each), in turn 16 rows of x each
constexpr int SK_DRAIN = SK_GROUPS * 128, SK_THREADS = 64 + SK_DRAIN;
constexpr int SK_A = SK_M * CT_K * 2;                       // 16 KiB of weights a stage
constexpr int SK_XCH = SK_GROUPS * 2 * 8 * 64 * 4;          // per group, g of eight rows and u of eight rows on their way to the threads that have the other
constexpr int SK_MOST_STAGES = 12;
constexpr int SK_SMEM = 227 * 1024;
constexpr int SK_RING = SK_SMEM - 1024 - 512 - SK_XCH;

__device__ __forceinline__ void mma_f16_one(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(tmem_d),
        "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Whether ok is true in all draining threads.
__device__ __forceinline__ bool all_drain(bool ok) {
    uint32_t r;
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        "setp.ne.b32 p, %1, 0;\n"
        "bar.red.and.pred q, 1, %2, p;\n"
        "selp.b32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r)
        : "r"((uint32_t)ok), "n"(SK_DRAIN)
        : "memory");
    return r != 0;
}
// This warp's 32 tensor-memory lanes x 16 columns, complete on return.
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;\n"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]),
          "=f"(v[14]), "=f"(v[15])
        : "r"(addr)
        : "memory");
}
// The same back; tmem_wait_st before it is read again.
__device__ __forceinline__ void tmem_st16(uint32_t addr, const float (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};\n" ::"r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]),
        "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
        : "memory");
}

}  // namespace

}  // namespace gad
