// Helpers of the kernels whose products run on the tensor cores: descriptions of operands in shared memory, the
// product instruction, its completion, and accumulators brought to registers.
#pragma once
#include <stdint.h>

#include "tma_common.cuh"

namespace fpde {

// 64-bit description of an operand slice in shared memory, 128-byte swizzle.  K-major: rows of 64 fp16,
// 1024 bytes per 8 rows.  MN-major: blocks of 64 columns, `block` bytes apart (64 k-rows: 8192); 1024 bytes
// per 8 k-rows.
__device__ __forceinline__ uint64_t slice_desc(uint32_t addr, bool mn_major, uint32_t block = 8192) {
    uint64_t d = (uint64_t)((addr & 0x3ffff) >> 4);
    d |= (uint64_t)((mn_major ? block : 16) >> 4) << 16;  // leading offset (K-major, swizzled: not used)
    d |= (uint64_t)(1024 >> 4) << 32;                     // stride offset
    d |= 1ull << 46;                                      // descriptor version of sm_100
    d |= 2ull << 61;                                      // 128-byte swizzle
    return d;
}

// The description of a slice `bytes` further on: the address field is the lowest, and no slice lies past its end.
__device__ __forceinline__ uint64_t desc_at(uint64_t d, uint32_t bytes) {
    return (d & 0xffffffff00000000ull) | (uint32_t)((uint32_t)d + (bytes >> 4));
}

template <int CG = 1>
__device__ __forceinline__ void mma_f16(uint32_t tmem, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
            : "memory");
}
// Arrives on the barrier when the products issued so far are done; CG = 2: on that of both blocks.
template <int CG = 1>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((uint16_t)3)
                     : "memory");
}
__device__ __forceinline__ void tmem_load32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, "
        "%18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

}  // namespace fpde
