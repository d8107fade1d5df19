// Wrappers and arithmetic shared by the kernels of 8-bit products.
#pragma once
#include "tc_ptx.cuh"

namespace mok {
namespace i8 {

// D[tmem] (+)= A[smem] B[smem]^T by one CTA: signed 8-bit operands, 32-bit integer sums, K = 32
__device__ __forceinline__ void mma_one(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

// silu(g) u.  The exponential is off by (2 + 1.2 |g|) 2^-23 of itself, the quotient by 2^-22: no more than what the three
// roundings of g to fp32 leave open (|g| 2^-22 of silu(g) for negative g, where it counts), and far below the rounding to 8-bit
// codes that follows, which an 11-bit tanh would move in one case of fifty.  (expf and an exact division: 131072 rows of 768
// from 2048 in 403 instead of 312 us.)
__device__ __forceinline__ float gated(float g, float u) { return __fdividef(g, 1.f + __expf(-g)) * u; }

}  // namespace i8
}  // namespace mok
