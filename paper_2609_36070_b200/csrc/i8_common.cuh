// 8-bit integer operands: the quantisation rule and the declarations shared by the kernels around the 8-bit products.
//
// A row of activations x is held as codes q = round(127 x / amax) in -127 .. 127, ties to the even code, and one scale
// amax / 127 (fp32), amax = max |x|.  127 x and the quotient are rounded to fp32 one after the other; for 16-bit x the
// product is exact and the quotient's rounding cannot cross a tie (two such quotients that are not tied differ from a tie
// by a relative 2^-17 or more for bf16 and 2^-20 for fp16), so the code is the one of exact arithmetic.  A row of zeros has
// scale 0 and codes 0; a row with an infinity or a NaN has that as its scale and codes 0, so its products are NaN and no
// other row's are touched.
#pragma once
#include "mok_internal.cuh"
#include <cuda_fp16.h>

namespace mok {
namespace i8 {

constexpr int MAX_CONTRACTION = 131072;     // |sum| <= 127 * 127 * K stays below 2^31

// Bits of |v| as an integer: ordered like the magnitudes, infinities above the finite ones and NaN above infinity.
__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ bool finite_bits(uint32_t b) { return b < 0x7f800000u; }

// round-to-nearest-even integer of v, |v| <= 127, in the low byte: adding 1.5 * 2^23 leaves it in the low mantissa bits
__device__ __forceinline__ uint32_t round_byte(float v) { return __float_as_uint(v + 12582912.f); }
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// The two factors of a row: q = (v * times) / by.  Above 2^120 the product 127 v would overflow: both are then 2^8 smaller.
struct RowRule { float times, by; };
__device__ __forceinline__ RowRule row_rule(float amax) {
    return amax > 1.329228e36f ? RowRule{127.f / 256.f, amax * (1.f / 256.f)} : RowRule{127.f, amax};
}
__device__ __forceinline__ uint32_t code_bits(float v, RowRule r) { return round_byte(__fdiv_rn(__fmul_rn(v, r.times), r.by)); }

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

inline bool type_ok(int t) { return t == MOK_TYPE_BF16 || t == MOK_TYPE_F16 || t == MOK_TYPE_F32; }
inline size_t type_bytes(int t) { return t == MOK_TYPE_F32 ? 4 : 2; }
inline int pitch_of(int K) { return (K + 15) / 16 * 16; }

// One product launch.  Rows live in the padded space of the schedule (grouped) or are 0 .. dense_rows - 1.
struct ProductArgs {
    const int8_t* A;             // codes [a_rows, K], lda bytes apart
    const int8_t* B;             // codes [E * (swiglu ? 2 : 1) * N, K], ldb bytes apart
    long long lda, ldb, a_rows;
    int32_t K, N, E;
    void* C;
    long long ldc;               // elements
    int32_t c_type;              // MOK_TYPE_* (plain epilogue)
    const float* a_scale;        // [a_rows] (plain, swiglu)
    const float* b_scale;        // [E * (swiglu ? 2 : 1) * N]
    const float* b_max;          // [E]: largest b_scale of the matrix (EPI_HALF)
    float y_unit;                // EPI_HALF: power of two that brings |sum| <= 127 * 127 * K below 65504
    const float* bias;           // [N] or NULL (plain)
    int32_t dense_rows;          // > 0: dense
    const int4* tiles;           // grouped: {first row, rows of the segment from there on, expert, -} of every 256-row tile
    const int32_t* n_mtiles;     // how many
    int32_t max_mt;              // at most
    int32_t c_mapped;            // set by the launcher: C is stored through a tensor map
    WsHeader* header;
};
enum { EPI_PLAIN = 0, EPI_GATED = 1, EPI_HALF = 2 };

// Where a token's codes go when its rows are wanted in expert order: row pos[t * k + s] for every routed slot s.
// The launch also writes the product's tile list from the schedule's tables.
struct RouteArgs {
    const int32_t *idx, *pos;
    int32_t E, k;
    int4* tiles;
    const int32_t *n_mtiles, *tile_expert, *mt_start, *pad_offsets, *counts;
};
cudaError_t launch_quantize(const void* x, int type, long long rows, int K, long long ldx, int8_t* codes, long long ldc,
                            float* scales, cudaStream_t s, const RouteArgs* routes = nullptr);
cudaError_t launch_product(const ProductArgs& a, int epi, cudaStream_t s);
cudaError_t status_header(WsHeader** out);

}  // namespace i8
}  // namespace mok
