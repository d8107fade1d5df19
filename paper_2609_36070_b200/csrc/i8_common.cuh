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
// `near` is their quotient to within 2^-22.
struct RowRule { float times, by, near; };
__device__ __forceinline__ RowRule row_rule(float amax) {
    const bool big = amax > 1.329228e36f;
    const float times = big ? 127.f / 256.f : 127.f, by = big ? amax * (1.f / 256.f) : amax;
    return RowRule{times, by, __fdividef(times, by)};
}
// The exact code costs a division.  v * near is within 4e-5 of the quotient, so unless it comes within 2e-4 of a tie its
// rounding is the quotient's: four codes cost a dozen instructions and one value in 2500 a division.
__device__ __forceinline__ uint32_t code_bits(float v, RowRule r) { return round_byte(__fdiv_rn(__fmul_rn(v, r.times), r.by)); }
static __device__ __noinline__ uint32_t four_exact_codes(float v0, float v1, float v2, float v3, float times, float by) {
    const RowRule r = {times, by, 0.f};
    return pack4(code_bits(v0, r), code_bits(v1, r), code_bits(v2, r), code_bits(v3, r));
}
// CALL: the divisions in a function, for code that runs once and should be short (a call costs its caller registers)
template <bool CALL = false>
__device__ __forceinline__ uint32_t four_codes(float v0, float v1, float v2, float v3, RowRule r) {
    constexpr float MAGIC = 12582912.f;
    const float m0 = fmaf(v0, r.near, MAGIC), m1 = fmaf(v1, r.near, MAGIC), m2 = fmaf(v2, r.near, MAGIC), m3 = fmaf(v3, r.near, MAGIC);
    const float d0 = fabsf(fmaf(v0, r.near, MAGIC - m0)), d1 = fabsf(fmaf(v1, r.near, MAGIC - m1));
    const float d2 = fabsf(fmaf(v2, r.near, MAGIC - m2)), d3 = fabsf(fmaf(v3, r.near, MAGIC - m3));
    if (d0 <= 0.4998f && d1 <= 0.4998f && d2 <= 0.4998f && d3 <= 0.4998f)      // (false for NaN, too)
        return pack4(__float_as_uint(m0), __float_as_uint(m1), __float_as_uint(m2), __float_as_uint(m3));
    if (CALL) return four_exact_codes(v0, v1, v2, v3, r.times, r.by);
    return pack4(code_bits(v0, r), code_bits(v1, r), code_bits(v2, r), code_bits(v3, r));
}

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }

template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

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
    const float* bias;           // [N] or NULL (plain)
    int32_t dense_rows;          // > 0: dense
    const int4* tiles;           // grouped: {first row, rows of the segment from there on, expert, -} of every row tile
    int32_t tile_rows;           // their rows: 256 (launch_product); 64, 128, 192 or 256 (launch_grouped)
    const int32_t* n_mtiles;     // how many
    int32_t max_mt;              // at most
    int32_t c_mapped;            // set by the launcher: C is stored through a tensor map
    int32_t bn;                  // set by the launcher: columns of a plain tile
    int32_t starve;              // test hook (set by the launchers): nothing is loaded, so the waits run out
    WsHeader* header;
};
enum { EPI_PLAIN = 0, EPI_GATED = 1, EPI_ROWS = 2 };

// Where a token's codes go when its rows are wanted in expert order: row pos[t * k + s] for every routed slot s.
//   n > 0     : the launch makes the whole schedule of the n routes itself (at most ROUTES_HERE): pos, tiles and their number
//   tiles     : it writes the products' list of row tiles from the schedule's tables
//   otherwise : all of it is there
constexpr int ROUTES_HERE = 1024;
struct RouteArgs {
    const int32_t* idx;
    int32_t* pos;
    int32_t E, k, n;
    int32_t tile_rows;
    int4* tiles;
    int32_t* n_tiles;
    const int32_t *tile_expert, *mt_start, *pad_offsets, *counts;
};
cudaError_t launch_quantize(const void* x, int type, long long rows, int K, long long ldx, int8_t* codes, long long ldc,
                            float* scales, cudaStream_t s, const RouteArgs* routes = nullptr);
cudaError_t launch_product(const ProductArgs& a, int epi, cudaStream_t s);
// few rows per expert (EPI_GATED, EPI_ROWS)
cudaError_t launch_grouped(const ProductArgs& a, int epi, cudaStream_t s);
// few tokens (EPI_PLAIN, dense): whether the kernel for them takes the product; quantises: from the activations (of x_type, -1:
// there are only codes)
bool narrow_product(int M, int K, int N, int x_type, unsigned long long x_align, bool* quantises);
cudaError_t launch_narrow(const ProductArgs& a, const void* x, int x_type, long long ldx, cudaStream_t s);
cudaError_t status_header(WsHeader** out);
extern thread_local bool g_starve;    // this thread's launches of products load nothing (mok_i8_starve)

}  // namespace i8
}  // namespace mok
