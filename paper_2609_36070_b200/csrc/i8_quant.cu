// Quantisation of activation rows to 8-bit codes with one scale per row (rule: i8_common.cuh).
#include "i8_common.cuh"

namespace mok {
namespace i8 {

constexpr int THREADS = 256;
constexpr int VEC_PER_THREAD = 8;      // 16-byte pieces of a row that one thread keeps in registers

// `TPR` threads share a row (32: eight rows per block; 256: the block); returns the maximum over them.
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* s_max) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (TPR > 32) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        __syncthreads();
        if (lane == 0) s_max[warp] = v;
        __syncthreads();
        v = __reduce_max_sync(0xffffffffu, lane < THREADS / 32 ? s_max[lane] : 0u);
    }
    return v;
}

// The rows that a quantised row is written to: itself, or with ROUTED one per routed slot of the token.
template <bool ROUTED>
struct Targets {
    long long first;
    const int32_t *idx, *pos;
    int E, n;
    __device__ __forceinline__ Targets(long long r, const RouteArgs& q) : first(r), idx(nullptr), pos(nullptr), E(q.E), n(1) {
        if (ROUTED) {
            n = q.k;
            idx = q.idx + r * q.k;
            pos = q.pos + r * q.k;
        }
    }
    __device__ __forceinline__ long long row(int s) const {          // -1: the slot is not routed
        if (!ROUTED) return first;
        return (unsigned)__ldg(idx + s) < (unsigned)E ? (long long)__ldg(pos + s) : -1;
    }
};

// The 256-row tiles of the experts' segments: {first row, rows of the segment from there on, expert, -}
__device__ __forceinline__ void write_tiles(const RouteArgs& q) {
    const int n = *q.n_mtiles;
    for (int i = blockIdx.x * THREADS + threadIdx.x; i < n; i += gridDim.x * THREADS) {
        const int e = q.tile_expert[i], m = i - q.mt_start[e];
        q.tiles[i] = make_int4(q.pad_offsets[e] + m * 2 * TILE_M, q.counts[e] - m * 2 * TILE_M, e, 0);
    }
}

// Rows of whole 16-byte pieces that fit into the registers of their threads: one pass over memory.
template <class T, int TPR, bool ROUTED>
__global__ void __launch_bounds__(THREADS)
quantize_vec_kernel(const T* __restrict__ x, long long rows, int K, long long ldx, int8_t* __restrict__ codes, long long ldc,
                    float* __restrict__ scales, const RouteArgs routes) {
    constexpr int PER = 16 / sizeof(T);
    __shared__ uint32_t s_max[THREADS / 32];
    pdl_enter();
    if (ROUTED) write_tiles(routes);
    const int sub = threadIdx.x % TPR, pieces = K / PER;
    constexpr int ROWS = THREADS / TPR;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < rows; r0 += (long long)gridDim.x * ROWS) {
        const long long r = r0 + threadIdx.x / TPR;
        const bool live = r < rows;                  // (whole warps: TPR >= 32)
        const uint4* src = reinterpret_cast<const uint4*>(x + (live ? r : 0) * ldx);
        uint4 raw[VEC_PER_THREAD];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < VEC_PER_THREAD; ++i) {
            const int c = sub + i * TPR;
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if (live && c < pieces) raw[i] = __ldg(src + c);
        }
#pragma unroll
        for (int i = 0; i < VEC_PER_THREAD; ++i) {
            const T* v = reinterpret_cast<const T*>(&raw[i]);
#pragma unroll
            for (int j = 0; j < PER; ++j) m = max(m, abs_bits(to_f(v[j])));
        }
        m = row_max<TPR>(m, s_max);
        if (!live) continue;
        const float amax = __uint_as_float(m);
        const bool codable = m > 0 && finite_bits(m);
        const RowRule rule = row_rule(amax);
        uint32_t o[VEC_PER_THREAD][PER / 4];
#pragma unroll
        for (int i = 0; i < VEC_PER_THREAD; ++i) {
            const T* v = reinterpret_cast<const T*>(&raw[i]);
#pragma unroll
            for (int q = 0; q < PER / 4; ++q) {
                o[i][q] = 0u;
                if (codable && sub + i * TPR < pieces)
                    o[i][q] = pack4(code_bits(to_f(v[4 * q]), rule), code_bits(to_f(v[4 * q + 1]), rule),
                                    code_bits(to_f(v[4 * q + 2]), rule), code_bits(to_f(v[4 * q + 3]), rule));
            }
        }
        const Targets<ROUTED> to(r, routes);
        for (int s = 0; s < to.n; ++s) {
            const long long row = to.row(s);
            if (row < 0) continue;
            int8_t* dst = codes + row * ldc;
#pragma unroll
            for (int i = 0; i < VEC_PER_THREAD; ++i) {
                const int c = sub + i * TPR;
                if (c >= pieces) break;
                if (PER == 8) *reinterpret_cast<uint2*>(dst + c * 8) = make_uint2(o[i][0], o[i][PER / 4 - 1]);
                else *reinterpret_cast<uint32_t*>(dst + c * 4) = o[i][0];
            }
            if (sub == 0) scales[row] = amax / 127.f;
            for (int c = K + sub; c < ldc && c < K + 16; c += TPR) dst[c] = 0;     // the pitch's tail
        }
    }
}

// Any length, stride and alignment: one block per row, two passes (the second one hits the caches).
template <class T, bool ROUTED>
__global__ void __launch_bounds__(THREADS)
quantize_any_kernel(const T* __restrict__ x, long long rows, int K, long long ldx, int8_t* __restrict__ codes, long long ldc,
                    float* __restrict__ scales, const RouteArgs routes) {
    __shared__ uint32_t s_max[THREADS / 32];
    pdl_enter();
    if (ROUTED) write_tiles(routes);
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* src = x + r * ldx;
        uint32_t m = 0;
        for (int c = threadIdx.x; c < K; c += THREADS) m = max(m, abs_bits(to_f(src[c])));
        m = row_max<THREADS>(m, s_max);
        const float amax = __uint_as_float(m);
        const bool codable = m > 0 && finite_bits(m);
        const RowRule rule = row_rule(amax);
        const Targets<ROUTED> to(r, routes);
        for (int s = 0; s < to.n; ++s) {
            const long long row = to.row(s);
            if (row < 0) continue;
            int8_t* dst = codes + row * ldc;
            for (int c = threadIdx.x; c < K; c += THREADS)
                dst[c] = codable ? (int8_t)(code_bits(to_f(src[c]), rule) & 0xffu) : (int8_t)0;
            if (threadIdx.x == 0) scales[row] = amax / 127.f;
            for (int c = K + threadIdx.x; c < ldc && c < K + 16; c += THREADS) dst[c] = 0;
        }
    }
}

template <class T, bool ROUTED>
static cudaError_t launch_typed(const void* xv, long long rows, int K, long long ldx, int8_t* codes, long long ldc, float* scales,
                                const RouteArgs& routes, cudaStream_t s) {
    constexpr int PER = 16 / sizeof(T);
    const T* x = reinterpret_cast<const T*>(xv);
    const bool one = rows == 1 && !ROUTED;
    const bool vec = (reinterpret_cast<uintptr_t>(x) & 15u) == 0 && K % PER == 0 && (ldx % PER == 0 || rows == 1) &&
                     (reinterpret_cast<uintptr_t>(codes) & 15u) == 0 && (ldc % 16 == 0 || one);
    const long long most = 148 * 16;
    if (vec && K <= 32 * VEC_PER_THREAD * PER && rows >= 148 * 8) {      // enough rows for a warp each
        const long long blocks = (rows + 7) / 8;
        return launch_pdl(quantize_vec_kernel<T, 32, ROUTED>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(THREADS), 0, s,
                          x, rows, K, ldx, codes, ldc, scales, routes);
    }
    const dim3 grid((unsigned)(rows < most ? rows : most));
    if (vec && K <= THREADS * VEC_PER_THREAD * PER)
        return launch_pdl(quantize_vec_kernel<T, THREADS, ROUTED>, grid, dim3(THREADS), 0, s, x, rows, K, ldx, codes, ldc, scales,
                          routes);
    return launch_pdl(quantize_any_kernel<T, ROUTED>, grid, dim3(THREADS), 0, s, x, rows, K, ldx, codes, ldc, scales, routes);
}

cudaError_t launch_quantize(const void* x, int type, long long rows, int K, long long ldx, int8_t* codes, long long ldc,
                            float* scales, cudaStream_t s, const RouteArgs* routes) {
    if (routes)          // (16-bit activations only)
        return type == MOK_TYPE_F16 ? launch_typed<__half, true>(x, rows, K, ldx, codes, ldc, scales, *routes, s)
                                    : launch_typed<__nv_bfloat16, true>(x, rows, K, ldx, codes, ldc, scales, *routes, s);
    const RouteArgs none = {};
    if (type == MOK_TYPE_F32) return launch_typed<float, false>(x, rows, K, ldx, codes, ldc, scales, none, s);
    if (type == MOK_TYPE_F16) return launch_typed<__half, false>(x, rows, K, ldx, codes, ldc, scales, none, s);
    return launch_typed<__nv_bfloat16, false>(x, rows, K, ldx, codes, ldc, scales, none, s);
}

}  // namespace i8
}  // namespace mok
