// Quantisation of activation rows to 8-bit codes with one scale per row (rule: i8_common.cuh).
#include "i8_common.cuh"

namespace mok {
namespace i8 {

constexpr int THREADS = 256;
constexpr int HELD = 4;                // 16-byte pieces of a row that one thread keeps in registers: with more, too few
                                       // blocks fit on an SM to cover the memory's latency

// `TPR` threads share a row (a warp, or the warps of a part of the block); returns the maximum over them.  Called by all threads.
template <int TPR, int BLOCK>
__device__ __forceinline__ uint32_t row_max(uint32_t v, uint32_t* s_max) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (TPR > 32) {
        constexpr int WARPS = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        __syncthreads();
        if (lane == 0) s_max[warp] = v;
        __syncthreads();
        v = __reduce_max_sync(0xffffffffu, lane < WARPS ? s_max[warp / WARPS * WARPS + lane] : 0u);
    }
    return v;
}

// The rows that a quantised row is written to: itself, or with ROUTED one per routed slot of the token (here: their places in
// shared memory, or NULL).
template <bool ROUTED>
struct Targets {
    long long first;
    const int32_t *idx, *pos, *here;
    int E, n;
    __device__ __forceinline__ Targets(long long r, const RouteArgs& q, const int32_t* places)
        : first(r), idx(nullptr), pos(nullptr), here(places), E(q.E), n(1) {
        if (ROUTED) {
            n = q.k;
            idx = q.idx + r * q.k;
            pos = q.pos + r * q.k;
        }
    }
    __device__ __forceinline__ long long row(int s) const {          // -1: the slot is not routed
        if (!ROUTED) return first;
        if (here) return here[s];
        return (unsigned)__ldg(idx + s) < (unsigned)E ? (long long)pos[s] : -1;
    }
};

// The schedule of a small batch, in every block of the quantisation (one block per token) instead of a launch before it: the
// counts of all experts, the starts of their segments, and the places of token r's rows (the routes of an expert in their
// order).  Block 0 also writes the list of row tiles.
template <int BLOCK>
__device__ __forceinline__ void schedule_here(const RouteArgs& q, long long r, int32_t* s_place) {
    constexpr int PER = MAX_E / BLOCK, WARPS = BLOCK / 32;           // experts per thread
    __shared__ int32_t s_cnt[MAX_E], s_row0[MAX_E], s_sums[2][WARPS];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int e = tid; e < MAX_E; e += BLOCK) s_cnt[e] = 0;
    __syncthreads();
    for (int j = tid; j < q.n; j += BLOCK) {
        const int e = __ldg(q.idx + j);
        if ((unsigned)e < (unsigned)q.E) atomicAdd(&s_cnt[e], 1);
    }
    __syncthreads();
    int pads = 0, tiles = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = s_cnt[tid * PER + i];
        pads += (c + TILE_M - 1) / TILE_M;
        tiles += (c + q.tile_rows - 1) / q.tile_rows;
    }
    int pads_to = pads, tiles_to = tiles;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int p = __shfl_up_sync(0xffffffffu, pads_to, off), t = __shfl_up_sync(0xffffffffu, tiles_to, off);
        if (lane >= off) { pads_to += p; tiles_to += t; }
    }
    if (lane == 31) { s_sums[0][warp] = pads_to; s_sums[1][warp] = tiles_to; }
    __syncthreads();
    for (int w = 0; w < warp; ++w) { pads_to += s_sums[0][w]; tiles_to += s_sums[1][w]; }
    int row0 = (pads_to - pads) * TILE_M, tile = tiles_to - tiles;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = tid * PER + i, c = s_cnt[e];
        s_row0[e] = row0;
        if (blockIdx.x == 0)
            for (int m = 0; m < c; m += q.tile_rows) q.tiles[tile++] = make_int4(row0 + m, c - m, e, 0);
        row0 += (c + TILE_M - 1) / TILE_M * TILE_M;
    }
    if (blockIdx.x == 0 && tid == BLOCK - 1) *q.n_tiles = tiles_to;
    __syncthreads();
    for (int s = warp; s < q.k; s += WARPS) {
        const int j0 = (int)r * q.k + s, e = __ldg(q.idx + j0);
        int before = 0;
        for (int j = lane; j < j0; j += 32) before += __ldg(q.idx + j) == e ? 1 : 0;
        before = __reduce_add_sync(0xffffffffu, before);
        if (lane == 0) {
            const bool routed = (unsigned)e < (unsigned)q.E;
            s_place[s] = routed ? s_row0[e] + before : -1;
            if (routed) q.pos[j0] = s_row0[e] + before;
        }
    }
    __syncthreads();
}

// The row tiles of the experts' segments: {first row, rows of the segment from there on, expert, -}
__device__ __forceinline__ void write_tiles(const RouteArgs& q) {
    const int n = *q.n_tiles;
    for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) {
        const int e = q.tile_expert[i], m = i - q.mt_start[e];
        q.tiles[i] = make_int4(q.pad_offsets[e] + m * q.tile_rows, q.counts[e] - m * q.tile_rows, e, 0);
    }
}

// Rows of whole 16-byte pieces that fit into the registers of their threads: one pass over memory.
template <class T, int TPR, int BLOCK, bool ROUTED>
__global__ void __launch_bounds__(BLOCK, 1280 / BLOCK)
quantize_vec_kernel(const T* __restrict__ x, long long rows, int K, long long ldx, int8_t* __restrict__ codes, long long ldc,
                    float* __restrict__ scales, const RouteArgs routes) {
    constexpr int PER = 16 / sizeof(T);
    __shared__ uint32_t s_max[BLOCK / 32];
    __shared__ int32_t s_place[ROUTED ? MAX_K : 1];
    pdl_enter();
    if (ROUTED && routes.n == 0 && routes.tiles) write_tiles(routes);
    const int sub = threadIdx.x % TPR, pieces = K / PER, padded = (K + 15) & ~15;
    constexpr int ROWS = BLOCK / TPR;
    for (long long r0 = (long long)blockIdx.x * ROWS; r0 < rows; r0 += (long long)gridDim.x * ROWS) {
        const long long r = r0 + threadIdx.x / TPR;
        const bool live = r < rows;
        const uint4* src = reinterpret_cast<const uint4*>(x + (live ? r : 0) * ldx);
        uint4 raw[HELD];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int c = sub + i * TPR;
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            if (live && c < pieces) raw[i] = __ldg(src + c);
        }
        if constexpr (ROUTED && TPR == BLOCK) {          // (while the row is on its way)
            if (routes.n > 0) schedule_here<BLOCK>(routes, r, s_place);
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const T* v = reinterpret_cast<const T*>(&raw[i]);
#pragma unroll
            for (int j = 0; j < PER; ++j) m = max(m, abs_bits(to_f(v[j])));
        }
        m = row_max<TPR, BLOCK>(m, s_max);
        if (!live) continue;
        const float amax = __uint_as_float(m);
        const bool codable = m > 0 && finite_bits(m);
        const RowRule rule = row_rule(amax);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {         // the codes take the place of the values
            const T* v = reinterpret_cast<const T*>(&raw[i]);
            uint2 o = make_uint2(0u, 0u);
            if (codable && sub + i * TPR < pieces) {
                o.x = four_codes(to_f(v[0]), to_f(v[1]), to_f(v[2]), to_f(v[3]), rule);
                if (PER == 8) o.y = four_codes(to_f(v[PER - 4]), to_f(v[PER - 3]), to_f(v[PER - 2]), to_f(v[PER - 1]), rule);
            }
            raw[i].x = o.x;
            raw[i].y = o.y;
        }
        const Targets<ROUTED> to(r, routes, ROUTED && routes.n > 0 ? s_place : nullptr);
        for (int s = 0; s < to.n; ++s) {
            const long long row = to.row(s);
            if (row < 0) continue;
            int8_t* dst = codes + row * ldc;
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int c = sub + i * TPR;
                if (c >= pieces) break;
                if (PER == 8) *reinterpret_cast<uint2*>(dst + c * 8) = make_uint2(raw[i].x, raw[i].y);
                else *reinterpret_cast<uint32_t*>(dst + c * 4) = raw[i].x;
            }
            if (sub == 0) scales[row] = amax / 127.f;
            if (K + sub < padded && K + sub < ldc) dst[K + sub] = 0;               // (fewer than 16 bytes)
        }
    }
}

// Any length, stride and alignment: one block per row, two passes (the second one hits the caches).
template <class T, bool ROUTED>
__global__ void __launch_bounds__(THREADS)
quantize_any_kernel(const T* __restrict__ x, long long rows, int K, long long ldx, int8_t* __restrict__ codes, long long ldc,
                    float* __restrict__ scales, const RouteArgs routes) {
    __shared__ uint32_t s_max[THREADS / 32];
    __shared__ int32_t s_place[ROUTED ? MAX_K : 1];
    pdl_enter();
    if (ROUTED && routes.n == 0 && routes.tiles) write_tiles(routes);
    const int padded = (K + 15) & ~15;
    for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* src = x + r * ldx;
        if constexpr (ROUTED) {
            if (routes.n > 0) schedule_here<THREADS>(routes, r, s_place);
        }
        uint32_t m = 0;
        for (int c = threadIdx.x; c < K; c += THREADS) m = max(m, abs_bits(to_f(src[c])));
        m = row_max<THREADS, THREADS>(m, s_max);
        const float amax = __uint_as_float(m);
        const bool codable = m > 0 && finite_bits(m);
        const RowRule rule = row_rule(amax);
        const Targets<ROUTED> to(r, routes, ROUTED && routes.n > 0 ? s_place : nullptr);
        for (int s = 0; s < to.n; ++s) {
            const long long row = to.row(s);
            if (row < 0) continue;
            int8_t* dst = codes + row * ldc;
            for (int c = threadIdx.x; c < K; c += THREADS)
                dst[c] = codable ? (int8_t)(code_bits(to_f(src[c]), rule) & 0xffu) : (int8_t)0;
            if (threadIdx.x == 0) scales[row] = amax / 127.f;
            if (K + (int)threadIdx.x < padded && K + (int)threadIdx.x < ldc) dst[K + threadIdx.x] = 0;
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
    // as few threads per row as hold it: a warp needs no barrier, but few rows want more threads each
    const bool many = rows >= 148 * 8;
    auto blocks = [&](int per_block) {
        const long long n = (rows + per_block - 1) / per_block;
        return dim3((unsigned)(n < most ? n : most));
    };
#define MOK_ROWS(TPR, BLOCK)                                                                                                   \
    return launch_pdl(quantize_vec_kernel<T, TPR, BLOCK, ROUTED>, blocks(BLOCK / TPR), dim3(BLOCK), 0, s, x, rows, K, ldx, codes, \
                      ldc, scales, routes)
    if (vec && many && K <= 32 * HELD * PER) MOK_ROWS(32, 256);
    if (vec && many && K <= 64 * HELD * PER) MOK_ROWS(64, 256);
    if (vec && many && K <= 128 * HELD * PER) MOK_ROWS(128, 256);
    if (vec && K <= 256 * HELD * PER) MOK_ROWS(256, 256);
    if (vec && K <= 512 * HELD * PER) MOK_ROWS(512, 512);
#undef MOK_ROWS
    const dim3 grid = blocks(1);
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
