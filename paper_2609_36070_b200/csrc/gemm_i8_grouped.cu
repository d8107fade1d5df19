// Expert products of 8-bit operands with few rows per expert (a decoding step, a chunk of a prompt): bound by streaming the
// weights of the experts that are met.  As in the dense kernel for few tokens the weights sit on the MMA's M side (128 rows),
// the tokens of one expert on its N side (16 to 256 columns, as many as the tile has), so an expert with two rows costs its
// weights and nothing else: 256-row tiles would pull 256 mostly empty token rows beside every weight tile.
//
// Persistent CTAs over the list of (row tile, channel tile):
//   warp 0       TMA producer: 128 weight rows and the tile's token rows per 128 bytes of K; eight, six, five or four stages for
//                tiles of at most 64, 128, 192 or 256 rows
//   warp 1       MMA issuer (tcgen05.mma.kind::i8, M = 128), two accumulators
//   warps 2..9   epilogue: lane = channel, so that stores are coalesced as they are
//   EPI_GATED : the M side holds 64 gate rows and the 64 matching up rows; the warps of the up lanes hand their values over
//               through shared memory, those of the gate lanes write h = silu(g) u as fp32
//   EPI_ROWS  : sums times the channel's scale, as fp32 (see gemm_i8.cu)
// All mbarrier waits are bounded; on a timeout the CTA records MOK_ERR_TIMEOUT and leaves cleanly.
#include "i8_common.cuh"
#include "i8_ptx.cuh"
#include "tensor_map.cuh"

namespace mok {
namespace i8 {

using namespace tc;

constexpr int G_EPI = 8, G_THREADS = 64 + 32 * G_EPI;
constexpr int G_MAX_STAGES = 8;
// ROWS: most rows of a tile
template <int ROWS> struct Grouped {
    static constexpr int STAGES = ROWS == 64 ? 8 : ROWS == 128 ? 6 : ROWS == 192 ? 5 : 4, STAGE = 16384 + ROWS * 128;      // weights, tokens
    static constexpr int XCHG = STAGES * STAGE;              // up values: 4 warp pairs x 2 buffers x [16 tokens][32 channels]
    static constexpr int CTRL = XCHG + 4 * 2 * 2048;
    static constexpr int SMEM = CTRL + 512;
    static_assert(SMEM <= 232448, "shared memory of one CTA");
};

struct GroupedCtrl {
    uint64_t full[G_MAX_STAGES], empty[G_MAX_STAGES], tfull[2], tempty[2];
    uint64_t xfull[4][2], xempty[4][2];          // the exchange buffers of the four warp pairs
    uint32_t tmem_base, abort;
};
static_assert(sizeof(GroupedCtrl) <= 512, "control block too large");

struct RowTile { int row0, n, e, valid; };
__device__ __forceinline__ RowTile row_tile(const ProductArgs& a, int L, int n_nt) {
    const int q = L / n_nt;
    const int4 d = __ldg(a.tiles + q);
    return RowTile{d.x, L - q * n_nt, d.z, min(d.y, a.tile_rows)};
}
__device__ __forceinline__ int columns(int valid) { return (valid + 15) & ~15; }      // N of the MMA

template <int EPI, int ROWS>
__global__ void __launch_bounds__(G_THREADS, 1)
product_grouped_kernel(const __grid_constant__ CUtensorMap tmapW, const __grid_constant__ CUtensorMap tmap16,
                       const __grid_constant__ CUtensorMap tmap64, const __grid_constant__ CUtensorMap tmap128,
                       const __grid_constant__ CUtensorMap tmapRows, const __grid_constant__ ProductArgs a, const int n_nt, const int k_blocks) {
    constexpr bool GATED = EPI == EPI_GATED;
    using G = Grouped<ROWS>;
    constexpr uint32_t TMEM_COLUMNS = ROWS <= 64 ? 128u : ROWS <= 128 ? 256u : 512u;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    GroupedCtrl* ctrl = reinterpret_cast<GroupedCtrl*>(smem + G::CTRL);
    volatile uint32_t* abort_flag = &ctrl->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < G::STAGES; ++s) {
            mbar_init(smem_u32(&ctrl->full[s]), 1);
            mbar_init(smem_u32(&ctrl->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&ctrl->tfull[b]), 1);
            mbar_init(smem_u32(&ctrl->tempty[b]), G_EPI);
            for (int p = 0; p < 4; ++p) {
                mbar_init(smem_u32(&ctrl->xfull[p][b]), 1);
                mbar_init(smem_u32(&ctrl->xempty[p][b]), 1);
            }
        }
        ctrl->abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&ctrl->tmem_base)), "r"(TMEM_COLUMNS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctrl->tmem_base;
    pdl_enter();
    int n_mt = *a.n_mtiles;
    if (n_mt > a.max_mt) n_mt = a.max_mt;
    const int total = n_mt * n_nt;

    if (warp == 0) {
        if (lane == 0 && !a.starve) {
            int s = 0;
            uint32_t ph = 0;
            RowTile next = {};
            if ((int)blockIdx.x < total) next = row_tile(a, blockIdx.x, n_nt);
            for (int L = blockIdx.x; L < total; L += gridDim.x) {
                const RowTile t = next;
                if (L + (int)gridDim.x < total) next = row_tile(a, L + gridDim.x, n_nt);
                const int cols = columns(t.valid);
                const CUtensorMap* map = cols <= 16 ? &tmap16 : ROWS == 64 || cols <= 64 ? &tmap64 : ROWS == 128 || cols <= 128 ? &tmap128 : &tmapRows;
                const uint32_t box = cols <= 16 ? 16u : ROWS == 64 || cols <= 64 ? 64u : ROWS == 128 || cols <= 128 ? 128u : (uint32_t)ROWS;
                const uint32_t bytes = 16384u + box * 128u;
                const int wrow = GATED ? t.e * 2 * a.N + t.n * 64 : t.e * a.N + t.n * 128;
                bool ok = true;
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = mbar_wait(smem_u32(&ctrl->empty[s]), ph ^ 1u, abort_flag, a.header, 31);
                    if (!ok) break;
                    const uint32_t full = smem_u32(&ctrl->full[s]), sw = base + s * G::STAGE;
                    mbar_expect_tx(full, bytes);
                    tma_load_2d(sw, &tmapW, full, kb * 128, wrow);               // 64 rows: gate, or the first half
                    tma_load_2d(sw + 8192, &tmapW, full, kb * 128, wrow + (GATED ? a.N : 64));
                    tma_load_2d(sw + 16384, map, full, kb * 128, t.row0);
                    if (++s == G::STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            int s = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            RowTile next = {};
            if ((int)blockIdx.x < total) next = row_tile(a, blockIdx.x, n_nt);
            for (int L = blockIdx.x; L < total; L += gridDim.x) {
                const RowTile t = next;
                if (L + (int)gridDim.x < total) next = row_tile(a, L + gridDim.x, n_nt);
                const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(columns(t.valid) >> 3) << 17) | (8u << 24);
                bool ok = mbar_wait(smem_u32(&ctrl->tempty[buf]), aph ^ 1u, abort_flag, a.header, 32);
                if (!ok) break;
                tc_fence_after();
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = mbar_wait(smem_u32(&ctrl->full[s]), ph, abort_flag, a.header, 33);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t adesc = make_smem_desc(base + s * G::STAGE), bdesc = make_smem_desc(base + s * G::STAGE + 16384);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_one(tmem + buf * ROWS, adesc + (uint64_t)(j * 2), bdesc + (uint64_t)(j * 2), idesc, (kb | j) ? 1u : 0u);
                    tc_commit<1>(smem_u32(&ctrl->empty[s]));
                    if (++s == G::STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                tc_commit<1>(smem_u32(&ctrl->tfull[buf]));
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        // warp's lanes of the accumulator (quad) and its 16-column groups: half, half + 2, ...
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const int pair = half * 2 + (quad & 1);
        float* xchg = reinterpret_cast<float*>(smem + G::XCHG + pair * 4096);
        int buf = 0, flip = 0;
        uint32_t aph = 0, xph = 0;
        RowTile next = {};
        if ((int)blockIdx.x < total) next = row_tile(a, blockIdx.x, n_nt);
        for (int L = blockIdx.x; L < total; L += gridDim.x) {
            const RowTile t = next;
            if (L + (int)gridDim.x < total) next = row_tile(a, L + gridDim.x, n_nt);
            const int n = GATED ? t.n * 64 + (quad & 1) * 32 + lane : t.n * 128 + quad * 32 + lane;     // the lane's channel
            const bool there = n < a.N;
            float f = 0.f;
            if (there) f = GATED ? __ldg(a.b_scale + ((size_t)t.e * 2 + (quad >> 1)) * a.N + n) : __ldg(a.b_scale + (size_t)t.e * a.N + n);
            float xs[ROWS / 32];                           // lane l: scale of the tile's rows l, l + 32, ...
            if (GATED) {
#pragma unroll
                for (int i = 0; i < ROWS / 32; ++i) xs[i] = lane + 32 * i < t.valid ? __ldg(a.a_scale + t.row0 + lane + 32 * i) : 0.f;
            }
            bool ok = mbar_wait(smem_u32(&ctrl->tfull[buf]), aph, abort_flag, a.header, 34);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem + buf * ROWS + ((uint32_t)(quad * 32) << 16);
#pragma unroll
            for (int i = 0; i < ROWS / 32; ++i) {
                const int c = i * 32 + half * 16;            // first token of the group
                if (c >= t.valid) break;
                uint32_t acc[16];
                tc_ld16(taddr + c, acc);
                tc_wait_ld();
                if (GATED) {
                    float v[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) v[j] = (float)(int)acc[j] * __shfl_sync(0xffffffffu, xs[i], half * 16 + j) * f;
                    float* mine = xchg + flip * 512;
                    const uint32_t filled = smem_u32(&ctrl->xfull[pair][flip]), freed = smem_u32(&ctrl->xempty[pair][flip]);
                    if (quad >= 2) {
                        ok = mbar_wait(freed, xph ^ 1u, abort_flag, a.header, 35);
#pragma unroll
                        for (int j = 0; j < 16; ++j) mine[j * 32 + lane] = v[j];
                        __syncwarp();
                        if (lane == 0) mbar_arrive(filled);
                    } else {
                        ok = mbar_wait(filled, xph, abort_flag, a.header, 36);
                    }
                    if (!__all_sync(0xffffffffu, ok)) break;
                    if (quad < 2 && there) {
                        float* dst = reinterpret_cast<float*>(a.C) + (long long)(t.row0 + c) * a.ldc + n;
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (c + j < t.valid) dst[j * a.ldc] = gated(v[j], mine[j * 32 + lane]);
                    }
                    if (quad < 2) {
                        __syncwarp();
                        if (lane == 0) mbar_arrive(freed);
                    }
                    flip ^= 1;
                    xph ^= flip ^ 1;                         // (both buffers have been used once more)
                } else if (there) {
                    float* dst = reinterpret_cast<float*>(a.C) + (long long)(t.row0 + c) * a.ldc + n;
#pragma unroll
                    for (int j = 0; j < 16; ++j)
                        if (c + j < t.valid) dst[j * a.ldc] = (float)(int)acc[j] * f;
                }
            }
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctrl->tempty[buf]));
            if (++buf == 2) { buf = 0; aph ^= 1u; }
        }
    }

    if (*abort_flag) {   // failure path only: give copies and MMAs already in flight time to land before leaving
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 200000ull) { }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLUMNS) : "memory");
    }
}

template <int EPI, int ROWS>
static cudaError_t launch_grouped_epi(const CUtensorMap& mW, const CUtensorMap (&mX)[4], const ProductArgs& a, int n_nt, int k_blocks,
                                      long long tiles, cudaStream_t s) {
    static PerDevice configured;
    auto kernel = product_grouped_kernel<EPI, ROWS>;
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    e = configured.get(dev, &sms, [&](int d, int* n) {
        cudaError_t e2 = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Grouped<ROWS>::SMEM);
        return e2 == cudaSuccess ? device_sm_count(d, n) : e2;
    });
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, dim3((unsigned)(tiles < sms ? tiles : sms)), dim3(G_THREADS), (size_t)Grouped<ROWS>::SMEM, s, mW, mX[0],
                      mX[1], mX[2], mX[3], a, n_nt, k_blocks);
}

cudaError_t launch_grouped(const ProductArgs& args, int epi, cudaStream_t s) {
    ProductArgs a = args;
    a.starve = g_starve;
    const bool is_gated = epi == EPI_GATED;
    CUtensorMap mW, mX[4];
    auto map = [&](CUtensorMap* m, const void* p, long long rows, long long pitch, uint32_t box) {
        return tmap::encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, p, (uint64_t)rows, (uint64_t)a.K, (uint64_t)pitch, 128, box,
                               CU_TENSOR_MAP_SWIZZLE_128B);
    };
    if (!map(&mW, a.B, (long long)a.E * (is_gated ? 2 : 1) * a.N, a.ldb, 64) || !map(&mX[0], a.A, a.a_rows, a.lda, 16) ||
        !map(&mX[1], a.A, a.a_rows, a.lda, 64) || !map(&mX[2], a.A, a.a_rows, a.lda, 128) ||
        !map(&mX[3], a.A, a.a_rows, a.lda, a.tile_rows == 192 ? 192 : 256))
        return cudaErrorInvalidValue;
    const int n_nt = is_gated ? (a.N + 63) / 64 : (a.N + 127) / 128, k_blocks = (a.K + 127) / 128;
    const long long tiles = (long long)a.max_mt * n_nt;
    if (tiles <= 0 || tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    if (a.tile_rows == 64)
        return is_gated ? launch_grouped_epi<EPI_GATED, 64>(mW, mX, a, n_nt, k_blocks, tiles, s)
                        : launch_grouped_epi<EPI_ROWS, 64>(mW, mX, a, n_nt, k_blocks, tiles, s);
    if (a.tile_rows == 128)
        return is_gated ? launch_grouped_epi<EPI_GATED, 128>(mW, mX, a, n_nt, k_blocks, tiles, s)
                        : launch_grouped_epi<EPI_ROWS, 128>(mW, mX, a, n_nt, k_blocks, tiles, s);
    if (a.tile_rows == 192)
        return is_gated ? launch_grouped_epi<EPI_GATED, 192>(mW, mX, a, n_nt, k_blocks, tiles, s)
                        : launch_grouped_epi<EPI_ROWS, 192>(mW, mX, a, n_nt, k_blocks, tiles, s);
    if (a.tile_rows != 256) return cudaErrorInvalidValue;
    return is_gated ? launch_grouped_epi<EPI_GATED, 256>(mW, mX, a, n_nt, k_blocks, tiles, s)
                    : launch_grouped_epi<EPI_ROWS, 256>(mW, mX, a, n_nt, k_blocks, tiles, s);
}

}  // namespace i8
}  // namespace mok
