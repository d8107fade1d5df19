// Products of 8-bit integer operands on the tensor cores (tcgen05.mma.kind::i8, K = 32 per instruction, exact 32-bit integer
// sums in TMEM), scaled in fp32 as they leave: out[r, n] = a_scale[r] * b_scale[n] * sum_k A[r, k] B[n, k].
//
// Persistent, warp-specialised, on CTA pairs: the two CTAs of a cluster compute one 256 x 256 tile with cta_group::2 MMAs
// issued by the even CTA.  Each CTA stages its own 128 rows of A and half of the 256 rows of B (128 bytes of K per stage, 32 KB,
// six stages), so an SM pulls 32 KB for 512 cycles of MMA; a 128 x 256 tile of one CTA would pull 48 KB for them, and with all
// SMs at work that rate, some 45 bytes per cycle, is the limit.  The plain product also takes narrower tiles (down to 128
// columns) where they spread the work better over the SMs.
//   warp 0       TMA producer : A and B tiles (128-byte swizzle)
//   warp 1       MMA issuer (even CTA)
//   warps 2..9   epilogue     : warp w drains TMEM lane quadrant w % 4 and one half of the tile's columns
// Two 256-column accumulators: a tile's epilogue runs beside the next tile's products.
//
//   EPI_PLAIN : C = scaled sums (+ bias) as bf16, fp16 or fp32, one rounding
//   EPI_GATED : B tile = 128 gate rows (even CTA) + the matching 128 up rows (odd CTA); h = silu(g) u in fp32 -> C fp32.  h is
//               quantised by a pass of its own, since its row maximum spans all N tiles; fp32 because a rounding before the
//               quantisation moves codes (bf16 moves one code in twenty).
//   EPI_ROWS  : C = b_scale[n] * sum as fp32, whatever the type of the layer's output: the combine puts a row's scale on with
//               its weight, adds up a token's rows in fp32 and rounds once.  (16-bit rows would spare half of the path's largest stream, but round every row a second
//               time, and a common unit for them loses the channels whose scales are far below their matrix's largest.)
// K, N and the rows may be ragged: TMA fills bytes past K and rows past the tensor with zeros, stores are masked.
// All mbarrier waits are bounded; on a timeout the CTA records MOK_ERR_TIMEOUT and leaves cleanly.
#include "i8_common.cuh"
#include "i8_ptx.cuh"
#include "tensor_map.cuh"

namespace mok {
namespace i8 {

using namespace tc;

constexpr int BM = 128, BN = 256, BKB = 128;
constexpr int A_BYTES = BM * BKB, B_BYTES = BN / 2 * BKB, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int STAGES = 6;
constexpr int EPI_WARPS = 8;
constexpr int SLAB_BYTES = 2048;                 // 32 rows of 64 bytes; two per epilogue warp
constexpr int SLAB_REGION = STAGES * STAGE_BYTES;
constexpr int SCALE_REGION = SLAB_REGION + EPI_WARPS * 2 * SLAB_BYTES;      // per epilogue warp: 2 x 32 column factors
constexpr int CTRL_REGION = SCALE_REGION + EPI_WARPS * 256;
constexpr int SMEM_BYTES = CTRL_REGION + 256;
constexpr int TMEM_COLS = 512;
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int GROUP_ROWS = 2048;

struct Ctrl {
    uint64_t full[STAGES], empty[STAGES], tfull[2], tempty[2];
    uint32_t tmem_base, abort;
};
static_assert(sizeof(Ctrl) <= 256, "control block too large");
static_assert(SMEM_BYTES <= 232448, "shared memory of one CTA");

// D s32, A and B signed 8-bit, both K-major
__device__ __forceinline__ constexpr uint32_t make_idesc(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void mma_pair(uint32_t d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void st_shared_f32(uint32_t addr, float v) {
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ float4 ld_shared_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

struct PairTile { int row0, n, e, valid; };     // n: column tile; valid: rows of the segment from row0 on

__device__ __forceinline__ PairTile pair_tile(const ProductArgs& a, int L, int n_nt, int n_mt) {
    PairTile t;
    if (a.dense_rows <= 0) {
        // one load from the tile list: a chain of look-ups (expert, first tile, offset) costs as much as a short tile's products
        const int q = L / n_nt;
        const int4 d = __ldg(a.tiles + q);
        t.row0 = d.x; t.valid = d.y; t.e = d.z;
        t.n = L - q * n_nt;
        return t;
    }
    // row tiles in groups of GROUP_ROWS rows, fastest inside a group: its rows stay in L2 while the weight tiles stream
    constexpr int group_m = GROUP_ROWS / (2 * BM);
    const int g = L / (group_m * n_nt);
    const int rem = L - g * group_m * n_nt;
    const int in_group = min(group_m, n_mt - g * group_m);
    t.e = 0;
    t.n = rem / in_group;
    t.row0 = (g * group_m + rem - t.n * in_group) * 2 * BM;
    t.valid = a.dense_rows - t.row0;
    return t;
}

template <class T> struct Pack;
template <> struct Pack<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t two(float a, float b) { return pack_bf16(a, b); }
    static __device__ __forceinline__ __nv_bfloat16 one(float a) { return __float2bfloat16_rn(a); }
};
template <> struct Pack<float> {
    static __device__ __forceinline__ float one(float a) { return a; }
};
template <> struct Pack<__half> {
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
    static __device__ __forceinline__ __half one(float a) { return __float2half_rn(a); }
};

// Puts 32 rows (lane = row) of 64 bytes into a slab, in the 64-byte swizzle of the tensor map that they are stored through.
__device__ __forceinline__ void stage_row(uint32_t slab, int lane, const uint32_t (&w)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
        st_shared_v4(slab + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
__device__ __forceinline__ void store_wait_read_1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }

// A warp's 32 rows x 32 columns (v = the columns of row `lane`) to C as one or two bulk tensor stores from the warp's slabs:
// no address arithmetic, and rows and columns past the tensor are clipped by the map.  `flip` alternates the slabs.
template <class T>
__device__ __forceinline__ void store_tile(const float (&v)[32], const CUtensorMap* map, uint32_t slabs, int& flip, int col,
                                           int row, int lane) {
    if constexpr (sizeof(T) == 4) {
        if (lane == 0) tma_store_wait_read();
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(v[16 * h + i]);
            stage_row(slabs + h * SLAB_BYTES, lane, w);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map, slabs, col, row);
            tma_store_2d(map, slabs + SLAB_BYTES, col + 16, row);
            tma_store_commit();
        }
    } else {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = Pack<T>::two(v[2 * i], v[2 * i + 1]);
        const uint32_t slab = slabs + flip * SLAB_BYTES;
        flip ^= 1;
        if (lane == 0) store_wait_read_1();          // (the store before the last one was the last user of this slab)
        __syncwarp();
        stage_row(slab, lane, w);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            tma_store_2d(map, slab, col, row);
            tma_store_commit();
        }
    }
}

// The same for a C whose rows are not 16-byte aligned (odd widths): row by row, lanes along the columns.
template <class T>
__device__ __forceinline__ void store_any(const float (&v)[32], uint32_t slabs, T* c, long long ldc, int n_rows, int n_cols, int lane) {
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 32; ++i) st_shared_f32(slabs + lane * 128 + ((i ^ lane) << 2), v[i]);
    __syncwarp();
    if (lane < n_cols) {
        for (int r = 0; r < n_rows; ++r) {
            float f;
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f) : "r"(slabs + r * 128 + ((lane ^ r) << 2)));
            c[(long long)r * ldc + lane] = Pack<T>::one(f);
        }
    }
}

template <int EPI>
__global__ void __launch_bounds__(THREADS, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap tmapA, const __grid_constant__ CUtensorMap tmapB,
                    const __grid_constant__ CUtensorMap tmapC, const __grid_constant__ ProductArgs a, const int n_nt, const int k_blocks) {
    constexpr bool GATED = EPI == EPI_GATED;
    extern __shared__ __align__(1024) uint8_t smem[];       // (the swizzled tiles want 1024-byte boundaries)
    const uint32_t base = smem_u32(smem);
    Ctrl* ctrl = reinterpret_cast<Ctrl*>(smem + CTRL_REGION);
    volatile uint32_t* abort_flag = &ctrl->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const int unit = blockIdx.x >> 1, n_units = gridDim.x >> 1;
    const int bn = EPI == EPI_PLAIN ? a.bn : BN;                     // columns of a tile

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_u32(&ctrl->full[s]), 1);
            mbar_init(smem_u32(&ctrl->empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(smem_u32(&ctrl->tfull[b]), 1);
            mbar_init(smem_u32(&ctrl->tempty[b]), EPI_WARPS * 2);
        }
        ctrl->abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&ctrl->tmem_base)), "r"((uint32_t)TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                              // the peer's barriers exist before anyone arrives on them remotely
    tc_fence_after();
    const uint32_t tmem_base = ctrl->tmem_base;
    pdl_enter();                                 // (the set-up above runs beside the predecessor)
    int n_mt = a.dense_rows > 0 ? (a.dense_rows + 2 * BM - 1) / (2 * BM) : *a.n_mtiles;
    if (n_mt > a.max_mt) n_mt = a.max_mt;
    const int total = n_mt * n_nt;

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0 && !a.starve) {
            int s = 0;
            uint32_t ph = 0;
            PairTile next = {};
            if (unit < total) next = pair_tile(a, unit, n_nt, n_mt);
            for (int L = unit; L < total; L += n_units) {
                const PairTile t = next;
                if (L + n_units < total) next = pair_tile(a, L + n_units, n_nt, n_mt);     // (on its way during this tile)
                const int brow = GATED ? t.e * 2 * a.N + rank * a.N + t.n * (BN / 2) : t.e * a.N + t.n * bn + rank * (bn / 2);
                bool ok = true;
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = mbar_wait(smem_u32(&ctrl->empty[s]), ph ^ 1u, abort_flag, a.header, 1);
                    if (!ok) break;
                    const uint32_t full = smem_u32(&ctrl->full[s]);
                    const uint32_t sa = base + s * STAGE_BYTES, sb = sa + A_BYTES;
                    // the even CTA's barrier collects the bytes of both CTAs of the pair
                    if (rank == 0) mbar_expect_tx(full, 2 * A_BYTES + bn * BKB);
                    tma_load_2d_peer(sa, &tmapA, full, kb * BKB, t.row0 + rank * BM);
                    tma_load_2d_peer(sb, &tmapB, full, kb * BKB, brow);
                    if (++s == STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        if (lane == 0 && rank == 0) {
            const uint32_t idesc = make_idesc(2 * BM, bn);
            int s = 0, buf = 0;
            uint32_t ph = 0, aph = 0;
            for (int L = unit; L < total; L += n_units) {
                bool ok = mbar_wait(smem_u32(&ctrl->tempty[buf]), aph ^ 1u, abort_flag, a.header, 2);
                if (!ok) break;
                tc_fence_after();
                const uint32_t d = tmem_base + (uint32_t)(buf * BN);
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = mbar_wait(smem_u32(&ctrl->full[s]), ph, abort_flag, a.header, 3);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t sa = base + s * STAGE_BYTES;
                    const uint64_t adesc = make_smem_desc(sa), bdesc = make_smem_desc(sa + A_BYTES);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        mma_pair(d, adesc + (uint64_t)(j * 2), bdesc + (uint64_t)(j * 2), idesc, (kb | j) ? 1u : 0u);
                    tc_commit<2>(smem_u32(&ctrl->empty[s]));
                    if (++s == STAGES) { s = 0; ph ^= 1u; }
                }
                if (!ok) break;
                tc_commit<2>(smem_u32(&ctrl->tfull[buf]));
                if (++buf == 2) { buf = 0; aph ^= 1u; }
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ epilogue
        const int quad = warp & 3, half = (warp - 2) >> 2;
        const uint32_t slabs = base + SLAB_REGION + (warp - 2) * 2 * SLAB_BYTES;
        const uint32_t factors = base + SCALE_REGION + (warp - 2) * 256;
        constexpr int CHUNKS = GATED ? 2 : 4;                        // 32-column pieces of this warp
        int buf = 0, flip = 0;
        uint32_t aph = 0;
        PairTile next = {};
        if (unit < total) next = pair_tile(a, unit, n_nt, n_mt);
        for (int L = unit; L < total; L += n_units) {
            const PairTile t = next;
            if (L + n_units < total) next = pair_tile(a, L + n_units, n_nt, n_mt);
            const int r0 = rank * BM + quad * 32;                    // first of the warp's rows inside the tile
            const int n_rows = min(32, t.valid - r0);
            // the row's scale and the warp's column scales, one column of each piece per lane, on their way while the
            // products finish
            const int first = t.n * (GATED ? BN / 2 : bn) + half * 32;           // pieces are dealt to the two halves in turn
            const float* bs = a.b_scale + (size_t)t.e * (GATED ? 2 : 1) * a.N;
            float rs = 0.f;
            if (EPI != EPI_ROWS && lane < n_rows) rs = __ldg(a.a_scale + t.row0 + r0 + lane);
            float s0[CHUNKS], s1[CHUNKS];                            // s1: up scales, or the bias
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int n = first + c * 64 + lane;
                s0[c] = n < a.N ? __ldg(bs + n) : 0.f;
                s1[c] = 0.f;
                if (GATED && n < a.N) s1[c] = __ldg(bs + a.N + n);
                if (EPI == EPI_PLAIN && a.bias && n < a.N) s1[c] = __ldg(a.bias + n);
            }
            bool ok = mbar_wait(smem_u32(&ctrl->tfull[buf]), aph, abort_flag, a.header, 4);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + (uint32_t)(buf * BN + half * 32) + ((uint32_t)(quad * 32) << 16);
            uint32_t acc[2][32], up[2][GATED ? 32 : 1];
            tc_ld32(taddr, acc[0]);
            if constexpr (GATED) tc_ld32(taddr + BN / 2, up[0]);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int b = c & 1;
                st_shared_f32(factors + lane * 4, s0[c]);
                if (EPI != EPI_ROWS) st_shared_f32(factors + 128 + lane * 4, s1[c]);
                tc_wait_ld();
                if (c + 1 < CHUNKS) {                                // the next piece comes while this one is worked on
                    tc_ld32(taddr + (c + 1) * 64, acc[b ^ 1]);       // (columns past a narrow tile: never stored)
                    if constexpr (GATED) tc_ld32(taddr + BN / 2 + (c + 1) * 64, up[b ^ 1]);
                    __syncwarp();
                } else {                                             // the accumulator goes back before the last arithmetic
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(smem_u32(&ctrl->tempty[buf]), 0);
                }
                const int n0 = first + c * 64, n_cols = a.N - n0;    // first output column of the piece, and how many exist
                if (n_rows > 0 && n_cols > 0 && (EPI != EPI_PLAIN || half * 32 + c * 64 < bn)) {
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float4 f = ld_shared_f4(factors + i * 4);
                        const float fs[4] = {f.x, f.y, f.z, f.w};
                        if constexpr (EPI == EPI_ROWS) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) v[i + j] = (float)(int)acc[b][i + j] * fs[j];
                        } else {
                            const float4 q = ld_shared_f4(factors + 128 + i * 4);
                            const float qs[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                v[i + j] = (float)(int)acc[b][i + j] * rs * fs[j];
                                if constexpr (GATED) v[i + j] = gated(v[i + j], (float)(int)up[b][i + j] * rs * qs[j]);
                                else v[i + j] += qs[j];
                            }
                        }
                    }
                    const int row = t.row0 + r0;
                    // (grouped rows are stored in whole blocks of 32: what follows a segment's last row is its own padding)
                    if constexpr (EPI != EPI_PLAIN) {
                        store_tile<float>(v, &tmapC, slabs, flip, n0, row, lane);
                    } else if (a.c_mapped) {
                        if (a.c_type == MOK_TYPE_F32) store_tile<float>(v, &tmapC, slabs, flip, n0, row, lane);
                        else if (a.c_type == MOK_TYPE_F16) store_tile<__half>(v, &tmapC, slabs, flip, n0, row, lane);
                        else store_tile<__nv_bfloat16>(v, &tmapC, slabs, flip, n0, row, lane);
                    } else {
                        const long long at = (long long)row * a.ldc + n0;
                        if (a.c_type == MOK_TYPE_F32) store_any(v, slabs, reinterpret_cast<float*>(a.C) + at, a.ldc, n_rows, n_cols, lane);
                        else if (a.c_type == MOK_TYPE_F16) store_any(v, slabs, reinterpret_cast<__half*>(a.C) + at, a.ldc, n_rows, n_cols, lane);
                        else store_any(v, slabs, reinterpret_cast<__nv_bfloat16*>(a.C) + at, a.ldc, n_rows, n_cols, lane);
                    }
                }
                __syncwarp();                                        // the factors have been read
            }
            if (++buf == 2) { buf = 0; aph ^= 1u; }
        }
        if (lane == 0) tma_store_wait_all();
    }

    // ---------------------------------------------------------------------- teardown
    if (*abort_flag) {   // failure path only: give copies and MMAs already in flight time to land before leaving
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 200000ull) { }
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync();                              // neither CTA frees TMEM or exits while the other may still touch it
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)TMEM_COLS) : "memory");
    }
}

__device__ WsHeader g_header;                    // status word of the 8-bit products of this device (sticky until read)

cudaError_t status_header(WsHeader** out) {
    static std::atomic<WsHeader*> at[MAX_DEVICES];
    int dev = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= MAX_DEVICES) return cudaErrorInvalidDevice;
    WsHeader* p = at[dev].load(std::memory_order_acquire);
    if (!p) {
        void* q = nullptr;
        if ((e = cudaGetSymbolAddress(&q, g_header)) != cudaSuccess) return e;
        p = reinterpret_cast<WsHeader*>(q);
        at[dev].store(p, std::memory_order_release);
    }
    *out = p;
    return cudaSuccess;
}

static bool byte_map(CUtensorMap* m, const void* ptr, long long rows, int cols, long long stride, uint32_t box_rows) {
    return tmap::encode_2d(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, ptr, (uint64_t)rows, (uint64_t)cols, (uint64_t)stride, BKB, box_rows,
                           CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int EPI>
static cudaError_t launch_pair(const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mC, const ProductArgs& a, int n_nt, int k_blocks,
                               long long tiles, cudaStream_t s) {
    static PerDevice configured;                 // per device: CTA pairs that run at once
    auto kernel = product_pair_kernel<EPI>;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM_BYTES;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int dev = 0, units = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    e = configured.get(dev, &units, [&](int d, int* n) {
        cudaError_t e2 = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
        int sms = 0, clusters = 0;
        if (e2 == cudaSuccess) e2 = device_sm_count(d, &sms);
        cfg.gridDim = dim3(sms / 2 * 2);
        if (e2 == cudaSuccess) e2 = cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg);
        if (e2 != cudaSuccess) return e2;
        if (clusters < 1) return cudaErrorInvalidConfiguration;
        *n = clusters < sms / 2 ? clusters : sms / 2;
        return cudaSuccess;
    });
    if (e != cudaSuccess) return e;
    cfg.gridDim = dim3((unsigned)(2 * (tiles < units ? tiles : units)));
    cfg.numAttrs = g_pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, mA, mB, mC, a, n_nt, k_blocks);
}

// Columns of a plain tile: those by which 74 pairs are done first.  A k-block of 128 bytes takes a pair two cycles per column on
// the tensor cores; all pairs together bring some 7500 bytes per cycle into their SMs.  (600 tokens, 8192 x 8192: 192 columns
// 52 us, 256 columns 58 us; 8192 tokens, 4096 x 7168: 256 columns.)
static int pair_columns(int M, int N) {
    int best = BN;
    double least = 0;
    for (int bn = BN; bn >= 128; bn -= 32) {
        const long long tiles = (long long)((M + 2 * BM - 1) / (2 * BM)) * ((N + bn - 1) / bn), waves = (tiles + 73) / 74;
        const double mma = (double)waves * 2 * bn, bytes = (double)tiles * 2 * (BM + bn / 2) * BKB / 7500;
        const double c = mma > bytes ? mma : bytes;
        if (bn == BN || c < least) {
            least = c;
            best = bn;
        }
    }
    return best;
}

cudaError_t launch_product(const ProductArgs& args, int epi, cudaStream_t s) {
    ProductArgs a = args;
    const bool gated = epi == EPI_GATED;
    a.bn = epi == EPI_PLAIN ? pair_columns(a.dense_rows, a.N) : BN;
    a.starve = g_starve;
    CUtensorMap mA, mB, mC;
    if (!byte_map(&mA, a.A, a.a_rows, a.K, a.lda, BM) ||
        !byte_map(&mB, a.B, (long long)a.E * (gated ? 2 : 1) * a.N, a.K, a.ldb, (uint32_t)a.bn / 2))
        return cudaErrorInvalidValue;
    // C in boxes of 32 rows of 64 bytes, where its rows allow it
    const int type = epi == EPI_PLAIN ? a.c_type : MOK_TYPE_F32;
    const uint64_t size = type_bytes(type);
    a.c_mapped = (reinterpret_cast<uintptr_t>(a.C) & 15u) == 0 && (a.ldc * size) % 16 == 0;
    if (!a.c_mapped) mC = mA;
    else if (!tmap::encode_2d(&mC, type == MOK_TYPE_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_UINT16, a.C,
                              (uint64_t)(a.dense_rows > 0 ? a.dense_rows : a.a_rows), (uint64_t)a.N, a.ldc * size,
                              (uint32_t)(64 / size), 32, CU_TENSOR_MAP_SWIZZLE_64B))
        return cudaErrorInvalidValue;
    const int n_nt = gated ? (a.N + BN / 2 - 1) / (BN / 2) : (a.N + a.bn - 1) / a.bn;
    const int k_blocks = (a.K + BKB - 1) / BKB;
    const long long tiles = (a.dense_rows > 0 ? (a.dense_rows + 2 * BM - 1) / (2 * BM) : a.max_mt) * (long long)n_nt;
    if (tiles <= 0 || tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    if (epi == EPI_PLAIN) return launch_pair<EPI_PLAIN>(mA, mB, mC, a, n_nt, k_blocks, tiles, s);
    if (gated) return launch_pair<EPI_GATED>(mA, mB, mC, a, n_nt, k_blocks, tiles, s);
    return launch_pair<EPI_ROWS>(mA, mB, mC, a, n_nt, k_blocks, tiles, s);
}

}  // namespace i8
}  // namespace mok
