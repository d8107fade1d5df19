// Products of 8-bit integer operands on the tensor cores (tcgen05.mma.kind::i8, K = 32 per instruction, exact 32-bit integer
// sums in TMEM), scaled in fp32 as they leave: out[r, n] = a_scale[r] * b_scale[n] * sum_k A[r, k] B[n, k].
//
// Persistent, warp-specialised, on CTA pairs: the two CTAs of a cluster compute one 256 x 256 tile with cta_group::2 MMAs
// issued by the even CTA.  Each CTA stages its own 128 rows of A and half of the 256 rows of B (128 bytes of K per stage, 32 KB,
// six stages), so an SM pulls 32 KB for 256 cycles of MMA; a 128 x 256 tile of one CTA would pull 48 KB for them, and one-byte
// operands are bound by that rate.
//   warp 0       TMA producer : A and B tiles (128-byte swizzle)
//   warp 1       MMA issuer (even CTA)
//   warps 2..9   epilogue     : warp w drains TMEM lane quadrant w % 4 and one half of the tile's columns
// Two 256-column accumulators: a tile's epilogue runs beside the next tile's products.
//
//   EPI_PLAIN : C = scaled sums (+ bias) as bf16, fp16 or fp32, one rounding
//   EPI_GATED : B tile = 128 gate rows (even CTA) + the matching 128 up rows (odd CTA); h = silu(g) u in fp32 -> C fp32.  h is
//               quantised by a pass of its own, since its row maximum spans all N tiles; fp32 because a rounding before the
//               quantisation moves codes (bf16 moves one code in twenty).
//   EPI_HALF  : C = fp16(sum * y_unit * b_scale[n] / b_max): the sums in the unit of the row, at most 65504 by construction
//               (|sum| <= 127 * 127 * K, y_unit a power of two), so that the combine can read two bytes per value with
//               eleven significant bits and put the row's factor a_scale * b_max / y_unit on in fp32.
// K, N and the rows may be ragged: TMA fills bytes past K and rows past the tensor with zeros, stores are masked.
// All mbarrier waits are bounded; on a timeout the CTA records MOK_ERR_TIMEOUT and leaves cleanly.
#include "i8_common.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.cuh"

namespace mok {
namespace i8 {

using namespace tc;

constexpr int BM = 128, BN = 256, BKB = 128;
constexpr int A_BYTES = BM * BKB, B_BYTES = BN / 2 * BKB, STAGE_BYTES = A_BYTES + B_BYTES;
constexpr int STAGES = 6;
constexpr int EPI_WARPS = 8;
constexpr int SLAB_BYTES = 4096;                 // per epilogue warp: 32 rows x 32 columns of up to four bytes
constexpr int SLAB_REGION = STAGES * STAGE_BYTES;
constexpr int CTRL_REGION = SLAB_REGION + EPI_WARPS * SLAB_BYTES;
constexpr int SMEM_BYTES = CTRL_REGION + 256 + 1024;
constexpr int TMEM_COLS = 512;
constexpr int THREADS = 64 + 32 * EPI_WARPS;     // + one gather warp
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

struct PairTile { int row0, n, e, valid; };     // valid: rows of the segment from row0 on

__device__ __forceinline__ PairTile pair_tile(const ProductArgs& a, int L, int n_nt, int n_mt) {
    PairTile t;
    int mt0 = 0, m_cnt = n_mt, pad0 = 0, rows = a.dense_rows;
    t.e = 0;
    if (a.dense_rows <= 0) {
        t.e = __ldg(a.tile_expert + L / n_nt);
        mt0 = __ldg(a.mt_start + t.e);
        m_cnt = __ldg(a.mt_start + t.e + 1) - mt0;
        pad0 = __ldg(a.pad_offsets + t.e);
        rows = __ldg(a.counts + t.e);
    }
    // row tiles in groups of GROUP_ROWS rows, fastest inside a group: its rows stay in L2 while the weight tiles stream
    constexpr int group_m = GROUP_ROWS / (2 * BM);
    const int r = L - n_nt * mt0;
    const int g = r / (group_m * n_nt);
    const int rem = r - g * group_m * n_nt;
    const int in_group = min(group_m, m_cnt - g * group_m);
    t.n = rem / in_group;
    const int m = g * group_m + (rem - t.n * in_group);
    t.row0 = pad0 + m * 2 * BM;
    t.valid = rows - m * 2 * BM;
    return t;
}

template <class T> struct Pack;
template <> struct Pack<__nv_bfloat16> {
    static __device__ __forceinline__ uint32_t two(float a, float b) { return pack_bf16(a, b); }
};
template <> struct Pack<__half> {
    static __device__ __forceinline__ uint32_t two(float a, float b) {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// Writes a warp's 32 rows x 32 columns (lane = row, v = its columns) to C through the warp's slab, so that a store
// instruction covers whole row segments.  n_rows, n_cols: how many of them exist.
template <class T>
__device__ __forceinline__ void store_block(const float (&v)[32], uint32_t slab, T* c, long long ldc, int n_rows, int n_cols,
                                            bool vec, int lane) {
    constexpr int PER = 16 / sizeof(T), SEGS = 32 / PER;             // elements of a 16-byte piece, pieces of a row
    __syncwarp();
#pragma unroll
    for (int i = 0; i < SEGS; ++i) {
        const uint32_t at = slab + lane * (32 * sizeof(T)) + ((sizeof(T) == 4 ? (i ^ (lane & 7)) : (i ^ ((lane >> 1) & 3))) << 4);
        if constexpr (sizeof(T) == 4)
            st_shared_v4(at, __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        else
            st_shared_v4(at, Pack<T>::two(v[8 * i], v[8 * i + 1]), Pack<T>::two(v[8 * i + 2], v[8 * i + 3]),
                         Pack<T>::two(v[8 * i + 4], v[8 * i + 5]), Pack<T>::two(v[8 * i + 6], v[8 * i + 7]));
    }
    __syncwarp();
    const int seg = lane % SEGS;
#pragma unroll
    for (int it = 0; it < SEGS; ++it) {
        const int r = it * (32 / SEGS) + lane / SEGS;
        uint4 val;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(val.x), "=r"(val.y), "=r"(val.z), "=r"(val.w)
                     : "r"(slab + r * (uint32_t)(32 * sizeof(T)) + ((sizeof(T) == 4 ? (seg ^ (r & 7)) : (seg ^ ((r >> 1) & 3))) << 4)));
        if (r >= n_rows) continue;
        T* dst = c + (long long)r * ldc + seg * PER;
        if (vec && (seg + 1) * PER <= n_cols) {
            *reinterpret_cast<uint4*>(dst) = val;
        } else {
            const T* e = reinterpret_cast<const T*>(&val);
#pragma unroll
            for (int j = 0; j < PER; ++j)
                if (seg * PER + j < n_cols) dst[j] = e[j];
        }
    }
}

// silu(g) u.  The exponential and the quotient are good to about 2^-21: what follows is a rounding to 8-bit codes, which an
// 11-bit tanh would move in one case of fifty.
__device__ __forceinline__ float gated(float g, float u) { return __fdividef(g, 1.f + __expf(-g)) * u; }

template <int EPI>
__global__ void __launch_bounds__(THREADS, 1)
product_pair_kernel(const __grid_constant__ CUtensorMap tmapA, const __grid_constant__ CUtensorMap tmapB,
                    const __grid_constant__ ProductArgs a, const int n_nt, const int k_blocks) {
    constexpr bool GATED = EPI == EPI_GATED;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base - raw);
    Ctrl* ctrl = reinterpret_cast<Ctrl*>(smem + CTRL_REGION);
    volatile uint32_t* abort_flag = &ctrl->abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_ctarank();
    const int unit = blockIdx.x >> 1, n_units = gridDim.x >> 1;

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
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            for (int L = unit; L < total; L += n_units) {
                const PairTile t = pair_tile(a, L, n_nt, n_mt);
                const int brow = GATED ? t.e * 2 * a.N + rank * a.N + t.n * (BN / 2) : t.e * a.N + t.n * BN + rank * (BN / 2);
                bool ok = true;
                for (int kb = 0; kb < k_blocks; ++kb) {
                    ok = mbar_wait(smem_u32(&ctrl->empty[s]), ph ^ 1u, abort_flag, a.header, 1);
                    if (!ok) break;
                    const uint32_t full = smem_u32(&ctrl->full[s]);
                    const uint32_t sa = base + s * STAGE_BYTES, sb = sa + A_BYTES;
                    // the even CTA's barrier collects the bytes of both CTAs of the pair
                    if (rank == 0) mbar_expect_tx(full, 2 * STAGE_BYTES);
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
            constexpr uint32_t idesc = make_idesc(2 * BM, BN);
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
        const uint32_t slab = base + SLAB_REGION + (warp - 2) * SLAB_BYTES;
        const size_t c_bytes = EPI == EPI_HALF ? 2 : (GATED || a.c_type == MOK_TYPE_F32) ? 4 : 2;
        const bool vec = (reinterpret_cast<uintptr_t>(a.C) & 15u) == 0 && ((a.ldc * c_bytes) & 15u) == 0;
        int buf = 0;
        uint32_t aph = 0;
        for (int L = unit; L < total; L += n_units) {
            const PairTile t = pair_tile(a, L, n_nt, n_mt);
            const int r0 = rank * BM + quad * 32;                    // first of the warp's rows inside the tile
            const int n_rows = min(32, t.valid - r0);
            float rs = 0.f;
            if (EPI != EPI_HALF && lane < n_rows) rs = __ldg(a.a_scale + t.row0 + r0 + lane);
            // the warp's column scales, one column of each piece per lane, on their way while the products finish
            constexpr int CHUNKS = GATED ? 2 : 4;                    // 32-column pieces of this warp
            const int first = t.n * (GATED ? BN / 2 : BN) + half * 32 * CHUNKS;
            const float* bs = a.b_scale + (size_t)t.e * (GATED ? 2 : 1) * a.N;
            float unit_n = 1.f;
            if constexpr (EPI == EPI_HALF) {
                const float top = __ldg(a.b_max + t.e);
                unit_n = top > 0.f ? a.y_unit / top : 0.f;
            }
            float s0[CHUNKS], s1[CHUNKS];                            // s1: up scales, or the bias
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                const int n = first + c * 32 + lane;
                s0[c] = n < a.N ? __ldg(bs + n) : 0.f;
                s1[c] = 0.f;
                if (GATED && n < a.N) s1[c] = __ldg(bs + a.N + n);
                if (EPI == EPI_PLAIN && a.bias && n < a.N) s1[c] = __ldg(a.bias + n);
                if (EPI == EPI_HALF) s0[c] *= unit_n;
            }
            bool ok = mbar_wait(smem_u32(&ctrl->tfull[buf]), aph, abort_flag, a.header, 4);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            tc_fence_after();
            const uint32_t taddr = tmem_base + (uint32_t)(buf * BN) + ((uint32_t)(quad * 32) << 16);
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c) {
                uint32_t acc[32], up[GATED ? 32 : 1];
                const int col = half * 32 * CHUNKS + c * 32;
                tc_ld32(taddr + col, acc);
                if constexpr (GATED) tc_ld32(taddr + BN / 2 + col, up);
                __syncwarp();                                        // the slab's previous block has been read
                st_shared_f32(slab + lane * 4, s0[c]);
                st_shared_f32(slab + 128 + lane * 4, s1[c]);
                __syncwarp();
                tc_wait_ld();
                if (c == CHUNKS - 1) {                               // the accumulator goes back before the last arithmetic
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_remote(smem_u32(&ctrl->tempty[buf]), 0);
                }
                const int n0 = first + c * 32, n_cols = a.N - n0;    // first output column of the piece, and how many exist
                if (n_rows <= 0 || n_cols <= 0) continue;
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const float4 f = ld_shared_f4(slab + i * 4);
                    if constexpr (EPI == EPI_HALF) {
                        v[i] = (float)(int)acc[i] * f.x;
                        v[i + 1] = (float)(int)acc[i + 1] * f.y;
                        v[i + 2] = (float)(int)acc[i + 2] * f.z;
                        v[i + 3] = (float)(int)acc[i + 3] * f.w;
                    } else {
                        const float4 q = ld_shared_f4(slab + 128 + i * 4);
                        v[i] = (float)(int)acc[i] * rs * f.x;
                        v[i + 1] = (float)(int)acc[i + 1] * rs * f.y;
                        v[i + 2] = (float)(int)acc[i + 2] * rs * f.z;
                        v[i + 3] = (float)(int)acc[i + 3] * rs * f.w;
                        if constexpr (GATED) {
                            v[i] = gated(v[i], (float)(int)up[i] * rs * q.x);
                            v[i + 1] = gated(v[i + 1], (float)(int)up[i + 1] * rs * q.y);
                            v[i + 2] = gated(v[i + 2], (float)(int)up[i + 2] * rs * q.z);
                            v[i + 3] = gated(v[i + 3], (float)(int)up[i + 3] * rs * q.w);
                        } else {
                            v[i] += q.x;
                            v[i + 1] += q.y;
                            v[i + 2] += q.z;
                            v[i + 3] += q.w;
                        }
                    }
                }
                const long long at = (long long)(t.row0 + r0) * a.ldc + n0;
                if constexpr (GATED) {
                    store_block(v, slab, reinterpret_cast<float*>(a.C) + at, a.ldc, n_rows, n_cols, vec, lane);
                } else if constexpr (EPI == EPI_HALF) {
                    store_block(v, slab, reinterpret_cast<__half*>(a.C) + at, a.ldc, n_rows, n_cols, vec, lane);
                } else {
                    if (a.c_type == MOK_TYPE_F32) store_block(v, slab, reinterpret_cast<float*>(a.C) + at, a.ldc, n_rows, n_cols, vec, lane);
                    else if (a.c_type == MOK_TYPE_F16) store_block(v, slab, reinterpret_cast<__half*>(a.C) + at, a.ldc, n_rows, n_cols, vec, lane);
                    else store_block(v, slab, reinterpret_cast<__nv_bfloat16*>(a.C) + at, a.ldc, n_rows, n_cols, vec, lane);
                }
            }
            if (++buf == 2) { buf = 0; aph ^= 1u; }
        }
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
static cudaError_t launch_pair(const CUtensorMap& mA, const CUtensorMap& mB, const ProductArgs& a, int n_nt, int k_blocks,
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
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, mA, mB, a, n_nt, k_blocks);
}

cudaError_t launch_product(const ProductArgs& a, int epi, cudaStream_t s) {
    const bool gated = epi == EPI_GATED;
    CUtensorMap mA, mB;
    if (!byte_map(&mA, a.A, a.a_rows, a.K, a.lda, BM) ||
        !byte_map(&mB, a.B, (long long)a.E * (gated ? 2 : 1) * a.N, a.K, a.ldb, BN / 2))
        return cudaErrorInvalidValue;
    const int n_nt = gated ? (a.N + BN / 2 - 1) / (BN / 2) : (a.N + BN - 1) / BN;
    const int k_blocks = (a.K + BKB - 1) / BKB;
    const long long tiles = (a.dense_rows > 0 ? (a.dense_rows + 2 * BM - 1) / (2 * BM) : a.max_mt) * (long long)n_nt;
    if (tiles <= 0 || tiles > 0x7fffffffll) return cudaErrorInvalidValue;
    if (epi == EPI_PLAIN) return launch_pair<EPI_PLAIN>(mA, mB, a, n_nt, k_blocks, tiles, s);
    if (gated) return launch_pair<EPI_GATED>(mA, mB, a, n_nt, k_blocks, tiles, s);
    return launch_pair<EPI_HALF>(mA, mB, a, n_nt, k_blocks, tiles, s);
}

}  // namespace i8
}  // namespace mok
