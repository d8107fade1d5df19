// Products of 8-bit operands with few tokens (a decoding step): bound by reading the weights once, so the shape is chosen for
// memory, not for the tensor cores.
//
// The weights sit on the MMA's M side (128 output channels per tile, tcgen05.mma.kind::i8), the tokens on its N side (16, 32
// or 64 columns).  A cluster of S CTAs shares one channel tile and splits K: with a few dozen channel tiles a split is what
// puts the reading onto all SMs.  Per CTA
//   1. a TMA ring starts to stream the CTA's K range of the 128 weight rows
//   2. meanwhile all warps bring the tokens' K range into shared memory as the (swizzled) B operand, which stays resident:
//      codes are copied; activations are quantised right here -- every CTA takes the maxima of its range, the cluster
//      exchanges them -- which spares a launch and a round trip through memory
//   3. one thread issues the MMAs as the stages land
//   4. the 32-bit sums go from TMEM to shared memory; each CTA of the cluster adds up its share of the tokens over the
//      cluster (integer sums: exact in any order), scales and stores them
#include "i8_common.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.cuh"

namespace mok {
namespace i8 {

using namespace tc;

constexpr int NARROW_THREADS = 512, NARROW_WARPS = NARROW_THREADS / 32;
constexpr int NARROW_STAGE = 128 * 128;          // 128 channels x 128 bytes of K
constexpr int NARROW_MAX_STAGES = 10;
constexpr int NARROW_SMEM = 232448;
constexpr int NARROW_CTRL = 1024;                // barriers, row maxima

struct NarrowCtrl {
    uint64_t full[NARROW_MAX_STAGES], empty[NARROW_MAX_STAGES], tfull;
    uint32_t tmem_base, abort;
    uint32_t amax[64], top[64];                  // row maxima over this CTA's K range, and over the cluster's
    float scale[64];
};
static_assert(sizeof(NarrowCtrl) <= NARROW_CTRL, "control block too large");

__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}
__device__ __forceinline__ uint32_t ld_cluster(uint32_t addr, uint32_t rank) {
    uint32_t v;
    asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %1, %2;\n\tld.shared::cluster.u32 %0, [ra];\n\t}"
                 : "=r"(v) : "r"(addr), "r"(rank) : "memory");
    return v;
}
__device__ __forceinline__ constexpr uint32_t narrow_idesc(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
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

// Pieces of eight activations that a thread holds.  Few, and no path for unaligned rows: code that runs once is paid for by
// its instruction fetches (twelve pieces: 3000 instructions per warp, 15 us).
template <class T> struct Held { static constexpr int pieces = sizeof(T) == 2 ? 4 : 2; };

struct NarrowArgs {
    const void* x;               // activations of x_type, or NULL: codes and scales are given
    const int8_t* codes;
    const float* scales;
    long long ldx, ldc;          // elements of x, bytes of codes
    int32_t M, K, N;
    int32_t bn;                  // columns of the MMA: 16, 32 or 64
    int32_t stages;
    const float* w_scale;
    const float* bias;
    void* out;
    long long ldo;
    WsHeader* header;
};

// The tokens' K range k0 .. k1 as codes into `tok`.  A unit is 256 elements of a row, eight per lane; a warp has all its units
// (at most Held<T>::pieces) in registers at once, so that memory is waited for once and read once.
template <class T>
__device__ __forceinline__ void quantise_range(const NarrowArgs& a, int k0, int k1, uint8_t* tok, NarrowCtrl* ctrl, int warp, int lane,
                                               int S) {
    constexpr int HELD = Held<T>::pieces;
    const int per_row = (k1 - k0 + 255) >> 8, units = a.M * per_row;
    uint4 v[HELD][sizeof(T) / 2];
    int row[HELD], at[HELD];                     // at: first element, relative to k0; the range's end for none
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int u = warp + i * NARROW_WARPS;
        row[i] = u / per_row;
        at[i] = u < units ? (u - row[i] * per_row) * 256 + lane * 8 : k1 - k0;
        const T* src = reinterpret_cast<const T*>(a.x) + row[i] * a.ldx + k0 + at[i];
#pragma unroll
        for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
            v[i][q] = make_uint4(0u, 0u, 0u, 0u);
            if (at[i] < k1 - k0 && k0 + at[i] < a.K) v[i][q] = __ldg(reinterpret_cast<const uint4*>(src) + q);   // (K: whole pieces)
        }
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if (warp + i * NARROW_WARPS >= units) break;
        const T* e = reinterpret_cast<const T*>(v[i]);
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, abs_bits(to_f(e[j])));
        m = __reduce_max_sync(0xffffffffu, m);
        if (lane == 0) atomicMax(&ctrl->amax[row[i]], m);
    }
    __syncthreads();
    if (S > 1) {
        cluster_sync();                          // every CTA's maxima are complete
        uint32_t m = 0;
        if ((int)threadIdx.x < a.M)
            for (int q = 0; q < S; ++q) m = max(m, ld_cluster(smem_u32(&ctrl->amax[threadIdx.x]), (uint32_t)q));
        if ((int)threadIdx.x < a.M) ctrl->top[threadIdx.x] = m;
    } else if ((int)threadIdx.x < a.M) {
        ctrl->top[threadIdx.x] = ctrl->amax[threadIdx.x];
    }
    __syncthreads();
    if ((int)threadIdx.x < a.M) ctrl->scale[threadIdx.x] = __uint_as_float(ctrl->top[threadIdx.x]) / 127.f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        if (at[i] >= k1 - k0) continue;
        const uint32_t m = ctrl->top[row[i]];
        uint2 o = make_uint2(0u, 0u);
        if (m > 0 && finite_bits(m)) {
            const RowRule rule = row_rule(__uint_as_float(m));
            const T* e = reinterpret_cast<const T*>(v[i]);
            o.x = four_codes<true>(to_f(e[0]), to_f(e[1]), to_f(e[2]), to_f(e[3]), rule);
            o.y = four_codes<true>(to_f(e[4]), to_f(e[5]), to_f(e[6]), to_f(e[7]), rule);
        }
        const int b = at[i] >> 7, c = at[i] & 127;
        *reinterpret_cast<uint2*>(tok + (size_t)(b * a.bn + row[i]) * 128 + (((c >> 4) ^ (row[i] & 7)) << 4) + (c & 8)) = o;
    }
}

// X: the activations' type, int8_t for codes
template <class X, class O>
__global__ void __launch_bounds__(NARROW_THREADS, 1)
product_narrow_kernel(const __grid_constant__ CUtensorMap tmapW, const __grid_constant__ NarrowArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = (int)cluster_size(), rank = (int)cluster_ctarank();
    const int tile = blockIdx.x / S;
    const int kb_all = (a.K + 127) / 128;
    const int kb0 = (int)((long long)kb_all * rank / S), kb1 = (int)((long long)kb_all * (rank + 1) / S), n_kb = kb1 - kb0;
    const int k0 = kb0 * 128, k1 = kb1 * 128;
    // ring of weight stages | tokens [n_kb][bn][128 bytes] | control block; the sums reuse the ring
    uint8_t* tok = smem + a.stages * NARROW_STAGE;
    const int most_kb = (kb_all + S - 1) / S;
    NarrowCtrl* ctrl = reinterpret_cast<NarrowCtrl*>(tok + (size_t)most_kb * a.bn * 128);
    volatile uint32_t* abort_flag = &ctrl->abort;

    if (threadIdx.x == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(smem_u32(&ctrl->full[s]), 1);
            mbar_init(smem_u32(&ctrl->empty[s]), 1);
        }
        mbar_init(smem_u32(&ctrl->tfull), 1);
        ctrl->abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (threadIdx.x < 64) ctrl->amax[threadIdx.x] = 0u;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&ctrl->tmem_base)), "r"(64u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctrl->tmem_base;
    pdl_enter();

    // the first stages of the weights are on their way before the tokens are looked at
    const int ahead = n_kb < a.stages ? n_kb : a.stages;
    if (threadIdx.x == 0) {
        for (int s = 0; s < ahead; ++s) {
            mbar_expect_tx(smem_u32(&ctrl->full[s]), NARROW_STAGE);
            tma_load_2d(base + s * NARROW_STAGE, &tmapW, smem_u32(&ctrl->full[s]), (kb0 + s) * 128, tile * 128);
        }
    }
    __syncwarp();
    if constexpr (sizeof(X) > 1) {
        quantise_range<X>(a, k0, k1, tok, ctrl, warp, lane, S);
    } else {
        // codes, in 16-byte pieces; zeros past K
        const int pieces = n_kb * 8;
        for (int i = threadIdx.x; i < a.M * pieces; i += NARROW_THREADS) {
            const int r = i / pieces, c = i - r * pieces;
            const uint32_t dst = smem_u32(tok) + ((c >> 3) * a.bn + r) * 128 + (((c & 7) ^ (r & 7)) << 4);
            const int left = a.K - (k0 + c * 16);
            cp_async_16(dst, left > 0 ? a.codes + r * a.ldc + k0 + c * 16 : a.codes, left >= 16 ? 16u : left > 0 ? (uint32_t)left : 0u);
        }
        if ((int)threadIdx.x < a.M) ctrl->scale[threadIdx.x] = __ldg(a.scales + threadIdx.x);
        asm volatile("cp.async.wait_all;" ::: "memory");
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the MMAs read what was just written
    __syncthreads();

    if (warp == 0) {
        if (lane == 0) {                                              // the rest of the weights
            int s = 0;
            uint32_t ph = 0;
            for (int kb = ahead; kb < n_kb; ++kb) {
                if (!mbar_wait(smem_u32(&ctrl->empty[s]), ph, abort_flag, a.header, 21)) break;
                mbar_expect_tx(smem_u32(&ctrl->full[s]), NARROW_STAGE);
                tma_load_2d(base + s * NARROW_STAGE, &tmapW, smem_u32(&ctrl->full[s]), (kb0 + kb) * 128, tile * 128);
                if (++s == a.stages) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = narrow_idesc(a.bn);
            int s = 0;
            uint32_t ph = 0;
            for (int kb = 0; kb < n_kb; ++kb) {
                if (!mbar_wait(smem_u32(&ctrl->full[s]), ph, abort_flag, a.header, 22)) break;
                tc_fence_after();
                const uint64_t adesc = make_smem_desc(base + s * NARROW_STAGE);
                const uint64_t bdesc = make_smem_desc(smem_u32(tok) + kb * a.bn * 128);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    mma_one(tmem, adesc + (uint64_t)(j * 2), bdesc + (uint64_t)(j * 2), idesc, (kb | j) ? 1u : 0u);
                tc_commit<1>(smem_u32(&ctrl->empty[s]));
                if (++s == a.stages) { s = 0; ph ^= 1u; }
            }
            tc_commit<1>(smem_u32(&ctrl->tfull));
        }
        __syncwarp();
    }
    // ---- sums: TMEM lane = channel, column = token -> shared memory [token][128 channels]
    bool ok = mbar_wait(smem_u32(&ctrl->tfull), 0u, abort_flag, a.header, 23);
    tc_fence_after();
    int32_t* sums = reinterpret_cast<int32_t*>(smem);
    ok = __all_sync(0xffffffffu, ok);
    if (ok && n_kb > 0) {
        const int c = (warp >> 2) * 16;          // four warps per 16 tokens
        if (c < a.M) {
            uint32_t r[16];
            tc_ld16(tmem + (uint32_t)c + ((uint32_t)((warp & 3) * 32) << 16), r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < a.M) sums[(c + i) * 128 + (warp & 3) * 32 + lane] = (int32_t)r[i];
        }
    } else {
        for (int i = threadIdx.x; i < a.M * 128; i += NARROW_THREADS) sums[i] = 0;       // an empty K range
    }
    tc_fence_before();
    __syncthreads();
    if (S > 1) cluster_sync();
    {
        const int ch = threadIdx.x & 127, n = tile * 128 + ch;
        if (n < a.N) {
            const float ws = __ldg(a.w_scale + n), b = a.bias ? __ldg(a.bias + n) : 0.f;
            for (int t = rank + S * (threadIdx.x >> 7); t < a.M; t += NARROW_THREADS / 128 * S) {
                int32_t sum = 0;
                if (S == 1) sum = sums[t * 128 + ch];
                else
                    for (int q = 0; q < S; ++q) sum += (int32_t)ld_cluster(base + (uint32_t)(t * 128 + ch) * 4, (uint32_t)q);
                const float v = (float)sum * ctrl->scale[t] * ws + b;
                reinterpret_cast<O*>(a.out)[(long long)t * a.ldo + n] = from_f<O>(v);
            }
        }
    }
    if (*abort_flag) {   // failure path only: give copies and MMAs already in flight time to land before leaving
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 200000ull) { }
    }
    __syncthreads();
    if (S > 1) cluster_sync();                   // the peers have read this CTA's sums
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(64u) : "memory");
    }
}

template <class X, class O>
static cudaError_t launch_narrow_typed(const CUtensorMap& mW, const NarrowArgs& a, int S, int tiles, size_t smem, cudaStream_t s) {
    static PerDevice configured;
    auto kernel = product_narrow_kernel<X, O>;
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    e = configured.get(dev, &sms, [&](int d, int* n) {
        cudaError_t e2 = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NARROW_SMEM);
        return e2 == cudaSuccess ? device_sm_count(d, n) : e2;
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)S;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)(tiles * S));
    cfg.blockDim = dim3(NARROW_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, mW, a);
}

// Split of K: the S of 1 .. 8 with the least k-blocks one after the other, if every CTA had an SM; false if the tokens' K
// range does not fit beside four stages of weights.
static bool narrow_shape(int M, int K, int N, int* bn, int* split, int* stages, size_t* smem) {
    if (M > 64) return false;
    *bn = M <= 16 ? 16 : M <= 32 ? 32 : 64;
    const int kb = (K + 127) / 128, tiles = (N + 127) / 128;
    int best = 0;
    long long cost = 0;
    for (int S = 1; S <= 8 && S <= kb; ++S) {
        const int most = (kb + S - 1) / S;
        const long long room = NARROW_SMEM - NARROW_CTRL - (long long)most * *bn * 128;
        if (room < 4 * NARROW_STAGE) continue;
        const long long c = ((long long)tiles * S + 147) / 148 * most * 8 + S;        // (a larger cluster exchanges more)
        if (!best || c < cost) {
            best = S;
            cost = c;
            const int n = (int)(room / NARROW_STAGE), least = (*bn * 128 * 4 + NARROW_STAGE - 1) / NARROW_STAGE;
            *stages = n < NARROW_MAX_STAGES ? n : NARROW_MAX_STAGES;
            if (*stages > most) *stages = most > least ? most : least;                // (the sums need room too)
            *smem = (size_t)*stages * NARROW_STAGE + (size_t)most * *bn * 128 + NARROW_CTRL;
        }
    }
    *split = best;
    return best > 0;
}

// Whether the narrow kernel takes a product, and whether it quantises the activations itself: as far as the registers hold a
// CTA's share, from whole 16-byte pieces (x_align: the bits that x's address and row pitch have set).
bool narrow_product(int M, int K, int N, int x_type, unsigned long long x_align, bool* quantises) {
    int bn, S, stages;
    size_t smem;
    if (!narrow_shape(M, K, N, &bn, &S, &stages, &smem)) return false;
    const int most = ((K + 127) / 128 + S - 1) / S;
    *quantises = K % 8 == 0 && (x_align & 15u) == 0 &&
                 M * ((most + 1) / 2) <= NARROW_WARPS * (x_type == MOK_TYPE_F32 ? Held<float>::pieces : Held<__half>::pieces);
    return true;
}

template <class X>
static cudaError_t launch_narrow_out(const CUtensorMap& mW, const NarrowArgs& a, int c_type, int S, int tiles, size_t smem,
                                     cudaStream_t s) {
    if (c_type == MOK_TYPE_F32) return launch_narrow_typed<X, float>(mW, a, S, tiles, smem, s);
    if (c_type == MOK_TYPE_F16) return launch_narrow_typed<X, __half>(mW, a, S, tiles, smem, s);
    return launch_narrow_typed<X, __nv_bfloat16>(mW, a, S, tiles, smem, s);
}

cudaError_t launch_narrow(const ProductArgs& g, const void* x, int x_type, long long ldx, cudaStream_t s) {
    NarrowArgs a = {};
    int S = 1;
    size_t smem = 0;
    if (!narrow_shape(g.dense_rows, g.K, g.N, &a.bn, &S, &a.stages, &smem)) return cudaErrorInvalidValue;
    a.x = x;
    a.ldx = ldx;
    a.codes = g.A;
    a.ldc = g.lda;
    a.scales = g.a_scale;
    a.M = g.dense_rows; a.K = g.K; a.N = g.N;
    a.w_scale = g.b_scale;
    a.bias = g.bias;
    a.out = g.C;
    a.ldo = g.ldc;
    a.header = g.header;
    CUtensorMap mW;
    if (!tmap::encode_2d(&mW, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.B, (uint64_t)g.N, (uint64_t)g.K, (uint64_t)g.ldb, 128, 128,
                         CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    const int tiles = (g.N + 127) / 128;
    if (!x) return launch_narrow_out<int8_t>(mW, a, g.c_type, S, tiles, smem, s);
    if (x_type == MOK_TYPE_F32) return launch_narrow_out<float>(mW, a, g.c_type, S, tiles, smem, s);
    if (x_type == MOK_TYPE_F16) return launch_narrow_out<__half>(mW, a, g.c_type, S, tiles, smem, s);
    return launch_narrow_out<__nv_bfloat16>(mW, a, g.c_type, S, tiles, smem, s);
}

}  // namespace i8
}  // namespace mok
