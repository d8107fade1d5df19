// Products of 8-bit operands with few tokens (a decoding step): bound by reading the weights once, so the shape is chosen for
// memory, not for the tensor cores.
//
// The weights sit on the MMA's M side (128 output channels per tile, tcgen05.mma.kind::i8), the tokens on its N side (16 to
// 256 columns).  A cluster of S CTAs shares one channel tile and splits K: with a few dozen channel tiles a split is what
// puts the reading onto all SMs.  Per CTA
//   1. a TMA ring streams the CTA's K range of the 128 weight rows and of the tokens' codes
//   2. or, a few rows of activations are quantised right here, into a (128-byte swizzled) B operand that stays: every CTA
//      takes the maxima of its range, the cluster exchanges them, which spares a launch and a round trip through memory
//   3. one thread issues the MMAs as the stages land
//   4. the 32-bit sums go from TMEM to shared memory; each CTA of the cluster adds up its share of the tokens over the
//      cluster (integer sums: exact in any order), scales and stores them
#include "i8_common.cuh"
#include "i8_ptx.cuh"
#include "tensor_map.cuh"

namespace mok {
namespace i8 {

using namespace tc;

constexpr int NARROW_THREADS = 512, NARROW_WARPS = NARROW_THREADS / 32;
constexpr int NARROW_STAGE = 128 * 128;          // 128 channels x 128 bytes of K
constexpr int NARROW_MAX_STAGES = 12;
constexpr int NARROW_SMEM = 232448;
constexpr int NARROW_CTRL = 2048;                // barriers, row maxima and scales
constexpr int NARROW_TOKENS = 256;               // most columns of the MMA
constexpr int NARROW_HELD = 64;                  // most rows that are quantised in the kernel

struct NarrowCtrl {
    uint64_t full[NARROW_MAX_STAGES], empty[NARROW_MAX_STAGES], tfull;
    uint32_t tmem_base, abort;
    uint32_t amax[NARROW_HELD], top[NARROW_HELD];    // row maxima over this CTA's K range, and over the cluster's
    float scale[NARROW_TOKENS];
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
__device__ __forceinline__ int4 ld_cluster4(uint32_t addr, uint32_t rank) {
    int4 v;
    asm volatile("{\n\t.reg .b32 ra;\n\tmapa.shared::cluster.u32 ra, %4, %5;\n\tld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [ra];\n\t}"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr), "r"(rank) : "memory");
    return v;
}
__device__ __forceinline__ constexpr uint32_t narrow_idesc(int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}
// Pieces of eight activations that a thread holds.  Few, and no path for unaligned rows: code that runs once is paid for by
// its instruction fetches (twelve pieces: 3000 instructions per warp, 15 us).
template <class T> struct Held { static constexpr int pieces = sizeof(T) == 2 ? 4 : 2; };

struct NarrowArgs {
    const void* x;               // activations, or NULL: codes and scales are given
    const float* scales;
    long long ldx;
    int32_t M, K, N;
    int32_t bn;                  // columns of the MMA: 16, 32, 64, 128 or 256
    int32_t stages;
    int32_t starve;              // (see ProductArgs)
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
        // eight threads per row, one for each CTA of the cluster: the reads go out together
        static_assert(NARROW_THREADS == 8 * NARROW_HELD, "a thread for each row and CTA");
        const int r = threadIdx.x >> 3, q = threadIdx.x & 7;
        uint32_t m = 0;
        if (r < a.M && q < S) m = ld_cluster(smem_u32(&ctrl->amax[r]), (uint32_t)q);
#pragma unroll
        for (int off = 1; off < 8; off <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, off));
        if (r < a.M && q == 0) ctrl->top[r] = m;
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
product_narrow_kernel(const __grid_constant__ CUtensorMap tmapW, const __grid_constant__ CUtensorMap tmapX,
                      const __grid_constant__ NarrowArgs a) {
    constexpr bool CODES = sizeof(X) == 1;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = (int)cluster_size(), rank = (int)cluster_ctarank();
    const int tiles_n = (a.N + 127) / 128, unit = blockIdx.x / S, tile = unit % tiles_n;     // channel tile ...
    const int t0 = unit / tiles_n * a.bn, M = min(a.bn, a.M - t0);                            // ... and tokens of this cluster
    const int kb_all = (a.K + 127) / 128;
    const int kb0 = (int)((long long)kb_all * rank / S), kb1 = (int)((long long)kb_all * (rank + 1) / S), n_kb = kb1 - kb0;
    const int k0 = kb0 * 128, k1 = kb1 * 128;
    // ring of stages (weights, codes) | quantised tokens [n_kb][bn][128 bytes] | control block; the sums reuse the ring
    const uint32_t tok_bytes = (uint32_t)a.bn * 128, stage_bytes = NARROW_STAGE + (CODES ? tok_bytes : 0u);
    uint8_t* tok = smem + a.stages * stage_bytes;
    const int most_kb = CODES ? 0 : (kb_all + S - 1) / S;
    const uint32_t tmem_cols = a.bn <= 64 ? 64u : (uint32_t)a.bn;
    NarrowCtrl* ctrl = reinterpret_cast<NarrowCtrl*>(tok + (size_t)most_kb * tok_bytes);
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
    if (threadIdx.x < NARROW_HELD) ctrl->amax[threadIdx.x] = 0u;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     ::"r"(smem_u32(&ctrl->tmem_base)), "r"(tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctrl->tmem_base;
    pdl_enter();

    // the first stages of the weights are on their way before the tokens are looked at
    const int ahead = n_kb < a.stages ? n_kb : a.stages;
    auto load = [&](int s, int kb) {
        if (a.starve) return;
        const uint32_t full = smem_u32(&ctrl->full[s]);
        mbar_expect_tx(full, stage_bytes);
        tma_load_2d(base + s * stage_bytes, &tmapW, full, (kb0 + kb) * 128, tile * 128);
        if (CODES) tma_load_2d(base + s * stage_bytes + NARROW_STAGE, &tmapX, full, (kb0 + kb) * 128, t0);
    };
    if (threadIdx.x == 0)
        for (int s = 0; s < ahead; ++s) load(s, s);
    __syncwarp();
    if constexpr (CODES) {
        if ((int)threadIdx.x < M) ctrl->scale[threadIdx.x] = __ldg(a.scales + t0 + threadIdx.x);
    } else {
        quantise_range<X>(a, k0, k1, tok, ctrl, warp, lane, S);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // the MMAs read what was just written
    __syncthreads();

    if (warp == 0) {
        if (lane == 0) {                                              // the rest of the weights
            int s = 0;
            uint32_t ph = 0;
            for (int kb = ahead; kb < n_kb; ++kb) {
                if (!mbar_wait(smem_u32(&ctrl->empty[s]), ph, abort_flag, a.header, 21)) break;
                load(s, kb);
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
                const uint64_t adesc = make_smem_desc(base + s * stage_bytes);
                const uint64_t bdesc = make_smem_desc(CODES ? base + s * stage_bytes + NARROW_STAGE : smem_u32(tok) + kb * tok_bytes);
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
        for (int c = (warp >> 2) * 16; c < M; c += NARROW_WARPS * 4) {     // four warps per 16 tokens
            uint32_t r[16];
            tc_ld16(tmem + (uint32_t)c + ((uint32_t)((warp & 3) * 32) << 16), r);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (c + i < M) sums[(c + i) * 128 + (warp & 3) * 32 + lane] = (int32_t)r[i];
        }
    } else {
        for (int i = threadIdx.x; i < M * 128; i += NARROW_THREADS) sums[i] = 0;       // an empty K range
    }
    tc_fence_before();
    __syncthreads();
    if (S > 1) cluster_sync();
    {
        // a warp takes a token, a lane four channels
        const int ch = lane * 4, n = tile * 128 + ch;
        float ws[4], bs[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ws[j] = n + j < a.N ? __ldg(a.w_scale + n + j) : 0.f;
            bs[j] = a.bias && n + j < a.N ? __ldg(a.bias + n + j) : 0.f;
        }
        const bool vec = n + 4 <= a.N && ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ldo * sizeof(O))) & (4 * sizeof(O) - 1)) == 0;
        for (int t = rank + S * warp; t < M; t += NARROW_WARPS * S) {
            int4 sum = make_int4(0, 0, 0, 0);
            if (S == 1) {
                sum = *reinterpret_cast<const int4*>(sums + t * 128 + ch);
            } else {
                for (int q = 0; q < S; ++q) {
                    const int4 p = ld_cluster4(base + (uint32_t)(t * 128 + ch) * 4, (uint32_t)q);
                    sum.x += p.x; sum.y += p.y; sum.z += p.z; sum.w += p.w;
                }
            }
            const float xs = ctrl->scale[t];
            const float v[4] = {(float)sum.x * xs * ws[0] + bs[0], (float)sum.y * xs * ws[1] + bs[1],
                                (float)sum.z * xs * ws[2] + bs[2], (float)sum.w * xs * ws[3] + bs[3]};
            O* dst = reinterpret_cast<O*>(a.out) + (long long)(t0 + t) * a.ldo + n;
            if (vec) {
                struct alignas(4 * sizeof(O)) { O e[4]; } o;
#pragma unroll
                for (int j = 0; j < 4; ++j) o.e[j] = from_f<O>(v[j]);
                *reinterpret_cast<decltype(o)*>(dst) = o;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (n + j < a.N) dst[j] = from_f<O>(v[j]);
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
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(tmem_cols) : "memory");
    }
}

template <class X, class O>
static cudaError_t launch_narrow_typed(const CUtensorMap& mW, const CUtensorMap& mX, const NarrowArgs& a, int S, int tiles, size_t smem, cudaStream_t s) {
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
    cfg.numAttrs = g_pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, mW, mX, a);
}

// Clusters of S CTAs with a whole SM each that run at once (how many fit depends on how the SMs are grouped: 148 SMs hold 33
// clusters of four, but only 15 of eight).
static const int* narrow_clusters() {
    static PerDevice ready;
    static int known[MAX_DEVICES][9];
    static const int guess[9] = {0, 148, 74, 45, 33, 26, 22, 15, 15};    // (without a device: the sizes of a workspace query)
    int dev = 0, one = 0;
    if (current_device(&dev) != cudaSuccess) return guess;
    const cudaError_t e = ready.get(dev, &one, [&](int d, int* out) {
        auto kernel = product_narrow_kernel<int8_t, __nv_bfloat16>;
        cudaError_t e2 = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NARROW_SMEM);
        for (int S = 1; S <= 8 && e2 == cudaSuccess; ++S) {
            cudaLaunchConfig_t cfg = {};
            cudaLaunchAttribute attr[1];
            attr[0].id = cudaLaunchAttributeClusterDimension;
            attr[0].val.clusterDim.x = (unsigned)S;
            attr[0].val.clusterDim.y = 1;
            attr[0].val.clusterDim.z = 1;
            cfg.gridDim = dim3((unsigned)(148 * S));
            cfg.blockDim = dim3(NARROW_THREADS);
            cfg.dynamicSmemBytes = NARROW_SMEM;
            cfg.attrs = attr;
            cfg.numAttrs = 1;
            e2 = cudaOccupancyMaxActiveClusters(&known[d][S], kernel, &cfg);
            if (known[d][S] < 1) known[d][S] = 1;
        }
        *out = 1;
        return e2;
    });
    return e == cudaSuccess ? known[dev] : guess;
}

// The tile width and the split of K by which the product is done first.  Measured: 4.8 us for a wave of CTAs and 15 us for
// each MB that one of them brings in (16 tokens, 4096 x 4096: 7.0; 256 tokens: 10.7).  held: the tokens are quantised in the
// kernel, their K range has to fit beside the ring.
struct NarrowShape { int bn, split, stages; size_t smem; double us; };
static bool narrow_shape(int M, int K, int N, bool held, NarrowShape* out) {
    if (held && M > NARROW_HELD) return false;
    const int kb = (K + 127) / 128, tiles_n = (N + 127) / 128;
    const int* at_once = narrow_clusters();
    out->split = 0;
    for (int bn = 16; bn <= NARROW_TOKENS; bn *= 2) {
        if (M > bn && bn < 128) continue;                                // (only the wide tiles are laid side by side)
        const long long tiles = (long long)tiles_n * ((M + bn - 1) / bn);
        if (tiles > 1 << 16) continue;
        for (int S = 1; S <= 8 && S <= kb; ++S) {
            const int most = (kb + S - 1) / S, stage = NARROW_STAGE + (held ? 0 : bn * 128);
            const long long tok = held ? (long long)most * bn * 128 : 0;
            int stages = (int)((NARROW_SMEM - NARROW_CTRL - tok) / stage);
            const int least = (bn * 128 * 4 + stage - 1) / stage;        // (the sums reuse the ring)
            if (stages < 4 || stages < least) continue;
            const double us = (double)((tiles + at_once[S] - 1) / at_once[S]) * (4.8 + 15e-6 * most * (NARROW_STAGE + bn * 128));
            if (out->split && us >= out->us) continue;
            if (stages > NARROW_MAX_STAGES) stages = NARROW_MAX_STAGES;
            if (stages > most) stages = most > least ? most : least;
            *out = NarrowShape{bn, S, stages, (size_t)stages * stage + (size_t)tok + NARROW_CTRL, us};
        }
        if (M <= bn) break;                                              // (a wider tile would only hold more padding)
    }
    return out->split > 0;
}

// Whether the narrow kernel takes a product: unless the pair tiles of 256 x 256 are done sooner (measured: 8.4 us and 6 to
// 11 us for each MB that a pair's SM brings in, 32 KB for each k-block).  quantises: it takes activations, as far as the registers hold a CTA's share of them, from whole 16-byte pieces
// (x_align: the bits that x's address and row pitch have set).
bool narrow_product(int M, int K, int N, int x_type, unsigned long long x_align, bool* quantises) {
    NarrowShape held, shape;
    *quantises = false;
    if (x_type >= 0 && K % 8 == 0 && (x_align & 15u) == 0 && narrow_shape(M, K, N, true, &held)) {
        const int most = ((K + 127) / 128 + held.split - 1) / held.split;
        *quantises = M * ((most + 1) / 2) <= NARROW_WARPS * (x_type == MOK_TYPE_F32 ? Held<float>::pieces : Held<__half>::pieces);
    }
    if (*quantises) return true;
    if (!narrow_shape(M, K, N, false, &shape)) return false;
    const long long waves = ((long long)((N + 255) / 256) * ((M + 255) / 256) + 73) / 74;
    return shape.us <= 8.4 + 8e-6 * (double)waves * ((K + 127) / 128) * 32768;
}

template <class X>
static cudaError_t launch_narrow_out(const CUtensorMap& mW, const CUtensorMap& mX, const NarrowArgs& a, int c_type, int S, int tiles, size_t smem,
                                     cudaStream_t s) {
    if (c_type == MOK_TYPE_F32) return launch_narrow_typed<X, float>(mW, mX, a, S, tiles, smem, s);
    if (c_type == MOK_TYPE_F16) return launch_narrow_typed<X, __half>(mW, mX, a, S, tiles, smem, s);
    return launch_narrow_typed<X, __nv_bfloat16>(mW, mX, a, S, tiles, smem, s);
}

cudaError_t launch_narrow(const ProductArgs& g, const void* x, int x_type, long long ldx, cudaStream_t s) {
    NarrowArgs a = {};
    NarrowShape shape;
    if (!narrow_shape(g.dense_rows, g.K, g.N, x != nullptr, &shape)) return cudaErrorInvalidValue;
    const int S = shape.split;
    const size_t smem = shape.smem;
    a.bn = shape.bn;
    a.stages = shape.stages;
    a.starve = g_starve;
    a.x = x;
    a.ldx = ldx;
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
    CUtensorMap mX = mW;
    if (!x && !tmap::encode_2d(&mX, CU_TENSOR_MAP_DATA_TYPE_UINT8, g.A, (uint64_t)a.M, (uint64_t)g.K, (uint64_t)g.lda, 128,
                               (uint32_t)a.bn, CU_TENSOR_MAP_SWIZZLE_128B))
        return cudaErrorInvalidValue;
    if (!x) return launch_narrow_out<int8_t>(mW, mX, a, g.c_type, S, tiles * ((g.dense_rows + a.bn - 1) / a.bn), smem, s);
    if (x_type == MOK_TYPE_F32) return launch_narrow_out<float>(mW, mX, a, g.c_type, S, tiles, smem, s);
    if (x_type == MOK_TYPE_F16) return launch_narrow_out<__half>(mW, mX, a, g.c_type, S, tiles, smem, s);
    return launch_narrow_out<__nv_bfloat16>(mW, mX, a, g.c_type, S, tiles, smem, s);
}

}  // namespace i8
}  // namespace mok
