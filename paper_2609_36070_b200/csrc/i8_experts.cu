// Routed expert FFNs in 8-bit integers: out[t] = add[t] + sum_s w[t, s] f_{idx[t, s]}(x[t]), every product with exact
// integer sums and one scale per row and per channel.
//   1. dispatch schedule (small batches: inside step 2; in one block; or the layer's own kernels)
//   2. token rows -> codes: found once per token, written once per route, in expert order.  (Gathering the rows in the product
//      instead, with gathering TMA loads of four rows, took 70 cycles per load and three times the product's own time.)
//   3. gate/up product, h = silu(g) u in fp32
//   4. rows of h -> codes and a scale
//   5. down product, fp32 rows
//   6. combine: slot order, fp32, no atomics, so the bits do not depend on the launch
#include "i8_common.cuh"
#include <string.h>

namespace mok {
namespace i8 {

constexpr int THREADS = 256;
constexpr int ONE_BLOCK = 1024, ONE_BLOCK_ROUTES = 32768;    // of the schedule in one block
// Rows per expert up to which launch_grouped is the faster one.  Grouped against pairs, at 80, 112 and 128 rows: 128 experts of
// 2048 x 768 185/191, 207/211, 222/227 us; 32 of 2880 x 2880 188/215, 221/243, 244/283; 16 of 4096 x 2048 118/131, 131/140, 140/141;
// 64 of 1024 x 512 60/67, 76/71, 79/73; at 200 rows the pairs are ahead of all but the third.
constexpr long long GROUPED_ROWS = 112;

// Rows of h (fp32) -> codes and a scale (which the combine puts on), one per route: route j's row is pos[j].
template <int TPR, int NV>
__global__ void __launch_bounds__(THREADS)
quantize_hidden_kernel(const float* __restrict__ h, int I, int8_t* __restrict__ codes, int ldc, float* __restrict__ scales,
                       const int32_t* __restrict__ idx, const int32_t* __restrict__ pos, int n, int E) {
    __shared__ uint32_t s_max[THREADS / 32];
    pdl_enter();
    constexpr int ROWS = THREADS / TPR, WARPS = TPR / 32;
    const int sub = threadIdx.x % TPR, pieces = I >> 2;
    for (int j0 = blockIdx.x * ROWS; j0 < n; j0 += gridDim.x * ROWS) {
        const int j = j0 + threadIdx.x / TPR;
        const int e = j < n ? __ldg(idx + j) : -1;
        const bool live = (unsigned)e < (unsigned)E;
        const int p = live ? __ldg(pos + j) : 0;
        const float4* src = reinterpret_cast<const float4*>(h + (size_t)p * I);
        float4 v[NV];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = sub + i * TPR;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (live && c < pieces) v[i] = __ldcs(src + c);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
            m = max(max(m, max(abs_bits(v[i].x), abs_bits(v[i].y))), max(abs_bits(v[i].z), abs_bits(v[i].w)));
        m = __reduce_max_sync(0xffffffffu, m);
        if (TPR > 32) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
            __syncthreads();
            if (lane == 0) s_max[warp] = m;
            __syncthreads();
            m = __reduce_max_sync(0xffffffffu, lane < WARPS ? s_max[warp / WARPS * WARPS + lane] : 0u);
        }
        if (!live) continue;
        const float amax = __uint_as_float(m);
        const bool codable = m > 0 && finite_bits(m);
        const RowRule rule = row_rule(amax);
        int8_t* dst = codes + (size_t)p * ldc;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = sub + i * TPR;
            if (c >= pieces) break;
            uint32_t o = 0u;
            if (codable) o = four_codes(v[i].x, v[i].y, v[i].z, v[i].w, rule);
            *reinterpret_cast<uint32_t*>(dst + c * 4) = o;
        }
        if (sub == 0) scales[p] = amax / 127.f;
    }
}

// A block per token and 1024 columns, four columns a thread.  Slots whose expert id is outside 0 .. E-1 are not routed: their
// weights are not read.  A routed row counts even with weight 0 (0 times NaN is NaN).
constexpr int COMBINE_THREADS = 256;
template <class T>
__global__ void __launch_bounds__(COMBINE_THREADS)
combine_rows_kernel(const float* __restrict__ y, const float* __restrict__ scales, const int32_t* __restrict__ idx, const float* __restrict__ w,
                    const int32_t* __restrict__ pos, const T* __restrict__ add, long long ld_add, int H, int E, int k,
                    T* __restrict__ out, long long ld_out) {
    struct alignas(4 * sizeof(T)) Four { T e[4]; };
    __shared__ int32_t s_pos[MAX_K];                 // -1: not routed
    __shared__ float s_w[MAX_K];
    pdl_enter();
    const size_t t = blockIdx.x;
    if (threadIdx.x < k) {
        const size_t j = t * k + threadIdx.x;
        const bool routed = (unsigned)idx[j] < (unsigned)E;
        const int p = routed ? pos[j] : -1;
        s_pos[threadIdx.x] = p;
        s_w[threadIdx.x] = routed ? w[j] * scales[p] : 0.f;
    }
    const int c = (blockIdx.y * COMBINE_THREADS + threadIdx.x) * 4;
    const bool mine = c < H;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    if (add && mine) {
        const Four v = *reinterpret_cast<const Four*>(add + t * ld_add + c);
        acc = make_float4(to_f(v.e[0]), to_f(v.e[1]), to_f(v.e[2]), to_f(v.e[3]));
    }
    __syncthreads();
    if (!mine) return;
    for (int s0 = 0; s0 < k; s0 += 8) {
        float4 row[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {            // eight rows on their way at once
            row[s] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s0 + s < k && s_pos[s0 + s] >= 0) row[s] = __ldg(reinterpret_cast<const float4*>(y + (size_t)s_pos[s0 + s] * H + c));
        }
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s0 + s >= k) break;
            const float f = s_w[s0 + s];
            acc.x = fmaf(f, row[s].x, acc.x);
            acc.y = fmaf(f, row[s].y, acc.y);
            acc.z = fmaf(f, row[s].z, acc.z);
            acc.w = fmaf(f, row[s].w, acc.w);
        }
    }
    Four o;
    o.e[0] = from_f<T>(acc.x);
    o.e[1] = from_f<T>(acc.y);
    o.e[2] = from_f<T>(acc.z);
    o.e[3] = from_f<T>(acc.w);
    *reinterpret_cast<Four*>(out + t * ld_out + c) = o;
}

// The schedule in one block, for batches of up to ONE_BLOCK_ROUTES routes: the layer's own schedule keeps an expert's rows in
// route order, which takes several passes (three launches); here a row's place inside its expert's segment is whatever an
// atomic counter gives, because no result depends on it: every row is computed by itself, and the combine reads rows by `pos`.
// Between the passes pos holds a route's place inside its expert.
__global__ void __launch_bounds__(ONE_BLOCK)
schedule_one_kernel(const int32_t* __restrict__ idx, int n, int E, int tile_rows, int32_t* pos, int4* __restrict__ tiles,
                    int32_t* __restrict__ n_tiles) {
    __shared__ int32_t s_cnt[MAX_E], s_row0[MAX_E], s_pads[MAX_E / 32], s_tiles[MAX_E / 32];
    constexpr int DEEP = 8;                      // routes on their way per thread
    pdl_enter();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < MAX_E) s_cnt[tid] = 0;
    __syncthreads();
    for (int j0 = tid; j0 < n; j0 += ONE_BLOCK * DEEP) {
        int e[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) e[i] = j0 + i * ONE_BLOCK < n ? __ldg(idx + j0 + i * ONE_BLOCK) : -1;
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if ((unsigned)e[i] < (unsigned)E) pos[j0 + i * ONE_BLOCK] = atomicAdd(&s_cnt[e[i]], 1);
    }
    __syncthreads();
    int c = 0, pads = 0, mine = 0, pads_to = 0, tiles_to = 0;       // of expert tid; the sums run up to and including it
    if (tid < MAX_E) {
        c = s_cnt[tid];
        pads_to = pads = (c + TILE_M - 1) / TILE_M;
        tiles_to = mine = (c + tile_rows - 1) / tile_rows;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int p = __shfl_up_sync(0xffffffffu, pads_to, off), t = __shfl_up_sync(0xffffffffu, tiles_to, off);
            if (lane >= off) { pads_to += p; tiles_to += t; }
        }
        if (lane == 31) { s_pads[warp] = pads_to; s_tiles[warp] = tiles_to; }
    }
    __syncthreads();
    if (tid < MAX_E) {
        for (int q = 0; q < warp; ++q) { pads_to += s_pads[q]; tiles_to += s_tiles[q]; }
        const int pad0 = pads_to - pads, tile0 = tiles_to - mine;
        s_row0[tid] = pad0 * TILE_M;
        for (int q = 0; q < mine; ++q) tiles[tile0 + q] = make_int4(pad0 * TILE_M + q * tile_rows, c - q * tile_rows, tid, 0);
        if (tid == MAX_E - 1) *n_tiles = tiles_to;
    }
    __syncthreads();
    for (int j0 = tid; j0 < n; j0 += ONE_BLOCK * DEEP) {
        int e[DEEP], place[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) {
            const int j = j0 + i * ONE_BLOCK;
            e[i] = j < n ? __ldg(idx + j) : -1;
            place[i] = (unsigned)e[i] < (unsigned)E ? pos[j] : 0;
        }
#pragma unroll
        for (int i = 0; i < DEEP; ++i)
            if ((unsigned)e[i] < (unsigned)E) pos[j0 + i * ONE_BLOCK] = s_row0[e[i]] + place[i];
    }
}

thread_local bool g_starve = false;

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Workspace of the routed experts: the schedule's tables (a WsLayout of which only those are set) and the activations.
struct ExpertsLayout {
    WsLayout L;
    size_t tiles, xq, xs, h, hq, hs, y, total;
    int pitch_h, pitch_i;
    bool grouped;                // the products for few rows per expert
    int tile_rows;               // of the products' row tiles
    long long max_tiles;         // upper bound of their number
};

static bool experts_layout(int T, int H, int I, int E, int k, ExpertsLayout* X) {
    if (T < 0 || H < 8 || I < 8 || (H % 8) || (I % 8) || E < 1 || E > MAX_E || k < 1 || k > MAX_K || k > E) return false;
    if (H > MAX_CONTRACTION || I > 16384 || (long long)T * k >= (1ll << 31) / 256) return false;
    memset(X, 0, sizeof(*X));
    WsLayout& L = X->L;
    const long long R = (long long)T * k, nonempty = R < E ? R : E;
    const long long rpad = (R + nonempty * (TILE_M - 1) + TILE_M - 1) / TILE_M * TILE_M;
    L.R = (int32_t)R;
    L.Rpad = (int32_t)(rpad > TILE_M ? rpad : TILE_M);
    L.max_mt = L.Rpad / TILE_M;
    L.n_blk = (int32_t)((R + SCHED_CHUNK - 1) / SCHED_CHUNK);
    if (L.n_blk < 1) L.n_blk = 1;
    // Few rows per expert: the weights, streamed once, are the time; from some hundred on it is the bytes that the tiles pull
    // into the SMs, of which the pair tiles pull fewer per product.  Small tiles leave room for more stages, a tile too small
    // streams its expert's weights twice.
    X->grouped = R <= GROUPED_ROWS * (long long)E;
    const bool any = R <= ONE_BLOCK_ROUTES;                 // (the layer's schedule knows tiles of 128 and 256 rows)
    X->tile_rows = !X->grouped ? 2 * TILE_M : any && R <= 32ll * E ? 64 : R <= 64ll * E ? TILE_M : any ? 192 : 2 * TILE_M;
    X->max_tiles = R / X->tile_rows + nonempty;
    X->pitch_h = pitch_of(H);
    X->pitch_i = pitch_of(I);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    const size_t r1 = sizeof(int32_t) * (size_t)(R > 0 ? R : 1);
    L.header = take(sizeof(WsHeader));
    L.counts = take(sizeof(int32_t) * E);
    L.offsets = take(sizeof(int32_t) * (E + 1));
    L.pad_offsets = take(sizeof(int32_t) * (E + 1));
    L.mt_start = take(sizeof(int32_t) * (E + 1));
    L.tile_expert = take(sizeof(int32_t) * (size_t)L.max_mt);
    L.mt_start2 = take(sizeof(int32_t) * (E + 1));
    L.tile_expert2 = take(sizeof(int32_t) * (size_t)L.max_mt);
    L.perm = take(r1);
    L.inv = take(r1);
    L.pos = take(r1);
    L.blk_hist = take(sizeof(int32_t) * (size_t)L.n_blk * E);
    L.row_token = take(sizeof(int32_t) * (size_t)L.Rpad);
    X->tiles = take(sizeof(int4) * (size_t)(R / 64 + nonempty + 1));      // (of the smallest tiles: no size falls as T grows)
    X->xq = take((size_t)L.Rpad * X->pitch_h);
    X->xs = take(sizeof(float) * (size_t)L.Rpad);
    X->h = take(sizeof(float) * (size_t)L.Rpad * I);
    X->hq = take((size_t)L.Rpad * X->pitch_i);
    X->hs = take(sizeof(float) * (size_t)L.Rpad);
    X->y = take(sizeof(float) * (size_t)L.Rpad * H);
    X->total = off;
    return true;
}

template <class T>
static cudaError_t launch_combine(const mok_i8_experts_args* a, const ExpertsLayout& X, char* ws, cudaStream_t s) {
    const dim3 grid((unsigned)a->T, (unsigned)((a->H + 4 * COMBINE_THREADS - 1) / (4 * COMBINE_THREADS)));
    return launch_pdl(combine_rows_kernel<T>, grid, dim3(COMBINE_THREADS), 0, s, reinterpret_cast<const float*>(ws + X.y),
                      reinterpret_cast<const float*>(ws + X.hs), a->topk_idx, a->topk_w,
                      reinterpret_cast<const int32_t*>(ws + X.L.pos), reinterpret_cast<const T*>(a->add), (long long)a->add_stride,
                      a->H, a->E, a->k, reinterpret_cast<T*>(a->out), (long long)a->out_stride);
}

}  // namespace i8
}  // namespace mok

using namespace mok;

extern "C" {

int mok_i8_quantize(const void* x, int type, long long rows, int K, long long x_stride, int8_t* codes, long long codes_stride,
                    float* scales, void* stream) {
    if (!i8::type_ok(type) || rows < 0 || K < 1 || K > i8::MAX_CONTRACTION) return MOK_ERR_SHAPE;
    if (rows > 1 && (x_stride < K || codes_stride < K)) return MOK_ERR_SHAPE;
    if (rows == 0) return MOK_OK;
    if (!x || !codes || !scales) return MOK_ERR_NULL;
    if (!i8::aligned(x, i8::type_bytes(type)) || !i8::aligned(scales, 4)) return MOK_ERR_ALIGN;
    const DependentLaunches dependent;
    const cudaError_t e = i8::launch_quantize(x, type, rows, K, x_stride, codes, codes_stride > K ? codes_stride : K, scales,
                                              reinterpret_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

static unsigned long long x_alignment(const mok_i8_linear_args* a) {
    return reinterpret_cast<uintptr_t>(a->x) | (a->M > 1 ? (unsigned long long)a->x_stride * i8::type_bytes(a->x_type) : 0ull);
}
static size_t codes_bytes(int M, int K) { return align_up((size_t)M * i8::pitch_of(K), 256) + align_up((size_t)M * sizeof(float), 256); }

size_t mok_i8_linear_workspace_bytes(const mok_i8_linear_args* a) {
    if (!a || !a->x || a->M < 1 || a->K < 1 || a->N < 1 || a->K > i8::MAX_CONTRACTION || !i8::type_ok(a->x_type)) return 0;
    bool quantises = false;
    return i8::narrow_product(a->M, a->K, a->N, a->x_type, x_alignment(a), &quantises) && quantises ? 0 : codes_bytes(a->M, a->K);
}

int mok_i8_linear(const mok_i8_linear_args* a) {
    if (!a) return MOK_ERR_NULL;
    const bool coded = a->x == nullptr && a->x_codes != nullptr;
    if (a->M < 0 || a->K < 1 || a->K > i8::MAX_CONTRACTION || a->N < 1 || !i8::type_ok(a->out_type) ||
        (!coded && !i8::type_ok(a->x_type)))
        return MOK_ERR_SHAPE;
    // (strides of single rows do not count)
    if ((a->M > 1 && ((coded ? a->codes_stride : a->x_stride) < a->K || a->out_stride < a->N)) || (a->N > 1 && a->w_stride < a->K))
        return MOK_ERR_SHAPE;
    if (a->M == 0) return MOK_OK;
    if ((!a->x && !a->x_codes) || (coded && !a->x_scales) || !a->W_codes || !a->W_scales || !a->out) return MOK_ERR_NULL;
    if (!i8::aligned(a->W_codes, 16) || (a->N > 1 && a->w_stride % 16) || !i8::aligned(a->W_scales, 4) || !i8::aligned(a->bias, 4) ||
        !i8::aligned(a->out, i8::type_bytes(a->out_type)))
        return MOK_ERR_ALIGN;
    if (coded ? !i8::aligned(a->x_codes, 16) || (a->M > 1 && a->codes_stride % 16) || !i8::aligned(a->x_scales, 4)
              : !i8::aligned(a->x, i8::type_bytes(a->x_type)))
        return MOK_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    const DependentLaunches dependent;
    i8::ProductArgs g = {};
    cudaError_t e = i8::status_header(&g.header);
    if (e != cudaSuccess) return cuda_fail(e);
    g.a_rows = a->M;
    g.B = a->W_codes;
    g.ldb = a->N > 1 ? a->w_stride : i8::pitch_of(a->K);
    g.b_scale = a->W_scales;
    g.bias = a->bias;
    g.K = a->K; g.N = a->N; g.E = 1;
    g.C = a->out;
    g.ldc = a->M > 1 ? a->out_stride : a->N;
    g.c_type = a->out_type;
    g.dense_rows = a->M;
    g.max_mt = (a->M + 2 * TILE_M - 1) / (2 * TILE_M);
    bool quantises = false;
    const bool narrow = i8::narrow_product(a->M, a->K, a->N, coded ? -1 : a->x_type, x_alignment(a), &quantises);
    if (coded) {
        g.A = a->x_codes;
        g.lda = a->M > 1 ? a->codes_stride : i8::pitch_of(a->K);
        g.a_scale = a->x_scales;
    } else {
        if (narrow && quantises) {
            e = i8::launch_narrow(g, a->x, a->x_type, a->x_stride, s);
            return e == cudaSuccess ? MOK_OK : cuda_fail(e);
        }
        if (!a->workspace || !i8::aligned(a->workspace, 256) || a->workspace_bytes < codes_bytes(a->M, a->K)) return MOK_ERR_WORKSPACE;
        char* ws = reinterpret_cast<char*>(a->workspace);
        int8_t* codes = reinterpret_cast<int8_t*>(ws);
        const int pitch = i8::pitch_of(a->K);
        float* scales = reinterpret_cast<float*>(ws + align_up((size_t)a->M * pitch, 256));
        e = i8::launch_quantize(a->x, a->x_type, a->M, a->K, a->x_stride, codes, pitch, scales, s);
        if (e != cudaSuccess) return cuda_fail(e);
        g.A = codes;
        g.lda = pitch;
        g.a_scale = scales;
    }
    e = narrow ? i8::launch_narrow(g, nullptr, 0, 0, s) : i8::launch_product(g, i8::EPI_PLAIN, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

size_t mok_i8_experts_workspace_bytes(int T, int H, int I, int E, int k) {
    i8::ExpertsLayout X;
    return i8::experts_layout(T, H, I, E, k, &X) ? X.total : 0;
}

int mok_i8_experts(const mok_i8_experts_args* a) {
    if (!a) return MOK_ERR_NULL;
    i8::ExpertsLayout X;
    if (!i8::experts_layout(a->T, a->H, a->I, a->E, a->k, &X) || (a->type != MOK_TYPE_BF16 && a->type != MOK_TYPE_F16))
        return MOK_ERR_SHAPE;
    if (a->gate_up_stride < a->H || a->down_stride < a->I ||
        (a->T > 1 && (a->x_stride < a->H || a->out_stride < a->H || (a->add && a->add_stride < a->H))))
        return MOK_ERR_SHAPE;
    if (a->T == 0) return MOK_OK;
    if (!a->x || !a->topk_idx || !a->topk_w || !a->gate_up_codes || !a->gate_up_scales || !a->down_codes || !a->down_scales ||
        !a->down_max || !a->out)
        return MOK_ERR_NULL;
    if (!i8::aligned(a->x, 2) || !i8::aligned(a->out, 16) || !i8::aligned(a->add, 16) || !i8::aligned(a->gate_up_codes, 16) ||
        !i8::aligned(a->down_codes, 16) || (a->gate_up_stride % 16) || (a->down_stride % 16) || (a->out_stride % 8) ||
        (a->add && a->add_stride % 8) || !i8::aligned(a->topk_idx, 4) || !i8::aligned(a->topk_w, 4) ||
        !i8::aligned(a->gate_up_scales, 4) || !i8::aligned(a->down_scales, 4) || !i8::aligned(a->down_max, 4))
        return MOK_ERR_ALIGN;
    if (!a->workspace || !i8::aligned(a->workspace, 256) || a->workspace_bytes < X.total) return MOK_ERR_WORKSPACE;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    char* ws = reinterpret_cast<char*>(a->workspace);
    WsHeader* hdr = reinterpret_cast<WsHeader*>(ws + X.L.header);
    const DependentLaunches dependent;
    i8::ProductArgs g = {};
    cudaError_t e = i8::status_header(&g.header);
    if (e != cudaSuccess) return cuda_fail(e);
    auto table = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
    int4* tiles = reinterpret_cast<int4*>(ws + X.tiles);
    i8::RouteArgs routes = {a->topk_idx, table(X.L.pos), a->E, a->k, 0, X.tile_rows, tiles, &hdr->n_ftiles};
    if (X.L.R <= i8::ROUTES_HERE) {
        routes.n = X.L.R;
    } else if (X.L.R <= i8::ONE_BLOCK_ROUTES) {
        e = launch_pdl(i8::schedule_one_kernel, dim3(1), dim3(i8::ONE_BLOCK), 0, s, a->topk_idx, X.L.R, a->E, X.tile_rows,
                       routes.pos, tiles, routes.n_tiles);
        routes.tiles = nullptr;
    } else {
        e = launch_schedule(a->topk_idx, a->T, a->E, a->k, TILE_M, TILE_M, X.L, ws, nullptr, nullptr, nullptr, nullptr, s);
        const bool half = X.tile_rows == TILE_M;
        routes.n_tiles = half ? &hdr->n_mtiles : &hdr->n_mtiles2;
        routes.tile_expert = table(half ? X.L.tile_expert : X.L.tile_expert2);
        routes.mt_start = table(half ? X.L.mt_start : X.L.mt_start2);
        routes.pad_offsets = table(X.L.pad_offsets);
        routes.counts = table(X.L.counts);
    }
    g.n_mtiles = routes.n_tiles;
    if (e != cudaSuccess) return cuda_fail(e);
    e = i8::launch_quantize(a->x, a->type, a->T, a->H, a->x_stride, reinterpret_cast<int8_t*>(ws + X.xq), X.pitch_h,
                            reinterpret_cast<float*>(ws + X.xs), s, &routes);
    if (e != cudaSuccess) return cuda_fail(e);
    g.E = a->E;
    g.tiles = tiles;
    g.tile_rows = X.tile_rows;
    g.max_mt = (int32_t)X.max_tiles;
    g.A = reinterpret_cast<const int8_t*>(ws + X.xq);
    g.lda = X.pitch_h;
    g.a_rows = X.L.Rpad;
    g.a_scale = reinterpret_cast<const float*>(ws + X.xs);
    g.B = a->gate_up_codes;
    g.ldb = a->gate_up_stride;
    g.b_scale = a->gate_up_scales;
    g.K = a->H; g.N = a->I;
    g.C = ws + X.h;
    g.ldc = a->I;
    e = X.grouped ? i8::launch_grouped(g, i8::EPI_GATED, s) : i8::launch_product(g, i8::EPI_GATED, s);
    if (e != cudaSuccess) return cuda_fail(e);
    {
        const float* h = reinterpret_cast<const float*>(ws + X.h);
        int8_t* hq = reinterpret_cast<int8_t*>(ws + X.hq);
        auto rows = [&](auto kernel, int per_block) {
            const int blocks = (X.L.R + per_block - 1) / per_block, most = 148 * 16;
            return launch_pdl(kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(i8::THREADS), 0, s, h, a->I, hq, X.pitch_i,
                              reinterpret_cast<float*>(ws + X.hs), a->topk_idx, table(X.L.pos), X.L.R, a->E);
        };
        e = a->I <= 1024 ? rows(i8::quantize_hidden_kernel<32, 8>, 8)
            : a->I <= 2048 ? rows(i8::quantize_hidden_kernel<128, 4>, 2)
            : a->I <= 4096 ? rows(i8::quantize_hidden_kernel<256, 4>, 1)
            : a->I <= 8192 ? rows(i8::quantize_hidden_kernel<256, 8>, 1) : rows(i8::quantize_hidden_kernel<256, 16>, 1);
        if (e != cudaSuccess) return cuda_fail(e);
    }
    g.A = reinterpret_cast<const int8_t*>(ws + X.hq);
    g.lda = X.pitch_i;
    g.a_scale = nullptr;
    g.B = a->down_codes;
    g.ldb = a->down_stride;
    g.b_scale = a->down_scales;
    g.K = a->I; g.N = a->H;
    g.C = ws + X.y;
    g.ldc = a->H;
    e = X.grouped ? i8::launch_grouped(g, i8::EPI_ROWS, s) : i8::launch_product(g, i8::EPI_ROWS, s);
    if (e != cudaSuccess) return cuda_fail(e);
    e = a->type == MOK_TYPE_BF16 ? i8::launch_combine<__nv_bfloat16>(a, X, ws, s) : i8::launch_combine<__half>(a, X, ws, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

int mok_i8_starve(int wait_limit_us, void* stream) {
    if (wait_limit_us < 0) return MOK_ERR_SHAPE;
    WsHeader* hdr = nullptr;
    cudaError_t e = i8::status_header(&hdr);
    if (e != cudaSuccess) return cuda_fail(e);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const uint32_t limit = (uint32_t)wait_limit_us;
    if ((e = cudaMemcpyAsync(&hdr->wait_limit_us, &limit, sizeof(limit), cudaMemcpyHostToDevice, s)) != cudaSuccess ||
        (e = cudaStreamSynchronize(s)) != cudaSuccess)
        return cuda_fail(e);
    i8::g_starve = wait_limit_us > 0;
    return MOK_OK;
}

int mok_i8_status(void* stream) {
    WsHeader* hdr = nullptr;
    cudaError_t e = i8::status_header(&hdr);
    if (e != cudaSuccess) return cuda_fail(e);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    int32_t status = 0;
    if ((e = cudaMemcpyAsync(&status, &hdr->status, sizeof(status), cudaMemcpyDeviceToHost, s)) != cudaSuccess ||
        (e = cudaMemsetAsync(&hdr->status, 0, sizeof(status), s)) != cudaSuccess || (e = cudaStreamSynchronize(s)) != cudaSuccess)
        return cuda_fail(e);
    return status;
}

}  // extern "C"
