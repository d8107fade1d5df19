// Routing scores -> experts and weights, and the gradient back to the logits.
//
//   s = sigmoid(l) or softmax(l) over the E experts of a token (fp32 whatever the logits' type)
//   c = s + bias                     the choice value; the bias decides the selection only, never a weight
//   groups of E / n_groups consecutive experts: a group's value is its best c, or the sum of its two best; the
//   topk_groups best groups stay.  The k best c among them are the token's experts, in descending order; every tie (of
//   groups and of experts) goes to the lowest id.
//   w_i = scale * s_i / sum_j s_j over the chosen (renormalise; 0 where the sum is 0), or scale * s_i
// The scores rise with the logits, so without a bias and without sums of two scores the logits themselves are compared:
// two logits that a score rounds to the same number keep their order, and no score but the chosen ones is computed.
//
// One warp per token, lane l holds experts l, l + 32, ...: a token's logits are read once, coalesced.  A round of the
// selection is a maximum over the lane's own values, a warp maximum of order-preserving integer keys (redux.sync) and,
// if several lanes hold it, a warp minimum of their ids.
#include "mok_internal.cuh"
#include <cuda_fp16.h>
#include <float.h>

namespace mok {
namespace gate {

constexpr int WARPS = 4;

__device__ __forceinline__ float load_f(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_f(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_f(__half* p, float v) { *p = __float2half_rn(v); }

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }

// Keys that compare as the values do: absent or taken experts 0, NaN 1, then -inf ... +inf.  -0 counts as 0.
__device__ __forceinline__ unsigned choice_key(float v) {
    if (v != v) return 1u;
    const unsigned u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
    return v;
}
// exp(l - m), 0 where everything is masked (m = -inf)
__device__ __forceinline__ float exp_below(float l, float m) { return m == -INFINITY ? 0.f : expf(l - m); }

struct Params {
    const void* logits;
    const float* bias;
    long long stride;
    int32_t T, E, k, softmax, n_groups, topk_groups, group_top, renormalise;
    float scale;
    int32_t* idx;
    float* w;
};

template <class L, int VPL>
__global__ void __launch_bounds__(32 * WARPS)
gate_kernel(const Params p) {
    extern __shared__ float s_choice[];              // [WARPS][E], group-limited routing only
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int E = p.E, k = p.k, G = p.n_groups, gs = E / G;
    const bool by_score = p.bias != nullptr || (G > 1 && p.group_top == 2);
    float bias[VPL];
    int group[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int e = lane + 32 * j;
        bias[j] = (p.bias && e < E) ? __ldg(p.bias + e) : 0.f;
        group[j] = G > 1 ? e / gs : 0;
    }
    int per = 1;                                     // lanes that share a group's experts: G * per <= 32
    while (G * per * 2 <= 32) per *= 2;
    for (int t = blockIdx.x * WARPS + warp; t < p.T; t += gridDim.x * WARPS) {
        const L* row = reinterpret_cast<const L*>(p.logits) + (long long)t * p.stride;
        float c[VPL];
        float m = -INFINITY, total = 1.f;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int e = lane + 32 * j;
            c[j] = e < E ? load_f(row + e) : -INFINITY;
        }
        const bool full_sum = p.softmax && (by_score || !p.renormalise);
        if (p.softmax) {
#pragma unroll
            for (int j = 0; j < VPL; ++j) m = fmaxf(m, c[j]);
            m = warp_max(m);
        }
        if (full_sum) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) sum += (lane + 32 * j < E) ? exp_below(c[j], m) : 0.f;
            total = m == -INFINITY ? 1.f : warp_sum(sum);
        }
        if (by_score) {
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const float s = p.softmax ? (m == -INFINITY ? 0.f : expf(c[j] - m) / total) : sigmoid(c[j]);
                c[j] = s + bias[j];
            }
        }
        unsigned kept = 0xffffffffu;
        if (G > 1) {
            float* mine = s_choice + warp * E;
#pragma unroll
            for (int j = 0; j < VPL; ++j)
                if (lane + 32 * j < E) mine[lane + 32 * j] = c[j];
            __syncwarp();
            // `per` neighbouring lanes find the two best of one group; its value is compared with every other group's
            const int g = lane / per;
            float b1 = -INFINITY, b2 = -INFINITY;
            if (g < G) {
                const int q = lane & (per - 1), n = (gs - q + per - 1) / per;
                int i = g % (n > 0 ? n : 1);         // staggered, so that equal places of the groups do not share a bank
                for (int it = 0; it < n; ++it) {
                    const float v = mine[g * gs + q + i * per];
                    i = i + 1 == n ? 0 : i + 1;
                    b2 = fmaxf(b2, fminf(b1, v));
                    b1 = fmaxf(b1, v);
                }
            }
            for (int off = 1; off < per; off <<= 1) {
                const float o1 = __shfl_xor_sync(0xffffffffu, b1, off), o2 = __shfl_xor_sync(0xffffffffu, b2, off);
                b2 = fmaxf(fminf(b1, o1), fmaxf(b2, o2));
                b1 = fmaxf(b1, o1);
            }
            const unsigned value = choice_key(p.group_top == 2 ? b1 + b2 : b1);
            int rank = 0;
            for (int q = 0; q < G; ++q) {
                const unsigned other = __shfl_sync(0xffffffffu, value, q * per);
                rank += (other > value || (other == value && q < g)) ? 1 : 0;
            }
            const unsigned lanes = __ballot_sync(0xffffffffu, g < G && rank < p.topk_groups);
            kept = 0u;
            for (int q = 0; q < G; ++q) kept |= ((lanes >> (q * per)) & 1u) << q;
            __syncwarp();                            // `mine` is rewritten by the next token
        }
        unsigned key[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            key[j] = (lane + 32 * j < E && ((kept >> group[j]) & 1u)) ? choice_key(c[j]) : 0u;
        int my_e = 0;
        for (int s = 0; s < k; ++s) {
            unsigned best = key[0];
            int bj = 0;
#pragma unroll
            for (int j = 1; j < VPL; ++j)
                if (key[j] > best) { best = key[j]; bj = j; }         // strict: the lowest id of the lane's equals
            const unsigned top = __reduce_max_sync(0xffffffffu, best);
            int e = best == top ? lane + 32 * bj : 0x7fffffff;
            const unsigned holders = __ballot_sync(0xffffffffu, best == top);
            const int e_win = (holders & (holders - 1)) ? __reduce_min_sync(0xffffffffu, e)
                                                        : __shfl_sync(0xffffffffu, e, __ffs(holders) - 1);
            if (e == e_win) {
#pragma unroll
                for (int j = 0; j < VPL; ++j)
                    if (j == bj) key[j] = 0u;
            }
            if (lane == s) my_e = e_win;
        }
        // the chosen experts' scores, one per lane
        float s = 0.f;
        if (lane < k) {
            const float l = load_f(row + my_e);
            s = !p.softmax ? sigmoid(l) : full_sum ? exp_below(l, m) / total : exp_below(l, m);
        }
        if (p.renormalise) {
            const float sum = warp_sum(s);
            s = sum > 0.f || sum != sum ? s / sum : 0.f;
        }
        if (lane < k) {
            p.idx[(size_t)t * k + lane] = my_e;
            p.w[(size_t)t * k + lane] = s * p.scale;
        }
    }
}

struct BwdParams {
    const void* logits;
    const int32_t* idx;
    const float* dw;
    long long stride, d_stride;
    int32_t T, E, k, softmax, renormalise;
    float scale;
    void* dlogits;
};

// dL/dlogits from dL/dw, g = scale * dw:
//   renormalised  sigmoid: dl_i = s_i (1 - s_i) (g_i - sum_j g_j s_j / S) / S      S = sum of the chosen scores
//                 softmax: dl_i = p_i (g_i - sum_j g_j p_j)                         p = softmax over the chosen logits
//   as they are   sigmoid: dl_i = g_i s_i (1 - s_i)
//                 softmax: dl_e = s_e (g_e - sum_j g_j s_j)                         for every expert e, g_e = 0 if not chosen
// Only the last one is non-zero outside the chosen experts (and reads all logits).  1 - s is sigmoid(-l), without the
// cancellation.  One warp per token; the row is put together in shared memory and written once, coalesced.  Chosen ids
// outside 0 .. E-1 (routes that were dropped) have no part in it.
template <class L>
__global__ void __launch_bounds__(32 * WARPS)
gate_backward_kernel(const BwdParams p) {
    extern __shared__ float s_row[];                 // [WARPS][E]
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int E = p.E, k = p.k;
    float* mine = s_row + warp * E;
    for (int t = blockIdx.x * WARPS + warp; t < p.T; t += gridDim.x * WARPS) {
        const L* row = reinterpret_cast<const L*>(p.logits) + (long long)t * p.stride;
        L* out = reinterpret_cast<L*>(p.dlogits) + (long long)t * p.d_stride;
        int e = -1;
        float g = 0.f, l = 0.f;
        if (lane < k) {
            e = p.idx[(size_t)t * k + lane];
            if ((unsigned)e >= (unsigned)E) e = -1;
            if (e >= 0) {
                g = p.dw[(size_t)t * k + lane] * p.scale;
                l = load_f(row + e);
            }
        }
        const bool dense = p.softmax && !p.renormalise;
        for (int i = lane; i < E; i += 32) mine[i] = 0.f;
        __syncwarp();
        if (!dense) {
            float d = 0.f;
            if (p.softmax) {
                const float m = warp_max(e >= 0 ? l : -INFINITY);
                const float q = e >= 0 ? exp_below(l, m) : 0.f;
                const float S = warp_sum(q);
                const float pi = S > 0.f ? q / S : 0.f;
                d = pi * (g - warp_sum(g * pi));
            } else {
                const float s = e >= 0 ? sigmoid(l) : 0.f;
                const float slope = s * sigmoid(-l);
                if (p.renormalise) {
                    const float S = warp_sum(s), inv = S > 0.f ? 1.f / S : 0.f;
                    d = slope * inv * (g - warp_sum(g * s) * inv);
                } else {
                    d = g * slope;
                }
            }
            if (e >= 0) mine[e] = d;
            __syncwarp();
            for (int i = lane; i < E; i += 32) store_f(out + i, mine[i]);
        } else {
            float m = -INFINITY, sum = 0.f;
            for (int i = lane; i < E; i += 32) m = fmaxf(m, load_f(row + i));
            m = warp_max(m);
            for (int i = lane; i < E; i += 32) sum += exp_below(load_f(row + i), m);
            sum = warp_sum(sum);
            const float inv = sum > 0.f ? 1.f / sum : 0.f;
            const float dot = warp_sum(e >= 0 ? g * exp_below(l, m) * inv : 0.f);
            if (e >= 0) mine[e] = g;
            __syncwarp();
            for (int i = lane; i < E; i += 32) {
                const float s = exp_below(load_f(row + i), m) * inv;
                store_f(out + i, s * (mine[i] - dot));
            }
        }
        __syncwarp();
    }
}

template <class L>
static cudaError_t launch_gate(const Params& p, cudaStream_t s) {
    long long blocks = ((long long)p.T + WARPS - 1) / WARPS;
    if (blocks > 148 * 12) blocks = 148 * 12;
    const size_t smem = p.n_groups > 1 ? sizeof(float) * WARPS * p.E : 0;
    const int vpl = (p.E + 31) / 32;
    const dim3 grid((unsigned)blocks), block(32 * WARPS);
    if (vpl <= 1) return launch_pdl(gate_kernel<L, 1>, grid, block, smem, s, p);
    if (vpl <= 2) return launch_pdl(gate_kernel<L, 2>, grid, block, smem, s, p);
    if (vpl <= 4) return launch_pdl(gate_kernel<L, 4>, grid, block, smem, s, p);
    if (vpl <= 8) return launch_pdl(gate_kernel<L, 8>, grid, block, smem, s, p);
    return launch_pdl(gate_kernel<L, 16>, grid, block, smem, s, p);
}

template <class L>
static cudaError_t launch_backward(const BwdParams& p, cudaStream_t s) {
    long long blocks = ((long long)p.T + WARPS - 1) / WARPS;
    if (blocks > 148 * 12) blocks = 148 * 12;
    return launch_pdl(gate_backward_kernel<L>, dim3((unsigned)blocks), dim3(32 * WARPS), sizeof(float) * WARPS * p.E, s, p);
}

static bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
static bool type_ok(int t) { return t == MOK_TYPE_BF16 || t == MOK_TYPE_F16 || t == MOK_TYPE_F32; }
static size_t type_bytes(int t) { return t == MOK_TYPE_F32 ? 4 : 2; }

}  // namespace gate
}  // namespace mok

using namespace mok;

extern "C" {

int mok_gate(const mok_gate_args* a) {
    if (!a) return MOK_ERR_NULL;
    if (a->T < 0 || a->E < 1 || a->E > MAX_E || a->k < 1 || a->k > MAX_K || a->n_groups < 1 || a->n_groups > 32 ||
        a->E % a->n_groups || a->topk_groups < 1 || a->topk_groups > a->n_groups || !gate::type_ok(a->logits_type) ||
        (a->score != MOK_SCORE_SOFTMAX && a->score != MOK_SCORE_SIGMOID))
        return MOK_ERR_SHAPE;
    const int gs = a->E / a->n_groups;
    if (a->k > a->topk_groups * gs) return MOK_ERR_SHAPE;
    if (a->n_groups > 1 && (a->group_top < 1 || a->group_top > 2 || a->group_top > gs)) return MOK_ERR_SHAPE;
    if (a->logits_stride < a->E && a->T > 1) return MOK_ERR_SHAPE;
    if (a->T == 0) return MOK_OK;
    if (!a->logits || !a->topk_idx || !a->topk_w) return MOK_ERR_NULL;
    if (!gate::aligned(a->logits, gate::type_bytes(a->logits_type)) || !gate::aligned(a->bias, 4) ||
        !gate::aligned(a->topk_idx, 4) || !gate::aligned(a->topk_w, 4))
        return MOK_ERR_ALIGN;
    const gate::Params p = {a->logits, a->bias, a->logits_stride, a->T, a->E, a->k, a->score == MOK_SCORE_SOFTMAX,
                            a->n_groups, a->topk_groups, a->group_top, a->renormalise != 0, a->scale, a->topk_idx, a->topk_w};
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    g_pdl = true;
    cudaError_t e = a->logits_type == MOK_TYPE_F32 ? gate::launch_gate<float>(p, s)
                    : a->logits_type == MOK_TYPE_BF16 ? gate::launch_gate<__nv_bfloat16>(p, s) : gate::launch_gate<__half>(p, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

int mok_gate_backward(const mok_gate_bwd_args* a) {
    if (!a) return MOK_ERR_NULL;
    if (a->T < 0 || a->E < 1 || a->E > MAX_E || a->k < 1 || a->k > MAX_K || a->k > a->E || !gate::type_ok(a->logits_type) ||
        (a->score != MOK_SCORE_SOFTMAX && a->score != MOK_SCORE_SIGMOID))
        return MOK_ERR_SHAPE;
    if ((a->logits_stride < a->E || a->dlogits_stride < a->E) && a->T > 1) return MOK_ERR_SHAPE;
    if (a->T == 0) return MOK_OK;
    if (!a->logits || !a->topk_idx || !a->dw || !a->dlogits) return MOK_ERR_NULL;
    const size_t tb = gate::type_bytes(a->logits_type);
    if (!gate::aligned(a->logits, tb) || !gate::aligned(a->dlogits, tb) || !gate::aligned(a->topk_idx, 4) ||
        !gate::aligned(a->dw, 4))
        return MOK_ERR_ALIGN;
    const gate::BwdParams p = {a->logits, a->topk_idx, a->dw, a->logits_stride, a->dlogits_stride, a->T, a->E, a->k,
                               a->score == MOK_SCORE_SOFTMAX, a->renormalise != 0, a->scale, a->dlogits};
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    g_pdl = true;
    cudaError_t e = a->logits_type == MOK_TYPE_F32 ? gate::launch_backward<float>(p, s)
                    : a->logits_type == MOK_TYPE_BF16 ? gate::launch_backward<__nv_bfloat16>(p, s)
                                                      : gate::launch_backward<__half>(p, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

}  // extern "C"
