// Routing scores -> experts and weights, and the gradient back to the logits.
//
//   s = sigmoid(l) or softmax(l) over the E experts of a token (fp32 whatever the logits' type)
//   c = s + bias                     the choice value; the bias decides the selection only, never a weight
//   groups of E / n_groups consecutive experts: a group's value is its best c, or the sum of its two best; experts that may
//   not be used (c of -inf or NaN) add nothing to it, and a group of such experts only is below all others.  The
//   topk_groups best groups stay.  The k best c among them are the token's experts, in descending order; every tie (of
//   groups and of experts) goes to the lowest id.
//   w_i = scale * s_i / sum_j s_j over the chosen (renormalise; 0 where the sum is 0), or scale * s_i
// The scores rise with the logits, so without a bias and without sums of two scores the logits themselves are compared:
// two logits that a score rounds to the same number keep their order, and no score but the chosen ones is computed.
//
// With many tokens the kernels are bound by instructions, not by the logits' bytes (32768 tokens of 256 experts: 5 us of
// memory traffic), so the common case, no groups or groups of a multiple of four experts, puts FOUR tokens into a warp,
// eight lanes each: every step across lanes then serves four tokens.  Lane p of a token holds pieces p, p + 8, ... of four
// consecutive experts and the largest value of each piece.  Two ways to the k largest:
//   - lists (k = 5 .. 16): the k-th largest of the lanes' two largest piece maxima is a lower bound of the k-th largest value; the
//     values that reach it, a few more than k, are listed in shared memory, and a value's place is the number of listed
//     values before it.
//   - rounds (small k, where they are cheaper; large k; and tokens with more than 32 values in reach, which equal values can
//     bring): a maximum over the lane's pieces, three shuffles across the eight lanes, and a refill of the one piece that
//     lost its largest value.
// 229 instructions per token (256 experts, k = 8; 395 with groups and a bias) against 610 (1300) with a warp per token: 12.2
// (20.7) us for 32768 tokens against 25 (53), one call after the other on rows that stay in L2; 23.2 with groups on changing rows.
// Issue slots are 55 % used, the pipe of comparisons 46 to 50 %; the rest is the latency of
// its steps, with the 20 warps per SM that the registers allow (more warps and spilled values, or the next rows copied ahead
// into shared memory, were 2 to 7 % slower).  Other groupings, and batches that do not fill the GPU (up to some 2300 tokens: 4.7
// against 7.4 us for 512 tokens), take the warp-per-token kernel, whose chain of steps is shorter.
#include "mok_internal.cuh"
#include <cuda_fp16.h>

namespace mok {
namespace gate {

constexpr int WARPS = 4;
static_assert(MAX_K == 32, "the kernels add up the chosen scores of four slots per lane, or of one");

__device__ __forceinline__ float load_f(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_f(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ float load_f(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ void store_f(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void store_f(__half* p, float v) { *p = __float2half_rn(v); }

__device__ __forceinline__ float sigmoid(float l) { return 1.f / (1.f + expf(-l)); }

// For the comparison of scores: within 2^-21 of the exact value, absolutely, as scores near 1 are in fp32.  (Relatively the
// exponent's rounding counts as well: 2^-24 |l|, 1e-6 of the score for l = -20.)  Weights are not made of it.
__device__ __forceinline__ float exp2_near(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
constexpr float LOG2_E = 1.44269504f;
__device__ __forceinline__ float sigmoid_near(float l) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + exp2_near(-LOG2_E * l)));
    return r;
}
// 1 where a > b, to be summed by additions: those run beside the comparisons, and integer additions do not.
__device__ __forceinline__ float one_if_above(float a, float b) {
    float r;
    asm("set.gt.f32.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// The next value below v, any but -inf and NaN.
__device__ __forceinline__ float next_below(float v) {
    const int u = __float_as_int(v);
    return __int_as_float(v > 0.f ? u - 1 : v == 0.f ? (int)0x80000001u : u + 1);
}
// For a 16-bit logit, whose last bits are free in fp32: expert e's place there sorts equals by their ids.  Finite v.
__device__ __forceinline__ float with_id(float v, int e) {
    const unsigned u = __float_as_uint(v + 0.f);
    return __uint_as_float(u | (unsigned)((u >> 31) ? e : MAX_E - 1 - e));
}
// What a choice value is compared as.  -inf stands for "not there", so NaN and -inf take the place of the lowest finite values,
// in this order; finite values that low count as AT_LOWEST, so that both kernels order all values alike.
constexpr float AT_NAN = -3.40282347e38f, AT_MINUS_INF = -3.40282326e38f, AT_LOWEST = -3.40282306e38f;
__device__ __forceinline__ float ranked(float v) {
    return v != v ? AT_NAN : v == -INFINITY ? AT_MINUS_INF : fmaxf(v, AT_LOWEST);
}
// A group's value from its two best ranked values, or its best one
__device__ __forceinline__ float group_value(float b1, float b2, bool two) {
    if (b1 <= AT_MINUS_INF) return AT_NAN;
    return two && b2 > AT_MINUS_INF ? fmaxf(b1 + b2, AT_LOWEST) : b1;
}
// Keys that compare as ranked values do; absent or taken experts are 0.  -0 counts as 0.
__device__ __forceinline__ unsigned choice_key(float v) {
    const unsigned u = __float_as_uint(v + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
// (Pairs of neighbours first.  The order of the sums is the one of the four-token kernel, where lane l's experts l, l + 32, ...
// are element l % 4 of the pieces of lane l / 4: a token's weights have the same bits in any batch.)
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
    return v;
}
// Reductions over the eight lanes of a token.
__device__ __forceinline__ float max8(float v) {
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, off));
    return v;
}
__device__ __forceinline__ float sum8(float v) {
#pragma unroll
    for (int off = 1; off < 8; off <<= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}
// 1 / sum where that is finite: a sum of subnormal scores, and the scores, are multiplied by lift(sum) first.  (One quotient for
// all scores: a quotient for each was 3 to 12 % slower.)
__device__ __forceinline__ float lift(float sum) { return sum < 0x1p-64f ? 0x1p+64f : 1.f; }
__device__ __forceinline__ float inverse(float sum, float up) { return sum == 0.f ? 0.f : 1.f / (sum * up); }
// What a row's exponentials are taken from: its maximum, 0 where everything is masked (so that they are 0), or NaN.
__device__ __forceinline__ float exp_from(float m) { return m == -INFINITY ? 0.f : m; }

struct Params {
    const void* logits;
    const float* bias;
    long long stride;
    int32_t T, E, k, softmax, n_groups, topk_groups, group_top, renormalise;
    float scale;
    int32_t* idx;
    float* w;
};

// Any grouping: one warp per token, lane l holds experts l, l + 32, ...; k rounds of a warp maximum.
template <class L, int VPL>
__global__ void __launch_bounds__(32 * WARPS)
gate_warp_kernel(const Params p) {
    extern __shared__ float s_choice[];              // [WARPS][E]
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
    for (long long t = (long long)blockIdx.x * WARPS + warp; t < p.T; t += (long long)gridDim.x * WARPS) {
        const L* row = reinterpret_cast<const L*>(p.logits) + t * p.stride;
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
            m = exp_from(warp_max(m));
        }
        if (full_sum) {
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < VPL; ++j) sum += expf(c[j] - m);
            sum = warp_sum(sum);
            total = sum == 0.f ? 1.f : sum;
        }
        if (by_score) {
            const float inv = 1.f / total;
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const float s = p.softmax ? __fmul_rn(expf(c[j] - m), inv) : sigmoid_near(c[j]);
                c[j] = c[j] == -INFINITY ? -INFINITY : __fadd_rn(s, bias[j]);  // (absent, or not to be used whatever its bias)
            }
        }
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            if (lane + 32 * j < E) c[j] = ranked(c[j]);
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
            const unsigned value = choice_key(group_value(b1, b2, p.group_top == 2));
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
        int my_e = 0;
        unsigned key[VPL];
#pragma unroll
        for (int j = 0; j < VPL; ++j)
            key[j] = (lane + 32 * j < E && ((kept >> group[j]) & 1u)) ? choice_key(c[j]) : 0u;
        for (int s = 0; s < k; ++s) {
            unsigned best = key[0];
            int bj = 0;
#pragma unroll
            for (int j = 1; j < VPL; ++j)
                if (key[j] > best) { best = key[j]; bj = j; }     // strict: the lowest id of the lane's equals
            const unsigned most = __reduce_max_sync(0xffffffffu, best);
            const int e = best == most ? lane + 32 * bj : 0x7fffffff;
            const int e_win = __reduce_min_sync(0xffffffffu, e);
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
            s = !p.softmax ? sigmoid(l) : full_sum ? expf(l - m) / total : expf(l - m);
        }
        if (p.renormalise) {
            float sum = s + __shfl_xor_sync(0xffffffffu, s, 8);      // (the order of the four-token kernel again)
            sum = sum8(sum + __shfl_xor_sync(0xffffffffu, sum, 16));
            const float up = lift(sum);
            s = s * up * inverse(sum, up);
        }
        if (lane < k) {
            p.idx[(size_t)t * k + lane] = my_e;
            p.w[(size_t)t * k + lane] = s * p.scale;
        }
    }
}

// Four consecutive values of a row, -inf past the E-th.
template <bool VEC>
__device__ __forceinline__ void load4(const float* row, int e, int E, float (&v)[4]) {
    if (VEC) {
        const float4 f = e < E ? __ldg(reinterpret_cast<const float4*>(row + e)) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w;
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = e + j < E ? __ldg(row + e + j) : -INFINITY;
    }
}
template <bool VEC, class H>
__device__ __forceinline__ void load4(const H* row, int e, int E, float (&v)[4]) {
    if (VEC) {
        if (e < E) {
            const uint2 raw = __ldg(reinterpret_cast<const uint2*>(row + e));
            const H* h = reinterpret_cast<const H*>(&raw);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = load_f(h + j);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = -INFINITY;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = e + j < E ? load_f(row + e + j) : -INFINITY;
    }
}
template <int NI> constexpr int GATE_FLOATS = 4 * (32 * NI + MAX_K + 64);      // shared memory of a warp

// Blocks of an SM: what the registers of 4 NI values and NI maxima per thread leave room for.  (7 of the small ones, not 8:
// 32768 tokens of 128 experts 8.9 us against 10.0, 8192 of 64 3.9 against 5.1, but 40000 of 30 9.5 against 8.4; 5 for NI = 8, not 4
// or 6: 32768 tokens of 256 experts in groups 20.7 against 22.3 and 21.1.)
constexpr int gate_blocks(int NI) { return NI <= 4 ? 7 : NI <= 6 ? 6 : NI <= 8 ? 5 : NI <= 12 ? 3 : 2; }

// No groups, or groups of whole pieces of four experts: four tokens per warp.  NI pieces of four experts per lane (E <= 32 NI).
template <class L, int NI, bool VEC>
__global__ void __launch_bounds__(32 * WARPS, gate_blocks(NI))
gate_kernel(const Params p) {
    extern __shared__ __align__(16) float s_mem[];   // per warp: values [4][32 NI], chosen ids [4][MAX_K], lists [4][2][32]
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & 7, own = lane >> 3;
    const int E = p.E, k = p.k, G = p.n_groups;
    // pieces of a group, and the factor by which a piece's number gives its group (of at most 128 pieces: exact)
    const int per_group = E / G / 4, group_magic = G > 1 ? (65536 + per_group - 1) / per_group : 0;
    const bool by_score = p.bias != nullptr || (G > 1 && p.group_top == 2);
    const bool full_sum = p.softmax && (by_score || !p.renormalise);
    float* space = s_mem + (size_t)warp * GATE_FLOATS<NI>;
    float* vals = space + own * 32 * NI;
    int* chosen = reinterpret_cast<int*>(space + 4 * 32 * NI) + own * MAX_K;
    float* list = space + 4 * (32 * NI + MAX_K) + own * 64;                             // the values in reach, and their ids
    int* list_id = reinterpret_cast<int*>(list + 32);
    for (long long t0 = ((long long)blockIdx.x * WARPS + warp) * 4; t0 < p.T; t0 += (long long)gridDim.x * WARPS * 4) {
        const long long t = t0 + own < p.T ? t0 + own : p.T - 1;       // (past the end: the last token again, not written)
        const L* row = reinterpret_cast<const L*>(p.logits) + t * p.stride;
        float c[NI][4];
#pragma unroll
        for (int i = 0; i < NI; ++i) load4<VEC>(row, (sub + 8 * i) * 4, E, c[i]);
        // a finite sum of magnitudes holds no NaN and no infinity; one below LOW nothing near the lowest finite values either, so
        // that ranked() changes nothing
        constexpr float LOW = 1e38f;
        auto magnitude = [&]() {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int e = (sub + 8 * i) * 4;
                if (e + 3 < E) sum += (fabsf(c[i][0]) + fabsf(c[i][1])) + (fabsf(c[i][2]) + fabsf(c[i][3]));
                else if (!VEC) {
#pragma unroll
                    for (int j = 0; j < 3; ++j) sum += e + j < E ? fabsf(c[i][j]) : 0.f;
                }
            }
            return sum;
        };
        float size = magnitude();
        const bool finite = size < INFINITY;
        float m = -INFINITY, total = 1.f;
        if (p.softmax) {
#pragma unroll
            for (int i = 0; i < NI; ++i) m = fmaxf(m, fmaxf(fmaxf(c[i][0], c[i][1]), fmaxf(c[i][2], c[i][3])));
            m = exp_from(max8(m));
        }
        if (full_sum) {
            float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float x = expf(c[i][j] - m);
                    part[j] += x;
                    if (by_score) c[i][j] = x;
                }
            const float sum = sum8((part[0] + part[1]) + (part[2] + part[3]));
            total = sum == 0.f ? 1.f : sum;
        }
        if (by_score) {
            const float inv = 1.f / total;
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int e = (sub + 8 * i) * 4;
                float b[4];
                if (p.bias) load4<VEC>(p.bias, e, E, b);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s = p.softmax ? __fmul_rn(c[i][j], inv) : sigmoid_near(c[i][j]);
                    c[i][j] = p.bias ? __fadd_rn(s, b[j]) : s;
                }
            }
            size = magnitude();
            if (E < 32 * NI) {
#pragma unroll
                for (int i = 0; i < NI; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if ((sub + 8 * i) * 4 + j >= E) c[i][j] = -INFINITY;
            }
        }
        const bool ordinary = size < LOW && finite;
        if (!ordinary) {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int e = (sub + 8 * i) * 4;
                float l[4];
                load4<VEC>(row, e, E, l);            // (an expert masked by -inf is not to be used whatever its bias)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[i][j] = e + j >= E ? -INFINITY : ranked(l[j] == -INFINITY ? -INFINITY : c[i][j]);
                }
            }
        }
        float top[NI];                               // the largest value of each piece
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            top[i] = fmaxf(fmaxf(c[i][0], c[i][1]), fmaxf(c[i][2], c[i][3]));
            *reinterpret_cast<float4*>(vals + (sub + 8 * i) * 4) = make_float4(c[i][0], c[i][1], c[i][2], c[i][3]);
        }
        constexpr int WORDS = (NI + 7) / 8;          // of a bit per value
        unsigned dropped[WORDS] = {};                // the values in groups left out
        if (G > 1) {
            // lane sub finds the two best of groups sub, sub + 8, ... from the values in shared memory; the lanes start at
            // different pieces, so that they do not meet in a bank.  Every group's value is then compared with all others.
            __syncwarp();
            float* value = list;
            for (int g = sub; g < G; g += 8) {
                const float4* mine = reinterpret_cast<const float4*>(vals) + g * per_group;
                float b1 = -INFINITY, b2 = -INFINITY;
                int at = sub < per_group ? sub : sub % per_group;
#pragma unroll 4
                for (int it = 0; it < per_group; ++it) {
                    const float4 f = mine[at];
                    at = at + 1 == per_group ? 0 : at + 1;
                    const float h0 = fmaxf(f.x, f.y), h1 = fmaxf(f.z, f.w), h = fmaxf(h0, h1);
                    const float second = fmaxf(fminf(h0, h1), fmaxf(fminf(f.x, f.y), fminf(f.z, f.w)));
                    b2 = fmaxf(fmaxf(b2, second), fminf(b1, h));
                    b1 = fmaxf(b1, h);
                }
                value[g] = group_value(b1, b2, p.group_top == 2) + 0.f;     // (no -0)
            }
            __syncwarp();
            unsigned kept = 0u;
            for (int g = sub; g < G; g += 8) {
                const float v = value[g], below = next_below(v);
                float rank = 0.f;
#pragma unroll 4
                for (int q = 0; q < G; ++q) rank += one_if_above(value[q], q < g ? below : v);      // (of equals the lower id)
                kept |= (rank < (float)p.topk_groups ? 1u : 0u) << g;
            }
#pragma unroll
            for (int off = 1; off < 8; off <<= 1) kept |= __shfl_xor_sync(0xffffffffu, kept, off);
#pragma unroll
            for (int i = 0; i < NI; ++i)
                if (!((kept >> ((unsigned)((sub + 8 * i) * group_magic) >> 16)) & 1u)) {
                    top[i] = -INFINITY;
                    dropped[i / 8] |= 0xfu << (4 * (i % 8));
                }
        }
        __syncwarp();
        bool listed = k > 4 && k <= 16;
        if (listed) {
            float h0 = top[0], h1 = -INFINITY;       // the two largest maxima of the lane's pieces
            if (NI == 1 && h0 > -INFINITY)           // (or values of its only one)
                h1 = fmaxf(fminf(fmaxf(c[0][0], c[0][1]), fmaxf(c[0][2], c[0][3])), fmaxf(fminf(c[0][0], c[0][1]), fminf(c[0][2], c[0][3])));
#pragma unroll
            for (int i = 1; i < NI; ++i) {
                h1 = fmaxf(h1, fminf(h0, top[i]));
                h0 = fmaxf(h0, top[i]);
            }
            float above0 = 0.f, above1 = 0.f;        // how many of the sixteen are larger
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float o0 = __shfl_sync(0xffffffffu, h0, (lane & 24) + q), o1 = __shfl_sync(0xffffffffu, h1, (lane & 24) + q);
                above0 += one_if_above(o0, h0) + one_if_above(o1, h0);
                above1 += one_if_above(o0, h1) + one_if_above(o1, h1);
            }
            float reach = fminf(above0 < (float)k ? h0 : INFINITY, above1 < (float)k ? h1 : INFINITY);
#pragma unroll
            for (int off = 1; off < 8; off <<= 1) reach = fminf(reach, __shfl_xor_sync(0xffffffffu, reach, off));
            if (reach == 0.f) reach = -0.f;          // (-0 - +0 would be -0, but both zeros reach a zero: v - -0 is +0 for them)
            // bit 4 i + j of the words: value j of piece i.  The sign of a difference is shifted in, one comparison's work for
            // two; the difference of equal infinities, NaN, has none (+inf; with -inf there is no list).
            unsigned mask[WORDS];
            int mine = 0;
#pragma unroll
            for (int w = 0; w < WORDS; ++w) {
                constexpr unsigned ALL = 0xffffffffu;
                const int pieces = NI - 8 * w < 8 ? NI - 8 * w : 8;
                mask[w] = 0u;
#pragma unroll
                for (int i = 7; i >= 0; --i)
                    if (i < pieces) {
#pragma unroll
                        for (int j = 3; j >= 0; --j)
                            mask[w] = __funnelshift_l(__float_as_uint(c[(8 * w + i) % NI][j] - reach), mask[w], 1);
                    }
                mask[w] = ~mask[w] & ~dropped[w] & (ALL >> (32 - 4 * pieces));
                mine += __popc(mask[w]);
            }
            int upto = mine;
#pragma unroll
            for (int off = 1; off < 8; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, upto, off, 8);
                if (sub >= off) upto += o;
            }
            const int n = __shfl_sync(0xffffffffu, upto, lane | 7);
            const int most = __reduce_max_sync(0xffffffffu, n);
            listed = most <= 32 && reach > -INFINITY && __all_sync(0xffffffffu, n >= k);
            listed = __all_sync(0xffffffffu, listed);
            if (listed) {
                const bool keyed = sizeof(L) == 2 && !by_score && __all_sync(0xffffffffu, ordinary);
                int at = upto - mine;
#pragma unroll
                for (int w = 0; w < WORDS; ++w)
                    while (mask[w]) {
                        const int b = __ffs(mask[w]) - 1, e = (sub + 8 * (8 * w + (b >> 2))) * 4 + (b & 3);
                        mask[w] &= mask[w] - 1;
                        list[at] = keyed ? with_id(vals[e], e) : vals[e];
                        list_id[at++] = e;
                    }
                for (int q = n + sub; q < ((most + 3) & ~3); q += 8) list[q] = -INFINITY;
                __syncwarp();
                // The values alone give each its place, unless two are equal; then the places, which should be 0 .. n - 1, add
                // up to less.  Of scores of 16-bit logits without a bias some mostly are.
                bool equals = sizeof(L) == 2 && !p.bias && !keyed;
                if (!equals) {
                    float places = 0.f;
                    for (int q0 = 0; q0 < most; q0 += 16) {  // two values per lane
                        const bool is_a = q0 + sub < n, is_b = q0 + 8 + sub < n;
                        const float a = is_a ? list[q0 + sub] : INFINITY, b = is_b ? list[q0 + 8 + sub] : INFINITY;
                        float ra = 0.f, rb = 0.f;
                        for (int x = 0; x < most; x += 4) {
                            const float4 o = *reinterpret_cast<const float4*>(list + x);
                            ra += (one_if_above(o.x, a) + one_if_above(o.y, a)) + (one_if_above(o.z, a) + one_if_above(o.w, a));
                            rb += (one_if_above(o.x, b) + one_if_above(o.y, b)) + (one_if_above(o.z, b) + one_if_above(o.w, b));
                        }
                        places += ra + rb;                   // (none is above infinity)
                        if (is_a && ra < (float)k) chosen[(int)ra] = list_id[q0 + sub];
                        if (is_b && rb < (float)k) chosen[(int)rb] = list_id[q0 + 8 + sub];
                    }
                    equals = __any_sync(0xffffffffu, sum8(places) != (float)(n * (n - 1) / 2));
                }
                if (equals) {
                    __syncwarp();
                    for (int q0 = 0; q0 < most; q0 += 16) {
                        const bool is_a = q0 + sub < n, is_b = q0 + 8 + sub < n;
                        const float a = is_a ? list[q0 + sub] : INFINITY, b = is_b ? list[q0 + 8 + sub] : INFINITY;
                        const int ia = is_a ? list_id[q0 + sub] : 0, ib = is_b ? list_id[q0 + 8 + sub] : 0;
                        int ra = 0, rb = 0;
                        for (int x = 0; x < n; ++x) {
                            const float o = list[x];
                            const int io = list_id[x];
                            ra += (o > a || (o == a && io < ia)) ? 1 : 0;
                            rb += (o > b || (o == b && io < ib)) ? 1 : 0;
                        }
                        if (is_a && ra < k) chosen[ra] = ia;
                        if (is_b && rb < k) chosen[rb] = ib;
                    }
                }
            }
        }
        if (!listed) {
            for (int s = 0; s < k; ++s) {
                float mine = top[0];
#pragma unroll
                for (int i = 1; i < NI; ++i) mine = fmaxf(mine, top[i]);
                const float best = max8(mine);
                unsigned holders = (__ballot_sync(0xffffffffu, mine == best) >> (lane & 24)) & 0xffu;
                int bi = 0;
                if (mine == best) {
#pragma unroll
                    for (int i = NI - 1; i >= 0; --i)
                        if (top[i] == best) bi = i;      // the lane's lowest ids
                }
                const int piece = sub + 8 * bi;
                if (__any_sync(0xffffffffu, holders & (holders - 1))) {    // equal values in several lanes: the lowest piece
                    int low = mine == best ? piece : 0x7fffffff;
#pragma unroll
                    for (int off = 1; off < 8; off <<= 1) low = min(low, __shfl_xor_sync(0xffffffffu, low, off));
                    holders = 1u << (low & 7);
                }
                if (holders == 1u << sub) {              // this lane's piece holds it: take it out, find the piece's next
                    const float4 v = *reinterpret_cast<const float4*>(vals + piece * 4);
                    const int j = v.x == best ? 0 : v.y == best ? 1 : v.z == best ? 2 : 3;
                    vals[piece * 4 + j] = -INFINITY;
                    chosen[s] = piece * 4 + j;
                    const float a = j == 0 ? v.y : v.x, b = j <= 1 ? v.z : v.y, d = j == 3 ? v.z : v.w;
                    const float next = fmaxf(fmaxf(a, b), d);
#pragma unroll
                    for (int i = 0; i < NI; ++i)
                        if (i == bi) top[i] = next;
                }
            }
        }
        __syncwarp();
        // the chosen experts' weights, slots sub, sub + 8, ...
        float s[MAX_K / 8];
#pragma unroll
        for (int q = 0; q < MAX_K / 8; ++q) {
            s[q] = 0.f;
            if (8 * q + sub < k) {
                const float l = load_f(row + chosen[8 * q + sub]);
                s[q] = !p.softmax ? sigmoid(l) : full_sum ? expf(l - m) / total : expf(l - m);
            }
        }
        if (p.renormalise) {
            const float sum = sum8((s[0] + s[1]) + (s[2] + s[3]));
            const float up = lift(sum), inv = inverse(sum, up);
#pragma unroll
            for (int q = 0; q < MAX_K / 8; ++q) s[q] = s[q] * up * inv;
        }
#pragma unroll
        for (int q = 0; q < MAX_K / 8; ++q) {
            if (8 * q + sub < k && t0 + own < p.T) {
                p.idx[(size_t)t * k + 8 * q + sub] = chosen[8 * q + sub];
                p.w[(size_t)t * k + 8 * q + sub] = s[q] * p.scale;
            }
        }
        __syncwarp();                                // vals and chosen are rewritten by the next tokens
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
// cancellation.  Four tokens per warp, eight lanes each, as in the forward kernel; a token's row is put together in shared
// memory and written once, in 16-byte pieces.  Chosen ids outside 0 .. E-1 (routes that were dropped) have no part in it.
// NI: pieces of four experts per lane, as in the forward kernel; 0 where only the chosen experts have a gradient.
template <class L, int NI, bool VEC>
__global__ void __launch_bounds__(32 * WARPS)
gate_backward_kernel(const BwdParams p) {
    constexpr int SLOTS = MAX_K / 8;                 // of a token's k routes per lane
    extern __shared__ __align__(16) float s_row[];   // [WARPS][4][E rounded up to 8], zero between tokens
    constexpr int PER = 16 / sizeof(L);
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane & 7, own = lane >> 3;
    const int E = p.E, k = p.k, pitch = (E + 7) & ~7;
    float* mine = s_row + (warp * 4 + own) * pitch;
    // (16-byte pieces; of four experts with NI > 0)
    constexpr int PIECE = NI == 0 ? PER : 4;
    const bool vec = E % PIECE == 0 && p.d_stride % PIECE == 0 && (reinterpret_cast<uintptr_t>(p.dlogits) & (PIECE * sizeof(L) - 1)) == 0;
    for (int i = sub; i < E; i += 8) mine[i] = 0.f;
    __syncwarp();
    for (long long t0 = ((long long)blockIdx.x * WARPS + warp) * 4; t0 < p.T; t0 += (long long)gridDim.x * WARPS * 4) {
        const bool live = t0 + own < p.T;
        const long long t = live ? t0 + own : p.T - 1;
        const L* row = reinterpret_cast<const L*>(p.logits) + t * p.stride;
        L* out = reinterpret_cast<L*>(p.dlogits) + t * p.d_stride;
        int e[SLOTS];                                // slots sub, sub + 8, ...
        float g[SLOTS], l[SLOTS];
#pragma unroll
        for (int q = 0; q < SLOTS; ++q) {
            e[q] = -1;
            g[q] = l[q] = 0.f;
            if (8 * q + sub < k) {
                e[q] = p.idx[t * k + 8 * q + sub];
                g[q] = p.dw[t * k + 8 * q + sub] * p.scale;
                if ((unsigned)e[q] >= (unsigned)E) e[q] = -1;
                if (e[q] >= 0) l[q] = load_f(row + e[q]);
                else g[q] = 0.f;
            }
        }
        if constexpr (NI == 0) {
            float s[SLOTS], total = 0.f, dot = 0.f, m = -INFINITY;
            if (p.softmax) {
#pragma unroll
                for (int q = 0; q < SLOTS; ++q) m = fmaxf(m, e[q] >= 0 ? l[q] : -INFINITY);
                m = exp_from(max8(m));
            }
#pragma unroll
            for (int q = 0; q < SLOTS; ++q) {
                s[q] = 0.f;
                if (e[q] >= 0) s[q] = p.softmax ? expf(l[q] - m) : sigmoid(l[q]);
                total += s[q];
            }
            if (p.renormalise) {
                total = sum8(total);
                const float up = lift(total), inv = inverse(total, up);
#pragma unroll
                for (int q = 0; q < SLOTS; ++q) {
                    s[q] = s[q] * up * inv;
                    dot += g[q] * s[q];
                }
                dot = sum8(dot);
            }
#pragma unroll
            for (int q = 0; q < SLOTS; ++q)
                if (e[q] >= 0) mine[e[q]] = s[q] * (g[q] - dot) * (p.softmax ? 1.f : sigmoid(-l[q]));
            __syncwarp();
            if (!live) {
            } else if (vec) {
                for (int i = sub; i < E / PER; i += 8) {
                    uint4 o;
                    L* v = reinterpret_cast<L*>(&o);
#pragma unroll
                    for (int j = 0; j < PER; j += 4) {
                        const float4 f = *reinterpret_cast<const float4*>(mine + i * PER + j);
                        store_f(v + j, f.x);
                        store_f(v + j + 1, f.y);
                        store_f(v + j + 2, f.z);
                        store_f(v + j + 3, f.w);
                    }
                    __stcs(reinterpret_cast<uint4*>(out + i * PER), o);
                }
            } else {
                for (int i = sub; i < E; i += 8) store_f(out + i, mine[i]);
            }
        } else {
            // every expert: the row's exponentials stay in registers, the chosen ones' gradients wait in shared memory
            float c[NI][4], m = -INFINITY, sum = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < NI; ++i) load4<VEC>(row, (sub + 8 * i) * 4, E, c[i]);
#pragma unroll
            for (int i = 0; i < NI; ++i) m = fmaxf(m, fmaxf(fmaxf(c[i][0], c[i][1]), fmaxf(c[i][2], c[i][3])));
            m = exp_from(max8(m));
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    c[i][j] = expf(c[i][j] - m);
                    sum += c[i][j];
                }
            sum = sum8(sum);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int q = 0; q < SLOTS; ++q) {
                if (e[q] < 0) continue;
                dot += g[q] * expf(l[q] - m) * inv;
                mine[e[q]] = g[q];
            }
            dot = sum8(dot);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int at = (sub + 8 * i) * 4;
                if (!live || at >= E) continue;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = c[i][j] * inv * ((VEC || at + j < E ? mine[at + j] : 0.f) - dot);
                if (VEC && vec) {
                    struct alignas(4 * sizeof(L)) { L v[4]; } o;
#pragma unroll
                    for (int j = 0; j < 4; ++j) store_f(o.v + j, v[j]);
                    *reinterpret_cast<decltype(o)*>(out + at) = o;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at + j < E) store_f(out + at + j, v[j]);
                }
            }
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < SLOTS; ++q)
            if (e[q] >= 0) mine[e[q]] = 0.f;
        __syncwarp();
    }
}

template <class L, int NI>
static cudaError_t launch_four(const Params& p, cudaStream_t s) {
    const bool vec = p.E % 4 == 0 && (p.T == 1 || p.stride % 4 == 0) && (reinterpret_cast<uintptr_t>(p.logits) & (4 * sizeof(L) - 1)) == 0 &&
                     (reinterpret_cast<uintptr_t>(p.bias) & 15u) == 0;
    // one wave of blocks
    const long long units = ((long long)p.T + 4 * WARPS - 1) / (4 * WARPS), wave = 148 * gate_blocks(NI);
    const long long blocks = units < wave ? units : wave;
    const size_t smem = sizeof(float) * WARPS * GATE_FLOATS<NI>;
    const dim3 grid((unsigned)blocks), block(32 * WARPS);
    return vec ? launch_pdl(gate_kernel<L, NI, true>, grid, block, smem, s, p) : launch_pdl(gate_kernel<L, NI, false>, grid, block, smem, s, p);
}

template <class L>
static cudaError_t launch_gate(const Params& p, cudaStream_t s) {
    const int n = (p.E + 31) / 32;
    if (p.T > 148 * 16 && (p.n_groups == 1 || p.E / p.n_groups % 4 == 0)) {
        if (n <= 1) return launch_four<L, 1>(p, s);
        if (n <= 2) return launch_four<L, 2>(p, s);
        if (n <= 4) return launch_four<L, 4>(p, s);
        if (n <= 6) return launch_four<L, 6>(p, s);
        if (n <= 8) return launch_four<L, 8>(p, s);
        if (n <= 12) return launch_four<L, 12>(p, s);
        return launch_four<L, 16>(p, s);
    }
    long long blocks = ((long long)p.T + WARPS - 1) / WARPS;
    if (blocks > 148 * 8) blocks = 148 * 8;
    const size_t smem = sizeof(float) * WARPS * p.E;
    const dim3 grid((unsigned)blocks), block(32 * WARPS);
    if (n <= 1) return launch_pdl(gate_warp_kernel<L, 1>, grid, block, smem, s, p);
    if (n <= 2) return launch_pdl(gate_warp_kernel<L, 2>, grid, block, smem, s, p);
    if (n <= 4) return launch_pdl(gate_warp_kernel<L, 4>, grid, block, smem, s, p);
    if (n <= 8) return launch_pdl(gate_warp_kernel<L, 8>, grid, block, smem, s, p);
    return launch_pdl(gate_warp_kernel<L, 16>, grid, block, smem, s, p);
}

template <class L, int NI>
static cudaError_t launch_backward_four(const BwdParams& p, cudaStream_t s) {
    const bool vec = p.E % 4 == 0 && (p.T == 1 || p.stride % 4 == 0) && (reinterpret_cast<uintptr_t>(p.logits) & (4 * sizeof(L) - 1)) == 0;
    // A block's chain of dependent loads is its time, so the blocks are many and short.  The rows are written past the caches'
    // usual order: where they and the logits exceed L2 the next loads do not wait for them to be evicted (32768 tokens of 256
    // experts, sigmoid, inputs and outputs beyond L2: 11.1 us; two rounds of blocks and plain stores 12.0; one slot per lane for
    // small k, which leaves more room on an SM, 12.3: the next call's blocks then crowd on the SMs that are done first).
    const long long units = ((long long)p.T + 4 * WARPS - 1) / (4 * WARPS), most = 148 * 64;
    const size_t smem = sizeof(float) * WARPS * 4 * ((p.E + 7) & ~7);
    const dim3 grid((unsigned)(units < most ? units : most)), block(32 * WARPS);
    return NI > 0 && vec ? launch_pdl(gate_backward_kernel<L, NI, true>, grid, block, smem, s, p)
                         : launch_pdl(gate_backward_kernel<L, NI, false>, grid, block, smem, s, p);
}

template <class L>
static cudaError_t launch_backward(const BwdParams& p, cudaStream_t s) {
    if (!p.softmax || p.renormalise) return launch_backward_four<L, 0>(p, s);
    const int n = (p.E + 31) / 32;
    if (n <= 2) return launch_backward_four<L, 2>(p, s);
    if (n <= 4) return launch_backward_four<L, 4>(p, s);
    if (n <= 8) return launch_backward_four<L, 8>(p, s);
    return launch_backward_four<L, 16>(p, s);
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
    const DependentLaunches dependent;
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
    const DependentLaunches dependent;
    cudaError_t e = a->logits_type == MOK_TYPE_F32 ? gate::launch_backward<float>(p, s)
                    : a->logits_type == MOK_TYPE_BF16 ? gate::launch_backward<__nv_bfloat16>(p, s)
                                                      : gate::launch_backward<__half>(p, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

}  // extern "C"
