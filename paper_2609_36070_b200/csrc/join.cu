// What lies between two blocks of a network, and its gradients:
//
//   u = norm_after(y);   v = gate .* u;   sum = x + scale * drop(v);   normed = norm_before(sum)
//   norm(v) = (v - m) r w + b,   r = 1 / sqrt(mean((v - m)^2) + eps),   m = mean(v) (layer norm) or 0 (rms)
//   drop(v)[t, h] = v[t, h] / (1 - p) where word h % 4 of Philox4x32-10 (Salmon et al. 2011) of counter (h / 4, t, offset) under key
//                   `seed` is at least p 2^32 (rounded), else 0: a function of the position, so that no mask is stored
// Backwards, with n = (v - m) r and the gradient g of norm's output, the gradient of v is r (g w - mean(g w) - n mean(g w n)) (the
// first mean for layer norms only), that of w is sum_t g n and that of b sum_t g.
//
// Both are bound by the rows' bytes: x, y in, sum, normed out; backwards d_sum, d_normed, sum, y in, dx, dy out.  A row's statistics
// are found from its values in registers, so everything is read once; a row belongs to one warp or to the warps of a block, eight
// consecutive elements (16 bytes of a 16-bit type) to a thread at a time.  All arithmetic is fp32, statistics are two-pass (mean
// first), and outputs are rounded once: `normed` is made from the sum before it is rounded.
//
// Measured: rms norms, 32768 x 7168 bf16 (1.9 GB): 331 to 353 us by the box, 0.81 to 0.87 of the copy bandwidth; 16384 x 2048: 49 (0.83).  Layer norms
// with gate and dropout, 8191 x 2880 fp16: 74 us for 28.8 of bytes; bound by its instructions, 78 per element at 71 % of the issue slots.
//
// The other direction: join_backward.cu.
#include "join_common.cuh"

namespace mok {
namespace join {

// ---------------------------------------------------------------------------------------------------------------------- forward
// S: x and sum; Y: y, normed and a gate of tokens or elements.  VPT pieces of eight elements per thread.  PLAIN: rms norms without a
// bias or none, no gate, no dropout; the code for everything else would cost this, the usual case, a fifth of its instructions.
template <class S, class Y, int M, int VPT, bool PLAIN>
__global__ void __launch_bounds__(VPT == 1 ? 1024 : 512)
join_kernel(const Params p) {
    __shared__ float s_part[1][2][32][4];
    pdl_enter();
    RowSum row_sum(s_part);
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.T) return;                              // (several rows per block: a warp each, which meets no barrier)
    const int H = p.H, step = blockDim.x * 8, shift = M == SHIFTED ? shift_of(row, p.ld8) : 0, at0 = first_of<M>(threadIdx.x) - shift;
    const S* x = reinterpret_cast<const S*>(p.x) + row * p.ldx;
    const Y* y = reinterpret_cast<const Y*>(p.y) + row * p.ldy;
    // SHIFTED: a piece that reaches into the rows beside this one is read whole where the matrix goes on so far (no matrix has fewer elements
    // behind this row), and what is not the row's is masked: loads by elements would be waited for one tensor after the other
    const long long behind = (long long)(p.T - 1 - row) * H;
    auto piece = [&](const auto* base, int at) { return M == SHIFTED && behind + H - at >= 8 ? load8<PIECES>(base, at, H) : load8<M>(base, at, H); };
    // pieces past the row are 0, and take part in everything but loads and stores
    Raw<S> rx[VPT];
    Raw<Y> ry[VPT];
    bool live[VPT], whole[VPT];
    int at[VPT];                                         // (of a vector's piece to multiply zeros with: the first)
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        live[i] = at0 + i * step < H;
        whole[i] = is_whole<M>(at0 + i * step, H);
        at[i] = live[i] || M == SHIFTED ? at0 + i * step : 0;
        ry[i] = Raw<Y>();
        rx[i] = Raw<S>();
        if (live[i] && p.y) ry[i] = piece(y, at[i]);
        if (live[i] && p.x) rx[i] = piece(x, at[i]);
    }
    F8 v[VPT];
    // v becomes (v - mean) / spread
    auto normalise = [&](int norm) {
        if (!PLAIN && norm == MOK_NORM_LAYER) {
            F2 t = two(0.f);
#pragma unroll
            for (int i = 0; i < VPT; ++i) t = sum8(v[i], t);
            float s[1] = {t.lo() + t.hi()};
            row_sum.template operator()<true>(s);
            const float m = -s[0] * p.inv_h;
#pragma unroll
            for (int i = 0; i < VPT; ++i) v[i] = M == PIECES ? v[i] + two(live[i] ? m : 0.f) : within<M>(v[i] + two(m), at0 + i * step, H);
        }
        F2 t = two(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) t = dot8(v[i], v[i], t);
        float s[1] = {t.lo() + t.hi()};
        row_sum.template operator()<true>(s);
        const F2 r = two(rsqrtf(fmaf(s[0], p.inv_h, p.eps)));
#pragma unroll
        for (int i = 0; i < VPT; ++i) v[i] = v[i] * r;
    };
    auto by_vectors = [&](const void* w, const void* b) {
        if (w) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (M != SHIFTED || live[i]) v[i] = v[i] * vector8<M>(w, p.vector_type, at[i], H);
        }
        if (!PLAIN && b) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (live[i]) v[i] = v[i] + vector8<M>(b, p.vector_type, at[i], H);
        }
    };
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        v[i] = widen(ry[i]);
        if (M == SHIFTED && !whole[i]) v[i] = within<M>(v[i], at0 + i * step, H);
    }
    if (p.y) {
        if (p.after != MOK_NORM_NONE) {
            normalise(p.after);
            by_vectors(p.after_w, p.after_b);
        }
        if (!PLAIN) {
            if (p.gate_kind == MOK_JOIN_GATE_CHANNEL) {
                by_vectors(p.gate, nullptr);
            } else if (p.gate_kind == MOK_JOIN_GATE_TOKEN) {
                const F2 g = two(to_f(reinterpret_cast<const Y*>(p.gate)[row * p.ldg]));
#pragma unroll
                for (int i = 0; i < VPT; ++i) v[i] = v[i] * g;
            } else if (p.gate_kind == MOK_JOIN_GATE_FULL) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) v[i] = v[i] * widen(load8<M>(reinterpret_cast<const Y*>(p.gate) + row * p.ldg, at[i], H));
            }
            if (p.drop) {
                const Drop drop(p);
#pragma unroll
                for (int i = 0; i < VPT; ++i) v[i] = drop.template apply<M>(v[i], (int)row, at0 + i * step);
            }
        }
    }
    const F2 scale = two(p.scale);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        v[i] = fma8(v[i], scale, widen(rx[i]));
        // (a bias or NaN in the padding of the last piece)
        if (M == ELEMENTS || (M == SHIFTED && !whole[i])) v[i] = within<M>(v[i], at0 + i * step, H);
        if (p.sum && live[i]) store8<M>(reinterpret_cast<S*>(p.sum) + row * p.ld_sum, at[i], H, v[i]);
    }
    if (p.before == MOK_NORM_NONE) return;
    if (M == PIECES && (!PLAIN || p.after_w)) {                  // (a NaN or infinity in a vector, times the zeros of a piece past the row)
#pragma unroll
        for (int i = 0; i < VPT; ++i)
            if (!live[i]) v[i] = zeros();
    }
    normalise(p.before);
    by_vectors(p.before_w, p.before_b);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
        if (live[i]) store8<M>(reinterpret_cast<Y*>(p.normed) + row * p.ld_normed, at[i], H, v[i]);
}

// ------------------------------------------------------------------------------------------------------------------- host side
static bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
template <class S, class Y, int M, int VPT>
static cudaError_t launch_rows(const Params& p, cudaStream_t s) {
    const int pieces = (p.H + (M == SHIFTED ? 14 : 7)) / 8, threads = (pieces + 32 * VPT - 1) / (32 * VPT) * 32, rows = threads == 32 ? 4 : 1;
    const dim3 grid((unsigned)((p.T + rows - 1) / rows)), block(threads, rows);
    if constexpr (M != SHIFTED)
        if (!plain(p)) return launch_pdl(join_kernel<S, Y, M, VPT, false>, grid, block, 0, s, p);
    return launch_pdl(join_kernel<S, Y, M, VPT, true>, grid, block, 0, s, p);
}
// How many pieces a thread holds (us; 2^25 elements, bf16; plain: rms norms, else layer norms with gate and dropout):
//   few rows, or rows of up to 256 elements: one, for the shortest time of a row (65536 x 256: 26 against 33 with two, else 49 against 72)
//   rows of one warp, and of three: as many as they need (65536 x 512, two: 45, one: 72; 43690 x 768, plain, four: 51, two: 59;
//   43747 x 767, else, one: 166, two: 213)
//   plain: four where they leave no more than an eighth of the places empty (4096 x 8192: 54 against 61, 8192 x 4096: 51 against 55), else two
//   (21845 x 1536: 50 against 56)
//   else two, for the sake of more warps (4681 x 7168: 125 against 150 with four, 198 with one)
template <class S, class Y, int M>
static cudaError_t launch_forward(const Params& p, cudaStream_t s) {
    if (p.T <= 592 || p.H <= 256) return launch_rows<S, Y, M, 1>(p, s);
    if constexpr (M == PIECES) {
        const int pieces = p.H / 8, places = (pieces + 127) / 128 * 128;
        if (plain(p) && p.H > 512 && (pieces <= 128 || 8 * pieces >= 7 * places)) return launch_rows<S, Y, M, 4>(p, s);
    }
    if ((M == ELEMENTS || (M == PIECES && !plain(p))) && p.H > 512 && p.H <= 768) return launch_rows<S, Y, M, 1>(p, s);
    return launch_rows<S, Y, M, 2>(p, s);
}
// The arguments that both directions share.
static int common(const mok_join_args* a, Params* p) {
    const bool stream_ok = a->x_type == a->type || a->x_type == MOK_TYPE_F32;
    if (a->T < 0 || a->H < 1 || a->H > MAX_H || !i8::type_ok(a->type) || !i8::type_ok(a->x_type) || !stream_ok || !i8::type_ok(a->vector_type) ||
        a->before < MOK_NORM_NONE || a->before > MOK_NORM_LAYER || a->after < MOK_NORM_NONE || a->after > MOK_NORM_LAYER ||
        a->gate_kind < MOK_JOIN_GATE_NONE || a->gate_kind > MOK_JOIN_GATE_FULL || !(a->p >= 0.0 && a->p <= 1.0) || !(a->eps >= 0.f))
        return MOK_ERR_SHAPE;
    const bool rows = a->T > 1;
    if (rows && ((a->x && a->x_stride < a->H) || (a->y && a->y_stride < a->H) || (a->gate_kind == MOK_JOIN_GATE_FULL && a->gate_stride < a->H) ||
                 (a->gate_kind == MOK_JOIN_GATE_TOKEN && a->gate_stride < 1)))
        return MOK_ERR_SHAPE;
    const size_t tb = i8::type_bytes(a->type), xb = i8::type_bytes(a->x_type), vb = i8::type_bytes(a->vector_type);
    if (!aligned(a->x, xb) || !aligned(a->y, tb) || !aligned(a->gate, a->gate_kind == MOK_JOIN_GATE_CHANNEL ? vb : tb) || !aligned(a->before_weight, vb) ||
        !aligned(a->before_bias, vb) || !aligned(a->after_weight, vb) || !aligned(a->after_bias, vb) || !aligned(a->seed_at, 8))
        return MOK_ERR_ALIGN;
    *p = Params();
    p->x = a->x;
    p->y = a->y;
    p->gate = a->gate_kind ? a->gate : nullptr;
    p->before_w = a->before ? a->before_weight : nullptr;
    p->before_b = a->before ? a->before_bias : nullptr;
    p->after_w = a->after ? a->after_weight : nullptr;
    p->after_b = a->after ? a->after_bias : nullptr;
    p->ldx = a->x_stride;
    p->ldy = a->y_stride;
    p->ldg = a->gate_stride;
    p->T = a->T;
    p->H = a->H;
    p->before = a->before;
    p->after = a->after;
    p->gate_kind = a->gate_kind;
    p->vector_type = a->vector_type;
    p->scale = a->scale;
    p->eps = a->eps;
    p->inv_h = (float)(1.0 / a->H);
    const double border = a->p * 4294967296.0 + 0.5;
    p->drop = a->p <= 0.0 ? 0 : border >= 4294967296.0 ? 2 : 1;
    p->threshold = p->drop == 1 ? (uint32_t)border : 0u;
    p->keep = a->p < 1.0 ? (float)(1.0 / (1.0 - a->p)) : 0.f;
    p->seed = a->seed;
    p->offset = a->offset;
    p->seed_at = reinterpret_cast<const unsigned long long*>(a->seed_at);
    return MOK_OK;
}
// How the rows of a call's matrices lie: whole 16-byte pieces in all of them, or all shifted alike, or neither.
struct Rows {
    int T, H, ld8;                                       // ld8: the rows' distance modulo 8 elements; -1: not known yet
    bool pieces, shifted;
    Rows(int t, int h) : T(t), H(h), ld8(t > 1 ? -1 : 0), pieces(h % 8 == 0), shifted(h <= MAX_H - 7) {}
    void matrix(const void* p, long long stride, size_t size) {
        if (!p) return;
        pieces = pieces && aligned(p, 16) && (T <= 1 || stride * (long long)size % 16 == 0);
        const int mod = (int)(stride & 7);
        if (T > 1 && ld8 < 0) ld8 = mod;
        shifted = shifted && aligned(p, 8 * size) && (T <= 1 || mod == ld8);
    }
    void vector(const void* p) {
        pieces = pieces && aligned(p, 16);
        shifted = shifted && aligned(p, 16);
    }
    Layout layout() const { return pieces ? PIECES : shifted ? SHIFTED : ELEMENTS; }
};
static Rows common_rows(const mok_join_args* a) {
    const size_t tb = i8::type_bytes(a->type), xb = i8::type_bytes(a->x_type);
    Rows r(a->T, a->H);
    r.matrix(a->x, a->x_stride, xb);
    r.matrix(a->y, a->y_stride, tb);
    if (a->gate_kind == MOK_JOIN_GATE_FULL) r.matrix(a->gate, a->gate_stride, tb);
    if (a->gate_kind == MOK_JOIN_GATE_CHANNEL) r.vector(a->gate);
    for (const void* v : {a->before_weight, a->before_bias, a->after_weight, a->after_bias}) r.vector(v);
    return r;
}
}  // namespace join
}  // namespace mok

using namespace mok;

extern "C" {

int mok_block_join(const mok_join_args* a) {
    if (!a) return MOK_ERR_NULL;
    join::Params p;
    const int status = join::common(a, &p);
    if (status != MOK_OK) return status;
    if (a->T > 1 && ((a->sum && a->sum_stride < a->H) || (a->before && a->normed_stride < a->H))) return MOK_ERR_SHAPE;
    if (a->T == 0) return MOK_OK;
    // without y the sum is x, which need not be written again
    if ((!a->x && !a->y) || (a->y && !a->sum) || (a->before && !a->normed) || (a->gate_kind && a->y && !a->gate)) return MOK_ERR_NULL;
    const size_t tb = i8::type_bytes(a->type), xb = i8::type_bytes(a->x_type);
    if (!join::aligned(a->sum, xb) || !join::aligned(a->normed, tb)) return MOK_ERR_ALIGN;
    p.sum = a->sum;
    p.normed = a->normed;
    p.ld_sum = a->sum_stride;
    p.ld_normed = a->normed_stride;
    join::Rows r = join::common_rows(a);
    r.matrix(a->sum, a->sum_stride, xb);
    r.matrix(a->normed, a->normed_stride, tb);
    join::Layout layout = r.layout();
    // Shifted pieces, beside elements: rms norms of 11646 x 2881 75 against 88 us, 4193 x 8001 83 against 106, 33520 x 1001 82 against 81.
    // There is no such form of the rest, whose instructions count more than its accesses.
    if (layout == join::SHIFTED && !(join::plain(p) && a->H > 1024)) layout = join::ELEMENTS;
    p.ld8 = r.ld8;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    const DependentLaunches dependent;
    const cudaError_t e = join::by_type(a->x_type, a->type, [&](auto x, auto y) {
        using S = decltype(x);
        using Y = decltype(y);
        return layout == join::PIECES    ? join::launch_forward<S, Y, join::PIECES>(p, s)
               : layout == join::SHIFTED ? join::launch_forward<S, Y, join::SHIFTED>(p, s)
                                         : join::launch_forward<S, Y, join::ELEMENTS>(p, s);
    });
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

size_t mok_join_bwd_workspace_bytes(int T, int H) {
    if (T < 0 || H < 1 || H > join::MAX_H) return 0;
    const int blocks = T < 1 ? 1 : T < 148 ? T : 148;    // (at most: several rows may share a block)
    return align_up((size_t)5 * blocks * H * sizeof(float), 256);
}

int mok_block_join_backward(const mok_join_bwd_args* b) {
    if (!b) return MOK_ERR_NULL;
    const mok_join_args* a = &b->forward;
    join::Params p;
    const int status = join::common(a, &p);
    if (status != MOK_OK) return status;
    if (a->T > 1 && ((b->d_sum && b->d_sum_stride < a->H) || (a->before && b->d_normed_stride < a->H) || (b->dx && b->dx_stride < a->H) ||
                     (b->dy && b->dy_stride < a->H) || (b->dgate && a->gate_kind == MOK_JOIN_GATE_FULL && b->dgate_stride < a->H) ||
                     (b->dgate && a->gate_kind == MOK_JOIN_GATE_TOKEN && b->dgate_stride < 1)))
        return MOK_ERR_SHAPE;
    float* const vectors[5] = {a->before ? b->d_before_weight : nullptr, a->after ? b->d_after_weight : nullptr, a->before ? b->d_before_bias : nullptr,
                               a->after ? b->d_after_bias : nullptr,
                               a->gate_kind == MOK_JOIN_GATE_CHANNEL ? reinterpret_cast<float*>(b->dgate) : nullptr};
    const bool of_y = b->dy || b->dgate || vectors[1] || vectors[3];
    const size_t tb = i8::type_bytes(a->type), xb = i8::type_bytes(a->x_type);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(b->stream);
    if (a->T == 0) {                                     // no rows: the sums over them are 0
        for (float* v : vectors)
            if (v) {
                const cudaError_t e = cudaMemsetAsync(v, 0, (size_t)a->H * sizeof(float), s);
                if (e != cudaSuccess) return cuda_fail(e);
            }
        return MOK_OK;
    }
    if ((!b->d_sum && !a->before) || (a->before && (!b->d_normed || !a->x)) || (of_y && a->after && !a->y) ||
        (of_y && a->gate_kind && (!a->gate || (b->dgate && !a->y))))
        return MOK_ERR_NULL;
    if (!join::aligned(b->d_sum, xb) || !join::aligned(b->d_normed, tb) || !join::aligned(b->dx, xb) || !join::aligned(b->dy, tb) ||
        !join::aligned(b->dgate, a->gate_kind == MOK_JOIN_GATE_CHANNEL ? 4 : tb) || !join::aligned(b->d_before_weight, 4) ||
        !join::aligned(b->d_before_bias, 4) || !join::aligned(b->d_after_weight, 4) || !join::aligned(b->d_after_bias, 4))
        return MOK_ERR_ALIGN;
    if (!of_y) {                                         // nothing of y is wanted, so nothing of it is read
        p.after = MOK_NORM_NONE;
        p.gate_kind = MOK_JOIN_GATE_NONE;
    }
    if (!a->y && p.after == MOK_NORM_NONE && !b->dgate) p.y = nullptr;
    p.d_sum = b->d_sum;
    p.ld_dsum = b->d_sum_stride;
    p.d_normed = b->d_normed;
    p.ld_dnormed = b->d_normed_stride;
    p.sum = b->dx;
    p.ld_sum = b->dx_stride;
    p.dy = b->dy;
    p.ld_dy = b->dy_stride;
    p.dgate = a->gate_kind == MOK_JOIN_GATE_CHANNEL ? nullptr : b->dgate;
    p.ld_dgate = b->dgate_stride;
    join::Finish f = {};
    int n = 0;
    for (int i = 0; i < 5; ++i) {
        p.slot[i] = vectors[i] ? n : -1;
        if (vectors[i]) f.out[n++] = vectors[i];
    }
    if (n) {
        if (!b->workspace || !join::aligned(b->workspace, 256) || b->workspace_bytes < mok_join_bwd_workspace_bytes(a->T, a->H)) return MOK_ERR_WORKSPACE;
        p.partial = reinterpret_cast<float*>(b->workspace);
    }
    join::Rows r = join::common_rows(a);
    r.matrix(b->d_sum, b->d_sum_stride, xb);
    r.matrix(b->d_normed, b->d_normed_stride, tb);
    r.matrix(b->dx, b->dx_stride, xb);
    r.matrix(b->dy, b->dy_stride, tb);
    if (a->gate_kind == MOK_JOIN_GATE_FULL) r.matrix(b->dgate, b->dgate_stride, tb);
    p.ld8 = r.ld8;
    const DependentLaunches dependent;
    const cudaError_t e = join::launch_backward(p, a->x_type, a->type, r.layout(), f, n, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

}  // extern "C"
