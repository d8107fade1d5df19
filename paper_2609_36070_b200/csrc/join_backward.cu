// The gradients of the join between two blocks (join.cu has the formulas).
//
// The backward kernel's blocks stay for many rows: the sums over tokens (the gradients of the norms' weights) are kept in registers
// by the thread that owns the columns (those of biases and of a channel gate, which are rarer, in shared memory), written once per
// block and added up by a second kernel, in a fixed order.  A row passes through two block-wide sums one after the other (three with a
// layer norm), so the next rows are on their way meanwhile: each thread copies its own pieces asynchronously into shared memory, two or
// more rows ahead, and needs no barrier to read them.
//
// Measured: rms norms, 32768 x 7168 bf16 (2.8 GB): 558 to 583 us by the box, 0.75 of the copy bandwidth, and 16384 x 2880: 130 us; bound by the
// chain of a row's two sums at 16 warps per SM (128 registers, of which two norms spill 4 to 40 bytes; more rows at once would spill more).
// Layer norms with biases, gate and dropout, 8192 x 2880: 178 us for 57.6 of bytes; bound by its instructions, 170 per element at 65 % of the
// issue slots, of which the row sums are an eighth and the generator a tenth.  The 896 threads that a block of one piece per thread may
// have leave 72 registers: it spills 44 to 60 bytes, by elements 216 to 232.
#include "join_common.cuh"

namespace mok {
namespace join {

// --------------------------------------------------------------------------------------------------------------------- backward
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// the first `bytes` of it, and zeros
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// Piece `at` of a row to shared memory.  SHIFTED: not what lies behind the row, while the elements in front of it (those of the row before,
// in the same buffer: a row that begins at the buffer's start has no shift) are copied and have to be masked.
template <int M, class T>
__device__ __forceinline__ void copy_piece(uint32_t dst, const T* src, int at, int H) {
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q) {
        constexpr int per = 16 / sizeof(T);
        if (M == SHIFTED) copy16(dst + q * 16, src + q * per, (uint32_t)(min(max(H - at - q * per, 0), per) * (int)sizeof(T)));
        else copy16(dst + q * 16, src + q * per);
    }
}
// Threads of a block, by the pieces of eight elements that a thread holds of a row.
constexpr int back_threads(int vpt) { return vpt == 1 ? 896 : 512; }

// A block's sums over its rows to memory: one row's threads after the other's where it has several.  In shared memory a row of sums is
// `wide` numbers (SHIFTED: from where the thread's first piece begins; the shift is the same in all rows that a thread meets).
template <int VPT, int M>
__device__ __forceinline__ void block_sums(const Params& p, const F8 (&sum_before)[VPT], const F8 (&sum_after)[VPT], char* s_mem) {
    const int H = p.H, step = blockDim.x * 8, at0 = first_of<M>(threadIdx.x), wide = M == SHIFTED ? step * VPT : H;
    const bool direct = M != SHIFTED && blockDim.y == 1;
    float* sums = reinterpret_cast<float*>(s_mem);
    for (int a = 0; a < 5; ++a) {
        if (p.slot[a] < 0) continue;
        float* out = p.partial + ((size_t)p.slot[a] * gridDim.x + blockIdx.x) * H;
        if (a < 2) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (M == SHIFTED) store8<PIECES>(sums + threadIdx.y * wide, at0 + i * step, wide, a == 0 ? sum_before[i] : sum_after[i]);
                else if (at0 + i * step < H) store8<M>(direct ? out : sums + threadIdx.y * H, at0 + i * step, H, a == 0 ? sum_before[i] : sum_after[i]);
            if (direct) continue;
        }
        __syncthreads();
        const float* in = a < 2 ? sums : reinterpret_cast<const float*>(s_mem + p.at_acc[a - 2]);
        for (int at = threadIdx.y * blockDim.x + threadIdx.x; at < H; at += blockDim.x * blockDim.y) {
            float v = 0.f;
            for (int w = 0; w < (int)blockDim.y; ++w)
                v += in[w * wide + at + (M == SHIFTED ? shift_of((long long)blockIdx.x * blockDim.y + w, p.ld8) : 0)];
            out[at] = v;
        }
    }
}
// A vector of the columns into shared memory, in fp32, zeros past the H-th; `otherwise` where there is none.  All threads of the block.
__device__ __forceinline__ void hold_vector(float* to, const void* from, int type, int H, int wide, float otherwise) {
    for (int c = (threadIdx.y * blockDim.x + threadIdx.x) * 8; c < wide; c += blockDim.x * blockDim.y * 8) {
        const F8 other = {two(otherwise), two(otherwise), two(otherwise), two(otherwise)};
        store8<PIECES>(to, c, wide, c >= H ? zeros() : from ? vector8<PIECES>(from, type, c, H) : other);
    }
}
// SHIFTED: every row of threads has its own, in the same place as its pieces.
__device__ __forceinline__ void hold_shifted(float* to, const void* from, int type, int H, int wide, int shift, float otherwise) {
    const F8 other = {two(otherwise), two(otherwise), two(otherwise), two(otherwise)};
    for (int c = threadIdx.x * 8; c < wide; c += blockDim.x * 8)
        store8<PIECES>(to + threadIdx.y * wide, c, wide, c - shift >= H ? zeros() : from ? vector8<SHIFTED>(from, type, c - shift, H) : other);
}

// A piece that begins at `to`, element `at` of its row
template <int M, class T>
__device__ __forceinline__ void store_piece(T* to, bool whole, int at, int H, const F8& v) {
    if (M == PIECES || whole) store8<PIECES>(to, 0, 8, v);
    else store8<SHIFTED>(to - at, at, H, v);
}

// The usual case: rms norms without a bias, or none; no gate, no dropout; rows of whole pieces.  Since n = v r, the mean of g w n is r
// times that of g w v, so the statistics and that mean are one block-wide sum, and a row passes through two of them.  The norms' weights
// lie in shared memory in fp32, in front of the ring.
template <class S, class Y, int M, bool BEFORE, bool AFTER, int VPT>
__global__ void __launch_bounds__(back_threads(VPT))
join_backward_plain_kernel(const Params p) {
    extern __shared__ __align__(16) char s_mem[];
    __shared__ float s_part[MAX_ROWS][2][32][4];
    pdl_enter();
    RowSum row_sum(s_part);
    // in shared memory rows are `wide` elements long: pieces past the row's H are zeros, and take part in everything but copies and stores
    const int H = p.H, step = blockDim.x * 8, at0 = threadIdx.x * 8, wide = step * VPT;
    const long long first = (long long)blockIdx.x * blockDim.y + threadIdx.y, stride = (long long)gridDim.x * blockDim.y;
    const int shift = M == SHIFTED ? shift_of(first, p.ld8) : 0;         // (at0 counts from where the first piece begins)
    float *wb = reinterpret_cast<float*>(s_mem + p.at_before_w), *wa = reinterpret_cast<float*>(s_mem + p.at_after_w);
    char* mine = s_mem + p.at_ring + (size_t)threadIdx.y * p.stages * p.stage_bytes;
    if (M == SHIFTED) {
        if (BEFORE) hold_shifted(wb, p.before_w, p.vector_type, H, wide, shift, 1.f);
        if (AFTER) hold_shifted(wa, p.after_w, p.vector_type, H, wide, shift, 1.f);
    } else {
        if (BEFORE) hold_vector(wb, p.before_w, p.vector_type, H, wide, 1.f);
        if (AFTER) hold_vector(wa, p.after_w, p.vector_type, H, wide, 1.f);
    }
    wb += at0 + (M == SHIFTED ? threadIdx.y * wide : 0);
    wa += at0 + (M == SHIFTED ? threadIdx.y * wide : 0);
    bool live[VPT], whole[VPT];
    F8 sum_before[VPT], sum_after[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = at0 + i * step;
        live[i] = at - shift < H;
        whole[i] = is_whole<M>(at - shift, H);
        sum_before[i] = sum_after[i] = zeros();
        if (!live[i])
            for (int q = 0; q < p.stages; ++q) {
                char* to = mine + q * p.stage_bytes;
                if (BEFORE) store8<PIECES>(reinterpret_cast<S*>(to + p.at_x), at, H, zeros());
                if (BEFORE) store8<PIECES>(reinterpret_cast<Y*>(to + p.at_dnormed), at, H, zeros());
                if (AFTER) store8<PIECES>(reinterpret_cast<Y*>(to + p.at_y), at, H, zeros());
                store8<PIECES>(reinterpret_cast<S*>(to + p.at_dsum), at, H, zeros());
            }
    }
    __syncthreads();
    // this thread's pieces of the next row to be copied, and where they go; a group per row, empty past the last one
    const S *x = reinterpret_cast<const S*>(p.x) + first * p.ldx + at0 - shift, *dsum = reinterpret_cast<const S*>(p.d_sum) + first * p.ld_dsum + at0 - shift;
    const Y *dn = reinterpret_cast<const Y*>(p.d_normed) + first * p.ld_dnormed + at0 - shift, *yy = reinterpret_cast<const Y*>(p.y) + first * p.ldy + at0 - shift;
    const long long x_step = stride * p.ldx, dsum_step = stride * p.ld_dsum, dn_step = stride * p.ld_dnormed, y_step = stride * p.ldy;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(mine);
    const uint32_t to_x = ring + p.at_x + at0 * sizeof(S), to_dsum = ring + p.at_dsum + at0 * sizeof(S), to_dn = ring + p.at_dnormed + at0 * sizeof(Y),
                   to_y = ring + p.at_y + at0 * sizeof(Y);
    long long ahead = first;
    auto copy = [&](int stage) {
        if (ahead < p.T) {
            const uint32_t off = stage * p.stage_bytes;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                if (!live[i]) continue;
                const int at = at0 + i * step - shift;
                if (BEFORE) copy_piece<M>(to_x + off + i * step * sizeof(S), x + i * step, at, H);
                copy_piece<M>(to_dsum + off + i * step * sizeof(S), dsum + i * step, at, H);
                if (BEFORE) copy_piece<M>(to_dn + off + i * step * sizeof(Y), dn + i * step, at, H);
                if (AFTER) copy_piece<M>(to_y + off + i * step * sizeof(Y), yy + i * step, at, H);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        x += x_step;
        dsum += dsum_step;
        dn += dn_step;
        yy += y_step;
        ahead += stride;
    };
    S* dx = reinterpret_cast<S*>(p.sum) + first * p.ld_sum + at0 - shift;
    Y* dy = reinterpret_cast<Y*>(p.dy) + first * p.ld_dy + at0 - shift;
    const long long dx_step = stride * p.ld_sum, dy_step = stride * p.ld_dy;
    const F2 scale = two(p.scale);
    int stage = 0;
    for (int i = 0; i + 1 < p.stages; ++i) copy(i);
    for (long long row = first; row < p.T; row += stride) {
        copy(stage == 0 ? p.stages - 1 : stage - 1);
        if (p.stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else if (p.stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 3;" ::: "memory");
        const char* held = mine + stage * p.stage_bytes;
        const S *hx = reinterpret_cast<const S*>(held + p.at_x) + at0, *hd = reinterpret_cast<const S*>(held + p.at_dsum) + at0;
        const Y *hn = reinterpret_cast<const Y*>(held + p.at_dnormed) + at0, *hy = reinterpret_cast<const Y*>(held + p.at_y) + at0;
        F8 v[VPT], y[VPT], d[VPT];
        F2 a = two(0.f), b = two(0.f), c = two(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            if (BEFORE) {
                v[i] = widen(load8<PIECES>(hx, i * step, H));
                d[i] = widen(load8<PIECES>(hn, i * step, H));
                if (M == SHIFTED && !whole[i]) {
                    v[i] = within<M>(v[i], at0 + i * step - shift, H);
                    d[i] = within<M>(d[i], at0 + i * step - shift, H);
                }
                a = dot8(v[i], v[i], a);
                c = dot8(d[i] * widen(load8<PIECES>(wb, i * step, H)), v[i], c);
            }
            if (AFTER) {
                y[i] = widen(load8<PIECES>(hy, i * step, H));
                if (M == SHIFTED && !whole[i]) y[i] = within<M>(y[i], at0 + i * step - shift, H);
                b = dot8(y[i], y[i], b);
            }
        }
        float r0 = 1.f, r1 = 1.f, mean = 0.f;
        if constexpr (BEFORE && AFTER) {
            float t[3] = {a.lo() + a.hi(), c.lo() + c.hi(), b.lo() + b.hi()};
            row_sum(t);
            r0 = rsqrtf(fmaf(t[0], p.inv_h, p.eps));
            r1 = rsqrtf(fmaf(t[2], p.inv_h, p.eps));
            mean = -t[1] * r0 * p.inv_h;
        } else if constexpr (BEFORE) {
            float t[2] = {a.lo() + a.hi(), c.lo() + c.hi()};
            row_sum(t);
            r0 = rsqrtf(fmaf(t[0], p.inv_h, p.eps));
            mean = -t[1] * r0 * p.inv_h;
        } else if constexpr (AFTER) {
            float t[1] = {b.lo() + b.hi()};
            row_sum(t);
            r1 = rsqrtf(fmaf(t[0], p.inv_h, p.eps));
        }
        a = two(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            F8 direct = widen(load8<PIECES>(hd, i * step, H));
            if (M == SHIFTED && !whole[i]) direct = within<M>(direct, at0 + i * step - shift, H);
            if (BEFORE) {
                v[i] = v[i] * two(r0);                   // n
                sum_before[i] = fma8(d[i], v[i], sum_before[i]);
                d[i] = fma8(fma8(v[i], two(mean), d[i] * widen(load8<PIECES>(wb, i * step, H))), two(r0), direct);
            } else {
                d[i] = direct;
            }
            if (live[i]) store_piece<M>(dx + i * step, whole[i], at0 + i * step - shift, H, d[i]);
            d[i] = d[i] * scale;
            if (AFTER) {
                y[i] = y[i] * two(r1);
                sum_after[i] = fma8(d[i], y[i], sum_after[i]);
                d[i] = d[i] * widen(load8<PIECES>(wa, i * step, H));
                a = dot8(d[i], y[i], a);
            }
        }
        if (AFTER) {
            float u[1] = {a.lo() + a.hi()};
            row_sum(u);
            const F2 m = two(-u[0] * p.inv_h);
#pragma unroll
            for (int i = 0; i < VPT; ++i) d[i] = fma8(y[i], m, d[i]) * two(r1);
        }
        if (p.dy) {
#pragma unroll
            for (int i = 0; i < VPT; ++i)
                if (live[i]) store_piece<M>(dy + i * step, whole[i], at0 + i * step - shift, H, d[i]);
        }
        dx += dx_step;
        dy += dy_step;
        stage = stage + 1 == p.stages ? 0 : stage + 1;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    block_sums<VPT, M>(p, sum_before, sum_after, s_mem);
}

#define MOK_EACH_PIECE _Pragma("unroll") for (int i = 0; i < VPT; ++i)
// Everything else.  RING: rows come through shared memory, as above, and the vectors lie there; otherwise (rows that are no whole pieces,
// or too much of all that) both are read from memory where they are needed.
template <class S, class Y, int M, bool RING, int VPT>
__global__ void __launch_bounds__(back_threads(VPT))
join_backward_kernel(const Params p) {
    extern __shared__ __align__(16) char s_mem[];
    __shared__ float s_part[MAX_ROWS][2][32][4];
    pdl_enter();
    RowSum row_sum(s_part);
    const int H = p.H, step = blockDim.x * 8, at0 = first_of<M>(threadIdx.x), wide = step * VPT;
    const long long first = (long long)blockIdx.x * blockDim.y + threadIdx.y, stride = (long long)gridDim.x * blockDim.y;
    const bool before = p.before != MOK_NORM_NONE, after = p.after != MOK_NORM_NONE, layer_before = p.before == MOK_NORM_LAYER,
               layer_after = p.after == MOK_NORM_LAYER, full = p.gate_kind == MOK_JOIN_GATE_FULL;
    const bool of_y = p.dy || p.dgate || p.slot[1] >= 0 || p.slot[3] >= 0 || p.slot[4] >= 0;
    char* mine = s_mem + p.at_ring + (RING ? (size_t)threadIdx.y * p.stages * p.stage_bytes : 0);
    if (RING) {
        if (p.at_before_w >= 0) hold_vector(reinterpret_cast<float*>(s_mem + p.at_before_w), p.before_w, p.vector_type, H, wide, 1.f);
        if (p.at_after_w >= 0) hold_vector(reinterpret_cast<float*>(s_mem + p.at_after_w), p.after_w, p.vector_type, H, wide, 1.f);
        if (p.at_after_b >= 0) hold_vector(reinterpret_cast<float*>(s_mem + p.at_after_b), p.after_b, p.vector_type, H, wide, 0.f);
        if (p.at_channel >= 0) hold_vector(reinterpret_cast<float*>(s_mem + p.at_channel), p.gate, p.vector_type, H, wide, 1.f);
    }
    bool live[VPT];
    F8 sum_before[VPT], sum_after[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int at = at0 + i * step;
        live[i] = at < H;
        sum_before[i] = sum_after[i] = zeros();
        if (RING && !live[i])
            for (int q = 0; q < p.stages; ++q) {
                char* to = mine + q * p.stage_bytes;
                if (p.at_x >= 0) store8<PIECES>(reinterpret_cast<S*>(to + p.at_x), at, H, zeros());
                if (p.at_dsum >= 0) store8<PIECES>(reinterpret_cast<S*>(to + p.at_dsum), at, H, zeros());
                if (p.at_dnormed >= 0) store8<PIECES>(reinterpret_cast<Y*>(to + p.at_dnormed), at, H, zeros());
                if (p.at_y >= 0) store8<PIECES>(reinterpret_cast<Y*>(to + p.at_y), at, H, zeros());
                if (p.at_gate >= 0) store8<PIECES>(reinterpret_cast<Y*>(to + p.at_gate), at, H, zeros());
            }
        for (int a = 0; a < 3; ++a)
            if (live[i] && p.at_acc[a] >= 0) store8<M>(reinterpret_cast<float*>(s_mem + p.at_acc[a]) + threadIdx.y * H, at, H, zeros());
    }
    __syncthreads();
    auto add_extra = [&](int a, int at, const F8& v) {
        if (at >= H) return;
        float* to = reinterpret_cast<float*>(s_mem + p.at_acc[a]) + threadIdx.y * H;
        store8<M>(to, at, H, widen(load8<M>(to, at, H)) + v);
    };
    auto vector = [&](int where, const void* from, int at) {
        return RING ? widen(load8<PIECES>(reinterpret_cast<const float*>(s_mem + where), at, H)) : vector8<M>(from, p.vector_type, at < H ? at : 0, H);
    };
    // one row's pieces of this thread into a stage; a group per row, empty past the last one.  (Addresses are made anew for every row:
    // five pointers to be kept would cost registers that the sums need.)
    auto copy = [&](long long row, int stage) {
        if (row < p.T) {
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(mine) + stage * p.stage_bytes;
            auto tensor = [&](int where, const auto* base, long long ld) {
                if (where < 0) return;
                constexpr int size = sizeof(*base);
                const auto* from = base + row * ld + at0;
#pragma unroll
                for (int i = 0; i < VPT; ++i)
                    if (live[i]) {
#pragma unroll
                        for (int q = 0; q < size / 2; ++q) copy16(to + where + (at0 + i * step) * size + q * 16, from + i * step + q * 4);
                    }
            };
            tensor(p.at_x, reinterpret_cast<const S*>(p.x), p.ldx);
            tensor(p.at_dsum, reinterpret_cast<const S*>(p.d_sum), p.ld_dsum);
            tensor(p.at_dnormed, reinterpret_cast<const Y*>(p.d_normed), p.ld_dnormed);
            tensor(p.at_y, reinterpret_cast<const Y*>(p.y), p.ldy);
            tensor(p.at_gate, reinterpret_cast<const Y*>(p.gate), p.ldg);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const Drop drop(p);
    int stage = 0;
    if (RING)
        for (int i = 0; i + 1 < p.stages; ++i) copy(first + i * stride, i);
    for (long long row = first; row < p.T; row += stride) {
        if (RING) {
            copy(row + (p.stages - 1) * stride, stage == 0 ? p.stages - 1 : stage - 1);
            if (p.stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");  // this row's copies have landed, those of the rows
            else if (p.stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");         // after it need not have
            else asm volatile("cp.async.wait_group 3;" ::: "memory");
        }
        const char* held = mine + stage * p.stage_bytes;
        auto take = [&](int where, const auto* base, long long ld, int i) {
            using E = std::remove_const_t<std::remove_pointer_t<decltype(base)>>;
            const int at = at0 + i * step;
            if (RING) return widen(load8<PIECES>(reinterpret_cast<const E*>(held + where), at, H));
            Raw<E> r = Raw<E>();
            if (live[i]) r = load8<M>(base + row * ld, at, H);
            return widen(r);
        };
        // Conditions stand outside of the loops over a thread's pieces: within them every piece would wait for its own loads.
        F8 s[VPT], y[VPT], d[VPT], u[VPT];               // s, y: n of the sum and of y, in place
#pragma unroll
        for (int i = 0; i < VPT; ++i) s[i] = y[i] = d[i] = zeros();
        if (before) {
            MOK_EACH_PIECE s[i] = take(p.at_x, reinterpret_cast<const S*>(p.x), p.ldx, i);
            MOK_EACH_PIECE d[i] = take(p.at_dnormed, reinterpret_cast<const Y*>(p.d_normed), p.ld_dnormed, i);
        }
        if (p.at_y >= 0) MOK_EACH_PIECE y[i] = take(p.at_y, reinterpret_cast<const Y*>(p.y), p.ldy, i);
        if (layer_before || layer_after) {
            F2 a = two(0.f), b = two(0.f);
            MOK_EACH_PIECE a = sum8(s[i], a), b = sum8(y[i], b);
            float m[2] = {a.lo() + a.hi(), b.lo() + b.hi()};
            row_sum(m);
            const float ms = layer_before ? -m[0] * p.inv_h : 0.f, my = layer_after ? -m[1] * p.inv_h : 0.f;
            MOK_EACH_PIECE {
                s[i] = M == PIECES ? s[i] + two(live[i] ? ms : 0.f) : within<M>(s[i] + two(ms), at0 + i * step, H);
                y[i] = M == PIECES ? y[i] + two(live[i] ? my : 0.f) : within<M>(y[i] + two(my), at0 + i * step, H);
            }
        }
        // the statistics, and with n = v r the means that the gradient of the sum takes
        F2 a = two(0.f), b = two(0.f), c = two(0.f), e = two(0.f);
        if (before) {
            MOK_EACH_PIECE u[i] = d[i];
            if (p.before_w) MOK_EACH_PIECE u[i] = d[i] * vector(p.at_before_w, p.before_w, at0 + i * step);
            MOK_EACH_PIECE c = dot8(u[i], s[i], c), e = sum8(u[i], e), a = dot8(s[i], s[i], a);
        }
        if (after) MOK_EACH_PIECE b = dot8(y[i], y[i], b);
        float r[4] = {a.lo() + a.hi(), b.lo() + b.hi(), c.lo() + c.hi(), e.lo() + e.hi()};
        if (before || after) {
            row_sum(r);
            r[0] = rsqrtf(fmaf(r[0], p.inv_h, p.eps));
            r[1] = rsqrtf(fmaf(r[1], p.inv_h, p.eps));
        }
        // d becomes the gradient of the sum
        if (before) {
            const F2 spread = two(r[0]), mean_n = two(-r[2] * r[0] * p.inv_h), mean = two(layer_before ? -r[3] * p.inv_h : 0.f);
            if (p.at_acc[0] >= 0) MOK_EACH_PIECE add_extra(0, at0 + i * step, d[i]);
            MOK_EACH_PIECE {
                s[i] = s[i] * spread;
                sum_before[i] = fma8(d[i], s[i], sum_before[i]);
                d[i] = fma8(s[i], mean_n, u[i] + mean) * spread;
            }
        }
        if (p.at_dsum >= 0) MOK_EACH_PIECE d[i] = d[i] + take(p.at_dsum, reinterpret_cast<const S*>(p.d_sum), p.ld_dsum, i);
        MOK_EACH_PIECE {
            if (M == ELEMENTS) d[i] = within<M>(d[i], at0 + i * step, H);
            else if (!live[i]) d[i] = zeros();
        }
        if (p.sum) MOK_EACH_PIECE if (live[i]) store8<M>(reinterpret_cast<S*>(p.sum) + row * p.ld_sum, at0 + i * step, H, d[i]);
        if (of_y) {
            const float token = p.gate_kind == MOK_JOIN_GATE_TOKEN ? to_f(reinterpret_cast<const Y*>(p.gate)[row * p.ldg]) : 1.f;
            a = b = c = two(0.f);
            const F2 scale = two(p.scale), spread_y = two(r[1]);
            MOK_EACH_PIECE d[i] = d[i] * scale;                    // the gradient of v
            if (drop.kind) MOK_EACH_PIECE d[i] = drop.template apply<M>(d[i], (int)row, at0 + i * step);
            if (after) MOK_EACH_PIECE y[i] = y[i] * spread_y;
            if (p.gate_kind != MOK_JOIN_GATE_NONE) {
                MOK_EACH_PIECE u[i] = y[i];
                if (p.after_w) MOK_EACH_PIECE u[i] = u[i] * vector(p.at_after_w, p.after_w, at0 + i * step);
                if (p.after_b) MOK_EACH_PIECE u[i] = u[i] + vector(p.at_after_b, p.after_b, at0 + i * step);
                MOK_EACH_PIECE u[i] = u[i] * d[i];                 // the gradient of the gate
                if (full) {
                    if (p.dgate) MOK_EACH_PIECE if (live[i]) store8<M>(reinterpret_cast<Y*>(p.dgate) + row * p.ld_dgate, at0 + i * step, H, u[i]);
                    MOK_EACH_PIECE d[i] = d[i] * take(p.at_gate, reinterpret_cast<const Y*>(p.gate), p.ldg, i);
                } else if (p.gate_kind == MOK_JOIN_GATE_CHANNEL) {
                    if (p.at_acc[2] >= 0) MOK_EACH_PIECE add_extra(2, at0 + i * step, u[i]);
                    MOK_EACH_PIECE d[i] = d[i] * vector(p.at_channel, p.gate, at0 + i * step);
                } else {
                    MOK_EACH_PIECE c = sum8(u[i], c), d[i] = d[i] * two(token);
                }
            }
            if (after) {                                 // d is the gradient of norm_after's output
                MOK_EACH_PIECE sum_after[i] = fma8(d[i], y[i], sum_after[i]);
                if (p.at_acc[1] >= 0) MOK_EACH_PIECE add_extra(1, at0 + i * step, d[i]);
                if (p.after_w) MOK_EACH_PIECE d[i] = d[i] * vector(p.at_after_w, p.after_w, at0 + i * step);
                MOK_EACH_PIECE a = dot8(d[i], y[i], a), b = sum8(d[i], b);
            }
            if (after || p.gate_kind == MOK_JOIN_GATE_TOKEN) {
                float t[3] = {a.lo() + a.hi(), b.lo() + b.hi(), c.lo() + c.hi()};
                row_sum(t);
                if (p.gate_kind == MOK_JOIN_GATE_TOKEN && p.dgate && threadIdx.x == 0)
                    reinterpret_cast<Y*>(p.dgate)[row * p.ld_dgate] = i8::from_f<Y>(t[2]);
                if (after) {
                    const F2 n = two(-t[0] * p.inv_h), m = two(layer_after ? -t[1] * p.inv_h : 0.f);
                    MOK_EACH_PIECE d[i] = fma8(y[i], n, d[i] + m) * spread_y;
                }
            }
            if (p.dy) MOK_EACH_PIECE if (live[i]) store8<M>(reinterpret_cast<Y*>(p.dy) + row * p.ld_dy, at0 + i * step, H, d[i]);
        }
        if (RING) stage = stage + 1 == p.stages ? 0 : stage + 1;
    }
    if (RING) asm volatile("cp.async.wait_group 0;" ::: "memory");
    block_sums<VPT, M>(p, sum_before, sum_after, s_mem);
}

#undef MOK_EACH_PIECE

// The blocks' sums, added up: 32 columns by 16 threads each, which take every 16th block.
__global__ void __launch_bounds__(512)
join_finish_kernel(const __grid_constant__ Finish f) {
    __shared__ float part[16][33];
    pdl_enter();
    const int col = blockIdx.x * 32 + threadIdx.x;
    const float* in = f.partial + (size_t)blockIdx.y * f.blocks * f.H + col;
    float v = 0.f;
    if (col < f.H) {
#pragma unroll 10
        for (int b = threadIdx.y; b < f.blocks; b += 16) v += in[(size_t)b * f.H];
    }
    part[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y == 0 && col < f.H) {
#pragma unroll
        for (int q = 1; q < 16; ++q) v += part[q][threadIdx.x];
        f.out[blockIdx.y][col] = v;
    }
}

// ------------------------------------------------------------------------------------------------------------------- host side
template <class K>
static cudaError_t launch_back(K kernel, PerDevice& configured, const Params& p, dim3 grid, dim3 block, int smem, cudaStream_t s) {
    int dev = 0, ok = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    e = configured.get(dev, &ok, [&](int, int* v) {
        *v = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM - (int)sizeof(float) * MAX_ROWS * 2 * 4 * 32);
    });
    if (e != cudaSuccess) return e;
    return launch_pdl(kernel, grid, block, (size_t)smem, s, p);
}
template <class S, class Y, int M, bool BEFORE, bool AFTER, int VPT>
static cudaError_t launch_plain(const Params& p, dim3 grid, dim3 block, int smem, cudaStream_t s) {
    static PerDevice configured;
    return launch_back(join_backward_plain_kernel<S, Y, M, BEFORE, AFTER, VPT>, configured, p, grid, block, smem, s);
}
template <class S, class Y, int M, bool RING, int VPT>
static cudaError_t launch_general(const Params& p, dim3 grid, dim3 block, int smem, cudaStream_t s) {
    static PerDevice configured;
    return launch_back(join_backward_kernel<S, Y, M, RING, VPT>, configured, p, grid, block, smem, s);
}
struct Shape {
    int threads, rows, blocks;
};
// Whether the usual kernel does a call.  It has no sums of a bias' or a channel gate's gradient (which are wanted of biases that are not there,
// too: NULL stands for zeros).
static bool usual_call(const Params& p, Layout layout) {
    const bool no_sums = p.slot[2] < 0 && p.slot[3] < 0 && p.slot[4] < 0;
    return layout != ELEMENTS && plain(p) && no_sums && p.d_sum && p.sum && (p.before != MOK_NORM_NONE || p.after != MOK_NORM_NONE);
}
// Blocks that stay, one per SM, of as many rows (at most `most`) as its threads are; fewer for few rows.
static Shape backward_shape(int T, int H, Layout layout, int ld8, int vpt, int most) {
    Shape s;
    const int pieces = (H + (layout == SHIFTED ? 14 : 7)) / 8;
    s.threads = (pieces + 32 * vpt - 1) / (32 * vpt) * 32;
    s.rows = back_threads(vpt) / s.threads;
    if (s.rows > most) s.rows = most;
    if (s.threads > 32 && s.rows > MAX_ROWS) s.rows = MAX_ROWS;
    // (rows of few tokens go to as many SMs as there are)
    while (s.rows > 1 && (long long)148 * s.rows > 2ll * T) s.rows /= 2;
    const int units = (T + s.rows - 1) / s.rows;
    s.blocks = units < 148 ? units : 148;
    // a thread's columns are the same in all of its rows: those are to begin behind the same multiples of eight elements
    if (layout == SHIFTED && units > s.blocks)
        while ((s.blocks * s.rows * ld8) & 7) --s.blocks;
    return s;
}
template <class S, class Y>
static cudaError_t launch_rows(const Params& p, Layout layout, cudaStream_t s, int* blocks);
template <class S, class Y, int VPT>
static cudaError_t launch_backward_of(Params p, Layout layout, cudaStream_t s, int* blocks, int most_rows = 16) {
    const Shape shape = backward_shape(p.T, p.H, layout, p.ld8, VPT, most_rows);
    const bool vec = layout != ELEMENTS, shifted = layout == SHIFTED;
    *blocks = shape.blocks;
    const bool before = p.before != MOK_NORM_NONE, after = p.after != MOK_NORM_NONE;
    const bool usual = VPT == 2 && usual_call(p, layout);
    const int wide = shape.threads * VPT * 8;       // elements of a row in shared memory
    const dim3 grid(shape.blocks), block(shape.threads, shape.rows);
    const int sums_wide = shifted ? wide : p.H;      // a row of sums
    const int sums = shape.rows > 1 || shifted ? 4 * sums_wide * shape.rows : 0, room = SMEM - 1024 - (int)sizeof(float) * MAX_ROWS * 2 * 4 * 32;
    // a stage
    int at = 0;
    auto piece = [&](int& where, bool needed, size_t size) {
        where = needed ? at : -1;
        if (needed) at += wide * (int)size;
    };
    piece(p.at_x, before, sizeof(S));
    piece(p.at_dsum, p.d_sum != nullptr, sizeof(S));
    piece(p.at_dnormed, before, sizeof(Y));
    piece(p.at_y, after || (p.gate_kind != MOK_JOIN_GATE_NONE && p.y), sizeof(Y));
    piece(p.at_gate, p.gate_kind == MOK_JOIN_GATE_FULL, sizeof(Y));
    p.stage_bytes = at;
    // vectors, ring, sums
    const bool gate = p.gate_kind != MOK_JOIN_GATE_NONE;
    at = 0;
    auto vector = [&](int& where, bool needed) {
        where = needed ? at : -1;
        if (needed) at += wide * 4 * (shifted ? shape.rows : 1);
    };
    vector(p.at_before_w, before && (usual || p.before_w));
    vector(p.at_after_w, after && (usual || p.after_w));
    vector(p.at_after_b, after && p.after_b && gate);
    vector(p.at_channel, p.gate_kind == MOK_JOIN_GATE_CHANNEL);
    p.at_ring = at;
    const int n_acc = (p.slot[2] >= 0) + (p.slot[3] >= 0) + (p.slot[4] >= 0), acc = n_acc * 4 * p.H * shape.rows;
    p.stages = p.stage_bytes > 0 ? (room - acc - p.at_ring) / (p.stage_bytes * shape.rows) : 0;
    if (p.stages > 4) p.stages = 4;
    if (vec && p.stages < 2 && shape.rows > 1) {
        if constexpr (VPT == 2)                          // (two pieces per thread were for two rows)
            if (!usual && shape.rows == 2 && p.H <= 8 * back_threads(1)) return launch_backward_of<S, Y, 1>(p, layout, s, blocks);
        return launch_backward_of<S, Y, VPT>(p, layout, s, blocks, shape.rows - 1);
    }
    const bool ring = vec && p.stages >= 2;
    if (shifted && !ring) return launch_rows<S, Y>(p, ELEMENTS, s, blocks);
    if (!ring) {
        p.stages = 1;
        p.at_ring = 0;
    }
    int end = ring ? p.at_ring + p.stages * p.stage_bytes * shape.rows : 0;
    if (end < sums) end = sums;
    for (int i = 0; i < 3; ++i) {
        p.at_acc[i] = p.slot[2 + i] >= 0 ? end : -1;
        if (p.slot[2 + i] >= 0) end += 4 * p.H * shape.rows;
    }
    if constexpr (VPT == 2) {
        if (ring && usual) {
            auto of = [&](auto m) {
                constexpr int M = decltype(m)::value;
                return before && after ? launch_plain<S, Y, M, true, true, VPT>(p, grid, block, end, s)
                       : before        ? launch_plain<S, Y, M, true, false, VPT>(p, grid, block, end, s)
                                       : launch_plain<S, Y, M, false, true, VPT>(p, grid, block, end, s);
            };
            return shifted ? of(std::integral_constant<int, SHIFTED>()) : of(std::integral_constant<int, PIECES>());
        }
    }
    if (ring) return launch_general<S, Y, PIECES, true, VPT>(p, grid, block, end, s);
    if (vec) return launch_general<S, Y, PIECES, false, VPT>(p, grid, block, end, s);
    return launch_general<S, Y, ELEMENTS, false, VPT>(p, grid, block, end, s);
}
template <class S, class Y>
static cudaError_t launch_rows(const Params& p, Layout layout, cudaStream_t s, int* blocks) {
    // The usual kernel has two pieces per thread (16384 x 2880: 130 us, with one 155).  The general one has one, for more warps (11650 x 2880,
    // layer norms, gate and dropout: 247 against 264; 9362 x 3584, a gate and a bias: 111 against 134), but two where a row then needs one
    // warp and no barrier (65536 x 512, layer norms and dropout: 130 against 163; not by elements, where the accesses count: 300 against
    // 262), and where a block then has two rows (8192 x 4096, the same: 172 against 240, by elements 342 against 457).
    // Shifted pieces, beside elements: rms norms of 16392 x 2047 145 against 240 us, 65536 x 505 127 against 201; but a row that only its shift
    // brings to a second warp, 65536 x 511, 240 against 202.
    if (layout == SHIFTED && p.H <= 512 && (p.H + 14) / 8 > 64) layout = ELEMENTS;
    const bool usual = usual_call(p, layout);
    // The general kernel has no shifted form: its vectors would lie in shared memory once for each of a block's rows, which leaves room for
    // fewer of them (16384 x 2047, layer norms, gate and dropout: 695 against 390 us by elements).
    if (!usual && layout == SHIFTED) layout = ELEMENTS;
    const int half = 4 * back_threads(1);
    const bool pairs = (layout == PIECES && p.H > 256 && p.H <= 512) || (p.H > half && p.H <= 8 * back_threads(2));
    if (!usual && !pairs && p.H <= 8 * back_threads(1)) return launch_backward_of<S, Y, 1>(p, layout, s, blocks);
    return launch_backward_of<S, Y, 2>(p, layout, s, blocks);
}

cudaError_t launch_backward(const Params& p, int x_type, int type, Layout layout, Finish f, int vectors, cudaStream_t s) {
    const cudaError_t e = by_type(x_type, type, [&](auto x, auto y) { return launch_rows<decltype(x), decltype(y)>(p, layout, s, &f.blocks); });
    if (e != cudaSuccess || !vectors) return e;
    f.partial = p.partial;
    f.H = p.H;
    return launch_pdl(join_finish_kernel, dim3((p.H + 31) / 32, vectors), dim3(32, 16), 0, s, f);
}

}  // namespace join
}  // namespace mok
