// The whole expert layer for a few tokens (a decoding step) in ONE launch:
//
//   logits = x W_router^T + router_bias;   routes and weights as mok_gate makes them
//   h[r]   = silu(W_gate_e x_t) .* (W_up_e x_t)                  for every route r = (t, slot), e its expert, and for the shared expert
//   y[r]   = W_down_e h[r]
//   out[t] = add[t] + y_shared[t] + sum_slot w[t, slot] y[t, slot]
//
// Its time is that of reading, once, the weights of the experts that are met (6 H I bytes each): a token multiplies a weight once
// or not at all, so the arithmetic (2 T k / E operations per byte and expert) is far below what mma.sync delivers, and tcgen05's
// 128-row tiles would only be wider.  What the layer for many tokens loses here is not bandwidth but the gaps: six launches, each
// of which starts reading when the one before has ended.  So one CTA per SM stays for the whole call (cooperative launch) and a
// warp of it keeps a ring of 128 KB of shared memory full of weights:
//
//   0  router     a warp takes 2048 columns of an expert's row of W_router; partial logits to memory       | grid barrier 0
//   1  routing    T <= 16: every CTA routes all tokens, one or two per warp; else CTA t routes token t     | grid barrier 1
//   2  gate/up    units of 8 gate and 8 up rows, or more, over all CTAs; h to memory                       | grid barrier 2
//   3  down       units of 16 rows of one expert, or more, all experts of a slice of the output in turn; y (fp32) to memory; the
//                 CTA that completes a slice adds up its tokens' rows in slot order
//
// Measured (one call among others, weights beyond L2): 16 tokens of 128 experts of 2048 x 768, k = 8, with 766 MB of weights that are met:
// 148 us, 5.2 TB/s from beginning to end (floor 119); 64 tokens of 8 experts of 4096 x 14336 (2.8 GB): 526 to 583 us by the box; one token of
// the first layer (75 MB): 37 us, of which 13 pass before the routes are known and 3 in the last slices' sums.
//
// The ring runs across the barriers: the shared expert's gate/up rows are on their way before the tokens are routed, and W_down's
// rows, which do not depend on h, while the last gate/up units of other CTAs run.  The down units are dealt out so that the bytes
// of BOTH phases are even over the CTAs: a CTA with a gate/up unit more gets so much less of W_down.
//
// A unit's product: mma.sync m16n8k16, weight rows on the M side, tokens on the N side (a matrix tile of 8 tokens is then the
// smallest price for one token).  Weights come by tiled TMA loads of 64 columns, 128-byte swizzled, the tokens' rows (of x or h) by
// 16-byte asynchronous copies of two loader warps into a ring of their own, in the same layout.  The k index of both operands is
// permuted alike so that a lane's fragments of two instructions are 16 consecutive bytes of a row: one 128-bit load, no ldmatrix;
// and a matrix tile's rows are permuted so that eight lanes in a row read different banks.  The eight consumer warps split a step's
// rows and columns and add partial sums through shared memory in a fixed order: no float atomics, the same bits on every run.
// A TMA load takes the same 120 cycles to issue whether it brings 2 KB or 16, so units have as many rows (up to 128) as leave every
// CTA a few units; a step of 128 rows also needs an eighth of the tokens' columns.
// (Left behind: a bulk copy for each row's piece of a step, 200 cycles each and 1.2 TB/s in all; tokens' fragments read from L2 into
// registers a step ahead, which made every step as long as an L2 access, 2 to 3.3 TB/s.)
//
// Code that runs once is paid for by fetching its instructions: the routing, unrolled as in gate.cu, took 10 to 25 us.  It is written
// in loops here, a loader warp goes through it while the logits are computed, and both products are one loop.
//
// Waits are bounded: one that runs out sets the status word and an abort flag, after which no wait of the CTA waits any more, so
// that every thread still meets every barrier of the CTA and the kernel ends.
#include "gate_token.cuh"
#include "tc_ptx.cuh"
#include "tensor_map.cuh"
#include <chrono>

namespace mok {
namespace few {

using namespace tc;

constexpr int MAX_T = MOK_FEW_MAX_TOKENS;
constexpr int WARPS = 8;                                 // consumer warps
constexpr int W_LOADERS = 2, T_LOADERS = 2;              // warps that load weights, and tokens' rows
constexpr int THREADS = 32 * (WARPS + W_LOADERS + T_LOADERS);
constexpr int MAX_GRID = 256;
constexpr int W_SLOTS = 4, W_STEP = 32768;               // ring of the weights: a slot holds a step
constexpr int T_STEPS = 16, T_BYTES = 57344;             // ring of the tokens: steps that are under way, room for their rows
constexpr int SMEM = 232448;
constexpr int ROUTER_CHUNK = 2048;                       // columns of a router row that a warp takes at once
constexpr int ROUTER_TOKENS = 16;                        // most tokens of such an item
constexpr int SELF_ROUTED = 2 * WARPS;                   // up to so many tokens every CTA routes them all
constexpr int MAX_ROUTES = MAX_T * MAX_K;

static_assert(MAX_T == 64, "an expert's tokens are the bits of a 64-bit word");

struct Ctrl {
    uint64_t w_full[W_SLOTS], w_empty[W_SLOTS], t_full[T_STEPS], t_empty[T_STEPS];
    uint32_t abort;
    uint64_t never_full, never_empty;                    // of the rehearsal (see few_kernel)
    int32_t n_active;
    int32_t sh0, sh1, r0, r1, v0, v1, sources;           // the CTA's units (Shares)
    unsigned long long mask[MAX_E];                      // an expert's tokens
    uint16_t start[MAX_E];                               // where its routes begin in `list`
    uint16_t active[MAX_E];                              // the experts that are met, ascending
    uint16_t list[MAX_ROUTES];                           // routes t * k + slot by expert, tokens ascending
    uint16_t expert[MAX_ROUTES];
    uint8_t token[MAX_ROUTES];                           // the token of each entry of `list`
    uint8_t last[32 * WARPS];
    float w[MAX_ROUTES];
};
constexpr int RED = 2 * WARPS * 2 * 4 * 32 * 4;          // the warps' partial sums, two buffers of one tile of eight tokens
constexpr int RED_AT = ((int)sizeof(Ctrl) + 127) / 128 * 128;
constexpr int W_AT = (RED_AT + RED + 1023) / 1024 * 1024, T_AT = W_AT + W_SLOTS * W_STEP;      // (the swizzle goes by address bits up to 1024)
static_assert(T_AT + T_BYTES <= SMEM, "shared memory");
// before the first token rows are loaded their ring is scratch of the routing: logits and choice values of a token, for every
// consumer warp and one more
static_assert((WARPS + 1) * 2 * MAX_E * 4 <= T_BYTES, "scratch of the routing");

// What the CTAs tell one another.  Barrier 0 makes do with memory that holds anything: every CTA sets its own flag to the call's
// number, a warp of CTA 0 looks at all flags and sets `go` to it, which the others look at.  (All CTAs looking at all flags took 5 us.)
// The counters of the other barriers are cleared by CTA 0 before that.  Whoever is past barrier 2 clears its flag for the next call.
struct Signals {
    unsigned long long flag[MAX_GRID], go;
    int32_t done[2];                                     // CTAs that have arrived at barriers 1 and 2
};
struct Args {
    const void *x, *add;
    const float *W_router, *router_bias;
    long long x_stride, add_stride, out_stride;
    int32_t T, H, I, Is, E, k;
    int32_t parts, router_tokens;                        // router items: parts of a row, ceil(H / ROUTER_CHUNK); tokens of one
    int32_t groups1, groups2;                            // row groups of a unit in the two phases
    int32_t t_tile, t_tiles;                             // ring of the tokens: bytes of eight tokens, how many of them it holds
    double per_cta;                                      // 1 / grid
    int32_t starve;                                      // test hook: no weights are loaded
    unsigned long long number, wait_ns;                  // the call's number
    gate::Params gate;                                   // idx and w: where the routes go
    void* out;
    WsHeader* header;
    Signals* signals;
    int32_t* counters;                                   // per slice of the output: units done
    float* logits;                                       // [parts][T][E]
    void *h, *hs;                                        // [T k, I], [T, Is]
    float* y;                                            // [T k + T, H]
};

__device__ __forceinline__ unsigned long long ld_relaxed64(const unsigned long long* p) {
    unsigned long long v;
    asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ void st_release64(unsigned long long* p, unsigned long long v) {
    asm volatile("st.release.gpu.global.u64 [%0], %1;" ::"l"(p), "l"(v) : "memory");
}
__device__ __forceinline__ int add_acq_rel(int32_t* p, int v) {
    int old;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], %2;" : "=r"(old) : "l"(p), "r"(v) : "memory");
    return old;
}
// [c2][c1 ..][c0 ..] of a three-dimensional tensor
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 2, %0;" ::"n"(32 * WARPS) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
template <class X>
__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16816<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16816<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float2 two_f(uint32_t v, __nv_bfloat16) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
__device__ __forceinline__ float2 two_f(uint32_t v, __half) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }

// ---------------------------------------------------------------------------------------------------- waits and barriers
struct Waits {
    volatile uint32_t* abort;
    WsHeader* header;
    unsigned long long limit;
    __device__ __forceinline__ void give_up(int site) const {
        *abort = 1u;
        atomicCAS(&header->status, 0, (int)MOK_ERR_TIMEOUT);
        header->where = site;
    }
    // false: the CTA is giving up (nothing was waited for any longer)
    // (In line: a call here would cost the accumulators their registers.)
    __device__ __forceinline__ bool mbar(uint32_t bar, uint32_t parity, int site) const {
        unsigned long long t0 = 0ull;                    // (the timer is slow to read: not before a wait is a long one)
        for (uint32_t spins = 1; !mbar_try_wait(bar, parity); ++spins) {
            if (*abort) return false;
            if ((spins & 63u) == 0u) {
                const unsigned long long now = globaltimer();
                if (t0 == 0ull) t0 = now;
                if (now - t0 > limit) {
                    give_up(site);
                    return false;
                }
            }
        }
        return true;
    }
    // A whole warp waits until looks() says true in all lanes.
    template <class Looks>
    __device__ __forceinline__ bool look(const Looks& looks, int lane, int site) const {
        unsigned long long t0 = 0ull;
        for (uint32_t spins = 1; !__all_sync(0xffffffffu, looks()); ++spins) {
            bool over = *abort;
            if ((spins & 63u) == 0u) {
                if (t0 == 0ull) t0 = globaltimer();
                else over |= globaltimer() - t0 > limit;
            }
            if (__any_sync(0xffffffffu, over)) {
                if (lane == 0) give_up(site);
                __syncwarp();
                return false;
            }
        }
        fence_gpu();                                     // with the loads: acquires what was released with the words looked at
        __syncwarp();
        return true;
    }
};

__device__ __forceinline__ void add_release(int32_t* p, int v) {
    asm volatile("red.release.gpu.global.add.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
__device__ __forceinline__ int ld_relaxed(const int32_t* p) {
    int v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ bool wait_first(const Waits& waits, Signals* s, int c, int G, unsigned long long number, int lane) {
    if (c != 0) return waits.look([&] { return lane != 0 || ld_relaxed64(&s->go) == number; }, lane, 4);
    const bool ok = waits.look([&] {
        unsigned long long seen[MAX_GRID / 32];
        bool all = true;
#pragma unroll
        for (int j = 0; j < MAX_GRID / 32; ++j) seen[j] = lane + 32 * j < G ? ld_relaxed64(s->flag + lane + 32 * j) : number;
#pragma unroll
        for (int j = 0; j < MAX_GRID / 32; ++j) all &= seen[j] == number;
        return all;
    }, lane, 4);
    if (ok && lane == 0) st_release64(&s->go, number);
    return ok;
}
__device__ __forceinline__ bool wait_done(const Waits& waits, const Signals* s, int i, int G, int lane) {
    return waits.look([&] { return lane != 0 || ld_relaxed(s->done + i) == G; }, lane, 5 + i);
}

// ------------------------------------------------------------------------------------------------------ division of the work
// Gate/up units of a CTA: its even share of the shared expert's (known before the routing), then of the routed ones.  Down units:
// v = slice * sources + j, the sources of a slice being the experts that are met and the shared one; dealt out so that a CTA's
// gate/up and down units together have an even share of all bytes.
__host__ __device__ inline int part_of(int n, int c, int G) {            // floor(c n / G), c <= G <= 256
    const int q = n / G;
    return c * q + c * (n - q * G) / G;
}
__host__ __device__ inline int quotient(long long a, long long b) {      // floor(a / b) < 2^22: 64-bit divisions are long subroutines
    int q = (int)((float)a * (1.f / (float)b));
    while ((long long)q * b > a) --q;
    while ((long long)(q + 1) * b <= a) ++q;
    return q;
}
// The first down unit of CTA c; c == G: the end
__host__ __device__ inline int first_down(int c, int G, double per_cta, int H, int I, int Is, int active, int n_shared, int n_routed, int rows1,
                                          int rows2) {
    const int sources = active + (Is ? 1 : 0), slices = (H + rows2 - 1) / rows2;
    if (c == G || sources == 0) return slices * sources;
    const long long unit = (long long)rows2 * I, slice_cost = active * unit + (long long)rows2 * Is;
    const long long cost2 = slice_cost * slices, unit1 = (long long)rows1 * H, cost = cost2 + unit1 * (n_shared + n_routed);
    long long even = (long long)((double)cost * per_cta), at;
    if (even * G > cost) --even;
    // a CTA's gate/up units may be more than an even share of everything: then the down units are dealt out by themselves
    const int most = (n_shared + G - 1) / G + (n_routed + G - 1) / G;
    if (most * unit1 > even) {
        even = (long long)((double)cost2 * per_cta);
        at = c * even;
    } else {
        at = c * even - (part_of(n_shared, c, G) + part_of(n_routed, c, G)) * unit1;
    }
    at = at < 0 ? 0 : at > cost2 ? cost2 : at;
    // the first unit that begins at `at` or later
    const int slice = quotient(at, slice_cost);
    const long long rem = at - slice * slice_cost;
    return slice * sources + (rem > active * unit ? sources : quotient(rem + unit - 1, unit));
}

// A unit as both sides of the ring see it.
struct Unit {
    int n;                                               // tokens
    int list;                                            // their routes in Ctrl::list; -1: the shared expert, all tokens
    int K;
    int first;                                           // its first row: of the intermediate (gate/up), of the output (down)
    int limit;                                           // rows there are: I, Is or H
    int matrix;                                          // third coordinate in its tensor map
};
// Unit i of the CTA: gate/up units, then down units
__device__ __forceinline__ Unit unit_of(const Args& a, const Ctrl* ctrl, int i, int n1, int blocks, int rows1, int rows2) {
    Unit u;
    int e = -1;                                          // its expert; -1: the shared one
    if (i < n1) {
        u.K = a.H;
        u.limit = a.I;
        const int shared = ctrl->sh1 - ctrl->sh0;
        if (i < shared) {
            u.first = (ctrl->sh0 + i) * rows1;
            u.limit = a.Is;
        } else {
            const int id = ctrl->r0 + i - shared, q = id / blocks;
            u.first = (id - q * blocks) * rows1;
            e = ctrl->active[q];
        }
    } else {
        const int v = ctrl->v0 + i - n1, slice = v / ctrl->sources, j = v - slice * ctrl->sources;
        u.first = slice * rows2;
        u.limit = a.H;
        if (j < ctrl->n_active) e = ctrl->active[j];
        u.K = e < 0 ? a.Is : a.I;
    }
    u.n = e < 0 ? a.T : __popcll(ctrl->mask[e]);
    u.list = e < 0 ? -1 : ctrl->start[e];
    u.matrix = e < 0 ? 0 : i < n1 ? 2 * e : e;           // (gate/up: the gate half, the up half is the next)
    return u;
}

// A step is 32 KB of weights: [64-column block][row][128 bytes].  Its tokens: per eight of them (Args::t_tile bytes apart)
// [64-column block][8 rows][128 bytes].
template <int MT> __host__ __device__ constexpr int columns(int groups) { return 1024 / MT / groups; }        // of a step
struct Ring {                                            // slots used in turn by both sides
    uint32_t base, full, empty;                          // addresses
    int bytes, slots, slot;
    uint32_t phase;                                      // of `slot`'s use, 0 or 1 in turn
    __device__ __forceinline__ Ring(uint32_t at, const uint64_t* f, const uint64_t* e, int slot_bytes, int n)
        : base(at), full(smem_u32(f)), empty(smem_u32(e)), bytes(slot_bytes), slots(n), slot(0), phase(0u) {}
    __device__ __forceinline__ uint32_t data() const { return base + slot * bytes; }
    __device__ __forceinline__ uint32_t is_full() const { return full + slot * 8; }
    __device__ __forceinline__ uint32_t is_empty() const { return empty + slot * 8; }
    __device__ __forceinline__ void advance() {
        if (++slot == slots) {
            slot = 0;
            phase ^= 1u;
        }
    }
};
__device__ __forceinline__ Ring weight_ring(const char* smem, const Ctrl* c) {
    return Ring(smem_u32(smem + W_AT), c->w_full, c->w_empty, W_STEP, W_SLOTS);
}
// The tokens' ring: barriers per step, room per eight tokens.
struct TokenRing {
    Ring steps;
    int tile, tiles, at;                                 // bytes of a tile, tiles; the next one
    __device__ __forceinline__ TokenRing(const char* smem, const Ctrl* c, const Args& a)
        : steps(smem_u32(smem + T_AT), c->t_full, c->t_empty, 0, T_STEPS), tile(a.t_tile), tiles(a.t_tiles), at(0) {}
    __device__ __forceinline__ uint32_t data(int q) const {              // tile q of the step, q < 8 <= tiles
        const int i = at + q;
        return steps.base + (i < tiles ? i : i - tiles) * tile;
    }
    __device__ __forceinline__ void advance(int n) {
        at += n;
        if (at >= tiles) at -= tiles;
        steps.advance();
    }
};
// The loaders' side: which steps are under way, and how much room they take.
struct TokenRoom {
    Ring oldest;
    unsigned long long sizes;                            // four bits per step: its tiles
    int used, steps;
    // false: the CTA is giving up
    __device__ __forceinline__ bool take(const TokenRing& ring, int n, const Waits& waits) {
        while (steps == T_STEPS || used + n > ring.tiles) {
            // (all lanes alike: after an abort one may still find the step free where another gives up)
            if (!__all_sync(0xffffffffu, waits.mbar(oldest.is_empty(), oldest.phase, 6))) return false;
            used -= (int)(sizes >> (4 * oldest.slot)) & 15;
            --steps;
            oldest.advance();
        }
        const int s = ring.steps.slot;
        sizes = (sizes & ~(15ull << (4 * s))) | (unsigned long long)n << (4 * s);
        used += n;
        ++steps;
        return true;
    }
};
// Where row j of eight lies, so that the lanes of a fragment load read different banks
__device__ __forceinline__ int row_of(int g) { return (g >> 1) + 4 * (g & 1); }

// One step of a unit's weights, always all of its columns: those past K, and rows past the matrix, come as zeros.
template <int MT>
__device__ __forceinline__ void load_step(const Ring& ring, const CUtensorMap* map, const Unit& u, int k0, int groups) {
    const int rows = 16 * MT * groups, width = columns<MT>(groups);
    mbar_expect_tx(ring.is_full(), (uint32_t)W_STEP);
    for (int b = 0; b < width; b += 64) tma_load_3d(ring.data() + b * rows * 2, map, ring.is_full(), k0 + b, u.first, u.matrix);
}

// The tokens' rows of a unit: loader warp `me` takes every second step (`turn`: whose turn it is).  Four lanes per row of eight.
// false: the CTA is giving up
template <class X, int MT>
__device__ __forceinline__ bool load_tokens(const Args& a, const Ctrl* ctrl, const Waits& waits, TokenRing& ring, TokenRoom& room, const Unit& u, bool gated, int groups,
                                            int me, int& turn, int lane) {
    const int width = columns<MT>(groups), j = lane >> 2, at = row_of(j), p0 = lane & 3;
    const X* base = reinterpret_cast<const X*>(gated ? a.x : u.list >= 0 ? a.h : a.hs);
    const size_t stride = gated ? (size_t)a.x_stride : (size_t)u.K;
    for (int k0 = 0; k0 < u.K; k0 += width) {
        const int tiles = (u.n + 7) >> 3;
        if (!room.take(ring, tiles, waits)) return false;
        if (turn == me) {
            for (int q = j; q < u.n; q += 8) {
                const uint32_t dst = ring.data(q >> 3) + at * 128;
                const int r = u.list < 0 ? q : gated ? ctrl->token[u.list + q] : ctrl->list[u.list + q];
                const X* row = base + r * stride + k0;
#pragma unroll 4
                for (int p = p0; p < width / 8; p += 4) {
                    const bool there = k0 + p * 8 < u.K; // (the rest are zeros)
                    cp_async_16(dst + (p >> 3) * 1024 + ((p ^ at) & 7) * 16, there ? row + p * 8 : row, there ? 16u : 0u);
                }
            }
            cp_async_mbar_arrive(ring.steps.is_full());
        }
        turn ^= 1;
        ring.advance(tiles);
    }
    return true;
}

// --------------------------------------------------------------------------------------------------------------- consumers
template <int N> struct Count { static constexpr int value = N; };
template <class X, int MT, int NT>
struct Consumer {
    static constexpr int KB = 4 / MT;                    // 32-column blocks of a step per warp
    const Args& a;
    Ctrl* ctrl;
    const Waits& waits;
    float* red;                                          // [2][WARPS][MT * 4][32]
    int warp, lane;
    Ring ring;
    TokenRing tokens;
    int flip;
    float acc[MT][NT][4];

    // the whole K of u, in code for its number of tiles of tokens: branches in the loop cost as much as its products
    __device__ __forceinline__ void multiply(const Unit& u, bool gated, int groups) { by_tiles(u, gated, groups, Count<NT>()); }
    template <int N>
    __device__ __forceinline__ void by_tiles(const Unit& u, bool gated, int groups, Count<N>) {
        if (N == 1 || u.n > 8 * (N - 1)) run<N>(u, gated, groups);
        else if constexpr (N > 1) by_tiles(u, gated, groups, Count<N - 1>());
    }
    template <int TILES>
    __device__ __forceinline__ void run(const Unit& u, bool gated, int groups) {
        // rows of a step from one matrix tile to the next, and from its first eight rows to the other eight: 8 gate rows and, behind
        // all gate rows, the 8 up rows that go with them; or 16 rows
        const int tile_step = gated ? 8 : 16, half_step = gated ? 8 * MT * groups : 8;
        const int width = columns<MT>(groups), per = WARPS / groups, rg = warp / per, kw = warp % per, rows = 16 * MT * groups;
        const int t = lane & 3, r = row_of(lane >> 2);
        uint32_t weights_at[KB], tokens_at[KB];          // this lane's part of a step's 32-column blocks
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            const int block = (kw * KB + b) >> 1;
            const uint32_t chunk = (uint32_t)((((kw * KB + b) & 1) * 4 + t) ^ r) * 16 + r * 128;
            weights_at[b] = (uint32_t)(block * rows + rg * MT * tile_step) * 128 + chunk;
            tokens_at[b] = (uint32_t)block * 1024 + chunk;
        }
        // Sets of accumulators, by which a chain of products is shorter.  Not by TILES: the order of a token's sums would depend on how many
        // others meet its expert.
        constexpr int SETS = MT == 1 ? 2 : 1;
        float other[MT][TILES][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int q = 0; q < TILES; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][q][i] = other[m][q][i] = 0.f;
        for (int k0 = 0; k0 < u.K; k0 += width) {
            waits.mbar(ring.is_full(), ring.phase, 2);
            waits.mbar(tokens.steps.is_full(), tokens.steps.phase, 7);
            const uint32_t data = ring.data();
            uint4 lo[MT][KB], hi[MT][KB];
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    lo[m][b] = lds128(data + weights_at[b] + m * tile_step * 128);
                    hi[m][b] = lds128(data + weights_at[b] + (m * tile_step + half_step) * 128);
                }
            constexpr int PAIR = TILES > 1 ? 2 : 1;      // tiles at a time, so that a product does not wait for the one before it
#pragma unroll
            for (int q = 0; q < TILES; q += PAIR) {
                uint4 v[PAIR][KB];
#pragma unroll
                for (int n = 0; n < PAIR; ++n) {
                    if (q + n >= TILES) continue;
                    const uint32_t held = tokens.data(q + n);
#pragma unroll
                    for (int b = 0; b < KB; ++b) v[n][b] = lds128(held + tokens_at[b]);
                }
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int n = 0; n < PAIR; ++n)
#pragma unroll
                            for (int m = 0; m < MT; ++m) {
                                if (q + n >= TILES) continue;
                                float(&c)[4] = half && SETS == 2 ? other[m][q + n] : acc[m][q + n];
                                if (half) mma16816<X>(c, lo[m][b].z, hi[m][b].z, lo[m][b].w, hi[m][b].w, v[n][b].z, v[n][b].w);
                                else mma16816<X>(c, lo[m][b].x, hi[m][b].x, lo[m][b].y, hi[m][b].y, v[n][b].x, v[n][b].y);
                            }
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(tokens.steps.is_empty());
                mbar_arrive(ring.is_empty());
            }
            tokens.advance(TILES);
            ring.advance();
        }
        if (SETS == 2) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int q = 0; q < TILES; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][q][i] += other[m][q][i];
        }
    }
    // sums over the warps that split K, for tile q of eight tokens: out(row group and matrix tile, register, lane, sum...)
    __device__ __forceinline__ float* publish(int q) {
        float* mine = red + (size_t)((flip & 1) * WARPS + warp) * MT * 4 * 32;
        flip ^= 1;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                if (n == q) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) mine[(m * 4 + i) * 32 + lane] = acc[m][n][i];
                }
        consumers_sync();
        return red + (size_t)((flip ^ 1) & 1) * WARPS * MT * 4 * 32;
    }
    // register i of lane l, and i + 2, of a matrix tile
    __device__ __forceinline__ float2 total(const float* part, int per, int rg, int m, int i, int l) const {
        const float* at = part + (rg * per * MT * 4 + m * 4 + i) * 32 + l;
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w)
            if (w < per) {
                v.x += at[w * MT * 128];
                v.y += at[w * MT * 128 + 64];
            }
        return v;
    }
    // h, or rows of y, of a unit
    __device__ __forceinline__ void store(const Unit& u, bool gated, int groups) {
        const int per = WARPS / groups, tiles = (u.n + 7) >> 3;
        for (int q = 0; q < tiles; ++q) {
            const float* part = publish(q);
            for (int o = warp * 32 + lane; o < groups * MT * 64; o += 32 * WARPS) {
                // lane l of a matrix tile has columns (tokens) 2 (l % 4) + i of rows row_of(l / 4) and eight further
                const int l = o & 31, i = (o >> 5) & 1, tile = o >> 6, m = tile % MT, rg = tile / MT;
                const int col = q * 8 + 2 * (l & 3) + i;
                const float2 sum = total(part, per, rg, m, i, l);
                if (col >= u.n) continue;
                const int r = u.list >= 0 ? ctrl->list[u.list + col] : col;
                if (gated) {
                    const int row = u.first + tile * 8 + row_of(l >> 2);
                    // h in 16 bits, as the layer for many tokens keeps it: an operand of the next product
                    const float h = sum.x / (1.f + expf(-sum.x)) * sum.y;
                    X* dst = u.list >= 0 ? reinterpret_cast<X*>(a.h) + (size_t)r * a.I : reinterpret_cast<X*>(a.hs) + (size_t)r * a.Is;
                    if (row < u.limit) gate::store_f(dst + row, h);
                } else {
                    const int row = u.first + tile * 16 + row_of(l >> 2);
                    float* dst = a.y + (size_t)(u.list >= 0 ? r : a.T * a.k + r) * a.H + row;
                    if (row < u.limit) *dst = sum.x;
                    if (row + 8 < u.limit) dst[8] = sum.y;
                }
            }
        }
    }
    // The CTA's units are done.  Whoever completes a slice adds up its columns of every token.
    __device__ __forceinline__ void finish(int rows) {
        const int v0 = ctrl->v0, v1 = ctrl->v1, sources = ctrl->sources, me = warp * 32 + lane;
        if (v0 >= v1) return;
        const int first = v0 / sources, end = (v1 - 1) / sources + 1;
        for (int s0 = first; s0 < end; s0 += 32 * WARPS) {
            consumers_sync();
            const int slice = s0 + me, n = min(end - s0, 32 * WARPS);
            if (me < n) {
                const int units = min(v1, (slice + 1) * sources) - max(v0, slice * sources);
                ctrl->last[me] = add_acq_rel(a.counters + slice, units) + units == sources;
            }
            consumers_sync();
            // four columns of a token per thread (rows and H are multiples of four)
            for (int o = me; o < n * a.T * (rows / 4); o += 32 * WARPS) {
                const int q = o / (rows / 4), i = q / a.T, t = q - i * a.T, c = (s0 + i) * rows + (o - q * (rows / 4)) * 4;
                if (!ctrl->last[i] || c >= a.H) continue;
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (a.add) {
                    const X* add = reinterpret_cast<const X*>(a.add) + (size_t)t * a.add_stride + c;
                    v = make_float4(gate::load_f(add), gate::load_f(add + 1), gate::load_f(add + 2), gate::load_f(add + 3));
                }
                if (a.Is) {
                    const float4 y = __ldcg(reinterpret_cast<const float4*>(a.y + (size_t)(a.T * a.k + t) * a.H + c));
                    v = make_float4(v.x + y.x, v.y + y.y, v.z + y.z, v.w + y.w);
                }
                const float4* row = reinterpret_cast<const float4*>(a.y + (size_t)t * a.k * a.H + c);
#pragma unroll 8
                for (int k = 0; k < a.k; ++k) {
                    const float w = ctrl->w[t * a.k + k];
                    const float4 y = __ldcg(row + (size_t)k * (a.H / 4));
                    v = make_float4(fmaf(w, y.x, v.x), fmaf(w, y.y, v.y), fmaf(w, y.z, v.z), fmaf(w, y.w, v.w));
                }
                X* out = reinterpret_cast<X*>(a.out) + (size_t)t * a.out_stride + c;
                gate::store_f(out, v.x);
                gate::store_f(out + 1, v.y);
                gate::store_f(out + 2, v.z);
                gate::store_f(out + 3, v.w);
            }
        }
    }
};

// ------------------------------------------------------------------------------------------------------------------ routing
// Partial logits: item (expert, part of its row, group of tokens) per warp.
template <class X>
__device__ __forceinline__ void router(const Args& a, int warp, int lane) {
    const int token_groups = (a.T + a.router_tokens - 1) / a.router_tokens;
    const int items = a.E * a.parts * token_groups;
    constexpr int PIECES = ROUTER_CHUNK / 256;
    for (int item = warp * gridDim.x + blockIdx.x; item < items; item += WARPS * gridDim.x) {
        const int tg = item % token_groups, rest = item / token_groups, part = rest % a.parts, e = rest / a.parts;
        const int at = part * ROUTER_CHUNK + lane * 8, t0 = tg * a.router_tokens, t1 = min(a.T, t0 + a.router_tokens);
        uint4 v[PIECES], after[PIECES];
        auto fetch = [&](int t, uint4 (&to)[PIECES]) {
            const X* row = reinterpret_cast<const X*>(a.x) + (size_t)t * a.x_stride + at;
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                to[i] = at + i * 256 < a.H ? __ldg(reinterpret_cast<const uint4*>(row + i * 256)) : make_uint4(0u, 0u, 0u, 0u);
        };
        fetch(t0, v);
        float4 w[PIECES][2];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            w[i][0] = w[i][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (at + i * 256 < a.H) {
                const float4* src = reinterpret_cast<const float4*>(a.W_router + (size_t)e * a.H + at + i * 256);
                w[i][0] = __ldg(src);
                w[i][1] = __ldg(src + 1);
            }
        }
        for (int t = t0; t < t1; ++t) {
            if (t + 1 < t1) fetch(t + 1, after);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) {
                const uint32_t u[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                const float f[8] = {w[i][0].x, w[i][0].y, w[i][0].z, w[i][0].w, w[i][1].x, w[i][1].y, w[i][1].z, w[i][1].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = two_f(u[j], X());
                    sum = fmaf(x.x, f[2 * j], sum);
                    sum = fmaf(x.y, f[2 * j + 1], sum);
                }
            }
            sum = gate::warp_sum(sum);
            if (lane == 0) a.logits[((size_t)part * a.T + t) * a.E + e] = sum;
#pragma unroll
            for (int i = 0; i < PIECES; ++i) v[i] = after[i];
        }
    }
}
// A token's routes; lane s < k gets slot s's.  t < 0: only the motions, on no data.
__device__ __noinline__ void route(const Args& a, int t, float* row, float* choice, int lane, int& e, float& w) {
    for (int i = lane; i < a.E; i += 128) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = a.router_bias && i + 32 * j < a.E ? __ldg(a.router_bias + i + 32 * j) : 0.f;
#pragma unroll 2
        for (int p = 0; p < (t < 0 ? 0 : a.parts); ++p) {
            const float* part = a.logits + ((size_t)p * a.T + t) * a.E + i;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + 32 * j < a.E) v[j] += __ldcg(part + 32 * j);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + 32 * j < a.E) row[i + 32 * j] = v[j];
    }
    __syncwarp();
    gate::route_token(a.gate, row, choice, lane, e, w);
    w *= a.gate.scale;
    __syncwarp();
}

template <class X, int MT, int NT>
__global__ void __launch_bounds__(THREADS, 1)
few_kernel(const __grid_constant__ CUtensorMap m_gu, const __grid_constant__ CUtensorMap m_dn, const __grid_constant__ CUtensorMap m_sgu,
           const __grid_constant__ CUtensorMap m_sdn, const __grid_constant__ Args a) {
    extern __shared__ __align__(1024) char smem[];
    Ctrl* ctrl = reinterpret_cast<Ctrl*>(smem);
    float* scratch = reinterpret_cast<float*>(smem + T_AT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x, G = gridDim.x;
    const int rows1 = 8 * MT * a.groups1, rows2 = 16 * MT * a.groups2;
    const int blocks = (a.I + rows1 - 1) / rows1, n_shared = (a.Is + rows1 - 1) / rows1;
    const Waits waits = {&ctrl->abort, a.header, a.wait_ns};

    if (threadIdx.x == 0) {
        for (int s = 0; s < W_SLOTS; ++s) {
            mbar_init(smem_u32(&ctrl->w_full[s]), 1);
            mbar_init(smem_u32(&ctrl->w_empty[s]), WARPS);
        }
        for (int s = 0; s < T_STEPS; ++s) {
            mbar_init(smem_u32(&ctrl->t_full[s]), 32);
            mbar_init(smem_u32(&ctrl->t_empty[s]), WARPS);
        }
        ctrl->abort = 0u;
        ctrl->n_active = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_init(smem_u32(&ctrl->never_full), 1);
        mbar_init(smem_u32(&ctrl->never_empty), WARPS);
        if (c == 0) {
            a.signals->done[0] = a.signals->done[1] = 0;
            a.header->status = 0;
            a.header->where = 0;
        }
    }
    for (int e = threadIdx.x; e < a.E; e += THREADS) ctrl->mask[e] = 0ull;
    const int slices = (a.H + rows2 - 1) / rows2;
    for (int s = c * THREADS + threadIdx.x; s < slices; s += G * THREADS) a.counters[s] = 0;
    __syncthreads();

    if (warp >= WARPS && warp < WARPS + W_LOADERS) {
        // ------------------------------------------------------------------------------------------------------- weights
        Ring ring = weight_ring(smem, ctrl);
        // the shared expert's steps that fit into the empty ring go out before the routes are known
        const int shared = part_of(n_shared, c + 1, G) - part_of(n_shared, c, G), first = part_of(n_shared, c, G) * rows1;
        const int width1 = columns<MT>(a.groups1);
        int i = 0, k0 = 0, turn = warp - WARPS;          // the next step: unit and column; 0: it is this warp's
        if (lane == 0 && !a.starve) {
            while (i < shared && ring.phase == 0u) {     // (the first round: every slot is empty)
                if (turn == 0) load_step<MT>(ring, &m_sgu, Unit{0, -1, a.H, first + i * rows1, a.Is, 0}, k0, a.groups1);
                turn ^= 1;
                ring.advance();
                k0 += width1;
                if (k0 >= a.H) { k0 = 0; ++i; }
            }
        }
        __syncwarp();
        asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");       // the routes are in shared memory
        if (lane == 0 && !a.starve) {
            const int n1 = shared + ctrl->r1 - ctrl->r0, n = n1 + ctrl->v1 - ctrl->v0;
            bool go = true;
            for (; go && i < n; ++i, k0 = 0) {           // W_down does not depend on h: no wait for barrier 2 here
                const Unit u = unit_of(a, ctrl, i, n1, blocks, rows1, rows2);
                const CUtensorMap* map = i < n1 ? (u.list < 0 ? &m_sgu : &m_gu) : u.list < 0 ? &m_sdn : &m_dn;
                const int groups = i < n1 ? a.groups1 : a.groups2;
                for (; k0 < u.K; k0 += columns<MT>(groups)) {
                    if (turn == 0) {
                        go = waits.mbar(ring.is_empty(), ring.phase ^ 1u, 1);
                        if (!go) break;
                        load_step<MT>(ring, map, u, k0, groups);
                    }
                    turn ^= 1;
                    ring.advance();
                }
            }
        }
        __syncwarp();
    } else if (warp >= WARPS) {
        // --------------------------------------------------------------------------------------------------------- tokens
        const int me = warp - WARPS - W_LOADERS;
        int turn = 0;
        TokenRing ring(smem, ctrl, a);
        TokenRoom room = {ring.steps, 0ull, 0, 0};
        if (me == 0) {
            // The routing's instructions run once in a call and are not in any cache of the SM: this warp fetches them while the logits
            // are computed.
            int e;
            float w;
            float* rows = scratch + WARPS * 2 * MAX_E;
            route(a, -1, rows, rows + MAX_E, lane, e, w);
            if (lane == 0) ctrl->last[0] = (uint8_t)e;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
        const int n1 = ctrl->sh1 - ctrl->sh0 + ctrl->r1 - ctrl->r0, n = n1 + ctrl->v1 - ctrl->v0;
        bool go = true;
        for (int i = 0; go && i <= n; ++i) {
            if (i == n1) {
                go = wait_done(waits, a.signals, 1, G, lane);
                if (go && me == 0 && lane == 0) {        // every CTA is past barrier 0
                    a.signals->flag[c] = 0ull;
                    if (c == 0) a.signals->go = 0ull;
                }
            }
            if (go && i < n)
                go = load_tokens<X, MT>(a, ctrl, waits, ring, room, unit_of(a, ctrl, i, n1, blocks, rows1, rows2), i < n1, i < n1 ? a.groups1 : a.groups2,
                                        me, turn, lane);
        }
    } else {
        // ------------------------------------------------------------------------------------------------------ consumers
        router<X>(a, warp, lane);
        consumers_sync();
        if (threadIdx.x == 0) st_release64(a.signals->flag + c, a.number);
        Consumer<X, MT, NT> w = {a, ctrl, waits, reinterpret_cast<float*>(smem + RED_AT), warp, lane, weight_ring(smem, ctrl),
                                 TokenRing(smem, ctrl, a), 0};
        {
            // A rehearsal on no data while the barrier is waited for: it brings the instructions of the loop below.  Its rings' barriers
            // are as before their first use, so nothing waits (a parity of 1 counts as past), and limit = 0 stores nothing.
            const Ring held = w.ring;
            const TokenRing held_tokens = w.tokens;
            for (int i = 0; i < 2; ++i) {
                w.ring.full = w.tokens.steps.full = smem_u32(&ctrl->never_full);
                w.ring.empty = w.tokens.steps.empty = smem_u32(&ctrl->never_empty);
                w.ring.slot = w.tokens.steps.slot = 0;
                w.ring.phase = w.tokens.steps.phase = 1u;
                const Unit u = {8, -1, 64, 0, 0, 0};
                w.multiply(u, i == 0, i == 0 ? a.groups1 : a.groups2);
                w.store(u, i == 0, i == 0 ? a.groups1 : a.groups2);
            }
            w.ring = held;
            w.tokens = held_tokens;
        }
        if (warp == 0) wait_first(waits, a.signals, c, G, a.number, lane);
        consumers_sync();
        float *row = scratch + warp * 2 * MAX_E, *choice = row + MAX_E;
        const int n = a.T * a.k;
        if (a.T <= SELF_ROUTED) {
            for (int t = warp; t < a.T; t += WARPS) {
                int e;
                float w;
                route(a, t, row, choice, lane, e, w);
                if (lane < a.k) {
                    ctrl->expert[t * a.k + lane] = (uint16_t)e;
                    ctrl->w[t * a.k + lane] = w;
                    if (c == 0) {
                        a.gate.idx[t * a.k + lane] = e;
                        a.gate.w[t * a.k + lane] = w;
                    }
                }
            }
        } else {
            for (int t = warp * G + c; t < a.T; t += WARPS * G) {
                int e;
                float w;
                route(a, t, row, choice, lane, e, w);
                if (lane < a.k) {
                    a.gate.idx[t * a.k + lane] = e;
                    a.gate.w[t * a.k + lane] = w;
                }
            }
            consumers_sync();
            if (threadIdx.x == 0) add_release(a.signals->done, 1);
            if (warp == 0) wait_done(waits, a.signals, 0, G, lane);
            consumers_sync();
            for (int r = threadIdx.x; r < n; r += 32 * WARPS) {
                ctrl->expert[r] = (uint16_t)min(max(__ldcg(a.gate.idx + r), 0), a.E - 1);    // (out of range only after a timeout)
                ctrl->w[r] = __ldcg(a.gate.w + r);
            }
        }
        consumers_sync();
        for (int r = threadIdx.x; r < n; r += 32 * WARPS) atomicOr(&ctrl->mask[ctrl->expert[r]], 1ull << (r / a.k));
        consumers_sync();
        if (warp == 0) {
            int active = 0, routes = 0;
            for (int e0 = 0; e0 < a.E; e0 += 32) {
                const int e = e0 + lane, mine = e < a.E ? __popcll(ctrl->mask[e]) : 0;
                int upto = mine;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const int o = __shfl_up_sync(0xffffffffu, upto, off);
                    if (lane >= off) upto += o;
                }
                const unsigned met = __ballot_sync(0xffffffffu, mine > 0);
                if (mine) {
                    ctrl->active[active + __popc(met & ((1u << lane) - 1u))] = (uint16_t)e;
                    ctrl->start[e] = (uint16_t)(routes + upto - mine);
                }
                active += __popc(met);
                routes += __shfl_sync(0xffffffffu, upto, 31);
            }
            // after a wait that ran out the routes may be anything: there are none then
            if (__any_sync(0xffffffffu, *(volatile uint32_t*)&ctrl->abort)) active = 0;
            const int n_routed = active * blocks;
            if (lane < 2) {                              // the CTA's units begin, and the next CTA's
                const int at = c + lane;
                (lane ? ctrl->sh1 : ctrl->sh0) = part_of(n_shared, at, G);
                (lane ? ctrl->r1 : ctrl->r0) = part_of(n_routed, at, G);
                (lane ? ctrl->v1 : ctrl->v0) = first_down(at, G, a.per_cta, a.H, a.I, a.Is, active, n_shared, n_routed, rows1, rows2);
                ctrl->n_active = active;
                ctrl->sources = active + (a.Is ? 1 : 0);
            }
        }
        consumers_sync();
        for (int r = threadIdx.x; r < n; r += 32 * WARPS) {
            const int e = ctrl->expert[r], t = r / a.k;
            const int at = ctrl->start[e] + __popcll(ctrl->mask[e] & ((1ull << t) - 1ull));
            ctrl->list[at] = (uint16_t)r;
            ctrl->token[at] = (uint8_t)t;
        }
        asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
        const int n1 = ctrl->sh1 - ctrl->sh0 + ctrl->r1 - ctrl->r0, units = n1 + ctrl->v1 - ctrl->v0;
        for (int i = 0; i <= units; ++i) {
            if (i == n1) {
                consumers_sync();
                if (threadIdx.x == 0) add_release(a.signals->done + 1, 1);
            }
            if (i == units) break;
            const Unit u = unit_of(a, ctrl, i, n1, blocks, rows1, rows2);
            const int groups = i < n1 ? a.groups1 : a.groups2;
            w.multiply(u, i < n1, groups);
            w.store(u, i < n1, groups);
        }
        w.finish(rows2);
    }
    __syncthreads();                                     // no wait of the CTA is under way any more
    if (*(volatile uint32_t*)&ctrl->abort) {             // failure path only: copies in flight land before the CTA leaves
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 200000ull) { }
        // a replay of this call has the same number: it must not find its flags set (the token loader clears them behind barrier 2, which it
        // did not get past if it gave up)
        if (threadIdx.x == 0) {
            a.signals->flag[c] = 0ull;
            if (c == 0) a.signals->go = 0ull;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------- host side
struct Layout {
    size_t signals, counters, logits, idx, w, h, hs, y, total;
    int parts;
};
static bool layout(int T, int H, int I, int Is, int E, int k, Layout* L) {
    if (T < 0 || T > MAX_T || H < 8 || I < 8 || Is < 0 || H % 8 || I % 8 || Is % 8 || E < 1 || E > MAX_E || k < 1 || k > MAX_K || k > E) return false;
    if (H > (1 << 20) || I > (1 << 20) || Is > (1 << 20)) return false;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    const size_t n = (size_t)T * k;
    L->parts = (H + ROUTER_CHUNK - 1) / ROUTER_CHUNK;
    take(sizeof(WsHeader));
    L->signals = take(sizeof(Signals));
    L->counters = take((size_t)(H + 15) / 16 * sizeof(int32_t));
    L->logits = take((size_t)L->parts * T * E * sizeof(float));
    L->idx = take(n * sizeof(int32_t));
    L->w = take(n * sizeof(float));
    L->h = take(n * I * 2);
    L->hs = take((size_t)T * Is * 2);
    L->y = take((n + (Is ? T : 0)) * H * sizeof(float));
    L->total = at;
    return true;
}

// A number that no other call has and that leftover memory does not hold: what the flags of this call's barriers are set to.
static unsigned long long call_number() {
    static std::atomic<unsigned long long> count{(unsigned long long)std::chrono::steady_clock::now().time_since_epoch().count() ^
                                                 (unsigned long long)reinterpret_cast<uintptr_t>(&count)};
    unsigned long long z = count.fetch_add(0x9E3779B97F4A7C15ull) + 0x9E3779B97F4A7C15ull;     // splitmix64 (Steele et al. 2014)
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    z ^= z >> 31;
    return z ? z : 1ull;
}

// Row groups of a unit, `usual` of them: more where there are so few columns that warps would have none.
static int row_groups(int K, int usual, int most, int KC) {
    int g = usual;
    while (g < most && K <= KC / g / 2) g *= 2;
    return g;
}

// `matrices` matrices [rows, cols], one behind the other; a box is 64 columns of box_rows rows of `deep` matrices
template <class X>
static bool stack_map(CUtensorMap* m, const void* ptr, uint64_t matrices, uint64_t rows, uint64_t cols, uint32_t box_rows, uint32_t deep) {
    tmap::EncodeTiledFn enc = tmap::get_encode();
    if (!enc) return false;
    const cuuint64_t dims[3] = {cols, rows, matrices}, strides[2] = {cols * sizeof(X), rows * cols * sizeof(X)};
    const cuuint32_t box[3] = {64, box_rows, deep}, steps[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, const_cast<void*>(ptr), dims, strides, box, steps,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class X, int MT, int NT>
static cudaError_t launch(Args a, const mok_few_args* w, cudaStream_t s) {
    static PerDevice configured;
    auto kernel = few_kernel<X, MT, NT>;
    int dev = 0, sms = 0;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return e;
    e = configured.get(dev, &sms, [&](int d, int* v) {
        cudaError_t r = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
        return r != cudaSuccess ? r : device_sm_count(d, v);
    });
    if (e != cudaSuccess) return e;
    const int grid = sms < MAX_GRID ? sms : MAX_GRID;
    const int items = (int)(((long long)a.T * a.E * a.parts + WARPS * grid - 1) / (WARPS * grid));
    a.router_tokens = items < ROUTER_TOKENS ? items : ROUTER_TOKENS;
    // A load takes the same time to issue for few rows and for many, so units of more rows are faster; but the more rows, the further
    // apart the CTAs reach barrier 2.  16 tokens of 128 experts of 2048 x 768, gate/up units of 2 groups and down units of 4:
    // 148 us; 2 and 2: 157, 8 and 8: 155.
    a.groups1 = row_groups(a.H, 2, 8 / MT, columns<MT>(1));
    a.groups2 = row_groups(a.I, MT == 1 ? 4 : 2, 8 / MT, columns<MT>(1));
    a.t_tile = 8 * columns<MT>(a.groups1 < a.groups2 ? a.groups1 : a.groups2) * 2;
    a.t_tiles = T_BYTES / a.t_tile;
    static_assert(T_BYTES / (8 * columns<MT>(2) * 2) >= (NT > 2 ? 8 : NT), "a step's tokens have room");
    a.per_cta = 1.0 / grid;
    CUtensorMap m_gu, m_dn, m_sgu, m_sdn;
    const uint32_t box1 = 8 * MT * a.groups1, box2 = 16 * MT * a.groups2;
    if (!stack_map<X>(&m_gu, w->W_gate_up, 2 * (uint64_t)a.E, a.I, a.H, box1, 2) || !stack_map<X>(&m_dn, w->W_down, a.E, a.H, a.I, box2, 1))
        return cudaErrorInvalidValue;
    if (!a.Is) {                                         // (never used)
        m_sgu = m_gu;
        m_sdn = m_dn;
    } else if (!stack_map<X>(&m_sgu, w->W_shared_gate_up, 2, a.Is, a.H, box1, 2) || !stack_map<X>(&m_sdn, w->W_shared_down, 1, a.H, a.Is, box2, 1)) {
        return cudaErrorInvalidValue;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;         // the CTAs wait for one another: all of them have to be resident
    attr[0].val.cooperative = 1;
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, m_gu, m_dn, m_sgu, m_sdn, a);
}
template <class X>
static cudaError_t launch_for(const Args& a, const mok_few_args* w, cudaStream_t s) {
    // Two matrix tiles of weight rows per unit halve the loads of the tokens' fragments; with up to 16 tokens these are few, and
    // smaller units spread more evenly.
    if (a.T <= 8) return launch<X, 1, 1>(a, w, s);
    if (a.T <= 16) return launch<X, 1, 2>(a, w, s);
    if (a.T <= 32) return launch<X, 2, 4>(a, w, s);
    return launch<X, 2, 8>(a, w, s);
}
static bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace few
}  // namespace mok

using namespace mok;

extern "C" {

size_t mok_few_workspace_bytes(int T, int H, int I, int I_shared, int E, int k) {
    few::Layout L;
    return few::layout(T, H, I, I_shared, E, k, &L) ? L.total : 0;
}

int mok_moe_few(const mok_few_args* a) {
    if (!a) return MOK_ERR_NULL;
    few::Layout L;
    if (!few::layout(a->T, a->H, a->I, a->I_shared, a->E, a->k, &L) || (a->type != MOK_TYPE_BF16 && a->type != MOK_TYPE_F16) ||
        (a->score != MOK_SCORE_SOFTMAX && a->score != MOK_SCORE_SIGMOID) || a->n_groups < 1 || a->n_groups > 32 || a->E % a->n_groups ||
        a->topk_groups < 1 || a->topk_groups > a->n_groups || a->k > a->topk_groups * (a->E / a->n_groups) ||
        (a->n_groups > 1 && (a->group_top < 1 || a->group_top > 2 || a->group_top > a->E / a->n_groups)) ||
        (a->T > 1 && (a->x_stride < a->H || a->out_stride < a->H || (a->add && a->add_stride < a->H))))
        return MOK_ERR_SHAPE;
    if ((a->I_shared == 0) != (!a->W_shared_gate_up && !a->W_shared_down)) return MOK_ERR_SHAPE;
    if (a->T == 0) return MOK_OK;
    if (!a->x || !a->W_router || !a->W_gate_up || !a->W_down || !a->out || (a->I_shared && (!a->W_shared_gate_up || !a->W_shared_down)))
        return MOK_ERR_NULL;
    if (!few::aligned(a->x, 16) || (a->T > 1 && a->x_stride % 8) || !few::aligned(a->W_router, 16) || !few::aligned(a->W_gate_up, 16) ||
        !few::aligned(a->W_down, 16) || !few::aligned(a->W_shared_gate_up, 16) || !few::aligned(a->W_shared_down, 16) ||
        !few::aligned(a->out, 2) || !few::aligned(a->add, 2) || !few::aligned(a->router_bias, 4) || !few::aligned(a->bias, 4) ||
        !few::aligned(a->topk_idx, 4) || !few::aligned(a->topk_w, 4))
        return MOK_ERR_ALIGN;
    if (!a->workspace || !few::aligned(a->workspace, 256) || a->workspace_bytes < L.total) return MOK_ERR_WORKSPACE;
    char* ws = reinterpret_cast<char*>(a->workspace);
    few::Args g = {};
    g.x = a->x;
    g.W_router = a->W_router;
    g.router_bias = a->router_bias;
    g.add = a->add;
    g.x_stride = a->x_stride;
    g.add_stride = a->add_stride;
    g.out_stride = a->out_stride;
    g.T = a->T; g.H = a->H; g.I = a->I; g.Is = a->I_shared; g.E = a->E; g.k = a->k;
    g.parts = L.parts;
    g.starve = a->debug == MOK_DEBUG_STARVE;
    g.number = few::call_number();
    g.wait_ns = g.starve ? 2000000ull : tc::WAIT_LIMIT_NS;
    g.gate = {nullptr, a->bias, 0, a->T, a->E, a->k, a->score == MOK_SCORE_SOFTMAX, a->n_groups, a->topk_groups, a->group_top,
              a->renormalise != 0, a->scale, a->topk_idx ? a->topk_idx : reinterpret_cast<int32_t*>(ws + L.idx),
              a->topk_w ? a->topk_w : reinterpret_cast<float*>(ws + L.w)};
    g.out = a->out;
    g.header = reinterpret_cast<WsHeader*>(ws);
    g.signals = reinterpret_cast<few::Signals*>(ws + L.signals);
    g.counters = reinterpret_cast<int32_t*>(ws + L.counters);
    g.logits = reinterpret_cast<float*>(ws + L.logits);
    g.h = ws + L.h;
    g.hs = ws + L.hs;
    g.y = reinterpret_cast<float*>(ws + L.y);
    cudaStream_t s = reinterpret_cast<cudaStream_t>(a->stream);
    const cudaError_t e = a->type == MOK_TYPE_BF16 ? few::launch_for<__nv_bfloat16>(g, a, s) : few::launch_for<__half>(g, a, s);
    return e == cudaSuccess ? MOK_OK : cuda_fail(e);
}

}  // extern "C"
