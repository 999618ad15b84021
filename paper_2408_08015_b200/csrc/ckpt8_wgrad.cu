// Weight and bias gradient of a linear layer from the 8-bit checkpoint of its input:
//   dw[o][i] = sum over r of dy[r][o] * q[r][i] 2^(S[r][i / 32] - 133),   db[o] = sum over r of dy[r][o].
//
// One product on the tensor cores with the rows as the reduction, both operands MN-major as they lie in memory.  A kept value is a bfloat16 number,
// so the codes become the exact operand in registers on their way to shared memory and never exist in 16 bits in global memory.  float32 gradients
// are cut into three bfloat16 terms of 8 bits each, exact too but for bits below 2^-133, and three instructions take the place of one.
//
// What bounds it is shared memory, where the warps write the operand that the tensor core reads next to the other, and the issue of the warps that convert
// and of the one that feeds the tensor core: a step of 64 rows takes 750 to 800 cycles, 605 with the conversion left out, the instructions 512.  4096 -> 4096 over 32 768
// rows: 1.09 to 1.12 ms from one B200 to another, 0.98 to 1.01 PFLOP/s, at the 1.15 to 1.2 GHz that the power cap leaves; 512 -> 2048 over 16 384 rows: 50 to 52 us, 28 of them steps.  A pair of CTAs
// therefore shares one tile of 256 output by up to 256 input channels (tcgen05, cta_group::2): each holds 128 output channels of dy and half of the
// input channels, and converts half of the codes.  A step is 64 rows.
//   warp 0        tiled tensor copies of dy (the leading CTA's barrier counts the bytes of both)
//   warp 1        of the leading CTA: the instructions of the pair
//   warp 2        announces what the CTA's warps have written
//   warps 4-7     accumulators to memory
//   warps 8-23    codes to bfloat16, in two sets that take the steps in turn (where dy goes through registers: warps 8-15)
//   warps 16-31   where dy is float32, or does not lie as copies need it: dy through registers, in two sets as well
// db is the product with a column of ones, taken by the tiles of the first input channels.
//
// Every pair takes whole tiles while there is one for every pair, so that pairs that share operands read them from L2 at the same time.  What is
// left over is cut along the rows, into as many parts as suit the pairs, and a second kernel adds the parts in order.
#include <algorithm>

#include "../../include/asteroid.h"
#include "ckpt8.cuh"
#include "kernels.h"
#include "tc_common.cuh"
#include "tma.cuh"

namespace ast {
namespace {

using namespace q8;
using namespace tc;

constexpr int TILE_M = 256, HALF_M = 128, ROWS = 64;               // output channels of a pair and of a CTA; rows of a step
constexpr int PANEL = ROWS * 128;                                   // 64 channels of a step
constexpr int A_BYTES = 2 * PANEL, B_BYTES = 2 * PANEL;
constexpr int ONES_BYTES = 16 * 128;
constexpr int EPI_WARP = 4, Q_WARP = 8, Q_WARPS = 8, A_WARP = 16, A_WARPS = 8;      // Q_WARPS: of a set
// Columns of tensor memory: accumulators, those of the bias gradient (32 is the least a pair's instruction takes), and the sums of all accumulators but the
// first 32, which are held in shared memory.
constexpr int DB_COL = 256, DB_N = 32, SUM_COL = 288, NEAR_COLS = 32;
constexpr int NEAR_BYTES = (NEAR_COLS + 1) * HALF_M * 4, TURN_BYTES = 4 * 32 * 17 * 4;

enum { DY_COPY = 0, DY_F32 = 1, DY_F32_ANY = 2, DY_BF16_ANY = 3 };  // how dy is read
template <int MODE> struct Form {
    static constexpr int TERMS = MODE == DY_F32 || MODE == DY_F32_ANY ? 3 : 1;
    // The tensor core cuts a sum to 24 bits at every addition instead of rounding it, so that sums shrink by some 2^-24 of themselves with each of the four
    // instructions of a step: over 32768 rows the gradient was off by 2.8e-5 of its norm, over 4096 by 2.4e-6.  After SPAN steps the accumulators are therefore added
    // to sums of float32, rounded.  Normal values on both sides: 8e-7 over 32768 rows.  The worst case, sums of one sign: the at most 112 additions of a span cut up to
    // 2^-23 each, 1.4e-5, and the sums of the spans round, 2^-24 for each span: 6.3e-6 at 40 000 rows of float32 dy, growing with the rows.
    static constexpr int SPAN = TERMS == 3 ? 6 : 28;
    static constexpr int SETS = MODE == DY_COPY ? 2 : 1;                 // of warps that convert codes
    static constexpr int AHEAD = MODE == DY_COPY ? 1 : 2;                // of its steps whose codes a set requests ahead (three: 4 % slower at 4096 -> 4096)
    static constexpr int A_SETS = 2;                                     // of warps that dy goes through
    static constexpr int S = TERMS == 3 ? 3 : 6;                         // steps in shared memory
    static constexpr int STAGE = TERMS * A_BYTES + B_BYTES;
    static constexpr int THREADS = (Q_WARP + SETS * Q_WARPS + (MODE == DY_COPY ? 0 : A_SETS * A_WARPS)) * 32;
    static constexpr int SMEM = S * STAGE + ONES_BYTES + NEAR_BYTES + TURN_BYTES + 1024;
};

struct WArgs {
    const unsigned char *codes, *exps;
    const void* dy;
    size_t lddy, pitch, groups;
    unsigned rows;
    int ci, co, nt;                // nt: input channels of a tile, 128 or 256
    int tm, tn;                    // tiles
    int steps;                     // of all rows
    int whole, rest, parts;        // tiles taken whole; tiles cut into parts (parts == 1: not cut)
    float *dw, *db, *part;         // part [parts][rest][2] blocks of part_floats(nt)
    int add;
    int* err;                      // device error word, may be null
    int silent_after;              // self-test: steps after which the first pair's leading CTA announces nothing more
};
__host__ __device__ inline size_t part_floats(int nt) { return (size_t)HALF_M * nt + HALF_M; }     // a CTA's accumulators, then its bias gradient

// Unit u of work: a whole tile or a part of one, and its steps
struct Unit {
    int tile, part, k0, k1;
    bool cut;
};
__device__ __forceinline__ Unit unit_of(const WArgs& a, int u) {
    if (u < a.whole) return Unit{u, 0, 0, a.steps, false};
    const int v = u - a.whole, p = v / a.rest;
    return Unit{a.whole + v - p * a.rest, p, (int)((long long)a.steps * p / a.parts), (int)((long long)a.steps * (p + 1) / a.parts), a.parts > 1};
}
__device__ __forceinline__ int units(const WArgs& a) { return a.whole + a.rest * a.parts; }
// Tiles in blocks of 8 rows of tiles, column by column: those that run at the same time form a rectangle and share operands
__device__ __forceinline__ void tile_at(const WArgs& a, int t, int* m, int* n) {
    const int per = 8 * a.tn, b = t / per, h = min(8, a.tm - 8 * b), q = t - b * per;
    *n = q / h;
    *m = 8 * b + q - *n * h;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t leader_addr(uint32_t addr) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// The same without ordering the CTA's generic accesses for the other CTA, which would wait for every request of the thread: what is announced is read by the
// tensor core of the announcing CTA, behind a proxy fence.
__device__ __forceinline__ void announce_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// bounded (PROBE: some milliseconds); gives up as soon as another role of the CTA has
template <bool PROBE> __device__ __forceinline__ bool wait_for(uint32_t mbar, uint32_t parity, volatile int* gave_up) {
    return mbar_wait_abortable(mbar, parity, gave_up, PROBE ? 1u << 14 : WAIT_LIMIT);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t test_wait(uint32_t mbar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(mbar), "r"(parity)
        : "memory");
    return ok;
}
// ... by a whole warp, with one answer
template <bool PROBE> __device__ __forceinline__ bool warp_wait_for(uint32_t mbar, uint32_t parity, volatile int* gave_up) {
    if (__all_sync(0xffffffffu, mbar_try_wait(mbar, parity))) return true;
    return __all_sync(0xffffffffu, wait_for<PROBE>(mbar, parity, gave_up));
}
__device__ __forceinline__ void pair_load_2d(uint32_t dst, const CUtensorMap* m, int c0, int c1, uint32_t mbar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
                 "l"(reinterpret_cast<uint64_t>(m)), "r"(mbar), "r"(c0), "r"(c1)
                 : "memory");
}
// MN-major operand, 128-byte swizzle: panels of 64 channels PANEL bytes apart, groups of 8 rows 1024 bytes apart.  The lower word of its descriptor (16 rows
// on: + 2048 / 16) and the upper one.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr) { return ((addr & 0x3FFFFu) >> 4) | (uint32_t)(PANEL >> 4) << 16; }
constexpr uint32_t DESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;
// D (+)= A B over the 64 rows of a step: four instructions, the first of which adds to what is there if `more`; B moves on by b_next
__device__ __forceinline__ void pair_mma4(uint32_t d, uint32_t alo, uint32_t blo, uint32_t b_next, uint32_t idesc, uint32_t more, uint32_t leader) {
    asm volatile(
        "{\n"
        ".reg .pred p, q;\n"
        ".reg .b32 a1, a2, a3, b1, b2, b3;\n"
        ".reg .b64 da, db;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "setp.ne.b32 q, %6, 0;\n"
        "add.u32 a1, %1, 128;\n"
        "add.u32 a2, %1, 256;\n"
        "add.u32 a3, %1, 384;\n"
        "add.u32 b1, %2, %3;\n"
        "add.u32 b2, b1, %3;\n"
        "add.u32 b3, b2, %3;\n"
        "mov.b64 da, {%1, %7};\n"
        "mov.b64 db, {%2, %7};\n"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, p;\n"
        "mov.b64 da, {a1, %7};\n"
        "mov.b64 db, {b1, %7};\n"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n"
        "mov.b64 da, {a2, %7};\n"
        "mov.b64 db, {b2, %7};\n"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n"
        "mov.b64 da, {a3, %7};\n"
        "mov.b64 db, {b3, %7};\n"
        "@q tcgen05.mma.cta_group::2.kind::f16 [%0], da, db, %4, 1;\n"
        "}\n" ::"r"(d),
        "r"(alo), "r"(blo), "r"(b_next), "r"(idesc), "r"(more), "r"(leader), "r"(DESC_HI)
        : "memory");
}
// arrives at the barrier of this place in both CTAs when the instructions issued so far are done
__device__ __forceinline__ void pair_commit(uint32_t mbar, uint32_t leader) {
    asm volatile(
        "{\n"
        ".reg .pred q;\n"
        "setp.ne.b32 q, %1, 0;\n"
        "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %2;\n"
        "}\n" ::"r"(mbar),
        "r"(leader), "h"((uint16_t)3)
        : "memory");
}
// D = float32, A = B = bfloat16, both MN-major, M = 256
__device__ __forceinline__ uint32_t idesc_of(int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
}

// Four codes as two pairs of bfloat16, the first and third, then the second and fourth (the accumulators' columns are put right when they are stored).
// The bits of q + 128, eight of them, are the bfloat16 number (q + 128) 2^-133, across the border from subnormal to normal numbers; times 2^127, less 2, that
// is q / 64, exactly.  m: 64 times the group's scale.  The conversion is bound by the integer pipe, whose work this keeps to three instructions for four codes.
__device__ __forceinline__ uint32_t codes2(uint32_t w, __nv_bfloat162 m) {
    const uint32_t t = (w & 0x00ff00ffu) ^ 0x00800080u, two127 = 0x7f007f00u, minus2 = 0xc000c000u;
    const __nv_bfloat162 q = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&t), *reinterpret_cast<const __nv_bfloat162*>(&two127),
                                     *reinterpret_cast<const __nv_bfloat162*>(&minus2));
    const __nv_bfloat162 r = __hmul2(q, m);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint4 codes8(uint2 w, __nv_bfloat162 m) { return make_uint4(codes2(w.x, m), codes2(w.x >> 8, m), codes2(w.y, m), codes2(w.y >> 8, m)); }
// 2^(S - 127), or NaN
__device__ __forceinline__ __nv_bfloat162 scale64(unsigned s) {
    const uint32_t h = s == NOT_FINITE ? 0x7fc0u : s << 7, w = h | h << 16;
    return *reinterpret_cast<const __nv_bfloat162*>(&w);
}

// A float32 number as three bfloat16 numbers, cut (not rounded: the largest must not become infinite).  Infinities and NaN stand in the first alone.
__device__ __forceinline__ void cut3(float f, uint32_t* t) {
    const uint32_t u = __float_as_uint(f);
    const bool odd = (u & 0x7f800000u) == 0x7f800000u;
    t[0] = odd && (u & 0x7fffffu) ? 0x7fc00000u : u & 0xffff0000u;
    const float r = odd ? 0.f : f - __uint_as_float(t[0]);
    t[1] = __float_as_uint(r) & 0xffff0000u;
    t[2] = __float_as_uint(r - __uint_as_float(t[1])) & 0xffff0000u;
}

// PROBE: the self-test's, with short waits, which are made to run out
template <int MODE, bool PROBE> __global__ void __launch_bounds__(Form<MODE>::THREADS, 1) wgrad_kernel(const __grid_constant__ CUtensorMap tm_dy, const WArgs a) {
    constexpr int S = Form<MODE>::S, STAGE = Form<MODE>::STAGE, TERMS = Form<MODE>::TERMS, SPAN = Form<MODE>::SPAN;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[3 * S + 2];
    __shared__ uint32_t tmem_slot;
    __shared__ int gave_up_store;
    volatile int* gave_up = &gave_up_store;
    uint8_t* base = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);       // of a step: dy (its terms), then the converted codes
    uint8_t* ones = base + S * STAGE;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t rank = cluster_rank();
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1, n_units = units(a);
    // "full" and "accumulators read": the leading CTA's count for both
    const uint32_t bar0 = smem_u32(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (S + s); };
    auto written = [&](int s) { return bar0 + 8u * (2 * S + s); };
    const uint32_t acc_ready = bar0 + 8u * (3 * S), acc_read = acc_ready + 8u;

    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(full(s), MODE == DY_COPY ? 3 : 2);
            mbar_init(empty(s), 1);
            mbar_init(written(s), Q_WARPS + (MODE == DY_COPY ? 0 : A_WARPS));
        }
        mbar_init(acc_ready, 1);
        mbar_init(acc_read, 8);
        gave_up_store = 0;
        if (MODE == DY_COPY) tma::prefetch_map(&tm_dy);
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (warp == 2)
        for (int i = lane; i < ONES_BYTES / 16; i += 32) reinterpret_cast<uint4*>(ones)[i] = make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u);
    __syncwarp();
    fence_async_smem();
    fence_before_sync();
    cluster_barrier();
    fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_wait();
    pdl_launch();

    // The loops of warps 0 to 3 are kept to a few dozen instructions a step: beside the converting warps each takes 10 cycles, and a step is to take 512.
    if (warp == 0) {
        if (MODE == DY_COPY && lane == 0) {
            const uint32_t to = leader_addr(full(0));
            int s = 0;
            uint32_t parity = 1;                         // of a barrier that nothing has arrived at: waits of the first turn pass
            bool ok = true;
            for (int u = pair; u < n_units && ok; u += pairs) {
                const Unit w = unit_of(a, u);
                int m, n;
                tile_at(a, w.tile, &m, &n);
                const int x = m * TILE_M + (int)rank * HALF_M;
                for (int k = w.k0; k < w.k1; ++k) {
                    const int y = k * ROWS;              // below 2^31; the row behind the last step's need not be
                    if (!(ok = wait_for<PROBE>(empty(s), parity, gave_up))) break;
                    const uint32_t dst = smem_u32(base) + s * STAGE;
                    if (rank == 0) mbar_expect_tx(full(s), 2 * A_BYTES);
                    pair_load_2d(dst, &tm_dy, x, y, to + 8u * s);
                    pair_load_2d(dst + PANEL, &tm_dy, x + 64, y, to + 8u * s);
                    if (++s == S) {
                        s = 0;
                        parity ^= 1u;
                    }
                }
            }
            // copies in flight when a wait was given up land long before this ends
            for (int i = 0; !ok && i < 10000; ++i) __nanosleep(1000);
        }
    } else if (warp == 1) {
        if (rank == 0) {
            // The instructions of a step take the tensor core 512 cycles; this warp shares its scheduler with the converting ones and must not take longer
            const uint32_t leader = elect_leader();
            const uint32_t idesc = idesc_of(a.nt), idesc_db = idesc_of(DB_N);
            const uint32_t ones0 = desc_lo(smem_u32(ones)), d0 = desc_lo(smem_u32(base));
            int s = 0, done = 0;
            uint32_t parity = 0, ready = 0;
            bool ok = true;
            for (int u = pair; u < n_units && ok; u += pairs) {
                const Unit w = unit_of(a, u);
                int m, n;
                tile_at(a, w.tile, &m, &n);
                const bool bias = a.db && n == 0;
                uint32_t more = 0;
                for (int k = w.k0, left = 0; k < w.k1; ++k, --left) {
                    if (!left) {                         // a span begins
                        if (done && !(ok = warp_wait_for<PROBE>(acc_read, (uint32_t)((done - 1) & 1), gave_up))) break;
                        left = SPAN;
                        more = 0;
                        ++done;
                    }
                    // a look at a barrier takes 200 cycles while the converting warps use shared memory: the next step's is asked for before this one's work is issued
                    if (!__all_sync(0xffffffffu, ready) && !(ok = warp_wait_for<PROBE>(full(s), parity, gave_up))) break;
                    fence_after_sync();
                    const int ns = s + 1 == S ? 0 : s + 1;
                    const uint32_t np = ns ? parity : parity ^ 1u;
                    ready = test_wait(full(ns), np);
                    const uint32_t da = d0 + (uint32_t)s * (STAGE / 16), db = da + TERMS * (A_BYTES / 16);
#pragma unroll
                    for (int t = TERMS - 1; t >= 0; --t) {
                        pair_mma4(tmem, da + t * (A_BYTES / 16), db, 128u, idesc, more, leader);
                        if (bias) pair_mma4(tmem + DB_COL, da + t * (A_BYTES / 16), ones0, 0u, idesc_db, more, leader);
                        more = 1;
                    }
                    pair_commit(empty(s), leader);
                    if (left == 1 || k + 1 == w.k1) pair_commit(acc_ready, leader);
                    s = ns;
                    parity = np;
                }
            }
            for (int i = 0; !ok && i < 10000; ++i) __nanosleep(1000);            // ... and instructions in flight end
        }
    } else if (warp == 2) {
        // What the CTA's converting warps have written, made visible to the tensor core and announced to the leading CTA.  A warp of its own does that: the
        // fence waits for all of a thread's requests, and the converting warps have exponents in flight.
        if (lane == 0) {
            const uint32_t to = leader_addr(full(0));
            int s = 0;
            uint32_t parity = 0;
            bool ok = true;
            int announced = 0;
            for (int u = pair; u < n_units && ok; u += pairs) {
                const Unit w = unit_of(a, u);
                for (int k = w.k0; k < w.k1; ++k) {
                    if (!(ok = wait_for<PROBE>(written(s), parity, gave_up))) break;
                    if (PROBE && !(ok = blockIdx.x || announced++ < a.silent_after)) break;
                    fence_async_smem();
                    announce_at(to + 8u * s);
                    if (++s == S) {
                        s = 0;
                        parity ^= 1u;
                    }
                }
            }
        }
    } else if (warp >= EPI_WARP && warp < EPI_WARP + 4) {
        const int q = warp & 3, row = q * 32 + lane;
        const uint32_t read_at = leader_addr(acc_read);
        const bool vec = a.ci % 4 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 16 == 0;
        float* const turn = reinterpret_cast<float*>(ones + ONES_BYTES + NEAR_BYTES) + q * (32 * 17);        // of this warp
        const uint32_t mine = tmem + ((uint32_t)(q * 32) << 16), sums = mine + SUM_COL - NEAR_COLS;     // column c's sum: sums + c
        float* const here = reinterpret_cast<float*>(ones + ONES_BYTES) + row;      // [NEAR_COLS sums, bias gradient][128 rows]
        // Spans read; negative from the first wait on that ran out: nothing comes behind it, and the barrier's other parity, which the next wait would ask for, has long
        // passed.  This warp then reads no accumulators and announces none as read (the instructions stop, and with them the other CTA's warps); its results are NaN.
        int done = 0;
        for (int u = pair; u < n_units; u += pairs) {
            const Unit w = unit_of(a, u);
            int m, n;
            tile_at(a, w.tile, &m, &n);
            for (int k = w.k0; k < w.k1; k += SPAN, ++done) {
                const bool first = k == w.k0;
                if (done >= 0 && !warp_wait_for<PROBE>(acc_ready, (uint32_t)(done & 1), gave_up)) done = -1;
                if (done < 0) break;
                fence_after_sync();
                // 16 columns at a time: with 32 registers spill, and 4096 -> 4096 takes 4 % longer
                for (int g = 0; g < a.nt; g += 16) {
                    uint32_t r[16], t[16];
                    const bool near = g < NEAR_COLS;
                    tmem_ld16_issue(mine + g, r);
                    if (!first && !near) tmem_ld16_issue(sums + g, t);
                    tmem_ld_wait();
                    tmem_ld_pin16(r);
                    if (!first) {
                        if (near) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) t[e] = __float_as_uint(here[(g + e) * HALF_M]);
                        }
                        tmem_ld_pin16(t);
#pragma unroll
                        for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(t[e]) + __uint_as_float(r[e]));
                    }
                    if (near) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) here[(g + e) * HALF_M] = __uint_as_float(r[e]);
                    } else tmem_st16(sums + g, r);
                }
                if (a.db && n == 0) {
                    float b[8];
                    tmem_ld8(mine + DB_COL, b);
                    here[NEAR_COLS * HALF_M] = first ? b[0] : here[NEAR_COLS * HALF_M] + b[0];
                }
                tmem_st_wait();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) arrive_at(read_at);
            }
            const int o = m * TILE_M + (int)rank * HALF_M + row, i0 = n * a.nt;
            float* part = w.cut ? a.part + (((size_t)w.part * a.rest + (w.tile - a.whole)) * 2 + rank) * part_floats(a.nt) : nullptr;
            for (int g = 0; g < a.nt; g += 16) {
                float r[16], v[16];                      // v: channels in order, see codes2
                if (g < NEAR_COLS) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) r[e] = here[(g + e) * HALF_M];
                } else tmem_ld16(sums + g, r);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = done >= 0 ? r[(e & 3) == 1 ? e + 1 : (e & 3) == 2 ? e - 1 : e] : __uint_as_float(0x7fc00000u);
                if (w.cut) {
                    // four columns of 32 rows side by side
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        reinterpret_cast<float4*>(part)[(size_t)((g + e) >> 2) * HALF_M + row] = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                } else if (vec) {
                    float* d = a.dw + (size_t)o * a.ci + i0 + g;
                    const int left = o < a.co ? a.ci - i0 - g : 0;
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        if (e >= left) continue;
                        float4 x = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
                        if (a.add) {
                            const float4 y = *reinterpret_cast<const float4*>(d + e);
                            x = make_float4(x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w);
                        }
                        *reinterpret_cast<float4*>(d + e) = x;
                    }
                } else {
                    // Through shared memory, so that a row's 16 columns are written (and, where they are added to, read) side by side: 336 rows, 3858 -> 2760 85 -> 59 us.
                    // Rows of whole vectors take longer this way (300 rows, 1280 -> 1000 20 and 27 us).
                    __syncwarp();
#pragma unroll
                    for (int e = 0; e < 16; ++e) turn[lane * 17 + e] = v[e];
                    __syncwarp();
                    const int c = i0 + g + (lane & 15), o0 = o - lane + (lane >> 4);
                    float* d = a.dw + (size_t)o0 * a.ci + c;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float x = turn[(2 * e + (lane >> 4)) * 17 + (lane & 15)];
                        if (c < a.ci && o0 + 2 * e < a.co) *d = a.add ? *d + x : x;
                        d += 2 * (size_t)a.ci;
                    }
                }
            }
            if (a.db && n == 0) {
                const float b = done >= 0 ? here[NEAR_COLS * HALF_M] : __uint_as_float(0x7fc00000u);
                if (w.cut) part[(size_t)HALF_M * a.nt + row] = b;
                else if (o < a.co) a.db[o] = a.add ? a.db[o] + b : b;
            }
        }
    } else if (warp >= Q_WARP && warp < Q_WARP + Form<MODE>::SETS * Q_WARPS) {
        // A warp has 8 rows, a lane 16 channels of two of them: 8 lanes read the 128 bytes of a row.  They write it as 16 chunks of 8 channels, the even ones of
        // one panel next to the odd ones of the other, which the swizzle places in different banks.  The sets of warps take the steps in turn.  
        constexpr int SETS = Form<MODE>::SETS, AHEAD = Form<MODE>::AHEAD;
        const int set = (warp - Q_WARP) / Q_WARPS, row = (warp & 7) * 8 + (lane >> 3), u16 = lane & 7, panel = u16 >> 2;
        const int half_cols = a.nt >> 1, col0 = (int)rank * half_cols + u16 * 16;
        const bool have = u16 * 16 < half_cols;
        uint4 raw[AHEAD][2];
        unsigned ex[AHEAD][2];
        // the request cursor: unit, this set's steps left in it, this lane's places, the rows from its first one to the end (none where it has no columns)
        int ru = pair, skip = set, steps = 0, left = 0;
        const unsigned char *pc = nullptr, *pe = nullptr;
        const size_t next_c = SETS * ROWS * a.pitch, next_e = SETS * ROWS * a.groups, row4_c = 4 * a.pitch, row4_e = 4 * a.groups;
        auto open = [&]() {
            for (; ru < n_units; ru += pairs) {
                const Unit w = unit_of(a, ru);
                const int have_steps = w.k1 - w.k0 - skip;
                if (have_steps > 0) {
                    int m, n;
                    tile_at(a, w.tile, &m, &n);
                    const size_t col = (size_t)n * a.nt + col0, r0 = (size_t)(w.k0 + skip) * ROWS + row;
                    pc = a.codes + r0 * a.pitch + col;
                    pe = a.exps + r0 * a.groups + col / GROUP;
                    left = have && col < a.pitch ? (int)((long long)a.rows - (long long)r0) : 0;
                    steps = (have_steps + SETS - 1) / SETS;
                    skip += steps * SETS - (w.k1 - w.k0);        // into the next unit
                    return;
                }
                skip = -have_steps;
            }
        };
        auto request = [&](uint4* r, unsigned* e) {
            if (ru >= n_units) return;
            if (left > 4) {
                r[0] = __ldg(reinterpret_cast<const uint4*>(pc));
                r[1] = __ldg(reinterpret_cast<const uint4*>(pc + row4_c));
                e[0] = __ldg(pe);
                e[1] = __ldg(pe + row4_e);
            } else {
                const bool in = left > 0;
                r[0] = in ? __ldg(reinterpret_cast<const uint4*>(pc)) : make_uint4(0, 0, 0, 0);
                e[0] = in ? __ldg(pe) : 8u;
                r[1] = make_uint4(0, 0, 0, 0);
                e[1] = 8u;
            }
            pc += next_c;
            pe += next_e;
            left -= SETS * ROWS;
            if (--steps == 0) {
                ru += pairs;
                open();
            }
        };
        open();
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) request(raw[j], ex[j]);
        int total = 0;
        for (int u = pair; u < n_units; u += pairs) {
            const Unit w = unit_of(a, u);
            total += w.k1 - w.k0;
        }
        const int at = 2 * (u16 & 3), sw = row & 7;                  // 4 rows on the swizzle differs in its third bit
        uint8_t* const b0 = base + TERMS * A_BYTES + panel * PANEL + row * 128;
        const uint32_t o0 = (uint32_t)(((at + panel) ^ sw) << 4), o1 = (uint32_t)(((at + 1 - panel) ^ sw) << 4);
        bool ok = true;
        int s = set;
        uint32_t parity = 1;
        for (int i0 = set; i0 < total && ok; i0 += AHEAD * SETS)
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (i0 + j * SETS >= total || !ok) continue;
                if (!(ok = warp_wait_for<PROBE>(empty(s), parity, gave_up))) continue;
                if (have) {
                    uint8_t* b = b0 + s * STAGE;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const __nv_bfloat162 m = scale64(ex[j][i]);
                        const uint4 r = raw[j][i];
                        const uint2 lo = make_uint2(r.x, r.y), hi = make_uint2(r.z, r.w);
                        *reinterpret_cast<uint4*>(b + i * 512 + (o0 ^ (i * 64))) = codes8(panel ? hi : lo, m);
                        *reinterpret_cast<uint4*>(b + i * 512 + (o1 ^ (i * 64))) = codes8(panel ? lo : hi, m);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(written(s));
                s += SETS;
                if (s >= S) {
                    s -= S;
                    parity ^= 1u;
                }
                request(raw[j], ex[j]);
            }
    } else if (MODE != DY_COPY && warp >= A_WARP) {
        // dy through registers: a warp has 8 rows, a lane two channels of each of a row's two panels, so that a request and a store take a row's 64 channels side by side
        // (two sets of warps that take the steps in turn: one's requests are on the way while the other writes)
        const int set = (warp - A_WARP) / A_WARPS, row0 = ((warp - A_WARP) & 7) * 8;
        const uint32_t at = (uint32_t)row0 * 128u + (uint32_t)(lane & 3) * 4u;
        int it = 0;
        bool ok = true;
        for (int u = pair; u < n_units && ok; u += pairs) {
            const Unit w = unit_of(a, u);
            int m, n;
            tile_at(a, w.tile, &m, &n);
            const int o0 = m * TILE_M + (int)rank * HALF_M + 2 * lane;
            for (int k = w.k0; k < w.k1; ++k, ++it) {
                if (it % Form<MODE>::A_SETS != set) continue;
                const int s = it % S;
                float2 f[8][2];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const size_t rr = (size_t)k * ROWS + row0 + r;
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        const int o = o0 + 64 * p;
                        f[r][p] = make_float2(0.f, 0.f);
                        if (rr >= a.rows) continue;
                        if (MODE == DY_F32) {
                            if (o < a.co) f[r][p] = __ldg(reinterpret_cast<const float2*>(static_cast<const float*>(a.dy) + rr * a.lddy + o));
                        } else if (MODE == DY_F32_ANY) {
                            const float* q = static_cast<const float*>(a.dy) + rr * a.lddy + o;
                            if (o < a.co) f[r][p].x = __ldg(q);
                            if (o + 1 < a.co) f[r][p].y = __ldg(q + 1);
                        } else {
                            const unsigned short* q = static_cast<const unsigned short*>(a.dy) + rr * a.lddy + o;
                            // as they are: anything done to them here waits for each before the next is requested (512 -> 2048, 16384 rows: 250 us and 95)
                            if (o < a.co) f[r][p].x = __uint_as_float((unsigned)__ldg(q));
                            if (o + 1 < a.co) f[r][p].y = __uint_as_float((unsigned)__ldg(q + 1));
                        }
                    }
                }
                if (!(ok = warp_wait_for<PROBE>(empty(s), (uint32_t)((it / S + 1) & 1), gave_up))) break;
                uint8_t* const d = base + s * STAGE + at;
#pragma unroll
                for (int r = 0; r < 8; ++r)
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        uint32_t x[3], y[3];
                        if (TERMS == 3) {
                            cut3(f[r][p].x, x);
                            cut3(f[r][p].y, y);
                        } else {
                            x[0] = __float_as_uint(f[r][p].x);
                            y[0] = __float_as_uint(f[r][p].y);
                        }
#pragma unroll
                        for (int t = 0; t < TERMS; ++t)
                            *reinterpret_cast<uint32_t*>(d + t * A_BYTES + p * PANEL + r * 128 + (((lane >> 2) ^ r) << 4)) = __byte_perm(x[t], y[t], TERMS == 3 ? 0x7632 : 0x5410);
                    }
                __syncwarp();
                if (lane == 0) mbar_arrive(written(s));
            }
        }
    }
    __syncwarp();
    fence_before_sync();
    cluster_barrier();
    if (tid == 0 && gave_up_store && a.err) atomicExch(a.err, 1);
    __syncwarp();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

// The parts of the tiles that were cut, added in order.  A thread has one row and four columns of a CTA's half tile.
__global__ void __launch_bounds__(256) sum_parts_kernel(const WArgs a) {
    pdl_wait();
    pdl_launch();
    const int quads = a.nt / 4 * HALF_M;                                 // of a half tile
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x, per = (size_t)quads + HALF_M, total = per * 2 * a.rest;
    if (at >= total) return;
    const int half = (int)(at / per), e = (int)(at - half * per);
    int m, n;
    tile_at(a, a.whole + (half >> 1), &m, &n);
    const size_t step = (size_t)a.rest * 2 * part_floats(a.nt);
    const float* p = a.part + (size_t)half * part_floats(a.nt);
    const int o_base = m * TILE_M + (half & 1) * HALF_M;
    if (e >= quads) {
        const int o = o_base + e - quads;
        if (!a.db || n || o >= a.co) return;
        float s = a.add ? a.db[o] : 0.f;
        for (int k = 0; k < a.parts; ++k) s += p[k * step + (size_t)HALF_M * a.nt + (e - quads)];
        a.db[o] = s;
        return;
    }
    const int row = e % HALF_M, c = e / HALF_M * 4, o = o_base + row, i = n * a.nt + c;
    if (o >= a.co || i >= a.ci) return;
    float* d = a.dw + (size_t)o * a.ci + i;
    const int left = min(4, a.ci - i);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.add)
        for (int h = 0; h < left; ++h) s[h] = d[h];
#pragma unroll 4
    for (int k = 0; k < a.parts; ++k) {
        const float4 v = reinterpret_cast<const float4*>(p + k * step)[e];
        s[0] += v.x;
        s[1] += v.y;
        s[2] += v.z;
        s[3] += v.w;
    }
    if (left == 4 && a.ci % 4 == 0 && reinterpret_cast<uintptr_t>(a.dw) % 16 == 0) *reinterpret_cast<float4*>(d) = make_float4(s[0], s[1], s[2], s[3]);
    else
        for (int h = 0; h < left; ++h) d[h] = s[h];
}

// How the tiles are dealt out.  A step of 64 rows takes a pair 0.45 us (float32 1.5; bfloat16 dy through registers some 0.9, which the plan does not tell apart), starting a unit and
// storing its accumulators some 5 us; parts are written and read again at 6 bytes a picosecond by a kernel of 3 us.
struct Plan {
    int nt, tm, tn, steps, pairs, whole, rest, parts, all;
    double step_us;
    Plan(size_t rows, int ci, int co, int dtype) {
        nt = ci > 128 ? 256 : 128;
        tm = (co + TILE_M - 1) / TILE_M;
        tn = (ci + nt - 1) / nt;
        steps = (int)((rows + ROWS - 1) / ROWS);
        all = sm_count() / 2;
        const int tiles = tm * tn;
        whole = tiles / all * all;
        rest = tiles - whole;
        parts = 1;
        step_us = (dtype == AST_F32 ? 1.5 : 0.45) * nt / 256;
        double best = 1e300;
        for (int s = 1; rest && s <= MAX_PARTS && s <= std::max(1, steps / 2); ++s) {
            const double us = rounds(s) * ((steps + s - 1) / s * step_us + UNIT_US) + join_us(s);
            if (us < best) {
                best = us;
                parts = s;
            }
        }
        pairs = std::min(all, whole ? all : rest * parts);
    }
    static constexpr int MAX_PARTS = 64;
    static constexpr double UNIT_US = 5.0;
    int rounds(int s) const { return (rest * s + all - 1) / all; }
    double join_us(int s) const { return s > 1 ? 3.0 + 8e-6 * s * rest * TILE_M * nt / 6.0 : 0.0; }
    // No smaller number of rows takes more parts.  The number chosen goes up and down with the rows; s parts are chosen only where they cost less than any t < s, which
    // with the steps of a part rounded down for s and up for t bounds the number of steps on one side for each t.  The number chosen for this one rules out
    // most others by itself and is asked first: a call makes this check (0.4 us).
    int most_parts() const {
        for (int s = std::min(MAX_PARTS, steps / 2); s > parts && rest; --s) {
            double lo = 2.0 * s, hi = steps;
            const double rate = step_us * rounds(s) / s, fixed = rounds(s) * UNIT_US + join_us(s);
            auto ask = [&](int t) {
                // steps * slope < more, but for arithmetic errors far below 1e-6 us
                const int r = rounds(t);
                const double slope = rate - step_us * r / t, more = r * (step_us * (t - 1) / t + UNIT_US) + join_us(t) - fixed + 1e-6;
                if (slope > 1e-12) hi = std::min(hi, more / slope);
                else if (slope < -1e-12) lo = std::max(lo, more / slope);
                else if (more < 0) hi = 0;
                return lo <= hi;
            };
            bool can = ask(parts);
            for (int t = 1; can && t < s; ++t) can = ask(t);
            if (can) return s;
        }
        return parts;
    }
    size_t scratch(int p) const { return p > 1 ? (size_t)p * rest * 2 * part_floats(nt) : 0; }
};

template <int MODE, bool PROBE = false> void launch(const CUtensorMap& dy, const WArgs& a, int pairs, cudaStream_t st) {
    smem_limit_once<150 + 2 * MODE + PROBE>(wgrad_kernel<MODE, PROBE>, Form<MODE>::SMEM);
    launch_pdl_cluster(wgrad_kernel<MODE, PROBE>, 2 * pairs, Form<MODE>::THREADS, 2, Form<MODE>::SMEM, st, dy, a);
}

}  // namespace

size_t ckpt8_wgrad_scratch(int dtype, size_t rows, int ci, int co) {
    const Plan p(rows, ci, co, dtype);
    return p.scratch(p.parts);
}
size_t ckpt8_wgrad_most_scratch(int dtype, size_t rows, int ci, int co) {
    const Plan p(rows, ci, co, dtype);
    return p.scratch(p.most_parts());
}

void ckpt8_wgrad(int dtype, const void* codes, const void* exps, const void* dy, size_t lddy, size_t rows, int ci, int co, float* dw, float* db, bool accumulate,
                 float* scratch, int* err, cudaStream_t st, int silent_after) {
    if (!rows) {
        if (accumulate) return;
        cudaMemsetAsync(dw, 0, (size_t)ci * co * 4, st);
        if (db) cudaMemsetAsync(db, 0, (size_t)co * 4, st);
        return;
    }
    const Plan p(rows, ci, co, dtype);
    WArgs a{};
    a.codes = static_cast<const unsigned char*>(codes); a.exps = static_cast<const unsigned char*>(exps);
    a.dy = dy; a.lddy = lddy; a.groups = ((size_t)ci + GROUP - 1) / GROUP; a.pitch = a.groups * GROUP;
    a.rows = (unsigned)rows; a.ci = ci; a.co = co; a.nt = p.nt; a.tm = p.tm; a.tn = p.tn; a.steps = p.steps;
    a.whole = p.whole; a.rest = p.rest; a.parts = p.parts; a.dw = dw; a.db = db; a.part = scratch; a.add = accumulate ? 1 : 0; a.err = err;
    a.silent_after = silent_after;
    const bool probe = silent_after >= 0;
    const bool f32 = dtype == AST_F32;
    const bool pairs = reinterpret_cast<uintptr_t>(dy) % 8 == 0 && lddy % 2 == 0 && co % 2 == 0;
    alignas(64) CUtensorMap map{};
    int mode = f32 ? (pairs ? DY_F32 : DY_F32_ANY) : DY_BF16_ANY;
    if (!f32 && reinterpret_cast<uintptr_t>(dy) % 16 == 0 && lddy % 8 == 0) {
        const uint64_t dims[2] = {(uint64_t)co, (uint64_t)rows}, strides[1] = {(uint64_t)lddy * 2};
        const uint32_t box[2] = {64, ROWS};
        if (tma::encode_bf16(&map, dy, 2, dims, strides, box)) mode = DY_COPY;
    }
    {
        const double n_w = (double)ci * co;
        LaunchScope ls(K_CKPT8_WGRAD, rows * (a.pitch + a.groups + co * (f32 ? 4.0 : 2.0)) + 4.0 * (n_w + co), 2.0 * rows * n_w, st);
        switch (mode) {
            case DY_COPY: probe ? launch<DY_COPY, true>(map, a, p.pairs, st) : launch<DY_COPY>(map, a, p.pairs, st); break;
            case DY_F32: probe ? launch<DY_F32, true>(map, a, p.pairs, st) : launch<DY_F32>(map, a, p.pairs, st); break;
            case DY_F32_ANY: launch<DY_F32_ANY>(map, a, p.pairs, st); break;
            default: launch<DY_BF16_ANY>(map, a, p.pairs, st);
        }
    }
    if (p.parts > 1) {
        const size_t threads = ((size_t)p.nt / 4 * HALF_M + HALF_M) * 2 * p.rest;
        LaunchScope ls(K_REDUCE_SPLITS, 4.0 * p.scratch(p.parts) + 4.0 * p.rest * TILE_M * p.nt, 0.0, st);
        launch_pdl(sum_parts_kernel, (unsigned)((threads + 255) / 256), 256, 0, st, a);
    }
}

}  // namespace ast
