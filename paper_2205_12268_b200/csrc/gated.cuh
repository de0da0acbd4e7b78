// The gated pointwise block y = act(x Wg^T) * (x Wu^T) and its backward pass, bf16 on the tensor cores (tcgen05, accumulators in tensor memory).
//
// Four uses of one contraction kernel, D[128 x BN] += A[128 x 64] B[64 x BN] per step of the ring:
//   FORWARD  A = x (rows x channels), B = BN/2 rows of Wg and BN/2 of Wu: a gate and its partner are BN/2 columns apart in the same lane of
//            tensor memory, so the epilogue has both and writes y, rounded once.
//   PARTS    the same product again, its epilogue reads dy and writes dG and dU, operands of what follows
//   DX       A = dG then dU (rows x F), B = Wg then Wu as they lie: [F][Cin] has the contraction outside, an operand whose columns are contiguous
//   DW       A = dG or dU with the rows as contraction, B = x the same way: both lie with the contraction outside.  Few tiles (weights are small
//            next to maps) are cut along the rows, partial sums in fp32 are added in order by a kernel of their own.
// TMA (128-byte swizzle, no multicast) feeds a ring of stages, one thread issues the instructions, the accumulator is double-buffered, so the
// epilogue of a tile runs under the products of the next one.  Sizes that are no multiples of a tile arrive as zeros from TMA.
//
// dG and dU are fp16 with a power of two for each row, and so are x and the weights as operands of DX and DW.  Rounded to bf16, dG would add an error as large as
// the results' own rounding (2.4e-3 instead of 1.7e-3 against 64 bits); fp16 has three more bits at the same rate of the tensor cores, and bf16 values fit it
// exactly once the largest is near its end.  Row r's factor 2^k(r) comes from bounds, |dG| < 1.13 Cin max|dy_r| max|x_r| max|Wu| and |dU| the same with Wg (one for
// each: with the larger weights' bound for both, the other's part has fewer digits the more the two differ, none at 10^8).  With Cin and the maxima rounded up to
// powers of two the bound lies between 2^9 and 2^13.2, so nothing overflows, and a value has all of fp16's digits down to 2^-14: 2^-23 to 2^-27 of the bound.
// The weights have a factor each, their largest between 2^14 and 2^15; the products of DX then have the same power of two in both halves.  DW's need one
// for all rows: x_r is scaled by 2^(c - k(r)), with the c that brings the largest |dy_r| max|x_r|^2 to the end of fp16; x has all of its bits (bf16: eight) in rows
// where that is 2^-29 of the largest and more, times what x itself lies below its row's largest.
//
// Where the contraction is long, tiles of 256 columns are the work of two CTAs on neighbouring SMs (PAIR, cta_group::2): 128 rows each, and each brings in half
// of B for both, 32 KB a step instead of 48.  What bounds the loop then is the bytes that a ring can have on their way (192 KB at 1.5 us or so from L2):
// seven steps instead of four.  Forward with up to 256 channels, the weights of a column tile stay in shared memory (HOLD) while a CTA goes through the row
// tiles, and the ring holds rows alone.
#pragma once

#include <type_traits>

#include "tcgen05.cuh"
#include "tma.cuh"
#include "vec.cuh"

namespace wcc {
namespace gt {

using namespace tc;
using namespace tr;

enum Use { FORWARD, PARTS, DX, DW };

constexpr int BM = 128, KSTEP = 64;
constexpr int FEW = 32;                        // rows of a call that a stage of its own size holds
constexpr int FEW_STAGES = 17;
constexpr int HOLD_STEPS = 4;                  // HOLD: steps of weights that fit

// A variant of the kernel: its use, columns of a tile, whether two CTAs share a tile (PAIR), whether the weights of a column tile stay in shared memory
// (HOLD), rows of A that a step brings in (calls of few rows: the instruction then reads other steps' rows for the rest, whose results go nowhere).
template <int USE_, int BN_, bool PAIR_, bool HOLD_, int A_ROWS_ = BM> struct Form {
    static constexpr int USE = USE_, BN = BN_;
    static constexpr bool PAIR = PAIR_, HOLD = HOLD_;
    static constexpr bool GATES = USE == FORWARD || USE == PARTS;
    static_assert(GATES || !HOLD, "");
    static constexpr int B_COLS = PAIR ? BN / 2 : BN;                   // columns of B that a CTA brings in
    static constexpr int B_BYTES = B_COLS * KSTEP * 2;
    static constexpr int A_ROWS = A_ROWS_, A_BYTES = A_ROWS * KSTEP * 2;
    static constexpr int STAGE_BYTES = HOLD ? A_BYTES : A_BYTES + B_BYTES;
    static constexpr int HELD_BYTES = HOLD ? HOLD_STEPS * B_BYTES : 0;
    static constexpr int ROOM = (A_ROWS < BM ? 208 : 224) * 1024, MOST_STAGES = A_ROWS < BM ? FEW_STAGES : 8;
    static constexpr int FIT = (ROOM - HELD_BYTES) / STAGE_BYTES;
    static constexpr int STAGES = FIT < MOST_STAGES ? FIT : MOST_STAGES;
    static constexpr int SMEM = 1024 + STAGES * STAGE_BYTES + HELD_BYTES + (A_ROWS < BM ? BM * KSTEP * 2 : 0);      // and Ctl
    static constexpr int SHARES = BN == 64 ? 2 : 4;                     // warps of the epilogue: four for each share of a tile's columns
    static constexpr int THREADS = 64 + 128 * SHARES;
    static constexpr int ROWS = PAIR ? 2 * BM : BM;                     // of a tile
};

struct Ctl {
    uint64_t full[FEW_STAGES], empty[FEW_STAGES], tfull[2], tempty[2], bfull, bempty;
    uint32_t tmem_base;
    int abort_flag;
};

// Exponents E, |v| < 2^E, with BIAS added: of either weights and of x, and the largest over the rows of what they bring to DW, |dy_r| |x_r|^2.  (A row's own,
// E(r) of |dy_r| |x_r|, are a list.)
struct alignas(16) Exps { unsigned Wg, Wu, rows, x; };
constexpr int BIAS = 512;

struct Args {
    int rows, Cin, F;
    const Exps* exps;
    const short* row_exp;
    int log_cin;                           // Cin <= 2^log_cin
    int m_tiles, n_tiles, splits;          // DW: m_tiles counts those of dG and dU
    int act;
    const __nv_bfloat16* dy;
    __nv_bfloat16 *y, *y2;                 // FORWARD y; PARTS dG, dU; DX dx; DW dWg, dWu
    float* part;                           // DW with splits > 1: [splits][2 F][Cin]
    int* status;
};

__device__ __forceinline__ uint32_t cta_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
// Address of the pair's first CTA's copy of something in shared memory.
__device__ __forceinline__ uint32_t of_first(uint32_t addr)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(addr));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Bounded wait for a barrier that another CTA of the pair arrives at.
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag)
{
    const uint32_t limit = c_wait_limit;
    for (uint32_t it = 0; it < limit; ++it) {
        uint32_t ok;
        asm volatile("{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000u) : "memory");
        if (ok) return true;
        if (*abort_flag) return false;
    }
    return false;
}
// PAIR: bytes count at the first CTA's barrier.
template <bool PR> __device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* tm, int c0, int c1, uint32_t bar)
{
    if constexpr (PR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(c0), "r"(c1), "r"(bar) : "memory");
    else
        tma_load_2d(dst, tm, c0, c1, bar);
}
template <bool PR> __device__ __forceinline__ void multiply(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    if constexpr (PR)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        mma_ss<false>(d, a, b, idesc, accumulate);
}
// All products issued so far are done: arrive at this barrier (PAIR: of both CTAs).
template <bool PR> __device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (PR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
    else
        mma_commit(bar);
}

// ---- powers of two
__device__ __forceinline__ float power(int n) { return __int_as_float((min(max(n, -126), 127) + 127) << 23); }
// With row r's E(r): dG is scaled by 2^(dG - E(r)), dU by 2^(dU - E(r)), x of DW by 2^(x + E(r)), the weights by 2^Wg and 2^Wu.  No power is held to what fp32 has:
// where one goes beyond it (tiny rows, weights of zeros), it is multiplied by in two steps, dG's and dU's by way of dy.  What these do not reach is 0: of the sums
// u (or g) of rows where Cin max|x_r| max|Wu| is below 2^-114.
// With row r's e = row(E(r)): dG is scaled by 2^(dG - e), dU by 2^(dU - e), x of DW by 2^(x + e), the weights by 2^Wg and 2^Wu.  row() keeps dG's and dU's powers
// in fp32: below, for values that are larger than the bound allows; above, rows for which one of the two bounds is less than 2^-114 are scaled by less.  Weights of
// zeros go as large as the others.
struct Scales {
    int dG = 0, dU = 0, Wg = 0, Wu = 0, x = 0, lo = 0, hi = 0;
    __device__ __forceinline__ Scales() {}
    __device__ __forceinline__ Scales(const Exps* e, int log_cin)
    {
        const uint4 all = __ldcg(reinterpret_cast<const uint4*>(e));
        const int least = -126, er = (int)all.z - BIAS, ex = (int)all.w - BIAS;
        int eg = (int)all.x - BIAS, eu = (int)all.y - BIAS;
        if (eg == least) eg = eu;
        if (eu == least) eu = eg;
        dG = 13 - log_cin - eu;
        dU = 13 - log_cin - eg;
        Wg = 15 - eg;
        Wu = 15 - eu;
        lo = max(dG, dU) - 127;
        hi = min(dG, dU) + 126;
        x = 15 - max(er, lo + ex);
    }
    __device__ __forceinline__ int row(int E) const { return min(max(E, lo), hi); }
};
__device__ __forceinline__ uint32_t pack_half2(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

// Operand with the contraction outside: rows of 64 columns (128 bytes, swizzled), groups of 8 of the contraction 1024 bytes apart, the next 64 columns
// KSTEP rows further on.
__device__ __forceinline__ uint64_t smem_desc_outer(uint32_t addr)
{
    const uint32_t lo = ((addr & 0x3FFFFu) >> 4) | ((uint32_t)(KSTEP * 128 >> 4) << 16);
    const uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    return ((uint64_t)hi << 32) | lo;
}

// Value and derivative of the activation, two at a time.
// gelu: Phi by Abramowitz and Stegun 7.1.26 (erf to 1.5e-7 absolute; of Phi itself that is 1.6e-3 at z = -5 and 3.6e-3, a step of bf16, at -6, where the result is
// 10^-8), with one reciprocal for two; |z| beyond 42 is taken as 42 in it (the exponential is 0 there), so that their product does not overflow.
struct Act2 { f2 a, d; };
template <int ACT, bool SLOPE> __device__ __forceinline__ Act2 act_of(f2 z)
{
    const f2 one = both(1.0f);
    if constexpr (ACT == WCC_ACT_RELU)
        return {pair(z.x() < 0.0f ? 0.0f : z.x(), z.y() < 0.0f ? 0.0f : z.y()), pair(z.x() > 0.0f ? 1.0f : 0.0f, z.y() > 0.0f ? 1.0f : 0.0f)};
    if constexpr (ACT == WCC_ACT_SILU) {
        const Sigmoid2 q = sigmoid2(z);
        return {mul2(z, q.s), SLOPE ? silu_slope2(z, q) : one};
    }
    if constexpr (ACT == WCC_ACT_GELU) {
        const f2 x = pair(fminf(fabsf(z.x()), 42.0f), fminf(fabsf(z.y()), 42.0f));
        const f2 q = fma2(x, both(0.3275911f * 0.70710678118654752f), one);
        const f2 t = mul2(both(rcp_approx(q.x() * q.y())), pair(q.y(), q.x()));
        const f2 w = mul2(mul2(z, z), both(-0.72134752044448170f));                // e^(-z^2 / 2)
        const f2 e = pair(exp2_approx(w.x()), exp2_approx(w.y()));
        f2 p = fma2(t, both(0.5f * 1.061405429f), both(0.5f * -1.453152027f));
        p = fma2(p, t, both(0.5f * 1.421413741f));
        p = fma2(p, t, both(0.5f * -0.284496736f));
        p = fma2(p, t, both(0.5f * 0.254829592f));
        const f2 h = mul2(mul2(p, t), e), far = fma2(h, both(-1.0f), one);
        const f2 phi = pair(z.x() < 0.0f ? h.x() : far.x(), z.y() < 0.0f ? h.y() : far.y());
        return {mul2(z, phi), SLOPE ? fma2(mul2(z, both(0.39894228040143268f)), e, phi) : one};
    }
    return {z, one};
}

// N columns of this warp's lanes; what is read is there after tmem_wait.
template <int N> __device__ __forceinline__ void tmem_read(uint32_t taddr, uint32_t (&u)[N])
{
    static_assert(N == 16, "");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
                   "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 16 bf16 values, those of the first `cols` columns (a multiple of 8).  A lane's row is far from its neighbours', so a store goes to 32 lines: a whole
// 32-byte sector at once where the rows start on one.
__device__ __forceinline__ void store16(__nv_bfloat16* p, const uint32_t* w, int cols, bool sectors)
{
    if (sectors && cols >= 16) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        if (cols > 0) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        if (cols > 8) *reinterpret_cast<uint4*>(p + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// 16 columns of gates and their partners: y, or with dy (`d`, bf16 pairs) dG and dU times the row's factors.
template <int USE, int ACT>
__device__ __forceinline__ void gates16(const uint32_t (&g)[16], const uint32_t (&u)[16], const uint32_t* d, float fg, float fu, uint32_t* o, uint32_t* o2)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const f2 z = pair(__uint_as_float(g[2 * i]), __uint_as_float(g[2 * i + 1])), w = pair(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
        const Act2 v = act_of<ACT, USE == PARTS>(z);
        if constexpr (USE == FORWARD) {
            const f2 r = mul2(v.a, w);
            o[i] = pack_bf16x2(r.x(), r.y());
        } else {
            // (the factor last: dy alone times it might be too large)
            const f2 t = pair(bf16lo(d[i]), bf16hi(d[i])), r = mul2(mul2(mul2(t, w), v.d), both(fg)), r2 = mul2(mul2(t, v.a), both(fu));
            o[i] = pack_half2(r.x(), r.y());
            o2[i] = pack_half2(r2.x(), r2.y());
        }
    }
}

template <typename Fm>
__global__ void __launch_bounds__(Fm::THREADS, 1)
contract(const __grid_constant__ CUtensorMap tA0, const __grid_constant__ CUtensorMap tA1, const __grid_constant__ CUtensorMap tB0,
         const __grid_constant__ CUtensorMap tB1, const __grid_constant__ Args a)
{
    constexpr int USE = Fm::USE, BN = Fm::BN, ST = Fm::STAGES, SB = Fm::STAGE_BYTES, COLS = 2 * BN, BC = Fm::B_COLS, TM = Fm::ROWS;
    constexpr bool PR = Fm::PAIR, HOLD = Fm::HOLD;
    constexpr bool A_OUTER = USE == DW, B_OUTER = USE == DX || USE == DW;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    Ctl* ctl = reinterpret_cast<Ctl*>(smem_raw + (base - raw) + Fm::SMEM - 1024);
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int items = a.m_tiles * a.n_tiles * a.splits;
    // PAIR: both CTAs go through the same items, each with its half of the rows and of B
    const int rank = PR ? (int)cta_rank() : 0, worker = PR ? blockIdx.x / 2 : blockIdx.x, workers = PR ? gridDim.x / 2 : gridDim.x;
    // Items: HOLD: a stretch of them, row tiles within a column tile; else every workers'th, column tiles within a row tile within a part of the rows.
    const int w_first = HOLD ? (int)((long long)items * worker / workers) : worker, w_end = HOLD ? (int)((long long)items * (worker + 1) / workers) : items;
    const int w_step = HOLD ? 1 : workers;
    auto place = [&](int w, int& nt, int& mt, int& sp) {
        if constexpr (HOLD) {
            nt = w / a.m_tiles;
            mt = w - nt * a.m_tiles;
            sp = 0;
        } else {
            const int ms = w / a.n_tiles;
            nt = w - ms * a.n_tiles;
            sp = ms / a.m_tiles;
            mt = ms - sp * a.m_tiles;
        }
    };
    // steps of the ring for an item: along the channels, along F twice, along the rows
    const int f_steps = (a.F + KSTEP - 1) / KSTEP, row_steps = (a.rows + KSTEP - 1) / KSTEP;
    const int all_steps = USE == DX ? 2 * f_steps : USE == DW ? row_steps : (a.Cin + KSTEP - 1) / KSTEP;

    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->tfull[b]), 1); mbar_init(smem_u32(&ctl->tempty[b]), (PR ? 8 : 4) * Fm::SHARES); }
        mbar_init(smem_u32(&ctl->bfull), 1);
        mbar_init(smem_u32(&ctl->bempty), 1);
        ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        if constexpr (PR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"((uint32_t)COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"((uint32_t)COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    fence_before();
    __syncthreads();
    if constexpr (PR) cluster_sync();                          // the other CTA's barriers are ready
    fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    bool failed = false;
    pdl_wait();
    pdl_launch();

    if (warp == 0) {
        if (lane == 0) {
            // a step of weights: gates' columns, then their partners' (PAIR: one CTA has these, the other those)
            [[maybe_unused]] auto weights = [&](uint32_t dst, int k, int nt, uint32_t bar) {
                if constexpr (PR) {
                    load_tile<PR>(dst, rank == 0 ? &tB0 : &tB1, k * KSTEP, nt * (BN / 2), bar);
                } else {
                    load_tile<PR>(dst, &tB0, k * KSTEP, nt * (BN / 2), bar);
                    load_tile<PR>(dst + BN / 2 * 128, &tB1, k * KSTEP, nt * (BN / 2), bar);
                }
            };
            int s = 0, held = -1, swaps = 0;                   // column tile whose weights are here, times that they were brought in
            uint32_t ph = 1;
            for (int w = w_first; w < w_end && !failed; w += w_step) {
                int nt, mt, sp;
                place(w, nt, mt, sp);
                if (HOLD && nt != held) {
                    if (!mbar_wait(smem_u32(&ctl->bempty), (uint32_t)(swaps & 1) ^ 1u, abort_flag)) { failed = true; break; }
                    const uint32_t own = smem_u32(&ctl->bfull), bar = PR ? of_first(own) : own;
                    if (rank == 0) mbar_expect_tx(own, (uint32_t)((PR ? 2 : 1) * all_steps * Fm::B_BYTES));
                    for (int k = 0; k < all_steps; ++k) weights(base + ST * SB + k * Fm::B_BYTES, k, nt, bar);
                    held = nt;
                    ++swaps;
                }
                const int k0 = (int)((long long)all_steps * sp / a.splits), k1 = (int)((long long)all_steps * (sp + 1) / a.splits);
                for (int k = k0; k < k1; ++k) {
                    if (!mbar_wait(smem_u32(&ctl->empty[s]), ph, abort_flag)) { failed = true; break; }
                    const uint32_t sA = base + (uint32_t)s * SB, sB = sA + Fm::A_BYTES, own = smem_u32(&ctl->full[s]), bar = PR ? of_first(own) : own;
                    if (rank == 0) mbar_expect_tx(own, (uint32_t)(PR ? 2 * SB : SB));
                    if constexpr (USE == FORWARD || USE == PARTS) {
                        load_tile<PR>(sA, &tA0, k * KSTEP, mt * TM + rank * BM, bar);
                        if constexpr (!HOLD) weights(sB, k, nt, bar);
                    } else if constexpr (USE == DX) {
                        const bool up = k >= f_steps;
                        const int f0 = (up ? k - f_steps : k) * KSTEP;
                        load_tile<PR>(sA, up ? &tA1 : &tA0, f0, mt * TM + rank * BM, bar);
                        for (int i = 0; i < BC / 64; ++i) load_tile<PR>(sB + i * KSTEP * 128, up ? &tB1 : &tB0, nt * BN + rank * BC + 64 * i, f0, bar);
                    } else {
                        const int mhalf = a.m_tiles / 2;
                        const bool up = mt >= mhalf;
                        const int f0 = (up ? mt - mhalf : mt) * TM + rank * BM;
                        for (int i = 0; i < 2; ++i) load_tile<PR>(sA + i * KSTEP * 128, up ? &tA1 : &tA0, f0 + 64 * i, k * KSTEP, bar);
                        for (int i = 0; i < BC / 64; ++i) load_tile<PR>(sB + i * KSTEP * 128, &tB0, nt * BN + rank * BC + 64 * i, k * KSTEP, bar);
                    }
                    if (++s == ST) { s = 0; ph ^= 1u; }
                }
            }
            // the products' arrivals at this CTA's barriers (PAIR: from the other CTA) are all there before it goes
            for (int i = 0; i < ST && !failed; ++i) {
                failed = !mbar_wait(smem_u32(&ctl->empty[s]), ph, abort_flag);
                if (++s == ST) { s = 0; ph ^= 1u; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            // D fp32, A and B bf16 (bits 7 and 10) or fp16; bits 15 and 16: the contraction lies outside
            constexpr uint32_t idesc = (1u << 4) | (Fm::GATES ? (1u << 7) | (1u << 10) : 0u) | ((A_OUTER ? 1u : 0u) << 15) | ((B_OUTER ? 1u : 0u) << 16) |
                                       ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(TM >> 4) << 24);
            // (this thread issues next to the epilogue's warps: little more than the instructions themselves stands in its loop)
            int s = 0, item = 0, held = -1, swaps = 0;
            uint32_t ph = 0;
            const uint32_t full0 = smem_u32(&ctl->full[0]), empty0 = smem_u32(&ctl->empty[0]);
            const uint64_t a0 = A_OUTER ? smem_desc_outer(base) : smem_desc_sw128(base);
            const uint64_t b0 = HOLD ? smem_desc_sw128(base + ST * SB) : B_OUTER ? smem_desc_outer(base + Fm::A_BYTES) : smem_desc_sw128(base + Fm::A_BYTES);
            for (int w = w_first; w < w_end && !failed; w += w_step, ++item) {
                int nt, mt, sp;
                place(w, nt, mt, sp);
                if (HOLD && nt != held) {
                    if (held >= 0) commit<PR>(smem_u32(&ctl->bempty));         // the products with the old weights are done: they may go
                    if (!(PR ? wait_cluster(smem_u32(&ctl->bfull), (uint32_t)(swaps & 1), abort_flag) : mbar_wait(smem_u32(&ctl->bfull), (uint32_t)(swaps & 1), abort_flag))) { failed = true; break; }
                    held = nt;
                    ++swaps;
                }
                const int k0 = (int)((long long)all_steps * sp / a.splits), k1 = (int)((long long)all_steps * (sp + 1) / a.splits);
                const int buf = item & 1;
                const uint32_t bph = (uint32_t)(item >> 1) & 1u;
                if (!(PR ? wait_cluster(smem_u32(&ctl->tempty[buf]), bph ^ 1u, abort_flag) : mbar_wait(smem_u32(&ctl->tempty[buf]), bph ^ 1u, abort_flag))) { failed = true; break; }
                fence_after();
                const uint32_t d = tmem_base + (uint32_t)(buf * BN);
                uint32_t accumulate = 0;
                uint64_t bd = b0;
#pragma unroll 2
                for (int k = k0; k < k1; ++k) {
                    if (!(PR ? wait_cluster(full0 + 8 * s, ph, abort_flag) : mbar_wait(full0 + 8 * s, ph, abort_flag))) { failed = true; break; }
                    fence_after();
                    const uint64_t ad = a0 + (uint64_t)(s * (SB >> 4));
                    if constexpr (!HOLD) bd = b0 + (uint64_t)(s * (SB >> 4));
#pragma unroll
                    for (int kk = 0; kk < KSTEP / 16; ++kk) {      // 16 of the contraction: 32 bytes of a row, or 16 rows of 128 bytes
                        multiply<PR>(d, ad + (uint64_t)((A_OUTER ? 128 : 2) * kk), bd + (uint64_t)((B_OUTER ? 128 : 2) * kk), idesc, accumulate);
                        accumulate = 1;
                    }
                    commit<PR>(empty0 + 8 * s);
                    if constexpr (HOLD) bd += (uint64_t)(Fm::B_BYTES >> 4);
                    if (++s == ST) { s = 0; ph ^= 1u; }
                }
                if (failed) break;
                commit<PR>(smem_u32(&ctl->tfull[buf]));
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3, share = (warp - 2) >> 2;       // lanes of tensor memory that the warp may read; its share of the columns
        constexpr bool GATES = Fm::GATES;
        constexpr int MINE = (GATES ? BN / 2 : BN) / Fm::SHARES, N = 16;         // columns of the warp, and those at once
        const int width = GATES ? a.F : a.Cin, mhalf = a.m_tiles / 2;
        const bool sectors = width % 16 == 0 && ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.y2)) & 31u) == 0;
        const Scales scales = USE == FORWARD ? Scales{} : Scales(a.exps, a.log_cin);
        int item = 0;
        for (int w = w_first; w < w_end; w += w_step, ++item) {
            int nt, mt, sp;
            place(w, nt, mt, sp);
            const bool up = USE == DW && mt >= mhalf;
            const int row = (up ? mt - mhalf : mt) * TM + rank * BM + q * 32 + lane, col0 = nt * (GATES ? BN / 2 : BN) + share * MINE;
            const bool on = row < (USE == DW ? a.F : a.rows);
            const size_t at0 = (size_t)row * width + col0;
            // dy does not wait for the products
            uint32_t d[USE == PARTS ? MINE / 2 : 1];
            if constexpr (USE == PARTS) {
#pragma unroll
                for (int i = 0; i < MINE; i += 8) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (on && col0 + i < width) v = __ldg(reinterpret_cast<const uint4*>(a.dy + at0 + i));
                    d[i / 2] = v.x; d[i / 2 + 1] = v.y; d[i / 2 + 2] = v.z; d[i / 2 + 3] = v.w;
                }
            }
            // the row's factors of dG and dU, or what takes them and the other operands' away again (DX: the same of both halves)
            const int e = (USE == PARTS || USE == DX) && on ? scales.row(a.row_exp[row]) : 0;
            const int n = USE == DX ? e - scales.dG - scales.Wg : USE == DW ? -(up ? scales.dU : scales.dG) - scales.x : 0;
            [[maybe_unused]] const float factor = power(n / 2), second = power(n - n / 2);
            [[maybe_unused]] const float fg = power(scales.dG - e), fu = power(scales.dU - e);
            const int buf = item & 1;
            const uint32_t bph = (uint32_t)(item >> 1) & 1u;
            int ok = mbar_wait(smem_u32(&ctl->tfull[buf]), bph, abort_flag) ? 1 : 0;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) { failed = true; break; }
            fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * BN + share * MINE);
            // The accumulator is free as soon as it is in registers: with few steps a tile, what the next product but one waits for is this warp.
            uint32_t v[MINE / N][N], p[GATES ? MINE / N : 1][N];
#pragma unroll
            for (int c = 0; c < MINE / N; ++c) {
                tmem_read<N>(taddr + (uint32_t)(c * N), v[c]);
                if constexpr (GATES) tmem_read<N>(taddr + (uint32_t)(BN / 2 + c * N), p[c]);
            }
            tmem_wait();
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PR) asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(of_first(smem_u32(&ctl->tempty[buf]))) : "memory");
                else mbar_arrive(smem_u32(&ctl->tempty[buf]));
            }
            if constexpr (GATES) {
                uint32_t o[MINE / 2], o2[USE == PARTS ? MINE / 2 : 1];
                auto all = [&](auto act) {
#pragma unroll
                    for (int c = 0; c < MINE / N; ++c)
                        gates16<USE, decltype(act)::value>(v[c], p[c], USE == PARTS ? d + c * 8 : d, fg, fu, o + c * 8, USE == PARTS ? o2 + c * 8 : o2);
                };
                if (a.act == WCC_ACT_SILU) all(std::integral_constant<int, WCC_ACT_SILU>());
                else if (a.act == WCC_ACT_GELU) all(std::integral_constant<int, WCC_ACT_GELU>());
                else if (a.act == WCC_ACT_RELU) all(std::integral_constant<int, WCC_ACT_RELU>());
                else all(std::integral_constant<int, WCC_ACT_NONE>());
                if (on) {
#pragma unroll
                    for (int c = 0; c < MINE / N; ++c) {
                        const int cols = width - col0 - c * N;
                        if (cols <= 0) break;
                        store16(a.y + at0 + c * N, o + c * 8, cols, sectors);
                        if constexpr (USE == PARTS) store16(a.y2 + at0 + c * N, o2 + c * 8, cols, sectors);
                    }
                }
            } else if (on) {
#pragma unroll
                for (int c = 0; c < MINE / N; ++c) {
                    const int cols = width - col0 - c * N;
                    if (cols <= 0) break;
#pragma unroll
                    for (int i = 0; i < N; ++i) v[c][i] = __float_as_uint(__uint_as_float(v[c][i]) * factor * second);
                    if (USE == DW && a.splits > 1) {
                        float* o = a.part + (((size_t)sp * 2 + (up ? 1 : 0)) * a.F + row) * a.Cin + col0 + c * N;
#pragma unroll
                        for (int i = 0; i < N; i += 4)
                            if (i < cols) *reinterpret_cast<uint4*>(o + i) = make_uint4(v[c][i], v[c][i + 1], v[c][i + 2], v[c][i + 3]);
                    } else {
                        uint32_t o[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) o[k] = pack_bf16x2(__uint_as_float(v[c][2 * k]), __uint_as_float(v[c][2 * k + 1]));
                        store16((up ? a.y2 : a.y) + at0 + c * N, o, cols, sectors);
                    }
                }
            }
        }
        __syncwarp();
    }

    if (failed) {
        *abort_flag = 1;
        atomicExch(a.status, (int)WCC_ERR_TIMEOUT);
    }
    fence_before();
    __syncthreads();
    if (*abort_flag) {
        // copies that are on their way land before the CTA's shared memory goes away
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
        __syncthreads();
    }
    if constexpr (PR) cluster_sync();                          // the other CTA arrives at this one's barriers no more
    if (warp == 1) {
        fence_after();
        if constexpr (PR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)COLS) : "memory");
    }
}

// ---- operands in fp16
// Exponents of the rows, and of the weights (rows behind them): eight lanes a row, or a warp where rows are long.  What is not finite counts for nothing.
// (66306 rows of 64 and 256 values, a warp / eight lanes a row: 26 / 15 us; 8192 of 1024 and 4096 22 / 29.)
template <int LANES> __device__ __forceinline__ int exponent_of(const __nv_bfloat16* p, int n, int lane)
{
    const uint4* q = reinterpret_cast<const uint4*>(p);
    const int vectors = n / 8;
    unsigned m = 0;
#pragma unroll 8
    for (int i = lane; i < vectors; i += LANES) {
        const uint4 v = __ldg(q + i);
        m = __vmaxu2(m, __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu)));
    }
    unsigned top = max(m & 0xFFFFu, m >> 16);
    if (top >= 0x7F80u) {                                   // once more without what is not finite
        top = 0;
        for (int i = lane * 8; i < n; i += LANES * 8)
            for (int k = 0; k < 8; ++k) {
                const unsigned h = __bfloat16_as_ushort(p[i + k]) & 0x7FFFu;
                if (h < 0x7F80u) top = max(top, h);
            }
    }
    __syncwarp();
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    return (int)(top >> 7) - 126;
}
template <int LANES>
__global__ void __launch_bounds__(256) exponents(const __nv_bfloat16* __restrict__ dy, const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ Wg,
                                                        const __nv_bfloat16* __restrict__ Wu, int rows, int Cin, int F, short* __restrict__ row_exp, Exps* exps)
{
    __shared__ unsigned most[4];
    pdl_wait();
    pdl_launch();
    if (threadIdx.x < 4) most[threadIdx.x] = 0;
    __syncthreads();
    constexpr int EACH = 256 / LANES;
    const int lane = threadIdx.x & (LANES - 1);
    const long long all = (long long)rows + 2 * F, step = (long long)gridDim.x * EACH;
    unsigned top_g = 0, top_u = 0, top_r = 0, top_x = 0;
    for (long long r0 = (long long)blockIdx.x * EACH; r0 < all; r0 += step) {
        // (lanes without a row go along with the last one)
        const long long r = min(r0 + threadIdx.x / LANES, all - 1), f = r - rows;
        const bool row = r < rows;
        const int ex = exponent_of<LANES>(row ? x + r * Cin : f < F ? Wg + f * Cin : Wu + (f - F) * Cin, Cin, lane);
        const int ey = exponent_of<LANES>(row ? dy + r * F : dy, row ? F : 0, lane);
        if (row) {
            if (lane == 0) row_exp[r] = (short)(ey + ex);
            top_r = max(top_r, (unsigned)(ey + 2 * ex + BIAS));
            top_x = max(top_x, (unsigned)(ex + BIAS));
        } else if (f < F) {
            top_g = max(top_g, (unsigned)(ex + BIAS));
        } else {
            top_u = max(top_u, (unsigned)(ex + BIAS));
        }
    }
    if (lane == 0) {
        if (top_g) atomicMax(&most[0], top_g);
        if (top_u) atomicMax(&most[1], top_u);
        if (top_r) atomicMax(&most[2], top_r);
        if (top_x) atomicMax(&most[3], top_x);
    }
    __syncthreads();
    if (threadIdx.x < 4 && most[threadIdx.x]) atomicMax(reinterpret_cast<unsigned*>(exps) + threadIdx.x, most[threadIdx.x]);
}
// x and the weights in fp16 with their factors; x16 or W16 NULL: not wanted.
static __global__ void __launch_bounds__(256) to_half(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ Wg, const __nv_bfloat16* __restrict__ Wu,
                                                      int rows, int Cin, int F, const short* __restrict__ row_exp, const Exps* exps, int log_cin, Divisor by_row, uint4* x16, uint4* W16)
{
    pdl_wait();
    pdl_launch();
    const Scales s(exps, log_cin);
    const int per = Cin / 8;
    const long long nx = x16 ? (long long)rows * per : 0, nw = W16 ? (long long)F * per : 0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < nx + 2 * nw; i += (long long)gridDim.x * 256) {
        const uint4* from;
        uint4* to;
        int n;
        if (i < nx) {
            const long long row = nx < (1LL << 31) ? (long long)by_row.div((int)i) : i / per;
            n = s.x + s.row(row_exp[row]);
            from = reinterpret_cast<const uint4*>(x) + i;
            to = x16 + i;
        } else {
            const long long j = i - nx;
            n = j < nw ? s.Wg : s.Wu;
            from = j < nw ? reinterpret_cast<const uint4*>(Wg) + j : reinterpret_cast<const uint4*>(Wu) + (j - nw);
            to = W16 + j;
        }
        const uint4 v = __ldg(from);
        const float f = power(n / 2), g = power(n - n / 2);
        auto two = [&](uint32_t w) {
            float a = bf16lo(w) * f * g, b = bf16hi(w) * f * g;
            // (a finite value never becomes an infinity, whatever the exponents)
            if (fabsf(a) > 65504.0f && (w & 0x7F80u) != 0x7F80u) a = copysignf(65504.0f, a);
            if (fabsf(b) > 65504.0f && (w & 0x7F800000u) != 0x7F800000u) b = copysignf(65504.0f, b);
            return pack_half2(a, b);
        };
        *to = make_uint4(two(v.x), two(v.y), two(v.z), two(v.w));
    }
}

// Partial sums of the weights' gradients, added in order, two values a thread, sixteen parts on their way at once.
static __global__ void __launch_bounds__(128) add_parts(const float* __restrict__ part, int splits, size_t each, __nv_bfloat16* __restrict__ dWg,
                                                        __nv_bfloat16* __restrict__ dWu)
{
    pdl_wait();
    pdl_launch();
    const size_t i = ((size_t)blockIdx.x * 128 + threadIdx.x) * 2;
    if (i >= 2 * each) return;
    float2 v = make_float2(0.0f, 0.0f);
    for (int s0 = 0; s0 < splits; s0 += 16) {
        float2 p[16];
#pragma unroll
        for (int s = 0; s < 16; ++s) p[s] = s0 + s < splits ? __ldcg(reinterpret_cast<const float2*>(part + (size_t)(s0 + s) * 2 * each + i)) : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int s = 0; s < 16; ++s) { v.x += p[s].x; v.y += p[s].y; }
    }
    __nv_bfloat16* dst = i < each ? dWg + i : dWu + (i - each);
    *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(v.x, v.y);
}

// ---- host ------------------------------------------------------------------------------------------
// [outer][inner] bf16 or fp16, boxes of 64 x `box` rows.
inline bool map_of(CUtensorMap* tm, const void* p, int inner, int outer, int box, bool half = false)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer}, strides[1] = {(cuuint64_t)inner * 2};
    cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
    return fn(tm, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename Fm>
wcc_status launch(const CUtensorMap& A0, const CUtensorMap& A1, const CUtensorMap& B0, const CUtensorMap& B1, const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int smem = Fm::SMEM + (int)sizeof(Ctl) + 16;
    const wcc_status s = allow_smem<contract<Fm>>(di.dev, smem);
    if (s != WCC_OK) return s;
    const int items = a.m_tiles * a.n_tiles * a.splits, workers = Fm::PAIR ? di.sms / 2 : di.sms, grid = (items < workers ? items : workers) * (Fm::PAIR ? 2 : 1);
    return launch_overlapped(contract<Fm>, dim3((unsigned)grid), dim3(Fm::THREADS), smem, st, true, Fm::PAIR ? 2 : 1, A0, A1, B0, B1, a);
}

// Columns of a tile: as many as fill the SMs, 64 at least.  `cols` columns in all (FORWARD: gates and partners).
inline int tile_of(int m_tiles, long long cols, int sms)
{
    int bn = 256;
    while (bn > 64 && (cols <= bn / 2 || (long long)m_tiles * ((cols + bn - 1) / bn) < sms)) bn /= 2;
    return bn;
}
// Two CTAs a tile from this length of the contraction on: their barriers cost 1.3 us a tile instead of half of that, their loads a third less.  Forward with
// silu, 65536 rows to 1024 columns, one CTA / two: 256 channels 70 / 88 us, 512 119 / 112, 16384 x 1024 -> 4096 206 / 191.
constexpr int PAIR_FROM = 512;

template <int USE>
wcc_status gates(const void* x, const void* Wg, const void* Wu, Args a, const DeviceInfo& di, cudaStream_t st)
{
    // few rows: the weights are the traffic, so as many CTAs as there are, and the whole of their share on its way at once
    const bool few = a.rows <= FEW;
    const int bn = few ? 64 : tile_of(ceil_div(a.rows, BM), 2LL * a.F, di.sms);
    const bool two = bn == 256 && a.Cin >= PAIR_FROM;
    a.m_tiles = ceil_div(a.rows, two ? 2 * BM : BM);
    a.n_tiles = ceil_div(a.F, bn / 2);
    a.splits = 1;
    CUtensorMap A, G, U;
    if (!map_of(&A, x, a.Cin, a.rows, few ? FEW : BM) || !map_of(&G, Wg, a.Cin, a.F, bn / 2) || !map_of(&U, Wu, a.Cin, a.F, bn / 2)) return WCC_ERR_CUDA;
    if (two) return launch<Form<USE, 256, true, false>>(A, A, G, U, a, di, st);
    // Few channels: the weights stay (forward, to 1024 columns: 65536 x 256 72 -> 69 us, 66306 x 64 -> 256 18.8 -> 17.2).  Not where dy is read: the column
    // tiles of a row tile are then far apart in time, and its lines with them (gradients of the second 66 -> 70 us).
    if constexpr (USE == FORWARD)
        if (bn == 256 && a.Cin <= HOLD_STEPS * KSTEP) return launch<Form<USE, 256, false, true>>(A, A, G, U, a, di, st);
    if (bn == 256) return launch<Form<USE, 256, false, false>>(A, A, G, U, a, di, st);
    if (bn == 128) return launch<Form<USE, 128, false, false>>(A, A, G, U, a, di, st);
    if (few) return launch<Form<USE, 64, false, false, FEW>>(A, A, G, U, a, di, st);
    return launch<Form<USE, 64, false, false>>(A, A, G, U, a, di, st);
}

template <int USE>
wcc_status products(int bn, bool two, const CUtensorMap& A0, const CUtensorMap& A1, const CUtensorMap& B0, const CUtensorMap& B1, const Args& a, const DeviceInfo& di,
                    cudaStream_t st)
{
    if (two) return launch<Form<USE, 256, true, false>>(A0, A1, B0, B1, a, di, st);
    if (bn == 256) return launch<Form<USE, 256, false, false>>(A0, A1, B0, B1, a, di, st);
    if (bn == 128) return launch<Form<USE, 128, false, false>>(A0, A1, B0, B1, a, di, st);
    return launch<Form<USE, 64, false, false>>(A0, A1, B0, B1, a, di, st);
}

inline wcc_status dx(const void* dG, const void* dU, const void* Wg, const void* Wu, Args a, const DeviceInfo& di, cudaStream_t st)
{
    const int bn = tile_of(ceil_div(a.rows, BM), a.Cin, di.sms);
    const bool two = bn == 256 && 2 * a.F >= PAIR_FROM;
    a.m_tiles = ceil_div(a.rows, two ? 2 * BM : BM);
    a.n_tiles = ceil_div(a.Cin, bn);
    a.splits = 1;
    CUtensorMap A0, A1, B0, B1;
    if (!map_of(&A0, dG, a.F, a.rows, BM, true) || !map_of(&A1, dU, a.F, a.rows, BM, true) || !map_of(&B0, Wg, a.Cin, a.F, KSTEP, true) ||
        !map_of(&B1, Wu, a.Cin, a.F, KSTEP, true))
        return WCC_ERR_CUDA;
    return products<DX>(bn, two, A0, A1, B0, B1, a, di, st);
}

struct DwPlan { int bn; bool two; int m_tiles, n_tiles, splits; };
inline DwPlan dw_plan(int rows, int Cin, int F, int sms)
{
    DwPlan p;
    p.bn = Cin > 128 ? 256 : Cin > 64 ? 128 : 64;
    p.two = p.bn == 256 && F > BM && rows >= PAIR_FROM;        // (F up to 128: half a tile of two CTAs would be empty)
    if (p.two) sms /= 2;
    p.m_tiles = 2 * ceil_div(F, p.two ? 2 * BM : BM);
    p.n_tiles = ceil_div(Cin, p.bn);
    const long long tiles = (long long)p.m_tiles * p.n_tiles;
    const int steps = ceil_div(rows, KSTEP);
    long long s = tiles < sms ? sms / tiles : 1;
    if (s > (steps + 7) / 8) s = (steps + 7) / 8;
    p.splits = (int)s;
    return p;
}
inline wcc_status dw(const void* dG, const void* dU, const void* x, Args a, const DwPlan& p, const DeviceInfo& di, cudaStream_t st)
{
    a.m_tiles = p.m_tiles;
    a.n_tiles = p.n_tiles;
    a.splits = p.splits;
    CUtensorMap A0, A1, B;
    if (!map_of(&A0, dG, a.F, a.rows, KSTEP, true) || !map_of(&A1, dU, a.F, a.rows, KSTEP, true) || !map_of(&B, x, a.Cin, a.rows, KSTEP, true)) return WCC_ERR_CUDA;
    const wcc_status s = products<DW>(p.bn, p.two, A0, A1, B, B, a, di, st);
    if (s != WCC_OK || p.splits == 1) return s;
    const size_t each = (size_t)a.F * a.Cin;
    return launch_overlapped(add_parts, dim3((unsigned)((each + 127) / 128)), dim3(128), 0, st, true, 1, a.part, p.splits, each, a.y, a.y2);
}

struct Layout { size_t exps, row_exp, dG, dU, x16, W16, part, total; };
inline Layout layout_of(int rows, int Cin, int F)
{
    Layout l;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t a = at; at = align_up(at + bytes, 256); return a; };
    l.exps = take(sizeof(Exps));
    l.row_exp = take((size_t)rows * 2);
    l.dG = take((size_t)rows * F * 2);
    l.dU = take((size_t)rows * F * 2);
    l.x16 = take((size_t)rows * Cin * 2);
    l.W16 = take((size_t)2 * F * Cin * 2);
    const DwPlan p = dw_plan(rows, Cin, F, B200_SMS);
    l.part = take(p.splits > 1 ? (size_t)p.splits * 2 * F * Cin * 4 : 0);
    l.total = at;
    return l;
}

inline wcc_status operands(const void* dy, const void* x, const void* Wg, const void* Wu, const Args& a, Exps* exps, short* row_exp, void* x16, void* W16,
                           const DeviceInfo& di, cudaStream_t st)
{
    const __nv_bfloat16 *px = static_cast<const __nv_bfloat16*>(x), *pg = static_cast<const __nv_bfloat16*>(Wg), *pu = static_cast<const __nv_bfloat16*>(Wu);
    wcc_status s = launch_clear(exps, 256, st);
    if (s != WCC_OK) return s;
    const bool wide = a.F >= 2048 || a.Cin >= 2048;
    const int each = wide ? 8 : 32;
    const long long all = ((long long)a.rows + 2LL * a.F + each - 1) / each, most = (long long)di.sms * 8;
    s = launch_overlapped(wide ? exponents<32> : exponents<8>, dim3((unsigned)(all < most ? all : most)), dim3(256), 0, st, true, 1, static_cast<const __nv_bfloat16*>(dy), px, pg, pu, a.rows, a.Cin, a.F,
                          row_exp, exps);
    if (s != WCC_OK) return s;
    const long long n = ((x16 ? (long long)a.rows : 0) + (W16 ? 2LL * a.F : 0)) * (a.Cin / 8), want = (n + 255) / 256;
    return launch_overlapped(to_half, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, true, 1, px, pg, pu, a.rows, a.Cin, a.F, row_exp, exps, a.log_cin,
                             divisor_of((unsigned)(a.Cin / 8)), static_cast<uint4*>(x16), static_cast<uint4*>(W16));
}

}  // namespace gt
}  // namespace wcc
