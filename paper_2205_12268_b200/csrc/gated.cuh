// The gated pointwise block y = act(x Wg^T) * (x Wu^T) and its backward pass, bf16 on the tensor cores (tcgen05, accumulators in tensor memory).
//
// Four uses of one contraction kernel, D[128 x BN] += A[128 x 64] B[64 x BN] per step of the ring:
//   FORWARD  A = x (rows x channels), B = BN/2 rows of Wg and BN/2 of Wu: a gate and its partner are BN/2 columns apart in the same lane of
//            tensor memory, so the epilogue has both and writes y, rounded once.
//   PARTS    the same product again, its epilogue reads dy and writes dG and dU (bf16, operands of what follows)
//   DX       A = dG then dU (rows x F), B = Wg then Wu as they lie: [F][Cin] has the contraction outside, an operand whose columns are contiguous
//   DW       A = dG or dU with the rows as contraction, B = x the same way: both lie with the contraction outside.  Few tiles (weights are small
//            next to maps) are cut along the rows, partial sums in fp32 are added in order by a kernel of their own.
// TMA (128-byte swizzle, no multicast) feeds a ring of stages, one thread issues the instructions, the accumulator is double-buffered, so the
// epilogue of a tile runs under the products of the next one.  Sizes that are no multiples of a tile arrive as zeros from TMA.
#pragma once

#include "tcgen05.cuh"
#include "tma.cuh"
#include "vec.cuh"

namespace wcc {
namespace gt {

using namespace tc;
using tr::exp2_approx;
using tr::rcp_approx;
using tr::sigmoid;

enum Use { FORWARD, PARTS, DX, DW };

constexpr int BM = 128, KSTEP = 64, THREADS = 320;
constexpr int A_BYTES = BM * KSTEP * 2;

template <int BN> constexpr int STAGES_OF = BN == 256 ? 4 : BN == 128 ? 6 : 8;
template <int BN> constexpr int STAGE_BYTES_OF = A_BYTES + BN * KSTEP * 2;

struct Ctl {
    uint64_t full[8], empty[8], tfull[2], tempty[2];
    uint32_t tmem_base;
    int abort_flag;
};

struct Args {
    int rows, Cin, F;
    int m_tiles, n_tiles, splits;          // DW: m_tiles counts those of dG and dU
    int act;
    const __nv_bfloat16* dy;
    __nv_bfloat16 *y, *y2;                 // FORWARD y; PARTS dG, dU; DX dx; DW dWg, dWu
    float* part;                           // DW with splits > 1: [splits][2 F][Cin]
    int* status;
};

// Operand with the contraction outside: rows of 64 columns (128 bytes, swizzled), groups of 8 of the contraction 1024 bytes apart, the next 64 columns
// KSTEP rows further on.
__device__ __forceinline__ uint64_t smem_desc_outer(uint32_t addr)
{
    const uint32_t lo = ((addr & 0x3FFFFu) >> 4) | ((uint32_t)(KSTEP * 128 >> 4) << 16);
    const uint32_t hi = (1024u >> 4) | (1u << 14) | (2u << 29);
    return ((uint64_t)hi << 32) | lo;
}

// Value and derivative of the activation.
// gelu: Phi by Abramowitz and Stegun 7.1.26 (erf to 1.5e-7 absolute: far below the result's rounding).
struct Act { float a, d; };
template <int ACT> __device__ __forceinline__ Act act_of(float z)
{
    if constexpr (ACT == WCC_ACT_RELU) return {z < 0.0f ? 0.0f : z, z > 0.0f ? 1.0f : 0.0f};
    if constexpr (ACT == WCC_ACT_SILU) {
        const float s = sigmoid(z), a = z * s;
        return {a, __fmaf_rn(a, 1.0f - s, s)};
    }
    if constexpr (ACT == WCC_ACT_GELU) {
        const float x = fabsf(z) * 0.70710678118654752f;
        const float t = rcp_approx(__fmaf_rn(0.3275911f, x, 1.0f));
        const float e = exp2_approx(z * z * -0.72134752044448170f);                // e^(-z^2 / 2)
        float p = __fmaf_rn(1.061405429f, t, -1.453152027f);
        p = __fmaf_rn(p, t, 1.421413741f);
        p = __fmaf_rn(p, t, -0.284496736f);
        p = __fmaf_rn(p, t, 0.254829592f);
        const float h = 0.5f * p * t * e, phi = z < 0.0f ? h : 1.0f - h;
        return {z * phi, __fmaf_rn(z * 0.39894228040143268f, e, phi)};
    }
    return {z, 1.0f};
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&r)[16])
{
    uint32_t u[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
                   "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
                 : "r"(taddr));
#pragma unroll
    for (int i = 0; i < 16; ++i) r[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void tmem_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* f)
{
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* f)
{
    const uint4 w = __ldg(reinterpret_cast<const uint4*>(p));
    f[0] = bf16lo(w.x); f[1] = bf16hi(w.x); f[2] = bf16lo(w.y); f[3] = bf16hi(w.y);
    f[4] = bf16lo(w.z); f[5] = bf16hi(w.z); f[6] = bf16lo(w.w); f[7] = bf16hi(w.w);
}

// 16 columns of a gate and its partner: to y, or with dy to dG and dU.  `cols`: those inside the matrix (a multiple of 8).
template <int USE, int ACT>
__device__ __forceinline__ void gate16(const Args& a, const float (&g)[16], const float (&u)[16], size_t at, int cols)
{
    float o[16], o2[16], d[16];
    if constexpr (USE == PARTS) {
#pragma unroll
        for (int i = 0; i < 16; i += 8)
            if (i < cols) load8(a.dy + at + i, d + i);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const Act v = act_of<ACT>(g[i]);
        if constexpr (USE == FORWARD) {
            o[i] = v.a * u[i];
        } else {
            o[i] = d[i] * u[i] * v.d;
            o2[i] = d[i] * v.a;
        }
    }
#pragma unroll
    for (int i = 0; i < 16; i += 8)
        if (i < cols) {
            store8(a.y + at + i, o + i);
            if constexpr (USE == PARTS) store8(a.y2 + at + i, o2 + i);
        }
}

template <int USE, int BN>
__global__ void __launch_bounds__(THREADS, 1)
contract(const __grid_constant__ CUtensorMap tA0, const __grid_constant__ CUtensorMap tA1, const __grid_constant__ CUtensorMap tB0,
         const __grid_constant__ CUtensorMap tB1, const __grid_constant__ Args a)
{
    constexpr int ST = STAGES_OF<BN>, SB = STAGE_BYTES_OF<BN>, COLS = 2 * BN;
    constexpr bool A_OUTER = USE == DW, B_OUTER = USE == DX || USE == DW;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    Ctl* ctl = reinterpret_cast<Ctl*>(smem_raw + (base - raw) + (size_t)ST * SB);
    volatile int* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int items = a.m_tiles * a.n_tiles * a.splits;
    // steps of the ring for an item: along the channels, along F twice, along the rows
    const int f_steps = (a.F + KSTEP - 1) / KSTEP, row_steps = (a.rows + KSTEP - 1) / KSTEP;
    const int all_steps = USE == DX ? 2 * f_steps : USE == DW ? row_steps : (a.Cin + KSTEP - 1) / KSTEP;

    if (threadIdx.x == 0) {
        for (int s = 0; s < ST; ++s) { mbar_init(smem_u32(&ctl->full[s]), 1); mbar_init(smem_u32(&ctl->empty[s]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&ctl->tfull[b]), 1); mbar_init(smem_u32(&ctl->tempty[b]), 8); }
        ctl->abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&ctl->tmem_base)), "r"((uint32_t)COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem_base = ctl->tmem_base;
    bool failed = false;
    pdl_wait();
    pdl_launch();

    // item = (split * m_tiles + m) * n_tiles + n
    if (warp == 0) {
        if (lane == 0) {
            int it = 0;
            for (int w = blockIdx.x; w < items && !failed; w += gridDim.x) {
                const int nt = w % a.n_tiles, ms = w / a.n_tiles, mt = ms % a.m_tiles, sp = ms / a.m_tiles;
                const int k0 = (int)((long long)all_steps * sp / a.splits), k1 = (int)((long long)all_steps * (sp + 1) / a.splits);
                for (int k = k0; k < k1; ++k, ++it) {
                    const int s = it % ST;
                    const uint32_t ph = (uint32_t)(it / ST) & 1u;
                    if (!mbar_wait(smem_u32(&ctl->empty[s]), ph ^ 1u, abort_flag)) { failed = true; break; }
                    const uint32_t sA = base + (uint32_t)s * SB, sB = sA + A_BYTES, bar = smem_u32(&ctl->full[s]);
                    mbar_expect_tx(bar, (uint32_t)SB);
                    if constexpr (USE == FORWARD || USE == PARTS) {
                        tma_load_2d(sA, &tA0, k * KSTEP, mt * BM, bar);
                        tma_load_2d(sB, &tB0, k * KSTEP, nt * (BN / 2), bar);
                        tma_load_2d(sB + BN / 2 * 128, &tB1, k * KSTEP, nt * (BN / 2), bar);
                    } else if constexpr (USE == DX) {
                        const bool up = k >= f_steps;
                        const int f0 = (up ? k - f_steps : k) * KSTEP;
                        tma_load_2d(sA, up ? &tA1 : &tA0, f0, mt * BM, bar);
                        for (int i = 0; i < BN / 64; ++i) tma_load_2d(sB + i * KSTEP * 128, up ? &tB1 : &tB0, nt * BN + 64 * i, f0, bar);
                    } else {
                        const int half = a.m_tiles / 2;
                        const bool up = mt >= half;
                        const int f0 = (up ? mt - half : mt) * BM;
                        for (int i = 0; i < 2; ++i) tma_load_2d(sA + i * KSTEP * 128, up ? &tA1 : &tA0, f0 + 64 * i, k * KSTEP, bar);
                        for (int i = 0; i < BN / 64; ++i) tma_load_2d(sB + i * KSTEP * 128, &tB0, nt * BN + 64 * i, k * KSTEP, bar);
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            // D fp32, A and B bf16; bits 15 and 16: the contraction lies outside
            constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((A_OUTER ? 1u : 0u) << 15) | ((B_OUTER ? 1u : 0u) << 16) |
                                       ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);
            int it = 0, item = 0;
            for (int w = blockIdx.x; w < items && !failed; w += gridDim.x, ++item) {
                const int sp = w / a.n_tiles / a.m_tiles;
                const int k0 = (int)((long long)all_steps * sp / a.splits), k1 = (int)((long long)all_steps * (sp + 1) / a.splits);
                const int buf = item & 1;
                const uint32_t bph = (uint32_t)(item >> 1) & 1u;
                if (!mbar_wait(smem_u32(&ctl->tempty[buf]), bph ^ 1u, abort_flag)) { failed = true; break; }
                fence_after();
                const uint32_t d = tmem_base + (uint32_t)(buf * BN);
                uint32_t accumulate = 0;
                for (int k = k0; k < k1; ++k, ++it) {
                    const int s = it % ST;
                    const uint32_t ph = (uint32_t)(it / ST) & 1u;
                    if (!mbar_wait(smem_u32(&ctl->full[s]), ph, abort_flag)) { failed = true; break; }
                    fence_after();
                    const uint32_t sA = base + (uint32_t)s * SB, sB = sA + A_BYTES;
                    const uint64_t ad = A_OUTER ? smem_desc_outer(sA) : smem_desc_sw128(sA), bd = B_OUTER ? smem_desc_outer(sB) : smem_desc_sw128(sB);
#pragma unroll
                    for (int kk = 0; kk < KSTEP / 16; ++kk) {      // 16 of the contraction: 32 bytes of a row, or 16 rows of 128 bytes
                        mma_ss<false>(d, ad + (uint64_t)((A_OUTER ? 128 : 2) * kk), bd + (uint64_t)((B_OUTER ? 128 : 2) * kk), idesc, accumulate);
                        accumulate = 1;
                    }
                    mma_commit(smem_u32(&ctl->empty[s]));
                }
                if (failed) break;
                mma_commit(smem_u32(&ctl->tfull[buf]));
            }
        }
        __syncwarp();
    } else {
        const int q = warp & 3, half = (warp - 2) >> 2;        // lanes of tensor memory that the warp may read; its half of the columns
        int item = 0;
        for (int w = blockIdx.x; w < items; w += gridDim.x, ++item) {
            const int nt = w % a.n_tiles, ms = w / a.n_tiles, mt = ms % a.m_tiles, sp = ms / a.m_tiles;
            const int buf = item & 1;
            const uint32_t bph = (uint32_t)(item >> 1) & 1u;
            int ok = mbar_wait(smem_u32(&ctl->tfull[buf]), bph, abort_flag) ? 1 : 0;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) { failed = true; break; }
            fence_after();
            const uint32_t taddr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(buf * BN);
            if constexpr (USE == FORWARD || USE == PARTS) {
                const int row = mt * BM + q * 32 + lane;
                for (int c = half * (BN / 4); c < (half + 1) * (BN / 4); c += 16) {
                    const int col = nt * (BN / 2) + c;
                    if (col >= a.F) break;                      // (the whole warp)
                    float g[16], u[16];
                    tmem_ld16(taddr + (uint32_t)c, g);
                    tmem_ld16(taddr + (uint32_t)(BN / 2 + c), u);
                    tmem_wait();
                    if (row < a.rows) {
                        const size_t at = (size_t)row * a.F + col;
                        const int cols = a.F - col;
                        if (a.act == WCC_ACT_SILU) gate16<USE, WCC_ACT_SILU>(a, g, u, at, cols);
                        else if (a.act == WCC_ACT_GELU) gate16<USE, WCC_ACT_GELU>(a, g, u, at, cols);
                        else if (a.act == WCC_ACT_RELU) gate16<USE, WCC_ACT_RELU>(a, g, u, at, cols);
                        else gate16<USE, WCC_ACT_NONE>(a, g, u, at, cols);
                    }
                    __syncwarp();
                }
            } else {
                const int mhalf = a.m_tiles / 2;
                const bool up = USE == DW && mt >= mhalf;
                const int row = (up ? mt - mhalf : mt) * BM + q * 32 + lane, limit = USE == DW ? a.F : a.rows;
                for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += 16) {
                    const int col = nt * BN + c;
                    if (col >= a.Cin) break;
                    float v[16];
                    tmem_ld16(taddr + (uint32_t)c, v);
                    tmem_wait();
                    if (row < limit) {
                        if (USE == DW && a.splits > 1) {
                            float* p = a.part + (((size_t)sp * 2 + (up ? 1 : 0)) * a.F + row) * a.Cin + col;
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                if (col + i < a.Cin) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
                        } else {
                            __nv_bfloat16* p = (up ? a.y2 : a.y) + (size_t)row * a.Cin + col;
#pragma unroll
                            for (int i = 0; i < 16; i += 8)
                                if (col + i < a.Cin) store8(p + i, v + i);
                        }
                    }
                    __syncwarp();
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->tempty[buf]));
        }
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
    if (warp == 1) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)COLS) : "memory");
    }
}

// Partial sums of the weights' gradients, added in order, four values a thread.
static __global__ void __launch_bounds__(256) add_parts(const float* __restrict__ part, int splits, size_t each, __nv_bfloat16* __restrict__ dWg,
                                                        __nv_bfloat16* __restrict__ dWu)
{
    pdl_wait();
    pdl_launch();
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= 2 * each) return;
    float4 v = __ldcg(reinterpret_cast<const float4*>(part + i));
#pragma unroll 4
    for (int s = 1; s < splits; ++s) {
        const float4 p = __ldcg(reinterpret_cast<const float4*>(part + (size_t)s * 2 * each + i));
        v.x += p.x; v.y += p.y; v.z += p.z; v.w += p.w;
    }
    __nv_bfloat16* dst = i < each ? dWg + i : dWu + (i - each);
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// ---- host ------------------------------------------------------------------------------------------
// [outer][inner] bf16, boxes of 64 x `box` rows.
inline bool map_of(CUtensorMap* tm, const void* p, int inner, int outer, int box)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)outer}, strides[1] = {(cuuint64_t)inner * 2};
    cuuint32_t boxes[2] = {64, (cuuint32_t)box}, steps[2] = {1, 1};
    return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int USE, int BN>
wcc_status launch(const CUtensorMap& A0, const CUtensorMap& A1, const CUtensorMap& B0, const CUtensorMap& B1, const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int smem = 1024 + STAGES_OF<BN> * STAGE_BYTES_OF<BN> + (int)sizeof(Ctl) + 16;
    const wcc_status s = allow_smem<contract<USE, BN>>(di.dev, smem);
    if (s != WCC_OK) return s;
    const int items = a.m_tiles * a.n_tiles * a.splits;
    return launch_overlapped(contract<USE, BN>, dim3((unsigned)(items < di.sms ? items : di.sms)), dim3(THREADS), smem, st, true, 1, A0, A1, B0, B1, a);
}

// Columns of a tile: as many as fill the SMs, 64 at least.  `cols` columns in all (FORWARD: gates and partners).
inline int tile_of(int m_tiles, long long cols, int sms)
{
    int bn = 256;
    while (bn > 64 && (cols <= bn / 2 || (long long)m_tiles * ((cols + bn - 1) / bn) < sms)) bn /= 2;
    return bn;
}

template <int USE>
wcc_status gates(const void* x, const void* Wg, const void* Wu, Args a, const DeviceInfo& di, cudaStream_t st)
{
    a.m_tiles = ceil_div(a.rows, BM);
    const int bn = tile_of(a.m_tiles, 2LL * a.F, di.sms);
    a.n_tiles = ceil_div(a.F, bn / 2);
    a.splits = 1;
    CUtensorMap A, G, U;
    if (!map_of(&A, x, a.Cin, a.rows, BM) || !map_of(&G, Wg, a.Cin, a.F, bn / 2) || !map_of(&U, Wu, a.Cin, a.F, bn / 2)) return WCC_ERR_CUDA;
    if (bn == 256) return launch<USE, 256>(A, A, G, U, a, di, st);
    if (bn == 128) return launch<USE, 128>(A, A, G, U, a, di, st);
    return launch<USE, 64>(A, A, G, U, a, di, st);
}

inline wcc_status dx(const void* dG, const void* dU, const void* Wg, const void* Wu, Args a, const DeviceInfo& di, cudaStream_t st)
{
    a.m_tiles = ceil_div(a.rows, BM);
    const int bn = tile_of(a.m_tiles, a.Cin, di.sms);
    a.n_tiles = ceil_div(a.Cin, bn);
    a.splits = 1;
    CUtensorMap A0, A1, B0, B1;
    if (!map_of(&A0, dG, a.F, a.rows, BM) || !map_of(&A1, dU, a.F, a.rows, BM) || !map_of(&B0, Wg, a.Cin, a.F, KSTEP) || !map_of(&B1, Wu, a.Cin, a.F, KSTEP))
        return WCC_ERR_CUDA;
    if (bn == 256) return launch<DX, 256>(A0, A1, B0, B1, a, di, st);
    if (bn == 128) return launch<DX, 128>(A0, A1, B0, B1, a, di, st);
    return launch<DX, 64>(A0, A1, B0, B1, a, di, st);
}

struct DwPlan { int bn, m_tiles, n_tiles, splits; };
inline DwPlan dw_plan(int rows, int Cin, int F, int sms)
{
    DwPlan p;
    p.bn = Cin > 128 ? 256 : Cin > 64 ? 128 : 64;
    p.m_tiles = 2 * ceil_div(F, BM);
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
    if (!map_of(&A0, dG, a.F, a.rows, KSTEP) || !map_of(&A1, dU, a.F, a.rows, KSTEP) || !map_of(&B, x, a.Cin, a.rows, KSTEP)) return WCC_ERR_CUDA;
    wcc_status s;
    if (p.bn == 256) s = launch<DW, 256>(A0, A1, B, B, a, di, st);
    else if (p.bn == 128) s = launch<DW, 128>(A0, A1, B, B, a, di, st);
    else s = launch<DW, 64>(A0, A1, B, B, a, di, st);
    if (s != WCC_OK || p.splits == 1) return s;
    const size_t each = (size_t)a.F * a.Cin;
    return launch_overlapped(add_parts, dim3((unsigned)((2 * each / 4 + 255) / 256)), dim3(256), 0, st, true, 1, a.part, p.splits, each, a.y, a.y2);
}

struct Layout { size_t dG, dU, part, total; };
inline Layout layout_of(int rows, int Cin, int F)
{
    Layout l;
    l.dG = 0;
    l.dU = align_up((size_t)rows * F * 2, 256);
    l.part = 2 * l.dU;
    const DwPlan p = dw_plan(rows, Cin, F, B200_SMS);
    l.total = l.part + (p.splits > 1 ? align_up((size_t)p.splits * 2 * F * Cin * 4, 256) : 0);
    return l;
}

}  // namespace gt
}  // namespace wcc
