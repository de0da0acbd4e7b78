// Low-rank adapters of many requests beside a shared projection.  Image n of the batch has adapter a = ids[n] (or none) with factors
// A_a [r][Cin], B_a [Cout][r] and a scale t_a:
//     forward    U = A_a x_n,        y_n  = base_n + t_a B_a U
//     backward   V = t_a B_a^T dy_n, dx_n = base_n + A_a^T V,   dA_a = sum_n V x_n^T,   dB_a = t_a sum_n dy_n U^T
// The rank is at most 64 and the maps are long, so both products together do about r / 2 operations a byte: the maps are the bound, not the
// tensor pipes, and everything is arranged around reading and writing them once in whole lines.  A warp keeps the product of the first
// factor in registers as the operand of the second: nothing of rank r goes to memory in the forward pass.  (With accumulators in tensor memory it
// would go through there and shared memory between the two; the warp-level instructions reach 20 to 40 % of their rate when the maps come at 5 TB/s.)
//
// The products are warp-level matrix instructions on registers.  Their rows, columns and summation index can be any permutation of
// positions, ranks and channels that both operands agree on, and that freedom replaces every shuffle and transposition through shared memory:
//  - first product, D[position][rank]: lane (g, t) = (lane / 4, lane % 4) takes 16 bytes of a channel, NP positions from p0 + NP g on; its b-th
//    position is row g of row block b / 2 (upper half for odd b), its channels of a group are the CL from CL t on;
//  - second product, D[channel][position]: the accumulators of position b are its operand as they stand, one instruction column block per b,
//    and lane t ends up with 2 NP positions in a row of memory, 32 bytes, of the two channels g and g + 8.
// The factors are laid out in the order of the instructions, by each CTA in shared memory or, where they are large, once by prep_kernel.  The maps
// come through a ring of asynchronous copies that belongs to one warp (Feed).
// bf16 maps: the factors are bf16, U is split into two bf16 parts (relative error 2^-17), sums are fp32.  fp32 maps: every operand is split into
// two parts of 11 bits, three products of them are summed in fp32 (relative error about 2^-21 a term, beside 2^-24 of each fp32 addition).
#pragma once

#include <algorithm>

#include "common.cuh"

namespace wcc {
namespace ad {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int MAX_RANK = 64;
// What the sizes of a call decide against (us, bf16 project = 144 -> 24 on 4 x 128 x 256, fp32 headline = 64 -> 64 on 12 x 96 x 320, both rank 16):
constexpr int HALF_FROM = 8;            // blocks of 8 ranks from which a lane takes half as many positions (from 8 / 4 / 1: headline 66 / 65 / 73)
constexpr long long FILL = 12;          // warps an SM below which the warps of a CTA share tiles (12 / 24: 826 -> 899 on 14 x 18 x 72 59 / 72)
constexpr int STAGES = 3;               // of a warp's feed (3 / 4: headline 57 / 62); rows that start anywhere: 2 (58 -> 70 on 3 x 129 x 257: 3 32, 2 27)
constexpr int WAVES = 3;                // CTAs for each that fits at once, since images without an adapter are done early (1 / 3 / 6: headline 70 / 62 / 65;
                                        // its backward pass, 1 / 2 / 3: 120 / 117 / 112)

template <typename T> struct Geo;
template <> struct Geo<__nv_bfloat16> { static constexpr int NP = 8, TP = 64, CL = 8, GC = 32, PARTS = 1; };
template <> struct Geo<float> { static constexpr int NP = 4, TP = 32, CL = 4, GC = 16, PARTS = 2; };
// NP positions of a lane (16 bytes) and TP of a warp's tile in the widest form, CL channels of a lane in a group of GC, PARTS parts of a factor's
// element.  For the largest ranks a lane takes half as many positions, which halves the sums it has to hold.
template <typename T> __host__ __device__ constexpr int lane_positions(int rb) { return rb >= HALF_FROM ? Geo<T>::NP / 2 : Geo<T>::NP; }

// steps of the second product's summation index, ranks in blocks of 8
template <typename T> __host__ __device__ constexpr int steps2(int rb) { return sizeof(T) == 2 ? (rb + 1) / 2 : rb; }

// The matrix instructions cut their sums off instead of rounding them, an error with a sign: chains of them are kept short (a group of
// channels, a tile of positions) and added up by ordinary additions.  In one chain the gradients of the headline batch were off by 9e-6.
__device__ __forceinline__ void add(float (&s)[4], const float (&d)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += d[i];
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) { mma_bf16(d, a[0], a[1], a[2], a[3], b0, b1); }
__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) { mma_tf32(d, a[0], a[1], a[2], a[3], b0, b1); }
// x = hi + lo, hi rounded to 11 bits, lo cut to 11 bits: |x - hi - lo| <= 2^-21 |x|.  A NaN whose hi rounds over into a zero stays one in lo.
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t& hi, uint32_t& lo)
{
    hi = (x + 0x1000u) & 0xFFFFE000u;
    lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(hi)) & 0xFFFFE000u;
}
// u = hi + lo in bf16 pairs, |u - hi - lo| <= 2^-17 |u|; with a third part 2^-25
__device__ __forceinline__ void split_bf16(float u0, float u1, uint32_t& hi, uint32_t& lo)
{
    hi = pack_bf16x2(u0, u1);
    lo = pack_bf16x2(u0 - bf16lo(hi), u1 - bf16hi(hi));
}

// NP positions of a channel's row from p on as they lie in memory, those at P and beyond as zeros.  VEC: rows start on multiples of NP positions.
// Otherwise the two aligned pieces around them are loaded and shifted into place (`end`: behind the tensor's last element, nothing is read from
// there on).
template <int WORDS> struct Words { uint32_t w[WORDS]; };
template <int W> __device__ __forceinline__ Words<W> load_words(const void* p)
{
    Words<W> r;
    if constexpr (W == 4) {
        const uint4 u = *static_cast<const uint4*>(p);
        r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
    } else {
        const uint2 u = *static_cast<const uint2*>(p);
        r.w[0] = u.x; r.w[1] = u.y;
    }
    return r;
}
template <int W> __device__ __forceinline__ void store_words(void* p, const Words<W>& v)
{
    if constexpr (W == 8)
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     ::"l"(p), "r"(v.w[0]), "r"(v.w[1]), "r"(v.w[2]), "r"(v.w[3]), "r"(v.w[4]), "r"(v.w[5]), "r"(v.w[6]), "r"(v.w[7]) : "memory");
    else if constexpr (W == 4) *static_cast<uint4*>(p) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
    else *static_cast<uint2*>(p) = make_uint2(v.w[0], v.w[1]);
}
template <typename T, int NP, bool VEC>
__device__ __forceinline__ Words<NP * (int)sizeof(T) / 4> load_row(const T* row, size_t p, size_t P, const T* end)
{
    constexpr int W = NP * (int)sizeof(T) / 4;
    Words<W> r{};
    if (p >= P) return r;
    if constexpr (VEC) {
        return load_words<W>(row + p);
    } else {
        const T* q = row + p;
        const int m = (int)((reinterpret_cast<uintptr_t>(q) / sizeof(T)) % NP);
        q -= m;                                                         // (a tensor starts on 16 bytes)
        uint32_t w[2 * W];
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) w[i] = 0u;
#pragma unroll
        for (int h = 0; h < 2; ++h, q += NP) {
            if (h == 1 && m == 0) break;
            if (q + NP <= end) {
                const Words<W> u = load_words<W>(q);
#pragma unroll
                for (int i = 0; i < W; ++i) w[h * W + i] = u.w[i];
            } else {
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    if (q + i < end) {
                        if (sizeof(T) == 2) w[(h * W + (i >> 1)) % (2 * W)] |= (uint32_t)reinterpret_cast<const uint16_t*>(q)[i] << (16 * (i & 1));
                        else w[(h * W + i) % (2 * W)] = reinterpret_cast<const uint32_t*>(q)[i];
                    }
            }
        }
        const int sw = sizeof(T) == 2 ? m >> 1 : m;                     // whole words first
#pragma unroll
        for (int step = W / 2; step >= 1; step /= 2)
            if (sw & step) {
#pragma unroll
                for (int i = 0; i + step < 2 * W; ++i) w[i] = w[i + step];
            }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            r.w[i] = sizeof(T) == 2 ? __funnelshift_r(w[i], w[i + 1], 16 * (m & 1)) : w[i];
            if (p + NP > P) {
                if (sizeof(T) == 2) {
                    if (p + 2 * i >= P) r.w[i] = 0u;
                    else if (p + 2 * i + 1 >= P) r.w[i] &= 0xFFFFu;
                } else if (p + i >= P) r.w[i] = 0u;
            }
        }
        return r;
    }
}
template <typename T> __device__ __forceinline__ float load_one(const T* p)
{
    return sizeof(T) == 4 ? *reinterpret_cast<const float*>(p) : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16);
}
template <typename T> __device__ __forceinline__ void store_one(T* p, float v)
{
    if (sizeof(T) == 4) *reinterpret_cast<float*>(p) = v;
    else *reinterpret_cast<uint16_t*>(p) = (uint16_t)pack_bf16x2(v, 0.0f);
}

// ---- factors in the order of the matrix instructions -----------------------------------------
// A factor as seen by a product: element (j, c) at p[a * sa + j * sj + c * sc].
template <typename T>
struct Factor { const T* p; long long sa; int sj, sc; };

// First product: [group of GC channels][block of 8 ranks][part][lane] 16 bytes (CL channels of rank g).
// Second product: [block of 16 channels][step][part][lane] 16 bytes.
template <typename T> __host__ __device__ inline size_t first_words(int rb, int K) { return (size_t)((K + Geo<T>::GC - 1) / Geo<T>::GC) * rb * Geo<T>::PARTS * 32; }
template <typename T> __host__ __device__ inline size_t second_words(int rb, int M) { return (size_t)((M + 15) / 16) * steps2<T>(rb) * Geo<T>::PARTS * 32; }

template <typename T>
__device__ __forceinline__ uint32_t element(const T* f, int j, int c, int sj, int sc, int r, int C)
{
    if (j >= r || c >= C) return 0u;
    const T* q = f + (long long)j * sj + (long long)c * sc;
    return sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(q) : *reinterpret_cast<const uint32_t*>(q);
}
// Adapter a's factor into `out`; this thread takes words i0, i0 + step, ...
template <typename T>
__device__ __forceinline__ void lay_first(const Factor<T>& f, int a, int r, int rb, int K, uint4* out, int i0, int step)
{
    constexpr int GC = Geo<T>::GC, CL = Geo<T>::CL, PARTS = Geo<T>::PARTS;
    const T* p = f.p + a * f.sa;
    const int n = (int)(first_words<T>(rb, K) / PARTS);
    const bool wide = f.sc == 1 && K % CL == 0;                          // a lane's channels are 16 aligned bytes
    for (int i = i0; i < n; i += step) {
        const int lane = i & 31, jb = (i >> 5) % rb, grp = (i >> 5) / rb;
        const int j = 8 * jb + (lane >> 2), c = grp * GC + (lane & 3) * CL;
        uint32_t w[4] = {0u, 0u, 0u, 0u}, lo[4];
        if (wide) {
            if (j < r && c < K) {
                const uint4 u = *reinterpret_cast<const uint4*>(p + (long long)j * f.sj + c);
                w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < CL; ++k) {
                const uint32_t e = element(p, j, c + k, f.sj, f.sc, r, K);
                if (sizeof(T) == 2) w[(k >> 1) & 3] |= e << (16 * (k & 1));
                else w[k & 3] = e;
            }
        }
        if (PARTS == 2) {
#pragma unroll
            for (int k = 0; k < 4; ++k) split_tf32(w[k], w[k], lo[k]);
        }
        uint4* o = out + (i >> 5) * (PARTS * 32) + lane;
        o[0] = make_uint4(w[0], w[1], w[2], w[3]);
        if (PARTS == 2) o[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}
template <typename T>
__device__ __forceinline__ void lay_second(const Factor<T>& f, int a, int r, int rb, int M, uint4* out, int i0, int step)
{
    constexpr int PARTS = Geo<T>::PARTS;
    const T* p = f.p + a * f.sa;
    const int ns = steps2<T>(rb), n = (int)(second_words<T>(rb, M) / PARTS);
    const bool pairs = sizeof(T) == 2 && f.sj == 1 && r % 2 == 0;        // two neighbouring ranks are one aligned word
    for (int i = i0; i < n; i += step) {
        const int lane = i & 31, ks = (i >> 5) % ns, mo = (i >> 5) / ns, g = lane >> 2, t = lane & 3;
        uint32_t w[4], lo[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {                                   // registers: channel g, g + 8, then the other half of the step's ranks
            const int o = 16 * mo + g + 8 * (k & 1);
            if (sizeof(T) == 2) {
                const int j = 16 * ks + 8 * (k >> 1) + 2 * t;
                if (pairs) w[k] = j < r && o < M ? *reinterpret_cast<const uint32_t*>(p + (long long)o * f.sc + j) : 0u;
                else w[k] = element(p, j, o, f.sj, f.sc, r, M) | (element(p, j + 1, o, f.sj, f.sc, r, M) << 16);
            } else {
                split_tf32(element(p, 8 * ks + 2 * t + (k >> 1), o, f.sj, f.sc, r, M), w[k], lo[k]);
            }
        }
        uint4* op = out + (i >> 5) * (PARTS * 32) + lane;
        op[0] = make_uint4(w[0], w[1], w[2], w[3]);
        if (PARTS == 2) op[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// The ids of a call as the kernels take them: anything but 0 .. R - 1 is no adapter, and one at R or beyond is an error.  It enters a clear status word
// only: a wait that ran out leaves an output undefined, and nobody may miss that for an index.
__device__ __forceinline__ int adapter_of(const int32_t* ids, int n, int R, int* status)
{
    const int a = ids[n];
    if (a < R) return a < 0 ? -1 : a;
    if (status) atomicCAS(status, (int)WCC_OK, (int)WCC_ERR_INDEX);
    return -1;
}

// What the larger problems prepare in memory: factors too large for a CTA's shared memory, and the order of the images for grad_kernel.
template <typename T>
struct PrepArgs {
    Factor<T> first[2], second;         // p NULL: none
    uint4* first_out[2];
    uint4* second_out;
    int K[2], M;
    int R, r, rb, N;
    const int32_t* ids;
    int32_t* order;                     // images with an adapter by adapter, and per adapter the first of them [R + 1]; or NULL
    int32_t* start;
};

// CTA = one adapter (grid.x) and one stripe of its words (grid.y).  An adapter that no image uses is skipped.
template <typename T>
__global__ void __launch_bounds__(256) prep_kernel(PrepArgs<T> q)
{
    const int a = blockIdx.x;
    pdl_wait();
    pdl_launch();
    bool mine = false;
    for (int n = threadIdx.x; n < q.N; n += 256) mine |= q.ids[n] == a;
    const bool used = __syncthreads_or(mine);
    if (q.order && blockIdx.y == 0 && threadIdx.x < 32) {
        // first place of this adapter's images = images of the adapters before it; then those in ascending order
        int before = 0, total = 0;
        for (int n0 = 0; n0 < q.N; n0 += 32) {
            const int n = n0 + (int)threadIdx.x, v = n < q.N ? q.ids[n] : -1;
            before += __popc(__ballot_sync(FULL, v >= 0 && v < a));
            total += __popc(__ballot_sync(FULL, v >= 0 && v < q.R));
        }
        if (threadIdx.x == 0) { q.start[a] = before; if (a == q.R - 1) q.start[q.R] = total; }
        if (used)
            for (int n0 = 0; n0 < q.N; n0 += 32) {
                const int n = n0 + (int)threadIdx.x;
                const bool hit = n < q.N && q.ids[n] == a;
                const unsigned m = __ballot_sync(FULL, hit);
                if (hit) q.order[before + __popc(m & ((1u << threadIdx.x) - 1u))] = n;
                before += __popc(m);
            }
    }
    if (!used) return;
    const int i0 = blockIdx.y * 256 + threadIdx.x, step = gridDim.y * 256;
#pragma unroll
    for (int side = 0; side < 2; ++side)
        if (q.first[side].p) lay_first<T>(q.first[side], a, q.r, q.rb, q.K[side], q.first_out[side] + a * first_words<T>(q.rb, q.K[side]), i0, step);
    if (q.second.p) lay_second<T>(q.second, a, q.r, q.rb, q.M, q.second_out + a * second_words<T>(q.rb, q.M), i0, step);
}

// ---- the two products over a warp's tile of positions ---------------------------------------------
template <typename T, int RB, int NP_> struct Tile {
    static constexpr int NP = NP_, TP = 8 * NP, MB = NP / 2;
    float acc[MB][RB][4];               // of position NP g + b, rank 8 jb + 2 t + e: [b / 2][jb][2 (b % 2) + e]
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[mb][jb][i] = 0.0f;
    }
    // positions from `n` on of this lane's NP are nothing
    __device__ __forceinline__ void keep(int n)
    {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (2 * mb + (i >> 1) >= n) acc[mb][jb][i] = 0.0f;
    }
    __device__ __forceinline__ void scale(float s)
    {
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[mb][jb][i] *= s;
    }
};
template <bool SM> __device__ __forceinline__ uint4 load_factor(const uint4* p) { return SM ? *p : __ldg(p); }

// Adds a group of channels to the first product: x holds this lane's channels of it, wg points at this lane's words of the factor.
template <typename T, int RB, bool SM, int NP>
__device__ __forceinline__ void first_step(Tile<T, RB, NP>& tile, const Words<NP * (int)sizeof(T) / 4> (&x)[Geo<T>::CL], const uint4* wg)
{
    constexpr int MB = NP / 2, CL = Geo<T>::CL;
    if constexpr (sizeof(T) == 2) {
        uint32_t fa[2][MB][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                fa[s][mb][0] = __byte_perm(x[4 * s].w[mb], x[4 * s + 1].w[mb], 0x5410);
                fa[s][mb][1] = __byte_perm(x[4 * s].w[mb], x[4 * s + 1].w[mb], 0x7632);
                fa[s][mb][2] = __byte_perm(x[(4 * s + 2) % CL].w[mb], x[(4 * s + 3) % CL].w[mb], 0x5410);
                fa[s][mb][3] = __byte_perm(x[(4 * s + 2) % CL].w[mb], x[(4 * s + 3) % CL].w[mb], 0x7632);
            }
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            const uint4 w = load_factor<SM>(wg + jb * 32);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                mma_bf16(d, fa[0][mb], w.x, w.y);
                mma_bf16(d, fa[1][mb], w.z, w.w);
                add(tile.acc[mb][jb], d);
            }
        }
    } else {
        uint32_t hi[2][MB][4], lo[2][MB][4];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int i = 0; i < 4; ++i) split_tf32(x[2 * s + (i >> 1)].w[2 * mb + (i & 1)], hi[s][mb][i], lo[s][mb][i]);
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            const uint4 wh = load_factor<SM>(wg + (jb * 2) * 32), wl = load_factor<SM>(wg + (jb * 2 + 1) * 32);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                mma_tf32(d, lo[0][mb], wh.x, wh.y);
                mma_tf32(d, lo[1][mb], wh.z, wh.w);
                mma_tf32(d, hi[0][mb], wl.x, wl.y);
                mma_tf32(d, hi[1][mb], wl.z, wl.w);
                mma_tf32(d, hi[0][mb], wh.x, wh.y);
                mma_tf32(d, hi[1][mb], wh.z, wh.w);
                add(tile.acc[mb][jb], d);
            }
        }
    }
}

// The maps of first products and the bases of second ones on their way through shared memory: a warp copies the groups of channels ahead of
// their use, also those of its next tile while it writes the last one, and waits for nobody else.
//  - AL, rows that start on vectors: a stage is [GC rows][8 pieces of NP positions], pieces exchanged so that the eight lanes of a phase (two g,
//    four t) read from different banks.
//  - rows that start anywhere: the aligned pieces of 16 bytes around the tile's part of each row, as they lie; the reader shifts.  Single loads of 2
//    bytes cost eight times the instructions, and one after the other: 58 -> 70 channels of 129 x 257 bf16 77 us, shifted in registers 31.
// Rows behind the last channel arrive as zeros; positions behind the last one as zeros (AL) or as what follows them, and nobody keeps what is
// made of them.  Headline batch with the map fed and the base loaded into registers 62 us, both fed 56.
template <typename T, int NP, bool AL>
struct Feed {
    static constexpr int GC = Geo<T>::GC, CL = Geo<T>::CL, PIECE = NP * (int)sizeof(T), S = AL ? STAGES : 2, W = PIECE / 4;
    static constexpr int ROW = 8 * PIECE, PITCH = ROW + (AL ? 0 : 16), CH = PITCH / 16, STAGE = GC * PITCH;
    uint32_t base, fill, use;           // shared address, offsets of the stages to fill and to use next
    size_t off;                         // AL: this lane's first row and piece of a stage, from the stage's first channel at position 0; else p0
    bool in;                            // that piece exists
    __device__ __forceinline__ explicit Feed(void* warp_smem) : base((uint32_t)__cvta_generic_to_shared(warp_smem)), fill(0), use(0), off(0), in(false) {}
    // The following stages are of the tile at p0.
    __device__ __forceinline__ void at(size_t P, size_t p0)
    {
        const int lane = threadIdx.x & 31;
        const size_t p = p0 + (size_t)(NP * (lane & 7));
        in = p < P;
        off = AL ? (size_t)(lane >> 3) * P + (in ? p : 0) : p0;
    }
    // A stage of a first product's group, or (BASE) of 16 channels of a second product's base: rows from `row0` (its first channel, at position 0),
    // `left` > 0 channels of them exist; `end`: behind the tensor.  commit() follows; without an issue before it the stage stays empty.
    template <bool BASE>
    __device__ __forceinline__ void issue(const T* row0, int left, size_t P, const T* end)
    {
        constexpr int ROWS = BASE ? 16 : GC;
        const int lane = threadIdx.x & 31;
        if constexpr (AL) {
            const int r0 = lane >> 3, c = lane & 7;
            const T* src = row0 + off;
            const uint32_t dst = base + fill + (uint32_t)(r0 * ROW);
#pragma unroll
            for (int k = 0; k < ROWS / 4; ++k, src += 4 * P) {
                const bool have = r0 + 4 * k < left;
                const int sw = BASE ? r0 & 1 : PIECE == 16 ? 2 * ((4 * k / CL) & 3) : 4 * ((4 * k / CL) & 1);      // (r0 < 4 <= CL)
                const uint32_t d = dst + (uint32_t)(k * 4 * ROW + (c ^ sw) * PIECE);
                const int bytes = have && in ? PIECE : 0;
                if constexpr (PIECE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(have ? src : row0), "r"(bytes) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(d), "l"(have ? src : row0), "r"(bytes) : "memory");
            }
        } else {
#pragma unroll
            for (int k = 0; k < (ROWS * CH + 31) / 32; ++k) {
                const int i = lane + 32 * k, r = i / CH, ch = i - r * CH;
                if (r >= ROWS) break;
                const bool have = r < left;
                const T* row = row0 + (size_t)(have ? r : 0) * P;
                const char* src = reinterpret_cast<const char*>((reinterpret_cast<uintptr_t>(row + off) & ~(uintptr_t)15) + 16 * ch);
                const bool any = have && off < P && src < reinterpret_cast<const char*>(row + P);
                const long long rest = reinterpret_cast<const char*>(end) - src;      // (a tensor starts on 16 bytes, it may end anywhere)
                const int bytes = any ? (rest < 16 ? (int)rest : 16) : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;"
                             ::"r"(base + fill + (uint32_t)(r * PITCH + 16 * ch)), "l"(any ? src : reinterpret_cast<const char*>((reinterpret_cast<uintptr_t>(row0) & ~(uintptr_t)15))), "r"(bytes) : "memory");
            }
        }
    }
    __device__ __forceinline__ void commit()
    {
        asm volatile("cp.async.commit_group;" ::: "memory");
        fill = fill == (S - 1) * STAGE ? 0 : fill + STAGE;
    }
    // Waits for the next stage; the stage before it may be filled again behind this.
    __device__ __forceinline__ void wait()
    {
        asm volatile("cp.async.wait_group %0;" ::"n"(S - 2) : "memory");
        __syncwarp();
    }
    static __device__ __forceinline__ void read(uint32_t a, uint32_t* w)
    {
        if constexpr (PIECE == 16) asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
        else asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a));
    }
    // Where a row that starts at `row` (its address at p0) begins in the 16 bytes that hold it.
    static __device__ __forceinline__ uint32_t skew(const T* row0, size_t P, size_t p0, int r)
    {
        return ((uint32_t)reinterpret_cast<uintptr_t>(row0) + ((uint32_t)p0 + (uint32_t)r * (uint32_t)P) * (uint32_t)sizeof(T)) & 15u;
    }
    // row0, p0: as in issue and at (rows that start anywhere)
    __device__ __forceinline__ void take(Words<W> (&x)[CL], const T* row0, size_t P, size_t p0)
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
        if constexpr (AL) {
            const uint32_t a = base + use + (uint32_t)(t * CL * ROW + (g ^ (PIECE == 16 ? 2 * t : 4 * (t & 1))) * PIECE);
#pragma unroll
            for (int i = 0; i < CL; ++i) read(a + (uint32_t)(i * ROW), x[i].w);
        } else {
#pragma unroll
            for (int i = 0; i < CL; ++i) {
                const int r = t * CL + i;
                const uint32_t m = skew(row0, P, p0, r), a = base + use + (uint32_t)(r * PITCH + g * PIECE) + (m & ~3u);
                uint32_t w[W + 1];
#pragma unroll
                for (int k = 0; k < W + (sizeof(T) == 2 ? 1 : 0); ++k) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[k]) : "r"(a + 4u * k));
#pragma unroll
                for (int k = 0; k < W; ++k) x[i].w[k] = sizeof(T) == 2 ? __funnelshift_r(w[k], w[k + 1], 8 * (m & 3u)) : w[k];
            }
        }
        use = use == (S - 1) * STAGE ? 0 : use + STAGE;
    }
    // 2 NP positions of channels g and g + 8
    __device__ __forceinline__ void take_base(Words<2 * W> (&x)[2])
    {
        const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t a = base + use + (uint32_t)(g * ROW + ((2 * t + e) ^ (g & 1)) * PIECE);
            read(a, x[0].w + e * W);
            read(a + 8 * ROW, x[1].w + e * W);
        }
        use = use == (S - 1) * STAGE ? 0 : use + STAGE;
    }
    // rows that start anywhere: the stage itself
    __device__ __forceinline__ uint32_t take_stage()
    {
        const uint32_t a = base + use;
        use = use == (S - 1) * STAGE ? 0 : use + STAGE;
        return a;
    }
    static __device__ __forceinline__ void drain() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
};

// dst = base + second product, of the blocks kw, kw + ks, ... of 16 channels of an image (base, dst: its first channel; base may be NULL).
// next_base(x): this lane's part of the next block's base from the feed (VEC 0: the stage's address).  VEC: see row_form; with 2 a lane stores its 2 NP
// positions at once.  out: this warp's 16 x (TP + 4) floats, VEC 0 only.
template <typename T, int RB, int VEC, bool SM, int NP, typename Next>
__device__ __forceinline__ void second_product(const Tile<T, RB, NP>& tile, const T* base, T* dst, int M, size_t P, size_t p0, const uint4* w2, int kw, int ks,
                                               float* out, Next next_base)
{
    constexpr int TP = 8 * NP, PARTS = Geo<T>::PARTS;
    constexpr int NO = VEC == 2 ? 2 * NP : NP, PIECES = 2 * NP / NO;    // positions of a load or store
    constexpr bool HALF = sizeof(T) == 2;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int mo_n = (M + 15) / 16;
    const size_t pw = p0 + (size_t)(2 * NP * t);
    // the accumulators as operands: of position b, block jb of ranks
    constexpr int UW = HALF ? 1 : 2;
    uint32_t uh[NP][RB][UW], ul[NP][RB][UW];
#pragma unroll
    for (int b = 0; b < NP; ++b)
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            const float u0 = tile.acc[b >> 1][jb][2 * (b & 1)], u1 = tile.acc[b >> 1][jb][2 * (b & 1) + 1];
            if constexpr (HALF) split_bf16(u0, u1, uh[b][jb][0], ul[b][jb][0]);
            else {
                split_tf32(__float_as_uint(u0), uh[b][jb][0], ul[b][jb][0]);
                split_tf32(__float_as_uint(u1), uh[b][jb][UW - 1], ul[b][jb][UW - 1]);
            }
        }
    constexpr int NS = steps2<T>(RB);
    using Piece = Words<NO * (int)sizeof(T) / 4>;
    for (int mo = kw; mo < mo_n; mo += ks) {
        float d[NP][4];
#pragma unroll
        for (int b = 0; b < NP; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[b][i] = 0.0f;
        const uint4* wm = w2 + (size_t)mo * NS * PARTS * 32;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            if constexpr (HALF) {
                const uint4 w = load_factor<SM>(wm + s * 32);
#pragma unroll
                for (int b = 0; b < NP; ++b) {
                    mma_bf16(d[b], w.x, w.y, w.z, w.w, ul[b][2 * s][0], 2 * s + 1 < RB ? ul[b][(2 * s + 1) % RB][0] : 0u);
                    mma_bf16(d[b], w.x, w.y, w.z, w.w, uh[b][2 * s][0], 2 * s + 1 < RB ? uh[b][(2 * s + 1) % RB][0] : 0u);
                }
            } else {
                const uint4 wh = load_factor<SM>(wm + (s * 2) * 32), wl = load_factor<SM>(wm + (s * 2 + 1) * 32);
#pragma unroll
                for (int b = 0; b < NP; ++b) {
                    mma_tf32(d[b], wl.x, wl.y, wl.z, wl.w, uh[b][s][0], uh[b][s][UW - 1]);
                    mma_tf32(d[b], wh.x, wh.y, wh.z, wh.w, ul[b][s][0], ul[b][s][UW - 1]);
                    mma_tf32(d[b], wh.x, wh.y, wh.z, wh.w, uh[b][s][0], uh[b][s][UW - 1]);
                }
            }
        }
        // channel g + 8 h: accumulators 2 h + e of b are position pw + NP e + b
        if constexpr (VEC == 0) {
            // rows that start anywhere: through shared memory, so that the lanes of a warp write neighbours
            __syncwarp();
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int b = 0; b < NP; b += 2)
                        *reinterpret_cast<float2*>(out + (g + 8 * h) * (TP + 4) + 2 * NP * t + NP * e + b) = make_float2(d[b][2 * h + e], d[b + 1][2 * h + e]);
            __syncwarp();
            const int rows = min(16, M - 16 * mo), here = (int)min((size_t)TP, P - p0);
            using Fd = Feed<T, NP, false>;
            Words<1> none[1];
            const uint32_t stage = base ? next_base(none) : 0u;
            T* row = dst + (size_t)(16 * mo) * P + p0;
#pragma unroll 4
            for (int i = lane; i < rows * TP; i += 32) {
                const int r = i / TP, c = i % TP;
                if (c < here) {
                    float v = out[r * (TP + 4) + c];
                    if (base) {
                        const uint32_t a = stage + (uint32_t)(r * Fd::PITCH + c * (int)sizeof(T)) + Fd::skew(base + (size_t)(16 * mo) * P, P, p0, r);
                        if constexpr (HALF) {
                            uint16_t h;
                            asm volatile("ld.shared.b16 %0, [%1];" : "=h"(h) : "r"(a));
                            v += __uint_as_float((uint32_t)h << 16);
                        } else {
                            uint32_t h;
                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(h) : "r"(a));
                            v += __uint_as_float(h);
                        }
                    }
                    store_one(row + (size_t)r * P + c, v);
                }
            }
        } else {
            Words<NP * (int)sizeof(T) / 2> bs[2]{};
            if (base) next_base(bs);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int o = 16 * mo + g + 8 * h;
                if (o >= M) continue;
                T* row = dst + (size_t)o * P;
#pragma unroll
                for (int e = 0; e < PIECES; ++e) {
                    Piece v;
#pragma unroll
                    for (int i = 0; i < NO * (int)sizeof(T) / 4; ++i) {
                        const uint32_t bw = bs[h].w[e * (NO * (int)sizeof(T) / 4) + i];
                        if constexpr (HALF) {
                            const int at = NO * e + 2 * i;              // of the lane's 2 NP positions
                            v.w[i] = pack_bf16x2(d[at % NP][2 * h + at / NP] + bf16lo(bw), d[at % NP + 1][2 * h + at / NP] + bf16hi(bw));
                        } else {
                            const int at = NO * e + i;
                            v.w[i] = __float_as_uint(d[at % NP][2 * h + at / NP] + __uint_as_float(bw));
                        }
                    }
                    if (pw + NO * e < P) store_words(row + pw + NO * e, v);
                }
            }
        }
    }
}

// dst = base (or 0) at a tile of TP positions: what an image without an adapter gets.  The ks warps of the tile take turns at the rows.
template <typename T, int TP, bool VEC>
__device__ __forceinline__ void copy_tile(const T* base, T* dst, int M, size_t P, size_t p0, int kw, int ks)
{
    constexpr int NP = TP / 8, W = NP * (int)sizeof(T) / 4, BATCH = 8;   // loads before the first store: the two may be the same map
    const int lane = threadIdx.x & 31;
    if constexpr (VEC) {
        const size_t p = p0 + (size_t)NP * (lane & 7);
        if (p >= P) return;
        for (int o0 = 4 * kw + (lane >> 3); o0 < M; o0 += BATCH * 4 * ks) {
            Words<W> v[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) v[i] = base ? load_words<W>(base + min(o0 + 4 * i * ks, M - 1) * P + p) : Words<W>{};
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (o0 + 4 * i * ks < M) store_words(dst + (o0 + 4 * i * ks) * P + p, v[i]);
        }
    } else {
        for (size_t p = p0 + lane; p < min(P, p0 + TP); p += 32)
            for (int o0 = kw; o0 < M; o0 += BATCH * ks) {
                float v[BATCH];
#pragma unroll
                for (int i = 0; i < BATCH; ++i) v[i] = base ? load_one(base + min(o0 + i * ks, M - 1) * P + p) : 0.0f;
#pragma unroll
                for (int i = 0; i < BATCH; ++i)
                    if (o0 + i * ks < M) store_one(dst + (o0 + i * ks) * P + p, v[i]);
            }
    }
}

// This lane's part of a tile as planes of a [ranks][pitch] array, `at` = element (0, NP g): bf16 three parts `next` elements apart, or fp32.
template <typename T, int RB, int NP>
__device__ __forceinline__ void store_planes(const Tile<T, RB, NP>& tile, T* plane, size_t pitch, size_t next)
{
    constexpr int MB = NP / 2;
    const int t = threadIdx.x & 3;
#pragma unroll
    for (int jb = 0; jb < RB; ++jb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            T* q = plane + (8 * jb + 2 * t + e) * pitch;
            if constexpr (sizeof(T) == 2) {
                Words<MB> hi, mid, lo;
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    const float v0 = tile.acc[mb][jb][e], v1 = tile.acc[mb][jb][2 + e];
                    hi.w[mb] = pack_bf16x2(v0, v1);
                    split_bf16(v0 - bf16lo(hi.w[mb]), v1 - bf16hi(hi.w[mb]), mid.w[mb], lo.w[mb]);
                }
                store_words(q, hi);
                store_words(q + next, mid);
                store_words(q + 2 * next, lo);
            } else {
                Words<NP> v;
#pragma unroll
                for (int b = 0; b < NP; ++b) v.w[b] = __float_as_uint(tile.acc[b >> 1][jb][2 * (b & 1) + e]);
                store_words(q, v);
            }
        }
}

template <typename T>
struct ApplyArgs {
    const T* src;                       // [N][K][P]
    Factor<T> f1, f2;                   // f2.p NULL: the first product alone (tap)
    const uint4* w1;                    // laid out in memory, or NULL: each CTA lays them out in shared memory
    const uint4* w2;
    const float* scale;                 // NULL: 1
    const int32_t* ids;
    const T* base;                      // NULL: 0
    T* dst;                             // [N][M][P]
    T* tap;                             // first product with the scale as planes [N][8 RB][Pp], zero behind P; NULL: not kept
    size_t P, Pp;
    int N, K, M, R, r;
    int ks;                             // warps that share a position tile
    int groups, parts, per_part;        // of an image: tiles of a CTA's warps, CTAs, groups of a CTA
    int items;
    int* status;
};

// A CTA takes a run of tiles of one image.  Shared memory: the factors (SM), partial sums of warps that share a tile, tiles on their way out.
template <typename T, int RB, int NP, int VEC, bool SM>
__device__ __forceinline__ void apply_body(const ApplyArgs<T>& q, int item, uint4* sm)
{
    using Ti = Tile<T, RB, NP>;
    constexpr int TP = Ti::TP, MB = Ti::MB;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int n = item / q.parts, per = warps / q.ks;                   // per: position tiles at once
    const int kw = warp % q.ks;
    const int g0 = (item - n * q.parts) * q.per_part, g1 = min(q.groups, g0 + q.per_part);
    const int a = adapter_of(q.ids, n, q.R, q.status);
    const size_t P = q.P;
    const T* base = q.base ? q.base + (size_t)n * q.M * P : nullptr;
    T* dst = q.dst + (size_t)n * q.M * P;

    if (a < 0) {                                                        // (the whole CTA: it has one image)
        if (q.f2.p && q.dst != q.base)
            for (int gr = g0; gr < g1; ++gr) copy_tile<T, TP, (VEC > 0)>(base, dst, q.M, P, (size_t)(gr * per + warp / q.ks) * TP, kw, q.ks);
        return;
    }
    const size_t n1 = first_words<T>(RB, q.K), n2 = q.f2.p ? second_words<T>(RB, q.M) : 0;
    const uint4 *w1 = sm + lane, *w2 = sm + n1 + lane;
    if (SM) {
        lay_first<T>(q.f1, a, q.r, RB, q.K, sm, threadIdx.x, blockDim.x);
        if (n2) lay_second<T>(q.f2, a, q.r, RB, q.M, sm + n1, threadIdx.x, blockDim.x);
        sm += n1 + n2;
        __syncthreads();
    } else {
        w1 = q.w1 + a * n1 + lane;
        w2 = q.w2 + a * n2 + lane;
    }
    float4* red = reinterpret_cast<float4*>(sm);
    char* tail = reinterpret_cast<char*>(sm) + (q.ks > 1 ? (size_t)warps * (MB * RB * 512) : 0);      // tiles on their way out, or in
    float* out = reinterpret_cast<float*>(tail) + warp * 16 * (TP + 4);
    if (VEC == 0) tail += (size_t)warps * 16 * (TP + 4) * 4;
    void* feed_sm = tail + (size_t)warp * Feed<T, NP, (VEC > 0)>::S * Feed<T, NP, (VEC > 0)>::STAGE;
    const float sc = q.scale ? q.scale[a] : 1.0f;
    const T *src = q.src + (size_t)n * q.K * P, *src_end = q.src + (size_t)q.N * q.K * P, *base_end = q.base + (size_t)q.N * q.M * P;
    const size_t limit = q.tap ? q.Pp : P;

    using Fd = Feed<T, NP, (VEC > 0)>;
    constexpr int GC = Geo<T>::GC;
    Fd feed(feed_sm);
    // What the feed copies next: `fleft` channels from `fsrc` on, of the map or (fb) of the base, at the tile of round fr; this warp's groups of the
    // map and then its blocks of the base.
    const int groups = (q.K + GC - 1) / GC;
    const T* const base0 = q.f2.p ? base : nullptr;
    const size_t xstep = (size_t)(q.ks * GC) * P, bstep = (size_t)(q.ks * 16) * P;
    int fr = g0 - 1, fleft = 0;
    bool fb = true, fin = false;
    const T* fsrc = src;
    auto ahead = [&]() {
        while (fleft <= 0 && fr < g1) {
            if (!fb && base0 && fin) { fb = true; fsrc = base0 + (size_t)(kw * 16) * P; fleft = q.M - kw * 16; }
            else {
                const size_t p = (size_t)(++fr * per + warp / q.ks) * TP;
                if (fr == g1) break;
                fin = p < P;
                feed.at(P, p);
                fb = false; fsrc = src + (size_t)(kw * GC) * P; fleft = q.K - kw * GC;
            }
        }
        if (fr < g1) {
            if (fb) { feed.template issue<true>(fsrc, fleft, P, base_end); fsrc += bstep; fleft -= 16 * q.ks; }
            else { feed.template issue<false>(fsrc, fleft, P, src_end); fsrc += xstep; fleft -= GC * q.ks; }
        }
        feed.commit();
    };
    auto next_base = [&](auto& x) -> uint32_t {
        feed.wait();
        ahead();
        if constexpr (VEC > 0) { feed.take_base(x); return 0u; }
        else return feed.take_stage();
    };
    for (int i = 0; i < Fd::S - 1; ++i) ahead();
    for (int gr = g0; gr < g1; ++gr) {
        const size_t p0 = (size_t)(gr * per + warp / q.ks) * TP;
        Ti tile;
        tile.zero();
        for (int grp = kw; grp < groups; grp += q.ks) {
            Words<Fd::W> x[Fd::CL];
            feed.wait();
            ahead();
            feed.take(x, src + (size_t)(grp * GC) * P, P, p0);
            first_step<T, RB, SM, NP>(tile, x, w1 + (size_t)grp * RB * Geo<T>::PARTS * 32);
        }
        if (q.ks > 1) {
            // the warps of a tile add their partial sums, every warp all of them in the same order
            if (gr > g0) __syncthreads();                               // those of the group before have been read
            float4* mine = red + (size_t)warp * (MB * RB * 32) + lane;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int jb = 0; jb < RB; ++jb)
                    mine[(mb * RB + jb) * 32] = make_float4(tile.acc[mb][jb][0], tile.acc[mb][jb][1], tile.acc[mb][jb][2], tile.acc[mb][jb][3]);
            __syncthreads();
            const float4* all = red + (size_t)(warp - kw) * (MB * RB * 32) + lane;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int jb = 0; jb < RB; ++jb) {
                    float4 v = all[(mb * RB + jb) * 32];
                    for (int w = 1; w < q.ks; ++w) {
                        const float4 u = all[(size_t)w * (MB * RB * 32) + (mb * RB + jb) * 32];
                        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                    }
                    tile.acc[mb][jb][0] = v.x; tile.acc[mb][jb][1] = v.y; tile.acc[mb][jb][2] = v.z; tile.acc[mb][jb][3] = v.w;
                }
        }
        if (p0 >= limit) continue;
        tile.scale(sc);
        if (q.tap && kw == 0) {
            const size_t pl = p0 + (size_t)NP * (lane >> 2);
            if (pl + NP > P) tile.keep(pl < P ? (int)(P - pl) : 0);
            store_planes<T, RB, NP>(tile, q.tap + (size_t)n * (8 * RB) * q.Pp + pl, q.Pp, (size_t)q.N * (8 * RB) * q.Pp);
        }
        if (q.f2.p && p0 < P) second_product<T, RB, VEC, SM, NP>(tile, base, dst, q.M, P, p0, w2, kw, q.ks, out, next_base);
    }
    Fd::drain();
}

// Up to two maps in one launch (the backward pass projects dy and x): the second takes the CTAs from q0.items on.
template <typename T, int RB, int NP, int VEC, bool SM>
__global__ void __launch_bounds__(256, RB <= 2 ? 2 : 1) apply_kernel(ApplyArgs<T> q0, ApplyArgs<T> q1)
{
    extern __shared__ uint4 apply_sm[];
    pdl_wait();
    pdl_launch();
    const int item = blockIdx.x;
    if (item < q0.items) apply_body<T, RB, NP, VEC, SM>(q0, item, apply_sm);
    else apply_body<T, RB, NP, VEC, SM>(q1, item - q0.items, apply_sm);
}

// ---- single tokens (one position an image) --------------------------------------------------------
// A CTA takes one image and a stripe of its output channels.  Its warps compute the r products over the input channels (16-byte loads of the
// factor's rows), then every thread an output channel over the ranks.  The factors are the traffic; an adapter that several tokens
// share comes from the L2.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) token_kernel(const T* __restrict__ x, const T* __restrict__ A, const T* __restrict__ B, const float* __restrict__ scale,
                                                    const int32_t* __restrict__ ids, const T* base, T* y, int Cin, int Cout, int R, int r, int per,
                                                    int* status)
{
    __shared__ float u[MAX_RANK];
    constexpr int VE = 16 / (int)sizeof(T);
    const int n = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int a = adapter_of(ids, n, R, status);
    auto val = [](const T* p) { return sizeof(T) == 4 ? *reinterpret_cast<const float*>(p) : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16); };
    if (a >= 0) {
        const T* xr = x + (size_t)n * Cin;
        for (int j = warp; j < r; j += 8) {
            const T* ar = A + ((size_t)a * r + j) * Cin;
            float s = 0.0f;
            if (VEC) {
#pragma unroll 4
                for (int c = lane * VE; c < Cin; c += 32 * VE) {
                    const uint4 xv = *reinterpret_cast<const uint4*>(xr + c), av = __ldg(reinterpret_cast<const uint4*>(ar + c));
                    const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, aw[4] = {av.x, av.y, av.z, av.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (sizeof(T) == 4) s = fmaf(__uint_as_float(xw[i]), __uint_as_float(aw[i]), s);
                        else { s = fmaf(bf16lo(xw[i]), bf16lo(aw[i]), s); s = fmaf(bf16hi(xw[i]), bf16hi(aw[i]), s); }
                    }
                }
            } else {
                for (int c = lane; c < Cin; c += 32) s = fmaf(val(xr + c), val(ar + c), s);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
            if (lane == 0) u[j] = s * (scale ? scale[a] : 1.0f);
        }
    }
    __syncthreads();
    const int o1 = min(Cout, (int)(blockIdx.y + 1) * per);
    for (int o = blockIdx.y * per + threadIdx.x; o < o1; o += 256) {
        const size_t at = (size_t)n * Cout + o;
        float s = 0.0f;
        if (a >= 0) {
            const T* br = B + ((size_t)a * Cout + o) * r;
            if (r % VE == 0) {
                for (int j = 0; j < r; j += VE) {
                    const uint4 bv = __ldg(reinterpret_cast<const uint4*>(br + j));
                    const uint32_t bw[4] = {bv.x, bv.y, bv.z, bv.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        if (sizeof(T) == 4) s = fmaf(__uint_as_float(bw[i]), u[j + i], s);
                        else { s = fmaf(bf16lo(bw[i]), u[j + 2 * i], s); s = fmaf(bf16hi(bw[i]), u[j + 2 * i + 1], s); }
                    }
                }
            } else {
                for (int j = 0; j < r; ++j) s = fmaf(val(br + j), u[j], s);
            }
        }
        if (base) s += val(base + at);
        if (sizeof(T) == 4) reinterpret_cast<float*>(y)[at] = s;
        else reinterpret_cast<uint16_t*>(y)[at] = (uint16_t)pack_bf16x2(s, 0.0f);
    }
}

// ---- gradients of the factors ---------------------------------------------------------------------
// G[c][j] = sum over an adapter's images and positions of map[c][p] plane[j][p]: a matrix product over positions, which both operands have
// contiguous.  The images are taken in the order of their adapters, cut into `ranges` equal runs of tiles; a warp takes one run and 16
// channels, keeps its 16 x 8 RB sums in registers and writes them out where the adapter changes, to slot (run + adapter): runs and adapters
// only ascend, so no slot is written twice, and grad_reduce adds an adapter's slots in ascending order.
// One half tile of G[c][j] += map[c][p] plane[j][p]: 4 NP positions, channels g and g + 8 in x0 and x1, pl at rank g and this lane's positions.
template <typename T>
__device__ __forceinline__ void grad_step(float (&d)[4], const Words<Geo<T>::NP * (int)sizeof(T) / 4>& x0, const Words<Geo<T>::NP * (int)sizeof(T) / 4>& x1,
                                          const T* pl, size_t next)
{
    if constexpr (sizeof(T) == 2) {
        const uint32_t a0[4] = {x0.w[0], x1.w[0], x0.w[1], x1.w[1]}, a1[4] = {x0.w[2], x1.w[2], x0.w[3], x1.w[3]};
#pragma unroll
        for (int part = 2; part >= 0; --part) {
            const uint4 v = *reinterpret_cast<const uint4*>(pl + part * next);
            mma_bf16(d, a0, v.x, v.y);
            mma_bf16(d, a1, v.z, v.w);
        }
    } else {
        const uint4 v = *reinterpret_cast<const uint4*>(pl);
        const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
            for (int i = 0; i < 4; ++i) split_tf32(i & 1 ? x1.w[2 * s + (i >> 1)] : x0.w[2 * s + (i >> 1)], ah[i], al[i]);
            split_tf32(vw[2 * s], bh[0], bl[0]);
            split_tf32(vw[2 * s + 1], bh[1], bl[1]);
            mma_tf32(d, al, bh[0], bh[1]);
            mma_tf32(d, ah, bl[0], bl[1]);
            mma_tf32(d, ah, bh[0], bh[1]);
        }
    }
}

template <typename T>
struct GradArgs {
    const T* map[2];                    // x (with the plane of V) and dy (with that of U)
    const void* plane[2];
    float* part;                        // [slot][Cin + Cout in blocks of 16][8 RB]
    const int32_t* order;
    const int32_t* start;               // [R + 1]
    const int32_t* ids;
    size_t P, Pp;
    int C[2], blocks[2];                // channels, blocks of 16
    int N, R, ranges, tiles;            // tiles of an image
};

template <typename T, int RB, bool VEC>
__global__ void __launch_bounds__(256) grad_kernel(GradArgs<T> q)
{
    constexpr int TP = Geo<T>::TP, NP = Geo<T>::NP;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int all = q.blocks[0] + q.blocks[1];
    const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    pdl_wait();
    pdl_launch();
    const int k = (int)(w / all), blk = (int)(w - (long long)k * all);
    if (k >= q.ranges) return;
    const bool side = blk >= q.blocks[0];
    const int c0 = 16 * (side ? blk - q.blocks[0] : blk), C = side ? q.C[1] : q.C[0];
    const T* map = side ? q.map[1] : q.map[0];
    const T* map_end = map + (size_t)q.N * C * q.P;
    const void* plane = side ? q.plane[1] : q.plane[0];
    const long long total = (long long)q.start[q.R] * q.tiles, share = (total + q.ranges - 1) / q.ranges;
    const long long u0 = k * share, u1 = min(total, u0 + share);
    if (u0 >= u1) return;
    float acc[RB][4];
#pragma unroll
    for (int jb = 0; jb < RB; ++jb)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[jb][i] = 0.0f;

    int img = (int)(u0 / q.tiles), tile = (int)(u0 - (long long)img * q.tiles);
    int n = q.order[img], a = q.ids[n];
    auto flush = [&]() {
        float* o = q.part + ((size_t)(k + a) * all + blk) * (16 * 8 * RB);
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            *reinterpret_cast<float2*>(o + (g)*8 * RB + 8 * jb + 2 * t) = make_float2(acc[jb][0], acc[jb][1]);
            *reinterpret_cast<float2*>(o + (g + 8) * 8 * RB + 8 * jb + 2 * t) = make_float2(acc[jb][2], acc[jb][3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[jb][i] = 0.0f;
        }
    };
    for (long long u = u0; u < u1; ++u) {
        const T* m0 = map + ((size_t)n * C + c0 + g) * q.P;
        const T* m1 = m0 + 8 * q.P;
        const size_t pb = (size_t)tile * TP;
        Words<4> xr[2][2];              // [half of the tile][channel g, g + 8]: this lane's NP positions of it
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const size_t p = pb + h * (TP / 2) + t * NP;
            xr[h][0] = xr[h][1] = Words<4>{};
            if (c0 + g < C) xr[h][0] = load_row<T, NP, VEC>(m0, p, q.P, map_end);
            if (c0 + g + 8 < C) xr[h][1] = load_row<T, NP, VEC>(m1, p, q.P, map_end);
        }
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h)
                grad_step<T>(d, xr[h][0], xr[h][1], static_cast<const T*>(plane) + ((size_t)n * (8 * RB) + 8 * jb + g) * q.Pp + pb + h * (TP / 2) + t * NP,
                             (size_t)q.N * (8 * RB) * q.Pp);
            add(acc[jb], d);
        }
        if (++tile == q.tiles) {
            tile = 0;
            ++img;
            if (u + 1 < u1) {
                n = q.order[img];
                const int b = q.ids[n];
                if (b != a) { flush(); a = b; }
            }
        }
    }
    flush();
}

// dA [R][r][Cin] and dB [R][Cout][r] from the slots; adapters without an image get zeros.
template <int RB>
__global__ void __launch_bounds__(256) grad_reduce(const float* __restrict__ part, const int32_t* __restrict__ start, const float* __restrict__ scale,
                                                   float* __restrict__ dA, float* __restrict__ dB, int Cin, int Cout, int blocks0, int all, int r,
                                                   int R, int ranges, int tiles)
{
    pdl_wait();
    const int a = blockIdx.y;
    const int e = blockIdx.x * 256 + threadIdx.x;                       // (channel in blocks of 16, rank)
    const int j = e % (8 * RB), c = e / (8 * RB);
    if (c >= 16 * all) return;
    const long long total = (long long)start[R] * tiles, share = (total + ranges - 1) / ranges;
    const long long us = (long long)start[a] * tiles, ue = (long long)start[a + 1] * tiles;
    float s = 0.0f;
    if (ue > us) {
        const int k0 = (int)(us / share), k1 = (int)((ue - 1) / share);
        const size_t pitch = (size_t)all * (16 * 8 * RB);
        const float* q = part + (size_t)(k0 + a) * pitch + e;
        for (int k = k0; k <= k1; ++k, q += pitch) s += *q;
    }
    if (j >= r) return;
    if (c < 16 * blocks0) {
        if (c < Cin) dA[((size_t)a * r + j) * Cin + c] = s;
    } else {
        const int o = c - 16 * blocks0;
        if (o < Cout) dB[((size_t)a * Cout + o) * r + j] = scale ? scale[a] * s : s;
    }
}

// Shared memory of a warp for its feed, and for its tiles on their way out where rows start anywhere.
template <typename T> static size_t feed_smem(int np, bool vec)
{
    return (size_t)(vec ? STAGES : 2) * Geo<T>::GC * (8 * np * sizeof(T) + (vec ? 0 : 16)) + (vec ? 0 : (size_t)16 * (8 * np + 4) * 4);
}

// ---- the whole backward pass in one kernel --------------------------------------------------------
// Small ranks and maps with tiles enough.  A CTA takes a run of units of 4 warp tiles, in the order of the images.  For a unit its warps compute
// V and dx and then U of their tiles, leave V and U in shared memory, and then each of them takes blocks of 16 channels of x and dy over
// the unit's positions: G[c][j] += map[c][p] plane[j][p], from rows that were just read and come from the L1 or L2.  So x and dy cross the
// memory bus once.  The sums stay in registers until the image changes; run and image only ascend, so slot (run + image) is written once.
constexpr int BW = 4;                                                   // warps of a CTA
template <typename T>
struct BwdArgs {
    const T *dy, *x, *base;
    T* dx;                              // NULL: not wanted
    Factor<T> fB, fAt, fA;              // dy -> V, V -> dx, x -> U
    const float* scale;
    const int32_t* ids;
    float* part;                        // [slot][block of 16 channels][16][8 RB]
    size_t P;
    int N, Cin, Cout, R, r;
    int units, share;                   // units of an image, of a run
    int* status;
};
template <typename T> __host__ __device__ constexpr int plane_pitch(int np) { return BW * 8 * np + 64 / (int)sizeof(T); }      // 16 banks off per rank
template <typename T>
static size_t bwd_smem(int rb, int Cin, int Cout, bool dx, bool vec)
{
    const int np = lane_positions<T>(rb);
    return 16 * (first_words<T>(rb, Cout) + first_words<T>(rb, Cin) + (dx ? second_words<T>(rb, Cin) : 0)) +
           (size_t)2 * (sizeof(T) == 2 ? 3 : 1) * 8 * rb * plane_pitch<T>(np) * sizeof(T) + BW * feed_smem<T>(np, vec);
}

template <typename T, int RB, int VEC, int NB>
__global__ void __launch_bounds__(32 * BW, NB <= 4 ? 3 : 2) bwd_kernel(BwdArgs<T> q)
{
    constexpr int NP = lane_positions<T>(RB);
    using Ti = Tile<T, RB, NP>;
    constexpr int TP = Ti::TP, PITCH = plane_pitch<T>(NP), PARTS = sizeof(T) == 2 ? 3 : 1, PLANE = 8 * RB * PITCH;
    extern __shared__ uint4 bwd_sm[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const size_t P = q.P, nB = first_words<T>(RB, q.Cout), nA = first_words<T>(RB, q.Cin), nAt = q.dx ? second_words<T>(RB, q.Cin) : 0;
    T* planes = reinterpret_cast<T*>(bwd_sm + nB + nA + nAt);           // [U for dy, V for x][part][rank][position]
    float* out = reinterpret_cast<float*>(planes + 2 * PARTS * PLANE) + warp * 16 * (TP + 4);
    const int blocks0 = (q.Cin + 15) / 16, all = blocks0 + (q.Cout + 15) / 16;
    const T *x_end = q.x + (size_t)q.N * q.Cin * P, *dy_end = q.dy + (size_t)q.N * q.Cout * P,
            *base_end = q.base + (size_t)q.N * q.Cin * P;
    const int run = blockIdx.x;
    const long long total = (long long)q.N * q.units, u0 = (long long)run * q.share, u1 = min(total, u0 + q.share);

    float acc[NB][RB][4];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[i][jb][k] = 0.0f;
    };
    auto flush = [&](int n) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
            if (warp + BW * i < all) {
                float* o = q.part + ((size_t)(run + n) * all + warp + BW * i) * (16 * 8 * RB) + 2 * t;
#pragma unroll
                for (int jb = 0; jb < RB; ++jb) {
                    *reinterpret_cast<float2*>(o + g * 8 * RB + 8 * jb) = make_float2(acc[i][jb][0], acc[i][jb][1]);
                    *reinterpret_cast<float2*>(o + (g + 8) * 8 * RB + 8 * jb) = make_float2(acc[i][jb][2], acc[i][jb][3]);
                }
            }
        clear();
    };
    clear();
    // What the feed copies next: `fleft` channels from `fsrc` on, of dy (phase 0), the base (1) and x (2) of unit fu.  Units of images without an adapter
    // are stepped over.
    using Fd = Feed<T, NP, (VEC > 0)>;
    constexpr int GC = Geo<T>::GC;
    const int gB = (q.Cout + GC - 1) / GC, gA = (q.Cin + GC - 1) / GC;
    Fd feed(reinterpret_cast<char*>(planes + 2 * PARTS * PLANE) + (VEC > 0 ? 0 : (size_t)BW * 16 * (TP + 4) * 4) + (size_t)warp * Fd::S * Fd::STAGE);
    long long fu = u0 - 1;
    int fn = -1, fleft = 0, phase = 2;
    bool feeds = false, fin = false;
    const T* fsrc = q.dy;
    auto ahead = [&]() {
        if (fleft <= 0 && fu < u1) {
            if (phase == 2) {
                for (++fu; fu < u1; ++fu) {
                    const int n = (int)(fu / q.units);
                    if (n != fn) { fn = n; feeds = q.ids[n] >= 0 && q.ids[n] < q.R; }
                    if (feeds) break;
                }
                const size_t p = (size_t)(fu - (long long)fn * q.units) * (BW * TP) + (size_t)warp * TP;
                fin = p < P;
                feed.at(P, p);
                phase = 0; fsrc = q.dy + (size_t)fn * q.Cout * P; fleft = q.Cout;
            } else if (phase == 0 && fin && q.dx && q.base) { phase = 1; fsrc = q.base + (size_t)fn * q.Cin * P; fleft = q.Cin; }
            else { phase = 2; fsrc = q.x + (size_t)fn * q.Cin * P; fleft = q.Cin; }
        }
        if (fu < u1) {
            const int rows = phase == 1 ? 16 : GC;
            if (phase == 1) feed.template issue<true>(fsrc, fleft, P, base_end);
            else feed.template issue<false>(fsrc, fleft, P, phase ? x_end : dy_end);
            fsrc += (size_t)rows * P;
            fleft -= rows;
        }
        feed.commit();
    };
    auto next_base = [&](auto& x) -> uint32_t {
        feed.wait();
        ahead();
        if constexpr (VEC > 0) { feed.take_base(x); return 0u; }
        else return feed.take_stage();
    };
    // the first product of a map at this warp's tile
    auto project = [&](Ti& tile, const T* map, int groups, size_t p0, const uint4* w) {
        tile.zero();
        for (int grp = 0; grp < groups; ++grp) {
            Words<Fd::W> x[Fd::CL];
            feed.wait();
            ahead();
            feed.take(x, map + (size_t)(grp * GC) * P, P, p0);
            first_step<T, RB, true, NP>(tile, x, w + (size_t)grp * RB * Geo<T>::PARTS * 32);
        }
        const size_t pl = p0 + (size_t)NP * g;
        if (pl + NP > P) tile.keep(pl < P ? (int)(P - pl) : 0);
    };
    for (int i = 0; i < Fd::S - 1; ++i) ahead();
    int last = -1, a = -1, laid = -1;                                   // image at work, its adapter, the adapter in shared memory
    float sc = 1.0f;
    for (long long u = u0; u < u1; ++u) {
        const int n = (int)(u / q.units);
        const size_t pu = (size_t)(u - (long long)n * q.units) * (BW * TP), p0 = pu + (size_t)warp * TP;
        if (n != last) {
            if (a >= 0) flush(last);
            last = n;
            a = adapter_of(q.ids, n, q.R, q.status);
            if (a >= 0 && a != laid) {
                __syncthreads();
                lay_first<T>(q.fB, a, q.r, RB, q.Cout, bwd_sm, threadIdx.x, 32 * BW);
                lay_first<T>(q.fA, a, q.r, RB, q.Cin, bwd_sm + nB, threadIdx.x, 32 * BW);
                if (nAt) lay_second<T>(q.fAt, a, q.r, RB, q.Cin, bwd_sm + nB + nA, threadIdx.x, 32 * BW);
                laid = a;
                sc = q.scale ? q.scale[a] : 1.0f;
                __syncthreads();
            }
        }
        const T* base = q.base ? q.base + (size_t)n * q.Cin * P : nullptr;
        T* dx = q.dx + (size_t)n * q.Cin * P;
        if (a < 0) {
            if (q.dx && q.dx != q.base) copy_tile<T, TP, (VEC > 0)>(base, dx, q.Cin, P, p0, 0, 1);
            continue;
        }
        const T *xn = q.x + (size_t)n * q.Cin * P, *dyn = q.dy + (size_t)n * q.Cout * P;
        T* mine = planes + warp * TP + NP * g;
        Ti tile;
        project(tile, dyn, gB, p0, bwd_sm + lane);
        tile.scale(sc);
        store_planes<T, RB, NP>(tile, mine + PARTS * PLANE, PITCH, PLANE);
        if (nAt && p0 < P) second_product<T, RB, VEC, true, NP>(tile, base, dx, q.Cin, P, p0, bwd_sm + nB + nA + lane, 0, 1, out, next_base);
        project(tile, xn, gA, p0, bwd_sm + nB + lane);
        store_planes<T, RB, NP>(tile, mine, PITCH, PLANE);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int blk = warp + BW * i;
            if (blk >= all) continue;
            const bool side = blk >= blocks0;                           // dy
            const int c0 = 16 * (side ? blk - blocks0 : blk), C = side ? q.Cout : q.Cin;
            const T* m0 = (side ? dyn : xn) + (size_t)min(c0 + g, C - 1) * P;     // channels behind the last one: sums that nobody reads
            const T* m1 = (side ? dyn : xn) + (size_t)min(c0 + g + 8, C - 1) * P;
            const T* end = side ? dy_end : x_end;
            const T* plane = planes + (side ? 0 : PARTS * PLANE) + t * NP;
#pragma unroll 2
            for (int w = 0; w < BW; ++w) {
                Words<NP * (int)sizeof(T) / 4> xw[2][2];                // [half of the tile][channel g, g + 8]
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const size_t p = pu + w * TP + h * (TP / 2) + t * NP;
                    xw[h][0] = load_row<T, NP, (VEC > 0)>(m0, p, P, end);
                    xw[h][1] = load_row<T, NP, (VEC > 0)>(m1, p, P, end);
                }
#pragma unroll
                for (int jb = 0; jb < RB; ++jb) {
                    float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const T* pl = plane + (8 * jb + g) * PITCH + w * TP + h * (TP / 2);
                        grad_step<T>(d, xw[h][0], xw[h][1], pl, PLANE);
                    }
                    add(acc[i][jb], d);
                }
            }
        }
        __syncthreads();                                                // the planes are written again
    }
    if (a >= 0) flush(last);
    Fd::drain();
    pdl_launch();
}

// dA and dB from the slots of bwd_kernel: 32 elements (channel in blocks of 16, rank) a CTA, eight threads an element, added in a fixed order.
template <int RB>
__global__ void __launch_bounds__(256) bwd_reduce(const float* __restrict__ part, const int32_t* __restrict__ ids, const float* __restrict__ scale,
                                                  float* __restrict__ dA, float* __restrict__ dB, int N, int Cin, int Cout, int blocks0, int all, int r,
                                                  int units, int share)
{
    __shared__ float sm[8][33];
    pdl_wait();
    const int a = blockIdx.y, e = blockIdx.x * 32 + threadIdx.x;        // (all * 16 * 8 RB is a multiple of 32)
    const size_t pitch = (size_t)all * (16 * 8 * RB);
    float s = 0.0f;
    int count = 0;                                                      // slots of the adapter so far
    for (int n = 0; n < N; ++n) {
        if (ids[n] != a) continue;
        const int k0 = (int)((long long)n * units / share), k1 = (int)(((long long)(n + 1) * units - 1) / share);
        const int skip = (int)((threadIdx.y - (unsigned)count) & 7u);
#pragma unroll 4
        for (int k = k0 + skip; k <= k1; k += 8) s += part[(size_t)(k + n) * pitch + e];
        count += k1 - k0 + 1;
    }
    sm[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) s += sm[i][threadIdx.x];
    const int j = e % (8 * RB), c = e / (8 * RB);
    if (j >= r) return;
    if (c < 16 * blocks0) {
        if (c < Cin) dA[((size_t)a * r + j) * Cin + c] = s;
    } else {
        const int o = c - 16 * blocks0;
        if (o < Cout) dB[((size_t)a * Cout + o) * r + j] = scale ? scale[a] * s : s;
    }
}

// ---- plans and launches -----------------------------------------------------------------------------
inline int blocks_of(int rank) { return rank <= 8 ? 1 : rank <= 16 ? 2 : rank <= 32 ? 4 : 8; }

// The one-kernel backward pass: its sums are 4 NB RB registers a thread, its unit is 4 tiles.
template <typename T>
struct Fused {
    bool ok;
    int nb, units, share, runs;
};
template <typename T>
static Fused<T> fused_of(int N, int Cin, int Cout, size_t P, int rank)
{
    Fused<T> f{};
    const int rb = blocks_of(rank), all = ceil_div(Cin, 16) + ceil_div(Cout, 16), unit = BW * Geo<T>::TP;
    f.nb = all <= 2 * BW ? 2 : all <= 4 * BW ? 4 : 8;
    f.units = (int)((P + unit - 1) / unit);
    const long long total = (long long)N * f.units;
    if (rb > 2 || all > 8 * BW || N > 4096 || total < 2 * B200_SMS) return f;
    const size_t smem = bwd_smem<T>(rb, Cin, Cout, true, P % Geo<T>::NP == 0);
    if (smem > 113 * 1024) return f;                                      // two CTAs an SM
    f.runs = (int)std::min(total, (long long)WAVES * B200_SMS * std::min<int>(3, (int)(228 * 1024 / (smem + 1024))));
    // two units at least: factors laid out and a feed filled for a single one are not paid for.  512 units in runs of 1 / 2, 144 -> 24 on 4 x 128 x 256
    // with adapters 0 1 2 3: 64 / 62, 0 - 2 3: 63 / 60; but - - 1 2: 46 / 58, where half of the runs have nothing to do.
    f.share = (int)std::max(2LL, (total + f.runs - 1) / f.runs);
    f.runs = (int)((total + f.share - 1) / f.share);
    f.ok = true;
    return f;
}

// Factors that a CTA lays out for itself: while four CTAs of an SM have the room.
template <typename T> static bool staged(int rb, int K, int M) { return 16 * (first_words<T>(rb, K) + (M ? second_words<T>(rb, M) : 0)) <= 40 * 1024; }
struct Ws {
    void* first[2];
    void* second;
    void* tap[2];
    int32_t* order;
    int32_t* start;
    float* part;
    size_t Pp;
    int ranges;
    size_t total;
};

template <typename T>
static Ws carve(void* ws, int N, int Cin, int Cout, size_t P, int R, int rank, bool bwd)
{
    Ws w{};
    const int rb = blocks_of(rank), TP = Geo<T>::TP, all = ceil_div(Cin, 16) + ceil_div(Cout, 16);
    size_t off = 0;
    char* b = static_cast<char*>(ws);
    auto take = [&](size_t bytes) { char* p = b ? b + off : nullptr; off += align_up(bytes, 256); return p; };
    if (!bwd) {
        if (P > 1 && !staged<T>(rb, Cin, Cout)) {
            w.first[0] = take((size_t)R * first_words<T>(rb, Cin) * 16);
            w.second = take((size_t)R * second_words<T>(rb, Cout) * 16);
        }
        w.total = off;
        return w;
    }
    // dy -> V -> dx alone, x -> U, and what the sums of the gradients need
    w.first[0] = take((size_t)R * first_words<T>(rb, Cout) * 16);
    w.second = take((size_t)R * second_words<T>(rb, Cin) * 16);
    w.first[1] = take((size_t)R * first_words<T>(rb, Cin) * 16);
    const Fused<T> f = fused_of<T>(N, Cin, Cout, P, rank);
    if (f.ok) {
        w.part = reinterpret_cast<float*>(take((size_t)(f.runs + N) * all * 16 * 8 * rb * 4));
        w.total = off;
        return w;
    }
    w.Pp = (P + TP - 1) / TP * TP;
    for (int i = 0; i < 2; ++i) w.tap[i] = take((size_t)N * 8 * rb * w.Pp * (sizeof(T) == 2 ? 6 : 4));
    w.order = reinterpret_cast<int32_t*>(take((size_t)N * 4));
    w.start = reinterpret_cast<int32_t*>(take((size_t)(R + 1) * 4));
    const long long units = (long long)N * (w.Pp / TP);
    const long long want = (16LL * B200_SMS + all - 1) / all;
    w.ranges = (int)std::max(1LL, std::min(want, units));
    w.part = reinterpret_cast<float*>(take((size_t)(w.ranges + R) * all * 16 * 8 * rb * 4));
    w.total = off;
    return w;
}

// How rows start: 2 on 2 NP positions, which are stored at once, 1 on NP, 0 anywhere.  With all of a lane's positions the former are 32 bytes in one
// store, and such a store needs an address on 32 bytes, where every map is only promised to start on 16: the output's own address decides too.
template <typename T>
static int row_form(size_t P, const void* dst, int np)
{
    if (P % (2 * np) == 0 && reinterpret_cast<uintptr_t>(dst) % (2 * np * sizeof(T)) == 0) return 2;
    return P % np == 0 ? 1 : 0;
}
// Warps that share a tile: more only while the tiles alone do not fill the GPU.
template <typename T>
static void plan_apply(ApplyArgs<T>& q, int np, int most_ks, int& warps)
{
    const int tp = 8 * np;
    const long long tiles = (long long)(((q.tap ? q.Pp : q.P) + tp - 1) / tp);
    const int most = std::max(ceil_div(q.K, Geo<T>::GC), q.f2.p ? ceil_div(q.M, 16) : 1);
    q.ks = 1;
    while (q.ks < most_ks && q.ks * 2 <= most && (long long)q.N * tiles * q.ks < FILL * B200_SMS) q.ks *= 2;
    if (!warps) warps = q.ks == 8 ? 8 : 4;
    if (q.ks == 8) warps = 8;
}
template <typename T>
static void plan_parts(ApplyArgs<T>& q, int np, int warps, bool sm)
{
    const int tp = 8 * np, per = warps / q.ks;
    const long long tiles = (long long)(((q.tap ? q.Pp : q.P) + tp - 1) / tp);
    q.groups = (int)((tiles + per - 1) / per);
    // a CTA that lays out its factors takes as many groups as leave four CTAs an SM (eight warps: two)
    const int ctas = WAVES * B200_SMS * (warps == 8 ? 2 : 4);
    q.per_part = sm ? (int)std::max(1LL, std::min((long long)q.groups, (long long)q.N * q.groups / ctas)) : 1;
    q.parts = ceil_div(q.groups, q.per_part);
}
// Factors, partial sums of warps that share a tile, and the tiles on their way out where rows start anywhere.
template <typename T> static size_t apply_smem(const ApplyArgs<T>& q, int warps, int rb, int np, bool vec, bool sm)
{
    return (sm ? 16 * (first_words<T>(rb, q.K) + (q.f2.p ? second_words<T>(rb, q.M) : 0)) : 0) +
           (size_t)warps * ((q.ks > 1 ? (np / 2) * rb * 512 : 0) + feed_smem<T>(np, vec));
}

template <typename T, int RB, int NP, int VEC, bool SM>
static wcc_status run_apply(ApplyArgs<T> q0, ApplyArgs<T>* q1, int dev, bool overlap, cudaStream_t st)
{
    size_t smem = 0;
    int warps = 0;
    long long items1 = 0;
    for (int most_ks = 8; most_ks >= 4; most_ks /= 2) {                 // eight warps if their shared memory is there
        warps = 0;
        plan_apply(q0, NP, most_ks, warps);
        if (q1) plan_apply(*q1, NP, most_ks, warps);
        plan_parts(q0, NP, warps, SM);
        smem = apply_smem(q0, warps, RB, NP, VEC > 0, SM);
        if (q1) {
            plan_parts(*q1, NP, warps, SM);
            smem = std::max(smem, apply_smem(*q1, warps, RB, NP, VEC > 0, SM));
            items1 = (long long)q1->N * q1->parts;
        }
        if (smem <= 227 * 1024) break;
    }
    const long long items = (long long)q0.N * q0.parts;
    if (items + items1 > 0x7FFFFFFFLL) return WCC_ERR_SHAPE;
    q0.items = (int)items;
    if (q1) q1->items = (int)items1;
    wcc_status s = allow_smem<apply_kernel<T, RB, NP, VEC, SM>>(dev, (int)smem);
    if (s != WCC_OK) return s;
    return launch_overlapped(apply_kernel<T, RB, NP, VEC, SM>, dim3((unsigned)(items + items1)), dim3((unsigned)(32 * warps)), smem, st, overlap, 1, q0,
                             q1 ? *q1 : q0);
}
// overlap: the kernel before it in the stream is the preparation.
template <typename T>
static wcc_status launch_apply(const ApplyArgs<T>& q0, ApplyArgs<T>* q1, int rb, int dev, bool overlap, cudaStream_t st)
{
    constexpr int FULL_NP = Geo<T>::NP;
    const bool sm = !q0.w1;
    const int np = lane_positions<T>(rb), vec = row_form<T>(q0.P, q0.dst, np);
#define WCC_AD_APPLY(RB_, NP_, SM_)                                                                                                      \
    if (rb == (RB_) && np == (NP_) && sm == (SM_))                                                                                       \
        return vec == 2 ? run_apply<T, RB_, NP_, 2, SM_>(q0, q1, dev, overlap, st)                                                        \
                        : vec == 1 ? run_apply<T, RB_, NP_, 1, SM_>(q0, q1, dev, overlap, st) : run_apply<T, RB_, NP_, 0, SM_>(q0, q1, dev, overlap, st);
    WCC_AD_APPLY(1, FULL_NP, true) WCC_AD_APPLY(2, FULL_NP, true) WCC_AD_APPLY(4, FULL_NP, true) WCC_AD_APPLY(8, FULL_NP / 2, true)
    WCC_AD_APPLY(1, FULL_NP, false) WCC_AD_APPLY(2, FULL_NP, false) WCC_AD_APPLY(4, FULL_NP, false) WCC_AD_APPLY(8, FULL_NP / 2, false)
#undef WCC_AD_APPLY
    return WCC_ERR_SHAPE;
}

template <typename T>
static wcc_status launch_prep(const PrepArgs<T>& q, cudaStream_t st)
{
    const size_t words = std::max({q.first[0].p ? first_words<T>(q.rb, q.K[0]) : 1, q.first[1].p ? first_words<T>(q.rb, q.K[1]) : 1,
                                   q.second.p ? second_words<T>(q.rb, q.M) : 1});
    const int stripes = (int)std::min<size_t>(64, (words + 255) / 256);
    return launch_overlapped(prep_kernel<T>, dim3((unsigned)q.R, (unsigned)stripes), dim3(256), 0, st, false, 1, q);
}

template <typename T>
static wcc_status forward(const void* x, const void* A, const void* B, const float* scale, const int32_t* ids, const void* base, int N, int Cin, int Cout,
                          size_t P, int R, int rank, void* y, void* ws, cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    if (P == 1) {
        const int want = ceil_div(B200_SMS, N), per = std::max(256, ceil_div(ceil_div(Cout, want), 256) * 256);
        const bool vec = Cin % (16 / (int)sizeof(T)) == 0;
        return launch_overlapped(vec ? token_kernel<T, true> : token_kernel<T, false>, dim3((unsigned)N, (unsigned)ceil_div(Cout, per)), dim3(256), 0, st,
                                 false, 1, static_cast<const T*>(x), static_cast<const T*>(A), static_cast<const T*>(B), scale, ids,
                                 static_cast<const T*>(base), static_cast<T*>(y), Cin, Cout, R, rank, per, di.status);
    }
    const Ws w = carve<T>(ws, N, Cin, Cout, P, R, rank, false);
    const int rb = blocks_of(rank);
    ApplyArgs<T> q{};
    q.f1 = Factor<T>{static_cast<const T*>(A), (long long)rank * Cin, Cin, 1};
    q.f2 = Factor<T>{static_cast<const T*>(B), (long long)Cout * rank, 1, rank};
    if (w.first[0]) {
        PrepArgs<T> p{};
        p.first[0] = q.f1; p.second = q.f2;
        p.first_out[0] = static_cast<uint4*>(w.first[0]); p.second_out = static_cast<uint4*>(w.second);
        p.K[0] = Cin; p.M = Cout; p.R = R; p.r = rank; p.rb = rb; p.N = N; p.ids = ids;
        if ((s = launch_prep(p, st)) != WCC_OK) return s;
        q.w1 = p.first_out[0]; q.w2 = p.second_out;
    }
    q.src = static_cast<const T*>(x); q.scale = scale; q.ids = ids; q.base = static_cast<const T*>(base); q.dst = static_cast<T*>(y);
    q.P = P; q.N = N; q.K = Cin; q.M = Cout; q.R = R; q.r = rank; q.status = di.status;
    return launch_apply<T>(q, nullptr, rb, di.dev, q.w1 != nullptr, st);
}

template <typename T>
static wcc_status backward(const void* dy, const void* x, const void* A, const void* B, const float* scale, const int32_t* ids, const void* base, int N,
                           int Cin, int Cout, size_t P, int R, int rank, void* dx, float* dA, float* dB, void* ws, cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    const Ws w = carve<T>(ws, N, Cin, Cout, P, R, rank, true);
    const int rb = blocks_of(rank), all = ceil_div(Cin, 16) + ceil_div(Cout, 16);
    const bool vec = P % Geo<T>::NP == 0, params = dA != nullptr;
    const Factor<T> fB{static_cast<const T*>(B), (long long)Cout * rank, 1, rank}, fAt{static_cast<const T*>(A), (long long)rank * Cin, Cin, 1}, fA = fAt;
    const Fused<T> f = fused_of<T>(N, Cin, Cout, P, rank);
    if (params && f.ok) {
        BwdArgs<T> q{};
        q.dy = static_cast<const T*>(dy); q.x = static_cast<const T*>(x); q.base = static_cast<const T*>(base); q.dx = static_cast<T*>(dx);
        q.fB = fB; q.fAt = fAt; q.fA = fA; q.scale = scale; q.ids = ids; q.part = w.part; q.P = P; q.N = N; q.Cin = Cin; q.Cout = Cout; q.R = R;
        q.r = rank; q.units = f.units; q.share = f.share; q.status = di.status;
        const int v = row_form<T>(P, dx, lane_positions<T>(rb));
        const size_t smem = bwd_smem<T>(rb, Cin, Cout, dx != nullptr, v > 0);
        const dim3 rgrid((unsigned)(all * 4 * rb), (unsigned)R);
#define WCC_AD_BWD(RB_, VEC_, NB_)                                                                                                                \
    if (rb == (RB_) && v == (VEC_) && f.nb == (NB_)) {                                                                                            \
        if ((s = allow_smem<bwd_kernel<T, RB_, VEC_, NB_>>(di.dev, (int)smem)) != WCC_OK) return s;                                               \
        s = launch_overlapped(bwd_kernel<T, RB_, VEC_, NB_>, dim3((unsigned)f.runs), dim3(32 * BW), smem, st, false, 1, q);                       \
        if (s != WCC_OK) return s;                                                                                                                \
        return launch_overlapped(bwd_reduce<RB_>, rgrid, dim3(32, 8), 0, st, true, 1, w.part, ids, scale, dA, dB, N, Cin, Cout, ceil_div(Cin, 16), \
                                 all, rank, f.units, f.share);                                                                                    \
    }
#define WCC_AD_BWDS(RB_, VEC_) WCC_AD_BWD(RB_, VEC_, 2) WCC_AD_BWD(RB_, VEC_, 4) WCC_AD_BWD(RB_, VEC_, 8)
        WCC_AD_BWDS(1, 0) WCC_AD_BWDS(1, 1) WCC_AD_BWDS(1, 2) WCC_AD_BWDS(2, 0) WCC_AD_BWDS(2, 1) WCC_AD_BWDS(2, 2)
#undef WCC_AD_BWDS
#undef WCC_AD_BWD
        return WCC_ERR_SHAPE;
    }
    const bool sm = staged<T>(rb, Cout, dx ? Cin : 0) && (!params || staged<T>(rb, Cin, 0));
    ApplyArgs<T> q{}, u{};
    q.f1 = fB;
    if (dx) q.f2 = fAt;
    if (!sm || params) {
        PrepArgs<T> p{};
        if (!sm) {
            p.first[0] = fB;
            if (dx) p.second = fAt;
            if (params) p.first[1] = fA;
            p.first_out[0] = static_cast<uint4*>(w.first[0]); p.first_out[1] = static_cast<uint4*>(w.first[1]); p.second_out = static_cast<uint4*>(w.second);
            q.w1 = p.first_out[0]; q.w2 = p.second_out;
        }
        p.K[0] = Cout; p.K[1] = Cin; p.M = Cin; p.R = R; p.r = rank; p.rb = rb; p.N = N; p.ids = ids;
        if (params) { p.order = w.order; p.start = w.start; }
        if ((s = launch_prep(p, st)) != WCC_OK) return s;
    }
    q.src = static_cast<const T*>(dy); q.scale = scale; q.ids = ids; q.base = static_cast<const T*>(base); q.dst = static_cast<T*>(dx);
    q.tap = params ? static_cast<T*>(w.tap[0]) : nullptr;
    q.P = P; q.Pp = w.Pp; q.N = N; q.K = Cout; q.M = Cin; q.R = R; q.r = rank; q.status = di.status;
    u = q;
    u.src = static_cast<const T*>(x); u.f1 = fA; u.f2 = Factor<T>{}; u.scale = nullptr; u.base = nullptr; u.dst = nullptr;
    u.tap = static_cast<T*>(w.tap[1]); u.K = Cin; u.M = 0;
    if (!sm) u.w1 = static_cast<uint4*>(w.first[1]);
    if ((s = launch_apply<T>(q, params ? &u : nullptr, rb, di.dev, !sm || params, st)) != WCC_OK || !params) return s;
    GradArgs<T> h{};
    h.map[0] = static_cast<const T*>(x); h.map[1] = static_cast<const T*>(dy); h.plane[0] = w.tap[0]; h.plane[1] = w.tap[1];
    h.part = w.part; h.order = w.order; h.start = w.start; h.ids = ids; h.P = P; h.Pp = w.Pp;
    h.C[0] = Cin; h.C[1] = Cout; h.blocks[0] = ceil_div(Cin, 16); h.blocks[1] = ceil_div(Cout, 16);
    h.N = N; h.R = R; h.ranges = w.ranges; h.tiles = (int)(w.Pp / Geo<T>::TP);
    const dim3 grid((unsigned)(((long long)w.ranges * all + 7) / 8)), rgrid((unsigned)ceil_div(16 * all * 8 * rb, 256), (unsigned)R);
#define WCC_AD_GRAD(RB_)                                                                                                                          \
    if (rb == (RB_)) {                                                                                                                            \
        s = launch_overlapped(vec ? grad_kernel<T, RB_, true> : grad_kernel<T, RB_, false>, grid, dim3(256), 0, st, true, 1, h);                   \
        if (s != WCC_OK) return s;                                                                                                                \
        return launch_overlapped(grad_reduce<RB_>, rgrid, dim3(256), 0, st, true, 1, w.part, w.start, scale, dA, dB, Cin, Cout, h.blocks[0], all,  \
                                 rank, R, w.ranges, h.tiles);                                                                                     \
    }
    WCC_AD_GRAD(1) WCC_AD_GRAD(2) WCC_AD_GRAD(4) WCC_AD_GRAD(8)
#undef WCC_AD_GRAD
    return WCC_ERR_SHAPE;
}

// What wcc_debug_adapters_path answers.
template <typename T>
static int path_of(int N, int Cin, int Cout, size_t P, int rank, const void* dst, bool bwd)
{
    if (!bwd && P == 1) return WCC_PATH_ADAPTERS_TOKEN;
    const int rb = blocks_of(rank), form = WCC_PATH_FORM * row_form<T>(P, dst, lane_positions<T>(rb));
    const Fused<T> f = fused_of<T>(N, Cin, Cout, P, rank);
    if (bwd && f.ok) return WCC_PATH_ADAPTERS_ONE_KERNEL + form + WCC_PATH_BLOCKS * f.nb;
    const bool sm = bwd ? staged<T>(rb, Cout, Cin) && staged<T>(rb, Cin, 0) : staged<T>(rb, Cin, Cout);
    return (sm ? WCC_PATH_ADAPTERS_MAP : WCC_PATH_ADAPTERS_MAP_PREPARED) + form;
}

}  // namespace ad

static wcc_status check_adapter_args(int N, int Cin, int Cout, int H, int W, int R, int rank, wcc_dtype dt)
{
    if (N <= 0 || Cin <= 0 || Cout <= 0 || H <= 0 || W <= 0 || Cin > WCC_MAX_CHANNELS || Cout > WCC_MAX_CHANNELS) return WCC_ERR_SHAPE;
    if (R <= 0 || R > 65535 || rank <= 0 || rank > ad::MAX_RANK) return WCC_ERR_SHAPE;
    if ((long long)H * W > (1LL << 30) || (long long)N * H * W > (1LL << 30)) return WCC_ERR_SHAPE;
    if (dt != WCC_F32 && dt != WCC_BF16) return WCC_ERR_DTYPE;
    return WCC_OK;
}

}  // namespace wcc
