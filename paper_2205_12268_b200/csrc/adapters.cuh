// Low-rank adapters of many requests beside a shared projection.  Image n of the batch has adapter a = ids[n] (or none) with factors
// A_a [r][Cin], B_a [Cout][r] and a scale t_a:
//     forward    U = A_a x_n,        y_n  = base_n + t_a B_a U
//     backward   V = t_a B_a^T dy_n, dx_n = base_n + A_a^T V,   dA_a = sum_n V x_n^T,   dB_a = t_a sum_n dy_n U^T
// The rank is at most 64 and the maps are long, so both products together do about r / 2 operations a byte: the maps are the bound, not the
// tensor pipes, and everything is arranged around reading and writing them once in whole lines.  A warp keeps the product of the first
// factor in registers as the operand of the second: nothing of rank r goes to memory in the forward pass.
//
// The products are warp-level matrix instructions on registers.  Their rows, columns and summation index can be any permutation of
// positions, ranks and channels that both operands agree on, and that freedom replaces every shuffle and transposition through shared memory:
//  - first product, D[position][rank]: lane (g, t) = (lane / 4, lane % 4) loads 16 bytes of a channel, NP positions from p0 + NP g on; its b-th
//    position is row g of row block b / 2 (upper half for odd b), its channels of a group are the CL from CL t on;
//  - second product, D[channel][position]: the accumulators of position b are its operand as they stand, one instruction column block per b,
//    and lane t ends up with 2 NP positions in a row of memory, 32 bytes, of the two channels g and g + 8.
// bf16 maps: the factors are bf16, U is split into two bf16 parts (relative error 2^-17), sums are fp32.  fp32 maps: every operand is split into
// two parts of 11 bits, three products of them are summed in fp32 (relative error about 2^-21 a term, beside 2^-24 of each fp32 addition).
#pragma once

#include <algorithm>

#include "common.cuh"

namespace wcc {
namespace ad {

constexpr unsigned FULL = 0xFFFFFFFFu;
constexpr int MAX_RANK = 64;
#ifndef AD_HALF
#define AD_HALF 8
#define AD_FILL 12LL
#endif

template <typename T> struct Geo;
template <> struct Geo<__nv_bfloat16> { static constexpr int NP = 8, TP = 64, CL = 8, GC = 32, PARTS = 1; };
template <> struct Geo<float> { static constexpr int NP = 4, TP = 32, CL = 4, GC = 16, PARTS = 2; };
// NP positions of a lane (16 bytes) and TP of a warp's tile in the widest form, CL channels of a lane in a group of GC, PARTS parts of a factor's
// element.  For the largest ranks a lane takes half as many positions, which halves the sums it has to hold.
template <typename T> __host__ __device__ constexpr int lane_positions(int rb) { return rb >= AD_HALF ? Geo<T>::NP / 2 : Geo<T>::NP; }

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
// there on): single loads of 2 bytes cost eight times the instructions, a layer's odd map 76 us instead of the figure below.
template <int WORDS> struct Words { uint32_t w[WORDS]; };
template <int W> __device__ __forceinline__ Words<W> load_words(const void* p)
{
    Words<W> r;
    if constexpr (W == 8) {
        // volatile, so that it stays ahead of the products it is issued before
        asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
            : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7])
            : "l"(p));
    } else if constexpr (W == 4) {
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

// First product: [adapter][group of GC channels][block of 8 ranks][part][lane] 16 bytes (CL channels of rank g).
// Second product: [adapter][block of 16 channels][step][part][lane] 16 bytes.
template <typename T> __host__ __device__ inline size_t first_words(int rb, int K) { return (size_t)((K + Geo<T>::GC - 1) / Geo<T>::GC) * rb * Geo<T>::PARTS * 32; }
template <typename T> __host__ __device__ inline size_t second_words(int rb, int M) { return (size_t)((M + 15) / 16) * steps2<T>(rb) * Geo<T>::PARTS * 32; }

template <typename T>
__device__ __forceinline__ uint32_t element(const Factor<T>& f, int a, int j, int c, int r, int C)
{
    if (j >= r || c >= C) return 0u;
    const T* q = f.p + a * f.sa + (long long)j * f.sj + (long long)c * f.sc;
    return sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(q) : *reinterpret_cast<const uint32_t*>(q);
}

template <typename T>
struct PrepArgs {
    Factor<T> first[2], second[2];      // of up to two products of each kind (p NULL: none)
    uint4* first_out[2];
    uint4* second_out[2];
    int K[2], M[2];
    int R, r, rb, N;
    const int32_t* ids;
    int32_t* order;                     // backward: images with an adapter by adapter, and per adapter the first of them [R + 1]
    int32_t* start;
};

// The ids of a call as the kernels take them: anything but 0 .. R - 1 is no adapter, and one at R or beyond is an error.
__device__ __forceinline__ int adapter_of(const int32_t* ids, int n, int R, int* status)
{
    const int a = ids[n];
    if (a < R) return a < 0 ? -1 : a;
    if (status) atomicExch(status, (int)WCC_ERR_INDEX);
    return -1;
}

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
    constexpr int GC = Geo<T>::GC, CL = Geo<T>::CL, PARTS = Geo<T>::PARTS;
    for (int side = 0; side < 2; ++side) {
        if (q.first[side].p) {
            const size_t words = first_words<T>(q.rb, q.K[side]);
            uint4* out = q.first_out[side] + a * words;
            for (size_t i = (size_t)blockIdx.y * 256 + threadIdx.x; i < words / PARTS; i += (size_t)gridDim.y * 256) {
                const int lane = (int)(i & 31), jb = (int)((i >> 5) % q.rb), grp = (int)((i >> 5) / q.rb);
                const int j = 8 * jb + (lane >> 2), c = grp * GC + (lane & 3) * CL;
                uint32_t e[CL], w[4], lo[4];
#pragma unroll
                for (int k = 0; k < CL; ++k) e[k] = element(q.first[side], a, j, c + k, q.r, q.K[side]);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (sizeof(T) == 2) w[k] = e[(2 * k) % CL] | (e[(2 * k + 1) % CL] << 16);
                    else split_tf32(e[k], w[k], lo[k]);
                }
                uint4* o = out + (i >> 5) * (PARTS * 32) + lane;
                o[0] = make_uint4(w[0], w[1], w[2], w[3]);
                if (PARTS == 2) o[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
        if (q.second[side].p) {
            const int ns = steps2<T>(q.rb);
            const size_t words = second_words<T>(q.rb, q.M[side]);
            uint4* out = q.second_out[side] + a * words;
            for (size_t i = (size_t)blockIdx.y * 256 + threadIdx.x; i < words / PARTS; i += (size_t)gridDim.y * 256) {
                const int lane = (int)(i & 31), ks = (int)((i >> 5) % ns), mo = (int)((i >> 5) / ns), g = lane >> 2, t = lane & 3;
                const int o0 = 16 * mo + g, M = q.M[side];
                const Factor<T>& f = q.second[side];
                uint32_t w[4], lo[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {           // registers: channel o0, o0 + 8, then the other half of the step's ranks
                    const int o = o0 + 8 * (k & 1);
                    if (sizeof(T) == 2) {
                        const int j = 16 * ks + 8 * (k >> 1) + 2 * t;
                        w[k] = element(f, a, j, o, q.r, M) | (element(f, a, j + 1, o, q.r, M) << 16);
                    } else {
                        split_tf32(element(f, a, 8 * ks + 2 * t + (k >> 1), o, q.r, M), w[k], lo[k]);
                    }
                }
                uint4* op = out + (i >> 5) * (PARTS * 32) + lane;
                op[0] = make_uint4(w[0], w[1], w[2], w[3]);
                if (PARTS == 2) op[32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        }
    }
}

// ---- both products over a tile of positions -----------------------------------------------------
template <typename T>
struct ApplyArgs {
    const T* src;                       // [N][K][P]
    const uint4* w1;
    const uint4* w2;                    // NULL: the first product alone (tap)
    const float* scale;                 // NULL: 1
    const int32_t* ids;
    const T* base;                      // NULL: 0
    T* dst;                             // [N][M][P]
    void* tap;                          // first product with the scale: three bf16 parts, or fp32, [N][8 RB][Pp] each; NULL: not kept
    size_t P, Pp;
    int N, K, M, R;
    int tiles;                          // groups of CTA tiles of an image
    int ks;                             // warps that share a position tile
    int items;
    int* status;
};

// VEC: 0 single loads, 1 rows start on the NP positions of a lane's first product, 2 also on the 2 NP of the second.
template <typename T, int RB, int VEC>
__device__ __forceinline__ void apply_body(const ApplyArgs<T>& q, int item, float4* sm)
{
    constexpr int NP = lane_positions<T>(RB), TP = 8 * NP, CL = Geo<T>::CL, GC = Geo<T>::GC, PARTS = Geo<T>::PARTS, MB = NP / 2;
    constexpr int NO = VEC == 2 ? 2 * NP : NP, PIECES = 2 * NP / NO;    // positions of a load or store of the second product
    constexpr bool HALF = sizeof(T) == 2;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int n = item / q.tiles;
    const int per = (int)(blockDim.x >> 5) / q.ks;                    // position tiles of the CTA
    const int kw = warp % q.ks, tile = (item - n * q.tiles) * per + warp / q.ks;
    const size_t p0 = (size_t)tile * TP;
    const int a = adapter_of(q.ids, n, q.R, q.status);
    const size_t P = q.P;
    const int mo_n = (q.M + 15) / 16;
    const size_t pw = p0 + (size_t)(2 * NP * t);

    if (a < 0) {                                                        // (the whole CTA: it has one image)
        if (!q.w2 || q.dst == q.base || p0 >= P) return;
        // the warps of the tile copy its rows, eight pieces of 16 or 8 bytes (or 32 single elements) a row
        const T* from = q.base + (size_t)n * q.M * P;
        T* to = q.dst + (size_t)n * q.M * P;
        constexpr int BATCH = 8;                                        // loads before the first store: the two may be the same map
        if constexpr (VEC > 0) {
            constexpr int W = NP * (int)sizeof(T) / 4;
            const size_t p = p0 + (size_t)NP * (lane & 7);
            if (p < P)
                for (int o0 = 4 * kw + (lane >> 3); o0 < q.M; o0 += BATCH * 4 * q.ks) {
                    Words<W> v[BATCH];
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) v[i] = q.base ? load_words<W>(from + min(o0 + 4 * i * q.ks, q.M - 1) * P + p) : Words<W>{};
#pragma unroll
                    for (int i = 0; i < BATCH; ++i)
                        if (o0 + 4 * i * q.ks < q.M) store_words(to + (o0 + 4 * i * q.ks) * P + p, v[i]);
                }
        } else {
            for (size_t p = p0 + lane; p < min(P, p0 + TP); p += 32)
                for (int o0 = kw; o0 < q.M; o0 += BATCH * q.ks) {
                    float v[BATCH];
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) v[i] = q.base ? load_one(from + min(o0 + i * q.ks, q.M - 1) * P + p) : 0.0f;
#pragma unroll
                    for (int i = 0; i < BATCH; ++i)
                        if (o0 + i * q.ks < q.M) store_one(to + (o0 + i * q.ks) * P + p, v[i]);
                }
        }
        return;
    }

    float acc[MB][RB][4];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int jb = 0; jb < RB; ++jb)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[mb][jb][i] = 0.0f;

    const int groups = (q.K + GC - 1) / GC;
    const size_t pl = p0 + (size_t)NP * g;
    const T* src = q.src + (size_t)n * q.K * P;
    const size_t pc = pl < P ? pl : 0;
    const T* src_end = q.src + (size_t)q.N * q.K * P;
    const uint4* w1 = q.w1 + (size_t)a * first_words<T>(RB, q.K) + lane;
    const size_t limit = q.tap ? q.Pp : P;                             // the tap is zero behind P
    if (p0 < P)
#pragma unroll 2
        for (int grp = kw; grp < groups; grp += q.ks) {
            // Channels behind the last one meet zeros in the factor, positions behind the last one are never stored: both load something else that
            // exists, so that all loads of a group go out together.
            Words<NP * (int)sizeof(T) / 4> x[CL];
#pragma unroll
            for (int i = 0; i < CL; ++i) {
                const T* xp = src + (size_t)min(grp * GC + t * CL + i, q.K - 1) * P;
                if constexpr (VEC > 0) x[i] = load_words<NP * (int)sizeof(T) / 4>(xp + pc);
                else x[i] = load_row<T, NP, false>(xp, pl, P, src_end);
            }
            const uint4* wg = w1 + (size_t)grp * RB * PARTS * 32;
            if constexpr (HALF) {
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
                    const uint4 w = __ldg(wg + jb * 32);
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_bf16(d, fa[0][mb], w.x, w.y);
                        mma_bf16(d, fa[1][mb], w.z, w.w);
                        add(acc[mb][jb], d);
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
                    const uint4 wh = __ldg(wg + (jb * 2) * 32), wl = __ldg(wg + (jb * 2 + 1) * 32);
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        mma_tf32(d, lo[0][mb], wh.x, wh.y);
                        mma_tf32(d, lo[1][mb], wh.z, wh.w);
                        mma_tf32(d, hi[0][mb], wl.x, wl.y);
                        mma_tf32(d, hi[1][mb], wl.z, wl.w);
                        mma_tf32(d, hi[0][mb], wh.x, wh.y);
                        mma_tf32(d, hi[1][mb], wh.z, wh.w);
                        add(acc[mb][jb], d);
                    }
                }
            }
        }

    if (q.ks > 1) {
        // the warps of a tile add their partial sums, every warp all of them in the same order
        float4* mine = sm + (size_t)warp * (MB * RB * 32) + lane;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb) mine[(mb * RB + jb) * 32] = make_float4(acc[mb][jb][0], acc[mb][jb][1], acc[mb][jb][2], acc[mb][jb][3]);
        __syncthreads();
        const float4* all = sm + (size_t)(warp - kw) * (MB * RB * 32) + lane;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int jb = 0; jb < RB; ++jb) {
                float4 v = all[(mb * RB + jb) * 32];
                for (int w = 1; w < q.ks; ++w) {
                    const float4 u = all[(size_t)w * (MB * RB * 32) + (mb * RB + jb) * 32];
                    v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                }
                acc[mb][jb][0] = v.x; acc[mb][jb][1] = v.y; acc[mb][jb][2] = v.z; acc[mb][jb][3] = v.w;
            }
    }
    if (p0 >= limit) return;
    const float sc = q.scale ? q.scale[a] : 1.0f;
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int jb = 0; jb < RB; ++jb)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[mb][jb][i] *= sc;

    if (q.tap && kw == 0) {
        if (pl >= P) {
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int jb = 0; jb < RB; ++jb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[mb][jb][i] = 0.0f;
        }
        // rank j = 8 jb + 2 t + e: this lane's positions p0 + NP g + b are accumulators [b / 2][jb][2 (b % 2) + e]
#pragma unroll
        for (int jb = 0; jb < RB; ++jb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const size_t at = ((size_t)n * (8 * RB) + 8 * jb + 2 * t + e) * q.Pp + pl;
                if constexpr (HALF) {
                    Words<MB> hi, mid, lo;
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        const float v0 = acc[mb][jb][e], v1 = acc[mb][jb][2 + e];
                        hi.w[mb] = pack_bf16x2(v0, v1);
                        split_bf16(v0 - bf16lo(hi.w[mb]), v1 - bf16hi(hi.w[mb]), mid.w[mb], lo.w[mb]);
                    }
                    T* plane = static_cast<T*>(q.tap) + at;
                    const size_t next = (size_t)q.N * (8 * RB) * q.Pp;
                    store_words(plane, hi);
                    store_words(plane + next, mid);
                    store_words(plane + 2 * next, lo);
                } else {
                    Words<NP> v;
#pragma unroll
                    for (int b = 0; b < NP; ++b) v.w[b] = __float_as_uint(acc[b >> 1][jb][2 * (b & 1) + e]);
                    store_words(static_cast<T*>(q.tap) + at, v);
                }
            }
    }
    if (!q.w2 || p0 >= P) return;

    // the accumulators as operands: of position b, block jb of ranks
    constexpr int UW = HALF ? 1 : 2;
    uint32_t uh[NP][RB][UW], ul[NP][RB][UW];
#pragma unroll
    for (int b = 0; b < NP; ++b)
#pragma unroll
        for (int jb = 0; jb < RB; ++jb) {
            const float u0 = acc[b >> 1][jb][2 * (b & 1)], u1 = acc[b >> 1][jb][2 * (b & 1) + 1];
            if constexpr (HALF) split_bf16(u0, u1, uh[b][jb][0], ul[b][jb][0]);
            else {
                split_tf32(__float_as_uint(u0), uh[b][jb][0], ul[b][jb][0]);
                split_tf32(__float_as_uint(u1), uh[b][jb][UW - 1], ul[b][jb][UW - 1]);
            }
        }
    float* out = reinterpret_cast<float*>(sm) + (q.ks > 1 ? (size_t)(blockDim.x >> 5) * (MB * RB * 128) : 0) + warp * 16 * (TP + 4);
    const uint4* w2 = q.w2 + (size_t)a * second_words<T>(RB, q.M) + lane;
    constexpr int NS = steps2<T>(RB);
    // the base of the next 16 channels is loaded while these are computed: the loads of one iteration would be waited for in every one
    using Piece = Words<NO * (int)sizeof(T) / 4>;
    auto load_base = [&](int mo, Piece(&b)[2][PIECES]) {
        if (VEC > 0 && q.base && mo < mo_n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const T* row = q.base + ((size_t)n * q.M + min(16 * mo + g + 8 * h, q.M - 1)) * P;
#pragma unroll
                for (int e = 0; e < PIECES; ++e) b[h][e] = load_words<NO * (int)sizeof(T) / 4>(row + (pw + NO * e < P ? pw + NO * e : 0));
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < PIECES; ++e) b[h][e] = Piece{};
        }
    };
    Piece next[2][PIECES];
    load_base(kw, next);
    for (int mo = kw; mo < mo_n; mo += q.ks) {
        Piece bs[2][PIECES];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < PIECES; ++e) bs[h][e] = next[h][e];
        load_base(mo + q.ks, next);
        float d[NP][4];
#pragma unroll
        for (int b = 0; b < NP; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) d[b][i] = 0.0f;
        const uint4* wm = w2 + (size_t)mo * NS * PARTS * 32;
#pragma unroll
        for (int ks = 0; ks < NS; ++ks) {
            if constexpr (HALF) {
                const uint4 w = __ldg(wm + ks * 32);
#pragma unroll
                for (int b = 0; b < NP; ++b) {
                    mma_bf16(d[b], w.x, w.y, w.z, w.w, ul[b][2 * ks][0], 2 * ks + 1 < RB ? ul[b][(2 * ks + 1) % RB][0] : 0u);
                    mma_bf16(d[b], w.x, w.y, w.z, w.w, uh[b][2 * ks][0], 2 * ks + 1 < RB ? uh[b][(2 * ks + 1) % RB][0] : 0u);
                }
            } else {
                const uint4 wh = __ldg(wm + (ks * 2) * 32), wl = __ldg(wm + (ks * 2 + 1) * 32);
#pragma unroll
                for (int b = 0; b < NP; ++b) {
                    mma_tf32(d[b], wl.x, wl.y, wl.z, wl.w, uh[b][ks][0], uh[b][ks][UW - 1]);
                    mma_tf32(d[b], wh.x, wh.y, wh.z, wh.w, ul[b][ks][0], ul[b][ks][UW - 1]);
                    mma_tf32(d[b], wh.x, wh.y, wh.z, wh.w, uh[b][ks][0], uh[b][ks][UW - 1]);
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
            const int rows = min(16, q.M - 16 * mo);
            const size_t at = ((size_t)n * q.M + 16 * mo) * P + p0, here = P - p0;
#pragma unroll 8
            for (int i = lane; i < 16 * TP; i += 32) {
                const int r = i / TP, c = i % TP;
                if (r < rows && (size_t)c < here) {
                    const size_t j = at + r * P + c;
                    float v = out[r * (TP + 4) + c];
                    if (q.base) v += load_one(q.base + j);
                    store_one(q.dst + j, v);
                }
            }
        } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int o = 16 * mo + g + 8 * h;
            if (o >= q.M) continue;
            T* row = q.dst + ((size_t)n * q.M + o) * P;
#pragma unroll
            for (int e = 0; e < PIECES; ++e) {
                Piece v;
#pragma unroll
                for (int i = 0; i < NO * (int)sizeof(T) / 4; ++i) {
                    if constexpr (HALF) {
                        const int at = NO * e + 2 * i;                  // of the lane's 2 NP positions
                        v.w[i] = pack_bf16x2(d[at % NP][2 * h + at / NP] + bf16lo(bs[h][e].w[i]), d[at % NP + 1][2 * h + at / NP] + bf16hi(bs[h][e].w[i]));
                    } else {
                        const int at = NO * e + i;
                        v.w[i] = __float_as_uint(d[at % NP][2 * h + at / NP] + __uint_as_float(bs[h][e].w[i]));
                    }
                }
                if (pw + NO * e < P) store_words(row + pw + NO * e, v);
            }
        }
        }
    }
}

// Up to two maps in one launch (the backward pass projects dy and x): the second takes the CTAs from q0.items on.
template <typename T, int RB, int VEC>
__global__ void __launch_bounds__(256) apply_kernel(ApplyArgs<T> q0, ApplyArgs<T> q1)
{
    extern __shared__ float4 apply_sm[];
    pdl_wait();
    pdl_launch();
    const int item = blockIdx.x;
    if (item < q0.items) apply_body<T, RB, VEC>(q0, item, apply_sm);
    else apply_body<T, RB, VEC>(q1, item - q0.items, apply_sm);
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
            for (int h = 0; h < 2; ++h) {
                const Words<4>(&xw)[2] = xr[h];
                const size_t at = ((size_t)n * (8 * RB) + 8 * jb + g) * q.Pp + pb + h * (TP / 2) + t * NP;
                if constexpr (sizeof(T) == 2) {
                    const __nv_bfloat16* pl = static_cast<const __nv_bfloat16*>(plane) + at;
                    const uint32_t a0[4] = {xw[0].w[0], xw[1].w[0], xw[0].w[1], xw[1].w[1]}, a1[4] = {xw[0].w[2], xw[1].w[2], xw[0].w[3], xw[1].w[3]};
#pragma unroll
                    for (int part = 2; part >= 0; --part) {
                        const uint4 v = *reinterpret_cast<const uint4*>(pl + (size_t)part * q.N * (8 * RB) * q.Pp);
                        mma_bf16(d, a0, v.x, v.y);
                        mma_bf16(d, a1, v.z, v.w);
                    }
                } else {
                    const uint4 v = *reinterpret_cast<const uint4*>(static_cast<const float*>(plane) + at);
                    const uint32_t vw[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        uint32_t ah[4], al[4], bh[2], bl[2];
#pragma unroll
                        for (int i = 0; i < 4; ++i) split_tf32(xw[i & 1].w[2 * s + (i >> 1)], ah[i], al[i]);
                        split_tf32(vw[2 * s], bh[0], bl[0]);
                        split_tf32(vw[2 * s + 1], bh[1], bl[1]);
                        mma_tf32(d, al, bh[0], bh[1]);
                        mma_tf32(d, ah, bl[0], bl[1]);
                        mma_tf32(d, ah, bh[0], bh[1]);
                    }
                }
            }
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

// ---- plans and launches -----------------------------------------------------------------------------
struct Ws {
    void* first[2];
    void* second[2];
    void* tap[2];
    int32_t* order;
    int32_t* start;
    float* part;
    size_t Pp;
    int ranges;
    size_t total;
};

inline int blocks_of(int rank) { return rank <= 8 ? 1 : rank <= 16 ? 2 : rank <= 32 ? 4 : 8; }

template <typename T>
static Ws carve(void* ws, int N, int Cin, int Cout, size_t P, int R, int rank, bool bwd)
{
    Ws w{};
    const int rb = blocks_of(rank), TP = Geo<T>::TP;
    size_t off = 0;
    char* b = static_cast<char*>(ws);
    auto take = [&](size_t bytes) { char* p = b ? b + off : nullptr; off += align_up(bytes, 256); return p; };
    if (!bwd) {
        if (P > 1) {
            w.first[0] = take((size_t)R * first_words<T>(rb, Cin) * 16);
            w.second[0] = take((size_t)R * second_words<T>(rb, Cout) * 16);
        }
        w.total = off;
        return w;
    }
    w.Pp = (P + TP - 1) / TP * TP;
    w.first[0] = take((size_t)R * first_words<T>(rb, Cout) * 16);       // B^T: dy -> V
    w.second[0] = take((size_t)R * second_words<T>(rb, Cin) * 16);      // A^T: V -> dx
    w.first[1] = take((size_t)R * first_words<T>(rb, Cin) * 16);        // A: x -> U
    for (int i = 0; i < 2; ++i) w.tap[i] = take((size_t)N * 8 * rb * w.Pp * (sizeof(T) == 2 ? 6 : 4));
    w.order = reinterpret_cast<int32_t*>(take((size_t)N * 4));
    w.start = reinterpret_cast<int32_t*>(take((size_t)(R + 1) * 4));
    const int all = ceil_div(Cin, 16) + ceil_div(Cout, 16);
    const long long units = (long long)N * (w.Pp / TP);
    const long long want = (16LL * B200_SMS + all - 1) / all;
    w.ranges = (int)std::max(1LL, std::min(want, units));
    w.part = reinterpret_cast<float*>(take((size_t)(w.ranges + R) * all * 16 * 8 * rb * 4));
    w.total = off;
    return w;
}

// Warps that share a tile: more only while the tiles alone do not fill the GPU.
// Partial sums of warps that share a tile, and the tiles on their way out where rows start anywhere.
template <typename T> static size_t apply_smem(int warps, int rb, int ks, bool vec)
{
    const int np = lane_positions<T>(rb);
    return (size_t)warps * ((ks > 1 ? (np / 2) * rb * 512 : 0) + (vec ? 0 : 16 * (8 * np + 4) * 4));
}
template <typename T>
static void plan_apply(ApplyArgs<T>& q, int rb, int& warps)
{
    const int tp = 8 * lane_positions<T>(rb);
    const long long tiles = (long long)(((q.tap ? q.Pp : q.P) + tp - 1) / tp);
    const int parts = std::max(ceil_div(q.K, Geo<T>::GC), q.w2 ? ceil_div(q.M, 16) : 1);
    q.ks = 1;
    while (q.ks < 8 && q.ks * 2 <= parts && (long long)q.N * tiles * q.ks < AD_FILL * B200_SMS) q.ks *= 2;
    warps = q.ks == 8 ? 8 : 4;
    const int per = warps / q.ks;
    q.tiles = (int)((tiles + per - 1) / per);
}

template <typename T, int RB, int VEC>
static wcc_status run_apply(ApplyArgs<T> q0, ApplyArgs<T>* q1, int dev, cudaStream_t st)
{
    int warps, warps1 = 0;
    plan_apply(q0, RB, warps);
    if (q1) {
        plan_apply(*q1, RB, warps1);
        if (warps1 != warps) {          // one block size for the launch: the larger, whose other map then has more tiles a CTA
            warps = std::max(warps, warps1);
            for (ApplyArgs<T>* p : {&q0, q1}) {
                const int tp = 8 * lane_positions<T>(RB);
                const long long tiles = (long long)(((p->tap ? p->Pp : p->P) + tp - 1) / tp);
                p->tiles = (int)((tiles + warps / p->ks - 1) / (warps / p->ks));
            }
        }
    }
    size_t smem = apply_smem<T>(warps, RB, q0.ks, VEC > 0);
    if (q1) smem = std::max(smem, apply_smem<T>(warps, RB, q1->ks, VEC > 0));
    const long long items = (long long)q0.N * q0.tiles, items1 = q1 ? (long long)q1->N * q1->tiles : 0;
    if (items + items1 > 0x7FFFFFFFLL) return WCC_ERR_SHAPE;
    q0.items = (int)items;
    if (q1) q1->items = (int)items1;
    wcc_status s = allow_smem<apply_kernel<T, RB, VEC>>(dev, (int)smem);
    if (s != WCC_OK) return s;
    return launch_overlapped(apply_kernel<T, RB, VEC>, dim3((unsigned)(items + items1)), dim3((unsigned)(32 * warps)), smem, st, true, 1, q0, q1 ? *q1 : q0);
}
template <typename T>
static wcc_status launch_apply(const ApplyArgs<T>& q0, ApplyArgs<T>* q1, int rb, int dev, cudaStream_t st)
{
    const int np = lane_positions<T>(rb), vec = q0.P % (2 * np) == 0 ? 2 : q0.P % np == 0 ? 1 : 0;
#define WCC_AD_APPLY(RB_)                                                                      \
    if (rb == (RB_))                                                                           \
        return vec == 2 ? run_apply<T, RB_, 2>(q0, q1, dev, st) : vec == 1 ? run_apply<T, RB_, 1>(q0, q1, dev, st) : run_apply<T, RB_, 0>(q0, q1, dev, st);
    WCC_AD_APPLY(1) WCC_AD_APPLY(2) WCC_AD_APPLY(4) WCC_AD_APPLY(8)
#undef WCC_AD_APPLY
    return WCC_ERR_SHAPE;
}

template <typename T>
static wcc_status launch_prep(const PrepArgs<T>& q, cudaStream_t st)
{
    const size_t words = std::max({q.first[0].p ? first_words<T>(q.rb, q.K[0]) : 0, q.first[1].p ? first_words<T>(q.rb, q.K[1]) : 0,
                                   q.second[0].p ? second_words<T>(q.rb, q.M[0]) : 0, q.second[1].p ? second_words<T>(q.rb, q.M[1]) : 0});
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
    PrepArgs<T> p{};
    p.first[0] = Factor<T>{static_cast<const T*>(A), (long long)rank * Cin, Cin, 1};
    p.second[0] = Factor<T>{static_cast<const T*>(B), (long long)Cout * rank, 1, rank};
    p.first_out[0] = static_cast<uint4*>(w.first[0]); p.second_out[0] = static_cast<uint4*>(w.second[0]);
    p.K[0] = Cin; p.M[0] = Cout; p.R = R; p.r = rank; p.rb = rb; p.N = N; p.ids = ids;
    if ((s = launch_prep(p, st)) != WCC_OK) return s;
    ApplyArgs<T> q{};
    q.src = static_cast<const T*>(x); q.w1 = static_cast<const uint4*>(w.first[0]); q.w2 = static_cast<const uint4*>(w.second[0]);
    q.scale = scale; q.ids = ids; q.base = static_cast<const T*>(base); q.dst = static_cast<T*>(y);
    q.P = P; q.N = N; q.K = Cin; q.M = Cout; q.R = R; q.status = di.status;
    return launch_apply<T>(q, nullptr, rb, di.dev, st);
}

template <typename T>
static wcc_status backward(const void* dy, const void* x, const void* A, const void* B, const float* scale, const int32_t* ids, const void* base, int N,
                           int Cin, int Cout, size_t P, int R, int rank, void* dx, float* dA, float* dB, void* ws, cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    const Ws w = carve<T>(ws, N, Cin, Cout, P, R, rank, true);
    const int rb = blocks_of(rank);
    const bool vec = P % Geo<T>::NP == 0, params = dA != nullptr;
    PrepArgs<T> p{};
    p.first[0] = Factor<T>{static_cast<const T*>(B), (long long)Cout * rank, 1, rank};
    if (dx) p.second[0] = Factor<T>{static_cast<const T*>(A), (long long)rank * Cin, Cin, 1};
    if (params) p.first[1] = Factor<T>{static_cast<const T*>(A), (long long)rank * Cin, Cin, 1};
    p.first_out[0] = static_cast<uint4*>(w.first[0]); p.first_out[1] = static_cast<uint4*>(w.first[1]); p.second_out[0] = static_cast<uint4*>(w.second[0]);
    p.K[0] = Cout; p.K[1] = Cin; p.M[0] = Cin; p.R = R; p.r = rank; p.rb = rb; p.N = N; p.ids = ids;
    if (params) { p.order = w.order; p.start = w.start; }
    if ((s = launch_prep(p, st)) != WCC_OK) return s;
    ApplyArgs<T> q{}, u{};
    q.src = static_cast<const T*>(dy); q.w1 = static_cast<const uint4*>(w.first[0]); q.w2 = dx ? static_cast<const uint4*>(w.second[0]) : nullptr;
    q.scale = scale; q.ids = ids; q.base = static_cast<const T*>(base); q.dst = static_cast<T*>(dx); q.tap = params ? w.tap[0] : nullptr;
    q.P = P; q.Pp = w.Pp; q.N = N; q.K = Cout; q.M = Cin; q.R = R; q.status = di.status;
    u = q;
    u.src = static_cast<const T*>(x); u.w1 = static_cast<const uint4*>(w.first[1]); u.w2 = nullptr; u.scale = nullptr; u.base = nullptr;
    u.dst = nullptr; u.tap = w.tap[1]; u.K = Cin; u.M = 0;
    if ((s = launch_apply<T>(q, params ? &u : nullptr, rb, di.dev, st)) != WCC_OK || !params) return s;
    GradArgs<T> h{};
    h.map[0] = static_cast<const T*>(x); h.map[1] = static_cast<const T*>(dy); h.plane[0] = w.tap[0]; h.plane[1] = w.tap[1];
    h.part = w.part; h.order = w.order; h.start = w.start; h.ids = ids; h.P = P; h.Pp = w.Pp;
    h.C[0] = Cin; h.C[1] = Cout; h.blocks[0] = ceil_div(Cin, 16); h.blocks[1] = ceil_div(Cout, 16);
    h.N = N; h.R = R; h.ranges = w.ranges; h.tiles = (int)(w.Pp / Geo<T>::TP);
    const int all = h.blocks[0] + h.blocks[1];
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
