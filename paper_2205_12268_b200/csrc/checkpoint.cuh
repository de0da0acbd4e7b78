// Activation checkpoints in 8 bits: blocks of 128 consecutive values of a row, int8 codes and an fp32 scale each.
//     code = rint(x * (127 / top)),  scale = top / 127,  top = the block's largest magnitude
// The bytes bound both kernels: es + 1 a value.
#pragma once

#include "vec.cuh"

namespace wcc {
namespace ck {

using namespace tr;

constexpr int BLOCK = WCC_CKPT_BLOCK;
constexpr float SMALLEST = 7.8886090522101181e-31f;    // 2^-100: 127 / top stays far from the end of fp32

struct Scale { float inv, scale; };
__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u; }
// The larger magnitude; NaN if either is.
__device__ __forceinline__ float larger(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}
// Of a block with the largest magnitude `top` (NaN if a NaN is among its values).
__device__ __forceinline__ Scale scale_of(float top)
{
    if (not_finite(top)) return {0.0f, __int_as_float(0x7FC00000)};
    if (top < SMALLEST) return {0.0f, 0.0f};
    return {__fdiv_rn(127.0f, top), __fdiv_rn(top, 127.0f)};
}
// A value's code in the low byte: |x * inv| <= 127 (1 + 2^-23), and adding 1.5 * 2^23 rounds it to a whole number, ties to even.  (Two roundings: as a pair of
// packed instructions they came back as one multiply-add, whose ties are others.)
__device__ __forceinline__ uint32_t code_of(float x, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(x, inv), 12582912.0f)); }
__device__ __forceinline__ uint32_t pack_codes(f2 a, f2 b, float inv)
{
    return __byte_perm(__byte_perm(code_of(a.x(), inv), code_of(a.y(), inv), 0x0040), __byte_perm(code_of(b.x(), inv), code_of(b.y(), inv), 0x0040), 0x5410);
}
// The largest magnitude among 16 bytes of values and, by shuffles, among those of LANES lanes, for U such vectors; NaN if a NaN is among them.  bf16: by pairs.
template <int LANES, int U> __device__ __forceinline__ void largest(const uint4 (&w)[U], float (&top)[U], float)
{
#pragma unroll
    for (int u = 0; u < U; ++u)
        top[u] = larger(larger(fabsf(__uint_as_float(w[u].x)), __uint_as_float(w[u].y)), larger(fabsf(__uint_as_float(w[u].z)), __uint_as_float(w[u].w)));
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) top[u] = larger(top[u], __shfl_xor_sync(0xFFFFFFFFu, top[u], o));
}
__device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <int LANES, int U> __device__ __forceinline__ void largest(const uint4 (&w)[U], float (&top)[U], __nv_bfloat16)
{
    constexpr uint32_t ABS = 0x7FFF7FFFu;
    uint32_t m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = larger2(larger2(w[u].x & ABS, w[u].y & ABS), larger2(w[u].z & ABS, w[u].w & ABS));
#pragma unroll
    for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
        for (int u = 0; u < U; ++u) m[u] = larger2(m[u], __shfl_xor_sync(0xFFFFFFFFu, m[u], o));
#pragma unroll
    for (int u = 0; u < U; ++u) top[u] = larger(bf16lo(m[u]), bf16hi(m[u]));
}
template <int V> __device__ __forceinline__ void put_codes(const Pairs<V>& f, float inv, int8_t* codes)
{
    uint32_t q[V / 4];
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
        q[i] = pack_codes(f.v[2 * i], f.v[2 * i + 1], inv);
        if (inv == 0.0f) q[i] = 0u;                        // (what is not finite times 0 is no number)
    }
    if constexpr (V == 8) *reinterpret_cast<uint2*>(codes) = make_uint2(q[0], q[1]);
    else *reinterpret_cast<uint32_t*>(codes) = q[0];
}

// Where block b lies: its row and its first column.  SMALL: rows * L < 2^31.
template <bool SMALL> __device__ __forceinline__ void place(long long b, int nb, Divisor by_nb, long long& row, int& c0)
{
    row = SMALL ? (long long)by_nb.div((int)b) : b / nb;
    c0 = (int)(b - row * nb) * BLOCK;
}

// Rows that start on 16 bytes: 16 bytes a lane, 16 (bf16) or 32 (fp32) lanes a block, fewer (LANES) where rows are shorter than a block, U blocks on the way at once.
template <typename T, int LANES, bool SMALL>
__global__ void __launch_bounds__(256, 5) pack_vectors(const T* __restrict__ x, long long blocks, int L, int nb, Divisor by_nb, int8_t* __restrict__ codes,
                                                    float* __restrict__ scales)
{
    constexpr int V = 16 / (int)sizeof(T), EACH = 256 / LANES, U = 4;
    static_assert(LANES >= U, "a lane divides for each of the U blocks");
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x % LANES, col = lane * V;
    for (long long b0 = (long long)blockIdx.x * EACH * U + threadIdx.x / LANES; b0 - threadIdx.x / LANES < blocks; b0 += (long long)gridDim.x * EACH * U) {
        uint4 w[U];
        long long at[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long b = b0 + u * EACH;
            long long row = 0;
            int c0 = 0;
            if (b < blocks) place<SMALL>(b, nb, by_nb, row, c0);
            on[u] = b < blocks && c0 + col < L;
            at[u] = row * L + c0 + col;
            w[u] = on[u] ? *reinterpret_cast<const uint4*>(x + at[u]) : make_uint4(0u, 0u, 0u, 0u);
        }
        float top[U];
        largest<LANES, U>(w, top, T());
        // each of four lanes divides for one of the four blocks
        float inv[U];
        const int j = lane & (U - 1);
        const Scale s = scale_of(j == 1 ? top[1] : j == 2 ? top[2] : j == 3 ? top[3] : top[0]);
#pragma unroll
        for (int u = 0; u < U; ++u) inv[u] = __shfl_sync(0xFFFFFFFFu, s.inv, u, LANES);
        if (lane < U && b0 + j * EACH < blocks) scales[b0 + j * EACH] = s.scale;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on[u]) {
                Pairs<V> f;
                unpack2(w[u], f, T());
                put_codes(f, inv[u], codes + at[u]);
            }
    }
}

// Rows that start anywhere: a warp a block, lanes on neighbouring values, U blocks on the way at once.
template <typename T, bool SMALL>
__global__ void __launch_bounds__(256) pack_anywhere(const T* __restrict__ x, long long blocks, int L, int nb, Divisor by_nb, int8_t* __restrict__ codes,
                                                     float* __restrict__ scales)
{
    constexpr int U = 3;
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31;
    for (long long b0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * U; b0 < blocks; b0 += (long long)gridDim.x * 8 * U) {
        float v[U][4];
        long long at[U];
        int n[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            long long row = 0;
            int c0 = 0;
            n[u] = 0;
            if (b0 + u < blocks) {
                place<SMALL>(b0 + u, nb, by_nb, row, c0);
                n[u] = min(BLOCK, L - c0);
            }
            at[u] = row * L + c0 + lane;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] = lane + 32 * i < n[u] ? (float)x[at[u] + 32 * i] : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (n[u] == 0) break;
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) top = larger(top, v[u][i]);
#pragma unroll
            for (int o = 16; o; o >>= 1) top = larger(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            const Scale s = scale_of(top);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 32 * i < n[u]) codes[at[u] + 32 * i] = s.inv == 0.0f ? (int8_t)0 : (int8_t)__float2int_rn(v[u][i] * s.inv);
            if (lane == 0) scales[b0 + u] = s.scale;
        }
    }
}

// Rows of up to 32 values that start anywhere: LANES lanes a row, U rows on the way at once.
template <typename T, int LANES>
__global__ void __launch_bounds__(256) pack_short(const T* __restrict__ x, long long rows, int L, int8_t* __restrict__ codes, float* __restrict__ scales)
{
    constexpr int EACH = 256 / LANES, U = 4;
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x % LANES;
    for (long long r0 = (long long)blockIdx.x * EACH * U + threadIdx.x / LANES; r0 - threadIdx.x / LANES < rows; r0 += (long long)gridDim.x * EACH * U) {
        float v[U], top[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * EACH;
            v[u] = r < rows && lane < L ? (float)x[r * L + lane] : 0.0f;
            top[u] = larger(0.0f, v[u]);
        }
#pragma unroll
        for (int o = LANES / 2; o; o >>= 1)
#pragma unroll
            for (int u = 0; u < U; ++u) top[u] = larger(top[u], __shfl_xor_sync(0xFFFFFFFFu, top[u], o));
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * EACH;
            const Scale s = scale_of(top[u]);
            if (r < rows && lane < L) codes[r * L + lane] = s.inv == 0.0f ? (int8_t)0 : (int8_t)__float2int_rn(v[u] * s.inv);
            if (r < rows && lane == 0) scales[r] = s.scale;
        }
    }
}

// 16 bytes of output a thread, whatever the rows: codes and output are dense.  ROUND: a vector's values are of one block (L a multiple of V); else most often.
template <typename T, bool SMALL, bool ROUND>
__global__ void __launch_bounds__(256) restore_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, long long total, int L, int nb,
                                                      Divisor by_L, T* __restrict__ out)
{
    constexpr int V = 16 / (int)sizeof(T), U = 4;
    pdl_wait();
    pdl_launch();
    const long long step = 256 * V;
    for (long long f0 = (long long)blockIdx.x * step * U + threadIdx.x * V; f0 < total; f0 += (long long)gridDim.x * step * U) {
        Vec<int8_t, V> q[U];
        long long row[U];
        int col[U];
        float s[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long f = f0 + u * step;
            if (f < total) {
                row[u] = SMALL ? (long long)by_L.div((int)f) : f / L;
                col[u] = (int)(f - row[u] * L);
                s[u] = __ldg(scales + row[u] * nb + col[u] / BLOCK);
                if (f + V <= total) q[u].load(codes + f);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long f = f0 + u * step;
            if (f >= total) break;
            if (f + V > total) {                           // the tensor's last few
                for (int i = 0; i < (int)(total - f); ++i) {
                    const long long r = (f + i) / L;
                    out[f + i] = (T)((float)codes[f + i] * __ldg(scales + r * nb + (int)(f + i - r * L) / BLOCK));
                }
                break;
            }
            float v[V];
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                f2 a, b;
                codes4(reinterpret_cast<const uint32_t*>(&q[u].r.w)[i / 4], a, b);
                v[i] = a.x(); v[i + 1] = a.y(); v[i + 2] = b.x(); v[i + 3] = b.y();
            }
            const int here = min(L - col[u], BLOCK - col[u] % BLOCK);      // values left of this block
            if (ROUND || here >= V) {
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] *= s[u];
            } else {
                long long r = row[u];
                int c = col[u], left = here;
                float w = s[u];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[i] *= w;
                    ++c;
                    if (--left == 0 && i < V - 1) {
                        if (c == L) { c = 0; ++r; }
                        left = min(L - c, BLOCK);
                        w = __ldg(scales + r * nb + c / BLOCK);
                    }
                }
            }
            Vec<T, V> o;
            pack(o, v);
            o.store(out + f);
        }
    }
}

template <typename T, int LANES>
wcc_status launch_pack(const T* x, long long blocks, int L, int nb, bool small, int8_t* codes, float* scales, const DeviceInfo& di, cudaStream_t st)
{
    const long long each = 4 * (256 / LANES), want = (blocks + each - 1) / each, most = (long long)di.sms * 10;
    return launch_overlapped(small ? pack_vectors<T, LANES, true> : pack_vectors<T, LANES, false>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0,
                             st, true, 1, x, blocks, L, nb, divisor_of((unsigned)nb), codes, scales);
}
template <typename T>
wcc_status pack(const void* in, long long rows, int L, int8_t* codes, float* scales, cudaStream_t st)
{
    DeviceInfo di;
    const wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    constexpr int FULL = BLOCK * (int)sizeof(T) / 16;
    const T* x = static_cast<const T*>(in);
    const int nb = ceil_div(L, BLOCK);
    const long long blocks = rows * nb;
    const bool small = rows * L < (1LL << 31);
    if ((long long)L * sizeof(T) % 16 == 0) {
        if (L <= BLOCK / 4) return launch_pack<T, FULL / 4>(x, blocks, L, nb, small, codes, scales, di, st);
        if (L <= BLOCK / 2) return launch_pack<T, FULL / 2>(x, blocks, L, nb, small, codes, scales, di, st);
        return launch_pack<T, FULL>(x, blocks, L, nb, small, codes, scales, di, st);
    }
    const long long most = (long long)di.sms * 8;
    if (L <= 32) {
        const int lanes = L <= 2 ? 2 : L <= 4 ? 4 : L <= 8 ? 8 : L <= 16 ? 16 : 32;
        const long long each = 4 * (256 / lanes), ctas = (rows + each - 1) / each;
        auto kernel = lanes == 2 ? pack_short<T, 2> : lanes == 4 ? pack_short<T, 4> : lanes == 8 ? pack_short<T, 8> : lanes == 16 ? pack_short<T, 16> : pack_short<T, 32>;
        return launch_overlapped(kernel, dim3((unsigned)(ctas < most ? ctas : most)), dim3(256), 0, st, true, 1, x, rows, L, codes, scales);
    }
    const long long want = (blocks + 23) / 24;
    return launch_overlapped(small ? pack_anywhere<T, true> : pack_anywhere<T, false>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, true, 1,
                             x, blocks, L, nb, divisor_of((unsigned)nb), codes, scales);
}
template <typename T>
wcc_status restore(const int8_t* codes, const float* scales, long long rows, int L, void* out, cudaStream_t st)
{
    DeviceInfo di;
    const wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    constexpr int V = 16 / (int)sizeof(T);
    const int nb = ceil_div(L, BLOCK);
    const long long total = rows * L, want = (total + 1024 * V - 1) / (1024 * V), most = (long long)di.sms * 16;
    const bool small = total < (1LL << 31), round = L % V == 0;
    auto kernel = round ? (small ? restore_kernel<T, true, true> : restore_kernel<T, false, true>) : (small ? restore_kernel<T, true, false> : restore_kernel<T, false, false>);
    return launch_overlapped(kernel, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, true, 1, codes, scales, total, L, nb,
                             divisor_of((unsigned)L), static_cast<T*>(out));
}

}  // namespace ck
}  // namespace wcc
