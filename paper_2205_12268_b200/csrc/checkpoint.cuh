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
// top: the largest magnitude as fmaxf gives it (NaN values left out); bad: a NaN or an infinity is among the values
__device__ __forceinline__ Scale scale_of(float top, bool bad)
{
    if (bad) return {0.0f, __int_as_float(0x7FC00000)};
    if (top < SMALLEST) return {0.0f, 0.0f};
    return {__fdiv_rn(127.0f, top), __fdiv_rn(top, 127.0f)};
}
// |x * inv| <= 127 (1 + 2^-23) rounds to 127 at most.  A block that is not finite has inv = 0: its codes are 0 or, for NaN, what the
// conversion makes of NaN, which is 0 as well.
__device__ __forceinline__ int code_of(float x, float inv) { return __float2int_rn(x * inv); }
__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u; }

// One warp a block, lanes on neighbouring values: rows may start anywhere.
template <typename T>
__global__ void __launch_bounds__(256) pack_kernel(const T* __restrict__ x, long long rows, int L, int nb, int8_t* __restrict__ codes, float* __restrict__ scales)
{
    pdl_wait();
    pdl_launch();
    const int lane = threadIdx.x & 31;
    const long long blocks = rows * nb, step = (long long)gridDim.x * 8;
    for (long long b = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); b < blocks; b += step) {
        const long long row = b / nb;
        const int c0 = (int)(b - row * nb) * BLOCK, n = min(BLOCK, L - c0);
        const T* p = x + row * L + c0;
        float v[4], top = 0.0f;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = 0.0f;
            if (lane + 32 * i < n) v[i] = (float)p[lane + 32 * i];
            top = fmaxf(top, fabsf(v[i]));
            bad |= not_finite(v[i]);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        bad = __any_sync(0xFFFFFFFFu, bad);
        const Scale s = scale_of(top, bad);
        int8_t* q = codes + row * L + c0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 32 * i < n) q[lane + 32 * i] = (int8_t)code_of(v[i], s.inv);
        if (lane == 0) scales[b] = s.scale;
    }
}

// Sixteen neighbouring codes a thread, whatever the rows: codes and output are dense.
template <typename T>
__global__ void __launch_bounds__(256) restore_kernel(const int8_t* __restrict__ codes, const float* __restrict__ scales, long long total, int L, int nb,
                                                      T* __restrict__ out)
{
    pdl_wait();
    pdl_launch();
    constexpr int V = 16 / (int)sizeof(T);
    const long long step = (long long)gridDim.x * 256 * 16;
    for (long long f = ((long long)blockIdx.x * 256 + threadIdx.x) * 16; f < total; f += step) {
        long long row = f / L;
        int col = (int)(f - row * L);
        if (f + 16 <= total) {
            Vec<int8_t, 16> q;
            q.load(codes + f);
            float v[16];
            unpack(q, v);
            float s = __ldg(scales + row * nb + col / BLOCK);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                v[i] *= s;
                ++col;
                if (col == L) { col = 0; ++row; if (i < 15) s = __ldg(scales + row * nb); }
                else if (col % BLOCK == 0 && i < 15) s = __ldg(scales + row * nb + col / BLOCK);
            }
#pragma unroll
            for (int i = 0; i < 16; i += V) {
                float w[V];
#pragma unroll
                for (int j = 0; j < V; ++j) w[j] = v[i + j];
                Vec<T, V> o;
                pack(o, w);
                o.store(out + f + i);
            }
        } else {
            for (; f < total; ++f) {
                row = f / L;
                col = (int)(f - row * L);
                out[f] = (T)((float)codes[f] * __ldg(scales + row * nb + col / BLOCK));
            }
        }
    }
}

template <typename T>
wcc_status pack(const void* x, long long rows, int L, int8_t* codes, float* scales, cudaStream_t st)
{
    DeviceInfo di;
    const wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    const int nb = ceil_div(L, BLOCK);
    const long long want = (rows * nb + 7) / 8, most = (long long)di.sms * 8;
    return launch_overlapped(pack_kernel<T>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, true, 1, static_cast<const T*>(x), rows, L, nb,
                             codes, scales);
}
template <typename T>
wcc_status restore(const int8_t* codes, const float* scales, long long rows, int L, void* out, cudaStream_t st)
{
    DeviceInfo di;
    const wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    const int nb = ceil_div(L, BLOCK);
    const long long total = rows * L, want = (total + 4095) / 4096, most = (long long)di.sms * 8;
    return launch_overlapped(restore_kernel<T>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, true, 1, codes, scales, total, L, nb,
                             static_cast<T*>(out));
}

}  // namespace ck
}  // namespace wcc
