// Vectors of neighbouring values, packed fp32 arithmetic and activations, shared by the kernels for training (group norm, checkpoints, gated block).
#pragma once

#include "common.cuh"

namespace wcc {
namespace tr {

// ---- two fp32 operations in one instruction ------------------------------------------------------
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n fma.rn.f32x2 a, a, b, c;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

__device__ __forceinline__ float exp2_approx(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp_approx(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// ---- vectors of V values of type T, V * sizeof(T) <= 16 bytes ------------------------------------
template <int BYTES> struct Words;
template <> struct Words<16> { uint4 w; };
template <> struct Words<8> { uint2 w; };
template <> struct Words<4> { uint32_t w; };
template <> struct Words<2> { uint16_t w; };
template <> struct Words<1> { uint8_t w; };

template <typename T, int V> struct Vec {
    using W = Words<(int)sizeof(T) * V>;
    W r;
    __device__ __forceinline__ void load(const T* p) { r = *reinterpret_cast<const W*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<W*>(p) = r; }
};

template <int V> __device__ __forceinline__ void unpack(const Vec<float, V>& v, float (&f)[V])
{
    const float* p = reinterpret_cast<const float*>(&v.r);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = p[i];
}
template <int V> __device__ __forceinline__ void unpack(const Vec<__nv_bfloat16, V>& v, float (&f)[V])
{
    if constexpr (V == 1) {
        f[0] = __uint_as_float((uint32_t)v.r.w << 16);
    } else {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(&v.r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            f[2 * i] = bf16lo(p[i]);
            f[2 * i + 1] = bf16hi(p[i]);
        }
    }
}
template <int V> __device__ __forceinline__ void unpack(const Vec<int8_t, V>& v, float (&f)[V])
{
    const int8_t* p = reinterpret_cast<const int8_t*>(&v.r);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = (float)p[i];
}
template <int V> __device__ __forceinline__ void pack(Vec<float, V>& v, const float (&f)[V])
{
    float* p = reinterpret_cast<float*>(&v.r);
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = f[i];
}
template <int V> __device__ __forceinline__ void pack(Vec<__nv_bfloat16, V>& v, const float (&f)[V])
{
    if constexpr (V == 1) {
        v.r.w = __bfloat16_as_ushort(__float2bfloat16_rn(f[0]));
    } else {
        uint32_t* p = reinterpret_cast<uint32_t*>(&v.r);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) p[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
    }
}

// ---- activations ---------------------------------------------------------------------------------
// 1 / (1 + e^-z).  e^-z overflows to infinity below z = -88 and the result is 0, as it should be to fp32.
__device__ __forceinline__ float sigmoid(float z) { return rcp_approx(1.0f + exp2_approx(-1.4426950408889634f * z)); }

}  // namespace tr
}  // namespace wcc
