// Vectors of neighbouring values, packed fp32 arithmetic and activations, shared by the kernels for training (group norm, checkpoints, gated block).
#pragma once

#include "common.cuh"

namespace wcc {
namespace tr {

// ---- whole numbers -------------------------------------------------------------------------------
// n / d for 0 <= n < 2^31 by a multiplication: m = ceil(2^(32 + s) / d) < 2^32 with 2^s < d <= 2^(s + 1)
struct Divisor {
    unsigned m, s, d;
    __device__ __forceinline__ int div(int n) const { return d == 1 ? n : (int)(__umulhi((unsigned)n, m) >> s); }
    __device__ __forceinline__ int mod(int n) const { return n - div(n) * (int)d; }
};
inline Divisor divisor_of(unsigned d)
{
    unsigned s = 0;
    while ((2u << s) < d) ++s;             // 2^(s + 1) >= d
    return {d == 1 ? 0u : (unsigned)(((1ull << (32 + s)) + d - 1) / d), s, d};
}

// ---- two fp32 operations in one instruction ------------------------------------------------------
// The pair is a 64-bit value throughout, so that it stays in neighbouring registers.
struct f2 {
    unsigned long long w;
    __device__ __forceinline__ float x() const { return __uint_as_float((unsigned)w); }
    __device__ __forceinline__ float y() const { return __uint_as_float((unsigned)(w >> 32)); }
};
__device__ __forceinline__ f2 pair(float x, float y)
{
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.w) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ f2 both(float v) { return pair(v, v); }
__device__ __forceinline__ f2 add2(f2 a, f2 b)
{
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b)
{
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.w) : "l"(a.w), "l"(b.w));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c)
{
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.w) : "l"(a.w), "l"(b.w), "l"(c.w));
    return r;
}

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

// Two at once with one reciprocal, 1/a = b / (a b): the unit of 2^x and of reciprocals gives 16 results a clock and SM and bounds the backward pass of
// group norm with its four a value (three this way).  With t = e^z: 1 - s = 1 / (1 + t), s = t (1 - s), both to fp32's digits however small.  Above z = 43 t stays
// e^43, so that a b does not overflow: s is 1 long since.  (Held from below instead, as 1 / (1 + e^-z), s does not fall under e^-43, and z s is anything.)
struct Sigmoid2 { f2 s, rest; };           // sigmoid, 1 - sigmoid
__device__ __forceinline__ Sigmoid2 sigmoid2(f2 z)
{
    const f2 v = mul2(pair(fminf(z.x(), 43.0f), fminf(z.y(), 43.0f)), both(1.4426950408889634f));
    const f2 t = pair(exp2_approx(v.x()), exp2_approx(v.y())), a = add2(t, both(1.0f));
    const f2 rest = mul2(both(rcp_approx(a.x() * a.y())), pair(a.y(), a.x()));
    return {mul2(t, rest), rest};
}
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ f2 silu2(f2 z) { return mul2(z, sigmoid2(z).s); }
// s + z s (1 - s), z held at 43 as well: 1 - s is.  (A NaN stays one, and is its own value's alone.)
__device__ __forceinline__ f2 silu_slope2(f2 z, const Sigmoid2& q)
{
    return fma2(mul2(pair(min_nan(z.x(), 43.0f), min_nan(z.y(), 43.0f)), q.s), q.rest, q.s);
}

// Values of a vector as pairs.
template <int V> struct Pairs { f2 v[V / 2]; };

__device__ __forceinline__ void unpack2(const uint4& w, Pairs<4>& f, float)
{
    f.v[0] = pair(__uint_as_float(w.x), __uint_as_float(w.y));
    f.v[1] = pair(__uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ void unpack2(const uint4& w, Pairs<8>& f, __nv_bfloat16)
{
    f.v[0] = pair(bf16lo(w.x), bf16hi(w.x));
    f.v[1] = pair(bf16lo(w.y), bf16hi(w.y));
    f.v[2] = pair(bf16lo(w.z), bf16hi(w.z));
    f.v[3] = pair(bf16lo(w.w), bf16hi(w.w));
}
__device__ __forceinline__ uint4 pack2(const Pairs<4>& f, float)
{
    return make_uint4((unsigned)f.v[0].w, (unsigned)(f.v[0].w >> 32), (unsigned)f.v[1].w, (unsigned)(f.v[1].w >> 32));
}
__device__ __forceinline__ uint4 pack2(const Pairs<8>& f, __nv_bfloat16)
{
    return make_uint4(pack_bf16x2(f.v[0].x(), f.v[0].y()), pack_bf16x2(f.v[1].x(), f.v[1].y()), pack_bf16x2(f.v[2].x(), f.v[2].y()),
                      pack_bf16x2(f.v[3].x(), f.v[3].y()));
}
// Four int8 codes to fp32: with their sign bit flipped they are code + 128 in the low byte of 2^23, exact.
__device__ __forceinline__ void codes4(uint32_t w, f2& a, f2& b)
{
    w ^= 0x80808080u;
    const f2 off = both(-8388736.0f);
    a = add2(pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540)), __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7541))), off);
    b = add2(pair(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7542)), __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7543))), off);
}

}  // namespace tr
}  // namespace wcc
