// Layer norm over the channels of a map, forward and backward.  With C channels, at every position of every image
//     mu = 1/C sum_c x,   v = 1/C sum_c (x - mu)^2,   r = (v + eps)^-1/2,   xh = (x - mu) r
//     y  = xh gamma + beta
//     g  = dy gamma,  dx = r (g - 1/C sum_c g - xh 1/C sum_c g xh),  dgamma = sum dy xh,  dbeta = sum dy  (over images, positions).
// Both directions are bound by memory: every element is read once, kept on the SM until the statistics of its position are known, and
// written once.
//
// Maps: a CTA takes all channels of a tile of positions.  `segl` lanes cover 16 to 512 bytes of a channel's row in vectors of V elements; the
// groups of lanes hold channels g, g + G, ...: K vectors a thread.  Large maps whose rows start on 16 bytes go through a ring of TMA tiles
// (ln_ring), the others load straight into registers (ln_fwd_map, ln_bwd_map); channels beyond one CTA's registers go to a cluster whose
// CTAs exchange their sums through distributed shared memory.
// Rows (one position an image): the channels are contiguous.  Many rows: a warp a row, fed by copies of its own (ln_fwd_feed, ln_bwd_feed);
// few, wide or odd ones: 8, 32 or 256 threads a row.
// Statistics are fp32 sums over registers in two rounds, the mean and then the deviations from it, so that a large common offset of the
// channels costs no digits of the variance.
#pragma once

#include <algorithm>

#include "common.cuh"
#include "tma.cuh"

namespace wcc {
namespace ln {

constexpr int NT = 256;                 // threads of a CTA over rows
constexpr int WARPS = NT / 32;
constexpr int MAX_WARPS = 16;           // of a CTA over a map
constexpr unsigned FULL = 0xFFFFFFFFu;

// V elements of type T as they lie in memory.
template <typename T, int V>
struct Vec {
    static constexpr int BYTES = V * (int)sizeof(T);
    static constexpr int WORDS = BYTES >= 4 ? BYTES / 4 : 1;
    uint32_t w[WORDS];
    __device__ __forceinline__ void load(const T* p)
    {
        if (BYTES == 16) { const uint4 u = *reinterpret_cast<const uint4*>(p); w[0] = u.x; w[1 % WORDS] = u.y; w[2 % WORDS] = u.z; w[3 % WORDS] = u.w; }
        else if (BYTES == 8) { const uint2 u = *reinterpret_cast<const uint2*>(p); w[0] = u.x; w[1 % WORDS] = u.y; }
        else if (BYTES == 4) w[0] = *reinterpret_cast<const uint32_t*>(p);
        else w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    __device__ __forceinline__ void store(T* p) const
    {
        if (BYTES == 16) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1 % WORDS], w[2 % WORDS], w[3 % WORDS]);
        else if (BYTES == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1 % WORDS]);
        else if (BYTES == 4) *reinterpret_cast<uint32_t*>(p) = w[0];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
    }
    // Element i from p[i * stride]; only the first n.  (All of them but at the end of an image: without a test of each.)
    __device__ __forceinline__ void load(const T* p, int stride, int n)
    {
        if (n == V) {
#pragma unroll
            for (int i = 0; i < V; ++i, p += stride) put(i, p);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i, p += stride)
                if (i < n) put(i, p);
        }
    }
    __device__ __forceinline__ void put(int i, const T* p)
    {
        if (sizeof(T) == 4) w[i % WORDS] = *reinterpret_cast<const uint32_t*>(p);
        else {
            const uint32_t u = *reinterpret_cast<const uint16_t*>(p);
            w[(i >> 1) % WORDS] = i & 1 ? w[(i >> 1) % WORDS] | u << 16 : u;
        }
    }
    __device__ __forceinline__ void store(T* p, int stride, int n) const
    {
        if (n == V) {
#pragma unroll
            for (int i = 0; i < V; ++i, p += stride) take(i, p);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i, p += stride)
                if (i < n) take(i, p);
        }
    }
    __device__ __forceinline__ void take(int i, T* p) const
    {
        if (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(p) = w[i % WORDS];
        else *reinterpret_cast<uint16_t*>(p) = (uint16_t)(w[(i >> 1) % WORDS] >> (16 * (i & 1)));
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
    }
    // The values are unpacked again behind this: kept unpacked across a barrier they would take twice the registers.
    __device__ __forceinline__ void forget()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) asm volatile("" : "+r"(w[i]));
    }
    __device__ __forceinline__ float get(int i) const
    {
        if (sizeof(T) == 4) return __uint_as_float(w[i % WORDS]);
        return (i & 1) ? bf16hi(w[(i >> 1) % WORDS]) : bf16lo(w[(i >> 1) % WORDS]);
    }
    __device__ __forceinline__ void set(const float (&f)[V])
    {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) w[i % WORDS] = __float_as_uint(f[i]);
        } else if (V == 1) {
            w[0] = pack_bf16x2(f[0], 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 2) w[(i >> 1) % WORDS] = pack_bf16x2(f[i], f[(i + 1) % V]);
        }
    }
};

template <int V>
__device__ __forceinline__ void load_floats(const float* p, float (&f)[V])
{
    Vec<float, V >= 4 ? 4 : V> v;
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        v.load(p + i);
#pragma unroll
        for (int j = 0; j < (V < 4 ? V : 4); ++j) f[(i + j) % V] = v.get(j);
    }
}
template <int V>
__device__ __forceinline__ void store_floats(float* p, const float (&f)[V])
{
    constexpr int S = V >= 4 ? 4 : V;
    Vec<float, S> v;
#pragma unroll
    for (int i = 0; i < V; i += S) {
        float q[S];
#pragma unroll
        for (int j = 0; j < S; ++j) q[j] = f[i + j];
        v.set(q);
        v.store(p + i);
    }
}

// Element-wise fp32 arithmetic, two at a time where there are two.
__device__ __forceinline__ void add2(float& x0, float& x1, float a0, float a1, float b0, float b1)
{
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void mul2(float& x0, float& x1, float a0, float a1, float b0, float b1)
{
    asm("{\n .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ void fma2(float& x0, float& x1, float a0, float a1, float b0, float b1, float c0, float c1)
{
    asm("{\n .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n fma.rn.f32x2 a, a, b, c;\n mov.b64 {%0, %1}, a;\n}"
        : "=f"(x0), "=f"(x1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
template <int V> struct F {
    float f[V];
    __device__ __forceinline__ F() {}
    __device__ __forceinline__ explicit F(float s)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = s;
    }
};
template <int V> __device__ __forceinline__ F<V> operator+(const F<V>& a, const F<V>& b)
{
    F<V> r;
    if constexpr (V == 1) { r.f[0] = a.f[0] + b.f[0]; }
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) add2(r.f[i], r.f[i + 1], a.f[i], a.f[i + 1], b.f[i], b.f[i + 1]);
    }
    return r;
}
template <int V> __device__ __forceinline__ F<V> operator*(const F<V>& a, const F<V>& b)
{
    F<V> r;
    if constexpr (V == 1) { r.f[0] = a.f[0] * b.f[0]; }
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) mul2(r.f[i], r.f[i + 1], a.f[i], a.f[i + 1], b.f[i], b.f[i + 1]);
    }
    return r;
}
template <int V> __device__ __forceinline__ F<V> fma(const F<V>& a, const F<V>& b, const F<V>& c)
{
    F<V> r;
    if constexpr (V == 1) { r.f[0] = fmaf(a.f[0], b.f[0], c.f[0]); }
    else {
#pragma unroll
        for (int i = 0; i < V; i += 2) fma2(r.f[i], r.f[i + 1], a.f[i], a.f[i + 1], b.f[i], b.f[i + 1], c.f[i], c.f[i + 1]);
    }
    return r;
}
template <int V> __device__ __forceinline__ F<V> operator-(const F<V>& a)
{
    F<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.f[i] = -a.f[i];
    return r;
}
template <typename T, int V> __device__ __forceinline__ F<V> floats(const Vec<T, V>& v)
{
    F<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.f[i] = v.get(i);
    return r;
}

__device__ __forceinline__ uint32_t cluster_addr(const void* p, int rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float cluster_ld(uint32_t a)
{
    float f;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(a) : "memory");
    return f;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

struct MapGeom {
    size_t P;                           // positions of an image
    int C, Cs;                          // channels, and those of one CTA of a cluster
    int tiles, items;                   // tiles of an image, of the batch
    int segl_log2;
    int warps, groups_log2;             // of a CTA: warps, groups of lanes
    int pw_log2;                        // warps side by side over the positions (segl = 32)
    int cl;                             // CTAs of a cluster
};

// Sums of a tile's NS * V values per lane over all channels: over the groups of a warp, then over the warps, a thread per sum, through shared
// memory, and over the CTAs of a cluster.  Every thread ends up with the same bits.  Calls alternate between two buffers for the result:
// a neighbour of the cluster may still read the one before.
__host__ __device__ inline int tile_floats(const MapGeom& q, int tpos) { return ((q.warps >> q.pw_log2) + 2) * 2 * tpos; }
template <int V, int NS>
__device__ __forceinline__ void tile_sum(F<V> (&s)[NS], float* sm, const MapGeom& q, int l, int buf)
{
    const int segl = 1 << q.segl_log2, tpos = (segl << q.pw_log2) * V, parts = q.warps >> q.pw_log2;
    if (parts == 1 && segl == 32 && q.cl == 1) return;               // a warp has all channels of its positions
    for (int o = segl; o < 32; o <<= 1) {
#pragma unroll
        for (int j = 0; j < NS; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) s[j].f[i] += __shfl_xor_sync(FULL, s[j].f[i], o);
    }
    if ((int)(threadIdx.x & 31) < segl) {
#pragma unroll
        for (int j = 0; j < NS; ++j) store_floats<V>(sm + ((threadIdx.x >> (5 + q.pw_log2)) * NS + j) * tpos + l * V, s[j].f);
    }
    __syncthreads();
    float* res = sm + (parts + buf) * 2 * tpos;
    for (int i = threadIdx.x; i < NS * tpos; i += 32 * q.warps) {
        float a = sm[i];
        for (int w = 1; w < parts; ++w) a += sm[w * NS * tpos + i];
        res[i] = a;
    }
    if (q.cl > 1) {
        cluster_sync();
#pragma unroll
        for (int j = 0; j < NS; ++j) s[j] = F<V>(0.0f);
        for (int b = 0; b < q.cl; ++b) {
            const uint32_t a = cluster_addr(res, b);
#pragma unroll
            for (int j = 0; j < NS; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) s[j].f[i] += cluster_ld(a + 4u * (j * tpos + l * V + i));
        }
    } else {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NS; ++j) load_floats<V>(res + j * tpos + l * V, s[j].f);
    }
}

// Where a thread stands in a tile: column l of its positions, group g of its channels; its V positions run from `first` on, in a vector, or with
// STR every segl-th (rows that do not start on a vector: single loads, each of them coalesced).
template <int V, bool STR>
struct Place {
    int l, g, first, stride;
    __device__ __forceinline__ explicit Place(const MapGeom& q)
    {
        const int lane = threadIdx.x & 31, segl = 1 << q.segl_log2, wp = (threadIdx.x >> 5) & ((1 << q.pw_log2) - 1);
        l = wp * segl + (lane & (segl - 1));
        g = ((int)(threadIdx.x >> (5 + q.pw_log2)) << (5 - q.segl_log2)) + (lane >> q.segl_log2);
        first = STR ? wp * segl * V + (lane & (segl - 1)) : l * V;
        stride = segl;
    }
    // how many of the V positions from p on exist
    __device__ __forceinline__ int valid(size_t p, size_t P) const
    {
        if (p >= P) return 0;
        if (!STR) return V;
        const size_t n = (P - p + stride - 1) / stride;
        return n < V ? (int)n : V;
    }
};
template <typename T, int V, bool STR>
__device__ __forceinline__ void load_at(Vec<T, V>& v, const T* p, int stride, int nv)
{
    if (STR) v.load(p, stride, nv);
    else if (nv) v.load(p);
}
template <int V, bool STR>
__device__ __forceinline__ void load_floats_at(const float* p, int stride, int nv, float (&f)[V])
{
    if constexpr (STR) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < nv) f[i] = p[i * stride];
    } else if (nv) load_floats<V>(p, f);
}
template <int V, bool STR>
__device__ __forceinline__ void store_floats_at(float* p, int stride, int nv, const float (&f)[V])
{
    if constexpr (STR) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < nv) p[i * stride] = f[i];
    } else if (nv) store_floats<V>(p, f);
}

template <typename T, int V, int K>
__device__ __forceinline__ void forget(Vec<T, V> (&v)[K])
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k].forget();
}
// FULL: every thread has all K channels; tests of each slowed the large maps (4 x 1024 x 128 x 128 bf16 110 us instead of 65).
// A position's mean and reciprocal deviation from the channels that the tile's threads hold.  A first mean, then the sums of the deviations
// from it and of their squares: they correct it, and what it was off by enters the variance in second order only.
template <typename T, int V, int K, bool FULL>
__device__ __forceinline__ void statistics(Vec<T, V> (&v)[K], int nk, float eps, float* sm, const MapGeom& q, int l, F<V>& m, F<V>& r)
{
    const float inv_C = 1.0f / (float)q.C;
    F<V> s[2], one[1];
    one[0] = F<V>(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k) one[0] = one[0] + floats(v[k]);      // (zeros where there is no channel)
    forget<T, V, K>(v);
    tile_sum<V, 1>(one, sm, q, l, 0);
    m = one[0] * F<V>(inv_C);
    s[0] = s[1] = F<V>(0.0f);
    const F<V> neg = -m;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (FULL || k < nk) {
            const F<V> d = floats(v[k]) + neg;
            s[0] = s[0] + d;
            s[1] = fma(d, d, s[1]);
        }
    forget<T, V, K>(v);
    tile_sum<V, 2>(s, sm, q, l, 1);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float e = s[0].f[i] * inv_C, var = fmaf(s[1].f[i], inv_C, -e * e);
        m.f[i] += e;
        r.f[i] = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);      // (a NaN stays one)
    }
}
// y of a thread's channels, stored `step` elements apart; its k-th channel's parameters are at k * cstep.
template <typename T, int V, int K, bool STR, bool FULL>
__device__ __forceinline__ void normalise(Vec<T, V> (&v)[K], int nk, const F<V>& m, const F<V>& r, const float* pg, const float* pb, int cstep, T* py,
                                          size_t step, int stride, int nv)
{
    const F<V> neg = -m;
#pragma unroll
    for (int k = 0; k < K; ++k, py += step)
        if (FULL || k < nk) {
            const float ga = pg ? pg[k * cstep] : 1.0f, be = pb ? pb[k * cstep] : 0.0f;
            const F<V> o = fma((floats(v[k]) + neg) * r, F<V>(ga), F<V>(be));
            v[k].set(o.f);
            if constexpr (STR) v[k].store(py, stride, nv);
            else v[k].store(py);
        }
}
// The sums over the channels that a gradient needs (s: of g and of g xh), and this tile's share of the parameters' gradients.
template <typename T, int V, int K, bool FULL>
__device__ __forceinline__ void gradient_sums(const Vec<T, V> (&vx)[K], const Vec<T, V> (&vd)[K], int nk, const F<V>& neg, const F<V>& r, const float* pg,
                                              int cstep, F<V> (&s)[2], float (&dg)[K], float (&db)[K])
{
    s[0] = s[1] = F<V>(0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (FULL || k < nk) {
            const F<V> d = floats(vd[k]), xh = (floats(vx[k]) + neg) * r, gg = pg ? d * F<V>(pg[k * cstep]) : d;
            s[0] = s[0] + gg;
            s[1] = fma(gg, xh, s[1]);
#pragma unroll
            for (int i = 0; i < V; ++i) { dg[k] = fmaf(d.f[i], xh.f[i], dg[k]); db[k] += d.f[i]; }
        }
}
template <typename T, int V, int K, bool STR, bool FULL>
__device__ __forceinline__ void gradient(Vec<T, V> (&vx)[K], const Vec<T, V> (&vd)[K], int nk, const F<V>& neg, const F<V>& r, const float* pg, int cstep,
                                         const F<V> (&s)[2], float inv_C, T* po, size_t step, int stride, int nv)
{
    const F<V> c1 = s[0] * F<V>(-inv_C), c2 = s[1] * F<V>(-inv_C);
#pragma unroll
    for (int k = 0; k < K; ++k, po += step)
        if (FULL || k < nk) {
            const F<V> xh = (floats(vx[k]) + neg) * r;
            const F<V> o = r * fma(xh, c2, fma(floats(vd[k]), F<V>(pg ? pg[k * cstep] : 1.0f), c1));
            vx[k].set(o.f);
            if constexpr (STR) vx[k].store(po, stride, nv);
            else vx[k].store(po);
        }
}
// Where the sums of the parameters' gradients go: rows of partial sums [row][2][C], or, if there is one row only, the gradients themselves.
struct Partials {
    float *g, *b;                       // either may be NULL
    size_t pitch;
};
// The lanes of a channel add up and write row `row`; c: the thread's first channel.
template <int K>
__device__ __forceinline__ void store_partials(float (&dg)[K], float (&db)[K], int nk, int segl, int cstep, const Partials& out, int C, int row, int c)
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        for (int o = 1; o < segl; o <<= 1) { dg[k] += __shfl_xor_sync(FULL, dg[k], o); db[k] += __shfl_xor_sync(FULL, db[k], o); }
        if ((threadIdx.x & (segl - 1)) == 0 && k < nk) {
            if (out.g) out.g[row * out.pitch + c + k * cstep] = dg[k];
            if (out.b) out.b[row * out.pitch + c + k * cstep] = db[k];
        }
    }
}

// ---- forward, maps --------------------------------------------------------------------------
template <typename T, int V, int K, bool STR>
__global__ void __launch_bounds__(32 * MAX_WARPS, K * Vec<T, V>::WORDS <= 16 ? 2 : 1) ln_fwd_map(const T* x, const float* __restrict__ gamma,
                                                                                                 const float* __restrict__ beta, T* y,
                                                                                                 float* __restrict__ mean, float* __restrict__ rstd,
                                                                                                 MapGeom q, float eps)
{
    extern __shared__ float sm[];
    const Place<V, STR> w(q);
    const int item = blockIdx.x / q.cl, crank = blockIdx.x - item * q.cl;
    const int n = item / q.tiles;
    const size_t p = (size_t)(item - n * q.tiles) * ((size_t)V << (q.segl_log2 + q.pw_log2)) + w.first;
    const int nv = w.valid(p, q.P);
    const int c = crank * q.Cs + w.g, left = min(q.C, crank * q.Cs + q.Cs) - c;      // this thread's first channel, and how many there are from it on
    const int nk = (left + (1 << q.groups_log2) - 1) >> q.groups_log2;
    const size_t at = ((size_t)n * q.C + c) * q.P + p, step = q.P << q.groups_log2;

    Vec<T, V> v[K];
    const T* px = x + at;
#pragma unroll
    for (int k = 0; k < K; ++k, px += step) {
        v[k].zero();
        if (k < nk) load_at<T, V, STR>(v[k], px, w.stride, nv);
    }
    F<V> m, r;
    statistics<T, V, K, false>(v, nk, eps, sm, q, w.l, m, r);
    if (q.cl > 1) cluster_sync();       // nobody leaves while a neighbour reads
    if (w.g == 0 && crank == 0) {
        if (mean) store_floats_at<V, STR>(mean + (size_t)n * q.P + p, w.stride, nv, m.f);
        if (rstd) store_floats_at<V, STR>(rstd + (size_t)n * q.P + p, w.stride, nv, r.f);
    }
    if (STR || nv) normalise<T, V, K, STR, false>(v, nk, m, r, gamma ? gamma + c : nullptr, beta ? beta + c : nullptr, 1 << q.groups_log2, y + at, step, w.stride, nv);
}

// ---- backward, maps -------------------------------------------------------------------------
// Persistent: a thread keeps its channels from tile to tile, so the sums of the parameters' gradients stay in its registers; at the
// end each cluster writes one row of partial sums and ln_reduce adds the rows in a fixed order.
template <typename T, int V, int K, bool STR>
__global__ void __launch_bounds__(32 * MAX_WARPS, K * Vec<T, V>::WORDS <= 8 ? 2 : 1) ln_bwd_map(const T* dy, const T* x, const float* __restrict__ gamma,
                                                                                                const float* __restrict__ mean,
                                                                                                const float* __restrict__ rstd, T* dx,
                                                                                                Partials out, MapGeom q)
{
    extern __shared__ float sm[];
    const Place<V, STR> w(q);
    const int cid = blockIdx.x / q.cl, clusters = gridDim.x / q.cl, crank = blockIdx.x - cid * q.cl;
    const int c = crank * q.Cs + w.g, left = min(q.C, crank * q.Cs + q.Cs) - c;
    const int nk = (left + (1 << q.groups_log2) - 1) >> q.groups_log2, cstep = 1 << q.groups_log2;
    const size_t step = q.P << q.groups_log2;
    const float inv_C = 1.0f / (float)q.C;
    const float* pg = gamma ? gamma + c : nullptr;

    float dg[K], db[K];
#pragma unroll
    for (int k = 0; k < K; ++k) { dg[k] = 0.0f; db[k] = 0.0f; }
    int buf = 0;
    for (int item = cid; item < q.items; item += clusters, buf ^= 1) {
        const int n = item / q.tiles;
        const size_t p = (size_t)(item - n * q.tiles) * ((size_t)V << (q.segl_log2 + q.pw_log2)) + w.first;
        const int nv = w.valid(p, q.P);
        const size_t at = ((size_t)n * q.C + c) * q.P + p;
        Vec<T, V> vx[K], vd[K];
        const T *px = x + at, *pd = dy + at;
#pragma unroll
        for (int k = 0; k < K; ++k, px += step, pd += step) {
            vx[k].zero(); vd[k].zero();
            if (k < nk) { load_at<T, V, STR>(vx[k], px, w.stride, nv); load_at<T, V, STR>(vd[k], pd, w.stride, nv); }
        }
        F<V> neg(0.0f), r(0.0f), s[2];    // s: sums of g and of g xh
        load_floats_at<V, STR>(mean + (size_t)n * q.P + p, w.stride, nv, neg.f);
        load_floats_at<V, STR>(rstd + (size_t)n * q.P + p, w.stride, nv, r.f);
        neg = -neg;
        gradient_sums<T, V, K, false>(vx, vd, nk, neg, r, pg, cstep, s, dg, db);
        forget<T, V, K>(vx);
        forget<T, V, K>(vd);
        tile_sum<V, 2>(s, sm, q, w.l, buf);
        if (STR || nv) gradient<T, V, K, STR, false>(vx, vd, nk, neg, r, pg, cstep, s, inv_C, dx + at, step, w.stride, nv);
    }
    if (q.cl > 1) cluster_sync();       // nobody leaves while a neighbour reads
    pdl_launch();
    const int wp = (threadIdx.x >> 5) & ((1 << q.pw_log2) - 1);
    store_partials<K>(dg, db, nk, 1 << q.segl_log2, cstep, out, q.C, (cid << q.pw_log2) + wp, c);
}

// ---- large maps: tiles through a ring in shared memory -----------------------------------------
// The same arithmetic on tiles that TMA copies in and out, so that the copies of the next tiles and of the last one run while a tile is
// worked on, whatever the registers hold.  A stage is [rows][TP] of x (backward: then the same of dy), rows = channels in boxes of at most 256; the
// result takes x's place.  Persistent CTAs; thread 0 issues the copies.  A stage is loaded again when its store has read it, which thread 0
// waits for one tile later.
constexpr int STAGES = 3;
struct RingGeom {
    MapGeom q;
    int boxes, box_rows, tp;            // rows of a stage = boxes * box_rows, positions of a tile
    uint32_t half;                      // bytes of x's part of a stage
};
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, uint32_t src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];"
                 ::"l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(z), "r"(src) : "memory");
}
__device__ __forceinline__ void store_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void store_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

template <typename T, int V, int K, bool BWD, bool FULL_K>
__global__ void __launch_bounds__(32 * MAX_WARPS, 1) ln_ring(const __grid_constant__ CUtensorMap tmx, const __grid_constant__ CUtensorMap tmd,
                                                             const __grid_constant__ CUtensorMap tmo, const float* __restrict__ gamma,
                                                             const float* __restrict__ beta, float* __restrict__ mean, float* __restrict__ rstd,
                                                             Partials out, RingGeom h, float eps, int* __restrict__ status)
{
    extern __shared__ uint8_t ring_raw[];
    __shared__ uint64_t full[STAGES];
    const MapGeom& q = h.q;
    uint8_t* ring = ring_raw + ((128u - (tc::smem_u32(ring_raw) & 127u)) & 127u);
    const uint32_t stage_bytes = h.half * (BWD ? 2 : 1);
    float* sm = reinterpret_cast<float*>(ring + (size_t)STAGES * stage_bytes);
    float* par = sm + tile_floats(q, h.tp);                             // gamma [C], beta [C]
    for (int c = threadIdx.x; c < q.C; c += 32 * q.warps) {
        par[c] = gamma ? gamma[c] : 1.0f;
        if (!BWD) par[q.C + c] = beta ? beta[c] : 0.0f;
    }
    const int segl = 1 << q.segl_log2;
    const int l = threadIdx.x & (segl - 1), g = threadIdx.x >> q.segl_log2;
    const int cstep = 1 << q.groups_log2, left = q.C - g, nk = (left + cstep - 1) >> q.groups_log2;
    const size_t step = (size_t)h.tp << q.groups_log2;
    const float inv_C = 1.0f / (float)q.C;

    auto issue = [&](int i) {           // (thread 0) tile i of this CTA into its stage
        const long long item = (long long)blockIdx.x + (long long)i * gridDim.x;
        if (item >= q.items) return;
        const int n = (int)item / q.tiles, p = ((int)item - n * q.tiles) * h.tp;
        const uint32_t dst = tc::smem_u32(ring) + (uint32_t)(i % STAGES) * stage_bytes, bar = tc::smem_u32(&full[i % STAGES]);
        tc::mbar_expect_tx(bar, stage_bytes);
        const uint32_t box = (uint32_t)(h.box_rows * h.tp * (int)sizeof(T));
        for (int b = 0; b < h.boxes; ++b) {
            tma_load_3d(dst + b * box, &tmx, p, b * h.box_rows, n, bar);
            if (BWD) tma_load_3d(dst + h.half + b * box, &tmd, p, b * h.box_rows, n, bar);
        }
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) tc::mbar_init(tc::smem_u32(&full[s]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int i = 0; i < STAGES; ++i) issue(i);
    }
    __syncthreads();

    float dg[BWD ? K : 1], db[BWD ? K : 1];
#pragma unroll
    for (int k = 0; k < (BWD ? K : 1); ++k) { dg[k] = 0.0f; db[k] = 0.0f; }
    bool ok = true;
    int i = 0;
    for (int item = blockIdx.x; item < q.items; item += gridDim.x, ++i) {
        const int n = item / q.tiles;
        const size_t p = (size_t)(item - n * q.tiles) * h.tp + (size_t)l * V;
        const bool in = p < q.P;
        const size_t at = (size_t)n * q.P + p;
        F<V> m(0.0f), r(0.0f);
        if (BWD && in) { load_floats<V>(mean + at, m.f); load_floats<V>(rstd + at, r.f); }
        ok = tc::mbar_wait(tc::smem_u32(&full[i % STAGES]), (uint32_t)(i / STAGES) & 1u);
        if (__syncthreads_or(!ok)) { ok = false; break; }
        T* tile = reinterpret_cast<T*>(ring + (size_t)(i % STAGES) * stage_bytes) + (size_t)g * h.tp + l * V;
        Vec<T, V> v[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k].zero();
            if (FULL_K || k < nk) v[k].load(tile + k * step);
        }
        if constexpr (BWD) {
            Vec<T, V> vd[K];
            const T* td = tile + h.half / sizeof(T);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                vd[k].zero();
                if (FULL_K || k < nk) vd[k].load(td + k * step);
            }
            F<V> s[2];
            const F<V> neg = -m;
            const float* pg = par + g;
            gradient_sums<T, V, K, FULL_K>(v, vd, nk, neg, r, pg, cstep, s, dg, db);
            forget<T, V, K>(v);
            forget<T, V, K>(vd);
            tile_sum<V, 2>(s, sm, q, l, i & 1);
            gradient<T, V, K, false, FULL_K>(v, vd, nk, neg, r, pg, cstep, s, inv_C, tile, step, 0, V);
        } else {
            statistics<T, V, K, FULL_K>(v, nk, eps, sm, q, l, m, r);
            if (g == 0 && in) {
                if (mean) store_floats<V>(mean + at, m.f);
                if (rstd) store_floats<V>(rstd + at, r.f);
            }
            normalise<T, V, K, false, FULL_K>(v, nk, m, r, par + g, par + q.C + g, cstep, tile, step, 0, V);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
            const uint32_t src = tc::smem_u32(ring) + (uint32_t)(i % STAGES) * stage_bytes, box = (uint32_t)(h.box_rows * h.tp * (int)sizeof(T));
            const int p0 = (item - n * q.tiles) * h.tp;
            for (int b = 0; b < h.boxes; ++b) tma_store_3d(&tmo, src + b * box, p0, b * h.box_rows, n);
            store_commit();
            store_wait_read<1>();       // the store of the tile before has left its stage
            if (i >= 1) issue(i - 1 + STAGES);
        }
    }
    if (!ok) {
        // let the copies that are under way land before the shared memory goes away
        if (threadIdx.x == 0) atomicExch(status, (int)WCC_ERR_TIMEOUT);
        for (int w = 0; w < 2000; ++w) __nanosleep(1000);
        __syncthreads();
    }
    if (threadIdx.x == 0) store_wait_all();
    if constexpr (BWD) {
        pdl_launch();
        store_partials<K>(dg, db, nk, segl, cstep, out, q.C, blockIdx.x, g);
    }
}

// The gradients of the parameters from the sums of a CTA's warps, [warp][2][C] in shared memory: a thread a column, the warps in order.
__device__ __forceinline__ void add_warps(const float* acc, int warps, int C, const Partials& out, int row)
{
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * C; i += NT) {
        float a = acc[i];
        for (int w = 1; w < warps; ++w) a += acc[(size_t)w * 2 * C + i];
        float* o = i < C ? out.g : out.b;
        if (o) o[row * out.pitch + (i < C ? i : i - C)] = a;
    }
}

// ---- rows (one position an image) -------------------------------------------------------------
// TR threads take a row of C contiguous channels, vector j of thread t holds channels (t + j TR) V and on.
template <int TR>
__device__ __forceinline__ float2 row_sum(float2 a, float2* sm)
{
#pragma unroll
    for (int o = 1; o < (TR < 32 ? TR : 32); o <<= 1) { a.x += __shfl_xor_sync(FULL, a.x, o); a.y += __shfl_xor_sync(FULL, a.y, o); }
    if (TR > 32) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = a;
        __syncthreads();
        a = sm[0];
#pragma unroll
        for (int w = 1; w < WARPS; ++w) { a.x += sm[w].x; a.y += sm[w].y; }
    }
    return a;
}

template <typename T, int V, int K, int TR>
__global__ void __launch_bounds__(NT) ln_fwd_rows(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                                                  float* __restrict__ mean_out, float* __restrict__ rstd_out, int N, int C, float eps)
{
    __shared__ float2 sm[WARPS];
    const int t = threadIdx.x % TR;
    const float inv_C = 1.0f / (float)C;
    const long long row = (long long)blockIdx.x * (NT / TR) + threadIdx.x / TR;
    const bool in = row < N;
    const T* px = x + (size_t)(in ? row : 0) * C;
    Vec<T, V> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k].zero();
        const int c = (t + k * TR) * V;
        if (in && c < C) v[k].load(px + c);
    }
    // mean relative to the row's first channel, then the squared deviations: two passes over registers
    const float x0 = in ? (sizeof(T) == 4 ? *reinterpret_cast<const float*>(px) : __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(px) << 16)) : 0.0f;
    float2 a = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if ((t + k * TR) * V < C) {
#pragma unroll
            for (int i = 0; i < V; ++i) a.x += v[k].get(i) - x0;
        }
    a = row_sum<TR>(a, sm);
    const float m = fmaf(a.x, inv_C, x0);
    a = make_float2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < K; ++k)
        if ((t + k * TR) * V < C) {
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[k].get(i) - m; a.y = fmaf(d, d, a.y); }
        }
    a = row_sum<TR>(a, sm);
    const float r = 1.0f / sqrtf(fmaf(a.y, inv_C, eps));
    if (!in) return;
    if (t == 0) {
        if (mean_out) mean_out[row] = m;
        if (rstd_out) rstd_out[row] = r;
    }
    T* py = y + (size_t)row * C;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (t + k * TR) * V;
        if (c < C) {
            float f[V], ga[V], be[V];
#pragma unroll
            for (int i = 0; i < V; ++i) { ga[i] = 1.0f; be[i] = 0.0f; }
            if (gamma) load_floats<V>(gamma + c, ga);
            if (beta) load_floats<V>(beta + c, be);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = fmaf((v[k].get(i) - m) * r, ga[i], be[i]);
            v[k].set(f);
            v[k].store(py + c);
        }
    }
}

template <typename T, int V, int K, int TR>
__global__ void __launch_bounds__(NT) ln_bwd_rows(const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                  const float* __restrict__ rstd, T* dx, Partials out, int N, int C)
{
    extern __shared__ __align__(16) float acc_sm[];      // TR < 256: [warp][2][C], the sums of the CTA's warps
    __shared__ float2 sm[WARPS];
    const int t = threadIdx.x % TR, sub = threadIdx.x / TR;
    constexpr int R = NT / TR;
    const float inv_C = 1.0f / (float)C;
    float dg[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) { dg[k][i] = 0.0f; db[k][i] = 0.0f; }

    for (long long row0 = (long long)blockIdx.x * R; row0 < N; row0 += (long long)gridDim.x * R) {
        const long long row = row0 + sub;
        const bool in = row < N;
        const size_t at = (size_t)(in ? row : 0) * C;
        Vec<T, V> vx[K], vd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            vx[k].zero(); vd[k].zero();
            const int c = (t + k * TR) * V;
            if (in && c < C) { vx[k].load(x + at + c); vd[k].load(dy + at + c); }
        }
        const float mu = in ? mean[row] : 0.0f, r = in ? rstd[row] : 0.0f;
        float2 a = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (t + k * TR) * V;
            if (c < C) {
                float ga[V];
#pragma unroll
                for (int i = 0; i < V; ++i) ga[i] = 1.0f;
                if (gamma) load_floats<V>(gamma + c, ga);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = vd[k].get(i), xh = (vx[k].get(i) - mu) * r, gg = d * ga[i];
                    dg[k][i] = fmaf(d, xh, dg[k][i]);
                    db[k][i] += d;
                    a.x += gg;
                    a.y = fmaf(gg, xh, a.y);
                }
            }
        }
        a = row_sum<TR>(a, sm);
        a.x *= inv_C; a.y *= inv_C;
        if (in) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (t + k * TR) * V;
                if (c < C) {
                    float ga[V], f[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) ga[i] = 1.0f;
                    if (gamma) load_floats<V>(gamma + c, ga);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xh = (vx[k].get(i) - mu) * r;
                        f[i] = r * (fmaf(vd[k].get(i), ga[i], -a.x) - xh * a.y);
                    }
                    vx[k].set(f);
                    vx[k].store(dx + at + c);
                }
            }
        }
    }
    pdl_launch();
    if (!out.g && !out.b) return;
    // the row groups of a warp add up, then the warps: a fixed order
#pragma unroll
    for (int o = TR; o < 32; o <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                dg[k][i] += __shfl_xor_sync(FULL, dg[k][i], o);
                db[k][i] += __shfl_xor_sync(FULL, db[k][i], o);
            }
    if constexpr (TR < NT) {
        const int per = 32 / TR, warp = (int)threadIdx.x >> 5;         // rows of a warp at once
        const long long left = N - (long long)blockIdx.x * R;
        const int warps = (int)min((long long)WARPS, (left + per - 1) / per);      // those that had one
        if ((int)(threadIdx.x & 31) < TR && warp < warps) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (t + k * TR) * V;
                if (c < C) {
                    store_floats<V>(acc_sm + (size_t)warp * 2 * C + c, dg[k]);
                    store_floats<V>(acc_sm + (size_t)warp * 2 * C + C + c, db[k]);
                }
            }
        }
        add_warps(acc_sm, warps, C, out, blockIdx.x);
    } else {
        const size_t row = blockIdx.x * out.pitch;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (t + k * TR) * V;
            if (c < C) {
                if (out.g) store_floats<V>(out.g + row + c, dg[k]);
                if (out.b) store_floats<V>(out.b + row + c, db[k]);
            }
        }
    }
}

// ---- many rows --------------------------------------------------------------------------------
// A warp takes a row after the other and copies the next ones to its own ring in shared memory meanwhile; a lane copies what it reads itself,
// so nothing waits but the lane.  gamma and beta stay in shared memory: fetched for every row they would be more bytes than the row
// (8192 rows of 1024 bf16: forward 12.8 us, backward 34.8 us that way).
constexpr int ROW_STAGES = 3;
template <typename T, int K>
struct RowFeed {
    static constexpr int V = 16 / (int)sizeof(T), STAGE = K * 512;
    uint32_t base;
    __device__ __forceinline__ explicit RowFeed(const void* warp_smem) : base((uint32_t)__cvta_generic_to_shared(warp_smem) + 16u * (threadIdx.x & 31)) {}
    // row -> stage s; a row that does not exist leaves the stage as it is
    __device__ __forceinline__ void issue(const T* row, int C, bool have, int s)
    {
        const int lane = threadIdx.x & 31;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (have && (lane + 32 * k) * V < C)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(base + (uint32_t)(s * STAGE + k * 512)), "l"(row + (lane + 32 * k) * V) : "memory");
    }
    static __device__ __forceinline__ void commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
    static __device__ __forceinline__ void wait() { asm volatile("cp.async.wait_group %0;" ::"n"(ROW_STAGES - 2) : "memory"); }
    static __device__ __forceinline__ void drain() { asm volatile("cp.async.wait_group 0;" ::: "memory"); }
    __device__ __forceinline__ void take(int s, int k, Vec<T, V>& v) const
    {
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.w[0]), "=r"(v.w[1]), "=r"(v.w[2]), "=r"(v.w[3]) : "r"(base + (uint32_t)(s * STAGE + k * 512)));
    }
};
template <int NS> __device__ __forceinline__ void warp_sums(float (&a)[NS])
{
#pragma unroll
    for (int o = 16; o; o >>= 1)
#pragma unroll
        for (int i = 0; i < NS; ++i) a[i] += __shfl_xor_sync(FULL, a[i], o);
}
template <int V> __device__ __forceinline__ float total(const F<V>& f)
{
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) s += f.f[i];
    return s;
}

template <typename T, int K>
__global__ void __launch_bounds__(NT) ln_fwd_feed(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                                                  float* __restrict__ mean, float* __restrict__ rstd, int N, int C, float eps)
{
    extern __shared__ __align__(16) float feed_sm[];
    constexpr int V = RowFeed<T, K>::V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float *sg = feed_sm, *sb = feed_sm + C;
    for (int c = threadIdx.x; c < C; c += NT) { sg[c] = gamma ? gamma[c] : 1.0f; sb[c] = beta ? beta[c] : 0.0f; }
    const RowFeed<T, K> proto(reinterpret_cast<char*>(feed_sm + 2 * C) + (size_t)warp * ROW_STAGES * RowFeed<T, K>::STAGE);
    RowFeed<T, K> feed = proto;
    const long long step = (long long)gridDim.x * WARPS;
    long long row = (long long)blockIdx.x * WARPS + warp;
#pragma unroll
    for (int i = 0; i < ROW_STAGES - 1; ++i) { feed.issue(x + (row + i * step) * C, C, row + i * step < N, i); feed.commit(); }
    __syncthreads();
    const float inv_C = 1.0f / (float)C;
    for (int s = 0; row < N; row += step, s = s + 1 == ROW_STAGES ? 0 : s + 1) {
        feed.wait();
        const long long next = row + (ROW_STAGES - 1) * step;
        feed.issue(x + next * C, C, next < N, s == 0 ? ROW_STAGES - 1 : s - 1);
        feed.commit();
        Vec<T, V> v[K];
        F<V> a(0.0f), b(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            v[k].zero();
            if ((lane + 32 * k) * V < C) feed.take(s, k, v[k]);
            a = a + floats(v[k]);
        }
        float one[1] = {total(a)};
        warp_sums<1>(one);
        float m = one[0] * inv_C;
        a = F<V>(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if ((lane + 32 * k) * V < C) {
                const F<V> d = floats(v[k]) + F<V>(-m);
                a = a + d;
                b = fma(d, d, b);
            }
        float two[2] = {total(a), total(b)};
        warp_sums<2>(two);
        const float e = two[0] * inv_C, var = fmaf(two[1], inv_C, -e * e), r = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
        m += e;
        if (lane == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = r;
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + 32 * k) * V;
            if (c < C) {
                F<V> ga, be;
                load_floats<V>(sg + c, ga.f);
                load_floats<V>(sb + c, be.f);
                v[k].set(fma((floats(v[k]) + F<V>(-m)) * F<V>(r), ga, be).f);
                v[k].store(y + row * C + c);
            }
        }
    }
    RowFeed<T, K>::drain();
}

template <typename T, int K>
__global__ void __launch_bounds__(NT, 2) ln_bwd_feed(const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                     const float* __restrict__ rstd, T* dx, Partials out, int N, int C)
{
    extern __shared__ __align__(16) float feed_sm[];
    constexpr int V = RowFeed<T, K>::V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float* sg = feed_sm;
    for (int c = threadIdx.x; c < C; c += NT) sg[c] = gamma ? gamma[c] : 1.0f;
    char* mine = reinterpret_cast<char*>(feed_sm + C) + (size_t)warp * 2 * ROW_STAGES * RowFeed<T, K>::STAGE;
    RowFeed<T, K> fx(mine), fd(mine + ROW_STAGES * RowFeed<T, K>::STAGE);
    const long long step = (long long)gridDim.x * WARPS;
    long long row = (long long)blockIdx.x * WARPS + warp;
#pragma unroll
    for (int i = 0; i < ROW_STAGES - 1; ++i) {
        fx.issue(x + (row + i * step) * C, C, row + i * step < N, i);
        fd.issue(dy + (row + i * step) * C, C, row + i * step < N, i);
        fx.commit();
    }
    __syncthreads();
    const float inv_C = 1.0f / (float)C;
    F<V> dg[K], db[K];
#pragma unroll
    for (int k = 0; k < K; ++k) dg[k] = db[k] = F<V>(0.0f);
    float mu = row < N ? mean[row] : 0.0f, r = row < N ? rstd[row] : 0.0f;
    for (int s = 0; row < N; row += step, s = s + 1 == ROW_STAGES ? 0 : s + 1) {
        const float mu1 = row + step < N ? mean[row + step] : 0.0f, r1 = row + step < N ? rstd[row + step] : 0.0f;
        fx.wait();
        const long long next = row + (ROW_STAGES - 1) * step;
        const int sn = s == 0 ? ROW_STAGES - 1 : s - 1;
        fx.issue(x + next * C, C, next < N, sn);
        fd.issue(dy + next * C, C, next < N, sn);
        fx.commit();
        F<V> a(0.0f), b(0.0f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + 32 * k) * V;
            if (c < C) {
                Vec<T, V> vx, vd;
                fx.take(s, k, vx);
                fd.take(s, k, vd);
                F<V> ga;
                load_floats<V>(sg + c, ga.f);
                const F<V> d = floats(vd), xh = (floats(vx) + F<V>(-mu)) * F<V>(r), g = d * ga;
                dg[k] = fma(d, xh, dg[k]);
                db[k] = db[k] + d;
                a = a + g;
                b = fma(g, xh, b);
            }
        }
        float two[2] = {total(a), total(b)};
        warp_sums<2>(two);
        const F<V> c1(-two[0] * inv_C), c2(-two[1] * inv_C);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + 32 * k) * V;
            if (c < C) {
                Vec<T, V> vx, vd;
                fx.take(s, k, vx);
                fd.take(s, k, vd);
                F<V> ga;
                load_floats<V>(sg + c, ga.f);
                const F<V> xh = (floats(vx) + F<V>(-mu)) * F<V>(r);
                vx.set((F<V>(r) * fma(xh, c2, fma(floats(vd), ga, c1))).f);
                vx.store(dx + row * C + c);
            }
        }
        mu = mu1;
        r = r1;
    }
    RowFeed<T, K>::drain();
    pdl_launch();
    if (!out.g && !out.b) return;
    // the warps' sums, in the room of the rows
    float* acc = feed_sm + C;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (lane + 32 * k) * V;
        if (c < C) {
            store_floats<V>(acc + (size_t)warp * 2 * C + c, dg[k].f);
            store_floats<V>(acc + (size_t)warp * 2 * C + C + c, db[k].f);
        }
    }
    add_warps(acc, WARPS, C, out, blockIdx.x);
}

// dgamma and dbeta from the partial rows: 32 columns a CTA, 32 threads a column, added in a fixed order.
__global__ void __launch_bounds__(1024) ln_reduce(const float* __restrict__ part, int rows, int C, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float sm[32][33];
    pdl_wait();
    const int col = blockIdx.x * 32 + threadIdx.x;
    float a = 0.0f;
    if (col < 2 * C)
        for (int r = threadIdx.y; r < rows; r += 32) a += part[(size_t)r * 2 * C + col];
    sm[threadIdx.y][threadIdx.x] = a;
    __syncthreads();
    a = sm[threadIdx.x][threadIdx.y];   // a warp has one column now
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(FULL, a, o);
    const int c = blockIdx.x * 32 + threadIdx.y;
    if (threadIdx.x == 0 && c < 2 * C) {
        if (c < C) { if (dgamma) dgamma[c] = a; }
        else if (dbeta) dbeta[c - C] = a;
    }
}

// ---- plans and launches -----------------------------------------------------------------------
struct Plan {
    bool rows;
    int es, V, K, TR;                       // TR: rows only
    bool ring, strided, feed;
    MapGeom q;
    RingGeom h;                         // ring only; h.q == q
    int ctas;                           // ring and feed: CTAs of the launch
    size_t smem;
};

// Elements of a vector
inline int vec_elems(size_t len, int es)
{
    int v = 16 / es;
    while (len % v) v >>= 1;
    return v;
}

// The ring, where rows start on 16 bytes and there are two tiles or more for every CTA that fits at once.  Tiles of 32 KB (x and dy together), twice
// that where rows of 64 bytes would be cut otherwise; 8 bytes a lane (forward on 4 x 1024 x 128 x 128 bf16, us: 4 bytes -, 8 65, 16 72; backward
// on 12 x 64 x 96 x 320 fp32 8 54, 16 53).  Without the ring these take 114 and 74.
inline bool ring_plan(Plan& p, int N, int C, size_t P, int es, bool bwd)
{
    if (P * es % 16 != 0 || P * es < 64 || C < 8) return false;
    int row = 512;                                                       // bytes of a tile's row
    const int most = 32768 >> (bwd ? 1 : 0);
    while (row > 64 && (long long)row * C > most) row /= 2;
    while (row > 64 && (size_t)row > P * es) row /= 2;
    RingGeom& h = p.h;
    h.boxes = ceil_div(C, 256);
    h.box_rows = ceil_div(ceil_div(C, h.boxes), 2) * 2;                  // boxes start on 128 bytes of shared memory
    h.tp = row / es;
    h.half = (uint32_t)(h.boxes * h.box_rows * row);
    if (h.half > 65536u >> (bwd ? 1 : 0)) return false;
    const size_t tiles = (P + h.tp - 1) / h.tp;
    if (tiles * N > 0x7FFFFFFFull) return false;
    const int vb = std::min(row / 4, 8);
    p.V = vb / es;
    int lg = 0;
    while ((vb << lg) < row && lg < 5) ++lg;
    if ((vb << lg) != row) { p.V *= 2; if (p.V * es > 16) return false; }
    int warps = 4;
    const int kmax = (bwd ? 16 : 32) / (p.V * es / 4);
    while (warps < MAX_WARPS && ceil_div(C, warps << (5 - lg)) > kmax) warps *= 2;
    const int k = ceil_div(C, warps << (5 - lg));
    if (k > kmax) return false;
    p.K = k <= 2 ? 2 : k <= 4 ? 4 : k <= 8 ? 8 : 16;
    MapGeom& q = p.q;
    q.P = P; q.C = C; q.Cs = C; q.cl = 1; q.segl_log2 = lg; q.warps = warps;
    q.groups_log2 = 5 - lg + (warps == 4 ? 2 : warps == 8 ? 3 : 4);
    q.tiles = (int)tiles;
    q.items = N * q.tiles;
    h.q = q;
    p.smem = 128 + (size_t)STAGES * h.half * (bwd ? 2 : 1) + (size_t)tile_floats(q, h.tp) * 4 + (size_t)(bwd ? 1 : 2) * C * 4;
    const int per_sm = std::max(1, std::min((int)(225 * 1024 / (p.smem + 1200)), 512 / (32 * warps)));
    p.ctas = std::min(q.items, per_sm * B200_SMS);
    if (q.items < 2 * p.ctas) return false;
    p.ring = true;
    return true;
}

// Registers: a thread of the forward pass holds K vectors, one of the backward pass 2 K (and 2 K sums): at most 32 and 16 words of a map, and
// half of that while more warps can share the channels.
inline Plan plan_of(int N, int C, size_t P, int es, bool bwd)
{
    Plan p{};
    p.es = es;
    if (P == 1) {
        p.rows = true;
        p.V = C % (16 / es) == 0 ? 16 / es : 1;
        const int caps[5][2] = {{8, 8}, {8, 32}, {32, 32}, {256, 8}, {256, 32}};      // threads a row, channels a thread
        int i = 0;
        while (caps[i][0] * caps[i][1] < C) ++i;                                         // 256 x 32 = WCC_MAX_CHANNELS
        // a warp a row: forward from four rows a warp on, where gamma and beta have been paid for
        const int v16 = 16 / es, k = ceil_div(C, 32 * v16);
        if (C % v16 == 0 && k <= (es == 2 ? 4 : 8) && N >= (bwd ? 1 : 4) * WARPS * B200_SMS) {
            p.feed = true;
            p.K = k <= 1 ? 1 : k <= 2 ? 2 : k <= 4 ? 4 : 8;
            p.smem = (size_t)(bwd ? 1 : 2) * C * 4 + (size_t)WARPS * ROW_STAGES * p.K * 512 * (bwd ? 2 : 1);
            if (bwd) p.smem = std::max(p.smem, (size_t)(1 + 2 * WARPS) * C * 4);
            const int per_sm = bwd ? 2 : 4;
            p.ctas = std::min(ceil_div(N, WARPS), B200_SMS * std::min(per_sm, (int)(228 * 1024 / (p.smem + 1024))));
            return p;
        }
        p.TR = caps[i][0];
        p.K = caps[i][1] / p.V;
        p.smem = bwd && p.TR < NT ? (size_t)WARPS * 2 * C * 4 : 0;
        return p;
    }
    if (ring_plan(p, N, C, P, es, bwd)) return p;
    // single loads where rows start on no vector (a vector of two bf16 is hardly better)
    p.V = vec_elems(P, es);
    p.strided = p.V * es < (es == 2 ? 4 : 8);
    if (p.strided) p.V = 8 / es;
    const int words = p.V * es / 4, kmax = (bwd ? 16 : 32) / words, kgood = (bwd ? 8 : 16) / words;
    int lg = 0;
    while (lg < 5 && ((size_t)p.V << lg) < P) ++lg;
    auto tiles_of = [&](int s) { return (P + ((size_t)p.V << s) - 1) / ((size_t)p.V << s); };
    auto K_of = [&](int s, int w, int c) { return ceil_div(c, w << (5 - s)); };
    const int sector = [&] { int s = 0; while ((p.strided ? es << s : (p.V << s) * es) < 32 && s < lg) ++s; return s; }();
    int cl = 1;
    while (lg > sector && K_of(lg, MAX_WARPS, C) > kmax) --lg;
    while (lg > sector && (size_t)N * tiles_of(lg) < 2 * B200_SMS) --lg;
    while (K_of(lg, MAX_WARPS, ceil_div(C, cl)) > kmax && cl < 8) cl *= 2;
    while (K_of(lg, MAX_WARPS, ceil_div(C, cl)) > kmax) --lg;
    int warps = 1;
    while (warps < MAX_WARPS && K_of(lg, warps, ceil_div(C, cl)) > kgood) warps *= 2;
    p.q.P = P; p.q.C = C; p.q.cl = cl; p.q.Cs = ceil_div(C, cl); p.q.segl_log2 = lg;
    p.q.groups_log2 = 5 - lg;
    for (int w = 1; w < warps; w *= 2) ++p.q.groups_log2;
    const int k = K_of(lg, warps, p.q.Cs);
    p.K = k <= 2 ? 2 : k <= 4 ? 4 : k <= 8 ? 8 : k <= 16 ? 16 : 32;
    // few channels: warps side by side
    while (lg == 5 && warps < 8 && (size_t)N * tiles_of(lg + p.q.pw_log2 + 1) >= 2 * B200_SMS) { ++p.q.pw_log2; warps *= 2; }
    while (warps < 4 && lg < 5) { warps *= 2; ++p.q.groups_log2; }
    p.q.warps = warps;
    p.q.tiles = (int)tiles_of(lg + p.q.pw_log2);
    p.q.items = N * p.q.tiles;
    lg += p.q.pw_log2;
    const int tpos = p.V << lg;
    p.smem = (size_t)tile_floats(p.q, tpos) * 4;
    return p;
}

template <typename T, int V, int K, bool STR>
static wcc_status fwd_map(const Plan& p, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, float eps, cudaStream_t st)
{
    return launch_overlapped(ln_fwd_map<T, V, K, STR>, dim3((unsigned)(p.q.items * p.q.cl)), dim3((unsigned)(32 * p.q.warps)), p.smem, st, false, p.q.cl,
                             static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, p.q, eps);
}
template <typename T, int V, int K, bool STR>
static wcc_status bwd_map(const Plan& p, int ctas, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                          const Partials& part, cudaStream_t st)
{
    return launch_overlapped(ln_bwd_map<T, V, K, STR>, dim3((unsigned)ctas), dim3((unsigned)(32 * p.q.warps)), p.smem, st, false, p.q.cl, static_cast<const T*>(dy),
                             static_cast<const T*>(x), gamma, mean, rstd, static_cast<T*>(dx), part, p.q);
}
template <typename T, int V, int K, int TR>
static wcc_status fwd_rows(const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, int N, int C, float eps, cudaStream_t st)
{
    return launch_overlapped(ln_fwd_rows<T, V, K, TR>, dim3((unsigned)ceil_div(N, NT / TR)), dim3(NT), 0, st, false, 1, static_cast<const T*>(x), gamma,
                             beta, static_cast<T*>(y), mean, rstd, N, C, eps);
}
template <typename T, int V, int K, int TR>
static wcc_status bwd_rows(const Plan& p, int ctas, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                           const Partials& part, int N, int C, cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK || (s = allow_smem<ln_bwd_rows<T, V, K, TR>>(di.dev, (int)p.smem)) != WCC_OK) return s;
    return launch_overlapped(ln_bwd_rows<T, V, K, TR>, dim3((unsigned)ctas), dim3(NT), p.smem, st, false, 1, static_cast<const T*>(dy),
                             static_cast<const T*>(x), gamma, mean, rstd, static_cast<T*>(dx), part, N, C);
}

inline bool ring_map(CUtensorMap* tm, const void* ptr, int es, const Plan& p, int N)
{
    tc::EncodeTiledFn fn = tc::encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)p.q.P, (cuuint64_t)p.q.C, (cuuint64_t)N};
    cuuint64_t strides[2] = {(cuuint64_t)p.q.P * es, (cuuint64_t)p.q.P * p.q.C * es};
    cuuint32_t box[3] = {(cuuint32_t)p.h.tp, (cuuint32_t)p.h.box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(tm, es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, const_cast<void*>(ptr), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <typename T, int V, int K, bool BWD, bool FULL_K>
static wcc_status run_ring(const Plan& p, const void* x, const void* dy, void* out, const float* gamma, const float* beta, float* mean, float* rstd,
                           const Partials& part, int N, float eps, cudaStream_t st)
{
    CUtensorMap tx, td, to;
    if (!ring_map(&tx, x, sizeof(T), p, N) || !ring_map(&td, BWD ? dy : x, sizeof(T), p, N) || !ring_map(&to, out, sizeof(T), p, N)) return WCC_ERR_CUDA;
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK) return s;
    if ((s = allow_smem<ln_ring<T, V, K, BWD, FULL_K>>(di.dev, (int)p.smem)) != WCC_OK) return s;
    return launch_overlapped(ln_ring<T, V, K, BWD, FULL_K>, dim3((unsigned)p.ctas), dim3((unsigned)(32 * p.q.warps)), p.smem, st, false, 1, tx, td, to, gamma, beta,
                             mean, rstd, part, p.h, eps, di.status);
}
template <typename T, bool BWD>
static wcc_status ring(const Plan& p, const void* x, const void* dy, void* out, const float* gamma, const float* beta, float* mean, float* rstd,
                       const Partials& part, int N, float eps, cudaStream_t st)
{
    constexpr int V4 = 4 / (int)sizeof(T);
#define WCC_LN_RING(V_, K_) \
    if (p.V == (V_) && p.K == (K_))                                                                                              \
        return p.q.C == (K_) << p.q.groups_log2 ? run_ring<T, V_, K_, BWD, true>(p, x, dy, out, gamma, beta, mean, rstd, part, N, eps, st) \
                                                : run_ring<T, V_, K_, BWD, false>(p, x, dy, out, gamma, beta, mean, rstd, part, N, eps, st);
    WCC_LN_RING(2 * V4, 2) WCC_LN_RING(2 * V4, 4) WCC_LN_RING(2 * V4, 8) WCC_LN_RING(4 * V4, 2) WCC_LN_RING(4 * V4, 4)
    if constexpr (!BWD) { WCC_LN_RING(2 * V4, 16) WCC_LN_RING(4 * V4, 8) }
#undef WCC_LN_RING
    return WCC_ERR_SHAPE;
}

// CTAs of the backward pass = rows of partial sums (times the cluster): as many as run at once.
inline int bwd_ctas(const Plan& p, int N)
{
    if (p.ring || p.feed) return p.ctas;
    if (p.rows) {
        const long long want = ((long long)N * p.TR + NT - 1) / NT;
        return (int)(want < 2 * B200_SMS ? want : 2 * B200_SMS);
    }
    const int words = p.K * std::max(1, p.V * p.es / 4), room = B200_SMS * std::min(16, (words <= 8 ? 1024 : 512) / (32 * p.q.warps)) / p.q.cl;
    return (p.q.items < room ? p.q.items : room) * p.q.cl;
}
// Rows of partial sums.
inline int bwd_rows(const Plan& p, int N) { return p.rows || p.ring ? bwd_ctas(p, N) : (bwd_ctas(p, N) / p.q.cl) << p.q.pw_log2; }
inline size_t bwd_ws_bytes(const Plan& p, int N, int C) { return align_up((size_t)bwd_rows(p, N) * 2 * C * 4, 256); }

template <typename T, int K>
static wcc_status fwd_feed(const Plan& p, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, int N, int C, float eps,
                           cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK || (s = allow_smem<ln_fwd_feed<T, K>>(di.dev, (int)p.smem)) != WCC_OK) return s;
    return launch_overlapped(ln_fwd_feed<T, K>, dim3((unsigned)p.ctas), dim3(NT), p.smem, st, false, 1, static_cast<const T*>(x), gamma, beta,
                             static_cast<T*>(y), mean, rstd, N, C, eps);
}
template <typename T, int K>
static wcc_status bwd_feed(const Plan& p, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                           const Partials& part, int N, int C, cudaStream_t st)
{
    DeviceInfo di;
    wcc_status s = device_info(di);
    if (s != WCC_OK || (s = allow_smem<ln_bwd_feed<T, K>>(di.dev, (int)p.smem)) != WCC_OK) return s;
    return launch_overlapped(ln_bwd_feed<T, K>, dim3((unsigned)p.ctas), dim3(NT), p.smem, st, false, 1, static_cast<const T*>(dy),
                             static_cast<const T*>(x), gamma, mean, rstd, static_cast<T*>(dx), part, N, C);
}

template <typename T>
static wcc_status forward(const Plan& p, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, int N, int C, float eps,
                          cudaStream_t st)
{
    constexpr int VM = 16 / (int)sizeof(T);
    if (p.feed) {
#define WCC_LN_FEED(K_) if (p.K == (K_)) return fwd_feed<T, K_>(p, x, gamma, beta, y, mean, rstd, N, C, eps, st);
        WCC_LN_FEED(1) WCC_LN_FEED(2) WCC_LN_FEED(4)
        if constexpr (sizeof(T) == 4) { WCC_LN_FEED(8) }
#undef WCC_LN_FEED
        return WCC_ERR_SHAPE;
    }
    if (p.rows) {
#define WCC_LN_ROWS(V_, KV_, TR_) \
    if (p.V == (V_) && p.K == (KV_) / (V_) && p.TR == (TR_)) return fwd_rows<T, V_, (KV_) / (V_), TR_>(x, gamma, beta, y, mean, rstd, N, C, eps, st);
        WCC_LN_ROWS(VM, 8, 8) WCC_LN_ROWS(VM, 32, 8) WCC_LN_ROWS(VM, 32, 32) WCC_LN_ROWS(VM, 8, 256) WCC_LN_ROWS(VM, 32, 256)
        WCC_LN_ROWS(1, 8, 8) WCC_LN_ROWS(1, 32, 8) WCC_LN_ROWS(1, 32, 32) WCC_LN_ROWS(1, 8, 256) WCC_LN_ROWS(1, 32, 256)
#undef WCC_LN_ROWS
        return WCC_ERR_SHAPE;
    }
    if (p.ring) return ring<T, false>(p, x, nullptr, y, gamma, beta, mean, rstd, Partials{}, N, eps, st);
#define WCC_LN_MAP(V_, K_, STR_) \
    if (p.V == (V_) && p.K == (K_) && p.strided == (STR_)) return fwd_map<T, V_, K_, STR_>(p, x, gamma, beta, y, mean, rstd, eps, st);
    constexpr int V4 = 4 / (int)sizeof(T);
    WCC_LN_MAP(4 * V4, 2, false) WCC_LN_MAP(4 * V4, 4, false) WCC_LN_MAP(4 * V4, 8, false)
    WCC_LN_MAP(2 * V4, 2, false) WCC_LN_MAP(2 * V4, 4, false) WCC_LN_MAP(2 * V4, 8, false) WCC_LN_MAP(2 * V4, 16, false)
    WCC_LN_MAP(2 * V4, 2, true) WCC_LN_MAP(2 * V4, 4, true) WCC_LN_MAP(2 * V4, 8, true) WCC_LN_MAP(2 * V4, 16, true)
    if constexpr (V4 == 2) { WCC_LN_MAP(V4, 2, false) WCC_LN_MAP(V4, 4, false) WCC_LN_MAP(V4, 8, false) WCC_LN_MAP(V4, 16, false) WCC_LN_MAP(V4, 32, false) }
#undef WCC_LN_MAP
    return WCC_ERR_SHAPE;
}

template <typename T>
static wcc_status backward(const Plan& p, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                           const Partials& part, int N, int C, cudaStream_t st)
{
    constexpr int VM = 16 / (int)sizeof(T);
    const int ctas = bwd_ctas(p, N);
    if (p.feed) {
#define WCC_LN_FEED(K_) if (p.K == (K_)) return bwd_feed<T, K_>(p, dy, x, gamma, mean, rstd, dx, part, N, C, st);
        WCC_LN_FEED(1) WCC_LN_FEED(2) WCC_LN_FEED(4)
        if constexpr (sizeof(T) == 4) { WCC_LN_FEED(8) }
#undef WCC_LN_FEED
        return WCC_ERR_SHAPE;
    }
    if (p.rows) {
#define WCC_LN_ROWS(V_, KV_, TR_) \
    if (p.V == (V_) && p.K == (KV_) / (V_) && p.TR == (TR_)) return bwd_rows<T, V_, (KV_) / (V_), TR_>(p, ctas, dy, x, gamma, mean, rstd, dx, part, N, C, st);
        WCC_LN_ROWS(VM, 8, 8) WCC_LN_ROWS(VM, 32, 8) WCC_LN_ROWS(VM, 32, 32) WCC_LN_ROWS(VM, 8, 256) WCC_LN_ROWS(VM, 32, 256)
        WCC_LN_ROWS(1, 8, 8) WCC_LN_ROWS(1, 32, 8) WCC_LN_ROWS(1, 32, 32) WCC_LN_ROWS(1, 8, 256) WCC_LN_ROWS(1, 32, 256)
#undef WCC_LN_ROWS
        return WCC_ERR_SHAPE;
    }
    if (p.ring) return ring<T, true>(p, x, dy, dx, gamma, nullptr, const_cast<float*>(mean), const_cast<float*>(rstd), part, N, 0.0f, st);
#define WCC_LN_MAP(V_, K_, STR_) \
    if (p.V == (V_) && p.K == (K_) && p.strided == (STR_)) return bwd_map<T, V_, K_, STR_>(p, ctas, dy, x, gamma, mean, rstd, dx, part, st);
    constexpr int V4 = 4 / (int)sizeof(T);
    WCC_LN_MAP(4 * V4, 2, false) WCC_LN_MAP(4 * V4, 4, false)
    WCC_LN_MAP(2 * V4, 2, false) WCC_LN_MAP(2 * V4, 4, false) WCC_LN_MAP(2 * V4, 8, false)
    WCC_LN_MAP(2 * V4, 2, true) WCC_LN_MAP(2 * V4, 4, true) WCC_LN_MAP(2 * V4, 8, true)
    if constexpr (V4 == 2) { WCC_LN_MAP(V4, 2, false) WCC_LN_MAP(V4, 4, false) WCC_LN_MAP(V4, 8, false) WCC_LN_MAP(V4, 16, false) }
#undef WCC_LN_MAP
    return WCC_ERR_SHAPE;
}

}  // namespace ln

static wcc_status check_norm_args(int N, int C, int H, int W, wcc_dtype dt)
{
    if (N <= 0 || C <= 0 || H <= 0 || W <= 0 || C > WCC_MAX_CHANNELS) return WCC_ERR_SHAPE;
    if ((long long)H * W > (1LL << 30)) return WCC_ERR_SHAPE;
    // tiles and rows are counted in 32 bits
    if ((long long)N * H * W > (1LL << 30)) return WCC_ERR_SHAPE;
    if (dt != WCC_F32 && dt != WCC_BF16) return WCC_ERR_DTYPE;
    return WCC_OK;
}

}  // namespace wcc
