// Layer norm over the channels of a map, forward and backward.  With C channels, at every position of every image
//     mu = 1/C sum_c x,   v = 1/C sum_c (x - mu)^2,   r = (v + eps)^-1/2,   xh = (x - mu) r
//     y  = xh gamma + beta
//     g  = dy gamma,  dx = r (g - 1/C sum_c g - xh 1/C sum_c g xh),  dgamma = sum dy xh,  dbeta = sum dy  (over images, positions).
// Both directions are bound by memory: every element is read once, kept in registers until the statistics of its position are
// known, and written once.
//
// Maps: a CTA takes all channels of a tile of positions.  `segl` lanes cover the tile's positions in vectors of V elements, the
// CTA's threads form 256 / segl groups, and group g holds channels g, g + G, ...: K vectors a thread.  Wide segments load whole lines,
// narrow ones leave registers for more channels and make more tiles; ln_plan weighs them.  Channels beyond one CTA's registers go
// to a cluster whose CTAs exchange their statistics through distributed shared memory.
// Rows (one position an image): the channels are contiguous, 8, 32 or 256 threads take a row.
// Statistics are fp32 sums over registers in two rounds, the mean and then the deviations from it, so that a large common offset of the
// channels costs no digits of the variance.
#pragma once

#include <algorithm>

#include "common.cuh"

namespace wcc {
namespace ln {

constexpr int NT = 256;                 // threads of a CTA
constexpr int WARPS = NT / 32;
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
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) w[i] = 0u;
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
    int cl;                             // CTAs of a cluster
};

// Sums of a tile's NS * V values per lane over all channels: over the groups of a warp, over the warps through shared memory and over the CTAs of a
// cluster; every thread ends up with the same bits.  Calls alternate between two buffers, each of tile_floats(), so one barrier a call is
// enough: a buffer is written again only behind the barrier of the call in between.
__host__ __device__ inline int tile_parts(int segl_log2) { return (NT >> segl_log2) < WARPS ? (NT >> segl_log2) : WARPS; }
__host__ __device__ inline int tile_floats(const MapGeom& q, int tpos) { return (tile_parts(q.segl_log2) + (q.cl > 1 ? 1 : 0)) * 2 * tpos; }
template <int V, int NS>
__device__ __forceinline__ void tile_sum(float (&s)[2 * V], float* sm, const MapGeom& q, int l, int g, int buf)
{
    const int segl = 1 << q.segl_log2, tpos = segl * V, parts = tile_parts(q.segl_log2);
    for (int o = segl; o < 32; o <<= 1) {
#pragma unroll
        for (int i = 0; i < NS * V; ++i) s[i] += __shfl_xor_sync(FULL, s[i], o);
    }
    sm += buf * tile_floats(q, tpos);
    const int part = segl < 32 ? (int)threadIdx.x >> 5 : g;
    if ((threadIdx.x & 31) < segl || segl >= 32) {
#pragma unroll
        for (int i = 0; i < NS * V; ++i) sm[(part * 2 + i / V) * tpos + l * V + i % V] = s[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NS * V; ++i) s[i] = sm[(i / V) * tpos + l * V + i % V];
    for (int w = 1; w < parts; ++w) {
#pragma unroll
        for (int i = 0; i < NS * V; ++i) s[i] += sm[(w * 2 + i / V) * tpos + l * V + i % V];
    }
    if (q.cl > 1) {
        float* mine = sm + parts * 2 * tpos;
        if (g == 0) {
#pragma unroll
            for (int i = 0; i < NS * V; ++i) mine[(i / V) * tpos + l * V + i % V] = s[i];
        }
        cluster_sync();
#pragma unroll
        for (int i = 0; i < NS * V; ++i) s[i] = 0.0f;
        for (int b = 0; b < q.cl; ++b) {
            const uint32_t a = cluster_addr(mine, b);
#pragma unroll
            for (int i = 0; i < NS * V; ++i) s[i] += cluster_ld(a + 4u * ((i / V) * tpos + l * V + i % V));
        }
    }
}

// ---- forward, maps --------------------------------------------------------------------------
template <typename T, int V, int K>
__global__ void __launch_bounds__(NT) ln_fwd_map(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                                                 float* __restrict__ mean_out, float* __restrict__ rstd_out, MapGeom q, float eps)
{
    extern __shared__ float sm[];
    const int tid = threadIdx.x;
    const int segl = 1 << q.segl_log2, tpos = segl * V, G = NT >> q.segl_log2;
    const int l = tid & (segl - 1), g = tid >> q.segl_log2;
    const int item = blockIdx.x / q.cl, crank = blockIdx.x - item * q.cl;
    const int n = item / q.tiles;
    const size_t p = (size_t)(item - n * q.tiles) * tpos + (size_t)l * V;
    const bool in = p < q.P;
    const int c0 = crank * q.Cs, c1 = min(q.C, c0 + q.Cs);
    const size_t at = ((size_t)n * q.C + c0 + g) * q.P + p, step = (size_t)G * q.P;

    Vec<T, V> v[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        v[k].zero();
        if (in && c0 + g + k * G < c1) v[k].load(x + at + k * step);
    }

    // a first mean, then the sums of the deviations from it and of their squares: they correct it, and what it was off by enters the
    // variance in second order only
    const float inv_C = 1.0f / (float)q.C;
    float m[V], s[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) s[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] += v[k].get(i);              // (zeros where there is no channel)
    tile_sum<V, 1>(s, sm, q, l, g, 0);
#pragma unroll
    for (int i = 0; i < V; ++i) { m[i] = s[i] * inv_C; s[i] = 0.0f; }
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (c0 + g + k * G < c1) {
#pragma unroll
            for (int i = 0; i < V; ++i) { const float d = v[k].get(i) - m[i]; s[i] += d; s[V + i] = fmaf(d, d, s[V + i]); }
        }
    tile_sum<V, 2>(s, sm, q, l, g, 1);
    if (q.cl > 1) cluster_sync();       // nobody leaves while a neighbour reads
    float r[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float e = s[i] * inv_C;
        m[i] += e;
        const float var = fmaf(s[V + i], inv_C, -e * e);
        r[i] = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);        // (a NaN stays one)
    }
    if (!in) return;
    if (g == 0 && crank == 0) {
        if (mean_out) store_floats<V>(mean_out + (size_t)n * q.P + p, m);
        if (rstd_out) store_floats<V>(rstd_out + (size_t)n * q.P + p, r);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = c0 + g + k * G;
        if (c < c1) {
            const float ga = gamma ? gamma[c] : 1.0f, be = beta ? beta[c] : 0.0f;
            float f[V];
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] = fmaf((v[k].get(i) - m[i]) * r[i], ga, be);
            v[k].set(f);
            v[k].store(y + at + k * step);
        }
    }
}

// ---- backward, maps -------------------------------------------------------------------------
// Persistent: a thread keeps its channels from tile to tile, so the sums of the parameters' gradients stay in its registers; at the
// end each cluster writes one row of partial sums and ln_reduce adds the rows in a fixed order.
template <typename T, int V, int K>
__global__ void __launch_bounds__(NT) ln_bwd_map(const T* dy, const T* x, const float* __restrict__ gamma, const float* __restrict__ mean,
                                                 const float* __restrict__ rstd, T* dx, float* __restrict__ part_out, MapGeom q)
{
    extern __shared__ float sm[];
    const int tid = threadIdx.x;
    const int segl = 1 << q.segl_log2, tpos = segl * V, G = NT >> q.segl_log2;       // segl <= 32
    const int l = tid & (segl - 1), g = tid >> q.segl_log2;
    const int cid = blockIdx.x / q.cl, clusters = gridDim.x / q.cl, crank = blockIdx.x - cid * q.cl;
    const int c0 = crank * q.Cs, c1 = min(q.C, c0 + q.Cs);
    const size_t step = (size_t)G * q.P;
    const float inv_C = 1.0f / (float)q.C;

    float dg[K], db[K];
#pragma unroll
    for (int k = 0; k < K; ++k) { dg[k] = 0.0f; db[k] = 0.0f; }
    int buf = 0;
    for (int item = cid; item < q.items; item += clusters, buf ^= 1) {
        const int n = item / q.tiles;
        const size_t p = (size_t)(item - n * q.tiles) * tpos + (size_t)l * V;
        const bool in = p < q.P;
        const size_t at = ((size_t)n * q.C + c0 + g) * q.P + p;
        Vec<T, V> vx[K], vd[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            vx[k].zero(); vd[k].zero();
            if (in && c0 + g + k * G < c1) { vx[k].load(x + at + k * step); vd[k].load(dy + at + k * step); }
        }
        float mu[V], r[V], s[2 * V];      // s: sums of g and of g xh
#pragma unroll
        for (int i = 0; i < V; ++i) { mu[i] = 0.0f; r[i] = 0.0f; s[i] = 0.0f; s[V + i] = 0.0f; }
        if (in) { load_floats<V>(mean + (size_t)n * q.P + p, mu); load_floats<V>(rstd + (size_t)n * q.P + p, r); }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = c0 + g + k * G;
            if (c < c1) {
                const float ga = gamma ? gamma[c] : 1.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = vd[k].get(i), xh = (vx[k].get(i) - mu[i]) * r[i], gg = d * ga;
                    dg[k] = fmaf(d, xh, dg[k]);
                    db[k] += d;
                    s[i] += gg;
                    s[V + i] = fmaf(gg, xh, s[V + i]);
                }
            }
        }
        tile_sum<V, 2>(s, sm, q, l, g, buf);
        if (in) {
#pragma unroll
            for (int i = 0; i < 2 * V; ++i) s[i] *= inv_C;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = c0 + g + k * G;
                if (c < c1) {
                    const float ga = gamma ? gamma[c] : 1.0f;
                    float f[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float xh = (vx[k].get(i) - mu[i]) * r[i];
                        f[i] = r[i] * (fmaf(vd[k].get(i), ga, -s[i]) - xh * s[V + i]);
                    }
                    vx[k].set(f);
                    vx[k].store(dx + at + k * step);
                }
            }
        }
    }
    if (q.cl > 1) cluster_sync();       // nobody leaves while a neighbour reads
    pdl_launch();
    if (!part_out) return;
    float* row = part_out + (size_t)cid * 2 * q.C;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        for (int o = 1; o < segl; o <<= 1) { dg[k] += __shfl_xor_sync(FULL, dg[k], o); db[k] += __shfl_xor_sync(FULL, db[k], o); }
        const int c = c0 + g + k * G;
        if (l == 0 && c < c1) { row[c] = dg[k]; row[q.C + c] = db[k]; }
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
                                                  const float* __restrict__ rstd, T* dx, float* __restrict__ part_out, int N, int C)
{
    extern __shared__ float acc_sm[];   // TR < 256: [2][C], the sums of the CTA's row groups
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
    if (!part_out) return;
    float* row = part_out + (size_t)blockIdx.x * 2 * C;
    // the row groups add up one after the other: a fixed order
    for (int w = 0; w < R; ++w) {
        if (sub == w) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (t + k * TR) * V;
                if (c < C) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float a = dg[k][i], b = db[k][i];
                        if (R > 1 && w > 0) { a += acc_sm[c + i]; b += acc_sm[C + c + i]; }
                        if (R > 1 && w + 1 < R) { acc_sm[c + i] = a; acc_sm[C + c + i] = b; }
                        else { row[c + i] = a; row[C + c + i] = b; }
                    }
                }
            }
        }
        if (R > 1) __syncthreads();
    }
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
    int V, K, TR;                       // TR: rows only
    MapGeom q;
    size_t smem;
};

// Elements of a vector: 16 bytes while rows of `len` elements start on that.
inline int vec_elems(size_t len, int es)
{
    int v = 16 / es;
    while (len % v) v >>= 1;
    return v;
}

// Registers: a thread of the forward pass holds K vectors, one of the backward pass 2 K (and 2 K sums).
inline Plan plan_of(int N, int C, size_t P, int es, bool bwd)
{
    Plan p{};
    if (P == 1) {
        p.rows = true;
        p.V = C % (16 / es) == 0 ? 16 / es : 1;
        const int caps[5][2] = {{8, 8}, {8, 32}, {32, 32}, {256, 8}, {256, 32}};      // threads a row, channels a thread
        int i = 0;
        while (caps[i][0] * caps[i][1] < C) ++i;                                         // 256 x 32 = WCC_MAX_CHANNELS
        p.TR = caps[i][0];
        p.K = caps[i][1] / p.V;
        p.smem = bwd && p.TR < NT ? (size_t)2 * C * 4 : 0;
        return p;
    }
    p.V = vec_elems(P, es);
    const int kmax = bwd ? (p.V * es <= 4 ? 16 : 8) : (p.V * es <= 4 ? 32 : 16), kgood = 8;
    int lg = 0;
    const int top = bwd ? 5 : 8;
    while (lg < top && ((size_t)p.V << lg) < P) ++lg;
    // the widest segments that leave K at kgood; narrower down to a sector for more tiles than the GPU has room for at once, or for K
    auto K_of = [&](int s, int c) { return ceil_div(c, NT >> s); };
    auto tiles_of = [&](int s) { return (P + ((size_t)p.V << s) - 1) / ((size_t)p.V << s); };
    const int sector = [&] { int s = 0; while ((p.V << s) * es < 32 && s < lg) ++s; return s; }();
    while (lg > sector && K_of(lg, C) > kgood) --lg;
    while (lg > sector && (size_t)N * tiles_of(lg) < 2 * B200_SMS) --lg;
    int cl = 1;
    while (K_of(lg, ceil_div(C, cl)) > kmax && cl < 8) cl *= 2;
    while (K_of(lg, ceil_div(C, cl)) > kmax) --lg;
    p.q.P = P; p.q.C = C; p.q.cl = cl; p.q.Cs = ceil_div(C, cl); p.q.segl_log2 = lg;
    p.q.tiles = (int)tiles_of(lg);
    p.q.items = N * p.q.tiles;
    const int k = K_of(lg, p.q.Cs);
    p.K = k <= 2 ? 2 : k <= 4 ? 4 : k <= 8 ? 8 : k <= 16 ? 16 : 32;
    const int tpos = p.V << lg;
    p.smem = (size_t)2 * tile_floats(p.q, tpos) * 4;
    return p;
}

template <typename T, int V, int K>
static wcc_status fwd_map(const Plan& p, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, float eps, cudaStream_t st)
{
    return launch_overlapped(ln_fwd_map<T, V, K>, dim3((unsigned)(p.q.items * p.q.cl)), dim3(NT), p.smem, st, false, p.q.cl,
                             static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, p.q, eps);
}
template <typename T, int V, int K>
static wcc_status bwd_map(const Plan& p, int ctas, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                          float* part, cudaStream_t st)
{
    return launch_overlapped(ln_bwd_map<T, V, K>, dim3((unsigned)ctas), dim3(NT), p.smem, st, false, p.q.cl, static_cast<const T*>(dy),
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
                           float* part, int N, int C, cudaStream_t st)
{
    return launch_overlapped(ln_bwd_rows<T, V, K, TR>, dim3((unsigned)ctas), dim3(NT), p.smem, st, false, 1, static_cast<const T*>(dy),
                             static_cast<const T*>(x), gamma, mean, rstd, static_cast<T*>(dx), part, N, C);
}

// CTAs of the backward pass = rows of partial sums (times the cluster): as many as run at once.
inline int bwd_ctas(const Plan& p, int N)
{
    if (p.rows) {
        const long long want = ((long long)N * p.TR + NT - 1) / NT;
        return (int)(want < 2 * B200_SMS ? want : 2 * B200_SMS);
    }
    const int room = 2 * B200_SMS / p.q.cl;
    return (p.q.items < room ? p.q.items : room) * p.q.cl;
}
inline size_t bwd_ws_bytes(const Plan& p, int N, int C)
{
    return align_up((size_t)bwd_ctas(p, N) / (p.rows ? 1 : p.q.cl) * 2 * C * 4, 256);
}

template <typename T>
static wcc_status forward(const Plan& p, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd, int N, int C, float eps,
                          cudaStream_t st)
{
    constexpr int VM = 16 / (int)sizeof(T);
    if (p.rows) {
#define WCC_LN_ROWS(V_, KV_, TR_) \
    if (p.V == (V_) && p.K == (KV_) / (V_) && p.TR == (TR_)) return fwd_rows<T, V_, (KV_) / (V_), TR_>(x, gamma, beta, y, mean, rstd, N, C, eps, st);
        WCC_LN_ROWS(VM, 8, 8) WCC_LN_ROWS(VM, 32, 8) WCC_LN_ROWS(VM, 32, 32) WCC_LN_ROWS(VM, 8, 256) WCC_LN_ROWS(VM, 32, 256)
        WCC_LN_ROWS(1, 8, 8) WCC_LN_ROWS(1, 32, 8) WCC_LN_ROWS(1, 32, 32) WCC_LN_ROWS(1, 8, 256) WCC_LN_ROWS(1, 32, 256)
#undef WCC_LN_ROWS
        return WCC_ERR_SHAPE;
    }
#define WCC_LN_MAP(V_, K_) \
    if (p.V == (V_) && p.K == (K_)) return fwd_map<T, V_, K_>(p, x, gamma, beta, y, mean, rstd, eps, st);
    WCC_LN_MAP(VM, 2) WCC_LN_MAP(VM, 4) WCC_LN_MAP(VM, 8) WCC_LN_MAP(VM, 16)
    WCC_LN_MAP(VM / 2, 2) WCC_LN_MAP(VM / 2, 4) WCC_LN_MAP(VM / 2, 8) WCC_LN_MAP(VM / 2, 16)
    WCC_LN_MAP(VM / 4, 2) WCC_LN_MAP(VM / 4, 4) WCC_LN_MAP(VM / 4, 8) WCC_LN_MAP(VM / 4, 16) WCC_LN_MAP(VM / 4, 32)
    if constexpr (VM == 8) { WCC_LN_MAP(1, 2) WCC_LN_MAP(1, 4) WCC_LN_MAP(1, 8) WCC_LN_MAP(1, 16) WCC_LN_MAP(1, 32) }
#undef WCC_LN_MAP
    return WCC_ERR_SHAPE;
}

template <typename T>
static wcc_status backward(const Plan& p, const void* dy, const void* x, const float* gamma, const float* mean, const float* rstd, void* dx,
                           float* part, int N, int C, cudaStream_t st)
{
    constexpr int VM = 16 / (int)sizeof(T);
    const int ctas = bwd_ctas(p, N);
    if (p.rows) {
#define WCC_LN_ROWS(V_, KV_, TR_) \
    if (p.V == (V_) && p.K == (KV_) / (V_) && p.TR == (TR_)) return bwd_rows<T, V_, (KV_) / (V_), TR_>(p, ctas, dy, x, gamma, mean, rstd, dx, part, N, C, st);
        WCC_LN_ROWS(VM, 8, 8) WCC_LN_ROWS(VM, 32, 8) WCC_LN_ROWS(VM, 32, 32) WCC_LN_ROWS(VM, 8, 256) WCC_LN_ROWS(VM, 32, 256)
        WCC_LN_ROWS(1, 8, 8) WCC_LN_ROWS(1, 32, 8) WCC_LN_ROWS(1, 32, 32) WCC_LN_ROWS(1, 8, 256) WCC_LN_ROWS(1, 32, 256)
#undef WCC_LN_ROWS
        return WCC_ERR_SHAPE;
    }
#define WCC_LN_MAP(V_, K_) \
    if (p.V == (V_) && p.K == (K_)) return bwd_map<T, V_, K_>(p, ctas, dy, x, gamma, mean, rstd, dx, part, st);
    WCC_LN_MAP(VM, 2) WCC_LN_MAP(VM, 4) WCC_LN_MAP(VM, 8)
    WCC_LN_MAP(VM / 2, 2) WCC_LN_MAP(VM / 2, 4) WCC_LN_MAP(VM / 2, 8)
    WCC_LN_MAP(VM / 4, 2) WCC_LN_MAP(VM / 4, 4) WCC_LN_MAP(VM / 4, 8) WCC_LN_MAP(VM / 4, 16)
    if constexpr (VM == 8) { WCC_LN_MAP(1, 2) WCC_LN_MAP(1, 4) WCC_LN_MAP(1, 8) WCC_LN_MAP(1, 16) }
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
