// Group norm with an activation on channels-last maps [N][P][C], forward and backward.
//
// Statistics run over the positions and the D channels of a group, so every map is gone through twice: once for sums, once to apply them.  The
// bytes bound it: x and y (forward), x, dy and dx (backward), each once, if the second time finds the map in L2.  Four ways:
//  - images of one position whose groups are 2^k lanes of a warp (token rows): rows_forward, rows_backward, nothing is read twice;
//  - other images of one tile: a CTA does sums and result of an image, and goes on to its next;
//  - images of many tiles whose channels repeat within a CTA's vectors: groupnorm_ring.cuh;
//  - images of many tiles and more channels than that (beyond 2048 bf16 or 1024 fp32, odd numbers beyond 256): one launch works through a list of tiles,
//     sums of image 0 .. lag-1 | sums of image lag, apply image 0 (tile by tile in turn) | sums of image lag+1, apply image 1 | ...
//    with a lag of about 24 MB.  CTAs take tiles by a ticket, in order.  A tile only ever waits for tiles in front of it, so whichever CTAs are resident finish:
//    the lowest unfinished tile waits for nobody.  The last CTA to bring a tile's sums (by a count of arrivals) adds them all up in the tiles' order, so
//    results do not depend on the schedule, and raises the image's flag.
//
// A thread meets the same channels all along: its vectors (of V values) are a multiple of the period p = C / gcd(C, V) vectors apart, so its
// constants and sums sit in registers.  Periods longer than the CTA are gone through in slots of one vector a thread.
#pragma once

#include "checkpoint.cuh"
#include "tma.cuh"
#include "vec.cuh"

namespace wcc {
namespace gn {

using namespace tr;

constexpr int T = 256;                     // threads of a CTA
constexpr int FAN = 16;                    // tiles whose channel sums are added up in one step
constexpr int CTAS_FWD = 3, CTAS_BWD = 2;  // CTAs of an SM
constexpr size_t LAG_BYTES = (size_t)24 << 20;
constexpr int RING_GAP = B200_SMS * 3 / 2;         // ring: tiles of sums in flight, and what they finish behind

struct Plan {
    int V, p, lanes, reps, slots;          // period of p vectors; `reps` periods side by side, or one in `slots` turns of the CTA
    bool aligned;                          // all of a vector's channels are in one group
    bool ring;                             // groupnorm_ring.cuh; else the kernels of this file
    int tile, nt, supers;                  // positions (ring: vectors) of a tile, tiles of an image, steps of FAN tiles
    int lag;                               // images between sums and result
    // ring: a tile's result comes `delay` tiles behind its sums, an image's sums are finished by `fin` steps, `gap` tiles behind its last
    int delay, gap, fin;
    int copies;                            // ring: rows of C in a period
    int ctl;                               // words of control an image: arrivals of each step, of the steps, flag (ring: arrivals of warps)
    bool solo;
};

struct Args {
    const void *x, *dy;
    const int8_t* codes;                   // checkpoint of x, read (backward) ...
    const float* scales;
    const float *gamma, *beta, *mean, *rstd;
    void* out;
    float *mean_out, *rstd_out;
    float *part, *sup, *img;               // partial sums of tiles, of steps, of images (or the parameters' gradients themselves)
    long long img_beta, img_gamma, img_row;  // img + row * img_row + {img_beta, img_gamma}
    float2* coef;
    unsigned* ctl;                         // ticket, then Plan::ctl words an image
    int N, P, C, G, D, nb, act;
    float eps, inv_count;
    bool params;
    Divisor dC, dD, dW;                    // by C, D and the vectors (or values) of a group in a row
    Plan q;
    int* status;
};

inline int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

inline Plan plan_of(int N, int P, int C, int G, int es, bool backward, bool whole_rows)
{
    Plan q{};
    const long long E = (long long)P * C;
    const size_t bytes = (size_t)E * es * (backward ? 2 : 1);
    const long long lag = (long long)((LAG_BYTES + bytes - 1) / bytes);
    q.lag = (int)(lag < N ? lag : N);
    // The ring takes whole 16-byte vectors whatever the channels, if the period fits the CTA and the image has tiles enough; a checkpoint's where rows
    // start on 16 bytes of codes.
    q.V = 16 / es;
    q.p = C / gcd(C, q.V);
    if (q.p <= T && (!whole_rows || C % 16 == 0) && E / q.V < (1LL << 30)) {
        q.lanes = q.p;
        q.reps = T / q.p;
        q.slots = 1;
        q.aligned = C % q.V == 0 && (C / G) % q.V == 0;
        const long long nv = E / q.V, step = (long long)q.reps * q.p;
        long long hi = 4096, lo = 512;
        if (!backward) hi = 8192;
        if (hi < 64LL * C / q.V) hi = 64LL * C / q.V;
        // Small maps: two or three tiles of each kind for an SM, that the end of a tile is met once.  (us, forward / backward, with eight: 4 x 64 x 64 x 256
        // bf16 44 / 44, now 25 / 26; 24 x 60 x 50 x 40 fp32 39 / 40, now 24 / 27.)
        long long t = N * nv / (B200_SMS * (backward ? 2 : 3));
        t = t < lo ? lo : t > hi ? hi : t;
        if (t < (nv + 4095) / 4096) t = (nv + 4095) / 4096;
        q.tile = (int)((t + step - 1) / step * step);
        q.nt = (int)((nv + q.tile - 1) / q.tile);
        q.ctl = 1;
        q.copies = q.p * q.V / C;
        q.ring = q.nt > 1;
        const long long all = (long long)N * q.nt, gap = RING_GAP < all - q.nt ? RING_GAP : all - q.nt, delay = q.nt + gap + RING_GAP / 2;
        q.gap = (int)gap;
        q.delay = (int)(delay < all ? delay : all);
        // an item's threads have all of their loads on the way at once: 4096 channels' sums, or 512 groups' statistics
        const long long fin = backward ? (2LL * C * q.nt + 4095) / 4096 : ((long long)G * q.nt + 511) / 512;
        q.fin = (int)(fin < G ? fin : G);
        if (q.ring) return q;
    }
    // Vectors of 16 bytes where every image starts on one and the period fits the CTA; else as wide as the rows' own alignment.  (A checkpoint's
    // scale is that of a row, so a vector must not go over a row's end.)
    q.V = 16 / es;
    while (q.V > 1 && !(E % q.V == 0 && (C % q.V == 0 || (!whole_rows && C / gcd(C, q.V) <= T)))) q.V /= 2;
    q.p = C / gcd(C, q.V);
    q.lanes = q.p < T ? q.p : T;
    q.reps = q.p < T ? T / q.p : 1;
    q.slots = (q.p + T - 1) / T;
    const int D = C / G;
    q.aligned = C % q.V == 0 && D % q.V == 0;
    // Tiles: eight for each SM, of 8 to 64 KB, and of 64 positions at least where there are enough (the backward pass stores two sums a channel and tile).
    const int unit = q.p * q.V / C;        // positions of a period
    const long long row = (long long)C * es;
    long long hi = 65536 / row, lo = 8192 / row;
    if (hi < 64) hi = 64;
    if (lo < 1) lo = 1;
    long long t = (long long)N * P / (B200_SMS * 8);
    t = t < lo ? lo : t > hi ? hi : t;
    if (t < (P + 1023) / 1024) t = (P + 1023) / 1024;
    t = (t + unit - 1) / unit * unit;
    q.tile = (int)(t < P ? t : P);
    q.nt = (P + q.tile - 1) / q.tile;
    q.supers = (q.nt + FAN - 1) / FAN;
    q.solo = q.nt == 1;
    q.ctl = q.supers + 2;
    return q;
}

inline int grid_of(const Plan& q, int N, int sms, bool backward)
{
    const long long items = q.solo ? (long long)N : 2LL * N * q.nt, most = (long long)sms * (backward ? CTAS_BWD : CTAS_FWD);
    return (int)(items < most ? items : most);
}

struct Layout { size_t ctl, part, sup, img, coef, total; };
inline Layout layout_of(const Plan& q, int N, int C, int G, bool backward)
{
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t a = at; at = align_up(at + bytes, 256); return a; };
    if (!q.solo) {
        // (the words of control and the ring's coefficients start as zeros)
        l.ctl = take((1 + (size_t)N * q.ctl) * 4);
        l.coef = take((size_t)N * G * 8);
        l.part = take((size_t)N * q.nt * (backward ? 2 * C : 3 * G) * 4);
        if (backward && !q.ring) l.sup = take((size_t)N * q.supers * 2 * C * 4);
    }
    if (backward) l.img = take((size_t)(q.solo ? grid_of(q, N, B200_SMS, true) : N) * 2 * C * 4);
    l.total = at < 256 ? 256 : at;
    return l;
}

// Vectors that a thread has on their way at once (backward: of either map): the narrower, the more, as far as registers go.
template <int V> constexpr int LOADS_FWD = V == 1 ? 8 : 4;
template <int V> constexpr int LOADS_BWD = V >= 4 ? 2 : 8 / V;

// ---- pieces ----------------------------------------------------------------------------------------
struct Stat { float n, mean, m2; };       // (ring)
// Values put together: their number, their mean in two parts, base + off, and the sum of their squared deviations from it.  base is one of the values: between
// groups of a few values differences of means go into the deviations at first order, and the mean of values far from zero, rounded, has lost too much for
// that (a mean of 10^4 spreads: rstd of 23 values was off by 10^-4; one by one its parts lose what is of the spread's size).
struct Part { float n, base, off, m2; };
__device__ __forceinline__ Part merge(Part a, Part b)
{
    // (what is of no values adds nothing: the square of its distance may be no fp32 number.  By selections: with branches 3 x 40 x 200 x 1023 fp32 takes 253 us, so 185.)
    const bool none = a.n == 0.0f, both = !none && b.n != 0.0f;
    const float n = a.n + b.n, f = both ? __fdividef(b.n, n) : 0.0f, d = both ? (b.base - a.base) + (b.off - a.off) : 0.0f;
    return {n, none ? b.base : a.base, none ? b.off : __fmaf_rn(d, f, a.off), a.m2 + b.m2 + d * d * a.n * f};
}
__device__ __forceinline__ Part warp_merge(Part s)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        Part b{__shfl_xor_sync(0xFFFFFFFFu, s.n, o), __shfl_xor_sync(0xFFFFFFFFu, s.base, o), __shfl_xor_sync(0xFFFFFFFFu, s.off, o), __shfl_xor_sync(0xFFFFFFFFu, s.m2, o)};
        // the lower lane's part first on both sides: the same bits on all lanes
        s = (threadIdx.x & o) ? merge(b, s) : merge(s, b);
    }
    return s;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Channel of value e of vector q of a period.
template <int V> __device__ __forceinline__ int channel(const Args& a, int q, int e)
{
    const int f = q * V + e;
    return f < a.C ? f : f % a.C;
}

// ---- forward ---------------------------------------------------------------------------------------
// Sums of a tile.  Deviations are taken from the thread's first value (of the channel, or of its group), so a common offset costs nothing: a
// thread's sum of squares holds the pivot's own distance squared, and loses at most (values of the thread) * 2^-24 of itself.  Threads and tiles
// are then put together (Part).
template <typename X, int V, bool ALIGNED>
__device__ __forceinline__ void stats_tile(const Args& a, const X* x, int nvec, Part* entries)
{
    const Plan& q = a.q;
    const int sub = threadIdx.x / q.lanes, lane = threadIdx.x - sub * q.lanes;
    const int step = q.reps * q.p;
    for (int j = 0; j < q.slots; ++j) {
        const int vq = j * T + lane;
        if (sub >= q.reps || vq >= q.p) continue;
        const int v0 = sub * q.p + vq;
        if constexpr (ALIGNED) {
            f2 s = both(0.0f), ss = both(0.0f);
            float s1 = 0.0f, ss1 = 0.0f, pivot = 0.0f;
            int k = 0;
            if (v0 < nvec) {
                pivot = (float)x[(size_t)v0 * V];
                const f2 neg = both(-pivot);
#pragma unroll 4
                for (int v = v0; v < nvec; v += step, ++k) {
                    Vec<X, V> r;
                    r.load(x + (size_t)v * V);
                    float f[V];
                    unpack(r, f);
                    if constexpr (V == 1) {
                        const float d = f[0] - pivot;
                        s1 += d;
                        ss1 = __fmaf_rn(d, d, ss1);
                    } else {
#pragma unroll
                        for (int e = 0; e < V; e += 2) {
                            const f2 d = add2(pair(f[e], f[e + 1]), neg);
                            s = add2(s, d);
                            ss = fma2(d, d, ss);
                        }
                    }
                }
            }
            const float n = (float)(k * V), sum = s.x() + s.y() + s1, sq = ss.x() + ss.y() + ss1, m = k ? __fdividef(sum, n) : 0.0f;
            entries[v0] = {n, pivot, m, fmaxf(sq - sum * m, 0.0f)};
        } else {
            float s[V], ss[V], pivot[V];
#pragma unroll
            for (int e = 0; e < V; ++e) s[e] = ss[e] = pivot[e] = 0.0f;
            int k = 0;
            if (v0 < nvec) {
                Vec<X, V> r;
                r.load(x + (size_t)v0 * V);
                unpack(r, pivot);
#pragma unroll 2
                for (int v = v0; v < nvec; v += step, ++k) {
                    r.load(x + (size_t)v * V);
                    float f[V];
                    unpack(r, f);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float d = f[e] - pivot[e];
                        s[e] += d;
                        ss[e] = __fmaf_rn(d, d, ss[e]);
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float n = (float)k, m = k ? __fdividef(s[e], n) : 0.0f;
                entries[v0 * V + e] = {n, pivot[e], m, fmaxf(ss[e] - s[e] * m, 0.0f)};
            }
        }
    }
}

// Group g of the CTA's entries; the whole warp calls it.
template <int V, bool ALIGNED>
__device__ __forceinline__ Part group_of(const Args& a, int g, const Part* entries)
{
    const Plan& q = a.q;
    constexpr int W = ALIGNED ? V : 1;
    const int period = q.p * V / W, Cw = a.C / W, Dw = a.D / W, copies = period / Cw, each = copies * Dw, total = q.reps * each;
    Part s{0.0f, 0.0f, 0.0f, 0.0f};
    for (int m = threadIdx.x & 31; m < total; m += 32) {
        const int sub = m / each, rest = m - sub * each, i = rest / Dw;
        s = merge(s, entries[sub * period + i * Cw + g * Dw + (rest - i * Dw)]);
    }
    return warp_merge(s);
}

template <int V, int ACT> __device__ __forceinline__ void activate(float (&z)[V])
{
    if constexpr (ACT == WCC_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = z[e] < 0.0f ? 0.0f : z[e];       // (a NaN stays one)
    } else if constexpr (ACT == WCC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] = z[e] * sigmoid(z[e]);
    }
}

template <typename X, int V, int ACT>
__device__ __forceinline__ void apply_tile(const Args& a, const X* x, X* y, int nvec, const float2* coef)
{
    const Plan& q = a.q;
    const int sub = threadIdx.x / q.lanes, lane = threadIdx.x - sub * q.lanes;
    const int step = q.reps * q.p;
    constexpr int U = LOADS_FWD<V>;
    for (int j = 0; j < q.slots; ++j) {
        const int vq = j * T + lane;
        if (sub >= q.reps || vq >= q.p) continue;
        float m[V], k[V], b[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = channel<V>(a, vq, e);
            const float2 st = coef[c / a.D];
            m[e] = -st.x;
            k[e] = st.y * (a.gamma ? __ldg(a.gamma + c) : 1.0f);
            b[e] = a.beta ? __ldg(a.beta + c) : 0.0f;
        }
        for (int v = sub * q.p + vq; v < nvec; v += U * step) {
            Vec<X, V> r[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (v + u * step < nvec) r[u].load(x + (size_t)(v + u * step) * V);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * step >= nvec) break;
                float f[V];
                unpack(r[u], f);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] = __fmaf_rn(f[e] + m[e], k[e], b[e]);
                activate<V, ACT>(f);
                pack(r[u], f);
                r[u].store(y + (size_t)(v + u * step) * V);
            }
        }
    }
}
template <typename X, int V>
__device__ __forceinline__ void apply(const Args& a, const X* x, X* y, int nvec, const float2* coef)
{
    if (a.act == WCC_ACT_SILU) apply_tile<X, V, WCC_ACT_SILU>(a, x, y, nvec, coef);
    else if (a.act == WCC_ACT_RELU) apply_tile<X, V, WCC_ACT_RELU>(a, x, y, nvec, coef);
    else apply_tile<X, V, WCC_ACT_NONE>(a, x, y, nvec, coef);
}

// ---- the list of tiles -----------------------------------------------------------------------------
struct Item { bool sums; int n, tile; };
__device__ __forceinline__ Item item_of(const Args& a, long long i)
{
    const int nt = a.q.nt, lag = a.q.lag;
    const long long head = (long long)lag * nt, mid = 2LL * (a.N - lag) * nt;
    if (i < head) return {true, (int)(i / nt), (int)(i % nt)};
    i -= head;
    if (i < mid) {
        const long long round = i / (2 * nt);
        const int k = (int)(i - round * 2 * nt);
        return (k & 1) ? Item{false, (int)round, k >> 1} : Item{true, (int)round + lag, k >> 1};
    }
    i -= mid;
    return {false, a.N - lag + (int)(i / nt), (int)(i % nt)};
}

__device__ __forceinline__ unsigned load_acquire(const unsigned* p)
{
    unsigned v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void store_release(unsigned* p, unsigned v)
{
    asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// True on every thread if this CTA is the last of `of` to arrive; then what the others wrote before is visible.
__device__ __forceinline__ bool arrive_last(unsigned* count, unsigned of, int* flag)
{
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) *flag = atomicAdd(count, 1u) == of - 1;
    __syncthreads();
    const bool last = *flag != 0;
    if (last) __threadfence();
    return last;
}
// Bounded wait of the whole CTA for an image's flag.
__device__ __forceinline__ bool wait_flag(const unsigned* f, int* status, int* flag)
{
    if (threadIdx.x == 0) {
        bool ok = false;
        const uint32_t limit = tc::c_wait_limit;
        for (uint32_t i = 0; i < limit && !ok; ++i) {
            ok = load_acquire(f) != 0u;
            if (!ok) __nanosleep(100);
        }
        if (!ok) atomicExch(status, (int)WCC_ERR_TIMEOUT);
        *flag = ok;
    }
    __syncthreads();
    return *flag != 0;
}

template <typename X, int V, bool ALIGNED>
__global__ void __launch_bounds__(T, CTAS_FWD) forward_kernel(const __grid_constant__ Args a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ long long s_item;
    __shared__ int s_flag;
    Part* entries = reinterpret_cast<Part*>(smem);
    const Plan& q = a.q;
    const int warp = threadIdx.x >> 5;
    const X* x = static_cast<const X*>(a.x);
    X* y = static_cast<X*>(a.out);
    const long long E = (long long)a.P * a.C;
    pdl_wait();
    pdl_launch();
    if (q.solo) {
        const int words = q.slots > 1 ? q.p * V / (ALIGNED ? V : 1) : q.reps * q.p * (ALIGNED ? 1 : V);
        float2* coef = reinterpret_cast<float2*>(entries + words);
        const int nvec = (int)(E / V);
        for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
            stats_tile<X, V, ALIGNED>(a, x + n * E, nvec, entries);
            __syncthreads();
            for (int g = warp; g < a.G; g += T / 32) {
                const Part s = group_of<V, ALIGNED>(a, g, entries);
                if ((threadIdx.x & 31) == 0) {
                    const float r = __fdiv_rn(1.0f, __fsqrt_rn(s.m2 * a.inv_count + a.eps)), mean = s.base + s.off;
                    coef[g] = make_float2(mean, r);
                    if (a.mean_out) a.mean_out[(size_t)n * a.G + g] = mean;
                    if (a.rstd_out) a.rstd_out[(size_t)n * a.G + g] = r;
                }
            }
            __syncthreads();
            apply<X, V>(a, x + n * E, y + n * E, nvec, coef);
        }
        return;
    }
    const long long items = 2LL * a.N * q.nt;
    long long next = threadIdx.x == 0 ? (long long)atomicAdd(a.ctl, 1u) : 0;
    for (;;) {
        if (threadIdx.x == 0) s_item = next;
        __syncthreads();
        const long long i = s_item;
        if (i >= items) return;
        if (threadIdx.x == 0) next = (long long)atomicAdd(a.ctl, 1u);
        const Item it = item_of(a, i);
        const int p0 = it.tile * q.tile, positions = min(q.tile, a.P - p0);
        const long long at = it.n * E + (long long)p0 * a.C;
        const int nvec = (int)((long long)positions * a.C / V);
        unsigned* ctl = a.ctl + 1 + (size_t)it.n * q.ctl;
        float2* coef = a.coef + (size_t)it.n * a.G;
        if (it.sums) {
            float2* part = reinterpret_cast<float2*>(a.part) + (size_t)it.n * q.nt * a.G;
            stats_tile<X, V, ALIGNED>(a, x + at, nvec, entries);
            __syncthreads();
            for (int g = warp; g < a.G; g += T / 32) {
                const Part s = group_of<V, ALIGNED>(a, g, entries);
                // (a tile's mean in one number: the tile's values are many, and what their mean loses goes into the whole by less than a value's own rounding)
                if ((threadIdx.x & 31) == 0) part[(size_t)it.tile * a.G + g] = make_float2(s.base + s.off, s.m2);
            }
            if (arrive_last(ctl, (unsigned)q.nt, &s_flag)) {
                for (int g = warp; g < a.G; g += T / 32) {
                    Part s{0.0f, 0.0f, 0.0f, 0.0f};
                    for (int t = threadIdx.x & 31; t < q.nt; t += 32) {
                        const float2 v = __ldcg(part + (size_t)t * a.G + g);
                        s = merge(s, {(float)((long long)min(q.tile, a.P - t * q.tile) * a.D), v.x, 0.0f, v.y});
                    }
                    s = warp_merge(s);
                    if ((threadIdx.x & 31) == 0) {
                        const float r = __fdiv_rn(1.0f, __fsqrt_rn(s.m2 * a.inv_count + a.eps)), mean = s.base + s.off;
                        coef[g] = make_float2(mean, r);
                        if (a.mean_out) a.mean_out[(size_t)it.n * a.G + g] = mean;
                        if (a.rstd_out) a.rstd_out[(size_t)it.n * a.G + g] = r;
                    }
                }
                __threadfence();
                __syncthreads();
                if (threadIdx.x == 0) store_release(ctl + q.ctl - 1, 1u);
            }
        } else {
            if (!wait_flag(ctl + q.ctl - 1, a.status, &s_flag)) return;
            // through shared memory: written during this launch, so not to be read by the path of constant data
            float2* c = reinterpret_cast<float2*>(entries);
            for (int g = threadIdx.x; g < a.G; g += T) c[g] = __ldcg(coef + g);
            __syncthreads();
            apply<X, V>(a, x + at, y + at, nvec, c);
        }
        __syncthreads();
    }
}

// ---- backward --------------------------------------------------------------------------------------
template <int V, int ACT> __device__ __forceinline__ void slope_times(const float (&z)[V], float (&t)[V])
{
    if constexpr (ACT == WCC_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < V; ++e) t[e] = z[e] > 0.0f ? t[e] : 0.0f;
    } else if constexpr (ACT == WCC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float s = sigmoid(z[e]);
            t[e] *= __fmaf_rn(z[e] * s, 1.0f - s, s);
        }
    }
}

// What a thread's channels need: -mean, rstd * gamma, beta.
template <int V> struct Channels {
    float m[V], k[V], b[V];
    __device__ __forceinline__ void load(const Args& a, int n, int vq)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = channel<V>(a, vq, e);
            const size_t g = (size_t)n * a.G + c / a.D;
            m[e] = -__ldg(a.mean + g);
            k[e] = __ldg(a.rstd + g) * (a.gamma ? __ldg(a.gamma + c) : 1.0f);
            b[e] = a.beta ? __ldg(a.beta + c) : 0.0f;
        }
    }
};

// One vector of x: as it is, or from its checkpoint.
template <typename X, int V, bool KEPT> struct Source {
    const X* x;
    const int8_t* codes;
    const float* scales;                   // of the tile's first row
    Vec<X, V> r;
    Vec<int8_t, V> c;
    float s;
    __device__ __forceinline__ void load(int v, int row, int nb, int block)
    {
        if constexpr (KEPT) {
            c.load(codes + (size_t)v * V);
            s = __ldg(scales + (size_t)row * nb + block);
        } else {
            r.load(x + (size_t)v * V);
        }
    }
    __device__ __forceinline__ void get(float (&f)[V]) const
    {
        if constexpr (KEPT) {
            unpack(c, f);
#pragma unroll
            for (int e = 0; e < V; ++e) f[e] *= s;
        } else {
            unpack(r, f);
        }
    }
};

// Sums over the tile's positions of t and t * (x - mean) for each channel, to dst[0 .. C) and dst[C .. 2C).
template <typename X, int V, bool KEPT, int ACT>
__device__ __forceinline__ void sums_tile(const Args& a, int n, long long at, int nvec, float* sums, float* dst)
{
    const Plan& q = a.q;
    const int sub = threadIdx.x / q.lanes, lane = threadIdx.x - sub * q.lanes;
    const int step = q.reps * q.p, width = q.p * V;
    const X* dy = static_cast<const X*>(a.dy) + at;
    constexpr int U = LOADS_BWD<V>;
    for (int j = 0; j < q.slots; ++j) {
        const int vq = j * T + lane;
        if (sub >= q.reps || vq >= q.p) continue;
        Channels<V> ch;
        ch.load(a, n, vq);
        float s0[V], s1[V];
#pragma unroll
        for (int e = 0; e < V; ++e) s0[e] = s1[e] = 0.0f;
        const int block = vq * V / ck::BLOCK;
        int row = sub;
        for (int v = sub * q.p + vq; v < nvec; v += U * step, row += U * q.reps) {
            Source<X, V, KEPT> src[U];
            Vec<X, V> d[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * step >= nvec) break;
                src[u].x = static_cast<const X*>(a.x) + at;
                src[u].codes = a.codes + at;
                src[u].scales = a.scales + at / a.C * a.nb;
                src[u].load(v + u * step, row + u * q.reps, a.nb, block);
                d[u].load(dy + (size_t)(v + u * step) * V);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * step >= nvec) break;
                float xc[V], t[V], z[V];
                src[u].get(xc);
                unpack(d[u], t);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    xc[e] += ch.m[e];
                    z[e] = __fmaf_rn(xc[e], ch.k[e], ch.b[e]);
                }
                slope_times<V, ACT>(z, t);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    s0[e] += t[e];
                    s1[e] = __fmaf_rn(t[e], xc[e], s1[e]);
                }
            }
        }
        if (q.slots > 1) {                 // a channel is one thread's
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dst[vq * V + e] = s0[e];
                dst[a.C + vq * V + e] = s1[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sums[sub * width + vq * V + e] = s0[e];
                sums[(q.reps + sub) * width + vq * V + e] = s1[e];
            }
        }
    }
    __syncthreads();
    if (q.slots == 1) {
        const int copies = width / a.C;
        for (int c = threadIdx.x; c < a.C; c += T) {
            float s0 = 0.0f, s1 = 0.0f;
            for (int k = 0; k < q.reps; ++k)
                for (int i = 0; i < copies; ++i) {
                    s0 += sums[k * width + i * a.C + c];
                    s1 += sums[(q.reps + k) * width + i * a.C + c];
                }
            dst[c] = s0;
            dst[a.C + c] = s1;
        }
    }
}

template <typename X, int V, bool KEPT, int ACT>
__device__ __forceinline__ void dx_tile(const Args& a, int n, long long at, int nvec, const float2* coef)
{
    const Plan& q = a.q;
    const int sub = threadIdx.x / q.lanes, lane = threadIdx.x - sub * q.lanes;
    const int step = q.reps * q.p;
    const X* dy = static_cast<const X*>(a.dy) + at;
    X* out = static_cast<X*>(a.out) + at;
    constexpr int U = LOADS_BWD<V>;
    for (int j = 0; j < q.slots; ++j) {
        const int vq = j * T + lane;
        if (sub >= q.reps || vq >= q.p) continue;
        Channels<V> ch;
        ch.load(a, n, vq);
        float k0[V], k1[V];
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const float2 c = coef[channel<V>(a, vq, e) / a.D];
            k0[e] = c.x;
            k1[e] = c.y;
        }
        const int block = vq * V / ck::BLOCK;
        int row = sub;
        for (int v = sub * q.p + vq; v < nvec; v += U * step, row += U * q.reps) {
            Source<X, V, KEPT> src[U];
            Vec<X, V> d[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * step >= nvec) break;
                src[u].x = static_cast<const X*>(a.x) + at;
                src[u].codes = a.codes + at;
                src[u].scales = a.scales + at / a.C * a.nb;
                src[u].load(v + u * step, row + u * q.reps, a.nb, block);
                d[u].load(dy + (size_t)(v + u * step) * V);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (v + u * step >= nvec) break;
                float xc[V], t[V], z[V];
                src[u].get(xc);
                unpack(d[u], t);
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    xc[e] += ch.m[e];
                    z[e] = __fmaf_rn(xc[e], ch.k[e], ch.b[e]);
                }
                slope_times<V, ACT>(z, t);
#pragma unroll
                for (int e = 0; e < V; ++e) t[e] = __fmaf_rn(t[e], ch.k[e], __fmaf_rn(xc[e], k1[e], k0[e]));
                pack(d[u], t);
                d[u].store(out + (size_t)(v + u * step) * V);
            }
        }
    }
}
template <typename X, int V, bool KEPT>
__device__ __forceinline__ void sums_of(const Args& a, int n, long long at, int nvec, float* sums, float* dst)
{
    if (a.act == WCC_ACT_SILU) sums_tile<X, V, KEPT, WCC_ACT_SILU>(a, n, at, nvec, sums, dst);
    else if (a.act == WCC_ACT_RELU) sums_tile<X, V, KEPT, WCC_ACT_RELU>(a, n, at, nvec, sums, dst);
    else sums_tile<X, V, KEPT, WCC_ACT_NONE>(a, n, at, nvec, sums, dst);
}
template <typename X, int V, bool KEPT>
__device__ __forceinline__ void dx_of(const Args& a, int n, long long at, int nvec, const float2* coef)
{
    if (a.act == WCC_ACT_SILU) dx_tile<X, V, KEPT, WCC_ACT_SILU>(a, n, at, nvec, coef);
    else if (a.act == WCC_ACT_RELU) dx_tile<X, V, KEPT, WCC_ACT_RELU>(a, n, at, nvec, coef);
    else dx_tile<X, V, KEPT, WCC_ACT_NONE>(a, n, at, nvec, coef);
}

// The terms of a group's dx = rstd gamma t + k1 (x - mean) + k0 from its sums of g and g (x - mean): k0 = -rstd mean(g), k1 = -rstd^2 mean(g xh).  The mean of g xh
// comes first: it is of g's size, where rstd^3 alone would leave fp32 with a spread of 10^-13 or 10^13.
__device__ __forceinline__ float2 terms_of(const Args& a, float r, float c1, float c2)
{
    const float m = r * (c2 * a.inv_count);
    return make_float2(-r * (c1 * a.inv_count), -r * m * r);
}
// Of image n, from the sums of its channels.
__device__ __forceinline__ void group_terms(const Args& a, int n, const float* chan, float2* coef)
{
    for (int g = threadIdx.x >> 5; g < a.G; g += T / 32) {
        float c1 = 0.0f, c2 = 0.0f;
        for (int d = threadIdx.x & 31; d < a.D; d += 32) {
            const int c = g * a.D + d;
            const float w = a.gamma ? __ldg(a.gamma + c) : 1.0f;
            c1 = __fmaf_rn(w, chan[c], c1);
            c2 = __fmaf_rn(w, chan[a.C + c], c2);
        }
        c1 = warp_sum(c1);
        c2 = warp_sum(c2);
        if ((threadIdx.x & 31) == 0) {
            const float r = __ldg(a.rstd + (size_t)n * a.G + g);
            coef[g] = terms_of(a, r, c1, c2);
        }
    }
}

template <typename X, int V, bool KEPT>
__global__ void __launch_bounds__(T, CTAS_BWD) backward_kernel(const __grid_constant__ Args a)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ long long s_item;
    __shared__ int s_flag;
    const Plan& q = a.q;
    const long long E = (long long)a.P * a.C;
    float* chan = reinterpret_cast<float*>(smem);                      // [2][C]
    float2* coef_s = reinterpret_cast<float2*>(chan + 2 * a.C);        // [G]
    float* acc = reinterpret_cast<float*>(coef_s + a.G);               // [2][C], solo
    float* sums = acc + (q.solo ? 2 * a.C : 0);                        // [2][reps][p V] where slots == 1
    pdl_wait();
    pdl_launch();
    if (q.solo) {
        const int nvec = (int)(E / V);
        for (int c = threadIdx.x; c < 2 * a.C; c += T) acc[c] = 0.0f;
        for (int n = blockIdx.x; n < a.N; n += gridDim.x) {
            sums_of<X, V, KEPT>(a, n, n * E, nvec, sums, chan);
            __syncthreads();
            group_terms(a, n, chan, coef_s);
            for (int c = threadIdx.x; c < a.C; c += T) {
                acc[c] += chan[c];
                acc[a.C + c] = __fmaf_rn(__ldg(a.rstd + (size_t)n * a.G + c / a.D), chan[a.C + c], acc[a.C + c]);
            }
            __syncthreads();
            dx_of<X, V, KEPT>(a, n, n * E, nvec, coef_s);
        }
        if (a.params) {
            __syncthreads();
            float* row = a.img + (long long)blockIdx.x * a.img_row;
            for (int c = threadIdx.x; c < a.C; c += T) {
                row[a.img_beta + c] = acc[c];
                row[a.img_gamma + c] = acc[a.C + c];
            }
        }
        return;
    }
    const long long items = 2LL * a.N * q.nt;
    long long next = threadIdx.x == 0 ? (long long)atomicAdd(a.ctl, 1u) : 0;
    for (;;) {
        if (threadIdx.x == 0) s_item = next;
        __syncthreads();
        const long long i = s_item;
        if (i >= items) return;
        if (threadIdx.x == 0) next = (long long)atomicAdd(a.ctl, 1u);
        const Item it = item_of(a, i);
        const int p0 = it.tile * q.tile, positions = min(q.tile, a.P - p0);
        const long long at = it.n * E + (long long)p0 * a.C;
        const int nvec = (int)((long long)positions * a.C / V);
        unsigned* ctl = a.ctl + 1 + (size_t)it.n * q.ctl;
        float2* coef = a.coef + (size_t)it.n * a.G;
        if (it.sums) {
            const int s = it.tile / FAN, t0 = s * FAN, tn = min(FAN, q.nt - t0);
            float* part = a.part + (size_t)it.n * q.nt * 2 * a.C;
            float* sup = a.sup + (size_t)it.n * q.supers * 2 * a.C;
            sums_of<X, V, KEPT>(a, it.n, at, nvec, sums, part + (size_t)it.tile * 2 * a.C);
            if (arrive_last(ctl + s, (unsigned)tn, &s_flag)) {
                for (int c = threadIdx.x; c < 2 * a.C; c += T) {
                    float v = 0.0f;
#pragma unroll 8
                    for (int k = 0; k < tn; ++k) v += __ldcg(part + (size_t)(t0 + k) * 2 * a.C + c);
                    sup[(size_t)s * 2 * a.C + c] = v;
                }
                if (arrive_last(ctl + q.supers, (unsigned)q.supers, &s_flag)) {
                    for (int c = threadIdx.x; c < 2 * a.C; c += T) {
                        float v = 0.0f;
#pragma unroll 8
                        for (int k = 0; k < q.supers; ++k) v += __ldcg(sup + (size_t)k * 2 * a.C + c);
                        chan[c] = v;
                    }
                    __syncthreads();
                    group_terms(a, it.n, chan, coef);
                    if (a.params) {
                        float* row = a.img + it.n * a.img_row;
                        for (int c = threadIdx.x; c < a.C; c += T) {
                            row[a.img_beta + c] = chan[c];
                            row[a.img_gamma + c] = __ldg(a.rstd + (size_t)it.n * a.G + c / a.D) * chan[a.C + c];
                        }
                    }
                    __threadfence();
                    __syncthreads();
                    if (threadIdx.x == 0) store_release(ctl + q.ctl - 1, 1u);
                }
            }
        } else {
            if (!wait_flag(ctl + q.ctl - 1, a.status, &s_flag)) return;
            for (int g = threadIdx.x; g < a.G; g += T) coef_s[g] = __ldcg(coef + g);
            __syncthreads();
            dx_of<X, V, KEPT>(a, it.n, at, nvec, coef_s);
        }
        __syncthreads();
    }
}

// ---- images of one position ------------------------------------------------------------------------
// Rows of tokens: a group is D neighbouring values, 2^k lanes with a vector each, so its sums are shuffles and nothing is read twice.  A thread keeps its channels
// from row to row.  (us, 8192 x 1024 bf16, an image a CTA as above / this way: forward 198 / 13, backward 343 / 23.)
inline bool rows_path(int P, int C, int G, int es, bool whole_rows)
{
    const int V = 16 / es, D = C / G, lanes = D / V;
    return P == 1 && D % V == 0 && lanes <= 32 && (lanes & (lanes - 1)) == 0 && (!whole_rows || C % 16 == 0);
}
// Rows of a CTA at once, CTAs side by side along a row, CTAs along the rows: by the sizes alone, so that the order of the gradients' sums is, and their rows of
// partial sums fit a workspace (laid out without a device).
struct RowsGrid { int each, slots, blocks; };
inline RowsGrid rows_grid(int N, int C, int es, bool backward)
{
    RowsGrid g;
    const int per = C * es / 16;
    g.each = per < T ? T / per : 1;
    g.slots = (per + T - 1) / T;
    const int want = (N + g.each - 1) / g.each, most = B200_SMS * (backward ? CTAS_BWD : 8) / g.slots;
    g.blocks = want < most ? want : most > 0 ? most : 1;
    return g;
}
__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    for (int o = lanes / 2; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}
template <int V> __device__ __forceinline__ void load_floats(const float* p, int c, float other, f2 (&v)[V / 2])
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const float4 w = p ? __ldg(reinterpret_cast<const float4*>(p + c + i)) : make_float4(other, other, other, other);
        v[i / 2] = pair(w.x, w.y);
        v[i / 2 + 1] = pair(w.z, w.w);
    }
}

template <typename X>
__global__ void __launch_bounds__(T) rows_forward(const __grid_constant__ Args a, const int each)
{
    constexpr int V = 16 / (int)sizeof(X), VP = V / 2, U = 2;
    const int per = a.C / V, lanes = a.D / V, sub = each > 1 ? (int)threadIdx.x / per : 0;
    const int q = each > 1 ? (int)threadIdx.x - sub * per : (int)(blockIdx.y * T + threadIdx.x);
    const bool mine = sub < each && q < per;
    const int c = mine ? q * V : 0, g = c / a.D;
    pdl_wait();
    pdl_launch();
    f2 w[VP], b[VP];
    load_floats<V>(a.gamma, c, 1.0f, w);
    load_floats<V>(a.beta, c, 0.0f, b);
    const float inv = a.inv_count;
    const X* x = static_cast<const X*>(a.x);
    X* y = static_cast<X*>(a.out);
    for (long long r0 = (long long)blockIdx.x * each; r0 < a.N; r0 += (long long)gridDim.x * each * U) {
        uint4 raw[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + sub + (long long)u * gridDim.x * each;
            on[u] = mine && r < a.N;
            raw[u] = on[u] ? *reinterpret_cast<const uint4*>(x + r * a.C + c) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + sub + (long long)u * gridDim.x * each;
            Pairs<V> f;
            unpack2(raw[u], f, X());
            f2 s = f.v[0];
#pragma unroll
            for (int i = 1; i < VP; ++i) s = add2(s, f.v[i]);
            const float mean = lanes_sum(s.x() + s.y(), lanes) * inv;
            f2 ss = both(0.0f);
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                f.v[i] = add2(f.v[i], both(-mean));
                ss = fma2(f.v[i], f.v[i], ss);
            }
            const float rstd = __fdiv_rn(1.0f, __fsqrt_rn(lanes_sum(ss.x() + ss.y(), lanes) * inv + a.eps));
            if (!on[u]) continue;
            if (q % lanes == 0) {
                if (a.mean_out) a.mean_out[r * a.G + g] = mean;
                if (a.rstd_out) a.rstd_out[r * a.G + g] = rstd;
            }
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                f2 z = fma2(f.v[i], mul2(w[i], both(rstd)), b[i]);
                if (a.act == WCC_ACT_RELU) z = pair(z.x() < 0.0f ? 0.0f : z.x(), z.y() < 0.0f ? 0.0f : z.y());
                else if (a.act == WCC_ACT_SILU) z = silu2(z);
                f.v[i] = z;
            }
            *reinterpret_cast<uint4*>(y + r * a.C + c) = pack2(f, X());
        }
    }
}

template <typename X, bool KEPT>
__global__ void __launch_bounds__(T, CTAS_BWD) rows_backward(const __grid_constant__ Args a, const int each)
{
    constexpr int V = 16 / (int)sizeof(X), VP = V / 2;
    __shared__ float sums[2][T * V];
    const int per = a.C / V, lanes = a.D / V, sub = each > 1 ? (int)threadIdx.x / per : 0;
    const int q = each > 1 ? (int)threadIdx.x - sub * per : (int)(blockIdx.y * T + threadIdx.x);
    const bool mine = sub < each && q < per;
    const int c = mine ? q * V : 0, g = c / a.D;
    pdl_wait();
    pdl_launch();
    f2 w[VP], b[VP], s0[VP], s1[VP];
    load_floats<V>(a.gamma, c, 1.0f, w);
    load_floats<V>(a.beta, c, 0.0f, b);
#pragma unroll
    for (int i = 0; i < VP; ++i) s0[i] = s1[i] = both(0.0f);
    const float inv = a.inv_count;
    const X *x = static_cast<const X*>(a.x), *dy = static_cast<const X*>(a.dy);
    X* out = static_cast<X*>(a.out);
    for (long long r0 = (long long)blockIdx.x * each; r0 < a.N; r0 += (long long)gridDim.x * each) {
        const long long r = r0 + sub;
        const bool on = mine && r < a.N;
        const long long at = on ? r * a.C + c : 0, stat = on ? r * a.G + g : 0;
        Pairs<V> xc, t;
        const uint4 d = on ? *reinterpret_cast<const uint4*>(dy + at) : make_uint4(0u, 0u, 0u, 0u);
        const float mean = on ? __ldg(a.mean + stat) : 0.0f, rstd = on ? __ldg(a.rstd + stat) : 0.0f;
        if constexpr (KEPT) {
            const float sc = on ? __ldg(a.scales + r * a.nb + c / ck::BLOCK) : 0.0f;
            if constexpr (V == 8) {
                const uint2 k = on ? *reinterpret_cast<const uint2*>(a.codes + at) : make_uint2(0u, 0u);
                codes4(k.x, xc.v[0], xc.v[1]);
                codes4(k.y, xc.v[2], xc.v[3]);
            } else {
                codes4(on ? *reinterpret_cast<const uint32_t*>(a.codes + at) : 0u, xc.v[0], xc.v[1]);
            }
#pragma unroll
            for (int i = 0; i < VP; ++i) xc.v[i] = fma2(xc.v[i], both(sc), both(-mean));
        } else {
            unpack2(on ? *reinterpret_cast<const uint4*>(x + at) : make_uint4(0u, 0u, 0u, 0u), xc, X());
#pragma unroll
            for (int i = 0; i < VP; ++i) xc.v[i] = add2(xc.v[i], both(-mean));
        }
        unpack2(d, t, X());
        f2 c1 = both(0.0f), c2 = both(0.0f);
#pragma unroll
        for (int i = 0; i < VP; ++i) {
            xc.v[i] = mul2(xc.v[i], both(rstd));                       // xh
            if (a.act != WCC_ACT_NONE) {
                const f2 z = fma2(xc.v[i], w[i], b[i]);
                if (a.act == WCC_ACT_RELU) {
                    t.v[i] = pair(z.x() > 0.0f ? t.v[i].x() : 0.0f, z.y() > 0.0f ? t.v[i].y() : 0.0f);
                } else {
                    t.v[i] = mul2(t.v[i], silu_slope2(z, sigmoid2(z)));
                }
            }
            s0[i] = add2(s0[i], t.v[i]);
            s1[i] = fma2(t.v[i], xc.v[i], s1[i]);
            t.v[i] = mul2(t.v[i], w[i]);
            c1 = add2(c1, t.v[i]);
            c2 = fma2(t.v[i], xc.v[i], c2);
        }
        const float m1 = lanes_sum(c1.x() + c1.y(), lanes) * inv, m2 = lanes_sum(c2.x() + c2.y(), lanes) * inv;
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < VP; ++i) t.v[i] = mul2(both(rstd), add2(t.v[i], fma2(xc.v[i], both(-m2), both(-m1))));
        *reinterpret_cast<uint4*>(out + at) = pack2(t, X());
    }
    if (!a.params) return;
    // the CTA's sums of a channel, rows side by side in order
#pragma unroll
    for (int i = 0; i < VP; ++i) {
        const int k = threadIdx.x * V + 2 * i;
        sums[0][k] = s0[i].x(); sums[0][k + 1] = s0[i].y();
        sums[1][k] = s1[i].x(); sums[1][k + 1] = s1[i].y();
    }
    __syncthreads();
    float* row = a.img + (long long)blockIdx.x * a.img_row;
    const int wide = each > 1 ? a.C : min(T * V, a.C - (int)blockIdx.y * T * V), first = each > 1 ? 0 : (int)blockIdx.y * T * V;
    for (int k = threadIdx.x; k < wide; k += T) {
        float v0 = 0.0f, v1 = 0.0f;
        for (int e = 0; e < each; ++e) {
            v0 += sums[0][e * a.C + k];
            v1 += sums[1][e * a.C + k];
        }
        row[a.img_beta + first + k] = v0;
        row[a.img_gamma + first + k] = v1;
    }
}

// dbeta and dgamma from the rows of partial sums, 32 columns a block, rows in order of a warp's number.
static __global__ void __launch_bounds__(256) reduce_kernel(const float* __restrict__ img, int rows, int C, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float s[8][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    pdl_wait();
    pdl_launch();
    float v = 0.0f;
    if (c < 2 * C)
#pragma unroll 4
        for (int r = warp; r < rows; r += 8) v += __ldcg(img + (size_t)r * 2 * C + c);
    s[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && c < 2 * C) {
        for (int k = 1; k < 8; ++k) v += s[k][lane];
        float* dst = c < C ? dbeta : dgamma;
        if (dst) dst[c < C ? c : c - C] = v;
    }
}

// ---- host ------------------------------------------------------------------------------------------
template <typename X, int V, bool ALIGNED>
wcc_status launch_forward(const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    const Plan& q = a.q;
    const int words = (q.slots > 1 ? q.p : q.reps * q.p) * (ALIGNED ? 1 : V);
    size_t smem = (size_t)words * sizeof(Part) + (q.solo ? (size_t)a.G * 8 : 0);
    if (smem < (size_t)a.G * 8) smem = (size_t)a.G * 8;
    if (smem > 48 * 1024) {
        const wcc_status s = allow_smem<forward_kernel<X, V, ALIGNED>>(di.dev, (int)smem);
        if (s != WCC_OK) return s;
    }
    return launch_overlapped(forward_kernel<X, V, ALIGNED>, dim3((unsigned)grid_of(q, a.N, di.sms, false)), dim3(T), smem, st, true, 1, a);
}
template <typename X>
wcc_status forward(const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    const Plan& q = a.q;
    if (rows_path(a.P, a.C, a.G, (int)sizeof(X), false)) {
        const RowsGrid g = rows_grid(a.N, a.C, (int)sizeof(X), false);
        return launch_overlapped(rows_forward<X>, dim3((unsigned)g.blocks, (unsigned)g.slots), dim3(T), 0, st, true, 1, a, g.each);
    }
    if constexpr (sizeof(X) == 2)
        if (q.V == 8) return q.aligned ? launch_forward<X, 8, true>(a, di, st) : launch_forward<X, 8, false>(a, di, st);
    if (q.V == 4) return q.aligned ? launch_forward<X, 4, true>(a, di, st) : launch_forward<X, 4, false>(a, di, st);
    if (q.V == 2) return q.aligned ? launch_forward<X, 2, true>(a, di, st) : launch_forward<X, 2, false>(a, di, st);
    return launch_forward<X, 1, true>(a, di, st);
}
template <typename X, int V, bool KEPT>
wcc_status launch_backward(const Args& a, const DeviceInfo& di, int grid, cudaStream_t st)
{
    const Plan& q = a.q;
    const size_t smem = (size_t)(2 * a.C + 2 * a.G + (q.solo ? 2 * a.C : 0) + (q.slots == 1 ? 2 * q.reps * q.p * V : 0)) * 4;
    if (smem > 48 * 1024) {
        const wcc_status s = allow_smem<backward_kernel<X, V, KEPT>>(di.dev, (int)smem);
        if (s != WCC_OK) return s;
    }
    return launch_overlapped(backward_kernel<X, V, KEPT>, dim3((unsigned)grid), dim3(T), smem, st, true, 1, a);
}
template <typename X>
wcc_status backward(const Args& a, const DeviceInfo& di, int grid, cudaStream_t st)
{
    const Plan& q = a.q;
    const bool kept = a.x == nullptr;
    if (rows_path(a.P, a.C, a.G, (int)sizeof(X), kept)) {
        const RowsGrid g = rows_grid(a.N, a.C, (int)sizeof(X), true);
        return launch_overlapped(kept ? rows_backward<X, true> : rows_backward<X, false>, dim3((unsigned)g.blocks, (unsigned)g.slots), dim3(T), 0, st, true, 1, a, g.each);
    }
    if constexpr (sizeof(X) == 2)
        if (q.V == 8) return kept ? launch_backward<X, 8, true>(a, di, grid, st) : launch_backward<X, 8, false>(a, di, grid, st);
    if (q.V == 4) return kept ? launch_backward<X, 4, true>(a, di, grid, st) : launch_backward<X, 4, false>(a, di, grid, st);
    if (q.V == 2) return kept ? launch_backward<X, 2, true>(a, di, grid, st) : launch_backward<X, 2, false>(a, di, grid, st);
    return kept ? launch_backward<X, 1, true>(a, di, grid, st) : launch_backward<X, 1, false>(a, di, grid, st);
}

}  // namespace gn
}  // namespace wcc
