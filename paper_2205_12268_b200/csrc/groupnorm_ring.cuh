// Group norm of images of many tiles, fed by a ring in shared memory.
//
// One thread of a CTA takes tickets and brings the tiles' vectors in by bulk copies, chunk by chunk, as far ahead as the ring has room: across the ends of
// tiles, where the other 256 threads add up sums and hand them on.  So the memory stays busy meanwhile (48 to 96 KB in flight a CTA, two CTAs an SM),
// and the threads' registers hold constants and sums, not loads.
//
// The list of tiles has three kinds of items.  Step i of it: the sums of tile i; the result of tile i - delay; and, `gap` tiles behind the last sums of
// an image, `fin` items that each finish the sums of a share of its groups.  The gap is about the number of tiles of sums that are in flight, so an item
// seldom waits for what it needs, and the delay is as short as that allows, so that the second reading finds the map in L2.  Every item waits for items in
// front of it in the list only, and a CTA takes a ticket only shortly before it can use it: whichever CTAs are resident finish.
// A tile of sums ends with one barrier (the threads' sums are in shared memory), then each of the eight warps stores those of its share of the groups and
// counts itself done.  What the last kind of item needs of a group is one word of 64 bits, which is zero until it is there (coded so that no result is zero).
//
// Every wait has a limit, the meetings of the 256 threads among them (an mbarrier, not bar.sync): a warp whose wait ran out says so, and the others give up at
// their next wait, wherever they are.  What the threads of a warp do next goes by a vote, what the 256 do by a word that one of them wrote before they meet.
// Whoever leaves early stays until copies that are on their way have landed.
//
// Vectors are the aligned 16 bytes of the whole tensor.  An image that starts or ends inside one has up to V - 1 values at either end that
// belong to no vector of its own; they are the first and the last tile's edges, gone through one by one.
#pragma once

#include <type_traits>

#include "feed.h"
#include "groupnorm.cuh"

namespace wcc {
namespace gn {

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// The T threads that compute meet: false if this or another wait of the CTA ran out (the same on all lanes of a warp, not on all warps).
struct Meeting {
    uint32_t bar, parity;
    volatile int* abort_flag;
    __device__ __forceinline__ bool operator()()
    {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) tc::mbar_arrive(bar);
        const bool ok = tc::mbar_wait(bar, parity, abort_flag);
        parity ^= 1u;
        return __all_sync(0xFFFFFFFFu, ok);
    }
};
// A wait of this thread ran out, or another one's: the CTA stays until copies that are on their way have landed.
__device__ __noinline__ void give_up(volatile int* abort_flag, int* status)
{
    *abort_flag = 1;
    atomicExch(status, (int)WCC_ERR_TIMEOUT);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
}

// A group's two numbers as a word that is never zero: arithmetic gives no NaN of this pattern.
constexpr unsigned NONE = 0xFFE5A5A5u;
__device__ __forceinline__ void put_coef(float2* p, float a, float b)
{
    const unsigned ua = (a != a ? 0x7FFFFFFFu : __float_as_uint(a)) ^ NONE, ub = (b != b ? 0x7FFFFFFFu : __float_as_uint(b)) ^ NONE;
    asm volatile("st.relaxed.gpu.global.v2.u32 [%0], {%1, %2};" ::"l"(p), "r"(ua), "r"(ub) : "memory");
}
__device__ __forceinline__ unsigned long long load_coef(const float2* p)
{
    unsigned long long w;
    asm volatile("ld.relaxed.gpu.global.u64 %0, [%1];" : "=l"(w) : "l"(p) : "memory");
    return w;
}
__device__ __forceinline__ bool is_there(unsigned long long w) { return (unsigned)w != 0u && (unsigned)(w >> 32) != 0u; }
__device__ __forceinline__ float2 decode(unsigned long long w) { return make_float2(__uint_as_float((unsigned)w ^ NONE), __uint_as_float((unsigned)(w >> 32) ^ NONE)); }

// One chunk: where its image's whole vectors start, its first vector, its vectors; the image, the tile and its end; values at the image's ends; its first
// row among all images' (checkpoints).
struct Head { long long base; int v0, nvec, n, tile, vend, flags, front, back; long long row; };
enum { HEAD_APPLY = 1, HEAD_FIRST = 2, HEAD_LAST = 4, HEAD_END = 8, HEAD_FINISH = 16 };

// The list of items.  Items in front of step i: sums, results, and those that finish an image's sums, which stand at the end of a step.
__device__ __forceinline__ unsigned items_before(const Args& a, unsigned i)
{
    const Plan& q = a.q;
    const unsigned all = (unsigned)a.N * q.nt, done = i > (unsigned)q.gap ? min((i - q.gap) / q.nt, (unsigned)a.N) : 0u;
    return min(i, all) + (i > (unsigned)q.delay ? min(i - q.delay, all) : 0u) + q.fin * done;
}
struct Work { int n, tile, flags; };                                // a finishing item: tile is its share
__device__ __forceinline__ Work work_of(const Args& a, unsigned ticket)
{
    const Plan& q = a.q;
    const unsigned all = (unsigned)a.N * q.nt;
    unsigned lo = 0, hi = all + q.delay;                            // the last step with no more than `ticket` items in front of it
    while (hi - lo > 1) {
        const unsigned mid = lo + (hi - lo) / 2;
        if (items_before(a, mid) <= ticket) lo = mid;
        else hi = mid;
    }
    unsigned k = ticket - items_before(a, lo);
    if (lo < all && k-- == 0) return {(int)(lo / q.nt), (int)(lo % q.nt), 0};
    if (lo >= (unsigned)q.delay && k-- == 0) return {(int)((lo - q.delay) / q.nt), (int)((lo - q.delay) % q.nt), HEAD_APPLY};
    return {(int)((lo + 1 - q.gap) / q.nt) - 1, (int)k, HEAD_FINISH};
}

template <typename X, bool BWD, bool KEPT> struct Ring {
    static constexpr int V = 16 / (int)sizeof(X);
    // Vectors of a thread and chunk: waiting for a chunk, reading its head and letting it go cost as much as two vectors.  (us, backward, two a chunk / as
    // many as here: 12 x 96 x 320 x 64 fp32 95 / 86, 4 x 128 x 128 x 1024 bf16 148 / 136, from the checkpoint 198 / 156.)
    static constexpr int K = BWD ? 4 : 6;
    // and those whose instructions stand one after the other (a checkpoint's scales have to: they sit in registers)
    static constexpr int UNROLL = KEPT ? K : 2;
    static constexpr int X_BYTES = KEPT ? K * T * V : K * T * 16;
    static constexpr int BYTES = X_BYTES + (BWD ? K * T * 16 : 0);
};

constexpr int POSTS = 4;               // tiles whose sums are stored and not yet counted

struct RingCtl {
    uint64_t full[8], empty[8], stored[POSTS], meeting;
    int post[POSTS], posted;           // images of those tiles (-1: no more), tiles counted so far
    Head head[8];
    int abort, go;                     // a wait ran out; the sums to be finished are all there
    float partial[T];
};

// Finishes share `part_of` of image n's groups: all 256 threads.  scratch: room for the sums of a share's channels.  False: given up.
template <bool BWD> __device__ __forceinline__ bool finish(const Args& a, int n, int part_of, float* scratch, float* partial, Meeting& meet)
{
    const Plan& q = a.q;
    const int lo = (int)((long long)a.G * part_of / q.fin), hi = (int)((long long)a.G * (part_of + 1) / q.fin);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // loads that wait for one another cost a microsecond each while the memory is busy: as many as there are registers for go out together
    if constexpr (!BWD) {
        const float* all = a.part + (size_t)n * q.nt * a.G * 3;
        constexpr int U = 6;
        for (int g = lo + warp; g < hi; g += T / 32) {
            // the mean of the tiles' means, then the squared deviations from it; the tiles' numbers stay in registers if they fit
            Stat w[U];
            auto load = [&](int t0) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int t = t0 + 32 * u;
                    const float* p = all + ((size_t)t * a.G + g) * 3;
                    w[u] = t < q.nt ? Stat{__ldcg(p), __ldcg(p + 1), __ldcg(p + 2)} : Stat{0.0f, 0.0f, 0.0f};
                }
            };
            float ref = 0.0f, sum = 0.0f, m2 = 0.0f;
            Stat st{0.0f, 0.0f, 0.0f};
            for (int t0 = lane; t0 - lane < q.nt; t0 += 32 * U) {
                load(t0);
                if (t0 == lane) ref = __shfl_sync(0xFFFFFFFFu, w[0].mean, 0);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    st.n += w[u].n;
                    if (w[u].n > 0.0f) sum = __fmaf_rn(w[u].n, w[u].mean - ref, sum);
                }
            }
            st.n = warp_sum(st.n);
            sum = warp_sum(sum);
            st.mean = ref + __fdividef(sum, st.n);
            for (int t0 = lane; t0 - lane < q.nt; t0 += 32 * U) {
                if (q.nt > 32 * U) load(t0);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float d = w[u].mean - st.mean;
                    if (w[u].n > 0.0f) m2 += __fmaf_rn(w[u].n * d, d, w[u].m2);
                }
            }
            st.m2 = warp_sum(m2);
            if (lane == 0) {
                const float r = __fdiv_rn(1.0f, __fsqrt_rn(st.m2 * a.inv_count + a.eps));
                put_coef(a.coef + (size_t)n * a.G + g, st.mean, r);
                if (a.mean_out) a.mean_out[(size_t)n * a.G + g] = st.mean;
                if (a.rstd_out) a.rstd_out[(size_t)n * a.G + g] = r;
            }
        }
    } else {
        // columns: the sums of t, then of t (x - mean), of the share's channels; several threads a column where there are few
        const int c_lo = lo * a.D, cs = (hi - lo) * a.D, cols = 2 * cs;
        const float* part = a.part + (size_t)n * q.nt * 2 * a.C + c_lo;
        const int split = cols < T ? T / cols : 1, mine = split > 1 ? (int)threadIdx.x / cols : 0, col0 = (int)threadIdx.x - mine * cols;
        // the first group's numbers, on their way meanwhile
        const int g0 = lo + warp < hi ? lo + warp : lo;
        const float r0 = __ldg(a.rstd + (size_t)n * a.G + g0), w0 = a.gamma && lane < a.D ? __ldg(a.gamma + g0 * a.D + lane) : 1.0f;
        constexpr int U = 16;
        if (mine < split) {
            for (int col = col0; col < cols; col += T) {
                const float* p = part + (col < cs ? col : a.C + col - cs);
                float v = 0.0f;
                for (int t0 = mine; t0 < q.nt; t0 += split * U) {
                    float w[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) w[u] = t0 + u * split < q.nt ? __ldcg(p + (size_t)(t0 + u * split) * 2 * a.C) : 0.0f;
#pragma unroll
                    for (int u = 0; u < U; ++u) v += w[u];
                }
                if (split > 1) partial[mine * cols + col] = v;
                else scratch[col] = v;
            }
        }
        if (!meet()) return false;
        if (split > 1) {
            for (int col = threadIdx.x; col < cols; col += T) {
                float v = partial[col];
                for (int k = 1; k < split; ++k) v += partial[k * cols + col];
                scratch[col] = v;
            }
            if (!meet()) return false;
        }
        for (int g = lo + warp; g < hi; g += T / 32) {
            float c1 = 0.0f, c2 = 0.0f;
            const float r = g == g0 ? r0 : __ldg(a.rstd + (size_t)n * a.G + g);
            for (int d = lane; d < a.D; d += 32) {
                const int ch = g * a.D + d;
                const float w = !a.gamma ? 1.0f : g == g0 && d == lane ? w0 : __ldg(a.gamma + ch), v1 = scratch[ch - c_lo], v2 = scratch[cs + ch - c_lo];
                c1 = __fmaf_rn(w, v1, c1);
                c2 = __fmaf_rn(w, v2, c2);
                if (a.params) {
                    float* row = a.img + n * a.img_row;
                    row[a.img_beta + ch] = v1;
                    row[a.img_gamma + ch] = r * v2;
                }
            }
            c1 = warp_sum(c1);
            c2 = warp_sum(c2);
            if (lane == 0) {
                const float2 k = terms_of(a, r, c1, c2);
                put_coef(a.coef + (size_t)n * a.G + g, k.x, k.y);
            }
        }
    }
    return true;
}

template <typename X, bool ALIGNED, bool BWD, bool KEPT>
__global__ void __launch_bounds__(T + 64, 2) ring_kernel(const __grid_constant__ Args a, const int stages)
{
    using R = Ring<X, BWD, KEPT>;
    constexpr int V = R::V, K = R::K, VP = V / 2;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ RingCtl c;
    const Plan& q = a.q;
    const uint32_t ring = tc::smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { tc::mbar_init(tc::smem_u32(&c.full[s]), 1); tc::mbar_init(tc::smem_u32(&c.empty[s]), T / 32); }
        for (int i = 0; i < POSTS; ++i) { tc::mbar_init(tc::smem_u32(&c.stored[i]), T / 32); c.post[i] = -1; }
        tc::mbar_init(tc::smem_u32(&c.meeting), T / 32);
        c.abort = 0;
        c.posted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_launch();
    const int step = q.reps * q.p, chunk = K * step;
    volatile int* abort_flag = &c.abort;

    if (warp == T / 32) {
        // ---- the thread that feeds the ring
        if (lane != 0) return;
        const unsigned items = (unsigned)a.N * (2u * q.nt + q.fin);
        const long long E = (long long)a.P * a.C;
        int s = 0, sent = 0;                                       // stage of the next chunk, chunks sent
        uint32_t ph = 1;
        for (;;) {
            const unsigned ticket = atomicAdd(a.ctl, 1u);
            const bool end = ticket >= items || *abort_flag;
            const int first = sent;
            const Work it = end ? Work{0, 0, HEAD_END} : work_of(a, ticket);
            const bool loads = !(it.flags & (HEAD_END | HEAD_FINISH));
            // the image's values in front of its first whole vector, its whole vectors, the values behind them
            const long long at = it.n * E;
            const int front = (int)((V - at % V) % V), nvec = (int)((E - front) / V), back = (int)(E - front - (long long)nvec * V);
            int v = it.tile * q.tile;
            const int vend = min(v + q.tile, nvec);
            int flags = HEAD_FIRST | it.flags;
            for (;;) {
                if (!tc::mbar_wait(tc::smem_u32(&c.empty[s]), ph, abort_flag)) { give_up(abort_flag, a.status); return; }
                const int n = loads && vend > v ? min(vend - v, chunk) : 0;
                if (!loads || v + n >= vend) flags |= HEAD_LAST;
                c.head[s] = {at + front, v, n, it.n, it.tile, vend, flags, it.tile == 0 ? front : 0, it.tile == q.nt - 1 ? back : 0,
                             KEPT ? (long long)it.n * a.P + v / q.p : 0};
                const uint32_t bar = tc::smem_u32(&c.full[s]), dst = ring + (uint32_t)(s * R::BYTES);
                const uint32_t xb = (uint32_t)(KEPT ? n * V : n * 16), db = (uint32_t)(n * 16);
                tc::mbar_expect_tx(bar, xb + (BWD ? db : 0u));
                if (n > 0) {
                    const long long e = at + front + (long long)v * V;
                    if constexpr (KEPT) bulk_load(dst, a.codes + e, xb, bar);
                    else bulk_load(dst, static_cast<const X*>(a.x) + e, xb, bar);
                    if constexpr (BWD) bulk_load(dst + R::X_BYTES, static_cast<const X*>(a.dy) + e, db, bar);
                }
                if (++s == stages) { s = 0; ph ^= 1u; }
                ++sent;
                if (flags & HEAD_LAST) break;
                flags &= ~HEAD_FIRST;
                v += n;
            }
            if (end) {
                if (*abort_flag) give_up(abort_flag, a.status);
                return;
            }
            const int w = awaited_chunk(first, sent, stages);
            if (w >= 0 && !tc::mbar_wait(tc::smem_u32(&c.empty[w % stages]), (uint32_t)(w / stages) & 1u, abort_flag)) { give_up(abort_flag, a.status); return; }
        }
    }

    if (warp == T / 32 + 1) {
        // ---- the thread that counts stored sums.  The fence in front of the count waits for all stores that are on their way, results of other tiles
        // among them, some microseconds: not to be done by those who compute.
        if (lane != 0) return;
        for (int t = 0;; ++t) {
            if (!tc::mbar_wait(tc::smem_u32(&c.stored[t % POSTS]), (uint32_t)(t / POSTS) & 1u, abort_flag)) { give_up(abort_flag, a.status); return; }
            const int n = c.post[t % POSTS];
            if (n < 0) return;
            asm volatile("fence.acq_rel.gpu;" ::: "memory");
            atomicAdd(a.ctl + 1 + n, 1u);
            *const_cast<volatile int*>(&c.posted) = t + 1;
        }
    }

    // ---- the threads that compute
    const int sub = threadIdx.x / q.lanes, vq = threadIdx.x - sub * q.lanes, width = q.p * V;
    const bool active = sub < q.reps;
    const int v_mine = sub * q.p + vq;
    const X* x = static_cast<const X*>(a.x);
    const X* dy = static_cast<const X*>(a.dy);
    X* out = static_cast<X*>(a.out);
    // sums of a tile, two buffers in turn.  Forward: a Stat for each vector, or each value; backward: [2][rows][p V]
    const bool fold = BWD && q.p < 32 && 32 % q.p == 0;            // lanes of a warp that share channels are added up first
    const int rows = fold ? T / 32 : q.reps;
    constexpr int W = ALIGNED ? V : 1;
    uint8_t* const buffers = smem + (size_t)stages * R::BYTES;
    const size_t buffer_bytes = BWD ? (size_t)2 * T * V * 4 : (size_t)T * (V / W) * sizeof(Stat);
    int buffer = 0;
    // this warp's share of the groups
    const int g_lo = a.G * warp / (T / 32), g_hi = a.G * (warp + 1) / (T / 32);
    const int scale_block = vq * V / ck::BLOCK;
    const int c_first = ALIGNED ? vq * V : 0, g_first = ALIGNED ? a.dD.div(c_first) : 0;

    f2 mean[ALIGNED ? 1 : VP];                                 // minus the mean of the channels
    Pairs<V> k, b;                                                 // rstd gamma, beta; forward, not ALIGNED, sums: k holds the pivots
    Pairs<V> s1, s2;                                               // backward: sums of t and t (x - mean); forward: of deviations and their squares
    f2 k0[ALIGNED ? 1 : VP], k1[ALIGNED ? 1 : VP];                 // backward, apply: dx = k t + k1 (x - mean) + k0
    float pivot = 0.0f;
    int count = 0;
    float scale[K];

    Meeting meet{tc::smem_u32(&c.meeting), 0u, abort_flag};
    // the warp's part of a tile's sums is stored (n: its image; -1: there are no more tiles); false: given up, nothing is counted
    int posts = 0;
    auto post = [&](int n) {
        __syncwarp();
        bool room = true;
        if (lane == 0) {
            const uint32_t limit = tc::c_wait_limit;
            room = posts - *const_cast<volatile int*>(&c.posted) < POSTS;
            for (uint32_t i = 0; i < limit && !room && !*abort_flag; ++i) {
                __nanosleep(64);
                room = posts - *const_cast<volatile int*>(&c.posted) < POSTS;
            }
            if (room) {
                if (warp == 0) c.post[posts % POSTS] = n;
                tc::mbar_arrive(tc::smem_u32(&c.stored[posts % POSTS]));
            }
        }
        ++posts;
        return __all_sync(0xFFFFFFFFu, room) != 0;
    };
    int s = 0;
    uint32_t ph = 0;
    for (;;) {
        const bool here = tc::mbar_wait(tc::smem_u32(&c.full[s]), ph, abort_flag);
        if (!__all_sync(0xFFFFFFFFu, here)) { give_up(abort_flag, a.status); return; }
        const Head h = c.head[s];
        if (h.flags & HEAD_END) {
            if (!post(-1)) give_up(abort_flag, a.status);
            return;
        }
        const bool applying = (h.flags & HEAD_APPLY) != 0;
        // (asked for one chunk ahead)
        auto scales_of = [&](int ahead) {
            if constexpr (KEPT) {
                const float* p = a.scales + (h.row + ahead * (K * q.reps) + sub) * a.nb + scale_block;
#pragma unroll
                for (int u = 0; u < K; ++u)
                    scale[u] = active && h.v0 + ahead * chunk + u * step + v_mine < h.vend ? __ldg(p + (long long)(u * q.reps) * a.nb) : 0.0f;
            }
        };
        if (h.flags & HEAD_FINISH) {
            // everything of the stage is read: it holds nothing else
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(tc::smem_u32(&c.empty[s]));
            if (++s == stages) { s = 0; ph ^= 1u; }
            float* const scratch = reinterpret_cast<float*>(buffers + buffer * buffer_bytes);
            buffer ^= 1;
            if (threadIdx.x == 0) {
                bool ok = false;
                const uint32_t limit = tc::c_wait_limit;
                const unsigned want = (unsigned)q.nt;
                for (uint32_t i = 0; i < limit && !ok && !*abort_flag; ++i) {
                    ok = load_acquire(a.ctl + 1 + h.n) == want;
                    if (!ok) __nanosleep(64);
                }
                c.go = ok;
            }
            if (!meet() || !*const_cast<volatile int*>(&c.go) || !finish<BWD>(a, h.n, h.tile, scratch, c.partial, meet) || !meet()) { give_up(abort_flag, a.status); return; }
            continue;
        }
        if (h.flags & HEAD_FIRST) {
            scales_of(0);
            const float2* coef = a.coef + (size_t)h.n * a.G;
            const int shift = ALIGNED ? 0 : a.dC.mod((int)(h.base - (long long)h.n * a.P * a.C));
            // channel of value e of this thread's vectors
            auto channel_at = [&](int e) { return ALIGNED ? c_first + e : a.dC.mod(vq * V + e + shift); };
            if (applying) {
                // the image's sums are known: usually long since
                bool all = false;
                const uint32_t limit = tc::c_wait_limit;
                constexpr int NG = ALIGNED ? 1 : V;
                const float2* where[NG];
#pragma unroll
                for (int e = 0; e < NG; ++e) where[e] = coef + (ALIGNED ? g_first : a.dD.div(channel_at(e)));
                const float2* where_edge = coef;
                if (!ALIGNED && lane < h.front + h.back) {         // that of an edge too
                    const long long f = lane < h.front ? (long long)lane : (long long)a.P * a.C - h.back + (lane - h.front);
                    where_edge = coef + (int)(f % a.C) / a.D;
                }
                for (uint32_t i = 0; i < limit && !all && !__any_sync(0xFFFFFFFFu, *abort_flag != 0); ++i) {
                    if (!ALIGNED && !__all_sync(0xFFFFFFFFu, is_there(load_coef(where[0])))) { __nanosleep(256); continue; }
                    unsigned long long w[NG], we = ~0ull;          // (all on their way at once)
#pragma unroll
                    for (int e = 0; e < NG; ++e) w[e] = load_coef(where[e]);
                    if (!ALIGNED && h.front + h.back) we = load_coef(where_edge);
                    bool ok = is_there(we);
#pragma unroll
                    for (int e = 0; e < NG; ++e) ok = ok && is_there(w[e]);
#pragma unroll
                    for (int j = 0; j < (ALIGNED ? 1 : VP); ++j) {
                        const float2 p0 = decode(w[ALIGNED ? 0 : 2 * j]), p1 = ALIGNED ? p0 : decode(w[ALIGNED ? 0 : 2 * j + 1]);
                        k0[j] = pair(p0.x, p1.x);
                        k1[j] = pair(p0.y, p1.y);
                    }
                    all = __all_sync(0xFFFFFFFFu, ok);
                    if (!all) __nanosleep(128);
                }
                if (!all) { give_up(abort_flag, a.status); return; }
            }
            if (BWD || applying) {
                const float *mp = BWD ? a.mean + (size_t)h.n * a.G : nullptr, *rp = BWD ? a.rstd + (size_t)h.n * a.G : nullptr;
                if constexpr (ALIGNED) {
                    // one group, neighbouring channels
                    f2 m, r;
                    if constexpr (BWD) { m = both(-__ldg(mp + g_first)); r = both(__ldg(rp + g_first)); }
                    else { m = both(-k0[0].x()); r = k1[0]; }
                    mean[0] = m;
#pragma unroll
                    for (int i = 0; i < V; i += 4) {
                        const float4 w = a.gamma ? __ldg(reinterpret_cast<const float4*>(a.gamma + c_first + i)) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                        const float4 o = a.beta ? __ldg(reinterpret_cast<const float4*>(a.beta + c_first + i)) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        k.v[i / 2] = mul2(r, pair(w.x, w.y));
                        k.v[i / 2 + 1] = mul2(r, pair(w.z, w.w));
                        b.v[i / 2] = pair(o.x, o.y);
                        b.v[i / 2 + 1] = pair(o.z, o.w);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        const int c0 = channel_at(2 * i), c1 = channel_at(2 * i + 1);
                        f2 m, r;
                        if constexpr (BWD) {
                            const int g0 = a.dD.div(c0), g1 = a.dD.div(c1);
                            m = pair(-__ldg(mp + g0), -__ldg(mp + g1));
                            r = pair(__ldg(rp + g0), __ldg(rp + g1));
                        } else {
                            m = pair(-k0[i].x(), -k0[i].y());
                            r = k1[i];
                        }
                        mean[i] = m;
                        k.v[i] = a.gamma ? mul2(r, pair(__ldg(a.gamma + c0), __ldg(a.gamma + c1))) : r;
                        b.v[i] = a.beta ? pair(__ldg(a.beta + c0), __ldg(a.beta + c1)) : both(0.0f);
                    }
                }
            }
            if (!applying) {
#pragma unroll
                for (int i = 0; i < VP; ++i) s1.v[i] = s2.v[i] = both(0.0f);
            }
            count = 0;
        }
        const uint8_t* stage = smem + (size_t)s * R::BYTES;
        X* const dst = out + h.base + (long long)h.v0 * V;

        // one chunk: f(u, vector of the chunk) for each of this thread's vectors
        auto each = [&](auto f) {
#pragma unroll R::UNROLL
            for (int u = 0; u < K; ++u) {
                const int v = u * step + v_mine;
                if (active && v < h.nvec) f(u, v);
            }
        };
        auto centred = [&](int u, int v, Pairs<V>& xc) {           // x - mean
            if constexpr (KEPT) {
                const f2 sc = both(scale[u]);
                if constexpr (V == 8) {
                    const uint2 w = *reinterpret_cast<const uint2*>(stage + v * 8);
                    codes4(w.x, xc.v[0], xc.v[1]);
                    codes4(w.y, xc.v[2], xc.v[3]);
                } else {
                    codes4(*reinterpret_cast<const uint32_t*>(stage + v * 4), xc.v[0], xc.v[1]);
                }
#pragma unroll
                for (int i = 0; i < VP; ++i) xc.v[i] = fma2(xc.v[i], sc, mean[ALIGNED ? 0 : i]);
            } else {
                unpack2(*reinterpret_cast<const uint4*>(stage + v * 16), xc, X());
#pragma unroll
                for (int i = 0; i < VP; ++i) xc.v[i] = add2(xc.v[i], mean[ALIGNED ? 0 : i]);
            }
        };
        auto chunk_of = [&](auto tag, auto final) {
            constexpr int ACT = decltype(tag)::value;
            [[maybe_unused]] constexpr bool APPLY = decltype(final)::value;
            if constexpr (BWD) {
                each([&](int u, int v) {
                    Pairs<V> xc, t;
                    centred(u, v, xc);
                    unpack2(*reinterpret_cast<const uint4*>(stage + R::X_BYTES + v * 16), t, X());
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        if constexpr (ACT == WCC_ACT_RELU) {
                            const f2 z = fma2(xc.v[i], k.v[i], b.v[i]);
                            t.v[i] = pair(z.x() > 0.0f ? t.v[i].x() : 0.0f, z.y() > 0.0f ? t.v[i].y() : 0.0f);
                        } else if constexpr (ACT == WCC_ACT_SILU) {
                            const f2 z = fma2(xc.v[i], k.v[i], b.v[i]);
                            t.v[i] = mul2(t.v[i], silu_slope2(z, sigmoid2(z)));
                        }
                        if constexpr (!APPLY) {
                            s1.v[i] = add2(s1.v[i], t.v[i]);
                            s2.v[i] = fma2(t.v[i], xc.v[i], s2.v[i]);
                        } else {
                            t.v[i] = fma2(t.v[i], k.v[i], fma2(xc.v[i], k1[ALIGNED ? 0 : i], k0[ALIGNED ? 0 : i]));
                        }
                    }
                    if constexpr (APPLY) *reinterpret_cast<uint4*>(dst + v * V) = pack2(t, X());
                });
            } else {
                each([&](int u, int v) {
                    Pairs<V> f;
                    centred(u, v, f);
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        f.v[i] = fma2(f.v[i], k.v[i], b.v[i]);
                        if constexpr (ACT == WCC_ACT_RELU) f.v[i] = pair(f.v[i].x() < 0.0f ? 0.0f : f.v[i].x(), f.v[i].y() < 0.0f ? 0.0f : f.v[i].y());
                        else if constexpr (ACT == WCC_ACT_SILU) f.v[i] = silu2(f.v[i]);
                    }
                    *reinterpret_cast<uint4*>(dst + v * V) = pack2(f, X());
                });
            }
        };
        auto by_act = [&](auto final) {
            if (a.act == WCC_ACT_SILU) chunk_of(std::integral_constant<int, WCC_ACT_SILU>(), final);
            else if (a.act == WCC_ACT_RELU) chunk_of(std::integral_constant<int, WCC_ACT_RELU>(), final);
            else chunk_of(std::integral_constant<int, WCC_ACT_NONE>(), final);
        };
        if (applying) {
            by_act(std::true_type());
        } else if constexpr (BWD) {
            by_act(std::false_type());
        } else {
            if ((h.flags & HEAD_FIRST) && active && v_mine < h.nvec) {       // deviations are from the thread's first value, or its channels'
                Pairs<V> f;
                unpack2(*reinterpret_cast<const uint4*>(stage + v_mine * 16), f, X());
                pivot = f.v[0].x();
                if constexpr (!ALIGNED) k = f;
            }
            each([&](int u, int v) {
                Pairs<V> f;
                unpack2(*reinterpret_cast<const uint4*>(stage + v * 16), f, X());
                ++count;
#pragma unroll
                for (int i = 0; i < VP; ++i) {
                    if constexpr (ALIGNED) {
                        const f2 d = add2(f.v[i], both(-pivot));
                        s1.v[i & 1] = add2(s1.v[i & 1], d);
                        s2.v[i & 1] = fma2(d, d, s2.v[i & 1]);
                    } else {
                        const f2 d = fma2(k.v[i], both(-1.0f), f.v[i]);
                        s1.v[i] = add2(s1.v[i], d);
                        s2.v[i] = fma2(d, d, s2.v[i]);
                    }
                }
            });
        }
        if (!(h.flags & HEAD_LAST)) scales_of(1);
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(tc::smem_u32(&c.empty[s]));
        if (++s == stages) { s = 0; ph ^= 1u; }
        if (!(h.flags & HEAD_LAST)) continue;

        // ---- the end of a tile
        const int shift = ALIGNED ? 0 : a.dC.mod((int)(h.base - (long long)h.n * a.P * a.C));
        // the edge value that is this lane's: its place in the tensor and its channel
        const int edges = ALIGNED ? 0 : h.front + h.back;
        long long edge_at = 0;
        int edge_ch = -1;
        if (!ALIGNED && lane < edges) {
            const long long f = lane < h.front ? (long long)lane : (long long)a.P * a.C - h.back + (lane - h.front);
            edge_at = (long long)h.n * a.P * a.C + f;
            edge_ch = (int)(f % a.C);
        }
        const float2* const coef = a.coef + (size_t)h.n * a.G;
        if (applying) {
            if (!ALIGNED && warp == 0 && edge_ch >= 0) {
                const int g = edge_ch / a.D;
                const float2 cf = decode(load_coef(coef + g));
                const float w = a.gamma ? __ldg(a.gamma + edge_ch) : 1.0f, be = a.beta ? __ldg(a.beta + edge_ch) : 0.0f;
                float r[1];
                if constexpr (BWD) {
                    const float xc = (float)x[edge_at] - __ldg(a.mean + (size_t)h.n * a.G + g), kk = __ldg(a.rstd + (size_t)h.n * a.G + g) * w;
                    float z[1] = {__fmaf_rn(xc, kk, be)};
                    r[0] = (float)dy[edge_at];
                    if (a.act == WCC_ACT_SILU) slope_times<1, WCC_ACT_SILU>(z, r);
                    else if (a.act == WCC_ACT_RELU) slope_times<1, WCC_ACT_RELU>(z, r);
                    r[0] = __fmaf_rn(r[0], kk, __fmaf_rn(xc, cf.y, cf.x));
                } else {
                    r[0] = __fmaf_rn((float)x[edge_at] - cf.x, cf.y * w, be);
                    if (a.act == WCC_ACT_SILU) activate<1, WCC_ACT_SILU>(r);
                    else if (a.act == WCC_ACT_RELU) activate<1, WCC_ACT_RELU>(r);
                }
                out[edge_at] = (X)r[0];
            }
            continue;
        }
        uint8_t* const mine = buffers + buffer * buffer_bytes;
        buffer ^= 1;
        if constexpr (!BWD) {
            Stat* entries = reinterpret_cast<Stat*>(mine);
            if (active) {
                if constexpr (ALIGNED) {
                    const f2 sa = add2(s1.v[0], s1.v[1]), sb = add2(s2.v[0], s2.v[1]);
                    const float n = (float)(count * V), sum = sa.x() + sa.y(), m = count ? __fdividef(sum, n) : 0.0f;
                    // (a thread without a vector here has the pivot of another tile)
                    entries[v_mine] = {n, count ? pivot + m : 0.0f, fmaxf(sb.x() + sb.y() - sum * m, 0.0f)};
                } else {
                    const float n = (float)count;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float sum = e & 1 ? s1.v[e / 2].y() : s1.v[e / 2].x(), sq = e & 1 ? s2.v[e / 2].y() : s2.v[e / 2].x();
                        const float pv = count ? (e & 1 ? k.v[e / 2].y() : k.v[e / 2].x()) : 0.0f, m = count ? __fdividef(sum, n) : 0.0f;
                        entries[v_mine * V + e] = {n, pv + m, fmaxf(sq - sum * m, 0.0f)};
                    }
                }
            }
            if (!meet()) { give_up(abort_flag, a.status); return; }
            // The tile's groups: first the mean, then the squared deviations from it.  The group's channels among the entries: value f of a
            // period is channel (f + shift) mod C.
            Stat* part = reinterpret_cast<Stat*>(a.part) + ((size_t)h.n * q.nt + h.tile) * a.G;
            const int Cw = a.C / W, Dw = a.D / W, total = q.reps * q.copies * Dw;
            for (int g = g_lo; g < g_hi; ++g) {
                // (the rows of entries are `copies` times Cw wide: entry m is channel m mod Dw of the group in the (m / Dw)th stretch of Cw)
                auto entry = [&](int m) {
                    const int i = a.dW.div(m);
                    int f = g * Dw + (m - i * Dw) - shift;
                    if (f < 0) f += Cw;
                    return entries[i * Cw + f];
                };
                const float edge = !ALIGNED && edge_ch >= 0 && edge_ch / a.D == g ? 1.0f : 0.0f;
                const float edge_v = !ALIGNED && edge != 0.0f ? (float)x[edge_at] : 0.0f;
                const float ref = entry(0).mean;
                float n = edge, sum = edge != 0.0f ? edge_v - ref : 0.0f;
                for (int m = lane; m < total; m += 32) {
                    const Stat e = entry(m);
                    n += e.n;
                    sum = __fmaf_rn(e.n, e.mean - ref, sum);
                }
                n = warp_sum(n);
                sum = warp_sum(sum);
                const float mu = n > 0.0f ? ref + __fdividef(sum, n) : ref;
                float m2 = edge != 0.0f ? (edge_v - mu) * (edge_v - mu) : 0.0f;
                for (int m = lane; m < total; m += 32) {
                    const Stat e = entry(m);
                    const float d = e.mean - mu;
                    m2 += __fmaf_rn(e.n * d, d, e.m2);
                }
                m2 = warp_sum(m2);
                if (lane == 0) part[g] = {n, mu, m2};
            }
            if (!post(h.n)) { give_up(abort_flag, a.status); return; }
        } else {
            float* sums = reinterpret_cast<float*>(mine);
            const int second = rows * width;
            if (fold) {
                for (int o = 16; o >= q.p; o >>= 1) {
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        s1.v[i] = add2(s1.v[i], f2{__shfl_xor_sync(0xFFFFFFFFu, s1.v[i].w, o)});
                        s2.v[i] = add2(s2.v[i], f2{__shfl_xor_sync(0xFFFFFFFFu, s2.v[i].w, o)});
                    }
                }
            }
            if (fold ? lane < q.p : active) {
                const int row = (fold ? warp : sub) * width + vq * V;
#pragma unroll
                for (int i = 0; i < VP; ++i) {
                    *reinterpret_cast<unsigned long long*>(sums + row + 2 * i) = s1.v[i].w;
                    *reinterpret_cast<unsigned long long*>(sums + second + row + 2 * i) = s2.v[i].w;
                }
            }
            if (!meet()) { give_up(abort_flag, a.status); return; }
            float et = 0.0f, etx = 0.0f;
            if (!ALIGNED && edge_ch >= 0) {
                const int g = edge_ch / a.D;
                const float xc = (float)x[edge_at] - __ldg(a.mean + (size_t)h.n * a.G + g);
                float z[1] = {__fmaf_rn(xc, __ldg(a.rstd + (size_t)h.n * a.G + g) * (a.gamma ? __ldg(a.gamma + edge_ch) : 1.0f), a.beta ? __ldg(a.beta + edge_ch) : 0.0f)};
                float t[1] = {(float)dy[edge_at]};
                if (a.act == WCC_ACT_SILU) slope_times<1, WCC_ACT_SILU>(z, t);
                else if (a.act == WCC_ACT_RELU) slope_times<1, WCC_ACT_RELU>(z, t);
                et = t[0];
                etx = t[0] * xc;
            }
            const int c_lo = g_lo * a.D, c_n = (g_hi - g_lo) * a.D, copies = q.copies;
            float* part = a.part + ((size_t)h.n * q.nt + h.tile) * 2 * a.C;
            for (int i0 = 0; i0 < c_n; i0 += 32) {
                const int ch = c_lo + i0 + lane;
                const bool on = i0 + lane < c_n;
                int f = ch - shift;
                if (f < 0) f += a.C;
                float v1 = 0.0f, v2 = 0.0f;
                if (on) {
                    const int n = rows * copies;                   // (a row is `copies` times C wide)
#pragma unroll 8
                    for (int r = 0; r < n; ++r) {
                        v1 += sums[r * a.C + f];
                        v2 += sums[second + r * a.C + f];
                    }
                }
                if constexpr (!ALIGNED)
                    for (int i = 0; i < edges; ++i) {
                        const int ec = __shfl_sync(0xFFFFFFFFu, edge_ch, i);
                        const float e1 = __shfl_sync(0xFFFFFFFFu, et, i), e2 = __shfl_sync(0xFFFFFFFFu, etx, i);
                        if (ec == ch) { v1 += e1; v2 += e2; }
                    }
                if (on) {
                    part[ch] = v1;
                    part[a.C + ch] = v2;
                }
            }
            if (!post(h.n)) { give_up(abort_flag, a.status); return; }
        }
    }
}

template <typename X, bool ALIGNED, bool BWD, bool KEPT>
wcc_status launch_ring(const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    using R = Ring<X, BWD, KEPT>;
    const int extra = 2 * (BWD ? 2 * T * R::V * 4 : T * (ALIGNED ? 1 : R::V) * (int)sizeof(Stat));
    const int room = 111 * 1024 - (int)sizeof(RingCtl), most = (room - extra) / R::BYTES, stages = most < 3 ? most : 3, smem = stages * R::BYTES + extra;
    const wcc_status s = allow_smem<ring_kernel<X, ALIGNED, BWD, KEPT>>(di.dev, smem);
    if (s != WCC_OK) return s;
    const long long items = (long long)a.N * (2 * a.q.nt + a.q.fin), grid = 2LL * di.sms;
    return launch_overlapped(ring_kernel<X, ALIGNED, BWD, KEPT>, dim3((unsigned)(items < grid ? items : grid)), dim3(T + 64), (size_t)smem, st, true, 1, a, stages);
}
template <typename X> wcc_status ring_forward(const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    return a.q.aligned ? launch_ring<X, true, false, false>(a, di, st) : launch_ring<X, false, false, false>(a, di, st);
}
template <typename X> wcc_status ring_backward(const Args& a, const DeviceInfo& di, cudaStream_t st)
{
    if (a.x) return a.q.aligned ? launch_ring<X, true, true, false>(a, di, st) : launch_ring<X, false, true, false>(a, di, st);
    return a.q.aligned ? launch_ring<X, true, true, true>(a, di, st) : launch_ring<X, false, true, true>(a, di, st);
}

}  // namespace gn
}  // namespace wcc
