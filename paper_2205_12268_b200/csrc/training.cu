// C-ABI entry points of the operators for training around the layer (see include/wcc.h): group norm with an activation, 8-bit activation
// checkpoints, the gated pointwise block.  A translation unit of its own; device globals belong to libwcc.cu.
#define WCC_TRAINING_UNIT
#include "checkpoint.cuh"
#include "common.cuh"
#include "gated.cuh"
#include "groupnorm.cuh"
#include "groupnorm_ring.cuh"

namespace wcc {

wcc_status set_training_wait_limit(uint32_t polls)
{
    return cudaMemcpyToSymbol(tc::c_wait_limit, &polls, sizeof(polls)) == cudaSuccess ? WCC_OK : WCC_ERR_CUDA;
}

static bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
template <typename... P> static bool on16(const void* p, P... rest) { return on16(p) && on16(rest...); }

static wcc_status check_groupnorm(int N, int P, int C, int G, wcc_dtype dt, int act)
{
    if (N <= 0 || P <= 0 || C <= 0 || C > WCC_MAX_CHANNELS || G <= 0 || C % G != 0) return WCC_ERR_SHAPE;
    if ((long long)N * P > (1LL << 30) || (long long)N * P * C > (1LL << 40)) return WCC_ERR_SHAPE;
    if (act != WCC_ACT_NONE && act != WCC_ACT_RELU && act != WCC_ACT_SILU) return WCC_ERR_SHAPE;
    if (dt != WCC_F32 && dt != WCC_BF16) return WCC_ERR_DTYPE;
    return WCC_OK;
}

static gn::Args groupnorm_args(int N, int P, int C, int G, int act, const gn::Plan& q, const gn::Layout& l, void* ws, const DeviceInfo& di)
{
    gn::Args a{};
    char* w = static_cast<char*>(ws);
    a.N = N; a.P = P; a.C = C; a.G = G; a.D = C / G; a.nb = ceil_div(C, ck::BLOCK); a.act = act;
    a.inv_count = (float)(1.0 / ((double)P * a.D));
    a.q = q;
    a.dC = gn::divisor_of((unsigned)C);
    a.dD = gn::divisor_of((unsigned)a.D);
    a.dW = gn::divisor_of((unsigned)(q.aligned ? a.D / q.V : a.D));
    a.ctl = reinterpret_cast<unsigned*>(w + l.ctl);
    a.part = reinterpret_cast<float*>(w + l.part);
    a.sup = reinterpret_cast<float*>(w + l.sup);
    a.img = reinterpret_cast<float*>(w + l.img);
    a.coef = reinterpret_cast<float2*>(w + l.coef);
    a.status = di.status;
    return a;
}

static wcc_status check_gated(int rows, int Cin, int F, int act)
{
    if (rows <= 0 || rows > (1 << 30) || Cin <= 0 || F <= 0 || Cin > WCC_MAX_GATED || F > WCC_MAX_GATED || Cin % 8 != 0 || F % 8 != 0) return WCC_ERR_SHAPE;
    if (act < WCC_ACT_NONE || act > WCC_ACT_GELU) return WCC_ERR_SHAPE;
    if ((long long)ceil_div(rows, gt::BM) * ceil_div(F > Cin ? F : Cin, 32) > 0x7FFFFFFFLL) return WCC_ERR_SHAPE;
    return WCC_OK;
}

}  // namespace wcc

using namespace wcc;

extern "C" {

wcc_status wcc_checkpoint(const void* x, long long rows, int L, wcc_dtype dt, int8_t* codes, float* scales, void* stream)
{
    if (!x || !codes || !scales) return WCC_ERR_NULL;
    if (rows <= 0 || L <= 0 || rows > (1LL << 40) / L) return WCC_ERR_SHAPE;
    if (dt != WCC_F32 && dt != WCC_BF16) return WCC_ERR_DTYPE;
    if (!on16(x, codes, scales)) return WCC_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dt == WCC_BF16 ? ck::pack<__nv_bfloat16>(x, rows, L, codes, scales, st) : ck::pack<float>(x, rows, L, codes, scales, st);
}

wcc_status wcc_checkpoint_restore(const int8_t* codes, const float* scales, long long rows, int L, wcc_dtype dt, void* out, void* stream)
{
    if (!out || !codes || !scales) return WCC_ERR_NULL;
    if (rows <= 0 || L <= 0 || rows > (1LL << 40) / L) return WCC_ERR_SHAPE;
    if (dt != WCC_F32 && dt != WCC_BF16) return WCC_ERR_DTYPE;
    if (!on16(out, codes, scales)) return WCC_ERR_ALIGN;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dt == WCC_BF16 ? ck::restore<__nv_bfloat16>(codes, scales, rows, L, out, st) : ck::restore<float>(codes, scales, rows, L, out, st);
}

size_t wcc_groupnorm_workspace_bytes(int N, int P, int C, int groups, wcc_dtype dt, int backward)
{
    if (check_groupnorm(N, P, C, groups, dt, WCC_ACT_NONE) != WCC_OK) return 0;
    const int es = dt == WCC_BF16 ? 2 : 4;
    size_t n = gn::layout_of(gn::plan_of(N, P, C, groups, es, false, false), N, C, groups, false).total;
    for (int kept = 0; backward && kept < 2; ++kept) {
        const size_t b = gn::layout_of(gn::plan_of(N, P, C, groups, es, true, kept != 0), N, C, groups, true).total;
        if (b > n) n = b;
    }
    return n;
}

wcc_status wcc_groupnorm_fwd(const void* x, const float* gamma, const float* beta, int N, int P, int C, int groups, float eps, wcc_act act,
                             wcc_dtype dt, void* y, float* mean, float* rstd, int8_t* codes, float* scales, void* ws, size_t ws_bytes, void* stream)
{
    if (!x || !y || !ws || !codes != !scales) return WCC_ERR_NULL;
    wcc_status s = check_groupnorm(N, P, C, groups, dt, act);
    if (s != WCC_OK) return s;
    if (!(eps >= 0.0f) || eps > 3.0e38f) return WCC_ERR_SHAPE;
    if (!on16(x, gamma, beta, y, mean, rstd, codes, scales, ws)) return WCC_ERR_ALIGN;
    const gn::Plan q = gn::plan_of(N, P, C, groups, dt == WCC_BF16 ? 2 : 4, false, false);
    const gn::Layout l = gn::layout_of(q, N, C, groups, false);
    if (ws_bytes < l.total) return WCC_ERR_WORKSPACE;
    DeviceInfo di;
    if ((s = device_info(di)) != WCC_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    gn::Args a = groupnorm_args(N, P, C, groups, act, q, l, ws, di);
    a.x = x; a.out = y; a.gamma = gamma; a.beta = beta; a.mean_out = mean; a.rstd_out = rstd; a.eps = eps;
    if (codes && (s = wcc_checkpoint(x, (long long)N * P, C, dt, codes, scales, stream)) != WCC_OK) return s;
    if (!q.solo && (s = launch_clear(a.ctl, l.part - l.ctl, st)) != WCC_OK) return s;
    if (q.ring) return dt == WCC_BF16 ? gn::ring_forward<__nv_bfloat16>(a, di, st) : gn::ring_forward<float>(a, di, st);
    return dt == WCC_BF16 ? gn::forward<__nv_bfloat16>(a, di, st) : gn::forward<float>(a, di, st);
}

wcc_status wcc_groupnorm_bwd(const void* dy, const void* x, const int8_t* codes, const float* scales, const float* gamma, const float* beta,
                             const float* mean, const float* rstd, int N, int P, int C, int groups, wcc_act act, wcc_dtype dt, void* dx, float* dgamma,
                             float* dbeta, void* ws, size_t ws_bytes, void* stream)
{
    if (!dy || (!x && (!codes || !scales)) || !mean || !rstd || !dx || !ws) return WCC_ERR_NULL;
    wcc_status s = check_groupnorm(N, P, C, groups, dt, act);
    if (s != WCC_OK) return s;
    if (!on16(dy, x, codes, scales, gamma, beta, mean, rstd, dx, dgamma, dbeta, ws)) return WCC_ERR_ALIGN;
    const gn::Plan q = gn::plan_of(N, P, C, groups, dt == WCC_BF16 ? 2 : 4, true, x == nullptr);
    const gn::Layout l = gn::layout_of(q, N, C, groups, true);
    if (ws_bytes < l.total) return WCC_ERR_WORKSPACE;
    DeviceInfo di;
    if ((s = device_info(di)) != WCC_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    gn::Args a = groupnorm_args(N, P, C, groups, act, q, l, ws, di);
    a.dy = dy; a.x = x; a.codes = codes; a.scales = scales; a.out = dx; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
    a.params = dgamma || dbeta;
    const int grid = gn::grid_of(q, N, B200_SMS, true);
    a.img_beta = 0; a.img_gamma = C; a.img_row = 2LL * C;
    if (!q.solo && (s = launch_clear(a.ctl, l.part - l.ctl, st)) != WCC_OK) return s;
    if (q.ring) s = dt == WCC_BF16 ? gn::ring_backward<__nv_bfloat16>(a, di, st) : gn::ring_backward<float>(a, di, st);
    else s = dt == WCC_BF16 ? gn::backward<__nv_bfloat16>(a, di, grid, st) : gn::backward<float>(a, di, grid, st);
    if (s != WCC_OK || !a.params) return s;
    const int es = dt == WCC_BF16 ? 2 : 4, rows = gn::rows_path(P, C, groups, es, x == nullptr) ? gn::rows_grid(N, C, es, true).blocks : q.solo ? grid : N;
    return launch_overlapped(gn::reduce_kernel, dim3((unsigned)ceil_div(2 * C, 32)), dim3(256), 0, st, true, 1, a.img, rows, C, dgamma, dbeta);
}

wcc_status wcc_gated_fwd(const void* x, const void* Wg, const void* Wu, int rows, int Cin, int F, wcc_act act, void* y, void* stream)
{
    if (!x || !Wg || !Wu || !y) return WCC_ERR_NULL;
    wcc_status s = check_gated(rows, Cin, F, act);
    if (s != WCC_OK) return s;
    if (!on16(x, Wg, Wu, y)) return WCC_ERR_ALIGN;
    DeviceInfo di;
    if ((s = device_info(di)) != WCC_OK) return s;
    gt::Args a{};
    a.rows = rows; a.Cin = Cin; a.F = F; a.act = act; a.status = di.status;
    a.y = static_cast<__nv_bfloat16*>(y);
    return gt::gates<gt::FORWARD>(x, Wg, Wu, a, di, static_cast<cudaStream_t>(stream));
}

size_t wcc_gated_bwd_workspace_bytes(int rows, int Cin, int F)
{
    if (check_gated(rows, Cin, F, WCC_ACT_NONE) != WCC_OK) return 0;
    return gt::layout_of(rows, Cin, F).total;
}

wcc_status wcc_gated_bwd(const void* dy, const void* x, const void* Wg, const void* Wu, int rows, int Cin, int F, wcc_act act, void* dx, void* dWg,
                         void* dWu, void* ws, size_t ws_bytes, void* stream)
{
    if (!dy || !x || !Wg || !Wu || !ws || !dWg != !dWu || (!dx && !dWg)) return WCC_ERR_NULL;
    wcc_status s = check_gated(rows, Cin, F, act);
    if (s != WCC_OK) return s;
    if (!on16(dy, x, Wg, Wu, dx, dWg, dWu, ws)) return WCC_ERR_ALIGN;
    const gt::Layout l = gt::layout_of(rows, Cin, F);
    if (ws_bytes < l.total) return WCC_ERR_WORKSPACE;
    DeviceInfo di;
    if ((s = device_info(di)) != WCC_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    char* w = static_cast<char*>(ws);
    gt::Args a{};
    a.rows = rows; a.Cin = Cin; a.F = F; a.act = act; a.status = di.status;
    a.dy = static_cast<const __nv_bfloat16*>(dy);
    a.y = reinterpret_cast<__nv_bfloat16*>(w + l.dG);
    a.y2 = reinterpret_cast<__nv_bfloat16*>(w + l.dU);
    while ((1 << a.log_cin) < Cin) ++a.log_cin;
    gt::Exps* exps = reinterpret_cast<gt::Exps*>(w + l.exps);
    short* row_exp = reinterpret_cast<short*>(w + l.row_exp);
    a.exps = exps;
    a.row_exp = row_exp;
    char *x16 = w + l.x16, *W16 = w + l.W16;
    if ((s = gt::operands(dy, x, Wg, Wu, a, exps, row_exp, dWg ? x16 : nullptr, dx ? W16 : nullptr, di, st)) != WCC_OK) return s;
    if ((s = gt::gates<gt::PARTS>(x, Wg, Wu, a, di, st)) != WCC_OK) return s;
    if (dWg) {
        gt::Args b = a;
        b.y = static_cast<__nv_bfloat16*>(dWg);
        b.y2 = static_cast<__nv_bfloat16*>(dWu);
        b.part = reinterpret_cast<float*>(w + l.part);
        if ((s = gt::dw(a.y, a.y2, x16, b, gt::dw_plan(rows, Cin, F, B200_SMS), di, st)) != WCC_OK) return s;
    }
    if (dx) {
        gt::Args b = a;
        b.y = static_cast<__nv_bfloat16*>(dx);
        if ((s = gt::dx(a.y, a.y2, W16, W16 + (size_t)F * Cin * 2, b, di, st)) != WCC_OK) return s;
    }
    return WCC_OK;
}

}  // extern "C"
