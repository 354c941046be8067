// C-ABI of the sequence operators: validation and the calls of their launchers.  See include/ucd_seq.h for the contract.
#include "ucd_seq.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <new>

#include "seq.h"

using namespace ucd;

namespace {

constexpr int64_t kMaxStride = int64_t(1) << 40, kMaxInner = int64_t(1) << 25;   // a tile of 16 tokens and more in 32-bit offsets of bytes
constexpr int64_t kMaxElements = int64_t(1) << 40;
// Positions, sequences and what they are divided into are counted in 32 bits, and loops over them step up to 2^20 beyond their end.
constexpr int32_t kMaxExtent = 1 << 30;

template <class F>
int guarded(F body) noexcept
{
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return UCD_E_NOMEM;
    } catch (...) {
        return UCD_E_INVALID;
    }
}

int hip_status(hipError_t e)
{
    if (e == hipSuccess) return UCD_OK;
    static const bool verbose = getenv("UCD_VERBOSE_ERRORS") != nullptr;
    if (verbose) fprintf(stderr, "ucd: HIP error %d: %s\n", (int)e, hipGetErrorString(e));
    return UCD_E_HIP;
}

// Fills in dense strides; false where rows of `width` elements would overlap.  Those of an extent of one are never taken, and may be anything.
bool fill_strides(int64_t &outer, int64_t &inner, int64_t n_outer, int64_t n_inner, int64_t width)
{
    if (outer < 0 || inner < 0 || width > kMaxInner || (n_inner > 1 && inner > kMaxInner)) return false;
    if (inner == 0) inner = width;
    if (outer == 0) outer = inner * (n_inner > 1 ? n_inner : 1);
    if (n_inner <= 1) inner = width;
    if (n_outer <= 1) outer = width;
    if (outer > kMaxStride) return false;
    if (n_inner > 1 && inner < width) return false;
    if (n_outer > 1 && outer < width) return false;
    if (n_inner > 1 && n_outer > 1) {
        const bool rows_inside = inner <= outer;
        const int64_t lo = rows_inside ? inner : outer, hi = rows_inside ? outer : inner, n = rows_inside ? n_inner : n_outer;
        if (hi < lo * (n - 1) + width) return false;
    }
    return true;
}

bool extent_ok(int32_t n, int32_t least) { return n >= least && n <= kMaxExtent; }
bool dtype_ok(int dtype) { return dtype == 0 || dtype == 1; }
bool act_ok(int act) { return act == UCD_ACT_NONE || act == UCD_ACT_SILU; }
bool aligned(const void *p, int dtype) { return ((uintptr_t)p & (dtype == 1 ? 1u : 3u)) == 0; }
bool aligned4(const void *p) { return ((uintptr_t)p & 3u) == 0; }
bool beta_ok(float beta) { return beta == 0.f || beta == 1.f; }

// UCD_OK where a workspace of `need` bytes is there
int ws_status(size_t need, const void *ws, size_t ws_bytes)
{
    if (need == 0) return UCD_OK;
    if (!ws) return UCD_E_NULLPTR;
    if (((uintptr_t)ws & 15u) != 0) return UCD_E_INVALID;
    return ws_bytes < need ? UCD_E_WS_TOO_SMALL : UCD_OK;
}

bool norm_ok(const ucd_group_norm_t *in, ucd_group_norm_t &d)
{
    d = *in;
    if (!extent_ok(d.N, 1) || !extent_ok(d.S, 1) || !extent_ok(d.C, 1) || d.G < 1 || d.C % d.G != 0 || !act_ok(d.act) || !dtype_ok(d.dtype)) return false;
    if (!(d.eps >= 0.f) || std::isinf(d.eps)) return false;
    if ((double)d.N * d.S * d.C > (double)kMaxElements) return false;
    return fill_strides(d.x_n, d.x_s, d.N, d.S, d.C) && fill_strides(d.y_n, d.y_s, d.N, d.S, d.C);
}

bool conv_ok(const ucd_causal_conv_t *in, ucd_causal_conv_t &d)
{
    d = *in;
    if (!extent_ok(d.B, 0) || !extent_ok(d.L, 0) || !extent_ok(d.D, 1) || d.K < 1 || d.K > 8 || !act_ok(d.act) || !dtype_ok(d.dtype) || d.n_slots < 0) return false;
    if ((double)d.B * (d.L + 1) * d.D > (double)kMaxElements) return false;
    return fill_strides(d.x_b, d.x_l, d.B, d.L, d.D) && fill_strides(d.y_b, d.y_l, d.B, d.L, d.D);
}

bool scan_ok(const ucd_scan_t *in, ucd_scan_t &d)
{
    d = *in;
    if (!extent_ok(d.B, 0) || !extent_ok(d.L, 0) || !extent_ok(d.D, 1) || d.N < 1 || d.N > 64 || d.G < 1 || d.D % d.G != 0 || !dtype_ok(d.dtype)) return false;
    if (d.softplus != 0 && d.softplus != 1) return false;
    if (d.n_slots < 0 || (double)d.B * (d.L + 1) * d.D > (double)kMaxElements) return false;
    const int64_t GN = (int64_t)d.G * d.N;
    if ((double)d.B * (d.L + 1) * GN > (double)kMaxElements) return false;
    return fill_strides(d.u_b, d.u_l, d.B, d.L, d.D) && fill_strides(d.dt_b, d.dt_l, d.B, d.L, d.D) &&
           fill_strides(d.z_b, d.z_l, d.B, d.L, d.D) && fill_strides(d.y_b, d.y_l, d.B, d.L, d.D) &&
           fill_strides(d.Bm_b, d.Bm_l, d.B, d.L, GN) && fill_strides(d.Cm_b, d.Cm_l, d.B, d.L, GN);
}

// Workgroups of the convolution's launches, 32 channels by 4 runs of 8 tokens each at least: their kernels count them, and runs, in 32 bits.
bool conv_countable(const ucd_causal_conv_t &d)
{
    const double runs = (double)d.B * (d.L / 8 + 1);
    return runs < 1u << 31 && (d.D / 32 + 1.) * (runs / 4 + 1) < 1u << 31;
}

// No token at all: tensors of no elements have no address.
bool empty(int B, int L) { return B == 0 || L == 0; }

// Workgroups of the scan's launches, 16 channels each at least: their kernels count them in 32 bits.
double scan_workgroups(const ucd_scan_t &d) { return (double)d.B * (d.D / 16 + d.G); }

// A pool needs its slots, where there are any, and slots their pool.
bool slots_ok(int B, int n_slots, const int32_t *slots) { return n_slots > 0 ? slots != nullptr || B == 0 : slots == nullptr; }

int scan_inputs(const ucd_scan_t &d, const ucd_scan_in_t *in)
{
    if (!in->A || (!empty(d.B, d.L) && (!in->u || !in->dt || !in->Bm || !in->Cm))) return UCD_E_NULLPTR;
    if (!aligned(in->u, d.dtype) || !aligned(in->dt, d.dtype) || !aligned(in->Bm, d.dtype) || !aligned(in->Cm, d.dtype) ||
        !aligned(in->z, d.dtype) || !aligned4(in->A) || !aligned4(in->skip) || !aligned4(in->dt_bias) ||
        !aligned4(in->lengths) || !aligned4(in->slots))
        return UCD_E_INVALID;
    return UCD_OK;
}

}  // namespace

extern "C" {

size_t ucd_group_norm_workspace_size(const ucd_group_norm_t *norm, int dir)
{
    ucd_group_norm_t d;
    if (!norm || !norm_ok(norm, d) || (dir != UCD_SEQ_FWD && dir != UCD_SEQ_BWD)) return UCD_WS_NA;
    return group_norm_ws_bytes(d, dir);
}

int ucd_group_norm_fwd(const ucd_group_norm_t *norm, const void *x, const float *gamma, const float *beta_w, void *y,
                       float *stats, void *ws, size_t ws_bytes, void *stream)
{
    return guarded([&]() -> int {
        if (!norm || !x || !gamma || !beta_w || !y) return UCD_E_NULLPTR;
        ucd_group_norm_t d;
        if (!norm_ok(norm, d)) return UCD_E_INVALID;
        if (!aligned(x, d.dtype) || !aligned(y, d.dtype) || !aligned4(gamma) || !aligned4(beta_w) || !aligned4(stats))
            return UCD_E_INVALID;
        const int rc = ws_status(group_norm_ws_bytes(d, UCD_SEQ_FWD), ws, ws_bytes);
        if (rc != UCD_OK) return rc;
        (void)hipGetLastError();
        return hip_status(group_norm_fwd(d, x, gamma, beta_w, y, stats, ws, (hipStream_t)stream));
    });
}

int ucd_group_norm_bwd(const ucd_group_norm_t *norm, const void *x, const float *gamma, const float *beta_w,
                       const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, float beta, void *ws,
                       size_t ws_bytes, void *stream)
{
    return guarded([&]() -> int {
        if (!norm || !x || !gamma || !beta_w || !stats || !dy || !dx || !dgamma || !dbeta) return UCD_E_NULLPTR;
        ucd_group_norm_t d;
        if (!norm_ok(norm, d) || !beta_ok(beta)) return UCD_E_INVALID;
        if (!aligned(x, d.dtype) || !aligned(dy, d.dtype) || !aligned(dx, d.dtype) || !aligned4(gamma) || !aligned4(beta_w) ||
            !aligned4(stats) || !aligned4(dgamma) || !aligned4(dbeta))
            return UCD_E_INVALID;
        const int rc = ws_status(group_norm_ws_bytes(d, UCD_SEQ_BWD), ws, ws_bytes);
        if (rc != UCD_OK) return rc;
        (void)hipGetLastError();
        return hip_status(group_norm_bwd(d, x, gamma, beta_w, stats, dy, dx, dgamma, dbeta, beta != 0.f, ws, (hipStream_t)stream));
    });
}

size_t ucd_causal_conv_workspace_size(const ucd_causal_conv_t *conv)
{
    ucd_causal_conv_t d;
    if (!conv || !conv_ok(conv, d)) return UCD_WS_NA;
    return causal_conv_ws_bytes(d);
}

int ucd_causal_conv_fwd(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                        const int32_t *lengths, const int32_t *slots, const void *state_in, void *state_out, void *y,
                        void *stream)
{
    return guarded([&]() -> int {
        if (!conv || !w) return UCD_E_NULLPTR;
        ucd_causal_conv_t d;
        if (!conv_ok(conv, d) || !slots_ok(d.B, d.n_slots, slots)) return UCD_E_INVALID;
        if (!empty(d.B, d.L) && (!x || !y)) return UCD_E_NULLPTR;
        if (!aligned(x, d.dtype) || !aligned(w, d.dtype) || !aligned(y, d.dtype) || !aligned(state_in, d.dtype) ||
            !aligned(state_out, d.dtype) || !aligned4(bias) || !aligned4(lengths) || !aligned4(slots))
            return UCD_E_INVALID;
        if (!conv_countable(d)) return UCD_E_UNSUPPORTED;
        if (d.B == 0) return UCD_OK;
        CausalConvArgs a{};
        a.x = x; a.w = w; a.bias = bias; a.lengths = lengths; a.slots = slots;
        a.state_in = state_in; a.state_out = state_out; a.y = y;
        (void)hipGetLastError();
        return hip_status(causal_conv_fwd(d, a, (hipStream_t)stream));
    });
}

int ucd_causal_conv_bwd(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                        const int32_t *lengths, const void *state_in, const void *dy, const void *dstate_out, void *dx,
                        float *dw, float *dbias, void *dstate_in, float beta, void *ws, size_t ws_bytes, void *stream)
{
    return guarded([&]() -> int {
        if (!conv || !w || !dw) return UCD_E_NULLPTR;
        ucd_causal_conv_t d;
        if (!conv_ok(conv, d) || d.n_slots != 0 || !beta_ok(beta)) return UCD_E_INVALID;
        if (!empty(d.B, d.L) && (!x || !dy || !dx)) return UCD_E_NULLPTR;
        if (!aligned(x, d.dtype) || !aligned(w, d.dtype) || !aligned(dy, d.dtype) || !aligned(dx, d.dtype) ||
            !aligned(state_in, d.dtype) || !aligned(dstate_out, d.dtype) || !aligned(dstate_in, d.dtype) || !aligned4(bias) ||
            !aligned4(lengths) || !aligned4(dw) || !aligned4(dbias))
            return UCD_E_INVALID;
        const int rc = ws_status(causal_conv_ws_bytes(d), ws, ws_bytes);
        if (rc != UCD_OK) return rc;
        if (!conv_countable(d)) return UCD_E_UNSUPPORTED;
        CausalConvArgs a{};
        a.x = x; a.w = w; a.bias = bias; a.lengths = lengths; a.state_in = state_in; a.dy = dy; a.dstate_out = dstate_out;
        a.dx = dx; a.dw = dw; a.dbias = dbias; a.dstate_in = dstate_in;
        (void)hipGetLastError();
        return hip_status(causal_conv_bwd(d, a, beta != 0.f, ws, (hipStream_t)stream));
    });
}

int ucd_causal_conv_step(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                         const int32_t *slots, void *state, void *y, void *stream)
{
    return guarded([&]() -> int {
        if (!conv || !w) return UCD_E_NULLPTR;
        ucd_causal_conv_t d;
        if (!conv_ok(conv, d) || d.L != 1 || !slots_ok(d.B, d.n_slots, slots)) return UCD_E_INVALID;
        if (d.B > 0 && (!x || !y || (d.K > 1 && !state))) return UCD_E_NULLPTR;
        if (!aligned(x, d.dtype) || !aligned(w, d.dtype) || !aligned(y, d.dtype) || !aligned(state, d.dtype) || !aligned4(bias) ||
            !aligned4(slots))
            return UCD_E_INVALID;
        if (!conv_countable(d)) return UCD_E_UNSUPPORTED;
        if (d.B == 0) return UCD_OK;
        CausalConvArgs a{};
        a.x = x; a.w = w; a.bias = bias; a.slots = slots; a.state_in = state; a.state_out = state; a.y = y;
        (void)hipGetLastError();
        return hip_status(causal_conv_step(d, a, (hipStream_t)stream));
    });
}

size_t ucd_scan_workspace_size(const ucd_scan_t *scan, int dir)
{
    ucd_scan_t d;
    if (!scan || !scan_ok(scan, d) || (dir != UCD_SEQ_FWD && dir != UCD_SEQ_BWD)) return UCD_WS_NA;
    return scan_ws_bytes(d, dir);
}

size_t ucd_scan_saved_size(const ucd_scan_t *scan)
{
    ucd_scan_t d;
    if (!scan || !scan_ok(scan, d)) return UCD_WS_NA;
    return scan_saved_bytes(d);
}

int ucd_scan_fwd(const ucd_scan_t *scan, const ucd_scan_in_t *in, const float *state_in, float *state_out, void *y,
                 void *saved, size_t saved_bytes, void *ws, size_t ws_bytes, void *stream)
{
    return guarded([&]() -> int {
        if (!scan || !in) return UCD_E_NULLPTR;
        ucd_scan_t d;
        if (!scan_ok(scan, d) || !slots_ok(d.B, d.n_slots, in->slots)) return UCD_E_INVALID;
        if (!empty(d.B, d.L) && !y) return UCD_E_NULLPTR;
        int rc = scan_inputs(d, in);
        if (rc != UCD_OK) return rc;
        if (!aligned(y, d.dtype) || !aligned4(state_in) || !aligned4(state_out)) return UCD_E_INVALID;
        if (saved && (rc = ws_status(scan_saved_bytes(d), saved, saved_bytes)) != UCD_OK) return rc;
        if ((rc = ws_status(scan_ws_bytes(d, UCD_SEQ_FWD), ws, ws_bytes)) != UCD_OK) return rc;
        if (scan_workgroups(d) >= 1 << 30) return UCD_E_UNSUPPORTED;
        if (d.B == 0) return UCD_OK;
        (void)hipGetLastError();
        return hip_status(scan_fwd(d, *in, state_in, state_out, y, (float *)saved, ws, (hipStream_t)stream));
    });
}

int ucd_scan_bwd(const ucd_scan_t *scan, const ucd_scan_in_t *in, const void *dy, const float *dstate_out,
                 const void *saved, size_t saved_bytes, const ucd_scan_grad_t *grad, float beta, void *ws, size_t ws_bytes,
                 void *stream)
{
    return guarded([&]() -> int {
        if (!scan || !in || !grad) return UCD_E_NULLPTR;
        ucd_scan_t d;
        if (!scan_ok(scan, d) || d.n_slots != 0 || in->slots || !beta_ok(beta)) return UCD_E_INVALID;
        int rc = scan_inputs(d, in);
        if (rc != UCD_OK) return rc;
        if (!grad->A || (in->skip && !grad->skip) || (in->dt_bias && !grad->dt_bias)) return UCD_E_NULLPTR;
        if (!empty(d.B, d.L) && (!dy || !grad->u || !grad->dt || !grad->Bm || !grad->Cm || (in->z && !grad->z))) return UCD_E_NULLPTR;
        if (!aligned(dy, d.dtype) || !aligned(grad->u, d.dtype) || !aligned(grad->dt, d.dtype) || !aligned(grad->Bm, d.dtype) ||
            !aligned(grad->Cm, d.dtype) || !aligned(grad->z, d.dtype) || !aligned4(grad->A) || !aligned4(grad->skip) ||
            !aligned4(grad->dt_bias) || !aligned4(grad->state) || !aligned4(dstate_out))
            return UCD_E_INVALID;
        if ((rc = ws_status(scan_saved_bytes(d), saved, saved_bytes)) != UCD_OK) return rc;
        if ((rc = ws_status(scan_ws_bytes(d, UCD_SEQ_BWD), ws, ws_bytes)) != UCD_OK) return rc;
        if (scan_workgroups(d) >= 1 << 30) return UCD_E_UNSUPPORTED;
        (void)hipGetLastError();
        return hip_status(scan_bwd(d, *in, dy, dstate_out, (const float *)saved, *grad, beta != 0.f, ws, (hipStream_t)stream));
    });
}

int ucd_scan_step(const ucd_scan_t *scan, const ucd_scan_in_t *in, float *state, void *y, void *stream)
{
    return guarded([&]() -> int {
        if (!scan || !in) return UCD_E_NULLPTR;
        ucd_scan_t d;
        if (!scan_ok(scan, d) || d.L != 1 || !slots_ok(d.B, d.n_slots, in->slots)) return UCD_E_INVALID;
        if (d.B > 0 && (!state || !y)) return UCD_E_NULLPTR;
        const int rc = scan_inputs(d, in);
        if (rc != UCD_OK) return rc;
        if (!aligned(y, d.dtype) || !aligned4(state)) return UCD_E_INVALID;
        if (scan_workgroups(d) >= 1 << 30) return UCD_E_UNSUPPORTED;
        if (d.B == 0) return UCD_OK;
        (void)hipGetLastError();
        return hip_status(scan_step(d, *in, state, y, (hipStream_t)stream));
    });
}

}  // extern "C"
