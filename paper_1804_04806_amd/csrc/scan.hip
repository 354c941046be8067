// Selective state space scan: Forward, Backward and the single-token step.
#include <algorithm>

#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace {
using namespace seq;

constexpr int kMaxN = 64;

__device__ int length_of(const ucd_scan_t &d, const int32_t *lengths, int b)
{
    if (!lengths) return d.L;
    const int n = lengths[b];
    return n < 0 ? 0 : n < d.L ? n : d.L;
}

__device__ float softplus(float v) { return v > 20.f ? v : log1pf(__expf(v)); }

// One channel of one sequence per thread, its states in memory; saved holds every token's and those before the first.
template <class T>
__global__ __launch_bounds__(64) void scan_fwd_simple(ucd_scan_t d, ucd_scan_in_t in, const float *state_in, float *state_out,
                                                      void *y_, float *saved)
{
    const long i = blockIdx.x * 64l + threadIdx.x;
    if (i >= (long)d.B * d.D) return;
    const int c = (int)(i % d.D), b = (int)(i / d.D), g = c / (d.D / d.G);
    const int slot = in.slots ? in.slots[b] : b;
    const bool idle = in.slots && (slot < 0 || slot >= d.n_slots);
    const int n = idle ? 0 : length_of(d, in.lengths, b);
    float h[kMaxN];
    for (int k = 0; k < d.N; ++k) {
        h[k] = state_in && !idle ? state_in[((long)slot * d.D + c) * d.N + k] : 0.f;
        if (saved) saved[((long)b * (d.L + 1) * d.D + c) * d.N + k] = h[k];
    }
    for (int t = 0; t < d.L; ++t) {
        float y = 0.f;
        if (t < n) {
            const float u = to_f(((const T *)in.u)[b * d.u_b + t * d.u_l + c]);
            float dt = to_f(((const T *)in.dt)[b * d.dt_b + t * d.dt_l + c]) + (in.dt_bias ? in.dt_bias[c] : 0.f);
            if (d.softplus) dt = softplus(dt);
            for (int k = 0; k < d.N; ++k) {
                h[k] = __expf(dt * in.A[(long)c * d.N + k]) * h[k] + dt * u * to_f(((const T *)in.Bm)[b * d.Bm_b + t * d.Bm_l + g * d.N + k]);
                y += h[k] * to_f(((const T *)in.Cm)[b * d.Cm_b + t * d.Cm_l + g * d.N + k]);
            }
            if (in.skip) y += in.skip[c] * u;
            if (in.z) {
                const float z = to_f(((const T *)in.z)[b * d.z_b + t * d.z_l + c]);
                y *= z * sigmoid(z);
            }
        }
        ((T *)y_)[b * d.y_b + t * d.y_l + c] = from_f<T>(y);
        if (saved)
            for (int k = 0; k < d.N; ++k) saved[(((long)b * (d.L + 1) + t + 1) * d.D + c) * d.N + k] = h[k];
    }
    if (state_out && !idle)
        for (int k = 0; k < d.N; ++k) state_out[((long)slot * d.D + c) * d.N + k] = h[k];
}

// One channel per thread; ws receives every token's dh.  part: [B][D][N + 2] sums over a sequence's tokens (dA, dskip, ddt_bias).
template <class T>
__global__ __launch_bounds__(64) void scan_bwd_simple(ucd_scan_t d, ucd_scan_in_t in, const void *dy_, const float *dstate_out,
                                                      const float *saved, ucd_scan_grad_t gr, float *ws, float *part)
{
    const long i = blockIdx.x * 64l + threadIdx.x;
    if (i >= (long)d.B * d.D) return;
    const int c = (int)(i % d.D), b = (int)(i / d.D), g = c / (d.D / d.G), n = length_of(d, in.lengths, b);
    float dh[kMaxN], dA[kMaxN], dskip = 0.f, dbias = 0.f;
    for (int k = 0; k < d.N; ++k) {
        dh[k] = dstate_out ? dstate_out[((long)b * d.D + c) * d.N + k] : 0.f;
        dA[k] = 0.f;
    }
    for (int t = d.L - 1; t >= 0; --t) {
        const long at = (((long)b * d.L + t) * d.D + c) * d.N, before = (((long)b * (d.L + 1) + t) * d.D + c) * d.N, after = before + (long)d.D * d.N;
        float du = 0.f, ddt = 0.f, dz = 0.f;
        if (t < n) {
            const float u = to_f(((const T *)in.u)[b * d.u_b + t * d.u_l + c]);
            const float raw = to_f(((const T *)in.dt)[b * d.dt_b + t * d.dt_l + c]) + (in.dt_bias ? in.dt_bias[c] : 0.f);
            const float dt = d.softplus ? softplus(raw) : raw;
            float dy = to_f(((const T *)dy_)[b * d.y_b + t * d.y_l + c]);
            if (in.z) {
                float y = in.skip ? in.skip[c] * u : 0.f;
                for (int k = 0; k < d.N; ++k) y += saved[after + k] * to_f(((const T *)in.Cm)[b * d.Cm_b + t * d.Cm_l + g * d.N + k]);
                const float z = to_f(((const T *)in.z)[b * d.z_b + t * d.z_l + c]), s = sigmoid(z);
                dz = dy * y * (s * (1.f + z * (1.f - s)));
                dy *= z * s;
            }
            float grown = 0.f;
            for (int k = 0; k < d.N; ++k) {
                const float A = in.A[(long)c * d.N + k], a = __expf(dt * A);
                const float bm = to_f(((const T *)in.Bm)[b * d.Bm_b + t * d.Bm_l + g * d.N + k]);
                dh[k] += dy * to_f(((const T *)in.Cm)[b * d.Cm_b + t * d.Cm_l + g * d.N + k]);
                ws[at + k] = dh[k];
                grown += dh[k] * bm;
                const float q = dh[k] * a * saved[before + k];
                ddt += q * A;
                dA[k] += q * dt;
                dh[k] *= a;
            }
            du = grown * dt;
            ddt += grown * u;
            if (in.skip) {
                du += in.skip[c] * dy;
                dskip += dy * u;
            }
            if (d.softplus) ddt *= sigmoid(raw);
            dbias += ddt;
        } else {
            for (int k = 0; k < d.N; ++k) ws[at + k] = 0.f;
        }
        ((T *)gr.u)[b * d.u_b + t * d.u_l + c] = from_f<T>(du);
        ((T *)gr.dt)[b * d.dt_b + t * d.dt_l + c] = from_f<T>(ddt);
        if (in.z) ((T *)gr.z)[b * d.z_b + t * d.z_l + c] = from_f<T>(dz);
    }
    float *p = part + i * (d.N + 2);
    for (int k = 0; k < d.N; ++k) {
        p[k] = dA[k];
        if (gr.state) gr.state[((long)b * d.D + c) * d.N + k] = dh[k];
    }
    p[d.N] = dskip;
    p[d.N + 1] = dbias;
}

// One state of one group at one token per thread.
template <class T>
__global__ __launch_bounds__(256) void scan_bc_simple(ucd_scan_t d, ucd_scan_in_t in, const void *dy_, const float *saved, const float *ws,
                                                      ucd_scan_grad_t gr)
{
    const long units = (long)d.B * d.L * d.G * d.N;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < units; i += gridDim.x * 256l) {
        const int k = (int)(i % d.N), g = (int)(i / d.N % d.G), t = (int)(i / d.N / d.G % d.L), b = (int)(i / d.N / d.G / d.L);
        float db = 0.f, dc = 0.f;
        if (t < length_of(d, in.lengths, b))
            for (int c = g * (d.D / d.G); c < (g + 1) * (d.D / d.G); ++c) {
                const long at = (((long)b * d.L + t) * d.D + c) * d.N + k;
                float dt = to_f(((const T *)in.dt)[b * d.dt_b + t * d.dt_l + c]) + (in.dt_bias ? in.dt_bias[c] : 0.f);
                if (d.softplus) dt = softplus(dt);
                float dy = to_f(((const T *)dy_)[b * d.y_b + t * d.y_l + c]);
                if (in.z) {
                    const float z = to_f(((const T *)in.z)[b * d.z_b + t * d.z_l + c]);
                    dy *= z * sigmoid(z);
                }
                db += ws[at] * dt * to_f(((const T *)in.u)[b * d.u_b + t * d.u_l + c]);
                dc += dy * saved[(((long)b * (d.L + 1) + t + 1) * d.D + c) * d.N + k];
            }
        ((T *)gr.Bm)[b * d.Bm_b + t * d.Bm_l + g * d.N + k] = from_f<T>(db);
        ((T *)gr.Cm)[b * d.Cm_b + t * d.Cm_l + g * d.N + k] = from_f<T>(dc);
    }
}

__global__ __launch_bounds__(256) void scan_weights_simple(ucd_scan_t d, const float *part, ucd_scan_grad_t gr, bool add)
{
    const long i = blockIdx.x * 256l + threadIdx.x;
    if (i >= (long)d.D * (d.N + 2)) return;
    const int k = (int)(i % (d.N + 2)), c = (int)(i / (d.N + 2));
    float v = 0.f;
    for (int b = 0; b < d.B; ++b) v += part[(long)b * d.D * (d.N + 2) + i];
    float *out = k < d.N ? gr.A + (long)c * d.N + k : k == d.N ? (gr.skip ? gr.skip + c : nullptr) : gr.dt_bias ? gr.dt_bias + c : nullptr;
    if (out) *out = v + (add ? *out : 0.f);
}

unsigned blocks_of(long units, int threads) { return (unsigned)std::min((units + threads - 1) / threads, 1l << 20); }

template <class T>
hipError_t fwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const float *state_in, float *state_out, void *y, float *saved, hipStream_t s)
{
    scan_fwd_simple<T><<<blocks_of((long)d.B * d.D, 64), 64, 0, s>>>(d, in, state_in, state_out, y, saved);
    return hipGetLastError();
}

template <class T>
hipError_t bwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const void *dy, const float *dstate_out, const float *saved, const ucd_scan_grad_t &g,
               bool add, float *ws, hipStream_t s)
{
    float *part = ws + (size_t)d.B * d.L * d.D * d.N;
    if (d.B > 0) scan_bwd_simple<T><<<blocks_of((long)d.B * d.D, 64), 64, 0, s>>>(d, in, dy, dstate_out, saved, g, ws, part);
    if (d.B > 0 && d.L > 0) scan_bc_simple<T><<<blocks_of((long)d.B * d.L * d.G * d.N, 256), 256, 0, s>>>(d, in, dy, saved, ws, g);
    scan_weights_simple<<<blocks_of((long)d.D * (d.N + 2), 256), 256, 0, s>>>(d, part, g, add);
    return hipGetLastError();
}

}  // namespace

size_t scan_ws_bytes(const ucd_scan_t &d, int dir)
{
    return dir == UCD_SEQ_FWD ? 0 : 4 * ((size_t)d.B * d.L * d.D * d.N + (size_t)d.B * d.D * (d.N + 2));
}
size_t scan_saved_bytes(const ucd_scan_t &d) { return (size_t)4 * d.B * (d.L + 1) * d.D * d.N; }

hipError_t scan_fwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const float *state_in, float *state_out, void *y, float *saved, void *,
                    hipStream_t s)
{
    return d.dtype == 1 ? fwd<bf16_t>(d, in, state_in, state_out, y, saved, s) : fwd<float>(d, in, state_in, state_out, y, saved, s);
}

hipError_t scan_bwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const void *dy, const float *dstate_out, const float *saved,
                    const ucd_scan_grad_t &g, bool add, void *ws, hipStream_t s)
{
    return d.dtype == 1 ? bwd<bf16_t>(d, in, dy, dstate_out, saved, g, add, (float *)ws, s)
                        : bwd<float>(d, in, dy, dstate_out, saved, g, add, (float *)ws, s);
}

hipError_t scan_step(const ucd_scan_t &d, const ucd_scan_in_t &in, float *state, void *y, hipStream_t s)
{
    return scan_fwd(d, in, state, state, y, nullptr, nullptr, s);
}

}  // namespace ucd
