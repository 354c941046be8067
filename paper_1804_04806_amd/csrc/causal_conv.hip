// Short causal convolution: Forward, Backward and the single-token step.
#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace {
using namespace seq;

__device__ int length_of(const ucd_causal_conv_t &d, const int32_t *lengths, int b)
{
    if (!lengths) return d.L;
    const int n = lengths[b];
    return n < 0 ? 0 : n < d.L ? n : d.L;
}

// a sequence's place among the states, -1 for an idle one
__device__ int slot_of(const ucd_causal_conv_t &d, const int32_t *slots, int b)
{
    if (!slots) return b;
    const int s = slots[b];
    return s >= 0 && s < d.n_slots ? s : -1;
}

// x_t of a channel; t < 0 reaches into the state
template <class T>
__device__ float token(const ucd_causal_conv_t &d, const T *x, const T *state, int t)
{
    if (t >= 0) return to_f(x[(long)t * d.x_l]);
    return state ? to_f(state[(long)(d.K - 1 + t) * d.D]) : 0.f;
}

template <class T>
__global__ __launch_bounds__(256) void conv_fwd_simple(ucd_causal_conv_t d, CausalConvArgs a)
{
    const long units = (long)d.B * d.L * d.D;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < units; i += gridDim.x * 256l) {
        const int c = (int)(i % d.D), t = (int)(i / d.D % d.L), b = (int)(i / d.D / d.L);
        const int slot = slot_of(d, a.slots, b);
        float u = 0.f;
        if (slot >= 0 && t < length_of(d, a.lengths, b)) {
            const T *x = (const T *)a.x + b * d.x_b + c;
            const T *st = a.state_in ? (const T *)a.state_in + (long)slot * (d.K - 1) * d.D + c : nullptr;
            const T *w = (const T *)a.w + (long)c * d.K;
            u = a.bias ? a.bias[c] : 0.f;
            for (int k = 0; k < d.K; ++k) u += to_f(w[k]) * token(d, x, st, t - d.K + 1 + k);
            if (d.act == UCD_ACT_SILU) u *= sigmoid(u);
        }
        ((T *)a.y)[b * d.y_b + t * d.y_l + c] = from_f<T>(u);
    }
}

// after the outputs: state_in may be state_out
template <class T>
__global__ __launch_bounds__(256) void conv_state_simple(ucd_causal_conv_t d, CausalConvArgs a)
{
    const long units = (long)d.B * d.D;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < units; i += gridDim.x * 256l) {
        const int c = (int)(i % d.D), b = (int)(i / d.D);
        const int slot = slot_of(d, a.slots, b), n = length_of(d, a.lengths, b);
        if (slot < 0) continue;
        const T *x = (const T *)a.x + b * d.x_b + c;
        const T *st = a.state_in ? (const T *)a.state_in + (long)slot * (d.K - 1) * d.D + c : nullptr;
        T *out = (T *)a.state_out + (long)slot * (d.K - 1) * d.D + c;
        for (int j = 0; j < d.K - 1; ++j) out[(long)j * d.D] = from_f<T>(token(d, x, st, n - d.K + 1 + j));
    }
}

template <class T>
__device__ float conv_du(const ucd_causal_conv_t &d, const CausalConvArgs &a, const T *x, const T *st, const T *dy, int c, int t)
{
    const float g = to_f(dy[(long)t * d.y_l]);
    if (d.act != UCD_ACT_SILU) return g;
    const T *w = (const T *)a.w + (long)c * d.K;
    float u = a.bias ? a.bias[c] : 0.f;
    for (int k = 0; k < d.K; ++k) u += to_f(w[k]) * token(d, x, st, t - d.K + 1 + k);
    const float s = sigmoid(u);
    return g * (s * (1.f + u * (1.f - s)));
}

// dx, and the gradient of the state at t < 0
template <class T>
__global__ __launch_bounds__(256) void conv_dx_simple(ucd_causal_conv_t d, CausalConvArgs a)
{
    const long rows = d.L + d.K - 1, units = (long)d.B * rows * d.D;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < units; i += gridDim.x * 256l) {
        const int c = (int)(i % d.D), t = (int)(i / d.D % rows) - (d.K - 1), b = (int)(i / d.D / rows);
        const int n = length_of(d, a.lengths, b);
        const T *x = (const T *)a.x + b * d.x_b + c;
        const T *st = a.state_in ? (const T *)a.state_in + (long)b * (d.K - 1) * d.D + c : nullptr;
        const T *dy = (const T *)a.dy + b * d.y_b + c;
        const T *w = (const T *)a.w + (long)c * d.K;
        float g = 0.f;
        if (t < n) {
            for (int k = 0; k < d.K; ++k) {
                const int at = t + d.K - 1 - k;
                if (at >= 0 && at < n) g += to_f(w[k]) * conv_du<T>(d, a, x, st, dy, c, at);
            }
            const int j = t - (n - d.K + 1);
            if (a.dstate_out && j >= 0) g += to_f(((const T *)a.dstate_out)[((long)b * (d.K - 1) + j) * d.D + c]);
        }
        if (t >= 0) ((T *)a.dx)[b * d.x_b + t * d.x_l + c] = from_f<T>(g);
        else if (a.dstate_in) ((T *)a.dstate_in)[((long)b * (d.K - 1) + t + d.K - 1) * d.D + c] = from_f<T>(g);
    }
}

template <class T>
__global__ __launch_bounds__(256) void conv_weights_simple(ucd_causal_conv_t d, CausalConvArgs a, bool add)
{
    __shared__ float lds[256];
    const int c = blockIdx.x;
    float acc[9] = {};
    for (int b = 0; b < d.B; ++b) {
        const int n = length_of(d, a.lengths, b);
        const T *x = (const T *)a.x + b * d.x_b + c;
        const T *st = a.state_in ? (const T *)a.state_in + (long)b * (d.K - 1) * d.D + c : nullptr;
        const T *dy = (const T *)a.dy + b * d.y_b + c;
        for (int t = threadIdx.x; t < n; t += 256) {
            const float g = conv_du<T>(d, a, x, st, dy, c, t);
            for (int k = 0; k < d.K; ++k) acc[k] += g * token(d, x, st, t - d.K + 1 + k);
            acc[8] += g;
        }
    }
    for (int k = 0; k < 9; ++k) {
        if (k >= d.K && k < 8) continue;
        __syncthreads();
        lds[threadIdx.x] = acc[k];
        __syncthreads();
        if (threadIdx.x == 0) {
            float v = 0.f;
            for (int i = 0; i < 256; ++i) v += lds[i];
            float *out = k < 8 ? a.dw + (long)c * d.K + k : a.dbias ? a.dbias + c : nullptr;
            if (out) *out = v + (add ? *out : 0.f);
        }
    }
}

unsigned blocks_of(long units)
{
    const long n = (units + 255) / 256;
    return (unsigned)(n < (1 << 20) ? n : (1 << 20));
}

template <class T>
hipError_t fwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s)
{
    if (d.L > 0) conv_fwd_simple<T><<<blocks_of((long)d.B * d.L * d.D), 256, 0, s>>>(d, a);
    if (a.state_out && d.K > 1) conv_state_simple<T><<<blocks_of((long)d.B * d.D), 256, 0, s>>>(d, a);
    return hipGetLastError();
}

template <class T>
hipError_t bwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, hipStream_t s)
{
    if (d.B > 0) conv_dx_simple<T><<<blocks_of((long)d.B * (d.L + d.K - 1) * d.D), 256, 0, s>>>(d, a);
    conv_weights_simple<T><<<d.D, 256, 0, s>>>(d, a, add);
    return hipGetLastError();
}

}  // namespace

size_t causal_conv_ws_bytes(const ucd_causal_conv_t &) { return 0; }

hipError_t causal_conv_fwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s)
{
    return d.dtype == 1 ? fwd<bf16_t>(d, a, s) : fwd<float>(d, a, s);
}

hipError_t causal_conv_bwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, void *, hipStream_t s)
{
    return d.dtype == 1 ? bwd<bf16_t>(d, a, add, s) : bwd<float>(d, a, add, s);
}

hipError_t causal_conv_step(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s) { return causal_conv_fwd(d, a, s); }

}  // namespace ucd
