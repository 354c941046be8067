// Group norm with an activation, channels last: Forward and Backward.
#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace {
using namespace seq;

// Sum over a workgroup of 256 threads, in every thread.
__device__ float block_sum(float v, float *lds)
{
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    return lds[0] + lds[1] + lds[2] + lds[3];
}

// One sample's group per workgroup: mean, variance around it, outputs.
template <class T>
__global__ __launch_bounds__(256) void norm_fwd_kernel(ucd_group_norm_t d, const T *x, const float *gamma, const float *beta,
                                                       T *y, float *stats)
{
    __shared__ float lds[4];
    const int cg = d.C / d.G;
    const long m = (long)d.S * cg, units = (long)d.N * d.G;
    for (long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const long n = unit / d.G;
        const int c0 = (int)(unit % d.G) * cg;
        const T *xs = x + n * d.x_n + c0;
        float sum = 0.f;
        for (long i = threadIdx.x; i < m; i += 256) sum += to_f(xs[i / cg * d.x_s + i % cg]);
        const float mean = block_sum(sum, lds) / m;
        float sq = 0.f;
        for (long i = threadIdx.x; i < m; i += 256) {
            const float v = to_f(xs[i / cg * d.x_s + i % cg]) - mean;
            sq += v * v;
        }
        const float rstd = 1.f / sqrtf(block_sum(sq, lds) / m + d.eps);
        if (stats && threadIdx.x == 0) {
            stats[unit] = mean;
            stats[units + unit] = rstd;
        }
        for (long i = threadIdx.x; i < m; i += 256) {
            const int c = (int)(i % cg);
            float u = (to_f(xs[i / cg * d.x_s + c]) - mean) * rstd * gamma[c0 + c] + beta[c0 + c];
            if (d.act == UCD_ACT_SILU) u *= sigmoid(u);
            y[n * d.y_n + i / cg * d.y_s + c0 + c] = from_f<T>(u);
        }
    }
}

__device__ float act_grad(const ucd_group_norm_t &d, float u)
{
    if (d.act != UCD_ACT_SILU) return 1.f;
    const float s = sigmoid(u);
    return s * (1.f + u * (1.f - s));
}

template <class T>
__global__ __launch_bounds__(256) void norm_bwd_kernel(ucd_group_norm_t d, const T *x, const float *gamma, const float *beta,
                                                       const float *stats, const T *dy, T *dx)
{
    __shared__ float lds[4];
    const int cg = d.C / d.G;
    const long m = (long)d.S * cg, units = (long)d.N * d.G;
    for (long unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const long n = unit / d.G;
        const int c0 = (int)(unit % d.G) * cg;
        const T *xs = x + n * d.x_n + c0;
        const T *dys = dy + n * d.y_n + c0;
        const float mean = stats[unit], rstd = stats[units + unit];
        float s1 = 0.f, s2 = 0.f;
        for (long i = threadIdx.x; i < m; i += 256) {
            const int c = (int)(i % cg);
            const float xhat = (to_f(xs[i / cg * d.x_s + c]) - mean) * rstd;
            const float g = gamma[c0 + c] * to_f(dys[i / cg * d.y_s + c]) * act_grad(d, xhat * gamma[c0 + c] + beta[c0 + c]);
            s1 += g;
            s2 += g * xhat;
        }
        s1 = block_sum(s1, lds) / m;
        s2 = block_sum(s2, lds) / m;
        for (long i = threadIdx.x; i < m; i += 256) {
            const int c = (int)(i % cg);
            const float xhat = (to_f(xs[i / cg * d.x_s + c]) - mean) * rstd;
            const float g = gamma[c0 + c] * to_f(dys[i / cg * d.y_s + c]) * act_grad(d, xhat * gamma[c0 + c] + beta[c0 + c]);
            dx[n * d.x_n + i / cg * d.x_s + c0 + c] = from_f<T>(rstd * (g - s1 - xhat * s2));
        }
    }
}

// One channel per workgroup.
template <class T>
__global__ __launch_bounds__(256) void norm_weights_kernel(ucd_group_norm_t d, const T *x, const float *gamma, const float *beta,
                                                           const float *stats, const T *dy, float *dgamma, float *dbeta, bool add)
{
    __shared__ float lds[4];
    const int c = blockIdx.x, g = c / (d.C / d.G);
    const long rows = (long)d.N * d.S, units = (long)d.N * d.G;
    float s1 = 0.f, s2 = 0.f;
    for (long i = threadIdx.x; i < rows; i += 256) {
        const long n = i / d.S, s = i % d.S;
        const float xhat = (to_f(x[n * d.x_n + s * d.x_s + c]) - stats[n * d.G + g]) * stats[units + n * d.G + g];
        const float du = to_f(dy[n * d.y_n + s * d.y_s + c]) * act_grad(d, xhat * gamma[c] + beta[c]);
        s1 += du;
        s2 += du * xhat;
    }
    s1 = block_sum(s1, lds);
    s2 = block_sum(s2, lds);
    if (threadIdx.x == 0) {
        dbeta[c] = s1 + (add ? dbeta[c] : 0.f);
        dgamma[c] = s2 + (add ? dgamma[c] : 0.f);
    }
}

unsigned blocks_of(long units) { return (unsigned)(units < (1 << 20) ? units : (1 << 20)); }

}  // namespace

size_t group_norm_ws_bytes(const ucd_group_norm_t &, int) { return 0; }

template <class T>
static hipError_t fwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w, void *y, float *stats,
                      hipStream_t s)
{
    norm_fwd_kernel<T><<<blocks_of((long)d.N * d.G), 256, 0, s>>>(d, (const T *)x, gamma, beta_w, (T *)y, stats);
    return hipGetLastError();
}

template <class T>
static hipError_t bwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w, const float *stats,
                      const void *dy, void *dx, float *dgamma, float *dbeta, bool add, hipStream_t s)
{
    norm_bwd_kernel<T><<<blocks_of((long)d.N * d.G), 256, 0, s>>>(d, (const T *)x, gamma, beta_w, stats, (const T *)dy, (T *)dx);
    norm_weights_kernel<T><<<d.C, 256, 0, s>>>(d, (const T *)x, gamma, beta_w, stats, (const T *)dy, dgamma, dbeta, add);
    return hipGetLastError();
}

hipError_t group_norm_fwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w, void *y,
                          float *stats, void *, hipStream_t s)
{
    return d.dtype == 1 ? fwd<bf16_t>(d, x, gamma, beta_w, y, stats, s) : fwd<float>(d, x, gamma, beta_w, y, stats, s);
}

hipError_t group_norm_bwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w,
                          const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, bool add, void *,
                          hipStream_t s)
{
    return d.dtype == 1 ? bwd<bf16_t>(d, x, gamma, beta_w, stats, dy, dx, dgamma, dbeta, add, s)
                        : bwd<float>(d, x, gamma, beta_w, stats, dy, dx, dgamma, dbeta, add, s);
}

}  // namespace ucd
