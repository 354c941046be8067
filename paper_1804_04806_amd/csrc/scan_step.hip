// Selective state space scan, one token of each sequence.
//
// The states, 4 bytes each, are read and written once, everything else is a sixteenth of that and less: memory bounds it.  One lane to 4 neighbouring
// states, so that a wave reads and writes whole lines; lanes of one channel each compute its step and gate (30 vector instructions, hidden
// behind the loads) rather than wait for each other.  256 sequences, 4096 channels, 16 states: 27.6 us, 5.2 TB/s, with the states of 67 MB in the card's
// cache, 39.7 (3.6) from memory; one sequence, 2048 channels: 3.1 us, which is a launch's own time.
#include <algorithm>

#include "scan_common.hpp"

namespace ucd {
namespace {
using namespace seq;

struct StepParams {
    ucd_scan_t d;
    ucd_scan_in_t in;
    int per_group;
    float *state;
    void *y;
};

// LPC lanes to a channel; grid.x over channels, grid.y over sequences
template <class T, int LPC, bool WIDE>
__global__ __launch_bounds__(256) void scan_step_kernel(StepParams p)
{
    const ucd_scan_t &d = p.d;
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    const int c = i / LPC, q = i % LPC, n0 = 4 * q;
    if (c >= d.D) return;       // whole channels: lanes that are summed up leave together
    const int haven = min(4, d.N - n0);
    const int g = d.G == 1 ? 0 : c / p.per_group;
    for (int b = blockIdx.y; b < d.B; b += gridDim.y) {
        const int slot = p.in.slots ? p.in.slots[b] : b;
        T *y_at = (T *)p.y + b * d.y_b + c;
        if (p.in.slots && (slot < 0 || slot >= d.n_slots)) {
            if (q == 0) *y_at = from_f<T>(0.f);
            continue;
        }
        float *state = p.state + ((long)slot * d.D + c) * d.N + n0;
        const Pack<float, 4> h0 = load_pack<WIDE, float, 4>(state, haven), A = load_pack<WIDE, float, 4>(p.in.A + (long)c * d.N + n0, haven);
        const Pack<T, 4> bm = load_pack<WIDE, T, 4>((const T *)p.in.Bm + b * d.Bm_b + (long)g * d.N + n0, haven);
        const Pack<T, 4> cm = load_pack<WIDE, T, 4>((const T *)p.in.Cm + b * d.Cm_b + (long)g * d.N + n0, haven);
        const float u = to_f(((const T *)p.in.u)[b * d.u_b + c]), raw = to_f(((const T *)p.in.dt)[b * d.dt_b + c]);
        const float z = p.in.z ? to_f(((const T *)p.in.z)[b * d.z_b + c]) : 0.f;
        const float skip = p.in.skip ? p.in.skip[c] : 0.f;
        float s = raw + (p.in.dt_bias ? p.in.dt_bias[c] : 0.f);
        if (d.softplus) s = softplus<T>(s);
        const float gain = s * u, s2 = s * kLog2e;
        Pack<float, 4> h;
        float y = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            h.v[j] = fmaf(exp2_fast(s2 * A.v[j]), h0.v[j], gain * to_f(bm.v[j]));
            y = fmaf(h.v[j], to_f(cm.v[j]), y);
        }
        store_pack<WIDE, float, 4>(state, h, haven);
        y = fmaf(skip, u, sum_lanes<LPC>(y));
        if (p.in.z) y *= z * sigmoid(z);
        if (q == 0) *y_at = from_f<T>(y);
    }
}

template <class T, int LPC>
hipError_t launch(const StepParams &p, bool wide, hipStream_t s)
{
    const dim3 grid((unsigned)(((long)p.d.D * LPC + 255) / 256), (unsigned)std::min(p.d.B, 65535));
    if (wide) scan_step_kernel<T, LPC, true><<<grid, 256, 0, s>>>(p);
    else scan_step_kernel<T, LPC, false><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <class T>
hipError_t launch(const StepParams &p, bool wide, hipStream_t s)
{
    const int N = p.d.N;
    if (N <= 4) return launch<T, 1>(p, wide, s);
    if (N <= 8) return launch<T, 2>(p, wide, s);
    if (N <= 16) return launch<T, 4>(p, wide, s);
    if (N <= 32) return launch<T, 8>(p, wide, s);
    return launch<T, 16>(p, wide, s);
}

}  // namespace

hipError_t scan_step(const ucd_scan_t &d, const ucd_scan_in_t &in, float *state, void *y, hipStream_t s)
{
    StepParams p{d, in, d.D / d.G, state, y};
    const bool wide = d.N % 4 == 0;
    return d.dtype == 1 ? launch<bf16_t>(p, wide, s) : launch<float>(p, wide, s);
}

}  // namespace ucd
