// Selective state space scan, Forward: scan_fwd_kernel.
#include <algorithm>
#include <type_traits>

#include "scan_common.hpp"

namespace ucd {
namespace {
using namespace seq;

// What neighbouring tokens bring from LDS: d_t and d_t u_t of the lane's channel, Bm and Cm of its states.
constexpr int kAhead = 2;

template <class W, bool WITH_C>
struct SomeTokens {
    float2 s[kAhead];
    Pack<float, W::NPL> b[kAhead], c[kAhead];
    __device__ __forceinline__ void load(const float2 *step, const float *bm, const float *cm, const ScanPlace<W> &at, int t)
    {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            s[i] = step[(t + i) * W::CW + at.c];
            b[i] = *reinterpret_cast<const Pack<float, W::NPL> *>(bm + (t + i) * W::NP + at.n0);
            if (WITH_C) c[i] = *reinterpret_cast<const Pack<float, W::NPL> *>(cm + (t + i) * W::NP + at.n0);
        }
    }
};

// One segment of a sequence, 4 x 64 / LPC channels per workgroup.  STATE_ONLY: from zero, without outputs; leaves the segment's end state
// and the sum of its steps, from which a second launch without STATE_ONLY finds its segments' first states.
template <class T, class W, bool WIDE, bool GATE, bool STATE_ONLY>
__global__ __launch_bounds__(64 * kWaves, 2) void scan_fwd_kernel(ScanParams p, unsigned units)
{
    constexpr int LPC = W::LPC, NPL = W::NPL;
    typedef SomeTokens<W, !STATE_ONLY> Ahead;
    __shared__ alignas(16) float2 lds_step[kWaves][kTile * W::CW];      // d_t, d_t u_t
    __shared__ alignas(16) float lds_bc[kWaves][2 * kTile * W::NP];
    __shared__ alignas(16) float lds_y[kWaves][STATE_ONLY ? 1 : kTile * W::CW];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float2 *step = lds_step[wave];
    float *bm = lds_bc[wave], *cm = bm + kTile * W::NP, *ys = lds_y[wave];
    const ucd_scan_t &d = p.d;

    for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const ScanPlace<W> at(p, unit);
        if (at.have == 0 || (STATE_ONLY && at.seg == p.segs - 1)) continue;     // nobody needs the last segment's end
        const int slot = p.in.slots ? p.in.slots[at.b] : at.b;
        const bool idle = p.in.slots && (slot < 0 || slot >= d.n_slots);
        const int n = idle ? 0 : scan_length(p, at.b);
        const int tile0 = at.seg * p.seg_tiles, tile1 = min(p.tiles, tile0 + p.seg_tiles);
        const long ch = at.c0 + at.c;

        float A2[NPL], h[NPL];
        load_states<WIDE>(A2, p.in.A + ch * d.N + at.n0, at.haven);
#pragma unroll
        for (int j = 0; j < NPL; ++j) A2[j] *= kLog2e;
        const long state_at = ((long)slot * d.D + ch) * d.N + at.n0;
        auto seg_at = [&](int s) { return (((long)at.b * p.segs + s) * d.D + ch) * d.N + at.n0; };
        if (STATE_ONLY || p.segs == 1) {
            load_states<WIDE>(h, p.state_in + state_at, p.state_in && !idle && at.seg == 0 ? at.haven : 0);
            // state_out may be state_in: the second launch takes the first state from here
            if (STATE_ONLY && at.seg == 0) store_states<WIDE>(p.seg_state + seg_at(0), h, at.haven);
            if (STATE_ONLY)
#pragma unroll
                for (int j = 0; j < NPL; ++j) h[j] = 0.f;
        } else {
            load_states<WIDE>(h, p.seg_state + seg_at(0), at.haven);
            for (int s = 0; s < at.seg; ++s) {
                float end[NPL];
                load_states<WIDE>(end, p.seg_state + seg_at(s + 1), at.haven);
                join_segment(h, A2, at.c < at.have ? p.seg_step[((long)at.b * p.segs + s) * d.D + ch] : 0.f, end);
            }
        }
        float bias[W::VE], skip[W::VE], steps = 0.f;
#pragma unroll
        for (int i = 0; i < W::VE; ++i) {
            const bool have = at.ch0 + i < at.have;
            bias[i] = have && p.in.dt_bias ? p.in.dt_bias[at.c0 + at.ch0 + i] : 0.f;
            skip[i] = have && p.in.skip ? p.in.skip[at.c0 + at.ch0 + i] : 0.f;
        }

        TileRows<T, W, WIDE> u, dt, z;
        TileStates<T, W, WIDE> bc;
        auto load = [&](int tile) {
            const int t0 = tile * kTile;
            if (t0 >= n) return;
            u.load(p.in.u, d.u_b, d.u_l, at, t0, n);
            dt.load(p.in.dt, d.dt_b, d.dt_l, at, t0, n);
            if (!STATE_ONLY && GATE) z.load(p.in.z, d.z_b, d.z_l, at, t0, n);
            bc.load(p, at, t0, n);
        };
        auto keep = [&](int tile, int part) {
            store_states<WIDE>(p.saved + ((((long)at.b * p.tiles + tile) * (kTile / kKeep) + part) * d.D + ch) * d.N + at.n0, h, at.haven);
        };
        load(tile0);
        for (int tile = tile0; tile < tile1; ++tile) {
            const int t0 = tile * kTile;
            float ut[W::P][W::VE], zt[W::P][W::VE];
            if (t0 < n) {
                bc.stage(bm, d.N);
#pragma unroll
                for (int i = 0; i < W::P; ++i) {
                    const int t = i * W::TP + at.tok;
#pragma unroll
                    for (int e = 0; e < W::VE; ++e) {
                        ut[i][e] = u.r[i].get(e);
                        float s = dt.r[i].get(e) + bias[e];
                        const float soft = softplus<T>(s);
                        s = d.softplus ? soft : s;
                        s = t0 + t < n ? s : 0.f;     // padding: the state stays
                        step[t * W::CW + at.ch0 + e] = make_float2(s, t0 + t < n ? s * ut[i][e] : 0.f);
                        if (!STATE_ONLY && GATE) {
                            const float v = z.r[i].get(e);
                            zt[i][e] = v * sigmoid(v);
                        }
                    }
                }
                if (tile + 1 < tile1) load(tile + 1);
                wave_lds_order();
                if (!STATE_ONLY && p.saved) keep(tile, 0);
                float kept = 0.f;
                // two tokens' values are on their way from LDS while the two before them are computed: left to itself the compiler reads them
                // just before their use, and a wave that has its SIMD to itself waits for each
                Ahead now, next;
                now.load(step, bm, cm, at, 0);
#pragma unroll
                for (int t = 0; t < kTile; ++t) {
                    if (t % kAhead == 0) {
                        if (t > 0) now = next;
                        if (t + kAhead < kTile) next.load(step, bm, cm, at, t + kAhead);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    const float2 s = now.s[t % kAhead];
                    const Pack<float, NPL> b = now.b[t % kAhead], c = now.c[t % kAhead];
                    float y = 0.f;
#pragma unroll
                    for (int j = 0; j < NPL; ++j) {
                        h[j] = fmaf(exp2_fast(s.x * A2[j]), h[j], s.y * b.v[j]);
                        if (!STATE_ONLY) y = fmaf(h[j], c.v[j], y);
                    }
                    if (STATE_ONLY) {
                        steps += s.x;
                    } else {
                        if (p.saved && t % kKeep == kKeep - 1 && t + 1 < kTile) keep(tile, (t + 1) / kKeep);
                        y = sum_lanes<LPC>(y);
                        kept = LPC == 1 || at.q == t % LPC ? y : kept;      // each lane of a channel keeps one token in LPC
                        if (t % LPC == LPC - 1) ys[(t - LPC + 1 + at.q) * W::CW + at.c] = kept;
                    }
                }
                wave_lds_order();
            }
            if (!STATE_ONLY) {
#pragma unroll
                for (int i = 0; i < W::P; ++i) {
                    const int t = i * W::TP + at.tok;
                    Pack<T, W::VE> out;
                    float yt[W::VE];
                    lds_row(yt, ys + t * W::CW + at.ch0);
#pragma unroll
                    for (int e = 0; e < W::VE; ++e) {
                        float y = fmaf(skip[e], ut[i][e], yt[e]);
                        if (GATE) y *= zt[i][e];
                        out.v[e] = from_f<T>(t0 + t < n ? y : 0.f);
                    }
                    TileRows<T, W, WIDE>::store(p.y, d.y_b, d.y_l, at, t0, i, out, t0 + t < d.L ? at.have - at.ch0 : 0);
                }
                wave_lds_order();
            }
        }
        if (STATE_ONLY) {
            store_states<WIDE>(p.seg_state + seg_at(at.seg + 1), h, at.haven);
            if (at.q == 0 && at.c < at.have) p.seg_step[((long)at.b * p.segs + at.seg) * d.D + ch] = steps;
        } else if (p.state_out && !idle && at.seg == p.segs - 1) {
            store_states<WIDE>(p.state_out + state_at, h, at.haven);
        }
    }
}

template <class T, class W, bool WIDE, bool GATE>
hipError_t launch(const ScanParams &p, hipStream_t s)
{
    const unsigned units = scan_units(p), grid = std::min(units, 1u << 22);
    if (p.segs > 1) scan_fwd_kernel<T, W, WIDE, false, true><<<grid, 64 * kWaves, 0, s>>>(p, units);
    scan_fwd_kernel<T, W, WIDE, GATE, false><<<grid, 64 * kWaves, 0, s>>>(p, units);
    return hipGetLastError();
}

template <class T, class W, bool WIDE>
hipError_t launch(const ScanParams &p, hipStream_t s)
{
    return p.in.z ? launch<T, W, WIDE, true>(p, s) : launch<T, W, WIDE, false>(p, s);
}

}  // namespace

hipError_t scan_fwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const float *state_in, float *state_out, void *y, float *saved, void *ws,
                    hipStream_t s)
{
    ScanParams p{};
    scan_params(d, in, UCD_SEQ_FWD, ws, p);
    p.state_in = state_in;
    p.state_out = state_out;
    p.y = y;
    p.saved = saved;
    const bool wide = scan_wide(d, in, y, state_in, state_out, nullptr);
    return scan_by_states(d, [&](auto wave) {
        typedef decltype(wave) W;
        if (d.dtype == 1) return wide ? launch<bf16_t, W, true>(p, s) : launch<bf16_t, W, false>(p, s);
        return wide ? launch<float, W, true>(p, s) : launch<float, W, false>(p, s);
    });
}

}  // namespace ucd
