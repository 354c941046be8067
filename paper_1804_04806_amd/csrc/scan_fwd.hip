// Selective state space scan, Forward: scan_fwd_kernel.
//
// Per channel c with its step d_t = softplus(dt_t + dt_bias), and per state n:
//   h_t = exp(d_t A) h_{t-1} + d_t u_t Bm_t,  y_t = (sum_n Cm_t h_t + skip u_t) SiLU(z_t).
// A state and token cost a multiplication, an exponential (two issue slots), a multiplication and two fused ones, where it moves 1 / N of some
// bytes: the vector units bound it, and a wave that has its SIMD to itself has to keep them fed.  8 x 2048 tokens, 2048 channels, 16 states, bf16:
// 196 us with the states that Backward needs, 182 without; the units issue in 67 % of the time, and six slots alone would take
// 82 us.  The tokens of a sequence follow each other, so lanes are states and channels, tiles of tokens are what is loaded at
// once, and sequences are cut only where there are too few channels.  (A tile's outputs written behind the next tile's sums: 316 us against 251 then;
// eight lanes to a channel instead of four: 256 against 205, and 539 against 380 for twice as many sequences.)
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
        const ScanPlace<W> at(p, unit, WIDE);
        if (at.have == 0 || (STATE_ONLY && at.seg == p.segs - 1)) continue;     // nobody needs the last segment's end
        const int slot = p.in.slots ? p.in.slots[at.b] : at.b;
        const bool idle = p.in.slots && (slot < 0 || slot >= d.n_slots);
        const int n = idle ? 0 : scan_length(p, at.b);
        const int tile0 = at.seg * p.seg_tiles, tile1 = min(p.tiles, tile0 + p.seg_tiles);
        const long ch = at.c0 + at.c;

        float A2[NPL], h[NPL];
        load_states(A2, p.in.A + ch * d.N + at.n0, at.haven);
#pragma unroll
        for (int j = 0; j < NPL; ++j) A2[j] *= kLog2e;
        const long state_at = ((long)slot * d.D + ch) * d.N + at.n0;
        auto seg_at = [&](int s) { return (((long)at.b * p.segs + s) * d.D + ch) * W::NP + at.n0; };
        const bool mine = at.c < at.have;
        if (STATE_ONLY || p.segs == 1) {
            load_states(h, p.state_in + state_at, p.state_in && !idle && at.seg == 0 ? at.haven : 0);
            // state_out may be state_in: the second launch takes the first state from here
            if (STATE_ONLY && at.seg == 0) store_own(p.seg_state + seg_at(0), h, mine);
            if (STATE_ONLY)
#pragma unroll
                for (int j = 0; j < NPL; ++j) h[j] = 0.f;
        } else {
            load_own(h, p.seg_state + seg_at(0), mine);
            for (int s = 0; s < at.seg; ++s) {
                float end[NPL];
                load_own(end, p.seg_state + seg_at(s + 1), mine);
                join_segment(h, A2, mine ? p.seg_step[((long)at.b * p.segs + s) * d.D + ch] : 0.f, end);
            }
        }
        float bias[W::VE], skip[W::VE], steps = 0.f;
#pragma unroll
        for (int i = 0; i < W::VE; ++i) {
            const bool have = at.channel(i);
            bias[i] = have && p.in.dt_bias ? p.in.dt_bias[at.c0 + at.ch0 + i] : 0.f;
            skip[i] = have && p.in.skip ? p.in.skip[at.c0 + at.ch0 + i] : 0.f;
        }

        const long t_first = (long)tile0 * kTile, e = sizeof(T);
        const char *u_at = row_base<T>(p.in.u, d.u_b, d.u_l, at, t_first), *dt_at = row_base<T>(p.in.dt, d.dt_b, d.dt_l, at, t_first);
        const char *z_at = row_base<T>(p.in.z, d.z_b, d.z_l, at, t_first);
        const char *bm_at = bc_base<T>(p.in.Bm, d.Bm_b, d.Bm_l, at, t_first, d.N), *cm_at = bc_base<T>(p.in.Cm, d.Cm_b, d.Cm_l, at, t_first, d.N);
        char *y_at = const_cast<char *>(row_base<T>(p.y, d.y_b, d.y_l, at, t_first));
        float *saved_at = p.saved + (((long)at.b * p.tiles + tile0) * (kTile / kKeep) * d.D + at.first) * W::NP;
        const uint32_t state_off = (uint32_t)(at.c0 - at.first + at.c) * W::NP + at.n0, y_off = row_offset<T>(at, d.y_l, kTile);
        Raw<T, W::VE, WIDE> u, dt, z;
        TileStates<T, W> bc;
        bc.clear(bm, d.N);
        uint32_t u_off, dt_off, z_off;
        auto place = [&](int last) {
            u_off = row_offset<T>(at, d.u_l, last);
            dt_off = row_offset<T>(at, d.dt_l, last);
            if (GATE) z_off = row_offset<T>(at, d.z_l, last);
            bc.place(p, last);
        };
        place(kTile);
        auto load = [&](int tile, auto full) {      // and on to the next tile; full: all its tokens are there
            constexpr bool FULL = decltype(full)::value;
            const int left = n - tile * kTile;
            if (!FULL && left <= 0) return;
            if (!FULL && left < kTile) place(left - 1);
            u.load(u_at, u_off, at.have - at.ch0);
            dt.load(dt_at, dt_off, at.have - at.ch0);
            if (GATE) z.load(z_at, z_off, at.have - at.ch0);
            bc.load(bm_at, cm_at);
            u_at += kTile * e * d.u_l;
            dt_at += kTile * e * d.dt_l;
            if (GATE) z_at += kTile * e * d.z_l;
            bm_at += kTile * e * d.Bm_l;
            cm_at += kTile * e * d.Cm_l;
        };
        // FULL: all tokens and channels of the segment are there, as is the rule.  Without masks and without branches around the stores, behind which the
        // loads' arrival could only be told by waiting for the stores too.  SAVE: states are kept for Backward.
        auto walk = [&](auto full, auto save) {
            constexpr bool FULL = decltype(full)::value, SAVE = decltype(save)::value;
            if (tile1 > tile0) load(tile0, full);
            for (int tile = tile0; tile < tile1; ++tile) {
                const int left = n - tile * kTile;
                const bool there = FULL || at.tok < left;
                float ut[W::VE], zt[W::VE];
                if (FULL || left > 0) {
                    bc.stage(bm, d.N);
#pragma unroll
                    for (int i = 0; i < W::VE; ++i) {
                        ut[i] = u.get(i);
                        float s = dt.get(i) + bias[i];
                        const float soft = softplus<T>(s);
                        s = d.softplus ? soft : s;
                        s = there ? s : 0.f;     // padding: the state stays
                        if (FULL || at.channel(i)) step[at.tok * W::CW + at.ch0 + i] = make_float2(s, there ? s * ut[i] : 0.f);
                        if (GATE) {
                            const float v = z.get(i);
                            zt[i] = v * sigmoid(v);
                        }
                    }
                    if (tile + 1 < tile1) load(tile + 1, full);
                    wave_lds_order();
                    auto keep = [&]() {
                        store_own(saved_at + state_off, h, FULL || mine);
                        saved_at += (long)d.D * W::NP;
                    };
                    if (SAVE) keep();
                    LaneSums<LPC> sums;
                    // the next tokens' values are on their way from LDS while these are computed: left to itself the compiler reads them just
                    // before their use, and a wave that has its SIMD to itself waits for each
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
                            if (SAVE && t % kKeep == kKeep - 1 && t + 1 < kTile) keep();
                            sums.add(t, y, at.q);
                            if (t % LPC == LPC - 1) ys[(t - LPC + 1 + at.q) * W::CW + at.c] = sums.get(at.q);
                        }
                    }
                    wave_lds_order();
                }
                if (!STATE_ONLY) {
                    Pack<T, W::VE> out;
                    float yt[W::VE];
                    lds_row<W, FULL>(yt, ys, at);
#pragma unroll
                    for (int i = 0; i < W::VE; ++i) {
                        float y = fmaf(skip[i], ut[i], yt[i]);
                        if (GATE) y *= zt[i];
                        out.v[i] = from_f<T>(there ? y : 0.f);
                    }
                    store_row<T, W, WIDE, FULL>(y_at, y_off, out, at, at.tok < d.L - tile * kTile);
                    y_at += kTile * e * d.y_l;
                    wave_lds_order();
                }
            }
        };
        const bool full = n >= tile1 * kTile && at.have == W::CW, save = !STATE_ONLY && p.saved;
        typedef std::integral_constant<bool, !STATE_ONLY> Save;
        if (full && save) walk(std::integral_constant<bool, WIDE>(), Save());
        else if (full) walk(std::integral_constant<bool, WIDE>(), std::false_type());
        else if (save) walk(std::false_type(), Save());
        else walk(std::false_type(), std::false_type());
        if (STATE_ONLY) {
            store_own(p.seg_state + seg_at(at.seg + 1), h, mine);
            if (at.q == 0 && mine) p.seg_step[((long)at.b * p.segs + at.seg) * d.D + ch] = steps;
        } else if (p.state_out && !idle && at.seg == p.segs - 1) {
            store_states(p.state_out + state_at, h, at.haven);
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
    const bool wide = scan_wide(d);
    return scan_by_states(d, [&](auto wave) {
        typedef decltype(wave) W;
        if (d.dtype == 1) return wide ? launch<bf16_t, W, true>(p, s) : launch<bf16_t, W, false>(p, s);
        return wide ? launch<float, W, true>(p, s) : launch<float, W, false>(p, s);
    });
}

}  // namespace ucd
