// Selective state space scan, Backward: scan_bwd_kernel and the joins of its partial sums.
//
// With x the decayed gradient of the state that a token receives from its successor, dyp = dy SiLU(z):
//   dh_t = dyp_t Cm_t + x_{t+1},  x_t = exp(d_t A) dh_t,  x behind the last token = dstate_out,
//   dCm_t = sum over channels dyp_t h_t,  dBm_t = sum over channels dh_t d_t u_t,
//   dd_t = sum_n x_t h_{t-1} A + u_t sum_n dh_t Bm_t,  dA = sum_t x_t h_{t-1} d_t,
//   du_t = d_t sum_n dh_t Bm_t + skip dyp_t,  dz_t = dy_t (sum_n Cm_t h_t + skip u_t) SiLU'(z_t).
// The states come again from those that Forward kept every eight tokens (all of them would be eight times the memory of u, dt, z and y together at 16
// states; recomputing costs five of the twenty slots that a state and token take).  Sums over the states stay in a channel's lanes, sums over the
// channels go through the waves' own exchanges, a workgroup's LDS and one row of partial sums per workgroup: no atomics, the order is fixed.
// The vector units bound it: 8 x 2048 tokens, 2048 channels, 16 states, bf16: 509 us, issuing in 75 % of the time, and 14 + 5 for the joins.
#include <algorithm>

#include "scan_common.hpp"

namespace ucd {
namespace {
using namespace seq;

// Sums of two tokens' dBm and dCm over the wave's channels: v[token][kind][state], channels are the lane bits from LPC up.  Each exchange of halves
// adds up two values at once; r[state] is then token (lane bit 5), kind (lane bit 4), in every lane of the row with that state quarter.
template <class W>
__device__ __forceinline__ void sum_channels(float (&v)[2][2][W::NPL], float (&r)[W::NPL])
{
    constexpr int LPC = W::LPC, NPL = W::NPL;
    float w[2][NPL];
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < NPL; ++j) {
            swap_halves(v[0][k][j], v[1][k][j]);
            w[k][j] = v[0][k][j] + v[1][k][j];
        }
#pragma unroll
    for (int j = 0; j < NPL; ++j) {
        swap_rows(w[0][j], w[1][j]);
        r[j] = w[0][j] + w[1][j];
        if (LPC < 16) r[j] += dpp<kRor8>(r[j]);
        if (LPC < 8) r[j] += dpp<kRor4>(r[j]);
    }
}

// What two tokens bring from LDS: d_t, d_t u_t and dyp_t of the lane's channel, Bm and Cm of its states.
template <class W>
struct TwoTokens {
    float2 s[2];
    float g[2];
    Pack<float, W::NPL> b[2], c[2];
    __device__ __forceinline__ void load(const float2 *step, const float *dys, const float *bm, const float *cm, const ScanPlace<W> &at, int t, bool all)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = step[(t + i) * W::CW + at.c];
            b[i] = *reinterpret_cast<const Pack<float, W::NPL> *>(bm + (t + i) * W::NP + at.n0);
            if (!all) continue;
            g[i] = dys[(t + i) * W::CW + at.c];
            c[i] = *reinterpret_cast<const Pack<float, W::NPL> *>(cm + (t + i) * W::NP + at.n0);
        }
    }
};

// One segment of a sequence from its last token to its first, 4 x 64 / LPC channels per workgroup.  STATE_ONLY: from zero, the gradient of the state
// before the segment alone.
template <class T, class W, bool WIDE, bool GATE, bool STATE_ONLY>
__global__ __launch_bounds__(64 * kWaves, 2) void scan_bwd_kernel(ScanParams p, unsigned units)
{
    constexpr int LPC = W::LPC, NPL = W::NPL;
    typedef TwoTokens<W> Ahead;
    constexpr int BC = 2 * kTile * W::NP;
    __shared__ alignas(16) float2 lds_step[kWaves][kTile * W::CW];      // d_t, d_t u_t
    __shared__ alignas(16) float lds_dy[kWaves][kTile * W::CW];         // dyp_t
    __shared__ alignas(16) float lds_bc[kWaves][BC];
    __shared__ alignas(16) float lds_out[kWaves][STATE_ONLY ? 1 : 3 * kTile * W::CW];   // sums over the states: dh Bm, x h A, Cm h
    __shared__ alignas(16) float lds_sum[STATE_ONLY ? 1 : 2][STATE_ONLY ? 1 : kWaves][STATE_ONLY ? 1 : BC];
    // the lane's dA of the tiles so far: a tile's sum first, then theirs, or thousands of tokens' roundings would add up
    __shared__ Pack<float, NPL> lds_dA[STATE_ONLY ? 1 : kWaves][STATE_ONLY ? 1 : 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    float2 *step = lds_step[wave];
    float *dys = lds_dy[wave], *bm = lds_bc[wave], *cm = bm + kTile * W::NP;
    float *gs = lds_out[wave], *es = gs + kTile * W::CW, *ys = es + kTile * W::CW;
    const ucd_scan_t &d = p.d;
    const int low = lane % 16 / LPC;       // the channel bits of a lane within its row

    for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const ScanPlace<W> at(p, unit, WIDE);
        if (STATE_ONLY && at.seg == 0) continue;
        const int n = scan_length(p, at.b);
        const int tile0 = at.seg * p.seg_tiles, tile1 = min(p.tiles, tile0 + p.seg_tiles);
        const long ch = at.c0 + at.c;
        const bool mine = at.c < at.have;

        float A2[NPL], x[NPL], dA[NPL] = {};
        Pack<float, NPL> &all_dA = lds_dA[STATE_ONLY ? 0 : wave][STATE_ONLY ? 0 : lane];
        auto add_dA = [&](bool first) {
            Pack<float, NPL> sum = all_dA;
#pragma unroll
            for (int j = 0; j < NPL; ++j) {
                sum.v[j] = dA[j] + (first ? 0.f : sum.v[j]);
                dA[j] = 0.f;
            }
            all_dA = sum;
        };
        if (!STATE_ONLY) add_dA(true);
        load_states(A2, p.in.A + ch * d.N + at.n0, at.haven);
#pragma unroll
        for (int j = 0; j < NPL; ++j) A2[j] *= kLog2e;
        auto seg_at = [&](int s) { return (((long)at.b * p.segs + s) * d.D + ch) * W::NP + at.n0; };
        const long state_at = ((long)at.b * d.D + ch) * d.N + at.n0;
        load_states(x, p.dstate_out + state_at, p.dstate_out && (at.seg == p.segs - 1 || !STATE_ONLY) ? at.haven : 0);
        if (!STATE_ONLY)
            for (int s = p.segs - 1; s > at.seg; --s) {
                float end[NPL];
                load_own(end, p.seg_state + seg_at(s), mine);
                // the last segment began with dstate_out
                if (s == p.segs - 1) {
#pragma unroll
                    for (int j = 0; j < NPL; ++j) x[j] = end[j];
                } else join_segment(x, A2, mine ? p.seg_step[((long)at.b * p.segs + s) * d.D + ch] : 0.f, end);
            }
        float bias[W::VE], skip[W::VE], dskip[W::VE] = {}, dbias[W::VE] = {}, steps = 0.f;
#pragma unroll
        for (int i = 0; i < W::VE; ++i) {
            bias[i] = at.channel(i) && p.in.dt_bias ? p.in.dt_bias[at.c0 + at.ch0 + i] : 0.f;
            skip[i] = at.channel(i) && p.in.skip ? p.in.skip[at.c0 + at.ch0 + i] : 0.f;
        }

        const long t_last = (long)(tile1 - 1) * kTile, e = sizeof(T);      // of the last tile
        const char *u_at = row_base<T>(p.in.u, d.u_b, d.u_l, at, t_last), *dt_at = row_base<T>(p.in.dt, d.dt_b, d.dt_l, at, t_last);
        const char *z_at = row_base<T>(p.in.z, d.z_b, d.z_l, at, t_last), *dy_at = row_base<T>(p.dy, d.y_b, d.y_l, at, t_last);
        const char *bm_at = bc_base<T>(p.in.Bm, d.Bm_b, d.Bm_l, at, t_last, d.N), *cm_at = bc_base<T>(p.in.Cm, d.Cm_b, d.Cm_l, at, t_last, d.N);
        char *du_at = const_cast<char *>(row_base<T>(p.g.u, d.u_b, d.u_l, at, t_last)), *ddt_at = const_cast<char *>(row_base<T>(p.g.dt, d.dt_b, d.dt_l, at, t_last));
        char *dz_at = const_cast<char *>(row_base<T>(p.g.z, d.z_b, d.z_l, at, t_last));
        const float *saved_at = p.saved + (((long)at.b * p.tiles + tile1 - 1) * (kTile / kKeep) * d.D + at.first) * W::NP;
        const uint32_t state_off = (uint32_t)(at.c0 - at.first + at.c) * W::NP + at.n0;
        Raw<T, W::VE, WIDE> u, dt, z, dy;
        TileStates<T, W> bc;
        bc.clear(bm, d.N);
        float kept[kTile / kKeep][NPL];
        uint32_t u_off, dt_off, z_off, dy_off;
        auto place = [&](int last) {
            u_off = row_offset<T>(at, d.u_l, last);
            dt_off = row_offset<T>(at, d.dt_l, last);
            dy_off = row_offset<T>(at, d.y_l, last);
            if (GATE) z_off = row_offset<T>(at, d.z_l, last);
            bc.place(p, last);
        };
        place(kTile);
        auto load = [&](int tile, auto whole) {      // and on to the tile before it; whole: all its tokens are there
            constexpr bool FULL = decltype(whole)::value;
            const int left = n - tile * kTile;
            if (FULL || left > 0) {
                if (!FULL && left < kTile) place(left - 1);
                u.load(u_at, u_off, at.have - at.ch0);
                dt.load(dt_at, dt_off, at.have - at.ch0);
                dy.load(dy_at, dy_off, at.have - at.ch0);
                if (GATE) z.load(z_at, z_off, at.have - at.ch0);
                bc.load(bm_at, cm_at);
                if (!STATE_ONLY)
#pragma unroll
                    for (int i = 0; i < kTile / kKeep; ++i) load_own(kept[i], saved_at + i * (long)d.D * W::NP + state_off, mine);
                if (!FULL && left < kTile) place(kTile);
            }
            u_at -= kTile * e * d.u_l;
            dt_at -= kTile * e * d.dt_l;
            dy_at -= kTile * e * d.y_l;
            if (GATE) z_at -= kTile * e * d.z_l;
            bm_at -= kTile * e * d.Bm_l;
            cm_at -= kTile * e * d.Cm_l;
            saved_at -= (kTile / kKeep) * (long)d.D * W::NP;
        };
        // FULL: all tokens and channels of the segment are there, as is the rule (see Forward).
        auto walk = [&](auto whole) {
        constexpr bool FULL = decltype(whole)::value;
        if (tile1 > tile0) load(tile1 - 1, whole);
        for (int tile = tile1 - 1; tile >= tile0; --tile) {
            const int left = n - tile * kTile;
            float ut[W::VE], st[W::VE], rate[W::VE], dyp[W::VE], dzt[W::VE];
            if (FULL || left > 0) {
                bc.stage(bm, d.N);
#pragma unroll
                for (int i = 0; i < W::VE; ++i) {
                    const bool there = FULL || (at.tok < left && at.channel(i));
                    ut[i] = u.get(i);
                    float s = dt.get(i) + bias[i], slope;
                    const float soft = softplus<T>(s, &slope);
                    s = d.softplus ? soft : s;
                    rate[i] = d.softplus ? slope : 1.f;
                    s = there ? s : 0.f;
                    st[i] = s;
                    float g = dy.get(i);
                    if (GATE) {
                        const float v = z.get(i), sg = sigmoid(v);
                        dzt[i] = g * sg * fmaf(v, 1.f - sg, 1.f);
                        g *= v * sg;
                    }
                    g = there ? g : 0.f;
                    dyp[i] = g;
                    if (FULL || at.channel(i)) {
                        step[at.tok * W::CW + at.ch0 + i] = make_float2(s, there ? s * ut[i] : 0.f);
                        dys[at.tok * W::CW + at.ch0 + i] = g;
                    }
                }
                float before[kTile / kKeep][NPL];
#pragma unroll
                for (int i = 0; i < kTile / kKeep; ++i)
#pragma unroll
                    for (int j = 0; j < NPL; ++j) before[i][j] = kept[i][j];
                if (tile > tile0) load(tile - 1, whole);
                wave_lds_order();
                if (STATE_ONLY) {
#pragma unroll
                    for (int t = kTile - 1; t >= 0; --t) {
                        const float s = step[t * W::CW + at.c].x, g = dys[t * W::CW + at.c];
                        const Pack<float, NPL> c = *reinterpret_cast<const Pack<float, W::NPL> *>(cm + t * W::NP + at.n0);
#pragma unroll
                        for (int j = 0; j < NPL; ++j) x[j] = exp2_fast(s * A2[j]) * fmaf(g, c.v[j], x[j]);
                        steps += s;
                    }
                } else {
                    float *sums = lds_sum[tile & 1][wave];
                    LaneSums<LPC> g_sums, e_sums, y_sums;
                    float v[2][2][NPL];
#pragma unroll
                    for (int part = kTile / kKeep - 1; part >= 0; --part) {
                        const int p0 = part * kKeep;
                        float a[kKeep][NPL], h[kKeep + 1][NPL];
#pragma unroll
                        for (int j = 0; j < NPL; ++j) h[0][j] = before[part][j];
                        // LDS is read two tokens ahead, as in Forward
                        Ahead now, next;
                        now.load(step, dys, bm, cm, at, p0, false);
#pragma unroll
                        for (int i = 0; i < kKeep; ++i) {
                            if (i % 2 == 0) {
                                if (i > 0) now = next;
                                if (i + 2 < kKeep) next.load(step, dys, bm, cm, at, p0 + i + 2, false);
                                else next.load(step, dys, bm, cm, at, p0 + kKeep - 2, true);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                            const float2 s = now.s[i % 2];
                            const Pack<float, NPL> b = now.b[i % 2];
#pragma unroll
                            for (int j = 0; j < NPL; ++j) {
                                a[i][j] = exp2_fast(s.x * A2[j]);
                                h[i + 1][j] = fmaf(a[i][j], h[i][j], s.y * b.v[j]);
                            }
                        }
#pragma unroll
                        for (int i = kKeep - 1; i >= 0; --i) {
                            const int t = p0 + i;
                            if (i % 2 == 1) {
                                now = next;
                                if (i > 1) next.load(step, dys, bm, cm, at, t - 3, true);
                                __builtin_amdgcn_sched_barrier(0);
                            }
                            const float2 s = now.s[i % 2];
                            const float g = now.g[i % 2];
                            const Pack<float, NPL> b = now.b[i % 2], c = now.c[i % 2];
                            float gt = 0.f, et = 0.f, yt = 0.f;
#pragma unroll
                            for (int j = 0; j < NPL; ++j) {
                                const float dh = fmaf(g, c.v[j], x[j]);
                                v[t % 2][0][j] = dh * s.y;
                                v[t % 2][1][j] = g * h[i + 1][j];
                                gt = fmaf(dh, b.v[j], gt);
                                if (GATE) yt = fmaf(c.v[j], h[i + 1][j], yt);
                                x[j] = a[i][j] * dh;
                                const float w = x[j] * h[i][j];
                                et = fmaf(w, A2[j], et);
                                dA[j] = fmaf(w, s.x, dA[j]);
                            }
                            g_sums.add(t, gt, at.q);
                            e_sums.add(t, et, at.q);
                            if (GATE) y_sums.add(t, yt, at.q);
                            if (t % LPC == 0) {
                                const int o = (t + at.q) * W::CW + at.c;
                                gs[o] = g_sums.get(at.q);
                                es[o] = e_sums.get(at.q);
                                if (GATE) ys[o] = y_sums.get(at.q);
                            }
                            if (t % 2 == 0) {
                                float r[NPL];
                                sum_channels<W>(v, r);
                                float *o = sums + ((t + lane / 32) * 2 + lane / 16 % 2) * W::NP + at.n0;
                                // the lanes of a row that differ in the channel share out its NPL sums
                                constexpr int SHARES = 16 / LPC < NPL ? 16 / LPC : NPL, EACH = NPL / SHARES;
                                Pack<float, EACH> mine_r;
#pragma unroll
                                for (int j = 0; j < EACH; ++j) {
                                    mine_r.v[j] = r[j];
#pragma unroll
                                    for (int k = 1; k < SHARES; ++k) mine_r.v[j] = low == k ? r[k * EACH + j] : mine_r.v[j];
                                }
                                if (low < SHARES) *reinterpret_cast<Pack<float, EACH> *>(o + low * EACH) = mine_r;
                            }
                        }
                    }
                    add_dA(false);
                }
                wave_lds_order();
            } else if (tile > tile0) {
                load(tile - 1, whole);
            }
            if (!STATE_ONLY) {
                const bool token = at.tok < d.L - tile * kTile;
                Pack<T, W::VE> du, ddt, dz;
                float g[W::VE], et[W::VE], yt[W::VE];
                lds_row<W, FULL>(g, gs, at);
                lds_row<W, FULL>(et, es, at);
                if (GATE) lds_row<W, FULL>(yt, ys, at);
#pragma unroll
                for (int i = 0; i < W::VE; ++i) {
                    const bool there = FULL || (at.tok < left && at.channel(i));
                    const float rise = fmaf(et[i], kLn2, g[i] * ut[i]) * rate[i];
                    du.v[i] = from_f<T>(there ? fmaf(g[i], st[i], skip[i] * dyp[i]) : 0.f);
                    ddt.v[i] = from_f<T>(there ? rise : 0.f);
                    if (GATE) dz.v[i] = from_f<T>(there ? dzt[i] * fmaf(skip[i], ut[i], yt[i]) : 0.f);
                    dskip[i] += there ? dyp[i] * ut[i] : 0.f;
                    dbias[i] += there ? rise : 0.f;
                }
                store_row<T, W, WIDE, FULL>(du_at, u_off, du, at, token);
                store_row<T, W, WIDE, FULL>(ddt_at, dt_off, ddt, at, token);
                if (GATE) store_row<T, W, WIDE, FULL>(dz_at, z_off, dz, at, token);
                du_at -= kTile * e * d.u_l;
                ddt_at -= kTile * e * d.dt_l;
                if (GATE) dz_at -= kTile * e * d.z_l;
                wave_lds_order();
                if (FULL || left > 0) {
                    // the waves' sums, in their order; the other of the two buffers is written meanwhile
                    lds_barrier();
                    float *o = p.part_bc + ((((long)at.b * p.tiles + tile) * d.G + at.g) * p.blocks + at.block) * BC;
                    constexpr int EACH = (BC + 64 * kWaves - 1) / (64 * kWaves);
#pragma unroll
                    for (int k = 0; k < EACH; ++k) {
                        const int i = (int)threadIdx.x + k * 64 * kWaves;
                        if (BC % (64 * kWaves) != 0 && i >= BC) continue;
                        float v = lds_sum[tile & 1][0][i];
#pragma unroll
                        for (int w = 1; w < kWaves; ++w) v += lds_sum[tile & 1][w][i];
                        o[i] = v;
                    }
                }
            }
        }
        };
        if (n >= tile1 * kTile && at.have == W::CW) {
            walk(std::integral_constant<bool, WIDE>());
        } else {
            // channels that are not there add zeros to the sums
#pragma unroll
            for (int i = 0; i < W::VE; ++i) {
                step[lane + i * 64] = make_float2(0.f, 0.f);
                dys[lane + i * 64] = 0.f;
            }
            walk(std::false_type());
        }
        if (STATE_ONLY) {
            store_own(p.seg_state + seg_at(at.seg), x, mine);
            if (at.q == 0 && mine) p.seg_step[((long)at.b * p.segs + at.seg) * d.D + ch] = steps;
        } else {
            if (p.g.state && at.seg == 0) store_states(p.g.state + state_at, x, at.haven);
            float *o = p.part_w + (((long)at.b * p.segs + at.seg) * d.D) * (d.N + 2);
#pragma unroll
            for (int j = 0; j < NPL; ++j)
                if (j < at.haven) o[ch * (d.N + 2) + at.n0 + j] = all_dA.v[j];
            // over the lanes that load other tokens of the same channels
#pragma unroll
            for (int e = 0; e < W::VE; ++e) {
                for (int k = W::LR; k < 64; k *= 2) {
                    dskip[e] += __shfl_xor(dskip[e], k);
                    dbias[e] += __shfl_xor(dbias[e], k);
                }
                if (lane < W::LR && at.channel(e)) {
                    float *w = o + (at.c0 + at.ch0 + e) * (long)(d.N + 2) + d.N;
                    w[0] = dskip[e];
                    w[1] = dbias[e];
                }
            }
            lds_barrier();      // lds_sum is written again by the next unit
        }
    }
}

// dBm and dCm: four neighbouring elements of either per thread, over the workgroups of a group's channels.
template <class T>
__global__ __launch_bounds__(256) void scan_join_bc_kernel(ScanParams p, int np, long total)
{
    const ucd_scan_t &d = p.d;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < total; i += gridDim.x * 256l) {
        const int k = (int)(i % (np / 4)) * 4, kind = (int)(i / (np / 4) % 2);
        const long row = i / (np / 4) / 2;
        const int g = (int)(row % d.G), t = (int)(row / d.G % d.L), b = (int)(row / d.G / d.L);
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (t < scan_length(p, b)) {
            const float *o = p.part_bc + ((((long)b * p.tiles + t / kTile) * d.G + g) * p.blocks) * (2l * kTile * np) + (t % kTile * 2 + kind) * np + k;
#pragma unroll 8
            for (unsigned s = 0; s < p.blocks; ++s) {
                const float4 w = *reinterpret_cast<const float4 *>(o + s * (2l * kTile * np));
                v.x += w.x;
                v.y += w.y;
                v.z += w.z;
                v.w += w.w;
            }
        }
        T *out = (kind ? (T *)p.g.Cm + b * d.Cm_b + (long)t * d.Cm_l : (T *)p.g.Bm + b * d.Bm_b + (long)t * d.Bm_l) + (long)g * d.N + k;
        const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k + j < d.N) out[j] = from_f<T>(f[j]);
    }
}

// dA, dskip and ddt_bias, over sequences and segments.
__global__ __launch_bounds__(kJoinThreads) void scan_join_weights_kernel(ScanParams p)
{
    const ucd_scan_t &d = p.d;
    join_columns(p.part_w, (long)d.B * p.segs, (long)d.D * (d.N + 2), [&](long i, float v) {
        const int k = (int)(i % (d.N + 2));
        const long c = i / (d.N + 2);
        float *out = k < d.N ? p.g.A + c * d.N + k : k == d.N ? (p.in.skip ? p.g.skip + c : nullptr) : p.in.dt_bias ? p.g.dt_bias + c : nullptr;
        if (out) *out = v + (p.add ? *out : 0.f);
    });
}

template <class T, class W, bool WIDE, bool GATE>
void launch_main(const ScanParams &p, hipStream_t s)
{
    const unsigned units = scan_units(p), grid = std::min(units, 1u << 22);
    if (units == 0) return;       // no sequences: the joins write the gradients of the weights
    if (p.segs > 1) scan_bwd_kernel<T, W, WIDE, GATE, true><<<grid, 64 * kWaves, 0, s>>>(p, units);
    scan_bwd_kernel<T, W, WIDE, GATE, false><<<grid, 64 * kWaves, 0, s>>>(p, units);
}

template <class T, class W, bool WIDE>
hipError_t launch(const ScanParams &p, hipStream_t s)
{
    if (p.in.z) launch_main<T, W, WIDE, true>(p, s);
    else launch_main<T, W, WIDE, false>(p, s);
    const ucd_scan_t &d = p.d;
    const long elements = (long)d.B * d.L * d.G * 2 * W::NP / 4;
    if (elements > 0)
        scan_join_bc_kernel<T><<<(unsigned)std::min((elements + 255) / 256, 1l << 22), 256, 0, s>>>(p, W::NP, elements);
    scan_join_weights_kernel<<<join_grid((long)d.D * (d.N + 2)), kJoinThreads, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t scan_bwd(const ucd_scan_t &d, const ucd_scan_in_t &in, const void *dy, const float *dstate_out, const float *saved,
                    const ucd_scan_grad_t &g, bool add, void *ws, hipStream_t s)
{
    ScanParams p{};
    scan_params(d, in, UCD_SEQ_BWD, ws, p);
    p.dy = dy;
    p.dstate_out = dstate_out;
    p.saved = const_cast<float *>(saved);
    p.g = g;
    p.add = add;
    const bool wide = scan_wide(d);
    return scan_by_states(d, [&](auto wave) {
        typedef decltype(wave) W;
        if (d.dtype == 1) return wide ? launch<bf16_t, W, true>(p, s) : launch<bf16_t, W, false>(p, s);
        return wide ? launch<float, W, true>(p, s) : launch<float, W, false>(p, s);
    });
}

}  // namespace ucd
