// What the scan's kernels share: how a wave is laid out over channels and states, and how it stages a tile of tokens.
//
// A lane holds 4 neighbouring states of one channel; LPC neighbouring lanes hold a channel's N <= 4 LPC states, a wave 64 / LPC
// neighbouring channels, which share Bm and Cm (they are of one group).  Waves walk over tiles of 16 tokens by themselves: what
// all states of a channel have in common (the step, its activation, the gate) is computed once per channel and token by the
// lane that loads it, and handed to the others through the wave's own part of LDS.  No workgroup barriers.
#pragma once
#include <type_traits>

#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace seq {

constexpr int kTile = 16;      // tokens
constexpr int kKeep = 8;       // tokens between the states that Forward keeps for Backward
constexpr int kWaves = 4;      // of a workgroup, on neighbouring channels

template <int LPC>
struct ScanWave {
    static constexpr int CW = 64 / LPC, NP = 4 * LPC;        // channels, states
    static constexpr int EPL = kTile * CW / 64;              // a tile's elements per lane,
    static constexpr int VE = EPL < 4 ? EPL : 4, P = EPL / VE;   // in P packs of VE neighbours
    static constexpr int LR = CW / VE, TP = 64 / LR;         // lanes to a token, tokens to a pack of all lanes
    static constexpr int BE = 2 * kTile * NP / 64;           // a tile's elements of Bm and Cm per lane
};

struct ScanParams {
    ucd_scan_t d;
    ucd_scan_in_t in;
    int per_group;               // channels of a group,
    unsigned blocks;             // and workgroups for them
    int segs, seg_tiles;         // a sequence's parts that are scanned side by side, and their length
    int tiles;                   // of a whole sequence
    bool wide_states;            // A and all states in packs of 4
    const float *state_in;
    float *state_out;
    void *y;
    float *saved;                // [B][tiles][kTile / kKeep][D][N]: states before each part of a tile
    // Forward: a sequence's first state, then the end states of its segments but the last, each from zero; Backward: the gradients of the
    // states before its segments but the first, each from zero.  And the sums of the segments' steps.
    float *seg_state, *seg_step; // [B][segs][D][N], [B][segs][D]
    // Backward
    const void *dy;
    const float *dstate_out;
    ucd_scan_grad_t g;
    float *part_bc;              // [B][tiles][G][blocks][16 tokens][2][NP]: a workgroup's sums of dBm and dCm over its channels
    float *part_w;               // [B][segs][D][N + 2]: a segment's sums of dA, dskip, ddt_bias
    bool add;
};

// The unit of a workgroup, its waves' channels and its lanes' states.
template <int LPC>
struct ScanPlace {
    int b, seg, g, c0, c, q, n0;
    int have, haven;      // channels of the wave, states of the lane
    __device__ __forceinline__ ScanPlace(const ScanParams &p, unsigned unit)
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        const int block = unit % p.blocks;
        unit /= p.blocks;
        g = unit % p.d.G;
        unit /= p.d.G;
        seg = unit % p.segs;
        b = unit / p.segs;
        const int at = (block * kWaves + wave) * ScanWave<LPC>::CW;
        have = p.per_group - at;
        have = have < 0 ? 0 : have < ScanWave<LPC>::CW ? have : ScanWave<LPC>::CW;
        c0 = g * p.per_group + at;
        q = lane % LPC;
        c = lane / LPC;
        n0 = 4 * q;
        haven = c < have ? p.d.N - n0 : 0;
        haven = haven < 0 ? 0 : haven < 4 ? haven : 4;
    }
};

__device__ __forceinline__ int scan_length(const ScanParams &p, int b)
{
    if (!p.in.lengths) return p.d.L;
    const int n = p.in.lengths[b];
    return n < 0 ? 0 : n < p.d.L ? n : p.d.L;
}

// 4 states (or a channel's 4 coefficients) of the lane
__device__ __forceinline__ void load_states(float (&h)[4], const float *at, int haven, bool wide)
{
    const Pack<float, 4> r = wide ? load_pack<true, float, 4>(at, haven) : load_pack<false, float, 4>(at, haven);
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = r.v[j];
}

__device__ __forceinline__ void store_states(float *at, const float (&h)[4], int haven, bool wide)
{
    Pack<float, 4> r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r.v[j] = h[j];
    if (wide) store_pack<true, float, 4>(at, r, haven);
    else store_pack<false, float, 4>(at, r, haven);
}

// A tile's values of a (B, L, D) tensor as they come from memory: pack i of a lane is token i * TP + lane / LR, channels (lane % LR) * VE on.
template <class T, int LPC>
struct TileRows {
    typedef ScanWave<LPC> W;
    Pack<T, W::VE> r[W::P];

    template <bool WIDE>
    __device__ __forceinline__ void load(const void *base, long sb, long sl, const ScanPlace<LPC> &at, int t0, int n)
    {
        const int lane = threadIdx.x % 64, ch = lane % W::LR * W::VE;
#pragma unroll
        for (int i = 0; i < W::P; ++i) {
            const int t = t0 + i * W::TP + lane / W::LR;
            const T *p = (const T *)base + at.b * sb + (long)t * sl + at.c0 + ch;
            r[i] = load_pack<WIDE, T, W::VE>(p, t < n ? at.have - ch : 0);
        }
    }
};

// The same of Bm and Cm: the tile's 16 rows of NP states of one, then of the other; in packs of 4 or one by one.
template <class T, int LPC, bool WIDE>
struct TileStates {
    typedef ScanWave<LPC> W;
    static constexpr int V = WIDE ? 4 : 1, P = (W::BE + V - 1) / V;
    Pack<T, V> r[P];

    static __device__ __forceinline__ int index(int i) { return (i * 64 + (int)threadIdx.x % 64) * V; }

    __device__ __forceinline__ void load(const ScanParams &p, const ScanPlace<LPC> &at, int t0, int n)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = index(i), k = e % W::NP, t = t0 + e / W::NP % kTile;
            const bool second = e >= kTile * W::NP;
            const int have = t < n && k < p.d.N && e < 2 * kTile * W::NP ? V : 0;
            const T *base = second ? (const T *)p.in.Cm + at.b * p.d.Cm_b + (long)t * p.d.Cm_l : (const T *)p.in.Bm + at.b * p.d.Bm_b + (long)t * p.d.Bm_l;
            r[i] = load_pack<WIDE, T, V>(base + (long)at.g * p.d.N + k, have);
        }
    }

    // into LDS: Bm's rows, then Cm's
    __device__ __forceinline__ void stage(float *lds)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = index(i);
            Pack<float, V> f;
#pragma unroll
            for (int j = 0; j < V; ++j) f.v[j] = to_f(r[i].v[j]);
            if (2 * kTile * W::NP % (64 * V) == 0 || e < 2 * kTile * W::NP) *reinterpret_cast<Pack<float, V> *>(lds + e) = f;
        }
    }
};

// The decay of a lane's states over a whole segment, whose steps add up to `step`, and its own end state on top.
__device__ __forceinline__ void join_segment(float (&h)[4], const float (&A2)[4], float step, const float (&end)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = fmaf(exp2_fast(step * A2[j]), h[j], end[j]);
}

}  // namespace seq

// Whether rows can be read in packs of 4 (a pack of one row is inside a group, and so of Bm and Cm).
bool scan_wide(const ucd_scan_t &d, const ucd_scan_in_t &in, const void *y, const ucd_scan_grad_t *g);
void scan_params(const ucd_scan_t &d, const ucd_scan_in_t &in, int dir, void *ws, seq::ScanParams &p);
int scan_lanes(const ucd_scan_t &d);   // LPC
// workgroups of a launch, below 2^31 (seq_api.cpp)
inline unsigned scan_units(const seq::ScanParams &p) { return (unsigned)p.d.B * p.segs * p.d.G * p.blocks; }

// f(std::integral_constant<int, LPC>) for the descriptor's number of states
template <class F>
hipError_t scan_by_lanes(const ucd_scan_t &d, F f)
{
    switch (scan_lanes(d)) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return f(std::integral_constant<int, 16>());
    }
}

}  // namespace ucd
