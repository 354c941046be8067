// What the scan's kernels share: how a wave is laid out over channels and states, and how it stages a tile of tokens.
//
// A lane holds NPL neighbouring states of one channel; LPC neighbouring lanes hold a channel's N <= LPC NPL states, a wave 64 / LPC
// neighbouring channels, which share Bm and Cm (they are of one group).  Waves walk over tiles of 16 tokens by themselves: what
// all states of a channel have in common (the step, its activation, the gate) is computed once per channel and token by the
// lane that loads it, and handed to the others through the wave's own part of LDS.  Workgroups meet in Backward only, once a tile, to add up
// their waves' sums over channels.
#pragma once
#include <type_traits>

#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace seq {

constexpr int kTile = 16;      // tokens
constexpr int kKeep = 8;       // tokens between the states that Forward keeps for Backward
constexpr int kWaves = 4;      // of a workgroup, on neighbouring channels

template <int LPC_, int NPL_>
struct ScanWave {
    static constexpr int LPC = LPC_, NPL = NPL_, CW = 64 / LPC, NP = NPL * LPC;        // channels, states
    static constexpr int VE = kTile * CW / 64;               // a tile's elements per lane, neighbours of one token
    static constexpr int LR = CW / VE;                       // lanes to a token
    static constexpr int BE = 2 * kTile * NP / 64;           // a tile's elements of Bm and Cm per lane
};

struct ScanParams {
    ucd_scan_t d;
    ucd_scan_in_t in;
    int per_group;               // channels of a group,
    unsigned blocks;             // and workgroups for them
    int segs, seg_tiles;         // a sequence's parts that are scanned side by side, and their length
    int tiles;                   // of a whole sequence
    const float *state_in;
    float *state_out;
    void *y;
    float *saved;                // [B][tiles][kTile / kKeep][D][NP]: states before each part of a tile
    // Forward: a sequence's first state, then the end states of its segments but the last, each from zero; Backward: the gradients of the
    // states before its segments but the first, each from zero.  And the sums of the segments' steps.
    float *seg_state, *seg_step; // [B][segs][D][NP], [B][segs][D]
    // Backward
    const void *dy;
    const float *dstate_out;
    ucd_scan_grad_t g;
    float *part_bc;              // [B][tiles][G][blocks][16 tokens][2][NP]: a workgroup's sums of dBm and dCm over its channels
    float *part_w;               // [B][segs][D][N + 2]: a segment's sums of dA, dskip, ddt_bias
    bool add;
};

// The unit of a workgroup, its waves' channels and its lanes' states.
template <class W>
struct ScanPlace {
    int b, seg, g, block;        // of the workgroup,
    int first, c0, have;         // its first channel, the wave's and how many of them there are
    int base;                    // no pack of a row begins before this channel
    int c, q, n0, haven;         // the lane's channel within the wave, states from n0 on and how many of them there are
    // What the lane loads: token (of a pack of all lanes) and first channel within the wave.  The last packs of a group are moved back to its end: they
    // may begin in another lane's channels, and then do the same as that lane, or in another wave's, which are left alone.
    int tok, ch0;
    __device__ __forceinline__ bool channel(int i) const { return ch0 + i >= 0 && ch0 + i < have; }     // is the wave's
    __device__ __forceinline__ ScanPlace(const ScanParams &p, unsigned unit, bool wide)
    {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        block = unit % p.blocks;
        unit /= p.blocks;
        g = unit % p.d.G;
        unit /= p.d.G;
        seg = unit % p.segs;
        b = unit / p.segs;
        first = g * p.per_group + block * kWaves * W::CW;
        const int at = (block * kWaves + wave) * W::CW;
        have = p.per_group - at;
        have = have < 0 ? 0 : have < W::CW ? have : W::CW;
        c0 = first + wave * W::CW;
        q = lane % W::LPC;
        c = lane / W::LPC;
        n0 = W::NPL * q;
        haven = c < have ? p.d.N - n0 : 0;
        haven = haven < 0 ? 0 : haven < W::NPL ? haven : W::NPL;
        tok = lane / W::LR;
        ch0 = lane % W::LR * W::VE;
        base = first;
        if (wide) {
            const int end = p.per_group - at;
            ch0 = end - W::VE < ch0 ? end - W::VE : ch0;
            base = first < W::VE ? 0 : first - W::VE;
        }
    }
};

__device__ __forceinline__ int scan_length(const ScanParams &p, int b)
{
    if (!p.in.lengths) return p.d.L;
    const int n = p.in.lengths[b];
    return n < 0 ? 0 : n < p.d.L ? n : p.d.L;
}

// The lane's states, or coefficients of a channel's states.
template <int N>
__device__ __forceinline__ void load_states(float (&h)[N], const float *at, int haven)
{
    const Pack<float, N> r = haven == N ? loose_load<float, N>(at) : load_pack<false, float, N>(at, haven);
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = r.v[j];
}

template <int N>
__device__ __forceinline__ void store_states(float *at, const float (&h)[N], int haven)
{
    Pack<float, N> r;
#pragma unroll
    for (int j = 0; j < N; ++j) r.v[j] = h[j];
    if (haven == N) loose_store<float, N>(at, r);
    else store_pack<false, float, N>(at, r, haven);
}

// The same in the library's own buffers, whose channels have NP states: always a whole pack.
template <int N>
__device__ __forceinline__ void load_own(float (&h)[N], const float *at, bool there)
{
    const Pack<float, N> r = load_pack<true, float, N>(at, there);
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = r.v[j];
}
template <int N>
__device__ __forceinline__ void store_own(float *at, const float (&h)[N], bool there)
{
    Pack<float, N> r;
#pragma unroll
    for (int j = 0; j < N; ++j) r.v[j] = h[j];
    store_pack<true, float, N>(at, r, there);
}

// Tokens behind the sequence's last repeat it and (one by one) channels that are not there repeat the workgroup's first: what is loaded of them is
// masked where it is used.  Offsets of a tile's elements from its first token and `base` are below 2^32 bytes (seq_api.cpp bounds the strides).
template <class T, class W>
__device__ __forceinline__ uint32_t row_offset(const ScanPlace<W> &at, long sl, int last)
{
    const int c = at.ch0 < at.have ? at.c0 - at.base + at.ch0 : at.first - at.base;
    return ((uint32_t)min(at.tok, last) * (uint32_t)sl + (uint32_t)c) * (uint32_t)sizeof(T);
}

// The tile's first element for a workgroup: of u, dt, z, y and of Bm, Cm.  Uniform: an address is this pointer, which a tile moves on by scalar
// arithmetic, and a lane's offset, which stays.
template <class T, class W>
__device__ __forceinline__ const char *row_base(const void *base, long sb, long sl, const ScanPlace<W> &at, long t0)
{
    return (const char *)base + (at.b * sb + t0 * sl + at.base) * (long)sizeof(T);
}
template <class T, class W>
__device__ __forceinline__ const char *bc_base(const void *base, long sb, long sl, const ScanPlace<W> &at, long t0, int N)
{
    return (const char *)base + (at.b * sb + t0 * sl + (long)at.g * N) * (long)sizeof(T);
}

// WIDE: rows have a pack's elements before their end (see ScanPlace); FULL: they are the wave's, as is the token.
template <class T, class W, bool WIDE, bool FULL>
__device__ __forceinline__ void store_row(char *base, uint32_t offset, const Pack<T, W::VE> &v, const ScanPlace<W> &at, bool token)
{
    T *to = reinterpret_cast<T *>(base + offset);
    if (FULL || (WIDE && token && at.ch0 >= 0)) {
        loose_store<T, W::VE>(to, v);
    } else if (token) {
#pragma unroll
        for (int i = 0; i < W::VE; ++i)
            if (at.channel(i)) to[i] = v.v[i];
    }
}

// A tile's Bm and Cm, 16 rows of NP states of one, then of the other, in packs of 4; a row's last pack is moved back to its end.  Up to 4 states: one by
// one.  In LDS a row's states behind the N-th stay 0.
template <class T, class W>
struct TileStates {
    static constexpr int V = W::NP > 4 ? 4 : 1, P = W::BE / V, ROWS = kTile * W::NP;
    static_assert(2 * ROWS == 64 * V * P, "all lanes have a pack");
    static constexpr bool WHOLE = ROWS % (64 * V) == 0;      // a pack of all lanes is of one tensor
    Raw<T, V, true> r[P];
    uint32_t offset[P];

    static __device__ __forceinline__ int index(int i) { return (i * 64 + (int)threadIdx.x % 64) * V; }
    static __device__ __forceinline__ bool second(int i) { return WHOLE ? i * 64 * V >= ROWS : index(i) >= ROWS; }
    static __device__ __forceinline__ int state(int e, int states) { return min(e % W::NP, states - V); }

    __device__ __forceinline__ void place(const ScanParams &p, int last)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = index(i), t = min(e / W::NP % kTile, last);
            offset[i] = ((uint32_t)t * (uint32_t)(second(i) ? p.d.Cm_l : p.d.Bm_l) + (uint32_t)state(e, p.d.N)) * (uint32_t)sizeof(T);
        }
    }

    __device__ __forceinline__ void load(const char *bm, const char *cm)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            if (WHOLE) r[i].load(second(i) ? cm : bm, offset[i], V);
            else if (second(i)) r[i].load(cm, offset[i], V);
            else r[i].load(bm, offset[i], V);
        }
    }

    // before the first tile
    static __device__ __forceinline__ void clear(float *lds, int states)
    {
        if (states == W::NP) return;
#pragma unroll
        for (int i = 0; i < P * V; ++i) lds[i * 64 + (int)threadIdx.x % 64] = 0.f;
    }
    __device__ __forceinline__ void stage(float *lds, int states)
    {
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const int e = index(i);
            Pack<float, V> f;
#pragma unroll
            for (int j = 0; j < V; ++j) f.v[j] = r[i].get(j);
            loose_store<float, V>(lds + e - e % W::NP + state(e, states), f);
        }
    }
};

// What a lane takes from its token's row in LDS; FULL: all of it is the wave's.
template <class W, bool FULL>
__device__ __forceinline__ void lds_row(float (&v)[W::VE], const float *rows, const ScanPlace<W> &at)
{
    const float *row = rows + at.tok * W::CW;
    if (FULL) {
        const Pack<float, W::VE> r = *reinterpret_cast<const Pack<float, W::VE> *>(row + at.ch0);
#pragma unroll
        for (int i = 0; i < W::VE; ++i) v[i] = r.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < W::VE; ++i) v[i] = row[max(at.ch0 + i, 0)];
    }
}

// The decay of a lane's states over a whole segment, whose steps add up to `step`, and its own end state on top.
template <int N>
__device__ __forceinline__ void join_segment(float (&h)[N], const float (&A2)[N], float step, const float (&end)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) h[j] = fmaf(exp2_fast(step * A2[j]), h[j], end[j]);
}

}  // namespace seq

// Whether rows can be read in packs of 4.
inline bool scan_wide(const ucd_scan_t &d) { return d.D / d.G >= 4; }
void scan_params(const ucd_scan_t &d, const ucd_scan_in_t &in, int dir, void *ws, seq::ScanParams &p);
// workgroups of a launch, below 2^31 (seq_api.cpp)
inline unsigned scan_units(const seq::ScanParams &p) { return (unsigned)p.d.B * p.segs * p.d.G * p.blocks; }

// f(ScanWave<LPC, NPL>()) for the descriptor's number of states
template <class F>
hipError_t scan_by_states(const ucd_scan_t &d, F f)
{
    using seq::ScanWave;
    if (d.N <= 4) return f(ScanWave<4, 1>());
    if (d.N <= 8) return f(ScanWave<4, 2>());
    if (d.N <= 16) return f(ScanWave<4, 4>());
    if (d.N <= 32) return f(ScanWave<8, 4>());
    return f(ScanWave<16, 4>());
}
inline int scan_lanes(const ucd_scan_t &d) { return d.N <= 16 ? 4 : d.N <= 32 ? 8 : 16; }
inline int scan_states(const ucd_scan_t &d) { return d.N <= 4 ? 4 : d.N <= 8 ? 8 : 4 * scan_lanes(d); }   // NP

}  // namespace ucd
