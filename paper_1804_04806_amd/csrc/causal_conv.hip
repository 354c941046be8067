// Short causal convolution: Forward, Backward and the single-token step.
//
// Every token is read once (K - 1 of them once more per run) and every result written once: memory bounds it.  A thread owns VE neighbouring channels
// and a run of tokens; the last K - 1 tokens of its channels, and in Backward the last K - 1 gradients of u, stay in registers while it walks.
// Workgroups are 32 packs of 16 bytes (64 of two channels) by 8 (4) runs: whole lines of a row, and neighbouring runs meet their common tokens in the
// same L1.  8 x 2048 tokens, 2048 channels, 4 taps, bf16, on inputs that change from call to call: Forward 32 us (4.2 TB/s; a copy of as many bytes takes
// 28), Backward 54 (3.7, its join included); fp32, 1024 channels: 30 (4.5) and 45 (4.5).  (Figures at the constants below compare two choices on one set
// of inputs, part of which stays in the card's cache: 27 and 48 us.)  Rows of few channels leave lanes idle: 16 x 8192 x 64 24 us in Forward, 1.4 TB/s.
#include <algorithm>
#include <type_traits>

#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace {
using namespace seq;

constexpr int kMaxK = 8;
constexpr int kAhead = 4;          // tokens that are loaded at once

struct ConvParams {
    ucd_causal_conv_t d;
    CausalConvArgs a;
    int run, runs;                 // tokens of a run, runs of a sequence (one at least)
    unsigned packs, blocks_x;      // packs of channels, and workgroups for them
    unsigned rows;                 // runs of all sequences
    float *part;                   // Backward: [workgroups for the runs][K + 1][D]
    unsigned part_rows;
    bool add;
};

template <int VE>
struct ConvBlock {
    static constexpr int PX = VE <= 2 ? 64 : 32, CY = 256 / PX;
};

// A row's last pack is moved back to the row's end: its first channels are another thread's.  That one alone stores them, as it may have replaced their
// state before this one read it, but for Backward, where nothing is replaced and both store the same.
template <int VE>
__device__ __forceinline__ int pack_channel(const ConvParams &p, unsigned pack)
{
    return min((int)pack * VE, p.d.D - VE);
}
template <int VE>
__device__ __forceinline__ int pack_own(const ConvParams &p, unsigned pack)     // its first channel that is its own
{
    return max(0, ((int)pack + 1) * VE - p.d.D);
}

// f(whether a lane of the wave has a pack that was moved back): the other waves, nearly all of them, store without a branch.
template <int VE, class F>
__device__ __forceinline__ void by_tail(int own, F f)
{
    if (VE > 1 && __any(own > 0)) f(std::integral_constant<bool, (VE > 1)>());
    else f(std::false_type());
}

// What a thread works on.
template <class T, int VE>
struct ConvPlace {
    int c0, own, b, t0, n, slot;
    bool active;
    __device__ __forceinline__ ConvPlace(const ConvParams &p, unsigned unit)
    {
        typedef ConvBlock<VE> B;
        const unsigned pack = unit % p.blocks_x * B::PX + threadIdx.x % B::PX, row = unit / p.blocks_x * B::CY + threadIdx.x / B::PX;
        active = pack < p.packs && row < p.rows;
        c0 = pack_channel<VE>(p, pack);
        own = pack_own<VE>(p, pack);
        b = active ? (int)(row / (unsigned)p.runs) : 0;
        t0 = (int)(row % (unsigned)p.runs) * p.run;
        slot = b;
        n = p.d.L;
        if (!active) return;
        if (p.a.slots) {
            slot = p.a.slots[b];
            if (slot < 0 || slot >= p.d.n_slots) slot = -1;
        }
        if (p.a.lengths) n = max(0, min(p.d.L, p.a.lengths[b]));
        if (slot < 0) n = 0;
    }
};

template <class T, int VE>
__device__ __forceinline__ void load_channels(float (&v)[VE], const T *at)
{
    const Pack<T, VE> r = loose_load<T, VE>(at);
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = to_f(r.v[i]);
}

// TAIL: a lane of the wave may have such a pack
template <class T, int VE, bool TAIL>
__device__ __forceinline__ void store_channels(T *at, const float (&v)[VE], int own = 0)
{
    Pack<T, VE> r;
#pragma unroll
    for (int i = 0; i < VE; ++i) r.v[i] = from_f<T>(v[i]);
    if (!TAIL || own == 0) {
        loose_store<T, VE>(at, r);
    } else {
#pragma unroll
        for (int i = 1; i < VE; ++i)
            if (i >= own) at[i] = r.v[i];
    }
}

// the K - 1 tokens before t0: of the sequence, of the state, or 0
template <class T, int VE, int K>
__device__ __forceinline__ void load_window(float (&win)[K][VE], const ConvParams &p, const ConvPlace<T, VE> &at, const T *x)
{
    const T *state = p.a.state_in && at.slot >= 0 ? (const T *)p.a.state_in + (long)at.slot * (K - 1) * p.d.D + at.c0 : nullptr;
#pragma unroll
    for (int k = 0; k < K - 1; ++k) {
        const int t = at.t0 - (K - 1) + k;
#pragma unroll
        for (int i = 0; i < VE; ++i) win[k][i] = 0.f;
        if (t >= 0) {
            if (t < at.n) load_channels<T, VE>(win[k], x + (long)t * p.d.x_l);
        } else if (state) {
            load_channels<T, VE>(win[k], state + (long)(K - 1 + t) * p.d.D);
        }
    }
}

template <class T, int VE, int K>
__device__ __forceinline__ void load_weights(float (&w)[K][VE], float (&bias)[VE], const ConvParams &p, int c0)
{
    const T *at = (const T *)p.a.w + (long)c0 * K;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
#pragma unroll
        for (int k = 0; k < K; ++k) w[k][i] = to_f(at[i * K + k]);
        bias[i] = p.a.bias ? p.a.bias[c0 + i] : 0.f;
    }
}

template <class T, int VE, int K, bool SILU, bool TAIL>
__device__ __forceinline__ void conv_fwd_run(const ConvParams &p, const ConvPlace<T, VE> &at)
{
    const T *x = (const T *)p.a.x + at.b * p.d.x_b + at.c0;
    T *y = (T *)p.a.y + at.b * p.d.y_b + at.c0;
    float win[K][VE], w[K][VE], bias[VE];      // win[K - 1] is the current token
    load_window<T, VE, K>(win, p, at, x);
    load_weights<T, VE, K>(w, bias, p, at.c0);
    // the new state is the first run's to write: it has read the old one, which may be in the same place
    float first[K][VE];
#pragma unroll
    for (int k = 0; k < K - 1; ++k)
#pragma unroll
        for (int i = 0; i < VE; ++i) first[k][i] = win[k][i];
    const int end = min(p.d.L, at.t0 + p.run), stop = min(end, at.n);
    int t = at.t0;
    Raw<T, VE, true> in[kAhead], next[kAhead];
    auto load = [&](int t) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) next[j].load((const char *)(x + (long)min(t + j, stop - 1) * p.d.x_l), 0, VE);
    };
    if (t < stop) load(t);
    for (; t < stop; t += kAhead) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) in[j] = next[j];
        if (t + kAhead < stop) load(t + kAhead);      // under way while these tokens are computed
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (t + j >= stop) break;
            float out[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                win[K - 1][i] = in[j].get(i);
                float u = bias[i];
#pragma unroll
                for (int k = 0; k < K; ++k) u = fmaf(w[k][i], win[k][i], u);
                out[i] = SILU ? u * sigmoid(u) : u;
#pragma unroll
                for (int k = 0; k < K - 1; ++k) win[k][i] = win[k + 1][i];
            }
            store_channels<T, VE, TAIL>(y + (long)(t + j) * p.d.y_l, out, at.own);
        }
    }
    const float zero[VE] = {};
    for (t = max(at.t0, stop); t < end; ++t) store_channels<T, VE, TAIL>(y + (long)t * p.d.y_l, zero, at.own);
    if (K > 1 && p.a.state_out && at.t0 == 0 && at.slot >= 0) {
        T *state = (T *)p.a.state_out + (long)at.slot * (K - 1) * p.d.D + at.c0;
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            const int s = at.n - (K - 1) + k;
            float v[VE];
            if (s >= 0) {
                load_channels<T, VE>(v, x + (long)s * p.d.x_l);
            } else {
                // token s of the old state: its place is K - 1 + s
#pragma unroll
                for (int i = 0; i < VE; ++i) v[i] = 0.f;
#pragma unroll
                for (int m = 0; m < K - 1; ++m)
                    if (m == K - 1 + s)
#pragma unroll
                        for (int i = 0; i < VE; ++i) v[i] = first[m][i];
            }
            store_channels<T, VE, TAIL>(state + (long)k * p.d.D, v, at.own);
        }
    }
}

template <class T, int VE, int K, bool SILU>
__global__ __launch_bounds__(256) void conv_fwd_kernel(ConvParams p, unsigned units)
{
    for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const ConvPlace<T, VE> at(p, unit);
        if (!at.active) continue;
        by_tail<VE>(at.own, [&](auto tail) { conv_fwd_run<T, VE, K, SILU, decltype(tail)::value>(p, at); });
    }
}

// One token: a thread to VE channels of a sequence, few of them, so that single sequences fill some hundred workgroups too; all loads but the state's
// place are under way at once.  64 sequences, 2048 channels, 4 taps, bf16: 3.0 us, which is a launch's own time.
template <class T, int VE, int K, bool SILU>
__global__ __launch_bounds__(256) void conv_step_kernel(ConvParams p)
{
    const unsigned pack = blockIdx.x * 256u + threadIdx.x;
    if (pack >= p.packs) return;
    const int c0 = pack_channel<VE>(p, pack), own = pack_own<VE>(p, pack);
    float w[K][VE], bias[VE];
    load_weights<T, VE, K>(w, bias, p, c0);
    by_tail<VE>(own, [&](auto tail) {
        constexpr bool TAIL = decltype(tail)::value;
        for (int b = blockIdx.y; b < p.d.B; b += gridDim.y) {
            float x[VE], out[VE] = {};
            load_channels<T, VE>(x, (const T *)p.a.x + b * p.d.x_b + c0);
            const int slot = p.a.slots ? p.a.slots[b] : b;
            if (!p.a.slots || (slot >= 0 && slot < p.d.n_slots)) {
                T *state = (T *)p.a.state_out + (long)slot * (K - 1) * p.d.D + c0;
                float before[K][VE];
    #pragma unroll
                for (int k = 0; k < K - 1; ++k) load_channels<T, VE>(before[k], state + (long)k * p.d.D);
    #pragma unroll
                for (int i = 0; i < VE; ++i) {
                    before[K - 1][i] = x[i];
                    float u = bias[i];
    #pragma unroll
                    for (int k = 0; k < K; ++k) u = fmaf(w[k][i], before[k][i], u);
                    out[i] = SILU ? u * sigmoid(u) : u;
                }
    #pragma unroll
                for (int k = 0; k < K - 1; ++k) store_channels<T, VE, TAIL>(state + (long)k * p.d.D, before[k + 1], own);
            }
            store_channels<T, VE, TAIL>((T *)p.a.y + b * p.d.y_b + c0, out, own);
        }
    });
}

// dx, the gradient of the state before the first token, and sums of dw and dbias over the workgroup's runs.
// At token t: du_t = dy_t act'(u_t), and dx of token t - K + 1, the last that du_t reaches, is complete.
template <class T, int VE, int K, bool SILU>
__global__ __launch_bounds__(256) void conv_bwd_kernel(ConvParams p)
{
    typedef ConvBlock<VE> B;
    __shared__ float lds[B::CY][B::PX * VE];
    float w[K][VE], bias[VE], dw[K][VE] = {}, db[VE] = {};
    bool have_w = false;
    const unsigned column = blockIdx.x % p.blocks_x, part_row = blockIdx.x / p.blocks_x, rows_y = (p.rows + B::CY - 1) / B::CY;
    const unsigned pack = column * B::PX + threadIdx.x % B::PX;
    const int own = pack < p.packs ? pack_own<VE>(p, pack) : 0;
    for (unsigned block = part_row; block < rows_y; block += p.part_rows) {
        const ConvPlace<T, VE> at(p, block * p.blocks_x + column);
        if (!at.active) continue;
        if (!have_w) load_weights<T, VE, K>(w, bias, p, at.c0);
        have_w = true;
        const T *x = (const T *)p.a.x + at.b * p.d.x_b + at.c0, *dy = (const T *)p.a.dy + at.b * p.d.y_b + at.c0;
        T *dx = (T *)p.a.dx + at.b * p.d.x_b + at.c0;
        const long state_at = (long)at.b * (K - 1) * p.d.D + at.c0;
        float win[K][VE], g[K][VE] = {};       // tokens t - K + 1 to t, and their du
        load_window<T, VE, K>(win, p, at, x);
        const int end = min(p.d.L, at.t0 + p.run), stop = min(end, at.n);      // the run's own tokens
        // and those that its last tokens reach; a first run emits the state's gradients too, whatever its length
        const int until = stop > at.t0 || at.t0 == 0 ? stop + K - 1 : at.t0;
        Raw<T, VE, true> xin[kAhead], gin[kAhead], xnext[kAhead], gnext[kAhead];
        const int seen = min(until, at.n);           // tokens that are read
        const T *x_at = x + (long)at.t0 * p.d.x_l, *dy_at = dy + (long)at.t0 * p.d.y_l;
        T *dx_at = dx + (long)(at.t0 - (K - 1)) * p.d.x_l;
        auto load = [&](int t) {                     // tokens t to t + 3, the last of them again behind it
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int k = min(j, seen - 1 - t);
                xnext[j].load((const char *)(x_at + k * p.d.x_l), 0, VE);
                gnext[j].load((const char *)(dy_at + k * p.d.y_l), 0, VE);
            }
            x_at += kAhead * p.d.x_l;
            dy_at += kAhead * p.d.y_l;
        };
        // one token: INSIDE, it is one of the run's own
        auto token = [&](int j, int t, auto inside) {
            constexpr bool INSIDE = decltype(inside)::value;
            const int s = t - (K - 1);
            const bool there = INSIDE || t < at.n, own = INSIDE || t < stop;
            float out[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                win[K - 1][i] = there ? xin[j].get(i) : 0.f;
                float du = there ? gin[j].get(i) : 0.f;
                if (SILU) {
                    float u = bias[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) u = fmaf(w[k][i], win[k][i], u);
                    const float sg = sigmoid(u);
                    du *= sg * fmaf(u, 1.f - sg, 1.f);
                    if (!INSIDE) du = there ? du : 0.f;
                }
                const float part = own ? du : 0.f;
                db[i] += part;
#pragma unroll
                for (int k = 0; k < K; ++k) dw[k][i] = INSIDE || own ? fmaf(part, win[k][i], dw[k][i]) : dw[k][i];
                g[K - 1][i] = du;
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < K; ++k) v = fmaf(w[K - 1 - k][i], g[k][i], v);
                out[i] = v;
#pragma unroll
                for (int k = 0; k < K - 1; ++k) {
                    g[k][i] = g[k + 1][i];
                    win[k][i] = win[k + 1][i];
                }
            }
            // a token that is part of the new state
            if (!INSIDE && p.a.dstate_out && s >= at.n - (K - 1)) {
                float more[VE];
                load_channels<T, VE>(more, (const T *)p.a.dstate_out + state_at + (long)(s - (at.n - (K - 1))) * p.d.D);
#pragma unroll
                for (int i = 0; i < VE; ++i) out[i] += more[i];
            }
            if (s >= at.t0) store_channels<T, VE, false>(dx_at, out);
            else if (at.t0 == 0 && p.a.dstate_in) store_channels<T, VE, false>((T *)p.a.dstate_in + state_at + (long)(K - 1 + s) * p.d.D, out);
            dx_at += p.d.x_l;
        };
        if (at.t0 < seen) load(at.t0);
        for (int t = at.t0; t < until; t += kAhead) {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                xin[j] = xnext[j];
                gin[j] = gnext[j];
            }
            if (t + kAhead < seen) load(t + kAhead);
            if (t + kAhead <= stop) {
#pragma unroll
                for (int j = 0; j < kAhead; ++j) token(j, t + j, std::true_type());
            } else {
#pragma unroll
                for (int j = 0; j < kAhead; ++j)
                    if (t + j < until) token(j, t + j, std::false_type());
            }
        }
        const float zero[VE] = {};
        for (int t = max(at.t0, stop); t < end; ++t) store_channels<T, VE, false>(dx + (long)t * p.d.x_l, zero);
    }
    // over the workgroup's runs, in their order
    const int x_lane = threadIdx.x % B::PX, y_lane = threadIdx.x / B::PX;
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VE; ++i)
            if (i >= own) lds[y_lane][x_lane * VE + i - own] = k < K ? dw[k % K][i] : db[i];
        __syncthreads();
        for (int i = threadIdx.x; i < B::PX * VE; i += 256) {
            float v = lds[0][i];
#pragma unroll
            for (int r = 1; r < B::CY; ++r) v += lds[r][i];
            const int c = (int)column * B::PX * VE + i;
            if (c < p.d.D) p.part[((long)part_row * (K + 1) + k) * p.d.D + c] = v;
        }
    }
}

// A channel's K + 1 sums over the workgroups.
__global__ __launch_bounds__(kJoinThreads) void conv_join_kernel(ConvParams p)
{
    const int K = p.d.K;
    join_columns(p.part, p.part_rows, (long)(K + 1) * p.d.D, [&](long i, float v) {
        const int c = (int)(i % p.d.D), k = (int)(i / p.d.D);
        float *out = k < K ? p.a.dw + (long)c * K + k : p.a.dbias ? p.a.dbias + c : nullptr;
        if (out) *out = v + (p.add ? *out : 0.f);
    });
}

// Packs: Forward 16 bytes.  Backward keeps four times as much of a channel in registers (its window of tokens and gradients, filter and their sums):
// two channels to a thread leave four waves to a SIMD.  bf16: 47.7 us where four take 48.5 and eight, two waves to a SIMD, 69 (8 x 2048 x 2048), of
// single sequences of 512 tokens, 4096 channels 11.8, 13.0 and 15.8; fp32: 38.5 where four take 40.3 (8 x 2048 x 1024), 26.1 and 28.1 (13 x 1021 x 509).
// Rows need not be whole packs nor begin at their multiples: 2047 channels instead of 2048 take 38 us instead of 26 in Forward, 58 instead of 48 in
// Backward, and took 42 and 76 channel by channel.
constexpr int kFwdPack[2] = {4, 8}, kBwdPack[2] = {2, 2}, kStepPack[2] = {2, 2};
static_assert(kBwdPack[0] == kBwdPack[1], "one division of Backward's workspace");
enum Form { FORWARD, BACKWARD, STEP };

// Runs are as long as leaves two waves to a SIMD, 8 to 32 tokens.
template <int VE>
void divide(const ucd_causal_conv_t &d, ConvParams &p)
{
    typedef ConvBlock<VE> B;
    p.d = d;
    p.packs = (unsigned)((d.D + VE - 1) / VE);
    p.blocks_x = (p.packs + B::PX - 1) / B::PX;
    p.run = 32;
    while (p.run > 8 && (double)d.B * ((d.L + p.run - 1) / p.run) * p.packs < 131072.) p.run /= 2;
    p.runs = std::max(1, (d.L + p.run - 1) / p.run);
    p.rows = (unsigned)d.B * (unsigned)p.runs;
    // Backward: a workgroup takes every part_rows-th row of runs, and adds one row of partial sums; about as many workgroups as run at once
    const unsigned rows_y = (p.rows + B::CY - 1) / B::CY;
    p.part_rows = std::max(1u, std::min(rows_y, 2048 / p.blocks_x));
}

template <class T, int VE, int K, bool SILU>
hipError_t run_fwd(const ConvParams &p, hipStream_t s)
{
    const unsigned units = p.blocks_x * ((p.rows + ConvBlock<VE>::CY - 1) / ConvBlock<VE>::CY);
    conv_fwd_kernel<T, VE, K, SILU><<<std::min(units, 1u << 22), 256, 0, s>>>(p, units);
    return hipGetLastError();
}

template <class T, int VE, int K, bool SILU>
hipError_t run_step(const ConvParams &p, hipStream_t s)
{
    conv_step_kernel<T, VE, K, SILU><<<dim3((p.packs + 255) / 256, (unsigned)std::min(p.d.B, 65535)), 256, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, int VE, int K, bool SILU>
hipError_t run_bwd(const ConvParams &p, hipStream_t s)
{
    conv_bwd_kernel<T, VE, K, SILU><<<p.blocks_x * p.part_rows, 256, 0, s>>>(p);
    conv_join_kernel<<<join_grid((long)(K + 1) * p.d.D), kJoinThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, int VE, int K, Form FORM>
hipError_t by_act(const ConvParams &p, hipStream_t s)
{
    const bool silu = p.d.act == UCD_ACT_SILU;
    if constexpr (FORM == BACKWARD) return silu ? run_bwd<T, VE, K, true>(p, s) : run_bwd<T, VE, K, false>(p, s);
    else if constexpr (FORM == STEP) return silu ? run_step<T, VE, K, true>(p, s) : run_step<T, VE, K, false>(p, s);
    else return silu ? run_fwd<T, VE, K, true>(p, s) : run_fwd<T, VE, K, false>(p, s);
}

template <class T, int VE, Form FORM>
hipError_t by_taps(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, void *ws, hipStream_t s)
{
    ConvParams p{};
    divide<VE>(d, p);
    p.a = a;
    p.part = (float *)ws;
    p.add = add;
    switch (d.K) {
    case 1: return by_act<T, VE, 1, FORM>(p, s);
    case 2: return by_act<T, VE, 2, FORM>(p, s);
    case 3: return by_act<T, VE, 3, FORM>(p, s);
    case 4: return by_act<T, VE, 4, FORM>(p, s);
    case 5: return by_act<T, VE, 5, FORM>(p, s);
    case 6: return by_act<T, VE, 6, FORM>(p, s);
    case 7: return by_act<T, VE, 7, FORM>(p, s);
    default: return by_act<T, VE, 8, FORM>(p, s);
    }
}

template <Form FORM>
hipError_t dispatch(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, void *ws, hipStream_t s)
{
    constexpr const int *packs = FORM == BACKWARD ? kBwdPack : FORM == STEP ? kStepPack : kFwdPack;
    // rows of fewer channels have none
    const bool whole = d.D >= packs[d.dtype];
    if (d.dtype == 1) return whole ? by_taps<bf16_t, packs[1], FORM>(d, a, add, ws, s) : by_taps<bf16_t, 1, FORM>(d, a, add, ws, s);
    return whole ? by_taps<float, packs[0], FORM>(d, a, add, ws, s) : by_taps<float, 1, FORM>(d, a, add, ws, s);
}

}  // namespace

size_t causal_conv_ws_bytes(const ucd_causal_conv_t &d)
{
    ConvParams p{};
    if (d.D < kBwdPack[d.dtype]) divide<1>(d, p);
    else divide<kBwdPack[0]>(d, p);
    return (size_t)4 * p.part_rows * (d.K + 1) * d.D;
}

hipError_t causal_conv_fwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s) { return dispatch<FORWARD>(d, a, false, nullptr, s); }

hipError_t causal_conv_bwd(const ucd_causal_conv_t &d, const CausalConvArgs &a, bool add, void *ws, hipStream_t s)
{
    return dispatch<BACKWARD>(d, a, add, ws, s);
}

hipError_t causal_conv_step(const ucd_causal_conv_t &d, const CausalConvArgs &a, hipStream_t s) { return dispatch<STEP>(d, a, false, nullptr, s); }

}  // namespace ucd
