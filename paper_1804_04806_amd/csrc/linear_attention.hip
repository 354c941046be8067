// Linear attention with a decay for each head, over chunks of 64 tokens.
//
//   S_t = e^{l_t} S_{t-1} + k_t^T v_t,  y_t = scale q_t S_t.  Within a chunk, G the sums of l up to a token and D[t, s] = e^{G_t - G_s} (s <= t):
//   y = scale ((q k^T) o D) v + scale e^{G_t} q S_in,   S_out = e^{G_C} S_in + sum_s e^{G_C - G_s} k_s^T v_s.
//
// The gradients are the same mixing of other rows.  With dS_t = scale q_t^T dy_t + e^{l_{t+1}} dS_{t+1}:
//   dq_t = scale sum_{s <= t} D (dy_t . v_s) k_s     mixes (dy, v, k) forward, its state is S^T;
//   dk_s = scale sum_{t >= s} D (v_s . dy_t) q_t     mixes (v, dy, q) backward, its state is dS^T;
//   dv_s = scale sum_{t >= s} D (k_s . q_t) dy_t     mixes (k, q, dy) backward, its state is dS.
// Backward in time a token's decay is its neighbour's, l_{t+1}, and 0 for the last.
//
// A workgroup walks over the chunks of a sequence's head with 64 columns of the state, fp32 in the matrix instructions' registers.  Long sequences with
// few heads are cut into segments: their own states first, then the states at their starts, then all segments at once.
//
// The gradient of a decay is that of all paths that cross it: pairs of tokens within the chunk, tokens with the states before and behind it, and the
// state that passes through:  dl_u = sum_{s < u <= t} W[t, s] + sum_{t >= u} a_t + sum_{s < u} b_s + c,
//   W = scale (q k^T) o (dy v^T) o D,  a_t = q_t . (dq_t's part of S_in),  b_s = k_s . (dk_s's part of dS_out),  c = e^{G_C} <S_in, dS_out>.
// Sums over whole sequences of q_t . dq_t - k_t . dk_t would be the same in exact arithmetic, but lose in their differences what the paths that do not
// cross the token leave of rounding.
#include <algorithm>

#include "linear_attention.hpp"

namespace ucd {
namespace {
using namespace attention;

struct Rows {
    const void *p;
    long b, l;      // strides
    int div;        // heads that share a row of it
    int width;
    template <class T>
    __device__ __forceinline__ const T *at(int seq, int head) const { return (const T *)p + seq * b + (long)(head / div) * width; }
};

struct Mix {
    Rows q, k, v, dot;           // dot: rows like the output's, multiplied with the part of the state at the chunk's start; may be none
    void *out;
    long out_b, out_l;
    bool out_f32;
    float p_scale, first_scale, last_scale;
    Decays decays;
    const int32_t *lengths, *slots;
    int B, L, H, n_slots, segments, per_segment;     // chunks of a segment
    // states: of a slot and head rows (of q's width) and columns (of v's) apart
    const float *state_in;
    float *state_out;
    long s_row, s_col, s_head;
    float *starts;               // (segments, B, H, rows, columns) with the strides of state_in, or null
    float *segment_decay;        // (segments, B, H)
    float *dots;                 // (column tiles, B, H, L), or null
    void *chunk_states;          // states at the chunks' starts, by workgroup, chunk and thread
    float *passes;               // (column tiles, B, H, chunks): c
    int tiles;
};

// Places of a launch: column tile, head, segment, sequence.  Column tiles of a head are neighbours that share q and k.
struct Place {
    int tile, head, seq, segment;
};
__device__ __forceinline__ Place place_of(const Mix &p, int segments)
{
    unsigned i = blockIdx.x;
    Place r;
    r.tile = i % p.tiles;
    i /= p.tiles;
    r.head = i % p.H;
    i /= p.H;
    r.segment = i % segments;
    r.seq = i / segments;
    return r;
}

// What a walk is for: outputs; outputs and what the gradient of the decays takes of them (forward: the states at the chunks' starts are kept, backward
// they are read); a segment's own state alone, from nothing.
enum { OUTPUTS, DECAYS, STATES };

// DK: q's width, 64 or 128.  WHOLE: of rows (Fetch).
template <class T, int DK, bool REV, int FOR, bool WHOLE>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 || DK == 64 ? 2 : 1) void mix_kernel(Mix p)
{
    constexpr bool OUT = FOR != STATES, DG = FOR == DECAYS;
    // what is added to a state that a caller gets, or the next segment, is as exact as the state; states that only go into 16-bit operands need less
    constexpr int PARTS = sizeof(T) == 4 ? 1 : DG ? 2 : 3;
    typedef Mma<T> M;
    typedef TileLds<T, DK> TQ;
    typedef TileLds<T, kCols> TV;
    constexpr int SD = DK / 64;         // a wave's tiles of the state: DK = 128: 32 rows and all 64 columns; 64: 32 rows and 32 columns
    __shared__ __attribute__((aligned(16))) char lds_q[OUT ? TQ::BYTES : 16], lds_k[TQ::BYTES], lds_v[TV::BYTES],
        lds_p[OUT ? TV::BYTES : 16], lds_s[OUT ? TQ::BYTES : 16];      // lds_s: the state's columns as rows of DK
    __shared__ ChunkDecays decays[2];
    __shared__ float lds_dot[2][kChunk], lds_pass[4];
    const Place at = place_of(p, OUT ? p.segments : p.segments - 1);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 32, half = lane / 32;
    const int col0 = at.tile * kCols, cols = min(kCols, p.v.width - col0);
    const int n = p.lengths ? max(0, min(p.L, p.lengths[at.seq])) : p.L;
    const int slot = p.slots ? p.slots[at.seq] : at.seq;
    const bool idle = p.slots && (slot < 0 || slot >= p.n_slots);
    const int chunks = (p.L + kChunk - 1) / kChunk;
    const int c0 = at.segment * p.per_segment, c1 = min(chunks, c0 + p.per_segment);       // in walking order
    // a chunk's first token, and the token of one of its rows
    auto token0 = [&](int chunk) { return (REV ? chunks - 1 - chunk : chunk) * kChunk; };
    auto token = [&](int chunk, int r) { return token0(chunk) + (REV ? kChunk - 1 - r : r); };
    const int osize = p.out_f32 ? 4 : (int)sizeof(T);
    const long o_l = p.out_l * osize;
    char *out = (char *)p.out + (at.seq * p.out_b + (long)at.head * p.v.width + col0) * osize;

    if (idle) {
        for (int c = c0; c < c1 && OUT; ++c)
            for (int i = threadIdx.x; i < kChunk * kCols; i += kThreads) {
                const int t = token(c, i / kCols), x = i % kCols;
                if (t < p.L && x < cols) *(T *)(out + t * o_l + x * sizeof(T)) = from_f<T>(0.f);
            }
        return;
    }

    // places of a wave's tiles of the state
    const int s_row = DK == 128 ? wave * 32 : wave % 2 * 32;
    auto s_col = [&](int i) { return DK == 128 ? 32 * i : wave / 2 * 32; };
    f32x16 state[SD];
#pragma unroll
    for (int i = 0; i < SD; ++i) state[i] = f32x16{};
    if (OUT) {
        const float *from = p.starts ? p.starts + (((long)at.segment * p.B + at.seq) * p.H + at.head) * p.s_head
                                     : p.state_in ? p.state_in + ((long)slot * p.H + at.head) * p.s_head : nullptr;
        if (from)
#pragma unroll
            for (int i = 0; i < SD; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int y = s_row + 8 * (r / 4) + 4 * half + r % 4, x = s_col(i) + row;
                    if (y < p.q.width && x < cols) state[i][r] = from[y * p.s_row + (col0 + x) * p.s_col];
                }
    }

    Fetch<T, DK, WHOLE> fq, fk;
    Fetch<T, kCols, WHOLE> fv;
    const long q_l = p.q.l * sizeof(T), k_l = p.k.l * sizeof(T), v_l = p.v.l * sizeof(T);
    const T *qp = p.q.template at<T>(at.seq, at.head), *kp = p.k.template at<T>(at.seq, at.head), *vp = p.v.template at<T>(at.seq, at.head) + col0;
    if (OUT) fq.init(p.q.width, q_l, REV);
    fk.init(p.k.width, k_l, REV);
    fv.init(cols, v_l, REV);
    auto fetch = [&](int chunk) {
        const long t = token0(chunk);
        const int there = n - (int)t;
        if (OUT) fq.load((const char *)qp + t * q_l, q_l, there);
        fk.load((const char *)kp + t * k_l, k_l, there);
        fv.load((const char *)vp + t * v_l, v_l, there);
    };
    // a lane's outputs: row t, columns x0 + 8 i + 4 half + 0 .. 3
    const int t0 = wave % 2 * 32, x0 = wave / 2 * 32, t_row = t0 + row, t_at = REV ? kChunk - 1 - t_row : t_row;
    const uint32_t o_first = (uint32_t)(t_at * o_l) + (x0 + 4 * half) * osize;
    const long d_l = DG ? p.dot.l * (long)sizeof(T) : 0;
    const T *dp = DG ? p.dot.template at<T>(at.seq, at.head) + col0 : nullptr;
    // the first wave has the decays of the chunk that comes, and those of the one behind it on their way
    T raw_decay = from_f<T>(0.f);
    auto fetch_decay = [&](int chunk) {
        const int t = token(chunk, lane) + (REV ? 1 : 0);
        raw_decay = chunk < c1 && t < n ? p.decays.raw<T>(at.seq, at.head, t) : from_f<T>(0.f);
    };
    auto set_decays = [&](int chunk) {
        const int t = token(chunk, lane) + (REV ? 1 : 0);
        decays[chunk & 1].set(t < n ? p.decays.get<T>(at.head, raw_decay) : 0.f, p.first_scale, p.last_scale);
        fetch_decay(chunk + 1);
    };
    double segment_decay = 0;
    // states at the chunks' starts: pieces of 16 bytes, a workgroup's threads side by side
    constexpr int PER = 16 / sizeof(T), PIECES = 16 * SD / PER;
    typedef Pack<T, PER> Piece;
    auto kept = [&](int c) {
        const long chunk = REV ? chunks - 1 - c : c;
        return (Piece *)p.chunk_states + ((((long)at.seq * p.H + at.head) * p.tiles + at.tile) * chunks + chunk) * (PIECES * kThreads) + threadIdx.x;
    };
    Piece before[DG && REV ? PIECES : 1];
    if (c0 < c1) {
        fetch(c0);
        if (wave == 0) {
            fetch_decay(c0);
            set_decays(c0);
        }
    }
    for (int c = c0; c < c1; ++c) {
        const ChunkDecays &dec = decays[c & 1];
        if (DG && REV) {
            const Piece *from = kept(c);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) before[i] = from[i * kThreads];
        }
        {
            const long t = token0(c);
            if (OUT) fq.store(lds_q, (const char *)qp + t * q_l);
            fk.store(lds_k, (const char *)kp + t * k_l);
            fv.store(lds_v, (const char *)vp + t * v_l);
        }
        if (OUT) {
            // the state as an operand, rounded once to its type
#pragma unroll
            for (int i = 0; i < SD; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4)
                    *reinterpret_cast<Pack<T, 4> *>(lds_s + TQ::at(s_col(i) + row, s_row + 2 * r + 4 * half)) =
                        pack_four<T>(state[i][r], state[i][r + 1], state[i][r + 2], state[i][r + 3]);
            if (DG && !REV) {
                Piece *to = kept(c);
#pragma unroll
                for (int i = 0; i < PIECES; ++i) {
                    Piece v;
#pragma unroll
                    for (int e = 0; e < PER; ++e) v.v[e] = from_f<T>(state[i * PER / 16][i * PER % 16 + e]);
                    to[i * kThreads] = v;
                }
            }
        }
        lds_barrier();
        if (DG && REV) {
            float pass = 0.f;
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int e = 0; e < PER; ++e) pass = fmaf(to_f(before[i % (DG && REV ? PIECES : 1)].v[e]), state[i * PER / 16][i * PER % 16 + e], pass);
            pass = sum_group(pass, 64);
            if (lane == 0) lds_pass[wave] = pass;
        }
        if (wave == 0 && c + 1 < c1) set_decays(c + 1);       // ahead of the loads, which it would wait for
        if (c + 1 < c1) fetch(c + 1);
        if (OUT) {
            // P[t, s]: a lane has row t and 16 s
            const int s0 = x0, t = t_row, tok0 = token0(c);
            const bool real = t_at < n - tok0;
            // what the part of the first state is multiplied with: on its way
            uint32_t dots[DG ? 4 : 1][4];
            if (DG) {
                const auto rsrc = buffer_of((const char *)dp + tok0 * d_l, chunk_bytes(d_l, n - tok0));
                const uint32_t first = (uint32_t)(t_at * d_l) + (x0 + 4 * half) * (uint32_t)sizeof(T);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int have = cols - (x0 + 8 * r + 4 * half);
                    const uint32_t o = first + 8 * r * (uint32_t)sizeof(T);
                    if (WHOLE && sizeof(T) == 2) {
                        const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(rsrc, have > 0 ? o : kOut, 0, 0);
                        dots[r][0] = x[0], dots[r][1] = x[1];
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            dots[r][e] = sizeof(T) == 4 ? __builtin_amdgcn_raw_buffer_load_b32(rsrc, e < have ? o + 4 * e : kOut, 0, 0)
                                                        : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, e < have ? o + 2 * e : kOut, 0, 0);
                    }
                }
            }
            f32x16 acc{};
            if (s0 <= t0)
#pragma unroll
                for (int k = 0; k < DK; k += M::K) acc = M::product(M::template along<DK>(lds_k, s0, k), M::template along<DK>(lds_q, t0, k), acc);
            const float hi = dec.hi[t], lo = dec.lo[t];
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                const int s = s0 + 2 * r + 4 * half;
                const auto shi = *reinterpret_cast<const Pack<float, 4> *>(&dec.hi[s]), slo = *reinterpret_cast<const Pack<float, 4> *>(&dec.lo[s]);
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = ChunkDecays::pair<T>(hi, lo, shi.v[e], slo.v[e]) * p.p_scale;
                    v[e] = s + e <= t ? acc[r + e] * w : 0.f;
                }
                *reinterpret_cast<Pack<T, 4> *>(lds_p + TV::at(t, s)) = pack_four<T>(v[0], v[1], v[2], v[3]);
            }
            lds_barrier();
            if (DG && REV && threadIdx.x == 0) {
                const int chunk = chunks - 1 - c;
                const float own = chunk * kChunk < n ? p.decays.get<T>(at.seq, at.head, (long)chunk * kChunk) : 0.f;
                p.passes[(((long)at.tile * p.B + at.seq) * p.H + at.head) * chunks + chunk] =
                    dec.whole * exp_full(own) * ((lds_pass[0] + lds_pass[1]) + (lds_pass[2] + lds_pass[3]));
            }
            // outputs: a lane has row t and 16 columns
            f32x16 y{};
#pragma unroll
            for (int k = 0; k < DK; k += M::K) y = M::product(M::template along<DK>(lds_s, x0, k), M::template along<DK>(lds_q, t0, k), y);
            const float first = dec.first[t];
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] *= first;
            if (DG) {
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const uint32_t(&d)[4] = dots[DG ? r / 4 : 0];
                    const float v = sizeof(T) == 4 ? __uint_as_float(d[r % 4])
                                    : WHOLE        ? __uint_as_float(r % 2 ? d[r % 4 / 2] & 0xFFFF0000u : d[r % 4 / 2] << 16)
                                                   : __uint_as_float(d[r % 4] << 16);
                    sum = fmaf(v, y[r], sum);
                }
                float other = sum;
                swap_halves(sum, other);
                sum += other;
                if (half == 0) lds_dot[wave / 2][t] = sum;
            }
#pragma unroll
            for (int k = 0; k < kChunk; k += M::K)
                if (k < 32 || t0 == 32) y = M::product(M::template across<kCols>(lds_v, x0, k), M::template along<kCols>(lds_p, t0, k), y);
            const auto rsrc = buffer_of(out + tok0 * o_l, chunk_bytes(o_l, p.L - tok0));
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] = real ? y[r] : 0.f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int have = cols - (x0 + 8 * r + 4 * half);
                const uint32_t o = o_first + 8 * r * osize;
                const auto four = pack_four<T>(y[4 * r], y[4 * r + 1], y[4 * r + 2], y[4 * r + 3]);
                if (sizeof(T) == 4 || p.out_f32) {
                    if (WHOLE) {
                        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, pack_four<float>(y[4 * r], y[4 * r + 1], y[4 * r + 2], y[4 * r + 3])), rsrc,
                                                               have > 0 ? o : kOut, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(y[4 * r + e]), rsrc, e < have ? o + 4 * e : kOut, 0, 0);
                    }
                } else if constexpr (sizeof(T) == 2) {
                    if (WHOLE) {
                        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, four), rsrc, have > 0 ? o : kOut, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, four.v[e]), rsrc, e < have ? o + 2 * e : kOut, 0, 0);
                    }
                }
            }
        }
        // the state behind the chunk
        const float whole = dec.whole;
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) state[i][r] *= whole;
#pragma unroll
        for (int k = 0; k < kChunk; k += M::K) {
            constexpr int E = M::K / 2;
            float w[E];
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                const auto four = *reinterpret_cast<const Pack<float, 4> *>(&dec.last[k + half * E + e]);
#pragma unroll
                for (int i = 0; i < 4; ++i) w[e + i] = four.v[i];
            }
            typename M::Frag a[PARTS];
            M::template weighted<PARTS>(M::template across<DK>(lds_k, s_row, k), w, a);
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                const auto b = M::template across<kCols>(lds_v, s_col(i), k);
#pragma unroll
                for (int e = PARTS; e-- > 0;) state[i] = M::product(a[e], b, state[i]);
            }
        }
        if (!OUT && threadIdx.x < 64) segment_decay += (double)dec.hi[63] + (double)dec.lo[63];
        lds_barrier();
        if (DG && threadIdx.x < kChunk) {
            const int t = token(c, threadIdx.x);
            if (t < p.L) p.dots[(((long)at.tile * p.B + at.seq) * p.H + at.head) * p.L + t] = lds_dot[0][threadIdx.x] + lds_dot[1][threadIdx.x];
        }
    }

    if (!OUT) {
        float *to = p.starts + ((((long)at.segment + 1) * p.B + at.seq) * p.H + at.head) * p.s_head;
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int y = s_row + 8 * (r / 4) + 4 * half + r % 4, x = s_col(i) + row;
                if (y < p.q.width && x < cols) to[y * p.s_row + (col0 + x) * p.s_col] = state[i][r];
            }
        if (threadIdx.x == 0 && at.tile == 0) p.segment_decay[((long)at.segment * p.B + at.seq) * p.H + at.head] = exp2_fast((float)segment_decay);
    } else if (p.state_out && at.segment == p.segments - 1) {
        const float factor = REV && n > 0 ? exp_full(p.decays.get<T>(at.seq, at.head, 0)) : 1.f;
        float *to = p.state_out + ((long)slot * p.H + at.head) * p.s_head;
#pragma unroll
        for (int i = 0; i < SD; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int y = s_row + 8 * (r / 4) + 4 * half + r % 4, x = s_col(i) + row;
                if (y < p.q.width && x < cols) to[y * p.s_row + (col0 + x) * p.s_col] = REV ? state[i][r] * factor : state[i][r];
            }
    }
}

// starts[0] = state_in or 0; starts[j + 1] = decay[j] starts[j] + the segment's own state, which stands there.  grid.y: sequences and heads
__global__ __launch_bounds__(256) void join_states_kernel(Mix p, int size)
{
    for (long sh = blockIdx.y; sh < (long)p.B * p.H; sh += gridDim.y) {
        const int seq = (int)(sh / p.H), head = (int)(sh % p.H), slot = p.slots ? p.slots[seq] : seq;
        const bool idle = p.slots && (slot < 0 || slot >= p.n_slots);
        const long step = (long)p.B * p.H * size;
        for (int i = blockIdx.x * 256 + threadIdx.x; i < size; i += gridDim.x * 256) {
            float s = p.state_in && !idle ? p.state_in[((long)slot * p.H + head) * size + i] : 0.f;
            float *at = p.starts + sh * size + i;
            *at = s;
            for (int j = 1; j < p.segments; ++j) {
                at += step;
                s = fmaf(p.segment_decay[(long)(j - 1) * p.B * p.H + sh], s, *at);
                *at = s;
            }
        }
    }
}

// sum_{s < t} W[t, s] - sum_{t > s} W[t, s] of the same token, for every token of a chunk: to pairs (B, H, L).
struct Pairs {
    Rows q, k, v, dy;
    float scale;
    Decays decays;
    const int32_t *lengths;
    int B, L, H;
    float *out;
};

template <class T, int DK, int DV, bool WHOLE>
__global__ __launch_bounds__(kThreads) void pairs_kernel(Pairs p)
{
    typedef Mma<T> M;
    constexpr int WIDE = DK > DV ? DK : DV;
    __shared__ __attribute__((aligned(16))) char lds_a[TileLds<T, WIDE>::BYTES], lds_b[TileLds<T, WIDE>::BYTES];
    __shared__ float w[kChunk][kChunk + 1];
    __shared__ ChunkDecays dec;
    __shared__ float parts[kThreads];
    const int chunks = (p.L + kChunk - 1) / kChunk;
    const int chunk = blockIdx.x % chunks, head = blockIdx.x / chunks % p.H, seq = blockIdx.x / chunks / p.H;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 32, half = lane / 32;
    const int n = p.lengths ? max(0, min(p.L, p.lengths[seq])) : p.L, first = chunk * kChunk;
    float *out = p.out + ((long)seq * p.H + head) * p.L + first;
    Fetch<T, DK, WHOLE> fq, fk;
    Fetch<T, DV, WHOLE> fv, fo;
    auto load = [&](auto &f, const Rows &r) {
        f.init(r.width, r.l * sizeof(T), false);
        f.load(r.template at<T>(seq, head) + first * r.l, r.l * sizeof(T), n - first);
    };
    auto store = [&](const auto &f, const Rows &r, char *to) { f.store(to, r.template at<T>(seq, head) + first * r.l); };
    load(fq, p.q);
    load(fk, p.k);
    load(fo, p.dy);
    load(fv, p.v);
    const int t0 = wave % 2 * 32, s0 = wave / 2 * 32, t = t0 + row;
    f32x16 acc{}, acc2{};
    if (wave == 0) dec.set(first + lane < n ? p.decays.get<T>(seq, head, first + lane) : 0.f, 1.f, 1.f);
    store(fq, p.q, lds_a);
    store(fk, p.k, lds_b);
    lds_barrier();
    if (s0 <= t0)
#pragma unroll
        for (int k = 0; k < DK; k += M::K) acc = M::product(M::template along<DK>(lds_b, s0, k), M::template along<DK>(lds_a, t0, k), acc);
    lds_barrier();
    store(fo, p.dy, lds_a);
    store(fv, p.v, lds_b);
    lds_barrier();
    if (s0 <= t0)
#pragma unroll
        for (int k = 0; k < DV; k += M::K) acc2 = M::product(M::template along<DV>(lds_b, s0, k), M::template along<DV>(lds_a, t0, k), acc2);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int s = s0 + 8 * (r / 4) + 4 * half + r % 4;
        const float d = ChunkDecays::pair<float>(dec.hi[t], dec.lo[t], dec.hi[s], dec.lo[s]);
        w[t][s] = s < t ? p.scale * acc[r] * acc2[r] * d : 0.f;
    }
    lds_barrier();
    // four threads to a token: half of its row, half of its column
    const int token = threadIdx.x % 64, part = threadIdx.x / 64;
    float sum = 0.f;
    for (int i = 0; i < 32; ++i) {
        const int o = part % 2 * 32 + i;
        sum += part < 2 ? w[token][o] : -w[o][token];
    }
    parts[threadIdx.x] = sum;
    lds_barrier();
    if (threadIdx.x < 64 && first + token < p.L) out[token] = (parts[token] + parts[64 + token]) + (parts[128 + token] + parts[192 + token]);
}

// dg of a chunk's tokens, one lane each: sums of pairs and a from the token to the chunk's end, of b before it, and c
template <class T>
__global__ __launch_bounds__(64) void decay_gradient_kernel(const float *pairs, const float *a, const float *b, const float *c, int tiles_a, int B, int L,
                                                            int H, const int32_t *lengths, T *dg, long g_b, long g_l)
{
    const int chunks = (L + kChunk - 1) / kChunk;
    const long tasks = (long)B * H * chunks, plane = (long)B * H * L;
    for (long i = blockIdx.x; i < tasks; i += gridDim.x) {
        const int chunk = (int)(i % chunks);
        const long sh = i / chunks;
        const int head = (int)(sh % H), seq = (int)(sh / H), lane = threadIdx.x, t = chunk * kChunk + lane;
        const int n = lengths ? max(0, min(L, lengths[seq])) : L;
        float ahead = 0.f, behind = 0.f, through = 0.f;
        if (t < n) {
            ahead = pairs[sh * L + t];
            for (int j = 0; j < tiles_a; ++j) {
                ahead += a[j * plane + sh * L + t];
                behind += b[j * plane + sh * L + t];
            }
        }
        for (int j = 0; j < tiles_a; ++j) through += c[((long)j * B * H + sh) * chunks + chunk];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float up = __shfl_down(ahead, d), down = __shfl_up(behind, d);
            if (lane + d < 64) ahead += up;
            if (lane >= d) behind += down;
        }
        const float before = __shfl_up(behind, 1);
        if (t < L) dg[seq * g_b + t * g_l + head] = from_f<T>(t < n ? ahead + (lane ? before : 0.f) + through : 0.f);
    }
}

// out (B, L, Hk, D) = sums over neighbouring heads of part (B, L, H, D)
template <class T>
__global__ __launch_bounds__(256) void sum_heads_kernel(const float *part, int L, int H, int Hk, int D, long tokens, T *out, long o_b, long o_l)
{
    const int width = Hk * D, shared = H / Hk;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < tokens * width; i += gridDim.x * 256l) {
        const long tok = i / width;
        const int c = (int)(i % width), hk = c / D, x = c % D;
        const float *at = part + (tok * H + (long)hk * shared) * D + x;
        float v = at[0];
        for (int j = 1; j < shared; ++j) v += at[(long)j * D];
        out[tok / L * o_b + tok % L * o_l + c] = from_f<T>(v);
    }
}

// ---- single tokens -------------------------------------------------------------------------------------------------
//
// The state is read and written once, 4 bytes an element: memory bounds it.  A workgroup has 32 columns of a head's state, 8 lanes of 4 columns to a row.

struct StepParams {
    ucd_linear_attention_t d;
    ucd_linear_attention_in_t in;
    Decays decays;
    float *state;
    void *y;
    int tiles;
};

template <class T>
__global__ __launch_bounds__(256) void attention_step_kernel(StepParams p)
{
    __shared__ float sums[32][33];
    const ucd_linear_attention_t &d = p.d;
    const int tile = blockIdx.x % p.tiles, head = blockIdx.x / p.tiles % d.H, seq = blockIdx.x / p.tiles / d.H;
    const int slot = p.in.slots ? p.in.slots[seq] : seq, x = tile * 32 + threadIdx.x % 8 * 4, group = threadIdx.x / 8, have = min(4, d.Dv - x);
    T *y = (T *)p.y + seq * d.y_b + (long)head * d.Dv;
    if (p.in.slots && (slot < 0 || slot >= d.n_slots)) {
        if (threadIdx.x < 32 && tile * 32 + (int)threadIdx.x < d.Dv) y[tile * 32 + threadIdx.x] = from_f<T>(0.f);
        return;
    }
    const int shared = d.H / d.Hk;
    const T *q = (const T *)p.in.q + seq * d.q_b + (long)(head / shared) * d.Dk, *k = (const T *)p.in.k + seq * d.k_b + (long)(head / shared) * d.Dk;
    float *s = p.state + ((long)slot * d.H + head) * d.Dk * d.Dv + x;
    const Pack<T, 4> v = load_pack<false, T, 4>((const T *)p.in.v + seq * d.v_b + (long)head * d.Dv + x, have);
    const float a = exp_full(p.decays.get<T>(seq, head, 0));
    Pack<float, 4> sum{};
#pragma unroll 4
    for (int i = group; i < d.Dk; i += 32) {
        float *at = s + (long)i * d.Dv;
        Pack<float, 4> h = have == 4 ? loose_load<float, 4>(at) : load_pack<false, float, 4>(at, have);
        const float ki = to_f(k[i]), qi = to_f(q[i]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h.v[e] = fmaf(a, h.v[e], ki * to_f(v.v[e]));
            sum.v[e] = fmaf(qi, h.v[e], sum.v[e]);
        }
        if (have == 4) loose_store<float, 4>(at, h);
        else store_pack<false, float, 4>(at, h, have);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[group][threadIdx.x % 8 * 4 + e] = sum.v[e];
    __syncthreads();
    const int c = threadIdx.x;
    if (c < 32 && tile * 32 + c < d.Dv) {
        float v = 0.f;
#pragma unroll
        for (int g = 0; g < 32; ++g) v += sums[g][c];
        y[tile * 32 + c] = from_f<T>(d.scale * v);
    }
}

// ---- plans ---------------------------------------------------------------------------------------------------------

int chunks_of(int L) { return (L + kChunk - 1) / kChunk; }
int tiles_of(int width) { return (width + kCols - 1) / kCols; }

// Segments of a walk: as many as fill the card with two workgroups to a unit, where there is not one to each anyway.
void segments_of(int B, int L, int H, int width, int &segments, int &per)
{
    const long have = (long)B * H * tiles_of(width), chunks = std::max(1, chunks_of(L));
    const long want = have >= 256 ? 1 : std::max(1l, std::min(512 / std::max(1l, have), chunks));
    per = (int)((chunks + want - 1) / want);
    segments = (int)((chunks + per - 1) / per);
}

struct Layout {
    int segments, per;          // columns of Dv: Forward, dv
    int segments_k, per_k;      // columns of Dk: dq, dk
    size_t starts, decay, starts_k, decay_k, transposed;
    size_t pairs, a, b, c, keep, heads, bytes;
};

size_t state_size(const ucd_linear_attention_t &d) { return (size_t)d.B * d.H * d.Dk * d.Dv; }

Layout layout_of(const ucd_linear_attention_t &d, int dir)
{
    Layout l{};
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    const size_t esize = d.dtype == 1 ? 2 : 4;
    segments_of(d.B, d.L, d.H, d.Dv, l.segments, l.per);
    segments_of(d.B, d.L, d.H, d.Dk, l.segments_k, l.per_k);
    const size_t bh = (size_t)d.B * d.H;
    if (l.segments > 1) {
        l.starts = take(l.segments * state_size(d) * 4);
        l.decay = take(l.segments * bh * 4);
    }
    if (dir == UCD_SEQ_BWD) {
        if (l.segments_k > 1) {
            l.starts_k = take(l.segments_k * state_size(d) * 4);
            l.decay_k = take(l.segments_k * bh * 4);
        }
        const size_t tiles = tiles_of(d.Dk);
        l.pairs = take(bh * d.L * 4);
        l.a = take(tiles * bh * d.L * 4);
        l.b = take(tiles * bh * d.L * 4);
        l.c = take(tiles * bh * chunks_of(d.L) * 4);
        l.keep = take(tiles * bh * chunks_of(d.L) * kThreads * (d.Dv > 64 ? 32 : 16) * esize);
        if (d.H != d.Hk) l.heads = take(bh * d.L * d.Dk * 4);
    }
    l.bytes = at;
    return l;
}

// Rows that Fetch can read by whole pieces
template <class T>
bool whole_rows(const Rows &r)
{
    constexpr int PER = 16 / sizeof(T), WORD = 4 / sizeof(T);
    return r.width % PER == 0 && r.l % WORD == 0 && r.b % WORD == 0 && ((uintptr_t)r.p & 3u) == 0;
}

template <class T, int DK, bool REV, bool WHOLE>
hipError_t run_mix(const Mix &p, hipStream_t s)
{
    const unsigned groups = (unsigned)((long)p.B * p.H * p.tiles);
    if (p.segments > 1) {
        mix_kernel<T, DK, REV, STATES, WHOLE><<<groups * (p.segments - 1), kThreads, 0, s>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.starts) {      // also of one segment, where Forward keeps the state that it begins with
        const int size = (int)p.s_head;
        join_states_kernel<<<dim3((unsigned)std::min(64, (size + 255) / 256), (unsigned)std::min(65535l, (long)p.B * p.H)), 256, 0, s>>>(p, size);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.dots) mix_kernel<T, DK, REV, DECAYS, WHOLE><<<groups * p.segments, kThreads, 0, s>>>(p);
    else mix_kernel<T, DK, REV, OUTPUTS, WHOLE><<<groups * p.segments, kThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, bool REV>
hipError_t run_mix(Mix &p, hipStream_t s)
{
    p.tiles = tiles_of(p.v.width);
    const Rows out{p.out, p.out_b, p.out_l, 1, p.v.width};
    const bool whole = whole_rows<T>(p.q) && whole_rows<T>(p.k) && whole_rows<T>(p.v) && whole_rows<T>(out) && (!p.dots || whole_rows<T>(p.dot));
    if (whole) return p.q.width > 64 ? run_mix<T, 128, REV, true>(p, s) : run_mix<T, 64, REV, true>(p, s);
    return p.q.width > 64 ? run_mix<T, 128, REV, false>(p, s) : run_mix<T, 64, REV, false>(p, s);
}

template <class T, bool WHOLE>
hipError_t run_pairs(const Pairs &r, unsigned grid, hipStream_t s)
{
    if (r.k.width > 64 && r.v.width > 64) pairs_kernel<T, 128, 128, WHOLE><<<grid, kThreads, 0, s>>>(r);
    else if (r.k.width > 64) pairs_kernel<T, 128, 64, WHOLE><<<grid, kThreads, 0, s>>>(r);
    else if (r.v.width > 64) pairs_kernel<T, 64, 128, WHOLE><<<grid, kThreads, 0, s>>>(r);
    else pairs_kernel<T, 64, 64, WHOLE><<<grid, kThreads, 0, s>>>(r);
    return hipGetLastError();
}

Mix mix_base(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in)
{
    Mix p{};
    p.decays = Decays{in.g, d.g_b, d.g_l, in.decay};
    p.lengths = in.lengths;
    p.slots = in.slots;
    p.B = d.B;
    p.L = d.L;
    p.H = d.H;
    p.n_slots = d.n_slots;
    p.s_head = (long)d.Dk * d.Dv;
    return p;
}

template <class T>
hipError_t fwd(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in, const float *state_in, float *state_out, void *y, float *saved,
               char *ws, hipStream_t s)
{
    const Layout l = layout_of(d, UCD_SEQ_FWD);
    Mix p = mix_base(d, in);
    const int shared = d.H / d.Hk;
    p.q = Rows{in.q, (long)d.q_b, (long)d.q_l, shared, d.Dk};
    p.k = Rows{in.k, (long)d.k_b, (long)d.k_l, shared, d.Dk};
    p.v = Rows{in.v, (long)d.v_b, (long)d.v_l, 1, d.Dv};
    p.out = y;
    p.out_b = d.y_b;
    p.out_l = d.y_l;
    p.p_scale = p.first_scale = d.scale;
    p.last_scale = 1.f;
    p.state_in = state_in;
    p.state_out = state_out;
    p.s_row = d.Dv;
    p.s_col = 1;
    p.segments = l.segments;
    p.per_segment = l.per;
    p.starts = saved ? saved : l.segments > 1 ? (float *)(ws + l.starts) : nullptr;
    p.segment_decay = (float *)(ws + l.decay);
    return run_mix<T, false>(p, s);
}

template <class T>
hipError_t bwd(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in, const void *dy, const float *dstate_out, const float *saved,
               const ucd_linear_attention_grad_t &grad, char *ws, hipStream_t s)
{
    const Layout l = layout_of(d, UCD_SEQ_BWD);
    const int shared = d.H / d.Hk;
    const Rows q{in.q, (long)d.q_b, (long)d.q_l, shared, d.Dk}, k{in.k, (long)d.k_b, (long)d.k_l, shared, d.Dk};
    const Rows v{in.v, (long)d.v_b, (long)d.v_l, 1, d.Dv}, o{dy, (long)d.y_b, (long)d.y_l, 1, d.Dv};
    const bool decays = grad.g != nullptr;
    hipError_t e;
    // dv, and the gradient of the first state
    Mix p = mix_base(d, in);
    p.q = k;
    p.k = q;
    p.v = o;
    p.out = grad.v;
    p.out_b = d.v_b;
    p.out_l = d.v_l;
    p.p_scale = p.last_scale = d.scale;
    p.first_scale = 1.f;
    p.state_in = dstate_out;
    p.state_out = grad.state;
    p.s_row = d.Dv;
    p.s_col = 1;
    p.segments = l.segments;
    p.per_segment = l.per;
    p.starts = l.segments > 1 ? (float *)(ws + l.starts) : nullptr;
    p.segment_decay = (float *)(ws + l.decay);
    if ((e = run_mix<T, true>(p, s)) != hipSuccess) return e;
    // dq: the states again, transposed
    Mix a = mix_base(d, in);
    a.q = o;
    a.k = v;
    a.v = k;
    a.dot = q;
    a.p_scale = a.first_scale = d.scale;
    a.last_scale = 1.f;
    a.state_in = saved;       // of the sequences' starts
    a.s_row = 1;
    a.s_col = d.Dv;
    a.segments = l.segments_k;
    a.per_segment = l.per_k;
    a.starts = l.segments_k > 1 ? (float *)(ws + l.starts_k) : nullptr;
    a.segment_decay = (float *)(ws + l.decay_k);
    a.dots = decays ? (float *)(ws + l.a) : nullptr;
    a.chunk_states = ws + l.keep;
    a.passes = (float *)(ws + l.c);
    auto heads = [&](Mix &m, void *out, long o_b, long o_l, bool rev) {
        m.out_f32 = shared > 1;
        m.out = shared > 1 ? ws + l.heads : out;
        m.out_l = shared > 1 ? (long)d.H * d.Dk : o_l;
        m.out_b = shared > 1 ? m.out_l * d.L : o_b;
        const hipError_t e = rev ? run_mix<T, true>(m, s) : run_mix<T, false>(m, s);
        if (shared == 1) return e;
        const long tokens = (long)d.B * d.L;
        if (e != hipSuccess || tokens == 0) return e;
        const unsigned grid = (unsigned)std::min((tokens * d.Hk * d.Dk + 255) / 256, 1l << 16);
        sum_heads_kernel<T><<<grid, 256, 0, s>>>((const float *)(ws + l.heads), d.L, d.H, d.Hk, d.Dk, tokens, (T *)out, o_b, o_l);
        return hipGetLastError();
    };
    if ((e = heads(a, grad.q, d.q_b, d.q_l, false)) != hipSuccess) return e;
    // dk
    Mix b = a;
    b.q = v;
    b.k = o;
    b.v = q;
    b.dot = k;
    b.p_scale = b.last_scale = d.scale;
    b.first_scale = 1.f;
    b.state_in = dstate_out;
    b.dots = decays ? (float *)(ws + l.b) : nullptr;
    if ((e = heads(b, grad.k, d.k_b, d.k_l, true)) != hipSuccess) return e;
    if (!decays || d.L == 0) return hipSuccess;
    Pairs r{q, k, v, o, d.scale, a.decays, in.lengths, d.B, d.L, d.H, (float *)(ws + l.pairs)};
    const unsigned grid = (unsigned)((long)d.B * d.H * chunks_of(d.L));
    const bool whole = whole_rows<T>(q) && whole_rows<T>(k) && whole_rows<T>(v) && whole_rows<T>(o);
    if ((e = whole ? run_pairs<T, true>(r, grid, s) : run_pairs<T, false>(r, grid, s)) != hipSuccess) return e;
    decay_gradient_kernel<T><<<std::min(grid, 1u << 20), 64, 0, s>>>(r.out, a.dots, b.dots, a.passes, tiles_of(d.Dk), d.B, d.L, d.H, in.lengths, (T *)grad.g,
                                                                    d.g_b, d.g_l);
    return hipGetLastError();
}

}  // namespace

size_t linear_attention_ws_bytes(const ucd_linear_attention_t &d, int dir)
{
    if (d.B == 0 || d.L == 0) return 0;
    return layout_of(d, dir).bytes;
}

size_t linear_attention_saved_bytes(const ucd_linear_attention_t &d)
{
    const Layout l = layout_of(d, UCD_SEQ_FWD);
    return l.segments * state_size(d) * 4;
}

// Workgroups of the launches, which are counted in 32 bits, and their threads
bool linear_attention_countable(const ucd_linear_attention_t &d)
{
    return (double)d.B * d.H * std::max({tiles_of(d.Dk), tiles_of(d.Dv), (d.Dv + 31) / 32, chunks_of(d.L)}) < 1 << 23;
}

hipError_t linear_attention_fwd(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in, const float *state_in, float *state_out, void *y,
                                float *saved, void *ws, hipStream_t s)
{
    return d.dtype == 1 ? fwd<bf16_t>(d, in, state_in, state_out, y, saved, (char *)ws, s) : fwd<float>(d, in, state_in, state_out, y, saved, (char *)ws, s);
}

hipError_t linear_attention_bwd(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in, const void *dy, const float *dstate_out,
                                const float *saved, const ucd_linear_attention_grad_t &grad, void *ws, hipStream_t s)
{
    return d.dtype == 1 ? bwd<bf16_t>(d, in, dy, dstate_out, saved, grad, (char *)ws, s) : bwd<float>(d, in, dy, dstate_out, saved, grad, (char *)ws, s);
}

hipError_t linear_attention_step(const ucd_linear_attention_t &d, const ucd_linear_attention_in_t &in, float *state, void *y, hipStream_t s)
{
    StepParams p{d, in, Decays{in.g, d.g_b, d.g_l, in.decay}, state, y, (d.Dv + 31) / 32};
    const unsigned grid = (unsigned)((long)d.B * d.H * p.tiles);
    if (d.dtype == 1) attention_step_kernel<bf16_t><<<grid, 256, 0, s>>>(p);
    else attention_step_kernel<float><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace ucd
