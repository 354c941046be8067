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
    __device__ __forceinline__ const T *at(int seq, int head, long t) const { return (const T *)p + seq * b + t * l + (long)(head / div) * width; }
};

struct Mix {
    Rows q, k, v, dot;           // dot: rows like the output's, multiplied with the part of the state at the chunk's start; may be none
    void *out;
    long out_b, out_l;
    float p_scale, first_scale, last_scale;
    Decays decays;
    const int32_t *lengths, *slots;
    int B, L, H, n_slots, segments, per_segment;     // chunks of a segment
    // states: of a slot and head rows (of q's width) and columns (of v's) apart
    const float *state_in;
    float *state_out;
    long s_row, s_col, s_head, s_out_row, s_out_col;
    float *starts;               // (segments, B, H, rows, columns) with the strides of state_in, or null
    float *segment_decay;        // (segments, B, H)
    float *dots;                 // (column tiles, B, H, L), or null
    void *chunk_states;          // states at the chunks' starts, by workgroup, chunk and thread; or null
    float *passes;               // (column tiles, B, H, chunks): c
    int tiles;
};

// Places of a launch: column tile, head, sequence, segment.  Column tiles of a head are neighbours that share q and k.
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

enum { KEEP_NONE = 0, KEEP_WRITE = 1, KEEP_READ = 2 };

// DK: q's width, 64 or 128.  STATES: only the segment's own state, from nothing.
template <class T, class OUT, int DK, bool REV, bool STATES, int KEEP>
__global__ __launch_bounds__(kThreads) void mix_kernel(Mix p)
{
    typedef Mma<T> M;
    typedef TileLds<T, DK> TQ;
    typedef TileLds<T, kCols> TV;
    constexpr int SD = DK / 64;         // a wave's tiles of the state: DK = 128: 32 rows and all 64 columns; 64: 32 rows and 32 columns
    __shared__ __attribute__((aligned(16))) char lds_q[STATES ? 16 : TQ::BYTES], lds_k[TQ::BYTES], lds_v[TV::BYTES],
        lds_p[STATES ? 16 : TV::BYTES], lds_s[STATES ? 16 : TQ::BYTES];      // lds_s: the state's columns as rows of DK
    __shared__ ChunkDecays dec;
    __shared__ float lds_dot[2][kChunk], lds_pass[4];
    const Place at = place_of(p, STATES ? p.segments - 1 : p.segments);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 32, half = lane / 32;
    const int col0 = at.tile * kCols, cols = min(kCols, p.v.width - col0);
    const int n = p.lengths ? max(0, min(p.L, p.lengths[at.seq])) : p.L;
    const int slot = p.slots ? p.slots[at.seq] : at.seq;
    const bool idle = p.slots && (slot < 0 || slot >= p.n_slots);
    const int chunks = (p.L + kChunk - 1) / kChunk;
    const int c0 = at.segment * p.per_segment, c1 = min(chunks, c0 + p.per_segment);       // in walking order

    // places of a wave's tiles of the state
    const int s_row = DK == 128 ? wave * 32 : wave % 2 * 32;
    auto s_col = [&](int i) { return DK == 128 ? 32 * i : wave / 2 * 32; };
    f32x16 state[SD];
#pragma unroll
    for (int i = 0; i < SD; ++i) state[i] = f32x16{};
    if (!STATES && !idle) {
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

    auto token = [&](int chunk, int r) { return (REV ? chunks - 1 - chunk : chunk) * kChunk + (REV ? kChunk - 1 - r : r); };
    Fetch<T, DK> fq, fk;
    Fetch<T, kCols> fv;
    auto fetch = [&](int chunk) {
        auto rows = [&](const Rows &s) {
            return [&s, &at, n, chunk, token](int r) {
                const int t = token(chunk, r);
                return t < n ? s.template at<T>(at.seq, at.head, t) : nullptr;
            };
        };
        if (!STATES) fq.load(rows(p.q), p.q.width);
        fk.load(rows(p.k), p.k.width);
        auto v = rows(p.v);
        fv.load([&](int r) { const T *s = v(r); return s ? s + col0 : nullptr; }, cols);
    };
    auto own_decay = [&](int chunk) {
        const int t = token(chunk, lane) + (REV ? 1 : 0);
        return t < n ? p.decays.get<T>(at.seq, at.head, t) : 0.f;
    };
    double segment_decay = 0;

    if (idle) {
        for (int c = c0; c < c1 && !STATES; ++c)
            for (int i = threadIdx.x; i < kChunk * kCols; i += kThreads) {
                const int t = token(c, i / kCols), x = i % kCols;
                if (t < p.L && x < cols) ((OUT *)p.out + at.seq * p.out_b + t * p.out_l + (long)at.head * p.v.width + col0)[x] = from_f<OUT>(0.f);
            }
        return;
    }
    if (c0 < c1) fetch(c0);
    for (int c = c0; c < c1; ++c) {
        if (!STATES) fq.store(lds_q);
        fk.store(lds_k);
        fv.store(lds_v);
        if (wave == 0) {
            const float own = own_decay(c);
            dec.set(own, p.first_scale, p.last_scale);
        }
        if (!STATES) {
            // the state as an operand, rounded once to its type
#pragma unroll
            for (int i = 0; i < SD; ++i)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    Pack<T, 4> v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v.v[e] = from_f<T>(state[i][r + e]);
                    *reinterpret_cast<Pack<T, 4> *>(lds_s + TQ::at(s_col(i) + row, s_row + 2 * r + 4 * half)) = v;
                }
            if (KEEP == KEEP_WRITE || KEEP == KEEP_READ) {
                // by thread: 16 SD values of T
                const long chunk = REV ? chunks - 1 - c : c;
                T *keep = (T *)p.chunk_states + (((((long)at.seq * p.H + at.head) * p.tiles + at.tile) * chunks + chunk) * kThreads + threadIdx.x) * (16 * SD);
                float pass = 0.f;
#pragma unroll
                for (int i = 0; i < SD; ++i)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        Pack<T, 4> v;
                        if (KEEP == KEEP_WRITE) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v.v[e] = from_f<T>(state[i][r + e]);
                            *reinterpret_cast<Pack<T, 4> *>(keep + 16 * i + r) = v;
                        } else {
                            v = *reinterpret_cast<const Pack<T, 4> *>(keep + 16 * i + r);
#pragma unroll
                            for (int e = 0; e < 4; ++e) pass = fmaf(to_f(v.v[e]), state[i][r + e], pass);
                        }
                    }
                if (KEEP == KEEP_READ) {
                    pass = sum_group(pass, 64);
                    if (lane == 0) lds_pass[wave] = pass;
                }
            }
        }
        __syncthreads();
        if (c + 1 < c1) fetch(c + 1);
        if (KEEP == KEEP_READ && threadIdx.x == 0) {
            const int chunk = chunks - 1 - c;
            const float own = chunk * kChunk < n ? p.decays.get<T>(at.seq, at.head, (long)chunk * kChunk) : 0.f;
            p.passes[(((long)at.tile * p.B + at.seq) * p.H + at.head) * chunks + chunk] =
                dec.whole * exp_full(own) * ((lds_pass[0] + lds_pass[1]) + (lds_pass[2] + lds_pass[3]));
        }
        if (!STATES) {
            // P[t, s]: a lane has row t and 16 s
            const int t0 = wave % 2 * 32, s0 = wave / 2 * 32, t = t0 + row;
            f32x16 acc{};
            if (s0 <= t0)
#pragma unroll
                for (int k = 0; k < DK; k += M::K) acc = M::product(M::template along<DK>(lds_k, s0, k), M::template along<DK>(lds_q, t0, k), acc);
            const float hi = dec.hi[t], lo = dec.lo[t];
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                Pack<T, 4> v;
                const int s = s0 + 2 * r + 4 * half;
                const auto shi = *reinterpret_cast<const Pack<float, 4> *>(&dec.hi[s]), slo = *reinterpret_cast<const Pack<float, 4> *>(&dec.lo[s]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float w = exp2_fast((hi - shi.v[e]) + (lo - slo.v[e])) * p.p_scale;
                    v.v[e] = from_f<T>(s + e <= t ? acc[r + e] * w : 0.f);
                }
                *reinterpret_cast<Pack<T, 4> *>(lds_p + TV::at(t, s)) = v;
            }
            __syncthreads();
            // outputs: a lane has row t and 16 columns
            const int x0 = wave / 2 * 32;
            f32x16 y{};
#pragma unroll
            for (int k = 0; k < DK; k += M::K) y = M::product(M::template along<DK>(lds_s, x0, k), M::template along<DK>(lds_q, t0, k), y);
            const float first = dec.first[t];
#pragma unroll
            for (int r = 0; r < 16; ++r) y[r] *= first;
            const int tok = token(c, t);
            if (p.dots) {
                const T *d = tok < n ? p.dot.template at<T>(at.seq, at.head, tok) + col0 : nullptr;
                float sum = 0.f;
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int x = x0 + 2 * r + 4 * half, have = d ? cols - x : 0;
                    const Pack<T, 4> v = have >= 4 ? loose_load<T, 4>(d + x) : load_pack<false, T, 4>(d + x, have);
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum = fmaf(to_f(v.v[e]), y[r + e], sum);
                }
                float other = sum;
                swap_halves(sum, other);
                sum += other;
                if (half == 0) lds_dot[wave / 2][t] = sum;
            }
#pragma unroll
            for (int k = 0; k < kChunk; k += M::K)
                if (k < t0 + 32) y = M::product(M::template across<kCols>(lds_v, x0, k), M::template along<kCols>(lds_p, t0, k), y);
            if (tok < p.L) {
                OUT *to = (OUT *)p.out + at.seq * p.out_b + tok * p.out_l + (long)at.head * p.v.width + col0;
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int x = x0 + 2 * r + 4 * half, have = min(4, cols - x);
                    Pack<OUT, 4> v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v.v[e] = from_f<OUT>(tok < n ? y[r + e] : 0.f);
                    if (have == 4) loose_store<OUT, 4>(to + x, v);
                    else if (have > 0) store_pack<false, OUT, 4>(to + x, v, have);
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
            for (int e = 0; e < E; e += 4) *reinterpret_cast<Pack<float, 4> *>(w + e) = *reinterpret_cast<const Pack<float, 4> *>(&dec.last[k + half * E + e]);
            typename M::Frag a[M::PARTS];
            M::weighted(M::template across<DK>(lds_k, s_row, k), w, a);
#pragma unroll
            for (int i = 0; i < SD; ++i) {
                const auto b = M::template across<kCols>(lds_v, s_col(i), k);
#pragma unroll
                for (int e = M::PARTS; e-- > 0;) state[i] = M::product(a[e], b, state[i]);
            }
        }
        if (STATES && threadIdx.x < 64) {
            const double all = (double)dec.hi[63] + (double)dec.lo[63];
            segment_decay += all;
        }
        __syncthreads();
        if (!STATES && p.dots && threadIdx.x < kChunk) {
            const int t = token(c, threadIdx.x);
            if (t < p.L) p.dots[(((long)at.tile * p.B + at.seq) * p.H + at.head) * p.L + t] = lds_dot[0][threadIdx.x] + lds_dot[1][threadIdx.x];
        }
    }

    if (STATES) {
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

template <class T, int DK, int DV>
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
    auto rows = [&](const Rows &s) {
        return [&s, seq, head, n, first](int r) { return first + r < n ? s.template at<T>(seq, head, first + r) : nullptr; };
    };
    const int t0 = wave % 2 * 32, s0 = wave / 2 * 32, t = t0 + row;
    f32x16 acc{}, acc2{};
    {
        Fetch<T, DK> f;
        f.load(rows(p.q), p.q.width);
        f.store(lds_a);
        f.load(rows(p.k), p.k.width);
        f.store(lds_b);
    }
    if (wave == 0) dec.set(first + lane < n ? p.decays.get<T>(seq, head, first + lane) : 0.f, 1.f, 1.f);
    __syncthreads();
    if (s0 <= t0)
#pragma unroll
        for (int k = 0; k < DK; k += M::K) acc = M::product(M::template along<DK>(lds_b, s0, k), M::template along<DK>(lds_a, t0, k), acc);
    __syncthreads();
    {
        Fetch<T, DV> f;
        f.load(rows(p.dy), p.dy.width);
        f.store(lds_a);
        f.load(rows(p.v), p.v.width);
        f.store(lds_b);
    }
    __syncthreads();
    if (s0 <= t0)
#pragma unroll
        for (int k = 0; k < DV; k += M::K) acc2 = M::product(M::template along<DV>(lds_b, s0, k), M::template along<DV>(lds_a, t0, k), acc2);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int s = s0 + 8 * (r / 4) + 4 * half + r % 4;
        const float d = exp2_fast((dec.hi[t] - dec.hi[s]) + (dec.lo[t] - dec.lo[s]));
        w[t][s] = s < t ? p.scale * acc[r] * acc2[r] * d : 0.f;
    }
    __syncthreads();
    // four threads to a token: half of its row, half of its column
    const int token = threadIdx.x % 64, part = threadIdx.x / 64;
    float sum = 0.f;
    for (int i = 0; i < 32; ++i) {
        const int o = part % 2 * 32 + i;
        sum += part < 2 ? w[token][o] : -w[o][token];
    }
    parts[threadIdx.x] = sum;
    __syncthreads();
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

// Segments of a walk: as many as fill the card with two workgroups to a unit, of 4 chunks at least.
void segments_of(int B, int L, int H, int width, int &segments, int &per)
{
    const long have = (long)B * H * tiles_of(width), chunks = std::max(1, chunks_of(L));
    const long want = std::max(1l, std::min(512 / std::max(1l, have), chunks / 4));
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

template <class T, class OUT, int DK, bool REV>
hipError_t run_mix(Mix &p, int keep, hipStream_t s)
{
    p.tiles = tiles_of(p.v.width);
    const unsigned groups = (unsigned)((long)p.B * p.H * p.tiles);
    if (p.segments > 1) {
        mix_kernel<T, OUT, DK, REV, true, KEEP_NONE><<<groups * (p.segments - 1), kThreads, 0, s>>>(p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        const int size = (int)p.s_head;
        join_states_kernel<<<dim3((unsigned)std::min(64, (size + 255) / 256), (unsigned)std::min(65535l, (long)p.B * p.H)), 256, 0, s>>>(p, size);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    } else if (p.starts) {      // Forward keeps the state that it begins with
        const int size = (int)p.s_head;
        join_states_kernel<<<dim3((unsigned)std::min(64, (size + 255) / 256), (unsigned)std::min(65535l, (long)p.B * p.H)), 256, 0, s>>>(p, size);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const unsigned grid = groups * p.segments;
    if (keep == KEEP_NONE) mix_kernel<T, OUT, DK, REV, false, KEEP_NONE><<<grid, kThreads, 0, s>>>(p);
    else if (!REV) mix_kernel<T, OUT, DK, REV, false, KEEP_WRITE><<<grid, kThreads, 0, s>>>(p);
    else mix_kernel<T, OUT, DK, REV, false, KEEP_READ><<<grid, kThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, class OUT, bool REV>
hipError_t run_mix(Mix &p, int keep, hipStream_t s)
{
    return p.q.width > 64 ? run_mix<T, OUT, 128, REV>(p, keep, s) : run_mix<T, OUT, 64, REV>(p, keep, s);
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
    return run_mix<T, T, false>(p, KEEP_NONE, s);
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
    if ((e = run_mix<T, T, true>(p, KEEP_NONE, s)) != hipSuccess) return e;
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
        const int keep = !decays ? KEEP_NONE : rev ? KEEP_READ : KEEP_WRITE;
        if (shared == 1) {
            m.out = out;
            m.out_b = o_b;
            m.out_l = o_l;
            return rev ? run_mix<T, T, true>(m, keep, s) : run_mix<T, T, false>(m, keep, s);
        }
        m.out = ws + l.heads;
        m.out_l = (long)d.H * d.Dk;
        m.out_b = m.out_l * d.L;
        const hipError_t e = rev ? run_mix<T, float, true>(m, keep, s) : run_mix<T, float, false>(m, keep, s);
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
    if (d.Dk > 64 && d.Dv > 64) pairs_kernel<T, 128, 128><<<grid, kThreads, 0, s>>>(r);
    else if (d.Dk > 64) pairs_kernel<T, 128, 64><<<grid, kThreads, 0, s>>>(r);
    else if (d.Dv > 64) pairs_kernel<T, 64, 128><<<grid, kThreads, 0, s>>>(r);
    else pairs_kernel<T, 64, 64><<<grid, kThreads, 0, s>>>(r);
    if ((e = hipGetLastError()) != hipSuccess) return e;
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
