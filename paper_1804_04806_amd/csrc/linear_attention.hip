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
// A workgroup walks over the chunks of a sequence's head with 64 or 128 columns of the state, fp32 in the matrix instructions' registers.  Long sequences with
// few heads are cut into segments: their own states first, then the states at their starts, then all segments at once.
//
// The gradient of a decay is that of all paths that cross it: pairs of tokens within the chunk, tokens with the states before and behind it, and the
// state that passes through.  With W[t, s] = scale (q_t . k_s) (dy_t . v_s) D,
//   dl_u = sum_{s < u <= t} W[t, s] + sum_{t >= u} a_t + sum_{s < u} b_s + c,
//   a_t = q_t . (dq_t's part of S_in),  b_s = k_s . (dk_s's part of dS_out),  c = e^{G_C} <S_in, dS_out>.
// A_t = q_t . dq_t without W[t, t] is a_t and W's row, B_s = k_s . dk_s without W[s, s] is b_s and W's column, so that
//   dl_u = sum_{t >= u} (A_t - (B_t - b_t)) + sum_{s < u} b_s + c.
// A pair that does not cross u is in a row and in a column, of the same product rounded to the same 16 bits (both walks take its decay from sums that are the
// same to far below 32 bits, and round it once): what is left of it is rounding of 32 bits.
// Sums of A - B over whole sequences would be the same as this in exact arithmetic, but the states' roundings are not the same on both sides.  (Pairs
// in a kernel of their own read all inputs again, 59 us of 526 for 8 x 2048 tokens of 16 heads of 128.)
#include <algorithm>

#include "linear_attention.hpp"

namespace ucd {
namespace attention {

// starts[0] = state_in or 0; starts[j + 1] = decay[j] starts[j] + the segment's own state, which stands there.  grid.y: sequences and heads.  Memory bounds it:
// the states of a few segments are on their way at once (four segments of 128 heads of 128 by 128, 59 MB: 12 us).
template <int N>
__global__ __launch_bounds__(256) void join_states_kernel(Mix p, int size)
{
    constexpr int AHEAD = 4;
    for (long sh = blockIdx.y; sh < (long)p.B * p.H; sh += gridDim.y) {
        const int seq = (int)(sh / p.H), head = (int)(sh % p.H), slot = p.slots ? p.slots[seq] : seq;
        const bool idle = p.slots && (slot < 0 || slot >= p.n_slots);
        const long heads = (long)p.B * p.H, step = heads * size;
        const float *decay = p.segment_decay + sh;
        for (int i = (blockIdx.x * 256 + threadIdx.x) * N; i < size; i += gridDim.x * 256 * N) {
            Pack<float, N> s{};
            if (p.state_in && !idle) s = loose_load<float, N>(p.state_in + ((long)slot * p.H + head) * size + i);
            float *at = p.starts + sh * size + i;
            loose_store<float, N>(at, s);
            for (int j = 1; j < p.segments; j += AHEAD) {
                const int there = min(AHEAD, p.segments - j);
                Pack<float, N> own[AHEAD];
                float d[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {      // behind the last one, that again
                    const long o = j + min(k, there - 1);
                    own[k] = loose_load<float, N>(at + o * step);
                    d[k] = decay[(o - 1) * heads];
                }
#pragma unroll
                for (int k = 0; k < AHEAD; ++k)
                    if (k < there) {
#pragma unroll
                        for (int e = 0; e < N; ++e) s.v[e] = fmaf(d[k], s.v[e], own[k].v[e]);
                        loose_store<float, N>(at + (j + k) * step, s);
                    }
            }
        }
    }
}

hipError_t join_states(const Mix &p, hipStream_t s)
{
    const int size = (int)p.s_head, packs = size % 4 == 0 ? size / 4 : size;
    const dim3 grid((unsigned)std::min(64, (packs + 255) / 256), (unsigned)std::min(65535l, (long)p.B * p.H));
    if (size % 4 == 0) join_states_kernel<4><<<grid, 256, 0, s>>>(p, size);
    else join_states_kernel<1><<<grid, 256, 0, s>>>(p, size);
    return hipGetLastError();
}

}  // namespace attention

namespace {
using namespace attention;

// dg of a chunk's tokens, one lane each: sums of A - (B - b) from the token to the chunk's end, of b before it, and c.  A, B and b are `planes` sums each
template <class T>
__global__ __launch_bounds__(64) void decay_gradient_kernel(const float *A, const float *B_, const float *b, const float *c, int planes, int tiles, int B,
                                                            int L, int H, const int32_t *lengths, Decays decays, T *dg, long g_b, long g_l)
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
            float crossing = 0.f;
            for (int j = 0; j < planes; ++j) {
                const long at = j * plane + sh * L + t;
                ahead += A[at];
                crossing += B_[at] - b[at];
                behind += b[at];
            }
            ahead -= crossing;
        }
        for (int j = 0; j < tiles; ++j) through += c[((long)j * B * H + sh) * chunks + chunk];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const float up = __shfl_down(ahead, d), down = __shfl_up(behind, d);
            if (lane + d < 64) ahead += up;
            if (lane >= d) behind += down;
        }
        const float before = __shfl_up(behind, 1);
        // a decay that forgets everything has none: what is left of sums around it is rounding
        const bool real = t < n && !(decays.get<T>(seq, head, t) <= kLeast);
        if (t < L) dg[seq * g_b + t * g_l + head] = from_f<T>(real ? ahead + (lane ? before : 0.f) + through : 0.f);
    }
}

// out (B, L, Hk, D) = sums over neighbouring heads of part (B, H, L, D), head by head so that a token's stride stays small whatever there are of heads
template <class T>
__global__ __launch_bounds__(256) void sum_heads_kernel(const float *part, int L, int H, int Hk, int D, long tokens, T *out, long o_b, long o_l)
{
    const int width = Hk * D, shared = H / Hk;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < tokens * width; i += gridDim.x * 256l) {
        const long tok = i / width;
        const int c = (int)(i % width), hk = c / D, x = c % D;
        const long seq = tok / L, t = tok % L;
        const float *at = part + ((seq * H + (long)hk * shared) * L + t) * D + x;
        float v = at[0];
        for (int j = 1; j < shared; ++j) v += at[(long)j * L * D];
        out[seq * o_b + t * o_l + c] = from_f<T>(v);
    }
}

// ---- single tokens -------------------------------------------------------------------------------------------------
//
// The state is read and written once, 4 bytes an element: memory bounds it (128 sequences of 16 heads of 128 by 128: 57 us, 4.7 TB/s).  A workgroup has 32
// columns of a head's state, 8 lanes of 4 columns to a row.

struct StepParams {
    ucd_linear_attention_t d;
    ucd_linear_attention_in_t in;
    Decays decays;
    float *state;
    void *y;
    int tiles;
};

// WIDE: rows of whole packs of 4, read through a buffer, all of a thread's at once and none under a condition.
template <class T, bool WIDE>
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
    float *s = p.state + ((long)slot * d.H + head) * d.Dk * d.Dv;
    const auto rsrc = buffer_of(s, (uint32_t)(d.Dk * d.Dv) * 4u);
    constexpr int ROWS = 4;      // 128 of them at most
    u32x4 held[WIDE ? ROWS : 1];
    auto place = [&](int j) { return group + 32 * j < d.Dk && have > 0 ? ((group + 32 * j) * d.Dv + x) * 4u : kOut; };
    if (WIDE)
#pragma unroll
        for (int j = 0; j < ROWS; ++j) held[WIDE ? j : 0] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, place(j), 0, 0);
    const Pack<T, 4> v = load_pack<WIDE, T, 4>((const T *)p.in.v + seq * d.v_b + (long)head * d.Dv + x, have);
    const float a = exp_full(p.decays.get<T>(seq, head, 0));
    Pack<float, 4> sum{};
    auto move = [&](Pack<float, 4> &h, float ki, float qi) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            h.v[e] = fmaf(a, h.v[e], ki * to_f(v.v[e]));
            sum.v[e] = fmaf(qi, h.v[e], sum.v[e]);
        }
    };
    if constexpr (WIDE) {
        float ks[ROWS], qs[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            const int i = group + 32 * j, there = min(i, d.Dk - 1);
            ks[j] = to_f(k[there]);
            qs[j] = i < d.Dk ? to_f(q[there]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            auto h = __builtin_bit_cast(Pack<float, 4>, held[j]);
            if (group + 32 * j < d.Dk) move(h, ks[j], qs[j]);      // what is not there may be multiplied to a NaN
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, h), rsrc, place(j), 0, 0);
        }
    } else {
        for (int i = group; i < d.Dk; i += 32) {
            float *at = s + (long)i * d.Dv + x;
            Pack<float, 4> h = have == 4 ? loose_load<float, 4>(at) : load_pack<false, float, 4>(at, have);
            move(h, to_f(k[i]), to_f(q[i]));
            if (have == 4) loose_store<float, 4>(at, h);
            else store_pack<false, float, 4>(at, h, have);
        }
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

// Segments of a walk: as many as fill the card where there are few heads, of one chunk at least.  A segment more is a walk over its keys for its own state.
void segments_of(int B, int L, int H, bool f32, int &segments, int &per)
{
    const long fit = f32 ? 256 : 512;       // workgroups that the card has at once, one or two on a compute unit
    const long have = (long)B * H, chunks = std::max(1, chunks_of(L));
    const long want = std::max(1l, std::min(fit / std::max(1l, have), chunks));
    per = (int)((chunks + want - 1) / want);
    segments = (int)((chunks + per - 1) / per);
}

struct Layout {
    int segments, per;
    size_t starts, decay;
    size_t a, b, all_b, c, keep, heads, bytes;
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
    segments_of(d.B, d.L, d.H, d.dtype == 0, l.segments, l.per);
    const size_t bh = (size_t)d.B * d.H;
    if (l.segments > 1) {
        l.starts = take(l.segments * state_size(d) * 4);
        l.decay = take(l.segments * bh * 4);
    }
    if (dir == UCD_SEQ_BWD) {
        const int cols = cols_of(d.Dv, d.Dk, d.dtype == 0);      // of dq's and dk's walks
        const size_t tiles = tiles_of(d.Dk, cols);
        const size_t planes = tiles * (cols / 32);
        l.a = take(planes * bh * d.L * 4);
        l.b = take(planes * bh * d.L * 4);
        l.all_b = take(planes * bh * d.L * 4);
        l.c = take(tiles * bh * chunks_of(d.L) * 4);
        l.keep = take(tiles * bh * chunks_of(d.L) * cols * (d.Dv > 64 ? 128 : 64) * esize);
        if (d.H != d.Hk) l.heads = take(bh * d.L * d.Dk * 4);
    }
    l.bytes = at;
    return l;
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
    p.out_h = d.Dv;
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
    const Rows out{y, (long)d.y_b, (long)d.y_l, 1, d.Dv};
    return run_mix<T, false>(p, whole_rows<T>(p.q) && whole_rows<T>(p.k) && whole_rows<T>(p.v) && whole_rows<T>(out), s);
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
    // of all together: what one walk keeps the other reads as it lies
    const bool whole = whole_rows<T>(q) && whole_rows<T>(k) && whole_rows<T>(v) && whole_rows<T>(o) &&
                       whole_rows<T>(Rows{grad.q, (long)d.q_b, (long)d.q_l, 1, d.Dk}) && whole_rows<T>(Rows{grad.k, (long)d.k_b, (long)d.k_l, 1, d.Dk}) &&
                       whole_rows<T>(Rows{grad.v, (long)d.v_b, (long)d.v_l, 1, d.Dv});
    hipError_t e;
    // dv, and the gradient of the first state
    Mix p = mix_base(d, in);
    p.q = k;
    p.k = q;
    p.v = o;
    p.out = grad.v;
    p.out_b = d.v_b;
    p.out_h = d.Dv;
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
    if ((e = run_mix<T, true>(p, whole, s)) != hipSuccess) return e;
    // dq: Forward's states, transposed, from those that it kept at the segments' starts on
    Mix a = mix_base(d, in);
    a.q = o;
    a.k = v;
    a.v = k;
    a.dot = q;
    a.p_scale = a.first_scale = d.scale;
    a.last_scale = 1.f;
    a.s_row = 1;
    a.s_col = d.Dv;
    a.segments = l.segments;
    a.per_segment = l.per;
    a.starts = const_cast<float *>(saved);
    a.started = true;
    a.dots = decays ? (float *)(ws + l.a) : nullptr;
    a.chunk_states = ws + l.keep;
    a.passes = (float *)(ws + l.c);
    auto heads = [&](Mix &m, void *out, long o_b, long o_l, bool rev) {
        m.out_f32 = shared > 1;
        m.out = shared > 1 ? ws + l.heads : out;
        m.out_l = shared > 1 ? d.Dk : o_l;
        m.out_h = shared > 1 ? (long)d.L * d.Dk : d.Dk;
        m.out_b = shared > 1 ? d.H * m.out_h : o_b;
        const hipError_t e = rev ? run_mix<T, true>(m, whole, s) : run_mix<T, false>(m, whole, s);
        if (shared == 1) return e;
        const long tokens = (long)d.B * d.L;
        if (e != hipSuccess || tokens == 0) return e;
        const unsigned grid = (unsigned)std::min((tokens * d.Hk * d.Dk + 255) / 256, 1l << 16);
        sum_heads_kernel<T><<<grid, 256, 0, s>>>((const float *)(ws + l.heads), d.L, d.H, d.Hk, d.Dk, tokens, (T *)out, o_b, o_l);
        return hipGetLastError();
    };
    if ((e = heads(a, grad.q, d.q_b, d.q_l, false)) != hipSuccess) return e;
    Mix b = a;
    b.q = v;
    b.k = o;
    b.v = q;
    b.dot = k;
    b.p_scale = b.last_scale = d.scale;
    b.first_scale = 1.f;
    // dk: dv's states, transposed
    b.state_in = dstate_out;
    b.starts = p.starts;
    b.dots = decays ? (float *)(ws + l.all_b) : nullptr;
    b.state_dots = (float *)(ws + l.b);
    if ((e = heads(b, grad.k, d.k_b, d.k_l, true)) != hipSuccess) return e;
    if (!decays || d.L == 0) return hipSuccess;
    const unsigned grid = (unsigned)std::min((long)d.B * d.H * chunks_of(d.L), 1l << 20);
    const int planes = b.tiles * (cols_of(d.Dv, d.Dk, d.dtype == 0) / 32);
    decay_gradient_kernel<T><<<grid, 64, 0, s>>>(a.dots, b.dots, b.state_dots, a.passes, planes, b.tiles, d.B, d.L, d.H, in.lengths, a.decays,
                                                 (T *)grad.g, d.g_b, d.g_l);
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
    return (double)d.B * d.H * std::max({tiles_of(d.Dk, 32), tiles_of(d.Dv, 32), chunks_of(d.L)}) < 1 << 23;
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
    const bool wide = d.Dv % 4 == 0;
    if (d.dtype == 1) wide ? attention_step_kernel<bf16_t, true><<<grid, 256, 0, s>>>(p) : attention_step_kernel<bf16_t, false><<<grid, 256, 0, s>>>(p);
    else wide ? attention_step_kernel<float, true><<<grid, 256, 0, s>>>(p) : attention_step_kernel<float, false><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace ucd
