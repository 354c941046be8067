// Linear attention's walk over the chunks of sequences (linear_attention.hip has the formulas): its kernel and launches.
#pragma once
#include <algorithm>

#include "linear_attention.hpp"

namespace ucd {
namespace attention {

// Places of a launch: column tile, head, segment, sequence.  Column tiles of a head are neighbours that share q and k.
struct Place {
    int tile, head, seq, segment;
};
__device__ __forceinline__ Place place_of(const Mix &p, int segments)
{
    unsigned i = xcd_place();
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

// DK: q's width, 64 or 128; COLS: the state's columns that a workgroup has, 64 or 128, 32 to a wave.  WHOLE: of rows (Fetch).
//
// A wave has its columns of the state as sums of the matrix instructions, DK rows of them, and uses those sums as they lie as an operand of q S: the
// reduction runs over the state's rows in the order in which the sums hold them, for q too, so that the state never goes through LDS.  v is
// weighted for the state's update, each wave its own columns, which stay in registers for the pairs' products.  Two barriers a chunk: behind the tiles,
// and behind the pairs, which the waves share out.  16-bit tensors have their pairs' weights, and the state where it is an operand, rounded to 16 bits: that
// is what their matrix instructions take, and errors grow from the output's own 1.7e-3 to 2.4e-3 in the 2-norm.  Memory bounds it, 16 bits, at two workgroups
// to a compute unit: 8 x 2048 tokens of 16 heads of 128, Forward 78 us for 270 MB, dv 73, dq and dk, with the decays' gradient, 113 and 128 for 470 MB each.
// fp32 is bound by its matrix instructions.
template <class T, int DK, int COLS, bool REV, int FOR, bool WHOLE, bool OUT32>
__global__ __launch_bounds__(2 * COLS, sizeof(T) == 2 && (COLS == 128 || DK == 64) ? 2 : 1) void mix_kernel(Mix p)
{
    constexpr int THREADS = 2 * COLS, WAVES = COLS / 32;
    constexpr bool OUT = FOR != STATES, DG = FOR == DECAYS;
    constexpr int PARTS = sizeof(T) == 4 ? 1 : 3;        // of what is added to a state: as exact as its 32 bits, whoever reads it
    typedef Mma<T> M;
    typedef TileLds<T, DK> TQ;
    typedef TileLds<T, COLS> TV;
    typedef TileLds<T, kChunk> TP;
    constexpr int ST = DK / 32, KS = kChunk / M::K;      // tiles of a wave's state, 32 by 32; reduction steps over a chunk's tokens
    __shared__ __attribute__((aligned(16))) char lds_q[OUT ? TQ::BYTES : 16], lds_k[TQ::BYTES], lds_v[TV::BYTES], lds_p[OUT ? TP::BYTES : 16];
    __shared__ ChunkDecays decays[2];
    __shared__ float lds_pass[WAVES];
    // a wave's outputs on their way to rows: 32 rows of 64 bytes (and what they are multiplied with from rows).  Stored from the sums as they lie, 16 bytes
    // each of 32 rows, they took 2900 cycles of a chunk's 13000
    constexpr int TURN_ROW = 80;
    __shared__ __attribute__((aligned(16))) char lds_turn[OUT ? WAVES * 32 * TURN_ROW : 16];
    const Place at = place_of(p, OUT ? p.segments : p.segments - 1);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), row = lane % 32, half = lane / 32;
    const int col0 = at.tile * COLS, cols = min(COLS, p.v.width - col0);
    const int n = p.lengths ? max(0, min(p.L, p.lengths[at.seq])) : p.L;
    const int slot = p.slots ? p.slots[at.seq] : at.seq;
    const bool idle = p.slots && (slot < 0 || slot >= p.n_slots);
    const int chunks = (p.L + kChunk - 1) / kChunk;
    const int c0 = at.segment * p.per_segment, c1 = min(chunks, c0 + p.per_segment);       // in walking order
    // a chunk's first token, and the token of one of its rows
    auto token0 = [&](int chunk) { return (REV ? chunks - 1 - chunk : chunk) * kChunk; };
    auto token = [&](int chunk, int r) { return token0(chunk) + (REV ? kChunk - 1 - r : r); };
    constexpr int osize = OUT32 ? 4 : (int)sizeof(T);      // fp32 outputs are parts that are summed up over the heads that share a row
    static_assert(!OUT32 || sizeof(T) == 2, "");
    const long o_l = p.out_l * osize;
    char *out = (char *)p.out + (at.seq * p.out_b + at.head * p.out_h + col0) * osize;

    if (idle) {
        for (int c = c0; c < c1 && OUT; ++c)
            for (int i = threadIdx.x; i < kChunk * COLS; i += THREADS) {
                const int t = token(c, i / COLS), x = i % COLS;
                if (t < p.L && x < cols) *(T *)(out + t * o_l + x * osize) = from_f<T>(0.f);
            }
        return;
    }

    // sum r of tile i: row 32 i + 8 (r / 4) + 4 half + r % 4, column x0 + lane % 32
    const int x0 = wave * 32;
    auto state_at = [&](int i, int r) {      // its place in a head's state, in bytes
        const int y = 32 * i + 8 * (r / 4) + 4 * half + r % 4, x = x0 + row;
        return y < p.q.width && x < cols ? 4u * (uint32_t)(y * (int)p.s_row + (col0 + x) * (int)p.s_col) : kOut;
    };
    f32x16 state[ST];
#pragma unroll
    for (int i = 0; i < ST; ++i) state[i] = f32x16{};
    if (OUT) {
        const float *from = p.starts ? p.starts + (((long)at.segment * p.B + at.seq) * p.H + at.head) * p.s_head
                                     : p.state_in ? p.state_in + ((long)slot * p.H + at.head) * p.s_head : nullptr;
        // through a buffer: all loads at once, none waited for under a condition
        const auto rsrc = buffer_of(from, from ? (uint32_t)p.s_head * 4u : 0u);
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) state[i][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, state_at(i, r), 0, 0));
    }

    Fetch<T, DK, WHOLE, THREADS> fq, fk;
    Fetch<T, COLS, WHOLE, THREADS> fv;
    const long q_l = p.q.l * sizeof(T), k_l = p.k.l * sizeof(T), v_l = p.v.l * sizeof(T);
    const T *qp = p.q.template at<T>(at.seq, at.head), *kp = p.k.template at<T>(at.seq, at.head), *vp = p.v.template at<T>(at.seq, at.head) + col0;
    if (OUT) fq.init(p.q.width, q_l, REV);
    fk.init(p.k.width, k_l, REV);
    fv.init(cols, v_l, REV);
    // of a chunk that is none nothing is read: loads and stores are the same ones for every chunk, so that a load's data is waited for without the stores
    // behind it
    auto fetch_q = [&](int chunk) {
        const long t = token0(chunk);
        fq.load((const char *)qp + t * q_l, q_l, chunk < c1 ? n - (int)t : 0);
    };
    auto fetch = [&](int chunk, bool all) {
        const long t = token0(chunk);
        const int there = chunk < c1 ? n - (int)t : 0;
        fk.load((const char *)kp + t * k_l, k_l, there);
        fv.load((const char *)vp + t * v_l, v_l, there);
        if (OUT && all) fetch_q(chunk);
    };
    // the first wave sets the decays of the chunk that comes; those of the one behind it are on their way
    uint32_t raw_decay = 0;
    const float head_decay = p.decays.decay ? p.decays.decay[at.head] : 0.f;
    auto fetch_decay = [&](int chunk) {
        const int t = token0(chunk) + (REV ? 1 : 0);
        raw_decay = p.decays.raw<T>(at.seq, at.head, t, chunk < c1 ? n - t : 0, REV);
    };
    auto set_decays = [&](int chunk) {
        const int t = token(chunk, lane) + (REV ? 1 : 0);
        if (wave == 0) decays[chunk & 1].set(t < n ? Decays::sum<T>(head_decay, raw_decay) : 0.f, p.first_scale, p.last_scale);
        fetch_decay(chunk + 1);
    };
    double segment_decay = 0;
    char *turn = lds_turn + (OUT ? wave * 32 * TURN_ROW : 0);
    // a lane's piece of the rows in `turn`: of row 16 i + lane / 4, 16 bytes
    const int turn_row = lane / 4, turn_at = lane % 4 * 16;
    // states at the chunks' starts, as the operands that they are: a workgroup's threads side by side
    typedef typename M::Frag Frag;
    constexpr int PIECES = DK / M::K;
    auto kept = [&](int c) {
        const long chunk = REV ? chunks - 1 - c : c;
        return (Frag *)p.chunk_states + ((((long)at.seq * p.H + at.head) * p.tiles + at.tile) * chunks + chunk) * (PIECES * THREADS) + threadIdx.x;
    };
    const long d_l = DG ? p.dot.l * (long)sizeof(T) : 0;
    const T *dp = DG ? p.dot.template at<T>(at.seq, at.head) + col0 : nullptr;
    // Dots of the outputs with rows of `dot` (what the output is the gradient of), for the decays' gradient: rows' pieces of 16 bytes, and the sums over a
    // wave's columns, one plane for each.  A second read of the pieces, from the cache, costs less than their registers.
    constexpr int DOT_PASSES = (int)sizeof(T) / 2, DOT_COLS = 64 / (int)sizeof(T), DOT_PER = 16 / (int)sizeof(T);
    u32x4 dots[DG ? 2 : 1][DG ? DOT_PASSES : 1][DG ? 2 : 1];
    auto load_dots = [&](long tok0, int tb) {
        const auto rsrc = buffer_of((const char *)dp + tok0 * d_l, chunk_bytes(d_l, n - (int)tok0));
#pragma unroll
        for (int pass = 0; pass < DOT_PASSES; ++pass)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = 32 * tb + 16 * i + turn_row, t_at = REV ? kChunk - 1 - t : t;
                const int x = x0 + pass * DOT_COLS + lane % 4 * DOT_PER, have = cols - x;
                const uint32_t o = (uint32_t)(t_at * d_l) + x * (uint32_t)sizeof(T);
                u32x4 &d = dots[DG ? tb : 0][DG ? pass : 0][DG ? i : 0];
                if (WHOLE) {
                    d = __builtin_amdgcn_raw_buffer_load_b128(rsrc, have > 0 ? o : kOut, 0, 0);
                } else {
                    Pack<T, DOT_PER> v;
#pragma unroll
                    for (int e = 0; e < DOT_PER; ++e) {
                        if constexpr (sizeof(T) == 4) v.v[e] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rsrc, e < have ? o + 4 * e : kOut, 0, 0));
                        else v.v[e] = __builtin_bit_cast(T, (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, e < have ? o + 2 * e : kOut, 0, 0));
                    }
                    d = __builtin_bit_cast(u32x4, v);
                }
            }
    };
    auto put_dots = [&](int tb, int pass) {
#pragma unroll
        for (int i = 0; i < 2; ++i) lds_put(turn + (16 * i + turn_row) * TURN_ROW + turn_at, dots[DG ? tb : 0][DG ? pass : 0][DG ? i : 0]);
        wave_lds_order();
    };
    // of rows 32 tb + 0 .. 31; `there`: their first pass is in `turn` already
    auto dot = [&](float *to, int c, int tb, const f32x16 &y, bool there) {
        float sum = 0.f;
#pragma unroll
        for (int pass = 0; pass < DOT_PASSES; ++pass) {
            if (!there || pass) put_dots(tb, pass);
            constexpr int QUADS = 4 / DOT_PASSES;
#pragma unroll
            for (int r = 0; r < QUADS; ++r) {
                const auto v = lds_get<Pack<T, 4>>(turn + row * TURN_ROW + (8 * r + 4 * half) * (int)sizeof(T));
#pragma unroll
                for (int e = 0; e < 4; ++e) sum = fmaf(to_f(v.v[e]), y[4 * (pass * QUADS + r) + e], sum);
            }
            wave_lds_order();
        }
        float other = sum;
        swap_halves(sum, other);
        sum += other;
        const int t = token(c, 32 * tb + row);
        if (half == 0 && t < p.L) to[(((long)(at.tile * WAVES + wave) * p.B + at.seq) * p.H + at.head) * p.L + t] = sum;
    };
    // A token's pair with itself crosses no decay and may be all there is beside the rest: outputs get it behind the dots.  Elements of step k of it, or
    // all others.
    auto diagonal = [&](const Frag &f, int k, bool its) {
        constexpr int WORDS = sizeof(Frag) / 4, PER = 4 / (int)sizeof(T), E = M::K / 2;
        struct Words {
            uint32_t w[WORDS];
        };
        Words v = __builtin_bit_cast(Words, f);
        const int d = row - k * M::K % 32 - half * E;
#pragma unroll
        for (int i = 0; i < WORDS; ++i) {
            const uint32_t of = PER == 2 ? 0xffffu << (d & 1) * 16 : 0xffffffffu, mask = (PER == 2 ? d >> 1 : d) == i ? of : 0u;
            v.w[i] &= its ? mask : ~mask;
        }
        return __builtin_bit_cast(Frag, v);
    };
    if (c0 < c1) {
        fetch_decay(c0);
        set_decays(c0);
        fetch(c0, true);
    }
    for (int c = c0; c < c1; ++c) {
        const ChunkDecays &dec = decays[c & 1];
        const long tok0 = token0(c);
        fk.store(lds_k, (const char *)kp + tok0 * k_l);
        fv.store(lds_v, (const char *)vp + tok0 * v_l);
        if (OUT) fq.template store<M::SUMS_ORDER>(lds_q, (const char *)qp + tok0 * q_l);
        lds_barrier();
        if (!OUT) fetch(c + 1, true);
        Frag before[DG && REV ? PIECES : 1];
        if (DG && REV) {
            const Frag *from = kept(c);
#pragma unroll
            for (int i = 0; i < PIECES; ++i) before[DG && REV ? i : 0] = from[i * THREADS];
        }
        if (DG) load_dots(tok0, 1);
        if (DG && REV) load_dots(tok0, 0);
        set_decays(c + 1);
        // Operands are read in batches ahead of their products: one by one each product would wait for its own.
        if (OUT) {
            // P[t, s] in tiles of 16 by 16: a lane has row t and 4 s.  A wave has a row of tiles of four, or two of them
            constexpr int NK = DK / M::K16, BATCH = sizeof(T) == 2 ? 2 : 1;      // tiles at a time
            constexpr bool BOTH = DG || sizeof(T) == 4;                          // floats of the sums of decays
#pragma unroll
            for (int part = 0; part < 4 / WAVES; ++part) {
                const int tb = (part ? 3 - wave : wave) * 16, t = tb + lane % 16;
                Frag fragq[NK];
#pragma unroll
                for (int k = 0; k < NK; ++k) fragq[k] = M::template along16<DK>(lds_q, tb, k * M::K16);
                const float hi = dec.hi[t], lo = dec.lo[t];
#pragma unroll
                for (int sb = 0; sb < kChunk; sb += 16 * BATCH) {
                    Frag fragk[BATCH][NK];
                    Pack<float, 4> shi[BATCH], slo[BOTH ? BATCH : 1];
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
#pragma unroll
                        for (int k = 0; k < NK; ++k) fragk[i][k] = M::template along16_other<DK>(lds_k, sb + 16 * i, k * M::K16);
                        const int s = sb + 16 * i + 4 * (lane / 16);
                        shi[i] = ChunkDecays::four(dec.hi + s);
                        if (BOTH) slo[BOTH ? i : 0] = ChunkDecays::four(dec.lo + s);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    f32x4 acc[BATCH] = {};
#pragma unroll
                    for (int k = 0; k < NK; ++k)
#pragma unroll
                        for (int i = 0; i < BATCH; ++i) acc[i] = M::product16(fragk[i][k], fragq[k], acc[i]);
#pragma unroll
                    for (int i = 0; i < BATCH; ++i) {
                        const int s = sb + 16 * i + 4 * (lane / 16);
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float w = ChunkDecays::pair<T, DG>(hi, lo, shi[i].v[e], BOTH ? slo[BOTH ? i : 0].v[e] : 0.f) * p.p_scale;
                            v[e] = s + e <= t ? acc[i][e] * w : 0.f;
                        }
                        lds_put(lds_p + TP::at(t, s), pack_four<T>(v[0], v[1], v[2], v[3]));
                    }
                }
            }
        }
        // outputs' part of the state: a lane has rows t and 16 columns
        f32x16 y[2] = {};
        if (OUT) {
            float pass = 0.f;
            constexpr int BATCH = DG && REV ? 2 : 4;      // steps at a time; registers are missing for more where the states before are there, too
            Frag fragq[2][BATCH][2];
            auto read = [&](int k) {
#pragma unroll
                for (int i = 0; i < BATCH; ++i)
#pragma unroll
                    for (int tb = 0; tb < 2; ++tb) fragq[k / BATCH % 2][i][tb] = M::template along<DK>(lds_q, 32 * tb, (k + i) * M::K);
            };
            read(0);
#pragma unroll
            for (int kb = 0; kb < DK / M::K; kb += BATCH) {
                if (kb + BATCH < DK / M::K) read(kb + BATCH);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < BATCH; ++i) {
                    const int k = (kb + i) * M::K, first = k % 32 / 16 * 8 + (M::K == 8 ? k % 16 / 8 * 4 : 0);
                    const f32x16 &s = state[k / 32];
                    const Frag f = M::from_sums(s, first);
                    y[0] = M::product(f, fragq[kb / BATCH % 2][i][0], y[0]);
                    y[1] = M::product(f, fragq[kb / BATCH % 2][i][1], y[1]);
                    if (DG && !REV) kept(c)[(kb + i) * THREADS] = f;
                    if (DG && REV) {
                        const auto values = __builtin_bit_cast(Pack<T, M::SUMS>, before[DG && REV ? kb + i : 0]);
#pragma unroll
                        for (int e = 0; e < M::SUMS; ++e) pass = fmaf(to_f(values.v[e]), s[first + e], pass);
                    }
                }
            }
            if (DG && REV) {
                pass = sum_group(pass, 64);
                if (lane == 0) lds_pass[wave] = pass;
            }
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const float first = dec.first[32 * tb + row];
#pragma unroll
                for (int r = 0; r < 16; ++r) y[tb][r] *= first;
                if (DG && REV) dot(p.state_dots, c, tb, y[tb], false);
            }
        }
        if (DG) {      // for what comes behind the pairs: rows 32 .. 63 wait in LDS (16 bits: there they are, if those behind the state were just multiplied)
            if (!REV || DOT_PASSES > 1) put_dots(1, 0);
            load_dots(tok0, 0);
        }
        // the state behind the chunk
        const float whole = dec.whole;
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) state[i][r] *= whole;
        Frag own[KS];
        {
            constexpr int E = M::K / 2;
            Frag a[2][ST];
            Pack<float, 4> w[2][E / 4];
            auto read = [&](int k) {
                own[k] = M::template across<COLS>(lds_v, x0, k * M::K);
#pragma unroll
                for (int e = 0; e < E / 4; ++e) w[k % 2][e] = ChunkDecays::four(dec.last + k * M::K + half * E + 4 * e);
#pragma unroll
                for (int i = 0; i < ST; ++i) a[k % 2][i] = M::template across<DK>(lds_k, 32 * i, k * M::K);
            };
            read(0);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if (k + 1 < KS) read(k + 1);
                __builtin_amdgcn_sched_barrier(0);
                float weights[E];
#pragma unroll
                for (int e = 0; e < E; ++e) weights[e] = w[k % 2][e / 4].v[e % 4];
                Frag b[PARTS];
                M::template weighted<PARTS>(own[k], weights, b);
#pragma unroll
                for (int e = PARTS; e-- > 0;)
#pragma unroll
                    for (int i = 0; i < ST; ++i) state[i] = M::product(a[k % 2][i], b[e], state[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (OUT) fetch(c + 1, !DG);      // not before: its registers would be missing above
        if (!OUT && threadIdx.x < 64) segment_decay += (double)dec.hi[63] + (double)dec.lo[63];
        lds_barrier();
        if (OUT) {
            Frag pairs[KS + KS / 2];      // of rows 32 .. 63, then of the others
#pragma unroll
            for (int k = 0; k < KS; ++k) pairs[k] = M::template along<kChunk>(lds_p, 32, k * M::K);
#pragma unroll
            for (int k = 0; k < KS / 2; ++k) pairs[KS + k] = M::template along<kChunk>(lds_p, 0, k * M::K);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                y[1] = M::product(own[k], DG && k >= KS / 2 ? diagonal(pairs[k], k, false) : pairs[k], y[1]);
                if (k < KS / 2) y[0] = M::product(own[k], DG ? diagonal(pairs[KS + k], k, false) : pairs[KS + k], y[0]);
            }
            if (DG) {
#pragma unroll
                for (int tb = 2; tb-- > 0;) dot(p.dots, c, tb, y[tb], tb == 1);
                fetch_q(c + 1);
#pragma unroll
                for (int k = 0; k < KS; ++k) {      // read again: registers are missing
                    const int tb = k / (KS / 2);
                    y[tb] = M::product(own[k], diagonal(M::template along<kChunk>(lds_p, 32 * tb, k * M::K), k, true), y[tb]);
                }
            }
#pragma unroll
            for (int tb = 0; tb < 2; ++tb) {
                const auto rsrc = buffer_of(out + tok0 * o_l, chunk_bytes(o_l, p.L - (int)tok0));
                const int t = 32 * tb + row, t_at = REV ? kChunk - 1 - t : t;
                const bool real = t_at < n - (int)tok0;
#pragma unroll
                for (int r = 0; r < 16; ++r) y[tb][r] = real ? y[tb][r] : 0.f;
                constexpr int PASSES = osize / 2, QUADS = 4 / PASSES, PER = 16 / osize;
#pragma unroll
                for (int pass = 0; pass < PASSES; ++pass) {
#pragma unroll
                    for (int r = 0; r < QUADS; ++r) {
                        const int q = 4 * (pass * QUADS + r);
                        char *to = turn + row * TURN_ROW + (8 * r + 4 * half) * osize;
                        if constexpr (osize == 4) lds_put(to, pack_four<float>(y[tb][q], y[tb][q + 1], y[tb][q + 2], y[tb][q + 3]));
                        else lds_put(to, pack_four<T>(y[tb][q], y[tb][q + 1], y[tb][q + 2], y[tb][q + 3]));
                    }
                    wave_lds_order();
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const u32x4 v = lds_get<u32x4>(turn + (16 * i + turn_row) * TURN_ROW + turn_at);
                        const int tr = 32 * tb + 16 * i + turn_row, tr_at = REV ? kChunk - 1 - tr : tr;
                        const int x = x0 + pass * (64 / osize) + lane % 4 * PER, have = cols - x;
                        const uint32_t o = (uint32_t)(tr_at * o_l) + x * osize;
                        if (WHOLE) {
                            __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, have > 0 ? o : kOut, 0, 0);
                        } else if constexpr (osize == 4) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) __builtin_amdgcn_raw_buffer_store_b32(v[e], rsrc, e < have ? o + 4 * e : kOut, 0, 0);
                        } else {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(v[e / 2] >> (e % 2 * 16)), rsrc, e < have ? o + 2 * e : kOut, 0, 0);
                        }
                    }
                    wave_lds_order();
                }
            }
            if (DG && REV && threadIdx.x == 64) {
                const int chunk = chunks - 1 - c;
                const float first = chunk * kChunk < n ? p.decays.get<T>(at.seq, at.head, (long)chunk * kChunk) : 0.f;
                float all = lds_pass[0];
#pragma unroll
                for (int i = 1; i < WAVES; ++i) all += lds_pass[i];
                p.passes[(((long)at.tile * p.B + at.seq) * p.H + at.head) * chunks + chunk] = whole * exp_full(first) * all;
            }
        }
    }

    float *to = nullptr;
    float factor = 1.f;
    if (!OUT) {
        to = p.starts + ((((long)at.segment + 1) * p.B + at.seq) * p.H + at.head) * p.s_head;
        if (threadIdx.x == 0 && at.tile == 0) p.segment_decay[((long)at.segment * p.B + at.seq) * p.H + at.head] = exp2_fast((float)segment_decay);
    } else if (p.state_out && at.segment == p.segments - 1) {
        to = p.state_out + ((long)slot * p.H + at.head) * p.s_head;
        if (REV && n > 0) factor = exp_full(p.decays.get<T>(at.seq, at.head, 0));
    }
    if (to) {
        const auto rsrc = buffer_of(to, (uint32_t)p.s_head * 4u);
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(REV && OUT ? state[i][r] * factor : state[i][r]), rsrc, state_at(i, r), 0, 0);
    }
}

// ---- launches ------------------------------------------------------------------------------------------------------

template <class T, int DK, int COLS, bool REV, bool WHOLE>
hipError_t run_mix_of(const Mix &p, hipStream_t s)
{
    const unsigned groups = (unsigned)((long)p.B * p.H * p.tiles);
    if (p.segments > 1 && !p.started) {
        mix_kernel<T, DK, COLS, REV, STATES, WHOLE, false><<<groups * (p.segments - 1), 2 * COLS, 0, s>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (p.starts && !p.started) {      // also of one segment, where Forward keeps the state that it begins with
        const hipError_t e = join_states(p, s);
        if (e != hipSuccess) return e;
    }
    const unsigned grid = groups * p.segments;
    if (sizeof(T) == 2 && p.out_f32) {
        if constexpr (sizeof(T) == 2) {
            if (p.dots) mix_kernel<T, DK, COLS, REV, DECAYS, WHOLE, true><<<grid, 2 * COLS, 0, s>>>(p);
            else mix_kernel<T, DK, COLS, REV, OUTPUTS, WHOLE, true><<<grid, 2 * COLS, 0, s>>>(p);
        }
    } else if (p.dots) mix_kernel<T, DK, COLS, REV, DECAYS, WHOLE, false><<<grid, 2 * COLS, 0, s>>>(p);
    else mix_kernel<T, DK, COLS, REV, OUTPUTS, WHOLE, false><<<grid, 2 * COLS, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, bool REV>
hipError_t run_mix(Mix &p, bool whole, hipStream_t s)
{
    const int cols = cols_of(p.q.width, p.v.width, sizeof(T) == 4);
    p.tiles = tiles_of(p.v.width, cols);
    const bool wide = p.q.width > 64;
    if (cols == 128) {
        if (whole) return wide ? run_mix_of<T, 128, 128, REV, true>(p, s) : run_mix_of<T, 64, 128, REV, true>(p, s);
        return wide ? run_mix_of<T, 128, 128, REV, false>(p, s) : run_mix_of<T, 64, 128, REV, false>(p, s);
    }
    if constexpr (sizeof(T) == 2)
        if (wide) return whole ? run_mix_of<T, 128, 64, REV, true>(p, s) : run_mix_of<T, 128, 64, REV, false>(p, s);
    return whole ? run_mix_of<T, 64, 64, REV, true>(p, s) : run_mix_of<T, 64, 64, REV, false>(p, s);
}

}  // namespace attention
}  // namespace ucd
