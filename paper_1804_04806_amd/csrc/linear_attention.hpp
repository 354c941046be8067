// What the linear attention's kernels share: tiles of 64 tokens in LDS, their products, decays.
#pragma once
#include <cstddef>

#include "piece_words.hpp"
#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace attention {
using namespace seq;

constexpr int kChunk = 64;      // tokens of a chunk
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// exp(-80) is as good as 0, and sums of 64 of them and their differences stay finite: what is below counts as -80.  A NaN stays one.
constexpr float kLeast = -80.f;

// A tile of rows of COLS elements in LDS.  Rows are 16 bytes longer than their elements and stand, 16 at a time, in an order of their own: 16 lanes that
// read 16 bytes each of 16 rows meet no bank twice (rows are an odd number of 16 bytes apart), and neither do transposing reads of 4 neighbouring rows by 64
// bytes (those rows are 64 bytes apart modulo 256).  An address is a lane's own plus a constant.
template <class T, int COLS>
struct TileLds {
    static constexpr int PER = 16 / sizeof(T), CELLS = COLS / PER, ROW = COLS * (int)sizeof(T) + 16, BYTES = kChunk * ROW;
    static constexpr int STEP = ROW / 16 % 16;                  // of rows, in 16 bytes modulo 256
    static_assert(STEP == 1 || STEP == 9, "its own inverse modulo 16");
    __device__ static __forceinline__ int place(int r) { return (r & ~15) | ((STEP * ((r & 3) << 2 | (r >> 2 & 3))) & 15); }
    __device__ static __forceinline__ int cell(int r, int c) { return place(r) * ROW + c * 16; }
    __device__ static __forceinline__ int at(int r, int col) { return place(r) * ROW + col * (int)sizeof(T); }
};

// Operands of v_mfma_f32_32x32: K reduction steps of a fragment; lanes 0-31 have the first half of them, lanes 32-63 the second, row lane % 32.
template <class T> struct Mma;

// Two values, rounded, as words of two; an instruction of its own, because the compiler turns the widening of one half into a second conversion.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(r) : "v"(lo), "v"(hi));
    return r;
}
template <class T> __device__ __forceinline__ Pack<T, 4> pack_four(float a, float b, float c, float d);
template <> __device__ __forceinline__ Pack<float, 4> pack_four<float>(float a, float b, float c, float d) { return Pack<float, 4>{{a, b, c, d}}; }
template <> __device__ __forceinline__ Pack<bf16_t, 4> pack_four<bf16_t>(float a, float b, float c, float d)
{
    struct Two {
        uint32_t w[2];
    };
    return __builtin_bit_cast(Pack<bf16_t, 4>, Two{{pack_bf16(a, b), pack_bf16(c, d)}});
}

template <> struct Mma<bf16_t> {
    static constexpr int K = 16;
    typedef bf16x8 Frag;
    // rows first .. first + 31 of a tile, reduction along its rows
    template <int COLS>
    __device__ static __forceinline__ Frag along(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        return lds_get<Frag>(tile + TileLds<bf16_t, COLS>::cell(lane % 32, lane / 32) + first * TileLds<bf16_t, COLS>::ROW + k0 * 2);
    }
    // sums i, i + 1, ... of a tile of them as an operand: lanes 0-31 have rows 0 .. 3 and 8 .. 11 of 16, lanes 32-63 rows 4 .. 7 and 12 .. 15.  What is
    // multiplied with them is stored in that order (SUMS_ORDER): 8, 8, 8 and 8 bytes of 32 as 0, 2, 1, 3
    __device__ static __forceinline__ Frag from_sums(const f32x16 &s, int i)
    {
        struct Words {
            uint32_t w[4];
        };
        return __builtin_bit_cast(Frag, Words{{pack_bf16(s[i], s[i + 1]), pack_bf16(s[i + 2], s[i + 3]), pack_bf16(s[i + 4], s[i + 5]), pack_bf16(s[i + 6], s[i + 7])}});
    }
    static constexpr int SUMS = 8;      // of an operand
    static constexpr bool SUMS_ORDER = true;
    // columns first .. first + 31, reduction over rows from k0 on: 16 lanes fetch 4 rows of 16 columns each and get 4 rows of a column each
    template <int COLS>
    __device__ static __forceinline__ Frag across(const char *tile, int first, int k0)
    {
        typedef TileLds<bf16_t, COLS> Tile;
        const int lane = threadIdx.x % 64, col = lane / 16 % 2 * 16 + lane % 4 * 4, k = lane / 32 * 8 + lane % 16 / 4;
        const char *p = tile + k0 * Tile::ROW + first * 2;
        typedef __attribute__((address_space(3))) s16x4 lds_t;
        struct Both {
            s16x4 lo, hi;
        } v;
        v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + Tile::at(k, col)));
        v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + Tile::at(k + 4, col)));
        return __builtin_bit_cast(Frag, v);
    }
    __device__ static __forceinline__ f32x16 product(const Frag &a, const Frag &b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // 16 rows by 32 steps, and their product: row lane % 16, steps 8 (lane / 16) + 0 .. 7
    static constexpr int K16 = 32;
    template <int COLS>
    __device__ static __forceinline__ Frag along16(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        return lds_get<Frag>(tile + TileLds<bf16_t, COLS>::cell(lane % 16, lane / 16) + first * TileLds<bf16_t, COLS>::ROW + k0 * 2);
    }
    // those steps of a tile in its own order that along16 gives of one in the sums'
    template <int COLS>
    __device__ static __forceinline__ Frag along16_other(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64, g = lane / 16;
        const char *p = tile + TileLds<bf16_t, COLS>::cell(lane % 16, g / 2 * 2) + g % 2 * 8 + first * TileLds<bf16_t, COLS>::ROW + k0 * 2;
        struct Both {
            s16x4 lo, hi;
        } v;
        v.lo = lds_get<s16x4>(p);
        v.hi = lds_get<s16x4>(p + 16);
        return __builtin_bit_cast(Frag, v);
    }
    __device__ static __forceinline__ f32x4 product16(const Frag &a, const Frag &b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
    // w a in PARTS bfloat16 parts, the largest first: three are as exact as the sums' 32 bits
    template <int PARTS>
    __device__ static __forceinline__ void weighted(const Frag &a, const float *w, Frag (&out)[PARTS])
    {
        struct Words {
            uint32_t w[4];
        };
        const Words x = __builtin_bit_cast(Words, a);
        Words part[PARTS];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo = __uint_as_float(x.w[i] << 16) * w[2 * i], hi = __uint_as_float(x.w[i] & 0xFFFF0000u) * w[2 * i + 1];
#pragma unroll
            for (int e = 0; e < PARTS; ++e) {
                const uint32_t r = pack_bf16(lo, hi);
                part[e].w[i] = r;
                if (e + 1 < PARTS) {
                    lo -= __uint_as_float(r << 16);
                    hi -= __uint_as_float(r & 0xFFFF0000u);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < PARTS; ++e) out[e] = __builtin_bit_cast(Frag, part[e]);
    }
};

template <> struct Mma<float> {
    static constexpr int K = 8;
    typedef Pack<float, 4> Frag;
    template <int COLS>
    __device__ static __forceinline__ Frag along(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        return lds_get<Frag>(tile + TileLds<float, COLS>::cell(lane % 32, lane / 32) + first * TileLds<float, COLS>::ROW + k0 * 4);
    }
    template <int COLS>
    __device__ static __forceinline__ Frag along16_other(const char *tile, int first, int k0) { return along16<COLS>(tile, first, k0); }
    __device__ static __forceinline__ Frag from_sums(const f32x16 &s, int i) { return Frag{{s[i], s[i + 1], s[i + 2], s[i + 3]}}; }
    static constexpr int SUMS = 4;
    static constexpr bool SUMS_ORDER = false;
    template <int COLS>
    __device__ static __forceinline__ Frag across(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        Frag v;
#pragma unroll
        for (int i = 0; i < 4; ++i)      // row 4 (lane / 32) + i of 8, from k0, of which there may be an odd number in 16
            v.v[i] = lds_get<float>(tile + TileLds<float, COLS>::at(k0 % 16 + lane / 32 * 4 + i, lane % 32) + k0 / 16 * 16 * TileLds<float, COLS>::ROW + first * 4);
        return v;
    }
    __device__ static __forceinline__ f32x16 product(const Frag &a, const Frag &b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
    static constexpr int K16 = 16;
    template <int COLS>
    __device__ static __forceinline__ Frag along16(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        return lds_get<Frag>(tile + TileLds<float, COLS>::cell(lane % 16, lane / 16) + first * TileLds<float, COLS>::ROW + k0 * 4);
    }
    __device__ static __forceinline__ f32x4 product16(const Frag &a, const Frag &b, f32x4 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
    template <int PARTS>
    __device__ static __forceinline__ void weighted(const Frag &a, const float *w, Frag (&out)[PARTS])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0].v[i] = a.v[i] * w[i];
    }
};

// The place of a workgroup among all: workgroups are dealt to the 8 XCDs in turn, and each XCD takes neighbours here.  Heads are neighbours, whose rows lie side
// by side in a token: an XCD that had every eighth head would use two of its L2's 16 channels.
__device__ __forceinline__ unsigned xcd_place()
{
    const unsigned n = gridDim.x, xcd = blockIdx.x % 8;
    return xcd * (n / 8) + min(xcd, n % 8) + blockIdx.x / 8;
}

constexpr long kMostStride = 1l << 23;          // of a token: 64 tokens in 32-bit offsets of bytes

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A buffer of `bytes` from p on.  All lanes have the same: the compiler does not see it of pointers that were multiplied, and would loop over the lanes.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void *p, uint32_t bytes)
{
    const uint64_t u = (uint64_t)p;
    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u);
    return __builtin_amdgcn_make_buffer_rsrc((void *)at, 0, __builtin_amdgcn_readfirstlane((int)bytes), 0x00020000);
}
// What is there of a chunk: bytes of its tokens.
__device__ __forceinline__ uint32_t chunk_bytes(long stride, int tokens) { return (uint32_t)(max(0, min(kChunk, tokens)) * stride); }

// A tile's pieces of 16 bytes on their way from memory: thread i has cells i, i + THREADS, ...  They are words that nothing looks at before they are stored
// (elements of 16 bits would be taken apart, and waited for, right behind the load), and are read through a buffer that ends behind the last token that
// there is: no branches.  WHOLE: rows of whole pieces at multiples of 4 bytes.  Otherwise word by word (piece_word), those that hold something of the piece;
// what does not belong to it goes when it is stored.
template <class T, int COLS, bool WHOLE, int THREADS>
struct Fetch {
    static constexpr int PER = 16 / sizeof(T), CELLS = COLS / PER, N = kChunk * CELLS / THREADS, ROWS = THREADS / CELLS;
    static constexpr int WORDS = WHOLE || sizeof(T) == 4 ? 4 : 5;
    uint32_t v[N][WORDS];
    uint32_t first, step;      // offsets: of the thread's first piece, from piece to piece
    int have;                  // elements of the row in a piece

    // `stride` bytes from token to token; reversed: row r is token 63 - r of the chunk
    __device__ __forceinline__ void init(int width, long stride, bool reversed)
    {
        const int r = threadIdx.x / CELLS, c = threadIdx.x % CELLS * PER;
        have = max(0, min(PER, width - c));
        first = (uint32_t)((reversed ? kChunk - 1 - r : r) * stride) + c * (uint32_t)sizeof(T);
        step = (uint32_t)(reversed ? -ROWS * stride : ROWS * stride);
    }
    // base: the chunk's first token; `tokens` of them are there
    __device__ __forceinline__ void load(const void *base, long stride, int tokens)
    {
        const uint32_t bytes = chunk_bytes(stride, tokens);
        if (WHOLE) {
            const auto rsrc = buffer_of(base, bytes);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rsrc, have > 0 ? first + i * step : kOut, 0, 0);
#pragma unroll
                for (int w = 0; w < 4; ++w) v[i][w] = x[w];
            }
        } else {
            const uint32_t odd = (uint32_t)(uintptr_t)base & 3u;
            const auto rsrc = buffer_of((const char *)base - odd, 0x80000000u);
#pragma unroll
            for (int i = 0; i < N; ++i) {
#pragma unroll
                for (int w = 0; w < WORDS; ++w)
                    v[i][w] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, piece_word(first + i * step, odd, have * (uint32_t)sizeof(T), bytes, w), 0, 0);
            }
        }
    }
    template <bool SUMS_ORDER = false>
    __device__ __forceinline__ void store(char *tile, const void *base) const
    {
        const int r = threadIdx.x / CELLS, c = threadIdx.x % CELLS;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            u32x4 x;
            if (WORDS == 4) {
#pragma unroll
                for (int w = 0; w < 4; ++w) x[w] = v[i][w];
            } else {
                const bool half = ((uint32_t)(uintptr_t)base + first + i * step) & 2u;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint32_t y = half ? v[i][w] >> 16 | v[i][WORDS == 5 ? w + 1 : w] << 16 : v[i][w];
                    x[w] = have >= 2 * w + 2 ? y : have == 2 * w + 1 ? y & 0xFFFFu : 0;
                }
            }
            char *to = tile + TileLds<T, COLS>::cell(ROWS % 16 == 0 ? r : r + i * ROWS, SUMS_ORDER ? c & ~1 : c) + (ROWS % 16 == 0 ? i * ROWS * TileLds<T, COLS>::ROW : 0);
            if (SUMS_ORDER) {
                to += c % 2 * 8;
                lds_put(to, u32x2{x[0], x[1]});
                lds_put(to + 16, u32x2{x[2], x[3]});
            } else {
                lds_put(to, x);
            }
        }
    }
};

// Log decays of a sequence's head.
struct Decays {
    const void *g;
    long g_b, g_l;
    const float *decay;
    // the words of 64 tokens from t on, `tokens` of them there, one lane each, from the last to the first where reversed
    template <class T>
    __device__ __forceinline__ uint32_t raw(int b, int h, long t, int tokens, bool reversed) const
    {
        const long l = g_l * (long)sizeof(T);
        const auto rsrc = buffer_of((const T *)g + b * g_b + t * g_l + h, g ? chunk_bytes(l, tokens) : 0u);
        const int lane = threadIdx.x % 64;
        const uint32_t at = (uint32_t)((reversed ? kChunk - 1 - lane : lane) * l);
        return sizeof(T) == 4 ? __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0) : (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0);
    }
    template <class T>
    __device__ __forceinline__ static float sum(float of_head, uint32_t raw)
    {
        const float v = of_head + (sizeof(T) == 4 ? __uint_as_float(raw) : __uint_as_float(raw << 16));
        return v < kLeast ? kLeast : v;
    }
    template <class T>
    __device__ __forceinline__ float get(int b, int h, long t) const
    {
        const float v = (decay ? decay[h] : 0.f) + (g ? to_f(((const T *)g)[b * g_b + t * g_l + h]) : 0.f);
        return v < kLeast ? kLeast : v;
    }
};

// A chunk's decays from its rows' own: `hi` + `lo` sums over the rows up to each, in units of 2 (two floats: their differences are exact to 32 bits
// whatever the sums), `first` 2^sum, `last` 2^(what is decayed behind a row).  A wave computes them, a row per lane, in 64 bits.  They are read in packs of
// four, which begin at multiples of 16 bytes, also those of the second of two chunks side by side.
struct alignas(16) ChunkDecays {
    float hi[kChunk], lo[kChunk], first[kChunk], last[kChunk], whole;

    // v + v of another lane, 0 where there is none: the steps of a sum over all lanes up to each
    template <int CTRL, int ROWS>
    __device__ static __forceinline__ double add_from(double v)
    {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_update_dpp(0u, (uint32_t)u, CTRL, ROWS, 0xF, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(0u, (uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
        return v + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
    }

    __device__ __forceinline__ void set(float own, float first_scale, float last_scale)
    {
        const int lane = threadIdx.x % 64;
        double sum = (double)own * 1.4426950408889634074;
        sum = add_from<0x111, 0xF>(sum);      // row_shr:1, 2, 4, 8
        sum = add_from<0x112, 0xF>(sum);
        sum = add_from<0x114, 0xF>(sum);
        sum = add_from<0x118, 0xF>(sum);
        sum = add_from<0x142, 0xA>(sum);      // row_bcast:15 to rows 1 and 3, row_bcast:31 to rows 2 and 3
        sum = add_from<0x143, 0xC>(sum);
        const uint64_t u = __builtin_bit_cast(uint64_t, sum);
        const double all = __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32 |
                                                          (uint32_t)__builtin_amdgcn_readlane((int)u, 63));
        hi[lane] = (float)sum;
        lo[lane] = (float)(sum - (double)(float)sum);
        first[lane] = first_scale * exp2_fast((float)sum);
        last[lane] = last_scale * exp2_fast((float)(all - sum));
        if (lane == 63) whole = exp2_fast((float)all);
    }
    // 2^(sums of row t less those of row s); 16-bit operands need no more than one float of each: sums are 64 * 80 / ln 2 at most, 2^-11 of a unit exact.
    // SAME: the same float whichever end the sums begin at, so that a walk forward and one backward round the same products to the same 16 bits.  The
    // difference is then rounded once: what the floats' own loses is put back with the second ones' difference.
    template <class T, bool SAME>
    __device__ static __forceinline__ float pair(float t_hi, float t_lo, float s_hi, float s_lo)
    {
        const float d = t_hi - s_hi;
        if (sizeof(T) == 4) return exp2_fast(d + (t_lo - s_lo));
        if (!SAME) return exp2_fast(d);
        const float of_s = d - t_hi, lost = (t_hi - (d - of_s)) - (s_hi + of_s);
        return exp2_fast(d + (lost + (t_lo - s_lo)));
    }
    __device__ static __forceinline__ Pack<float, 4> four(const float *p) { return lds_get<Pack<float, 4>>((const char *)p); }
};
static_assert(sizeof(ChunkDecays) % 16 == 0 && offsetof(ChunkDecays, lo) % 16 == 0 && offsetof(ChunkDecays, last) % 16 == 0, "whole packs");

// ---- a walk --------------------------------------------------------------------------------------------------------

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
    long out_b, out_h, out_l;    // of sequence, head and token; a token's is kMostStride at most
    bool out_f32;                // parts of T = bfloat16, for the heads that share a row of it
    float p_scale, first_scale, last_scale;
    Decays decays;
    const int32_t *lengths, *slots;
    int B, L, H, n_slots, segments, per_segment;     // chunks of a segment
    // states: of a slot and head rows (of q's width) and columns (of v's) apart
    const float *state_in;
    float *state_out;
    long s_row, s_col, s_head;
    float *starts;               // (segments, B, H, rows, columns) with the strides of state_in, or null
    bool started;                // starts are there already, from a walk over the same states
    float *segment_decay;        // (segments, B, H)
    float *dots, *state_dots;    // (column tiles' waves, B, H, L): rows of `dot` with the outputs and, backward, with the state's part of them; or null
    void *chunk_states;          // states at the chunks' starts, by workgroup, chunk and thread
    float *passes;               // (column tiles, B, H, chunks): c
    int tiles;
};

// Starts of the segments from their own states.
hipError_t join_states(const Mix &p, hipStream_t s);

// A walk, forward or (REV) backward in time; `whole`: whole_rows of all.  Sets p.tiles.
template <class T, bool REV>
hipError_t run_mix(Mix &p, bool whole, hipStream_t s);

inline int chunks_of(int L) { return (L + kChunk - 1) / kChunk; }
inline int tiles_of(int width, int cols) { return (width + cols - 1) / cols; }

// Columns of a state to a workgroup, 32 to a wave: all of them, so that pairs of tokens are computed once.  fp32 states of many rows have four waves also for
// few columns, two of them without any (two waves are out of registers: 5 x 677 tokens of 6 heads of 72 by 41, Forward's walk 71 us against 45).
inline int cols_of(int rows, int cols, bool f32) { return cols > 64 || (f32 && rows > 64) ? 128 : 64; }

// Rows that Fetch can read by whole pieces
template <class T>
bool whole_rows(const Rows &r)
{
    constexpr int PER = 16 / sizeof(T), WORD = 4 / sizeof(T);
    return r.width % PER == 0 && r.l % WORD == 0 && r.b % WORD == 0 && ((uintptr_t)r.p & 3u) == 0;
}

}  // namespace attention
}  // namespace ucd
