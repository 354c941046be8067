// What the linear attention's kernels share: tiles of 64 tokens in LDS, their products, decays.
#pragma once
#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace attention {
using namespace seq;

constexpr int kChunk = 64, kThreads = 256, kCols = 64;      // tokens of a chunk; columns of a state that a workgroup has
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// exp(-80) is as good as 0, and sums of 64 of them and their differences stay finite: what is below counts as -80.  A NaN stays one.
constexpr float kLeast = -80.f;

// A tile of rows of COLS elements in LDS, in cells of 16 bytes.  Cell c of row r stands at c ^ swizzle(r): 16 lanes that read a cell each of 16 rows meet
// no bank twice, and neither do transposing reads of 4 rows by 4 cells (bfloat16).
template <class T, int COLS>
struct TileLds {
    static constexpr int PER = 16 / sizeof(T), CELLS = COLS / PER, BYTES = kChunk * COLS * (int)sizeof(T);
    __device__ static __forceinline__ int swizzle(int r)
    {
        if (CELLS >= 16) return sizeof(T) == 2 ? (r & 3) << 2 | (r >> 2 & 3) : r & 15;
        return (r >> 1 & 1) << 2 | (r >> 2 & 3);
    }
    __device__ static __forceinline__ int cell(int r, int c) { return (r * CELLS + (c ^ swizzle(r))) * 16; }
    __device__ static __forceinline__ int at(int r, int col) { return cell(r, col / PER) + col % PER * (int)sizeof(T); }
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
        return *reinterpret_cast<const Frag *>(tile + TileLds<bf16_t, COLS>::cell(first + lane % 32, k0 / 8 + lane / 32));
    }
    // columns first .. first + 31, reduction over rows from k0 on: 16 lanes fetch 4 rows of 16 columns each and get 4 rows of a column each
    template <int COLS>
    __device__ static __forceinline__ Frag across(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64, col = first + lane / 16 % 2 * 16 + lane % 4 * 4, k = k0 + lane / 32 * 8 + lane % 16 / 4;
        typedef __attribute__((address_space(3))) s16x4 lds_t;
        struct Both {
            s16x4 lo, hi;
        } v;
        v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(tile + TileLds<bf16_t, COLS>::at(k, col)));
        v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(tile + TileLds<bf16_t, COLS>::at(k + 4, col)));
        return __builtin_bit_cast(Frag, v);
    }
    __device__ static __forceinline__ f32x16 product(const Frag &a, const Frag &b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
    // w a in PARTS bfloat16 parts, the largest first: three are as exact as the sums' 32 bits, two leave 2^-17
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
        return *reinterpret_cast<const Frag *>(tile + TileLds<float, COLS>::cell(first + lane % 32, k0 / 4 + lane / 32));
    }
    template <int COLS>
    __device__ static __forceinline__ Frag across(const char *tile, int first, int k0)
    {
        const int lane = threadIdx.x % 64;
        Frag v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = *reinterpret_cast<const float *>(tile + TileLds<float, COLS>::at(k0 + lane / 32 * 4 + i, first + lane % 32));
        return v;
    }
    __device__ static __forceinline__ f32x16 product(const Frag &a, const Frag &b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
        return c;
    }
    template <int PARTS>
    __device__ static __forceinline__ void weighted(const Frag &a, const float *w, Frag (&out)[PARTS])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0].v[i] = a.v[i] * w[i];
    }
};

// Reads behind a buffer's end give 0.
constexpr uint32_t kOut = 0x80000000u;
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

// A tile's pieces of 16 bytes on their way from memory: thread i has cells i, i + 256, ...  They are words that nothing looks at before they are stored
// (elements of 16 bits would be taken apart, and waited for, right behind the load), and are read through a buffer that ends behind the last token that
// there is: no branches.  WHOLE: rows of whole pieces at multiples of 4 bytes.  Otherwise word by word: those that begin before the row's end, from the
// multiple of 4 bytes at or below the piece's begin; what does not belong to the piece goes when it is stored.
template <class T, int COLS, bool WHOLE>
struct Fetch {
    static constexpr int PER = 16 / sizeof(T), CELLS = COLS / PER, N = kChunk * CELLS / kThreads, ROWS = kThreads / CELLS;
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
                const uint32_t at = first + i * step, from = (at + odd) & ~3u, end = at + odd + have * (uint32_t)sizeof(T);
#pragma unroll
                for (int w = 0; w < WORDS; ++w)
                    v[i][w] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, at < bytes && from + 4 * w < end ? from + 4 * w : kOut, 0, 0);
            }
        }
    }
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
            *reinterpret_cast<u32x4 *>(tile + TileLds<T, COLS>::cell(r + i * ROWS, c)) = x;
        }
    }
};

// Log decays of a sequence's head.
struct Decays {
    const void *g;
    long g_b, g_l;
    const float *decay;
    template <class T>
    __device__ __forceinline__ T raw(int b, int h, long t) const { return g ? ((const T *)g)[b * g_b + t * g_l + h] : from_f<T>(0.f); }
    template <class T>
    __device__ __forceinline__ float get(int h, T raw) const
    {
        const float v = (decay ? decay[h] : 0.f) + to_f(raw);
        return v < kLeast ? kLeast : v;
    }
    template <class T>
    __device__ __forceinline__ float get(int b, int h, long t) const { return get<T>(h, raw<T>(b, h, t)); }
};

// A chunk's decays from its rows' own: `hi` + `lo` sums over the rows up to each, in units of 2 (two floats: their differences are exact to 32 bits
// whatever the sums), `first` 2^sum, `last` 2^(what is decayed behind a row).  A wave computes them, a row per lane, in 64 bits.
struct ChunkDecays {
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
    // 2^(sums of row t less those of row s); 16-bit operands need no more than one float of each: sums are 64 * 80 / ln 2 at most, 2^-11 of a unit exact
    template <class T>
    __device__ static __forceinline__ float pair(float t_hi, float t_lo, float s_hi, float s_lo)
    {
        return exp2_fast(sizeof(T) == 2 ? t_hi - s_hi : (t_hi - s_hi) + (t_lo - s_lo));
    }
};

}  // namespace attention
}  // namespace ucd
