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
    // (w a) b with the weighted operand in three parts: as exact as the sums' 32 bits
    __device__ static __forceinline__ void weighted(const Frag &a, const float *w, Frag (&out)[3])
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = (float)a[i] * w[i];
            const bf16_t h = (bf16_t)v;
            const float r = v - (float)h;
            const bf16_t m = (bf16_t)r;
            out[0][i] = h;
            out[1][i] = m;
            out[2][i] = (bf16_t)(r - (float)m);
        }
    }
    static constexpr int PARTS = 3;
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
    __device__ static __forceinline__ void weighted(const Frag &a, const float *w, Frag (&out)[1])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) out[0].v[i] = a.v[i] * w[i];
    }
    static constexpr int PARTS = 1;
};

// A tile's pieces on their way from memory: thread i has cells i, i + 256, ...
template <class T, int COLS>
struct Fetch {
    static constexpr int PER = 16 / sizeof(T), CELLS = COLS / PER, N = kChunk * CELLS / kThreads;
    Pack<T, PER> v[N];
    // row(r): the address of row r's first element, null where there is none; `width` elements a row
    template <class F>
    __device__ __forceinline__ void load(F row, int width)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = i * kThreads + threadIdx.x, r = at / CELLS, c = at % CELLS * PER;
            const T *p = row(r);
            const int have = p ? width - c : 0;
            if (have >= PER) v[i] = loose_load<T, PER>(p + c);
            else v[i] = load_pack<false, T, PER>(p + c, have);
        }
    }
    __device__ __forceinline__ void store(char *tile) const
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = i * kThreads + threadIdx.x;
            *reinterpret_cast<Pack<T, PER> *>(tile + TileLds<T, COLS>::cell(at / CELLS, at % CELLS)) = v[i];
        }
    }
};

// Log decays of a sequence's head.
struct Decays {
    const void *g;
    long g_b, g_l;
    const float *decay;
    template <class T>
    __device__ __forceinline__ float get(int b, int h, long t) const
    {
        float v = decay ? decay[h] : 0.f;
        if (g) v += to_f(((const T *)g)[b * g_b + t * g_l + h]);
        return v < kLeast ? kLeast : v;
    }
};

// A chunk's decays from its rows' own: `total` sums over the rows up to each, in units of 2 and in two floats (their differences are exact to 32 bits
// whatever the sums), `first` 2^total, `last` 2^(what is decayed behind a row).  A wave computes them, a row per lane, in 64 bits.
struct ChunkDecays {
    float hi[kChunk], lo[kChunk], first[kChunk], last[kChunk];
    __device__ __forceinline__ void set(float own, float first_scale, float last_scale)
    {
        const int lane = threadIdx.x % 64;
        double sum = (double)own * 1.4426950408889634074;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const double other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        const double all = __shfl(sum, 63);
        hi[lane] = (float)sum;
        lo[lane] = (float)(sum - (double)(float)sum);
        first[lane] = first_scale * exp2_fast((float)sum);
        last[lane] = last_scale * exp2_fast((float)(all - sum));
        if (lane == 63) whole = exp2_fast((float)all);
    }
    float whole;
};

}  // namespace attention
}  // namespace ucd
