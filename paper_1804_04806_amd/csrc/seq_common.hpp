// What the sequence operators' kernels share: element types, wide loads, activations, sums over lanes.
#pragma once
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace ucd {
namespace seq {

typedef __bf16 bf16_t;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16_t v) { return (float)v; }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16_t from_f<bf16_t>(float v) { return (bf16_t)v; }   // to nearest, ties to even

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// N neighbours: one load or store where WIDE says that they are all there or none, the first `have` of them otherwise.  Global memory is read and
// written in such packs from any element's address on.
template <class T, int N>
struct alignas(sizeof(T) * N) Pack {
    T v[N];
};
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) LoosePack {
    T v[N];
};
template <class T, int N>
__device__ __forceinline__ Pack<T, N> loose_load(const T *p)
{
    return __builtin_bit_cast(Pack<T, N>, *reinterpret_cast<const LoosePack<T, N> *>(p));
}
template <class T, int N>
__device__ __forceinline__ void loose_store(T *p, const Pack<T, N> &r)
{
    *reinterpret_cast<LoosePack<T, N> *>(p) = __builtin_bit_cast(LoosePack<T, N>, r);
}

template <bool WIDE, class T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p, int have)
{
    Pack<T, N> r;
    if (WIDE) {
        if (have > 0) r = loose_load<T, N>(p);
        else
            for (int i = 0; i < N; ++i) r.v[i] = from_f<T>(0.f);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = i < have ? p[i] : from_f<T>(0.f);
    }
    return r;
}

template <bool WIDE, class T, int N>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, N> &r, int have)
{
    if (WIDE) {
        if (have > 0) loose_store<T, N>(p, r);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) p[i] = r.v[i];
    }
}

// N elements as they come from memory, in words (WIDE: one load; otherwise a word each, the last of `have` of them again behind it): a lane's prefetched
// values stay as they are until they are used.  As elements of 16 bits the compiler takes them apart, and waits for them, right behind the load.
template <class T, int N, bool WIDE>
struct Raw {
    static constexpr bool PACKED = WIDE && N * sizeof(T) % 4 == 0;
    static constexpr int WORDS = PACKED ? N * (int)sizeof(T) / 4 : N;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const char *base, uint32_t offset, int have)
    {
        if (PACKED) {
            struct __attribute__((packed, aligned(sizeof(T)))) Words {
                uint32_t v[WORDS];
            };
            const Words r = *reinterpret_cast<const Words *>(base + offset);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = r.v[i];
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) {
                const uint32_t at = offset + (uint32_t)sizeof(T) * (WIDE ? i : max(0, min(i, have - 1)));
                if (sizeof(T) == 4) w[i] = *reinterpret_cast<const uint32_t *>(base + at);
                else w[i] = *reinterpret_cast<const uint16_t *>(base + at);
            }
        }
    }
    __device__ __forceinline__ float get(int i) const
    {
        if (sizeof(T) == 4) return __builtin_bit_cast(float, w[i]);
        if (!PACKED) return __builtin_bit_cast(float, w[i % WORDS] << 16);
        return __builtin_bit_cast(float, i % 2 ? w[i / 2 % WORDS] & 0xFFFF0000u : w[i / 2 % WORDS] << 16);
    }
};

// 2^v on the transcendental unit, to an ulp of the result.  Where v is a rounded product w log2(e), as in sigmoid and in the scan's decays, its rounding
// adds up to |w| 2^-24 of the result: 6e-7 of a decay to 5e-5, the more the less is left.  exp_full's correction costs six instructions more, which the
// decays would pay for every state and token.
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }

// exp(v) to about an ulp: the rounding of v * log2(e), up to 2^-24 |v log2(e)| in the exponent, is put back as a factor.
__device__ __forceinline__ float exp_full(float v)
{
    const float t = v * kLog2e;
    const float lost = fmaf(v, kLog2e, -t) + v * 1.92596298e-8f;   // log2(e) is kLog2e + 1.92596298e-8
    const float e = exp2_fast(t);
    // an infinite v leaves a NaN in `lost`, where e is 0 or infinite
    return fabsf(t) < 256.f ? fmaf(e * kLn2, lost, e) : e;
}

// 1 / (1 + exp(-v)).  exp(-v) overflows to infinity below -88: the quotient is then 0, as it should be.
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + exp2_fast(v * -kLog2e)); }

// log(1 + exp(v)) = max(v, 0) + log1p(e), e = exp(-|v|); with w = 1 + e rounded, log1p(e) = log(w) e / (w - 1) to an ulp or two, because w - 1 is
// exact and log(w) / (w - 1) hardly changes between 1 + e and w.  Also the function's derivative, 1 / (1 + exp(-v)).  For bf16 activations exp(-|v|)
// without its correction: |v| 2^-24 of it off at most, which is also what the rounding of v = dt + dt_bias to 32 bits may leave of it.
template <class T>
__device__ __forceinline__ float softplus(float v, float *derivative = nullptr)
{
    const float e = sizeof(T) == 4 ? exp_full(-fabsf(v)) : exp2_fast(-fabsf(v) * kLog2e), w = 1.f + e, d = w - 1.f;
    const float l = d == 0.f ? e : __builtin_amdgcn_logf(w) * kLn2 * (e * __builtin_amdgcn_rcpf(d));
    if (derivative) *derivative = (v >= 0.f ? 1.f : e) * __builtin_amdgcn_rcpf(w);
    return fmaxf(v, 0.f) + l;
}

// Lane i's value from another lane of its row of 16, by the data path's own permutations.
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;   // quad_perm [1,0,3,2], [2,3,0,1]; row_half_mirror; row_mirror
constexpr int kRor8 = 0x128, kRor4 = 0x124;                                       // row_ror

// Sum over groups of N neighbouring lanes, N = 1, 2, 4, 8, 16, in every lane.
template <int N>
__device__ __forceinline__ float sum_lanes(float v)
{
    if (N > 1) v += dpp<kXor1>(v);
    if (N > 2) v += dpp<kXor2>(v);
    if (N > 4) v += dpp<kHalfMirror>(v);
    if (N > 8) v += dpp<kMirror>(v);
    return v;
}

// The sums over LPC neighbouring lanes of values that come token by token (up or down); after LPC of them, of which t is the last and first the lowest,
// lane q of each group has that of token first + q.
template <int LPC>
struct LaneSums {
    float v[4], kept = 0.f;
    __device__ __forceinline__ void add(int t, float value, int q)
    {
        if (LPC == 4) {
            v[t % 4] = value;
            return;
        }
        value = sum_lanes<LPC>(value);
        kept = q == t % LPC ? value : kept;
    }
    __device__ __forceinline__ float get(int q) const
    {
        if (LPC != 4) return kept;
        // pairs of lanes share out pairs of tokens, then pairs of pairs: 9 instructions where sums in every lane and a choice are 12
        const bool odd = q & 1, high = q & 2;
        const float low = (odd ? v[1] : v[0]) + dpp<kXor1>(odd ? v[0] : v[1]), top = (odd ? v[3] : v[2]) + dpp<kXor1>(odd ? v[2] : v[3]);
        return (high ? top : low) + dpp<kXor2>(high ? low : top);
    }
};

// a = {a of the lower half of the wave, b of the lower half}, b = {a of the upper half, b of the upper half}
__device__ __forceinline__ void swap_halves(float &a, float &b)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned lo = r[0], hi = r[1];      // bit_cast of a vector's element takes its first
    a = __builtin_bit_cast(float, lo);
    b = __builtin_bit_cast(float, hi);
}

// the same of odd and even rows of 16 lanes
__device__ __forceinline__ void swap_rows(float &a, float &b)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    const unsigned lo = r[0], hi = r[1];      // bit_cast of a vector's element takes its first
    a = __builtin_bit_cast(float, lo);
    b = __builtin_bit_cast(float, hi);
}

// Sum over groups of `lanes` neighbouring lanes, a power of two up to the wave, in every lane.  All lanes of a wave take part.
__device__ __forceinline__ float sum_group(float v, int lanes)
{
    if (lanes > 1) v += dpp<kXor1>(v);
    if (lanes > 2) v += dpp<kXor2>(v);
    if (lanes > 4) v += dpp<kHalfMirror>(v);
    if (lanes > 8) v += dpp<kMirror>(v);
    if (lanes > 16) {
        float w = v;
        swap_rows(v, w);
        v += w;
    }
    if (lanes > 32) {
        float w = v;
        swap_halves(v, w);
        v += w;
    }
    return v;
}

// Sum over the lanes that differ in the bits from `from` (a power of two) up, in every lane.
__device__ __forceinline__ float sum_apart(float v, int from)
{
    if (from <= 32) {
        float w = v;
        swap_halves(v, w);
        v += w;
    }
    if (from <= 16) {
        float w = v;
        swap_rows(v, w);
        v += w;
    }
    if (from <= 8) v += dpp<kRor8>(v);
    if (from <= 4) v += dpp<kRor4>(v);
    if (from <= 2) v += dpp<kXor2>(v);
    if (from <= 1) v += dpp<kXor1>(v);
    return v;
}

// Joins of partial sums: workgroups of 64 columns by 16 groups of rows.  The sum over `rows` rows of a column, rows of one group apart by 16, then
// over the groups in their order; valid in the threads of the first group.
constexpr int kJoinColumns = 64, kJoinThreads = 1024;

__device__ __forceinline__ float join_rows(const float *part, long rows, long row_length, long column)
{
    constexpr int GROUPS = kJoinThreads / kJoinColumns;
    __shared__ float lds[GROUPS][kJoinColumns];
    const int x = threadIdx.x % kJoinColumns, group = threadIdx.x / kJoinColumns;
    float v = 0.f;
    if (column < row_length)
#pragma unroll 8
        for (long r = group; r < rows; r += GROUPS) v += part[r * row_length + column];
    lds[group][x] = v;
    __syncthreads();
    v = lds[0][x];
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) v += lds[g][x];
    return v;
}

// out(column, sum) for all columns.  A grid of 2^32 threads is none, so that workgroups may have several times 64 columns.
inline unsigned join_grid(long columns) { return (unsigned)std::min((columns + kJoinColumns - 1) / kJoinColumns, 1l << 21); }

template <class F>
__device__ __forceinline__ void join_columns(const float *part, long rows, long row_length, F out)
{
    for (long first = blockIdx.x * (long)kJoinColumns; first < row_length; first += gridDim.x * (long)kJoinColumns) {
        const long column = first + threadIdx.x % kJoinColumns;
        const float v = join_rows(part, rows, row_length, column);
        if (column < row_length && threadIdx.x < kJoinColumns) out(column, v);
        __syncthreads();
    }
}

// Orders a wave's own LDS accesses: the hardware runs them in program order, the compiler has to keep them so.
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A workgroup's barrier for what is in LDS alone: __syncthreads() waits for all stores to memory too, and for loads that are meant to be under way.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace seq
}  // namespace ucd
