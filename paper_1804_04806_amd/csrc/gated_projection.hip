// Gated projection: y = act(x Wg^T) * (x Wu^T), and its gradients.
//
// Products bound it from some hundred tokens on, the weights' bytes below.  Forward is one product whose tiles hold the same columns of both
// projections, so that a lane has both sides of a gate in registers and writes y alone (for Backward, both sides in fp32 too).  Backward first turns
// dy and what was kept into dG = [dgate | dup], bfloat16 (rounded once, the products' operand: gradients are 2.3e-3 off instead of their own rounding's
// 1.7e-3), then dx = dG [Wg; Wu] and [dWg; dWu] = dG^T x, each
// one product.  Operands that the products cannot read as they lie (fp32, rows of no whole 16 bytes) are copied first.
#include <algorithm>

#include "gated_plan.hpp"
#include "product.hpp"
#include "seq.h"

namespace ucd {
namespace gated {
using namespace seq;
using namespace product;
static_assert(kStep == BK, "plans count the products' steps");

constexpr float kGelu = 1.59576912160573071176f, kCube = 0.044715f;    // 2 sqrt(2 / pi)

// act(v) and its derivative; GELU in its tanh form is v sigmoid(2 sqrt(2/pi) (v + 0.044715 v^3)).  The cube of a v beyond 1e12 overflows to an infinity of
// its sign, whose sigmoid is 0 or 1 as it should be; v times 0 is left out there.
__device__ __forceinline__ float gate_sigmoid(int act, float v)
{
    const float w = act == UCD_ACT_GELU ? kGelu * fmaf(kCube * v * v, v, v) : v;
    return __builtin_amdgcn_rcpf(1.f + exp_full(-w));
}
__device__ __forceinline__ float gate_act(int act, float v)
{
    return act == UCD_ACT_NONE ? v : v * gate_sigmoid(act, v);
}
__device__ __forceinline__ float gate_slope(int act, float v, float &value)
{
    value = v;
    if (act == UCD_ACT_NONE) return 1.f;
    const float s = gate_sigmoid(act, v), inner = act == UCD_ACT_GELU ? kGelu * fmaf(3.f * kCube * v, v, 1.f) : 1.f;
    value = v * s;
    const float rest = s * (1.f - s);
    return rest == 0.f ? s : fmaf(v * inner, rest, s);
}

// ---- copies --------------------------------------------------------------------------------------------------------

// The three bfloat16 parts of an fp32 value: the first is the largest finite one where it would be rounded to an infinity.
__device__ __forceinline__ void parts_of(float v, bf16_t &h, bf16_t &m, bf16_t &l)
{
    constexpr float kMost = 3.38953139e38f;
    h = (bf16_t)(fabsf(v) < INFINITY ? fminf(fmaxf(v, -kMost), kMost) : v);
    const float a = v - (float)h;
    m = (bf16_t)a;
    l = (bf16_t)(a - (float)m);
}

template <class T>
struct Planes {
    static constexpr int N = sizeof(T) == 4 ? 3 : 1;
};

template <class T>
__device__ __forceinline__ void store_planes(bf16_t *to, long plane, const float (&v)[8])
{
    Pack<bf16_t, 8> p[3];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (sizeof(T) == 4) parts_of(v[i], p[0].v[i], p[1].v[i], p[2].v[i]);
        else p[0].v[i] = from_f<bf16_t>(v[i]);
    }
#pragma unroll
    for (int i = 0; i < Planes<T>::N; ++i) *reinterpret_cast<Pack<bf16_t, 8> *>(to + i * plane) = p[i];
}

// rows x cols elements, rows `stride` apart -> planes of rows of `width`, a multiple of 8 from cols on, filled up with 0.  Up to three matrices in a launch,
// grid.y: of small ones most of a copy's 5 us is its launch.
struct Copy {
    const void *from;
    long stride, rows, plane;
    bf16_t *to;
};
struct Copies {
    Copy c[3];
    int count, cols, width;
};

template <class T>
__global__ __launch_bounds__(256) void copy_rows_kernel(Copies all)
{
    const Copy &p = all.c[blockIdx.y];
    const int packs = all.width / 8;
    const long size = p.rows * packs;
    const bool small = size <= 0x7fffffffl;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < size; i += gridDim.x * 256l) {
        const long row = small ? (long)((uint32_t)i / (uint32_t)packs) : i / packs;
        const int c = (int)(i - row * packs) * 8, have = min(8, all.cols - c);
        const T *src = (const T *)p.from + row * p.stride + c;
        float v[8];
        if (have == 8) {
            const Pack<T, 8> r = loose_load<T, 8>(src);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = to_f(r.v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < have ? to_f(src[j]) : 0.f;
        }
        store_planes<T>(p.to + row * all.width + c, p.plane, v);
    }
}

// ---- forward -------------------------------------------------------------------------------------------------------

struct GateOut {
    void *y;
    long y_m;
    float *saved;      // M rows of two rows of `wide` floats, or null
    int M, F, wide, act;
};

template <class T>
__device__ __forceinline__ void gate_store(const GateOut &o, long m, int f, const Pack<float, 4> &g, const Pack<float, 4> &u)
{
    const int have = min(4, o.F - f);
    if (m >= o.M || have <= 0) return;
    Pack<T, 4> y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y.v[i] = from_f<T>(gate_act(o.act, g.v[i]) * u.v[i]);
    T *at = (T *)o.y + m * o.y_m + f;
    if (have == 4) loose_store<T, 4>(at, y);
    else store_pack<false, T, 4>(at, y, have);
    if (o.saved) {      // whole packs: rows are a multiple of 4
        float *s = o.saved + m * 2 * o.wide + f;
        *reinterpret_cast<Pack<float, 4> *>(s) = g;
        *reinterpret_cast<Pack<float, 4> *>(s + o.wide) = u;
    }
}

// Products bound it; what a tile writes is not overlapped with them.  8192 x 2048 -> 8192, bf16: 509 us (1080 TFLOP/s), 561 with both sides for Backward.
template <class TILE, class T>
__global__ __launch_bounds__(TILE::THREADS) void gated_forward_kernel(Problem p, GateOut o, float *part)
{
    __shared__ __attribute__((aligned(16))) char lds[TILE::LDS];
    const int tm = blockIdx.x % p.tiles_m, tn = blockIdx.x / p.tiles_m;
    const int m0 = tm * TILE::BM, f0 = tn * (TILE::BN / 2);
    int t0, t1;
    split_range(p, blockIdx.y, t0, t1);
    TILE tile;
    tile.run(p, m0, f0, t0, t1, lds);
    constexpr int SIDE = TILE::FN / 2;
    auto sums = [&](int i, int j, int r) { return tile.sums(i, j, r); };
    // both sides in fp32: partial sums, for every split and row a row of either side, or what Backward reads
    float *both = part ? part + (long)blockIdx.y * o.M * 2 * o.wide : o.saved;
    if (both) {
        auto sink = [&](int m, int n, const Pack<float, 4> &v) {
            const int side = n >= TILE::BN / 2, f = f0 + n - side * (TILE::BN / 2);
            if (m0 + m < o.M && f < o.F) *reinterpret_cast<Pack<float, 4> *>(both + (m0 + m) * 2l * o.wide + side * o.wide + f) = v;
        };
        tile.template rows<float, 0, SIDE>(lds, sums, sink);
        tile.template rows<float, SIDE, SIDE>(lds, sums, sink);
    }
    if (part) return;
    tile.template rows<T, 0, SIDE>(
        lds,
        [&](int i, int j, int r) {
            Pack<float, 4> g = tile.sums(i, j, r);
            const Pack<float, 4> u = tile.sums(i + SIDE, j, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) g.v[e] = gate_act(o.act, g.v[e]) * u.v[e];
            return g;
        },
        [&](int m, int n, const auto &v) {
            constexpr int PER = 16 / sizeof(T);
            const int f = f0 + n, have = min(PER, o.F - f);
            if (m0 + m >= o.M || have <= 0) return;
            T *at = (T *)o.y + (m0 + m) * o.y_m + f;
            if (have == PER) loose_store<T, PER>(at, v);
            else store_pack<false, T, PER>(at, v, have);
        });
}

template <class T>
__global__ __launch_bounds__(256) void gated_join_kernel(const float *part, int splits, GateOut o)
{
    const int packs = o.wide / 4;
    const long size = (long)o.M * 2 * o.wide;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < (long)o.M * packs; i += gridDim.x * 256l) {
        const long m = i / packs;
        const int f = (int)(i % packs) * 4;
        const float *at = part + m * 2 * o.wide + f;
        Pack<float, 4> g{}, u{};
        for (int s = 0; s < splits; ++s) {
            const auto a = *reinterpret_cast<const Pack<float, 4> *>(at + s * size), b = *reinterpret_cast<const Pack<float, 4> *>(at + s * size + o.wide);
#pragma unroll
            for (int e = 0; e < 4; ++e) g.v[e] += a.v[e], u.v[e] += b.v[e];
        }
        gate_store<T>(o, m, f, g, u);
    }
}

// ---- few tokens ----------------------------------------------------------------------------------------------------
//
// Up to 64 tokens: the weights are read once, straight into the matrix instructions' operands, 16 bytes a lane.  A workgroup has 16 CT columns of both
// sides and all tokens; its eight waves share the reduction out, two steps of 32 (16 for fp32), 128 bytes of a row, each by turns, and join their sums
// in LDS.  Loads are without branches, AHEAD turns before their use.  Memory bounds it for few tokens, what is read of the tokens for many.

constexpr int kFewWaves = 8;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Rows from `base` on, read in pieces of 16 bytes.  WHOLE: rows of whole pieces at multiples of 4 bytes, through a buffer: what is not there is 0.
// Otherwise element by element at a row's end.
template <class T, bool WHOLE>
struct FewRows {
    static constexpr int N = 16 / sizeof(T);
    __amdgpu_buffer_rsrc_t rsrc;
    const T *base;
    long stride;

    __device__ __forceinline__ FewRows(const T *p, long stride_) : base(p), stride(stride_)
    {
        if (WHOLE) rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)uniform(p), 0, (int)0x80000000u, 0x00020000);
    }
    // the piece at k of a row, of which `have` elements are there
    __device__ __forceinline__ u32x4 load(int row, bool real, int k, int have) const
    {
        if constexpr (WHOLE) {
            const uint32_t at = (uint32_t)(row * stride + k) * (uint32_t)sizeof(T);
            const auto v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, real && have > 0 ? (int)at : (int)0x80000000u, 0, 0);
            return __builtin_bit_cast(u32x4, v);
        } else {
            const int n = real ? have : 0;
            const T *p = base + row * stride + k;
            return __builtin_bit_cast(u32x4, n >= N ? loose_load<T, N>(p) : load_pack<false, T, N>(p, n));
        }
    }
};

__device__ __forceinline__ f32x4 few_product(bf16_t, const u32x4 &w, const u32x4 &x, f32x4 acc)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 few_product(float, const u32x4 &w, const u32x4 &x, f32x4 acc)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i]), __uint_as_float(x[i]), acc, 0, 0, 0);
    return acc;
}

template <class T, int MT, int CT, int AHEAD, bool WHOLE>
__global__ __launch_bounds__(64 * kFewWaves) void gated_few_kernel(const T *x, long x_m, const T *wg, const T *wu, int D, GateOut o)
{
    constexpr int N = 16 / sizeof(T), STEP = 4 * N, TURN = 2 * STEP;
    __shared__ f32x4 sums[kFewWaves][2 * CT * MT][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, row = lane % 16;
    const long f0 = blockIdx.x * (16l * CT);
    const int left = (int)min(16l * CT, o.F - f0);
    const FewRows<T, WHOLE> rg(wg + f0 * D, D), ru(wu + f0 * D, D), rx(x, x_m);
    f32x4 acc[2][CT][MT] = {};
    struct Turn {
        u32x4 w[2][2][CT], x[2][MT];
    } turn[AHEAD];
    const auto load = [&](Turn &r, int k0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = k0 + h * STEP + lane / 16 * N, have = D - k;
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                r.w[h][0][c] = rg.load(16 * c + row, 16 * c + row < left, k, have);
                r.w[h][1][c] = ru.load(16 * c + row, 16 * c + row < left, k, have);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) r.x[h][t] = rx.load(16 * t + row, 16 * t + row < o.M, k, have);
        }
    };
    // Workgroups begin at turns of their own: x's lines are then not asked for by all of them at once.
    const int turns = (D + kFewWaves * TURN - 1) / (kFewWaves * TURN);
    int at = blockIdx.x / 8 % turns, next = 0;
    const auto load_next = [&](Turn &r) {
        load(r, next < turns ? (at * kFewWaves + (wave + blockIdx.x / 8) % kFewWaves) * TURN : D);
        ++next;
        at = at + 1 < turns ? at + 1 : 0;
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_next(turn[i]);
    for (int done = 0; done < turns; done += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            Turn &r = turn[i];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int side = 0; side < 2; ++side) acc[side][c][t] = few_product(T(), r.w[h][side][c], r.x[h][t], acc[side][c][t]);
            load_next(r);
        }
    }
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int side = 0; side < 2; ++side) sums[wave][2 * (c * MT + t) + side][lane] = acc[side][c][t];
    __syncthreads();
    // a lane's sums: column 4 (lane / 16) + 0 .. 3, token lane % 16
    for (int i = wave; i < CT * MT; i += kFewWaves) {
        Pack<float, 4> gate{}, up{};
        for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) gate.v[e] += sums[w][2 * i][lane][e], up.v[e] += sums[w][2 * i + 1][lane][e];
        gate_store<T>(o, 16 * (i % MT) + row, (int)f0 + 16 * (i / MT) + 4 * (lane / 16), gate, up);
    }
}

// ---- backward ------------------------------------------------------------------------------------------------------

// dG's planes, M rows of 2 * half: [dgate | dup], columns behind F are 0.  Memory bounds it: 8192 by 8192, bf16, 197 us for 940 MB.
template <class T>
__global__ __launch_bounds__(256) void gated_gradient_kernel(const T *dy, long dy_m, const float *saved, GateOut o, int half, long row, bf16_t *out, long plane)
{
    const int packs = half / 8;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < (long)o.M * packs; i += gridDim.x * 256l) {
        const long m = i / packs;
        const int f = (int)(i % packs) * 8, have = min(8, o.F - f);
        float dg[8] = {}, du[8] = {};
        if (have > 0) {
            const T *d = dy + m * dy_m + f;
            const float *s = saved + m * 2 * o.wide + f;
            Pack<T, 8> v;
            Pack<float, 8> g, u;
            if (have == 8) {
                v = loose_load<T, 8>(d);
                g = loose_load<float, 8>(s);
                u = loose_load<float, 8>(s + o.wide);
            } else {
                v = load_pack<false, T, 8>(d, have);
                g = load_pack<false, float, 8>(s, have);
                u = load_pack<false, float, 8>(s + o.wide, have);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float value;
                const float slope = gate_slope(o.act, g.v[e], value), dv = to_f(v.v[e]);
                dg[e] = e < have ? dv * u.v[e] * slope : 0.f;
                du[e] = e < have ? dv * value : 0.f;
            }
        }
        store_planes<T>(out + m * row + f, plane, dg);
        store_planes<T>(out + m * row + half + f, plane, du);
    }
}

// out(m, n), rows `stride` apart, of one matrix or of two: rows from `half` on are the second's
struct MatrixOut {
    void *p[2];
    long stride;
    long rows, half;      // rows of each; rows from `half` on are the second's, which one alone has beyond any tile
    int cols;
    bool add;
};

template <class T, int N>
__device__ __forceinline__ void matrix_store(const MatrixOut &o, long m, int n, const Pack<float, N> &v)
{
    const int second = m >= o.half, have = min(N, o.cols - n);
    m -= second ? o.half : 0;
    if (m >= o.rows || have <= 0) return;
    T *at = (T *)o.p[second] + m * o.stride + n;
    Pack<T, N> r;
    if (have == N) {
        Pack<T, N> old{};
        if (o.add) old = loose_load<T, N>(at);
#pragma unroll
        for (int e = 0; e < N; ++e) r.v[e] = from_f<T>(o.add ? to_f(old.v[e]) + v.v[e] : v.v[e]);
        loose_store<T, N>(at, r);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < have) at[e] = from_f<T>(o.add ? to_f(at[e]) + v.v[e] : v.v[e]);
    }
}

// dx (dG along its rows, the weights across) and the weights' gradients (both across).  8192 x 2048 -> 8192, bf16: 462 and 472 us, 1190 and 1165 TFLOP/s.
template <class TILE, class T>
__global__ __launch_bounds__(TILE::THREADS) void product_kernel(Problem p, MatrixOut o, float *part, long part_rows, int part_cols)
{
    __shared__ __attribute__((aligned(16))) char lds[TILE::LDS];
    const int tm = blockIdx.x % p.tiles_m, tn = blockIdx.x / p.tiles_m;
    const int m0 = tm * TILE::BM, n0 = tn * TILE::BN;
    int t0, t1;
    split_range(p, blockIdx.y, t0, t1);
    TILE tile;
    tile.run(p, m0, n0, t0, t1, lds);
    auto sums = [&](int i, int j, int r) { return tile.sums(i, j, r); };
    if (part) {
        float *at = part + (long)blockIdx.y * part_rows * part_cols;
        tile.template rows<float, 0, TILE::FN>(lds, sums, [&](int m, int n, const Pack<float, 4> &v) {
            if (m0 + m < part_rows && n0 + n < part_cols) *reinterpret_cast<Pack<float, 4> *>(at + (long)(m0 + m) * part_cols + n0 + n) = v;
        });
        return;
    }
    if (o.add) {       // added to in fp32: old values and sums are rounded together
        tile.template rows<float, 0, TILE::FN>(lds, sums, [&](int m, int n, const Pack<float, 4> &v) { matrix_store<T, 4>(o, (long)m0 + m, n0 + n, v); });
        return;
    }
    tile.template rows<T, 0, TILE::FN>(lds, sums, [&](int m, int n, const auto &v) {
        constexpr int PER = 16 / sizeof(T);
        long row = (long)m0 + m;
        const int second = row >= o.half, col = n0 + n, have = min(PER, o.cols - col);
        row -= second ? o.half : 0;
        if (row >= o.rows || have <= 0) return;
        T *at = (T *)o.p[second] + row * o.stride + col;
        if (have == PER) loose_store<T, PER>(at, v);
        else store_pack<false, T, PER>(at, v, have);
    });
}

// dx's and the weights' products
template <class T> using LargeAlong = Tile<T, 256, 256, 2, 4, 2, true, false, true>;
template <class T> using MiddleAlong = Tile<T, 192, 256, 2, 4, 2, true, false, true>;
template <class T> using SmallAlong = Tile<T, 128, 128, 2, 2, 2, true, false, true>;
template <class T> using LargeAcross = Tile<T, 256, 256, 2, 4, 2, false, false, false>;
template <class T> using SmallAcross = Tile<T, 128, 128, 2, 2, 2, false, false, false>;

template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(const float *part, int splits, MatrixOut o, long rows, int cols)
{
    const int packs = cols / 4;
    for (long i = blockIdx.x * 256l + threadIdx.x; i < rows * packs; i += gridDim.x * 256l) {
        const long m = i / packs;
        const int n = (int)(i % packs) * 4;
        Pack<float, 4> v{};
        for (int s = 0; s < splits; ++s) {
            const auto a = *reinterpret_cast<const Pack<float, 4> *>(part + (s * rows + m) * cols + n);
#pragma unroll
            for (int e = 0; e < 4; ++e) v.v[e] += a.v[e];
        }
        matrix_store<T, 4>(o, m, n, v);
    }
}

__global__ __launch_bounds__(256) void clear_kernel(char *p, long row_bytes, long rows, long stride_bytes)
{
    for (long i = blockIdx.x * 256l + threadIdx.x; i < rows * row_bytes; i += gridDim.x * 256l) p[i / row_bytes * stride_bytes + i % row_bytes] = 0;
}

// ---- plans ---------------------------------------------------------------------------------------------------------

unsigned grid_for(long n) { return (unsigned)std::min((n + 255) / 256, 1l << 16); }

// Up to 64 tokens: straight from memory (gated_few_kernel), whose work on the tokens grows with them, or tiles, which have a join.  bf16, 17, 32 and 64 tokens,
// us: 1024 -> 2816 6.1, 6.8 and 8.9 against 10.5, 10.8 and 11.5; 2048 -> 4096 8.9, 10.2 and 14.2 against 12.3, 12.5 and 13.1; 2048 -> 6144 15.5, 17.8 and 25.5
// against 14.1, 14.7 and 16.0; 4096 -> 16384 57, 64 and 86 against 57, 59 and 63.  fp32 and what has to be copied first would be read and written before tiles.
// The border of 2^23 is the middle of these: just below it 64 tokens lose some 5 %, and more where F is small and with it the number of workgroups
// (4096 -> 2048 15.1, 18.3 and 27.1 against 15.8, 16.2 and 16.9).
bool few_tokens(const ucd_gated_projection_t &d)
{
    return d.M <= 16 || (d.M <= kFewTokens && (d.dtype == 0 || (long)d.D * d.F <= 1l << 23));
}

// What a call has in its workspace, in bytes from its begin; a part of no bytes is not needed.
struct Layout {
    int planes, phases;
    int width;               // a row of x's and the weights' copies
    bool copy_x, copy_w;
    size_t x, wg, wu, dg, part, bytes;
    int half;                // dG's columns of one side
    long dg_row;             // elements from row to row
    long x_plane, w_plane, dg_plane;
    bool few;
    Shape fwd, dx, dw;
};

int wide_of(const ucd_gated_projection_t &d) { return (int)round_up(d.F, 4); }

Layout layout_of(const ucd_gated_projection_t &d, int dir, bool x_aligned, bool w_aligned)
{
    Layout l{};
    const bool f32 = d.dtype == 0;
    l.planes = f32 ? 3 : 1;
    l.phases = f32 ? 6 : 1;
    l.width = (int)round_up(d.D, 8);
    l.half = (int)round_up(d.F, BK);
    l.dg_row = 2l * l.half + BK;      // rows that are a power of two apart meet in few of the caches' channels (dx of 8192 x 2048 x 8192: 870 TFLOP/s against 979)
    l.copy_w = f32 || d.D % 8 != 0 || !w_aligned;
    l.copy_x = f32 || d.D % 8 != 0 || !x_aligned || (d.M > 1 && d.x_m % 8 != 0);
    l.few = few_tokens(d) || (d.M <= kFewTokens && (l.copy_x || l.copy_w));
    size_t at = 0;
    auto take = [&](size_t n) {
        const size_t here = at;
        at += (n + 255) / 256 * 256;
        return here;
    };
    l.x_plane = round_up((long)d.M * l.width, 128);
    l.w_plane = round_up((long)d.F * l.width, 128);
    if (dir == UCD_SEQ_FWD) {
        l.fwd = forward_shape(d.M, d.D, d.F, l.phases);
        if (l.few) {
            l.bytes = 0;
            return l;
        }
    } else {
        l.dx = dx_shape(d.M, d.D, d.F, l.phases);
        l.dw = dw_shape(d.M, d.D, d.F, l.phases);
        l.dg_plane = (long)d.M * l.dg_row;
        l.dg = take((size_t)l.planes * l.dg_plane * 2);
    }
    if (l.copy_x) l.x = take((size_t)l.planes * l.x_plane * 2);
    if (l.copy_w) {
        l.wg = take((size_t)l.planes * l.w_plane * 2);
        l.wu = take((size_t)l.planes * l.w_plane * 2);
    }
    size_t part = 0;
    if (dir == UCD_SEQ_FWD) {
        if (l.fwd.splits > 1) part = (size_t)l.fwd.splits * d.M * 2 * wide_of(d) * 4;
    } else {
        const size_t cols = (size_t)round_up(d.D, 4);
        if (l.dx.splits > 1) part = (size_t)l.dx.splits * d.M * cols * 4;
        if (l.dw.splits > 1) part = std::max(part, (size_t)l.dw.splits * 2 * l.half * cols * 4);
    }
    l.part = take(part);
    l.bytes = at;
    return l;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// x and the weights as operands, copied where they have to be
template <class T>
hipError_t operands(const ucd_gated_projection_t &d, const Layout &l, const void *x, const void *wg, const void *wu, char *ws, Operand &ox, Operand &ow,
                    hipStream_t s)
{
    ox.p[0] = ox.p[1] = (const bf16_t *)x;
    ox.stride = d.x_m;
    ow.p[0] = (const bf16_t *)wg;
    ow.p[1] = (const bf16_t *)wu;
    ow.stride = d.D;
    ox.plane = l.x_plane;
    ow.plane = l.w_plane;
    Copies all{};
    all.cols = d.D;
    all.width = l.width;
    if (l.copy_x) {
        bf16_t *to = (bf16_t *)(ws + l.x);
        ox.p[0] = ox.p[1] = to;
        ox.stride = l.width;
        all.c[all.count++] = Copy{x, (long)d.x_m, d.M, l.x_plane, to};
    }
    if (l.copy_w) {
        bf16_t *gate = (bf16_t *)(ws + l.wg), *up = (bf16_t *)(ws + l.wu);
        ow.p[0] = gate;
        ow.p[1] = up;
        ow.stride = l.width;
        all.c[all.count++] = Copy{wg, d.D, d.F, l.w_plane, gate};
        all.c[all.count++] = Copy{wu, d.D, d.F, l.w_plane, up};
    }
    if (all.count == 0) return hipSuccess;
    const long rows = std::max(l.copy_x ? (long)d.M : 0l, l.copy_w ? (long)d.F : 0l);
    copy_rows_kernel<T><<<dim3(grid_for(rows * (l.width / 8)), (unsigned)all.count), 256, 0, s>>>(all);
    return hipGetLastError();
}

template <class T, int MT, int CT, int AHEAD>
void few_of(const ucd_gated_projection_t &d, const T *x, const T *wg, const T *wu, const GateOut &o, bool whole, hipStream_t s)
{
    const unsigned grid = (unsigned)((d.F + 16 * CT - 1) / (16 * CT));
    if (whole) gated_few_kernel<T, MT, CT, AHEAD, true><<<grid, 64 * kFewWaves, 0, s>>>(x, d.x_m, wg, wu, d.D, o);
    else gated_few_kernel<T, MT, CT, 1, false><<<grid, 64 * kFewWaves, 0, s>>>(x, d.x_m, wg, wu, d.D, o);
}

template <class T>
hipError_t few(const ucd_gated_projection_t &d, const void *x, const void *wg, const void *wu, const GateOut &o, hipStream_t s)
{
    const T *px = (const T *)x, *pg = (const T *)wg, *pu = (const T *)wu;
    const bool whole = d.D * sizeof(T) % 16 == 0 && (d.M == 1 || d.x_m * sizeof(T) % 4 == 0) && (((uintptr_t)x | (uintptr_t)wg | (uintptr_t)wu) & 3u) == 0;
    // 32 columns to a workgroup read the tokens half as often as 16, but need enough of them: 2048 -> 8192, 32 and 64 tokens, 17.2 and 23.0 us against 19.7 and
    // 28.9 (two turns ahead)
    const bool two = d.F >= 32 * kUnits;
    // two turns ahead pay for one token where there are many: rows of 4096, 6144 and 8192 -> 8192, bf16, 25.9, 36.2 and 53.1 us against 28.0, 37.6 and 56.0 (fp32 of
    // half as many the same), and make no difference to 16 tokens.  Of fewer or an odd number the last is empty: 1024, 1536 and 2560 10.0, 13.1 and 18.8 against
    // 9.0, 11.9 and 17.5; at the border, 2048, 14.8 against 15.7 from memory, 13.4 against 12.6 where the card's cache has part of it.
    if (d.M <= 16 && d.D * sizeof(T) <= 4096) few_of<T, 1, 1, 1>(d, px, pg, pu, o, whole, s);
    else if (d.M <= 16) few_of<T, 1, 1, 2>(d, px, pg, pu, o, whole, s);
    else if (d.M <= 32 && two) few_of<T, 2, 2, 1>(d, px, pg, pu, o, whole, s);
    else if (d.M <= 32) few_of<T, 2, 1, 1>(d, px, pg, pu, o, whole, s);
    else if (two) few_of<T, 4, 2, 1>(d, px, pg, pu, o, whole, s);
    else few_of<T, 4, 1, 1>(d, px, pg, pu, o, whole, s);
    return hipGetLastError();
}

template <class T, class TILE>
hipError_t forward(const Problem &p, const GateOut &o, float *part, hipStream_t s)
{
    gated_forward_kernel<TILE, T><<<dim3((unsigned)(p.tiles_m * p.tiles_n), (unsigned)p.splits), TILE::THREADS, 0, s>>>(p, o, part);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part) return e;
    gated_join_kernel<T><<<grid_for((long)o.M * (o.wide / 4)), 256, 0, s>>>(part, p.splits, o);
    return hipGetLastError();
}

template <class T, class TILE>
hipError_t multiply(const Problem &p, const MatrixOut &o, float *part, long rows, hipStream_t s)
{
    const int cols = (int)round_up(o.cols, 4);
    product_kernel<TILE, T><<<dim3((unsigned)(p.tiles_m * p.tiles_n), (unsigned)p.splits), TILE::THREADS, 0, s>>>(p, o, part, rows, cols);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !part) return e;
    product_join_kernel<T><<<grid_for(rows * (cols / 4)), 256, 0, s>>>(part, p.splits, o, rows, cols);
    return hipGetLastError();
}

void shape_into(Problem &p, const Shape &s)
{
    p.tiles_m = s.tiles_m;
    p.tiles_n = s.tiles_n;
    p.splits = s.splits;
}

template <class T>
hipError_t fwd(const ucd_gated_projection_t &d, const void *x, const void *wg, const void *wu, const GateOut &o, char *ws, hipStream_t s)
{
    const Layout l = layout_of(d, UCD_SEQ_FWD, aligned16(x), aligned16(wg) && aligned16(wu));
    if (l.few) return few<T>(d, x, wg, wu, o, s);
    Problem p{};
    const hipError_t e = operands<T>(d, l, x, wg, wu, ws, p.m, p.n, s);
    if (e != hipSuccess) return e;
    p.m.rows = d.M;
    p.n.rows = d.F;
    p.m.k = p.n.k = l.width;
    p.k_tiles = (l.width + BK - 1) / BK;
    p.phases = l.phases;
    shape_into(p, l.fwd);
    float *part = p.splits > 1 ? (float *)(ws + l.part) : nullptr;
    if (l.fwd.side == 256) return forward<T, Tile<T, 256, 256, 2, 4, 2, true, true, true>>(p, o, part, s);
    if (l.fwd.side == 192) return forward<T, Tile<T, 192, 256, 2, 4, 2, true, true, true>>(p, o, part, s);
    if (l.fwd.side == 64) return forward<T, Tile<T, 64, 128, 2, 2, 2, true, true, true>>(p, o, part, s);
    return forward<T, Tile<T, 128, 128, 2, 2, 2, true, true, true>>(p, o, part, s);
}

template <class T>
hipError_t bwd(const ucd_gated_projection_t &d, const void *x, const void *wg, const void *wu, const void *dy, const GateOut &o, void *dx, void *dwg,
               void *dwu, bool add, char *ws, hipStream_t s)
{
    const Layout l = layout_of(d, UCD_SEQ_BWD, aligned16(x), aligned16(wg) && aligned16(wu));
    Operand ox{}, ow{}, og{};
    hipError_t e = operands<T>(d, l, x, wg, wu, ws, ox, ow, s);
    if (e != hipSuccess) return e;
    gated_gradient_kernel<T><<<grid_for((long)d.M * (l.half / 8)), 256, 0, s>>>((const T *)dy, d.y_m, o.saved, o, l.half, l.dg_row, (bf16_t *)(ws + l.dg), l.dg_plane);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    og.p[0] = og.p[1] = (const bf16_t *)(ws + l.dg);
    og.stride = l.dg_row;
    og.plane = l.dg_plane;
    // dx = dG [Wg; Wu]: dG along its rows, the weights across
    Problem p{};
    p.m = og;
    p.m.rows = d.M;
    p.m.k = 2 * l.half;
    p.n = ow;
    p.n.rows = l.width;
    p.n.k = d.F;
    p.n.half = l.half;
    p.k_tiles = 2 * l.half / BK;
    p.phases = l.phases;
    shape_into(p, l.dx);
    MatrixOut out{};
    out.p[0] = out.p[1] = dx;
    out.stride = d.x_m;
    out.rows = d.M;
    out.half = 1l << 40;
    out.cols = d.D;
    float *part = p.splits > 1 ? (float *)(ws + l.part) : nullptr;
    e = l.dx.side == 256   ? multiply<T, LargeAlong<T>>(p, out, part, d.M, s)
        : l.dx.side == 192 ? multiply<T, MiddleAlong<T>>(p, out, part, d.M, s)
                           : multiply<T, SmallAlong<T>>(p, out, part, d.M, s);
    if (e != hipSuccess) return e;
    // [dWg; dWu] = dG^T x: both across
    p.m = og;
    p.m.rows = 2 * l.half;
    p.m.k = d.M;
    p.n = ox;
    p.n.rows = l.width;
    p.n.k = d.M;
    p.k_tiles = (d.M + BK - 1) / BK;
    shape_into(p, l.dw);
    out.p[0] = dwg;
    out.p[1] = dwu;
    out.stride = d.D;
    out.rows = d.F;
    out.half = l.half;
    out.add = add;
    part = p.splits > 1 ? (float *)(ws + l.part) : nullptr;
    return l.dw.side == 256 ? multiply<T, LargeAcross<T>>(p, out, part, 2l * l.half, s)
                            : multiply<T, SmallAcross<T>>(p, out, part, 2l * l.half, s);
}

GateOut gate_out(const ucd_gated_projection_t &d, void *y, float *saved)
{
    return GateOut{y, (long)d.y_m, saved, d.M, d.F, wide_of(d), d.act};
}

}  // namespace gated

using namespace gated;

size_t gated_projection_ws_bytes(const ucd_gated_projection_t &d, int dir)
{
    if (d.M == 0) return 0;
    return std::max(layout_of(d, dir, false, false).bytes, layout_of(d, dir, true, true).bytes);      // few tokens that lie askew need none
}

size_t gated_projection_saved_bytes(const ucd_gated_projection_t &d) { return (size_t)d.M * 2 * wide_of(d) * 4; }

bool gated_projection_countable(const ucd_gated_projection_t &d)
{
    // tiles of the smaller kind, 128 by 128 (64 columns of either side): a grid has fewer than 2^32 threads
    const double m = (d.M + 127) / 128, f = (d.F + 63) / 64, c = (d.D + 127) / 128;
    return m * f < 1 << 23 && m * c < 1 << 23 && 2 * f * c < 1 << 23;
}

hipError_t gated_projection_fwd(const ucd_gated_projection_t &d, const void *x, const void *wg, const void *wu, void *y, float *saved, void *ws,
                                hipStream_t s)
{
    const GateOut o = gate_out(d, y, saved);
    return d.dtype == 1 ? fwd<bf16_t>(d, x, wg, wu, o, (char *)ws, s) : fwd<float>(d, x, wg, wu, o, (char *)ws, s);
}

hipError_t gated_projection_bwd(const ucd_gated_projection_t &d, const void *x, const void *wg, const void *wu, const void *dy, const float *saved,
                                void *dx, void *dwg, void *dwu, bool add, void *ws, hipStream_t s)
{
    if (d.M == 0) {
        if (add) return hipSuccess;
        const long bytes = (long)d.F * d.D * (d.dtype == 1 ? 2 : 4);
        clear_kernel<<<grid_for(bytes), 256, 0, s>>>((char *)dwg, bytes, 1, 0);
        clear_kernel<<<grid_for(bytes), 256, 0, s>>>((char *)dwu, bytes, 1, 0);
        return hipGetLastError();
    }
    const GateOut o = gate_out(d, nullptr, const_cast<float *>(saved));
    return d.dtype == 1 ? bwd<bf16_t>(d, x, wg, wu, dy, o, dx, dwg, dwu, add, (char *)ws, s)
                        : bwd<float>(d, x, wg, wu, dy, o, dx, dwg, dwu, add, (char *)ws, s);
}

}  // namespace ucd
