// Group norm with an activation, channels last: Forward and Backward.
//
// Forward reads x and writes y, Backward reads x and dy and writes dx: memory bounds both, and what counts is to read each of them once.  So a group's
// elements stay in registers between the sums and what is made of them, wherever a workgroup can hold them:
//   rows   single positions with groups of up to a few packs per lane: a group to 1 to 64 neighbouring lanes, samples one after the other;
//   slabs  a sample's positions by a strip of neighbouring groups, some hundred bytes of a row, in the registers of one workgroup;
//   parts  what fits neither: a first kernel leaves sums of parts of a group, the second joins them and reads its part again.
// Sums of Forward are means and squares around them (two passes over registers), joined as such: no difference of large numbers is taken.
// The gradients of gamma and beta are sums over positions, which threads keep per channel while they walk, and a join over the workgroups.
// bf16, Forward and Backward, on inputs that change from call to call: rows 8192 x 1 x 2048 in 16 groups 13 us (5.1 TB/s) and 29 (3.5; 4 of it the join);
// slabs 64 x 1024 x 512 in 32 groups with SiLU 39 (3.4) and 67 (3.0): all workgroups read, sum and write at the same time; parts 8 x 4096 x 2000 in one
// group 99 (2.6) and 145 (2.7).  (Figures at the constants below compare two choices on one set of inputs, part of which stays in the card's cache:
// 34 and 58 us for those slabs.)  Few samples are slow: 1 x 1024 x 512 in 32 groups is 8 workgroups of one XCD, 14 us in Forward.
#include <algorithm>

#include "seq.h"
#include "seq_common.hpp"

namespace ucd {
namespace {
using namespace seq;

constexpr int kRowsR = 4;                   // packs of a group per lane at most
// Backward of rows (8192 x 1 x 2048 in 16 groups, bf16): 25.6 us; with 256 threads in 1024 workgroups, and twice the partial sums, 32; with 512 in 2048
// 44; with 1024 in 256 24.5, but 16.9 instead of 16.2 for 512 channels in 4 groups.
constexpr int kRowsBwdThreads = 512, kRowsBwdGroups = 512;
// A slab's threads at most, and packs per thread: as many as fill 32 registers of the 128 that a thread has then (and 32 of dy in Backward), or a quarter.
constexpr int kMaxThreads = 1024;
template <class T, int VE>
constexpr int slab_packs(bool few) { return 32 / Raw<T, VE, true>::WORDS / (few ? 4 : 1); }
// Waves to a SIMD that Forward is built for: two workgroups to a CU, but for full slabs of 16-byte packs, whose weights would go to memory then.
template <class T, int VE, int R>
constexpr int slab_waves() { return R == slab_packs<T, VE>(false) && VE * sizeof(T) == 16 ? 4 : 8; }
inline int slab_packs(int dtype, int VE, bool few) { return 32 / std::max(1, VE / (dtype == 1 ? 2 : 1)) / (few ? 4 : 1); }

struct NormParams {
    ucd_group_norm_t d;
    const void *x, *dy;
    const float *gamma, *beta;
    const float *stats_in;
    void *y, *dx;
    float *stats;
    float *part;                 // Backward: [part_rows][2][C], sums of dgamma and dbeta
    float *sums;                 // parts: [N][chunks][G * cs][2]: Forward mean and squares around it, Backward the two sums of dx
    float *dgamma, *dbeta;
    bool add;
    int cg, pgl;                 // channels and packs of a group
    float share;                 // 1 / a group's elements
    int part_rows;               // rows of workgroups that share out the samples
    // rows
    int lanes, gx, ry, columns;  // lanes to a group; groups and samples of a workgroup; workgroups for all groups
    // slabs, parts
    int px, py, strips;          // packs of a strip, positions of a pass; strips of a row
    unsigned unit0;              // slabs: a launch's first workgroup
    int gps, cs;                 // groups of a strip, or strips of a group
    int chunk, chunks;           // positions of a part, parts of a sample's positions
    bool in_wave;                // strips and their groups are powers of two of lanes
};

template <class T, int VE>
__device__ __forceinline__ void load_f(float (&v)[VE], const Raw<T, VE, true> &r)
{
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = r.get(i);
}

template <int VE>
__device__ __forceinline__ void load_weights(float (&v)[VE], const float *at)
{
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = at[i];
}

// 1 / sqrt(v); the unit takes numbers below the smallest normal one for 0.
__device__ __forceinline__ float inverse_root(float v)
{
    const bool tiny = v < 0x1p-100f;
    return __builtin_amdgcn_rsqf(tiny ? v * 0x1p100f : v) * (tiny ? 0x1p50f : 1.f);
}

// y of one pack
template <bool SILU, class T, int VE>
__device__ __forceinline__ Pack<T, VE> norm_pack(const Raw<T, VE, true> &r, float mean, float rstd, const float (&gamma)[VE], const float (&beta)[VE])
{
    Pack<T, VE> out;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        float u = fmaf((r.get(i) - mean) * rstd, gamma[i], beta[i]);
        if (SILU) u *= sigmoid(u);
        out.v[i] = from_f<T>(u);
    }
    return out;
}

// xhat and du = dy act'(u) of one element
template <bool SILU>
__device__ __forceinline__ float norm_du(float xhat, float dy, float gamma, float beta)
{
    if (!SILU) return dy;
    const float u = fmaf(xhat, gamma, beta), s = sigmoid(u);
    return dy * s * fmaf(u, 1.f - s, 1.f);
}

template <bool SILU, class T, int VE>
__device__ __forceinline__ Pack<T, VE> dx_pack(const Raw<T, VE, true> &x, const Raw<T, VE, true> &dy, float mean, float rstd, float m1, float m2,
                                               const float (&gamma)[VE], const float (&beta)[VE])
{
    Pack<T, VE> out;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
        // rounded as in the sums m1 is made of: of a group of one element nothing must be left
#pragma clang fp contract(off)
        const float xhat = (x.get(i) - mean) * rstd, g = norm_du<SILU>(xhat, dy.get(i), gamma[i], beta[i]) * gamma[i];
        out.v[i] = from_f<T>(rstd * fmaf(-xhat, m2, g - m1));
    }
    return out;
}

// ---- rows ----------------------------------------------------------------------------------------------------------------------------------------

// A lane's group and its R packs of it.  A group's last pack is moved back to the group's end, where its first elements are the pack's before it too:
// they are left out of sums over the group, and what becomes of them comes out twice, the same.
template <int VE, int R>
struct RowPlace {
    int lane, g, row;
    int own[R];                 // the pack's first element that no other has; VE: there is no pack
    bool active, have[R];
    __device__ __forceinline__ RowPlace(const NormParams &p)
    {
        const int group = threadIdx.x / p.lanes;
        lane = threadIdx.x % p.lanes;
        g = blockIdx.x % p.columns * p.gx + group % p.gx;
        row = group / p.gx;
        active = row < p.ry && g < p.d.G;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            have[i] = active && lane + i * p.lanes < p.pgl;
            own[i] = have[i] ? max(0, (lane + i * p.lanes + 1) * VE - p.cg) : VE;
        }
    }
    __device__ __forceinline__ int channel(const NormParams &p, int i) const { return g * p.cg + min((lane + i * p.lanes) * VE, p.cg - VE); }
};

template <bool SILU, class T, int VE, int R>
__global__ __launch_bounds__(256) void norm_rows_fwd_kernel(NormParams p)
{
    const RowPlace<VE, R> at(p);
    float gamma[R][VE], beta[R][VE];
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (at.have[i]) {
            load_weights<VE>(gamma[i], p.gamma + at.channel(p, i));
            load_weights<VE>(beta[i], p.beta + at.channel(p, i));
        }
    const int step = p.part_rows * p.ry;
    Raw<T, VE, true> next[R], r[R];
    auto load = [&](int n) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (at.have[i]) next[i].load((const char *)((const T *)p.x + n * p.d.x_n + at.channel(p, i)), 0, VE);
    };
    // a workgroup's samples are side by side: all of its lanes go round as often
    const int n0 = blockIdx.x / p.columns * p.ry;
    if (n0 + at.row < p.d.N) load(n0 + at.row);
    for (int base = n0; base < p.d.N; base += step) {
        const int n = base + at.row;
        const bool there = n < p.d.N;
#pragma unroll
        for (int i = 0; i < R; ++i) r[i] = next[i];
        if (step < p.d.N - n) load(n + step);
        float sum = 0.f, sq = 0.f;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) sum += e >= at.own[i] ? r[i].get(e) : 0.f;
        const float mean = sum_group(sum, p.lanes) * p.share;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float v = r[i].get(e) - mean;
                sq += e >= at.own[i] ? v * v : 0.f;
            }
        const float rstd = inverse_root(fmaf(sum_group(sq, p.lanes), p.share, p.d.eps));
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (at.have[i] && there)
                loose_store<T, VE>((T *)p.y + n * p.d.y_n + at.channel(p, i), norm_pack<SILU, T, VE>(r[i], mean, rstd, gamma[i], beta[i]));
        if (p.stats && at.active && there && at.lane == 0) {
            p.stats[(long)n * p.d.G + at.g] = mean;
            p.stats[((long)p.d.N + n) * p.d.G + at.g] = rstd;
        }
    }
}

template <bool SILU, class T, int VE, int R>
__global__ __launch_bounds__(kRowsBwdThreads) void norm_rows_bwd_kernel(NormParams p)
{
    __shared__ float lds[kRowsBwdThreads];
    const RowPlace<VE, R> at(p);
    float gamma[R][VE], beta[R][VE], dg[R][VE] = {}, db[R][VE] = {};
    const int step = p.part_rows * p.ry, part_row = blockIdx.x / p.columns;
    {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (at.have[i]) {
                load_weights<VE>(gamma[i], p.gamma + at.channel(p, i));
                load_weights<VE>(beta[i], p.beta + at.channel(p, i));
            }
        Raw<T, VE, true> xn[R], gn[R], x[R], dy[R];
        float next_mean = 0.f, next_rstd = 0.f;
        auto load = [&](int n) {
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (at.have[i]) {
                    xn[i].load((const char *)((const T *)p.x + n * p.d.x_n + at.channel(p, i)), 0, VE);
                    gn[i].load((const char *)((const T *)p.dy + n * p.d.y_n + at.channel(p, i)), 0, VE);
                }
            if (!at.active) return;
            next_mean = p.stats_in[(long)n * p.d.G + at.g];
            next_rstd = p.stats_in[((long)p.d.N + n) * p.d.G + at.g];
        };
        const int n0 = part_row * p.ry;
        if (n0 + at.row < p.d.N) load(n0 + at.row);
        for (int base = n0; base < p.d.N; base += step) {
            const int n = base + at.row;
            const bool there = n < p.d.N;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                x[i] = xn[i];
                dy[i] = gn[i];
            }
            const float mean = next_mean, rstd = next_rstd;
            if (step < p.d.N - n) load(n + step);
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (!at.have[i] || !there) continue;
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float xhat = (x[i].get(e) - mean) * rstd, du = norm_du<SILU>(xhat, dy[i].get(e), gamma[i][e], beta[i][e]);
                    db[i][e] += du;
                    dg[i][e] = fmaf(du, xhat, dg[i][e]);
                    const float g = e >= at.own[i] ? du * gamma[i][e] : 0.f;
                    s1 += g;
                    s2 = fmaf(g, xhat, s2);
                }
            }
            s1 = sum_group(s1, p.lanes) * p.share;
            s2 = sum_group(s2, p.lanes) * p.share;
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (at.have[i] && there)
                    loose_store<T, VE>((T *)p.dx + n * p.d.x_n + at.channel(p, i),
                                       dx_pack<SILU, T, VE>(x[i], dy[i], mean, rstd, s1, s2, gamma[i], beta[i]));
        }
    }
    // over the samples side by side in the workgroup, in their order
    const int apart = p.gx * p.lanes;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float v = k ? db[i][e] : dg[i][e];
                if (p.ry > 1) {
                    __syncthreads();
                    lds[threadIdx.x] = v;
                    __syncthreads();
                    if (at.row == 0)
                        for (int r = 1; r < p.ry; ++r) v += lds[threadIdx.x + r * apart];
                }
                if (at.have[i] && at.row == 0) p.part[((long)part_row * 2 + k) * p.d.C + at.channel(p, i) + e] = v;
            }
}

// ---- slabs and parts -----------------------------------------------------------------------------------------------------------------------------

// Workgroups are dealt to the chip's 8 XCDs in turn, each of which has an L2 of its own: the strips of a sample, whose rows meet inside cache lines, go to
// the same one.  The grid is whole rounds of 8 samples (or rows of samples); false for those that there are not.
constexpr unsigned kXcds = 8;

__device__ __forceinline__ bool strip_of(unsigned block, int strips, int rows, int &strip, int &row)
{
    const unsigned k = block / kXcds;
    strip = (int)(k % (unsigned)strips);
    row = (int)(k / (unsigned)strips * kXcds + block % kXcds);
    return row < rows;
}

// The first channel of a group's k-th pack; the last is moved back to the group's end, as in rows.
template <int VE>
__device__ __forceinline__ int pack_channel(const NormParams &p, int g, int k)
{
    return g * p.cg + min(k * VE, p.cg - VE);
}

// A thread's pack of a strip and its positions.
template <int VE>
struct SlabPlace {
    int strip, local, g, c0, ty;     // local: the group within the strip
    int own;                         // as in rows; only where groups are no whole packs
    bool active;
    __device__ __forceinline__ SlabPlace(const NormParams &p, int strip_) : strip(strip_)
    {
        const int tx = threadIdx.x % p.px;
        ty = threadIdx.x / p.px;
        active = ty < p.py;
        int k;
        if (p.cs > 1) {
            k = strip % p.cs * p.px + tx;
            g = strip / p.cs;
            local = 0;
            active = active && k < p.pgl;
        } else {
            local = tx / p.pgl;       // < gps
            k = tx % p.pgl;
            g = strip * p.gps + local;
            active = active && g < p.d.G;
        }
        c0 = pack_channel<VE>(p, g, k);
        own = max(0, (k + 1) * VE - p.cg);
    }
};

// Sums over a workgroup's threads of one group, for each of its groups; in every thread that of its own.
__device__ __forceinline__ float2 sum_slab(const NormParams &p, float a, float b, bool active, int local)
{
    __shared__ float2 lds[kMaxThreads], res[kMaxThreads];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
    float2 v = active ? make_float2(a, b) : make_float2(0.f, 0.f);
    if (p.in_wave) {
        // a wave's lanes are whole rows of the strip: over its rows, then over a group's packs, then over the waves
        v.x = sum_group(sum_apart(v.x, p.px), p.pgl);
        v.y = sum_group(sum_apart(v.y, p.px), p.pgl);
        if (waves == 1) return v;
        if (lane < p.px && lane % p.pgl == 0) lds[wave * p.gps + local] = v;
        __syncthreads();
        // 16 lanes to a group, one to a wave's sum
        for (int j = 4 * wave + lane / 16; j - lane / 16 < p.gps; j += 4 * waves) {
            float2 o = make_float2(0.f, 0.f);
            if (lane % 16 < waves && j < p.gps) o = lds[lane % 16 * p.gps + j];
            o.x = sum_lanes<16>(o.x);
            o.y = sum_lanes<16>(o.y);
            if (lane % 16 == 0 && j < p.gps) res[j] = o;
        }
        __syncthreads();
        return res[local];
    }
    lds[threadIdx.x] = v;
    __syncthreads();
    const int groups = p.cs > 1 ? 1 : p.gps, width = p.cs > 1 ? p.px : p.pgl, count = width * p.py;
    for (int j = wave; j < groups; j += waves) {
        v = make_float2(0.f, 0.f);
        for (int i = lane; i < count; i += 64) {
            const float2 w = lds[i / width * p.px + j * width + i % width];
            v.x += w.x;
            v.y += w.y;
        }
        v.x = sum_group(v.x, 64);
        v.y = sum_group(v.y, 64);
        if (lane == 0) res[j] = v;
    }
    __syncthreads();
    return res[active ? local : 0];
}

// One pass over a thread's positions: f(i, there, q), q the place of its pack in a tensor.  Position and place are made opaque at the start, or the compiler
// keeps those of all passes, 3 registers for each of up to 32 packs, from the first pass to the last.
template <class T, int R, class F>
__device__ __forceinline__ void slab_pass(const void *tensor, long sn, long ss, const NormParams &p, bool active, int ty, int c0, int n, int s0, int count, F f)
{
    T *q = (T *)tensor + n * sn + (long)(s0 + ty) * ss + c0;
    const long stride = p.py * ss;
    int s = active ? ty : count;
    asm volatile("" : "+v"(s), "+v"(q));
#pragma unroll
    for (int i = 0; i < R; ++i) {
        f(i, s < count, q);
        s += p.py;
        q += stride;
    }
}

template <class T, int VE, int R>
struct Slab {
    Raw<T, VE, true> r[R];
    // The words as they are: floats made of them before are made again behind this, instead of being kept beside them from one pass to the next.
    __device__ __forceinline__ void fresh()
    {
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int k = 0; k < Raw<T, VE, true>::WORDS; ++k) asm volatile("" : "+v"(r[i].w[k]));
    }
    // positions that are not there as zeros
    __device__ __forceinline__ void load(const void *base, long sn, long ss, const NormParams &p, const SlabPlace<VE> &at, int n, int s0, int count)
    {
        slab_pass<T, R>(base, sn, ss, p, at.active, at.ty, at.c0, n, s0, count, [&](int i, bool there, const T *q) {
#pragma unroll
            for (int k = 0; k < Raw<T, VE, true>::WORDS; ++k) r[i].w[k] = 0;
            if (there) r[i].load((const char *)q, 0, VE);
        });
    }
};

// A part's mean and the squares around it, in every thread of its group.
template <bool TAIL, class T, int VE, int R>
__device__ __forceinline__ float2 slab_moments(const NormParams &p, Slab<T, VE, R> &x, const SlabPlace<VE> &at, int count, float share)
{
    float sum = 0.f, sq = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
        for (int e = 0; e < VE; ++e) sum += !TAIL || e >= at.own ? x.r[i].get(e) : 0.f;
    const float mean = sum_slab(p, sum, 0.f, at.active, at.local).x * share;
    x.fresh();
    int s = at.ty;
    asm volatile("" : "+v"(s));
#pragma unroll
    for (int i = 0; i < R; ++i, s += p.py) {
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float v = !TAIL || e >= at.own ? x.r[i].get(e) - mean : 0.f;
            part = fmaf(v, v, part);
        }
        sq += s < count ? part : 0.f;
    }
    x.fresh();
    return make_float2(mean, sum_slab(p, sq, 0.f, at.active, at.local).x);
}

template <bool SILU, class T, int VE, int R>
__device__ __forceinline__ void slab_store_y(const NormParams &p, const Slab<T, VE, R> &x, const SlabPlace<VE> &at, int n, int s0, int count, float mean,
                                             float rstd, const float (&gamma)[VE], const float (&beta)[VE])
{
    slab_pass<T, R>(p.y, p.d.y_n, p.d.y_s, p, at.active, at.ty, at.c0, n, s0, count, [&](int i, bool there, T *q) {
        const Pack<T, VE> out = norm_pack<SILU, T, VE>(x.r[i], mean, rstd, gamma, beta);
        if (there) loose_store<T, VE>(q, out);
    });
}

// The first thread of each group of a workgroup.
template <int VE>
__device__ __forceinline__ bool leads(const NormParams &p, const SlabPlace<VE> &at)
{
    return at.active && at.ty == 0 && (p.cs > 1 ? threadIdx.x == 0 : threadIdx.x % p.px == at.local * p.pgl);
}

template <bool SILU, bool TAIL, class T, int VE, int R>
__global__ __launch_bounds__(kMaxThreads, (slab_waves<T, VE, R>())) void norm_slab_fwd_kernel(NormParams p)
{
    int strip, first;
    if (!strip_of(p.unit0 + blockIdx.x, p.strips, p.part_rows, strip, first)) return;
    const SlabPlace<VE> at(p, strip);
    for (int n = first; n < p.d.N; n += p.part_rows) {
        Slab<T, VE, R> x;
        x.load(p.x, p.d.x_n, p.d.x_s, p, at, n, 0, p.d.S);
        const float2 m = slab_moments<TAIL, T, VE, R>(p, x, at, p.d.S, p.share);
        const float rstd = inverse_root(fmaf(m.y, p.share, p.d.eps));
        float gamma[VE] = {}, beta[VE] = {};
        if (at.active) {
            load_weights<VE>(gamma, p.gamma + at.c0);
            load_weights<VE>(beta, p.beta + at.c0);
        }
        slab_store_y<SILU, T, VE, R>(p, x, at, n, 0, p.d.S, m.x, rstd, gamma, beta);
        if (p.stats && leads<VE>(p, at)) {
            p.stats[(long)n * p.d.G + at.g] = m.x;
            p.stats[((long)p.d.N + n) * p.d.G + at.g] = rstd;
        }
    }
}

// The two sums of dx over a part of a sample, and per-channel sums on top of dg, db.  (x and dy of positions that are not there are 0, and so is du.)
template <bool SILU, bool TAIL, class T, int VE, int R>
__device__ __forceinline__ float2 slab_grads(const NormParams &p, Slab<T, VE, R> &x, Slab<T, VE, R> &dy, const SlabPlace<VE> &at, float mean, float rstd,
                                             const float (&gamma)[VE], const float (&beta)[VE], float (&dg)[VE], float (&db)[VE])
{
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float xhat = (x.r[i].get(e) - mean) * rstd, du = norm_du<SILU>(xhat, dy.r[i].get(e), gamma[e], beta[e]);
            db[e] += du;
            dg[e] = fmaf(du, xhat, dg[e]);
            const float weight = !TAIL || e >= at.own ? gamma[e] : 0.f;
            s1 = fmaf(du, weight, s1);
            s2 = fmaf(du * weight, xhat, s2);
            // now: the compiler would add up all du and du xhat behind the sums s1, s2, and keep them until then
            asm volatile("" : "+v"(db[e]), "+v"(dg[e]));
        }
    }
    x.fresh();
    dy.fresh();
    return sum_slab(p, s1, s2, at.active, at.local);
}

template <bool SILU, class T, int VE, int R>
__device__ __forceinline__ void slab_store_dx(const NormParams &p, const Slab<T, VE, R> &x, const Slab<T, VE, R> &dy, const SlabPlace<VE> &at, int n, int s0,
                                              int count, float mean, float rstd, float m1, float m2, const float (&gamma)[VE], const float (&beta)[VE])
{
    slab_pass<T, R>(p.dx, p.d.x_n, p.d.x_s, p, at.active, at.ty, at.c0, n, s0, count, [&](int i, bool there, T *q) {
        const Pack<T, VE> out = dx_pack<SILU, T, VE>(x.r[i], dy.r[i], mean, rstd, m1, m2, gamma, beta);
        if (there) loose_store<T, VE>(q, out);
    });
}

// A row of the partial sums of dgamma and dbeta: over the threads of a channel, in a fixed order; within a wave first, where its lanes hold whole rows of
// the strip.
template <int VE>
__device__ __forceinline__ void slab_store_part(const NormParams &p, const SlabPlace<VE> &at, long part_row, float (&dg)[VE], float (&db)[VE])
{
    __shared__ float2 lds[VE][kMaxThreads];
    const bool in_wave = p.px <= 64 && (p.px & (p.px - 1)) == 0;
    if (in_wave)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            dg[e] = sum_apart(dg[e], p.px);
            db[e] = sum_apart(db[e], p.px);
        }
    const int lane = threadIdx.x % 64, slot = in_wave ? (int)threadIdx.x / 64 * p.px + lane : (int)threadIdx.x;
    if (!in_wave || lane < p.px)
#pragma unroll
        for (int e = 0; e < VE; ++e) lds[e][slot] = make_float2(dg[e], db[e]);
    __syncthreads();
    const int rows = in_wave ? (int)blockDim.x / 64 : p.py;
    for (int i = threadIdx.x; i < p.px * VE; i += blockDim.x) {
        const int pack = i / VE, e = i % VE;
        const int g = p.cs > 1 ? at.strip / p.cs : at.strip * p.gps + pack / p.pgl, k = p.cs > 1 ? at.strip % p.cs * p.px + pack : pack % p.pgl;
        if (g >= p.d.G || k >= p.pgl) continue;
        float2 v = lds[e][pack];
        for (int r = 1; r < rows; ++r) {
            const float2 w = lds[e][r * p.px + pack];
            v.x += w.x;
            v.y += w.y;
        }
        const long c = pack_channel<VE>(p, g, k) + e;
        p.part[part_row * 2 * p.d.C + c] = v.x;
        p.part[(part_row * 2 + 1) * p.d.C + c] = v.y;
    }
    __syncthreads();
}

template <bool SILU, bool TAIL, class T, int VE, int R>
__global__ __launch_bounds__(kMaxThreads) void norm_slab_bwd_kernel(NormParams p)
{
    int strip, part_row;
    if (!strip_of(p.unit0 + blockIdx.x, p.strips, p.part_rows, strip, part_row)) return;
    const SlabPlace<VE> at(p, strip);
    float gamma[VE] = {}, beta[VE] = {}, dg[VE] = {}, db[VE] = {};
    if (at.active) {
        load_weights<VE>(gamma, p.gamma + at.c0);
        load_weights<VE>(beta, p.beta + at.c0);
    }
    for (int n = part_row; n < p.d.N; n += p.part_rows) {
        Slab<T, VE, R> x, dy;
        x.load(p.x, p.d.x_n, p.d.x_s, p, at, n, 0, p.d.S);
        dy.load(p.dy, p.d.y_n, p.d.y_s, p, at, n, 0, p.d.S);
        const float mean = at.active ? p.stats_in[(long)n * p.d.G + at.g] : 0.f, rstd = at.active ? p.stats_in[((long)p.d.N + n) * p.d.G + at.g] : 0.f;
        const float2 s = slab_grads<SILU, TAIL, T, VE, R>(p, x, dy, at, mean, rstd, gamma, beta, dg, db);
        slab_store_dx<SILU, T, VE, R>(p, x, dy, at, n, 0, p.d.S, mean, rstd, s.x * p.share, s.y * p.share, gamma, beta);
    }
    slab_store_part<VE>(p, at, part_row, dg, db);
}

// Channels of a group's part k of p.cs.
template <int VE>
__device__ __forceinline__ int part_channels(const NormParams &p, int k)
{
    return p.cs > 1 ? min(p.px * VE, p.cg - k * p.px * VE) : p.cg;
}

// Parts, first kernel: moments, or the sums of dx and those of dgamma and dbeta, of one part.
template <bool SILU, bool TAIL, class T, int VE, int R, bool BACKWARD>
__global__ __launch_bounds__(kMaxThreads, BACKWARD || VE * sizeof(T) == 16 ? 4 : 8) void norm_part_kernel(NormParams p, unsigned units)
{
    for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int strip, row;                                             // row: sample and chunk
        if (!strip_of(unit, p.strips, p.part_rows, strip, row)) continue;
        const SlabPlace<VE> at(p, strip);
        const int n = row / p.chunks, s0 = row % p.chunks * p.chunk, count = min(p.chunk, p.d.S - s0);
        Slab<T, VE, R> x, dy;
        x.load(p.x, p.d.x_n, p.d.x_s, p, at, n, s0, count);
        float2 out;
        if (BACKWARD) {
            dy.load(p.dy, p.d.y_n, p.d.y_s, p, at, n, s0, count);
            float gamma[VE] = {}, beta[VE] = {}, dg[VE] = {}, db[VE] = {}, mean = 0.f, rstd = 0.f;
            if (at.active) {
                load_weights<VE>(gamma, p.gamma + at.c0);
                load_weights<VE>(beta, p.beta + at.c0);
                mean = p.stats_in[(long)n * p.d.G + at.g];
                rstd = p.stats_in[((long)p.d.N + n) * p.d.G + at.g];
            }
            out = slab_grads<SILU, TAIL, T, VE, R>(p, x, dy, at, mean, rstd, gamma, beta, dg, db);
            slab_store_part<VE>(p, at, row, dg, db);
        } else {
            out = slab_moments<TAIL, T, VE, R>(p, x, at, count, 1.f / ((float)count * part_channels<VE>(p, strip % p.cs)));
        }
        if (leads<VE>(p, at)) {
            float *to = p.sums + 2 * ((long)row * p.d.G * p.cs + (p.cs > 1 ? at.strip : at.g));
            to[0] = out.x;
            to[1] = out.y;
        }
        __syncthreads();
    }
}

// The parts of a group joined, by one wave: Forward the mean of the means, weighted by their elements, and all squares around it.
template <int VE, bool BACKWARD>
__device__ __forceinline__ float2 join_parts(const NormParams &p, int n, int g)
{
    const int lane = threadIdx.x % 64, parts = p.chunks * p.cs;
    auto at = [&](int i) { return p.sums + 2 * (((long)n * p.chunks + i / p.cs) * p.d.G * p.cs + (long)g * p.cs + i % p.cs); };
    auto elements = [&](int i) {
        return (float)min(p.chunk, p.d.S - i / p.cs * p.chunk) * part_channels<VE>(p, i % p.cs);
    };
    float2 v = make_float2(0.f, 0.f);
    for (int i = lane; i < parts; i += 64) {
        const float *s = at(i);
        v.x += BACKWARD ? s[0] : s[0] * (elements(i) * p.share);
        v.y += BACKWARD ? s[1] : 0.f;
    }
    v.x = sum_group(v.x, 64);
    v.y = sum_group(v.y, 64);
    if (BACKWARD) return make_float2(v.x * p.share, v.y * p.share);
    for (int i = lane; i < parts; i += 64) {
        const float *s = at(i), off = s[0] - v.x;
        v.y += s[1] + off * off * elements(i);
    }
    v.y = sum_group(v.y, 64);
    return make_float2(v.x, inverse_root(fmaf(v.y, p.share, p.d.eps)));
}

// Parts, second kernel: y or dx of one part.
template <bool SILU, class T, int VE, int R, bool BACKWARD>
__global__ __launch_bounds__(kMaxThreads, BACKWARD || VE * sizeof(T) == 16 ? 4 : 8) void norm_apply_kernel(NormParams p, unsigned units)
{
    __shared__ float2 lds[kMaxThreads];
    const int wave = threadIdx.x / 64, waves = blockDim.x / 64;
    for (unsigned unit = blockIdx.x; unit < units; unit += gridDim.x) {
        int strip, row;
        if (!strip_of(unit, p.strips, p.part_rows, strip, row)) continue;
        const SlabPlace<VE> at(p, strip);
        const int n = row / p.chunks, s0 = row % p.chunks * p.chunk, count = min(p.chunk, p.d.S - s0);
        Slab<T, VE, R> x, dy;
        x.load(p.x, p.d.x_n, p.d.x_s, p, at, n, s0, count);
        if (BACKWARD) dy.load(p.dy, p.d.y_n, p.d.y_s, p, at, n, s0, count);
        const int g0 = p.cs > 1 ? at.strip / p.cs : at.strip * p.gps, groups = p.cs > 1 ? 1 : min(p.gps, p.d.G - g0);
        for (int j = wave; j < groups; j += waves) {
            const float2 v = join_parts<VE, BACKWARD>(p, n, g0 + j);
            if (threadIdx.x % 64 == 0) lds[j] = v;
        }
        __syncthreads();
        const float2 m = lds[at.active ? at.local : 0];
        if (at.active) {
            float gamma[VE], beta[VE];
            load_weights<VE>(gamma, p.gamma + at.c0);
            load_weights<VE>(beta, p.beta + at.c0);
            if (BACKWARD) {
                const float mean = p.stats_in[(long)n * p.d.G + at.g], rstd = p.stats_in[((long)p.d.N + n) * p.d.G + at.g];
                slab_store_dx<SILU, T, VE, R>(p, x, dy, at, n, s0, count, mean, rstd, m.x, m.y, gamma, beta);
            } else {
                slab_store_y<SILU, T, VE, R>(p, x, at, n, s0, count, m.x, m.y, gamma, beta);
                if (p.stats && s0 == 0 && leads<VE>(p, at) && (p.cs == 1 || at.strip % p.cs == 0)) {
                    p.stats[(long)n * p.d.G + at.g] = m.x;
                    p.stats[((long)p.d.N + n) * p.d.G + at.g] = m.y;
                }
            }
        }
        __syncthreads();
    }
}

__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(NormParams p)
{
    join_columns(p.part, p.part_rows, 2l * p.d.C, [&](long i, float v) {
        float *out = i < p.d.C ? p.dgamma + i : p.dbeta + (i - p.d.C);
        *out = v + (p.add ? *out : 0.f);
    });
}

// ---- which way, and how it is divided ------------------------------------------------------------------------------------------------------------

// Strips of 64 bytes: 34 us instead of 35 in Forward, 61 instead of 59 in Backward (64 x 1024 x 512, bf16, 32 groups), but 30 instead of 23 and 59
// instead of 38 where rows are no whole lines (37 x 1305 x 231, fp32, 77 groups); of 256 bytes: the same within 1 us.
constexpr int kStripBytes = 128;
// Slabs below 1024 packs are widened (2048 x 16 x 512, bf16, 32 groups: 20 and 37 us, 31 and 76 as they are); to 4096 where that leaves 1024 workgroups
// (256 x 49 x 2048, 32 groups: Forward 27 us instead of 33; 256 x 196 x 1024: 56 and 100 instead of 66 and 115; but 16 x 196 x 1024, with fewer
// workgroups: 12 and 18 instead of 8 and 14).
constexpr int kWidenPacks = 1024, kWidenMost = 4096, kWidenGroups = 1024;
enum Way { ROWS, SLABS, PARTS };

int ceil_div(long a, long b) { return (int)((a + b - 1) / b); }

// Packs of rows, from any element on; 0: not rows.
int rows_pack(const ucd_group_norm_t &d)
{
    const int cg = d.C / d.G;
    int ve = d.dtype == 1 ? 8 : 4;
    while (ve > cg) ve /= 2;
    return d.S == 1 && ceil_div(cg, ve) <= 64 * kRowsR ? ve : 0;
}

// With packs of VE.
Way divide(const ucd_group_norm_t &d, int VE, bool backward, NormParams &p, int &threads, int &R)
{
    const int e = d.dtype == 1 ? 2 : 4;
    p.d = d;
    p.cg = d.C / d.G;
    p.pgl = ceil_div(p.cg, VE);
    p.share = (float)(1. / ((double)d.S * p.cg));
    if (VE == rows_pack(d)) {
        R = p.pgl <= 64 ? 1 : kRowsR;
        p.lanes = 1;
        while (p.lanes * R < p.pgl) p.lanes *= 2;
        // Backward: larger workgroups, which add up the partial sums of the samples that they take side by side, and no more of them than run at once
        threads = backward ? kRowsBwdThreads : 256;
        const int groups = threads / p.lanes;
        p.gx = std::min(d.G, groups);
        p.ry = std::min(groups / p.gx, d.N);
        p.columns = ceil_div(d.G, p.gx);
        p.part_rows = std::max(1, std::min(ceil_div(d.N, p.ry), (backward ? kRowsBwdGroups : 2048) / p.columns));
        return ROWS;
    }
    // a strip is as many groups as make 128 bytes of a row, fewer down to 32 bytes where their slab would not fit, more where
    // it would be a few waves' work; or a workgroup's part of a group
    const int most = slab_packs(d.dtype, VE, false), few = slab_packs(d.dtype, VE, true);
    p.cs = ceil_div(p.pgl, kMaxThreads);
    p.gps = p.cs > 1 ? 1 : std::min({d.G, std::max(1, ceil_div(kStripBytes, p.cg * e)), kMaxThreads / p.pgl});
    auto fits = [&](int groups) { return (long)ceil_div(d.S, kMaxThreads / (groups * p.pgl)) <= most; };
    if (p.cs == 1 && !fits(p.gps)) {
        int groups = p.gps;
        while (groups > 1 && !fits(groups)) --groups;
        if (fits(groups) && (groups * p.cg * e >= 32 || groups == d.G)) p.gps = groups;
    }
    auto widen = [&] {
        const long packs = (long)d.S * p.gps * p.pgl;
        return packs < kWidenPacks || (packs < kWidenMost && (long)d.N * ceil_div(d.G, 2 * p.gps) >= kWidenGroups);
    };
    while (p.cs == 1 && 2 * p.gps <= d.G && 2 * p.gps * p.pgl <= 64 && widen() && fits(2 * p.gps)) p.gps *= 2;
    p.px = p.cs > 1 ? kMaxThreads : p.gps * p.pgl;
    p.strips = p.cs > 1 ? d.G * p.cs : ceil_div(d.G, p.gps);
    auto power = [](int n) { return (n & (n - 1)) == 0; };
    p.in_wave = p.cs == 1 && p.px <= 64 && power(p.px) && power(p.pgl);
    if (p.cs == 1 && fits(p.gps)) {
        // few packs to a thread while there are threads
        const bool small = (long)d.S * p.px <= (long)kMaxThreads * few;
        threads = 64;
        while (threads < kMaxThreads && (threads < p.px || ceil_div(d.S, threads / p.px) > (small ? few : most))) threads *= 2;
        R = ceil_div(d.S, threads / p.px) <= few ? few : most;
        p.py = threads / p.px;
        // Backward's workgroups leave a row of partial sums each: as many as run at once.  Forward's leave nothing.
        p.part_rows = std::max(1, std::min(d.N, (backward ? 256 * kMaxThreads / threads : 1 << 20) / p.strips));
        return SLABS;
    }
    threads = kMaxThreads;
    R = most;
    p.py = threads / p.px;
    p.chunk = std::min(d.S, p.py * R);
    p.chunks = ceil_div(d.S, p.chunk);
    p.part_rows = d.N * p.chunks;
    return PARTS;
}

size_t ws_bytes(const ucd_group_norm_t &d, int VE, int dir)
{
    NormParams p{};
    int threads, R;
    const Way way = divide(d, VE, dir == UCD_SEQ_BWD, p, threads, R);
    size_t n = dir == UCD_SEQ_BWD ? (size_t)8 * p.part_rows * d.C : 0;
    if (way == PARTS) n += (size_t)8 * d.N * p.chunks * d.G * p.cs;
    return n;
}

// Packs: those of rows, or the largest up to 16 bytes that hold a group in 1.3 times its elements (17 bf16 channels in packs of 4 instead of single ones:
// Forward 48 us instead of 65, 64 x 1024 x 510; but 3 fp32 channels in packs of 2 29 instead of 23, and in Backward 56 instead of 37, 37 x 1305 x 231).
// Up to 8 bytes where Backward keeps slabs of x and dy of many positions: with packs of 16 the sums per channel and the weights take 16 registers more
// (256 x 49 x 2048, bf16: 75 us against 57); for single positions 16 take 23 us and 8 take 32 (2000 x 1 x 4096 in one group).
constexpr int kMostBytes[2] = {16, 8};

int pack_of(const ucd_group_norm_t &d, int dir)
{
    if (const int ve = rows_pack(d)) return ve;
    const int cg = d.C / d.G;
    int ve = (d.S == 1 ? 16 : kMostBytes[dir]) / (d.dtype == 1 ? 2 : 4);
    while (ve > 1 && 10l * ceil_div(cg, ve) * ve > 13l * cg) ve /= 2;
    while (ve > cg) ve /= 2;
    return ve;
}

unsigned strip_units(const NormParams &p) { return (unsigned)p.strips * ((p.part_rows + kXcds - 1) / kXcds * kXcds); }

// TAIL: groups are no whole packs
template <bool SILU, bool TAIL, class T, int VE, bool BACKWARD>
hipError_t launch(NormParams &p, void *ws, hipStream_t s)
{
    const ucd_group_norm_t d = p.d;
    int threads, R;
    const Way way = divide(d, VE, BACKWARD, p, threads, R);
    char *at = (char *)ws;
    if (BACKWARD) {
        p.part = (float *)at;
        at += (size_t)8 * p.part_rows * d.C;
    }
    p.sums = (float *)at;
    constexpr int MOST = slab_packs<T, VE>(false), FEW = slab_packs<T, VE>(true);
    // 2^21 workgroups of up to 1024 threads to a launch: 2^32 threads are no grid
    const unsigned units = strip_units(p), grid = std::min(units, 1u << 21);
    if (way == PARTS) {
        norm_part_kernel<SILU, TAIL, T, VE, MOST, BACKWARD><<<grid, threads, 0, s>>>(p, units);
        norm_apply_kernel<SILU, T, VE, MOST, BACKWARD><<<grid, threads, 0, s>>>(p, units);
    } else if (way == SLABS) {
        for (p.unit0 = 0; p.unit0 < units; p.unit0 += grid) {
            const unsigned now = std::min(grid, units - p.unit0);
            if constexpr (BACKWARD) {
                if (R == FEW) norm_slab_bwd_kernel<SILU, TAIL, T, VE, FEW><<<now, threads, 0, s>>>(p);
                else norm_slab_bwd_kernel<SILU, TAIL, T, VE, MOST><<<now, threads, 0, s>>>(p);
            } else {
                if (R == FEW) norm_slab_fwd_kernel<SILU, TAIL, T, VE, FEW><<<now, threads, 0, s>>>(p);
                else norm_slab_fwd_kernel<SILU, TAIL, T, VE, MOST><<<now, threads, 0, s>>>(p);
            }
        }
    } else {
        const unsigned grid = (unsigned)p.columns * p.part_rows;
        if constexpr (BACKWARD) {
            if (R == 1) norm_rows_bwd_kernel<SILU, T, VE, 1><<<grid, threads, 0, s>>>(p);
            else norm_rows_bwd_kernel<SILU, T, VE, kRowsR><<<grid, threads, 0, s>>>(p);
        } else {
            if (R == 1) norm_rows_fwd_kernel<SILU, T, VE, 1><<<grid, threads, 0, s>>>(p);
            else norm_rows_fwd_kernel<SILU, T, VE, kRowsR><<<grid, threads, 0, s>>>(p);
        }
    }
    if (BACKWARD) norm_join_kernel<<<join_grid(2l * d.C), kJoinThreads, 0, s>>>(p);
    return hipGetLastError();
}

template <class T, int VE, bool BACKWARD>
hipError_t by_act(NormParams &p, void *ws, hipStream_t s)
{
    const bool silu = p.d.act == UCD_ACT_SILU;
    if (VE > 1 && p.d.C / p.d.G % VE != 0)
        return silu ? launch<true, (VE > 1), T, VE, BACKWARD>(p, ws, s) : launch<false, (VE > 1), T, VE, BACKWARD>(p, ws, s);
    return silu ? launch<true, false, T, VE, BACKWARD>(p, ws, s) : launch<false, false, T, VE, BACKWARD>(p, ws, s);
}

template <bool BACKWARD>
hipError_t dispatch(NormParams &p, int pack, void *ws, hipStream_t s)
{
    if (p.d.dtype == 1) {
        if (pack == 8) return by_act<bf16_t, 8, BACKWARD>(p, ws, s);
        if (pack == 4) return by_act<bf16_t, 4, BACKWARD>(p, ws, s);
        if (pack == 2) return by_act<bf16_t, 2, BACKWARD>(p, ws, s);
        return by_act<bf16_t, 1, BACKWARD>(p, ws, s);
    }
    if (pack == 4) return by_act<float, 4, BACKWARD>(p, ws, s);
    if (pack == 2) return by_act<float, 2, BACKWARD>(p, ws, s);
    return by_act<float, 1, BACKWARD>(p, ws, s);
}

}  // namespace

size_t group_norm_ws_bytes(const ucd_group_norm_t &d, int dir)
{
    return ws_bytes(d, pack_of(d, dir), dir);
}

hipError_t group_norm_fwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w, void *y,
                          float *stats, void *ws, hipStream_t s)
{
    NormParams p{};
    p.d = d;
    p.x = x; p.gamma = gamma; p.beta = beta_w; p.y = y; p.stats = stats;
    return dispatch<false>(p, pack_of(d, UCD_SEQ_FWD), ws, s);
}

hipError_t group_norm_bwd(const ucd_group_norm_t &d, const void *x, const float *gamma, const float *beta_w,
                          const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, bool add, void *ws,
                          hipStream_t s)
{
    NormParams p{};
    p.d = d;
    p.x = x; p.gamma = gamma; p.beta = beta_w; p.stats_in = stats; p.dy = dy; p.dx = dx; p.dgamma = dgamma; p.dbeta = dbeta; p.add = add;
    return dispatch<true>(p, pack_of(d, UCD_SEQ_BWD), ws, s);
}

}  // namespace ucd
