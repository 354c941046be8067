// Products of matrices of bfloat16 with sums in fp32, as the gated projection's kernels use them: out(m, n) = sum_k M(m, k) N(n, k), where either
// operand is read along its rows (k contiguous) or across them (m or n contiguous).
//
// A workgroup has a tile of BM by BN outputs and walks over k in steps of 64.  Both operands' steps go from memory to LDS directly, 16 bytes a lane,
// one step ahead of the products (two buffers, one barrier a step).  Lanes fetch permuted pieces, so that reads of LDS meet no bank twice:
//   along: rows of 64 k, 8 cells of 16 bytes; cell c of row r stands at c ^ (r / 2 % 8), a lane reads one cell (8 neighbouring k of its row);
//   across: rows of BM or BN columns, one for each k; cell c of row k stands at c ^ (k % 4 * 4), transposing reads (ds_read_b64_tr_b16) give a lane 4
//   neighbouring k of its column.
// The n side is the matrix instruction's first operand: a lane's sums are then neighbours in n, which is where outputs are contiguous.
//
// fp32 operands are three planes of bfloat16 each, x = h + m + l (8 + 8 + 8 significant bits), and a product of them six products of planes,
// hh', hm', mh', mm', hl', lh': the k axis six times over.  What is left out is below 2^-24 of a product.
#pragma once
#include "seq_common.hpp"

namespace ucd {
namespace product {
using namespace seq;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int BK = 64;
constexpr uint32_t kOut = 0x80000000u;            // behind any buffer's end: reads as 0

// An operand.  along: `rows` rows of `k` elements.  across: `k` rows of `rows` elements.  Rows are `stride` elements apart, a multiple of 8 like the
// length of a row, addresses are multiples of 16 bytes.  There may be two such matrices, p[0] and p[1]: along, the tile's first half of rows
// is the first's and its second half the same rows of the second; across, rows from `half` on are the second's, from its first on (`half` is a
// multiple of BK and at least k, the rows that each has).  Planes are `plane` elements apart.
struct Operand {
    const bf16_t *p[2];
    long stride, plane;
    int rows, k, half;
};

struct Problem {
    Operand m, n;
    int k_tiles;          // steps of one phase
    int phases;           // 1, or 6 for fp32 operands
    int tiles_m, tiles_n;
    int splits;           // of the steps of all phases
};

__device__ __forceinline__ uint64_t uniform(const void *p)
{
    const uint64_t u = (uint64_t)p;
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)u);
}

// One operand's way to LDS, step by step.  A lane's offsets stay; what moves from step to step is the buffer, which ends behind the last row that there is.
template <int R, bool ALONG, bool PAIR, int THREADS>
struct Stage {
    static constexpr int BYTES = R * BK * 2, LOADS = BYTES / (THREADS * 16);
    static_assert(LOADS * THREADS * 16 == BYTES, "whole loads");
    static constexpr int CELLS = ALONG ? BK / 8 : R / 8, ROWS = THREADS / CELLS;      // cells of a row; rows of a load
    static_assert(ROWS % 16 == 0 || (!ALONG && ROWS % 4 == 0), "all of a lane's cells have one place in their rows");
    uint32_t offset[LOADS];
    int column;                // of the lane's cells, in elements

    __device__ __forceinline__ void init(const Operand &o, int origin)
    {
        const int r = threadIdx.x / CELLS, c = (threadIdx.x % CELLS) ^ (ALONG ? r / 2 % 8 : r % 4 * 4);
        column = 8 * c;
        const bool there = ALONG || origin + column < o.rows;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            // along, a pair's second matrix has a buffer of its own
            const int row = ALONG && PAIR ? (r + i * ROWS) % (R / 2) : r + i * ROWS;
            offset[i] = there ? (uint32_t)row * (uint32_t)o.stride * 2u + 16u * c : kOut;
        }
    }

    // Moves step k0 of a plane, rows (columns) from `origin` on, to `lds`.
    __device__ __forceinline__ void move(const Operand &o, int plane, int k0, int origin, char *lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const bool second = !ALONG && PAIR && k0 >= o.half;
        const int k = k0 - (second ? o.half : 0);
        const long from = plane * o.plane + (ALONG ? origin * o.stride + k : k * o.stride + origin);
        const int rows = ALONG ? max(0, min(ALONG && PAIR ? R / 2 : R, o.rows - origin)) : max(0, min(BK, o.k - k));
        const uint32_t bytes = rows ? (uint32_t)(ALONG ? (rows - 1) * o.stride * 2 + (o.k - k) * 2 : rows * o.stride * 2) : 0u;
        const bool there = !ALONG || k + column < o.k;
        const uint64_t first = uniform(o.p[second ? 1 : 0] + from), other = ALONG && PAIR ? uniform(o.p[1] + from) : first;
        const int size = __builtin_amdgcn_readfirstlane((int)bytes);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            typedef __attribute__((address_space(3))) void lds_t;
            const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(i >= LOADS / 2 ? other : first), 0, size, 0x00020000);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_t *)(lds + (i * THREADS + wave * 64) * 16), 16, there ? offset[i] : kOut, 0, 0, 0);
        }
    }

    // A lane's 8 elements of 16 k from 16 kk on, of the 32 rows (columns) from `first` on: row lane % 32, k 8 (lane / 32) + 0 .. 7.
    __device__ static __forceinline__ bf16x8 read(const char *lds, int first, int kk)
    {
        const int lane = threadIdx.x % 64;
        if (ALONG) {
            const int r = lane % 32, c = (lane / 32) ^ (r / 2 % 8) ^ (2 * kk);
            return *reinterpret_cast<const bf16x8 *>(lds + r * (BK * 2) + c * 16 + first * (BK * 2));
        }
        // 16 lanes fetch 4 rows of 16 columns each, 4 columns a lane, and get a column each
        const int at = first + lane / 16 % 2 * 16 + lane % 4 * 4, k = lane / 32 * 8 + lane % 16 / 4;
        const int cell = (at / 8) ^ (k % 4 * 4);
        const char *p = lds + k * (R * 2) + cell * 16 + at % 8 * 2 + kk * (32 * R);
        typedef __attribute__((address_space(3))) s16x4 lds_t;
        struct Both {
            s16x4 lo, hi;
        } v;
        v.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)p);
        v.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + 4 * R * 2));       // four rows on: the same place in them
        return __builtin_bit_cast(bf16x8, v);
    }
};

// The planes of a phase: hh', hm', mh', mm', hl', lh'.
__device__ __forceinline__ int plane_m(int phase) { return phase == 2 || phase == 3 ? 1 : phase == 5 ? 2 : 0; }
__device__ __forceinline__ int plane_n(int phase) { return phase == 1 || phase == 3 ? 1 : phase == 4 ? 2 : 0; }

// Of T, the outputs' type: a tile for each.  N_PAIR: the n side is two matrices; along, its tile is the same rows of both, and so is a wave's part of it.
template <class T, int BM_, int BN_, int WAVES_M, int WAVES_N, bool M_ALONG, bool N_ALONG, bool N_PAIR>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, THREADS = 64 * WAVES_M * WAVES_N;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, FM = WM / 32, FN = WN / 32;
    static constexpr bool ROW_PAIR = N_PAIR && N_ALONG;
    typedef Stage<BM, M_ALONG, false, THREADS> SM;
    typedef Stage<BN, N_ALONG, N_PAIR, THREADS> SN;
    static constexpr int LDS = 2 * (SM::BYTES + SN::BYTES);
    f32x16 acc[FN][FM];
    int wm, wn, lane;

    // first row of fragment i within the tile's n side
    __device__ __forceinline__ int n_first(int i) const
    {
        return ROW_PAIR ? (i < FN / 2 ? 0 : BN / 2) + wn * (WN / 2) + i % (FN / 2) * 32 : wn * WN + 32 * i;
    }

    __device__ __forceinline__ void run(const Problem &p, int m0, int n0, int t0, int t1, char *lds)
    {
        lane = threadIdx.x % 64;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        wm = wave % WAVES_M;
        wn = wave / WAVES_M;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = f32x16{};
        if (t0 >= t1) return;
        int phase = t0 / p.k_tiles, k0 = t0 % p.k_tiles * BK;
        SM sm;
        SN sn;
        sm.init(p.m, m0);
        sn.init(p.n, n0);
        auto stage = [&](int buffer) {
            char *at = lds + buffer * (SM::BYTES + SN::BYTES);
            sm.move(p.m, plane_m(phase), k0, m0, at);
            sn.move(p.n, plane_n(phase), k0, n0, at + SM::BYTES);
            k0 += BK;
            if (k0 == p.k_tiles * BK) k0 = 0, ++phase;
        };
        stage(0);
        for (int t = t0; t < t1; ++t) {
            const int buffer = (t - t0) & 1;
            __builtin_amdgcn_s_waitcnt(0x0F70);      // vmcnt(0): this wave's part of the step has come
            lds_barrier();                           // everybody's has, and nobody reads the step before any more
            if (t + 1 < t1) stage(buffer ^ 1);
            const char *at = lds + buffer * (SM::BYTES + SN::BYTES);
            // operands are read 16 k ahead of their products
            bf16x8 n[2][FN], m[2][FM];
            auto read = [&](int kk) {
#pragma unroll
                for (int i = 0; i < FN; ++i) n[kk % 2][i] = SN::read(at + SM::BYTES, n_first(i), kk);
#pragma unroll
                for (int j = 0; j < FM; ++j) m[kk % 2][j] = SM::read(at, wm * WM + 32 * j, kk);
            };
            read(0);
#pragma unroll
            for (int kk = 0; kk < BK / 16; ++kk) {
                if (kk + 1 < BK / 16) read(kk + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < FM; ++j)
#pragma unroll
                    for (int i = 0; i < FN; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(n[kk % 2][i], m[kk % 2][j], acc[i][j], 0, 0, 0);
            }
        }
    }

    // f(m, n, values): four neighbours in n, places within the tile; each fragment of the n side by itself
    template <class F>
    __device__ __forceinline__ void each(F f) const
    {
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int i = 0; i < FN; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    f(wm * WM + 32 * j + lane % 32, n_first(i) + 8 * r + 4 * (lane / 32),
                      Pack<float, 4>{{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]}});
    }
};

// The steps of a split.
__device__ __forceinline__ void split_range(const Problem &p, int split, int &t0, int &t1)
{
    const int all = p.k_tiles * p.phases;
    t0 = (int)((long)all * split / p.splits);
    t1 = (int)((long)all * (split + 1) / p.splits);
}

}  // namespace product
}  // namespace ucd
