// Products of matrices of bfloat16 with sums in fp32, as the gated projection's kernels use them: out(m, n) = sum_k M(m, k) N(n, k), where either
// operand is read along its rows (k contiguous) or across them (m or n contiguous).
//
// A workgroup has a tile of BM by BN outputs and walks over k in steps of 64.  Both operands' steps go from memory to LDS directly, 16 bytes a lane,
// ahead of the products (a ring of buffers, one barrier a step).  Lanes fetch permuted pieces, so that reads of LDS meet no bank twice:
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

    // Step k0 of a plane, rows (columns) from `origin` on, is what comes next; 0 where it is no real one.
    uint64_t first, other;
    int size;
    bool there;
    __device__ __forceinline__ void aim(const Operand &o, int plane, int k0, int origin, bool real)
    {
        const bool second = !ALONG && PAIR && k0 >= o.half;
        const int k = k0 - (second ? o.half : 0);
        const long from = plane * o.plane + (ALONG ? origin * o.stride + k : k * o.stride + origin);
        const int rows = ALONG ? max(0, min(ALONG && PAIR ? R / 2 : R, o.rows - origin)) : max(0, min(BK, o.k - k));
        const uint32_t bytes = real && rows ? (uint32_t)(ALONG ? (rows - 1) * o.stride * 2 + (o.k - k) * 2 : rows * o.stride * 2) : 0u;
        there = !ALONG || k + column < o.k;
        first = uniform(o.p[second ? 1 : 0] + from);
        other = ALONG && PAIR ? uniform(o.p[1] + from) : first;
        size = __builtin_amdgcn_readfirstlane((int)bytes);
    }
    // Load i of it, to `lds`.
    __device__ __forceinline__ void move(int i, char *lds) const
    {
        typedef __attribute__((address_space(3))) void lds_t;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void *)(i >= LOADS / 2 ? other : first), 0, size, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_t *)(lds + (i * THREADS + wave * 64) * 16), 16, there ? offset[i] : kOut, 0, 0, 0);
    }

    // A lane's 8 elements of 16 k from 16 kk on, of the 32 rows (columns) from `first` on: row lane % 32, k 8 (lane / 32) + 0 .. 7.
    __device__ static __forceinline__ bf16x8 read(const char *lds, int first, int kk)
    {
        const int lane = threadIdx.x % 64;
        if (ALONG) {
            const int r = lane % 32, c = (lane / 32) ^ (r / 2 % 8) ^ (2 * kk);
            return lds_get<bf16x8>(lds + r * (BK * 2) + c * 16 + first * (BK * 2));
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
template <class T, int BM_, int BN_, int WAVES_M, int WAVES_N, int BUFFERS, bool M_ALONG, bool N_ALONG, bool N_PAIR>
struct Tile {
    static constexpr int BM = BM_, BN = BN_, THREADS = 64 * WAVES_M * WAVES_N;
    static constexpr int WM = BM / WAVES_M, WN = BN / WAVES_N, FM = WM / 32, FN = WN / 32;
    static constexpr bool ROW_PAIR = N_PAIR && N_ALONG;
    typedef Stage<BM, M_ALONG, false, THREADS> SM;
    typedef Stage<BN, N_ALONG, N_PAIR, THREADS> SN;
    static constexpr int STEP = SM::BYTES + SN::BYTES, LDS = BUFFERS * STEP;
    f32x16 acc[FN][FM];
    int wm, wn, lane;
    bf16x8 n[2][FN], m[2][FM];      // operands, 16 k ahead of their products
    SM sm;
    SN sn;

    // first row of fragment i within the tile's n side
    __device__ __forceinline__ int n_first(int i) const
    {
        return ROW_PAIR ? (i < FN / 2 ? 0 : BN / 2) + wn * (WN / 2) + i % (FN / 2) * 32 : wn * WN + 32 * i;
    }

    __device__ __forceinline__ void read(const char *at, int kk)
    {
#pragma unroll
        for (int i = 0; i < FN; ++i) n[kk % 2][i] = SN::read(at + SM::BYTES, n_first(i), kk);
#pragma unroll
        for (int j = 0; j < FM; ++j) m[kk % 2][j] = SM::read(at, wm * WM + 32 * j, kk);
    }
    __device__ __forceinline__ void multiply(int kk)
    {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < FM; ++j)
#pragma unroll
            for (int i = 0; i < FN; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(n[kk % 2][i], m[kk % 2][j], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
    // A step's loads in three parts between products: all at once they would hold up the waves that issue them.
    __device__ __forceinline__ void load(int part, char *into) const
    {
        constexpr int ALL = SM::LOADS + SN::LOADS;
#pragma unroll
        for (int i = ALL * part * 3 / 8; i < min(ALL, ALL * (part + 1) * 3 / 8); ++i) {
            if (i < SM::LOADS) sm.move(i, into);
            else sn.move(i - SM::LOADS, into + SM::BYTES);
        }
    }
    // Between two barriers: the last products of the step before, this step's others, and loads of a later step.  The pointers are told to be of different
    // memory, as they are: otherwise every transposing read waits for all loads on their way.
    __device__ __forceinline__ void step(const char *__restrict__ at, char *__restrict__ into)
    {
        load(0, into);
        read(at, 0);
        multiply(3);
        load(1, into);
        read(at, 1);
        multiply(0);
        load(2, into);
        read(at, 2);
        multiply(1);
        read(at, 3);
        multiply(2);
    }

    __device__ __forceinline__ void run(const Problem &p, int m0, int n0, int t0, int t1, char *lds)
    {
        static_assert(BK == 64, "four reads a step");
        lane = threadIdx.x % 64;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
        wm = wave % WAVES_M;
        wn = wave / WAVES_M;
#pragma unroll
        for (int i = 0; i < FN; ++i)
#pragma unroll
            for (int j = 0; j < FM; ++j) acc[i][j] = f32x16{};
        if (t0 >= t1) return;      // of all waves
        // the first step's "last products of the step before" are of zeros
#pragma unroll
        for (int i = 0; i < FN; ++i) n[1][i] = bf16x8{};
#pragma unroll
        for (int j = 0; j < FM; ++j) m[1][j] = bf16x8{};
        int phase = t0 / p.k_tiles, k0 = t0 % p.k_tiles * BK, aimed = t0;
        sm.init(p.m, m0);
        sn.init(p.n, n0);
        // Steps stand in a ring of buffers, BUFFERS - 1 of them on their way or there; behind the last one nothing is read, but as many loads stand in the
        // queue.
        auto aim = [&]() {
            sm.aim(p.m, plane_m(phase), k0, m0, aimed < t1);
            sn.aim(p.n, plane_n(phase), k0, n0, aimed < t1);
            ++aimed;
            k0 += BK;
            if (k0 == p.k_tiles * BK) k0 = 0, ++phase;
        };
        constexpr int LOADS = (SM::LOADS + SN::LOADS) * (BUFFERS - 2);      // in the queue behind the step that is waited for
        static_assert(LOADS < 64, "counted in six bits");
        constexpr int WAIT = (LOADS & 15) | LOADS >> 4 << 14 | 0x70;        // vmcnt(LOADS) lgkmcnt(0)
#pragma unroll
        for (int i = 0; i < BUFFERS - 1; ++i) {
            aim();
            load(0, lds + i * STEP), load(1, lds + i * STEP), load(2, lds + i * STEP);
        }
        int at = 0, into = (BUFFERS - 1) * STEP;
        for (int t = t0; t < t1; ++t) {
            __builtin_amdgcn_s_waitcnt(WAIT);      // this wave's part of the step has come, and it has read all of the one before
            lds_barrier();
            aim();
            step(lds + at, lds + into);
            at = at + STEP == LDS ? 0 : at + STEP;
            into = into + STEP == LDS ? 0 : into + STEP;
        }
        multiply(3);
        __builtin_amdgcn_s_waitcnt(0x0070);      // vmcnt(0) lgkmcnt(0): nothing is on its way to this LDS any more, and nobody reads it
        lds_barrier();
    }

    // Outputs in rows: a lane's sums are 16 bytes of a row at most, so that they go through LDS, 32 rows of a wave's COUNT fragments from FIRST on at a time.
    // value(i, j, r): four neighbours of fragment (i, j), from 8 r + 4 (lane / 32) on; sink(m, n, pack): 16 bytes of O at places within the tile.
    // Stored from the sums as they lie, tiles' ends took 18 us of each round of forward (8192 x 2048 x 8192).
    template <class O, int FIRST, int COUNT, class V, class S>
    __device__ __forceinline__ void rows(char *lds, V value, S sink) const
    {
        constexpr int WIDTH = COUNT * 32 * (int)sizeof(O), ROW = WIDTH + 16, PER = 16 / (int)sizeof(O), LANES = WIDTH / 16, EACH = 64 / LANES;
        constexpr int REGION = 32 * (FN * 32 * 4 + 16);      // a wave's, the same for all widths: the waves go from one to the next each in its own time
        static_assert(32 * ROW <= REGION && WAVES_M * WAVES_N * REGION <= LDS, "");
        char *own = lds + (wn * WAVES_M + wm) * REGION;
#pragma unroll
        for (int j = 0; j < FM; ++j) {
#pragma unroll
            for (int i = 0; i < COUNT; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const Pack<float, 4> v = value(FIRST + i, j, r);
                    Pack<O, 4> o;
#pragma unroll
                    for (int e = 0; e < 4; ++e) o.v[e] = from_f<O>(v.v[e]);
                    lds_put(own + lane % 32 * ROW + (32 * i + 8 * r + 4 * (lane / 32)) * (int)sizeof(O), o);
                }
            wave_lds_order();
#pragma unroll
            for (int i = 0; i < 32 / EACH; ++i) {
                const int row = i * EACH + lane / LANES, col = lane % LANES * PER;
                const Pack<O, PER> v = lds_get<Pack<O, PER>>(own + row * ROW + col * (int)sizeof(O));
                sink(wm * WM + 32 * j + row, n_first(FIRST) + col, v);
            }
            wave_lds_order();
        }
    }
    __device__ __forceinline__ Pack<float, 4> sums(int i, int j, int r) const
    {
        return Pack<float, 4>{{acc[i][j][4 * r], acc[i][j][4 * r + 1], acc[i][j][4 * r + 2], acc[i][j][4 * r + 3]}};
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
