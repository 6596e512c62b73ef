// Training of a block's 16-bit experts: products of grouped rows with the matrices of their expert, forward and backward.
//
//   up        a = W1 x, u = W3 x, h = silu(a) u            rows [K] x matrix rows [K]
//   down      y = W2 h                                     rows [K] x matrix rows [K]
//   d_hidden  q = W2^T d_out, then d_a, d_u, g h, d_gate   rows [K] x matrix columns
//   d_rows    y = W1^T d_a + W3^T d_u                      rows [K] x matrix columns
//   d_weights W1: d_a^T x, W3: d_u^T x, W2: d_out^T (g h)  columns x columns, over the rows of an expert
//
// An operand whose contraction runs along memory ("rows") lies in LDS as rows of 64 elements, one whose contraction runs across it
// ("columns") as 64 rows of 256 columns, and ds_read_b64_tr_b16 hands its columns to the lanes: no transposed copy of a matrix is made.
#include <algorithm>
#include <type_traits>

#include "experts_train.hpp"
#include "kernels.hpp"
#include "mfma_common.hpp"

namespace moemix {

namespace {

constexpr int kLdsBytes = 163840;        // of a compute unit
constexpr int kUnit = 32768;             // 256 rows of 64 elements, or 64 rows of 256
constexpr int kThreads = 512;

// Are a call's matrices more than the last-level cache holds?
bool matrices_past_caches(int E, int d, int f) { return (size_t)E * 3 * d * f * 2 > 256ull << 20; }

enum Form { kUp, kDown, kDHidden, kDRows };

typedef const int32_t __attribute__((address_space(4)))* const_ints_t;

typedef short short4v_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v_t* lds_short4_t;

// ---- operands in LDS

// "Columns": slabs of 16 columns (32 bytes) of row r are stored at slab ^ slab_swizzle(r): the 16 rows that one transposed read takes
// then lie in 16 different slabs, so no two of them in the same bank.
__device__ __forceinline__ int slab_swizzle(int r) { return (r & 3) | (((r >> 3) & 3) << 2); }

// 8 consecutive contraction elements (kk: 32 kk + 8 q ..) of column r16 of a slab; at: the lane's address for it (columns_at) in the unit.
template <int ROW = 512>   // bytes of a row
__device__ __forceinline__ half8_t read_columns(uint32_t at, int kk) {
    const short4v_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(uintptr_t)(at + kk * 32 * ROW));
    const short4v_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(uintptr_t)(at + kk * 32 * ROW + 4 * ROW));
    const half4_t l = __builtin_bit_cast(half4_t, lo), h = __builtin_bit_cast(half4_t, hi);
    return half8_t{l[0], l[1], l[2], l[3], h[0], h[1], h[2], h[3]};
}
__device__ __forceinline__ uint32_t columns_at(int lane, int slab) {
    const int r16 = lane & 15, q = lane >> 4, row = 8 * q + (r16 >> 2);
    return row * 512 + (r16 & 3) * 8 + ((slab ^ slab_swizzle(row)) << 5);
}
// "Rows": 16-byte pieces of row r at piece ^ rows_swizzle(r).  A 16-byte read serves lanes 0-3, 12-15 and 20-27 together, then 4-11, 16-19 and 28-31, and so on: of the
// operand's 16 rows each time some of one piece and the others of its neighbour, in 16 different places of 256 bytes.
__device__ __forceinline__ int rows_swizzle(int r) { return (r >> 1) & 7; }
__device__ __forceinline__ half8_t read_rows(uint32_t at) {
    return *(const half8_t __attribute__((address_space(3)))*)(uintptr_t)at;
}
__device__ __forceinline__ uint32_t rows_at(int lane, int kk) {
    const int r16 = lane & 15, q = lane >> 4;
    return r16 * 128 + (((4 * kk + q) ^ rows_swizzle(r16)) << 4);
}

// A pointer that is the same in every lane, whatever the compiler knows about it.
__device__ __forceinline__ gptr_t uniform_ptr(const void* p) {
    const uint64_t v = (uint64_t)(uintptr_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    gptr_t g = (gptr_t)(uintptr_t)(((uint64_t)hi << 32) | lo);
    asm volatile("s_nop 4" : "+s"(g));       // (what a memory instruction asks for after a lane read of its base)
    return g;
}

// As bring(), past the caches.
__device__ __forceinline__ void bring_past(uint32_t lds, gptr_t p, uint32_t v) {
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"{m0}"(lds), "v"(v), "s"(p) : "memory");
}

__device__ __forceinline__ float sigmoid(float a) { return 1.0f / (1.0f + __expf(-a)); }

// ---- who does what when
//
// The 8 wavefronts of a workgroup are two groups of four, one of each per SIMD; group g multiplies half g of the tile's rows.  A step of the contraction (64 elements)
// takes each group two phases: it reads the operands of the step from LDS into registers, then it multiplies them.  The groups are one phase apart, so that in
// every phase one of them feeds the matrix cores (64 instructions of 16 cycles) and the other reads, and all meet at its end.  Each group also asks for 8 KB per wavefront and step,
// straight into LDS, always of a step that lies ahead:
//   phase 2k:      group 0 reads step k, asks for rows' half 1 of step k + nA - 1 and the first half of the matrix's unit of step k + nB - 1;  group 1 multiplies step k - 1
//   phase 2k + 1:  group 1 reads step k, asks for rows' half 0 of step k + nA and the second half of the matrix's unit of step k + nB - 1;  group 0 multiplies step k
// (past the last step the last one again, so that the waits can count).
// Each half of the rows has a ring of nA units, the matrix one of nB; what is written then was read last in the phase before, or earlier.  A transfer has three phases or more
// to arrive (nA = 2, nB = 3, 160 KB of LDS; with two phases for the matrix's side a step took 2400 cycles in place of 2048).
// Transfers and reads go by turns: a transfer waits for its place in the compute unit's address path, 64 bytes per cycle for all wavefronts, and LDS delivers meanwhile.  (One after the
// other 450 + 550 cycles.)  kLate: the matrix's transfers are asked for among the products that follow instead, and by group 1 a step further ahead: where both operands take transposed
// reads, twice as many instructions, a phase of reading has no room for them (970 cycles with, backward of 4096 tokens in the Mixtral shape 5850 -> 5760 us; elsewhere they delay
// the products: forward 2780 -> 2817).
//
// What bounds it: 2048 cycles of products in the 2240 of a step; and power.  The clock falls to 1.4-1.5 GHz (8192 rows of one expert of 4096 x 14336, d_rows: 1390 us, 1.38 PFLOP/s; with operands
// of zeros, the same instructions, 1028 us).  So what saves energy counts: two products in a row share an operand (g goes to and fro over j), 0.7-1 % of the time.

// Up to COUNT of the wavefront's own transfers are under way.
template <int COUNT>
__device__ __forceinline__ void wait_transfers() {
    static_assert(COUNT < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(COUNT) : "memory");
}
// The wavefront's LDS accesses are done (said in a way that the compiler counts on: else it waits for the operands again among the products, and for the tokens that are being
// looked up with them), then all meet.
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0), nothing else
    asm volatile("s_barrier" ::: "memory");
}

// TILE: kA, kB (units of the rings), kRuns (transfers of a wavefront for its half of the rows; for its half of the matrix's unit it is four), kReads (operands of a step), kLate (multiply() calls
// bring_matrix()), bring_rows(k), bring_matrix(k) (transfer k of the next stage), rows_asked(more), matrix_asked(more) (all of a stage's have been made; is there another one?), look_up_rows(), look_up_matrix() (asks for
// what the next ones need), rows_there(step), matrix_there(step) (what the wavefront brought of a step has arrived and nobody reads it yet), read(r) (operand r of the next step),
// step_read(), multiply().
template <typename TILE>
__device__ __forceinline__ void run_steps(TILE& t, int n, int group) {
    constexpr bool kLate = TILE::kLate;
    constexpr int kA = TILE::kA, kB = TILE::kB, kRuns = TILE::kRuns, kPer = kRuns + 4, kTurns = kLate ? kRuns : kPer;
    static_assert(kA <= kB && kB <= kA + 1, "what follows counts on it");
    // transfers after those of the step that is read next
    constexpr int kRowsLate = (kA - 1) * kPer + (kLate ? 0 : 4), kMatrixLate = (kB - 2) * kPer, kMatrixLate1 = kMatrixLate + (kLate ? kRuns : 0);
    const int rows_ahead = kA - 1 + group, matrix_ahead = kB - 1 + (kLate ? group : 0);
    for (int k = -kB; k < 0; ++k) {
        if (k + rows_ahead >= 0) {
#pragma unroll
            for (int i = 0; i < kRuns; ++i) t.bring_rows(i);
            t.rows_asked(k + rows_ahead + 1 < n);
        }
        if (k + matrix_ahead >= 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i) t.bring_matrix(i);
            t.matrix_asked(k + matrix_ahead + 1 < n);
        }
        t.look_up_rows();
        t.look_up_matrix();
    }
    wait_transfers<kMatrixLate>();
    if (group) t.rows_there(0);
    t.matrix_there(0);
    meet();
    if (group) meet();
    for (int k = 0; k < n; ++k) {
        t.look_up_matrix();
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            if (i < kRuns) t.bring_rows(i);
            else t.bring_matrix(i - kRuns);
#pragma unroll
            for (int r = i * TILE::kReads / kTurns; r < (i + 1) * TILE::kReads / kTurns; ++r) t.read(r);
        }
        t.rows_asked(k + rows_ahead + 1 < n);
        if (!kLate) t.matrix_asked(k + matrix_ahead + 1 < n);
        t.step_read();
        if (group) wait_transfers<kRowsLate < kMatrixLate1 ? kRowsLate : kMatrixLate1>();
        else wait_transfers<kRowsLate>();
        t.rows_there(k + group);
        if (group) t.matrix_there(k + 1);
        pin_schedule();
        meet();
        pin_schedule();
        __builtin_amdgcn_s_setprio(1);
        t.multiply();
        __builtin_amdgcn_s_setprio(0);
        pin_schedule();
        if (kLate) t.matrix_asked(k + matrix_ahead + 1 < n);
        if (!group) {
            wait_transfers<kMatrixLate>();
            t.matrix_there(k + 1);
        }
        if (!group || k + 1 < n) meet();
    }
    wait_transfers<0>();
}

// ---- results

// A wavefront's sums: lane l of tile (j, i) holds row l & 15 of 16 i .., columns 16 j + 4 (l >> 4) .. + 3.  Written as they lie, rows would go to memory in pieces of 32 bytes (fp16), which
// took 30 000 cycles for 128 KB of a workgroup.  So the four j are exchanged among each four neighbouring lanes: afterwards v[k] of lane l is row (l & 12) + k, columns
// 16 (l & 3) + 4 (l >> 4) .. + 3, and one instruction writes whole lines of four rows.

// c odd (bit of the lane): `mine` stays in place of `theirs`
template <int CTRL, typename V>
__device__ __forceinline__ void exchange(bool odd, V& v0, V& v1) {
    constexpr int N = sizeof(V) / 4;
    typedef uint32_t words_t __attribute__((ext_vector_type(N)));
    const words_t a = __builtin_bit_cast(words_t, v0), b = __builtin_bit_cast(words_t, v1);
    words_t x, y;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint32_t ai = a[i], bi = b[i];
        const uint32_t other_a = __builtin_amdgcn_update_dpp(0, ai, CTRL, 0xF, 0xF, true), other_b = __builtin_amdgcn_update_dpp(0, bi, CTRL, 0xF, 0xF, true);
        x[i] = odd ? other_b : ai;
        y[i] = odd ? bi : other_a;
    }
    v0 = __builtin_bit_cast(V, x);
    v1 = __builtin_bit_cast(V, y);
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E;      // quad_perm: lanes 1 and 2 apart
template <typename V>
__device__ __forceinline__ void transpose4(int lane, V& v0, V& v1, V& v2, V& v3) {
    exchange<kSwap1>(lane & 1, v0, v1);
    exchange<kSwap1>(lane & 1, v2, v3);
    exchange<kSwap2>(lane & 2, v0, v2);
    exchange<kSwap2>(lane & 2, v1, v3);
}

// ---- products of rows

// What a workgroup works on: a chunk of up to 32 MT rows (group g the tiles of 16 rows MT g .. MT g + MT - 1), 256 columns from n0 on (up: 128 of each matrix; wavefront
// w of a group a quarter), contraction steps [s0, s1).
struct RowsWork {
    int expert, begin, rows, n0, s0, s1, split;
};

// PAST: the matrices are more than the caches hold.  Then chunks of up to 128 rows read theirs past them: most are their expert's only one, and each matrix is read once (4 and 64 tokens in the
// Mixtral shape, forward 540 -> 504 and 526 -> 493 us, 5.7 TB/s; with matrices that fit, 16 tokens of 256 x 512, 19.4 -> 21.3).  How many chunks an expert has is not looked at: several
// short ones of one expert all read past the caches, and so does a short one beside a long one.
template <int FORM, int MT, bool PAST>
struct RowsTile {
    static constexpr bool kColumns = FORM == kDHidden || FORM == kDRows;     // how the matrix lies
    static constexpr int kA = MT > 4 ? 2 : MT > 2 ? 3 : 4, kB = MT > 2 ? 3 : 4;
    static constexpr int kHalf = MT * 2048;                                 // bytes of a unit of half of the rows
    static constexpr int kRuns = (MT + 1) / 2;                              // (of 2 MT over four wavefronts; odd: two bring the same one at the end)
    static constexpr int kRingB = 2 * kA * kHalf;                           // where the matrix's ring begins
    static constexpr bool kLate = false;
    static_assert(kRingB + kB * kUnit <= kLdsBytes, "LDS");
    const TrainRows& a;
    const RowsWork& c;
    uint32_t lds0, put_a, put_b, get_a, get_b;      // LDS addresses: units that are filled next, units that are read next
    int lane, group, wn;
    gptr_t base_a, base_b;
    uint32_t va[kRuns], vb[4];
    int step_a, step_b;                             // d_rows: the next one to bring
    uint32_t ra[2], rb[kColumns ? 4 : 2];
    float4_t acc[4][MT];
    half8_t fa[2][MT], fb[2][4];

    __device__ __forceinline__ RowsTile(const TrainRows& a_, const RowsWork& c_, uint8_t* lds) : a(a_), c(c_) {
        lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
        lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        group = wave >> 2;
        wn = wave & 3;
        const int N = a.N, K = a.K, row_in_run = lane >> 3;
        const int piece = ((lane & 7) ^ rows_swizzle(8 * (wn & 1) + row_in_run)) * 16;
        const bool gathered = FORM == kUp || FORM == kDHidden;
        // half 1 - group of the rows, runs wn, wn + 4 .. of 8 rows
#pragma unroll
        for (int k = 0; k < kRuns; ++k) {
            const int row = min((1 - group) * 16 * MT + run_of(k) * 8 + row_in_run, c.rows - 1);     // (past the last row: the last one again)
            va[k] = (uint32_t)(gathered ? a.tok[c.begin + row] : row) * (uint32_t)K * 2 + piece;
        }
        // half `group` of the matrix's unit: 128 rows of 64 elements (up: of W1, of W3), or 32 rows of 256, runs of two
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (kColumns) {
                const int row = 32 * group + 8 * wn + 2 * k + (lane >> 5), p = lane & 31;
                const int col = ((((p >> 1) ^ slab_swizzle(row)) << 1) | (p & 1)) * 8;
                vb[k] = (uint32_t)row * (uint32_t)N * 2 + (uint32_t)min(col, N - 8 - c.n0) * 2;
            } else {
                const int row = (FORM == kUp ? 0 : 128 * group) + (wn + 4 * k) * 8 + row_in_run;
                vb[k] = (uint32_t)min(row, N - 1 - c.n0) * (uint32_t)K * 2 + piece;
            }
        }
        if (kColumns) {
#pragma unroll
            for (int j = 0; j < 4; ++j) rb[j] = columns_at(lane, 4 * wn + j);
        } else {
            rb[0] = rows_at(lane, 0);
            rb[1] = rows_at(lane, 1);
        }
        ra[0] = rows_at(lane, 0);
        ra[1] = rows_at(lane, 1);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        put_a = lds0 + (1 - group) * kA * kHalf;
        get_a = lds0 + group * kA * kHalf;
        put_b = get_b = lds0 + kRingB;
        step_a = step_b = c.s0;
        seek_rows(c.s0);
        seek_matrix(c.s0);
    }

    __device__ __forceinline__ int run_of(int k) const { return MT % 2 && k == MT / 2 ? 4 * k + (wn & 1) : 4 * k + wn; }
    // d_rows: the second half of the steps is d_u's and W3's.
    __device__ __forceinline__ int steps_of_one() const { return a.K / kTrainStep; }

    // The next step to bring is s.
    __device__ __forceinline__ void seek_rows(int s) {
        const bool second = FORM == kDRows && s >= steps_of_one();
        const size_t k0 = (size_t)(second ? s - steps_of_one() : s) * kTrainStep;
        base_a = uniform_ptr((second ? a.in2 : a.in) + (FORM == kDown || FORM == kDRows ? (size_t)c.begin * a.K : 0) + k0);
    }
    __device__ __forceinline__ void seek_matrix(int s) {
        const bool second = FORM == kDRows ? s >= steps_of_one() : FORM == kUp && group;
        const size_t k0 = (size_t)(FORM == kDRows && second ? s - steps_of_one() : s) * kTrainStep;
        const half_t* const w = second ? a.w3[c.expert] : a.w[c.expert];
        base_b = uniform_ptr(kColumns ? w + k0 * a.N + c.n0 : w + (size_t)c.n0 * a.K + k0);
    }

    __device__ __forceinline__ void bring_rows(int k) { moemix::bring<0>(put_a + run_of(k) * 1024, base_a, va[k]); }
    __device__ __forceinline__ void rows_asked(bool more) {
        const uint32_t ring = lds0 + (1 - group) * kA * kHalf;
        put_a = put_a == ring + (kA - 1) * kHalf ? ring : put_a + kHalf;
        if (!more) return;
        if (FORM == kDRows && ++step_a == steps_of_one()) seek_rows(step_a);
        else base_a += kTrainStep * 2;
    }
    __device__ __forceinline__ void bring_matrix(int k) {
        const uint32_t to = put_b + group * (kUnit / 2) + wn * (kColumns ? 4096 : 1024) + k * (kColumns ? 1024 : 4096);
        if (PAST && MT <= 4) bring_past(to, base_b, vb[k]);
        else moemix::bring<0>(to, base_b, vb[k]);
    }
    __device__ __forceinline__ void matrix_asked(bool more) {
        put_b = put_b == lds0 + kRingB + (kB - 1) * kUnit ? lds0 + kRingB : put_b + kUnit;
        if (!more) return;
        if (FORM == kDRows && ++step_b == steps_of_one()) seek_matrix(step_b);
        else base_b += kColumns ? (size_t)a.N * (kTrainStep * 2) : kTrainStep * 2;
    }
    __device__ __forceinline__ void look_up_rows() {}
    __device__ __forceinline__ void look_up_matrix() {}
    __device__ __forceinline__ void rows_there(int) {}
    __device__ __forceinline__ void matrix_there(int) {}

    static constexpr int kReads = 2 * (4 + MT);
    __device__ __forceinline__ void read(int r) {
        if (r < 8) {
            const int kk = r & 1, j = r >> 1;
            if (kColumns) fb[kk][j] = read_columns(get_b + rb[j], kk);
            else fb[kk][j] = read_rows(get_b + (FORM == kUp ? (j >> 1) * 128 + wn * 32 + (j & 1) * 16 : wn * 64 + j * 16) * 128 + rb[kk]);
        } else {
            const int kk = r & 1, i = (r - 8) >> 1;
            fa[kk][i] = read_rows(get_a + i * 2048 + ra[kk]);
        }
    }
    __device__ __forceinline__ void step_read() {
        const uint32_t ring = lds0 + group * kA * kHalf;
        get_a = get_a == ring + (kA - 1) * kHalf ? ring : get_a + kHalf;
        get_b = get_b == lds0 + kRingB + (kB - 1) * kUnit ? lds0 + kRingB : get_b + kUnit;
    }
    __device__ __forceinline__ void multiply() {
#pragma unroll
        for (int g = 0; g < 2 * MT; ++g) {
            const int kk = g / MT, i = g % MT;
#pragma unroll
            for (int to = 0; to < 4; ++to) {
                const int j = g & 1 ? 3 - to : to;
                acc[j][i] = mfma16(fb[kk][j], fa[kk][i], acc[j][i]);
            }
        }
    }

    __device__ __forceinline__ void write(uint8_t* lds) {
        if (FORM == kUp) write_up();
        else if (FORM == kDHidden) write_d_hidden(lds);
        else write_rows();
    }

    // a and u together: their two tiles of 16 columns each make the four that are exchanged.  Then h: rows of 32 columns, two lanes exchange theirs.  a and u go past the caches, h is
    // read next (forward of 333 tokens, 1024 x 2816, 55.6 -> 53.5 us; 512 in the Mixtral shape 607 -> 596; 4096 of them 2575 -> 2595).
    __device__ __forceinline__ void write_up() {
        const int n0 = c.n0 + wn * 32, N = a.N;
        if (n0 >= N) return;
        const int q = lane >> 4, r0 = group * 16 * MT;
        half_t* const au = (lane & 2 ? a.u : a.a) + (size_t)c.begin * N + n0 + (lane & 1) * 16 + 4 * q;
        half_t* const ph = a.h + (size_t)c.begin * N + n0 + (lane & 1) * 16 + 4 * q;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            half4_t v[4], h[2];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j][k] = (half_t)acc[j][i][k];
#pragma unroll
                for (int j = 0; j < 2; ++j) h[j][k] = (half_t)silu_mul(acc[j][i][k], acc[j + 2][i][k]);
            }
            transpose4(lane, v[0], v[1], v[2], v[3]);
            exchange<kSwap1>(lane & 1, h[0], h[1]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = r0 + 16 * i + (lane & 12) + k;
                if (r < c.rows) __builtin_nontemporal_store(v[k], (half4_t*)(au + (size_t)r * N));
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = r0 + 16 * i + (lane & 14) + k;
                if (r < c.rows) *(half4_t*)(ph + (size_t)r * N) = h[k];
            }
        }
    }

    // The operands' rings are free by now: a wavefront turns its sums, up to 64 rows at a time, into whole lines of rows in LDS of its own, eight columns of eight rows per instruction.
    __device__ __forceinline__ void write_d_hidden(uint8_t* lds) {
        constexpr int kRow = 272, kMost = MT < 4 ? MT : 4;
        __syncthreads();                                     // (the rings are read no more)
        uint8_t* const region = lds + (4 * group + wn) * (kLdsBytes / 8);
        const int N = a.N, n0 = c.n0 + wn * 64, r8 = lane >> 3, c8 = (lane & 7) * 8;
        if (n0 >= N) return;                                 // (64 divides N)
#pragma unroll
        for (int i0 = 0; i0 < MT; i0 += 4) {
            half8_t va[2 * kMost], vu[2 * kMost];
            float gate[2 * kMost];
            const int r0 = (group * MT + i0) * 16 + r8;
#pragma unroll
            for (int p = 0; p < 2 * kMost; ++p) {
                if (i0 * 2 + p >= 2 * MT) continue;
                const size_t row = (size_t)(c.begin + (r0 + 8 * p < c.rows ? r0 + 8 * p : 0));
                va[p] = *(const half8_t*)(a.a + row * N + n0 + c8);
                vu[p] = *(const half8_t*)(a.u + row * N + n0 + c8);
                gate[p] = a.gate[row];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i0 + i < MT)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *(float4_t*)(region + (i * 16 + (lane & 15)) * kRow + (j * 16 + 4 * (lane >> 4)) * 4) = acc[j][i0 + i];
            wave_lds_handover();
#pragma unroll
            for (int p = 0; p < 2 * kMost; ++p) {
                if (i0 * 2 + p >= 2 * MT) continue;
                const float* const sums = (const float*)(region + (8 * p + r8) * kRow) + c8;
                const float4_t lo = *(const float4_t*)sums, hi = *(const float4_t*)(sums + 4);
                const float g = gate[p];
                half8_t da, du, gh;
                float share = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = (float)va[p][k], y = (float)vu[p][k], s = sigmoid(x), z = x * s, h = z * y, v = k < 4 ? lo[k & 3] : hi[k & 3];
                    share = fmaf(v, h, share);
                    du[k] = (half_t)(g * v * z);
                    da[k] = (half_t)(g * v * y * (s * (1.0f + x * (1.0f - s))));
                    gh[k] = (half_t)(g * h);
                }
                share += dpp_move<kSwap1>(share);
                share += dpp_move<kSwap2>(share);
                share += __shfl_xor(share, 4, kWave);
                const int r = r0 + 8 * p;
                if (r < c.rows) {
                    const size_t at = (size_t)(c.begin + r) * N + n0 + c8;
                    *(half8_t*)(a.d_a + at) = da;
                    *(half8_t*)(a.d_u + at) = du;
                    *(half8_t*)(a.h + at) = gh;
                    if ((lane & 7) == 0) a.part[(size_t)(c.begin + r) * (N / 64) + n0 / 64] = share;
                }
            }
            wave_lds_handover();
        }
    }

    __device__ __forceinline__ void write_rows() {
        if (c.n0 + wn * 64 >= a.N) return;
        float* const y = a.y + ((size_t)c.split * a.P + c.begin) * a.N + c.n0 + wn * 64 + (lane & 3) * 16 + 4 * (lane >> 4);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            transpose4(lane, acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int r = group * 16 * MT + 16 * i + (lane & 12) + k;
                if (r < c.rows) *(float4_t*)(y + (size_t)r * a.N) = acc[k][i];
            }
        }
    }
};

template <int FORM, int MT, bool PAST>
__device__ __forceinline__ void rows_body(const TrainRows& a, const RowsWork& c, uint8_t* lds) {
    RowsTile<FORM, MT, PAST> t(a, c, lds);
    run_steps(t, c.s1 - c.s0, t.group);
    t.write(lds);
}

// Workgroups go to the 8 XCDs in turn, each XCD with an L2 of its own and 32 compute units: n tiles are dealt out to the XCDs in blocks of 32 neighbours (fewer than 256 tiles: eight
// blocks), so that those that run at once in an XCD share what they read, and that tiles of every length come to every XCD.
__device__ __host__ __forceinline__ int block_of(int n) { return n >= 256 ? 32 : (n + 7) / 8; }
__device__ __host__ __forceinline__ int slots_of(int n) {
    const int block = block_of(n);
    return block ? (n + 8 * block - 1) / (8 * block) * block : 0;
}
// (-1: none)
__device__ __forceinline__ int place_in_blocks(int n, int slot, int xcd) {
    const int block = block_of(n);
    if (slot >= slots_of(n)) return -1;
    const int round = slot / block, t = (round * 8 + xcd) * block + slot - round * block;
    return t < n ? t : -1;
}

constexpr int kMostSplit = 512;          // workgroups of split chunks

template <int FORM, bool PAST>
__global__ __launch_bounds__(kThreads, 2) void train_rows_kernel(TrainRows a, int n_tiles) {
    extern __shared__ uint8_t lds[];
    const TrainMeta* const meta = a.meta;
    const TrainSplit sp = FORM == kDown ? meta->down : FORM == kDRows ? meta->d_rows : meta->whole;
    const int first = sp.first_split, others = meta->n_chunks - first, n_a = first * n_tiles, units = others * n_tiles, n_b = units * sp.splits;
    const int slot = blockIdx.x >> 3, xcd = blockIdx.x & 7, slots_a = slots_of(n_a);
    const bool split = slot >= slots_a;
    int t = split ? place_in_blocks(n_b, slot - slots_a, xcd) : place_in_blocks(n_a, slot, xcd);
    if (t < 0) return;
    RowsWork c;
    c.split = split ? __builtin_amdgcn_readfirstlane(t / units) : 0;
    t -= c.split * units;
    // up to eight chunks of one expert side by side, column after column (where a group reaches over the line between the split chunks and the others: its part); what any of
    // them says tells of all
    const int zero = split ? first : 0, chunk0 = __builtin_amdgcn_readfirstlane(zero + t / n_tiles);
    const TrainChunk ch = a.chunks[chunk0];
    const int start = chunk0 - (ch.form >> 4 & 15), size = (ch.form & 15) * 32;
    const int of = max(start, zero), n = min(start + (ch.form >> 8), split ? first + others : first) - of, rest = t - (of - zero) * n_tiles;
    const int tile = __builtin_amdgcn_readfirstlane(rest / n);
    c.expert = __builtin_amdgcn_readfirstlane(ch.expert);
    c.begin = __builtin_amdgcn_readfirstlane(ch.begin + (of + rest - tile * n - chunk0) * size);
    c.rows = __builtin_amdgcn_readfirstlane(min(size, ch.end - c.begin));
    c.n0 = tile * (FORM == kUp ? kTrainCols / 2 : kTrainCols);
    const int steps = a.K / kTrainStep * (FORM == kDRows ? 2 : 1), shares = split ? sp.splits : 1;
    c.s0 = __builtin_amdgcn_readfirstlane(steps * c.split / shares);
    c.s1 = __builtin_amdgcn_readfirstlane(steps * (c.split + 1) / shares);
    switch ((c.rows + 31) >> 5) {
        case 1: rows_body<FORM, 1, PAST>(a, c, lds); break;
        case 2: rows_body<FORM, 2, PAST>(a, c, lds); break;
        case 3: rows_body<FORM, 3, PAST>(a, c, lds); break;
        case 4: rows_body<FORM, 4, PAST>(a, c, lds); break;
        case 5: rows_body<FORM, 5, PAST>(a, c, lds); break;
        case 6: rows_body<FORM, 6, PAST>(a, c, lds); break;
        default: rows_body<FORM, 8, PAST>(a, c, lds);
    }
}

template <int FORM, bool PAST>
void launch_rows_kernel(const TrainRows& a, hipStream_t st) {
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = train_rows_kernel<FORM, PAST>;
    allow_lds((const void*)kernel, kLdsBytes, configured);
    constexpr int kOut = FORM == kUp ? kTrainCols / 2 : kTrainCols;
    const int n_tiles = (a.N + kOut - 1) / kOut, most_chunks = a.P / a.most_rows + (a.E < a.P ? a.E : a.P);
    const int most_a = most_chunks * n_tiles, most_b = FORM == kDown || FORM == kDRows ? kMostSplit : 0;
    const int slots = (most_a + 255) / 256 * 32 + (most_b + 255) / 256 * 32;
    kernel<<<(unsigned)slots * 8, kThreads, kLdsBytes, st>>>(a, n_tiles);
}

template <int FORM>
void launch_rows(const TrainRows& a, hipStream_t st) {
    if (matrices_past_caches(a.E, a.N, a.K)) launch_rows_kernel<FORM, true>(a, st);
    else launch_rows_kernel<FORM, false>(a, st);
}

// ---- gradients of the matrices

struct WeightsWork {
    int begin, rows;             // of the expert
    const half_t *m, *n;         // [., lm], [., ln]
    int lm, ln, m0, n0;
    void* out;                   // [lm, ln]
};

// 16 rows from row m on of 64 columns of a gradient, lm x ln.  Stored past the caches, which hold what the next workgroups read (backward of 2048 tokens, 32 experts of 2048 x 1408, four per token:
// 558 -> 530 us; 256 tokens: 328 -> 278).
template <typename OUT>
__device__ __forceinline__ void write_sums(int lane, float4_t s0, float4_t s1, float4_t s2, float4_t s3, OUT* out, int m, int lm, int ln, bool accumulate) {
    typedef OUT out4_t __attribute__((ext_vector_type(4)));
    out += (lane & 3) * 16 + 4 * (lane >> 4);
    m += lane & 12;
    if (accumulate) {
        transpose4(lane, s0, s1, s2, s3);
        const float4_t sums[4] = {s0, s1, s2, s3};
        out4_t before[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) before[k] = *(const out4_t*)(out + (size_t)min(m + k, lm - 1) * ln);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            out4_t v;
#pragma unroll
            for (int w = 0; w < 4; ++w) v[w] = (OUT)(sums[k][w] + (float)before[k][w]);
            if (m + k < lm) __builtin_nontemporal_store(v, (out4_t*)(out + (size_t)(m + k) * ln));
        }
    } else {
        const float4_t sums[4] = {s0, s1, s2, s3};
        out4_t v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int w = 0; w < 4; ++w) v[j][w] = (OUT)sums[j][w];
        transpose4(lane, v[0], v[1], v[2], v[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (m + k < lm) __builtin_nontemporal_store(v[k], (out4_t*)(out + (size_t)(m + k) * ln));
    }
}

// Half a unit of "columns": rows of 8 slabs.  One transposed read takes its 16 rows in two goes of 8.
__device__ __forceinline__ int half_swizzle(int r) { return (r & 3) | (((r >> 3) & 1) << 2); }

// GM: the tokens' side is m (W2: d_out), else it is n (x).
template <typename OUT, bool GM>
struct WeightsTile {
    static constexpr int kA = 2, kB = 3, kRuns = 4, kHalf = 16384;          // a half of m: 64 rows of 128 columns
    static constexpr int kRingB = 2 * kA * kHalf;
    static constexpr bool kLate = true;
    const TrainWeights& a;
    const WeightsWork& c;
    uint8_t* lds;
    uint32_t lds0, put_a, put_b, get_a, get_b;
    int lane, group, wn;
    gptr_t base_a, base_b;
    uint32_t ld_a, ld_b;                 // bytes of a row
    const_ints_t tok;                    // tokens of the rows that are brought next of the gathered operand: 16 of m, 8 of n
    int next[GM ? 16 : 8];               // the same, asked for a phase before they are used
    uint32_t va[4], vb[4];               // gathered: what the lane brings of a row
    uint32_t at_m, at_n;
    float4_t acc[4][8];
    half8_t fm[2][8], fn[2][4];

    __device__ __forceinline__ int row_a(int k) const { return 16 * wn + 4 * k + (lane >> 4); }
    __device__ __forceinline__ int row_b(int k) const { return 32 * group + 8 * wn + 2 * k + (lane >> 5); }

    __device__ __forceinline__ WeightsTile(const TrainWeights& a_, const WeightsWork& c_, uint8_t* lds_) : a(a_), c(c_), lds(lds_) {
        lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
        lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        group = wave >> 2;
        wn = wave & 3;
        ld_a = (uint32_t)c.lm * 2;
        ld_b = (uint32_t)c.ln * 2;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int pa = lane & 15, pb = lane & 31;
            const int col_a = (1 - group) * 128 + ((((pa >> 1) ^ half_swizzle(row_a(k))) << 1) | (pa & 1)) * 8;
            const int col_b = ((((pb >> 1) ^ slab_swizzle(row_b(k))) << 1) | (pb & 1)) * 8;
            va[k] = (uint32_t)(c.m0 + min(col_a, c.lm - 8 - c.m0)) * 2 + (GM ? 0 : (uint32_t)row_a(k) * ld_a);
            vb[k] = (uint32_t)(c.n0 + min(col_b, c.ln - 8 - c.n0)) * 2 + (!GM ? 0 : (uint32_t)row_b(k) * ld_b);
        }
        tok = (const_ints_t)(uintptr_t)uniform_ptr(a.tok + c.begin + (GM ? 16 * wn : 32 * group + 8 * wn));
        look_up();
        base_a = uniform_ptr(c.m + (GM ? 0 : (size_t)c.begin * c.lm));
        base_b = uniform_ptr(c.n + (!GM ? 0 : (size_t)c.begin * c.ln));
        put_a = lds0 + (1 - group) * kA * kHalf;
        get_a = lds0 + group * kA * kHalf;
        put_b = get_b = lds0 + kRingB;
        const int row = 8 * (lane >> 4) + ((lane & 15) >> 2);
        at_m = row * 256 + (lane & 3) * 8 + (half_swizzle(row) << 5);
        at_n = columns_at(lane, 4 * wn);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    __device__ __forceinline__ void look_up() {
#pragma unroll
        for (int k = 0; k < (GM ? 16 : 8); ++k) next[k] = tok[k];
    }
    __device__ __forceinline__ void look_up_rows() {
        if (GM) look_up();
    }
    __device__ __forceinline__ void look_up_matrix() {
        if (!GM) look_up();
    }
    // Where a token's row begins, worked out by the scalar unit.
    __device__ __forceinline__ uint32_t row_at(int i, uint32_t ld) const {
        uint32_t v = (uint32_t)next[i] * ld;
        asm volatile("" : "+s"(v));
        return v;
    }
    // (Past the last row of the expert: other rows, cleared before they are read.)
    __device__ __forceinline__ void bring_rows(int k) {
        uint32_t v = va[k];
        if (GM) {
            const uint32_t r0 = row_at(4 * k, ld_a), r1 = row_at(4 * k + 1, ld_a), r2 = row_at(4 * k + 2, ld_a), r3 = row_at(4 * k + 3, ld_a);
            const uint32_t lo = lane & 16 ? r1 : r0, hi = lane & 16 ? r3 : r2;
            v += lane & 32 ? hi : lo;
        }
        moemix::bring<0>(put_a + wn * 4096 + k * 1024, base_a, v);
    }
    __device__ __forceinline__ void rows_asked(bool more) {
        const uint32_t ring = lds0 + (1 - group) * kA * kHalf;
        put_a = put_a == ring + (kA - 1) * kHalf ? ring : put_a + kHalf;
        if (!more) return;
        if (GM) tok += kTrainStep;
        else base_a += (size_t)ld_a * kTrainStep;
    }
    __device__ __forceinline__ void bring_matrix(int k) {
        uint32_t v = vb[k];
        if (!GM) {
            const uint32_t r0 = row_at(2 * k, ld_b), r1 = row_at(2 * k + 1, ld_b);
            v += lane & 32 ? r1 : r0;
        }
        moemix::bring<0>(put_b + group * (kUnit / 2) + wn * 4096 + k * 1024, base_b, v);
    }
    __device__ __forceinline__ void matrix_asked(bool more) {
        put_b = put_b == lds0 + kRingB + (kB - 1) * kUnit ? lds0 + kRingB : put_b + kUnit;
        if (!more) return;
        if (!GM) tok += kTrainStep;
        else base_b += (size_t)ld_b * kTrainStep;
    }
    // Rows past the expert's last one, whatever they hold, are zeros on both sides.
    __device__ __forceinline__ void rows_there(int step) {
        const int there = c.rows - step * kTrainStep;
        if (there >= kTrainStep || there <= 0) return;
        const int l = (int)fresh_offset(lane);      // (worked out here: hoisted, the addresses would cost registers in every step)
        uint8_t* const at = lds + (1 - group) * kA * kHalf + step % kA * kHalf + wn * 4096 + l * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (16 * wn + 4 * k + (l >> 4) >= there) *(uint4_t*)(at + k * 1024) = uint4_t{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void matrix_there(int step) {
        const int there = c.rows - step * kTrainStep;
        if (there >= kTrainStep || there <= 0) return;
        const int l = (int)fresh_offset(lane);
        uint8_t* const at = lds + kRingB + step % kB * kUnit + group * (kUnit / 2) + wn * 4096 + l * 16;
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (32 * group + 8 * wn + 2 * k + (l >> 5) >= there) *(uint4_t*)(at + k * 1024) = uint4_t{0u, 0u, 0u, 0u};
    }
    static constexpr int kReads = 24;
    __device__ __forceinline__ void read(int r) {
        if (r < 8) fn[r & 1][r >> 1] = read_columns<512>((get_b + at_n) ^ ((r >> 1) << 5), r & 1);
        else fm[r & 1][(r - 8) >> 1] = read_columns<256>((get_a + at_m) ^ (((r - 8) >> 1) << 5), r & 1);
    }
    __device__ __forceinline__ void step_read() {
        const uint32_t ring = lds0 + group * kA * kHalf;
        get_a = get_a == ring + (kA - 1) * kHalf ? ring : get_a + kHalf;
        get_b = get_b == lds0 + kRingB + (kB - 1) * kUnit ? lds0 + kRingB : get_b + kUnit;
    }
    __device__ __forceinline__ void multiply() {
#pragma unroll
        for (int g = 0; g < 16; ++g) {
            const int kk = g / 8, i = g % 8;
#pragma unroll
            for (int to = 0; to < 4; ++to) {
                const int j = g & 1 ? 3 - to : to;
                acc[j][i] = mfma16(fn[kk][j], fm[kk][i], acc[j][i]);
            }
            if (g % 4 == 0) {
                pin_schedule();
                if (g == 0) look_up_rows();
                bring_matrix(g / 4);
                pin_schedule();
            }
        }
    }
    __device__ __forceinline__ void write() {
        if (c.n0 + wn * 64 >= c.ln) return;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            write_sums<OUT>(lane, acc[0][i], acc[1][i], acc[2][i], acc[3][i], (OUT*)c.out + c.n0 + wn * 64, c.m0 + (group * 8 + i) * 16, c.lm, c.ln, a.accumulate);
    }
};

template <typename OUT>
__global__ __launch_bounds__(kThreads, 2) void train_weights_kernel(TrainWeights a, int tiles_f, int tiles_d) {
    extern __shared__ uint8_t lds[];
    // Workgroups go to the 8 XCDs in turn: each takes an eighth of every matrix, neighbouring tiles, the matrices of the experts with most rows first.
    const int per_xcd = (tiles_f * tiles_d + 7) >> 3, slot = blockIdx.x >> 3;
    const int matrix = __builtin_amdgcn_readfirstlane(slot / per_xcd), t = (blockIdx.x & 7) * per_xcd + slot - matrix * per_xcd;
    if (t >= tiles_f * tiles_d) return;
    const int place = matrix / 3, which = matrix - 3 * place, e = __builtin_amdgcn_readfirstlane(a.meta->order[place]);
    WeightsWork c;
    c.out = which == 0 ? a.w1[e] : which == 1 ? a.w3[e] : a.w2[e];
    if (!c.out) return;
    c.begin = __builtin_amdgcn_readfirstlane(a.meta->offsets[e]);
    c.rows = __builtin_amdgcn_readfirstlane(a.meta->offsets[e + 1]) - c.begin;
    if (c.rows == 0 && a.accumulate) return;
    // eight tiles of m side by side
    const int tiles_m = which == 2 ? tiles_d : tiles_f, tiles_n = which == 2 ? tiles_f : tiles_d;
    const int group = t / (8 * tiles_n), rest = t - group * 8 * tiles_n, in_group = min(8, tiles_m - group * 8);
    const int tn = rest / in_group, tm = group * 8 + rest - tn * in_group;
    c.m = which == 0 ? a.d_a : which == 1 ? a.d_u : a.d_out;
    c.n = which == 2 ? a.h : a.x;
    c.lm = which == 2 ? a.d : a.f;
    c.ln = which == 2 ? a.f : a.d;
    c.m0 = tm * kTrainCols;
    c.n0 = tn * kTrainCols;
    auto body = [&](auto gather_m) {
        WeightsTile<OUT, decltype(gather_m)::value> w(a, c, lds);
        if (c.rows) run_steps(w, (c.rows + kTrainStep - 1) / kTrainStep, w.group);
        w.write();
    };
    if (which == 2) body(std::true_type{});
    else body(std::false_type{});
}

// Few rows for each expert, or little work in all: what counts is that the gradients are written, so a workgroup is small (four wavefronts, 32 KB of LDS, three of them per compute unit: two,
// with 180 registers, took 238 us in place of 230 for 256 tokens, 32 experts of 2048 x 1408) and goes over `turns` tiles of 128 x 128 side by side; what the next one multiplies is on
// the way, through registers, while a tile is written (16 tokens in the Mixtral shape with 1, 2, 4, 8 tiles: 1217, 1114, 1075, 1047 us; of 2048 x 1408: 278, 272, 266, 279).
// Bound by the writes: 2.8 GB of fp16 gradients, 16 tokens in the Mixtral shape, in 550 us, 5.1 TB/s.
constexpr int kFewTile = 128, kFewThreads = 256, kFewTurns = 4;

template <typename OUT>
__global__ __launch_bounds__(kFewThreads, 3) void train_weights_few_kernel(TrainWeights a, int per_matrix, int turns) {
    __shared__ uint4_t lds[2][kTrainStep * kFewTile * 2 / 16];
    const int matrix = __builtin_amdgcn_readfirstlane(blockIdx.x / per_matrix), t = blockIdx.x - matrix * per_matrix, e = matrix / 3, which = matrix - 3 * e;
    const bool gather_m = which == 2;
    const int lm = gather_m ? a.d : a.f, ln = gather_m ? a.f : a.d, tiles_m = (lm + kFewTile - 1) / kFewTile, tiles_n = (ln + kFewTile - 1) / kFewTile;
    const int tn0 = __builtin_amdgcn_readfirstlane(t / tiles_m), m0 = (t - tn0 * tiles_m) * kFewTile, first = tn0 * turns, n_turns = min(turns, tiles_n - first);
    OUT* const out = (OUT*)(which == 0 ? a.w1[e] : which == 1 ? a.w3[e] : a.w2[e]);
    if (n_turns <= 0 || !out) return;
    const int begin = __builtin_amdgcn_readfirstlane(a.meta->offsets[e]), rows = __builtin_amdgcn_readfirstlane(a.meta->offsets[e + 1]) - begin;
    if (rows == 0 && a.accumulate) return;
    const gptr_t m = uniform_ptr(which == 0 ? a.d_a + (size_t)begin * lm : which == 1 ? a.d_u + (size_t)begin * lm : a.d_out);
    const gptr_t n = uniform_ptr(which == 2 ? a.h + (size_t)begin * ln : a.x);
    const int steps = (rows + kTrainStep - 1) / kTrainStep, all = steps * n_turns;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1, row0 = tid >> 4, col = (tid & 15) * 8;
    const int col_m = m0 + min(col, lm - 8 - m0);
    const int put = row0 * 16 + (((((tid & 15) >> 1) ^ half_swizzle(row0)) << 1) | (tid & 1));     // in 16 bytes; 16 rows on the swizzle is the same
    const int row = 8 * (lane >> 4) + ((lane & 15) >> 2);
    const uint32_t at = row * 256 + (lane & 3) * 8 + (half_swizzle(row) << 5);
    const uint32_t get_m = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4_t*)lds[0] + at, get_n = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4_t*)lds[1] + at;
    int tok[4];
    uint4_t vm[4], vn[4];
    float4_t acc[4][4];
    auto look_up = [&](int step) {
        const int at = begin + step * kTrainStep + (int)fresh_offset(row0);
#pragma unroll
        for (int k = 0; k < 4; ++k) tok[k] = a.tok[at + 16 * k];
    };
    auto ask = [&](int step, int turn) {
        const int n0 = (first + turn) * kFewTile, col_n = n0 + min(col, ln - 8 - n0), at = (int)fresh_offset(row0);
        // (32-bit offsets of tokens, and of rows within a step)
        const gptr_t step_m = gather_m ? m : m + (size_t)step * kTrainStep * lm * 2, step_n = gather_m ? n + (size_t)step * kTrainStep * ln * 2 : n;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t r = at + 16 * k, of_m = gather_m ? tok[k] : r, of_n = gather_m ? r : tok[k];
            vm[k] = *(const uint4_t __attribute__((address_space(1)))*)(step_m + (of_m * (uint32_t)lm * 2 + col_m * 2));
            vn[k] = *(const uint4_t __attribute__((address_space(1)))*)(step_n + (of_n * (uint32_t)ln * 2 + col_n * 2));
        }
    };
    auto clear = [&]() {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    };
    auto write = [&](int turn) {
        const int n0 = (first + turn) * kFewTile + wn * 64;
        if (n0 >= ln) return;
        const int l = (int)fresh_offset(lane);               // (worked out here: hoisted, the addresses would cost a workgroup its place beside two others)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            write_sums<OUT>(l, acc[0][i], acc[1][i], acc[2][i], acc[3][i], out + n0, m0 + wm * 64 + 16 * i, lm, ln, a.accumulate);
            pin_schedule();
        }
    };
    clear();
    if (rows == 0) {
        for (int turn = 0; turn < n_turns; ++turn) write(turn);
        return;
    }
    look_up(0);
    ask(0, 0);
    if (steps > 1) look_up(1);
    int step = 0, turn = 0;
    for (int k = 0; k < all; ++k) {
        const int there = rows - step * kTrainStep;          // rows past the expert's last one, whatever they hold, are zeros on both sides
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool is = row0 + 16 * i < there;
            lds[0][put + 256 * i] = is ? vm[i] : uint4_t{0u, 0u, 0u, 0u};
            lds[1][put + 256 * i] = is ? vn[i] : uint4_t{0u, 0u, 0u, 0u};
        }
        __syncthreads();
        const int step1 = step + 1 == steps ? 0 : step + 1, turn1 = step1 ? turn : turn + 1;
        if (k + 1 < all) {
            ask(step1, turn1);
            if (steps > 1) look_up(step1 + 1 == steps ? 0 : step1 + 1);
        }
        pin_schedule();
        const uint32_t at_m = fresh_offset(get_m), at_n = fresh_offset(get_n);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            if (kk * 32 >= there) break;
            half8_t fm[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) fm[i] = read_columns<256>(at_m ^ ((4 * wm + i) << 5), kk);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const half8_t fn = read_columns<256>(at_n ^ ((4 * wn + j) << 5), kk);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[j][i] = mfma16(fn, fm[i], acc[j][i]);
            }
        }
        if (!step1) {
            write(turn);
            clear();
        }
        step = step1;
        turn = turn1;
    }
}

int few_workgroups(int E, int d, int f) { return E * 3 * ((f + kFewTile - 1) / kFewTile) * ((d + kFewTile - 1) / kFewTile); }

template <typename OUT>
void launch_weights(const TrainWeights& a, int P, hipStream_t st) {
    const int few_f = (a.f + kFewTile - 1) / kFewTile, few_d = (a.d + kFewTile - 1) / kFewTile, few = few_workgroups(a.E, a.d, a.f);
    if (train_small_tiles(P, a.E, a.d, a.f)) {
        const int turns = few >= kFewTurns * 4 * 3 * (int)kComputeUnits ? kFewTurns : 1;
        const int per_matrix = std::max(few_f * ((few_d + turns - 1) / turns), few_d * ((few_f + turns - 1) / turns));
        train_weights_few_kernel<OUT><<<(unsigned)(a.E * 3 * per_matrix), kFewThreads, 0, st>>>(a, per_matrix, turns);
        return;
    }
    const int tiles_f = (a.f + kTrainCols - 1) / kTrainCols, tiles_d = (a.d + kTrainCols - 1) / kTrainCols;
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = train_weights_kernel<OUT>;
    allow_lds((const void*)kernel, kLdsBytes, configured);
    kernel<<<(unsigned)(a.E * 3 * ((tiles_f * tiles_d + 7) / 8) * 8), kThreads, kLdsBytes, st>>>(a, tiles_f, tiles_d);
}

// ---- the grouping, and the rows of a token

// Which chunks share their contraction, and among how many workgroups.  What fills whole rounds of the chip is left alone; of the rest, which would leave most of it idle
// or add a round, each is cut in s parts.  In units of a full tile's time (steps of the contraction at 2250 cycles): `cost` of all tiles of the rest, the longest `most`; a workgroup's
// beginning and end are 7.5 steps, a partial result is written and read back.
// Lane l < 32 of a wavefront reckons with l % 16 + 1 parts, for down (l < 16) or d_rows.
__device__ TrainSplit choose_splits(int lane, int n_chunks, int whole, float chunk_cost, float most, int rows, int n_tiles, int steps, int most_splits) {
    const int s = (lane & 15) + 1, left = n_chunks - whole, workgroups = left * n_tiles * s;
    const float parts = __builtin_amdgcn_rcpf((float)s), step = __builtin_amdgcn_rcpf((float)steps);
    const float rounds = (float)((workgroups + kComputeUnits - 1) / kComputeUnits), partial = ((float)rows * (float)n_tiles * 3e-4f + 0.15f) * step;
    float time = (rounds == 1.0f ? most * parts : (float)n_tiles * chunk_cost / kComputeUnits + 0.5f * most * parts) + rounds * 7.5f * step + (float)(s - 1) * partial;
    if (s > 1) time *= 1.03f;                                // (worth it only if it is more than nothing)
    if (s > most_splits || s > steps || (s > 1 && workgroups > kMostSplit)) time = 1e30f;
    int best = s;
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        const float other = __shfl_xor(time, m, kWave);
        const int other_s = __shfl_xor(best, m, kWave);
        if (other < time || (other == time && other_s < best)) {
            time = other;
            best = other_s;
        }
    }
    return best == 1 || !left ? TrainSplit{n_chunks, 1} : TrainSplit{whole, best};
}

__global__ __launch_bounds__(256) void train_group_kernel(TrainGrouping g, TrainWorkspace w, int d, int f) {
    __shared__ int32_t off[MOE_MAX_EXPERTS + 1], first_chunk[MOE_MAX_EXPERTS], chunk_rows[MOE_MAX_EXPERTS];
    __shared__ TrainSplit split[2];
    const int tid = threadIdx.x, P = g.T * g.k, E = g.E;
    if (tid < 64) {                                          // lane e looks after expert e
        int o = g.offsets ? (tid <= E ? g.offsets[tid] : 0) : tid ? P : 0;
        o = min(max(o, 0), P);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {                   // increasing, whatever they were
            const int before = __shfl_up(o, m, kWave);
            if (tid >= m) o = max(o, before);
        }
        const int begin = __shfl(o, tid < E ? tid : E, kWave), end = __shfl(o, tid < E ? tid + 1 : E, kWave);
        const int rows = end - begin, fewest = (rows + w.most_rows - 1) / w.most_rows;
        const int size = fewest ? (rows + 32 * fewest - 1) / (32 * fewest) * 32 : 0, chunks = size ? (rows + size - 1) / size : 0;
        int first = 0, n_chunks = 0, rank = 0;
        for (int e = 0; e < E; ++e) {
            const int s = __builtin_amdgcn_readlane(size, e), n = __builtin_amdgcn_readlane(chunks, e), r = __builtin_amdgcn_readlane(rows, e);
            n_chunks += n;
            if (s > size || (s == size && e < tid)) first += n;
            rank += r > rows || (r == rows && e < tid);
        }
        const int tiles = (d + kTrainCols - 1) / kTrainCols, whole = n_chunks * tiles / (int)kComputeUnits * (int)kComputeUnits / tiles;
        // what is left of whole rounds: the lane's part
        const int mine = chunks ? max(0, min(first + chunks, n_chunks) - max(first, whole)) : 0;
        float cost = (float)mine * (0.25f + 0.75f / kTrainRows * (float)size), most = mine ? 0.25f + 0.75f / kTrainRows * (float)size : 0.0f;
        int left_rows = mine * size;
#pragma unroll
        for (int m = 32; m >= 1; m >>= 1) {
            cost += __shfl_xor(cost, m, kWave);
            most = fmaxf(most, __shfl_xor(most, m, kWave));
            left_rows += __shfl_xor(left_rows, m, kWave);
        }
        if (tid <= E) off[tid] = o;
        if (tid < E) {
            first_chunk[tid] = first;
            chunk_rows[tid] = size;
        }
        const TrainSplit chosen = choose_splits(tid, n_chunks, whole, cost, most, left_rows, tiles, f / kTrainStep * (tid < 16 ? 1 : 2), w.splits);
        if (tid == 0 || tid == 16) split[tid >> 4] = chosen;
        if (blockIdx.x == 0) {
            if (tid == 0) w.meta->down = chosen;
            if (tid == 16) w.meta->d_rows = chosen;
            if (tid <= E) w.meta->offsets[tid] = o;
            if (tid < E) w.meta->order[rank] = tid;
            if (tid == 0) {
                w.meta->lo = o;
                w.meta->n_chunks = n_chunks;
                w.meta->whole = TrainSplit{n_chunks, 1};
            }
            if (tid == E) w.meta->hi = o;
        }
    }
    __syncthreads();
    const int lo = off[0], hi = off[E];
    const int r = blockIdx.x * 256 + tid;
    if (r >= P + kTrainStep) return;
    int tok = 0;
    float gate = 0.0f;
    if (r >= lo && r < hi) {
        const int p = g.perm ? g.perm[r] : r;
        if ((unsigned)p < (unsigned)P) {
            tok = p / g.k;
            gate = g.topk_gate ? g.topk_gate[p] : 1.0f;
            w.inv[p] = r;
        }
        int e = 0;                                           // the last expert that begins at r or before, and has rows
        for (int m = MOE_MAX_EXPERTS / 2; m >= 1; m >>= 1)
            if (e + m < E && off[e + m] <= r) e += m;
        const int in_expert = r - off[e], rows = off[e + 1] - off[e], size = chunk_rows[e], c = in_expert / size, chunk = first_chunk[e] + c;
        w.shares[r] = (chunk >= split[0].first_split ? split[0].splits : 1) | (chunk >= split[1].first_split ? split[1].splits : 1) << 8;
        if (in_expert == c * size) {                         // the chunk's first row
            const int chunks = (rows + size - 1) / size, groups = (chunks + 7) / 8, most = (chunks + groups - 1) / groups, of = c / most * most;
            w.chunks[chunk] = TrainChunk{e, r, off[e + 1], size / 32 + (c - of) * 16 + min(most, chunks - of) * 256};
        }
    }
    w.tok[r] = tok;
    w.gate[r] = gate;
}

// One workgroup per token.  inv[p] is looked up in perm again: a pair in no group has whatever lay there.
template <typename OUT>
__global__ __launch_bounds__(256) void train_gather_kernel(TrainGrouping g, TrainWorkspace w, int forward, int d, OUT* __restrict__ out,
                                                           float* __restrict__ d_gate, int n_part) {
    typedef OUT out4_t __attribute__((ext_vector_type(4)));
    const int t = blockIdx.x, lane = threadIdx.x & 63, P = g.T * g.k, lo = w.meta->lo, hi = w.meta->hi;
    // lane s looks after slot s
    int row = -1, shares = 0;
    float gate = 1.0f;
    if (lane < g.k) {
        const int p = t * g.k + lane, r = w.inv[p];
        if (r >= lo && r < hi && (g.perm ? g.perm[r] : r) == p) {
            row = r;
            shares = forward ? w.shares[r] & 255 : w.shares[r] >> 8;
            if (forward) gate = w.gate[r];
        }
    }
    if (out)
        for (int c = threadIdx.x * 4; c < d; c += 1024) {
            float4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int s = 0; s < g.k; ++s) {
                const int r = __builtin_amdgcn_readlane(row, s), n = __builtin_amdgcn_readlane(shares, s);
                if (r < 0) continue;
                const float* const y = w.y + (size_t)r * d + c;
                float4_t v = *(const float4_t*)y;
                for (int p0 = 1; p0 < n; p0 += 4) {          // (four asked for at once)
                    float4_t part[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) part[p] = *(const float4_t*)(y + (size_t)min(p0 + p, n - 1) * P * d);
#pragma unroll
                    for (int p = 0; p < 4; ++p)
                        if (p0 + p < n) v += part[p];
                }
                sum += __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, gate), s)) * v;
            }
            out4_t o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = (OUT)sum[k];
            *(out4_t*)(out + (size_t)t * d + c) = o;
        }
    if (d_gate)                                              // a wavefront per slot: its n_part shares lie side by side
        for (int s = threadIdx.x >> 6; s < g.k; s += 4) {
            const int r = __builtin_amdgcn_readlane(row, s);
            float sum = 0.0f;
            if (r >= 0)
                for (int i = lane; i < n_part; i += 64) sum += w.part[(size_t)r * n_part + i];
            sum = wave_sum(sum);
            if (lane == 0) d_gate[t * g.k + s] = sum;
        }
}

}  // namespace

// Which of the two kernels, estimated (us) from the mean number of rows (how they are spread is known on the GPU only) for fp16 gradients that overwrite: a round of large tiles takes 9 and 1
// per step, one of three small workgroups per compute unit 4 and 1.8 per step, 1 where each is alone.  Backward pass, large and small tiles: 64 rows for each of 32 experts of 2048 x 1408, 297, 261 us; 128 for each, 368, 346; 256, 542, 564; 300 for each of 6 of
// 320 x 1408, 77, 64; 4096 for each of 2 of 2048 x 1408, 369, 408; 8 for each of 4 of 256 x 512, 33, 27.
bool train_small_tiles(int P, int E, int d, int f) {
    const int workgroups = few_workgroups(E, d, f);
    const int tiles = ((f + kTrainCols - 1) / kTrainCols) * ((d + kTrainCols - 1) / kTrainCols), per_xcd = E * 3 * ((tiles + 7) / 8);
    const float steps = (float)((P / E + kTrainStep - 1) / kTrainStep), full = 3.0f * kComputeUnits;
    const float large = (float)((per_xcd + 31) / 32) * (9.0f + steps);
    const float small = std::max((float)workgroups / full, 1.0f) * (4.0f + steps * (workgroups <= (int)kComputeUnits ? 1.0f : workgroups <= 2 * (int)kComputeUnits ? 1.4f : 1.8f));
    return small <= large;
}

int train_most_splits(int P, int d) {
    const float rounds = (float)P / kTrainRows * (float)((d + kTrainCols - 1) / kTrainCols) / kComputeUnits;
    return rounds >= 8.0f ? 1 : rounds >= 4.0f ? 2 : rounds >= 1.0f ? 4 : rounds >= 0.25f ? 8 : kTrainMostSplits;
}

// As long as all chunks, were they half as long, still made one round of workgroups, they are: steps of few rows are quicker (forward of 400 tokens, 2 experts of 1024 x 1024, 47 -> 27 us, of 200
// tokens, 4096 x 4096, 104 -> 58; up to two rounds in place of one: of 333 tokens, 8 experts of 1024 x 2816, 53 -> 60).  Each chunk reads its matrix, so where that comes from memory they stay
// longer (backward of 150 tokens, 2 experts of 4096 x 8192, chunks of up to 256, 128, 64, 32 rows: 222, 222, 214, 239 us; 120 tokens, one of 4096 x 14336: 241, 241, 221, 235).
int train_most_rows(int P, int E, int d, int f, int tiles_f, int tiles_d) {
    const int least = matrices_past_caches(E, d, f) ? 64 : 32;
    int rows = kTrainRows;
    while (rows > least && (long long)(P / (rows / 2) + std::min(E, P)) * std::max(tiles_f, tiles_d) <= kComputeUnits) rows /= 2;
    return rows;
}

void launch_train_group(const TrainGrouping& g, const TrainWorkspace& w, int d, int f, hipStream_t st) {
    const int P = g.T * g.k;
    train_group_kernel<<<(P + kTrainStep + 255) / 256, 256, 0, st>>>(g, w, d, f);
}

void launch_train_up(const TrainRows& a, hipStream_t st) { launch_rows<kUp>(a, st); }
void launch_train_down(const TrainRows& a, hipStream_t st) { launch_rows<kDown>(a, st); }
void launch_train_d_hidden(const TrainRows& a, hipStream_t st) { launch_rows<kDHidden>(a, st); }
void launch_train_d_rows(const TrainRows& a, hipStream_t st) { launch_rows<kDRows>(a, st); }
void launch_train_d_weights(const TrainWeights& a, int P, bool half_out, hipStream_t st) {
    if (half_out) launch_weights<half_t>(a, P, st);
    else launch_weights<float>(a, P, st);
}

void launch_train_gather(const TrainGrouping& g, const TrainWorkspace& w, bool forward, int d, void* out, bool half_out, float* d_gate, int n_part,
                         hipStream_t st) {
    if (half_out) train_gather_kernel<half_t><<<g.T, 256, 0, st>>>(g, w, forward, d, (half_t*)out, d_gate, n_part);
    else train_gather_kernel<float><<<g.T, 256, 0, st>>>(g, w, forward, d, (float*)out, d_gate, n_part);
}

}  // namespace moemix
