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
#include "experts_train.hpp"
#include "kernels.hpp"
#include "mfma_common.hpp"

namespace moemix {

namespace {

constexpr int kLdsBytes = 163840;        // of a compute unit
constexpr int kUnit = 32768;             // 256 rows of 64 elements, or 64 rows of 256
constexpr int kThreads = 512;

enum Form { kUp, kDown, kDHidden, kDRows };

typedef const int32_t __attribute__((address_space(4)))* const_ints_t;

typedef short short4v_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v_t* lds_short4_t;

// ---- operands in LDS

// "Columns": slabs of 16 columns (32 bytes) of row r are stored at slab ^ slab_swizzle(r): the 16 rows that one transposed read takes
// then lie in 16 different slabs, so no two of them in the same bank.
__device__ __forceinline__ int slab_swizzle(int r) { return (r & 3) | (((r >> 3) & 3) << 2); }

// 8 consecutive contraction elements (kk: 32 kk + 8 q ..) of column r16 of a slab; at: the lane's address for it (columns_at) in the unit.
__device__ __forceinline__ half8_t read_columns(uint32_t at, int kk) {
    const short4v_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(uintptr_t)(at + kk * 16384));
    const short4v_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4_t)(uintptr_t)(at + kk * 16384 + 2048));
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

__device__ __forceinline__ float sigmoid(float a) { return 1.0f / (1.0f + __expf(-a)); }

// ---- who does what when
//
// The 8 wavefronts of a workgroup are two groups of four, one of each per SIMD.  A step of the contraction (64 elements) takes each group two phases: it reads the
// operands of the step from LDS into registers, then it multiplies them.  The groups are one phase apart, so that in every phase one of them feeds the matrix cores and
// the other reads, and all meet at its end.  Group 0 brings the matrix's side into LDS while it reads, group 1 the other side:
//   phase 2k:     group 0 reads step k and asks for B of step k + nB - 1; group 1 multiplies step k - 1
//   phase 2k + 1: group 1 reads step k and asks for A of step k + nA - 1; group 0 multiplies step k
// A ring of nA (nB) units holds them: the unit that is written was read last in phase 2k - 1.  What is read from phase 2k + 2 on has been waited for by who
// brought it before the end of phase 2k + 1.

// The wavefront's own transfers but the last `later` stages of RUNS each are done.
template <int RUNS>
__device__ __forceinline__ void wait_stages(int later) {
    if (later <= 0) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if (later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(RUNS) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * RUNS) : "memory");
}
__device__ __forceinline__ void meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// TILE: kRunsA, kRunsB (transfers of a wavefront per stage), kStagesA, kStagesB (units of the rings, at most 4), bring() (the next stage of the wavefront's side),
// landed(step) (after its transfers have ended, before others read them), read() (the next step), multiply().
template <typename TILE>
__device__ __forceinline__ void run_steps(TILE& t, int n, int group) {
    const int ahead = group ? TILE::kStagesA - 1 : TILE::kStagesB - 1;     // stages asked for before step k's
    auto wait = [&](int step) {                                            // step's stage is there
        const int later = min(ahead - 1, n - 1 - step);
        if (group) wait_stages<TILE::kRunsA>(later);
        else wait_stages<TILE::kRunsB>(later);
        t.landed(step);
    };
    for (int k = 0; k < ahead && k < n; ++k) t.bring();
    {
        const int later = min(ahead, n) - 1;
        if (group) wait_stages<TILE::kRunsA>(later);
        else wait_stages<TILE::kRunsB>(later);
        t.landed(0);
    }
    meet();
    if (group) meet();
    for (int k = 0; k < n; ++k) {
        if (k + ahead < n) t.bring();
        t.read();
        if (group && k + 1 < n) wait(k + 1);
        pin_schedule();
        meet();
        pin_schedule();
        __builtin_amdgcn_s_setprio(1);
        t.multiply();
        __builtin_amdgcn_s_setprio(0);
        pin_schedule();
        if (!group && k + 1 < n) wait(k + 1);
        if (!group || k + 1 < n) meet();
    }
}

// ---- products of rows

// What a workgroup works on: a chunk of up to 32 MT rows (group g the tiles of 16 rows MT g .. MT g + MT - 1), 256 columns from n0 on (up: 128 of each matrix; wavefront
// w of a group a quarter), contraction steps [s0, s1).
struct RowsWork {
    int expert, begin, rows, n0, s0, s1, split;
};

template <int FORM, int MT>
struct RowsTile {
    static constexpr bool kColumns = FORM == kDHidden || FORM == kDRows;     // how the matrix lies
    static constexpr int kA = MT * 4096;                                    // bytes of a unit of rows
    static constexpr int kRunsA = MT, kRunsB = 8;
    static constexpr int kStagesA = MT > 4 ? 3 : 4, kStagesB = MT > 4 ? 2 : MT > 2 ? 3 : 4;
    static_assert(kStagesA * kA + kStagesB * kUnit <= kLdsBytes, "LDS");
    static constexpr int kRingB = kStagesA * kA;                            // where the matrix's ring begins
    const TrainRows& a;
    const RowsWork& c;
    uint32_t lds0, put, get_a, get_b;    // LDS addresses: the ring of what the wavefront brings, where its next stage goes; the next step to read
    int lane, group, wn;
    gptr_t base[2];
    uint32_t v[8];
    int left;                            // d_rows: stages before the second half
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
        // run k of the wavefront: rows: 8 rows of 64 elements, run wn + 4 k of the unit; columns: two rows of 256, run 8 wn + k
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (group) {
                const int row = min((wn + 4 * k) * 8 + row_in_run, c.rows - 1);     // (past the last row: the last one again)
                v[k] = k < MT ? (uint32_t)(gathered ? a.tok[c.begin + row] : row) * (uint32_t)K * 2 + piece : 0;
            } else if (kColumns) {
                const int row = 16 * wn + 2 * k + (lane >> 5), p = lane & 31;
                const int col = ((((p >> 1) ^ slab_swizzle(row)) << 1) | (p & 1)) * 8;
                v[k] = (uint32_t)row * (uint32_t)N * 2 + (uint32_t)min(col, N - 8 - c.n0) * 2;
            } else {
                const int row = (wn + 4 * (FORM == kUp ? k & 3 : k)) * 8 + row_in_run;
                v[k] = (uint32_t)min(row, N - 1 - c.n0) * (uint32_t)K * 2 + piece;
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
        put = group ? lds0 : lds0 + kRingB;
        get_a = lds0;
        get_b = lds0 + kRingB;
        seek(c.s0);
    }

    // The next stage to bring is step s.  (d_rows: the second half of the steps is d_u's and W3's.)
    __device__ __forceinline__ void seek(int s) {
        const size_t N = a.N, K = a.K;
        const int e = c.expert, half = FORM == kDRows ? a.K / kTrainStep : 0;
        const bool second = FORM == kDRows && s >= half;
        const size_t k0 = (size_t)(second ? s - half : s) * kTrainStep;
        const half_t* p[2];
        if (group) {
            p[0] = p[1] = (second ? a.in2 : a.in) + (FORM == kDown || FORM == kDRows ? (size_t)c.begin * K : 0) + k0;
        } else if (kColumns) {
            p[0] = p[1] = (second ? a.w3[e] : a.w[e]) + k0 * N + c.n0;
        } else {
            p[0] = a.w[e] + (size_t)c.n0 * K + k0;
            p[1] = (FORM == kUp ? a.w3[e] : a.w[e]) + (size_t)c.n0 * K + k0;
        }
        base[0] = uniform_ptr(p[0]);
        base[1] = FORM == kUp ? uniform_ptr(p[1]) : base[0];
        left = second || FORM != kDRows ? 1 << 30 : half - s;
    }

    __device__ __forceinline__ void bring() {
        const uint32_t first = group ? put + wn * 1024 : put + wn * (kColumns ? 8192 : 1024);
        const uint32_t apart = group || !kColumns ? 4096 : 1024;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < MT || !group) moemix::bring<0>(first + k * apart, base[FORM == kUp && k >= 4], v[k]);
        if (group) put = put == lds0 + (kStagesA - 1) * kA ? lds0 : put + kA;
        else put = put == lds0 + kRingB + (kStagesB - 1) * kUnit ? lds0 + kRingB : put + kUnit;
        if (FORM == kDRows && --left == 0) {
            seek(a.K / kTrainStep);
            return;
        }
        const size_t step = !group && kColumns ? (size_t)a.N * (kTrainStep * 2) : kTrainStep * 2;
        base[0] += step;
        if (FORM == kUp) base[1] += step;
    }
    __device__ __forceinline__ void landed(int) {}

    __device__ __forceinline__ void read() {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (kColumns) fb[kk][j] = read_columns(get_b + rb[j], kk);
                else {
                    const uint32_t row0 = FORM == kUp ? (j >> 1) * 128 + wn * 32 + (j & 1) * 16 : wn * 64 + j * 16;
                    fb[kk][j] = read_rows(get_b + row0 * 128 + rb[kk]);
                }
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) fa[kk][i] = read_rows(get_a + (group * MT + i) * 2048 + ra[kk]);
        }
        get_a = get_a == lds0 + (kStagesA - 1) * kA ? lds0 : get_a + kA;
        get_b = get_b == lds0 + kRingB + (kStagesB - 1) * kUnit ? lds0 + kRingB : get_b + kUnit;
    }
    __device__ __forceinline__ void multiply() {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][i] = mfma16(fb[kk][j], fa[kk][i], acc[j][i]);
    }

    // lane: row r16 of a tile of rows, columns 4 q .. 4 q + 3 of a tile of the matrix
    __device__ __forceinline__ void write(uint8_t* lds) {
        const int r16 = lane & 15, q = lane >> 4, N = a.N;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = (group * MT + i) * 16 + r16;
            const bool there = r < c.rows;
            const size_t row = (size_t)(c.begin + (there ? r : 0));
            if (FORM == kUp) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int n = c.n0 + wn * 32 + j * 16 + 4 * q;
                    if (!there || n >= N) continue;
                    half4_t va, vu, vh;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        va[k] = (half_t)acc[j][i][k];
                        vu[k] = (half_t)acc[j + 2][i][k];
                        vh[k] = (half_t)silu_mul(acc[j][i][k], acc[j + 2][i][k]);
                    }
                    *(half4_t*)(a.a + row * N + n) = va;
                    *(half4_t*)(a.u + row * N + n) = vu;
                    *(half4_t*)(a.h + row * N + n) = vh;
                }
            } else if (FORM == kDHidden) {
                const float g = a.gate[row];
                float share = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int col = c.n0 + wn * 64 + j * 16 + 4 * q, n = min(col, N - 4);
                    const bool mine = there && col < N;
                    const half4_t va = *(const half4_t*)(a.a + row * N + n), vu = *(const half4_t*)(a.u + row * N + n);
                    half4_t da, du, gh;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float x = (float)va[k], y = (float)vu[k], s = sigmoid(x), z = x * s, h = z * y, v = acc[j][i][k];
                        share = mine ? fmaf(v, h, share) : share;
                        du[k] = (half_t)(g * v * z);
                        da[k] = (half_t)(g * v * y * (s * (1.0f + x * (1.0f - s))));
                        gh[k] = (half_t)(g * h);
                    }
                    if (mine) {
                        *(half4_t*)(a.d_a + row * N + n) = da;
                        *(half4_t*)(a.d_u + row * N + n) = du;
                        *(half4_t*)(a.h + row * N + n) = gh;
                    }
                }
                share += __shfl_xor(share, 16, kWave);
                share += __shfl_xor(share, 32, kWave);
                if (q == 0) ((float*)lds)[wn * kTrainRows + r] = share;
            } else {
                float* const y = a.y + (size_t)c.split * a.P * N + row * N;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = c.n0 + wn * 64 + j * 16 + 4 * q;
                    if (there && n < N) *(float4_t*)(y + n) = acc[j][i];
                }
            }
        }
        if (FORM == kDHidden) {
            __syncthreads();
            const float* const s = (const float*)lds;
            for (int r = threadIdx.x; r < c.rows; r += kThreads)
                a.part[(size_t)(c.n0 / kTrainCols) * a.P + c.begin + r] =
                    (s[r] + s[kTrainRows + r]) + (s[2 * kTrainRows + r] + s[3 * kTrainRows + r]);
        }
    }
};

template <int FORM, int MT>
__device__ __forceinline__ void rows_body(const TrainRows& a, const RowsWork& c, uint8_t* lds) {
    RowsTile<FORM, MT> t(a, c, lds);
    run_steps(t, c.s1 - c.s0, t.group);
    __syncthreads();                     // (LDS is read no more)
    t.write(lds);
}

template <int FORM>
__global__ __launch_bounds__(kThreads, 2) void train_rows_kernel(TrainRows a, int n_tiles) {
    extern __shared__ uint8_t lds[];
    // Workgroups go to the 8 XCDs in turn: each XCD takes a run of neighbouring tiles, eight chunks side by side.
    const int n_chunks = __builtin_amdgcn_readfirstlane(a.meta->n_chunks);
    const int units = n_chunks * n_tiles, total = units * a.splits, per_xcd = (total + 7) >> 3;
    const int slot = blockIdx.x >> 3, t0 = (blockIdx.x & 7) * per_xcd + slot;
    if (slot >= per_xcd || t0 >= total) return;
    RowsWork c;
    c.split = __builtin_amdgcn_readfirstlane(t0 / units);
    const int t = t0 - c.split * units;
    const int group = t / (8 * n_tiles), rest = t - group * 8 * n_tiles, in_group = min(8, n_chunks - group * 8);
    const int tile = __builtin_amdgcn_readfirstlane(rest / in_group);
    const TrainChunk ch = a.chunks[group * 8 + rest - tile * in_group];
    c.expert = __builtin_amdgcn_readfirstlane(ch.expert);
    c.begin = __builtin_amdgcn_readfirstlane(ch.begin);
    c.rows = __builtin_amdgcn_readfirstlane(ch.rows);
    c.n0 = tile * (FORM == kUp ? kTrainCols / 2 : kTrainCols);
    const int steps = a.K / kTrainStep * (FORM == kDRows ? 2 : 1);
    c.s0 = __builtin_amdgcn_readfirstlane(steps * c.split / a.splits);
    c.s1 = __builtin_amdgcn_readfirstlane(steps * (c.split + 1) / a.splits);
    if (c.rows <= 32) rows_body<FORM, 1>(a, c, lds);
    else if (c.rows <= 64) rows_body<FORM, 2>(a, c, lds);
    else if (c.rows <= 128) rows_body<FORM, 4>(a, c, lds);
    else rows_body<FORM, 8>(a, c, lds);
}

template <int FORM>
void launch_rows(const TrainRows& a, hipStream_t st) {
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = train_rows_kernel<FORM>;
    allow_lds((const void*)kernel, kLdsBytes, configured);
    constexpr int kOut = FORM == kUp ? kTrainCols / 2 : kTrainCols;
    const int n_tiles = (a.N + kOut - 1) / kOut;
    const long long total = (long long)n_tiles * a.most_chunks * a.splits;
    kernel<<<(unsigned)((total + 7) / 8 * 8), kThreads, kLdsBytes, st>>>(a, n_tiles);
}

// ---- gradients of the matrices

struct WeightsWork {
    int begin, rows;             // of the expert
    const half_t *m, *n;         // [., lm], [., ln]
    bool gather_m, gather_n;
    int lm, ln, m0, n0;
    void* out;                   // [lm, ln]
};

template <typename OUT>
struct WeightsTile {
    static constexpr int kRunsA = 8, kRunsB = 8, kStagesA = 3, kStagesB = 2;
    static constexpr int kRingB = kStagesA * kUnit;
    const TrainWeights& a;
    const WeightsWork& c;
    uint8_t* lds;
    uint32_t lds0, put, get_a, get_b;
    int lane, group, wn;
    bool gather;
    gptr_t base;
    uint32_t ld;                         // bytes of a row of what the wavefront brings
    const_ints_t tok;                    // tokens of the rows that it brings next
    uint32_t v[8];                       // run k: rows 16 wn + 2 k, + 1 of a stage; gathered: what the lane brings of a row (v[0 .. 3])
    uint32_t at_m, at_n;
    float4_t acc[4][8];
    half8_t fm[2][8], fn[2][4];

    __device__ __forceinline__ WeightsTile(const TrainWeights& a_, const WeightsWork& c_, uint8_t* lds_) : a(a_), c(c_), lds(lds_) {
        lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
        lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        group = wave >> 2;
        wn = wave & 3;
        gather = group ? c.gather_m : c.gather_n;
        const int width = group ? c.lm : c.ln, col0 = group ? c.m0 : c.n0;
        ld = (uint32_t)width * 2;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int row = 16 * wn + 2 * k + (lane >> 5), p = lane & 31;
            const int col = ((((p >> 1) ^ slab_swizzle(row)) << 1) | (p & 1)) * 8;
            v[k] = (uint32_t)(col0 + min(col, width - 8 - col0)) * 2;
        }
        if (gather) {                    // (the pattern of a run depends on k & 1 and k >> 2)
            v[2] = v[4];
            v[3] = v[5];
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += (uint32_t)(16 * wn + 2 * k + (lane >> 5)) * ld;
        }
        tok = (const_ints_t)(uintptr_t)uniform_ptr(a.tok + c.begin + 16 * wn);
        base = uniform_ptr((group ? c.m : c.n) + (gather ? 0 : (size_t)c.begin * width));
        put = group ? lds0 : lds0 + kRingB;
        get_a = lds0;
        get_b = lds0 + kRingB;
        at_m = columns_at(lane, 8 * group);
        at_n = columns_at(lane, 4 * wn);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // (Past the last row of the expert: other rows, cleared before they are read.)
    __device__ __forceinline__ void bring() {
        const uint32_t first = put + wn * 8192;
        if (gather) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int t0 = tok[2 * k], t1 = tok[2 * k + 1];
                moemix::bring<0>(first + k * 1024, base, (uint32_t)(lane < 32 ? t0 : t1) * ld + v[(k >> 2) * 2 + (k & 1)]);
            }
            tok += kTrainStep;
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) moemix::bring<0>(first + k * 1024, base, v[k]);
            base += (size_t)ld * kTrainStep;
        }
        if (group) put = put == lds0 + (kStagesA - 1) * kUnit ? lds0 : put + kUnit;
        else put = put == lds0 + kRingB + (kStagesB - 1) * kUnit ? lds0 + kRingB : put + kUnit;
    }
    // Rows past the expert's last one, whatever they hold, are zeros on both sides.
    __device__ __forceinline__ void landed(int step) {
        const int there = c.rows - step * kTrainStep;
        if (there >= kTrainStep) return;
        uint8_t* const at = lds + (group ? step % kStagesA * kUnit : kRingB + step % kStagesB * kUnit) + wn * 8192 + lane * 16;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (16 * wn + 2 * k + (lane >> 5) >= there) *(uint4_t*)(at + k * 1024) = uint4_t{0u, 0u, 0u, 0u};
    }
    __device__ __forceinline__ void read() {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
#pragma unroll
            for (int j = 0; j < 4; ++j) fn[kk][j] = read_columns((get_b + at_n) ^ (j << 5), kk);
#pragma unroll
            for (int i = 0; i < 8; ++i) fm[kk][i] = read_columns((get_a + at_m) ^ (i << 5), kk);
        }
        get_a = get_a == lds0 + (kStagesA - 1) * kUnit ? lds0 : get_a + kUnit;
        get_b = get_b == lds0 + kRingB + (kStagesB - 1) * kUnit ? lds0 + kRingB : get_b + kUnit;
    }
    __device__ __forceinline__ void multiply() {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j][i] = mfma16(fn[kk][j], fm[kk][i], acc[j][i]);
    }
    __device__ __forceinline__ void write() {
        typedef OUT out4_t __attribute__((ext_vector_type(4)));
        const int r16 = lane & 15, q = lane >> 4;
        OUT* const out = (OUT*)c.out;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int m = c.m0 + (group * 8 + i) * 16 + r16;
            if (m >= c.lm) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int n = c.n0 + wn * 64 + j * 16 + 4 * q;
                if (n >= c.ln) continue;
                out4_t* const o = (out4_t*)(out + (size_t)m * c.ln + n);
                float4_t v = acc[j][i];
                if (a.accumulate) {
                    const out4_t before = *o;
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += (float)before[k];
                }
                out4_t w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = (OUT)v[k];
                *o = w;
            }
        }
    }
};

template <typename OUT>
__global__ __launch_bounds__(kThreads, 2) void train_weights_kernel(TrainWeights a, int tiles_f, int tiles_d) {
    extern __shared__ uint8_t lds[];
    const int per_matrix = tiles_f * tiles_d, total = a.E * 3 * per_matrix, per_xcd = (total + 7) >> 3;
    const int slot = blockIdx.x >> 3, t0 = (blockIdx.x & 7) * per_xcd + slot;
    if (slot >= per_xcd || t0 >= total) return;
    const int matrix = t0 / per_matrix, t = t0 - matrix * per_matrix, e = matrix / 3, which = matrix - 3 * e;
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
    c.gather_m = which == 2;
    c.gather_n = which != 2;
    c.lm = which == 2 ? a.d : a.f;
    c.ln = which == 2 ? a.f : a.d;
    c.m0 = tm * kTrainCols;
    c.n0 = tn * kTrainCols;
    WeightsTile<OUT> w(a, c, lds);
    if (c.rows) run_steps(w, (c.rows + kTrainStep - 1) / kTrainStep, w.group);
    w.write();
}

template <typename OUT>
void launch_weights(const TrainWeights& a, hipStream_t st) {
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = train_weights_kernel<OUT>;
    allow_lds((const void*)kernel, kLdsBytes, configured);
    const int tiles_f = (a.f + kTrainCols - 1) / kTrainCols, tiles_d = (a.d + kTrainCols - 1) / kTrainCols;
    const int total = a.E * 3 * tiles_f * tiles_d;
    kernel<<<(unsigned)((total + 7) / 8 * 8), kThreads, kLdsBytes, st>>>(a, tiles_f, tiles_d);
}

// ---- the grouping, and the rows of a token

__global__ __launch_bounds__(256) void train_group_kernel(TrainGrouping g, TrainWorkspace w, int per) {
    __shared__ int32_t off[MOE_MAX_EXPERTS + 1];
    const int tid = threadIdx.x, P = g.T * g.k;
    if (tid == 0) {
        int run = 0;
        for (int e = 0; e <= g.E; ++e) {
            const int o = g.offsets ? g.offsets[e] : e ? P : 0;
            run = max(run, min(max(o, 0), P));
            off[e] = run;
        }
    }
    __syncthreads();
    const int lo = off[0], hi = off[g.E];
    const int r = blockIdx.x * 256 + tid;
    if (r < P + 64) {
        int tok = 0;
        float gate = 0.0f;
        if (r >= lo && r < hi) {
            const int p = g.perm ? g.perm[r] : r;
            if ((unsigned)p < (unsigned)P) {
                tok = p / g.k;
                gate = g.topk_gate ? g.topk_gate[p] : 1.0f;
                w.inv[p] = r;
            }
        }
        w.tok[r] = tok;
        w.gate[r] = gate;
    }
    if (blockIdx.x == 0 && tid < MOE_MAX_EXPERTS) {
        int at = 0;
        for (int e = 0; e < tid && e < g.E; ++e) at += (off[e + 1] - off[e] + per - 1) / per;
        if (tid < g.E) {
            const int begin = off[tid], end = off[tid + 1];
            for (int b = begin; b < end; b += per) w.chunks[at++] = TrainChunk{tid, b, min(per, end - b), 0};
            if (tid == g.E - 1) {
                w.meta->lo = lo;
                w.meta->hi = hi;
                w.meta->n_chunks = at;
            }
        }
    }
    if (blockIdx.x == 0 && tid <= g.E) w.meta->offsets[tid] = off[tid];
}

// One workgroup per token.  inv[p] is looked up in perm again: a pair in no group has whatever lay there.
template <typename OUT>
__global__ __launch_bounds__(256) void train_gather_kernel(TrainGrouping g, TrainWorkspace w, int gates, int d, OUT* __restrict__ out,
                                                           float* __restrict__ d_gate, int n_part) {
    typedef OUT out4_t __attribute__((ext_vector_type(4)));
    const int t = blockIdx.x, P = g.T * g.k, lo = w.meta->lo, hi = w.meta->hi;
    auto row_of_pair = [&](int p) {
        const int r = w.inv[p];
        if (r < lo || r >= hi) return -1;
        return (g.perm ? g.perm[r] : r) == p ? r : -1;
    };
    if (out)
        for (int c = threadIdx.x * 4; c < d; c += 1024) {
            float4_t sum = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int s = 0; s < g.k; ++s) {
                const int r = row_of_pair(t * g.k + s);
                if (r < 0) continue;
                float4_t v = *(const float4_t*)(w.y + (size_t)r * d + c);
                for (int p = 1; p < w.splits; ++p) v += *(const float4_t*)(w.y + ((size_t)p * P + r) * d + c);
                if (gates) v *= w.gate[r];
                sum += v;
            }
            out4_t o;
#pragma unroll
            for (int k = 0; k < 4; ++k) o[k] = (OUT)sum[k];
            *(out4_t*)(out + (size_t)t * d + c) = o;
        }
    if (d_gate && threadIdx.x < g.k) {
        const int p = t * g.k + threadIdx.x, r = row_of_pair(p);
        float sum = 0.0f;
        if (r >= 0)
            for (int i = 0; i < n_part; ++i) sum += w.part[(size_t)i * P + r];
        d_gate[p] = sum;
    }
}

}  // namespace

TrainPlan plan_train(int P, int d, int f, int E) {
    TrainPlan p;
    p.per = kTrainRows;
    p.splits_down = p.splits_dx = 1;
    return p;
}

void launch_train_group(const TrainGrouping& g, const TrainWorkspace& w, int per, hipStream_t st) {
    const int P = g.T * g.k;
    train_group_kernel<<<(P + 64 + 255) / 256, 256, 0, st>>>(g, w, per);
}

void launch_train_up(const TrainRows& a, hipStream_t st) { launch_rows<kUp>(a, st); }
void launch_train_down(const TrainRows& a, hipStream_t st) { launch_rows<kDown>(a, st); }
void launch_train_d_hidden(const TrainRows& a, hipStream_t st) { launch_rows<kDHidden>(a, st); }
void launch_train_d_rows(const TrainRows& a, hipStream_t st) { launch_rows<kDRows>(a, st); }
void launch_train_d_weights(const TrainWeights& a, bool half_out, hipStream_t st) {
    if (half_out) launch_weights<half_t>(a, st);
    else launch_weights<float>(a, st);
}

void launch_train_gather(const TrainGrouping& g, const TrainWorkspace& w, bool gates, int d, void* out, bool half_out, float* d_gate, int n_part,
                         hipStream_t st) {
    if (half_out) train_gather_kernel<half_t><<<g.T, 256, 0, st>>>(g, w, gates, d, (half_t*)out, d_gate, n_part);
    else train_gather_kernel<float><<<g.T, 256, 0, st>>>(g, w, gates, d, (float*)out, d_gate, n_part);
}

}  // namespace moemix
