// Products of e4m3 rows and matrices where a matrix has many rows: tiles that stay in LDS and registers.
//
// Within a block of 128 columns the sum over k of x[m,k] w[n,k] is a plain product of codes; the two scales multiply it once per block, as it is added to
// the 32-bit result: one fused multiply-add per result and block beside 1/4 (fp8) or 1 (fp16) matrix instruction per 16 x 16 results and 32 columns.
//
// What multiplies the codes: v_mfma_f32_16x16x128_f8f6f4 takes them as they are, 4.6 PFLOP/s in registers, but of eight neighbouring products drops what lies
// more than 13 binary places below the largest (1.5e-5 of a result for normal operands; fp16 results round at 4.9e-4).  Results in 32 bits
// and hidden values, which are rounded again to three bits, get exact sums instead: codes expanded to fp16 (a conversion instruction for two) and
// v_mfma_f32_16x16x32_f16, half the rate.
//
// Bound: 2 n in out operations against n in + out in bytes; from some 200 rows of a matrix on the matrix cores.  4096 rows, 4096 -> 14336, fp16 results: 262-278 us,
// 1.73-1.84 PFLOP/s; matrix cores busy 0.46 of the cycles at 1.9 GHz (the clock gives way under load), no LDS conflicts.  Without the loads 245 us, without the
// scaling 243, without both 204: what is left are the waits of eight wavefronts that meet once a block.  A library product with one scale for a whole
// matrix, without the quantizer: 222 us.  1000 rows, 14336 -> 4096, exact sums: 143-150 us, 0.8 PFLOP/s, matrix cores busy 0.40.
//
// Why this tile: 256 rows of w and up to 256 of x are 128 results per lane, what the registers hold without a spill at two wavefronts per SIMD; and two are
// needed, since the scaling of one wavefront's products has to run beside the matrix instructions of the other (2.1 PFLOP/s in registers with one, 4.1 with two).
// Every code brought into LDS serves 256 results then; a stage is 66 KB at most (256 rows of x), so two to four are under way.
#include <atomic>
#include <cmath>
#include <type_traits>

#include "fp8.hpp"
#include "kernels.hpp"
#include "mfma_common.hpp"

namespace moemix {

namespace {

typedef int int8v_t __attribute__((ext_vector_type(8)));
typedef float4_t __attribute__((aligned(4))) float4_anywhere_t;
typedef half4_t __attribute__((aligned(2))) half4_anywhere_t;

__device__ __forceinline__ int8v_t join(uint4_t a, uint4_t b) {
    return int8v_t{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

constexpr int kLds = 163840;             // of a compute unit
constexpr int kCols = 256;               // rows of w per tile (up: 128 of w1 and 128 of w3)

// A chunk of TT tiles of 16 rows of x: 8 wavefronts = 2 (rows of x) x 4 (rows of w).  A wavefront multiplies half of the tiles (an odd one is the first
// half's) with 64 rows of w; the two that share a SIMD are one of each half.  A stage of LDS holds a block of 128 columns: x [16 TT][128], w [256][128],
// scales [8][64].
template <int TT>
struct Tile {
    static constexpr int kX = TT * 2048, kW = kCols * 128, kScales = 2048;
    static constexpr int kStage = kX + kW + kScales;
    static constexpr int kStages = 4 * kStage <= kLds ? 4 : 3 * kStage <= kLds ? 3 : 2;
    static_assert(kStages * kStage <= kLds, "LDS");
    static constexpr int kRuns = 2 * TT;                     // runs of 8 rows (1 KB) of x; the first kRuns % 8 wavefronts (0: all) bring one more
    static constexpr int kMost = (kRuns + 7) / 8, kMore = kRuns % 8;
};

struct TileWork {
    int expert, n0, begin, rows;         // rows [begin, begin + rows) of y, results from n0 on
};

// MT tiles of the chunk, those from `tile0` on, are the wavefront's.
template <int TT, int MT, bool F8, bool UP, typename OUT>
__device__ __forceinline__ void tile_body(const Fp8Args& a, const TileWork& c, uint8_t* lds, int tile0) {
    typedef Tile<TT> L;
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wn = wave & 3;
    const int N = a.N, K = a.K, e = c.expert, n0 = c.n0, rows = c.rows;
    const int blocks = (K + kFp8Block - 1) / kFp8Block, tail = K - (blocks - 1) * kFp8Block;   // bytes of the last block
    const bool more = !L::kMore || wave < L::kMore;
    // ---- what it brings: lane l the 16-byte slot l & 7 of row l >> 3 of a run of 8 rows; runs wave, wave + 8, ...
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    // a run's first row modulo 16 is 8 (run & 1), and run and wave have the same parity
    const int piece = ((lane & 7) ^ swizzle128(8 * (wave & 1) + (lane >> 3))) * 16;
    uint32_t xv[L::kMost], wv[4];
    gptr_t xb = scalar_ptr(a.perm ? a.x : a.x + (size_t)c.begin * K);
#pragma unroll
    for (int k = 0; k < L::kMost; ++k) {
        const int row = min((wave + 8 * k) * 8 + (lane >> 3), rows - 1);      // (rows past the last one: the last one again)
        xv[k] = (uint32_t)(a.perm ? row_of(a, c.begin + row) : row) * (uint32_t)K + piece;
    }
    // w: runs wave, wave + 8, .. of 32; up: the first 16 are w1's
    gptr_t wb[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const Fp8Mat& m = UP && t ? a.w3[e] : a.w[e];
        const int row0 = min(UP ? n0 : n0 + 128 * t, N - 1);
        wb[t] = scalar_ptr(m.data + (size_t)row0 * K);
#pragma unroll
        for (int k = 0; k < 2; ++k) wv[2 * t + k] = (uint32_t)min((wave + 8 * k) * 8 + (lane >> 3), N - 1 - row0) * (uint32_t)K + piece;
    }
    // scales of a block: wavefront k < 4 those of rows 64 k .. of x, wavefronts 6 and 7 a scale of w each (up: of w1 and w3; else of the tile's
    // two blocks of 128 rows), 64 times over
    const int nb = UP ? n0 / kFp8Block : min(n0 / kFp8Block + (wave & 1), (N - 1) / kFp8Block);
    gptr_t sb = scalar_ptr(wave < 6 ? a.xs : (UP && wave == 7 ? a.w3[e].scale : a.w[e].scale) + (size_t)nb * blocks);
    const uint32_t sv = wave < 6 ? (uint32_t)row_of(a, c.begin + min((wave & 3) * 64 + lane, rows - 1)) * 4 : 0u;
    const size_t scales_of_block = wave < 6 ? (size_t)a.x_rows * 4 : 4;
    uint32_t put = lds0;                                     // the stage that is filled next
    auto bring_stage = [&](bool last) {                      // (of the blocks in order)
        uint32_t back = 0;
        if (last && tail < kFp8Block) back = piece > tail - 16 ? piece - (tail - 16) : 0;   // pieces past the end of a row: its last one
#pragma unroll
        for (int k = 0; k < L::kMost; ++k)
            if (k < L::kMost - 1 || more) bring<0>(put + (wave + 8 * k) * 1024, xb, xv[k] - back);
#pragma unroll
        for (int k = 0; k < 4; ++k) bring<0>(put + L::kX + (wave + 8 * k) * 1024, wb[k >> 1], wv[k] - back);
        bring_words(put + L::kX + L::kW + wave * 256, sb, sv);
        xb += kFp8Block;
        wb[0] += kFp8Block;
        wb[1] += kFp8Block;
        sb += scales_of_block;
        put = put == lds0 + (L::kStages - 1) * L::kStage ? lds0 : put + L::kStage;
    };
    // Up to `later` stages may be under way.
    auto wait = [&](int later) {
        if (later <= 0) wait_and_meet<0>();
        else if (later == 1 && more) wait_and_meet<L::kMost + 5>();
        else if (later == 1) wait_and_meet<L::kMost + 4>();
        else if (later == 2 && more) wait_and_meet<2 * (L::kMost + 5)>();
        else if (later == 2) wait_and_meet<2 * (L::kMost + 4)>();
        else if (more) wait_and_meet<3 * (L::kMost + 5)>();
        else wait_and_meet<3 * (L::kMost + 4)>();
    };
    // Stage b is there, and nobody reads stage b - 1 any more.  The pieces past the end of the rows are cleared by who brought them.
    auto meet = [&](int b, uint32_t at) {
        if (b == blocks - 1 && tail < kFp8Block) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            if (piece >= tail) {
#pragma unroll
                for (int k = 0; k < L::kMost; ++k)
                    if (k < L::kMost - 1 || more) *(uint4_t*)(lds + at + (wave + 8 * k) * 1024 + lane * 16) = uint4_t{0u, 0u, 0u, 0u};
#pragma unroll
                for (int k = 0; k < 4; ++k) *(uint4_t*)(lds + at + L::kX + (wave + 8 * k) * 1024 + lane * 16) = uint4_t{0u, 0u, 0u, 0u};
            }
        }
        wait(min(L::kStages - 2, blocks - 1 - b));
    };
    // ---- what it reads: lane l row r16 of 16, bytes 32 q .. 32 q + 31
    uint32_t off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) off[h] = r16 * 128 + (((2 * q + h) ^ swizzle128(r16)) * 16);
    // operand j of w: rows 64 wn + 16 j; up: 32 wn + 16 j of w1 (j < 2) and of w3
    auto read_w = [&](uint32_t at, int j, uint4_t (&v)[2]) {
        const uint32_t row0 = UP ? (j >> 1) * 128 + wn * 32 + (j & 1) * 16 : wn * 64 + j * 16;
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = *(const uint4_t*)(lds + at + L::kX + row0 * 128 + off[h]);
    };
    auto read_x = [&](uint32_t at, int i, uint4_t (&v)[2]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = *(const uint4_t*)(lds + at + (tile0 + i) * 2048 + off[h]);
    };
    float4_t acc[4][MT ? MT : 1];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};

    // ---- The operands that a block starts with are read while the last products of the block before it are under way, after the
    // wavefronts have met for it: then they find the matrix cores busy whenever they meet.
    uint4_t w[4][2], x[2], x_next[2];
    float w0, w1 = 0.0f;
    auto read_first = [&](uint32_t at) {                     // half 0 of w, tile 0 of x, the scales of w
        read_w(at, 0, w[0]);
        read_w(at, 1, w[1]);
        read_x(at, 0, x_next);
        const float* const sw = (const float*)(lds + at + L::kX + L::kW) + 6 * 64;
        w0 = sw[UP ? 0 : (wn >> 1) * 64];
        if (UP) w1 = sw[64];
    };
    for (int b = 0; b < L::kStages && b < blocks; ++b) bring_stage(b == blocks - 1);
    if (blocks == 1) meet(0, 0);
    else wait(min(L::kStages, blocks) - 1);
    uint32_t at = 0;
    if constexpr (MT > 0) read_first(0);
    else w0 = 0.0f;
    // F8: codes go to the matrix cores as they are; else expanded to fp16.
    half8_t wf[F8 ? 1 : 4][4], xf[4];
    auto expand = [](const uint4_t (&v)[2], half8_t (&o)[4]) {
#pragma unroll
        for (int p = 0; p < 4; ++p) o[p] = fp8_expand(v[p >> 1][2 * (p & 1)], v[p >> 1][2 * (p & 1) + 1]);
    };
    for (int b = 0; b < blocks; ++b) {
        const uint32_t next = at == (L::kStages - 1) * L::kStage ? 0u : at + L::kStage;
        const float* const sx = (const float*)(lds + at + L::kX + L::kW) + 16 * tile0 + r16;
        float4_t part[2][2];
        const float scale_w0 = w0, scale_w1 = w1;
        float s_now = 0.0f, s_before = 0.0f;
        auto add = [&](int i, int h, float s) {              // half h of tile i (up: 0 is w1's, 1 w3's)
            const float f = s * (UP && h ? scale_w1 : scale_w0);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[2 * h + j][i][k] = fmaf(part[h][j][k], f, acc[2 * h + j][i][k]);
                asm volatile("" : "+v"(acc[2 * h + j][i]));  // added here: sinking it to the end of the block would keep all products alive
            }
        };
        auto products = [&](int h) {
            if constexpr (F8) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    part[h][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(join(w[2 * h + j][0], w[2 * h + j][1]), join(x[0], x[1]),
                                                                                  float4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j) part[h][j] = mfma16(wf[2 * h + j][p], xf[p], p ? part[h][j] : float4_t{0.0f, 0.0f, 0.0f, 0.0f});
            }
        };
        if constexpr (MT > 0) {
            read_w(at, 2, w[2]);
            read_w(at, 3, w[3]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            x[0] = x_next[0];
            x[1] = x_next[1];
            if (i + 1 < MT) read_x(at, i + 1, x_next);
            s_now = sx[16 * i];
            if constexpr (!F8) expand(x, xf);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (!F8) {
                    if (i == 0) {
                        expand(w[2 * h], wf[2 * h]);
                        expand(w[2 * h + 1], wf[2 * h + 1]);
                    }
                }
                products(h);
                pin_schedule();
                if (i == MT - 1 && h == 0) {                 // (past the last block: whatever lies there, never used)
                    meet(b + 1, next);
                    if (b + L::kStages < blocks) bring_stage(b + L::kStages == blocks - 1);
                    read_first(next);                        // (w's half 0 has been handed to the matrix cores)
                    pin_schedule();
                }
                if (h) add(i, 0, s_now);
                else if (i) add(i - 1, 1, s_before);
                pin_schedule();
            }
            s_before = s_now;
        }
        if constexpr (MT > 0) {
            add(MT - 1, 1, s_before);
        } else {
            meet(b + 1, next);
            if (b + L::kStages < blocks) bring_stage(b + L::kStages == blocks - 1);
        }
        at = next;
    }
    // ---- lane: row r16 of a tile of x, results 4 q .. 4 q + 3 of a tile of w
    if constexpr (UP) {
        // The tile's 128 hidden values of a row are a block: rounded to fp16 as everywhere, then quantized here.  The largest magnitude of a row
        // goes over the four lanes that hold it and, through LDS, over the four wavefronts.
        uint32_t* const tops = (uint32_t*)lds;               // [4][16 TT]
        half4_t h[MT ? MT : 1][2];
        __syncthreads();                                     // (the stages have been read)
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            uint32_t top = 0;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const half_t v = n0 + wn * 32 + j * 16 + 4 * q + k < N ? (half_t)silu_mul(acc[j][i][k], acc[j + 2][i][k]) : (half_t)0.0f;
                    const uint32_t bits = __builtin_bit_cast(uint16_t, v) & 0x7FFFu;
                    h[i][j][k] = v;
                    top = top > bits ? top : bits;
                }
#pragma unroll
            for (int m = 16; m <= 32; m <<= 1) {
                const uint32_t o = __shfl_xor(top, m, kWave);
                top = top > o ? top : o;
            }
            if (q == 0) tops[wn * (16 * TT) + (tile0 + i) * 16 + r16] = top;
        }
        __syncthreads();
        uint8_t* const codes = (uint8_t*)a.y;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int r = (tile0 + i) * 16 + r16;
            uint32_t top = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t o = tops[k * (16 * TT) + r];
                top = top > o ? top : o;
            }
            const float m = magnitude_value(top), f = fp8_factor(m);
            if (r >= rows) continue;
            if (wn == 0 && q == 0) a.y_scale[(size_t)(n0 / kFp8Block) * a.P + c.begin + r] = fp8_scale(m);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int n = n0 + wn * 32 + j * 16 + 4 * q;     // (N is a multiple of 64)
                const half4_t v = h[i][j];
                if (n < N)
                    *(uint32_t*)(codes + (size_t)(c.begin + r) * N + n) = fp8_pack((float)v[0] * f, (float)v[1] * f, (float)v[2] * f, (float)v[3] * f);
            }
        }
        return;
    }
    OUT* const y = (OUT*)a.y;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int r = (tile0 + i) * 16 + r16;
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int n = n0 + wn * 64 + j * 16 + 4 * q;
            const float4_t v = acc[j][i];
            OUT* const o = y + (size_t)(c.begin + r) * N + n;
            if (n + 4 <= N) {
                if (sizeof(OUT) == 4) *(float4_anywhere_t*)o = v;
                else *(half4_anywhere_t*)o = half4_t{(half_t)v[0], (half_t)v[1], (half_t)v[2], (half_t)v[3]};
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (n + k < N) o[k] = (OUT)v[k];
            }
        }
    }
}

constexpr int most_tiles(bool f8) { return f8 ? 16 : 10; }   // (operands expanded to fp16 need more registers)

template <int TT, bool F8, bool UP, typename OUT>
__device__ __forceinline__ void tile_halves(const Fp8Args& a, const TileWork& c, uint8_t* lds) {
    if constexpr (TT <= most_tiles(F8)) {
        if (TT % 2 == 0) tile_body<TT, TT / 2, F8, UP, OUT>(a, c, lds, __builtin_amdgcn_readfirstlane(threadIdx.x >> 8) * (TT / 2));
        else if (threadIdx.x < 256) tile_body<TT, (TT + 1) / 2, F8, UP, OUT>(a, c, lds, 0);
        else tile_body<TT, TT / 2, F8, UP, OUT>(a, c, lds, (TT + 1) / 2);
    }
}

// Chunks of up to `per` rows of an expert; a chunk runs in the body for its number of tiles.
template <bool F8, bool UP, typename OUT>
__global__ __launch_bounds__(512, 2) void fp8_tile_kernel(Fp8Args a, int per, int n_tiles) {
    extern __shared__ uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63;
    // Workgroups go to the 8 XCDs in turn: each XCD takes a run of neighbouring tiles, eight chunks side by side.
    const Chunks chunks = count_chunks(a, per, lane);
    const int n_chunks = chunks.total(), total = n_chunks * n_tiles, per_xcd = (total + 7) >> 3;
    const int slot = blockIdx.x >> 3, t = (blockIdx.x & 7) * per_xcd + slot;
    if (slot >= per_xcd || t >= total) return;
    const int group = t / (8 * n_tiles), rest = t - group * 8 * n_tiles, in_group = min(8, n_chunks - group * 8);
    const int tile = rest / in_group;
    constexpr int kOut = UP ? kCols / 2 : kCols;             // results of a tile
    TileWork c;
    c.n0 = tile * kOut;
    if (!chunks.find(group * 8 + rest - tile * in_group, c.expert, c.begin, c.rows)) return;
    c.expert = __builtin_amdgcn_readfirstlane(c.expert);
    const int todo = a.todo[c.expert], N = a.N;
    if (todo == kFp8Skip) return;
    if (todo == kFp8Missing) {
        if (tid == 0 && tile == 0 && a.status) atomicOr(a.status, kStatusNotResident);
        if (!UP)
            for (int i = tid; i < c.rows * kOut; i += 512)
                if (c.n0 + i % kOut < N) ((OUT*)a.y)[(size_t)(c.begin + i / kOut) * N + c.n0 + i % kOut] = (OUT)0.0f;
        return;
    }
    switch ((c.rows + 15) >> 4) {
#define MOEMIX_TILE_CASE(n) case n: tile_halves<(n), F8, UP, OUT>(a, c, lds); break;
        MOEMIX_TILE_CASE(1)
        MOEMIX_TILE_CASE(2)
        MOEMIX_TILE_CASE(3)
        MOEMIX_TILE_CASE(4)
        MOEMIX_TILE_CASE(5)
        MOEMIX_TILE_CASE(6)
        MOEMIX_TILE_CASE(7)
        MOEMIX_TILE_CASE(8)
        MOEMIX_TILE_CASE(9)
        MOEMIX_TILE_CASE(10)
        MOEMIX_TILE_CASE(11)
        MOEMIX_TILE_CASE(12)
        MOEMIX_TILE_CASE(13)
        MOEMIX_TILE_CASE(14)
        MOEMIX_TILE_CASE(15)
        MOEMIX_TILE_CASE(16)
#undef MOEMIX_TILE_CASE
    }
}

template <bool F8, bool UP, typename OUT>
void launch(const Fp8Args& a, int per, hipStream_t st) {
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = fp8_tile_kernel<F8, UP, OUT>;
    allow_lds((const void*)kernel, kLds, configured);
    constexpr int kOut = UP ? kCols / 2 : kCols;
    const int n_tiles = (a.N + kOut - 1) / kOut;
    const long long total = (long long)n_tiles * most_chunks(a, per);
    kernel<<<(unsigned)((total + 7) / 8 * 8), 512, kLds, st>>>(a, per, n_tiles);
}

}  // namespace

// Rows per chunk: the number (of 16s) whose rounds of workgroups over the chip cost least, a block of 128 columns costing
// 4 + TT in a workgroup of TT tiles (measured, 4096 rows 4096 -> 14336: 0.88 us a block for TT = 4, 1.40 for 8, 1.81 for 12, 2.18 for 16).
// Of several experts some have more rows than the mean: an eighth or two standard deviations more is reckoned with (16 experts of 1024 x 4096, 128 rows
// on average: chunks of 144 rows, which some experts exceed, 37.5 us, of 160 24.7).
static int rows_per_chunk(const Fp8Args& a, bool up, bool exact, long long* best_cost) {
    const int out = up ? kCols / 2 : kCols, tiles = (a.N + out - 1) / out;
    const int with_rows = a.E < a.P ? a.E : a.P, even = (a.P + with_rows - 1) / with_rows;
    const float eighth = (float)even / 8.0f, deviations = 2.0f * sqrtf((float)even);
    const int mean = even + (with_rows > 1 ? (int)(eighth > deviations ? eighth : deviations) : 0);
    int per = 16, best_chunks = 0;
    for (int tt = 1; tt <= most_tiles(!exact); ++tt) {
        const int chunks = (mean + 16 * tt - 1) / (16 * tt), rows = (mean + chunks - 1) / chunks;
        const long long rounds = ((long long)tiles * chunks * with_rows + kComputeUnits - 1) / kComputeUnits, cost = rounds * (4 + (rows + 15) / 16);
        if (tt == 1 || cost < *best_cost || (cost == *best_cost && chunks < best_chunks)) {     // (of equal ones fewer chunks, then shorter ones)
            *best_cost = cost;
            best_chunks = chunks;
            per = 16 * tt;
        }
    }
    return per;
}

// Gathered rows are found by 32-bit offsets.
bool fp8_tile_can(const Fp8Args& a) { return a.K > 0 && (!a.perm || (size_t)a.x_rows * a.K < (1ull << 32) - 4096); }

// Microseconds, roughly: the rounds at 0.087 us per block of 128 columns and unit of cost (0.123 with rows expanded to fp16), or 6 TB/s of weights.
float fp8_tile_us(const Fp8Args& a, bool up, bool exact) {
    long long cost = 0;
    rows_per_chunk(a, up, exact, &cost);
    const float with_rows = (float)(a.E < a.P ? a.E : a.P), mb = 1e-6f * (float)a.N * (float)a.K * (up ? 2.0f : 1.0f) * with_rows;
    const float blocks = (float)((a.K + kFp8Block - 1) / kFp8Block), busy = (float)cost * blocks * (exact ? 0.123f : 0.087f);
    return 4.5f + (busy > mb / 6.0f ? busy : mb / 6.0f);
}

int fp8_tile_rows(const Fp8Args& a, bool up, bool exact) {
    long long cost = 0;
    return rows_per_chunk(a, up, exact, &cost);
}

void launch_fp8_tile(const Fp8Args& a, bool up, bool half_out, bool exact, hipStream_t st) {
    const int per = fp8_tile_rows(a, up, exact);
    if (up) launch<false, true, uint8_t>(a, per, st);
    else if (half_out) launch<true, false, half_t>(a, per, st);
    else if (exact) launch<false, false, float>(a, per, st);
    else launch<true, false, float>(a, per, st);
}

}  // namespace moemix
