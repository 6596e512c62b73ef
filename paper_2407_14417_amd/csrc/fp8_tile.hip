// Products of e4m3 rows and matrices where a matrix has many rows: tiles that stay in LDS and registers.
#include <atomic>
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

// 8 wavefronts = 2 (rows of x) x 4 (rows of w); each multiplies 16 MT rows of x with 64 rows of w.
template <int MT>
struct Tile {
    static constexpr int kRows = 32 * MT, kCols = 256;
    static constexpr int kX = kRows * 128, kW = kCols * 128, kScales = 8 * 64 * 4;
    static constexpr int kStage = kX + kW + kScales, kStages = MT == 8 ? 2 : 3;
    static constexpr int kXRuns = kRows / 64;               // 1 KB runs (8 rows) of x per wavefront and stage
    static constexpr int kTransfers = kXRuns + 4 + 1;       // ... with those of w and the scales
    static constexpr int kLds = kStage * kStages;
    static_assert(kLds <= 163840, "LDS");
};

template <int MT, bool F8, bool UP, typename OUT>
__global__ __launch_bounds__(512, 2) void fp8_tile_kernel(Fp8Args a, int n_tiles) {
    typedef Tile<MT> L;
    extern __shared__ uint8_t lds[];
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
    // ---- which tile
    const Chunks chunks = count_chunks(a, L::kRows, lane);
    const int n_chunks = chunks.total(), total = n_chunks * n_tiles, per_xcd = (total + 7) >> 3;
    const int slot = blockIdx.x >> 3, t = (blockIdx.x & 7) * per_xcd + slot;
    if (slot >= per_xcd || t >= total) return;
    const int group = t / (8 * n_tiles), rest = t - group * 8 * n_tiles, in_group = min(8, n_chunks - group * 8);
    const int tile = rest / in_group;
    int e, begin, rows;
    if (!chunks.find(group * 8 + rest - tile * in_group, e, begin, rows)) return;
    e = __builtin_amdgcn_readfirstlane(e);
    constexpr int kOut = UP ? 128 : 256;                     // results of a tile
    const int todo = a.todo[e], n0 = tile * kOut, N = a.N, K = a.K;
    if (todo == kFp8Skip) return;
    OUT* const y = (OUT*)a.y;
    if (todo == kFp8Missing) {
        if (tid == 0 && tile == 0 && a.status) atomicOr(a.status, kStatusNotResident);
        if (!UP)
            for (int i = tid; i < rows * kOut; i += 512)
                if (n0 + i % kOut < N) y[(size_t)(begin + i / kOut) * N + n0 + i % kOut] = (OUT)0.0f;
        return;
    }
    const int blocks = (K + kFp8Block - 1) / kFp8Block, tail = K - (blocks - 1) * kFp8Block;   // bytes of the last block
    // ---- what it brings: lane l the 16-byte slot l & 7 of row l >> 3 of a run of 8 rows
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds;
    uint32_t xv[L::kXRuns], wv[4], sv;
    const int piece_of[2] = {((lane & 7) ^ swizzle128(lane >> 3)) * 16, ((lane & 7) ^ swizzle128(8 + (lane >> 3))) * 16};
    gptr_t xb = scalar_ptr(a.perm ? a.x : a.x + (size_t)begin * K);
#pragma unroll
    for (int k = 0; k < L::kXRuns; ++k) {
        const int run = wave * L::kXRuns + k, row = min(run * 8 + (lane >> 3), rows - 1);
        xv[k] = (uint32_t)(a.perm ? row_of(a, begin + row) : row) * (uint32_t)K + piece_of[run & 1];
    }
    {
        const int row = min((wave % L::kXRuns) * 64 + lane, rows - 1);
        sv = (uint32_t)row_of(a, begin + row) * 4;
    }
    gptr_t sb = scalar_ptr(a.xs);
    const Fp8Mat m = UP && wave >= 4 ? a.w3[e] : a.w[e];
    const int row0 = min(UP ? n0 + (wave & 3) * 32 : n0 + wave * 32, N - 1);      // (rows past the last one: the last one again)
    gptr_t wb = scalar_ptr(m.data + (size_t)row0 * K);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = min(row0 + k * 8 + (lane >> 3), N - 1) - row0;
        wv[k] = (uint32_t)row * (uint32_t)K + piece_of[k & 1];
    }
    auto bring_stage = [&](int b) {
        const uint32_t at = lds0 + (b % L::kStages) * L::kStage;
        const gptr_t x = xb + (size_t)b * kFp8Block, w = wb + (size_t)b * kFp8Block;
        if (b == blocks - 1 && tail < kFp8Block) {            // pieces past the end of a row: its last one, cleared when it is read
            const int most = tail - 16;
#pragma unroll
            for (int k = 0; k < L::kXRuns; ++k) {
                const int p = piece_of[(wave * L::kXRuns + k) & 1];
                bring<0>(at + (wave * L::kXRuns + k) * 1024, x, xv[k] - (p > most ? p - most : 0));
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int p = piece_of[k & 1];
                bring<0>(at + L::kX + (wave * 4 + k) * 1024, w, wv[k] - (p > most ? p - most : 0));
            }
        } else {
#pragma unroll
            for (int k = 0; k < L::kXRuns; ++k) bring<0>(at + (wave * L::kXRuns + k) * 1024, x, xv[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k) bring<0>(at + L::kX + (wave * 4 + k) * 1024, w, wv[k]);
        }
        bring_words(at + L::kX + L::kW + wave * 256, sb + (size_t)b * a.x_rows * 4, sv);
    };
    // ---- scales of w: one (up: one of each matrix) per block and wavefront
    const int last = (N - 1) / kFp8Block;
    const float* ws[2] = {a.w[e].scale, a.w3[e].scale};
    ws[0] += (size_t)min(UP ? n0 / kFp8Block : n0 / kFp8Block + (wn >> 1), last) * blocks;
    if (UP) ws[1] += (size_t)(n0 / kFp8Block) * blocks;
    // ---- what it reads
    uint32_t off[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) off[h] = r16 * 128 + (((2 * q + h) ^ swizzle128(r16)) * 16);
    auto w_tile = [&](int j) { return UP ? (j >> 1) * 8 + wn * 2 + (j & 1) : wn * 4 + j; };
    float4_t acc[4][MT];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};

    for (int b = 0; b < L::kStages - 1; ++b)
        if (b < blocks) bring_stage(b);
    auto step = [&](int b, auto cut_c) {
        constexpr bool kCut = decltype(cut_c)::value;         // the block ends within 128 columns
        if (L::kStages == 3 && b + 1 < blocks) wait_and_meet<L::kTransfers>();
        else wait_and_meet<0>();
        if (b + L::kStages - 1 < blocks) bring_stage(b + L::kStages - 1);
        const uint8_t* const xs = lds + (b % L::kStages) * L::kStage;
        const uint8_t* const wl = xs + L::kX;
        const float* const sl = (const float*)(wl + L::kW) + wm * 16 * MT + r16;
        const float w0 = ws[0][b], w1 = UP ? ws[1][b] : 0.0f;
        auto read = [&](const uint8_t* base, int rows16, uint4_t (&v)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) v[h] = *(const uint4_t*)(base + rows16 * 2048 + off[h]);
            if (kCut) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    if ((2 * q + h) * 16 >= tail) v[h] = uint4_t{0u, 0u, 0u, 0u};
            }
        };
        if (F8) {
            int8v_t wf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint4_t v[2];
                read(wl, w_tile(j), v);
                wf[j] = join(v[0], v[1]);
            }
            // A pair of products is under way while the one before it is scaled and added.
            float4_t part[2][2];
            int8v_t xf[2];
            uint4_t v[2];
            read(xs, wm * MT, v);
            xf[0] = join(v[0], v[1]);
            float s_before = 0.0f;
            auto add = [&](int i, int h, float s) {           // pair h of tile i
#pragma unroll
                for (int c2 = 0; c2 < 2; ++c2) {
                    const float f = s * (UP && h ? w1 : w0);
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[2 * h + c2][i][c] = fmaf(part[h][c2][c], f, acc[2 * h + c2][i][c]);
                }
            };
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i + 1 < MT) {
                    read(xs, wm * MT + i + 1, v);
                    xf[(i + 1) & 1] = join(v[0], v[1]);
                }
                const float s = sl[16 * i];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int c2 = 0; c2 < 2; ++c2)
                        part[h][c2] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wf[2 * h + c2], xf[i & 1], float4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
                    if (h) add(i, 0, s);
                    else if (i) add(i - 1, 1, s_before);
                }
                s_before = s;
                pin_schedule();
            }
            add(MT - 1, 1, s_before);
        } else {
            half8_t wf[4][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint4_t v[2];
                read(wl, w_tile(j), v);
#pragma unroll
                for (int p = 0; p < 4; ++p) wf[j][p] = fp8_expand(v[p >> 1][2 * (p & 1)], v[p >> 1][2 * (p & 1) + 1]);
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                uint4_t v[2];
                read(xs, wm * MT + i, v);
                half8_t xf[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) xf[p] = fp8_expand(v[p >> 1][2 * (p & 1)], v[p >> 1][2 * (p & 1) + 1]);
                float4_t part[4];
#pragma unroll
                for (int p = 0; p < 4; ++p)
#pragma unroll
                    for (int j = 0; j < 4; ++j) part[j] = mfma16(wf[j][p], xf[p], p ? part[j] : float4_t{0.0f, 0.0f, 0.0f, 0.0f});
                const float s = sl[16 * i], s0 = s * w0, s1 = s * w1;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[j][i][c] = fmaf(part[j][c], UP && j >= 2 ? s1 : s0, acc[j][i][c]);
            }
        }
    };
    for (int b = 0; b < blocks - 1; ++b) step(b, std::false_type{});
    if (tail < kFp8Block) step(blocks - 1, std::true_type{});
    else step(blocks - 1, std::false_type{});
    // ---- lane: row r16 of a tile of x, results 4 q .. 4 q + 3 of a tile of w
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int r = (wm * MT + i) * 16 + r16;
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < (UP ? 2 : 4); ++j) {
            const int n = n0 + w_tile(j) * 16 + 4 * q;
            float4_t v = acc[j][i];
            if (UP) {
#pragma unroll
                for (int c = 0; c < 4; ++c) v[c] = silu_mul(v[c], acc[(j + 2) & 3][i][c]);
            }
            OUT* const o = y + (size_t)(begin + r) * N + n;
            if (n + 4 <= N) {
                if (sizeof(OUT) == 4) *(float4_anywhere_t*)o = v;
                else *(half4_anywhere_t*)o = half4_t{(half_t)v[0], (half_t)v[1], (half_t)v[2], (half_t)v[3]};
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (n + c < N) o[c] = (OUT)v[c];
            }
        }
    }
}

template <int MT, bool F8, bool UP, typename OUT>
void launch(const Fp8Args& a, hipStream_t st) {
    typedef Tile<MT> L;
    static std::atomic<unsigned long long> configured{0};
    const auto kernel = fp8_tile_kernel<MT, F8, UP, OUT>;
    allow_lds((const void*)kernel, L::kLds, configured);
    const int n_tiles = (a.N + (UP ? 127 : 255)) / (UP ? 128 : 256);
    const long long total = (long long)n_tiles * most_chunks(a, L::kRows);
    kernel<<<(unsigned)((total + 7) / 8 * 8), 512, L::kLds, st>>>(a, n_tiles);
}

template <int MT>
void launch_any(const Fp8Args& a, bool up, bool half_out, hipStream_t st) {
    if (up) launch<MT, true, true, half_t>(a, st);
    else if (half_out) launch<MT, true, false, half_t>(a, st);
    else launch<MT, true, false, float>(a, st);
}

}  // namespace

bool fp8_tile_serves(const Fp8Args& a) {
    const int mean = (a.P + a.E - 1) / a.E;
    // gathered rows are found by 32-bit offsets
    return mean > 64 && a.K > 0 && (!a.perm || (size_t)a.x_rows * a.K < (1ull << 32) - 4096) && a.K <= 1 << 20;
}

void launch_fp8_tile(const Fp8Args& a, bool up, bool half_out, bool exact, hipStream_t st) {
    const int mean = (a.P + a.E - 1) / a.E;
    if (exact) launch<4, false, false, float>(a, st);
    else if (mean > 192) launch_any<8>(a, up, half_out, st);
    else launch_any<4>(a, up, half_out, st);
}

}  // namespace moemix
