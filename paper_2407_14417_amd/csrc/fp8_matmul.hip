// Products of rows and matrices held in 8-bit floating point with a scale for each block of 128:
//   y[m, n] = sum_b xs[b, m] ws[n/128, b] sum_{k in block b} x[m, k] w[n, k]
// over one matrix or over the experts of a grouping (rows offsets[e] .. offsets[e+1] belong to expert e).  Here: few rows, and the choice between the kernels.
//
// Few rows are bound by the bytes of the matrix: 16 to 24 wavefronts a compute unit have one or two blocks of 16 rows x 128 codes each on their way.  One
// row, 4096 -> 14336: 14.9 us, 3.9 TB/s (59 MB; a copy of 1 GiB reads and writes 5.2 TB/s), of which 4 us are the kernel's beginning and end;
// 8 matrices of 14336 -> 4096 with a row each: 83 us, 5.0 TB/s.
#include <cmath>

#include "fp8.hpp"
#include "kernels.hpp"

namespace moemix {

namespace {

typedef uint4_t __attribute__((aligned(2))) uint4_half_aligned_t;    // (tokens may lie anywhere)

__device__ const uint32_t zeros[4] __attribute__((aligned(16))) = {0u, 0u, 0u, 0u};

// Few rows: one workgroup = 16 weight rows (up: of w1 and of w3) and up to 16 CT rows; its wavefronts take the blocks of 128
// columns in turn and their sums are added at the end, in order.  Codes go from memory to registers, DEPTH blocks ahead, are
// expanded to fp16 (exact) and multiplied by v_mfma_f32_16x16x32_f16, so a block's sum is as exact as 32 bits allow.
// Wavefronts side by side hide the way to memory better than blocks under way in one, whose registers they would take: one row 4096 -> 14336 with four
// ahead 16.0 us, with two 14.9 (one 15.1; 14336 -> 4096 13.2, 12.3, 15.3); 40 rows 4096 -> 4096 with two 12.0, with one 11.1.
constexpr int kFewWaves = 8;

template <int CT, int NT, bool UP, typename OUT>
__global__ __launch_bounds__(64 * kFewWaves) void fp8_few_kernel(Fp8Args a) {
    constexpr int T = UP ? 2 : NT, DEPTH = CT * T == 1 ? 2 : 1, kCols = UP ? 16 : 16 * NT;
    __shared__ float sums[kFewWaves][T * CT][256];
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int e, begin, rows;
    if (!count_chunks(a, 16 * CT, lane).find(blockIdx.y, e, begin, rows)) return;
    e = __builtin_amdgcn_readfirstlane(e);
    const int todo = a.todo[e], n0 = blockIdx.x * kCols;
    if (todo == kFp8Skip) return;
    OUT* const y = (OUT*)a.y;
    if (todo == kFp8Missing) {
        if (tid == 0 && blockIdx.x == 0 && a.status) atomicOr(a.status, kStatusNotResident);
        if (!UP)
            for (int i = tid; i < rows * kCols; i += 64 * kFewWaves)
                if (n0 + i % kCols < a.N) y[(size_t)(begin + i / kCols) * a.N + n0 + i % kCols] = (OUT)0.0f;
        return;
    }
    const int K = a.K, blocks = (K + kFp8Block - 1) / kFp8Block;
    const uint8_t* wp[T];
    const float* wsp[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const Fp8Mat& m = UP && t ? a.w3[e] : a.w[e];
        const int first = UP ? n0 : n0 + 16 * t;
        wp[t] = m.data + (size_t)min(first + r16, a.N - 1) * K;
        wsp[t] = m.scale + (size_t)(min(first, a.N - 1) / kFp8Block) * blocks;
    }
    const uint8_t* xp[CT];
    const float* xsp[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int token = row_of(a, begin + min(16 * c + r16, rows - 1));
        xp[c] = a.x + (size_t)token * K;
        xsp[c] = a.xs + token;
    }
    struct Step {
        uint4_t w[T][2], x[CT][2];
        float ws[T], xs[CT];
    } ring[DEPTH];
    // columns past the end of the rows count as zeros
    auto load = [&](Step& s, int b) {
        const int col = b * kFp8Block + q * 32;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const bool in = col + 16 * h < K;
#pragma unroll
            for (int t = 0; t < T; ++t) s.w[t][h] = *(const uint4_t*)(in ? wp[t] + col + 16 * h : (const uint8_t*)zeros);
#pragma unroll
            for (int c = 0; c < CT; ++c) s.x[c][h] = *(const uint4_t*)(in ? xp[c] + col + 16 * h : (const uint8_t*)zeros);
        }
#pragma unroll
        for (int t = 0; t < T; ++t) s.ws[t] = wsp[t][b];
#pragma unroll
        for (int c = 0; c < CT; ++c) s.xs[c] = xsp[c][(size_t)b * a.x_rows];
    };
    float4_t acc[T][CT];
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) acc[t][c] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](const Step& s) {
        half8_t wf[T][4];
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int p = 0; p < 4; ++p) wf[t][p] = fp8_expand(s.w[t][p >> 1][2 * (p & 1)], s.w[t][p >> 1][2 * (p & 1) + 1]);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            half8_t xf[4];
#pragma unroll
            for (int p = 0; p < 4; ++p) xf[p] = fp8_expand(s.x[c][p >> 1][2 * (p & 1)], s.x[c][p >> 1][2 * (p & 1) + 1]);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                float4_t part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int p = 0; p < 4; ++p) part = __builtin_amdgcn_mfma_f32_16x16x32_f16(wf[t][p], xf[p], part, 0, 0, 0);
                const float f = s.ws[t] * s.xs[c];
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][c][i] = fmaf(part[i], f, acc[t][c][i]);
            }
        }
    };
    const int steps = (blocks - wave + kFewWaves - 1) / kFewWaves;
    auto block_of = [&](int s) { return wave + s * kFewWaves; };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < steps) load(ring[d], block_of(d));
    int s = 0;
    for (; s + 2 * DEPTH <= steps; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            multiply(ring[d]);
            load(ring[d], block_of(s + d + DEPTH));
        }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        if (s + d < steps) multiply(ring[d]);
        if (s + d + DEPTH < steps) load(ring[d], block_of(s + d + DEPTH));
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (s + DEPTH + d < steps) multiply(ring[d]);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < CT; ++c) *(float4_t*)&sums[wave][t * CT + c][lane * 4] = acc[t][c];
    __syncthreads();
    for (int i = tid; i < CT * 16 * kCols; i += 64 * kFewWaves) {
        const int m = i / kCols, col = i % kCols, n = col & 15, c = m >> 4, at = ((n >> 2) * 16 + (m & 15)) * 4 + (n & 3);
        if (m >= rows || n0 + col >= a.N) continue;
        float v[2];
#pragma unroll
        for (int t = 0; t < (UP ? 2 : 1); ++t) {
            const int of = (UP ? t : col >> 4) * CT + c;
            v[t] = sums[0][of][at];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) v[t] += sums[w][of][at];
        }
        y[(size_t)(begin + m) * a.N + n0 + col] = (OUT)(UP ? silu_mul(v[0], v[UP ? 1 : 0]) : v[0]);
    }
}

// One token: workgroup (tile of 16 rows of w1 and of w3, slot) of the up-projection, or tile of 16 rows of the down-projection with all slots, whose
// outputs it adds weighted.  Rows come as fp16 and every wavefront quantizes what it multiplies (the same operations as quantize_fp8_rows_kernel), so a block of one
// token is three launches: gating, up, down.  Mixtral shape, top-2: 75 us, 4.7 TB/s of weights over the three (up 41 us, 5.7 TB/s; down 27, 4.3), and 101 with grouping,
// quantizers and average as launches of their own.
// Down: at 4096 columns a workgroup per compute unit, which needs 16 wavefronts to have enough on its way (Mixtral shape, block 79.5 us with 8, 76.5 with 16);
// of 16 one block each is enough (three ahead 76.9, two 74.9, one 74.6; up, 8 wavefronts: one 78.5, two 79.4, three and four 76.4 and 77.0).
constexpr int one_waves(bool up) { return up ? 8 : 16; }
constexpr size_t one_sums(bool up) { return one_waves(up) * (up ? 2 : 1) * 16 * sizeof(float); }

template <bool UP>
__global__ __launch_bounds__(64 * one_waves(UP)) void fp8_one_kernel(Fp8OneArgs a) {
    constexpr int kWaves = one_waves(UP), T = UP ? 2 : 1, DEPTH = UP ? 4 : 1;
    extern __shared__ uint8_t lds[];                          // sums [wavefronts][T][16]; per wavefront its quantized pieces [most][128], then scales [most]
    float* const sums = (float*)lds;
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4, n0 = blockIdx.x * 16, K = a.K;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int blocks = (K + kFp8Block - 1) / kFp8Block, total = UP ? blocks : a.k * blocks;
    const int steps = (total - wave + kWaves - 1) / kWaves, most = (total + kWaves - 1) / kWaves;
    uint8_t* const codes = lds + one_sums(UP) + wave * most * kFp8Block;
    float* const scales = (float*)(lds + one_sums(UP) + kWaves * most * kFp8Block) + wave * most;
    static_assert(kWaves * T * 16 * sizeof(float) == one_sums(UP), "LDS");
    // step s of the wavefront: block and slot
    auto place = [&](int s, int& slot, int& b) {
        const int g = wave + s * kWaves;
        slot = UP ? (int)blockIdx.y : g / blocks;
        b = UP ? g : g - slot * blocks;
    };
    auto expert_of = [&](int slot) { return a.idx[slot] & (MOE_MAX_EXPERTS - 1); };
    if (UP && a.todo[expert_of(blockIdx.y)] != kFp8Run) return;          // (the down-projection reports it)
    struct Step {
        uint4_t w[T][2];
        float f[T];
    } ring[DEPTH];
    auto load = [&](Step& r, int s) {
        int slot, b;
        place(s, slot, b);
        const int e = expert_of(slot);
        const bool run = UP || a.todo[e] == kFp8Run;
        const int col = b * kFp8Block + q * 32;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const Fp8Mat& m = UP && t ? a.w3[e] : a.w[e];
            const uint8_t* const row = m.data + (size_t)min(n0 + r16, a.N - 1) * K + col;
#pragma unroll
            for (int h = 0; h < 2; ++h) r.w[t][h] = *(const uint4_t*)(run && col + 16 * h < K ? row + 16 * h : (const uint8_t*)zeros);
            const float* const f = m.scale + (size_t)(n0 / kFp8Block) * blocks + b;
            r.f[t] = *(run ? f : (const float*)zeros);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (d < steps) load(ring[d], d);
    // ---- its pieces of the rows: 16 lanes a block, four blocks at a time
    for (int s0 = 0; s0 < steps; s0 += 4) {
        const int s = s0 + q;
        if (s >= steps) continue;
        int slot, b;
        place(s, slot, b);
        const int col = b * kFp8Block + r16 * 8;
        half8_t v = {};
        float weight = 1.0f;
        if (UP) {
            if (col < K) v = __builtin_bit_cast(half8_t, (uint4_t) * (const uint4_half_aligned_t*)(a.x + col));
        } else if (a.todo[expert_of(slot)] == kFp8Run) {
            weight = a.gate[slot];
            if (col < K) v = *(const half8_t*)(a.x + (size_t)slot * K + col);
        }
        uint32_t top = magnitude_max(0u, v);
        top = dpp_max<0xB1>(top);        // lanes 1 apart,
        top = dpp_max<0x4E>(top);        // 2 apart,
        top = dpp_max<0x141>(top);       // the other four of the eight,
        top = dpp_max<0x140>(top);       // and the other eight of the sixteen
        const float m = magnitude_value(top), f = fp8_factor(m);
        uint2_t c;
#pragma unroll
        for (int i = 0; i < 2; ++i) c[i] = fp8_pack((float)v[4 * i] * f, (float)v[4 * i + 1] * f, (float)v[4 * i + 2] * f, (float)v[4 * i + 3] * f);
        *(uint2_t*)(codes + s * kFp8Block + r16 * 8) = c;
        if (r16 == 0) scales[s] = fp8_scale(m) * weight;
    }
    wave_lds_handover();
    float4_t acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    // (every row of the second operand is the token: all columns of the product are alike)
    auto multiply = [&](const Step& r, int s) {
        half8_t xf[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4_t v = *(const uint4_t*)(codes + s * kFp8Block + q * 32 + h * 16);
            xf[2 * h] = fp8_expand(v[0], v[1]);
            xf[2 * h + 1] = fp8_expand(v[2], v[3]);
        }
        const float xs = scales[s];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            float4_t part = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < 4; ++p)
                part = __builtin_amdgcn_mfma_f32_16x16x32_f16(fp8_expand(r.w[t][p >> 1][2 * (p & 1)], r.w[t][p >> 1][2 * (p & 1) + 1]), xf[p], part, 0, 0, 0);
            const float f = r.f[t] * xs;
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = fmaf(part[i], f, acc[t][i]);
        }
    };
    int s = 0;
    for (; s + 2 * DEPTH <= steps; s += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            multiply(ring[d], s + d);
            load(ring[d], s + d + DEPTH);
        }
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
        if (s + d < steps) multiply(ring[d], s + d);
        if (s + d + DEPTH < steps) load(ring[d], s + d + DEPTH);
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (s + DEPTH + d < steps) multiply(ring[d], s + DEPTH + d);
    // lane 16 q holds results 4 q ..
    if (r16 == 0)
#pragma unroll
        for (int t = 0; t < T; ++t) *(float4_t*)(sums + (wave * T + t) * 16 + 4 * q) = acc[t];
    __syncthreads();
    const int n = n0 + tid;
    if (tid >= 16 || n >= a.N) return;
    float v[2];
#pragma unroll
    for (int t = 0; t < (UP ? 2 : 1); ++t) {
        const float* const from = sums + t * 16 + tid;
        v[t] = from[0];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v[t] += from[w * T * 16];
    }
    if (UP) a.y[(size_t)blockIdx.y * a.N + n] = (half_t)silu_mul(v[0], v[UP ? 1 : 0]);
    else a.y[n] = (half_t)(v[0] + (a.residual ? (float)a.residual[n] : 0.0f));
    if (!UP && blockIdx.x == 0 && tid < a.k && a.todo[expert_of(tid)] == kFp8Missing) atomicOr(a.status, kStatusNotResident);
}

template <int CT, int NT>
void launch_few(const Fp8Args& a, bool up, bool half_out, hipStream_t st) {
    const int cols = up ? 16 : 16 * NT;
    const dim3 grid((a.N + cols - 1) / cols, most_chunks(a, 16 * CT));
    if (up) fp8_few_kernel<CT, 1, true, half_t><<<grid, 64 * kFewWaves, 0, st>>>(a);
    else if (half_out) fp8_few_kernel<CT, NT, false, half_t><<<grid, 64 * kFewWaves, 0, st>>>(a);
    else fp8_few_kernel<CT, NT, false, float><<<grid, 64 * kFewWaves, 0, st>>>(a);
}

// Two tiles of 16 weight rows per wavefront halve what is read of x: with more than 16 rows, where that still leaves every compute unit a workgroup
// (4096 -> 14336, 32 rows, 448 workgroups: 24.1 -> 20.6 us; 14336 -> 4096, 128 workgroups: 32 rows 23.0 and 29.7, 64 rows 36.3 and 44.5).
int few_tiles(const Fp8Args& a, int ct, bool up) {
    return !up && ct > 1 && (long long)((a.N + 31) / 32) * most_chunks(a, 16 * ct) >= 256 ? 2 : 1;
}
int few_rows16(const Fp8Args& a) {
    const int mean = (a.P + a.E - 1) / a.E;
    return mean <= 16 ? 1 : mean <= 32 ? 2 : 4;
}

// Microseconds of the kernel above, roughly: 7.6 TB/s of weights and 7 TB/s of rows (every workgroup reads its chunk's) on top of 1.65 us (2.6 with more than
// one tile of rows) for every round of workgroups, two per compute unit with one tile of rows, else one.  Beside fp8_tile_us this says which kernel serves
// a product; both were fitted to 290 products of 1 to 256 rows and 1 to 32 matrices, where the choice costs 0.5 % over the better kernel (a fifth at worst).
// Few and tile, us: 4096 -> 14336, fp16 results, 8 rows 16.7 and 18.6, 48 rows 25.0 and 18.9; fp32 results, 32 rows 21.3 and 24.5; 14336 -> 4096, fp32, 64 rows
// 37.4 and 61; 8 experts 14336 -> 4096 with a row each 83 and 106; 32 experts 1408 -> 2048, 8 rows in all 6.3 and 9.1; a block of two tokens of the Mixtral
// shape, both projections, 149 and 193, of 16 tokens 286 and 302.
float few_us(const Fp8Args& a, bool up) {
    const int ct = few_rows16(a), cols = up ? 16 : 16 * few_tiles(a, ct, up), with_rows = a.E < a.P ? a.E : a.P;
    const int mean = (a.P + with_rows - 1) / with_rows, chunks = with_rows * ((mean + 16 * ct - 1) / (16 * ct));
    const float tiles = (float)((a.N + cols - 1) / cols), mb = 1e-6f * (float)a.N * (float)a.K * (up ? 2.0f : 1.0f);
    const float rounds = ceilf(tiles * (float)chunks / (ct == 1 ? 512.0f : 256.0f));
    return 1.0f + (ct == 1 ? 1.65f : 2.6f) * rounds + mb * (float)chunks / 7.6f + 1e-6f * tiles * (float)a.P * (float)a.K / 7.0f;
}

}  // namespace

size_t fp8_one_lds(int k, int K, bool up) {
    const int waves = one_waves(up), total = (up ? 1 : k) * ((K + kFp8Block - 1) / kFp8Block), most = (total + waves - 1) / waves;
    return one_sums(up) + (size_t)waves * most * (kFp8Block + sizeof(float));
}
// Up to 64 KB of LDS, so that two workgroups share a compute unit; past that the launches for several tokens serve one as well (us, these launches and those:
// 8 experts of 4096 x 14336, two slots 73 and 85, four 131 and 143; 4096 x 7168, eight 128 and 141; past the line, with as much LDS as there is, 4096 x 14336,
// eight 249 and 258, 1024 x 16384, eight 144 and 106, 16 experts of 2048 x 8192, eight 96 and 94).
bool fp8_one_serves(int k, int d, int f) { return fp8_one_lds(k, d, true) <= 65536 && fp8_one_lds(k, f, false) <= 65536; }

void launch_fp8_one(const Fp8OneArgs& a, bool up, hipStream_t st) {
    TraceScope trace(up ? kKernelUp : kKernelDown, st);
    const unsigned tiles = (unsigned)((a.N + 15) / 16);
    if (up) fp8_one_kernel<true><<<dim3(tiles, a.k), 64 * one_waves(true), fp8_one_lds(a.k, a.K, true), st>>>(a);
    else fp8_one_kernel<false><<<tiles, 64 * one_waves(false), fp8_one_lds(a.k, a.K, false), st>>>(a);
}

static void launch_few_any(const Fp8Args& a, bool up, bool half_out, hipStream_t st) {
    const int ct = few_rows16(a), nt = few_tiles(a, ct, up);
    if (ct == 1) launch_few<1, 1>(a, up, half_out, st);
    else if (ct == 2 && nt == 1) launch_few<2, 1>(a, up, half_out, st);
    else if (ct == 2) launch_few<2, 2>(a, up, half_out, st);
    else if (nt == 1) launch_few<4, 1>(a, up, half_out, st);
    else launch_few<4, 2>(a, up, half_out, st);
}

int fp8_rows_per_chunk(const Fp8Args& a, bool up, bool exact) {
    return fp8_tile_can(a) && fp8_tile_us(a, up, exact) < few_us(a, up) ? fp8_tile_rows(a, up, exact) : 0;
}

void launch_fp8_matmul(const Fp8Args& a, bool half_out, bool exact, hipStream_t st) {
    if (a.P == 0 || a.N == 0) return;
    if (fp8_rows_per_chunk(a, false, exact)) launch_fp8_tile(a, false, half_out, exact, st);
    else launch_few_any(a, false, half_out, st);
}

// The tile kernel holds a row's whole block of 128 hidden values and quantizes it; after the other kernel that is a launch of its own.
void launch_fp8_up(const Fp8Args& args, half_t* h, uint8_t* codes, float* scale, hipStream_t st) {
    Fp8Args a = args;
    if (fp8_rows_per_chunk(a, true, true)) {
        a.y = codes;
        a.y_scale = scale;
        TraceScope trace(kKernelUp, st);
        launch_fp8_tile(a, true, false, true, st);
        return;
    }
    a.y = h;
    {
        TraceScope trace(kKernelUp, st);
        launch_few_any(a, true, true, st);
    }
    launch_quantize_fp8_rows(h, a.P, a.N, codes, scale, st);
}

}  // namespace moemix
