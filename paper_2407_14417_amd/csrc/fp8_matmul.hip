// Products of rows and matrices held in 8-bit floating point with a scale for each block of 128:
//   y[m, n] = sum_b xs[b, m] ws[n/128, b] sum_{k in block b} x[m, k] w[n, k]
// over one matrix or over the experts of a grouping (rows offsets[e] .. offsets[e+1] belong to expert e).
#include "fp8.hpp"
#include "kernels.hpp"

namespace moemix {

namespace {

__device__ const uint32_t zeros[4] __attribute__((aligned(16))) = {0u, 0u, 0u, 0u};

// Few rows: one workgroup = 16 weight rows (up: of w1 and of w3) and up to 16 CT rows; its wavefronts take the blocks of 128
// columns in turn and their sums are added at the end, in order.  Codes go from memory to registers, DEPTH blocks ahead, are
// expanded to fp16 (exact) and multiplied by v_mfma_f32_16x16x32_f16, so a block's sum is as exact as 32 bits allow.
constexpr int kFewWaves = 8;

template <int CT, bool UP, typename OUT>
__global__ __launch_bounds__(64 * kFewWaves) void fp8_few_kernel(Fp8Args a) {
    constexpr int T = UP ? 2 : 1, DEPTH = CT == 1 ? 4 : 2;
    __shared__ float sums[kFewWaves][T * CT][256];
    const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int e, begin, rows;
    if (!count_chunks(a, 16 * CT, lane).find(blockIdx.y, e, begin, rows)) return;
    e = __builtin_amdgcn_readfirstlane(e);
    const int todo = a.todo[e], n0 = blockIdx.x * 16;
    if (todo == kFp8Skip) return;
    OUT* const y = (OUT*)a.y;
    if (todo == kFp8Missing) {
        if (tid == 0 && blockIdx.x == 0 && a.status) atomicOr(a.status, kStatusNotResident);
        if (!UP)
            for (int i = tid; i < rows * 16; i += 64 * kFewWaves)
                if (n0 + (i & 15) < a.N) y[(size_t)(begin + (i >> 4)) * a.N + n0 + (i & 15)] = (OUT)0.0f;
        return;
    }
    const int K = a.K, blocks = (K + kFp8Block - 1) / kFp8Block;
    const int wrow = min(n0 + r16, a.N - 1);
    const uint8_t* wp[T];
    const float* wsp[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const Fp8Mat& m = t ? a.w3[e] : a.w[e];
        wp[t] = m.data + (size_t)wrow * K;
        wsp[t] = m.scale + (size_t)(n0 / kFp8Block) * blocks;
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
    for (int i = tid; i < CT * 256; i += 64 * kFewWaves) {
        const int m = i >> 4, n = i & 15, c = m >> 4, at = ((n >> 2) * 16 + (m & 15)) * 4 + (n & 3);
        if (m >= rows || n0 + n >= a.N) continue;
        float v[T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            v[t] = sums[0][t * CT + c][at];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) v[t] += sums[w][t * CT + c][at];
        }
        y[(size_t)(begin + m) * a.N + n0 + n] = (OUT)(UP ? silu_mul(v[0], v[T - 1]) : v[0]);
    }
}

template <int CT>
void launch_few(const Fp8Args& a, bool up, bool half_out, dim3 grid, hipStream_t st) {
    if (up) fp8_few_kernel<CT, true, half_t><<<grid, 64 * kFewWaves, 0, st>>>(a);
    else if (half_out) fp8_few_kernel<CT, false, half_t><<<grid, 64 * kFewWaves, 0, st>>>(a);
    else fp8_few_kernel<CT, false, float><<<grid, 64 * kFewWaves, 0, st>>>(a);
}

}  // namespace

void launch_fp8_matmul(const Fp8Args& a, bool up, bool half_out, bool exact, hipStream_t st) {
    if (a.P == 0 || a.N == 0) return;
    if (fp8_tile_serves(a)) {
        launch_fp8_tile(a, up, half_out, exact, st);
        return;
    }
    const int mean = (a.P + a.E - 1) / a.E;
    const int ct = mean <= 16 ? 1 : mean <= 32 ? 2 : 4;
    dim3 grid((a.N + 15) / 16, most_chunks(a, 16 * ct));
    if (ct == 1) launch_few<1>(a, up, half_out, grid, st);
    else if (ct == 2) launch_few<2>(a, up, half_out, grid, st);
    else launch_few<4>(a, up, half_out, grid, st);
}

}  // namespace moemix
