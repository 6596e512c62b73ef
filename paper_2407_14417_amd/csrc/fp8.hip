// The 8-bit floating-point form on the device: rows quantized with a scale per 128 columns, matrices with a scale per block
// of 128 x 128, back to fp16, and the transposed codes that a gradient with respect to the rows multiplies with.
#include "fp8.hpp"
#include "kernels.hpp"

namespace moemix {

typedef uint4_t __attribute__((aligned(2))) uint4_half_aligned_t;    // (tokens may lie anywhere)

// A lane holds 16 consecutive columns of a row, eight lanes a block of 128: the largest magnitude of a block takes three
// steps on the DPP network.  Columns past `in` (a multiple of 16) count as zeros.
__global__ __launch_bounds__(256) void quantize_fp8_rows_kernel(const half_t* __restrict__ x, int n, int in, int blocks,
                                                                 uint8_t* __restrict__ codes, float* __restrict__ scale) {
    const size_t g = ((size_t)blockIdx.x * 256 + threadIdx.x) >> 3;     // row * blocks + block
    if (g >= (size_t)n * blocks) return;                                // (the eight lanes of a block agree)
    const size_t row = g / (unsigned)blocks;
    const int b = (int)(g - row * blocks), col = b * kFp8Block + (threadIdx.x & 7) * 16;
    const bool inside = col < in;
    half8_t v[2] = {};
    if (inside) {
        const uint4_half_aligned_t* p = (const uint4_half_aligned_t*)(x + row * in + col);
        v[0] = __builtin_bit_cast(half8_t, (uint4_t)p[0]);
        v[1] = __builtin_bit_cast(half8_t, (uint4_t)p[1]);
    }
    uint32_t most = magnitude_max(magnitude_max(0u, v[0]), v[1]);
    most = dpp_max<0xB1>(most);      // lanes 1 apart,
    most = dpp_max<0x4E>(most);      // 2 apart,
    most = dpp_max<0x141>(most);     // and the other four of the eight
    const float m = magnitude_value(most), f = fp8_factor(m);
    if (inside) {
        uint4_t o;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            o[i] = fp8_pack((float)v[i >> 1][4 * (i & 1)] * f, (float)v[i >> 1][4 * (i & 1) + 1] * f, (float)v[i >> 1][4 * (i & 1) + 2] * f,
                            (float)v[i >> 1][4 * (i & 1) + 3] * f);
        *(uint4_t*)(codes + row * in + col) = o;
    }
    if ((threadIdx.x & 7) == 0) scale[(size_t)b * n + row] = fp8_scale(m);
}

void launch_quantize_fp8_rows(const half_t* x, int n, int in, uint8_t* codes, float* scale, hipStream_t st) {
    const int blocks = (in + kFp8Block - 1) / kFp8Block;
    const size_t pieces = (size_t)n * blocks * 8;
    if (pieces) quantize_fp8_rows_kernel<<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(x, n, in, blocks, codes, scale);
}

// One workgroup per block of 128 x 128: every lane holds four pieces of 16 columns.
__global__ __launch_bounds__(256) void quantize_fp8_kernel(const half_t* __restrict__ w, int out, int in, uint8_t* __restrict__ codes,
                                                            float* __restrict__ scale) {
    __shared__ uint32_t wave_most[4];
    const int col = blockIdx.x * kFp8Block + (threadIdx.x & 7) * 16, row0 = blockIdx.y * kFp8Block + (threadIdx.x >> 3);
    half8_t v[4][2] = {};
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row0 + 32 * i < out && col < in) {
            const uint4_half_aligned_t* p = (const uint4_half_aligned_t*)(w + (size_t)(row0 + 32 * i) * in + col);
            v[i][0] = __builtin_bit_cast(half8_t, (uint4_t)p[0]);
            v[i][1] = __builtin_bit_cast(half8_t, (uint4_t)p[1]);
        }
        most = magnitude_max(magnitude_max(most, v[i][0]), v[i][1]);
    }
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) {
        const uint32_t o = __shfl_xor(most, m, kWave);
        most = most > o ? most : o;
    }
    if ((threadIdx.x & 63) == 0) wave_most[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) most = most > wave_most[i] ? most : wave_most[i];
    const float m = magnitude_value(most), f = fp8_factor(m);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (row0 + 32 * i >= out || col >= in) continue;
        uint4_t o;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const half8_t h = v[i][j >> 1];
            const int c = 4 * (j & 1);
            o[j] = fp8_pack((float)h[c] * f, (float)h[c + 1] * f, (float)h[c + 2] * f, (float)h[c + 3] * f);
        }
        *(uint4_t*)(codes + (size_t)(row0 + 32 * i) * in + col) = o;
    }
    if (threadIdx.x == 0) scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = fp8_scale(m);
}

void launch_quantize_fp8(const half_t* w, int out, int in, uint8_t* codes, float* scale, hipStream_t st) {
    if (out == 0 || in == 0) return;
    dim3 grid((in + kFp8Block - 1) / kFp8Block, (out + kFp8Block - 1) / kFp8Block);
    quantize_fp8_kernel<<<grid, 256, 0, st>>>(w, out, in, codes, scale);
}

// fp16_rne( fp32(code) * scale ), one thread per 8 codes.
__global__ __launch_bounds__(256) void dequant_fp8_kernel(Fp8Mat m, size_t n8, int in, half_t* __restrict__ w) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n8) return;
    const size_t row = i * 8 / (unsigned)in, col = i * 8 - row * in;
    const float s = m.scale[row / kFp8Block * ((in + kFp8Block - 1) / kFp8Block) + col / kFp8Block];
    const uint2_t c = ((const uint2_t*)m.data)[i];
    const half8_t v = fp8_expand(c[0], c[1]);
    half8_t o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = f32_to_f16_rne(__fmul_rn((float)v[j], s));
    *(half8_t*)(w + i * 8) = o;
}

void launch_dequant_fp8(const Fp8Mat& m, int out, int in, half_t* w, hipStream_t st) {
    const size_t n8 = (size_t)out * in / 8;
    if (n8) dequant_fp8_kernel<<<(unsigned)((n8 + 255) / 256), 256, 0, st>>>(m, n8, in, w);
}

// One workgroup per block: 16-byte pieces of rows into LDS, 16 bytes of columns out of it.  Rows of 132 bytes there: the
// bytes of a column lie in different banks.
__global__ __launch_bounds__(256) void transpose_fp8_kernel(Fp8Mat m, int out, int in, uint8_t* __restrict__ codes,
                                                             float* __restrict__ scale) {
    __shared__ uint32_t tile[kFp8Block][kFp8Block / 4 + 1];
    const int piece = threadIdx.x & 7, r0 = threadIdx.x >> 3;
    const int row0 = blockIdx.y * kFp8Block, col0 = blockIdx.x * kFp8Block;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = r0 + 32 * i;
        uint4_t v = {0u, 0u, 0u, 0u};
        if (row0 + r < out && col0 + piece * 16 < in) v = *(const uint4_t*)(m.data + (size_t)(row0 + r) * in + col0 + piece * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) tile[r][piece * 4 + j] = v[j];
    }
    __syncthreads();
    const uint8_t* const bytes = (const uint8_t*)tile;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = r0 + 32 * i;                           // column of the block, row of the result
        if (col0 + c >= in || row0 + piece * 16 >= out) continue;
        uint4_t v = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < 16; ++j) v[j >> 2] |= (uint32_t)bytes[(piece * 16 + j) * (kFp8Block + 4) + c] << (8 * (j & 3));
        *(uint4_t*)(codes + (size_t)(col0 + c) * out + row0 + piece * 16) = v;
    }
    if (threadIdx.x == 0) scale[(size_t)blockIdx.x * gridDim.y + blockIdx.y] = m.scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x];
}

void launch_transpose_fp8(const Fp8Mat& m, int out, int in, uint8_t* codes, float* scale, hipStream_t st) {
    if (out == 0 || in == 0) return;
    dim3 grid((in + kFp8Block - 1) / kFp8Block, (out + kFp8Block - 1) / kFp8Block);
    transpose_fp8_kernel<<<grid, 256, 0, st>>>(m, out, in, codes, scale);
}

}  // namespace moemix
