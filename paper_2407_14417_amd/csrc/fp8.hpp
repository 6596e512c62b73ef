// 8-bit floating point (e4m3: 1 sign, 4 exponent, 3 mantissa bits, largest value 448, no infinity) with an fp32 scale per
// block of 128: arguments of the launches, and the conversions every kernel uses.
#pragma once

#include "common.hpp"

namespace moemix {

constexpr int kFp8Block = MOE_FP8_BLOCK;
constexpr float kFp8Top = 448.0f;

struct Fp8Mat {
    const uint8_t* data;   // [out, in]
    const float* scale;    // [ceil(out/128), ceil(in/128)]
};

// What a launch of products does for an expert.
enum Fp8Todo : int32_t { kFp8Skip = 0, kFp8Run = 1, kFp8Missing = 2 };   // (missing: rows of zeros, status bit)

// y[r, :] = x[row(r), :] W_e^T for the rows r of expert e.
struct Fp8Args {
    Fp8Mat w[MOE_MAX_EXPERTS];    // up: w1
    Fp8Mat w3[MOE_MAX_EXPERTS];   // up
    int32_t todo[MOE_MAX_EXPERTS];
    const uint8_t* x;             // [x_rows, K] codes
    const float* xs;              // [ceil(K/128), x_rows]
    const int32_t* offsets;       // [E+1] or null: all P rows belong to expert 0
    const int32_t* perm;          // [P] or null; row r reads x row perm[r] / top_k (null: r)
    int32_t* status;              // or null
    void* y;                      // [P, N]
    float* y_scale;               // up, tile kernel: [ceil(N/128), P], y are codes
    int E, P, top_k, x_rows, N, K;
};

// Up-projection: hidden rows fp16( silu(W1 x) * (W3 x) ) quantized into codes [P, N] and scale [ceil(N/128), P]; h [P, N]: room for the rows in fp16.
// Sums are exact.
void launch_fp8_up(const Fp8Args& a, half_t* h, uint8_t* codes, float* scale, hipStream_t st);
// Rows of W x, fp32 or fp16 (half_out).  exact: sums as exact as 32 bits allow (else they
// may come from the matrix instructions for 8-bit operands, see fp8_tile.hip).
void launch_fp8_matmul(const Fp8Args& a, bool half_out, bool exact, hipStream_t st);
bool fp8_tile_can(const Fp8Args& a);
float fp8_tile_us(const Fp8Args& a, bool up, bool exact);
int fp8_tile_rows(const Fp8Args& a, bool up, bool exact);
// Rows per chunk of the tile kernel, 0: the kernel for few rows.
int fp8_rows_per_chunk(const Fp8Args& a, bool up, bool exact);
void launch_fp8_tile(const Fp8Args& a, bool up, bool half_out, bool exact, hipStream_t st);

// One token: up (y: [k, N] hidden rows of the slots, x: the token) or down (y: [N] the block's output, x: the hidden rows), rows quantized on the way.
struct Fp8OneArgs {
    Fp8Mat w[MOE_MAX_EXPERTS];    // up: w1
    Fp8Mat w3[MOE_MAX_EXPERTS];   // up
    int32_t todo[MOE_MAX_EXPERTS];
    const int32_t* idx;           // [k]
    const float* gate;            // [k], down
    const half_t* x;
    const half_t* residual;       // [N] or null, down
    half_t* y;
    int32_t* status;
    int k, N, K;
};
bool fp8_one_serves(int k, int d, int f);
void launch_fp8_one(const Fp8OneArgs& a, bool up, hipStream_t st);

// Chunks of `per` rows that P rows over E experts make at most.
inline int most_chunks(const Fp8Args& a, int per) {
    if (!a.offsets) return (a.P + per - 1) / per;
    const int with_rows = a.E < a.P ? a.E : a.P;
    return (a.P - with_rows) / per + with_rows;
}
void launch_quantize_fp8_rows(const half_t* x, int n, int in, uint8_t* codes, float* scale, hipStream_t st);
void launch_quantize_fp8(const half_t* w, int out, int in, uint8_t* codes, float* scale, hipStream_t st);
void launch_dequant_fp8(const Fp8Mat& m, int out, int in, half_t* w, hipStream_t st);
void launch_transpose_fp8(const Fp8Mat& m, int out, int in, uint8_t* codes, float* scale, hipStream_t st);

#if defined(__HIPCC__)

// The scale of a block whose largest magnitude is `most`, and the factor its values are multiplied with before the
// rounding to e4m3: both correctly rounded quotients.  A block of zeros: scale 0, factor 0.
__device__ __forceinline__ float fp8_scale(float most) { return __fdiv_rn(most, kFp8Top); }
__device__ __forceinline__ float fp8_factor(float most) { return most > 0.0f ? __fdiv_rn(kFp8Top, most) : most; }

// Four codes e4m3_rne(v[i]), v[0] in the lowest byte.  Magnitudes reach 448 (1 + 2^-23) at most, which rounds to 448; NaN
// stays NaN.
__device__ __forceinline__ uint32_t fp8_pack(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Eight codes -> fp16, exactly (every e4m3 value is an fp16 value).
__device__ __forceinline__ half8_t fp8_expand(uint32_t lo, uint32_t hi) {
    const half2_t a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
    const half2_t c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
    return half8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Magnitude bits of an fp16 value: their order is that of the magnitudes, infinities after all finite ones and NaN last.
__device__ __forceinline__ uint32_t magnitude_max(uint32_t most, half8_t v) {
    const uint4_t w = __builtin_bit_cast(uint4_t, v);
    uint32_t m = most;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = w[i] & 0x7FFFu, b = (w[i] >> 16) & 0x7FFFu;
        m = m > a ? m : a;
        m = m > b ? m : b;
    }
    return m;
}
__device__ __forceinline__ float magnitude_value(uint32_t bits) { return (float)__builtin_bit_cast(half_t, (uint16_t)bits); }

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
    return v > o ? v : o;
}

// The chunks of `per` rows of all experts, in expert order, for a whole wavefront: lane e holds expert e's rows and the chunks up
// to its last one.  (Offsets come from the caller: whatever they hold, rows stay within [0, P).)
struct Chunks {
    int lo, hi, mine, end, per, E;
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(end, E - 1); }
    // chunk i: its expert, first row and number of rows; false if there is none
    __device__ __forceinline__ bool find(int i, int& expert, int& begin, int& rows) const {
        const unsigned long long past = __ballot((int)(threadIdx.x & 63) < E && end > i);
        if (!past) return false;
        expert = __builtin_ctzll(past);
        const int first = i - (__builtin_amdgcn_readlane(end, expert) - __builtin_amdgcn_readlane(mine, expert));
        const int from = __builtin_amdgcn_readlane(lo, expert), to = __builtin_amdgcn_readlane(hi, expert);
        // an expert's chunks are of equal length, to a whole number of 16 rows
        const int even = (to - from - 1) / __builtin_amdgcn_readlane(mine, expert) + 1, size = min(per, (even + 15) & ~15);
        begin = from + first * size;
        rows = min(size, to - begin);
        return rows > 0;
    }
};

__device__ __forceinline__ Chunks count_chunks(const Fp8Args& a, int per, int lane) {
    Chunks c{0, 0, 0, 0, per, a.offsets ? a.E : 1};
    if (!a.offsets) {
        c.hi = lane == 0 ? a.P : 0;
    } else if (lane < a.E) {
        c.lo = min(max(a.offsets[lane], 0), a.P);
        c.hi = min(max(a.offsets[lane + 1], c.lo), a.P);
    }
    c.mine = (c.hi - c.lo + per - 1) / per;
    c.end = c.mine;                                   // inclusive prefix sum over the experts
#pragma unroll
    for (int m = 1; m < MOE_MAX_EXPERTS; m <<= 1) {
        const int below = __shfl_up(c.end, m, kWave);
        if (lane >= m) c.end += below;
    }
    return c;
}

// The row of x that row r of y multiplies.
__device__ __forceinline__ int row_of(const Fp8Args& a, int r) {
    if (!a.perm) return r;
    const int t = a.perm[r] / a.top_k;
    return min(max(t, 0), a.x_rows - 1);
}

#endif

}  // namespace moemix
