// Training of the gate: the balance loss with per-expert counts, and the gradients of gates and loss with respect to the logits,
// the tokens, the gate matrix and its bias.
//
// Lanes: LANES = 1, 2, 4 or 8 neighbouring lanes share a token, each holds four of its (up to 32) experts.  A softmax is two
// reductions over them on the DPP network; sums over tokens stay in the lane, which always sees the same experts.
//
// Bound: the loss by its launches and the way to memory and back (65536 tokens, 32 experts, four slots: 9.5 MB, 1.8 us of a copy's rate; 7.3 us and a finish of
// 4.1; few tokens: one launch, 4.7).  The backward pass by x read and d_x written once (16384 tokens, 4096 columns, 32 experts, fp16: 272 MB, 52 us; 69-71 us,
// 3.9 TB/s, beside 6.8 for d_logits and 4.9 for the sums of d_w).  d_x and d_w share the one pass over x's tokens and columns, since both
// need a tile's d_logits.
#include <type_traits>

#include "gate_grad.hpp"
#include "kernels.hpp"

namespace moemix {

namespace {

typedef uint4_t __attribute__((aligned(2))) uint4_anywhere_t;    // (tokens may lie anywhere)
typedef float4_t __attribute__((aligned(4))) float4_anywhere_t;

template <int LANES, class F>
__device__ __forceinline__ float over_experts(float v, F f) {
    if (LANES > 1) v = f(v, dpp_move<0xB1>(v));      // lanes 1 apart,
    if (LANES > 2) v = f(v, dpp_move<0x4E>(v));      // 2 apart,
    if (LANES > 4) v = f(v, dpp_move<0x141>(v));     // and the other four of the eight
    return v;
}
template <int LANES>
__device__ __forceinline__ float sum_experts(float v) { return over_experts<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES>
__device__ __forceinline__ float max_experts(float v) { return over_experts<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }

// Sum over the lanes of a wavefront that hold the same experts.
template <int LANES, class V>
__device__ __forceinline__ V over_tokens(V v) {
#pragma unroll
    for (int m = 32; m >= LANES; m >>= 1) v += __shfl_xor(v, m, kWave);
    return v;
}

// A lane's four logits; experts past the last one have -infinity.  WIDE: E is a multiple of 4 and rows start on 16 bytes.
template <bool WIDE>
__device__ __forceinline__ float4_t load_logits(const float* __restrict__ logits, size_t t, int E, int e0) {
    float4_t l;
    const float* const p = logits + t * E + e0;
    if (WIDE) {
        if (e0 < E) return *(const float4_t*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = -__builtin_inff();
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) l[i] = e0 + i < E ? p[i] : -__builtin_inff();
    }
    return l;
}

// What a lane reads of a token, all of it asked for before anything is used: up to eight slots (past the k-th: the k-th again).
struct Token {
    float4_t logits;
    int32_t idx[MOE_MAX_TOPK];
    bool counts;
};
template <bool WIDE>
__device__ __forceinline__ void load_token(Token& r, const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                           const uint8_t* __restrict__ valid, size_t t, int E, int k, int e0) {
    r.logits = load_logits<WIDE>(logits, t, E, e0);
    const int32_t* const p = idx + t * k;
#pragma unroll
    for (int s = 0; s < 4; ++s) r.idx[s] = p[min(s, k - 1)];
    if (k > 4)
#pragma unroll
        for (int s = 4; s < MOE_MAX_TOPK; ++s) r.idx[s] = p[min(s, k - 1)];
    r.counts = !valid || valid[t];
}

// Softmax over the experts with weights: p[i] = m[i] exp(l[i] - most) / sum, most over the experts with m != 0.  All of those at
// -infinity: zeros.  NaN and +infinity make NaN.
template <int LANES, class M>
__device__ __forceinline__ void softmax(const float4_t l, M m, float (&p)[4]) {
    float most = -__builtin_inff(), any = 0.0f, sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (m(i) == 0.0f) continue;
        most = fmaxf(most, l[i]);
        any = l[i] != -__builtin_inff() ? 1.0f : any;
    }
    most = max_experts<LANES>(most);
    any = max_experts<LANES>(any);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        p[i] = m(i) != 0.0f && any != 0.0f ? m(i) * expf(l[i] - most) : 0.0f;
        sum += p[i];
    }
    sum = sum_experts<LANES>(sum);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = any != 0.0f ? p[i] / sum : 0.0f;
}

// ---------------------------------------------------------------- loss

constexpr int kLossWaves = 16;    // (so that few workgroups leave partial sums for the finish)

// What is known at the end: counts, mean probabilities and the loss, from a lane's (e = lane, up to 31) sums over all tokens, by half a
// wavefront; and the status of the call.
__device__ __forceinline__ void finish_loss(int e, double sum, int32_t c, int32_t n, bool bad, int E, int k, int32_t* __restrict__ counts,
                                            float* __restrict__ mean_prob, float* __restrict__ loss, int32_t* __restrict__ status) {
    const double mean = n > 0 ? sum / n : 0.0;
    double l = e < E ? mean * c : 0.0;
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) l += __shfl_xor(l, m, kWave);
    if (e < E) {
        counts[e] = c;
        mean_prob[e] = (float)mean;
    }
    if (e == 0) {
        counts[E] = n;
        *loss = n > 0 ? (float)(l * E / ((double)n * k)) : 0.0f;
        *status = bad ? kStatusBadIndex : 0;
    }
}

// Sums over the workgroup's tokens.  A token's lanes count, each for its own four experts, the slots that chose them.  Few tokens: one
// workgroup finishes as well (ONE); else partial sums go to `sums` and `partial`.
template <int LANES, bool WIDE, bool ONE>
__global__ __launch_bounds__(64 * kLossWaves) void balance_sums_kernel(
    const float* __restrict__ logits, const int32_t* __restrict__ idx, const uint8_t* __restrict__ valid, int T, int E, int k,
    float* __restrict__ sums, int32_t* __restrict__ partial, int32_t* __restrict__ counts, float* __restrict__ mean_prob,
    float* __restrict__ loss, int32_t* __restrict__ status) {
    constexpr int kWaves = kLossWaves, kTokens = 64 / LANES;
    __shared__ float wave_sums[kWaves][32];
    __shared__ int32_t wave_counts[kWaves][34];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LANES, e0 = 4 * j;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    int32_t n[4] = {0, 0, 0, 0}, tokens = 0;
    bool bad = false;
    const long long step = (long long)gridDim.x * kWaves * kTokens;
    long long t = (long long)(blockIdx.x * kWaves + wave) * kTokens + lane / LANES;
    Token now, next;
    if (t < T) load_token<WIDE>(next, logits, idx, valid, t, E, k, e0);
    for (; t < T; t += step) {                        // (a token's lanes agree)
        now = next;
        if (t + step < T) load_token<WIDE>(next, logits, idx, valid, t + step, E, k, e0);
        if (!now.counts) continue;
        float p[4];
        softmax<LANES>(now.logits, [&](int i) { return e0 + i < E ? 1.0f : 0.0f; }, p);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += p[i];
#pragma unroll
        for (int s = 0; s < MOE_MAX_TOPK; ++s) {
            if (s >= k) break;
            const int e = now.idx[s];
            bad |= (unsigned)e >= (unsigned)E;
#pragma unroll
            for (int i = 0; i < 4; ++i) n[i] += e == e0 + i ? 1 : 0;
        }
        tokens += j == 0 ? 1 : 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc[i] = over_tokens<LANES>(acc[i]);
        n[i] = over_tokens<LANES>(n[i]);
    }
    tokens = over_tokens<1>(tokens);
    const bool any_bad = __ballot(bad) != 0;
    if (lane < LANES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            wave_sums[wave][e0 + i] = acc[i];
            wave_counts[wave][e0 + i] = n[i];
        }
    }
    if (lane == 0) {
        wave_counts[wave][32] = tokens;
        wave_counts[wave][33] = any_bad;
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
    const int at = lane < E ? lane : 32 + (lane - E);    // lane E: tokens, lane E + 1: an index out of range
    if (ONE) {
        int32_t c = 0, all = 0, flags = 0;
        double v = 0.0;
        for (int w = 0; w < kWaves; ++w) {
            if (lane < E) {
                c += wave_counts[w][lane];
                v += wave_sums[w][lane];
            }
            all += wave_counts[w][32];
            flags |= wave_counts[w][33];
        }
        finish_loss(lane, v, c, all, flags != 0, E, k, counts, mean_prob, loss, status);
    } else if (lane < E + 2) {
        int32_t c = 0;
        for (int w = 0; w < kWaves; ++w) c += wave_counts[w][at];
        partial[(size_t)blockIdx.x * (E + 2) + lane] = c;
        if (lane < E) {
            float v = 0.0f;
            for (int w = 0; w < kWaves; ++w) v += wave_sums[w][lane];
            sums[(size_t)blockIdx.x * E + lane] = v;
        }
    }
}

// One workgroup: adds the partial sums of up to 32 ROWS workgroups up (in 64 bits, in a fixed order) and forms the loss.
template <int ROWS>
__global__ __launch_bounds__(1024) void balance_finish_kernel(const float* __restrict__ sums, const int32_t* __restrict__ partial, int blocks,
                                                              int E, int k, int32_t* __restrict__ counts, float* __restrict__ mean_prob,
                                                              float* __restrict__ loss, int32_t* __restrict__ status) {
    __shared__ double part[32][33];
    __shared__ int32_t part_n[32][35];
    const int e = threadIdx.x & 31, g = threadIdx.x >> 5;
    double v = 0.0;
    int32_t c = 0, more = 0;
    float s[ROWS];                                    // all of a thread's values are asked for before the first is added
    int32_t cs[ROWS], ms[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const size_t b = min(g + 32 * i, blocks - 1);
        s[i] = sums[b * E + min(e, E - 1)];
        cs[i] = partial[b * (E + 2) + min(e, E - 1)];
        ms[i] = partial[b * (E + 2) + E + (e & 1)];
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
        if (g + 32 * i < blocks) {
            v += e < E ? s[i] : 0.0f;
            c += e < E ? cs[i] : 0;
            more += ms[i];
        }
    part[g][e] = v;
    part_n[g][e] = c;
    if (e < 2) part_n[g][32 + e] = more;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    int32_t n = 0, flags = 0;
    v = 0.0;
    c = 0;
    for (int i = 0; i < 32; ++i) {
        n += part_n[i][32];
        flags |= part_n[i][33];
        if (threadIdx.x < 32) {
            v += part[i][e];
            c += part_n[i][e];
        }
    }
    finish_loss(threadIdx.x, v, c, n, flags != 0, E, k, counts, mean_prob, loss, status);
}

// ---------------------------------------------------------------- backward

constexpr int kGradTokenWaves = 4;   // (16: 333 tokens 14.4 -> 16.1 us a backward pass)

// d_logits, and partial sums of them over the workgroup's tokens for the bias.
template <int LANES, bool WIDE>
__global__ __launch_bounds__(64 * kGradTokenWaves) void gate_dlogits_kernel(GateGradArgs a, float* __restrict__ sums, int32_t* __restrict__ flags) {
    __shared__ float wave_sums[kGradTokenWaves][32];
    __shared__ int32_t wave_bad[kGradTokenWaves];
    constexpr int kTokens = 64 / LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LANES, e0 = 4 * j, E = a.E;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, c[4] = {0.0f, 0.0f, 0.0f, 0.0f}, coef = 0.0f;
    if (a.d_loss) {
        const float n = (float)a.counts[E];
        coef = n > 0.0f ? *a.d_loss * (float)E / (n * (float)a.k) / n : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) c[i] = e0 + i < E ? (float)a.counts[e0 + i] : 0.0f;
    }
    bool bad = false;
    const long long step = (long long)gridDim.x * kGradTokenWaves * kTokens;
    long long t = (long long)(blockIdx.x * kGradTokenWaves + wave) * kTokens + lane / LANES;
    Token now, next;
    float dgs[MOE_MAX_TOPK], dgs_next[MOE_MAX_TOPK];
    auto ask = [&](long long at) {
        load_token<WIDE>(next, a.logits, a.idx, a.valid, at, E, a.k, e0);
        if (!a.d_gate) return;
        const float* const p = a.d_gate + at * a.k;
#pragma unroll
        for (int s = 0; s < 4; ++s) dgs_next[s] = p[min(s, a.k - 1)];
        if (a.k > 4)
#pragma unroll
            for (int s = 4; s < MOE_MAX_TOPK; ++s) dgs_next[s] = p[min(s, a.k - 1)];
    };
    if (t < a.T) ask(t);
    for (; t < a.T; t += step) {
        now = next;
#pragma unroll
        for (int s = 0; s < MOE_MAX_TOPK; ++s) dgs[s] = dgs_next[s];
        if (t + step < a.T) ask(t + step);
        float dl[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (now.counts) {
            const float4_t l = now.logits;
            if (a.d_loss) {
                float p[4], mean = 0.0f;
                softmax<LANES>(l, [&](int i) { return e0 + i < E ? 1.0f : 0.0f; }, p);
#pragma unroll
                for (int i = 0; i < 4; ++i) mean += p[i] * c[i];
                mean = sum_experts<LANES>(mean);
#pragma unroll
                for (int i = 0; i < 4; ++i) dl[i] = coef * p[i] * (c[i] - mean);
            }
            if (a.d_gate) {
                // the chosen experts with how often they were chosen (an expert chosen twice has two gates)
                float times[4] = {0.0f, 0.0f, 0.0f, 0.0f}, dg[4] = {0.0f, 0.0f, 0.0f, 0.0f}, g[4], dot = 0.0f;
#pragma unroll
                for (int s = 0; s < MOE_MAX_TOPK; ++s) {
                    if (s >= a.k) break;
                    const int e = now.idx[s];
                    const float d = dgs[s];
                    bad |= (unsigned)e >= (unsigned)E;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (e == e0 + i && e < E) {
                            times[i] += 1.0f;
                            dg[i] += d;
                        }
                }
                softmax<LANES>(l, [&](int i) { return times[i]; }, g);        // times * gate
                // one gate of the expert is g / times: sum_s gate_s d_gate_s
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    g[i] = times[i] > 0.0f ? g[i] / times[i] : 0.0f;
                    dot += times[i] > 0.0f ? g[i] * dg[i] : 0.0f;
                }
                dot = sum_experts<LANES>(dot);
#pragma unroll
                for (int i = 0; i < 4; ++i) dl[i] += times[i] > 0.0f ? g[i] * (dg[i] - times[i] * dot) : 0.0f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += dl[i];
        float* const out = a.d_logits + (size_t)t * E + e0;
        if (WIDE) {
            if (e0 < E) *(float4_t*)out = float4_t{dl[0], dl[1], dl[2], dl[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e0 + i < E) out[i] = dl[i];
        }
    }
    const bool any_bad = __ballot(bad) != 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = over_tokens<LANES>(acc[i]);
    if (lane < LANES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) wave_sums[wave][e0 + i] = acc[i];
    }
    if (lane == 0) wave_bad[wave] = any_bad;
    __syncthreads();
    if ((int)threadIdx.x < E) {
        float v = 0.0f;
        for (int w = 0; w < kGradTokenWaves; ++w) v += wave_sums[w][threadIdx.x];
        sums[(size_t)blockIdx.x * E + threadIdx.x] = v;
    }
    if (threadIdx.x == 0) {
        int32_t f = 0;
        for (int w = 0; w < kGradTokenWaves; ++w) f |= wave_bad[w];
        flags[blockIdx.x] = f;
    }
}

// One workgroup of 32 GROUPS threads: d_bias (in 64 bits, in a fixed order, of up to GROUPS ROWS workgroups' sums) and the status of the call, from
// what gate_dlogits_kernel left.
template <int GROUPS, int ROWS>
__device__ __forceinline__ void finish_bias(const float* __restrict__ sums, const int32_t* __restrict__ flags, int blocks, int E,
                                            float* __restrict__ d_bias, int32_t* __restrict__ status) {
    __shared__ double part[GROUPS][33];
    __shared__ int32_t bad;
    const int e = threadIdx.x & 31, g = threadIdx.x >> 5;
    if (threadIdx.x == 0) bad = 0;
    double v = 0.0;
    float r[ROWS];                                       // all of a thread's values are asked for before the first is added
#pragma unroll
    for (int i = 0; i < ROWS; ++i) r[i] = sums[(size_t)min(g + GROUPS * i, blocks - 1) * E + min(e, E - 1)];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) v += e < E && g + GROUPS * i < blocks ? r[i] : 0.0f;
    part[g][e] = v;
    int32_t f = 0;
    for (int b = threadIdx.x; b < blocks; b += 32 * GROUPS) f |= flags[b];
    __syncthreads();
    if (f) atomicOr(&bad, 1);
    __syncthreads();
    if (d_bias && (int)threadIdx.x < E) {
        v = 0.0;
        for (int i = 0; i < GROUPS; ++i) v += part[i][e];
        d_bias[e] = (float)v;
    }
    if (threadIdx.x == 0) *status = bad ? kStatusBadIndex : 0;
}

// Workgroup 0: d_bias and the status; the others: d_w from its partial sums, in order, four values per thread.
__global__ __launch_bounds__(256) void gate_finish_kernel(const float* __restrict__ sums, const int32_t* __restrict__ flags, int blocks, int E,
                                                          float* __restrict__ d_bias, int32_t* __restrict__ status,
                                                          const float* __restrict__ dw, int splits, size_t n, float* __restrict__ d_w) {
    if (blockIdx.x == 0) {
        finish_bias<8, kGateBlocks / 8>(sums, flags, blocks, E, d_bias, status);
        return;
    }
    const size_t i = ((size_t)(blockIdx.x - 1) * 256 + threadIdx.x) * 4;
    if (i >= n) return;                                  // (n = E d is a multiple of 64)
    float4_t v = *(const float4_t*)(dw + i);
#pragma unroll 8
    for (int s = 1; s < splits; ++s) v += *(const float4_t*)(dw + s * n + i);
    *(float4_anywhere_t*)(d_w + i) = v;
}

// ---- d_x = d_logits W and d_w = d_logits^T x in one pass over x, on the matrix cores
//
// A wavefront works on units of 32 tokens x 128 columns: a lane loads 8 columns of 8 tokens, lane l columns 8 (l & 15) .. and tokens
// 8 (l >> 4) .. of the unit.  Its 8 x 8 halves are transposed in registers (32 byte permutes) into the operands of d_w, whose
// contraction runs over tokens; the contraction of d_x over (up to 32) experts is one v_mfma_f32_16x16x32_f16 long.
// x and W are fp16 as they are.  d_logits are 32-bit: a power of two brings the largest of a contraction's values to 2^14, then
// each is the sum of two halves, hi = fp16(v), lo = fp16(v - hi), good to 2^-22 of the value (or 2^-39 of the largest): two products each.
// With fp32 products of the vector units this took 64 multiply-adds per element of x at 32 experts, twice the time of its
// bytes, and the registers of 256 accumulators spilled: 16384 tokens, 4096 columns, 32 experts 3757 us.

constexpr int kGradWaves = 8;

// v, w -> 2^k with the largest magnitude `most` brought to 2^14 .. 2^15 (1 for zeros, infinities and NaN)
__device__ __forceinline__ float half_scale(float most) {
    const int e = (int)(__builtin_bit_cast(uint32_t, most) >> 23) & 255;
    const int k = e == 255 || most == 0.0f ? 0 : min(14 + 127 - e, 120);
    return __builtin_bit_cast(float, (uint32_t)(127 + k) << 23);
}
__device__ __forceinline__ void split_halves(const float (&v)[8], float scale, half8_t& hi, half8_t& lo) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float f = v[i] * scale;
        hi[i] = (half_t)f;
        lo[i] = (half_t)(f - (float)hi[i]);
    }
}
__device__ __forceinline__ float largest(const float (&v)[8]) {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
    return m;
}

// ET: tiles of 16 experts.  Workgroup (x, y): columns 128 x .., the y-th share of the units' token tiles, its wavefronts in turn.  One share alone: the
// workgroup behind the last column finishes what gate_dlogits_kernel left.
struct GradRest {
    const float* sums;
    const int32_t* flags;
    int blocks;
    int32_t* status;
};
template <int ET, typename OUT>
__global__ __launch_bounds__(64 * kGradWaves, 2) void gate_dx_dw_kernel(GateGradArgs a, int tiles_per_split, float* __restrict__ dw, GradRest rest) {
    if ((int)blockIdx.x * 128 >= a.d) {
        if (rest.blocks <= 64) finish_bias<2 * kGradWaves, 4>(rest.sums, rest.flags, rest.blocks, a.E, a.d_bias, rest.status);
        else finish_bias<2 * kGradWaves, kGateBlocks / (2 * kGradWaves)>(rest.sums, rest.flags, rest.blocks, a.E, a.d_bias, rest.status);
        return;
    }
    __shared__ float4_t sums[kGradWaves / 2][16][64];
    const int lane = threadIdx.x & 63, r16 = lane & 15, q = lane >> 4, E = a.E, d = a.d;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int col0 = blockIdx.x * 128, col = col0 + 8 * r16;
    const bool in = col < d;                             // (d is a multiple of 64)
    // W for d_x: row r of tile j is column 32 (j >> 1) + 8 (r >> 2) + 4 (j & 1) + (r & 3), so that a lane's results of two tiles
    // are eight neighbouring columns
    half8_t w[8] = {};
    if (a.d_x) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int c = col0 + 32 * (j >> 1) + 8 * (r16 >> 2) + 4 * (j & 1) + (r16 & 3);
            const half_t* const src = a.wg + (c < d ? c : 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[j][i] = src[(size_t)min(8 * q + i, E - 1) * d];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)                      // (experts past the last one; columns past the last one are not stored)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (8 * q + i >= E) w[j][i] = (half_t)0.0f;
    }
    float4_t acc[8][ET];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int s = 0; s < ET; ++s) acc[j][s] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
    const int tiles = (a.T - 1) / 32 + 1;
    const int first = blockIdx.y * tiles_per_split, end = min(first + tiles_per_split, tiles);
    float* const dl = (float*)sums + wave * 1024;        // the unit's d_logits, [32][E]
    // What the next unit needs is asked for between the two products of this one.  Tokens past the last one: the last one again; their d_logits are 0.
    uint4_t x[8];
    float4_t part[4];
    uint32_t valid[8] = {1, 1, 1, 1, 1, 1, 1, 1};
    auto ask = [&](int tile) {
        const size_t t0 = (size_t)tile * 32;
        const int left = a.T - tile * 32;
        if (a.d_w) {
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = *(const uint4_anywhere_t*)(a.x + (t0 + min(8 * q + k, left - 1)) * d + (in ? col : 0));
        }
        if (a.valid)
#pragma unroll
            for (int k = 0; k < 8; ++k) valid[k] = a.valid[t0 + min(8 * q + k, left - 1)];
        const int n = min(left, 32) * E;
        const float* const src = a.d_logits + t0 * E;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 256 * i + 4 * lane;
            part[i] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (at + 4 <= n) {
                part[i] = *(const float4_anywhere_t*)(src + at);
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (at + c < n) part[i][c] = src[at + c];
            }
        }
    };
    if (first + wave < end) ask(first + wave);
    for (int tile = first + wave; tile < end; tile += kGradWaves) {
        const size_t t0 = (size_t)tile * 32;
        const int left = a.T - tile * 32;                // tokens of the tile (32 or more: all)
        wave_lds_handover();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (256 * i < 32 * E) *(float4_t*)(dl + 256 * i + 4 * lane) = part[i];
        wave_lds_handover();
        uint32_t live = ~0u;                             // bit t: token t of the unit is no padding (its d_x is 0 whatever W holds)
        if (a.valid) {
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) m |= (valid[k] ? 1u : 0u) << k;
            live = __builtin_amdgcn_readlane(m, 0) | __builtin_amdgcn_readlane(m, 16) << 8 | __builtin_amdgcn_readlane(m, 32) << 16 |
                   __builtin_amdgcn_readlane(m, 48) << 24;
        }
        if (a.d_w) {
            if (a.valid) {                               // padding may hold anything
#pragma unroll
                for (int k = 0; k < 8; ++k)
#pragma unroll
                    for (int c = 0; c < 4; ++c) x[k][c] = valid[k] ? x[k][c] : 0u;
            }
            half8_t hi[ET], lo[ET];
            float back[ET];
#pragma unroll
            for (int s = 0; s < ET; ++s) {
                const int e = min(16 * s + r16, E - 1);  // (columns past the last expert are not stored)
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = dl[(8 * q + k) * E + e];
                float most = largest(v);
                most = fmaxf(most, __shfl_xor(most, 16, kWave));
                most = fmaxf(most, __shfl_xor(most, 32, kWave));
                const float scale = half_scale(most);
                back[s] = 1.0f / scale;                  // (a power of two: exact)
                split_halves(v, scale, hi[s], lo[s]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {                // row r of tile j is column 8 r + j: its halves of the 8 tokens
                uint4_t op;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    op[k] = __builtin_amdgcn_perm(x[2 * k + 1][j >> 1], x[2 * k][j >> 1], (j & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
                for (int s = 0; s < ET; ++s) {
                    float4_t o = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, op), lo[s], float4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
                    o = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8_t, op), hi[s], o, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[j][s][i] = fmaf(o[i], back[s], acc[j][s][i]);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (tile + kGradWaves < end) ask(tile + kGradWaves);
        __builtin_amdgcn_sched_barrier(0);
        if (a.d_x) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int t = 16 * h + r16;
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = 8 * q + i < E ? dl[t * E + 8 * q + i] : 0.0f;
                float most = largest(v);
                most = fmaxf(most, __shfl_xor(most, 16, kWave));
                most = fmaxf(most, __shfl_xor(most, 32, kWave));
                const float scale = half_scale(most), back = 1.0f / scale;
                half8_t hi, lo;
                split_halves(v, scale, hi, lo);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    float4_t o[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[2 * p + c], lo, float4_t{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
                        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_f16(w[2 * p + c], hi, o[c], 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[c][i] = live >> t & 1 ? o[c][i] * back : 0.0f;
                    }
                    const int c = col0 + 32 * p + 8 * q;
                    if (t >= left || c >= d) continue;
                    OUT* const out = (OUT*)a.d_x + (t0 + t) * d + c;
                    if (sizeof(OUT) == 2) {
                        half8_t r;
#pragma unroll
                        for (int i = 0; i < 8; ++i) r[i] = (half_t)o[i >> 2][i & 3];
                        *(uint4_anywhere_t*)out = __builtin_bit_cast(uint4_t, r);
                    } else {
                        *(uint4_anywhere_t*)out = __builtin_bit_cast(uint4_t, o[0]);
                        *(uint4_anywhere_t*)(out + 4) = __builtin_bit_cast(uint4_t, o[1]);
                    }
                }
            }
        }
    }
    if (!a.d_w) return;
    // the wavefronts' sums: the upper half adds to the lower one, three times
#pragma unroll
    for (int half = kGradWaves / 2; half >= 1; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int s = 0; s < ET; ++s) sums[wave - half][j * ET + s][lane] = acc[j][s];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int s = 0; s < ET; ++s) acc[j][s] += sums[wave][j * ET + s][lane];
    }
    if (wave) return;
#pragma unroll
    for (int s = 0; s < ET; ++s) {
        const int e = 16 * s + r16;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = col0 + 8 * (4 * q + i);
            if (e >= E || c >= d) continue;
            float* const o = dw + ((size_t)blockIdx.y * E + e) * d + c;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = acc[j][s][i];
        }
    }
}

template <class F>
void by_lanes(int E, F f) {
    if (E <= 4) f(std::integral_constant<int, 1>{});
    else if (E <= 8) f(std::integral_constant<int, 2>{});
    else if (E <= 16) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 8>{});
}

bool wide_rows(const void* p, int E) { return E % 4 == 0 && (uintptr_t)p % 16 == 0; }

// Up to so many workgroups' tokens one workgroup takes alone.
constexpr int kOneBlock = 2;

int token_blocks(int T, int E, int waves, int most) {
    const int lanes = E <= 4 ? 1 : E <= 8 ? 2 : E <= 16 ? 4 : 8, per = 64 / lanes * waves;
    const int blocks = (T - 1) / per + 1;
    return blocks < most ? blocks : most;
}

}  // namespace

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* valid, int T, int E, int k, int32_t* counts,
                         float* mean_prob, float* loss, const GateWorkspace& w, hipStream_t st) {
    const int blocks = token_blocks(T, E, kLossWaves, kGateBlocks / 2);
    const bool one = blocks <= kOneBlock;
    by_lanes(E, [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        const auto go = [&](auto wide) {
            constexpr bool WIDE = decltype(wide)::value;
            if (one)
                balance_sums_kernel<LANES, WIDE, true><<<1, 64 * kLossWaves, 0, st>>>(logits, idx, valid, T, E, k, w.sums, w.counts, counts, mean_prob,
                                                                           loss, w.status);
            else
                balance_sums_kernel<LANES, WIDE, false><<<blocks, 64 * kLossWaves, 0, st>>>(logits, idx, valid, T, E, k, w.sums, w.counts,
                                                                                            counts, mean_prob, loss, w.status);
        };
        if (wide_rows(logits, E)) go(std::true_type{});
        else go(std::false_type{});
    });
    static_assert(kGateBlocks / 2 == 32 * 8, "rows");
    if (one) return;
    if (blocks <= 64) balance_finish_kernel<2><<<1, 1024, 0, st>>>(w.sums, w.counts, blocks, E, k, counts, mean_prob, loss, w.status);
    else balance_finish_kernel<8><<<1, 1024, 0, st>>>(w.sums, w.counts, blocks, E, k, counts, mean_prob, loss, w.status);
}

// A compute unit per workgroup, as far as every wavefront has a tile of 32 tokens; up to two tiles a wavefront one share takes alone, which saves the
// launch that adds shares up.
int gate_dw_splits(int T, int d, int) {
    const int by_work = ((T - 1) / 32 + kGradWaves) / kGradWaves, by_chip = 256 / ((d + 127) / 128);
    const int s = by_work < by_chip ? by_work : by_chip;
    return by_work <= 2 || s < 1 ? 1 : s;
}

void launch_route_backward(const GateGradArgs& a, const GateWorkspace& w, hipStream_t st) {
    const int blocks = token_blocks(a.T, a.E, kGradTokenWaves, kGateBlocks);
    by_lanes(a.E, [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        if (wide_rows(a.logits, a.E) && wide_rows(a.d_logits, a.E))
            gate_dlogits_kernel<LANES, true><<<blocks, 64 * kGradTokenWaves, 0, st>>>(a, w.sums, w.counts);
        else
            gate_dlogits_kernel<LANES, false><<<blocks, 64 * kGradTokenWaves, 0, st>>>(a, w.sums, w.counts);
    });
    const auto finish = [&](int splits) {
        const size_t n = splits > 1 ? (size_t)a.E * a.d : 0;
        gate_finish_kernel<<<1 + (unsigned)((n / 4 + 255) / 256), 256, 0, st>>>(w.sums, w.counts, blocks, a.E, a.d_bias, w.status, w.dw, splits, n,
                                                                                a.d_w);
    };
    if (!a.d_x && !a.d_w) {
        finish(1);
        return;
    }
    const int splits = w.dw_splits, tiles_per_split = (a.T - 1) / 32 / splits + 1;
    float* const dw = splits > 1 ? w.dw : a.d_w;
    const GradRest rest{w.sums, w.counts, blocks, w.status};
    const dim3 grid((a.d + 127) / 128 + (splits == 1), splits);
    const auto go = [&](auto tiles) {
        constexpr int ET = decltype(tiles)::value;
        if (a.d_x_half) gate_dx_dw_kernel<ET, half_t><<<grid, 64 * kGradWaves, 0, st>>>(a, tiles_per_split, dw, rest);
        else gate_dx_dw_kernel<ET, float><<<grid, 64 * kGradWaves, 0, st>>>(a, tiles_per_split, dw, rest);
    };
    if (a.E <= 16) go(std::integral_constant<int, 1>{});
    else go(std::integral_constant<int, 2>{});
    if (splits > 1) finish(a.d_w ? splits : 1);
}

}  // namespace moemix
