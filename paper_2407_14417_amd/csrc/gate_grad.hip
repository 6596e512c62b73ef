// Training of the gate: the balance loss with per-expert counts, and the gradients of gates and loss with respect to the logits,
// the tokens, the gate matrix and its bias.
//
// Lanes: LANES = 1, 2, 4 or 8 neighbouring lanes share a token, each holds four of its (up to 32) experts.  A softmax is two
// reductions over them on the DPP network; sums over tokens stay in the lane, which always sees the same experts.
#include <type_traits>

#include "gate_grad.hpp"
#include "kernels.hpp"

namespace moemix {

namespace {

typedef half4_t __attribute__((aligned(2))) half4_anywhere_t;    // (tokens may lie anywhere)

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

constexpr int kLossWaves = 4;

// Partial sums over the workgroup's tokens.  A token's lanes count, each for its own four experts, the slots that chose them.
template <int LANES, bool WIDE>
__global__ __launch_bounds__(64 * kLossWaves) void balance_sums_kernel(const float* __restrict__ logits, const int32_t* __restrict__ idx,
                                                                       const uint8_t* __restrict__ valid, int T, int E, int k,
                                                                       float* __restrict__ sums, int32_t* __restrict__ counts,
                                                                       int32_t* __restrict__ status) {
    __shared__ float wave_sums[kLossWaves][32];
    __shared__ int32_t wave_counts[kLossWaves][33];
    constexpr int kTokens = 64 / LANES;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane % LANES, e0 = 4 * j;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    int32_t n[4] = {0, 0, 0, 0}, tokens = 0;
    bool bad = false;
    for (long long t = (long long)(blockIdx.x * kLossWaves + wave) * kTokens + lane / LANES; t < T;
         t += (long long)gridDim.x * kLossWaves * kTokens) {
        if (valid && !valid[t]) continue;             // (a token's lanes agree)
        float p[4];
        softmax<LANES>(load_logits<WIDE>(logits, t, E, e0), [&](int i) { return e0 + i < E ? 1.0f : 0.0f; }, p);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] += p[i];
        for (int s = 0; s < k; ++s) {
            const int e = idx[t * k + s];
            bad |= (unsigned)e >= (unsigned)E;
#pragma unroll
            for (int i = 0; i < 4; ++i) n[i] += e == e0 + i ? 1 : 0;
        }
        tokens += j == 0 ? 1 : 0;
    }
    if (bad && status) atomicOr(status, kStatusBadIndex);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        acc[i] = over_tokens<LANES>(acc[i]);
        n[i] = over_tokens<LANES>(n[i]);
    }
    tokens = over_tokens<1>(tokens);
    if (lane < LANES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            wave_sums[wave][e0 + i] = acc[i];
            wave_counts[wave][e0 + i] = n[i];
        }
    }
    if (lane == 0) wave_counts[wave][32] = tokens;
    __syncthreads();
    if ((int)threadIdx.x <= E) {
        const int e = threadIdx.x;
        int32_t c = 0;
        for (int w = 0; w < kLossWaves; ++w) c += wave_counts[w][e < E ? e : 32];
        counts[(size_t)blockIdx.x * (E + 1) + e] = c;
        if (e < E) {
            float v = 0.0f;
            for (int w = 0; w < kLossWaves; ++w) v += wave_sums[w][e];
            sums[(size_t)blockIdx.x * E + e] = v;
        }
    }
}

// One workgroup: adds the partial sums up (in 64 bits, in a fixed order) and forms the loss.
__global__ __launch_bounds__(1024) void balance_finish_kernel(const float* __restrict__ sums, const int32_t* __restrict__ partial, int blocks,
                                                              int E, int k, int32_t* __restrict__ counts, float* __restrict__ mean_prob,
                                                              float* __restrict__ loss) {
    __shared__ double part[32][33];
    __shared__ int32_t part_n[32][33];
    const int e = threadIdx.x & 31, g = threadIdx.x >> 5;
    double v = 0.0;
    int32_t c = 0;
    if (e < E)
        for (int b = g; b < blocks; b += 32) {
            v += sums[(size_t)b * E + e];
            c += partial[(size_t)b * (E + 1) + e];
        }
    part[g][e] = v;
    part_n[g][e] = c;
    if (e == 0) {
        int32_t t = 0;
        for (int b = g; b < blocks; b += 32) t += partial[(size_t)b * (E + 1) + E];
        part_n[g][32] = t;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int32_t n = 0;
        v = 0.0;
        c = 0;
        for (int i = 0; i < 32; ++i) {
            n += part_n[i][32];
            v += part[i][e];
            c += part_n[i][e];
        }
        const double mean = n > 0 ? v / n : 0.0;
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
        }
    }
}

// ---------------------------------------------------------------- backward

// d_logits, and partial sums of them over the workgroup's tokens for the bias.
template <int LANES, bool WIDE>
__global__ __launch_bounds__(64 * kLossWaves) void gate_dlogits_kernel(GateGradArgs a, float* __restrict__ sums, int32_t* __restrict__ status) {
    __shared__ float wave_sums[kLossWaves][32];
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
    for (long long t = (long long)(blockIdx.x * kLossWaves + wave) * kTokens + lane / LANES; t < a.T;
         t += (long long)gridDim.x * kLossWaves * kTokens) {
        float dl[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (!a.valid || a.valid[t]) {
            const float4_t l = load_logits<WIDE>(a.logits, t, E, e0);
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
                for (int s = 0; s < a.k; ++s) {
                    const int e = a.idx[t * a.k + s];
                    const float d = a.d_gate[t * a.k + s];
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
    if (bad && status) atomicOr(status, kStatusBadIndex);
    if (!a.d_bias) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] = over_tokens<LANES>(acc[i]);
    if (lane < LANES) {
#pragma unroll
        for (int i = 0; i < 4; ++i) wave_sums[wave][e0 + i] = acc[i];
    }
    __syncthreads();
    if ((int)threadIdx.x < E) {
        float v = 0.0f;
        for (int w = 0; w < kLossWaves; ++w) v += wave_sums[w][threadIdx.x];
        sums[(size_t)blockIdx.x * E + threadIdx.x] = v;
    }
}

__global__ __launch_bounds__(1024) void gate_dbias_kernel(const float* __restrict__ sums, int blocks, int E, float* __restrict__ d_bias) {
    __shared__ double part[32][33];
    const int e = threadIdx.x & 31, g = threadIdx.x >> 5;
    double v = 0.0;
    if (e < E)
        for (int b = g; b < blocks; b += 32) v += sums[(size_t)b * E + e];
    part[g][e] = v;
    __syncthreads();
    if ((int)threadIdx.x < E) {
        v = 0.0;
        for (int i = 0; i < 32; ++i) v += part[i][e];
        d_bias[e] = (float)v;
    }
}

// Four columns per lane, 256 per workgroup; its four wavefronts take the range's tokens in turn.  Rows of padding have d_logits of 0
// and are left out, whatever x holds there.
template <int EMAX, typename OUT>
__global__ __launch_bounds__(256) void gate_dx_dw_kernel(GateGradArgs a, int per_split, float* __restrict__ dw) {
    __shared__ float wave_sums[2][EMAX][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), E = a.E;
    const int col = (blockIdx.x * 64 + lane) * 4;
    const bool in = col < a.d;                           // (d is a multiple of 64: a lane has all four or none)
    float4_t acc[EMAX], w[EMAX];
#pragma unroll
    for (int e = 0; e < EMAX; ++e) {
        acc[e] = w[e] = float4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (a.d_x && in && e < E) {
            const half4_t h = *(const half4_t*)(a.wg + (size_t)e * a.d + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[e][i] = (float)h[i];
        }
    }
    const long long t0 = (long long)blockIdx.y * per_split, t1 = t0 + per_split < a.T ? t0 + per_split : a.T;
    for (long long t = t0 + wave; t < t1; t += 4) {
        const bool counts = !a.valid || a.valid[t];
        half4_t h = {};
        if (in && a.d_w && counts) h = *(const half4_anywhere_t*)(a.x + (size_t)t * a.d + col);
        float4_t dx = {0.0f, 0.0f, 0.0f, 0.0f};
        if (counts)
#pragma unroll
            for (int e = 0; e < EMAX; ++e) {
                if (e >= E) break;
                const float g = a.d_logits[(size_t)t * E + e];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[e][i] = fmaf(g, (float)h[i], acc[e][i]);
                    dx[i] = fmaf(g, w[e][i], dx[i]);
                }
            }
        if (a.d_x && in) {
            OUT* const o = (OUT*)a.d_x + (size_t)t * a.d + col;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = (OUT)dx[i];
        }
    }
    if (!a.d_w) return;
    // wavefronts 2 and 3 add to 0 and 1, 1 to 0
    for (int half = 2; half >= 1; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half)
#pragma unroll
            for (int e = 0; e < EMAX; ++e) *(float4_t*)&wave_sums[wave - half][e][lane * 4] = acc[e];
        __syncthreads();
        if (wave < half)
#pragma unroll
            for (int e = 0; e < EMAX; ++e) acc[e] += *(const float4_t*)&wave_sums[wave][e][lane * 4];
    }
    if (wave == 0 && in) {
        float* const o = dw + (size_t)blockIdx.y * E * a.d + col;
#pragma unroll
        for (int e = 0; e < EMAX; ++e)
            if (e < E) *(float4_t*)(o + (size_t)e * a.d) = acc[e];
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

int token_blocks(int T, int E) {
    const int lanes = E <= 4 ? 1 : E <= 8 ? 2 : E <= 16 ? 4 : 8, per = 64 / lanes * kLossWaves;
    const int blocks = (T - 1) / per + 1;
    return blocks < kGateBlocks ? blocks : kGateBlocks;
}

}  // namespace

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* valid, int T, int E, int k, int32_t* counts,
                         float* mean_prob, float* loss, const GateWorkspace& w, hipStream_t st) {
    const int blocks = token_blocks(T, E);
    launch_zero_words(w.status, 1, st);
    by_lanes(E, [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        if (wide_rows(logits, E))
            balance_sums_kernel<LANES, true><<<blocks, 64 * kLossWaves, 0, st>>>(logits, idx, valid, T, E, k, w.sums, w.counts, w.status);
        else
            balance_sums_kernel<LANES, false><<<blocks, 64 * kLossWaves, 0, st>>>(logits, idx, valid, T, E, k, w.sums, w.counts, w.status);
    });
    balance_finish_kernel<<<1, 1024, 0, st>>>(w.sums, w.counts, blocks, E, k, counts, mean_prob, loss);
}

int gate_dw_splits(int T, int d, int E) {
    const int by_work = (T + 63) / 64, by_chip = 1024 / ((d + 255) / 256) + 1;
    const int s = by_work < by_chip ? by_work : by_chip;
    return s < 1 ? 1 : s;
}

void launch_route_backward(const GateGradArgs& a, const GateWorkspace& w, hipStream_t st) {
    const int blocks = token_blocks(a.T, a.E);
    launch_zero_words(w.status, 1, st);
    by_lanes(a.E, [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        if (wide_rows(a.logits, a.E) && wide_rows(a.d_logits, a.E))
            gate_dlogits_kernel<LANES, true><<<blocks, 64 * kLossWaves, 0, st>>>(a, w.sums, w.status);
        else
            gate_dlogits_kernel<LANES, false><<<blocks, 64 * kLossWaves, 0, st>>>(a, w.sums, w.status);
    });
    if (a.d_bias) gate_dbias_kernel<<<1, 1024, 0, st>>>(w.sums, blocks, a.E, a.d_bias);
    if (!a.d_x && !a.d_w) return;
    const int splits = w.dw_splits, per_split = (a.T - 1) / splits + 1;
    float* const dw = splits > 1 ? w.dw : a.d_w;
    const dim3 grid((a.d + 255) / 256, splits);
    const auto go = [&](auto most) {
        constexpr int EMAX = decltype(most)::value;
        if (a.d_x_half) gate_dx_dw_kernel<EMAX, half_t><<<grid, 256, 0, st>>>(a, per_split, dw);
        else gate_dx_dw_kernel<EMAX, float><<<grid, 256, 0, st>>>(a, per_split, dw);
    };
    if (a.E <= 8) go(std::integral_constant<int, 8>{});
    else if (a.E <= 16) go(std::integral_constant<int, 16>{});
    else go(std::integral_constant<int, 32>{});
    const size_t n = (size_t)a.E * a.d;
    if (a.d_w && splits > 1) launch_reduce_splits(w.dw, splits, n, n, a.d_w, st);
}

}  // namespace moemix
