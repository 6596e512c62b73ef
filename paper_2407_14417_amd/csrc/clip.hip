// Global norm over many gradients, and clipping.
//
//   norm = unscale sqrt(sum over all elements of v^2),  c = unscale min(1, max_norm / (norm + 1e-6)),  out = c v
//
// A list of up to 65536 elements (kClipAloneSize) is done by one workgroup.  Else two launches for each 96 tensors: sums of squares, one per workgroup, then the product, before which every
// workgroup adds the sums of all launches in the same order: up to 2048 of a launch, 16 KB from L2, and so 176 KB for 1024 tensors, whose eleven launches each do it again (96, 400, 1024 tensors
// of 2^20 elements, fp32, in place: 220, 960, 2657 us, 5.5, 5.2, 4.9 TB/s over three passes).  Sums are held in 64 bits: squares of fp32 gradients leave the range of 32, and billions of them their precision; two
// 64-bit instructions per element are a twentieth of what the vector units do in the time that its load takes.
// Bound: every gradient is read twice, since the norm has to be known before the first is scaled (24 tensors of 4096 x 14336 in fp32: 16.9 GB in 3110 us, 5.4 TB/s; 48 of
// 2048 x 1408 from fp16 to fp32: 1.11 GB in 208 us).  Results are stored past the caches: with ordinary stores the last of these took 257 us, of which 27 for this.
#include "clip.hpp"
#include "kernels.hpp"

namespace moemix {

namespace {

// The tensor that chunk c lies in.
__device__ __forceinline__ int tensor_of(const ClipTable& t, uint32_t c) {
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= c) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Sum of one value of each thread, the same in all of them.
template <int THREADS>
__device__ __forceinline__ double block_total(double v) {
    __shared__ double lds[THREADS / 64];
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, kWave);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = lds[0];
#pragma unroll
    for (int i = 1; i < THREADS / 64; ++i) sum += lds[i];
    return sum;
}

// What a group of 256 threads does with a chunk: f(i) for 16 bytes of values from element i on, f1(i) for single ones at the end; everything with f1 where the tensor is not
// on a 16-byte boundary.
template <int W, typename F, typename F1>
__device__ __forceinline__ void each(bool wide, unsigned long long begin, unsigned long long end, F f, F1 f1) {
    const int tid = threadIdx.x & 255;
    unsigned long long at = begin;
    if (wide) {
        const unsigned long long whole = begin + (end - begin) / W * W;
        if (end - begin == kClipChunk) {
#pragma unroll 4
            for (int i = 0; i < kClipChunk / (256 * W); ++i) f(begin + (unsigned long long)(i * 256 + tid) * W);
        } else {
            for (unsigned long long i = begin + tid * W; i < whole; i += 256 * W) f(i);
        }
        at = whole;
    }
    for (unsigned long long i = at + tid; i < end; i += 256) f1(i);
}

// PAST: past the caches.
template <bool PAST, typename V>
__device__ __forceinline__ V load(const V* p) {
    return PAST ? __builtin_nontemporal_load(p) : *p;
}

template <bool PAST, typename IN>
__device__ __forceinline__ double chunk_sum(const IN* g, unsigned long long begin, unsigned long long end) {
    constexpr int W = 16 / sizeof(IN);
    typedef IN wide_t __attribute__((ext_vector_type(W)));
    double sum[2] = {0.0, 0.0};
    each<W>((uintptr_t)g % 16 == 0, begin, end,
             [&](unsigned long long i) {
                 const wide_t v = load<PAST>((const wide_t*)(g + i));
#pragma unroll
                 for (int k = 0; k < W; ++k) sum[k & 1] = fma((double)v[k], (double)v[k], sum[k & 1]);
             },
             [&](unsigned long long i) { sum[0] = fma((double)g[i], (double)g[i], sum[0]); });
    return sum[0] + sum[1];
}

// The factor as first * second: first is 1, or where 32 bits hold the factor with less than their precision a power of two near its root.  (Then v * first is exact, or the product is below
// what 32 bits hold.)
struct Factor {
    float first, second;
};
__device__ __forceinline__ Factor factor_of(double c) {
    const int half = c > 0.0 && c < 0x1p-100 ? ilogb(c) / 2 : 0;
    return Factor{(float)ldexp(1.0, half), (float)ldexp(c, -half)};
}

template <bool PAST, typename IN, typename OUT>
__device__ __forceinline__ void chunk_scale(const IN* g, OUT* o, Factor c, unsigned long long begin, unsigned long long end) {
    constexpr int W = 16 / (sizeof(IN) > sizeof(OUT) ? sizeof(IN) : sizeof(OUT));     // (eight values from fp16 to fp32: pieces of lines, 1.1 GB 967 -> 808 us)
    typedef IN wide_t __attribute__((ext_vector_type(W)));
    typedef OUT wide_out_t __attribute__((ext_vector_type(W)));
    each<W>(((uintptr_t)g % sizeof(wide_t) | (uintptr_t)o % sizeof(wide_out_t)) == 0, begin, end,
             [&](unsigned long long i) {
                 const wide_t v = load<PAST>((const wide_t*)(g + i));
                 wide_out_t w;
#pragma unroll
                 for (int k = 0; k < W; ++k) w[k] = (OUT)((float)v[k] * c.first * c.second);
                 __builtin_nontemporal_store(w, (wide_out_t*)(o + i));
             },
             [&](unsigned long long i) { o[i] = (OUT)((float)g[i] * c.first * c.second); });
}

// Workgroups have GROUPS groups of 256 threads; group i of all takes chunks i, i + n ..
template <int GROUPS>
__device__ __forceinline__ uint32_t first_chunk() {
    return GROUPS == 1 ? blockIdx.x : blockIdx.x * GROUPS + __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
}

// Sum of squares of the workgroup's chunks.
template <int GROUPS, bool PAST>
__device__ __forceinline__ double sum_of_chunks(const ClipTable& t) {
    double sum = 0.0;
    for (uint32_t c = first_chunk<GROUPS>(); c < t.first[t.n]; c += gridDim.x * GROUPS) {
        const int i = tensor_of(t, c);
        const unsigned long long n = t.size[i] & kClipSize, begin = (unsigned long long)(c - t.first[i]) * kClipChunk;
        const unsigned long long end = n - begin < kClipChunk ? n : begin + kClipChunk;
        if (t.size[i] & kClipGradHalf) sum += chunk_sum<PAST>((const half_t*)t.grad[i], begin, end);
        else sum += chunk_sum<PAST>((const float*)t.grad[i], begin, end);
    }
    return block_total<256 * GROUPS>(sum);
}

// total: the sum of all squares.
template <int GROUPS, bool PAST>
__device__ __forceinline__ void scale_chunks(const ClipTable& t, double total, float max_norm, float unscale, float* __restrict__ norm_out) {
    const double norm = sqrt(total) * (double)unscale;
    const float rounded = (float)norm;
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = rounded;
    if (!isfinite(rounded)) return;
    const double ratio = (double)max_norm / (norm + 1e-6);
    const Factor c = factor_of((double)unscale * (ratio < 1.0 ? ratio : 1.0));
    for (uint32_t b = first_chunk<GROUPS>(); b < t.first[t.n]; b += gridDim.x * GROUPS) {
        const int i = tensor_of(t, b);
        if (c.first == 1.0f && c.second == 1.0f && t.grad[i] == t.out[i]) continue;
        const unsigned long long n = t.size[i] & kClipSize, begin = (unsigned long long)(b - t.first[i]) * kClipChunk;
        const unsigned long long end = n - begin < kClipChunk ? n : begin + kClipChunk;
        const bool from16 = t.size[i] & kClipGradHalf, to16 = t.size[i] & kClipOutHalf;
        if (from16 && to16) chunk_scale<PAST>((const half_t*)t.grad[i], (half_t*)t.out[i], c, begin, end);
        else if (from16) chunk_scale<PAST>((const half_t*)t.grad[i], (float*)t.out[i], c, begin, end);
        else if (to16) chunk_scale<PAST>((const float*)t.grad[i], (half_t*)t.out[i], c, begin, end);
        else chunk_scale<PAST>((const float*)t.grad[i], (float*)t.out[i], c, begin, end);
    }
}

template <bool PAST>
__global__ __launch_bounds__(256) void clip_sums_kernel(ClipTable t, double* __restrict__ part) {
    const double sum = sum_of_chunks<1, PAST>(t);
    if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

template <bool PAST>
__global__ __launch_bounds__(256) void clip_scale_kernel(ClipTable t, const double* __restrict__ part, int n_part, float max_norm, float unscale,
                                                         float* __restrict__ norm_out) {
    double sum = 0.0;
    for (int i = threadIdx.x; i < n_part; i += 256) sum += part[i];
    scale_chunks<1, PAST>(t, block_total<256>(sum), max_norm, unscale, norm_out);
}

// One workgroup does it all.
__global__ __launch_bounds__(1024) void clip_alone_kernel(ClipTable t, float max_norm, float unscale, float* __restrict__ norm_out) {
    scale_chunks<4, false>(t, sum_of_chunks<4, false>(t), max_norm, unscale, norm_out);
}

}  // namespace

void launch_clip_sums(const ClipTable& t, bool past_caches, double* part, hipStream_t st) {
    const auto kernel = past_caches ? clip_sums_kernel<true> : clip_sums_kernel<false>;
    if (clip_blocks(t)) kernel<<<clip_blocks(t), 256, 0, st>>>(t, part);
}

void launch_clip_scale(const ClipTable& t, bool past_caches, const double* part, int n_part, float max_norm, float unscale, float* norm, hipStream_t st) {
    const auto kernel = past_caches ? clip_scale_kernel<true> : clip_scale_kernel<false>;
    if (clip_blocks(t) || norm) kernel<<<clip_blocks(t) ? clip_blocks(t) : 1, 256, 0, st>>>(t, part, n_part, max_norm, unscale, norm);
}

void launch_clip_alone(const ClipTable& t, float max_norm, float unscale, float* norm, hipStream_t st) {
    clip_alone_kernel<<<1, 1024, 0, st>>>(t, max_norm, unscale, norm);
}

}  // namespace moemix
