// Global norm over many gradients, and clipping (clip.hip).
#pragma once

#include "common.hpp"

namespace moemix {

constexpr int kClipMost = 96;                  // tensors of one launch: their table travels as a kernel argument (2.8 KB)
constexpr int kClipChunk = 16384;              // elements that a workgroup takes at a time
// Lists of up to so many chunks and elements are one workgroup's (two launches, one: 32776 elements 10.2, 7.4 us; 65428, 11.1, 9.4; 98196, 11.3, 14.4; 9 tensors of 300, 10.2,
// 7.1; 17 of them, 10.3, 11.6).
constexpr uint32_t kClipAloneChunks = 12;
constexpr unsigned long long kClipAloneSize = 65536;
// Gradients of more bytes than the last-level cache holds are read past the caches, so that none of them drives out what could be read again (both ways: 201 MB, fp32 103, 110 us; 277 MB,
// fp16 to fp32 219, 208; 335 MB, fp32 179, 182; 470 MB 263, 252; 5.6 GB 3260, 3110).
constexpr unsigned long long kClipCached = 256ull << 20;
constexpr int kClipBlocks = 2048;              // most workgroups of a launch, eight per compute unit

struct ClipTable {
    const void* grad[kClipMost];
    void* out[kClipMost];
    unsigned long long size[kClipMost];        // elements; bit 62: the gradient is fp16, bit 63: out is
    uint32_t first[kClipMost + 1];             // chunks of the tensors before
    int n;
};
constexpr unsigned long long kClipGradHalf = 1ull << 62, kClipOutHalf = 1ull << 63, kClipSize = kClipGradHalf - 1;

inline int clip_blocks(const ClipTable& t) { return t.first[t.n] < kClipBlocks ? (int)t.first[t.n] : kClipBlocks; }

// part[0 .. clip_blocks(t)) = sums of squares
void launch_clip_sums(const ClipTable& t, bool past_caches, double* part, hipStream_t st);
// From n_part sums: norm (written if norm != null), and out = c * grad unless the norm is not finite.
void launch_clip_scale(const ClipTable& t, bool past_caches, const double* part, int n_part, float max_norm, float unscale, float* norm, hipStream_t st);
// Both for a table of all tensors.
void launch_clip_alone(const ClipTable& t, float max_norm, float unscale, float* norm, hipStream_t st);

}  // namespace moemix
