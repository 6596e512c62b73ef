// Training of the 16-bit experts: arguments and launchers (experts_train.hip), the workspace of its calls.
#pragma once

#include "common.hpp"

namespace moemix {

constexpr int kTrainStep = 64;          // contraction elements per stage
constexpr int kTrainCols = 256;         // columns of a tile
constexpr int kTrainRows = 256;         // most rows of a tile, of a chunk

// What the first launch of a call finds out about the grouping, whatever offsets and perm hold.
// Chunk i is rows [begin, min(begin + size, end)) of the grouped rows; up to eight chunks of an expert go side by side: i is number `at` of `abreast`.
struct TrainChunk {
    int32_t expert, begin, end;
    int32_t form;                          // size / 32 + 16 at + 256 abreast
};
// An expert's chunks are as even as 32s of rows allow; the experts with the longest come first.  Those from `first_split` on share their contraction among `splits` workgroups each.
struct TrainSplit {
    int32_t first_split, splits;
};
struct TrainMeta {
    int32_t lo, hi;                        // grouped rows [lo, hi) belong to an expert
    int32_t n_chunks;
    TrainSplit whole, down, d_rows;        // of the launches that cannot be split, of down and of d_rows
    int32_t offsets[MOE_MAX_EXPERTS + 1];  // increasing, within [0, P]
    int32_t order[MOE_MAX_EXPERTS];        // experts, the one with most rows first
};

constexpr int kTrainMostSplits = 16;

struct TrainWorkspace {
    TrainMeta* meta;
    TrainChunk* chunks;   // [E + P / 32]
    int32_t* tok;         // [P + 64]  grouped row -> token (0 for a row of no expert and past the end)
    float* gate;          // [P + 64]  grouped row -> its gate
    int32_t* inv;         // [P]       pair -> grouped row; anything for a pair in no group
    int32_t* shares;      // [P]       grouped row -> workgroups that share its contraction: down's, 256 times d_rows'
    half_t* h;            // [P + 64, f]  hidden rows; backward: times the gate (d_weights reads whole steps of 64 rows)
    half_t* d_a;          // [P + 64, f]
    half_t* d_u;          // [P + 64, f]
    float* part;          // [P][f / 64]  shares of d_gate
    float* y;             // [splits][P, d]  rows of the down-projection; backward: of d_x
    int splits;           // most of a chunk
    int most_rows;        // of a chunk: 32 .. 256
    size_t bytes;
};

inline TrainWorkspace carve_train_workspace(void* base, int T, int d, int f, int E, int k, int splits) {
    TrainWorkspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? (char*)base + off : nullptr;
        off += align_up(bytes, 256);
        return (void*)p;
    };
    const size_t P = (size_t)T * k;
    w.meta = (TrainMeta*)take(sizeof(TrainMeta));
    w.chunks = (TrainChunk*)take((E + P / 32) * sizeof(TrainChunk));
    w.tok = (int32_t*)take((P + kTrainStep) * sizeof(int32_t));
    w.gate = (float*)take((P + kTrainStep) * sizeof(float));
    w.inv = (int32_t*)take(P * sizeof(int32_t));
    w.shares = (int32_t*)take(P * sizeof(int32_t));
    w.h = (half_t*)take((P + kTrainStep) * f * sizeof(half_t));
    w.d_a = (half_t*)take((P + kTrainStep) * f * sizeof(half_t));
    w.d_u = (half_t*)take((P + kTrainStep) * f * sizeof(half_t));
    w.part = (float*)take(P * (f / 64) * sizeof(float));
    w.y = (float*)take((size_t)splits * P * d * sizeof(float));
    w.splits = splits;
    w.bytes = off;
    return w;
}

// offsets null: all P rows belong to expert 0; perm null: row r is pair r; topk_gate null: all gates are 1.
struct TrainGrouping {
    const int32_t* offsets;
    const int32_t* perm;
    const float* topk_gate;
    int T, k, E;
};

// Products of grouped rows with their expert's matrices.
struct TrainRows {
    const half_t* w[MOE_MAX_EXPERTS];
    const half_t* w3[MOE_MAX_EXPERTS];
    const half_t* in;          // [T, K] by tok, or [P, K]
    const half_t* in2;         // d_x: the second half of the contraction
    half_t* a;                 // [P, f] (d_hidden: read)
    half_t* u;
    half_t* h;
    half_t* d_a;
    half_t* d_u;
    float* y;
    float* part;
    const TrainMeta* meta;
    const TrainChunk* chunks;
    const int32_t* tok;
    const float* gate;
    int N, K, P, E;
    int most_rows;             // of a chunk
};

// Gradients of the matrices: for expert e  w1 = d_a^T x, w3 = d_u^T x, w2 = d_out^T h.  Null: not asked for.
struct TrainWeights {
    void* w1[MOE_MAX_EXPERTS];
    void* w3[MOE_MAX_EXPERTS];
    void* w2[MOE_MAX_EXPERTS];
    const half_t* x;           // [T, d]
    const half_t* d_out;       // [T, d]
    const half_t* h;           // [P, f], times the gate
    const half_t* d_a;
    const half_t* d_u;
    const TrainMeta* meta;
    const int32_t* tok;
    int d, f, E;
    int accumulate;
};

// Most workgroups that share a chunk's contraction in down and d_rows: partial results cost room, and pay where a launch has few rounds of workgroups.
int train_most_splits(int P, int d);

// Most rows of a chunk, where the widest launch has tiles_f or tiles_d tiles of columns.
int train_most_rows(int P, int E, int d, int f, int tiles_f, int tiles_d);

// Are the gradients of the matrices made of small tiles (train_weights_few_kernel)?
bool train_small_tiles(int P, int E, int d, int f);

void launch_train_group(const TrainGrouping& g, const TrainWorkspace& w, int d, int f, hipStream_t st);
// a = W1 x, u = W3 x, h = silu(a) u
void launch_train_up(const TrainRows& a, hipStream_t st);
// y = W2 h
void launch_train_down(const TrainRows& a, hipStream_t st);
// q = W2^T d_out; shares of d_gate, d_a, d_u, gate * h
void launch_train_d_hidden(const TrainRows& a, hipStream_t st);
// y = W1^T d_a + W3^T d_u
void launch_train_d_rows(const TrainRows& a, hipStream_t st);
void launch_train_d_weights(const TrainWeights& a, int P, bool half_out, hipStream_t st);
// out[t,:] = sum over the token's pairs in a group of (forward: topk_gate *) the sum of the shares of y; d_gate [T, k] (or null) from n_part shares of each.
void launch_train_gather(const TrainGrouping& g, const TrainWorkspace& w, bool forward, int d, void* out, bool half_out, float* d_gate,
                         int n_part, hipStream_t st);

}  // namespace moemix
