// The balance loss of the gate and the gate's backward pass: arguments and workspace of their launches.
#pragma once

#include "common.hpp"

namespace moemix {

// Workspace, computed identically by moe_gate_workspace_bytes and the entry points.
constexpr int kGateBlocks = 512;       // most workgroups that leave partial sums over tokens
struct GateWorkspace {
    int32_t* status;    // [64] first word is the status word
    float* sums;        // [kGateBlocks][E]  partial sums over tokens: probabilities, or d_logits
    int32_t* counts;    // [kGateBlocks][E + 2]  pairs per expert, valid tokens, and whether an index was out of range
    float* dl;          // [T, E]  d_logits where the caller does not ask for them
    float* dw;          // [dw_splits][E, d]  partial d_w_gate
    int dw_splits;
    size_t bytes;
};

int gate_dw_splits(int T, int d, int E);

inline GateWorkspace carve_gate_workspace(void* base, int T, int d, int E) {
    GateWorkspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) {
        char* p = base ? (char*)base + off : nullptr;
        off += align_up(bytes, 256);
        return (void*)p;
    };
    w.status = (int32_t*)take(64 * sizeof(int32_t));
    w.sums = (float*)take((size_t)kGateBlocks * E * sizeof(float));
    w.counts = (int32_t*)take((size_t)kGateBlocks * (E + 2) * sizeof(int32_t));
    w.dl = (float*)take((size_t)T * E * sizeof(float));
    w.dw_splits = gate_dw_splits(T, d, E);
    w.dw = (float*)take(w.dw_splits > 1 ? (size_t)w.dw_splits * E * d * sizeof(float) : 0);
    w.bytes = off;
    return w;
}

void launch_balance_loss(const float* logits, const int32_t* idx, const uint8_t* valid, int T, int E, int k, int32_t* counts,
                         float* mean_prob, float* loss, const GateWorkspace& w, hipStream_t st);

struct GateGradArgs {
    const half_t* x;            // [T, d]
    const half_t* wg;           // [E, d]
    const float* logits;        // [T, E]
    const int32_t* idx;         // [T, k]
    const uint8_t* valid;       // [T] or null
    const int32_t* counts;      // [E + 1], with d_loss
    const float* d_gate;        // [T, k] or null
    const float* d_loss;        // [1] or null
    float* d_logits;            // [T, E]  (the caller's or the workspace's)
    void* d_x;                  // [T, d] or null
    float* d_w;                 // [E, d] or null
    float* d_bias;              // [E] or null
    int T, d, E, k;
    bool d_x_half;
};
void launch_route_backward(const GateGradArgs& a, const GateWorkspace& w, hipStream_t st);

}  // namespace moemix
