// Interface of the router's training operators (router.hip): load balance loss, gate backward.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "host_common.h"

namespace ec2moe {

struct BalanceArgs {
    const float* probs;
    const int32_t* topk_idx;
    const uint8_t* valid;  // or null
    float coef;
    int n_tokens, n_experts, top_k;
    int32_t* counts;       // or null
    float* loss;
    float* d_probs;        // or null
    void* ws;              // balance_ws_bytes()
};
size_t balance_ws_bytes(int n_tokens, int n_experts);
hipError_t launch_balance(const BalanceArgs& a, hipStream_t s);

struct GateBackwardArgs {
    const void* x;
    const void* w_global;
    const void* w_local;
    const float* probs;
    const int32_t* topk_idx;
    const float* d_topk_w;   // or null, as the next three
    const float* d_probs;
    const float* d_balance;
    const uint8_t* valid;
    void* d_x;               // or null
    float* d_w_global;       // both or neither of the two
    float* d_w_local;
    float* d_b_global;       // or null
    float* d_b_local;        // or null
    int n_tokens, d, n_experts, n_groups, top_k;
    bool renormalize;
    int32_t goff[161];       // group k = experts goff[k] .. goff[k + 1] - 1
    int group_size;          // of equal groups; 0: see goff
    void* ws;                // gate_backward_ws_bytes()
};
size_t gate_backward_ws_bytes(DType dt, int n_tokens, int d, int n_experts, int n_groups);
hipError_t launch_gate_backward(DType dt, const GateBackwardArgs& a, hipStream_t s);

}  // namespace ec2moe
