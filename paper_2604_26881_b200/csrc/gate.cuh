// Arguments of the gating-rule kernel (gate.cu).
#pragma once

#include "internal.h"

namespace faasmoe {

struct GateArgs {
    const void* logits;             // f32 or bf16 [T, ld]
    int bf16_logits;
    int64_t ld;
    int T, E, k;
    int score, n_groups, keep, group_score, renormalize;
    float scale;
    const float* bias;              // f32 [M, E] or null
    const int32_t* tenant_id;       // [T] or null: every token uses model 0
    const int32_t* model_of_tenant; // [n_tenants] or null: every tenant uses model 0
    int n_tenants, M;
    int32_t* topk_idx;
    float* topk_w;
    uint8_t* tie_flag;              // or null
    int32_t* status;                // or null
    // set by launch_gate
    int group_size, lanes_per_group, eligible, vec, vec_bias;
};

void apply_gating(GateArgs& args, const moe_gating& rule);
cudaError_t launch_gate(const GateArgs& args, cudaStream_t st);

}  // namespace faasmoe
