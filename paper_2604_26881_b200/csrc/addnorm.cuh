// Arguments of the residual-add / RMSNorm / 8-bit output kernel (addnorm.cu).
#pragma once

#include "internal.h"

namespace faasmoe {

constexpr int kAddNormMaxH = 16384;      // 16 warps x 32 lanes x 4 vectors of 8 elements

struct AddNormArgs {
    const bf16* x;
    const bf16* residual;      // or null
    bf16* residual_out;        // or null; may be residual or x themselves
    const bf16* weight;
    bf16* out;                 // or null; may be x itself
    uint8_t* q;                // e4m3, or null
    float* q_scale;
    int64_t ldx, ldr, ldro, ldo, ldq;
    int group;                 // 0: one scale per row, 128: one per 128 columns
    int n_groups;              // scales per row
    int T, H;
    float eps;
    // set by launch_addnorm
    int vec, vec_weight, vec_q;
};

cudaError_t launch_addnorm(const AddNormArgs& args, cudaStream_t st);

}  // namespace faasmoe
