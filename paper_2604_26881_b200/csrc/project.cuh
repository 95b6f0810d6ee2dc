// Arguments of the shared projection with low-rank adapters (project.cu).
#pragma once

#include "internal.h"

namespace faasmoe {

constexpr int kAdapterMaxRank = 128;
constexpr int kProjectHeader = 256;       // bytes of the workspace in front of the adapters' first products

struct ProjectArgs {
    const bf16* x;                  // [T, ldx]
    const bf16* w;                  // [N, ldw] or null
    const bf16* a;                  // [n_adapters, rank, K]
    const bf16* b;                  // [n_adapters, N, rank]
    const float* scale;             // [n_adapters] or null (1)
    const int32_t* tenant_id;       // [T]
    const int32_t* adapter_of_tenant;   // [n_tenants] or null (tenant u uses adapter u)
    const void* base;               // [T, ldbase] of the output's type, or null
    void* out;                      // [T, ldo]
    int64_t ldx, ldw, ldbase, ldo;
    int out_f32;
    int T, K, N, n_adapters, rank, n_tenants;
    unsigned char* workspace;       // kProjectHeader bytes, then u [T][rank]: f32, or two bf16 arrays hi and lo
    int32_t* status;                // the caller's, or a word of the workspace
    // set by launch_project
    float* u;
    int u_pair;                     // u is stored as hi and lo
    int u_splits;                   // parts of K of the first product (a cluster)
    int ksteps, splits, n_stages, stage_bytes, a_bytes, a_rows;
    int slots;                      // adapters per CTA of the first product
};

// bytes of the workspace for T tokens (n_adapters = 0: none)
int64_t project_workspace(int T, int rank, int n_adapters);
cudaError_t launch_project(const ProjectArgs& args, cudaStream_t st);

}  // namespace faasmoe
