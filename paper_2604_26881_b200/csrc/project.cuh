// Arguments of the shared projection with low-rank adapters (project.cu).
#pragma once

#include "internal.h"

namespace faasmoe {

constexpr int kAdapterMaxRank = 128;

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
    float* u;                       // workspace: [T][rank], f32 or three bf16 arrays; not used where the first product is fused
    int32_t* status;                // the caller's, or null
    // set by launch_project
    int u_split;                    // u is stored as three bf16 terms, not as f32
    int u_splits;                   // parts of K of the first product (a cluster)
    int ksteps, splits, n_stages, stage_bytes, a_bytes, a_rows;
    int u_own;                      // tokens of a tile that one CTA of such a cluster adds up
    int kb, lanes;                  // first product: slices of 64 per stage, lanes that issue MMAs
    int u_rows;                     // most rows of A that the tokens may need (fused)
    int scratch;                    // bytes of the ring (or of the sums put together in it) in front of the sums received
    int sums_bytes;                 // of the sums received
    int slots;                      // adapters per CTA of the first product
};

// bytes of the workspace (0: none is needed)
int64_t project_workspace(int T, int K, int N, int rank, int n_adapters);
cudaError_t launch_project(const ProjectArgs& args, cudaStream_t st);
// the status bits of the calls that had no word for them, read and cleared (waits for the device)
cudaError_t take_project_status(int32_t* status_host);

}  // namespace faasmoe
