// Arguments of the projection in 8-bit integers (project_i8.cu).
#pragma once

#include "internal.h"

namespace faasmoe {

constexpr int kI8MaxK = 131071;         // (|q| <= 128: sums of K products fit 32 bits)

struct I8Args {
    const int8_t* x;           // [T, K]
    const int8_t* w;           // [N, K]
    const float* x_scale;
    const float* w_scale;
    const float* bias;         // [N] or null
    const void* base;          // [T, N] or null
    void* out;
    int64_t ldx, ldw, ldbase, ldo;
    int T, K, N, out_f32;
    int32_t* status;           // the caller's, or null
    // set by launch_project_i8
    int ksteps;                // slices of 128 bytes of K
    int splits;                // few tokens: CTAs of a cluster that share K
    int nt;                    // few tokens: tokens of a tile
    int kb;                    // few tokens: slices of a stage
    int columns;               // few tokens: TMEM columns
    int n_stages;
    int scratch;               // few tokens: offset of the received sums behind the ring
};

cudaError_t launch_project_i8(const I8Args& args, cudaStream_t st);
// the status bits of the calls that had no word for them, read and cleared (the device is idle)
cudaError_t take_project_i8_status(int32_t* status_host);

}  // namespace faasmoe
