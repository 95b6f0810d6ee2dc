// The residual's addition, the RMSNorm behind it and an 8-bit output with scales, in one pass over the rows:
//
//   h = bf16(x + residual)                   (h = x without a residual; stored to residual_out)
//   y = h * (1 / sqrt(mean(h^2) + eps)) * weight      (fp32)
//   out = bf16(y);   q = e4m3(y / s),  s = max |y| / 448 over the row or over each 128 columns
//
// Bound by HBM: every element is read and written once, kept in registers in between (W warps hold a row, up to four
// 16-byte vectors a lane), so the only other cost is the latency of one or two reductions per row.  The sum of
// squares, the scales and the quotients are fp32; h is rounded once because it is the residual stream that the caller
// keeps (the norm is that of the stored value), out and q are each one rounding of the same fp32 y.
#include <cuda_fp8.h>

#include "addnorm.cuh"

namespace faasmoe {

namespace {

constexpr uint32_t kFull = 0xffffffffu;

// max |y| that keeps a NaN, as the row's outputs do
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// eight consecutive elements of a row, of which the first n are there
__device__ __forceinline__ void load8(const bf16* p, int n, bool vec, float* f)
{
    if (vec) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 t = __bfloat1622float2(h[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < n ? __bfloat162float(p[i]) : 0.f;
    }
}
__device__ __forceinline__ void store8(bf16* p, int n, bool vec, const float* f)
{
    if (vec) {
        uint4 v;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        *reinterpret_cast<uint4*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(f[i]);
    }
}
__device__ __forceinline__ uint16_t e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// R rows per block, W warps per row, V vectors of 8 elements per lane
template <int V, bool QUANT>
__global__ void __launch_bounds__(512)
addnorm_kernel(const AddNormArgs p, int W)
{
    __shared__ float s_part[2][16];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row_in_block = warp / W, wr = warp - row_in_block * W;
    const int t = blockIdx.x * (blockDim.x / (32 * W)) + row_in_block;
    const bool live = t < p.T;
    float h[V][8];
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = ((v * W + wr) * 32 + lane) * 8, n = p.H - col;
        if (live && n > 0) {
            load8(p.x + (size_t)t * p.ldx + col, n, p.vec && n >= 8, h[v]);
            if (p.residual) {
                float r[8];
                load8(p.residual + (size_t)t * p.ldr + col, n, p.vec && n >= 8, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] = __bfloat162float(__float2bfloat16_rn(h[v][i] + r[i]));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] = 0.f;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = ((v * W + wr) * 32 + lane) * 8, n = p.H - col;
        if (p.residual_out && live && n > 0) store8(p.residual_out + (size_t)t * p.ldro + col, n, p.vec && n >= 8, h[v]);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(kFull, ss, o);
    if (W > 1) {
        if (lane == 0) s_part[0][warp] = ss;
        __syncthreads();
        ss = 0.f;
        for (int i = 0; i < W; ++i) ss += s_part[0][row_in_block * W + i];
    }
    const float r = 1.f / sqrtf(ss / (float)p.H + p.eps);
    float top = 0.f;                        // max |y| of this lane's elements (row scales)
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = ((v * W + wr) * 32 + lane) * 8, n = p.H - col;
        if (n > 0) {
            float g[8];
            load8(p.weight + col, n, p.vec_weight && n >= 8, g);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r * g[i];
            if (live && p.out) store8(p.out + (size_t)t * p.ldo + col, n, p.vec && n >= 8, h[v]);
        }
        if (QUANT && p.group == 0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < n) top = max_nan(top, fabsf(h[v][i]));
        }
    }
    if (!QUANT) return;
    float scale = 0.f;
    if (p.group == 0) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = max_nan(top, __shfl_xor_sync(kFull, top, o));
        if (W > 1) {
            if (lane == 0) s_part[1][warp] = top;
            __syncthreads();
            top = 0.f;
            for (int i = 0; i < W; ++i) top = max_nan(top, s_part[1][row_in_block * W + i]);
        }
        scale = top / 448.f;
        if (live && wr == 0 && lane == 0) p.q_scale[t] = scale;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int vec_id = (v * W + wr) * 32 + lane, col = vec_id * 8, n = p.H - col;
        if (p.group != 0) {
            // sixteen lanes hold 128 columns
            float a = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < n) a = max_nan(a, fabsf(h[v][i]));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) a = max_nan(a, __shfl_xor_sync(kFull, a, o));
            scale = a / 448.f;
            if (live && n > 0 && (lane & 15) == 0) p.q_scale[(size_t)t * p.n_groups + (vec_id >> 4)] = scale;
        }
        if (!live || n <= 0) continue;
        // (the reciprocal of a scale below 2^-126 is not a number to multiply with)
        const bool tiny = scale < 1e-37f;
        const float inv = tiny ? 0.f : 1.f / scale;
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = tiny ? (scale > 0.f ? h[v][i] / scale : 0.f) : h[v][i] * inv;
        uint8_t* dst = p.q + (size_t)t * p.ldq + col;
        if (p.vec_q && n >= 8) {
            uint2 o;
            o.x = e4m3x2(y[0], y[1]) | ((uint32_t)e4m3x2(y[2], y[3]) << 16);
            o.y = e4m3x2(y[4], y[5]) | ((uint32_t)e4m3x2(y[6], y[7]) << 16);
            *reinterpret_cast<uint2*>(dst) = o;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < n) dst[i] = (uint8_t)(e4m3x2(y[i], 0.f) & 0xff);
        }
    }
}

template <int V>
cudaError_t launch_v(const AddNormArgs& p, int W, int rows, cudaStream_t st)
{
    const dim3 grid((p.T + rows - 1) / rows), block(32 * W * rows);
    return p.q ? launch_pdl(addnorm_kernel<V, true>, grid, block, 0, st, p, W)
               : launch_pdl(addnorm_kernel<V, false>, grid, block, 0, st, p, W);
}

}  // namespace

cudaError_t launch_addnorm(const AddNormArgs& in, cudaStream_t st)
{
    AddNormArgs p = in;
    auto al = [](const void* q, size_t n) { return (uintptr_t)q % n == 0; };
    p.vec = al(p.x, 16) && p.ldx % 8 == 0 && al(p.residual, 16) && p.ldr % 8 == 0 && al(p.residual_out, 16) && p.ldro % 8 == 0 &&
            al(p.out, 16) && p.ldo % 8 == 0;
    p.vec_weight = al(p.weight, 16);
    p.vec_q = al(p.q, 8) && p.ldq % 8 == 0;
    const int vecs = (p.H + 7) / 8;
    const int V = vecs <= 32 ? 1 : (vecs <= 512 ? 2 : 4);
    int W = (vecs + 32 * V - 1) / (32 * V);
    const int rows = W >= 4 ? 1 : 4 / W;
    if (V == 1) return launch_v<1>(p, W, rows, st);
    if (V == 2) return launch_v<2>(p, W, rows, st);
    return launch_v<4>(p, W, rows, st);
}

}  // namespace faasmoe
