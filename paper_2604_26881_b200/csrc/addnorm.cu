// The residual's addition, the RMSNorm behind it and an 8-bit output with scales, in one pass over the rows:
//
//   h = bf16(x + residual)                   (h = x without a residual; stored to residual_out)
//   y = h * (1 / sqrt(mean(h^2) + eps)) * weight      (fp32)
//   out = bf16(y);   q = e4m3(y / s),  s = max |y| / 448 over the row or over each 128 columns
//
// Bound by HBM: every element is read and written once, kept in registers in between (W warps hold a row, up to four
// 16-byte vectors a lane).  16384 x 2048 with a bf16 output alone: 268 MB in 46 us, 5.9 TB/s (0.89 of the measured copy
// bandwidth); with both outputs and a scale per row 302 MB in 55 us, 5.5 TB/s (0.84), where the two roundings of every
// quotient are instructions that the loads do not hide; 4096 x 8192 with 128-column scales 58 us; 32 x 2048: 2.0 us, launch and
// latency.  The sum of squares (of the row in units of a power of two, where its squares leave the range), the scales and the
// quotients are fp32; h is rounded once because it is the residual stream that the caller keeps (the norm is that of the stored
// value), out is one rounding of the fp32 y, q one of the fp32 quotient y / s.
#include <cuda_fp8.h>
#include <float.h>

#include "addnorm.cuh"

namespace faasmoe {

namespace {

constexpr uint32_t kFull = 0xffffffffu;

// |y| as an unsigned number: of the same order, and a NaN is above everything, as it is to be in the outputs
__device__ __forceinline__ uint32_t magnitude(float y) { return __float_as_uint(y) & 0x7fffffffu; }

__device__ __forceinline__ void unpack8(const uint4& v, float* f)
{
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = __bfloat1622float2(h[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
}
__device__ __forceinline__ uint4 pack8(const float* f)
{
    uint4 v;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    return v;
}
// Eight consecutive elements of a row, of which the first n (possibly none) are there; the others read as zero.  VEC: n is
// 8 or not positive and the address is on a 16-byte boundary.
template <bool VEC>
__device__ __forceinline__ uint4 load8(const bf16* p, int n)
{
    uint4 v = make_uint4(0, 0, 0, 0);
    if (VEC) {
        if (n > 0) v = *reinterpret_cast<const uint4*>(p);
    } else {
        unsigned short e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = i < n ? reinterpret_cast<const unsigned short*>(p)[i] : (unsigned short)0;
        v = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
    }
    return v;
}
template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float* f)
{
    if (VEC) {
        if (n > 0) *reinterpret_cast<uint4*>(p) = pack8(f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(f[i]);
    }
}
__device__ __forceinline__ uint16_t e4m3x2(float a, float b)
{
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// Eight values times one factor as e4m3, element i in byte i.
__device__ __forceinline__ uint2 e4m3x8(const float* h, float by)
{
    uint2 o;
    o.x = e4m3x2(h[0] * by, h[1] * by) | ((uint32_t)e4m3x2(h[2] * by, h[3] * by) << 16);
    o.y = e4m3x2(h[4] * by, h[5] * by) | ((uint32_t)e4m3x2(h[6] * by, h[7] * by) << 16);
    return o;
}

// e4m3 of the fp32 quotients of eight values by one scale.  A product with the reciprocal is off by up to two fp32 steps, which
// is another 8-bit float next to the middle of two.  So the products with a reciprocal that is 2^-21 too small and with one that is
// as much too large, which have the quotient between them, are rounded both: where they agree that is its 8-bit float, and
// where they do not (a vector in 10^4) the quotients are taken, one after the other so that the code stays short.  (16384 x 2048:
// 53.8 us without the units below; 51.7 with one product that is not looked at again, 55.9 with eight quotients in the
// code, 11 us more than 51.7 with quotients of everything.)
template <bool VEC>
__device__ __forceinline__ void store_q(uint8_t* dst, int n, bool vec_q, const float* h, float scale)
{
    const float inv = 1.f / scale;
    uint2 o = e4m3x8(h, inv * (1.f - 0x1p-21f));
    const uint2 up = e4m3x8(h, inv * (1.f + 0x1p-21f));
    // (a scale below 1e-37 has no finite reciprocal)
    uint64_t doubt = scale < 1e-37f ? ~0ull : (uint64_t)(o.y ^ up.y) << 32 | (o.x ^ up.x);
#pragma unroll 1
    while (doubt) {                                           // (one division in the code, not eight)
        const int i = (__ffsll(doubt) - 1) >> 3;
        doubt &= ~(0xffull << (8 * i));
        float x = h[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) x = i == j ? h[j] : x;
        const uint32_t q = e4m3x2(scale != 0.f ? x / scale : 0.f, 0.f) & 0xffu, at = 8 * (i & 3);
        if (i < 4) o.x = (o.x & ~(0xffu << at)) | q << at;
        else o.y = (o.y & ~(0xffu << at)) | q << at;
    }
    if (VEC && vec_q) {
        *reinterpret_cast<uint2*>(dst) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) dst[i] = (uint8_t)((i < 4 ? o.x : o.y) >> (8 * (i & 3)) & 0xffu);
    }
}

// a barrier of the warps of one row of the block (rows of several warps: two in a block at most)
__device__ __forceinline__ void row_sync(int row, int W)
{
    if (row == 0) asm volatile("bar.sync 1, %0;" ::"r"(32 * W) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"r"(32 * W) : "memory");
}

// Mean of squares and eps of a row whose squares are beyond the range of fp32, or below it with no eps that counts beside them: of the
// row times a power of two that is exact and brings them inside (h is scaled by it, so that 1 / sqrt of what is returned is its factor).
template <int V>
__device__ __forceinline__ float mean_in_units(const AddNormArgs& p, float (&h)[V][8], float mean, int W, int warp, int lane, int row, float* sums)
{
    const float scale = mean < 1.f ? 0x1p100f : 0x1p-72f;
    float ss = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[v][i] *= scale;
            ss = fmaf(h[v][i], h[v][i], ss);
        }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(kFull, ss, o);
    if (W > 1) {
        row_sync(row, W);                                     // (everybody has read what was there)
        if (lane == 0) sums[warp] = ss;
        row_sync(row, W);
        ss = 0.f;
        for (int i = 0; i < W; ++i) ss += sums[row * W + i];
    }
    return ss / (float)p.H + p.eps * scale * scale;
}

// W warps per row, V vectors of 8 elements per lane, blockDim / (32 W) rows at a time; a block goes on with every gridDim-th set
// of rows and has the next set's loads in flight while it works on this one.  All loads of a row are issued before the first is
// used (a load inside a branch of its own waits for the one before it: 78 us instead of 58 for 16384 x 2048 with V = 2).
template <int V, bool QUANT, bool VEC>
__global__ void __launch_bounds__(512)
addnorm_kernel(const AddNormArgs p, int W)
{
    __shared__ float s_sum[2][16];
    __shared__ uint32_t s_top[2][16];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int row_in_block = warp / W, wr = warp - row_in_block * W;
    const int rows = blockDim.x / (32 * W);
    const int first = (wr * 32 + lane) * 8, step = W * 256;               // this lane's columns: first + v * step ...
    uint4 gv[V], xv[V], rv[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int col = first + v * step;
        gv[v] = p.vec_weight ? load8<VEC>(p.weight + col, p.H - col) : load8<false>(p.weight + col, p.H - col);
        rv[v] = make_uint4(0, 0, 0, 0);
    }
    auto fetch = [&](int t) {
        const int H = t < p.T ? p.H : 0;
#pragma unroll
        for (int v = 0; v < V; ++v) xv[v] = load8<VEC>(p.x + (size_t)t * p.ldx + first + v * step, H - first - v * step);
        if (p.residual) {
#pragma unroll
            for (int v = 0; v < V; ++v) rv[v] = load8<VEC>(p.residual + (size_t)t * p.ldr + first + v * step, H - first - v * step);
        }
    };
    int t = blockIdx.x * rows + row_in_block;
    fetch(t);
    int buf = 0;
    for (int set = blockIdx.x; set * rows < p.T; set += gridDim.x, t += gridDim.x * rows, buf ^= 1) {
        const bool live = t < p.T;
        float h[V][8];
        float ss = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            unpack8(xv[v], h[v]);
            if (p.residual) {
                float r[8];
                unpack8(rv[v], r);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[v][i] += r[i];
                const uint4 sum = pack8(h[v]);                // (rounded: the residual stream that is stored)
                unpack8(sum, h[v]);
            }
        }
        if (set + gridDim.x < (p.T + rows - 1) / rows) fetch(t + gridDim.x * rows);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (p.residual_out) store8<VEC>(p.residual_out + (size_t)t * p.ldro + first + v * step, live ? p.H - first - v * step : 0, h[v]);
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(h[v][i], h[v][i], ss);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(kFull, ss, o);
        if (W > 1) {
            // (two sets of partial sums in turn: a warp may be one set ahead of another, never two)
            if (lane == 0) s_sum[buf][warp] = ss;
            __syncthreads();
            ss = 0.f;
            for (int i = 0; i < W; ++i) ss += s_sum[buf][row_in_block * W + i];
        }
        float mean = ss / (float)p.H + p.eps;
        // (all warps of a row have the same sum, and so go the same way)
        const bool far = !(mean >= 0x1p-100f && mean <= FLT_MAX);
        if (QUANT && far) mean = mean_in_units<V>(p, h, mean, W, warp, lane, row_in_block, s_sum[buf]);
        const bool now = live && (QUANT || !far);
        const float r = 1.f / sqrtf(mean);
        uint32_t top = 0;                                     // largest |y| of the row
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = first + v * step, n = now ? p.H - col : 0;
            float g[8];
            unpack8(gv[v], g);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r * g[i];
            if (p.out) store8<VEC>(p.out + (size_t)t * p.ldo + col, n, h[v]);
            if (QUANT && p.group == 0) {
                // (columns that are not there hold 0, or 0 * r with r not finite)
#pragma unroll
                for (int i = 0; i < 8; ++i) if (VEC ? n > 0 : i < n) top = max(top, magnitude(h[v][i]));
            }
        }
        if (!QUANT) {
            // Here such a row is worked on behind all others' work, out of memory.  (In place, as with an 8-bit output, it costs 16384 x 2048
            // 51 us instead of 46, though no row takes the branch; there 55 instead of 54, and this 64.)
            if (far && live) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int col = first + v * step, n = p.H - col;
                    unpack8(p.residual_out ? load8<VEC>(p.residual_out + (size_t)t * p.ldro + col, n) : load8<VEC>(p.x + (size_t)t * p.ldx + col, n), h[v]);
                    if (p.residual && !p.residual_out) {
                        float r[8];
                        unpack8(load8<VEC>(p.residual + (size_t)t * p.ldr + col, n), r);
#pragma unroll
                        for (int i = 0; i < 8; ++i) h[v][i] += r[i];
                        const uint4 sum = pack8(h[v]);
                        unpack8(sum, h[v]);
                    }
                }
                const float r = 1.f / sqrtf(mean_in_units<V>(p, h, mean, W, warp, lane, row_in_block, s_sum[buf]));
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    float g[8];
                    unpack8(gv[v], g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[v][i] = h[v][i] * r * g[i];
                    if (p.out) store8<VEC>(p.out + (size_t)t * p.ldo + first + v * step, p.H - first - v * step, h[v]);
                }
            }
            continue;
        }
        if (p.group == 0) {
            top = __reduce_max_sync(kFull, top);
            if (W > 1) {
                if (lane == 0) s_top[buf][warp] = top;
                __syncthreads();
                top = 0;
                for (int i = 0; i < W; ++i) top = max(top, s_top[buf][row_in_block * W + i]);
            }
            const float scale = __uint_as_float(top) / 448.f;
            if (live && wr == 0 && lane == 0) p.q_scale[t] = scale;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int col = first + v * step, n = now ? p.H - col : 0;
                if (n > 0) store_q<VEC>(p.q + (size_t)t * p.ldq + col, n, p.vec_q, h[v], scale);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // sixteen lanes hold 128 columns
                const int col = first + v * step, n = now ? p.H - col : 0;
                uint32_t a = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) if (VEC ? n > 0 : i < n) a = max(a, magnitude(h[v][i]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(kFull, a, o));
                const float scale = __uint_as_float(a) / 448.f;
                if (n > 0) {
                    if ((lane & 15) == 0) p.q_scale[(size_t)t * p.n_groups + (col >> 7)] = scale;
                    store_q<VEC>(p.q + (size_t)t * p.ldq + col, n, p.vec_q, h[v], scale);
                }
            }
        }
    }
}

template <int V, bool QUANT, bool VEC>
cudaError_t launch_one(const AddNormArgs& p, int W, int rows, cudaStream_t st)
{
    // As many blocks as are resident at once (64 registers with V = 1, up to 128 above): 16384 x 2048 with a row's scale, V = 2,
    // takes 55 us with 4 blocks of 4 warps per SM, 72 with 3, 67 with 6 and 83 with a block for every row (bf16 alone: 46, 52, 51, 64).
    const int sets = (p.T + rows - 1) / rows, most = 148 * ((V == 1 ? 32 : 16) / (W * rows));
    return launch_pdl(addnorm_kernel<V, QUANT, VEC>, dim3(sets < most ? sets : most), dim3(32 * W * rows), 0, st, p, W);
}
template <int V>
cudaError_t launch_v(const AddNormArgs& p, int W, int rows, cudaStream_t st)
{
    if (p.vec) return p.q ? launch_one<V, true, true>(p, W, rows, st) : launch_one<V, false, true>(p, W, rows, st);
    return p.q ? launch_one<V, true, false>(p, W, rows, st) : launch_one<V, false, false>(p, W, rows, st);
}

}  // namespace

cudaError_t launch_addnorm(const AddNormArgs& in, cudaStream_t st)
{
    AddNormArgs p = in;
    auto al = [](const void* q, size_t n) { return (uintptr_t)q % n == 0; };
    p.vec = p.H % 8 == 0 && al(p.x, 16) && p.ldx % 8 == 0 && al(p.residual, 16) && p.ldr % 8 == 0 && al(p.residual_out, 16) && p.ldro % 8 == 0 &&
            al(p.out, 16) && p.ldo % 8 == 0;
    p.vec_weight = al(p.weight, 16);
    p.vec_q = al(p.q, 8) && p.ldq % 8 == 0;
    // Vectors per lane: two where a row has more than one warp's worth, four beyond 4096 columns (16384 x 2048 with a row's scale, us:
    // V = 1 65, V = 2 and 4 55; bf16 alone 46, 46, 47; 4096 x 8192 in groups: V = 2 63, V = 4 58).  Element by element (VEC false) one is
    // faster: 333 x 1411 4.2 against 4.8.
    const int vecs = (p.H + 7) / 8;
    const int V = vecs <= 32 || (!p.vec && vecs <= 512) ? 1 : (vecs <= 512 ? 2 : 4);
    const int W = (vecs + 32 * V - 1) / (32 * V), rows = W >= 4 ? 1 : 4 / W;
    if (V == 1) return launch_v<1>(p, W, rows, st);
    if (V == 2) return launch_v<2>(p, W, rows, st);
    return launch_v<4>(p, W, rows, st);
}

}  // namespace faasmoe
