// The residual's addition, the RMSNorm behind it and an 8-bit output with scales, in one pass over the rows:
//
//   h = bf16(x + residual)                   (h = x without a residual; stored to residual_out)
//   y = h * (1 / sqrt(mean(h^2) + eps)) * weight      (fp32)
//   out = bf16(y);   q = e4m3(y / s),  s = max |y| / 448 over the row or over each 128 columns
//
// Bound by HBM: every element is read and written once, kept in registers in between (W warps hold a row, up to four
// 16-byte vectors a lane).  16384 x 2048 with both outputs and a scale per row: 302 MB in 52 us, 5.8 TB/s (0.89 of the
// measured copy bandwidth); 4096 x 8192 with 128-column scales the same; 32 x 2048: 1.9 us, launch and latency.  The sum of
// squares (of the row in units of a power of two, where its squares leave the range), the scales and the quotients are fp32; h is
// rounded once because it is the residual stream that the caller keeps (the norm is that of the stored value), out is one rounding
// of the fp32 y, q one of the fp32 quotient y / s.
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
// where they do not (a vector in 10^4) the quotients are taken.  (16384 x 2048, calls back to back: 59 us,
// 55 with one product that is not looked at again, 66 with quotients of everything.)
template <bool VEC>
__device__ __forceinline__ void store_q(uint8_t* dst, int n, bool vec_q, const float* h, float scale)
{
    const float inv = 1.f / scale;
    uint2 o = e4m3x8(h, inv * (1.f - 0x1p-21f));
    const uint2 up = e4m3x8(h, inv * (1.f + 0x1p-21f));
    // (a scale below 1e-37 has no finite reciprocal)
    if (o.x != up.x || o.y != up.y || scale < 1e-37f) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = scale != 0.f ? h[i] / scale : 0.f;
        o = e4m3x8(y, 1.f);
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

// W warps per row, V vectors of 8 elements per lane, blockDim / (32 W) rows at a time; a block goes on with every gridDim-th set
// of rows and has the next set's loads in flight while it works on this one.  All loads of a row are issued before the first is
// used (a load inside a branch of its own waits for the one before it: 78 us instead of 58 for 16384 x 2048 with V = 2).
template <int V, bool QUANT, bool VEC>
__global__ void __launch_bounds__(512)
addnorm_kernel(const AddNormArgs p, int W)
{
    __shared__ float s_sum[2][16];
    __shared__ uint32_t s_top[2][16];
    __shared__ uint32_t s_big[16];
    __shared__ float s_again[16];
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
        // Squares beyond the range of fp32, or below it with no eps that counts beside them: the row again, in units of a power of two near
        // its largest element (or near the root of eps).  (All warps of a row have the same sum, and so go the same way.)
        // (16384 x 2048: 1.3 us; as a call that is not inlined 8 us.)
        if (!(mean >= 0x1p-100f && mean <= FLT_MAX)) {
            uint32_t big = 0;                                 // (columns that are not there hold 0)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) big = max(big, magnitude(h[v][i]));
            big = __reduce_max_sync(kFull, big);
            if (W > 1) {
                if (lane == 0) s_big[warp] = big;
                row_sync(row_in_block, W);
                big = 0;
                for (int i = 0; i < W; ++i) big = max(big, s_big[row_in_block * W + i]);
            }
            const float unit = fmaxf(__uint_as_float(big), sqrtf(p.eps));
            if (big > 0 && big < 0x7f800000u && unit <= FLT_MAX) {       // (rows of zeros, with infinities or NaN: as they are)
                const int e = min(max((int)(__float_as_uint(unit) >> 23) - 127, -126), 126);
                const float scale = __uint_as_float((uint32_t)(127 - e) << 23);        // 2^-e: exact, as are its products
                ss = 0.f;
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
                    if (lane == 0) s_again[warp] = ss;
                    row_sync(row_in_block, W);
                    ss = 0.f;
                    for (int i = 0; i < W; ++i) ss += s_again[row_in_block * W + i];
                }
                mean = ss / (float)p.H + p.eps * scale * scale;
            }
        }
        const float r = 1.f / sqrtf(mean);
        uint32_t top = 0;                                     // largest |y| of the row
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int col = first + v * step, n = live ? p.H - col : 0;
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
        if (!QUANT) continue;
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
                const int col = first + v * step, n = live ? p.H - col : 0;
                if (n > 0) store_q<VEC>(p.q + (size_t)t * p.ldq + col, n, p.vec_q, h[v], scale);
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // sixteen lanes hold 128 columns
                const int col = first + v * step, n = live ? p.H - col : 0;
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
    // As many blocks as are resident at once (57 registers with V = 1, up to 128 above): 16384 x 2048 with a row's scale, V = 2,
    // takes 52 us with 4 blocks of 4 warps per SM, 63 with 3, 66 with 6 and 81 with a block for every row.
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
    // Vectors per lane: two where a row has more than one warp's worth, four beyond 4096 columns (16384 x 2048, us: V = 1 57, V = 2
    // 52, V = 4 54; 4096 x 8192: V = 2 58, V = 4 52).  Element by element (VEC false) one is faster: 333 x 1411 4.8 against 5.5.
    const int vecs = (p.H + 7) / 8;
    const int V = vecs <= 32 || (!p.vec && vecs <= 512) ? 1 : (vecs <= 512 ? 2 : 4);
    const int W = (vecs + 32 * V - 1) / (32 * V), rows = W >= 4 ? 1 : 4 / W;
    if (V == 1) return launch_v<1>(p, W, rows, st);
    if (V == 2) return launch_v<2>(p, W, rows, st);
    return launch_v<4>(p, W, rows, st);
}

}  // namespace faasmoe
