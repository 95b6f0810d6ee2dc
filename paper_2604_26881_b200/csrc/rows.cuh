// Rows of bf16 in registers: eight elements at a time, in 16-byte accesses where the addresses allow.  Shared by the row kernels.
#pragma once

#include "internal.h"

namespace faasmoe {

// Two fp32 operations in one instruction (each rounded as the single one): the row kernels are bound by issue as much as by memory.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(d))
        : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// eight elements as four pairs
__device__ __forceinline__ void unpack8(const uint4& v, float2* f)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack8(const float2* f)
{
    uint4 v;
    __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[i].x, f[i].y);
    return v;
}
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

template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float2* f)
{
    if (VEC) {
        if (n > 0) *reinterpret_cast<uint4*>(p) = pack8(f);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = __float2bfloat16_rn(i & 1 ? f[i / 2].y : f[i / 2].x);
    }
}

// |y| as an unsigned number: of the same order, and a NaN is above everything, as it is to be in the outputs
__device__ __forceinline__ uint32_t magnitude(float y) { return __float_as_uint(y) & 0x7fffffffu; }

// a barrier of the warps of one row of the block (rows of several warps: two in a block at most)
__device__ __forceinline__ void row_sync(int row, int W)
{
    if (row == 0) asm volatile("bar.sync 1, %0;" ::"r"(32 * W) : "memory");
    else asm volatile("bar.sync 2, %0;" ::"r"(32 * W) : "memory");
}

}  // namespace faasmoe
