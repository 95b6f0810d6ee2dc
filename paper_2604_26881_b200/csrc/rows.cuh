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

__device__ __forceinline__ void store8_anywhere(bf16* p, int n, const uint4& v);
// (VEC false: all lanes of a warp take part, n elements of this lane, 8 less of the next)
template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float2* f)
{
    if (!VEC) store8_anywhere(p, n, pack8(f));
    else if (n > 0) *reinterpret_cast<uint4*>(p) = pack8(f);
}

// Eight of sixteen consecutive elements (two vectors), from element k on (0 .. 7; the same for all lanes).
__device__ __forceinline__ uint4 eight_from(const uint4& a, const uint4& b, int k)
{
    const bool four = k & 4, two = k & 2, one = k & 1;
    const uint32_t x0 = four ? a.z : a.x, x1 = four ? a.w : a.y, x2 = four ? b.x : a.z, x3 = four ? b.y : a.w, x4 = four ? b.z : b.x, x5 = four ? b.w : b.y;
    const uint32_t y0 = two ? x1 : x0, y1 = two ? x2 : x1, y2 = two ? x3 : x2, y3 = two ? x4 : x3, y4 = two ? x5 : x4;
    return make_uint4(one ? __funnelshift_r(y0, y1, 16) : y0, one ? __funnelshift_r(y1, y2, 16) : y1, one ? __funnelshift_r(y2, y3, 16) : y2,
                      one ? __funnelshift_r(y3, y4, 16) : y3);
}
// A vector whose elements from n on read as zero.
__device__ __forceinline__ uint4 first_of(const uint4& v, int n)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = 2 * i + 1 < n ? w[i] : (2 * i < n ? w[i] & 0xffffu : 0u);
    return make_uint4(o[0], o[1], o[2], o[3]);
}
// A row's vectors, one after the other in a warp's lanes, to a row that is on no 16-byte boundary: each lane writes the aligned 16 bytes
// that its predecessor's last elements and its own first ones make; elements at the ends of the warp's share, and of the row, are
// written one by one.  All lanes take part; n: elements of this lane (possibly none, the next lane's are 8 less).  (Element by element,
// each of eight instructions touches all of the warp's lines: 16384 x 2047 forward 216 us.)
__device__ __forceinline__ void store8_anywhere(bf16* p, int n, const uint4& v)
{
    const int s = (int)((uintptr_t)p & 15) >> 1, lane = threadIdx.x & 31;
    if (s == 0) {
        if (n >= 8) {
            *reinterpret_cast<uint4*>(p) = v;
            return;
        }
    } else {
        const uint4 before = make_uint4(__shfl_up_sync(0xffffffffu, v.x, 1), __shfl_up_sync(0xffffffffu, v.y, 1), __shfl_up_sync(0xffffffffu, v.z, 1),
                                        __shfl_up_sync(0xffffffffu, v.w, 1));
        if (lane > 0 && n >= 8 - s) *reinterpret_cast<uint4*>(p - s) = eight_from(before, v, 8 - s);
    }
    const bool head = s == 0 || lane == 0 || n < 8 - s, tail = s == 0 || lane == 31 || n < 16 - s;      // not written with a neighbour's
    if (n > 0 && (head || tail)) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n && (i < 8 - s ? head : tail)) reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(w[i / 2] >> (16 * (i & 1)));
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
