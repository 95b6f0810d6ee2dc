// Eight values of a row as 8-bit integers: q = x / scale in fp32, rounded to the nearest integer (ties to even).  Shared by the
// kernels that write 8-bit rows.
#pragma once

#include <float.h>

#include "rows.cuh"

namespace faasmoe {

// The fp32 quotient is what the rule rounds, but a division per element costs more than the memory traffic.  fma(x, 1 / scale,
// 1.5 * 2^23) rounds x / scale to an integer in one step, from a reciprocal that is off by 2^-24: by less than 8e-6 at 127, and the
// quotient's own rounding is half as much.  So only where that product is within 2e-5 of the middle of two integers (one
// element in 25000, and all of a row whose scale has no ordinary reciprocal) is the quotient itself taken, one after the other so that
// the code stays short.  A scale that is 0, infinite or NaN gives zeros.
struct RowScale {
    float scale, inv;
    bool plain;                 // the reciprocal can be used
    bool none;                  // zeros
};
__device__ __forceinline__ RowScale row_scale(float scale)
{
    RowScale s;
    s.scale = scale;
    s.inv = 1.f / scale;
    s.plain = scale >= 1e-37f;
    s.none = !(scale > 0.f && scale <= FLT_MAX);
    return s;
}
__device__ __forceinline__ uint2 to_i8x8(const float* x, const RowScale& s)
{
    constexpr float kMagic = 12582912.f;                      // 1.5 * 2^23: the integer is in the low bits of the sum
    uint32_t b[8];
    uint32_t doubt = s.plain ? 0u : 0xffu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float m = fmaf(x[i], s.inv, kMagic), k = m - kMagic;
        b[i] = __float_as_uint(m);
        if (fabsf(fmaf(x[i], s.inv, -k)) > 0.5f - 2e-5f) doubt |= 1u << i;
    }
    if (s.none) return make_uint2(0u, 0u);
#pragma unroll 1
    while (doubt) {
        const int i = __ffs(doubt) - 1;
        doubt &= doubt - 1;
        float v = x[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) v = i == j ? x[j] : v;
        const int q = (int)fminf(fmaxf(rintf(__fdiv_rn(v, s.scale)), -127.f), 127.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = i == j ? (uint32_t)q : b[j];
    }
    uint2 o;
    o.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    o.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    return o;
}
template <bool VEC>
__device__ __forceinline__ void store_i8(int8_t* dst, int n, bool vec_q, const float* x, const RowScale& s)
{
    const uint2 o = to_i8x8(x, s);
    if (VEC && vec_q) {
        *reinterpret_cast<uint2*>(dst) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) dst[i] = (int8_t)((i < 4 ? o.x : o.y) >> (8 * (i & 3)) & 0xffu);
    }
}

}  // namespace faasmoe
