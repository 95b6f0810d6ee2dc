// Eight values of a row as 8-bit integers: q = x / scale in fp32, rounded to the nearest integer (ties to even).  Shared by the
// kernels that write 8-bit rows.
#pragma once

#include <float.h>

#include "rows.cuh"

namespace faasmoe {

// The fp32 quotient is what the rule rounds (a product with the reciprocal is another number next to the middle of two integers,
// where bf16 values by bf16 maxima lie more often than chance has it: 0.1 % of them exactly on it).  It comes from the reciprocal y by
// Markstein's corrections (P. Markstein, IBM Journal of Research and Development 34, 1990): q + (x - q s) y with fused products is
// the quotient rounded once, if q is off by a unit in the last place at most; x y may be off by two, so there are two corrections.
// Scales that have no ordinary reciprocal, or are so small that x - q s would not be exact, take one division after the other.  A
// scale that is 0, infinite or NaN gives zeros.
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
    s.plain = scale >= 0x1p-70f && scale <= 0x1p100f;
    s.none = !(scale > 0.f && scale <= FLT_MAX);
    return s;
}
__device__ __forceinline__ uint2 to_i8x8(const float2 (&x)[4], const RowScale& s)
{
    constexpr float kMagic = 12582912.f;                      // 1.5 * 2^23: added to, it leaves the nearest integer in the low bits
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float2 q = mul2(x[i], both(s.inv));
        q = fma2(fma2(q, both(-s.scale), x[i]), both(s.inv), q);
        q = fma2(fma2(q, both(-s.scale), x[i]), both(s.inv), q);
        q = add2(q, both(kMagic));
        b[2 * i] = __float_as_uint(q.x); b[2 * i + 1] = __float_as_uint(q.y);
    }
    if (s.none) return make_uint2(0u, 0u);
    if (!s.plain) {                                           // (of the whole row)
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {                         // (one division in the code, not eight)
            float v = x[0].x;
#pragma unroll
            for (int j = 1; j < 8; ++j) v = i == j ? (j & 1 ? x[j / 2].y : x[j / 2].x) : v;
            const int q = (int)fminf(fmaxf(rintf(__fdiv_rn(v, s.scale)), -127.f), 127.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) b[j] = i == j ? (uint32_t)q : b[j];
        }
    }
    uint2 o;
    o.x = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
    o.y = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
    return o;
}
template <bool VEC>
__device__ __forceinline__ void store_i8(int8_t* dst, int n, bool vec_q, const float2 (&x)[4], const RowScale& s)
{
    const uint2 o = to_i8x8(x, s);
    if (vec_q && (VEC || n >= 8)) {
        *reinterpret_cast<uint2*>(dst) = o;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) dst[i] = (int8_t)((i < 4 ? o.x : o.y) >> (8 * (i & 3)) & 0xffu);
    }
}

}  // namespace faasmoe
