// Gating rules (paper Sec. 2.1: a gating network picks the k best experts of a token) beyond the plain softmax:
// softmax or sigmoid scores, a bias that balances the experts' load and takes part in the choice only, a choice in two
// steps (groups of experts first), renormalised and scaled weights.  From router logits z:
//
//   s[e] = exp(z[e] - max z) / sum exp(z - max z)   or   1 / (1 + exp(-z[e]))
//   v[e] = s[e] + b[e]           (without a bias the experts are ordered by z itself: s grows with z)
//   group score = max of v, or the sum of the two largest v of the group; the best groups stay (ties: lower group)
//   chosen      = the k largest v of the experts in those groups, in order (ties: lower expert id)
//   w[j]        = s[chosen j]  [ / sum of the chosen s ]  * scale
//
// WHICH experts are chosen is defined in double precision, so the answer does not hang on a rounding of s.  One warp
// takes one token, lane l the C experts l*C .. l*C+C-1 (C = 2, 4 or 8 for up to 64, 128, 256 experts), and orders them in 32 bits:
//   - a value becomes an unsigned key of the same order whose lowest bits hold the expert's id (lower id: larger key), so
//     that keys are unique and the largest one names its expert;
//   - a lane sorts its C keys once (a sorting network in registers), then every one of the k + 1 rounds is one
//     redux.sync over the heads of the lists and a shift in the winner's lane;
//   - neighbours of the result that are closer than the error bound of key and 32-bit value, and are not the same pair
//     (z, b), are put in order by their 64-bit values, one candidate per lane (in_order64); where the groups are that close, the
//     groups' scores are taken in 64 bits (keep64).
// Bound by the length of a warp's chain of dependent integer steps, not by the logits' bytes (16384 x 256 in fp32 are 2.7 us of HBM
// time) nor by issue (the SMs are busy 23 % of the time, with 19 % of their warps): about 870 instructions per token with 256
// experts in groups with a bias (gate_kernel), 470 in gate_many_kernel (22.9 us).  One token: 1.9 us, 32 tokens of the widest
// rule 3.0 us, both launch and latency; more at launch_gate.
// With random logits about 3 % of the tokens of that rule have neighbours that the keys leave undecided.
#include <float.h>

#include "gate.cuh"

namespace faasmoe {

namespace {

constexpr int kGateWarps = 4;
constexpr uint32_t kFull = 0xffffffffu;

__device__ __forceinline__ uint32_t order_key(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);                 // -0 and +0 are the same value
    return b ^ (0x80000000u | (uint32_t)((int32_t)b >> 31));
}
__device__ __forceinline__ float key_value(uint32_t k)
{
    return __uint_as_float(k ^ (0x80000000u | (uint32_t)(~(int32_t)k >> 31)));
}
// a logit as the rules see it: NaN counts as -inf, +inf as the largest finite value
__device__ __forceinline__ float clean(float z) { return fminf(fmaxf(z, -INFINITY), FLT_MAX); }
// a bias likewise, NaN as -inf
__device__ __forceinline__ float clean_bias(float b) { return fmaxf(b, -INFINITY); }
__device__ __forceinline__ float finite(float v) { return fminf(fmaxf(v, -FLT_MAX), FLT_MAX); }
__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float load_logit(const GateArgs& p, int t, int e)
{
    const size_t i = (size_t)t * p.ld + e;
    return clean(p.bf16_logits ? __bfloat162float(((const bf16*)p.logits)[i]) : ((const float*)p.logits)[i]);
}

// sigmoid(z) = exp(min(z, 0) - ref) / (1 + exp(-|z|)) for ref = 0; another ref scales it by exp(-ref) without underflow
__device__ __forceinline__ float sigmoid_from(float z, float ref)
{
    return __fdividef(expf(fminf(z, 0.f) - ref), 1.f + expf(-fabsf(z)));
}
__device__ __forceinline__ double sigmoid64(double z)
{
    const double e = exp(-fabs(z));
    return z >= 0 ? 1. / (1. + e) : e / (1. + e);
}

// The choice of one token in 64 bits: returns rank j's expert in lane j < p.k.
template <int C>
__device__ __noinline__ int choose64(const GateArgs& p, int t, const float* bias, double* row)
{
    const int lane = threadIdx.x & 31;
    double v[C], s[C];
    double zmax = -INFINITY;
    for (int i = 0; i < C; ++i) {
        const int e = lane * C + i;
        v[i] = e < p.E ? (double)load_logit(p, t, e) : -INFINITY;
        zmax = fmax(zmax, v[i]);
    }
    for (int o = 16; o > 0; o >>= 1) zmax = fmax(zmax, __shfl_xor_sync(kFull, zmax, o));
    double sum = 0;
    for (int i = 0; i < C; ++i) {
        if (p.score == MOE_SCORE_SIGMOID) s[i] = sigmoid64(v[i]);
        else { s[i] = v[i] == -INFINITY ? 0. : exp(v[i] - zmax); sum += s[i]; }
    }
    if (p.score == MOE_SCORE_SOFTMAX) {
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        for (int i = 0; i < C; ++i) s[i] = sum > 0 ? s[i] / sum : 0.;
    }
    for (int i = 0; i < C; ++i) {
        const int e = lane * C + i;
        if (bias) {
            s[i] += (double)clean_bias(e < p.E ? bias[e] : 0.f);
            v[i] = s[i];
        }
    }
    uint32_t kept = kFull;
    if (p.keep < p.n_groups) {
        const int size = p.E / p.n_groups;
        const bool by_logit = !bias && (p.group_score == MOE_GROUP_MAX || size == 1);
        for (int i = 0; i < C; ++i) row[lane * C + i] = by_logit ? v[i] : s[i];
        __syncwarp();
        double a = -INFINITY, b = -INFINITY;
        if (lane < p.n_groups)
            for (int i = 0; i < size; ++i) {
                const double x = row[lane * size + i];
                if (x > a) { b = a; a = x; } else if (x > b) b = x;
            }
        if (p.group_score == MOE_GROUP_TOP2 && size > 1) a += b;
        int rank = 0;
        for (int g = 0; g < p.n_groups; ++g) {
            const double x = __shfl_sync(kFull, a, g);
            rank += x > a || (x == a && g < lane);
        }
        kept = __ballot_sync(kFull, lane < p.n_groups && rank < p.keep);
        __syncwarp();
    }
    uint32_t left = 0;                       // bit i: this lane's expert i may still be chosen
    for (int i = 0; i < C; ++i) {
        const int e = lane * C + i;
        if (e < p.E && (p.keep >= p.n_groups || (kept >> (e / (p.E / p.n_groups)) & 1))) left |= 1u << i;
    }
    int mine = 0;
    for (int j = 0; j < p.k; ++j) {
        double best = -INFINITY;
        int id = 1 << 30;
        for (int i = 0; i < C; ++i)
            if ((left >> i & 1) && (id == (1 << 30) || v[i] > best)) { best = v[i]; id = lane * C + i; }
        for (int o = 16; o > 0; o >>= 1) {
            const double ob = __shfl_xor_sync(kFull, best, o);
            const int oi = __shfl_xor_sync(kFull, id, o);
            if (oi < (1 << 30) && (id == (1 << 30) || ob > best || (ob == best && oi < id))) { best = ob; id = oi; }
        }
        if (id / C == lane) left &= ~(1u << (id % C));
        if (lane == j) mine = id;
    }
    return mine;
}

template <int C>
__device__ __forceinline__ void sort_desc(uint32_t (&a)[C])
{
    auto cs = [&](int i, int j) { const uint32_t x = max(a[i], a[j]), y = min(a[i], a[j]); a[i] = x; a[j] = y; };
    if constexpr (C == 2) { cs(0, 1); }
    if constexpr (C == 4) { cs(0, 1); cs(2, 3); cs(0, 2); cs(1, 3); cs(1, 2); }
    if constexpr (C == 8) {                  // Batcher's odd-even merge sort, 19 exchanges
        cs(0, 1); cs(2, 3); cs(4, 5); cs(6, 7); cs(0, 2); cs(1, 3); cs(4, 6); cs(5, 7); cs(1, 2); cs(5, 6);
        cs(0, 4); cs(1, 5); cs(2, 6); cs(3, 7); cs(2, 4); cs(3, 5); cs(1, 2); cs(3, 4); cs(5, 6);
    }
}

// The next largest key of the warp's lists: every lane gets it, the lane that held it moves its list up.
template <int C>
__device__ __forceinline__ uint32_t pop(uint32_t (&key)[C])
{
    const uint32_t m = __reduce_max_sync(kFull, key[0]);
    if (key[0] == m) {
#pragma unroll
        for (int i = 0; i + 1 < C; ++i) key[i] = key[i + 1];
        key[C - 1] = 0u;
    }
    return m;
}

// The groups that stay, decided in 64 bits (bit g: group g).
template <int C, bool SIGMOID, bool BIAS>
__device__ __noinline__ uint32_t keep64(const GateArgs& p, int t, const float* bias, double* row)
{
    const int lane = threadIdx.x & 31;
    const bool by_logit = !BIAS && (p.group_score == MOE_GROUP_MAX || p.group_size == 1);
    float z[C];
    double v[C];
#pragma unroll
    for (int i = 0; i < C; ++i) z[i] = lane * C + i < p.E ? load_logit(p, t, lane * C + i) : -INFINITY;
    if (by_logit) {
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = z[i];
    } else if (SIGMOID) {
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = sigmoid64(z[i]);
    } else {
        float m = z[0];
#pragma unroll
        for (int i = 1; i < C; ++i) m = fmaxf(m, z[i]);
        m = key_value(__reduce_max_sync(kFull, order_key(m)));
        double sum = 0;
#pragma unroll
        for (int i = 0; i < C; ++i) { v[i] = z[i] == -INFINITY ? 0. : exp((double)z[i] - (double)m); sum += v[i]; }
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = sum > 0 ? v[i] / sum : 0.;
    }
    if (BIAS) {
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] += (double)clean_bias(lane * C + i < p.E ? __ldg(bias + lane * C + i) : 0.f);
    }
    double a = -INFINITY, b = -INFINITY;
    if (p.lanes_per_group) {
#pragma unroll
        for (int i = 0; i < C; ++i) { if (v[i] > a) { b = a; a = v[i]; } else if (v[i] > b) b = v[i]; }
        for (int o = 1; o < p.lanes_per_group; o <<= 1) {
            const double oa = __shfl_xor_sync(kFull, a, o), ob = __shfl_xor_sync(kFull, b, o);
            if (oa > a) { b = a > ob ? a : ob; a = oa; } else if (oa > b) b = oa;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) row[lane * C + i] = v[i];
        __syncwarp();
        if (lane < p.n_groups)
            for (int i = 0; i < p.group_size; ++i) {
                const double x = row[lane * p.group_size + i];
                if (x > a) { b = a; a = x; } else if (x > b) b = x;
            }
        __syncwarp();
    }
    if (p.group_score == MOE_GROUP_TOP2 && p.group_size > 1) a += b;
    if (p.lanes_per_group) a = __shfl_sync(kFull, a, (lane * p.lanes_per_group) & 31);
    int rank = 0;
    for (int g = 0; g < p.n_groups; ++g) {
        const double x = __shfl_sync(kFull, a, g);
        rank += x > a || (x == a && g < lane);
    }
    return __ballot_sync(kFull, lane < p.n_groups && rank < p.keep);
}

template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
struct Gate {
    static constexpr uint32_t kIdMask = 32 * C - 1;
    // Error bound of the difference of two 32-bit values:
    //   softmax: the argument (z - zmax) * log2 e is off by 3 * 2^-24 of itself, which is at most 0.37 * 1.8e-7 in p (p |ln p| <= 0.37)
    //            and, averaged over a row of 256, ln 256 * 1.8e-7 of the sum; ex2 by 2 ulp, 2.4e-7, in either; the sum by its C + 5
    //            additions in a row, 7.8e-7; quotient and product 6e-8 each: below 2.5e-6 of p, and two p add up to 1 at most;
    //   sigmoid: the exponential below 2^-21 + 2^-24 |z| relative, times s (1 - s) <= 1/4, and a reciprocal of 1 ulp: below 4e-7;
    // twice that for two sigmoids, with room.  Ordered by logits the values are exact (1e-37: the key of a denormal has cleared bits too).
    static constexpr float kSlack = !BIAS ? 1e-37f : (SIGMOID ? 2e-6f : 4e-6f);
    static constexpr __device__ float score_slack() { return SIGMOID ? 2e-6f : 4e-6f; }
    // the cleared bits of two keys (32 C ulp each at most) and the rounding of s + b
    static constexpr float kRel = 2.f * 32 * C / 8388608.f + 5e-7f;

    // The largest p.k of the lane's candidates (lanes below n, in the order of their keys) in 64-bit order: lane j gets rank j's
    // expert.  First the list is continued until its last two are clearly apart: what follows is below all but the last.
    static __device__ __noinline__ int in_order64(const GateArgs& p, int t, const float* bias, uint32_t (&key)[C], uint32_t my_key, int my_e, int n,
                                                  double* row)
    {
        const int lane = threadIdx.x & 31;
        for (;;) {
            const float v = key_value(__shfl_sync(kFull, my_key, n - 1)), pv = key_value(__shfl_sync(kFull, my_key, n - 2));
            if (n == p.eligible || pv - v > kSlack + kRel * fmaxf(fabsf(pv), fabsf(v))) break;
            if (n == 32) return choose64<C>(p, t, bias, row);
            const uint32_t m = pop<C>(key);
            if (lane == n) { my_key = m; my_e = (int)(kIdMask - (m & kIdMask)); }
            ++n;
        }
        double v = -INFINITY;
        const float z = lane < n ? load_logit(p, t, my_e) : -INFINITY;
        if (!BIAS) {
            v = (double)z;
        } else {
            double s;
            if (SIGMOID) {
                s = sigmoid64((double)z);
            } else {
                float zmax = -INFINITY;
                for (int e = lane; e < p.E; e += 32) zmax = fmaxf(zmax, load_logit(p, t, e));
                zmax = key_value(__reduce_max_sync(kFull, order_key(zmax)));
                double sum = 0;
                for (int e = lane; e < p.E; e += 32) {
                    const float q = load_logit(p, t, e);
                    if (q != -INFINITY) sum += exp((double)q - (double)zmax);
                }
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
                s = z != -INFINITY && sum > 0 ? exp((double)z - (double)zmax) / sum : 0.;
            }
            if (lane < n) v = s + (double)clean_bias(bias[my_e]);
        }
        int rank = 0;
        for (int j = 0; j < n; ++j) {
            const double o = __shfl_sync(kFull, v, j);
            const int oe = __shfl_sync(kFull, my_e, j);
            rank += o > v || (o == v && oe < my_e);
        }
        if (lane < n) row[rank] = (double)my_e;
        __syncwarp();
        const int mine = lane < p.k ? (int)row[lane] : 0;
        __syncwarp();
        return mine;
    }
};

// Weights and outputs of one token, by a warp: lane j < p.k has the expert of rank j and its logit.
template <bool SIGMOID>
__device__ __forceinline__ void write_token(const GateArgs& p, int t, int lane, int my_e, float my_z, float zmax, float inv_sum, bool bad)
{
    float w, s = 0.f;
    if (p.renormalize) {
        // exp(-ref) scales every chosen score alike, so small scores do not underflow before the division
        float top = lane < p.k ? my_z : -INFINITY;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
        const float ref = SIGMOID ? fminf(top, 0.f) : top;
        if (lane < p.k && my_z != -INFINITY) s = SIGMOID ? sigmoid_from(my_z, ref) : expf(my_z - ref);
        float sum = s;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        w = sum > 0.f ? s * (p.scale / sum) : 0.f;
    } else {
        if (my_z != -INFINITY) s = SIGMOID ? sigmoid_from(my_z, 0.f) : expf(my_z - zmax) * inv_sum;
        w = s * p.scale;
    }
    if (lane < p.k) {
        p.topk_idx[(size_t)t * p.k + lane] = bad ? lane : my_e;
        p.topk_w[(size_t)t * p.k + lane] = bad ? 0.f : w;
    }
}

// a lane's share of a row of logits (as they are) and of biases, with vector loads where the rows allow them
template <int C>
__device__ __forceinline__ void load_logits(const GateArgs& p, int t, int lane, int held, float (&z)[C])
{
    if (p.vec && held == C) {
        if (p.bf16_logits) {
            const bf16* src = (const bf16*)p.logits + (size_t)t * p.ld + lane * C;
            uint32_t h[C / 2];
            if constexpr (C == 8) { const uint4 q = *reinterpret_cast<const uint4*>(src); h[0] = q.x; h[1] = q.y; h[2] = q.z; h[3] = q.w; }
            else if constexpr (C == 4) { const uint2 q = *reinterpret_cast<const uint2*>(src); h[0] = q.x; h[1] = q.y; }
            else h[0] = *reinterpret_cast<const uint32_t*>(src);
#pragma unroll
            for (int i = 0; i < C; ++i) z[i] = __uint_as_float(i & 1 ? h[i / 2] & 0xffff0000u : h[i / 2] << 16);
        } else {
            const float* src = (const float*)p.logits + (size_t)t * p.ld + lane * C;
            if constexpr (C >= 4) {
#pragma unroll
                for (int i = 0; i < C; i += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(src + i);
                    z[i] = q.x; z[i + 1] = q.y; z[i + 2] = q.z; z[i + 3] = q.w;
                }
            } else {
                const float2 q = *reinterpret_cast<const float2*>(src);
                z[0] = q.x; z[1] = q.y;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) z[i] = i < held ? load_logit(p, t, lane * C + i) : -INFINITY;
    }
}
template <int C>
__device__ __forceinline__ void load_bias(const GateArgs& p, const float* bias, int lane, int held, float (&b)[C])
{
    if (p.vec_bias && held == C) {
        if constexpr (C >= 4) {
#pragma unroll
            for (int i = 0; i < C; i += 4) {
                const float4 q = __ldg(reinterpret_cast<const float4*>(bias + lane * C + i));
                b[i] = q.x; b[i + 1] = q.y; b[i + 2] = q.z; b[i + 3] = q.w;
            }
        } else {
            const float2 q = __ldg(reinterpret_cast<const float2*>(bias + lane * C));
            b[0] = q.x; b[1] = q.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) b[i] = i < held ? __ldg(bias + lane * C + i) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) b[i] = clean_bias(b[i]);
}

// One token by one warp; row: scratch of 32 C doubles.
template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
__device__ __forceinline__ void gate_token(const GateArgs& p, int t, int lane, double* row)
{
    using G = Gate<C, SIGMOID, BIAS, GROUPS>;
    constexpr uint32_t kIdMask = G::kIdMask;
    bool bad = false;
    int model = 0;
    if (p.tenant_id) {
        const int u = p.tenant_id[t];
        bad = u < 0 || u >= p.n_tenants;
        model = p.model_of_tenant ? p.model_of_tenant[bad ? 0 : u] : 0;
        if (model < 0 || model >= p.M) model = 0;
    }
    const float* bias = BIAS ? p.bias + (size_t)model * p.E : nullptr;
    const int held = min(max(p.E - lane * C, 0), C);          // experts of this lane
    float z[C], b[C];
    load_logits<C>(p, t, lane, held, z);
    if (BIAS) load_bias<C>(p, bias, lane, held, b);
#pragma unroll
    for (int i = 0; i < C; ++i) z[i] = clean(z[i]);
    // scores: softmax needs the maximum and the sum of the whole row; sigmoids only if they are compared
    float zmax = 0.f, inv_sum = 0.f;
    constexpr float kLog2e = 1.4426950408889634f;
    const bool sums = GROUPS && p.group_score == MOE_GROUP_TOP2 && p.group_size > 1;      // groups are compared by sums of scores
    float v[C];                                               // what orders the experts: s + b, or z
    float sc[C];
    if constexpr (!SIGMOID) {
        float m = z[0];
#pragma unroll
        for (int i = 1; i < C; ++i) m = fmaxf(m, z[i]);
        zmax = key_value(__reduce_max_sync(kFull, order_key(m)));
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            sc[i] = z[i] == -INFINITY ? 0.f : ex2((z[i] - zmax) * kLog2e);
            sum += sc[i];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        inv_sum = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] *= inv_sum;
    } else if (BIAS || sums) {
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] = rcp(1.f + ex2(-z[i] * kLog2e));
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) v[i] = BIAS ? __fadd_rn(sc[i], b[i]) : z[i];       // (never fused with the product before it)

    uint32_t key[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        // (finite values: the id bits must not make a NaN of an infinity)
        key[i] = (order_key(finite(v[i])) & ~kIdMask) | (kIdMask - lane * C - i);
        if (i >= held) key[i] = 0u;
    }

    // groups of experts
    bool undecided = false;                                   // 32 bits did not decide
    if constexpr (GROUPS) {
        float score;                                          // lane g < n_groups: score of group g
        if (p.lanes_per_group) {
            float a = -INFINITY, c = -INFINITY;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const float x = !BIAS && sums ? sc[i] : v[i];
                c = fmaxf(c, fminf(a, x));
                a = fmaxf(a, x);
            }
            for (int o = 1; o < p.lanes_per_group; o <<= 1) {
                const float oa = __shfl_xor_sync(kFull, a, o), oc = __shfl_xor_sync(kFull, c, o);
                c = fmaxf(fmaxf(c, oc), fminf(a, oa));
                a = fmaxf(a, oa);
            }
            score = __shfl_sync(kFull, sums ? a + c : a, (lane * p.lanes_per_group) & 31);
        } else {
            float* frow = reinterpret_cast<float*>(row);
#pragma unroll
            for (int i = 0; i < C; ++i) frow[lane * C + i] = !BIAS && sums ? sc[i] : v[i];
            __syncwarp();
            float a = -INFINITY, c = -INFINITY;
            if (lane < p.n_groups)
                for (int i = 0; i < p.group_size; ++i) {
                    const float x = frow[lane * p.group_size + i];
                    c = fmaxf(c, fminf(a, x));
                    a = fmaxf(a, x);
                }
            score = sums ? a + c : a;
            __syncwarp();
        }
        const uint32_t gkey = lane < p.n_groups ? order_key(BIAS ? finite(score) : score) : 0u;      // (infinite ones are decided below)
        int rank = 0;
        for (int g = 0; g < p.n_groups; ++g) {
            const uint32_t o = __shfl_sync(kFull, gkey, g);
            rank += o > gkey || (o == gkey && g < lane);
        }
        const bool in = lane < p.n_groups && rank < p.keep;
        uint32_t kept = __ballot_sync(kFull, in);
        if (BIAS || sums) {
            // the last kept against the best dropped group (a largest logit is exact: nothing to ask)
            const float lo = key_value(__reduce_min_sync(kFull, in ? gkey : kFull));
            const float hi = key_value(__reduce_max_sync(kFull, in ? 0u : gkey));
            undecided = !(lo - hi > (sums ? 2.f : 1.f) * G::score_slack() + 1e-6f * (fabsf(lo) + fabsf(hi)));
            if (undecided) kept = keep64<C, SIGMOID, BIAS>(p, t, bias, row);
        }
        if (p.lanes_per_group) {
            if (!(kept >> (lane / p.lanes_per_group) & 1)) {
#pragma unroll
                for (int i = 0; i < C; ++i) key[i] = 0u;
            }
        } else {
#pragma unroll
            for (int i = 0; i < C; ++i)
                if (!(kept >> (((lane * C + i) / p.group_size) & 31) & 1)) key[i] = 0u;
        }
    }

    // k + 1 rounds over the heads of the sorted lists; lane j keeps rank j
    int my_e;
    float my_z, flag_v = 0.f;
    const int rounds = min(p.k + 1, p.eligible);
    {
        sort_desc<C>(key);
        uint32_t my_key = 0;
#pragma unroll
        for (int j = 0; j <= kMaxTopK; ++j) {
            if (j < rounds) {
                const uint32_t m = pop<C>(key);
                if (lane == j) my_key = m;
            }
        }
        my_e = (int)(kIdMask - (my_key & kIdMask));
        // is lane j in order with rank j - 1?
        my_z = lane < rounds ? load_logit(p, t, my_e) : -INFINITY;
        if (BIAS || !p.bf16_logits) {                         // (bf16 logits lose nothing in the key's cleared bits)
            const float my_b = BIAS && lane < rounds ? __ldg(bias + my_e) : 0.f;
            const float kv = key_value(my_key);
            const float pv = __shfl_up_sync(kFull, kv, 1), pz = __shfl_up_sync(kFull, my_z, 1), pb = __shfl_up_sync(kFull, my_b, 1);
            const bool same = pz == my_z && pb == my_b && lane < p.k;     // equal pairs: the lower id, which came first
            const bool near = lane > 0 && lane < rounds && !same && !(pv - kv > G::kSlack + G::kRel * fmaxf(fabsf(pv), fabsf(kv)));
            if (__any_sync(kFull, near)) {
                undecided = true;
                my_e = G::in_order64(p, t, bias, key, my_key, my_e, rounds, row);
                if (lane < p.k) my_z = load_logit(p, t, my_e);
            }
        }
    }

    write_token<SIGMOID>(p, t, lane, my_e, my_z, zmax, inv_sum, bad);
    if (p.tie_flag) {
        // two neighbours among ranks 1..k+1 closer than 1e-5 relative, in the values that order them (without a bias: the scores, up
        // to a common factor)
        if (my_z != -INFINITY) flag_v = SIGMOID ? sigmoid_from(my_z, 0.f) : expf(my_z - zmax) * (BIAS ? inv_sum : 1.f);
        if (BIAS && lane < rounds) flag_v += clean_bias(__ldg(bias + my_e));
        const float pv = __shfl_up_sync(kFull, flag_v, 1);
        const bool near = __any_sync(kFull, lane > 0 && lane < rounds && !(pv - flag_v >= 1e-5f * fabsf(pv)));
        if (lane == 0) p.tie_flag[t] = near || undecided;
    }
    if (bad && lane == 0 && p.status) atomicOr(p.status, MOE_DEV_BAD_TENANT);
}

template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(kGateWarps * 32)
gate_kernel(const GateArgs p)
{
    __shared__ double s_row[kGateWarps][32 * C];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, t = blockIdx.x * kGateWarps + warp;
    if (t < p.T) gate_token<C, SIGMOID, BIAS, GROUPS>(p, t, threadIdx.x & 31, s_row[warp]);
}

// (a call, so that the registers of its rare use do not count in the kernel below)
template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
__device__ __noinline__ void gate_token_again(const GateArgs& p, int t, int lane, double* row)
{
    gate_token<C, SIGMOID, BIAS, GROUPS>(p, t, lane, row);
}

// Many tokens: four lanes per token.  A warp's instructions are what bounds the choice (the kernel above needs about 870 per
// token with 256 experts, groups and a bias), and most of its rounds keep 31 lanes waiting for one.  Here the lanes
// of a token go over its experts in blocks of 32 (lane r: experts 32 b + 16 h + 4 r + i), sort the eight of a block with the
// network, read the block's two largest off its top, and merge block after block into a list of the eight largest (pairwise
// maxima of one list and the other reversed are a bitonic sequence with the eight largest of both); two more merges join the
// four lanes.  The two largest of what the merges drop are ranks 9 and 10.  Groups are runs of whole blocks.  All loads of a token are in
// flight at once; its logits, then its sorted blocks, wait in shared memory at places that only their lane touches, so
// that the blocks can be a short loop.
template <int NB, bool SIGMOID, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(kGateWarps * 32)
gate_many_kernel(const GateArgs p)
{
    using G = Gate<NB, SIGMOID, BIAS, GROUPS>;
    constexpr uint32_t kIdMask = G::kIdMask;
    __shared__ double s_row[kGateWarps][32 * NB];
    __shared__ float4 s_z[kGateWarps][2 * NB][32];                        // [half block][lane]: logits, then sorted keys
    __shared__ float4 s_bias[BIAS ? 8 * NB : 1];
    __shared__ uint2 s_top[kGateWarps][GROUPS ? NB : 1][8];               // a block's two largest keys, per token
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane & 3;
    const int t0 = (blockIdx.x * kGateWarps + warp) * 8, t = t0 + (lane >> 2);
    const bool live = t < p.T;
    const int blocks = (p.E + 31) >> 5;
    const bool whole = (p.E & 31) == 0;
    {
        float4 q[2 * NB];
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c) {
            const int e = 16 * c + 4 * r;
            q[c] = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            if (p.vec && live && e + 4 <= p.E) {
                if (p.bf16_logits) {
                    const uint2 v = *reinterpret_cast<const uint2*>((const bf16*)p.logits + (size_t)t * p.ld + e);
                    q[c] = make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                                       __uint_as_float(v.y & 0xffff0000u));
                } else {
                    q[c] = *reinterpret_cast<const float4*>((const float*)p.logits + (size_t)t * p.ld + e);
                }
            } else if (live && e < p.E) {
                q[c].x = load_logit(p, t, e);
                if (e + 1 < p.E) q[c].y = load_logit(p, t, e + 1);
                if (e + 2 < p.E) q[c].z = load_logit(p, t, e + 2);
                if (e + 3 < p.E) q[c].w = load_logit(p, t, e + 3);
            }
        }
        if constexpr (BIAS) {
            if (p.M == 1)
                for (int e = threadIdx.x; e < 32 * NB; e += kGateWarps * 32) reinterpret_cast<float*>(s_bias)[e] = e < p.E ? __ldg(p.bias + e) : 0.f;
        }
#pragma unroll
        for (int c = 0; c < 2 * NB; ++c)
            s_z[warp][c][lane] = make_float4(clean(q[c].x), clean(q[c].y), clean(q[c].z), clean(q[c].w));
    }
    __syncthreads();
    if (t0 >= p.T) return;
    bool bad = false;
    int model = 0;
    if (p.tenant_id && live) {
        const int u = p.tenant_id[t];
        bad = u < 0 || u >= p.n_tenants;
        model = p.model_of_tenant ? p.model_of_tenant[bad ? 0 : u] : 0;
        if (model < 0 || model >= p.M) model = 0;
    }
    const float* bias = BIAS ? p.bias + (size_t)model * p.E : nullptr;
    auto block_logits = [&](int b, float (&z)[8]) {
        const float4 x = s_z[warp][2 * b][lane], y = s_z[warp][2 * b + 1][lane];
        z[0] = x.x; z[1] = x.y; z[2] = x.z; z[3] = x.w; z[4] = y.x; z[5] = y.y; z[6] = y.z; z[7] = y.w;
    };
    // softmax: maximum, then sum of the row (for scores, and for weights that are not renormalised).  A block's eight terms are a tree, so
    // that a sum is as many additions deep as in the kernel above, C + 5 at most: the bounds in Gate hold for both.
    constexpr float kLog2e = 1.4426950408889634f;
    float zmax = 0.f, inv_sum = 0.f;
    if (!SIGMOID && (BIAS || !p.renormalize || p.tie_flag)) {
        float m = -INFINITY, sum = 0.f;
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
            float z[8];
            block_logits(b, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, z[i]);
        }
        m = fmaxf(m, __shfl_xor_sync(kFull, m, 1));
        zmax = fmaxf(m, __shfl_xor_sync(kFull, m, 2));
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
            float z[8];
            block_logits(b, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = z[i] == -INFINITY ? 0.f : ex2((z[i] - zmax) * kLog2e);
            sum += ((z[0] + z[1]) + (z[2] + z[3])) + ((z[4] + z[5]) + (z[6] + z[7]));
        }
        sum += __shfl_xor_sync(kFull, sum, 1);
        sum += __shfl_xor_sync(kFull, sum, 2);
        inv_sum = sum > 0.f ? 1.f / sum : 0.f;
    }

    uint32_t list[8], dropped = 0, dropped2 = 0;              // the eight largest, and the next two
#pragma unroll
    for (int i = 0; i < 8; ++i) list[i] = 0u;
    auto merge = [&](const uint32_t (&other)[8]) {
        uint32_t d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = min(list[i], other[7 - i]);
            list[i] = max(list[i], other[7 - i]);
        }
        auto top2 = [](uint32_t& a, uint32_t& b, uint32_t c, uint32_t e) { b = max(min(a, c), max(b, e)); a = max(a, c); };
#pragma unroll
        for (int i = 0; i < 8; i += 2) { const uint32_t x = max(d[i], d[i + 1]); d[i + 1] = min(d[i], d[i + 1]); d[i] = x; }
        top2(d[0], d[1], d[2], d[3]);
        top2(d[4], d[5], d[6], d[7]);
        top2(d[0], d[1], d[4], d[5]);
        top2(dropped, dropped2, d[0], d[1]);
        auto cs = [&](int i, int j) { const uint32_t x = max(list[i], list[j]), y = min(list[i], list[j]); list[i] = x; list[j] = y; };
        cs(0, 4); cs(1, 5); cs(2, 6); cs(3, 7); cs(0, 2); cs(1, 3); cs(4, 6); cs(5, 7); cs(0, 1); cs(2, 3); cs(4, 5); cs(6, 7);
    };
    {
#pragma unroll 1
        for (int b = 0; b < blocks; ++b) {
            float z[8];
            block_logits(b, z);
            uint32_t key[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int e = 32 * b + 16 * h + 4 * r;
                float bv[4] = {0.f, 0.f, 0.f, 0.f};
                if constexpr (BIAS) {
                    if (p.M == 1) {
                        const float4 q = s_bias[e >> 2];
                        bv[0] = q.x; bv[1] = q.y; bv[2] = q.z; bv[3] = q.w;
                    } else if (p.vec_bias && e + 4 <= p.E) {
                        const float4 q = __ldg(reinterpret_cast<const float4*>(bias + e));
                        bv[0] = q.x; bv[1] = q.y; bv[2] = q.z; bv[3] = q.w;
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) bv[i] = e + i < p.E ? __ldg(bias + e + i) : 0.f;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float v = z[4 * h + i];
                    if constexpr (BIAS) {
                        // (the softmax of -inf is 0 also where the whole row is -inf)
                        v = (SIGMOID ? rcp(1.f + ex2(-v * kLog2e)) : (v == -INFINITY ? 0.f : ex2((v - zmax) * kLog2e) * inv_sum)) + clean_bias(bv[i]);
                    }
                    key[4 * h + i] = (order_key(finite(v)) & ~kIdMask) | (kIdMask - e - i);
                    if (!whole && e + i >= p.E) key[4 * h + i] = 0u;
                }
            }
            sort_desc<8>(key);
            if constexpr (GROUPS) {
                uint32_t a = key[0], c = key[1];
#pragma unroll
                for (int o = 1; o <= 2; o <<= 1) {
                    const uint32_t oa = __shfl_xor_sync(kFull, a, o), oc = __shfl_xor_sync(kFull, c, o);
                    c = max(min(a, oa), max(c, oc));
                    a = max(a, oa);
                }
                if (r == 0) s_top[warp][b][lane >> 2] = make_uint2(a, c);
                uint4* keys = reinterpret_cast<uint4*>(&s_z[warp][2 * b][lane]);
                keys[0] = make_uint4(key[0], key[1], key[2], key[3]);
                keys[32] = make_uint4(key[4], key[5], key[6], key[7]);
            } else {
                merge(key);
            }
        }
    }

    bool unsure = false;                                      // this token goes through gate_token
    if constexpr (GROUPS) {
        __syncwarp();
        const bool top2 = p.group_score == MOE_GROUP_TOP2;
        const int run = p.group_size >> 5;                    // blocks per group: 1, 2, 4 or 8
        // lane r scores the groups r, r + 4 of its token and counts the better ones
        const int groups = p.n_groups;                        // at most 8
        float score[2], big = 0.f;
        uint32_t best[2], second[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int g = r + 4 * h;
            uint32_t a = 0, c = 0;
            if (g < groups)
                for (int o = 0; o < run; ++o) {
                    const uint2 q = s_top[warp][g * run + o][lane >> 2];
                    c = max(min(a, q.x), max(c, q.y));
                    a = max(a, q.x);
                }
            best[h] = a; second[h] = c;
            score[h] = g < groups ? key_value(a) + (top2 ? key_value(c) : 0.f) : -INFINITY;
            if (g < groups) big = fmaxf(big, fabsf(key_value(a)) + fabsf(key_value(c)));
        }
        int above[2] = {0, 0};
#pragma unroll
        for (int o = 0; o < 8; ++o) {
            const float other = __shfl_sync(kFull, o < 4 ? score[0] : score[1], (lane & ~3) | (o & 3));
            if (o < groups) {
                above[0] += other > score[0] || (other == score[0] && o < r);
                above[1] += other > score[1] || (other == score[1] && o < r + 4);
            }
        }
        float lo = INFINITY, hi = -INFINITY;
        uint32_t kept = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int g = r + 4 * h;
            if (g >= groups) continue;
            if (above[h] < p.keep) { kept |= 1u << g; lo = fminf(lo, score[h]); } else hi = fmaxf(hi, score[h]);
        }
#pragma unroll
        for (int o = 1; o <= 2; o <<= 1) {
            kept |= __shfl_xor_sync(kFull, kept, o);
            lo = fminf(lo, __shfl_xor_sync(kFull, lo, o));
            hi = fmaxf(hi, __shfl_xor_sync(kFull, hi, o));
            big = fmaxf(big, __shfl_xor_sync(kFull, big, o));
        }
        // (scores are sums of values read off keys; bf16 logits lose nothing there)
        const bool close = (BIAS || !p.bf16_logits) && !(lo - hi > (top2 ? 2.f : 1.f) * G::kSlack + G::kRel * big);
        if (!SIGMOID && BIAS) unsure = close;                 // (a softmax in 64 bits needs the whole row)
        if ((SIGMOID || !BIAS) && __any_sync(kFull, close)) {
            // The groups' scores in 64 bits, from the group's best (two); a group with a further expert that close to them
            // sends the token through gate_token.
            bool more = false;
            double part[2][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int g = r + 4 * h;
                const bool here = g < groups && live;
                if (here) {
                    const float least = key_value(top2 ? second[h] : best[h]);
                    const uint32_t edge = order_key(least - (G::kSlack + G::kRel * fabsf(least)));
                    int near = 0;
                    for (int o = 0; o < run; ++o)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {         // the four lanes' eight keys of the block
                            const uint4 k4 = reinterpret_cast<const uint4*>(&s_z[warp][2 * (g * run + o) + (i >> 2)][(lane & ~3) + (i & 3)])[0];
                            near += (k4.x >= edge) + (k4.y >= edge) + (k4.z >= edge) + (k4.w >= edge);
                        }
                    more |= near > (top2 ? 2 : 1);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int e = (int)(kIdMask - ((j ? second[h] : best[h]) & kIdMask));
                    const bool on = here && (j == 0 || top2);
                    const double z = on ? load_logit(p, t, e) : 0.f;
                    part[h][j] = BIAS ? sigmoid64(z) + (double)(on ? clean_bias(__ldg(bias + e)) : 0.f) : z;
                    if (!on) part[h][j] = 0.;
                }
            }
            const double exact[2] = {r < groups ? part[0][0] + part[0][1] : -INFINITY, r + 4 < groups ? part[1][0] + part[1][1] : -INFINITY};
            int rank[2] = {0, 0};
#pragma unroll
            for (int o = 0; o < 8; ++o) {
                const double other = __shfl_sync(kFull, o < 4 ? exact[0] : exact[1], (lane & ~3) | (o & 3));
                if (o < groups) {
                    rank[0] += other > exact[0] || (other == exact[0] && o < r);
                    rank[1] += other > exact[1] || (other == exact[1] && o < r + 4);
                }
            }
            uint32_t again = (r < groups && rank[0] < p.keep ? 1u << r : 0u) | (r + 4 < groups && rank[1] < p.keep ? 16u << r : 0u);
#pragma unroll
            for (int o = 1; o <= 2; o <<= 1) {
                again |= __shfl_xor_sync(kFull, again, o);
                more |= __shfl_xor_sync(kFull, (int)more, o) != 0;
            }
            if (close) { kept = again; unsure = more; }
        }
        // (The flag is gate_token's to say wherever it might find the groups undecided.  Its values differ from these by the cleared bits
        // of keys, half of kRel, and with a softmax by the order of the sum, 2.1e-6.)
        if (BIAS && p.tie_flag) unsure |= !(lo - hi > (SIGMOID ? 1.f : 2.f) * ((top2 ? 2.f : 1.f) * G::kSlack + G::kRel * big));
        // (every token goes over its own groups, keep of them: the places of a lane in s_z are its own in any block)
#pragma unroll 1
        for (uint32_t left = kept; left; left &= left - 1) {
            const int first = (__ffs(left) - 1) * run;
#pragma unroll 1
            for (int o = 0; o < run; ++o) {
                const uint4* keys = reinterpret_cast<const uint4*>(&s_z[warp][2 * (first + o)][lane]);
                const uint4 x = keys[0], y = keys[32];
                const uint32_t key[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                merge(key);
            }
        }
    }

    // the four lanes' lists into one
#pragma unroll 1
    for (int o = 1; o <= 2; o <<= 1) {
        uint32_t other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl_xor_sync(kFull, list[i], o);
        {
            const uint32_t od = __shfl_xor_sync(kFull, dropped, o), od2 = __shfl_xor_sync(kFull, dropped2, o);
            dropped2 = max(min(dropped, od), max(dropped2, od2));
            dropped = max(dropped, od);
        }
        merge(other);
    }

    // Neighbours that the keys do not tell apart are put in order below, in 64 bits, the first rank behind the choice among them;
    // if the one behind that is as close, gate_token does it.
    const int k = p.k;
    bool mixed = false;
    if (BIAS || !p.bf16_logits) {
        float f[10];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = key_value(list[j]);
        f[8] = key_value(dropped);
        f[9] = key_value(dropped2);
        const int last = min(k + 1, p.eligible - 1);          // the last rank looked at, from 0
        float least = f[0];
#pragma unroll
        for (int j = 1; j < 10; ++j) if (j == last) least = f[j];
        const float need = G::kSlack + G::kRel * fmaxf(fabsf(f[0]), fabsf(least));        // (sorted: the largest magnitude is at an end)
        bool edge = false, behind = false;
#pragma unroll
        for (int j = 0; j < 9; ++j) {
            const bool near = j + 1 <= last && !(f[j] - f[j + 1] > need);
            if (j + 1 < k) mixed |= near;
            if (j + 1 == k) edge = near;
            if (j == k) behind = near;
        }
        mixed |= edge;
        unsure |= edge && behind;
        if (!SIGMOID && BIAS) {
            unsure |= mixed;                                  // (a softmax in 64 bits needs the whole row)
            if (p.tie_flag) {                                 // (the flag as for the groups; 2 kRel is above 1e-5 and what values differ by)
#pragma unroll
                for (int j = 0; j < 9; ++j) unsure |= j + 1 <= last && !(f[j] - f[j + 1] > 2.f * need);
            }
        }
    }

    // lane r has ranks 2 r and 2 r + 1 (and every lane the first rank behind the eight)
    const uint32_t k0 = r == 0 ? list[0] : r == 1 ? list[2] : r == 2 ? list[4] : list[6], k1 = r == 0 ? list[1] : r == 1 ? list[3] : r == 2 ? list[5] : list[7];
    const int e0 = (int)(kIdMask - (k0 & kIdMask)), e1 = (int)(kIdMask - (k1 & kIdMask)), e8 = (int)(kIdMask - (dropped & kIdMask));
    const int ranks = min(k + 1, p.eligible);                 // ranks that may take part in the order
    bool on0 = live && 2 * r < k, on1 = live && 2 * r + 1 < k;
    float z0 = live && 2 * r < ranks ? load_logit(p, t, e0) : -INFINITY, z1 = live && 2 * r + 1 < ranks ? load_logit(p, t, e1) : -INFINITY;
    int at0 = 2 * r, at1 = 2 * r + 1, at8 = 8;
    float z8 = -INFINITY;
    if (__any_sync(kFull, mixed && !unsure)) {
        if (live && ranks > 8) z8 = load_logit(p, t, e8);
        double v0 = z0, v1 = z1, v8 = z8;
        if (BIAS) {
            v0 = live && 2 * r < ranks ? sigmoid64(z0) + (double)clean_bias(__ldg(bias + e0)) : 0.;
            v1 = live && 2 * r + 1 < ranks ? sigmoid64(z1) + (double)clean_bias(__ldg(bias + e1)) : 0.;
            v8 = live && ranks > 8 ? sigmoid64(z8) + (double)clean_bias(__ldg(bias + e8)) : 0.;
        }
        int n0 = 0, n1 = 0, n8 = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from = (lane & ~3) | q;
                const double ov = __shfl_sync(kFull, h ? v1 : v0, from);
                const int oe = __shfl_sync(kFull, h ? e1 : e0, from);
                if (2 * q + h < ranks) {
                    n0 += ov > v0 || (ov == v0 && oe < e0);
                    n1 += ov > v1 || (ov == v1 && oe < e1);
                    n8 += ov > v8 || (ov == v8 && oe < e8);
                }
            }
        if (ranks > 8) {
            n0 += v8 > v0 || (v8 == v0 && e8 < e0);
            n1 += v8 > v1 || (v8 == v1 && e8 < e1);
        }
        if (mixed) {
            at0 = n0; at1 = n1; at8 = n8;
            on0 = live && 2 * r < ranks && n0 < k;
            on1 = live && 2 * r + 1 < ranks && n1 < k;
        }
    }
    const bool on8 = mixed && live && ranks > 8 && at8 < k && r == 0;     // (rank 9 has moved up: lane 0 writes it)
    if (!on0) z0 = -INFINITY;
    if (!on1) z1 = -INFINITY;
    if (!on8) z8 = -INFINITY;
    {
        float w0, w1, w8, s0 = 0.f, s1 = 0.f, s8 = 0.f;
        if (p.renormalize) {
            float top = fmaxf(fmaxf(z0, z1), z8);
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
            top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
            const float ref = SIGMOID ? fminf(top, 0.f) : top;
            if (z0 != -INFINITY) s0 = SIGMOID ? sigmoid_from(z0, ref) : expf(z0 - ref);
            if (z1 != -INFINITY) s1 = SIGMOID ? sigmoid_from(z1, ref) : expf(z1 - ref);
            if (z8 != -INFINITY) s8 = SIGMOID ? sigmoid_from(z8, ref) : expf(z8 - ref);
            float sum = s0 + s1 + s8;
            sum += __shfl_xor_sync(kFull, sum, 1);
            sum += __shfl_xor_sync(kFull, sum, 2);
            const float share = sum > 0.f ? p.scale / sum : 0.f;
            w0 = s0 * share; w1 = s1 * share; w8 = s8 * share;
        } else {
            if (z0 != -INFINITY) s0 = SIGMOID ? sigmoid_from(z0, 0.f) : expf(z0 - zmax) * inv_sum;
            if (z1 != -INFINITY) s1 = SIGMOID ? sigmoid_from(z1, 0.f) : expf(z1 - zmax) * inv_sum;
            if (z8 != -INFINITY) s8 = SIGMOID ? sigmoid_from(z8, 0.f) : expf(z8 - zmax) * inv_sum;
            w0 = s0 * p.scale; w1 = s1 * p.scale; w8 = s8 * p.scale;
        }
        const size_t out = (size_t)t * k;
        if (on0 && !unsure) { p.topk_idx[out + at0] = bad ? at0 : e0; p.topk_w[out + at0] = bad ? 0.f : w0; }
        if (on1 && !unsure) { p.topk_idx[out + at1] = bad ? at1 : e1; p.topk_w[out + at1] = bad ? 0.f : w1; }
        if (on8 && !unsure) { p.topk_idx[out + at8] = bad ? at8 : e8; p.topk_w[out + at8] = bad ? 0.f : w8; }
    }
    if (p.tie_flag) {
        // what gate_token looks at, in the same values: neighbours among ranks 1..k+1 that the keys leave undecided, or closer than 1e-5
        // relative (with a softmax and a bias it has been asked wherever either may be)
        bool near = false;
        if (SIGMOID || !BIAS) {
            float zz[3] = {0.f, 0.f, 0.f}, bb[3] = {0.f, 0.f, 0.f}, vv[3] = {0.f, 0.f, 0.f};      // ranks 2 r, 2 r + 1, 2 r + 2
            float kv[3] = {key_value(k0), key_value(k1), key_value(dropped)};
            bool in[3];
            const int ids[3] = {e0, e1, e8};
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                in[q] = live && 2 * r + q < ranks && (q < 2 || r == 3);
                if (!in[q]) continue;
                zz[q] = load_logit(p, t, ids[q]);
                if (BIAS) bb[q] = __ldg(bias + ids[q]);
                if (zz[q] != -INFINITY) vv[q] = SIGMOID ? sigmoid_from(zz[q], 0.f) : expf(zz[q] - zmax);
                if (BIAS) vv[q] += clean_bias(bb[q]);
            }
            const float nz = __shfl_down_sync(kFull, zz[0], 1), nb = __shfl_down_sync(kFull, bb[0], 1), nv = __shfl_down_sync(kFull, vv[0], 1),
                        nk = __shfl_down_sync(kFull, kv[0], 1);
            const bool next = __shfl_down_sync(kFull, (int)in[0], 1) != 0;
            if (r < 3) { zz[2] = nz; bb[2] = nb; vv[2] = nv; kv[2] = nk; in[2] = next; }
#pragma unroll
            for (int q = 1; q < 3; ++q) {
                const bool same = zz[q - 1] == zz[q] && bb[q - 1] == bb[q] && 2 * r + q < k;
                const bool apart = kv[q - 1] - kv[q] > G::kSlack + G::kRel * fmaxf(fabsf(kv[q - 1]), fabsf(kv[q]));
                near |= in[q] && ((!apart && !same && (BIAS || !p.bf16_logits)) || !(vv[q - 1] - vv[q] >= 1e-5f * fabsf(vv[q - 1])));
            }
        }
        const uint32_t any = __ballot_sync(kFull, near);
        if (live && r == 0 && !unsure) p.tie_flag[t] = (any >> lane & 15u) != 0;
    }
    if (bad && live && r == 0 && p.status) atomicOr(p.status, MOE_DEV_BAD_TENANT);

    // what 32 bits could not decide, token by token
    uint32_t todo = __ballot_sync(kFull, unsure && live && r == 0);
    while (todo) {
        const int from = __ffs(todo) - 1;
        todo &= todo - 1;
        gate_token_again<NB, SIGMOID, BIAS, GROUPS>(p, t0 + (from >> 2), lane, s_row[warp]);
        __syncwarp();
    }
}

template <int NB>
cudaError_t launch_many(const GateArgs& p, cudaStream_t st)
{
    const int which = (p.score == MOE_SCORE_SIGMOID ? 4 : 0) + (p.bias ? 2 : 0) + (p.keep < p.n_groups ? 1 : 0);
    const dim3 grid((p.T + 8 * kGateWarps - 1) / (8 * kGateWarps)), block(kGateWarps * 32);
    switch (which) {
        case 0: return launch_pdl(gate_many_kernel<NB, false, false, false>, grid, block, 0, st, p);
        case 1: return launch_pdl(gate_many_kernel<NB, false, false, true>, grid, block, 0, st, p);
        case 2: return launch_pdl(gate_many_kernel<NB, false, true, false>, grid, block, 0, st, p);
        case 3: return launch_pdl(gate_many_kernel<NB, false, true, true>, grid, block, 0, st, p);
        case 4: return launch_pdl(gate_many_kernel<NB, true, false, false>, grid, block, 0, st, p);
        case 5: return launch_pdl(gate_many_kernel<NB, true, false, true>, grid, block, 0, st, p);
        case 6: return launch_pdl(gate_many_kernel<NB, true, true, false>, grid, block, 0, st, p);
        default: return launch_pdl(gate_many_kernel<NB, true, true, true>, grid, block, 0, st, p);
    }
}

template <int C>
cudaError_t launch_c(const GateArgs& p, dim3 grid, dim3 block, cudaStream_t st)
{
    const int which = (p.score == MOE_SCORE_SIGMOID ? 4 : 0) + (p.bias ? 2 : 0) + (p.keep < p.n_groups ? 1 : 0);
    switch (which) {
        case 0: return launch_pdl(gate_kernel<C, false, false, false>, grid, block, 0, st, p);
        case 1: return launch_pdl(gate_kernel<C, false, false, true>, grid, block, 0, st, p);
        case 2: return launch_pdl(gate_kernel<C, false, true, false>, grid, block, 0, st, p);
        case 3: return launch_pdl(gate_kernel<C, false, true, true>, grid, block, 0, st, p);
        case 4: return launch_pdl(gate_kernel<C, true, false, false>, grid, block, 0, st, p);
        case 5: return launch_pdl(gate_kernel<C, true, false, true>, grid, block, 0, st, p);
        case 6: return launch_pdl(gate_kernel<C, true, true, false>, grid, block, 0, st, p);
        default: return launch_pdl(gate_kernel<C, true, true, true>, grid, block, 0, st, p);
    }
}

}  // namespace

cudaError_t launch_gate(const GateArgs& in, cudaStream_t st)
{
    GateArgs p = in;
    const int C = p.E <= 64 ? 2 : (p.E <= 128 ? 4 : 8);
    p.group_size = p.E / p.n_groups;
    const size_t esz = p.bf16_logits ? 2 : 4;
    p.eligible = p.keep < p.n_groups ? p.keep * p.group_size : p.E;
    // Four lanes per token where there are tokens enough for its longer chain, and the groups are runs of 1, 2, 4 or 8 blocks of
    // 32 compared by what orders the experts (sums of scores beside an order by logits stay with the other kernel).  Measured, one
    // warp per token / four lanes per token, us: 60 experts, softmax: 2048 tokens 3.7 / 4.5, 4096 5.0 / 4.7, 32768 24 / 11; 96, sigmoid,
    // bias: 4096 6.6 / 5.7; 128 in 4 groups, sigmoid, bias: 4096 7.2 / 7.7, 8192 10.8 / 9.1; 256, softmax: 4096 7.1 / 7.7, 8192
    // 11.7 / 9.8; 256 in 8 groups, sigmoid, bias: 8192 14.8 / 17.4, 16384 25.4 / 23.0, 32768 47 / 37.  With a softmax and a bias, whose
    // near ties go through gate_token: 128 in 4 groups 8192 12.3 / 15.5, 16384 20.6 / 19.0; 256: 16384 24.9 / 31.5, 32768 45.5 / 45.2,
    // in 8 groups 51.7 / 50.0.
    const int run = p.group_size / 32;
    const bool grouped = p.keep < p.n_groups;
    const bool blocks = !grouped || (p.group_size % 32 == 0 && (run & (run - 1)) == 0 && (p.bias || p.group_score == MOE_GROUP_MAX));
    int many_from = p.E <= 128 ? (grouped ? 8192 : 4096) : (p.bias ? 16384 : 8192);
    if (p.score == MOE_SCORE_SOFTMAX && p.bias) many_from = p.E <= 128 ? 16384 : 32768;
    // groups that fall on whole lanes, a power of two of them, are reduced by shuffles, others through shared memory
    const int lanes = p.group_size / C;
    p.lanes_per_group = p.group_size % C == 0 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
    if (p.T >= many_from && blocks) {
        // (aligned for a lane's eight here and for its C in gate_token)
        p.vec = p.ld % 8 == 0 && (uintptr_t)p.logits % 16 == 0;
        p.vec_bias = (uintptr_t)p.bias % 16 == 0 && p.E % 4 == 0;
        return C == 2 ? launch_many<2>(p, st) : (C == 4 ? launch_many<4>(p, st) : launch_many<8>(p, st));
    }
    // vectors of a lane's share of a row (16 bytes at most)
    const size_t share = C * esz < 16 ? C * esz : 16;
    p.vec = p.ld * esz % share == 0 && (uintptr_t)p.logits % share == 0;
    const size_t bias_share = C * 4 < 16 ? C * 4 : 16;
    p.vec_bias = (uintptr_t)p.bias % bias_share == 0 && p.E * 4 % bias_share == 0;
    const dim3 grid((p.T + kGateWarps - 1) / kGateWarps), block(kGateWarps * 32);
    if (C == 2) return launch_c<2>(p, grid, block, st);
    if (C == 4) return launch_c<4>(p, grid, block, st);
    return launch_c<8>(p, grid, block, st);
}

}  // namespace faasmoe
