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
//     warp does the whole token in 64 bits (choose64).
// Bound by instruction issue: see launch_gate for the counts and times.
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
    return expf(fminf(z, 0.f) - ref) / (1.f + expf(-fabsf(z)));
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

template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
struct Gate {
    static constexpr uint32_t kIdMask = 32 * C - 1;
    // Error bound of the difference of two 32-bit values:
    //   softmax: (z - zmax) * log2 e rounds by 2^-24 relative (p * |ln p| <= 0.37), ex2 by 2 ulp, a sum of at most C + 5
    //            additions in a row and the product by 1.5 ulp each: below 1.2e-6 * p;
    //   sigmoid: the exponential below 2^-21 + 2^-24 |z| relative, times s (1 - s) <= 1/4, and a reciprocal of 1 ulp: below 4e-7;
    // twice that for two, with room.  Ordered by logits the values are exact (1e-37: the key of a denormal has cleared bits too).
    static constexpr float kSlack = !BIAS ? 1e-37f : (SIGMOID ? 2e-6f : 4e-6f);
    static constexpr float kScoreSlack = SIGMOID ? 2e-6f : 4e-6f;
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

template <int C, bool SIGMOID, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(kGateWarps * 32)
gate_kernel(const GateArgs p)
{
    using G = Gate<C, SIGMOID, BIAS, GROUPS>;
    constexpr uint32_t kIdMask = G::kIdMask;
    __shared__ double s_row[kGateWarps][32 * C];
    pdl_wait();
    pdl_launch_dependents();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t = blockIdx.x * kGateWarps + warp;
    if (t >= p.T) return;
    bool bad = false;
    int model = 0;
    if (p.tenant_id) {
        const int u = p.tenant_id[t];
        bad = u < 0 || u >= p.n_tenants;
        model = p.model_of_tenant ? p.model_of_tenant[bad ? 0 : u] : 0;
        if (model < 0 || model >= p.M) model = 0;
    }
    const float* bias = BIAS ? p.bias + (size_t)model * p.E : nullptr;

    // the logits and biases of this lane's experts (vector loads where the rows allow them)
    float z[C], b[C];
    const int held = min(max(p.E - lane * C, 0), C);          // experts of this lane
    if (p.vec && held == C) {
        if (p.bf16_logits) {
            const bf16* src = (const bf16*)p.logits + (size_t)t * p.ld + lane * C;
            uint32_t h[C / 2];
            if constexpr (C == 8) *reinterpret_cast<uint4*>(h) = *reinterpret_cast<const uint4*>(src);
            else if constexpr (C == 4) *reinterpret_cast<uint2*>(h) = *reinterpret_cast<const uint2*>(src);
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
#pragma unroll
        for (int i = 0; i < C; ++i) z[i] = clean(z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) z[i] = i < held ? load_logit(p, t, lane * C + i) : -INFINITY;
    }
    if constexpr (BIAS) {
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
    }
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
    for (int i = 0; i < C; ++i) v[i] = BIAS ? sc[i] + clean_bias(b[i]) : z[i];

    uint32_t key[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        // (from the lowest finite value up: the id bits must not make a NaN of -inf)
        key[i] = (order_key(fmaxf(v[i], -FLT_MAX)) & ~kIdMask) | (kIdMask - lane * C - i);
        if (i >= held) key[i] = 0u;
    }

    // groups of experts
    bool undecided = false;                                   // the groups, or the last rank against the next
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
            float* row = reinterpret_cast<float*>(s_row[warp]);
#pragma unroll
            for (int i = 0; i < C; ++i) row[lane * C + i] = !BIAS && sums ? sc[i] : v[i];
            __syncwarp();
            float a = -INFINITY, c = -INFINITY;
            if (lane < p.n_groups)
                for (int i = 0; i < p.group_size; ++i) {
                    const float x = row[lane * p.group_size + i];
                    c = fmaxf(c, fminf(a, x));
                    a = fmaxf(a, x);
                }
            score = sums ? a + c : a;
            __syncwarp();
        }
        const uint32_t gkey = lane < p.n_groups ? order_key(score) : 0u;
        int rank = 0;
        for (int g = 0; g < p.n_groups; ++g) {
            const uint32_t o = __shfl_sync(kFull, gkey, g);
            rank += o > gkey || (o == gkey && g < lane);
        }
        const bool in = lane < p.n_groups && rank < p.keep;
        const uint32_t kept = __ballot_sync(kFull, in);
        if (BIAS || sums) {
            // the last kept against the best dropped group (a largest logit is exact: nothing to ask)
            const float lo = key_value(__reduce_min_sync(kFull, in ? gkey : kFull));
            const float hi = key_value(__reduce_max_sync(kFull, in ? 0u : gkey));
            undecided = !(lo - hi > (sums ? 2.f : 1.f) * G::kScoreSlack + 1e-6f * (fabsf(lo) + fabsf(hi)));
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
    if (!undecided) {
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
                my_e = G::in_order64(p, t, bias, key, my_key, my_e, rounds, s_row[warp]);
                if (lane < p.k) my_z = load_logit(p, t, my_e);
            }
        }
    } else {
        my_e = choose64<C>(p, t, bias, s_row[warp]);
        my_z = lane < p.k ? load_logit(p, t, my_e) : -INFINITY;
    }

    // weights
    float w, s;
    if (p.renormalize) {
        // exp(-ref) scales every chosen score alike, so small scores do not underflow before the division
        float top = lane < p.k ? my_z : -INFINITY;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
        const float ref = SIGMOID ? fminf(top, 0.f) : top;
        s = 0.f;
        if (lane < p.k && my_z != -INFINITY) s = SIGMOID ? sigmoid_from(my_z, ref) : expf(my_z - ref);
        float sum = s;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        w = sum > 0.f ? s / sum * p.scale : 0.f;
    } else {
        s = 0.f;
        if (my_z != -INFINITY) s = SIGMOID ? sigmoid_from(my_z, 0.f) : expf(my_z - zmax) * inv_sum;
        w = s * p.scale;
    }
    if (lane < p.k) {
        p.topk_idx[(size_t)t * p.k + lane] = bad ? lane : my_e;
        p.topk_w[(size_t)t * p.k + lane] = bad ? 0.f : w;
    }
    if (p.tie_flag) {
        // two neighbours among ranks 1..k+1 closer than 1e-5 relative, in the values that order them (without a bias: the scores)
        if (my_z != -INFINITY) flag_v = SIGMOID ? sigmoid_from(my_z, 0.f) : expf(my_z - zmax) * inv_sum;
        if (BIAS && lane < rounds) flag_v += clean_bias(__ldg(bias + my_e));
        const float pv = __shfl_up_sync(kFull, flag_v, 1);
        const bool near = __any_sync(kFull, lane > 0 && lane < rounds && !(pv - flag_v >= 1e-5f * fabsf(pv)));
        if (lane == 0) p.tie_flag[t] = near || undecided;
    }
    if (bad && lane == 0 && p.status) atomicOr(p.status, MOE_DEV_BAD_TENANT);
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
    // groups that fall on whole lanes, a power of two of them, are reduced by shuffles, others through shared memory
    const int lanes = p.group_size / C;
    p.lanes_per_group = p.group_size % C == 0 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
    p.eligible = p.keep < p.n_groups ? p.keep * p.group_size : p.E;
    // vectors of a lane's share of a row (16 bytes at most)
    const size_t esz = p.bf16_logits ? 2 : 4;
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
