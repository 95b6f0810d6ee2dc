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
//   - a value becomes an unsigned key of the same order whose lowest log2(C) bits hold the expert's place in the lane;
//   - a lane sorts its C keys once (a sorting network in registers), then every one of the k + 1 rounds is one
//     redux.sync over the heads of the lists, one ballot (lowest lane among equals) and a shift in the winner's lane;
//   - if two neighbours of the result (or the last kept and the first dropped group) are closer than the error
//     bound of the 32-bit values and are not the same pair (z, b), the warp does the token again in 64 bits (choose64).
// Measured shares of such tokens and times stand at launch_gate.
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
__device__ __forceinline__ float clean(float z) { return z != z ? -INFINITY : fminf(z, FLT_MAX); }

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
            const float b = e < p.E ? bias[e] : 0.f;
            s[i] += b != b ? -INFINITY : (double)b;
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

template <int C>
__global__ void __launch_bounds__(kGateWarps * 32)
gate_kernel(const GateArgs p)
{
    constexpr uint32_t kSlotMask = C - 1;
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
    const float* bias = p.bias ? p.bias + (size_t)model * p.E : nullptr;

    // the logits of this lane's experts (16-byte loads where the rows allow them)
    float z[C], b[C];
    if (p.vec && lane * C < p.E) {
        if (p.bf16_logits) {
            const bf16* src = (const bf16*)p.logits + (size_t)t * p.ld + lane * C;
            bf16 h[C];
            if constexpr (C == 8) *reinterpret_cast<uint4*>(h) = *reinterpret_cast<const uint4*>(src);
            else if constexpr (C == 4) *reinterpret_cast<uint2*>(h) = *reinterpret_cast<const uint2*>(src);
            else *reinterpret_cast<uint32_t*>(h) = *reinterpret_cast<const uint32_t*>(src);
#pragma unroll
            for (int i = 0; i < C; ++i) z[i] = __bfloat162float(h[i]);
        } else {
            const float* src = (const float*)p.logits + (size_t)t * p.ld + lane * C;
            if constexpr (C >= 4) {
#pragma unroll
                for (int i = 0; i < C; i += 4) *reinterpret_cast<float4*>(z + i) = *reinterpret_cast<const float4*>(src + i);
            } else {
                *reinterpret_cast<float2*>(z) = *reinterpret_cast<const float2*>(src);
            }
        }
#pragma unroll
        for (int i = 0; i < C; ++i) z[i] = clean(z[i]);
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) z[i] = lane * C + i < p.E ? load_logit(p, t, lane * C + i) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < C; ++i) {
        b[i] = bias && lane * C + i < p.E ? __ldg(bias + lane * C + i) : 0.f;
        if (b[i] != b[i]) b[i] = -INFINITY;
    }
    // softmax needs the maximum and the sum of the whole row
    float zmax = 0.f, inv_sum = 0.f;
    const bool softmax = p.score == MOE_SCORE_SOFTMAX;
    constexpr float kLog2e = 1.4426950408889634f;
    float sc[C];
    if (softmax) {
        zmax = z[0];
#pragma unroll
        for (int i = 1; i < C; ++i) zmax = fmaxf(zmax, z[i]);
        zmax = key_value(__reduce_max_sync(kFull, order_key(zmax)));
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) {
            sc[i] = z[i] == -INFINITY ? 0.f : exp2f((z[i] - zmax) * kLog2e);
            sum += sc[i];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        inv_sum = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] *= inv_sum;
    } else if (bias || (p.keep < p.n_groups && p.group_score == MOE_GROUP_TOP2)) {
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] = __fdividef(1.f, 1.f + exp2f(fminf(-z[i] * kLog2e, 120.f)));
    } else {
#pragma unroll
        for (int i = 0; i < C; ++i) sc[i] = 0.f;
    }
    // v orders the experts; by_logit: in the order of the logits themselves
    const bool by_logit = !bias;
    uint32_t key[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
        const float v = by_logit ? z[i] : sc[i] + b[i];
        // (from the lowest finite value up: the place bits must not make a NaN of -inf)
        key[i] = lane * C + i < p.E ? ((order_key(fmaxf(v, -FLT_MAX)) & ~kSlotMask) | (kSlotMask - i)) : 0u;
    }
    // error bound of a 32-bit value v: the score's own error, the rounding of the sum and the key's cleared bits
    //   softmax: (z - zmax) * log2e rounds by 2^-24 relative (p * |ln p| <= 0.37), exp2f by 2 ulp, a sum of at most
    //            C + 5 additions in a row and the product by 1.5 ulp each: below 1.2e-6 * p;
    //   sigmoid: exp2f and its argument below 2^-21 + 2^-24 |z|, times s (1 - s) <= 1/4, and a quotient of 2 ulp: below 4e-7.
    // Two values are in order if they differ by more than twice that; kSlack adds a factor of about 1.5.
    constexpr float kSlack = 4e-6f;
    constexpr float kRel = 2.f * C / 8388608.f + 5e-7f;       // cleared key bits: C ulp at most
    auto margin = [&](float v, float abs_err) { return (by_logit ? 1e-37f : abs_err) + kRel * fabsf(v); };

    // groups of experts
    bool undecided = false;
    if (p.keep < p.n_groups) {
        const int size = p.E / p.n_groups;
        const int lanes = size / C;                           // lanes that hold one group, if the groups fall on lanes
        const bool top2 = p.group_score == MOE_GROUP_TOP2 && size > 1;
        const bool use_s = top2 && by_logit;                  // sums need the scores themselves
        float score;                                          // lane g < n_groups: score of group g
        if (p.aligned_groups) {
            float a = -INFINITY, c = -INFINITY;
#pragma unroll
            for (int i = 0; i < C; ++i) {
                const float v = use_s ? sc[i] : (by_logit ? z[i] : sc[i] + b[i]);
                c = fmaxf(c, fminf(a, v));
                a = fmaxf(a, v);
            }
            for (int o = 1; o < lanes; o <<= 1) {
                const float oa = __shfl_xor_sync(kFull, a, o), oc = __shfl_xor_sync(kFull, c, o);
                c = fmaxf(fmaxf(c, oc), fminf(a, oa));
                a = fmaxf(a, oa);
            }
            score = __shfl_sync(kFull, top2 ? a + c : a, (lane * lanes) & 31);
        } else {
            float* row = reinterpret_cast<float*>(s_row[warp]);
#pragma unroll
            for (int i = 0; i < C; ++i) row[lane * C + i] = use_s ? sc[i] : (by_logit ? z[i] : sc[i] + b[i]);
            __syncwarp();
            float a = -INFINITY, c = -INFINITY;
            if (lane < p.n_groups)
                for (int i = 0; i < size; ++i) {
                    const float v = row[lane * size + i];
                    c = fmaxf(c, fminf(a, v));
                    a = fmaxf(a, v);
                }
            score = top2 ? a + c : a;
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
        if (!by_logit || top2) {
            // the last kept against the best dropped group (max of logits: exact, nothing to ask)
            const float lo = key_value(__reduce_min_sync(kFull, in ? gkey : kFull));
            const float hi = key_value(__reduce_max_sync(kFull, in ? 0u : gkey));
            const float m = (top2 ? 2.f : 1.f) * kSlack + 1e-6f * (fabsf(lo) + fabsf(hi));
            undecided = !(lo - hi > m);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int e = lane * C + i;
            const int g = p.aligned_groups ? lane / lanes : e / size;
            if (!(kept >> (g & 31) & 1)) key[i] = 0u;
        }
    }

    // k + 1 rounds over the heads of the sorted lists; lane j keeps rank j
    sort_desc<C>(key);
    const int rounds = min(p.k + 1, p.eligible);
    uint32_t my_key = 0;
    int my_e = 0;
#pragma unroll
    for (int j = 0; j <= kMaxTopK; ++j) {
        if (j < rounds) {
            // (the place bits take no part between lanes: among equals the lowest lane holds the lowest ids)
            const uint32_t head = key[0] & ~kSlotMask;
            const uint32_t m = __reduce_max_sync(kFull, head);
            const int w = __ffs(__ballot_sync(kFull, head == m)) - 1;
            const uint32_t won = __shfl_sync(kFull, key[0], w);
            if (lane == j) { my_key = won; my_e = w * C + (int)(kSlotMask - (won & kSlotMask)); }
            if (lane == w) {
#pragma unroll
                for (int i = 0; i + 1 < C; ++i) key[i] = key[i + 1];
                key[C - 1] = 0u;
            }
        }
    }
    // lane j's logit, bias and value, and whether it is in order with rank j - 1
    float my_z = lane < rounds ? load_logit(p, t, my_e) : -INFINITY;
    if (!(by_logit && p.bf16_logits)) {                       // bf16 logits lose nothing in the key's cleared bits
        float my_b = lane < rounds && bias ? __ldg(bias + my_e) : 0.f;
        const float v = key_value(my_key);
        const float pv = __shfl_up_sync(kFull, v, 1), pz = __shfl_up_sync(kFull, my_z, 1), pb = __shfl_up_sync(kFull, my_b, 1);
        const bool same = pz == my_z && pb == my_b && lane < p.k;       // equal pairs: the lower id, which came first
        const bool near = lane > 0 && lane < rounds && !same && !(pv - v > margin(fmaxf(fabsf(pv), fabsf(v)), kSlack));
        undecided |= __any_sync(kFull, near);
    }
    if (undecided) {
        my_e = choose64<C>(p, t, bias, s_row[warp]);
        if (lane < p.k) my_z = load_logit(p, t, my_e);
    }

    // weights
    float w;
    if (p.renormalize) {
        // exp(-ref) scales every chosen score alike, so small scores do not underflow before the division
        float top = lane < p.k ? my_z : -INFINITY;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
        const float ref = softmax ? top : fminf(top, 0.f);
        float s = 0.f;
        if (lane < p.k && my_z != -INFINITY) s = softmax ? expf(my_z - ref) : sigmoid_from(my_z, ref);
        float sum = s;
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        w = sum > 0.f ? s / sum * p.scale : 0.f;
    } else {
        float s = 0.f;
        if (my_z != -INFINITY) s = softmax ? expf(my_z - zmax) * inv_sum : sigmoid_from(my_z, 0.f);
        w = s * p.scale;
    }
    if (lane < p.k) {
        p.topk_idx[(size_t)t * p.k + lane] = bad ? lane : my_e;
        p.topk_w[(size_t)t * p.k + lane] = bad ? 0.f : w;
    }
    if (p.tie_flag) {
        // two neighbours among ranks 1..k+1 closer than 1e-5 relative, in the values that order them (without a bias: the scores)
        float v = key_value(my_key);
        if (by_logit) v = my_z == -INFINITY ? 0.f : (softmax ? expf(my_z - zmax) * inv_sum : sigmoid_from(my_z, 0.f));
        const float pv = __shfl_up_sync(kFull, v, 1);
        const bool near = __any_sync(kFull, lane > 0 && lane < rounds && !(pv - v >= 1e-5f * fabsf(pv)));
        if (lane == 0) p.tie_flag[t] = near || undecided;
    }
    if (bad && lane == 0 && p.status) atomicOr(p.status, MOE_DEV_BAD_TENANT);
}

}  // namespace

cudaError_t launch_gate(const GateArgs& in, cudaStream_t st)
{
    GateArgs p = in;
    const int C = p.E <= 64 ? 2 : (p.E <= 128 ? 4 : 8);
    const int size = p.E / p.n_groups, lanes = size / C;
    p.aligned_groups = size % C == 0 && (lanes & (lanes - 1)) == 0;
    p.eligible = p.keep < p.n_groups ? p.keep * size : p.E;
    // whole lanes of vectors: rows and experts in multiples of a lane's share, 16 bytes (or the lane's share) aligned
    const size_t esz = p.bf16_logits ? 2 : 4;
    const size_t share = C * esz < 16 ? C * esz : 16;
    p.vec = p.E % C == 0 && p.ld * esz % share == 0 && (uintptr_t)p.logits % share == 0;
    const dim3 grid((p.T + kGateWarps - 1) / kGateWarps), block(kGateWarps * 32);
    if (C == 2) return launch_pdl(gate_kernel<2>, grid, block, 0, st, p);
    if (C == 4) return launch_pdl(gate_kernel<4>, grid, block, 0, st, p);
    return launch_pdl(gate_kernel<8>, grid, block, 0, st, p);
}

}  // namespace faasmoe
