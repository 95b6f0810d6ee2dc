// The balance loss of a router with its per-expert counts, and the gradient of the logits.  Per token, from its logits z:
//
//   p[e] = softmax(z)[e]    or    s[e] / sum s,  s = sigmoid(z)              lse = log sum exp z
//   loss = E / (k n) sum_e c[e] P[e],   c = counts of the choices, P = mean of p, n = tokens        z_loss = mean of lse^2
//
//   dz[e] = g_w[e]  +  p[e] (1 - s[e]) (f[e] - sum_i f[i] p[i])  +  softmax(z)[e] 2 lse d_z / n       f = d_loss E / (k n^2) c
//
// with (1 - s) only for sigmoid scores and g_w the part that comes by way of the chosen experts' weights w = s, or s over the sum
// of the chosen s.  A token is taken by 4, 8 or 16 lanes with 16 experts each (up to 64, 128, 256 experts).
#include <float.h>

#include "balance.cuh"

namespace faasmoe {

namespace {

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kC = 16;                  // experts of a lane
constexpr int kWarps = 8;

// a logit as the rules see it: NaN counts as -inf, +inf as the largest finite value
__device__ __forceinline__ float clean(float z) { return fminf(fmaxf(z, -INFINITY), FLT_MAX); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(bf16 x) { return __bfloat162float(x); }

// sigmoid(z) = exp(min(z, 0) - ref) / (1 + exp(-|z|)) for ref = 0; another ref scales it by exp(-ref) without underflow
__device__ __forceinline__ float sigmoid_from(float z, float ref) { return __fdividef(expf(fminf(z, 0.f) - ref), 1.f + expf(-fabsf(z))); }

template <int L>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    return v;
}
template <int L>
__device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

// The expert in place i of a lane: vectors of VW neighbours, the lanes of a token taking them in turn.
template <int L, int VW>
__device__ __forceinline__ int expert_of(int sub, int i) { return ((i / VW) * L + sub) * VW + i % VW; }

// This lane's 16 logits of a row, -inf where there is no expert.
template <int L, int VW, typename TL>
__device__ __forceinline__ void load_row(const TL* row, int E, int sub, bool live, float (&z)[kC])
{
#pragma unroll
    for (int q = 0; q < kC / VW; ++q) {
        const int e0 = (q * L + sub) * VW, n = live ? E - e0 : 0;
        TL v[VW];
        if (VW > 1 && n >= VW) {
            const uint4 u = *reinterpret_cast<const uint4*>(row + e0);
            memcpy(v, &u, sizeof(v) < sizeof(u) ? sizeof(v) : sizeof(u));
        } else {
#pragma unroll
            for (int j = 0; j < VW; ++j) if (j < n) v[j] = row[e0 + j];
        }
#pragma unroll
        for (int j = 0; j < VW; ++j) z[q * VW + j] = j < n ? clean(to_float(v[j])) : -INFINITY;
    }
}

// Model of a token, or -1 if it takes no part.
__device__ __forceinline__ int model_of(const RouterBatch& b, int t, bool report)
{
    if (b.mask && b.mask[t] == 0) return -1;
    if (!b.tenant_id) return 0;
    const int u = b.tenant_id[t];
    if (u < 0 || u >= b.n_tenants) {
        if (report && b.status) atomicOr(b.status, MOE_DEV_BAD_TENANT);
        return -1;
    }
    if (!b.model_of_tenant) return 0;
    const int m = b.model_of_tenant[u];
    return m >= 0 && m < b.M ? m : 0;
}

// The shares p of a token, out of its logits (which become p); its log of the sum of exponentials.  A token without any logit
// above -inf has p = 0 and 0.
template <int L, bool SIGMOID, bool LSE>
__device__ __forceinline__ void shares(float (&z)[kC], float& lse)
{
    float top = z[0];
#pragma unroll
    for (int i = 1; i < kC; ++i) top = fmaxf(top, z[i]);
    top = group_max<L>(top);
    const bool some = top > -INFINITY;
    const float from = some ? top : 0.f;
    lse = 0.f;
    float sum = 0.f;
    if (!SIGMOID || LSE) {
        float e[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) { e[i] = expf(z[i] - from); sum += e[i]; }
        sum = group_sum<L>(sum);
        if (LSE) lse = some ? top + logf(sum) : 0.f;
        if (!SIGMOID) {
#pragma unroll
            for (int i = 0; i < kC; ++i) z[i] = e[i];
        }
    }
    if (SIGMOID) {
        const float ref = top > -60.f ? 0.f : from;           // (sigmoids of far negative logits in units of their largest)
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kC; ++i) { z[i] = sigmoid_from(z[i], ref); sum += z[i]; }
        sum = group_sum<L>(sum);
    }
    const float inv = some ? 1.f / sum : 0.f;
#pragma unroll
    for (int i = 0; i < kC; ++i) z[i] *= inv;
}

__host__ __device__ constexpr int padded(int E) { return (E + 3) & ~3; }
__host__ __device__ constexpr int record(int E) { return 2 * padded(E) + 4; }      // sums of p, counts, sum of lse^2, tokens

constexpr int kFinishMost = 4096;       // floats of a finishing block's table

// Adds up the records of a model (n of them, `stride` floats apart) in a fixed order and writes its outputs.
__device__ __forceinline__ void finish(const BalanceArgs& p, int m, const float* rec, int n, size_t stride, float* s_p, int* s_c)
{
    __shared__ double s_red[2][32];
    __shared__ int s_n[32];
    const int E = p.b.E, Ep = padded(E), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    int width = 1;                                            // lanes that share a record: one for four experts
    while (width * 4 < Ep) width *= 2;
    const int c = (tid & (width - 1)) * 4, r = tid / width;
    int rows = (int)blockDim.x / width;
    if (rows > n) rows = n;
    if (r < rows && c < Ep) {
        float4 sp = make_float4(0.f, 0.f, 0.f, 0.f);
        int4 sc = make_int4(0, 0, 0, 0);
#pragma unroll 4
        for (int x = r; x < n; x += rows) {
            const float4 f = *reinterpret_cast<const float4*>(rec + x * stride + c);
            const int4 q = *reinterpret_cast<const int4*>(rec + x * stride + Ep + c);
            sp.x += f.x; sp.y += f.y; sp.z += f.z; sp.w += f.w;
            sc.x += q.x; sc.y += q.y; sc.z += q.z; sc.w += q.w;
        }
        *reinterpret_cast<float4*>(s_p + r * Ep + c) = sp;
        *reinterpret_cast<int4*>(s_c + r * Ep + c) = sc;
    }
    double z = 0;
    int tokens = 0;
    for (int x = tid; x < n; x += blockDim.x) {
        z += (double)rec[x * stride + 2 * Ep];
        tokens += __float_as_int(rec[x * stride + 2 * Ep + 1]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) { z += __shfl_xor_sync(kFull, z, o); tokens += __shfl_xor_sync(kFull, tokens, o); }
    if (lane == 0) { s_red[0][warp] = z; s_n[warp] = tokens; }
    __syncthreads();
    z = 0; tokens = 0;
    for (int w = 0; w < warps; ++w) { z += s_red[0][w]; tokens += s_n[w]; }
    const double over = tokens > 0 ? 1.0 / tokens : 0.0;
    double part = 0;
    for (int e = tid; e < E; e += blockDim.x) {
        double sum = 0;
        int count = 0;
        for (int i = 0; i < rows; ++i) { sum += (double)s_p[i * Ep + e]; count += s_c[i * Ep + e]; }
        p.counts[(size_t)m * E + e] = count;
        p.mean_prob[(size_t)m * E + e] = (float)(sum * over);
        part += (double)count * sum * over;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) part += __shfl_xor_sync(kFull, part, o);
    if (lane == 0) s_red[1][warp] = part;
    __syncthreads();
    if (tid == 0) {
        part = 0;
        for (int w = 0; w < warps; ++w) part += s_red[1][w];
        p.tokens[m] = tokens;
        p.loss[m] = (float)(part * over * E / p.b.k);
        if (p.z_loss) p.z_loss[m] = (float)(z * over);
    }
}

// blockIdx.y: model; the model's blocks take chunks of 32 tokens per warp in turn.  A lane keeps the sums of its 16 experts.
template <int L, int VW, bool SIGMOID, typename TL>
__global__ void __launch_bounds__(32 * kWarps)
balance_kernel(const BalanceArgs p)
{
    constexpr int G = 32 / L;                                 // tokens of a warp at a time
    __shared__ __align__(16) float s_p[kWarps][kC * L];
    __shared__ __align__(16) int s_count[kC * L];
    __shared__ float s_z[kWarps];
    __shared__ int s_n[kWarps];
    __shared__ unsigned char s_list[kWarps][32];
    __shared__ __align__(16) float s_rec[record(kC * L)];
    pdl_wait();
    pdl_launch_dependents();
    const RouterBatch& b = p.b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % L, group = lane / L;
    const int m = blockIdx.y;
    for (int i = threadIdx.x; i < kC * L; i += blockDim.x) s_count[i] = 0;
    __syncthreads();
    float acc[kC], z2 = 0.f;
#pragma unroll
    for (int i = 0; i < kC; ++i) acc[i] = 0.f;
    int tokens = 0;
    const int chunks = (b.T + 31) / 32;
    for (int chunk = blockIdx.x * kWarps + warp; chunk < chunks; chunk += gridDim.x * kWarps) {
        const int t0 = chunk * 32, t = t0 + lane;
        const bool mine = t < b.T && model_of(b, t, m == 0) == m;
        const uint32_t set = __ballot_sync(kFull, mine);
        const int count = __popc(set);
        tokens += count;
        if (mine) {
            s_list[warp][__popc(set & ((1u << lane) - 1))] = (unsigned char)lane;
            for (int j = 0; j < b.k; ++j) {
                const int e = b.topk_idx[(size_t)t * b.k + j];
                if (e >= 0 && e < b.E) atomicAdd(&s_count[e], 1);
                else if (b.status) atomicOr(b.status, MOE_DEV_BAD_EXPERT);
            }
        }
        __syncwarp();
        for (int base = 0; base < count; base += G) {
            const bool live = base + group < count;
            const int row = t0 + (live ? s_list[warp][base + group] : 0);
            float z[kC], lse;
            load_row<L, VW>((const TL*)b.logits + (size_t)row * b.ld, b.E, sub, live, z);
            if (p.z_loss) shares<L, SIGMOID, true>(z, lse); else shares<L, SIGMOID, false>(z, lse);
#pragma unroll
            for (int i = 0; i < kC; ++i) acc[i] += z[i];
            z2 = fmaf(lse, lse, z2);
        }
        __syncwarp();
    }
#pragma unroll
    for (int o = L; o < 32; o <<= 1) {
#pragma unroll
        for (int i = 0; i < kC; ++i) acc[i] += __shfl_xor_sync(kFull, acc[i], o);
        z2 += __shfl_xor_sync(kFull, z2, o);
    }
    if (group == 0) {
#pragma unroll
        for (int i = 0; i < kC; ++i) s_p[warp][expert_of<L, VW>(sub, i)] = acc[i];
    }
    if (lane == 0) { s_z[warp] = z2; s_n[warp] = tokens; }
    __syncthreads();
    const int Ep = padded(b.E);
    for (int e = threadIdx.x; e < Ep; e += blockDim.x) {
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) sum += s_p[w][e];
        s_rec[e] = sum;
        s_rec[Ep + e] = __int_as_float(s_count[e]);
    }
    if (threadIdx.x == 0) {
        float sum = 0.f;
        int n = 0;
        for (int w = 0; w < kWarps; ++w) { sum += s_z[w]; n += s_n[w]; }
        s_rec[2 * Ep] = sum;
        s_rec[2 * Ep + 1] = __int_as_float(n);
    }
    __syncthreads();
    if (gridDim.x == 1) {
        finish(p, m, s_rec, 1, 0, &s_p[0][0], s_count);
    } else {
        float* dst = p.parts + ((size_t)blockIdx.x * b.M + m) * record(b.E);
        for (int i = threadIdx.x; i < record(b.E); i += blockDim.x) dst[i] = s_rec[i];
    }
}

__global__ void __launch_bounds__(1024)
balance_finish_kernel(const BalanceArgs p)
{
    __shared__ __align__(16) float s_p[kFinishMost];
    __shared__ __align__(16) int s_c[kFinishMost];
    pdl_wait();
    pdl_launch_dependents();
    const int m = blockIdx.x;
    finish(p, m, p.parts + (size_t)m * record(p.b.E), p.blocks, (size_t)p.b.M * record(p.b.E), s_p, s_c);
}

// ---------------------------------------------------------------------------------------------------------------------

template <int L, int VW, bool SIGMOID, typename TL>
__global__ void __launch_bounds__(32 * kWarps)
gate_grad_kernel(const GateGradArgs p)
{
    constexpr int G = 32 / L;                                 // tokens of a warp at a time
    constexpr int J = L < 8 ? 2 : 1;                          // chosen experts of a lane: j = sub and sub + L
    __shared__ __align__(16) float s_add[kWarps][G][kC * L];  // what comes by way of the weights, at the chosen experts
    pdl_wait();
    pdl_launch_dependents();
    const RouterBatch& b = p.b;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane % L, group = lane / L;
    float* const add = s_add[warp][group];
    for (int i = sub; i < kC * L; i += L) add[i] = 0.f;
    __syncwarp();
    const int steps = (b.T + G - 1) / G;
    for (int step = blockIdx.x * kWarps + warp; step < steps; step += gridDim.x * kWarps) {
        const int t = step * G + group;
        const int m = t < b.T ? model_of(b, t, sub == 0) : -1;
        const bool live = m >= 0;
        float z[kC];
        load_row<L, VW>((const TL*)b.logits + (size_t)t * b.ld, b.E, sub, live, z);
        // the chosen experts, their weights' gradients and their logits
        int id[J];
        float gw[J], zj[J];
#pragma unroll
        for (int q = 0; q < J; ++q) {
            const int j = sub + q * L;
            id[q] = -1; gw[q] = 0.f; zj[q] = -INFINITY;
            if (p.d_w && live && j < b.k) {
                const int e = b.topk_idx[(size_t)t * b.k + j];
                if (e >= 0 && e < b.E) {
                    id[q] = e;
                    gw[q] = p.d_w[(size_t)t * b.k + j] * p.scale;
                    zj[q] = clean(to_float(((const TL*)b.logits)[(size_t)t * b.ld + e]));
                } else if (b.status) {
                    atomicOr(b.status, MOE_DEV_BAD_EXPERT);
                }
            }
        }
        float top = z[0];
#pragma unroll
        for (int i = 1; i < kC; ++i) top = fmaxf(top, z[i]);
        top = group_max<L>(top);
        const bool some = top > -INFINITY;
        const float from = some ? top : 0.f;
        // softmax (of sigmoid scores only where the second loss asks for it)
        float soft[kC], soft_inv = 0.f, lse = 0.f;
        if (!SIGMOID || p.d_z) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < kC; ++i) { soft[i] = expf(z[i] - from); sum += soft[i]; }
            sum = group_sum<L>(sum);
            soft_inv = some ? 1.f / sum : 0.f;
            lse = some ? top + logf(sum) : 0.f;
        }
        float d[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) d[i] = 0.f;
        if (p.d_w) {
            float ws[J], inner[J], s = 0.f;
            if (p.renormalize) {
                float best = zj[0];
                if (J > 1) best = fmaxf(best, zj[J - 1]);
                best = group_max<L>(best);
                const float ref = best > -INFINITY ? (SIGMOID ? fminf(best, 0.f) : best) : 0.f;
#pragma unroll
                for (int q = 0; q < J; ++q) { ws[q] = SIGMOID ? sigmoid_from(zj[q], ref) : expf(zj[q] - ref); s += ws[q]; }
                s = group_sum<L>(s);
                const float inv = s > 0.f ? 1.f / s : 0.f;
                s = 0.f;
#pragma unroll
                for (int q = 0; q < J; ++q) { ws[q] *= inv; s = fmaf(gw[q], ws[q], s); }
                s = group_sum<L>(s);
#pragma unroll
                for (int q = 0; q < J; ++q) inner[q] = ws[q] * (gw[q] - s);
            } else {
#pragma unroll
                for (int q = 0; q < J; ++q) {
                    ws[q] = SIGMOID ? sigmoid_from(zj[q], 0.f) : expf(zj[q] - from) * soft_inv;
                    inner[q] = gw[q] * ws[q];
                    s += inner[q];
                }
                if (!SIGMOID) {                               // every expert has its share of the whole
                    s = group_sum<L>(s) * soft_inv;
#pragma unroll
                    for (int i = 0; i < kC; ++i) d[i] = -soft[i] * s;
                }
            }
#pragma unroll
            for (int q = 0; q < J; ++q) if (SIGMOID) inner[q] *= sigmoid_from(-zj[q], 0.f);
            // an expert that was chosen twice gets both, in the order of the choices
            float total[J];
#pragma unroll
            for (int q = 0; q < J; ++q) total[q] = 0.f;
            for (int j = 0; j < b.k; ++j) {
                int other = __shfl_sync(kFull, id[0], (group * L) + (j % L));
                float x = __shfl_sync(kFull, inner[0], (group * L) + (j % L));
                if (J > 1) {
                    const int other1 = __shfl_sync(kFull, id[J - 1], (group * L) + (j % L));
                    const float x1 = __shfl_sync(kFull, inner[J - 1], (group * L) + (j % L));
                    if (j >= L) { other = other1; x = x1; }
                }
#pragma unroll
                for (int q = 0; q < J; ++q) if (other == id[q]) total[q] += x;
            }
#pragma unroll
            for (int q = 0; q < J; ++q) if (id[q] >= 0) add[id[q]] = total[q];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < kC; ++i) d[i] += add[expert_of<L, VW>(sub, i)];
            __syncwarp();
#pragma unroll
            for (int q = 0; q < J; ++q) if (id[q] >= 0) add[id[q]] = 0.f;
            __syncwarp();
        }
        const float n = live && (p.d_loss || p.d_z) ? (float)max(p.tokens[m], 1) : 1.f;
        if (p.d_z) {
            const float c = live ? 2.f * p.d_z[m] / n * soft_inv : 0.f;
#pragma unroll
            for (int i = 0; i < kC; ++i) d[i] = fmaf(soft[i] * c, lse, d[i]);      // (in this order: a share of 0 stays 0)
        }
        if (p.d_loss) {
            const float coef = live ? p.d_loss[m] * ((float)b.E / (float)b.k) / n / n : 0.f;
            float f[kC], share[kC], sum = 0.f;
#pragma unroll
            for (int i = 0; i < kC; ++i) {
                const int e = expert_of<L, VW>(sub, i);
                f[i] = live && e < b.E ? (float)p.counts[(size_t)m * b.E + e] : 0.f;
            }
            if (SIGMOID) {
                const float ref = top > -60.f ? 0.f : from;
#pragma unroll
                for (int i = 0; i < kC; ++i) { share[i] = sigmoid_from(z[i], ref); sum += share[i]; }
                sum = group_sum<L>(sum);
                const float inv = some ? 1.f / sum : 0.f;
#pragma unroll
                for (int i = 0; i < kC; ++i) share[i] *= inv;
            } else {
#pragma unroll
                for (int i = 0; i < kC; ++i) share[i] = soft[i] * soft_inv;
            }
            float mean = 0.f;
#pragma unroll
            for (int i = 0; i < kC; ++i) mean = fmaf(f[i], share[i], mean);
            mean = group_sum<L>(mean);
#pragma unroll
            for (int i = 0; i < kC; ++i) {
                float x = share[i] * (f[i] - mean) * coef;
                if (SIGMOID) x *= sigmoid_from(-z[i], 0.f);
                d[i] += x;
            }
        }
        if (t < b.T) {
            TL* const row = (TL*)p.d_logits + (size_t)t * p.ld_d;
#pragma unroll
            for (int q = 0; q < kC / VW; ++q) {
                const int e0 = (q * L + sub) * VW, n_here = b.E - e0;
                TL v[VW];
#pragma unroll
                for (int j = 0; j < VW; ++j) v[j] = (TL)(live ? d[q * VW + j] : 0.f);
                if (VW > 1 && n_here >= VW) {
                    uint4 u;
                    memcpy(&u, v, sizeof(v) < sizeof(u) ? sizeof(v) : sizeof(u));
                    *reinterpret_cast<uint4*>(row + e0) = u;
                } else {
#pragma unroll
                    for (int j = 0; j < VW; ++j) if (j < n_here) row[e0 + j] = v[j];
                }
            }
        }
    }
}

bool wide_rows(const void* p, int64_t ld, int size) { return (uintptr_t)p % 16 == 0 && ld * size % 16 == 0; }

// the block count of balance_kernel, per model
int balance_blocks(int T, int E, int M)
{
    const int chunks = (T + 31) / 32, all = (chunks + kWarps - 1) / kWarps;
    int most = 148 * 2 / M;
    if (most < 1) most = 1;
    const int blocks = all < most ? all : most;
    return blocks < 1 ? 1 : blocks;
}

template <int L, int VW, typename TL>
cudaError_t run_balance(const BalanceArgs& p, cudaStream_t st)
{
    const dim3 grid(p.blocks, p.b.M), block(32 * kWarps);
    return p.b.score == MOE_SCORE_SIGMOID ? launch_pdl(balance_kernel<L, VW, true, TL>, grid, block, 0, st, p)
                                          : launch_pdl(balance_kernel<L, VW, false, TL>, grid, block, 0, st, p);
}
template <int L, int VW, typename TL>
cudaError_t run_grad(const GateGradArgs& p, cudaStream_t st)
{
    const int steps = (p.b.T + 32 / L - 1) / (32 / L), all = (steps + kWarps - 1) / kWarps, most = 148 * 4;
    const dim3 grid(all < most ? all : most), block(32 * kWarps);
    return p.b.score == MOE_SCORE_SIGMOID ? launch_pdl(gate_grad_kernel<L, VW, true, TL>, grid, block, 0, st, p)
                                          : launch_pdl(gate_grad_kernel<L, VW, false, TL>, grid, block, 0, st, p);
}
// (a macro: the shapes of both kernels)
#define FAASMOE_BY_SHAPE(run, E, wide, bf, ...)                                                                            \
    ((E) <= 64 ? ((bf) ? ((wide) ? run<4, 8, bf16>(__VA_ARGS__) : run<4, 1, bf16>(__VA_ARGS__))                            \
                       : ((wide) ? run<4, 4, float>(__VA_ARGS__) : run<4, 1, float>(__VA_ARGS__)))                         \
   : (E) <= 128 ? ((bf) ? ((wide) ? run<8, 8, bf16>(__VA_ARGS__) : run<8, 1, bf16>(__VA_ARGS__))                           \
                        : ((wide) ? run<8, 4, float>(__VA_ARGS__) : run<8, 1, float>(__VA_ARGS__)))                        \
                : ((bf) ? ((wide) ? run<16, 8, bf16>(__VA_ARGS__) : run<16, 1, bf16>(__VA_ARGS__))                         \
                        : ((wide) ? run<16, 4, float>(__VA_ARGS__) : run<16, 1, float>(__VA_ARGS__))))

}  // namespace

int64_t balance_workspace(int T, int E, int M)
{
    const int blocks = balance_blocks(T, E, M);
    return blocks == 1 ? 0 : (int64_t)blocks * M * record(E) * (int64_t)sizeof(float);
}

cudaError_t launch_balance(const BalanceArgs& in, cudaStream_t st)
{
    BalanceArgs p = in;
    const RouterBatch& b = p.b;
    p.blocks = balance_blocks(b.T, b.E, b.M);
    const bool wide = wide_rows(b.logits, b.ld, b.bf16_logits ? 2 : 4);
    const cudaError_t e = FAASMOE_BY_SHAPE(run_balance, b.E, wide, b.bf16_logits, p, st);
    if (e != cudaSuccess || p.blocks == 1) return e;
    return launch_pdl(balance_finish_kernel, dim3(b.M), dim3(1024), 0, st, p);
}

cudaError_t launch_gate_grad(const GateGradArgs& p, cudaStream_t st)
{
    const RouterBatch& b = p.b;
    const int size = b.bf16_logits ? 2 : 4;
    const bool wide = wide_rows(b.logits, b.ld, size) && wide_rows(p.d_logits, p.ld_d, size);
    return FAASMOE_BY_SHAPE(run_grad, b.E, wide, b.bf16_logits, p, st);
}

}  // namespace faasmoe
