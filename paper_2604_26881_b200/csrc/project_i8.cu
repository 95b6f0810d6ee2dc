// A shared projection in 8-bit integers with a scale for each token and each channel:
//
//   out[t, n] = base[t, n] + bias[n] + xs[t] ws[n] sum_k x[t, k] w[n, k]
//
// The sum runs on the tensor cores (tcgen05.mma, kind::i8: 32-bit integer accumulators in TMEM) and is exact, so it does not depend
// on how K is cut.  Two shapes: for few tokens the weight rows are the M operand and the tokens the N operand, and the CTAs of a
// cluster share K (project_i8_kernel); for many tokens, pairs of CTAs (cta_group::2) walk over tiles of 256 tokens x 256 weight
// rows (project_i8_many_kernel).
#include <cstring>

#include "cluster_ptx.cuh"
#include "project_i8.cuh"

namespace faasmoe {

namespace {

using namespace tc;

__device__ int32_t g_status;            // where the status bits go of calls that have no word for them
__device__ int32_t g_taken;
__global__ void take_status_kernel() { g_taken = atomicExch(&g_status, 0); }

// TMEM: as in the projection in bf16, the CTAs of clusters that fit one SM together ask for 512 columns at most, so that an
// allocation never waits for a cluster that waits for it: project_i8_kernel takes 128 columns at most and more than 12288
// registers (five with 40 a thread do not fit beside one another), project_i8_many_kernel all columns and 198 KB of shared memory.
constexpr uint32_t kFull = 0xffffffffu;
constexpr int kRow = 128;               // bytes of K of a slice: one row of a swizzled tile
constexpr int kRows = 128;              // rows of an operand tile of one CTA
constexpr int kTile = kRows * kRow;     // its bytes
constexpr int kMaxStages = 8;
constexpr int kFewThreads = 352;        // warp 0: TMA (weights), 1: MMA, 2..9: epilogue, 10: TMA (tokens)
constexpr int kMaxSmem = 212 * 1024;

// instruction descriptor: int8 x int8 -> int32, K-major operands
__device__ __forceinline__ uint32_t idesc_i8(int m, int n)
{
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void umma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma_i8_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}

__device__ __forceinline__ float load_base(const I8Args& p, int t, int n)
{
    const size_t at = (size_t)t * p.ldbase + n;
    return p.out_f32 ? ((const float*)p.base)[at] : __bfloat162float(((const bf16*)p.base)[at]);
}
__device__ __forceinline__ void store_out(const I8Args& p, int t, int n, float v)
{
    const size_t at = (size_t)t * p.ldo + n;
    if (p.out_f32) ((float*)p.out)[at] = v;
    else ((bf16*)p.out)[at] = __float2bfloat16_rn(v);
}

struct I8Maps { CUtensorMap x, w; };

// Few tokens: a cluster of `splits` CTAs per tile of 128 weight rows x nt tokens.  Each CTA contracts over its share of K into its
// own accumulator (lane <-> weight row, column <-> token) and sends the others their weight rows' sums (distributed shared memory);
// a CTA adds up, scales and writes 128 / splits rows.
__global__ void __launch_bounds__(kFewThreads)
project_i8_kernel(const I8Args p, const __grid_constant__ I8Maps maps)
{
    extern __shared__ __align__(16) unsigned char smem_dyn[];
    int32_t* const status = p.status ? p.status : &g_status;
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* const ring_ptr = smem_dyn + (ring - smem_u32(smem_dyn));
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_done = bar_full + 16 * kMaxStages, bar_got = bar_done + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = p.splits, nt = p.nt;
    const int rank = blockIdx.x % S;                        // (in a cluster: its rank there)
    const int n0 = (blockIdx.x / S) * kRows, t0 = blockIdx.y * nt;
    const int rows = min(nt, p.T - t0);
    const int nw = kRows / S;                               // weight rows of a CTA
    const int pitch = nt * nw + 16;                         // of an owner's block of sums (16: two owners in a warp meet in no bank)
    const int stage_bytes = kTile + nt * kRow;
    int* const own = reinterpret_cast<int*>(ring_ptr);      // [owner][token][its weight row], in the ring when its stages are done
    int* const part = reinterpret_cast<int*>(ring_ptr + p.scratch);      // [part][token][own weight row]
    const int k0 = (int)((long long)p.ksteps * rank / S), k1 = (int)((long long)p.ksteps * (rank + 1) / S);

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.n_stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_done, 1);
        mbar_init(bar_got, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"((uint32_t)p.columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (S > 1) cluster_arrive();                            // (waited for before anything is sent: the peers run and their barriers are there)
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();

    if (warp == 0 || warp == 10) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
            bool ok = true;
            for (int ks = k0; ks < k1; ++ks) {
                if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, status)) { ok = false; break; }
                const uint32_t sa = ring + stage * stage_bytes, full = bar_full + 8 * stage;
                if (warp == 0) {
                    armed |= 1u << stage;
                    armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                    mbar_expect_tx(full, stage_bytes);
                    tma_load_2d(sa, &maps.w, full, ks * kRow, n0);
                } else {
                    tma_load_2d(sa + kTile, &maps.x, full, ks * kRow, t0);
                }
                if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
            }
            if (!ok && warp == 0)                           // gave up: the copies in flight land before the block exits
                for (int s = 0; s < p.n_stages; ++s)
                    if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, acc = 0;
            bool ok = true;
            const uint32_t idesc = idesc_i8(kRows, nt);
            for (int ks = k0; ks < k1; ++ks) {
                if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
                tc_fence_after();
                const uint32_t lo_a = smem_desc_lo(ring + stage * stage_bytes), lo_b = lo_a + (kTile >> 4);
#pragma unroll
                for (int kk = 0; kk < kRow / 32; ++kk) {
                    umma_i8(tmem, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                    acc = 1;
                }
                umma_commit(bar_empty + 8 * stage);
                if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
            }
            if (ok) umma_commit(bar_done);
        }
        __syncwarp();
    } else {
        // thread <-> weight row (TMEM lane); two groups of four warps take every other 16 tokens each
        const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane, n = n0 + row;
        const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16);
        float ws = 0.f, bias = 0.f;
        if (S == 1 && n < p.N) { ws = p.w_scale[n]; bias = p.bias ? p.bias[n] : 0.f; }
        if (__all_sync(kFull, mbar_wait(bar_done, 0, &s_abort, status))) {
            tc_fence_after();
            int* const dst = own + (row / nw) * pitch + row % nw;
            for (int c = half * 16; c < rows; c += 32) {
                uint32_t r[16];
                tmem_ld16(from + c, r);
                tmem_ld_wait();
                if (S > 1) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) if (c + i < rows) dst[(c + i) * nw] = (int)r[i];
                } else if (n < p.N) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (c + i < rows) {
                            const int t = t0 + c + i;
                            float v = (float)(int)r[i] * p.x_scale[t] * ws + bias;
                            if (p.base) v += load_base(p, t, n);
                            store_out(p, t, n, v);
                        }
                }
            }
            if (S > 1) fence_async_shared();                // (the sums leave by bulk copies)
        }
    }
    tc_fence_before();
    __syncthreads();
    if (S > 1) {
        cluster_wait();
        const int bytes = rows * nw * 4;
        if (warp == 0) {
            if (lane == 0) mbar_expect_tx(bar_got, S * bytes);
            __syncwarp();
            if (lane < S) send_bulk(map_to_cta(smem_u32(part + rank * nt * nw), lane), smem_u32(own + lane * pitch), bytes, map_to_cta(bar_got, lane));
        }
        mbar_wait(bar_got, 0, &s_abort, status);
        __syncwarp();
        cluster_arrive_relaxed();                           // (waited for at the end: nobody leaves while its copies may still be on their way)
        if (!s_abort) {
            for (int e = threadIdx.x; e < rows * nw; e += kFewThreads) {
                const int r = e / nw, n = n0 + rank * nw + e % nw, t = t0 + r;
                if (n >= p.N) continue;
                int sum = 0;
                for (int z = 0; z < S; ++z) sum += part[z * nt * nw + e];
                float v = (float)sum * p.x_scale[t] * p.w_scale[n];
                if (p.bias) v += p.bias[n];
                if (p.base) v += load_base(p, t, n);
                store_out(p, t, n, v);
            }
        }
        __syncwarp();
        cluster_wait();
    }
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)p.columns) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Many tokens: 256 tokens x 256 weight rows per pair of CTAs (each holds 128 of either), pairs that walk over the tiles, two
// accumulators of 256 TMEM columns so that a tile's epilogue runs behind the next tile's MMAs.
constexpr int kManyTile = 256;
constexpr int kManyStages = 5;
constexpr int kManyStageBytes = 2 * kTile;
constexpr int kManyThreads = 352;                      // warp 0: TMA (weights), 1: MMA, 2..9: epilogue, 10: TMA (tokens)
constexpr int kOutPitch = 36;                          // floats per row of a warp's staging area (32 columns, 16-byte rows)
constexpr int kOutStage = 8 * 32 * kOutPitch * (int)sizeof(float);

// 32 tokens x 32 columns (from row t, column n) by a warp, out of its staging area, where the sums are scaled by their tokens: a
// row's columns are read, scaled, added to and written by neighbouring lanes.
template <typename T>
__device__ __forceinline__ void write_block(const I8Args& p, const float* stage, int t, int n, int lane, bool vec)
{
    constexpr int kPer = 16 / sizeof(T), kLanes = 32 / kPer;    // columns of a 16-byte vector; lanes per row, and vectors per lane
    if (vec && n + 32 <= p.N) {
        const int c = (lane % kLanes) * kPer;
        float ws[kPer], add[kPer];
#pragma unroll
        for (int j = 0; j < kPer; j += 4) {
            const float4 f = __ldg(reinterpret_cast<const float4*>(p.w_scale + n + c + j));
            ws[j] = f.x; ws[j + 1] = f.y; ws[j + 2] = f.z; ws[j + 3] = f.w;
            const float4 g = p.bias ? __ldg(reinterpret_cast<const float4*>(p.bias + n + c + j)) : make_float4(0.f, 0.f, 0.f, 0.f);
            add[j] = g.x; add[j + 1] = g.y; add[j + 2] = g.z; add[j + 3] = g.w;
        }
        uint4 q[kLanes];
        if (p.base) {
#pragma unroll
            for (int i = 0; i < kLanes; ++i) {
                const int r = t + i * (32 / kLanes) + lane / kLanes;
                q[i] = r < p.T ? *reinterpret_cast<const uint4*>((const T*)p.base + (size_t)r * p.ldbase + n + c) : make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kLanes; ++i) {
            const int r = i * (32 / kLanes) + lane / kLanes;
            const float4* from = reinterpret_cast<const float4*>(stage + r * kOutPitch + c);
            float v[kPer];
#pragma unroll
            for (int j = 0; j < kPer / 4; ++j) { const float4 f = from[j]; v[4 * j] = f.x; v[4 * j + 1] = f.y; v[4 * j + 2] = f.z; v[4 * j + 3] = f.w; }
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = v[j] * ws[j] + add[j];
            uint4 o;
            if constexpr (sizeof(T) == 4) {
                if (p.base) {
                    v[0] += __uint_as_float(q[i].x); v[1] += __uint_as_float(q[i].y); v[2] += __uint_as_float(q[i].z); v[3] += __uint_as_float(q[i].w);
                }
                o = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
            } else {
                if (p.base) {
                    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q[i]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { const float2 f = __bfloat1622float2(h[j]); v[2 * j] += f.x; v[2 * j + 1] += f.y; }
                }
                __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            }
            if (t + r < p.T) *reinterpret_cast<uint4*>((T*)p.out + (size_t)(t + r) * p.ldo + n + c) = o;
        }
    } else if (n + lane < p.N) {
        // rows that are not on 16-byte boundaries: a row's 32 columns at a time, eight rows' bases on their way at once
        T* out = (T*)p.out + (size_t)t * p.ldo + n + lane;
        const T* base = (const T*)p.base + (size_t)t * p.ldbase + n + lane;
        const float ws = p.w_scale[n + lane], add = p.bias ? p.bias[n + lane] : 0.f;
        const int rows = min(32, p.T - t);
#pragma unroll 1
        for (int r0 = 0; r0 < rows; r0 += 8) {
            T b[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = p.base && r0 + i < rows ? base[(r0 + i) * p.ldbase] : (T)0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r0 + i < rows) {
                    const float v = stage[(r0 + i) * kOutPitch + lane] * ws + add;
                    out[(r0 + i) * p.ldo] = (T)(p.base ? v + (float)b[i] : v);
                }
        }
    }
}

__global__ void __launch_bounds__(kManyThreads, 1)
project_i8_many_kernel(const I8Args p, const __grid_constant__ I8Maps maps)
{
    extern __shared__ __align__(16) unsigned char smem_dyn[];
    int32_t* const status = p.status ? p.status : &g_status;
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* const ring_ptr = smem_dyn + (ring - smem_u32(smem_dyn));
    __shared__ __align__(8) uint64_t s_bars[2 * kManyStages + 4];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kManyStages, bar_tfull = bar_full + 16 * kManyStages, bar_tempty = bar_tfull + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const int n_tiles = (p.N + kManyTile - 1) / kManyTile, m_tiles = (p.T + kManyTile - 1) / kManyTile;
    const long long total = (long long)n_tiles * m_tiles;
    const int pair0 = blockIdx.x >> 1, pairs = gridDim.x >> 1;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kManyStages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bar_tfull + 8 * b, 1); mbar_init(bar_tempty + 8 * b, 2 * 8); }
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                     // the peer's barriers are there before anything is signalled on them
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();

    if (warp == 0 || warp == 10) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
            bool ok = true;
            for (long long tile = pair0; tile < total && ok; tile += pairs) {
                const int n0 = (int)(tile / m_tiles) * kManyTile + rank * kRows, t0 = (int)(tile % m_tiles) * kManyTile + rank * kRows;
                for (int ks = 0; ks < p.ksteps; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, status)) { ok = false; break; }
                    const uint32_t sa = ring + stage * kManyStageBytes, full = bar_full + 8 * stage;
                    if (warp == 0) {
                        armed |= 1u << stage;
                        armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                        if (leader) mbar_expect_tx(full, 2 * kManyStageBytes);
                        tma_load_2d_pair(sa + kTile, &maps.w, full, ks * kRow, n0);
                    } else {
                        tma_load_2d_pair(sa, &maps.x, full, ks * kRow, t0);
                    }
                    if (++stage == (uint32_t)kManyStages) { stage = 0; phase ^= 1; }
                }
            }
            if (!ok && leader && warp == 0)                 // gave up: the copies in flight land before the block exits
                for (int s = 0; s < kManyStages; ++s)
                    if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            const uint32_t idesc = idesc_i8(256, 256);
            int it = 0;
            for (long long tile = pair0; tile < total && ok; tile += pairs, ++it) {
                const uint32_t buf = it & 1, d = tmem + buf * 256;
                if (!mbar_wait_cluster(bar_tempty + 8 * buf, ((it >> 1) & 1) ^ 1, &s_abort, status)) { ok = false; break; }
                tc_fence_after();
                uint32_t acc = 0;
                for (int ks = 0; ks < p.ksteps; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t lo_a = smem_desc_lo(ring + stage * kManyStageBytes), lo_b = lo_a + (kTile >> 4);
#pragma unroll
                    for (int kk = 0; kk < kRow / 32; ++kk) {
                        umma_i8_pair(d, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                        acc = 1;
                    }
                    umma_commit_pair(bar_empty + 8 * stage);
                    if (++stage == (uint32_t)kManyStages) { stage = 0; phase ^= 1; }
                }
                if (ok) umma_commit_pair(bar_tfull + 8 * buf);
            }
        }
        __syncwarp();
    } else {
        // ---- epilogue: thread <-> token (TMEM lane), four warps per half of the columns ----
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t tempty_leader = map_to_cta(bar_tempty, 0);
        const int esz = p.out_f32 ? 4 : 2;
        const bool vec = (uintptr_t)p.out % 16 == 0 && p.ldo * esz % 16 == 0 && (!p.base || ((uintptr_t)p.base % 16 == 0 && p.ldbase * esz % 16 == 0)) &&
                         (uintptr_t)p.w_scale % 16 == 0 && (uintptr_t)p.bias % 16 == 0;
        float* const stage = reinterpret_cast<float*>(ring_ptr + kManyStages * kManyStageBytes) + (warp - 2) * 32 * kOutPitch;
        int it = 0;
        for (long long tile = pair0; tile < total; tile += pairs, ++it) {
            const int n0 = (int)(tile / m_tiles) * kManyTile + half * 128, t = (int)(tile % m_tiles) * kManyTile + (int)rank * kRows + quarter * 32;
            const uint32_t buf = it & 1, from = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16) + half * 128;
            const float xs = t + lane < p.T ? p.x_scale[t + lane] : 0.f;
            if (!__all_sync(kFull, mbar_wait(bar_tfull + 8 * buf, (it >> 1) & 1, &s_abort, status))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 128; c += 32) {
                uint32_t r[32];
                tmem_ld16(from + c, r);
                tmem_ld16(from + c + 16, r + 16);
                tmem_ld_wait();
                if (c == 96) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(tempty_leader + 8 * buf);
                }
                if (n0 + c >= p.N || t >= p.T) continue;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    reinterpret_cast<float4*>(stage + lane * kOutPitch)[i] = make_float4((float)(int)r[4 * i] * xs, (float)(int)r[4 * i + 1] * xs,
                                                                                          (float)(int)r[4 * i + 2] * xs, (float)(int)r[4 * i + 3] * xs);
                __syncwarp();
                if (p.out_f32) write_block<float>(p, stage, t, n0 + c, lane, vec);
                else write_block<bf16>(p, stage, t, n0 + c, lane, vec);
                __syncwarp();
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                     // nobody leaves while the peer may still read this CTA's memory or signal it
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// 2-D map over `rows` x `k` bytes whose rows are ld apart; box = 128 x box_rows, 128-byte swizzle
bool make_map_i8(CUtensorMap* m, const void* base, uint64_t rows, uint64_t k, uint64_t ld, uint32_t box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {k, rows};
    cuuint64_t strides[1] = {ld};
    cuuint32_t box[2] = {(cuuint32_t)kRow, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// the opt-in to large dynamic shared memory is a per-device attribute of a kernel
template <typename K>
cudaError_t allow_smem(K kern, bool (&done)[kMaxDevices])
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
    if (done[dev]) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem);
    if (e == cudaSuccess) done[dev] = true;
    return e;
}

int div_up(int a, int b) { return (a + b - 1) / b; }

}  // namespace

cudaError_t take_project_i8_status(int32_t* status_host)
{
    take_status_kernel<<<1, 1>>>();
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? cudaMemcpyFromSymbol(status_host, g_taken, sizeof(int32_t)) : e;
}

cudaError_t launch_project_i8(const I8Args& in, cudaStream_t st)
{
    I8Args p = in;
    static bool few_ok[kMaxDevices] = {false}, many_ok[kMaxDevices] = {false};
    p.ksteps = div_up(p.K, kRow);

    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.stream = st;
    I8Maps maps;

    if (p.T > 128) {
        cudaError_t e = allow_smem(project_i8_many_kernel, many_ok);
        if (e != cudaSuccess) return e;
        if (!make_map_i8(&maps.x, p.x, p.T, p.K, p.ldx, kRows) || !make_map_i8(&maps.w, p.w, p.N, p.K, p.ldw, kRows)) return cudaErrorInvalidValue;
        const long long tiles = (long long)div_up(p.N, kManyTile) * div_up(p.T, kManyTile);
        const int pairs = tiles < 74 ? (int)tiles : 74;
        attr[1].val.clusterDim.x = 2;
        cfg.gridDim = dim3(2 * pairs); cfg.blockDim = dim3(kManyThreads); cfg.numAttrs = 2;
        cfg.dynamicSmemBytes = kManyStages * kManyStageBytes + kOutStage + 1024;
        return cudaLaunchKernelEx(&cfg, project_i8_many_kernel, p, maps);
    }
    cudaError_t e = allow_smem(project_i8_kernel, few_ok);
    if (e != cudaSuccess) return e;
    p.nt = ((p.T < 128 ? p.T : 128) + 15) & ~15;
    p.columns = p.nt <= 32 ? 32 : (p.nt <= 64 ? 64 : 128);
    const int n_tiles = div_up(p.N, kRows), m_tiles = div_up(p.T, p.nt);
    p.splits = 8;
    while (p.splits > 1 && ((long long)p.splits * n_tiles * m_tiles > 148 || p.ksteps < 2 * p.splits)) p.splits /= 2;
    const int stage_bytes = kTile + p.nt * kRow, want = div_up(p.ksteps, p.splits);
    const int own = p.splits > 1 ? p.splits * (p.nt * (kRows / p.splits) + 16) * 4 : 0, got = p.splits > 1 ? p.nt * kRows * 4 : 0;
    p.n_stages = (kMaxSmem - 1024 - got) / stage_bytes;
    if (p.n_stages > 6) p.n_stages = 6;
    if (p.n_stages > want) p.n_stages = want;
    p.scratch = p.n_stages * stage_bytes;
    if (p.scratch < own) p.scratch = own;
    if (!make_map_i8(&maps.x, p.x, p.T, p.K, p.ldx, p.nt) || !make_map_i8(&maps.w, p.w, p.N, p.K, p.ldw, kRows)) return cudaErrorInvalidValue;
    cfg.gridDim = dim3(n_tiles * p.splits, m_tiles); cfg.blockDim = dim3(kFewThreads);
    cfg.dynamicSmemBytes = (size_t)p.scratch + got + 1024;
    attr[1].val.clusterDim.x = p.splits;
    cfg.numAttrs = p.splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, project_i8_kernel, p, maps);
}

}  // namespace faasmoe
