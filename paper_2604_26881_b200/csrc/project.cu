// A shared projection with the tenants' low-rank adapters:
//
//   out[t] = base[t] + x[t] . W^T + scale[a] * (x[t] . A[a]^T) . B[a]^T,     a = adapter of token t's tenant
//
// Two launches.  The first computes u[t] = scale[a] * x[t] . A[a]^T (adapter_kernel): per 128 tokens the distinct adapters
// are listed, their rows are gathered by TMA as the N operand of one tcgen05.mma per 16 elements of K, and each token keeps
// the columns of its own adapter.  K is cut over CTAs; the parts of u are stored apart in fp32 and summed in a
// fixed order by the second launch, which is resident and streams W meanwhile (programmatic dependent launch) and adds
// u . B^T behind its main loop.
#include <cstring>

#include "project.cuh"
#include "tc_ptx.cuh"

namespace faasmoe {

namespace {

using namespace tc;

constexpr uint32_t kFull = 0xffffffffu;
constexpr int kTok = 128;               // tokens per tile: the M operand, one TMEM lane each
constexpr int kBK = 64;                 // K elements per slice: one 128-byte row of a swizzled tile
constexpr int kMaxStages = 8;
constexpr int kUCols = 128;             // columns of one CTA of the first product
constexpr int kUThreads = 192;          // warp 0: TMA, 1: MMA, 2..5: lists and epilogue
constexpr int kPN = 128;                // weight rows per tile of the projection
constexpr int kPThreads = 352;          // warp 0: TMA (weights), 1: MMA, 2..9: epilogue, 10: TMA (tokens)

__device__ __forceinline__ uint32_t cluster_ctarank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t map_to_cta(uint32_t local_addr, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(local_addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// instruction descriptor: bf16 x bf16 -> fp32, K-major operands, M = 128
__device__ __forceinline__ uint32_t idesc_bf16(int n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}

// Adapter of token t, or -1.  Ids outside their range set a status bit and count as none.
__device__ __forceinline__ int adapter_of(const ProjectArgs& p, int t, bool report)
{
    const int u = p.tenant_id[t];
    if (u < 0 || u >= p.n_tenants) {
        if (report) atomicOr(p.status, MOE_DEV_BAD_TENANT);
        return -1;
    }
    const int a = p.adapter_of_tenant ? p.adapter_of_tenant[u] : u;
    if (a < 0) return -1;
    if (a >= p.n_adapters) {
        if (report && p.adapter_of_tenant) atomicOr(p.status, MOE_DEV_BAD_ADAPTER);
        return -1;
    }
    return a;
}

struct UMaps { CUtensorMap x, a; };

// blockIdx: x = token tile, y = chunk of the tile's distinct adapters, z = part of K
__global__ void __launch_bounds__(kUThreads)
adapter_kernel(const ProjectArgs p, const __grid_constant__ UMaps maps)
{
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 1];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_count;
    __shared__ int s_adapter[kTok], s_first[kTok], s_list[kTok], s_warp_count[4];
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_done = bar_full + 16 * kMaxStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t0 = blockIdx.x * kTok;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.n_stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_done, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"((uint32_t)kUCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    pdl_launch_dependents();        // (after the wait: the projection may read x before it waits itself)

    // the tile's distinct adapters, in the order of their first token
    const int tok = threadIdx.x - 64, t = t0 + tok;
    if (warp >= 2) s_adapter[tok] = t < p.T ? adapter_of(p, t, blockIdx.y == 0 && blockIdx.z == 0) : -1;
    __syncthreads();
    int mine = -1, first = kTok;
    bool leads = false;
    uint32_t leaders = 0;
    if (warp >= 2) {
        mine = s_adapter[tok];
        for (int j = kTok - 1; j >= 0; --j) if (s_adapter[j] == mine) first = j;
        leads = mine >= 0 && first == tok;
        leaders = __ballot_sync(kFull, leads);
        if (lane == 0) s_warp_count[warp - 2] = __popc(leaders);
    }
    __syncthreads();
    if (warp >= 2) {
        int at = 0;
        for (int w = 0; w < warp - 2; ++w) at += s_warp_count[w];
        at += __popc(leaders & ((1u << lane) - 1));
        if (leads) { s_list[at] = mine; s_first[tok] = at; }
        if (threadIdx.x == 64) s_count = s_warp_count[0] + s_warp_count[1] + s_warp_count[2] + s_warp_count[3];
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    const int slot0 = blockIdx.y * p.slots;
    const int n_slots = min(p.slots, s_count - slot0);                 // adapters of this CTA
    if (n_slots > 0) {
        const int k0 = (int)((long long)p.ksteps * blockIdx.z / p.u_splits), k1 = (int)((long long)p.ksteps * (blockIdx.z + 1) / p.u_splits);
        const int cols = (n_slots * p.rank + 15) & ~15;                 // (rank 8 and an odd number: eight stale columns, never read)
        if (warp == 0) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
                bool ok = true;
                for (int ks = k0; ks < k1; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, p.status)) { ok = false; break; }
                    const uint32_t sa = ring + stage * p.stage_bytes, sb = sa + p.a_bytes, full = bar_full + 8 * stage;
                    armed |= 1u << stage;
                    armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                    mbar_expect_tx(full, (p.a_rows + n_slots * p.rank) * kBK * 2);
                    tma_load_2d(sa, &maps.x, full, ks * kBK, t0);
                    for (int j = 0; j < n_slots; ++j)
                        tma_load_2d(sb + j * p.rank * kBK * 2, &maps.a, full, ks * kBK, s_list[slot0 + j] * p.rank);
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (!ok)
                    for (int s = 0; s < p.n_stages; ++s)
                        if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, p.status);
            }
            __syncwarp();
        } else if (warp == 1) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, acc = 0;
                bool ok = true;
                const uint32_t idesc = idesc_bf16(cols);
                for (int ks = k0; ks < k1; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, p.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t lo_a = smem_desc_lo(ring + stage * p.stage_bytes), lo_b = lo_a + (p.a_bytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) {
                        umma_bf16(tmem, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                        acc = 1;
                    }
                    umma_commit(bar_empty + 8 * stage);
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (ok) umma_commit(bar_done);
            }
            __syncwarp();
        } else {
            // thread <-> token; a warp reads the TMEM lanes of its quarter
            const int quarter = warp & 3, row = quarter * 32 + lane, tr = t0 + row;
            const int a = s_adapter[row];
            int f = 0;
            if (a >= 0) {
                while (s_adapter[f] != a) ++f;                          // the adapter's first token knows its place in the list
                f = s_first[f] - slot0;
            }
            const bool live = a >= 0 && f >= 0 && f < n_slots;
            const float s = live ? (p.scale ? p.scale[a] : 1.f) : 0.f;
            float* dst = p.u + ((size_t)blockIdx.z * p.T + tr) * p.rank;
            const int c_lo = live ? f * p.rank : cols, c_hi = live ? c_lo + p.rank : 0;
            if (__all_sync(kFull, mbar_wait(bar_done, 0, &s_abort, p.status))) {
                tc_fence_after();
                for (int c = 0; c < cols; c += 16) {
                    if (!__any_sync(kFull, c + 16 > c_lo && c < c_hi)) continue;
                    uint32_t r[16];
                    tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int h = 0; h < 16; h += 8)
                        if (c + h >= c_lo && c + h < c_hi) {
                            float4* o = reinterpret_cast<float4*>(dst + (c + h - c_lo));
                            o[0] = make_float4(s * __uint_as_float(r[h]), s * __uint_as_float(r[h + 1]), s * __uint_as_float(r[h + 2]), s * __uint_as_float(r[h + 3]));
                            o[1] = make_float4(s * __uint_as_float(r[h + 4]), s * __uint_as_float(r[h + 5]), s * __uint_as_float(r[h + 6]), s * __uint_as_float(r[h + 7]));
                        }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kUCols) : "memory");
    }
}

struct PMaps { CUtensorMap x, w; };

// One cluster of `splits` CTAs per tile of 128 tokens x 128 weight rows; each CTA contracts over its share of K into its
// own TMEM accumulator, leaves the sums in shared memory, and adds up a share of the columns over the cluster (distributed
// shared memory, ranks in order: the same bits every time).  The adapters' second product and the base are added there, in fp32.
__global__ void __launch_bounds__(kPThreads)
project_kernel(const ProjectArgs p, const __grid_constant__ PMaps maps)
{
    extern __shared__ unsigned char smem_dyn[];
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    float* const part = reinterpret_cast<float*>(smem_dyn + (ring - smem_u32(smem_dyn)));      // the ring, when its stages are done
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 1];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ int s_adapter[kTok];
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_done = bar_full + 16 * kMaxStages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = p.splits;
    const uint32_t rank = S > 1 ? cluster_ctarank() : 0u;
    const int n0 = (blockIdx.x / S) * kPN, t0 = blockIdx.y * kTok;
    const int rows = min(kTok, p.T - t0);
    const int pitch = p.a_rows + 1;                       // part[column][token], odd pitch: no bank conflicts either way
    const bool product = p.ksteps > 0, adapters = p.n_adapters > 0;

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.n_stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_done, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"((uint32_t)kPN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    // With adapters the launch before this one is adapter_kernel, which had waited for everything before it when it let this
    // kernel start: x, W and the tenant ids are complete.  Without, it is some other kernel.
    if (!adapters) pdl_wait();
    pdl_launch_dependents();

    if (product) {
        const int k0 = (int)((long long)p.ksteps * rank / S), k1 = (int)((long long)p.ksteps * (rank + 1) / S);
        if (warp == 0 || warp == 10) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
                bool ok = true;
                for (int ks = k0; ks < k1; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, p.status)) { ok = false; break; }
                    const uint32_t sa = ring + stage * p.stage_bytes, full = bar_full + 8 * stage;
                    armed |= 1u << stage;
                    armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                    if (warp == 0) {
                        mbar_expect_tx(full, (p.a_rows + kPN) * kBK * 2);
                        tma_load_2d(sa + p.a_bytes, &maps.w, full, ks * kBK, n0);
                    } else {
                        tma_load_2d(sa, &maps.x, full, ks * kBK, t0);
                    }
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (!ok && warp == 0)
                    for (int s = 0; s < p.n_stages; ++s)
                        if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, p.status);
            }
            __syncwarp();
        } else if (warp == 1) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, acc = 0;
                bool ok = true;
                const uint32_t idesc = idesc_bf16(kPN);
                for (int ks = k0; ks < k1; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, p.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t lo_a = smem_desc_lo(ring + stage * p.stage_bytes), lo_b = lo_a + (p.a_bytes >> 4);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) {
                        umma_bf16(tmem, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                        acc = 1;
                    }
                    umma_commit(bar_empty + 8 * stage);
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (ok) umma_commit(bar_done);
            }
            __syncwarp();
        } else {
            const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane;
            if (__all_sync(kFull, mbar_wait(bar_done, 0, &s_abort, p.status)) && quarter * 32 < rows) {
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < kPN / 2; c += 16) {
                    uint32_t r[16];
                    tmem_ld16(tmem + ((uint32_t)(quarter * 32) << 16) + half * (kPN / 2) + c, r);
                    tmem_ld_wait();
                    if (row < rows) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) part[(half * (kPN / 2) + c + i) * pitch + row] = __uint_as_float(r[i]);
                    }
                }
            }
        }
    }
    if (adapters) {
        pdl_wait();                                        // u
        for (int i = threadIdx.x; i < rows; i += kPThreads) s_adapter[i] = adapter_of(p, t0 + i, false);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    float* const su = part + (size_t)kPN * pitch;          // u of the tile's tokens, summed over the parts of K
    if (adapters) {
        for (int i = threadIdx.x; i < rows * p.rank; i += kPThreads) {
            const int r = i / p.rank;
            float v = 0.f;
            if (s_adapter[r] >= 0) {
                const float* src = p.u + (size_t)t0 * p.rank + i;
                for (int s = 0; s < p.u_splits; ++s) v += __ldcg(src + (size_t)s * p.T * p.rank);
            }
            su[i] = v;
        }
    }
    if (S > 1) cluster_sync_all(); else __syncthreads();
    if (!s_abort) {
        const int nc = kPN / S, c0 = rank * nc;            // this CTA's columns of the tile
        const uint32_t part_addr = smem_u32(part);
        for (int e = threadIdx.x; e < rows * nc; e += kPThreads) {
            const int c = c0 + (e & (nc - 1)), r = e / nc, n = n0 + c;
            if (n >= p.N) continue;
            float v = 0.f;
            if (product) {
                if (S > 1) {
                    for (int s = 0; s < S; ++s) v += ld_cluster_f32(map_to_cta(part_addr + 4 * (c * pitch + r), s));
                } else {
                    v = part[c * pitch + r];
                }
            }
            if (adapters) {
                const int a = s_adapter[r];
                if (a >= 0) {
                    const uint4* bp = reinterpret_cast<const uint4*>(p.b + ((size_t)a * p.N + n) * p.rank);
                    const float* up = su + r * p.rank;
                    float d = 0.f;
                    for (int i = 0; i < p.rank / 8; ++i) {
                        const uint4 q = __ldg(bp + i);
                        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 f = __bfloat1622float2(h[j]);
                            d = fmaf(up[8 * i + 2 * j], f.x, d);
                            d = fmaf(up[8 * i + 2 * j + 1], f.y, d);
                        }
                    }
                    v += d;
                }
            }
            const size_t row = t0 + r;
            if (p.out_f32) {
                if (p.base) v += ((const float*)p.base)[row * p.ldbase + n];
                ((float*)p.out)[row * p.ldo + n] = v;
            } else {
                if (p.base) v += __bfloat162float(((const bf16*)p.base)[row * p.ldbase + n]);
                ((bf16*)p.out)[row * p.ldo + n] = __float2bfloat16_rn(v);
            }
        }
    }
    tc_fence_before();
    if (S > 1) cluster_sync_all(); else __syncthreads();   // nobody leaves while a peer may still read its sums
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kPN) : "memory");
    }
}

// 2-D map over `rows` x `k` bf16 whose rows are ld elements apart; box = 64 x box_rows, 128-byte swizzle
bool make_map_ld(CUtensorMap* m, const void* base, uint64_t rows, uint64_t k, uint64_t ld, uint32_t box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {k, rows};
    cuuint64_t strides[1] = {ld * 2};
    cuuint32_t box[2] = {(cuuint32_t)kBK, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kMaxSmem = 224 * 1024;

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

// Parts of K of the first product: about one CTA per SM over the token tiles, at least two slices each
int u_parts(int T, int K)
{
    const int tiles = div_up(T, kTok), steps = div_up(K, kBK);
    int s = 1;
    while (s < 8 && tiles * s * 2 <= 148 && steps / (s * 2) >= 2) s *= 2;
    return s;
}

}  // namespace

int64_t project_workspace(int T, int K, int rank, int n_adapters)
{
    if (n_adapters == 0 || T == 0) return kProjectHeader;
    return kProjectHeader + (int64_t)u_parts(T, K) * T * rank * (int64_t)sizeof(float);
}

cudaError_t launch_project(const ProjectArgs& in, cudaStream_t st)
{
    ProjectArgs p = in;
    static bool u_ok[kMaxDevices] = {false}, p_ok[kMaxDevices] = {false};
    const int m_tiles = div_up(p.T, kTok);
    p.a_rows = p.T >= kTok ? kTok : ((p.T + 7) & ~7);
    p.a_bytes = (p.a_rows * kBK * 2 + 1023) & ~1023;
    p.u = reinterpret_cast<float*>(p.workspace + kProjectHeader);
    p.u_splits = u_parts(p.T, p.K);
    if (p.n_adapters > 0) {
        cudaError_t e = allow_smem(adapter_kernel, u_ok);
        if (e != cudaSuccess) return e;
        UMaps um;
        if (!make_map_ld(&um.x, p.x, p.T, p.K, p.ldx, p.a_rows) ||
            !make_map_ld(&um.a, p.a, (uint64_t)p.n_adapters * p.rank, p.K, p.K, p.rank))
            return cudaErrorInvalidValue;
        ProjectArgs q = p;
        q.slots = kUCols / p.rank;
        q.ksteps = div_up(p.K, kBK);
        q.stage_bytes = p.a_bytes + kUCols * kBK * 2;
        q.n_stages = 4;
        const int chunks = div_up(p.T < kTok ? (p.T < p.n_adapters ? p.T : p.n_adapters) : (kTok < p.n_adapters ? kTok : p.n_adapters), q.slots);
        // (an MMA always reads 128 token rows: the last stage's tile is followed by the rows it may reach)
        const size_t smem = (size_t)q.n_stages * q.stage_bytes + kTok * kBK * 2 + 1024;
        e = launch_pdl(adapter_kernel, dim3(m_tiles, chunks, p.u_splits), dim3(kUThreads), smem, st, q, um);
        if (e != cudaSuccess) return e;
    }
    cudaError_t e = allow_smem(project_kernel, p_ok);
    if (e != cudaSuccess) return e;
    PMaps pm;
    memset(&pm, 0, sizeof(pm));
    p.ksteps = p.w ? div_up(p.K, kBK) : 0;
    if (p.w && (!make_map_ld(&pm.x, p.x, p.T, p.K, p.ldx, p.a_rows) || !make_map_ld(&pm.w, p.w, p.N, p.K, p.ldw, kPN)))
        return cudaErrorInvalidValue;
    const int n_tiles = div_up(p.N, kPN);
    p.splits = 1;
    while (p.splits < 8 && n_tiles * m_tiles * p.splits * 2 <= 148 && p.ksteps / (p.splits * 2) >= 2) p.splits *= 2;
    p.stage_bytes = p.a_bytes + kPN * kBK * 2;
    p.n_stages = div_up(p.ksteps, p.splits);
    if (p.n_stages > 6) p.n_stages = 6;
    if (p.n_stages < 1) p.n_stages = 1;
    size_t smem = (size_t)p.n_stages * p.stage_bytes + kTok * kBK * 2;
    const size_t scratch = ((size_t)kPN * (p.a_rows + 1) + (size_t)(p.n_adapters > 0 ? p.a_rows * p.rank : 0)) * sizeof(float);
    if (smem < scratch) smem = scratch;
    smem += 1024;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cfg.gridDim = dim3(n_tiles * p.splits, m_tiles); cfg.blockDim = dim3(kPThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = p.splits; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = p.splits > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, project_kernel, p, pm);
}

}  // namespace faasmoe
