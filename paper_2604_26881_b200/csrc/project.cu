// A shared projection with the tenants' low-rank adapters:
//
//   out[t] = base[t] + x[t] . W^T + scale[a] * (x[t] . A[a]^T) . B[a]^T,     a = adapter of token t's tenant
//
// u[t] = scale[a] * x[t] . A[a]^T, the first product, comes from a launch of its own (adapter_kernel): per 128 tokens the
// distinct adapters are listed, their rows are gathered by TMA as the N operand of one tcgen05.mma per 16 elements of K, and
// each token keeps the columns of its own adapter; K is cut over the CTAs of a cluster, which add up their parts in a fixed
// order.  The projection (project_kernel for few tokens, project_many_kernel for many) is resident and streams W meanwhile
// (programmatic dependent launch) and adds u . B^T behind its main loop.  For a handful of tokens it computes u itself, in the
// same pass over x, and there is one launch only.
//
// Few tokens are a chain of latencies (ids, list, TMA, MMA, exchange in the cluster, the launch boundary, second product), not
// bytes: 2048 -> 2048, rank 16, one token 9.8 us (8.5 MB, 1.3 us of HBM time); 2048 -> 5632, 32 tokens of 32 adapters 13.6 us
// (31.8 MB, 4.9 us).  Many tokens are bound by the tensor cores: 5632 -> 2048, 4096 tokens of 16 adapters of rank 16 77 to 78 us (95
// GFLOP, 1.23 PFLOP/s, 0.75 of the measured burst peak) in short runs, 87 to 92 back to back, where the power cap lowers the clock; the
// adapters alone beside a base, 1126 tokens, 13 of rank 64: 28 us, first product 12 of them.
#include <cstring>

#include "project.cuh"
#include "tc_ptx.cuh"

namespace faasmoe {

namespace {

using namespace tc;

__device__ int32_t g_project_status;      // where the status bits go of calls that have no word for them
__device__ int32_t g_project_taken;
__global__ void take_status_kernel() { g_project_taken = atomicExch(&g_project_status, 0); }

// TMEM: the CTAs of these kernels that fit one SM together ask for 512 columns at most (by registers two of project_kernel, 256
// columns each at most, or one and two of adapter_kernel, 128, or four of those), and a kernel that takes all 512 leaves no
// shared memory for a cluster of either.  So an allocation never waits for a cluster that waits for it, whatever other streams run.
constexpr uint32_t kFull = 0xffffffffu;
constexpr int kTok = 128;               // tokens per tile: the M operand, one TMEM lane each
constexpr int kBK = 64;                 // K elements per slice: one 128-byte row of a swizzled tile
constexpr int kMaxStages = 8;
constexpr int kUTerms = 3;              // bf16 numbers that add up to an fp32 one: 8 bits each
constexpr int kUCols = 128;             // columns of one CTA of the first product
constexpr int kUThreads = 288;          // warp 0: TMA (tokens), 1, 7: MMA, 2..5: lists and epilogue, 6, 8: TMA (rows of A)
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
// Copies shared memory of this CTA to another of the cluster; the bytes are counted on a barrier of the receiver.  (Single
// remote stores were measured at about 30 cycles each, one after the other: 4 us for one token's sums in a cluster of eight.)
__device__ __forceinline__ void send_bulk(uint32_t dst, uint32_t src, uint32_t bytes, uint32_t bar)
{
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "r"(src), "r"(bytes), "r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
// (nothing that was written before is handed over: only that this CTA has come so far)
__device__ __forceinline__ void cluster_arrive_relaxed() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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
__device__ __forceinline__ int32_t* status_of(const ProjectArgs& p) { return p.status ? p.status : &g_project_status; }
__device__ __forceinline__ int adapter_of(const ProjectArgs& p, int t, bool report)
{
    const int u = p.tenant_id[t];
    if (u < 0 || u >= p.n_tenants) {
        if (report) atomicOr(status_of(p), MOE_DEV_BAD_TENANT);
        return -1;
    }
    const int a = p.adapter_of_tenant ? p.adapter_of_tenant[u] : u;
    if (a < 0) return -1;
    if (a >= p.n_adapters) {
        if (report && p.adapter_of_tenant) atomicOr(status_of(p), MOE_DEV_BAD_ADAPTER);
        return -1;
    }
    return a;
}

// The distinct adapters of a tile of 32 * G tokens, in the order of their first token; four warps work on it, warp w on the
// groups of 32 tokens w and w + 4.  `sync` is a barrier of (at least) those warps.  Every token looks for the first one with its
// adapter by comparing with all earlier ones, four at a time: no step depends on how many there are or whose turn it is
// (walks along lists of the adapters found so far took up to 1 us).
template <int G>
struct AdapterList {
    alignas(16) int adapter[32 * G];    // of every token, -1: none
    int list[32 * G];
    uint32_t fresh[G];                  // the tokens that are the first with their adapter
    int count;
};
template <int G, typename Sync>
__device__ __forceinline__ void list_adapters(const ProjectArgs& p, AdapterList<G>& s, int t0, int w, int lane, bool report, Sync sync, int (&slot)[G / 4])
{
    int a[G / 4], first[G / 4];
#pragma unroll
    for (int i = 0; i < G / 4; ++i) {
        const int g = w + 4 * i, t = t0 + g * 32 + lane;
        a[i] = t < p.T ? adapter_of(p, t, report) : -1;
        s.adapter[g * 32 + lane] = a[i];
        first[i] = g * 32 + __ffs(__match_any_sync(kFull, a[i])) - 1;
    }
    sync();
#pragma unroll
    for (int i = 0; i < G / 4; ++i) {
        const int g = w + 4 * i;
        for (int h = g - 1; h >= 0; --h) {
#pragma unroll
            for (int q = 7; q >= 0; --q) {
                const int4 v = reinterpret_cast<const int4*>(s.adapter)[h * 8 + q];
                const int at = h * 32 + q * 4;
                if (v.w == a[i]) first[i] = at + 3;
                if (v.z == a[i]) first[i] = at + 2;
                if (v.y == a[i]) first[i] = at + 1;
                if (v.x == a[i]) first[i] = at;
            }
        }
        const uint32_t fresh = __ballot_sync(kFull, a[i] >= 0 && first[i] == g * 32 + lane);
        if (lane == 0) s.fresh[g] = fresh;
    }
    sync();
    uint32_t fresh[G];
    int count = 0;
#pragma unroll
    for (int h = 0; h < G; ++h) {
        fresh[h] = s.fresh[h];
        count += __popc(fresh[h]);
    }
#pragma unroll
    for (int i = 0; i < G / 4; ++i) {
        int at = 0;
#pragma unroll
        for (int h = 0; h < G; ++h) {
            const int d = first[i] - 32 * h;                // (bits of the group that are before the first token)
            at += __popc(d >= 32 ? fresh[h] : (d > 0 ? fresh[h] & ((1u << d) - 1) : 0u));
        }
        slot[i] = a[i] >= 0 ? at : -1;
        if (a[i] >= 0 && first[i] == (w + 4 * i) * 32 + lane) s.list[at] = a[i];
    }
    if (w == 0 && lane == 0) s.count = count;
    sync();
}

struct UMaps { CUtensorMap x, a; };

// blockIdx: x = token tile, y = every gridDim.y-th chunk of the tile's distinct adapters, z = part of K (a cluster holds the
// parts of one tile and adds them up in a fixed order)
__global__ void __launch_bounds__(kUThreads)
adapter_kernel(const ProjectArgs p, const __grid_constant__ UMaps maps)
{
    extern __shared__ unsigned char smem_dyn[];
    int32_t* const status = status_of(p);
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 4];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ AdapterList<4> s_al;
    __shared__ int s_slot[kTok];
    __shared__ int s_mine[kTok];            // the token's adapter is in a chunk of this CTA
    __shared__ float s_scale[kTok];
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_done = bar_full + 16 * kMaxStages,
                   bar_free = bar_done + 8, bar_list = bar_done + 16, bar_got = bar_done + 24;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int t0 = blockIdx.x * kTok;
    // Behind the ring (and the rows that the MMA of a short tile may read): this part's sums, [owner][column][token of the
    // owner], and those that the cluster's CTAs send here, [part][column][own token].  A CTA owns a share of the tokens.
    const int own = p.u_own, pitch = own + 1, block = p.rank * pitch;     // (own is even: an odd pitch has no bank conflicts)
    float* const sums = reinterpret_cast<float*>(smem_dyn + (ring - smem_u32(smem_dyn)) + p.scratch);
    float* const got = p.u_splits > 1 ? sums + p.u_splits * block : sums;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.n_stages; ++s) { mbar_init(bar_full + 8 * s, 2); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_done, 2);
        mbar_init(bar_free, 4);
        mbar_init(bar_list, 4);
        mbar_init(bar_got, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"((uint32_t)kUCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (p.u_splits > 1) cluster_arrive();       // (waited for before anything is sent: the peers run and their barriers are there)
    const uint32_t tmem = s_tmem;
    pdl_wait();
    pdl_launch_dependents();        // (after the wait: the projection may read x before it waits itself)

    const int k0 = (int)((long long)p.ksteps * blockIdx.z / p.u_splits), k1 = (int)((long long)p.ksteps * (blockIdx.z + 1) / p.u_splits);
    const int kb = p.kb, per_chunk = (k1 - k0 + kb - 1) / kb;           // slices per stage, stages per chunk
    const uint32_t b_bytes = (uint32_t)(p.stage_bytes / kb) - p.a_bytes;
    int count = 0, n_chunks = 0;
    auto know_list = [&] {                      // (every role but the listing warps)
        if (!mbar_wait(bar_list, 0, &s_abort, status)) return false;
        count = s_al.count;
        n_chunks = (count + p.slots - 1) / p.slots;
        return true;
    };
    if (warp == 0 || warp == 6 || warp == 8) {
        // One lane loads tokens, two load rows of A, even and odd stages (a load costs its lane about 140 cycles, a barrier 290);
        // the tokens need not wait for the list.
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
            bool ok = true;
            int i = 0;                          // stages so far
            if (warp != 0) ok = know_list();
            bool known = warp != 0;
            for (int c = blockIdx.y; ok && (!known || c < n_chunks); c += gridDim.y) {
                for (int ks = k0; ks < k1; ks += kb, ++i) {
                    if (!known && (i == p.n_stages || blockIdx.y > 0)) {
                        if (!know_list()) { ok = false; break; }
                        known = true;
                        if (c >= n_chunks) break;
                    }
                    if (warp == 0 || (i & 1) == (warp == 8)) {
                        if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, status)) { ok = false; break; }
                        const uint32_t sa = ring + stage * p.stage_bytes, sb = sa + kb * p.a_bytes, full = bar_full + 8 * stage;
                        const int n = min(kb, k1 - ks);
                        armed |= 1u << stage;
                        armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                        if (warp == 0) {
                            mbar_expect_tx(full, n * p.a_rows * kBK * 2);
                            for (int q = 0; q < n; ++q) tma_load_2d(sa + q * p.a_bytes, &maps.x, full, (ks + q) * kBK, t0);
                        } else {
                            const int n_slots = min(p.slots, count - c * p.slots);
                            mbar_expect_tx(full, n * n_slots * p.rank * kBK * 2);
                            for (int q = 0; q < n; ++q)
                                for (int j = 0; j < n_slots; ++j)
                                    tma_load_2d(sb + q * b_bytes + j * p.rank * kBK * 2, &maps.a, full, (ks + q) * kBK, s_al.list[c * p.slots + j] * p.rank);
                        }
                    }
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (ok && !known) {
                    ok = know_list();
                    known = true;
                }
            }
            if (ok && warp == 0 && n_chunks <= (int)blockIdx.y) {
                // no adapter to work on: the slices that were asked for early still have to land before the block exits; the
                // other lane's arrival, which completes a stage, is made here
                for (int s = 0; s < p.n_stages; ++s)
                    if (armed & (1u << s)) { mbar_arrive(bar_full + 8 * s); mbar_wait(bar_full + 8 * s, 0, &s_abort, status); }
            }
            if (!ok && warp == 0)
                for (int s = 0; s < p.n_stages; ++s)
                    if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, status);
        }
        __syncwarp();
    } else if (warp == 1 || warp == 7) {
        // Two lanes issue the MMAs, even and odd stages into accumulators of their own (TMEM columns 0.. and 64..): a narrow MMA
        // costs its lane about 100 cycles, a wait and a commit some 500, whatever its width.
        if (lane == 0) {
            const int mine = warp == 7;
            uint32_t stage = 0, phase = 0;
            bool ok = know_list();
            int it = 0, i = 0;
            for (int c = blockIdx.y; c < n_chunks && ok; c += gridDim.y, ++it) {
                // (rank 8 and an odd number of adapters: eight stale columns, never read)
                const int cols = (min(p.slots, count - c * p.slots) * p.rank + 15) & ~15;
                const uint32_t idesc = idesc_bf16(cols), d = tmem + mine * (kUCols / 2) * (p.slots * p.rank <= kUCols / 2);
                if (!mbar_wait(bar_free, (it & 1) ^ 1, &s_abort, status)) { ok = false; break; }
                tc_fence_after();
                uint32_t acc = 0;
                for (int ks = k0; ks < k1; ks += kb, ++i) {
                    if (p.lanes == 1 ? mine == 0 : (i & 1) == mine) {
                        if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
                        tc_fence_after();
                        uint32_t lo_a = smem_desc_lo(ring + stage * p.stage_bytes), lo_b = lo_a + ((kb * p.a_bytes) >> 4);
                        const int n = min(kb, k1 - ks);
                        for (int q = 0; q < n; ++q) {
#pragma unroll
                            for (int kk = 0; kk < kBK / 16; ++kk) {
                                umma_bf16(d, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                                acc = 1;
                            }
                            lo_a += p.a_bytes >> 4; lo_b += b_bytes >> 4;
                        }
                        umma_commit(bar_empty + 8 * stage);
                    }
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (ok) umma_commit(bar_done);
            }
        }
        __syncwarp();
    } else {
        int slot[1];
        list_adapters<4>(p, s_al, t0, warp - 2, lane, blockIdx.y == 0 && blockIdx.z == 0,
                         [] { asm volatile("bar.sync 1, 128;" ::: "memory"); }, slot);
        s_slot[threadIdx.x - 64] = slot[0];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_list);
        __all_sync(kFull, know_list());
        // thread <-> token; a warp reads the TMEM lanes of its quarter
        const int quarter = warp & 3, row = quarter * 32 + lane, my_slot = s_slot[row];
        s_mine[row] = my_slot >= 0 && (my_slot / p.slots) % gridDim.y == blockIdx.y;
        s_scale[row] = my_slot >= 0 && p.scale ? p.scale[s_al.adapter[row]] : 1.f;
        float* const dst = sums + (row / own) * block + row % own;
        int it = 0;
        for (int c0 = blockIdx.y; c0 < n_chunks; c0 += gridDim.y, ++it) {
            const int f = my_slot - c0 * p.slots;
            const bool live = my_slot >= 0 && f >= 0 && f < p.slots;
            const int cols = min(p.slots, count - c0 * p.slots) * p.rank;
            const int c_lo = live ? f * p.rank : cols, c_hi = live ? c_lo + p.rank : 0;
            if (!__all_sync(kFull, mbar_wait(bar_done, it & 1, &s_abort, status))) break;
            tc_fence_after();
            // (a chunk of one stage has filled one accumulator only: that of its stage's lane)
            const int lone = per_chunk == 1 ? (it * per_chunk) & 1 : -1;
            for (int c = 0; c < cols; c += 16) {
                if (!__any_sync(kFull, c + 16 > c_lo && c < c_hi)) continue;
                uint32_t r[16], r2[16];
                const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + c;
                tmem_ld16(p.lanes == 2 && lone == 1 ? from + kUCols / 2 : from, r);
                if (p.lanes == 2 && lone < 0) tmem_ld16(from + kUCols / 2, r2);
                tmem_ld_wait();
                if (p.lanes == 2 && lone < 0) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) + __uint_as_float(r2[i]));
                }
#pragma unroll
                for (int h = 0; h < 16; h += 8)
                    if (c + h >= c_lo && c + h < c_hi) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) dst[(c + h + i - c_lo) * pitch] = __uint_as_float(r[h + i]);
                    }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_free);
        }
        fence_async_shared();                   // (the sums leave by bulk copies)
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (p.u_splits > 1) cluster_wait();
    if (p.slots * (int)blockIdx.y < s_al.count) {           // there was a chunk for this cluster
        if (p.u_splits > 1) {
            if (warp == 0) {
                if (lane == 0) mbar_expect_tx(bar_got, p.u_splits * block * 4);
                __syncwarp();
                if (lane < p.u_splits)
                    send_bulk(map_to_cta(smem_u32(got + blockIdx.z * block), lane), smem_u32(sums + lane * block), block * 4, map_to_cta(bar_got, lane));
            }
            mbar_wait(bar_got, 0, &s_abort, status);
            __syncwarp();
            cluster_arrive_relaxed();           // (waited for below: nobody leaves while its copies may still be on their way)
        }
        // this CTA adds up its share of the tokens over the parts, in their order
        if (!s_abort) {
            const int pairs = p.rank >> 1, at_once = kUThreads / pairs;      // a thread adds two columns, of every at_once-th token
            const int r0 = threadIdx.x / pairs, c = 2 * (threadIdx.x - r0 * pairs);
            for (int r = r0; r0 < at_once && r < own; r += at_once) {
                const int row = own * blockIdx.z + r;
                if (row >= kTok || !s_mine[row]) continue;
                float v = 0.f, w = 0.f;
                for (int z = 0; z < p.u_splits; ++z) {
                    v += got[z * block + c * pitch + r];
                    w += got[z * block + (c + 1) * pitch + r];
                }
                v *= s_scale[row];
                w *= s_scale[row];
                const size_t at = (size_t)(t0 + row) * p.rank + c;
                if (p.u_split) {
                    // Each term is cut, not rounded, and the next is what it left over, so all have the sign of u: with an infinity in B
                    // terms of both signs, or a zero, would add up to NaN.  For the same reason nothing left over is handed on as
                    // 2^-32 of u, which 24 bits do not see (but for u below 2^-101), and what is left of an infinity as that infinity.
                    bf16* u = reinterpret_cast<bf16*>(p.u) + at;
                    const float2 trace = make_float2(v * 0x1p-32f, w * 0x1p-32f);
                    for (int h = 0; h < kUTerms; ++h, u += (size_t)p.T * p.rank) {
                        const __nv_bfloat162 term = __halves2bfloat162(__float2bfloat16_rz(v), __float2bfloat16_rz(w));
                        const float2 f = __bfloat1622float2(term);
                        *reinterpret_cast<__nv_bfloat162*>(u) = term;
                        if (!isinf(f.x)) v -= f.x;
                        if (!isinf(f.y)) w -= f.y;
                        if (v == 0.f) v = trace.x;
                        if (w == 0.f) w = trace.y;
                    }
                } else {
                    *reinterpret_cast<float2*>(p.u + at) = make_float2(v, w);
                }
            }
        }
        if (p.u_splits > 1) cluster_wait();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)kUCols) : "memory");
    }
}

struct PMaps { CUtensorMap x, w, a; };

// The columns of a tile that CTA i of n adds up and writes.
__host__ __device__ constexpr int first_column(int i, int n) { return kPN / 2 * i / n * 2; }
__host__ __device__ constexpr int most_columns(int n) { return (kPN / 2 + n - 1) / n * 2; }

// Few tokens: one cluster of `splits` CTAs per tile of 128 tokens x 128 weight rows; each CTA contracts over its share of K
// into its own TMEM accumulator and sends every column's sums to the CTA that adds that column up (distributed shared
// memory; the parts are added in their order: the same bits every time).  The adapters' second product and the base
// are added there, in fp32 on the CUDA cores: with few tokens that is a few hundred thousand products, and every token may
// have an adapter of its own.
//
// FUSED: the rows of A of the tile's adapters ride as further columns of the same MMA, so u comes out of the same pass (every
// cluster computes it for itself) and there is no first launch.
template <bool FUSED>
__global__ void __launch_bounds__(kPThreads, 2)
project_kernel(const ProjectArgs p, const __grid_constant__ PMaps maps)
{
    extern __shared__ __align__(16) unsigned char smem_dyn[];
    int32_t* const status = status_of(p);
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 3];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ int s_adapter[kTok];
    __shared__ AdapterList<4> s_al;
    __shared__ int s_slot[kTok];
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_done = bar_full + 16 * kMaxStages,
                   bar_list = bar_done + 8, bar_got = bar_done + 16;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int S = p.splits;
    const uint32_t rank = blockIdx.x % S;                   // (in a cluster: its rank there)
    const int n0 = (blockIdx.x / S) * kPN, t0 = blockIdx.y * kTok;
    const int rows = min(kTok, p.T - t0);
    const bool product = p.w != nullptr, adapters = p.n_adapters > 0;
    const bool joint = S > 1 && (product || FUSED);         // a cluster that shares the sums over K; otherwise S CTAs only share the columns
    const int w_rows = product ? kPN : 0;
    constexpr uint32_t kTmem = FUSED ? 256u : (uint32_t)kPN;
    // Behind the ring (and the rows that the MMA of a short tile may read): the sums sent here, [part][own column][token], then
    // (fused) the parts of u, [part][rank][token], then u itself, [token][rank].  This CTA's own sums, [column][token] of
    // the product and of u, are put together in the ring when its stages are done.
    // (columns in twos and a pitch of twice an odd number: a CTA's share is whole 16 bytes, and neighbouring columns meet in a bank in
    // pairs only; in fours and with an odd pitch never, but the largest share would be an extra round of outputs for 64 tokens)
    const int c0 = first_column((int)rank, S), nc = first_column((int)rank + 1, S) - c0, nc_max = most_columns(S);
    const int pitch = p.a_rows + 2;
    float* const own = reinterpret_cast<float*>(smem_dyn + (ring - smem_u32(smem_dyn)));
    float* const own_u = own + kPN * pitch;
    float* const part = reinterpret_cast<float*>(smem_dyn + (ring - smem_u32(smem_dyn)) + p.scratch);
    float* const u_part = part + S * nc_max * pitch;
    float* const su = u_part + (FUSED ? S * p.rank * pitch : 0);

    if (threadIdx.x == 0) {
        for (int s = 0; s < p.n_stages; ++s) { mbar_init(bar_full + 8 * s, FUSED ? 2 : 1); mbar_init(bar_empty + 8 * s, 1); }
        mbar_init(bar_done, 1);
        mbar_init(bar_list, 4);
        mbar_init(bar_got, 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(kTmem) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (joint) cluster_arrive();                            // (waited for before anything is sent: the peers run and their barriers are there)
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    // With a first launch that one is adapter_kernel, which had waited for everything before it when it let this kernel start:
    // x, W and the tenant ids are complete.  Otherwise the kernel before this one is some other's.
    if (FUSED || !adapters) pdl_wait();
    pdl_launch_dependents();

    if (!FUSED && adapters && warp >= 2 && warp < 6) {
        const int row = (warp & 3) * 32 + lane;
        s_adapter[row] = row < rows ? adapter_of(p, t0 + row, false) : -1;
    }
    const int ks_n = product || FUSED ? p.ksteps : 0;
    const int k0 = (int)((long long)ks_n * rank / S), k1 = (int)((long long)ks_n * (rank + 1) / S);
    if (k1 > k0) {
        if (warp == 0 || warp == 10) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
                bool ok = true;
                int count = -1;
                for (int ks = k0; ks < k1; ++ks) {
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, status)) { ok = false; break; }
                    const uint32_t sa = ring + stage * p.stage_bytes, full = bar_full + 8 * stage;
                    if (warp == 0) {
                        armed |= 1u << stage;
                        armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                        mbar_expect_tx(full, (p.a_rows + w_rows) * kBK * 2);
                        if (product) tma_load_2d(sa + p.a_bytes, &maps.w, full, ks * kBK, n0);
                        if (FUSED) tma_load_2d(sa, &maps.x, full, ks * kBK, t0);
                    } else if (FUSED) {
                        if (count < 0) {
                            if (!mbar_wait(bar_list, 0, &s_abort, status)) { ok = false; break; }
                            count = s_al.count;
                        }
                        const uint32_t sb = sa + p.a_bytes + w_rows * kBK * 2;
                        mbar_expect_tx(full, count * p.rank * kBK * 2);
                        for (int j = 0; j < count; ++j)
                            tma_load_2d(sb + j * p.rank * kBK * 2, &maps.a, full, ks * kBK, s_al.list[j] * p.rank);
                    } else {
                        tma_load_2d(sa, &maps.x, full, ks * kBK, t0);
                    }
                    if (++stage == (uint32_t)p.n_stages) { stage = 0; phase ^= 1; }
                }
                if (!ok && warp == 0)
                    for (int s = 0; s < p.n_stages; ++s)
                        if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, status);
            }
            __syncwarp();
        } else if (warp == 1) {
            if (lane == 0) {
                uint32_t stage = 0, phase = 0, acc = 0;
                bool ok = true;
                uint32_t idesc = idesc_bf16(kPN);
                if (FUSED) {
                    ok = mbar_wait(bar_list, 0, &s_abort, status);
                    // (rank 8 and an odd number of adapters: eight stale columns, never read; no adapter and no product: none used)
                    const int cols = w_rows + ((s_al.count * p.rank + 15) & ~15);
                    idesc = idesc_bf16(cols > 0 ? cols : 16);
                }
                for (int ks = k0; ks < k1 && ok; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
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
            // thread <-> token (TMEM lane); two groups of four warps take half of the columns each
            const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane;
            int a = -1;
            if (FUSED) {
                if (half == 0) {
                    int slot[1];
                    list_adapters<4>(p, s_al, t0, warp - 2, lane, blockIdx.x == 0, [] { asm volatile("bar.sync 1, 128;" ::: "memory"); }, slot);
                    s_slot[(warp - 2) * 32 + lane] = slot[0];
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar_list);
                }
                __all_sync(kFull, mbar_wait(bar_list, 0, &s_abort, status));
                a = s_al.adapter[row];
            } else if (adapters && half == 0) {
                a = s_adapter[row];
            }
            if (adapters && half == 0) {
                // The rows of the adapters' B that this CTA will multiply come into L2 while the product runs; every token asks for
                // its own adapter's, the first of a warp for all that share it.
                const int n_lo = n0 + c0, n_hi = min(n0 + c0 + nc, p.N);
                const uint32_t same = __match_any_sync(kFull, a);
                if (a >= 0 && lane == __ffs(same) - 1 && n_lo < n_hi) {
                    const char* lo = reinterpret_cast<const char*>(p.b + ((size_t)a * p.N + n_lo) * p.rank);
                    const char* hi = reinterpret_cast<const char*>(p.b + ((size_t)a * p.N + n_hi) * p.rank);
                    for (const char* q = lo; q < hi; q += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q));
                }
            }
            if (__all_sync(kFull, mbar_wait(bar_done, 0, &s_abort, status)) && quarter * 32 < rows) {
                tc_fence_after();
                const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
                if (product) {
#pragma unroll
                    for (int c = 0; c < kPN / 2; c += 16) {
                        uint32_t r[16];
                        tmem_ld16(tmem + lanes + half * (kPN / 2) + c, r);
                        tmem_ld_wait();
                        if (row < rows) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) own[(half * (kPN / 2) + c + i) * pitch + row] = __uint_as_float(r[i]);
                        }
                    }
                }
                if (FUSED && half == 1) {
                    const int slot = s_slot[row], cols = s_al.count * p.rank;
                    const int c_lo = slot >= 0 ? slot * p.rank : cols, c_hi = slot >= 0 ? c_lo + p.rank : 0;
                    for (int c = 0; c < cols; c += 16) {
                        if (!__any_sync(kFull, c + 16 > c_lo && c < c_hi)) continue;
                        uint32_t r[16];
                        tmem_ld16(tmem + lanes + w_rows + c, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int h = 0; h < 16; h += 8)
                            if (c + h >= c_lo && c + h < c_hi) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) own_u[(c + h + i - c_lo) * pitch + row] = __uint_as_float(r[h + i]);
                            }
                    }
                }
                fence_async_shared();                       // (the sums leave by bulk copies)
            }
        }
    }
    __syncthreads();
    if (joint) {
        cluster_wait();
        if (warp == 0) {
            // every CTA gets its columns of the product, and (fused) u whole
            if (lane == 0) mbar_expect_tx(bar_got, S * ((product ? nc : 0) + (FUSED ? p.rank : 0)) * pitch * 4);
            __syncwarp();
            if (lane < S) {
                const int to = lane, d0 = first_column(to, S), dn = first_column(to + 1, S) - d0;
                const uint32_t bar = map_to_cta(bar_got, to);
                if (product)
                    send_bulk(map_to_cta(smem_u32(part + (int)rank * nc_max * pitch), to), smem_u32(own + d0 * pitch), dn * pitch * 4, bar);
                if (FUSED) send_bulk(map_to_cta(smem_u32(u_part + (int)rank * p.rank * pitch), to), smem_u32(own_u), p.rank * pitch * 4, bar);
            }
        }
    }
    // The outputs: four of a thread at a time, so that their loads overlap.  The first rows of B and of the base are asked for
    // before u and the sums have arrived.
    const int* const adapter = FUSED ? s_al.adapter : s_adapter;
    const int total = rows * nc, vecs = p.rank / 8;
    const float* const got = joint ? part : own;
    int r[4], c[4], a[4];
    bool on[4];
    uint4 bq[4][2];
    float at_base[4];
    auto pick = [&](int e0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = e0 + q * kPThreads;
            r[q] = e / nc;
            c[q] = e - r[q] * nc;
            on[q] = e < total && n0 + c0 + c[q] < p.N;
            a[q] = on[q] && adapters ? adapter[r[q]] : -1;
            at_base[q] = 0.f;
            if (on[q] && p.base) {
                const size_t at = (size_t)(t0 + r[q]) * p.ldbase + n0 + c0 + c[q];
                at_base[q] = p.out_f32 ? ((const float*)p.base)[at] : __bfloat162float(((const bf16*)p.base)[at]);
            }
        }
    };
    auto load_b = [&](int i) {                             // vectors i and i + 1 of the four rows of B
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                bq[q][h] = a[q] >= 0 && i + h < vecs ? __ldg(reinterpret_cast<const uint4*>(p.b + ((size_t)a[q] * p.N + n0 + c0 + c[q]) * p.rank) + i + h)
                                                     : make_uint4(0, 0, 0, 0);
    };
    pick(threadIdx.x);
    if (adapters) load_b(0);
    if (!FUSED && adapters) {
        pdl_wait();                                        // u
        // (rows of tokens without an adapter hold anything and are not looked at)
        const float* src = p.u + (size_t)t0 * p.rank;
        for (int i = threadIdx.x; i < rows * p.rank / 4; i += kPThreads)
            reinterpret_cast<float4*>(su)[i] = __ldcg(reinterpret_cast<const float4*>(src) + i);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (joint) {
        mbar_wait(bar_got, 0, &s_abort, status);
        __syncwarp();
        cluster_arrive_relaxed();                          // (waited for at the end: nobody leaves while its copies may still be on their way)
    }
    if (FUSED) {
        const float* const up = joint ? u_part : own_u;
        for (int i = threadIdx.x; i < rows * p.rank; i += kPThreads) {
            const int ur = i / p.rank, uc = i - ur * p.rank, ua = s_al.adapter[ur];
            float v = 0.f;
            if (ua >= 0) {
                for (int z = 0; z < S; ++z) v += up[(z * p.rank + uc) * pitch + ur];
                if (p.scale) v *= p.scale[ua];
            }
            su[i] = v;
        }
        __syncthreads();
    }
    if (!s_abort) {
        for (int e0 = threadIdx.x; e0 < total; e0 += 4 * kPThreads) {
            if (e0 != threadIdx.x) {
                pick(e0);
                if (adapters) load_b(0);
            }
            float v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                v[q] = 0.f;
                if (on[q] && product)
                    for (int z = 0; z < S; ++z) v[q] += got[(z * nc_max + c[q]) * pitch + r[q]];
            }
            if (adapters) {
                float d[4] = {0.f, 0.f, 0.f, 0.f};
                for (int i = 0; i < vecs; i += 2) {
                    if (i > 0) load_b(i);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (a[q] < 0) continue;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (i + h >= vecs) break;
                            const __nv_bfloat162* b2 = reinterpret_cast<const __nv_bfloat162*>(&bq[q][h]);
                            const float4* up = reinterpret_cast<const float4*>(su + r[q] * p.rank + 8 * (i + h));
                            const float4 u0 = up[0], u1 = up[1];
                            const float2 f0 = __bfloat1622float2(b2[0]), f1 = __bfloat1622float2(b2[1]), f2 = __bfloat1622float2(b2[2]),
                                         f3 = __bfloat1622float2(b2[3]);
                            d[q] = fmaf(u0.x, f0.x, d[q]); d[q] = fmaf(u0.y, f0.y, d[q]); d[q] = fmaf(u0.z, f1.x, d[q]); d[q] = fmaf(u0.w, f1.y, d[q]);
                            d[q] = fmaf(u1.x, f2.x, d[q]); d[q] = fmaf(u1.y, f2.y, d[q]); d[q] = fmaf(u1.z, f3.x, d[q]); d[q] = fmaf(u1.w, f3.y, d[q]);
                        }
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += d[q];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (!on[q]) continue;
                const size_t row = t0 + r[q];
                const int n = n0 + c0 + c[q];
                v[q] += at_base[q];
                if (p.out_f32) ((float*)p.out)[row * p.ldo + n] = v[q];
                else ((bf16*)p.out)[row * p.ldo + n] = __float2bfloat16_rn(v[q]);
            }
        }
    }
    if (joint) cluster_wait();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmem) : "memory");
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Many tokens: 256 tokens x 256 weight rows per pair of CTAs (tcgen05.mma.cta_group::2; each CTA holds 128 of either), pairs
// that walk over the tiles, two accumulators of 256 TMEM columns so that a tile's epilogue runs behind the next tile's MMAs.
//
// The adapters' second products go into the same accumulator: u of the tile's tokens is one more M operand, three bf16 tiles that
// add up to the fp32 value, and
// for every distinct adapter of the tile the rows of its B are one more N operand.  Which tokens that MMA may change is said by
// its disable-output-lane mask, so u needs no masked copy per adapter and an infinity or a NaN in one tenant's B
// cannot reach another's tokens (a zeroed row of u would: 0 * inf).
constexpr int kMStages = 5;
constexpr int kMStageBytes = 2 * kTok * kBK * 2;       // 16 KB of tokens, 16 KB of weight rows per CTA
constexpr int kMTile = 256;
constexpr int kMThreads = 480;                         // warp 0: TMA (weights), 1: MMA, 2..9: epilogue, 10: TMA (tokens), 11..14: u
constexpr int kBRows = kTok / 2;                       // rows of an adapter's B in one load
constexpr int kUTile = kTok * kBK * 2;                 // one bf16 tile of 64 columns of u

__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar & 0xFEFFFFFFu), "r"(x), "r"(y) : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar & 0xFEFFFFFFu), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void umma_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// lanes (tokens of the pair) whose bit is set are left as they are
__device__ __forceinline__ void umma_pair_masked(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, const uint32_t* m)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, {%5, %6, %7, %8, %9, %10, %11, %12}, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(m[0]), "r"(m[1]), "r"(m[2]), "r"(m[3]), "r"(m[4]), "r"(m[5]),
                 "r"(m[6]), "r"(m[7]) : "memory");
}
// arrives on the barrier at the same offset in both CTAs of the pair
__device__ __forceinline__ void umma_commit_pair(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((unsigned short)3) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t cluster_addr)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ void builders_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

struct MMaps { CUtensorMap x, w, b, u; };

constexpr int kOutPitch = 36;                          // floats per row of a warp's staging area (32 columns, 16-byte rows)
constexpr size_t kOutStage = 8 * 32 * kOutPitch * sizeof(float);

// 32 tokens x 32 columns (from row t, column n) by a warp, out of its staging area: a row's columns are read, added to the base
// and written by neighbouring lanes, `kLanes` of them per row.
template <typename T>
struct Block {
    static constexpr int kPer = 16 / sizeof(T);         // columns of a 16-byte vector: 4 or 8
    static constexpr int kLanes = 32 / kPer;            // lanes per row, and vectors per lane: 8 or 4
    uint4 q[kLanes];                                    // the base

    __device__ __forceinline__ void load_base(const ProjectArgs& p, int t, int n, int lane, bool vec)
    {
        if (!p.base || !vec || n + 32 > p.N) return;
#pragma unroll
        for (int i = 0; i < kLanes; ++i) {
            const int r = t + i * (32 / kLanes) + lane / kLanes;
            q[i] = r < p.T ? *reinterpret_cast<const uint4*>((const T*)p.base + (size_t)r * p.ldbase + n + (lane % kLanes) * kPer) : make_uint4(0, 0, 0, 0);
        }
    }
    __device__ __forceinline__ void store(const ProjectArgs& p, const float* stage, int t, int n, int lane, bool vec)
    {
        if (vec && n + 32 <= p.N) {
            const int c = (lane % kLanes) * kPer;
#pragma unroll
            for (int i = 0; i < kLanes; ++i) {
                const int r = i * (32 / kLanes) + lane / kLanes;
                const float4* from = reinterpret_cast<const float4*>(stage + r * kOutPitch + c);
                float v[kPer];
#pragma unroll
                for (int j = 0; j < kPer / 4; ++j) { const float4 f = from[j]; v[4 * j] = f.x; v[4 * j + 1] = f.y; v[4 * j + 2] = f.z; v[4 * j + 3] = f.w; }
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
            const float* from = stage + lane;
            const int rows = min(32, p.T - t);
            if (p.base) {
                const T* base = (const T*)p.base + (size_t)t * p.ldbase + n + lane;
#pragma unroll 1
                for (int r0 = 0; r0 < rows; r0 += 8) {
                    T b[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (r0 + i < rows) b[i] = base[i * p.ldbase];
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (r0 + i < rows) out[i * p.ldo] = (T)(from[i * kOutPitch] + (float)b[i]);
                    base += 8 * p.ldbase; out += 8 * p.ldo; from += 8 * kOutPitch;
                }
            } else {
#pragma unroll 8
                for (int r = 0; r < rows; ++r, out += p.ldo, from += kOutPitch) *out = (T)*from;
            }
        }
    }
};

// One tile's 32 tokens (from t) x 128 columns (from n0) of a warp: out of TMEM, through the staging area, into the output.
template <typename T>
__device__ __forceinline__ bool write_tile(const ProjectArgs& p, uint32_t from, float* stage, int t, int n0, int lane, bool vec, bool empty, uint32_t bar_full,
                                           uint32_t parity, uint32_t bar_read, volatile int* abort_flag, int32_t* status)
{
    if (!__all_sync(kFull, mbar_wait(bar_full, parity, abort_flag, status))) return false;
    tc_fence_after();
#pragma unroll 1
    for (int c = 0; c < 128; c += 32) {
        Block<T> base;
        if (n0 + c < p.N) base.load_base(p, t, n0 + c, lane, vec);
        uint32_t r[32];
        tmem_ld16(from + c, r);
        tmem_ld16(from + c + 16, r + 16);
        tmem_ld_wait();
        if (c == 96) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(bar_read);
        }
        if (n0 + c < p.N) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                reinterpret_cast<float4*>(stage + lane * kOutPitch)[i] =
                    empty ? make_float4(0.f, 0.f, 0.f, 0.f)
                          : make_float4(__uint_as_float(r[4 * i]), __uint_as_float(r[4 * i + 1]), __uint_as_float(r[4 * i + 2]), __uint_as_float(r[4 * i + 3]));
            __syncwarp();
            base.store(p, stage, t, n0 + c, lane, vec);
            __syncwarp();
        }
    }
    return true;
}

__global__ void __launch_bounds__(kMThreads, 1)
project_many_kernel(const ProjectArgs p, const __grid_constant__ MMaps maps)
{
    extern __shared__ unsigned char smem_dyn[];
    int32_t* const status = status_of(p);
    const uint32_t ring = (smem_u32(smem_dyn) + 1023u) & ~1023u;
    unsigned char* const ring_ptr = smem_dyn + (ring - smem_u32(smem_dyn));
    const int n_stages = p.n_stages;
    // u: [64-column chunk][term] tiles; once the tile's MMAs have read it, its memory is the epilogue's staging area
    const uint32_t ua = ring + n_stages * kMStageBytes;
    __shared__ __align__(8) uint64_t s_bars[2 * kMaxStages + 9];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ AdapterList<8> s_al;
    __shared__ uint32_t s_mask[kMTile][8];
    const uint32_t bar_full = smem_u32(s_bars), bar_empty = bar_full + 8 * kMaxStages, bar_tfull = bar_full + 16 * kMaxStages,
                   bar_tempty = bar_tfull + 16, bar_ufull = bar_tfull + 32, bar_uempty = bar_tfull + 40, bar_list = bar_tfull + 48, bar_staged = bar_tfull + 56;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const bool adapters = p.n_adapters > 0;
    const int n_tiles = (p.N + kMTile - 1) / kMTile, m_tiles = (p.T + kMTile - 1) / kMTile, total = n_tiles * m_tiles;
    const int pair0 = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int chunks = (p.rank + kBK - 1) / kBK;            // of u and of the adapters' B

    if (threadIdx.x == 0) {
        for (int s = 0; s < n_stages; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(bar_tfull + 8 * b, 1); mbar_init(bar_tempty + 8 * b, 2 * 8); }
        mbar_init(bar_ufull, 1);
        mbar_init(bar_uempty, 3);                           // the tile's MMAs, and both loading lanes: nobody needs its list any more
        mbar_init(bar_list, 4);
        mbar_init(bar_staged, 8);
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
    // (with adapters the kernel before this one is adapter_kernel: see project_kernel)
    if (!adapters) pdl_wait();
    pdl_launch_dependents();

    if (warp == 0 || warp == 10) {
        // ---- TMA: one lane for the weight rows, one for the tokens; a lane needs about 430 cycles per stage (140 for a load,
        // 290 for the barrier), the MMAs of a stage 512.  Of the adapters' B each loads half of the rows, so that neither lane
        // can fall a turn of the ring behind the other and take a later phase of a barrier for its own.
        if (lane == 0) {
            uint32_t stage = 0, phase = 0, armed = 0, armed_phase = 0;
            bool ok = true;
            int it = 0, u_loads = 0;
            for (int tile = pair0; tile < total && ok; tile += pairs, ++it) {
                const int n0 = (tile / m_tiles) * kMTile + rank * kTok, t0 = (tile % m_tiles) * kMTile + rank * kTok;
                const int steps = p.ksteps;
                int extra = -1;                             // stages of adapters' B behind the product's
                for (int ks = 0; ok; ++ks) {
                    if (ks >= steps && extra < 0) {
                        extra = 0;
                        if (adapters) {
                            if (!mbar_wait(bar_list, it & 1, &s_abort, status)) { ok = false; break; }
                            extra = s_al.count * chunks;
                            if (warp == 10) {
                                // u of this CTA's tokens (rows of tokens without an adapter hold anything)
                                if (it == 0) pdl_wait();
                                // (the MMAs of the tile before have read theirs, and its epilogue is through with the memory)
                                if (!mbar_wait(bar_uempty, (it & 1) ^ 1, &s_abort, status) ||
                                    !mbar_wait(bar_staged, (it & 1) ^ 1, &s_abort, status)) { ok = false; break; }
                                if (leader) mbar_expect_tx(bar_ufull, 2 * kUTerms * chunks * kUTile);
                                u_loads = it + 1;
                                for (int c = 0; c < chunks; ++c)
                                    for (int h = 0; h < kUTerms; ++h)
                                        tma_load_3d_pair(ua + (c * kUTerms + h) * kUTile, &maps.u, bar_ufull, c * kBK, t0, h);
                            }
                        }
                    }
                    if (ks >= steps && ks >= steps + extra) break;
                    const uint32_t sa = ring + stage * kMStageBytes, full = bar_full + 8 * stage;
                    if (!mbar_wait(bar_empty + 8 * stage, phase ^ 1, &s_abort, status)) { ok = false; break; }
                    if (warp == 0) {
                        armed |= 1u << stage;
                        armed_phase = (armed_phase & ~(1u << stage)) | (phase << stage);
                        if (ks < steps) {
                            if (leader) mbar_expect_tx(full, 2 * kMStageBytes);
                            tma_load_2d_pair(sa + kTok * kBK * 2, &maps.w, full, ks * kBK, n0);
                        } else {
                            const int j = (ks - steps) / chunks, c = (ks - steps) - j * chunks;
                            if (leader) mbar_expect_tx(full, kMStageBytes);
                            tma_load_3d_pair(sa + kTok * kBK * 2, &maps.b, full, c * kBK, n0, s_al.list[j]);
                        }
                    } else if (ks < steps) {
                        tma_load_2d_pair(sa, &maps.x, full, ks * kBK, t0);
                    } else {
                        const int j = (ks - steps) / chunks, c = (ks - steps) - j * chunks;
                        tma_load_3d_pair(sa + (kTok + kBRows) * kBK * 2, &maps.b, full, c * kBK, n0 + kBRows, s_al.list[j]);
                    }
                    if (++stage == (uint32_t)n_stages) { stage = 0; phase ^= 1; }
                }
                if (ok && adapters) mbar_arrive(bar_uempty);
            }
            if (!ok && leader && warp == 0) {               // gave up: the copies in flight land before the block exits
                for (int s = 0; s < n_stages; ++s)
                    if (armed & (1u << s)) mbar_wait(bar_full + 8 * s, (armed_phase >> s) & 1u, &s_abort, status);
            }
            if (!ok && leader && u_loads > 0) mbar_wait(bar_ufull, (u_loads - 1) & 1, &s_abort, status);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            uint32_t stage = 0, phase = 0;
            bool ok = true;
            const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((256u >> 3) << 17) | ((256u >> 4) << 24);
            int it = 0;
            for (int tile = pair0; tile < total && ok; tile += pairs, ++it) {
                const uint32_t buf = it & 1, d = tmem + buf * 256;
                if (!mbar_wait_cluster(bar_tempty + 8 * buf, ((it >> 1) & 1) ^ 1, &s_abort, status)) { ok = false; break; }
                tc_fence_after();
                uint32_t acc = 0;
                for (int ks = 0; ks < p.ksteps; ++ks) {
                    if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t lo_a = smem_desc_lo(ring + stage * kMStageBytes), lo_b = lo_a + ((kTok * kBK * 2) >> 4);
#pragma unroll
                    for (int kk = 0; kk < kBK / 16; ++kk) {
                        umma_pair(d, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, acc);
                        acc = 1;
                    }
                    umma_commit_pair(bar_empty + 8 * stage);
                    if (++stage == (uint32_t)n_stages) { stage = 0; phase ^= 1; }
                }
                if (!ok) break;
                if (adapters) {
                    if (!mbar_wait(bar_list, it & 1, &s_abort, status) || !mbar_wait(bar_ufull, it & 1, &s_abort, status)) { ok = false; break; }
                    tc_fence_after();
                    const int count = s_al.count;
                    for (int j = 0; j < count && ok; ++j) {
                        // (without the product the first MMA of an adapter overwrites its tokens' lanes)
                        uint32_t first = acc, mask[8];
#pragma unroll
                        for (int g = 0; g < 8; ++g) mask[g] = s_mask[j][g];
                        for (int c = 0; c < chunks; ++c) {
                            if (!mbar_wait(bar_full + 8 * stage, phase, &s_abort, status)) { ok = false; break; }
                            tc_fence_after();
                            const uint32_t lo_b = smem_desc_lo(ring + stage * kMStageBytes + kTok * kBK * 2);
                            const int kks = (min(kBK, p.rank - c * kBK) + 15) >> 4;
                            for (int h = 0; h < kUTerms; ++h) {
                                const uint32_t lo_a = smem_desc_lo(ua + (c * kUTerms + h) * kUTile);
                                for (int kk = 0; kk < kks; ++kk) {
                                    umma_pair_masked(d, smem_desc_pack(lo_a + 2 * kk), smem_desc_pack(lo_b + 2 * kk), idesc, first, mask);
                                    first = 1;
                                }
                            }
                            umma_commit_pair(bar_empty + 8 * stage);
                            if (++stage == (uint32_t)n_stages) { stage = 0; phase ^= 1; }
                        }
                    }
                    if (!ok) break;
                    umma_commit_pair(bar_uempty);
                }
                umma_commit_pair(bar_tfull + 8 * buf);
            }
        }
        __syncwarp();
    } else if (warp < 10) {
        // ---- epilogue: thread <-> token (TMEM lane), four warps per half of the columns ----
        const int quarter = warp & 3, half = (warp - 2) >> 2;
        const uint32_t tempty_leader = map_to_cta(bar_tempty, 0);
        const int esz = p.out_f32 ? 4 : 2;
        const bool vec = (uintptr_t)p.out % 16 == 0 && p.ldo * esz % 16 == 0 && (!p.base || ((uintptr_t)p.base % 16 == 0 && p.ldbase * esz % 16 == 0));
        float* const stage = reinterpret_cast<float*>(ring_ptr + n_stages * kMStageBytes) + (warp - 2) * 32 * kOutPitch;
        if (adapters) {
            // the base of the first tile comes into L2 while u is being computed (a tile's epilogue of 4 blocks of columns, one
            // after the other, waits for it otherwise)
            const int n0 = (pair0 / m_tiles) * kMTile + half * 128, t = (pair0 % m_tiles) * kMTile + (int)rank * kTok + quarter * 32 + lane;
            if (p.base && t < p.T && n0 < p.N) {
                const char* row = (const char*)p.base + ((size_t)t * p.ldbase + n0) * esz;
                const int bytes = min(128, p.N - n0) * esz;
                for (int b = 0; b < bytes; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + b));
            }
            pdl_wait();
        }
        bool ok = true;
        int it = 0;
        for (int tile = pair0; tile < total; tile += pairs, ++it) {
            const int n0 = (tile / m_tiles) * kMTile + half * 128, t = (tile % m_tiles) * kMTile + (int)rank * kTok + quarter * 32 + lane;
            const uint32_t buf = it & 1;
            // a token that no MMA has written (no product, no adapter): its lane holds some earlier tile
            const bool empty = p.ksteps == 0 && !(t < p.T && adapters && adapter_of(p, t, false) >= 0);
            const uint32_t from = tmem + buf * 256 + ((uint32_t)(quarter * 32) << 16) + half * 128, parity = (it >> 1) & 1;
            ok = p.out_f32 ? write_tile<float>(p, from, stage, t - lane, n0, lane, vec, empty, bar_tfull + 8 * buf, parity, tempty_leader + 8 * buf, &s_abort, status)
                           : write_tile<bf16>(p, from, stage, t - lane, n0, lane, vec, empty, bar_tfull + 8 * buf, parity, tempty_leader + 8 * buf, &s_abort, status);
            if (!ok) break;
            fence_async_shared();                           // (u of the next tile comes into the staging area by TMA)
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_staged);
        }
    } else if (adapters) {
        // ---- four warps that list the adapters of the pair's tokens, and which lanes each MMA leaves alone ----
        const int w = warp - 11;
        int it = 0;
        for (int tile = pair0; tile < total; tile += pairs, ++it) {
            if (!__all_sync(kFull, mbar_wait(bar_uempty, (it & 1) ^ 1, &s_abort, status))) break;
            int slot[2];
            list_adapters<8>(p, s_al, (tile % m_tiles) * kMTile, w, lane, false, [] { builders_sync(); }, slot);
            for (int j = w; j < s_al.count; j += 4) {
                const int a = s_al.list[j];
#pragma unroll
                for (int g = 0; g < 8; ++g) {
                    const uint32_t other = __ballot_sync(kFull, s_al.adapter[g * 32 + lane] != a);
                    if (lane == g) s_mask[j][g] = other;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_list);
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

// 3-D map over n matrices [N][rank] (the adapters' B; u's terms); box = 64 x box_rows of one matrix
bool make_map_3d(CUtensorMap* m, const void* base, uint64_t n, uint64_t N, uint64_t rank, uint32_t box_rows)
{
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {rank, N, n};
    cuuint64_t strides[2] = {rank * 2, N * rank * 2};
    cuuint32_t box[3] = {(cuuint32_t)kBK, box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int kMaxSmem = 212 * 1024;      // dynamic; with the static arrays below the 227 KB of an SM

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

// tiles of `tile` tokens x `tile` columns (of sizes that no memory holds, which only a question for the workspace can have: many)
int tiles_of(const ProjectArgs& p, int tile)
{
    const int64_t n = (int64_t)div_up(p.N, tile) * div_up(p.T, tile);
    return n < (1 << 24) ? (int)n : 1 << 24;
}

constexpr int kSmSmem = 228 * 1024, kStaticSmem = 8 * 1024;     // of an SM; of one CTA of either launch, static and reserved
constexpr int kHalfSmem = 108 * 1024;      // dynamic shared memory up to which two CTAs share an SM

// How many clusters of `size` CTAs run at once, with one CTA per SM or two.  The SMs of a cluster belong to one GPC, so a few of
// each GPC stay unused: on the part measured 15 clusters of eight, not 18, with one CTA per SM (and 33 with two), 33 of
// four, 45 of three.  A cluster more is a second wave: 20 us instead of 10 for 16 clusters of eight.
int cluster_room(int size, bool two)
{
    static int room[kMaxDevices][9][2] = {};
    int dev = 0;
    if (size < 2 || size > 8 || cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return size == 1 ? 148 * (two ? 2 : 1) : 0;
    int& n = room[dev][size][two];
    if (n == 0) {
        static bool allowed[kMaxDevices] = {false};
        if (allow_smem(project_kernel<false>, allowed) != cudaSuccess) cudaGetLastError();      // (the query asks for that much)
        cudaLaunchConfig_t cfg;
        memset(&cfg, 0, sizeof(cfg));
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = size; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
        cfg.gridDim = dim3(size * 148); cfg.blockDim = dim3(kPThreads); cfg.dynamicSmemBytes = two ? kHalfSmem : kMaxSmem;
        cfg.attrs = &attr; cfg.numAttrs = 1;
        int most = 0;
        if (cudaOccupancyMaxActiveClusters(&most, project_kernel<false>, &cfg) != cudaSuccess || most < 1) {
            cudaGetLastError();
            most = (two ? 256 : 112) / size;                // (no answer: a cautious guess)
        }
        n = most;
    }
    return n;
}

// Parts of K, stages and shared memory of project_kernel; false if it does not fit.  `behind`: bytes behind the last stage
// that the MMA of a short token tile may read; `beside`: shared memory of a CTA of the first launch, 0 without one.
bool few_geometry(ProjectArgs& p, bool fused, int u_rows, int behind, int beside = 0)
{
    static_assert(kPN == kTok, "");
    const int tiles = tiles_of(p, kPN), pitch = p.a_rows + 2;
    const bool joint = p.w || fused;                        // (otherwise the parts only share the columns)
    p.stage_bytes = p.a_bytes + (p.w ? kPN * kBK * 2 : 0) + ((u_rows + 15) & ~15) * kBK * 2;
    // as many parts as there are SMs for the tiles (a cluster holds eight), of two slices at least, all clusters at once
    for (p.splits = 8; ; --p.splits) {
        if (p.splits > 1 && (p.splits == 5 || p.splits == 7 || p.splits * tiles > 148 || (joint && p.splits > p.ksteps / 2))) continue;
        // received: the parts of this CTA's columns, (fused) the parts of u; and u itself
        p.sums_bytes = (p.splits * most_columns(p.splits) * pitch + (fused ? p.splits * p.rank * pitch : 0) + p.a_rows * p.rank) * (int)sizeof(float);
        const int own = (kPN + (fused ? p.rank : 0)) * pitch * (int)sizeof(float);
        const int want = joint ? div_up(p.ksteps, p.splits) : 1;
        auto stages = [&](int bytes) {                      // the ring, or this CTA's own sums that are put together in it
            const int room = bytes - 1024 - p.sums_bytes;
            int n = (room - behind) / p.stage_bytes;
            if (n > want) n = want;
            if (n > 6) n = 6;
            return room < own || n < 0 ? 0 : n;
        };
        // two CTAs per SM if three stages (or all there are) fit, so that the next launch of a chain finds room beside this one
        const int half = stages(kHalfSmem), full = stages(kMaxSmem);
        bool two = half >= 3 || (half >= 1 && half == want);
        p.n_stages = two ? half : full;
        // (behind a first launch what has to fit beside a CTA is one of that launch, not a second one of these)
        const int left = beside > 0 ? stages(min(kMaxSmem, kSmSmem - kStaticSmem - beside)) : 0;
        if (two && left > half) { two = false; p.n_stages = left; }
        p.scratch = p.n_stages * p.stage_bytes + behind;
        if (p.scratch < own) p.scratch = own;
        const bool fits = p.n_stages >= 2 || (p.n_stages == 1 && want == 1);
        if (p.splits == 1) return fits;
        if (fits && (!joint || tiles <= cluster_room(p.splits, two))) return true;
    }
}

// Which shape, by what either costs (us), a model fitted to some thousand measured pairs of 1 to 1024 tokens, 512 to 5632 rows and
// columns, ranks 8 to 128 of 1 to 32 adapters (in 110 other draws of those, the choice is within 1.15 of the better one in all but
// two).  The pair shape: its slices of K, and a masked MMA per adapter that a tile may have.  The other: parts of K, and the
// adapters' products on the CUDA cores.  (few / many tokens' shape, 2048 -> 2048: rank 16, 4 adapters, 64 tokens 11 / 21, 128 15 / 22, 512 27 / 21; 32 adapters, 128
// tokens 21 / 41; rank 64, 2 adapters, 48 tokens 18 / 21, 96 28 / 21; no adapters, 200 tokens 13 / 15, 512 19 / 15.  2048 -> 5632:
// rank 16, 4 adapters, 24 tokens 12 / 22, 96 23 / 22; 5632 -> 2048: rank 32, 4 adapters, 128 tokens 22 / 39, rank 16, 1024 tokens 69 / 38.)
bool use_many(const ProjectArgs& p)
{
    const int steps = p.w ? div_up(p.K, kBK) : 0, tiles = tiles_of(p, kPN), rows = p.T < kTok ? p.T : kTok;
    int parts = tiles < 148 ? 148 / tiles : 1;
    if (parts > 8) parts = 8;
    if (p.w && parts > steps / 2) parts = steps / 2;
    if (parts < 1) parts = 1;
    const int waves = div_up(tiles * parts, 148), rounds = div_up(tiles_of(p, kMTile), 74);
    int distinct = p.T < kMTile ? p.T : kMTile;
    if (distinct > p.n_adapters) distinct = p.n_adapters;
    const bool adapters = p.n_adapters > 0;
    const float few = (adapters ? 8.8f : 7.7f) + waves * (0.6f * steps / parts + 0.009f * rows + 1.2e-4f * rows * kPN / parts * (adapters ? p.rank : 0));
    const float many = (p.w ? 10.3f : 13.5f) - (adapters ? 0.f : 3.1f) + rounds * (0.25f * steps + distinct * (0.48f + 0.0125f * p.rank));
    return many < few;
}

// Parts of K, chunks of adapters, stages and shared memory (returned) of adapter_kernel.
size_t adapter_geometry(const ProjectArgs& p, bool many, ProjectArgs& q, int& chunks)
{
    const int m_tiles = div_up(p.T, kTok), behind = kTok * kBK * 2 - p.a_bytes;
    q = p;
    // K is cut into as many parts as there are SMs for the token tiles, of two slices at least.  Beside a product of many
    // tokens the SMs that count are those that the product leaves: it starts on the others at once and needs u only at the
    // end of its first tiles (4096 tokens, 5632 -> 2048: 32 CTAs on all of K instead of 128 on quarters).  A product that leaves
    // none gives up 36.  (At least 12 / 20 / 36 / 52 / 74, us, adapters in ragged runs: 4096 tokens, 2048 -> 5632, 16 of rank 16
    // 91 / 96 / 94 / 96 / 99; 2048 tokens, 8 of them 61 / 57 / 52 / 53 / 58; 4096, 2048 -> 2048, 8 of rank 64 54 / 51 / 50 / 50 / 51.)
    int sms = 148;
    if (many && p.w) {
        const int busy = 2 * tiles_of(p, kMTile);
        sms = busy > 148 - 36 ? 36 : 148 - busy;
    }
    q.u_splits = 1;
    while (q.u_splits < (m_tiles == 1 ? 8 : 4) && m_tiles * q.u_splits * 2 <= sms && q.ksteps / (q.u_splits * 2) >= 2) q.u_splits *= 2;
    // Chunks of 64 columns: with one tile they are more CTAs, with many the ring has more stages for x, which is what is read.
    // From rank 32 on they would hold one or two adapters, so that beside a product, where CTAs are few, x would be read often:
    // 128 columns.  (64 / 128 columns, us, 5632 -> 2048, tokens of mixed tenants / in ragged runs of one: 4096 tokens, 4 adapters of
    // rank 16 80 / 101 and 80 / 101, 16 of rank 32 177 / 150 and 88 / 112, 13 of rank 64 236 / 171 and 130 / 101; 2048 tokens 67 / 64
    // and 54 / 60, 95 / 81 and 64 / 64, 120 / 95 and 67 / 67.)
    const int columns = many && p.w && p.rank >= 32 ? kUCols : kUCols / 2;
    q.slots = columns / p.rank > 0 ? columns / p.rank : 1;
    const int most = p.T < kTok ? p.T : kTok;
    const int all = div_up(most < p.n_adapters ? most : p.n_adapters, q.slots);      // chunks that a tile may have
    // (beyond rank 64 one accumulator takes all columns, and one lane issues the MMAs)
    q.lanes = q.slots * p.rank <= kUCols / 2 ? 2 : 1;
    // shared memory: the ring, and the sums of a_rows tokens twice (sent and received); at high ranks fewer parts, then fewer stages
    size_t sums;
    for (;; q.u_splits /= 2) {
        q.u_own = (div_up(p.a_rows, q.u_splits) + 3) & ~3;
        sums = (size_t)q.u_splits * (q.u_own + 1) * p.rank * sizeof(float) * (q.u_splits > 1 ? 2 : 1);
        // two slices per stage where a CTA has many: its lanes wait and commit half as often
        q.kb = div_up(q.ksteps, q.u_splits) >= 16 ? 2 : 1;
        q.stage_bytes = q.kb * (p.a_bytes + (q.lanes == 2 ? kUCols / 2 : kUCols) * kBK * 2);
        if (2 * q.stage_bytes + behind + sums + 1024 > kMaxSmem && q.kb == 2) { q.kb = 1; q.stage_bytes /= 2; }
        if (q.u_splits == 1 || 2 * q.stage_bytes + behind + sums + 1024 <= kMaxSmem) break;
    }
    // two CTAs per SM where four stages (or all of a chunk, two at least) fit
    const int per_chunk = div_up(div_up(q.ksteps, q.u_splits), q.kb);
    auto fit = [&](int bytes) { const int n = (bytes - 1024 - behind - (int)sums) / q.stage_bytes; return n < 0 ? 0 : (n > kMaxStages ? kMaxStages : n); };
    const bool two = fit(kHalfSmem) >= (per_chunk < 2 ? 2 : (per_chunk < 4 ? per_chunk : 4));
    q.n_stages = two ? fit(kHalfSmem) : fit(kMaxSmem);
    // Chunks have CTAs of their own, as many as run at once, and are walked over beyond that.  A CTA whose tile has no such chunk
    // ends at once, so they are counted for all SMs also beside a product.  (4096 tokens, 5632 -> 2048, 32 adapters of rank 16,
    // every token another: 290 us with the SMs that the product leaves, 170 to 195 with all; the same in runs of one tenant: 76, 79.)
    int room = q.u_splits > 1 ? cluster_room(q.u_splits, two) : 148 * (two ? 2 : 1);
    if (room > 148 / q.u_splits) room = 148 / q.u_splits;
    room /= m_tiles;
    chunks = all < room ? all : (room < 1 ? 1 : room);
    const int steps = per_chunk * div_up(all, chunks);
    if (q.n_stages > steps) q.n_stages = steps;
    // (an even number where the ring wraps: a stage then belongs to the same loading and issuing lanes every time around.  With
    // an odd one they would take turns on its barriers, and a lane that is ahead could take an older phase for its own.)
    if (q.n_stages < steps) q.n_stages &= ~1;
    q.scratch = q.n_stages * q.stage_bytes + behind;
    return q.scratch + sums + 1024;
}

// Tile sizes, and for few tokens the shape of project_kernel; returns whether u comes out of the same pass (fused).  That
// saves a launch, some 2 us of the caller's time, and costs every CTA all of u: up to four tokens of a product of at most 512 tiles of
// 128 x 64 weights (8 MB), where the launches are what a call waits for.  (2048 -> 2048, rank 16, one token: 9.9 us on the GPU
// and 11 on the host in one launch, 9.6 and 12.5 in two; 2048 -> 5632: 12.6 and 10.7 on the GPU; 2048 -> 2048, 4 adapters of rank 32:
// 8 tokens 12.7 and 11.1, 64 tokens 18 and 14.)
bool plan_few(ProjectArgs& p)
{
    const bool adapters = p.n_adapters > 0;
    p.a_rows = p.T >= kTok ? kTok : ((p.T + 7) & ~7);
    p.a_bytes = (p.a_rows * kBK * 2 + 1023) & ~1023;
    p.ksteps = p.w || adapters ? div_up(p.K, kBK) : 0;
    const int behind = kTok * kBK * 2 - p.a_bytes;          // an MMA reads 128 token rows, also of a short tile in the last stage
    p.u_rows = adapters ? (p.T < p.n_adapters ? p.T : p.n_adapters) * (p.rank <= kUCols ? p.rank : kUCols) : 0;
    if (adapters && p.T <= 4 && (int64_t)tiles_of(p, kPN) * p.ksteps <= 512 && p.u_rows <= kUCols && few_geometry(p, true, p.u_rows, behind)) return true;
    if (!use_many(p)) few_geometry(p, false, 0, behind);
    return false;
}

}  // namespace

int64_t project_workspace(int T, int K, int N, int rank, int n_adapters)
{
    if (n_adapters == 0 || T == 0) return 0;
    ProjectArgs p = {};
    p.T = T; p.K = K; p.N = N; p.rank = rank; p.n_adapters = n_adapters;
    if (plan_few(p) && (p.w = reinterpret_cast<const bf16*>(16), plan_few(p))) return 0;      // (with w and without)
    return (int64_t)T * rank * 2 * kUTerms;        // bf16 terms (fp32, which few tokens take, is less)
}

cudaError_t take_project_status(int32_t* status_host)
{
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return e;
    take_status_kernel<<<1, 1>>>();
    e = cudaGetLastError();
    return e == cudaSuccess ? cudaMemcpyFromSymbol(status_host, g_project_taken, sizeof(int32_t)) : e;
}

cudaError_t launch_project(const ProjectArgs& in, cudaStream_t st)
{
    ProjectArgs p = in;
    static bool u_ok[kMaxDevices] = {false}, p_ok[kMaxDevices] = {false}, f_ok[kMaxDevices] = {false}, m_ok[kMaxDevices] = {false};
    const int m_tiles = div_up(p.T, kTok), n_tiles = div_up(p.N, kPN);
    const bool adapters = p.n_adapters > 0, fused = plan_few(p), many = !fused && use_many(p);
    p.u_split = many;
    ProjectArgs q;
    int chunks = 0;
    const size_t u_smem = adapters && !fused ? adapter_geometry(p, many, q, chunks) : 0;
    if (u_smem && !many) few_geometry(p, false, 0, kTok * kBK * 2 - p.a_bytes, (int)u_smem);

    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof(cfg));
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 1; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.stream = st;

    if (adapters && !fused) {
        cudaError_t e = allow_smem(adapter_kernel, u_ok);
        if (e != cudaSuccess) return e;
        UMaps um;
        if (!make_map_ld(&um.x, p.x, p.T, p.K, p.ldx, p.a_rows) ||
            !make_map_ld(&um.a, p.a, (uint64_t)p.n_adapters * p.rank, p.K, p.K, p.rank))
            return cudaErrorInvalidValue;
        cfg.attrs[1].val.clusterDim.z = q.u_splits;
        cfg.numAttrs = q.u_splits > 1 ? 2 : 1;
        cfg.gridDim = dim3(m_tiles, chunks, q.u_splits); cfg.blockDim = dim3(kUThreads); cfg.dynamicSmemBytes = u_smem;
        e = cudaLaunchKernelEx(&cfg, adapter_kernel, q, um);
        if (e != cudaSuccess) return e;
        attr[1].val.clusterDim.z = 1;

    }
    if (many) {
        cudaError_t e = allow_smem(project_many_kernel, m_ok);
        if (e != cudaSuccess) return e;
        MMaps mm;
        memset(&mm, 0, sizeof(mm));
        if (!p.w) p.ksteps = 0;
        if (p.w && (!make_map_ld(&mm.x, p.x, p.T, p.K, p.ldx, kTok) || !make_map_ld(&mm.w, p.w, p.N, p.K, p.ldw, kTok)))
            return cudaErrorInvalidValue;
        if (adapters && (!make_map_3d(&mm.b, p.b, p.n_adapters, p.N, p.rank, kBRows) || !make_map_3d(&mm.u, p.u, kUTerms, p.T, p.rank, kTok)))
            return cudaErrorInvalidValue;
        const int u_tiles = adapters ? kUTerms * div_up(p.rank, kBK) : 0;      // 48 or 96 KB, which leave five or three stages
        p.n_stages = (kMaxSmem - 1024 - u_tiles * kUTile) / kMStageBytes;
        if (p.n_stages > kMStages) p.n_stages = kMStages;
        size_t behind_ring = (size_t)u_tiles * kUTile;
        if (behind_ring < kOutStage) behind_ring = kOutStage;
        const int tiles = tiles_of(p, kMTile), pairs = tiles < 74 ? tiles : 74;
        attr[1].val.clusterDim.x = 2;
        cfg.gridDim = dim3(2 * pairs); cfg.blockDim = dim3(kMThreads); cfg.numAttrs = 2;
        cfg.dynamicSmemBytes = (size_t)p.n_stages * kMStageBytes + behind_ring + 1024;
        return cudaLaunchKernelEx(&cfg, project_many_kernel, p, mm);
    }
    PMaps pm;
    memset(&pm, 0, sizeof(pm));
    if ((p.w || fused) && !make_map_ld(&pm.x, p.x, p.T, p.K, p.ldx, p.a_rows)) return cudaErrorInvalidValue;
    if (p.w && !make_map_ld(&pm.w, p.w, p.N, p.K, p.ldw, kPN)) return cudaErrorInvalidValue;
    if (fused && !make_map_ld(&pm.a, p.a, (uint64_t)p.n_adapters * p.rank, p.K, p.K, p.rank)) return cudaErrorInvalidValue;
    cfg.gridDim = dim3(n_tiles * p.splits, m_tiles); cfg.blockDim = dim3(kPThreads);
    cfg.dynamicSmemBytes = (size_t)p.scratch + p.sums_bytes + 1024;
    attr[1].val.clusterDim.x = p.splits;
    cfg.numAttrs = p.splits > 1 && (p.w || fused) ? 2 : 1;
    cudaError_t e = fused ? allow_smem(project_kernel<true>, f_ok) : allow_smem(project_kernel<false>, p_ok);
    if (e != cudaSuccess) return e;
    return fused ? cudaLaunchKernelEx(&cfg, project_kernel<true>, p, pm) : cudaLaunchKernelEx(&cfg, project_kernel<false>, p, pm);
}

}  // namespace faasmoe
