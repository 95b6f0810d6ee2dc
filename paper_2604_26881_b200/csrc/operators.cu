// C-ABI entry points that need no context: argument checks, then one launcher each.
#include <cmath>

#include "addnorm.cuh"
#include "gate.cuh"
#include "project.cuh"

using namespace faasmoe;

namespace {

constexpr int kMaxRows = 1 << 28;
constexpr int kProjectMaxTokens = 1 << 22;
constexpr int kProjectMaxDim = 1 << 30;      // K, N, and the rows of all adapters' A

bool off(const void* p, size_t align) { return ((uintptr_t)p & (align - 1)) != 0; }

// an output in the place of an input needs the input's row distance: a row would be overwritten before it is read
bool shifted(const void* out, int64_t ld_out, const void* in, int64_t ld_in, int T) { return out && out == in && T > 1 && ld_out != ld_in; }

}  // namespace

namespace faasmoe {

int check_gating(const moe_gating* rule, int E, int k)
{
    if (!rule) return MOE_ERR_NULL;
    if (rule->score != MOE_SCORE_SOFTMAX && rule->score != MOE_SCORE_SIGMOID) return MOE_ERR_SHAPE;
    if (rule->group_score != MOE_GROUP_MAX && rule->group_score != MOE_GROUP_TOP2) return MOE_ERR_SHAPE;
    if (rule->n_groups < 1 || rule->n_groups > 32 || E % rule->n_groups) return MOE_ERR_SHAPE;
    if (rule->keep_groups < 1 || rule->keep_groups > rule->n_groups) return MOE_ERR_SHAPE;
    if (k > rule->keep_groups * (E / rule->n_groups)) return MOE_ERR_SHAPE;
    if (!std::isfinite(rule->scale)) return MOE_ERR_SHAPE;
    return MOE_OK;
}

void apply_gating(GateArgs& a, const moe_gating& rule)
{
    a.score = rule.score; a.n_groups = rule.n_groups; a.keep = rule.keep_groups; a.group_score = rule.group_score;
    a.renormalize = rule.renormalize != 0; a.scale = rule.scale;
}

}  // namespace faasmoe

extern "C" {

int moe_gate(const void* logits, int logits_type, int64_t ld, int T, int E, int k, const moe_gating* rule,
             const float* balance_bias, const int32_t* tenant_id, const int32_t* model_of_tenant, int n_tenants, int M,
             int32_t* topk_idx, float* topk_w, uint8_t* tie_flag, int32_t* status_out, void* stream)
{
    if (!rule) return MOE_ERR_NULL;
    if (T < 0 || T > kMaxRows || E < 1 || E > kMaxExperts || k < 1 || k > kMaxTopK || k > E || ld < E) return MOE_ERR_SHAPE;
    if (M < 1 || M > kMaxExperts || (tenant_id && n_tenants < 1)) return MOE_ERR_SHAPE;
    if (logits_type != MOE_TYPE_F32 && logits_type != MOE_TYPE_BF16) return MOE_ERR_UNSUPPORTED;
    if (off(logits, logits_type == MOE_TYPE_BF16 ? 2 : 4) || off(balance_bias, 4) || off(tenant_id, 4) || off(model_of_tenant, 4) ||
        off(topk_idx, 4) || off(topk_w, 4) || off(status_out, 4))
        return MOE_ERR_SHAPE;
    const int rc = check_gating(rule, E, k);
    if (rc != MOE_OK) return rc;
    if (T == 0) return MOE_OK;
    if (!logits || !topk_idx || !topk_w || (M > 1 && (!tenant_id || !model_of_tenant))) return MOE_ERR_NULL;
    GateArgs a = {};
    a.logits = logits; a.bf16_logits = logits_type == MOE_TYPE_BF16; a.ld = ld; a.T = T; a.E = E; a.k = k;
    apply_gating(a, *rule);
    a.bias = balance_bias; a.tenant_id = tenant_id; a.model_of_tenant = model_of_tenant; a.n_tenants = n_tenants; a.M = M;
    a.topk_idx = topk_idx; a.topk_w = topk_w; a.tie_flag = tie_flag; a.status = status_out;
    return cuda_result("moe_gate", launch_gate(a, (cudaStream_t)stream));
}

int moe_add_rmsnorm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const void* weight, float eps,
                    int T, int H, void* residual_out, int64_t ld_residual_out, void* out, int64_t ld_out, void* out_q,
                    int64_t ld_q, float* q_scale, int group, void* stream)
{
    if (T < 0 || T > kMaxRows || H < 1) return MOE_ERR_SHAPE;
    if (H > kAddNormMaxH) return MOE_ERR_UNSUPPORTED;
    if (ldx < H || (residual && ld_residual < H) || (residual_out && ld_residual_out < H) || (out && ld_out < H) || (out_q && ld_q < H))
        return MOE_ERR_SHAPE;
    if (!(eps >= 0.f) || (out_q && group != 0 && group != 128)) return MOE_ERR_SHAPE;
    if (off(x, 2) || off(residual, 2) || off(weight, 2) || off(residual_out, 2) || off(out, 2) || off(q_scale, 4)) return MOE_ERR_SHAPE;
    if (T == 0) return MOE_OK;
    if (!x || !weight || (!residual_out && !out && !out_q) || (out_q && !q_scale)) return MOE_ERR_NULL;
    if ((out && out == residual_out) || (out_q && (out_q == x || out_q == residual || out_q == out || out_q == residual_out))) return MOE_ERR_SHAPE;
    if (shifted(out, ld_out, x, ldx, T) || shifted(out, ld_out, residual, ld_residual, T) || shifted(residual_out, ld_residual_out, x, ldx, T) ||
        shifted(residual_out, ld_residual_out, residual, ld_residual, T))
        return MOE_ERR_SHAPE;
    AddNormArgs a = {};
    a.x = (const bf16*)x; a.residual = (const bf16*)residual; a.residual_out = (bf16*)residual_out; a.weight = (const bf16*)weight;
    a.out = (bf16*)out; a.q = (uint8_t*)out_q; a.q_scale = q_scale;
    a.ldx = ldx; a.ldr = residual ? ld_residual : 0; a.ldro = residual_out ? ld_residual_out : 0; a.ldo = out ? ld_out : 0;
    a.ldq = out_q ? ld_q : 0;
    a.group = group; a.n_groups = group ? (H + group - 1) / group : 1; a.T = T; a.H = H; a.eps = eps;
    return cuda_result("moe_add_rmsnorm", launch_addnorm(a, (cudaStream_t)stream));
}

int64_t moe_project_workspace(int T, int K, int N, int rank, int n_adapters)
{
    if (T < 0 || T > kProjectMaxTokens || K < 1 || K > kProjectMaxDim || N < 1 || N > kProjectMaxDim || n_adapters < 0) return MOE_ERR_SHAPE;
    if (n_adapters > 0 && (rank < 1 || rank > kAdapterMaxRank || n_adapters > kProjectMaxDim / rank)) return MOE_ERR_SHAPE;
    return project_workspace(T, K, N, rank, n_adapters);
}

int moe_project_status(int32_t* status_host)
{
    if (!status_host) return MOE_ERR_NULL;
    return cuda_result("moe_project_status", take_project_status(status_host));
}

int moe_project(const void* x, int64_t ldx, const void* w, int64_t ldw, int T, int K, int N, const void* a, const void* b,
                const float* scale, int n_adapters, int rank, const int32_t* tenant_id, const int32_t* adapter_of_tenant,
                int n_tenants, const void* base, int64_t ld_base, void* out, int64_t ld_out, int out_type, void* workspace,
                int64_t workspace_bytes, int32_t* status_out, void* stream)
{
    const bool adapters = n_adapters > 0;
    if (T < 0 || T > kProjectMaxTokens || K < 1 || K > kProjectMaxDim || N < 1 || N > kProjectMaxDim || n_adapters < 0) return MOE_ERR_SHAPE;
    if (ld_out < N || (base && ld_base < N)) return MOE_ERR_SHAPE;
    if ((w || adapters) && ldx < K) return MOE_ERR_SHAPE;
    if (w && ldw < K) return MOE_ERR_SHAPE;
    if (adapters && (rank < 1 || rank > kAdapterMaxRank || n_adapters > kProjectMaxDim / rank || n_tenants < 1)) return MOE_ERR_SHAPE;
    if (out_type != MOE_TYPE_F32 && out_type != MOE_TYPE_BF16) return MOE_ERR_UNSUPPORTED;
    // the operands travel as TMA tiles: rows on 16-byte boundaries
    if (K % 8 || ((w || adapters) && ldx % 8) || (w && ldw % 8) || (adapters && rank % 8)) return MOE_ERR_UNSUPPORTED;
    const size_t out_align = out_type == MOE_TYPE_F32 ? 4 : 2;
    if (((w || adapters) && off(x, 16)) || off(w, 16) || off(out, out_align) || off(base, out_align) || off(status_out, 4)) return MOE_ERR_SHAPE;
    if (adapters && (off(a, 16) || off(b, 16) || off(scale, 4) || off(tenant_id, 4) || off(adapter_of_tenant, 4))) return MOE_ERR_SHAPE;
    if (off(workspace, 256)) return MOE_ERR_SHAPE;
    if (T == 0) return MOE_OK;
    if (!out || (!w && !adapters && !base)) return MOE_ERR_NULL;
    if (((w || adapters) && !x) || (adapters && (!a || !b || !tenant_id))) return MOE_ERR_NULL;
    const int64_t need = project_workspace(T, K, N, rank, n_adapters);
    if (need > 0 && !workspace) return MOE_ERR_NULL;
    if (workspace_bytes < need) return MOE_ERR_ALLOC;
    if (((w || adapters) && out == x) || out == w || (adapters && (out == a || out == b)) || shifted(out, ld_out, base, ld_base, T)) return MOE_ERR_SHAPE;
    ProjectArgs p = {};
    p.x = (const bf16*)x; p.w = (const bf16*)w; p.ldx = ldx; p.ldw = ldw; p.T = T; p.K = K; p.N = N;
    if (adapters) {
        p.a = (const bf16*)a; p.b = (const bf16*)b; p.scale = scale; p.n_adapters = n_adapters; p.rank = rank;
        p.tenant_id = tenant_id; p.adapter_of_tenant = adapter_of_tenant; p.n_tenants = n_tenants;
    }
    p.base = base; p.ldbase = ld_base; p.out = out; p.ldo = ld_out; p.out_f32 = out_type == MOE_TYPE_F32;
    p.u = (float*)workspace;
    p.status = status_out;
    return cuda_result("moe_project", launch_project(p, (cudaStream_t)stream));
}

}  // extern "C"
