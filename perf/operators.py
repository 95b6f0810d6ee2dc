"""Cases of the operators around the MoE layer: the gating rules (moe_gate), the residual's addition with the RMSNorm
in front of a layer (moe_add_rmsnorm) and a shared projection with the tenants' low-rank adapters (moe_project).

``run`` computes an operator in its plain form (elementary torch operations), or, where ``own`` is true, calls the
library.  Shapes are those of the package's workloads (hidden 2048, 60 experts of 1408, a shared expert of 5632, top 4,
4 or 16 tenants) and, for the routers with groups, the largest router the library takes (256 experts, top 8).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------------------------------------------------
# cases

def _gate(name, T, E, k, score, *, bias=False, groups=1, keep=1, group_score="max", renorm=True, scale=1.0, M=1,
          tenants=1, dtype="f32", pad=0):
    return dict(name=name, op="gate", T=T, E=E, k=k, score=score, bias=bias, groups=groups, keep=keep,
                group_score=group_score, renorm=renorm, scale=scale, M=M, tenants=tenants, dtype=dtype, pad=pad)


def _norm(name, T, H, *, residual=True, out=True, q="none", pad=0):
    return dict(name=name, op="norm", T=T, H=H, residual=residual, out=out, q=q, pad=pad)


def _project(name, T, K, N, *, weight=True, base=False, rank=16, adapters=4, tenants=4, layout="contiguous", out="bf16"):
    return dict(name=name, op="project", T=T, K=K, N=N, weight=weight, base=base, rank=rank, adapters=adapters,
                tenants=tenants, layout=layout, out=out)


def listed():
    return [
        # one sequence being decoded: softmax scores of the 60 experts, renormalised weights of the top 4
        _gate("gate_one_token", 1, 60, 4, "softmax"),
        # a decode batch on a wide router: sigmoid scores, a bias for balance, the best 4 of 8 groups
        _gate("gate_decode_grouped", 32, 256, 8, "sigmoid", bias=True, groups=8, keep=4, group_score="top2", scale=2.5),
        # the pool of 4 tenant models, each with its own bias; the logits are columns of a wider matrix in bf16
        _gate("gate_pool", 2048, 60, 4, "softmax", bias=True, groups=4, keep=2, M=4, tenants=4, dtype="bf16", pad=4),
        # a long prefill on the wide router
        _gate("gate_prefill_grouped", 16384, 256, 8, "sigmoid", bias=True, groups=8, keep=4, group_score="top2", scale=2.5),
        # the norm in front of the layer, decode batch, bf16 output
        _norm("norm_decode", 32, 2048),
        # ragged batch of 16 tenants: bf16 for the router and e4m3 in groups of 128 for an 8-bit projection
        _norm("norm_ragged_q128", 1126, 2048, q="group"),
        # odd sizes and a strided input, 8-bit output alone with one scale for a row
        _norm("norm_odd_qrow", 333, 1411, out=False, q="row", pad=5),
        # a large prefill
        _norm("norm_prefill_qrow", 16384, 2048, q="row"),
        # one token of one tenant
        _project("project_one_token", 1, 2048, 2048),
        # decode: every token another tenant's adapter; fp32 output, as the aggregation takes the shared expert's
        _project("project_decode", 32, 2048, 5632, rank=16, adapters=32, tenants=32, layout="uniform", out="f32"),
        # adapters added beside a projection that is already there, ragged requests of 16 tenants, three of them without
        _project("project_beside", 1126, 2048, 2048, weight=False, base=True, rank=64, adapters=13, tenants=16, layout="ragged"),
        # prefill through the shared expert's down projection, ragged requests of 16 tenants
        _project("project_prefill", 4096, 5632, 2048, rank=16, adapters=16, tenants=16, layout="ragged"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["gate", "norm", "project"])
    if op == "gate":
        groups = rng.choice([1, 1, 2, 4, 8])
        E = groups * rng.randint(max(2, -(-8 // groups)), 256 // groups)
        keep = rng.randint(1, groups)
        k = rng.randint(1, min(8, keep * (E // groups)))
        M = rng.choice([1, 1, 1, 4])
        c = _gate("", _log_int(rng, 1, 16384), E, k, rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.6, groups=groups,
                  keep=keep, group_score=rng.choice(["max", "top2"]), renorm=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]),
                  M=M, tenants=M * rng.randint(1, 4), dtype=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0, 0, 3, 4]))
    elif op == "norm":
        H = rng.choice([_log_int(rng, 1, 8192), 128 * rng.randint(1, 64)])
        T = _log_int(rng, 1, min(16384, 16384 * 2048 // H))
        q = rng.choice(["none", "row", "group"])
        c = _norm("", T, H, residual=rng.random() < 0.8, out=q == "none" or rng.random() < 0.6, q=q, pad=rng.choice([0, 0, 5, 8]))
    else:
        K, N = 8 * _log_int(rng, 16, 704), _log_int(rng, 64, 5632)
        T = _log_int(rng, 1, min(4096, 4096 * 5632 * 2048 // (K * N)))
        weight = rng.random() < 0.8
        tenants = rng.choice([1, 4, 16, 32])
        layout = rng.choice(["contiguous", "ragged", "uniform"])
        c = _project("", T, K, N, weight=weight, base=not weight or rng.random() < 0.3, rank=8 * _log_int(rng, 1, 16),
                     adapters=rng.randint(1, tenants), tenants=tenants, layout=layout, out=rng.choice(["bf16", "bf16", "f32"]))
    c.pop("name")
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 13)
    return g


def _normal(g, shape, std, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _tenants(case, seed):
    """Tenant of every token: requests one after another, of even or of ragged lengths, or tokens in any order."""
    T, n = case["T"], case["tenants"]
    rng = np.random.RandomState(seed % (1 << 31))
    if case.get("layout", "uniform") == "uniform":
        t = rng.randint(0, n, T)
    elif case["layout"] == "contiguous":
        t = np.arange(T) * n // T
    else:
        t = np.sort(rng.choice(n, T, p=rng.dirichlet(np.full(n, 1.5))))
    return torch.from_numpy(t.astype(np.int32)).to(DEV)


def prepare(case, seed):
    g = _generator(seed)
    T = case["T"]
    s = {"case": case}
    if case["op"] == "gate":
        E, M, k = case["E"], case["M"], case["k"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # router logits of normalised tokens: about one unit wide, some experts more popular than others
        logits = torch.randn(T, E + case["pad"], generator=g, device=DEV) + 0.5 * torch.randn(E + case["pad"], generator=g, device=DEV)
        s["logits"] = logits.to(dtype)[:, :E]
        s["bias"] = torch.randn(M, E, generator=g, device=DEV) * 0.05 if case["bias"] else None
        s["tenant_id"] = _tenants(case, seed) if M > 1 else None
        s["model_of_tenant"] = (torch.arange(case["tenants"], device=DEV) % M).to(torch.int32) if M > 1 else None
        s["topk_idx"] = torch.empty(T, k, dtype=torch.int32, device=DEV)
        s["topk_w"] = torch.empty(T, k, dtype=torch.float32, device=DEV)
    elif case["op"] == "norm":
        H = case["H"]
        s["x"] = _normal(g, (T, H + case["pad"]), 0.5, torch.bfloat16)[:, :H]
        s["residual"] = _normal(g, (T, H), 2.0, torch.bfloat16) if case["residual"] else None
        s["weight"] = (1 + 0.02 * torch.randn(H, generator=g, device=DEV)).to(torch.bfloat16)
        s["residual_out"] = torch.empty(T, H, dtype=torch.bfloat16, device=DEV) if case["residual"] else None
        s["out"] = torch.empty(T, H, dtype=torch.bfloat16, device=DEV) if case["out"] else None
        s["q"] = s["q_scale"] = None
        if case["q"] != "none":
            s["q"] = torch.empty(T, H, dtype=torch.float8_e4m3fn, device=DEV)
            s["q_scale"] = torch.empty(T, -(-H // 128) if case["q"] == "group" else 1, dtype=torch.float32, device=DEV)
    else:
        K, N, r, n = case["K"], case["N"], case["rank"], case["adapters"]
        out = torch.float32 if case["out"] == "f32" else torch.bfloat16
        s["x"] = _normal(g, (T, K), 1.0, torch.bfloat16)
        s["w"] = _normal(g, (N, K), 0.02, torch.bfloat16) if case["weight"] else None
        s["base"] = _normal(g, (T, N), 1.0, out) if case["base"] else None
        s["a"] = _normal(g, (n, r, K), 0.02, torch.bfloat16)
        s["b"] = _normal(g, (n, N, r), 0.02, torch.bfloat16)
        s["scale"] = 0.5 + torch.rand(n, generator=g, device=DEV)
        s["tenant_id"] = _tenants(case, seed)
        # tenants beyond the last adapter have none
        s["adapter_of_tenant"] = torch.tensor([u if u < n else -1 for u in range(case["tenants"])], dtype=torch.int32, device=DEV)
        s["out"] = torch.empty(T, N, dtype=out, device=DEV)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass

def run(state):
    return {"gate": _run_gate, "norm": _run_norm, "project": _run_project}[state["case"]["op"]](state)


def _run_gate(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        rule = B.moe_gating(score=c["score"], n_groups=c["groups"], keep_groups=c["keep"], group_score=c["group_score"],
                            renormalize=c["renorm"], scale=c["scale"])
        B.moe_gate(s["logits"], rule, s["topk_idx"], s["topk_w"], balance_bias=s["bias"], tenant_id=s["tenant_id"],
                   model_of_tenant=s["model_of_tenant"])
        return {"topk_idx": s["topk_idx"], "topk_w": s["topk_w"]}
    T, E = s["logits"].shape
    # the order of two experts is decided in 64 bits
    z = s["logits"].double()
    score = torch.softmax(z, 1) if c["score"] == "softmax" else torch.sigmoid(z)
    choice = z
    value = score
    if c["bias"]:
        bias = s["bias"].double()
        bias = bias[s["model_of_tenant"].long()[s["tenant_id"].long()]] if c["M"] > 1 else bias
        value = score + bias
        choice = value
    if c["keep"] < c["groups"]:
        size = E // c["groups"]
        if c["group_score"] == "max" or size == 1:
            group = choice.reshape(T, c["groups"], size).amax(2)
        else:
            group = torch.sort(value.reshape(T, c["groups"], size), dim=2, descending=True)[0][:, :, :2].sum(2)
        kept = torch.sort(group, dim=1, descending=True, stable=True)[1][:, :c["keep"]]
        mask = torch.zeros(T, c["groups"], dtype=torch.bool, device=z.device).scatter_(1, kept, True)
        choice = choice.masked_fill(~mask.repeat_interleave(size, 1), -math.inf)
    idx = torch.sort(choice, dim=1, descending=True, stable=True)[1][:, :c["k"]]
    w = score.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    return {"topk_idx": idx.to(torch.int32), "topk_w": (w * c["scale"]).float()}


def _run_norm(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        B.moe_add_rmsnorm(s["x"], s["weight"], 1e-6, residual=s["residual"], residual_out=s["residual_out"], out=s["out"],
                          out_q=s["q"], q_scale=s["q_scale"])
        return {"residual": s["residual_out"], "out": s["out"], "q": s["q"], "q_scale": s["q_scale"]}
    x = s["x"].float()
    res = None
    if c["residual"]:
        res = (x + s["residual"].float()).to(torch.bfloat16)
        x = res.float()
    y = x * torch.rsqrt((x * x).mean(1, keepdim=True) + 1e-6) * s["weight"].float()
    q = scale = None
    if c["q"] != "none":
        T, H = y.shape
        size = 128 if c["q"] == "group" else H
        n = -(-H // size)
        blocks = torch.nn.functional.pad(y, (0, n * size - H)).reshape(T, n, size)
        scale = blocks.abs().amax(2) / E4M3_MAX
        q = torch.where(scale[:, :, None] > 0, blocks / scale[:, :, None], torch.zeros((), device=y.device))
        q = q.reshape(T, n * size)[:, :H].clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return {"residual": res, "out": y.to(torch.bfloat16) if c["out"] else None, "q": q, "q_scale": scale}


def _run_project(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        B.moe_project(s["x"], s["w"], s["out"], base=s["base"], a=s["a"], b=s["b"], scale=s["scale"], tenant_id=s["tenant_id"],
                      adapter_of_tenant=s["adapter_of_tenant"])
        return s["out"]
    x = s["x"].float()
    n, r, K = s["a"].shape
    # every adapter's first product, the other adapters' columns of a token set to zero, every adapter's second product
    adapter = s["adapter_of_tenant"][s["tenant_id"].long()].long()
    u = (x @ s["a"].float().reshape(n * r, K).t()).reshape(-1, n, r)
    pick = (adapter[:, None] == torch.arange(n, device=x.device)).float() * s["scale"]
    y = (u * pick[:, :, None]).reshape(-1, n * r) @ s["b"].float().permute(0, 2, 1).reshape(n * r, -1)
    if c["weight"]:
        y = y + x @ s["w"].float().t()
    if c["base"]:
        y = y + s["base"].float()
    return y.to(s["out"].dtype)


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    T = case["T"]
    if case["op"] == "gate":
        E, k = case["E"], case["k"]
        b = T * E * (2 if case["dtype"] == "bf16" else 4) + T * k * 8
        b += 4 * case["M"] * E if case["bias"] else 0
        b += 4 * T if case["M"] > 1 else 0
        return {"bytes": b, "flops": 6.0 * T * E}
    if case["op"] == "norm":
        H = case["H"]
        b = 2 * T * H + 2 * H + (4 * T * H if case["residual"] else 0) + (2 * T * H if case["out"] else 0)
        if case["q"] != "none":
            b += T * H + 4 * T * (-(-H // 128) if case["q"] == "group" else 1)
        return {"bytes": b, "flops": 6.0 * T * H}
    K, N, r = case["K"], case["N"], case["rank"]
    used = min(case["adapters"], T)
    size = 4 if case["out"] == "f32" else 2
    b = 2 * T * K + 2 * used * r * (K + N) + 4 * T + size * T * N
    b += 2 * N * K if case["weight"] else 0
    b += size * T * N if case["base"] else 0
    return {"bytes": b, "flops": 2.0 * T * r * (K + N) + (2.0 * T * K * N if case["weight"] else 0.0)}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"gate": _exact_gate, "norm": _exact_norm, "project": _exact_project}[case["op"]](case, s)


def _exact_gate(case, s):
    z = s["logits"].double().cpu().numpy()
    T, E = z.shape
    if case["score"] == "softmax":
        e = np.exp(z - z.max(1, keepdims=True))
        p = e / e.sum(1, keepdims=True)
    else:
        p = np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))
    value = p.copy()
    if case["bias"]:
        bias = s["bias"].double().cpu().numpy()
        model = np.zeros(T, dtype=int)
        if case["M"] > 1:
            model = s["model_of_tenant"].cpu().numpy()[s["tenant_id"].cpu().numpy()]
        value += bias[model]
    order = np.argsort(-(value if case["bias"] else z), axis=1, kind="stable")       # (value descending, id ascending)
    size = E // case["groups"]
    if case["keep"] < case["groups"]:
        key = value if case["bias"] or case["group_score"] == "top2" else z
        best = -np.sort(-key.reshape(T, case["groups"], size), axis=2)
        score = best[:, :, 0] + (best[:, :, 1] if case["group_score"] == "top2" and size > 1 else 0)
        rank = np.argsort(np.argsort(-score, axis=1, kind="stable"), axis=1, kind="stable")
        allowed = np.take_along_axis(rank, order // size, 1) < case["keep"]
        # the first k of each row's order whose group is kept
        seen = np.cumsum(allowed, 1)
        idx = np.stack([order[t][allowed[t] & (seen[t] <= case["k"])] for t in range(T)])
    else:
        idx = order[:, :case["k"]]
    w = np.take_along_axis(p, idx, 1)
    if case["renorm"]:
        w = w / w.sum(1, keepdims=True)
    return {"topk_idx": idx.astype(np.int32), "topk_w": w * case["scale"]}


def _exact_norm(case, s):
    h = s["x"].double()
    total = None
    if case["residual"]:
        total = h + s["residual"].double()
        h = total.to(torch.bfloat16).double()            # the norm is that of the stored sum
    T, H = h.shape
    norm = torch.linalg.vector_norm(h, dim=1).square() / H + 1e-6
    y = h / norm.sqrt()[:, None] * s["weight"].double()
    q = scale = None
    if case["q"] == "row":
        scale = y.abs().max(1)[0][:, None] / E4M3_MAX
        q = y / scale
    elif case["q"] == "group":
        parts = [y[:, i:i + 128] for i in range(0, H, 128)]
        scale = torch.stack([p.abs().max(1)[0] / E4M3_MAX for p in parts], 1)
        q = torch.cat([p / scale[:, i:i + 1] for i, p in enumerate(parts)], 1)
    return {"residual": total, "out": y if case["out"] else None, "q": q, "q_scale": scale}


def _exact_project(case, s):
    T, N = s["out"].shape
    x = s["x"].double()
    y = s["base"].double() if case["base"] else torch.zeros(T, N, dtype=torch.float64, device=x.device)
    if case["weight"]:
        y = y + x @ s["w"].double().t()
    tenant = s["tenant_id"].cpu().numpy()
    table = s["adapter_of_tenant"].cpu().numpy()
    for a in range(case["adapters"]):
        rows = torch.from_numpy(np.nonzero(table[tenant] == a)[0]).to(x.device)
        if rows.numel():
            u = x[rows] @ s["a"][a].double().t()
            y[rows] += s["scale"][a].double() * (u @ s["b"][a].double().t())
    return y
