"""Cases of three operators around the MoE layer: the norms after and before a block with its gate and the residual's scale
(moe_block_norm, moe_block_norm_backward), a shared projection in 8-bit integers with a scale for each token and each channel
(moe_quantize_i8, moe_project_i8), and the balance loss of a router with its per-expert counts and the gradient of its logits
(moe_balance_loss, moe_gate_backward).

``run`` computes an operator in its plain form (elementary torch operations), or, where ``own`` is true, calls the
library.  Shapes are those of the package's workloads (hidden 2048, 60 experts, a shared expert of 5632, top 4, 4 or 16
tenants) and, for the large router, the largest one the library takes (256 experts, top 8).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


# ---------------------------------------------------------------------------------------------------------------------
# cases

def _block(name, op, T, H, *, post=True, pre=True, gate="none", act="none", residual_scale=1.0, block_scale=1.0, pad=0):
    return dict(name=name, op=op, T=T, H=H, post=post, pre=pre, gate=gate, act=act, residual_scale=residual_scale,
                block_scale=block_scale, pad=pad)


def _i8(name, T, K, N, *, source="tensor", bias=False, base=False, out="bf16", pad=0):
    return dict(name=name, op="i8", T=T, K=K, N=N, source=source, bias=bias, base=base, out=out, pad=pad)


def _router(name, T, E, k, score, *, renorm=True, scale=1.0, z=True, M=1, tenants=1, mask=False, dtype="f32", pad=0):
    return dict(name=name, op="router", T=T, E=E, k=k, score=score, renorm=renorm, scale=scale, z=z, M=M, tenants=tenants,
                mask=mask, dtype=dtype, pad=pad)


def listed():
    return [
        # one sequence being decoded: norm of the block's output, a learned scale per channel, the stream, the next block's norm
        _block("block_one_token", "block", 1, 2048, gate="channel"),
        # ragged batch of 16 tenants, the block's output gated element by element by a sigmoid
        _block("block_ragged_gated", "block", 1126, 2048, gate="element", act="sigmoid"),
        # a long prefill, one gate per token (a shared expert's), the stream scaled down as in deep stacks
        _block("block_prefill", "block", 16384, 2048, gate="token", residual_scale=0.5, block_scale=0.7),
        # training on odd sizes out of a wider buffer, a learned scale per channel
        _block("block_grad_odd", "block_grad", 333, 1411, gate="channel", pad=5),
        # training on a long batch: gradients of both norms' weights, of the block, the stream and the sigmoid gate
        _block("block_grad_long", "block_grad", 16384, 2048, gate="element", act="sigmoid"),
        # one token through a square projection
        _i8("i8_one_token", 1, 2048, 2048),
        # decode: the norm writes 8 bits that the shared expert's up projection takes
        _i8("i8_decode_block", 32, 2048, 5632, source="block"),
        # ragged batch of 16 tenants through the down projection, with a bias, added to what is there
        _i8("i8_ragged_base", 1126, 5632, 2048, bias=True, base=True),
        # a long prefill through the up projection
        _i8("i8_prefill", 16384, 2048, 5632),
        # a small training step on the 60 experts' router
        _router("router_small", 32, 60, 4, "softmax"),
        # the pool of 4 tenant models in one batch, padded rows among the tokens; bf16 logits out of a wider matrix
        _router("router_pool", 4096, 60, 4, "softmax", renorm=False, M=4, tenants=4, mask=True, dtype="bf16", pad=4),
        # a long step on the wide router with sigmoid scores
        _router("router_long", 65536, 256, 8, "sigmoid", scale=2.5),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["block", "block_grad", "i8", "router"])
    if op in ("block", "block_grad"):
        H = rng.choice([_log_int(rng, 8, 8192), 128 * rng.randint(1, 64)])
        T = _log_int(rng, 1, min(16384, 16384 * 2048 // H))
        c = _block("", op, T, H, post=rng.random() < 0.8, pre=rng.random() < 0.8, gate=rng.choice(["none", "channel", "token", "element"]),
                   act=rng.choice(["none", "sigmoid"]), residual_scale=rng.choice([1.0, 0.5]), block_scale=rng.choice([1.0, 0.7]),
                   pad=rng.choice([0, 0, 5, 8]))
    elif op == "i8":
        K = rng.choice([_log_int(rng, 64, 5632), 16 * _log_int(rng, 8, 352)])
        N = _log_int(rng, 64, 5632)
        T = _log_int(rng, 1, min(16384, 16384 * 5632 * 2048 // (K * N)))
        c = _i8("", T, K, N, source=rng.choice(["tensor", "block"]), bias=rng.random() < 0.4, base=rng.random() < 0.3,
                out=rng.choice(["bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 16]))
        if c["source"] == "block":
            c["out"] = "bf16"
    else:
        E = rng.choice([_log_int(rng, 2, 256), 8 * rng.randint(1, 32)])
        M = rng.choice([1, 1, 1, 4])
        c = _router("", _log_int(rng, 1, 65536), E, rng.randint(1, min(8, E)), rng.choice(["softmax", "sigmoid"]),
                    renorm=rng.random() < 0.7, scale=rng.choice([1.0, 2.5]), z=rng.random() < 0.7, M=M, tenants=M * rng.randint(1, 4),
                    mask=rng.random() < 0.4, dtype=rng.choice(["f32", "f32", "bf16"]), pad=rng.choice([0, 0, 3, 4]))
    c.pop("name")
    return c


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 17)
    return g


def _normal(g, shape, std, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _empty(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV)


def _weight(g, n):
    return (1 + 0.05 * torch.randn(n, generator=g, device=DEV)).to(torch.bfloat16)


def _gate_of(g, form, T, H):
    if form == "channel":                       # a learned scale per channel
        return _normal(g, (H,), 0.3)
    if form == "token":                         # a probability per token, in fp32 as the router gives it
        return torch.rand(T, generator=g, device=DEV)
    return _normal(g, (T, H), 1.0) if form == "element" else None


def prepare(case, seed):
    g = _generator(seed)
    T = case["T"]
    s = {"case": case}
    if case["op"] in ("block", "block_grad"):
        H = case["H"]
        s["y"] = _normal(g, (T, H + case["pad"]), 0.5)[:, :H]
        s["post"] = _weight(g, H) if case["post"] else None
        s["pre"] = _weight(g, H) if case["pre"] else None
        s["gate"] = _gate_of(g, case["gate"], T, H)
        if case["op"] == "block":
            s["residual"] = _normal(g, (T, H), 2.0)
            s["h"] = _empty(T, H)
            s["out"] = _empty(T, H) if case["pre"] else None
        else:
            # what the forward pass has stored, and the gradients that come back
            s["h"] = _normal(g, (T, H), 2.0)
            s["d_out"] = _normal(g, (T, H), 0.1) if case["pre"] else None
            s["d_h"] = _normal(g, (T, H), 0.1)
            s["d_y"], s["d_residual"] = _empty(T, H), _empty(T, H)
            s["d_post"] = _empty(H, dtype=torch.float32) if case["post"] else None
            s["d_pre"] = _empty(H, dtype=torch.float32) if case["pre"] else None
            s["d_gate"] = None
            if s["gate"] is not None:
                s["d_gate"] = torch.empty_like(s["gate"], dtype=torch.bfloat16 if case["gate"] == "element" else torch.float32)
    elif case["op"] == "i8":
        K, N = case["K"], case["N"]
        wide = -(-K // 16) * 16 + case["pad"]
        out = torch.float32 if case["out"] == "f32" else torch.bfloat16
        s["x"] = _normal(g, (T, K), 1.0)
        if case["source"] == "block":
            s["residual"], s["h"] = _normal(g, (T, K), 2.0), _empty(T, K)
            s["post"], s["pre"] = _weight(g, K), _weight(g, K)
        # the weights were laid out in 8 bits once, each row (output channel) with its scale
        w = torch.randn(N, K, generator=g, device=DEV) * 0.02
        s["w_scale"] = w.abs().amax(1) / 127
        s["w_q"] = torch.zeros(N, wide, dtype=torch.int8, device=DEV)[:, :K]
        s["w_q"].copy_(torch.round(w / s["w_scale"][:, None]).clamp(-127, 127))
        s["x_q"] = _empty(T, wide, dtype=torch.int8)[:, :K]
        s["x_scale"] = _empty(T, dtype=torch.float32)
        s["bias"] = torch.randn(N, generator=g, device=DEV) if case["bias"] else None
        s["base"] = _normal(g, (T, N), 1.0, out) if case["base"] else None
        s["out"] = _empty(T, N, dtype=out)
    else:
        E, M, k = case["E"], case["M"], case["k"]
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        # router logits of normalised tokens: about one unit wide, some experts more popular than others
        logits = torch.randn(T, E + case["pad"], generator=g, device=DEV) + 0.5 * torch.randn(E + case["pad"], generator=g, device=DEV)
        s["logits"] = logits.to(dtype)[:, :E]
        s["topk_idx"] = torch.sort(s["logits"].float(), dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32).contiguous()
        s["mask"] = (torch.rand(T, generator=g, device=DEV) < 0.8).to(torch.uint8) if case["mask"] else None
        s["tenant_id"] = s["model_of_tenant"] = None
        if M > 1:
            rng = np.random.RandomState(seed % (1 << 31))
            s["tenant_id"] = torch.from_numpy(rng.randint(0, case["tenants"], T).astype(np.int32)).to(DEV)
            s["model_of_tenant"] = (torch.arange(case["tenants"], device=DEV) % M).to(torch.int32)
        # gradients that come back: of the weights from the experts' outputs, of the losses their coefficients
        s["d_w"] = torch.randn(T, k, generator=g, device=DEV) * 0.01
        s["d_loss"] = 0.01 * (0.5 + torch.rand(M, generator=g, device=DEV))
        s["d_z"] = 0.001 * (0.5 + torch.rand(M, generator=g, device=DEV)) if case["z"] else None
        s["counts"], s["tokens"] = _empty(M, E, dtype=torch.int32), _empty(M, dtype=torch.int32)
        s["mean_prob"], s["loss"] = _empty(M, E, dtype=torch.float32), _empty(M, dtype=torch.float32)
        s["z_loss"] = _empty(M, dtype=torch.float32) if case["z"] else None
        s["d_logits"] = _empty(T, E, dtype=dtype)
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass

def run(state):
    return {"block": _run_block, "block_grad": _run_block_grad, "i8": _run_i8, "router": _run_router}[state["case"]["op"]](state)


def _run_block(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        B.moe_block_norm(s["y"], s["residual"], s["h"], EPS, post_weight=s["post"], pre_weight=s["pre"], gate=s["gate"],
                         gate_act=c["act"], residual_scale=c["residual_scale"], block_scale=c["block_scale"], out=s["out"])
        return {"h": s["h"], "out": s["out"]}
    a = _normed(s["y"].float(), s["post"])
    g = _gate_values(s["gate"], c)
    h = (c["residual_scale"] * s["residual"].float() + c["block_scale"] * (a if g is None else g * a)).to(torch.bfloat16)
    return {"h": h, "out": _normed(h.float(), s["pre"]).to(torch.bfloat16) if c["pre"] else None}


def _normed(x, weight):
    if weight is None:
        return x
    return x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS) * weight.float()


def _gate_values(gate, c):
    """The gate as a matrix that broadcasts over [T, H]."""
    if gate is None:
        return None
    g = gate.float()
    if c["gate"] == "token":
        g = g[:, None]
    return torch.sigmoid(g) if c["act"] == "sigmoid" else g


def _run_block_grad(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        B.moe_block_norm_backward(s["y"], s["h"], EPS, post_weight=s["post"], pre_weight=s["pre"], gate=s["gate"], gate_act=c["act"],
                                  residual_scale=c["residual_scale"], block_scale=c["block_scale"], d_out=s["d_out"], d_h=s["d_h"],
                                  d_block=s["d_y"], d_residual=s["d_residual"], d_gate=s["d_gate"], d_post_weight=s["d_post"],
                                  d_pre_weight=s["d_pre"])
        return {"d_y": s["d_y"], "d_residual": s["d_residual"], "d_gate": s["d_gate"], "d_post": s["d_post"], "d_pre": s["d_pre"]}
    dh, d_pre, d_post, d_gate = s["d_h"].float(), None, None, None
    if c["pre"]:
        d, d_pre = _norm_gradient(s["h"].float(), s["pre"].float(), s["d_out"].float())
        dh = dh + d
    y = s["y"].float()
    g = _gate_values(s["gate"], c)
    da = c["block_scale"] * dh
    if g is not None:
        dg = da * _normed(y, s["post"])
        if c["act"] == "sigmoid":
            dg = dg * (g * (1 - g))
        d_gate = {"channel": lambda: dg.sum(0), "token": lambda: dg.sum(1), "element": lambda: dg.to(torch.bfloat16)}[c["gate"]]()
        da = da * g
    dy = da
    if c["post"]:
        dy, d_post = _norm_gradient(y, s["post"].float(), da)
    return {"d_y": dy.to(torch.bfloat16), "d_residual": (c["residual_scale"] * dh).to(torch.bfloat16), "d_gate": d_gate,
            "d_post": d_post, "d_pre": d_pre}


def _norm_gradient(x, weight, d):
    """Gradients of RMSNorm(x) * weight in x and in weight, d coming back."""
    r = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    n = x * r
    dn = d * weight
    return r * (dn - n * (dn * n).mean(1, keepdim=True)), (d * n).sum(0)


def _run_i8(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        if c["source"] == "block":
            B.moe_block_norm(s["x"], s["residual"], s["h"], EPS, post_weight=s["post"], pre_weight=s["pre"], out_q=s["x_q"], q_scale=s["x_scale"])
        else:
            B.moe_quantize_i8(s["x"], s["x_q"], s["x_scale"])
        B.moe_project_i8(s["x_q"], s["x_scale"], s["w_q"], s["w_scale"], s["out"], bias=s["bias"], base=s["base"])
        return {"h": s.get("h"), "out": s["out"]}
    x, h = s["x"].float(), None
    if c["source"] == "block":
        h = (s["residual"].float() + _normed(x, s["post"])).to(torch.bfloat16)
        x = _normed(h.float(), s["pre"])
    scale = x.abs().amax(1) / torch.full((), 127.0, device=x.device)        # (a quotient, not a product with 1 / 127)
    q = torch.where(scale[:, None] > 0, torch.round(x / scale[:, None]), torch.zeros((), device=x.device))
    # (whole numbers: the sums of these products are exact as long as they stay below 2^24)
    y = (q @ s["w_q"].float().t()) * scale[:, None] * s["w_scale"]
    if c["bias"]:
        y = y + s["bias"]
    if c["base"]:
        y = y + s["base"].float()
    return {"h": h, "out": y.to(s["out"].dtype)}


def _run_router(s):
    c = s["case"]
    if own:
        from paper_2604_26881_b200 import binding as B
        rule = B.moe_gating(score=c["score"], renormalize=c["renorm"], scale=c["scale"])
        same = dict(mask=s["mask"], tenant_id=s["tenant_id"], model_of_tenant=s["model_of_tenant"])
        B.moe_balance_loss(s["logits"], s["topk_idx"], s["counts"], s["tokens"], s["mean_prob"], s["loss"], score=c["score"], z_loss=s["z_loss"], **same)
        B.moe_gate_backward(s["logits"], rule, s["topk_idx"], s["d_logits"], d_topk_w=s["d_w"], counts=s["counts"], tokens=s["tokens"],
                            d_loss=s["d_loss"], d_z_loss=s["d_z"], **same)
        return {"counts": s["counts"], "tokens": s["tokens"], "mean_prob": s["mean_prob"], "loss": s["loss"], "z_loss": s["z_loss"],
                "d_logits": s["d_logits"]}
    T, E, k, M = c["T"], c["E"], c["k"], c["M"]
    z = s["logits"].float()
    idx = s["topk_idx"].long()
    live = torch.ones(T, device=z.device) if s["mask"] is None else (s["mask"] != 0).float()
    model = torch.zeros(T, dtype=torch.long, device=z.device) if M == 1 else s["model_of_tenant"].long()[s["tenant_id"].long()]
    member = (model[:, None] == torch.arange(M, device=z.device)).float() * live[:, None]        # [T, M]
    # scores, and their shares of the token's whole
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    lse = top[:, 0] + torch.log(e.sum(1))
    soft = e / e.sum(1, keepdim=True)
    if c["score"] == "softmax":
        score, slope, p = soft, 1.0, soft
    else:
        score = 1 / (1 + torch.exp(-z))
        slope = 1 / (1 + torch.exp(z))                             # 1 - score
        p = score / score.sum(1, keepdim=True)
    # counts, means and losses of every model
    chosen = torch.zeros(T, E, device=z.device).scatter_add_(1, idx, torch.ones(T, k, device=z.device))
    counts = (member.double().t() @ chosen.double()).round()
    tokens = member.double().sum(0)
    over = 1 / tokens.clamp(min=1)
    mean = (member.double().t() @ p.double()) * over[:, None]
    loss = E / k * over * (counts * mean).sum(1)
    z_loss = (member.double() * lse.double()[:, None].square()).sum(0) * over if c["z"] else None
    # the gradient of the logits: by way of the weights, of the shares and of the log of the sum
    gw = s["d_w"] * c["scale"]
    ws = score.gather(1, idx)
    if c["renorm"]:
        ws = ws / ws.sum(1, keepdim=True)
        inner = ws * (gw - (gw * ws).sum(1, keepdim=True))
        d = torch.zeros(T, E, device=z.device).scatter_add_(1, idx, inner) * slope
    else:
        d = torch.zeros(T, E, device=z.device).scatter_add_(1, idx, gw * ws)
        d = d - soft * (gw * ws).sum(1, keepdim=True) if c["score"] == "softmax" else d * slope
    f = (member @ (counts * (s["d_loss"].double() * E / k * over * over)[:, None]).float())
    d = d + p * (f - (f * p).sum(1, keepdim=True)) * slope
    if c["z"]:
        d = d + soft * (2 * lse * (member @ (s["d_z"].double() * over).float()))[:, None]
    return {"counts": counts.to(torch.int32), "tokens": tokens.to(torch.int32), "mean_prob": mean.float(), "loss": loss.float(),
            "z_loss": z_loss.float() if c["z"] else None, "d_logits": (d * live[:, None]).to(s["d_logits"].dtype)}


# ---------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without

def work(case):
    T = case["T"]
    if case["op"] in ("block", "block_grad"):
        H = case["H"]
        gate = {"none": 0, "channel": 2 * H, "token": 4 * T, "element": 2 * T * H}[case["gate"]]
        weights = 2 * H * (int(case["post"]) + int(case["pre"]))
        if case["op"] == "block":
            return {"bytes": 2 * T * H * (3 + int(case["pre"])) + gate + weights, "flops": 12.0 * T * H}
        b = 2 * T * H * (5 + int(case["pre"])) + weights + 2 * weights        # y, h, d_h, d_out; d_y, d_residual; the weights and theirs
        b += gate * (2 if case["gate"] == "channel" else 1) + gate
        return {"bytes": b, "flops": 30.0 * T * H}
    if case["op"] == "i8":
        K, N = case["K"], case["N"]
        size = 4 if case["out"] == "f32" else 2
        b = 2 * T * K * (3 if case["source"] == "block" else 1) + N * K + 4 * N + size * T * N
        b += (4 * N if case["bias"] else 0) + (size * T * N if case["base"] else 0)
        return {"bytes": b, "flops": 2.0 * T * K * N}
    E, k, M = case["E"], case["k"], case["M"]
    size = 2 if case["dtype"] == "bf16" else 4
    b = 2 * T * E * size + T * k * 8 + M * E * 8 + (4 * T if M > 1 else 0) + (T if case["mask"] else 0)
    return {"bytes": b, "flops": 20.0 * T * E}


# ---------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"block": _exact_block, "block_grad": _exact_block_grad, "i8": _exact_i8, "router": _exact_router}[case["op"]](case, s)


def _unit(x):
    """x over the root of its mean square, and that root's inverse."""
    inv = 1 / (torch.linalg.vector_norm(x, dim=1).square() / x.shape[1] + EPS).sqrt()[:, None]
    return x * inv, inv


def _exact_gate(case, s):
    g = s["gate"].double()
    if case["gate"] == "token":
        g = g[:, None]
    if case["act"] == "sigmoid":
        s1 = 1 / (1 + (-g).exp())
        return s1, s1 * (1 / (1 + g.exp()))
    return g, torch.ones_like(g)


def _exact_stream(case, s, y, residual, post):
    a = y.double()
    if post is not None:
        a = _unit(a)[0] * post.double()
    if case.get("gate", "none") != "none":
        a = a * _exact_gate(case, s)[0]
    return case.get("residual_scale", 1.0) * residual.double() + case.get("block_scale", 1.0) * a


def _exact_block(case, s):
    h = _exact_stream(case, s, s["y"], s["residual"], s["post"])
    if not case["pre"]:
        return {"h": h, "out": None}
    return {"h": h, "out": _unit(h.to(torch.bfloat16).double())[0] * s["pre"].double()}      # the norm is that of the stored stream


def _exact_block_grad(case, s):
    H = case["H"]
    total = s["d_h"].double()
    out = {"d_gate": None, "d_post": None, "d_pre": None}
    if case["pre"]:
        n, r = _unit(s["h"].double())
        d = s["d_out"].double()
        out["d_pre"] = torch.einsum("th,th->h", d, n)
        d = d * s["pre"].double()
        total = total + r * (d - n * (torch.einsum("th,th->t", d, n) / H)[:, None])
    out["d_residual"] = case["residual_scale"] * total
    y = s["y"].double()
    n, r = _unit(y)
    back = case["block_scale"] * total
    if s["gate"] is not None:
        value, slope = _exact_gate(case, s)
        dg = back * slope * (n * s["post"].double() if case["post"] else y)
        out["d_gate"] = dg.sum(0) if case["gate"] == "channel" else dg.sum(1) if case["gate"] == "token" else dg
        back = back * value
    if case["post"]:
        out["d_post"] = torch.einsum("th,th->h", back, n)
        back = back * s["post"].double()
        back = r * (back - n * (torch.einsum("th,th->t", back, n) / H)[:, None])
    out["d_y"] = back
    return out


def _exact_i8(case, s):
    x, h = s["x"].double(), None
    if case["source"] == "block":
        h = _exact_stream(case, s, s["x"], s["residual"], s["post"])
        x = _unit(h.to(torch.bfloat16).double())[0] * s["pre"].double()
    scale = x.abs().max(1)[0][:, None] / 127
    q = torch.nan_to_num(torch.round(x / scale))
    y = (q @ s["w_q"].double().t()) * (scale * s["w_scale"].double())
    if case["bias"]:
        y += s["bias"].double()
    if case["base"]:
        y += s["base"].double()
    return {"h": h, "out": y}


def _exact_router(case, s):
    T, E, k, M = case["T"], case["E"], case["k"], case["M"]
    z = s["logits"].double().cpu().numpy()
    idx = s["topk_idx"].cpu().numpy()
    gw = s["d_w"].double().cpu().numpy() * case["scale"]
    live = np.ones(T, dtype=bool) if s["mask"] is None else s["mask"].cpu().numpy() != 0
    model = np.zeros(T, dtype=int) if M == 1 else s["model_of_tenant"].cpu().numpy()[s["tenant_id"].cpu().numpy()]
    lse = np.logaddexp.reduce(z, axis=1)
    soft = np.exp(z - lse[:, None])
    if case["score"] == "softmax":
        score, slope = soft, np.ones_like(z)
    else:
        score, slope = np.exp(-np.logaddexp(0, -z)), np.exp(-np.logaddexp(0, z))
    p = score / score.sum(1, keepdims=True)
    rows = np.arange(T)[:, None]
    w = score[rows, idx]
    d = np.zeros_like(z)
    if case["renorm"]:
        w = w / w.sum(1, keepdims=True)
        d[rows, idx] = w * (gw - (gw * w).sum(1, keepdims=True)) * slope[rows, idx]
    else:
        d[rows, idx] = gw * w * slope[rows, idx]
        if case["score"] == "softmax":
            d -= soft * (gw * w).sum(1, keepdims=True)
    counts, tokens = np.zeros((M, E), dtype=np.int32), np.zeros(M, dtype=np.int32)
    mean, loss, z_loss = np.zeros((M, E)), np.zeros(M), np.zeros(M)
    for m in range(M):
        t = np.nonzero(live & (model == m))[0]
        tokens[m] = t.size
        if t.size == 0:
            continue
        counts[m] = np.bincount(idx[t].ravel(), minlength=E)
        mean[m] = p[t].mean(0)
        loss[m] = E / (k * t.size) * (counts[m] * mean[m]).sum()
        z_loss[m] = (lse[t] ** 2).mean()
        f = counts[m] * (float(s["d_loss"][m]) * E / (k * t.size ** 2))
        d[t] += p[t] * (f - (p[t] @ f)[:, None]) * slope[t]
        if case["z"]:
            d[t] += soft[t] * (2 * lse[t] * float(s["d_z"][m]) / t.size)[:, None]
    d[~live] = 0
    return {"counts": counts, "tokens": tokens, "mean_prob": mean, "loss": loss, "z_loss": z_loss if case["z"] else None, "d_logits": d}
