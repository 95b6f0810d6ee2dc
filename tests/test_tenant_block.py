"""One block of a multi-tenant model from the calls that take no context and the layer's own: residual add and norm, router logits,
gating rule, dispatch, routed experts, a shared expert whose three projections carry the tenants' adapters, combine.

Checked against the formulas in 64 bits at the layer's own tolerances (rtol 2e-2, atol 2e-3: bf16 operands and stored
intermediates, fp32 accumulation); the choice of experts must equal the 64-bit rule wherever its values are not closer than the
fp32 logits can tell (1e-4, far above the rounding of sums of 256 products of order one).
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from harness import ATOL, RTOL
from paper_2604_26881_b200 import binding as B
from paper_2604_26881_b200 import workloads as W
from test_gate import reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 40, 300])
@pytest.mark.parametrize("graph", [False, True])
def test_block_with_tenants_adapters(T, graph):
    H, E, I, k, Is, n_tenants, n, rank = 256, 16, 128, 4, 256, 6, 4, 8
    dev = torch.device("cuda:0")
    wl = W.MoEWorkload("block", T=T, H=H, E=E, I=I, k=k, Is=Is, n_tenants=n_tenants, G=4, tenant_layout="uniform")
    wts = W.make_weights(wl, seed=9)
    _, tenant, _ = W.make_tokens(wl, seed=9)
    g = torch.Generator().manual_seed(4)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16)
    attn, res = rnd(T, H, std=0.5), rnd(T, H)
    table = torch.tensor([0, 1, 2, 3, -1, 1], dtype=torch.int32)
    scale = torch.rand(n, generator=g) + 0.5
    bias = torch.randn(1, E, generator=g) * 0.05
    low = {name: (rnd(n, rank, kk, std=0.1), rnd(n, nn, rank, std=0.1)) for name, kk, nn in (("gate", H, Is), ("up", H, Is), ("down", Is, H))}
    layer = B.MoELayer(H=H, E=E, I=I, k=k, Is=Is, n_tenants=n_tenants, max_tokens=T)
    try:
        layer.set_layer_weights(0, wts)
        d = {name: v.to(dev) for name, v in dict(attn=attn, res=res, rms=wts["rms_w"], tenant=tenant, table=table, scale=scale, bias=bias,
                                                 router=wts["router_w"][0], ws_gate=wts["ws_gate"][0], ws_up=wts["ws_up"][0],
                                                 ws_down=wts["ws_down"][0]).items()}
        ad = {name: dict(a=a.to(dev), b=b.to(dev), scale=d["scale"], tenant_id=d["tenant"], adapter_of_tenant=d["table"]) for name, (a, b) in low.items()}
        rule = B.moe_gating(score="sigmoid", n_groups=4, keep_groups=2, group_score="top2", renormalize=True, scale=1.5)
        R = T * k
        e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device=dev)
        o = dict(h=e(T, H, dt=torch.bfloat16), xn=e(T, H, dt=torch.bfloat16), q=e(T, H).to(torch.float8_e4m3fn), qs=e(T, 2), logits=e(T, E),
                 idx=e(T, k, dt=torch.int32), w=e(T, k), perm=e(R, dt=torch.int32), inv=e(R, dt=torch.int32), off=e(E + 1, dt=torch.int32),
                 xp=e(R + 128, H, dt=torch.bfloat16), yp=e(R, H), g=e(T, Is, dt=torch.bfloat16), u=e(T, Is, dt=torch.bfloat16), ys=e(T, H),
                 sg=torch.ones(T, device=dev), out=e(T, H, dt=torch.bfloat16))

        def block():
            B.moe_add_rmsnorm(d["attn"], d["rms"], 1e-6, residual=d["res"], residual_out=o["h"], out=o["xn"], out_q=o["q"], q_scale=o["qs"])
            B.moe_project(o["xn"], d["router"], o["logits"])
            B.moe_gate(o["logits"], rule, o["idx"], o["w"], balance_bias=d["bias"])
            B.moe_dispatch(layer.ctx, o["xn"], o["idx"], d["tenant"], T, 4, o["perm"], o["inv"], None, o["off"], None, o["xp"])
            B.moe_experts(layer.ctx, 0, o["xn"], o["xp"], o["perm"], o["off"], d["tenant"], T, 4, o["yp"])
            B.moe_project(o["xn"], d["ws_gate"], o["g"], **ad["gate"])
            B.moe_project(o["xn"], d["ws_up"], o["u"], **ad["up"])
            act = torch.nn.functional.silu(o["g"].float()).mul_(o["u"].float()).to(torch.bfloat16)
            o["act"] = act
            B.moe_project(act, d["ws_down"], o["ys"], **ad["down"])
            B.moe_combine(layer.ctx, o["yp"], o["inv"], o["w"], o["ys"], o["sg"], T, o["out"])

        block()
        torch.cuda.synchronize()
        assert B.moe_last_status(layer.ctx)[0] == 0
        if graph:
            first = {name: v.clone() for name, v in o.items()}
            for v in o.values():
                if v is not o["sg"] and v is not o["act"]:
                    v.zero_()
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr):
                block()
            gr.replay()
            gr.replay()
            torch.cuda.synchronize()
            for name in ("h", "xn", "logits", "idx", "w", "perm", "yp", "g", "u", "ys", "out"):
                assert torch.equal(o[name], first[name]), name
    finally:
        layer.close()
    c = {name: v.cpu() for name, v in o.items()}
    close = lambda got, ref: ((got.double() - ref).abs() <= ATOL + RTOL * ref.abs()).all()
    # stage by stage, each on the inputs that the stage before really gave
    h = (attn.float() + res.float()).to(torch.bfloat16)
    assert torch.equal(c["h"], h)
    xn = h.double() / torch.sqrt((h.double() ** 2).mean(1, keepdim=True) + 1e-6) * wts["rms_w"].double()
    assert ((c["xn"].double() - xn).abs() <= 2.0 ** -8 * 1.001 * xn.abs() + 1e-30).all()
    full = c["q"].double() * c["qs"].double().repeat_interleave(128, 1)
    assert ((full - xn).abs() <= 2.0 ** -4 * 1.001 * xn.abs() + 2.0 ** -10 * 1.001 * c["qs"].double().repeat_interleave(128, 1)).all()
    xb = c["xn"].double()
    z = xb @ wts["router_w"][0].double().t()
    assert (c["logits"].double() - z).abs().max() < 1e-4
    br = bias.double().numpy().repeat(T, 0)
    ref_idx, ref_w = reference(z.numpy(), k, score="sigmoid", n_groups=4, keep=2, group_score="top2", renorm=True, scale=1.5, bias=br)
    v = torch.sigmoid(z).numpy() + br
    gs = np.sort(np.sort(v.reshape(T, 4, 4), 2)[:, :, -2:].sum(2), 1)
    clear = (np.diff(np.sort(v, 1), axis=1).min(1) > 1e-4) & (np.diff(gs, axis=1).min(1) > 2e-4)
    assert T < 10 or clear.sum() > T // 2
    assert np.array_equal(c["idx"].numpy()[clear], ref_idx[clear])
    np.testing.assert_allclose(c["w"].numpy()[clear], ref_w[clear], rtol=1e-3)
    routed = torch.zeros(T, H, dtype=torch.float64)
    for t in range(T):
        for j in range(k):
            ex = int(c["idx"][t, j])
            y = torch.nn.functional.silu(wts["pool_gate"][ex].double() @ xb[t]) * (wts["pool_up"][ex].double() @ xb[t])
            routed[t] += float(c["w"][t, j]) * (wts["pool_down"][ex].double() @ y)
    adapter = table.long()[tenant.long()]

    def projected(x, name):
        y = x @ wts["ws_" + name][0].double().t()
        for i in range(n):
            t = adapter == i
            y[t] += float(scale[i]) * (x[t] @ low[name][0][i].double().t()) @ low[name][1][i].double().t()
        return y
    assert close(c["g"], projected(xb, "gate")) and close(c["u"], projected(xb, "up"))
    ys = projected(c["act"].double(), "down")
    assert close(c["ys"], ys)
    assert close(c["out"], routed + ys)


FIRST_CALLS = """
import torch
from paper_2604_26881_b200 import binding as B
dev = "cuda:0"
rnd = lambda *s: torch.randn(*s, device=dev).bfloat16()
w, a, b = rnd(320, 256), rnd(3, 16, 256), rnd(3, 320, 16)
calls = []
for T in (2, 40, 700, 9000):
    x, out, y, z = rnd(T, 256), torch.zeros(T, 320, device=dev), rnd(T, 256), torch.randn(T, 64, device=dev)
    idx, wt, tenant = torch.zeros(T, 4, dtype=torch.int32, device=dev), torch.zeros(T, 4, device=dev), (torch.arange(T, device=dev) % 3).int()
    calls.append((lambda x=x, out=out, tenant=tenant: B.moe_project(x, w, out, a=a, b=b, tenant_id=tenant), out))
    calls.append((lambda z=z, idx=idx, wt=wt: B.moe_gate(z, B.moe_gating(), idx, wt), wt))
    calls.append((lambda x=x, y=y: B.moe_add_rmsnorm(x, w.view(-1)[:256], 1e-6, out=y), y))
torch.cuda.synchronize()
for run, out in calls:
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    replayed = out.clone()
    run()
    torch.cuda.synchronize()
    assert torch.equal(replayed, out) and out.float().abs().sum() > 0
print("captured")
"""


def test_first_calls_of_a_process_may_be_captured():
    """Kernels are loaded, and launch shapes looked up, inside the capture."""
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, timeout=300,
                          cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0 and "captured" in done.stdout, done.stdout + done.stderr


def test_calls_on_three_streams_at_once():
    """Launches of different shapes share the SMs, their tensor memory included; each gives what it gives alone."""
    g = torch.Generator(device="cuda:0").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda:0").mul_(0.1).bfloat16()
    w, a, b = rnd(1408, 1024), rnd(40, 16, 1024), rnd(40, 1408, 16)
    sizes = (3, 50, 200, 700, 2000, 4)
    work = []
    for T in sizes:
        x, tenant = rnd(T, 1024), (torch.arange(T, device="cuda:0") % 40).int()
        alone, out = torch.empty(T, 1408, device="cuda:0"), torch.empty(T, 1408, device="cuda:0")
        call = lambda o, x=x, tenant=tenant: B.moe_project(x, w, o, a=a, b=b, tenant_id=tenant)
        call(alone)
        work.append((call, alone, out))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for rep in range(20):
        for i, (call, alone, out) in enumerate(work):
            out.zero_()
        torch.cuda.synchronize()
        for i, (call, alone, out) in enumerate(work):
            with torch.cuda.stream(streams[(i + rep) % 3]):
                for _ in range(3):
                    call(out)
        torch.cuda.synchronize()
        for call, alone, out in work:
            assert torch.equal(alone, out)
