"""The operators around the layer together, as a block of a model runs them: the norms on both sides of an attention block with its gate, in
8 bits, a shared projection in 8-bit integers with the tenants' adapters beside it, the router's logits, choice and balance loss, and
the gradients back to the block and to the stream; each stage against the formulas in 64 bits on what the stage before it gave.

Tolerances as in the operators' own tests (bf16 half a step, 2^-8; integers half a step of 127; fp32 sums counted in u = 2^-24).
"""
import numpy as np
import pytest
import torch

from paper_2604_26881_b200 import binding as B
from test_balance import U, gradient, reference

pytestmark = pytest.mark.gpu
BF, HALF = torch.bfloat16, 2.0 ** -8


@pytest.mark.parametrize("T", [1, 33, 700])
@pytest.mark.parametrize("graph", [False, True])
def test_block(T, graph):
    H, N, E, k, M, n_tenants, rank = 512, 640, 60, 4, 2, 5, 8
    g = torch.Generator().manual_seed(T)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(BF)
    host = dict(y=rnd(T, H, std=0.5), res=rnd(T, H, std=2.0), post=rnd(H, std=0.1) + 1, pre=rnd(H, std=0.1) + 1, gate=rnd(T, H), w=rnd(N, H, std=0.05),
                a=rnd(n_tenants, rank, H, std=0.05), b=rnd(n_tenants, N, rank, std=0.05), router=rnd(E, H, std=0.05),
                tenant=torch.randint(0, n_tenants, (T,), generator=g, dtype=torch.int32), mot=(torch.arange(n_tenants) % M).to(torch.int32),
                mask=(torch.rand(T, generator=g) < 0.8).to(torch.uint8), d_w=torch.randn(T, k, generator=g), d_out=rnd(T, H, std=0.1), d_h=rnd(T, H, std=0.1))
    d = {n: t.cuda() for n, t in host.items()}
    e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda:0")
    o = dict(h=e(T, H, dt=BF), xn=e(T, H, dt=BF), q=e(T, H, dt=torch.int8), qs=e(T), wq=e(N, H, dt=torch.int8), ws=e(N), p=e(T, N), logits=e(T, E),
             idx=e(T, k, dt=torch.int32), tw=e(T, k), counts=e(M, E, dt=torch.int32), tokens=e(M, dt=torch.int32), mean=e(M, E), loss=e(M), z=e(M),
             dl=e(T, E), dy=e(T, H, dt=BF), dr=e(T, H, dt=BF), dg=e(T, H, dt=BF), dpost=e(H), dpre=e(H))
    rule = B.moe_gating(score="sigmoid", renormalize=True, scale=2.5)
    one = torch.ones(M, device="cuda:0")
    models = dict(tenant_id=d["tenant"], model_of_tenant=d["mot"])
    norm = dict(post_weight=d["post"], pre_weight=d["pre"], gate=d["gate"], gate_act="sigmoid", residual_scale=0.5)

    def block():
        B.moe_quantize_i8(d["w"], o["wq"], o["ws"])
        B.moe_block_norm(d["y"], d["res"], o["h"], 1e-6, out=o["xn"], out_q=o["q"], q_scale=o["qs"], **norm)
        B.moe_project_i8(o["q"], o["qs"], o["wq"], o["ws"], o["p"])
        B.moe_project(o["xn"], None, o["p"], base=o["p"], a=d["a"], b=d["b"], tenant_id=d["tenant"])
        B.moe_project(o["xn"], d["router"], o["logits"])
        B.moe_gate(o["logits"], rule, o["idx"], o["tw"], **models)
        B.moe_balance_loss(o["logits"], o["idx"], o["counts"], o["tokens"], o["mean"], o["loss"], score="sigmoid", z_loss=o["z"], mask=d["mask"], **models)
        B.moe_gate_backward(o["logits"], rule, o["idx"], o["dl"], d_topk_w=d["d_w"], counts=o["counts"], tokens=o["tokens"], d_loss=one, d_z_loss=one,
                            mask=d["mask"], **models)
        B.moe_block_norm_backward(d["y"], o["h"], 1e-6, d_out=d["d_out"], d_h=d["d_h"], d_block=o["dy"], d_residual=o["dr"], d_gate=o["dg"],
                                  d_post_weight=o["dpost"], d_pre_weight=o["dpre"], **norm)

    block()
    torch.cuda.synchronize()
    if graph:
        first = {n: t.clone() for n, t in o.items()}
        for t in o.values():
            t.zero_()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            block()
        gr.replay()
        gr.replay()
        torch.cuda.synchronize()
        for n in o:
            assert torch.equal(o[n], first[n]), n
    c = {n: t.cpu() for n, t in o.items()}
    rms = lambda x: x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-6)
    f = {n: t.double() for n, t in host.items() if t.dtype == BF}
    a = rms(f["y"]) * f["post"] * torch.sigmoid(f["gate"])
    h = 0.5 * f["res"] + a
    assert ((c["h"].double() - h).abs() <= HALF * h.abs() + 64 * U * (h.abs() + a.abs())).all()
    xn = rms(c["h"].double()) * f["pre"]
    assert ((c["xn"].double() - xn).abs() <= (HALF + 80 * U) * xn.abs()).all()
    assert ((c["q"].double() * c["qs"].double()[:, None] - xn).abs() <= (0.5 + 0.001) * c["qs"].double()[:, None]).all()
    ad = torch.stack([f["b"][u] @ (f["a"][u] @ c["xn"][t].double()) for t, u in enumerate(host["tenant"].tolist())])
    size = torch.stack([f["b"][u].abs() @ (f["a"][u].abs() @ c["xn"][t].double().abs()) for t, u in enumerate(host["tenant"].tolist())])
    full = (c["q"].double() @ c["wq"].double().t()) * c["qs"].double()[:, None] * c["ws"].double()
    assert ((c["p"].double() - full - ad).abs() <= 530 * U * (full.abs() + size)).all()
    exact = xn @ f["w"].t()
    lim = 0.502 * (c["qs"].double()[:, None] * f["w"].abs().sum(1) + xn.abs().sum(1)[:, None] * c["ws"].double()) + 0.26 * H * c["qs"].double()[:, None] * c["ws"].double()
    assert ((full - exact).abs() <= lim).all()
    z = c["logits"].double().numpy()
    model = host["mot"].numpy()[host["tenant"].numpy()]
    live = host["mask"].numpy() != 0
    ref = reference(z, c["idx"].numpy(), "sigmoid", M, live, model)
    assert np.array_equal(c["counts"].numpy(), ref["counts"]) and np.array_equal(c["tokens"].numpy(), ref["tokens"])
    for n in ("mean", "loss", "z"):
        np.testing.assert_allclose(c[n].numpy(), ref[n], rtol=300 * U, atol=300 * U)
    want, mag = gradient(z, c["idx"].numpy(), dict(score="sigmoid", renorm=True, scale=2.5), ref, host["d_w"].numpy(), np.ones(M, np.float32),
                         np.ones(M, np.float32), live, model)
    assert (np.abs(c["dl"].double().numpy() - want) <= 300 * U * mag + U * np.abs(want) + 1e-12).all()
    # the gradients to the block, the stream, the gate and the weights: differentiation of the forward formula at the stored stream
    y, gate, post, pre, hh = (t.clone().requires_grad_() for t in (f["y"], f["gate"], f["post"], f["pre"], c["h"].double()))
    dh, dpre = torch.autograd.grad(rms(hh) * pre, (hh, pre), f["d_out"])
    total = f["d_h"] + dh
    dy, dg, dpost = torch.autograd.grad(rms(y) * post * torch.sigmoid(gate), (y, gate, post), total)
    for name, ref_g in (("dr", 0.5 * total), ("dy", dy), ("dg", dg)):
        scale = ref_g.abs().mean(1, keepdim=True)                      # (sums over a row: their errors are those of its magnitudes)
        assert ((c[name].double() - ref_g).abs() <= HALF * 1.001 * ref_g.abs() + 400 * U * (ref_g.abs() + 4 * scale)).all(), name
    for name, ref_g, terms in (("dpost", dpost, (total * torch.sigmoid(f["gate"]) * rms(f["y"])).abs().sum(0)), ("dpre", dpre, (f["d_out"] * rms(c["h"].double())).abs().sum(0))):
        assert ((c[name].double() - ref_g).abs() <= 400 * U * terms + U * ref_g.abs()).all(), name
