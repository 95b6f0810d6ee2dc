"""Gating rules (moe_gate, moe_set_gating) against a plain statement of the rules in 64 bits.

The choice is defined in double precision, so the expert ids must be equal wherever the 64-bit values of two experts are not
within a few double ulps of each other (random fp32 inputs never are).  Weights are fp32: an exponential (2 ulp), a sum of
at most 8 + 5 terms, a quotient and a product, below 32 roundings of 2^-24 relative; the argument z - ref of the exponential is
rounded too, which costs 2^-24 |z - ref| relative (at most 40 units for the logits used here where a weight matters).
"""
import ctypes
import math

import numpy as np
import pytest
import torch

from harness import GpuLayer
from paper_2604_26881_b200 import binding as B
from paper_2604_26881_b200 import workloads as W

FMAX = float(np.finfo(np.float32).max)
W_RTOL = 2.0 ** -24 * (32 + 40)


def reference(z, k, *, score, n_groups=1, keep=1, group_score="max", renorm=False, scale=1.0, bias=None):
    """One row at a time, as the rules read.  z [T, E] float64; bias [T, E] or None.  (idx [T, k], w [T, k])."""
    T, E = z.shape
    idx, w = np.zeros((T, k), np.int64), np.zeros((T, k))
    size = E // n_groups
    for t in range(T):
        zt = np.where(np.isnan(z[t]), -np.inf, np.minimum(z[t], FMAX))
        with np.errstate(over="ignore", under="ignore", invalid="ignore"):
            if score == "softmax":
                s = np.where(np.isneginf(zt), 0.0, np.exp(zt - zt.max()))
                s = s / s.sum() if s.sum() > 0 else s
            else:
                s = np.where(zt >= 0, 1 / (1 + np.exp(-np.abs(zt))), np.exp(-np.abs(zt)) / (1 + np.exp(-np.abs(zt))))
        v = zt if bias is None else s + np.where(np.isnan(bias[t]), -np.inf, bias[t])
        vg = v if bias is not None or group_score == "max" or size == 1 else s
        groups = []
        for g in range(n_groups):
            best = sorted(vg[g * size:(g + 1) * size], reverse=True)
            groups.append(best[0] + (best[1] if group_score == "top2" and size > 1 else 0.0))
        kept = sorted(range(n_groups), key=lambda g: (-groups[g], g))[:keep]
        allowed = [e for e in range(E) if e // size in kept]
        chosen = sorted(allowed, key=lambda e: (-v[e], e))[:k]
        idx[t] = chosen
        if renorm:
            # relative to the largest chosen score, so that nothing underflows
            zc = zt[chosen]
            logs = zc if score == "softmax" else -np.logaddexp(0.0, -zc)
            if np.isneginf(logs).all():
                continue
            x = np.exp(logs - logs.max())
            w[t] = x / x.sum() * scale
        else:
            w[t] = s[chosen] * scale
    return idx, w


def run(z, k, dev="cuda:0", bias=None, tenant=None, mot=None, dtype=torch.float32, pad=0, tie=False, **rule):
    T, E = z.shape
    full = torch.full((T, E + pad), 9.0, dtype=dtype, device=dev)
    full[:, :E] = torch.as_tensor(z, dtype=torch.float64).to(dtype).to(dev)
    n = 64
    idx_flat = torch.full((T * k + n,), -7, dtype=torch.int32, device=dev)
    w_flat = torch.full((T * k + n,), -7.0, dtype=torch.float32, device=dev)
    idx, w = idx_flat[:T * k].view(T, k), w_flat[:T * k].view(T, k)
    flag = torch.full((T,), 9, dtype=torch.uint8, device=dev) if tie else None
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    r = B.moe_gating(score=rule.get("score", "softmax"), n_groups=rule.get("n_groups", 1), keep_groups=rule.get("keep", 1),
                     group_score=rule.get("group_score", "max"), renormalize=rule.get("renorm", False), scale=rule.get("scale", 1.0))
    as_dev = lambda t, d: None if t is None else torch.as_tensor(t).to(d).to(dev)
    B.moe_gate(full[:, :E], r, idx, w, balance_bias=as_dev(bias, torch.float32), tenant_id=as_dev(tenant, torch.int32),
               model_of_tenant=as_dev(mot, torch.int32), tie_flag=flag, status_out=status)
    torch.cuda.synchronize()
    assert (idx_flat[T * k:] == -7).all() and (w_flat[T * k:] == -7).all(), "written past the end"
    return idx.cpu().numpy(), w.double().cpu().numpy(), (flag.cpu().numpy() if tie else None), int(status.item())


def check(z, k, bias=None, dtype=torch.float32, pad=0, **rule):
    zr = torch.as_tensor(z, dtype=torch.float64).to(dtype).double().numpy()
    br = None if bias is None else np.broadcast_to(torch.as_tensor(bias).float().double().numpy().reshape(1, -1), zr.shape)
    scale = float(np.float32(rule.get("scale", 1.0)))
    ref_idx, ref_w = reference(zr, k, bias=br, **{**rule, "scale": scale})
    idx, w, _, status = run(z, k, bias=None if bias is None else np.asarray(bias).reshape(1, -1), dtype=dtype, pad=pad, **rule)
    assert status == 0
    bad = np.nonzero((idx != ref_idx).any(1))[0]
    assert bad.size == 0, f"{bad.size} rows differ, first {bad[:3]}: got {idx[bad[:3]]}, want {ref_idx[bad[:3]]}"
    np.testing.assert_allclose(w, ref_w, rtol=W_RTOL, atol=1e-37)
    return idx


gpu = pytest.mark.gpu
RULES = [
    dict(score="softmax"),
    dict(score="softmax", renorm=True, scale=2.5),
    dict(score="sigmoid", renorm=True),
    dict(score="sigmoid", scale=0.5),
]


@gpu
@pytest.mark.parametrize("E,k", [(1, 1), (2, 2), (7, 3), (8, 8), (60, 4), (63, 8), (64, 1), (65, 8), (100, 5), (128, 8), (129, 2), (200, 8), (255, 8), (256, 8)])
@pytest.mark.parametrize("with_bias", [False, True])
def test_every_router_width(E, k, with_bias):
    g = np.random.default_rng(E * 10 + k)
    z = g.standard_normal((37, E)) * 2
    bias = g.standard_normal(E) * 0.1 if with_bias else None
    for i, rule in enumerate(RULES):
        check(z, k, bias=bias, pad=(0, 1, 4, 8)[i], **rule)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("E,n_groups,keep", [(256, 8, 4), (256, 32, 8), (256, 1, 1), (64, 8, 3), (60, 4, 2), (60, 12, 5), (252, 6, 3),
                                             (32, 32, 9), (96, 3, 1), (248, 31, 30), (128, 2, 1), (16, 2, 2)])
@pytest.mark.parametrize("group_score", ["max", "top2"])
def test_groups(dtype, E, n_groups, keep, group_score):
    g = np.random.default_rng(E + n_groups)
    k = min(8, keep * (E // n_groups))
    z = g.standard_normal((65, E))
    for score in ("softmax", "sigmoid"):
        for bias in (None, g.standard_normal(E) * 0.05):
            check(z, k, bias=bias, dtype=dtype, score=score, n_groups=n_groups, keep=keep, group_score=group_score, renorm=True)


@gpu
@pytest.mark.parametrize("T,ld,E", [(140, 1 << 24, 60), (9000, 1 << 18, 60), (16400, 1 << 18, 256)])
def test_rows_beyond_32_bit_offsets(T, ld, E):
    g = np.random.default_rng(T)
    z = torch.as_tensor(g.standard_normal((T, E))).to(torch.bfloat16)
    far = torch.empty(T * ld, dtype=torch.bfloat16, device="cuda:0").as_strided((T, E), (ld, 1))
    far.copy_(z)
    rule = B.moe_gating(score="sigmoid", renormalize=True)
    outs = []
    for logits in (z.to("cuda:0"), far):
        idx, w = torch.empty(T, 4, dtype=torch.int32, device="cuda:0"), torch.empty(T, 4, device="cuda:0")
        B.moe_gate(logits, rule, idx, w)
        outs.append((idx, w))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


@gpu
@pytest.mark.parametrize("T", [0, 1, 2, 3, 4, 5, 127, 1000, 4099])
def test_numbers_of_tokens(T):
    g = np.random.default_rng(T)
    z = g.standard_normal((T, 60))
    if T == 0:
        idx, w, _, _ = run(z, 4, score="softmax")
        assert idx.shape == (0, 4)
        return
    check(z, 4, bias=g.standard_normal(60) * 0.1, score="sigmoid", n_groups=4, keep=2, group_score="top2", renorm=True)


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_values_take_the_lower_id(score, with_bias, dtype):
    """Few distinct logits: nearly every neighbour is an exact tie, inside a lane, between lanes and at the k-th rank."""
    g = np.random.default_rng(5)
    for E, n_groups, keep in [(60, 1, 1), (256, 8, 3), (96, 6, 2)]:
        z = g.integers(-2, 3, (50, E)).astype(float)
        z[0] = 0.0
        z[1] = -0.0
        z[2, ::2] = 0.0
        z[2, 1::2] = -0.0
        bias = np.full(E, 0.25) if with_bias else None
        check(z, 8, bias=bias, dtype=dtype, score=score, n_groups=n_groups, keep=keep, renorm=True)
        if with_bias:
            check(z, 8, bias=g.integers(0, 2, E) * 0.5, dtype=dtype, score=score, n_groups=n_groups, keep=keep, renorm=True)


@gpu
def test_order_is_decided_in_64_bits():
    """Pairs whose values differ by less than fp32 can hold: v = sigmoid(z) + b with b stepping by one fp32 ulp of 1."""
    g = np.random.default_rng(9)
    T, E = 64, 256
    z = np.zeros((T, E))
    z += g.integers(0, 4, (T, E)) * 1e-7
    bias = 1.0 + g.integers(0, 3, E) * 2.0 ** -23
    for score in ("sigmoid", "softmax"):
        check(z, 8, bias=bias, score=score, n_groups=8, keep=3, group_score="top2")
        check(z, 8, bias=bias, score=score)
    # neighbouring fp32 logits without a bias
    base = np.float32(1.5)
    steps = g.integers(0, 30, (T, E))
    zz = (base + steps * np.spacing(base)).astype(np.float64)
    check(zz, 8, score="sigmoid")
    check(zz, 8, score="softmax", n_groups=8, keep=2)


@gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_masked_and_extreme_logits(score, renorm):
    g = np.random.default_rng(3)
    E, k = 60, 4
    z = g.standard_normal((16, E))
    z[0] = -np.inf                                  # nothing is left
    z[1, :] = -np.inf
    z[1, [7, 33]] = [0.5, 1.5]                      # fewer than k are left
    z[2, ::2] = -np.inf
    z[3, ::3] = -FMAX                               # the lowest finite value as a mask
    z[4, :] = -FMAX
    z[5, 10] = np.nan
    z[5, 11] = 50.0
    z[6, :] = np.nan
    z[7, 20] = np.inf
    z[8, [3, 30]] = np.inf
    z[9] = 1e30 * np.sign(z[9])
    z[10] = -200.0 + z[10]                          # scores below the smallest fp32 number
    z[11] = 200.0 + z[11]
    z[12] = z[12] * 1e-42                           # denormal logits
    z[13, 5:] = -np.inf
    z[14] = -1000.0
    z[15, :] = -np.inf
    z[15, 59] = -FMAX
    check(z, k, score=score, renorm=renorm)
    check(z, k, score=score, renorm=renorm, n_groups=6, keep=3)
    check(z, k, score=score, renorm=renorm, n_groups=6, keep=3, bias=g.standard_normal(E) * 0.1, group_score="top2")
    bias = g.standard_normal(E) * 0.1
    bias[[4, 9]] = -np.inf
    bias[12] = np.nan
    check(z, k, score=score, renorm=renorm, bias=bias)


def check_repeated(rows, T, k, bias=None, dtype=torch.float32, pad=0, seed=0, **rule):
    """A long batch: `rows` in random order, many times over.  The reference looks at every row once."""
    pick = np.random.default_rng(seed).integers(0, len(rows), T)
    pick[:len(rows)] = np.arange(len(rows))
    zr = torch.as_tensor(rows, dtype=torch.float64).to(dtype).double().numpy()
    br = None if bias is None else np.broadcast_to(torch.as_tensor(bias).float().double().numpy().reshape(1, -1), zr.shape)
    ref_idx, ref_w = reference(zr, k, bias=br, **{**rule, "scale": float(np.float32(rule.get("scale", 1.0)))})
    idx, w, flag, status = run(rows[pick], k, bias=None if bias is None else np.asarray(bias).reshape(1, -1), dtype=dtype, pad=pad, tie=True, **rule)
    assert status == 0
    bad = np.nonzero((idx != ref_idx[pick]).any(1))[0]
    assert bad.size == 0, f"{bad.size} tokens differ, first {bad[:3]}: got {idx[bad[:3]]}, want {ref_idx[pick[bad[:3]]]}"
    np.testing.assert_allclose(w, ref_w[pick], rtol=W_RTOL, atol=1e-37)
    # what a token gets does not depend on the token beside it
    for i in range(len(rows)):
        assert len(np.unique(w[pick == i], axis=0)) == 1 and len(set(flag[pick == i])) == 1


# batches that four lanes per token work on: from 8192 tokens with up to 128 experts, from 16384 or 32768 beyond
LONG = [(8192, 60, 4, {}), (8199, 64, 8, {}), (8192, 7, 3, {}), (8193, 1, 1, {}), (8200, 100, 8, {}), (8192, 128, 8, dict(n_groups=4, keep=2)),
        (8195, 128, 5, dict(n_groups=2, keep=1)), (8192, 96, 8, dict(n_groups=3, keep=2)), (8192, 60, 4, dict(n_groups=4, keep=2)),
        (8192, 8, 8, {}), (8192, 64, 7, dict(n_groups=2, keep=1)), (16387, 256, 8, {}), (16384, 256, 8, dict(n_groups=8, keep=4)), (16390, 200, 6, {}),
        (16384, 256, 7, dict(n_groups=4, keep=1)), (16384, 256, 1, dict(n_groups=2, keep=1)), (32768, 256, 8, dict(n_groups=8, keep=3)),
        (16385, 60, 4, {}), (16391, 128, 8, dict(n_groups=4, keep=3)), (4097, 64, 8, {}), (4100, 128, 6, {}), (8193, 256, 8, dict(n_groups=8, keep=2))]


@gpu
@pytest.mark.parametrize("T,E,k,groups", LONG)
def test_long_batches(T, E, k, groups):
    g = np.random.default_rng(T + E + k)
    rows = g.standard_normal((300, E)) * 1.5
    for score in ("softmax", "sigmoid"):
        for bias in (None, g.standard_normal(E) * 0.05):
            for group_score in ("max", "top2") if groups else ("max",):
                for renorm, dtype, pad in ((True, torch.float32, 0), (False, torch.bfloat16, 8), (True, torch.float32, 3)):
                    check_repeated(rows, T, k, bias=bias, dtype=dtype, pad=pad, score=score, renorm=renorm, group_score=group_score, **groups)


@gpu
@pytest.mark.parametrize("T,E,groups", [(8192, 60, {}), (8192, 128, dict(n_groups=4, keep=2)), (16384, 256, dict(n_groups=8, keep=4)), (16384, 256, {}),
                                        (32768, 256, dict(n_groups=2, keep=1)), (16384, 60, {}), (16384, 128, dict(n_groups=4, keep=2))])
@pytest.mark.parametrize("k", [1, 5, 7, 8])
def test_long_batches_of_ties_and_near_ties(T, E, groups, k):
    """Exact ties, values that only 64 bits tell apart, masked and extreme rows, at the k-th rank and between groups."""
    g = np.random.default_rng(E + k)
    ties = g.integers(-2, 3, (40, E)).astype(float)
    near = g.integers(0, 4, (40, E)) * 1e-7
    ulps = (np.float32(1.5) + g.integers(0, 30, (40, E)) * np.spacing(np.float32(1.5))).astype(float)
    odd = g.standard_normal((12, E))
    odd[0] = -np.inf
    odd[1, 3:] = -np.inf
    odd[2, ::2] = -FMAX
    odd[3] = np.nan
    odd[4, 5] = np.inf
    odd[5] = 1e30 * np.sign(odd[5])
    odd[6] -= 200
    odd[7] *= 1e-42
    odd[8] = -FMAX
    odd[9] = 0.0
    odd[10] += 200
    rows = np.concatenate([ties, near, ulps, odd])
    for score in ("softmax", "sigmoid"):
        for bias in (None, 1.0 + g.integers(0, 3, E) * 2.0 ** -23, np.zeros(E)):
            for group_score in ("max", "top2") if groups else ("max",):
                check_repeated(rows, T, k, bias=bias, score=score, renorm=True, group_score=group_score, **groups)
        check_repeated(ties, T, k, dtype=torch.bfloat16, score=score, **groups)


@gpu
@pytest.mark.parametrize("T,score", [(8300, "sigmoid"), (16400, "softmax")])
def test_long_batches_of_several_models(T, score):
    g = np.random.default_rng(21)
    E, M, k = 60, 4, 4
    z = g.standard_normal((T, E))
    tenant, mot = g.integers(0, 9, T), np.arange(9) % M
    tenant[[3, T - 1]] = [9, -2]
    bias = g.standard_normal((M, E)) * 0.2
    rule = dict(score=score, renorm=True)
    idx, w, _, status = run(z, k, bias=bias, tenant=tenant, mot=mot, **rule)
    assert status == B.MOE_DEV_BAD_TENANT
    ok = (tenant >= 0) & (tenant < 9)
    safe = np.where(ok, tenant, 0)
    ref_idx, ref_w = reference(z.astype(np.float32).astype(float), k, bias=bias.astype(np.float32).astype(float)[mot[safe]], **rule)
    assert np.array_equal(idx[ok], ref_idx[ok])
    np.testing.assert_allclose(w[ok], ref_w[ok], rtol=W_RTOL)
    assert (idx[~ok] == np.arange(k)).all() and (w[~ok] == 0).all()


@gpu
def test_models_and_bad_tenants():
    g = np.random.default_rng(11)
    T, E, M, k = 130, 60, 3, 4
    z = g.standard_normal((T, E))
    tenant = g.integers(0, 6, T)
    mot = np.arange(6) % M
    bias = g.standard_normal((M, E)) * 0.3
    rule = dict(score="sigmoid", renorm=True, n_groups=4, keep=2, group_score="top2")
    tenant[[5, 90]] = [-1, 6]
    idx, w, _, status = run(z, k, bias=bias, tenant=tenant, mot=mot, **rule)
    assert status == B.MOE_DEV_BAD_TENANT
    safe = np.where((tenant < 0) | (tenant >= 6), 0, tenant)
    ref_idx, ref_w = reference(z.astype(np.float32).astype(float), k, bias=bias.astype(np.float32).astype(float)[mot[safe]], **rule)
    ok = (tenant >= 0) & (tenant < 6)
    assert np.array_equal(idx[ok], ref_idx[ok])
    np.testing.assert_allclose(w[ok], ref_w[ok], rtol=W_RTOL)
    assert (idx[~ok] == np.arange(k)).all() and (w[~ok] == 0).all()


@gpu
def test_tie_flag():
    z = np.linspace(-3, 3, 60)[None].repeat(3, 0).copy()
    z[1, 57] = z[1, 58]                     # ranks 2 and 3 equal
    z[2, 0] = z[2, 1]                       # equal far behind the choice
    for score in ("softmax", "sigmoid"):
        _, _, flag, _ = run(z, 4, tie=True, score=score)
        assert flag.tolist() == [0, 1, 0]


@gpu
def test_graph_stream_and_repeated_calls_agree():
    g = np.random.default_rng(2)
    dev = torch.device("cuda:0")
    T, E, k = 513, 256, 8
    z = torch.from_numpy(g.standard_normal((T, E))).float().to(dev)
    bias = torch.from_numpy(g.standard_normal((1, E)) * 0.05).float().to(dev)
    rule = B.moe_gating(score="sigmoid", n_groups=8, keep_groups=4, group_score="top2", renormalize=True)
    mk = lambda: (torch.empty(T, k, dtype=torch.int32, device=dev), torch.empty(T, k, device=dev))
    a, b, c = mk(), mk(), mk()
    B.moe_gate(z, rule, *a, balance_bias=bias)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.moe_gate(z, rule, *b, balance_bias=bias, stream=side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_gate(z, rule, *c, balance_bias=bias)
    graph.replay()
    torch.cuda.synchronize()
    for o in (b, c):
        assert torch.equal(a[0], o[0]) and torch.equal(a[1], o[1])
    z2 = z.roll(1, 0).contiguous()
    z.copy_(z2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c[0], a[0].roll(1, 0)) and torch.equal(c[1], a[1].roll(1, 0))


def _layer(E, k, M, T, seed=0, Is=128, H=256):
    wl = W.MoEWorkload("rule", T=T, H=H, E=E, I=128, k=k, Is=Is, M=M, n_tenants=2 * M, G=3, zipf_bias=True, tenant_layout="uniform")
    return wl, W.make_weights(wl, seed=seed)


@gpu
@pytest.mark.parametrize("E,M,path", [(60, 1, B.MOE_PATH_AUTO), (12, 3, B.MOE_PATH_AUTO), (60, 2, B.MOE_PATH_FMA), (96, 1, B.MOE_PATH_AUTO)])
def test_layer_with_a_rule(E, M, path):
    """moe_set_gating: the layer's own logits, then the rule.  The router without a rule (raw softmax) gives the logits' order
    of the same kernels; the rule's choice is checked against the 64-bit rule wherever fp32 logits decide it."""
    T, k = 200, 4
    wl, wts = _layer(E, k, M, T)
    x, tenant, mot = W.make_tokens(wl, seed=1)
    gl = GpuLayer(wl, [wts], max_tokens=T, model_of_tenant=mot)
    try:
        B.moe_set_option(gl.ctx, B.MOE_OPT_ROUTE_PATH, path)
        G = 3
        before = gl.forward(x, tenant, G)
        dev = gl.dev
        bias = (torch.randn(M, E, generator=torch.Generator().manual_seed(4)) * 0.1)
        n_groups, keep = (4, 2)
        rule = B.moe_gating(score="sigmoid", n_groups=n_groups, keep_groups=keep, group_score="top2", renormalize=True, scale=1.5)
        bias_dev = bias.to(dev)
        B.moe_set_gating(gl.ctx, 0, rule, bias_dev)
        o = gl.four_calls(x, tenant, G)
        assert o["status"] == 0
        # logits in 64 bits from the exact bf16 values
        model = mot.long()[tenant.long()]
        z = torch.einsum("th,teh->te", x.double(), wts["router_w"].double()[model]) + wts["router_bias"].double()[model]
        bt = bias.double()[model].numpy()
        s = torch.sigmoid(z).numpy() + bt
        ref_idx, ref_w = reference(z.numpy(), k, score="sigmoid", n_groups=n_groups, keep=keep, group_score="top2", renorm=True,
                                   scale=1.5, bias=bt)
        # fp32 logits: H products summed in fp32, |z| of a few units: 1e-4 is far above their error; rows without a
        # closer call anywhere among their values and group scores must agree
        size = E // n_groups
        srt = np.sort(s, 1)
        grp = np.sort(np.sort(s.reshape(T, n_groups, size), 2)[:, :, -2:].sum(2), 1)
        clear = (np.diff(srt, axis=1)[:, -3 * k:].min(1) > 1e-4) & (np.diff(grp, axis=1).min(1) > 2e-4)
        idx = o["topk_idx"].cpu().numpy()
        assert clear.sum() > T // 4
        assert np.array_equal(idx[clear], ref_idx[clear])
        np.testing.assert_allclose(o["topk_w"].cpu().numpy()[clear], ref_w[clear], rtol=1e-3)
        # the whole layer runs on it: fused call = four calls, bit for bit
        out = gl.forward(x, tenant, G)
        assert torch.equal(out, o["out"])
        assert not torch.equal(out, before)
        # every token's weights sum to the scale
        torch.testing.assert_close(o["topk_w"].sum(1).cpu(), torch.full((T,), 1.5), rtol=1e-5, atol=0)
        # and back: the layer's own rule, the same bits as before
        B.moe_set_gating(gl.ctx, 0, None)
        assert torch.equal(gl.forward(x, tenant, G), before)
    finally:
        gl.close()


@gpu
def test_every_call_that_runs_the_layer_uses_the_rule():
    """Fused dispatch, the timed, host, pipelined and paged calls and the stack: the same bits as the layer call."""
    T, k = 100, 4
    wl = W.MoEWorkload("rule", T=T, H=256, E=60, I=128, k=k, Is=128, n_tenants=3, G=3, tenant_layout="uniform")
    wts = W.make_weights(wl, seed=5)
    x, tenant, mot = W.make_tokens(wl, seed=5)
    gl = GpuLayer(wl, [wts], max_tokens=T, model_of_tenant=mot)
    try:
        rule = B.moe_gating(score="sigmoid", n_groups=4, keep_groups=2, group_score="max", renormalize=True)
        bias = (torch.randn(1, 60, generator=torch.Generator().manual_seed(1)) * 0.1).to(gl.dev)
        plain = gl.forward(x, tenant, 3)
        B.moe_set_gating(gl.ctx, 0, rule, bias)
        ref = gl.forward(x, tenant, 3)
        assert not torch.equal(ref, plain)
        B.moe_set_option(gl.ctx, B.MOE_OPT_FUSED_DISPATCH, 1)
        assert torch.equal(gl.forward(x, tenant, 3), ref)
        B.moe_set_option(gl.ctx, B.MOE_OPT_FUSED_DISPATCH, 0)
        assert torch.equal(gl.forward_host(x, tenant, 3), ref.cpu())
        xd, td, out = x.to(gl.dev), tenant.to(gl.dev), torch.zeros_like(ref)
        B.moe_layer_forward_timed(gl.ctx, 0, xd, td, T, 3, out)
        assert torch.equal(out, ref)
        xh, th, oh = x.pin_memory(), tenant.pin_memory(), torch.zeros_like(x).pin_memory()
        B.moe_layer_forward_host_wait(gl.ctx, B.moe_layer_forward_host_submit(gl.ctx, 0, xh, th, T, 3, oh))
        assert torch.equal(oh, ref.cpu())
        # the stack's one block on inputs that its norm leaves as the layer's tokens
        sx, dbg_in, dbg_out = xd.clone(), torch.empty(1, T, 256, dtype=torch.bfloat16, device=gl.dev), torch.empty(1, T, 256, dtype=torch.bfloat16, device=gl.dev)
        B.moe_stack_forward(gl.ctx, sx, td, T, 3, dbg_layer_inputs=dbg_in, dbg_layer_outputs=dbg_out)
        o = torch.zeros_like(ref)
        B.moe_layer_forward(gl.ctx, 0, dbg_in[0], td, T, 3, o)
        d = (sx.double() - (xd.double() + o.double())).abs()                   # (the stack rounds once, this sum twice)
        assert (d <= 2.0 ** -8 * (o.double().abs() + sx.double().abs()) + 1e-30).all()
        # paged residency: routes by the rule, then pages in what the rule chose
        host = [wts[n].pin_memory() for n in ("pool_gate", "pool_up", "pool_down")]
        pool = [torch.zeros_like(h, device=gl.dev) for h in host]
        B.moe_residency_enable(gl.ctx, 0, *host, *pool)
        out.zero_()
        B.moe_layer_forward_paged(gl.ctx, 0, xd, td, T, 3, out)
        assert torch.equal(out, ref)
    finally:
        gl.close()


@gpu
def test_a_layers_rule_is_its_own():
    """Two layers, a rule in the second only; a layer index or a rule that does not fit is refused and changes nothing."""
    wl = W.MoEWorkload("two", T=40, H=256, E=12, I=128, k=2, Is=128, n_tenants=2, G=3, n_layers=2)
    wts = [W.make_weights(wl, seed=6, layer=i) for i in range(2)]
    x, tenant, mot = W.make_tokens(wl, seed=6)
    gl = GpuLayer(wl, wts, max_tokens=40, model_of_tenant=mot)
    try:
        a0, a1 = gl.forward(x, tenant, 3, 0), gl.forward(x, tenant, 3, 1)
        B.moe_set_gating(gl.ctx, 1, B.moe_gating(score="sigmoid", renormalize=True))
        assert torch.equal(gl.forward(x, tenant, 3, 0), a0) and not torch.equal(gl.forward(x, tenant, 3, 1), a1)
        for layer, rule in ((2, B.moe_gating()), (-1, None), (0, B.moe_gating(n_groups=5)), (0, B.moe_gating(n_groups=12, keep_groups=1))):
            with pytest.raises(B.MoeError) as e:
                B.moe_set_gating(gl.ctx, layer, rule)
            assert e.value.status == B.MOE_ERR_SHAPE
        assert torch.equal(gl.forward(x, tenant, 3, 0), a0)
    finally:
        gl.close()


@gpu
def test_softmax_rule_without_anything_is_the_layers_own_rule():
    T = 300
    wl, wts = _layer(60, 4, 1, T)
    x, tenant, mot = W.make_tokens(wl, seed=2)
    gl = GpuLayer(wl, [wts], max_tokens=T, model_of_tenant=mot)
    try:
        a = gl.four_calls(x, tenant, 3)
        B.moe_set_gating(gl.ctx, 0, B.moe_gating(score="softmax"))
        b = gl.four_calls(x, tenant, 3)
        assert torch.equal(a["topk_idx"], b["topk_idx"])
        torch.testing.assert_close(a["topk_w"], b["topk_w"], rtol=2e-6, atol=0)
        assert torch.equal(a["shared_gate"], b["shared_gate"])
    finally:
        gl.close()


def _raw(**kw):
    """moe_gate's C arguments; pointers are never followed by a refused call."""
    a = dict(logits=64, type=0, ld=8, T=4, E=8, k=2, rule=B.moe_gating(), bias=None, tenant=None, mot=None, n_tenants=1, M=1, idx=64,
             w=64, tie=None, status=None)
    a.update(kw)
    rule = a["rule"]
    return B.load_library().moe_gate(a["logits"], a["type"], a["ld"], a["T"], a["E"], a["k"], ctypes.byref(rule) if rule else None,
                                     a["bias"], a["tenant"], a["mot"], a["n_tenants"], a["M"], a["idx"], a["w"], a["tie"], a["status"], None)


def test_refusals_need_no_gpu():
    assert _raw(logits=None) == B.MOE_ERR_NULL
    assert _raw(rule=None) == B.MOE_ERR_NULL
    assert _raw(idx=None) == B.MOE_ERR_NULL
    assert _raw(w=None) == B.MOE_ERR_NULL
    assert _raw(M=2, tenant=None) == B.MOE_ERR_NULL
    for bad in (dict(T=-1), dict(E=0, ld=0), dict(E=257, ld=257), dict(k=0), dict(k=9, E=64, ld=64), dict(k=3, E=2, ld=2), dict(ld=7), dict(M=0),
                dict(M=257, tenant=64, mot=64), dict(tenant=64, n_tenants=0), dict(logits=66), dict(idx=66), dict(w=65), dict(status=2),
                dict(bias=66), dict(type=1, logits=65)):
        assert _raw(**bad) == B.MOE_ERR_SHAPE, bad
    assert _raw(type=7) == B.MOE_ERR_UNSUPPORTED
    for rule in (B.moe_gating(n_groups=3), B.moe_gating(n_groups=0, keep_groups=0), B.moe_gating(n_groups=4, keep_groups=5),
                 B.moe_gating(n_groups=4, keep_groups=0), B.moe_gating(scale=math.inf), B.moe_gating(scale=math.nan), B.MoeGating(2, 1, 1, 0, 0, 1.0),
                 B.MoeGating(0, 1, 1, 2, 0, 1.0)):
        assert _raw(rule=rule) == B.MOE_ERR_SHAPE
    assert _raw(rule=B.moe_gating(n_groups=8, keep_groups=1), k=2) == B.MOE_ERR_SHAPE      # one expert is left for k = 2
    assert _raw(rule=B.moe_gating(n_groups=64, keep_groups=64), E=64, ld=64) == B.MOE_ERR_SHAPE
    assert _raw(T=0) == B.MOE_OK
    assert B.load_library().moe_set_gating(None, 0, None, None) == B.MOE_ERR_NULL


def test_binding_checks_tensors():
    z, idx, w = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    rule = B.moe_gating()
    with pytest.raises(ValueError, match="CUDA"):
        B.moe_gate(z, rule, idx, w)
    for bad in (dict(logits=z.double()), dict(logits=z.t()), dict(topk_idx=idx.long()), dict(topk_w=w[:3]), dict(logits=z[0]), dict(rule=None)):
        a = dict(logits=z, rule=rule, topk_idx=idx, topk_w=w)
        a.update(bad)
        with pytest.raises(ValueError):
            B.moe_gate(a["logits"], a["rule"], a["topk_idx"], a["topk_w"])
    with pytest.raises(ValueError):
        B.moe_gate(z, rule, idx, w, balance_bias=torch.zeros(1, 7))
    with pytest.raises(ValueError):
        B.moe_gate(z, rule, idx, w, tenant_id=torch.zeros(4))
    with pytest.raises(ValueError):
        B.moe_set_gating(None, 0, rule, torch.zeros(1, 8))
    with pytest.raises(KeyError):
        B.moe_gating(score="tanh")


@gpu
@pytest.mark.parametrize("T,E,n_groups,keep,k", [(90, 256, 8, 4, 8), (16384, 256, 8, 4, 8), (16384, 256, 4, 1, 5), (16384, 128, 4, 2, 3), (32768, 256, 8, 2, 8)])
def test_experts_forced_by_an_infinite_bias(T, E, n_groups, keep, k):
    """A bias of +inf (or of the largest finite value, which is below it) puts its expert in front, ties to the lower id, and its group
    among those that stay."""
    g = np.random.default_rng(T + E + n_groups)
    rows = g.standard_normal((60, E))
    size = E // n_groups
    for forced in ([3], [size + 1, E - 1], [5, 2 * size - 1, E - 2], list(range(0, E, size)), [2, 3, 4, 7, E - 3]):
        for value in (np.inf, FMAX):
            bias = g.standard_normal(E) * 0.05
            bias[forced] = value
            for score in ("softmax", "sigmoid"):
                for group_score in ("max", "top2"):
                    check_repeated(rows, T, k, bias=bias, score=score, n_groups=n_groups, keep=keep, group_score=group_score, renorm=True)
    bias = g.standard_normal(E) * 0.05
    bias[[1, size + 2]] = [FMAX, np.inf]
    check_repeated(rows, T, k, bias=bias, score="sigmoid", n_groups=n_groups, keep=keep, renorm=True)


@gpu
@pytest.mark.parametrize("T,E,groups", [(40, 256, {}), (8192, 256, {}), (8192, 128, {}), (8192, 64, {}), (16384, 256, dict(n_groups=8, keep=8))])
def test_softmax_sums_of_one_dominant_expert(T, E, groups):
    """One expert has nearly all of the weight and the others 2^-24 of it or less, not half an fp32 step beside it: added to it one after
    the other they would all be lost.  At most 13 additions lie between an exponential and the sum, each 2^-24 relative, then a quotient and
    a product: below 16 * 2^-24 with the rounding of the tail's own exponentials.  (The others are 2e-3 apart, so that nothing is near a tie.)"""
    g = np.random.default_rng(E)
    rows = -24 * math.log(2) - 2e-3 * np.stack([g.permutation(E) for _ in range(E)])
    rows[np.arange(E), np.arange(E)] = 0.0
    for tie in (False, True):
        pick = np.arange(T) % E
        idx, w, _, _ = run(rows[pick], 2, score="softmax", tie=tie, **groups)
        zr = rows.astype(np.float32).astype(float)
        p = np.exp(zr) / np.exp(zr).sum(1, keepdims=True)
        assert np.array_equal(idx[:, 0], pick)
        np.testing.assert_allclose(w[:, 0], p[pick, pick], rtol=16 * 2.0 ** -24, atol=0)


@gpu
@pytest.mark.parametrize("T", [300, 32768])
def test_softmax_scores_that_a_bias_brings_close_to_zero(T):
    """One dominant logit early in a lane, the others 2^-24 of it, and a bias that leaves a few 1e-6 between it and the next ones: what a
    sum in 32 bits may be off by must not decide."""
    g = np.random.default_rng(31)
    E, k = 256, 4
    rows = -24 * math.log(2) - 1e-3 * g.random((256, E))
    top = g.integers(0, 8, 256) * 32 + g.integers(0, 4, 256)
    rows[np.arange(256), top] = 0.0
    p = 1 / (1 + 255 * 2.0 ** -24)                  # (to 1e-8)
    bias = g.uniform(-4e-6, 4e-6, E)
    bias[np.unique(top)] = -p + g.uniform(-4e-6, 4e-6, np.unique(top).size)
    for groups in ({}, dict(n_groups=8, keep=3)):
        check_repeated(rows, T, k, bias=bias, score="softmax", renorm=True, **groups)


@gpu
def test_a_layers_bias_has_one_number_for_every_expert_of_every_model():
    """moe_set_gating takes no bias that is shorter or longer than what the kernels read, and leaves the layer as it was."""
    T, M, E = 40, 3, 12
    wl, wts = _layer(E, 4, M, T)
    x, tenant, mot = W.make_tokens(wl, seed=1)
    gl = GpuLayer(wl, [wts], max_tokens=T, model_of_tenant=mot)
    try:
        cfg, device = B.moe_get_config(gl.ctx)
        assert (cfg.n_models, cfg.n_experts, cfg.top_k, cfg.max_tokens, device) == (M, E, 4, T, torch.device(gl.dev))
        before = gl.forward(x, tenant, 3)
        rule = B.moe_gating(score="sigmoid", renormalize=True)
        for shape in ((E,), (1, E), (M, E - 1), (E, M), (M, E, 1), (M * E,), (2 * M, E), (0,)):
            with pytest.raises(ValueError, match="balance_bias"):
                B.moe_set_gating(gl.ctx, 0, rule, torch.zeros(shape, device=gl.dev))
        assert torch.equal(gl.forward(x, tenant, 3), before)
        bias = torch.full((M, E), -1.0, device=gl.dev)
        bias[:, :4] = 1.0
        B.moe_set_gating(gl.ctx, 0, rule, bias)
        assert (gl.four_calls(x, tenant, 3)["topk_idx"].sort(1)[0].cpu() == torch.arange(4)).all()
    finally:
        gl.close()


def test_a_layers_bias_is_checked_before_the_call(monkeypatch):
    class OnDevice(torch.Tensor):
        is_cuda, device = True, torch.device("cuda", 0)

    class Library:
        def __init__(self, M, E, index=0):
            self.M, self.E, self.index, self.set = M, E, index, 0

        def moe_get_config(self, ctx, cfg, device):
            cfg._obj.n_models, cfg._obj.n_experts, device._obj.value = self.M, self.E, self.index
            return B.MOE_OK

        def moe_set_gating(self, ctx, layer, rule, bias):
            self.set += 1
            return B.MOE_OK
    rule = B.moe_gating()
    for M, E, index, shape, good in ((4, 8, 0, (4, 8), True), (1, 8, 0, (8,), True), (1, 8, 0, (1, 8), True), (4, 8, 0, (8,), False), (4, 8, 0, (1, 8), False),
                                     (4, 8, 0, (8, 4), False), (4, 8, 0, (4, 9), False), (4, 8, 0, (4, 7), False), (4, 8, 0, (32,), False), (4, 8, 1, (4, 8), False)):
        lib = Library(M, E, index)
        monkeypatch.setattr(B, "load_library", lambda lib=lib: lib)
        bias = torch.zeros(shape).as_subclass(OnDevice)
        if good:
            B.moe_set_gating(1, 0, rule, bias)
        else:
            with pytest.raises(ValueError, match="balance_bias"):
                B.moe_set_gating(1, 0, rule, bias)
        assert lib.set == good


def test_the_configuration_of_no_context():
    assert B.load_library().moe_get_config(None, ctypes.byref(B.MoeConfig()), None) == B.MOE_ERR_NULL


def flagged_rows(g, E):
    """Rows of every degree of closeness: random ones, neighbours from 1e-3 down to one fp32 step apart (of the logits, and of the scores
    where the bias is flat), exact ties, masked rows."""
    near = []
    for step in 2.0 ** -np.arange(8, 25, dtype=float):
        z = g.standard_normal((12, E))
        z[:, 1::2] = z[:, ::2][:, :z[:, 1::2].shape[1]] + step * g.integers(-3, 4, z[:, 1::2].shape)
        near.append(g.permuted(z, axis=1))
    odd = g.standard_normal((6, E))
    odd[0] = -np.inf
    odd[1, 1:] = -np.inf
    odd[2] = 0.0
    odd[3] -= 200
    odd[4, ::2] = -FMAX
    odd[5] = g.integers(-2, 3, E)
    return np.concatenate([g.standard_normal((60, E)), *near, odd])


@gpu
@pytest.mark.parametrize("T,E,k,groups", [(16384, 60, 4, {}), (16384, 64, 8, dict(n_groups=2, keep=1)), (16384, 128, 8, dict(n_groups=4, keep=2)), (16384, 128, 7, {}),
                                          (32768, 256, 8, dict(n_groups=8, keep=4)), (32768, 256, 8, {}), (32768, 200, 1, {}), (32768, 8, 8, {})])
def test_the_tie_flag_does_not_depend_on_the_batch(T, E, k, groups):
    """A row has the same flag in a short batch and in a long one, whichever kernel looks at it; so have its experts."""
    g = np.random.default_rng(E + k)
    rows = flagged_rows(g, E)
    pick = g.integers(0, len(rows), T)
    pick[:len(rows)] = np.arange(len(rows))
    # (a bias that undoes the scores in part, so that sums of the two come close to each other and to zero)
    s = 1 / (1 + np.exp(-rows[70]))
    odd = g.standard_normal(E) * 0.05
    odd[[1, E // 2, 2, 3]] = np.inf, np.inf, -np.inf, np.nan
    seen = set()
    for score in ("softmax", "sigmoid"):
        for bias in (None, np.zeros(E), g.standard_normal(E) * 0.05, odd, -s if score == "sigmoid" else -np.exp(rows[70]) / np.exp(rows[70]).sum()):
            for group_score in ("max", "top2") if groups else ("max",):
                for dtype in (torch.float32, torch.bfloat16):
                    kw = dict(bias=None if bias is None else bias.reshape(1, -1), dtype=dtype, tie=True, score=score, group_score=group_score, renorm=True, **groups)
                    idx, _, flag, _ = run(rows, k, **kw)
                    long_idx, _, long_flag, _ = run(rows[pick], k, **kw)
                    assert np.array_equal(long_idx, idx[pick])
                    bad = np.nonzero(long_flag != flag[pick])[0]
                    assert bad.size == 0, f"{bad.size} tokens, rows {sorted(set(pick[bad]))[:8]}: flag {long_flag[bad[0]]}, alone {flag[pick[bad[0]]]}, {kw}"
                    seen |= set(flag.tolist())
    assert seen == {0, 1}
