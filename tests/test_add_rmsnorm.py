"""moe_add_rmsnorm against the formula in 64 bits.

Tolerances, from the roundings: h is one rounding to bf16 of an fp32 sum of two bf16 numbers (exact unless their exponents are
more than 16 apart, where the fp32 rounding adds 2^-24).  y in fp32: a sum of squares whose partial sums are at most 64 deep
(32 in a lane, 5 + 16 across lanes and warps) -- relative 64 * 2^-24, halved by the root --, a root, a quotient and two
products: below 40 * 2^-24.  out adds half a bf16 step (2^-8 relative), q half an e4m3 step (2^-4 relative, 2^-10 below
2^-6) of y / s, and s itself is y's error plus one rounding.
"""
import numpy as np
import pytest
import torch

from paper_2604_26881_b200 import binding as B
from paper_2604_26881_b200 import workloads as W
from harness import GpuLayer

gpu = pytest.mark.gpu
Y_REL = 40 * 2.0 ** -24
BF16_HALF, E4M3_HALF, E4M3_SMALL = 2.0 ** -8, 2.0 ** -4, 2.0 ** -10


def reference(x, r, w, eps):
    h = x.double()
    if r is not None:
        h = (x.float() + r.float()).to(torch.bfloat16).double()
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * w.double()
    return h, y


def strided(T, H, pad, dtype, fill, shift=0):
    """A [T, H] view with rows H + pad apart, `shift` elements into its storage; the whole storage is returned too."""
    store = torch.full((T * (H + pad) + shift + 16,), fill, device="cuda:0", dtype=torch.float32).to(dtype)
    return store[shift:shift + T * (H + pad)].view(T, H + pad)[:, :H], store


def check(T, H, *, residual=True, residual_out=True, out=True, q=None, pads=(0, 0, 0, 0, 0), shift=0, eps=1e-6, seed=0, x_values=None, r_values=None):
    g = torch.Generator().manual_seed(seed + 7 * T + H)
    x0 = (torch.randn(T, H, generator=g) * 0.5).to(torch.bfloat16) if x_values is None else x_values
    r0 = (torch.randn(T, H, generator=g) * 2).to(torch.bfloat16) if r_values is None else r_values
    w0 = (1 + 0.2 * torch.randn(H, generator=g)).to(torch.bfloat16)
    x, _ = strided(T, H, pads[0], torch.bfloat16, 3.0, shift)
    x.copy_(x0)
    r = None
    if residual:
        r, _ = strided(T, H, pads[1], torch.bfloat16, 3.0, shift)
        r.copy_(r0)
    ro, ro_s = strided(T, H, pads[2], torch.bfloat16, 7.0, shift) if residual_out else (None, None)
    o, o_s = strided(T, H, pads[3], torch.bfloat16, 7.0, shift) if out else (None, None)
    qt = qs = q_s = None
    groups = 0
    if q:
        qt, q_s = strided(T, H, pads[4], torch.float8_e4m3fn, 7.0, shift)
        groups = 1 if q == "row" else -(-H // 128)
        qs = torch.full((T * groups + 8,), -5.0, device="cuda:0")
    B.moe_add_rmsnorm(x, w0.cuda(), eps, residual=r, residual_out=ro, out=o, out_q=qt, q_scale=qs[:T * groups].view(T, groups) if q else None)
    torch.cuda.synchronize()
    h, y = reference(x0, r0 if residual else None, w0, eps)
    if residual_out:
        assert torch.equal(ro.cpu().double().nan_to_num(nan=12345.0), h.nan_to_num(nan=12345.0))
    for view, store in ((ro, ro_s), (o, o_s), (qt, q_s)):
        if view is not None:                     # everything outside the rows is as it was
            keep = torch.ones(store.numel(), dtype=torch.bool)
            idx = (torch.arange(T)[:, None] * view.stride(0) + torch.arange(H) + shift).flatten()
            keep[idx] = False
            assert (store.cpu().float()[keep] == 7.0).all(), "written outside the rows"
    if out:
        got = o.cpu().double()
        assert torch.equal(got.isnan(), y.isnan())
        ok = ~y.isnan()
        assert ((got - y).abs()[ok] <= (BF16_HALF + 2 * Y_REL) * y.abs()[ok] + 1e-40).all()
    if q:
        assert (qs[T * groups:] == -5.0).all()
        s = qs[:T * groups].view(T, groups).cpu().double()
        size = H if q == "row" else 128
        ref_s = torch.stack([y[:, i:i + size].abs().amax(1) / 448 for i in range(0, H, size)], 1)
        assert torch.equal(s.isnan(), ref_s.isnan())
        fine = ~ref_s.isnan()
        assert ((s - ref_s).abs()[fine] <= 2 * Y_REL * ref_s[fine] + 2e-45).all()
        full = s.repeat_interleave(size, 1)[:, :H]
        val = qt.cpu().double()
        live = (full > 1e-30) & ~full.isnan()
        assert (val[full == 0] == 0).all()
        assert val[full.isnan()].isnan().all()
        lim = E4M3_HALF * (y / full).abs() * (1 + 1e-5) + E4M3_SMALL
        assert ((val - y / full).abs()[live] <= lim[live]).all()
        assert (val.abs()[~val.isnan()] <= 448).all()
    return o, qt, qs


@gpu
@pytest.mark.parametrize("H", [1, 2, 7, 8, 9, 127, 128, 129, 255, 256, 257, 511, 1000, 1408, 1411, 2048, 4096, 5632, 8192, 8200, 16384])
@pytest.mark.parametrize("q", [None, "row", "group"])
def test_every_width(H, q):
    check(5, H, q=q)


@gpu
@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 33, 1126])
def test_numbers_of_tokens(T):
    for H in (64, 512, 768, 2048):
        check(T, H, q="row", seed=1)
        check(T, H, q="group", seed=2, residual=False)


@gpu
def test_no_tokens():
    e = torch.empty(0, 256, dtype=torch.bfloat16, device="cuda:0")
    B.moe_add_rmsnorm(e, torch.ones(256, dtype=torch.bfloat16, device="cuda:0"), 1e-6, residual=e, out=e)


@gpu
@pytest.mark.parametrize("pads,shift", [((8, 0, 16, 8, 8), 0), ((1, 2, 3, 4, 5), 0), ((0, 0, 0, 0, 0), 1), ((5, 0, 0, 0, 0), 8), ((0, 0, 0, 0, 3), 0), ((7, 7, 7, 7, 7), 3)])
def test_strides_and_alignment(pads, shift):
    for H in (200, 1411, 2048):
        for q in (None, "row", "group"):
            check(6, H, q=q, pads=pads, shift=shift)


@gpu
def test_rows_beyond_32_bit_offsets():
    """Rows 2^25 elements apart: the last ones lie beyond 2^31 elements."""
    T, H, ld = 70, 520, 1 << 25
    g = torch.Generator().manual_seed(4)
    far = lambda dtype: torch.empty(T * ld, dtype=dtype, device="cuda:0").as_strided((T, H), (ld, 1))
    x0, r0, w0 = torch.randn(T, H, generator=g).to(torch.bfloat16), torch.randn(T, H, generator=g).to(torch.bfloat16), torch.ones(H, dtype=torch.bfloat16)
    near = dict(out=torch.empty(T, H, dtype=torch.bfloat16, device="cuda:0"), out_q=torch.empty(T, H, dtype=torch.float8_e4m3fn, device="cuda:0"),
                q_scale=torch.empty(T, 1, device="cuda:0"), residual_out=torch.empty(T, H, dtype=torch.bfloat16, device="cuda:0"))
    B.moe_add_rmsnorm(x0.cuda(), w0.cuda(), 1e-6, residual=r0.cuda(), **near)
    x, o, q = far(torch.bfloat16), far(torch.bfloat16), far(torch.float8_e4m3fn)
    x.copy_(x0)
    s = torch.empty(T, 1, device="cuda:0")
    B.moe_add_rmsnorm(x, w0.cuda(), 1e-6, residual=r0.cuda(), residual_out=x, out=o, out_q=q, q_scale=s)
    torch.cuda.synchronize()
    assert torch.equal(x, near["residual_out"]) and torch.equal(o, near["out"]) and torch.equal(s, near["q_scale"])
    assert torch.equal(q.contiguous().view(torch.uint8), near["out_q"].view(torch.uint8))


@gpu
def test_each_output_alone_and_without_a_residual():
    for residual in (False, True):
        check(9, 520, residual=residual, residual_out=True, out=False)
        check(9, 520, residual=residual, residual_out=False, out=True)
        check(9, 520, residual=residual, residual_out=False, out=False, q="row")
        check(9, 520, residual=residual, residual_out=False, out=False, q="group")


@gpu
def test_zeros_huge_tiny_and_non_finite_rows():
    T, H = 10, 300
    g = torch.Generator().manual_seed(0)
    x = torch.randn(T, H, generator=g).to(torch.bfloat16)
    x[0] = 0
    x[1, 128:256] = 0                        # one group of zeros
    x[2] = x[2] * 1e15
    x[3] = x[3] * 1e-18                      # mean of squares far below eps
    x[4, 7] = float("inf")
    x[5, 290] = float("nan")
    x[6, 3] = -float("inf")
    x[7] = 0
    x[7, 299] = 1
    x[8, :] = torch.finfo(torch.bfloat16).tiny
    for q in ("row", "group"):
        check(T, H, residual=False, q=q, x_values=x)
        check(T, H, residual=True, q=q, x_values=x, r_values=torch.zeros(T, H, dtype=torch.bfloat16))
    check(T, H, residual=False, q="row", x_values=x[[1, 2, 7]].repeat(4, 1)[:T], eps=0.0)


@gpu
def test_in_place():
    T, H = 77, 2048
    g = torch.Generator().manual_seed(0)
    x = torch.randn(T, H, generator=g).to(torch.bfloat16).cuda()
    r = torch.randn(T, H, generator=g).to(torch.bfloat16).cuda()
    w = torch.rand(H, generator=g).to(torch.bfloat16).cuda()
    ro, o = torch.empty_like(x), torch.empty_like(x)
    B.moe_add_rmsnorm(x, w, 1e-5, residual=r, residual_out=ro, out=o)
    x2, r2 = x.clone(), r.clone()
    B.moe_add_rmsnorm(x2, w, 1e-5, residual=r2, residual_out=r2, out=x2)
    torch.cuda.synchronize()
    assert torch.equal(r2, ro) and torch.equal(x2, o)


@gpu
def test_the_stack_block_from_its_parts():
    """One block of moe_stack_forward = norm, layer, residual add: the norm's output feeds moe_layer_forward, and the next
    norm adds its output to the residual stream.  The stack adds its residual before the rounding of the layer's output,
    so the two streams differ by that one rounding: half a bf16 step of the layer's output and of the sum."""
    wl = W.MoEWorkload("blk", T=90, H=256, E=8, I=128, k=2, Is=128, n_tenants=2, G=2)
    wts = [W.make_weights(wl, seed=3, layer=i) for i in range(1)]
    x, tenant, _ = W.make_tokens(wl, seed=3)
    gl = GpuLayer(wl, wts, max_tokens=90)
    try:
        dev = gl.dev
        xd, td = x.to(dev), tenant.to(dev)
        w = wts[0]["rms_w"].to(dev)
        xn, o, h, nxt = (torch.empty_like(xd) for _ in range(4))
        B.moe_add_rmsnorm(xd, w, wl.rms_eps, out=xn)
        B.moe_layer_forward(gl.ctx, 0, xn, td, 90, 2, o)
        B.moe_add_rmsnorm(o, w, wl.rms_eps, residual=xd, residual_out=h, out=nxt)
        stack_x, dbg_in = xd.clone(), torch.empty(1, 90, 256, dtype=torch.bfloat16, device=dev)
        B.moe_stack_forward(gl.ctx, stack_x, td, 90, 2, dbg_layer_inputs=dbg_in)
        torch.cuda.synchronize()
        d = (dbg_in[0].double() - xn.double()).abs()
        assert (d <= 2 * BF16_HALF * xn.double().abs() + 1e-30).all()          # the two norms: one bf16 rounding apart
        same = (dbg_in[0] == xn).all(1)                                        # tokens whose normed input is the same
        assert same.sum() > 45
        lim = BF16_HALF * (o.double().abs() + 2 * h.double().abs()) + 1e-6
        assert ((stack_x.double() - h.double()).abs() <= lim)[same].all()
    finally:
        gl.close()


@gpu
def test_graph_and_stream():
    T, H = 64, 1408
    x = torch.randn(T, H, device="cuda:0").to(torch.bfloat16)
    w = torch.ones(H, device="cuda:0", dtype=torch.bfloat16)
    a, b, c = (torch.empty_like(x) for _ in range(3))
    B.moe_add_rmsnorm(x, w, 1e-6, out=a)
    torch.cuda.synchronize()
    B.moe_add_rmsnorm(x, w, 1e-6, out=b, stream=torch.cuda.Stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.moe_add_rmsnorm(x, w, 1e-6, out=c)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c)


def _raw(**kw):
    a = dict(x=64, ldx=16, r=None, ldr=0, w=64, eps=1e-6, T=4, H=16, ro=None, ldro=0, o=64, ldo=16, q=None, ldq=0, qs=None, group=0)
    a.update(kw)
    return B.load_library().moe_add_rmsnorm(*a.values(), None)


def test_refusals_need_no_gpu():
    for bad in (dict(x=None), dict(w=None), dict(o=None), dict(q=64, ldq=16)):
        assert _raw(**bad) == B.MOE_ERR_NULL, bad
    for bad in (dict(T=-1), dict(H=0), dict(ldx=15), dict(ldo=15), dict(r=64, ldr=15), dict(ro=64, ldro=15), dict(q=64, ldq=15, qs=64), dict(eps=-1.0),
                dict(eps=float("nan")), dict(q=64, ldq=16, qs=64, group=64), dict(x=65), dict(o=65), dict(q=64, ldq=16, qs=66), dict(w=63)):
        assert _raw(**bad) == B.MOE_ERR_SHAPE, bad
    for bad in (dict(ldo=24), dict(x=128, r=64, ldr=24), dict(o=None, ro=64, ldro=24), dict(x=128, ro=64, ldro=16), dict(q=64, ldq=16, qs=64)):      # overlapping
        assert _raw(**bad) == B.MOE_ERR_SHAPE, bad
    assert _raw(H=16385, ldx=16385, ldo=16385) == B.MOE_ERR_UNSUPPORTED
    assert _raw(T=0) == B.MOE_OK


def test_binding_checks_tensors():
    x, w = torch.zeros(4, 16, dtype=torch.bfloat16), torch.ones(16, dtype=torch.bfloat16)
    f8 = torch.zeros(4, 16).to(torch.float8_e4m3fn)
    with pytest.raises(ValueError, match="CUDA"):
        B.moe_add_rmsnorm(x, w, 1e-6, out=x.clone())
    for kw in (dict(out=x.float()), dict(out=x[:3]), dict(residual=x[:, :8]), dict(out=x, out_q=f8), dict(out_q=f8, q_scale=torch.zeros(4, 2)),
               dict(out_q=x, q_scale=torch.zeros(4, 1)), dict(out=x.t().contiguous().t())):
        with pytest.raises(ValueError):
            B.moe_add_rmsnorm(x, w, 1e-6, **kw)
    with pytest.raises(ValueError):
        B.moe_add_rmsnorm(x, w.float(), 1e-6, out=x)


@gpu
@pytest.mark.parametrize("q", ["row", "group"])
def test_quotients_are_rounded_once_to_8_bits(q):
    """out_q = e4m3(y / s) of the fp32 y and s, bit for bit.  With h = +-1 and eps = 0 the mean is 1 and y = +-weight, both exact,
    so y / s is an fp32 quotient of known numbers; some of them are in the middle of two 8-bit floats, or an fp32 step beside it."""
    g = torch.Generator().manual_seed(0)
    H, size = 16384, 16384 if q == "row" else 128
    for _ in range(8 if q == "row" else 3):
        w = (torch.randn(H, generator=g) * 2).to(torch.bfloat16)
        x = torch.where(torch.rand(2, H, generator=g) < 0.5, -1.0, 1.0).to(torch.bfloat16)
        y = (x.float() * w.float()).view(2, H // size, size)
        s = y.abs().amax(2) / 448
        want = (y / s[:, :, None]).view(2, H).to(torch.float8_e4m3fn)
        out_q, scale = torch.empty(2, H, dtype=torch.float8_e4m3fn, device="cuda:0"), torch.empty(2, H // size, device="cuda:0")
        B.moe_add_rmsnorm(x.cuda(), w.cuda(), 0.0, out_q=out_q, q_scale=scale)
        torch.cuda.synchronize()
        assert torch.equal(scale.cpu(), s)
        bad = out_q.cpu().view(torch.uint8) != want.view(torch.uint8)
        assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} differ"


@gpu
@pytest.mark.parametrize("H", [5, 300, 512, 768, 1411, 2048, 8192])
def test_finite_rows_whose_squares_leave_the_range_of_32_bits(H):
    """The formula holds for every finite row: squares beyond the largest fp32 number, squares that vanish and no eps beside them, and
    an eps of either kind.  Ordinary rows between them keep their results."""
    g = torch.Generator().manual_seed(H)
    sizes = torch.tensor([1e18, 1.0, 3e19, 1e25, 1e-30, 1e30, 1e37, 1e-12, 1e-18, 1e-23, 2.0 ** -110, 2.0 ** -120, 1.0, 1e20])
    x = (torch.rand(len(sizes), H, generator=g) + 0.5) * torch.where(torch.rand(len(sizes), H, generator=g) < 0.5, -1, 1)
    x = (x * sizes[:, None]).to(torch.bfloat16)
    x[13, 1:] = 1.0                                     # one element alone is beyond the range
    tiny = x.clone()
    tiny[[0, 3]] = (2.0 ** -133 * torch.randint(1, 100, (2, H), generator=g)).to(torch.bfloat16)           # (numbers below the normal ones)
    far = torch.where(torch.rand(len(sizes), H, generator=g) < 0.5, -1, 1) * torch.finfo(torch.bfloat16).max
    for q in (None, "row", "group"):
        for eps in (0.0, 2.0 ** -20, 2.0 ** -110, 2.0 ** -126, 2.0 ** 126):
            check(len(sizes), H, residual=False, q=q, x_values=x, eps=eps)
            check(len(sizes), H, residual=True, q=q, x_values=tiny, r_values=torch.zeros_like(x), eps=eps)
            check(len(sizes), H, residual=False, q=q, x_values=far.to(torch.bfloat16), eps=eps)


@gpu
@pytest.mark.parametrize("H", [5, 200, 768, 2048, 5632])
@pytest.mark.parametrize("q", [False, True])
def test_rows_out_of_range_in_place(H, q):
    """Rows whose squares leave the range beside ordinary ones, with every output in the place of an input that may be there: the bits
    of a call whose outputs are elsewhere, in a batch that blocks go over several times."""
    g = torch.Generator().manual_seed(H)
    T = 3000
    size = torch.tensor([1.0, 1e20, 1e-3, 3e37, 1.0, 1e-30])[torch.randint(0, 6, (T,), generator=g)]
    x = (torch.randn(T, H, generator=g) * size[:, None]).to(torch.bfloat16).cuda()
    r = (torch.randn(T, H, generator=g) * size[:, None]).to(torch.bfloat16).cuda()
    w = (1 + 0.2 * torch.randn(H, generator=g)).to(torch.bfloat16).cuda()
    for residual in (False, True):
        for eps in (1e-6, 0.0):
            def call(x, r, ro, o):
                oq, s = (torch.zeros(T, H, dtype=torch.float8_e4m3fn, device="cuda:0"), torch.zeros(T, 1, device="cuda:0")) if q else (None, None)
                B.moe_add_rmsnorm(x, w, eps, residual=r, residual_out=ro, out=o, out_q=oq, q_scale=s)
                torch.cuda.synchronize()
                return (oq.view(torch.uint8), s) if q else ()
            ro, o = torch.empty_like(x), torch.empty_like(x)
            want = call(x, r if residual else None, ro, o)
            assert bool(o[size.cuda() > 1e19].isfinite().all()) and bool((o[size.cuda() > 1e19].abs().amax(1) > 0.1).all())
            for place in ("out", "residual", "both", "x"):
                x2, r2 = x.clone(), r.clone() if residual else None
                o2 = x2 if place in ("out", "both") else torch.empty_like(x)
                ro2 = {"out": None, "residual": r2, "both": r2, "x": x2}[place]
                got = call(x2, r2, ro2, o2)
                assert torch.equal(o2.view(torch.int16), o.view(torch.int16)), place
                if ro2 is not None:
                    assert torch.equal(ro2, ro), place
                assert all(torch.equal(a, b) for a, b in zip(got, want)), place
