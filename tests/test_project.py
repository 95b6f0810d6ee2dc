"""moe_project (shared projection with the tenants' low-rank adapters) against the formula in 64 bits.

Tolerances.  A sum over K on the tensor cores is rounded or cut at most once per 16 products and once per part of K that is
added up: (K/16 + 16) * 2^-23 of the sum of the terms' absolute values.  An adapter's inner product u carries that error, the
factor's rounding, and at most 2^-16 relative where it is held as bf16 numbers (2^-24 for an fp32 output); the outer product adds (rank + 4)
fp32 roundings.  The last addition and base: 3 * 2^-24 of the absolute values.  A bf16 output adds half a bf16 step (2^-8).
All of it is propagated through the absolute values of the very inputs.
"""
import numpy as np
import pytest
import torch

from paper_2604_26881_b200 import binding as B

gpu = pytest.mark.gpu
DEV = "cuda:0"


def reference(x, w, base, a, b, scale, adapter, exact_u=False):
    """(y, error bound) in 64 bits; adapter [T] holds each token's adapter or -1.  exact_u: of an fp32 output."""
    x = x.double()
    K = x.shape[1]
    T, N = x.shape[0], (w if w is not None else base if base is not None else b[0]).shape[0 if w is not None else 1 if base is not None else 0]
    e_sum = (K / 16 + 16) * 2.0 ** -23
    y = torch.zeros(T, N, dtype=torch.float64)
    mag = torch.zeros(T, N, dtype=torch.float64)
    err = torch.zeros(T, N, dtype=torch.float64)
    if w is not None:
        y += x @ w.double().t()
        m = x.abs() @ w.double().abs().t()
        mag += m
        err += e_sum * m
    if a is not None:
        for i in sorted(set(adapter.tolist()) - {-1}):
            t = adapter == i
            s = 1.0 if scale is None else float(scale[i].double())
            ai, bi = a[i].double(), b[i].double()
            u, um = s * (x[t] @ ai.t()), abs(s) * (x[t].abs() @ ai.abs().t())
            u_err = e_sum * um + (2.0 ** -22 + (2.0 ** -24 if exact_u else 2.0 ** -16)) * u.abs()
            y[t] += u @ bi.t()
            m = (u.abs() + u_err) @ bi.abs().t()
            mag[t] += m
            err[t] += u_err @ bi.abs().t() + (ai.shape[0] + 4 + ai.shape[0] / 8) * 2.0 ** -23 * m
    if base is not None:
        y += base.double()
        mag += base.double().abs()
    return y, err + 3 * 2.0 ** -23 * mag


def view(t, pad, fill=3.0):
    """t on the device as the first columns of a wider matrix."""
    if t is None:
        return None
    s = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=DEV)
    s[:, :t.shape[1]] = t.to(DEV)
    return s[:, :t.shape[1]]


def inputs(T, K, N, rank, n, seed, weight=True, base=False, out=torch.bfloat16, scale=True):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std).to(torch.bfloat16)
    return dict(x=rnd(T, K), w=rnd(N, K, std=0.05) if weight else None, base=torch.randn(T, N, generator=g).to(out) if base else None,
                a=rnd(n, rank, K, std=0.05) if n else None, b=rnd(n, N, rank, std=0.05) if n else None,
                scale=(torch.rand(n, generator=g) + 0.5) if n and scale else None)


def tenants(T, n_tenants, layout, seed):
    g = np.random.default_rng(seed)
    if layout == "uniform":
        t = g.integers(0, n_tenants, T)
    elif layout == "contiguous":
        t = np.arange(T) * n_tenants // max(T, 1)
    else:
        t = np.sort(g.integers(0, n_tenants, T) ** 2 // n_tenants)
    return torch.from_numpy(t.astype(np.int32))


def check(T, K, N, rank=16, n=4, n_tenants=None, layout="uniform", out=torch.float32, pads=(0, 0, 0, 0), table="some", seed=0, mutate=None, **kw):
    d = inputs(T, K, N, rank, n, seed + T + K + N, out=out, **kw)
    if mutate:
        mutate(d)
    n_tenants = n_tenants or max(n, 1)
    tenant = tenants(T, n_tenants, layout, seed)
    mot = None
    adapter = tenant.long()
    if n and table:
        mot = torch.tensor([(u * 7 + 1) % (n + 1) - 1 for u in range(n_tenants)], dtype=torch.int32)       # -1 now and then
        adapter = mot.long()[adapter]
    elif n:
        adapter = torch.where(adapter < n, adapter, torch.full_like(adapter, -1))
    y, err = reference(d["x"], d["w"], d["base"], d["a"], d["b"], d["scale"], adapter, out == torch.float32)
    store = torch.full((T + 2, N + pads[3] + 3), 7.0, dtype=out, device=DEV)
    o = store[1:T + 1, :N]
    dev = lambda t: None if t is None else t.to(DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.moe_project(view(d["x"], pads[0], float("nan")), view(d["w"], pads[1], float("nan")), o, base=view(d["base"], pads[2]), a=dev(d["a"]), b=dev(d["b"]),
                  scale=dev(d["scale"]), tenant_id=dev(tenant) if n else None, adapter_of_tenant=dev(mot), status_out=status,
                  **({"n_tenants": n_tenants} if n and mot is None else {}))
    torch.cuda.synchronize()
    assert int(status) == 0
    keep = torch.ones_like(store, dtype=torch.bool)
    keep[1:T + 1, :N] = False
    assert (store[keep] == 7.0).all(), "written outside the output"
    got = o.double().cpu()
    assert torch.equal(got.isnan(), y.isnan()), "NaN where none belongs, or missing"
    ok = y.isfinite() & err.isfinite()
    lim = err + (2.0 ** -8 * (y.abs() + err) if out == torch.bfloat16 else 0) + 1e-30
    bad = ((got - y).abs() > lim) & ok
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, worst {((got - y).abs() / lim)[ok].max():.2f} of the bound at {bad.nonzero()[0].tolist()}"
    return o


@gpu
@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 64, 65, 127, 128, 129, 255, 256, 257, 300, 513])
@pytest.mark.parametrize("K,N", [(64, 128), (200, 129), (1024, 260)])
def test_numbers_of_tokens(T, K, N):
    check(T, K, N, out=torch.float32)
    check(T, K, N, out=torch.bfloat16, base=True)


@gpu
@pytest.mark.parametrize("K,N", [(8, 1), (8, 300), (16, 127), (72, 64), (120, 255), (136, 256), (2048, 7), (2048, 1411), (5632, 130), (1408, 2048)])
def test_shapes(K, N):
    for T in (5, 140, 600):
        check(T, K, N, rank=8)


@gpu
@pytest.mark.parametrize("rank", [8, 16, 24, 40, 64, 72, 104, 128])
@pytest.mark.parametrize("n,layout", [(1, "uniform"), (3, "contiguous"), (40, "uniform"), (200, "uniform"), (17, "ragged")])
def test_ranks_and_adapters(rank, n, layout):
    for T in (1, 33, 130, 700):
        check(T, 192, 200, rank=rank, n=n, layout=layout)
        check(T, 320, 130, rank=rank, n=n, layout=layout, weight=False, base=True, table=None, n_tenants=n + 2)


@gpu
def test_parts_can_be_left_out():
    for T in (3, 200, 1000):
        check(T, 256, 256, n=0)
        check(T, 256, 256, n=0, base=True, out=torch.bfloat16)
        check(T, 256, 256, weight=False)
        check(T, 256, 256, weight=False, scale=False, out=torch.bfloat16)
        check(T, 256, 256, weight=False, n=0, base=True)
        check(T, 256, 300, scale=False)


@gpu
@pytest.mark.parametrize("pads", [(8, 0, 0, 0), (0, 16, 3, 1), (40, 8, 1, 5), (8, 8, 8, 8)])
def test_strides(pads):
    for T in (17, 150, 520):
        for out in (torch.float32, torch.bfloat16):
            check(T, 136, 261, pads=pads, base=True, out=out)


@gpu
def test_long_batches_and_long_sums():
    check(4096, 512, 512, rank=16, n=16, layout="ragged", out=torch.bfloat16)
    check(2048, 2048, 1411, rank=64, n=13, layout="ragged", out=torch.float32)
    check(1126, 5632, 2048, rank=16, n=4, layout="contiguous", out=torch.bfloat16)
    check(3000, 256, 640, rank=32, n=200, layout="uniform", out=torch.float32)


@gpu
@pytest.mark.parametrize("rank", [16, 40, 64, 72, 128])
def test_rings_that_wrap_many_times(rank):
    """Long sums over K in one CTA, at every ring depth that the rank leaves room for, with several chunks of adapters."""
    for T, n in ((140, 16), (128, 40), (257, 3), (640, 16)):
        check(T, 5632, 200, rank=rank, n=n, layout="ragged")
        check(T, 2048, 130, rank=rank, n=n, layout="uniform", weight=False, base=True)


@gpu
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [2, 20, 130, 300, 900])
def test_what_the_workspace_held_does_not_matter(T, out):
    """Tokens without an adapter leave their rows of the workspace as they were: NaN there reaches nobody."""
    K, N, rank, n = 512, 300, 24, 5
    d = inputs(T, K, N, rank, n, 8, base=True, out=out)
    g = {k: v.to(DEV) for k, v in d.items()}
    tenant = tenants(T, n + 3, "uniform", 2).to(DEV)                # (three tenants have no adapter)
    results = []
    for weight in (g["w"], None):
        for fill in (0, 255):
            ws = torch.full((max(256, B.moe_project_workspace(T, K, N, rank, n)),), fill, dtype=torch.uint8, device=DEV)
            o = torch.empty(T, N, dtype=out, device=DEV)
            B.moe_project(g["x"], weight, o, base=g["base"], a=g["a"], b=g["b"], scale=g["scale"], tenant_id=tenant, n_tenants=n + 3, workspace=ws)
            results.append(o)
    torch.cuda.synchronize()
    assert torch.equal(results[0], results[1]) and torch.equal(results[2], results[3])
    assert all(bool(o.isfinite().all()) for o in results)


@gpu
@pytest.mark.parametrize("T,what", [(100, "x"), (100, "w"), (100, "out"), (600, "x"), (600, "w"), (600, "out")])
def test_rows_beyond_32_bit_offsets(T, what):
    """Rows so far apart that the last ones lie beyond 2^31 elements, of each matrix in turn, in either shape."""
    K, N, rank, n = 128, 260, 16, 4
    d = inputs(T, K, N, rank, n, 3, base=True)
    g = {k: v.to(DEV) for k, v in d.items()}
    tenant = tenants(T, n, "uniform", 1).to(DEV)
    kw = dict(a=g["a"], b=g["b"], scale=g["scale"], tenant_id=tenant)
    near = torch.empty(T, N, dtype=torch.bfloat16, device=DEV)
    B.moe_project(g["x"], g["w"], near, base=g["base"], **kw)

    def far(t):
        ld = -(-(1 << 32) // t.shape[0] // 8) * 8
        v = torch.empty(t.shape[0] * ld + 1024, dtype=t.dtype, device=DEV).as_strided(t.shape, (ld, 1))
        v.copy_(t)
        return v
    x, w, out, base = g["x"], g["w"], torch.empty_like(near), g["base"]
    if what == "x":
        x = far(x)
    elif what == "w":
        w = far(w)
    else:
        out = base = far(base)                                       # (in place)
    B.moe_project(x, w, out, base=base, **kw)
    torch.cuda.synchronize()
    assert torch.equal(out, near)


@gpu
@pytest.mark.parametrize("T", [3, 40, 600])
def test_adapters_beyond_32_bit_offsets(T):
    """a and b of more than 2^31 elements: the last adapters give what they give alone."""
    K, N, rank, n = 4096, 4096, 128, 4100
    g = torch.Generator(device=DEV).manual_seed(2)
    rnd = lambda *s: (torch.randn(*s, generator=g, device=DEV) * 0.05).to(torch.bfloat16)
    x, a2, b2 = rnd(T, K), rnd(2, rank, K), rnd(2, N, rank)
    a, b = torch.empty(n, rank, K, dtype=torch.bfloat16, device=DEV), torch.empty(n, N, rank, dtype=torch.bfloat16, device=DEV)
    a[n - 2:], b[n - 2:] = a2, b2
    pick = torch.arange(T, dtype=torch.int32, device=DEV) % 2
    one, two = (torch.empty(T, N, device=DEV) for _ in range(2))
    B.moe_project(x, None, one, a=a2, b=b2, tenant_id=pick)
    B.moe_project(x, None, two, a=a, b=b, tenant_id=pick + (n - 2))
    torch.cuda.synchronize()
    y, err = reference(x.cpu(), None, None, a2.cpu(), b2.cpu(), None, pick.cpu().long())
    for o in (one, two):                                             # (of other numbers of adapters: other shapes, other orders of the sums)
        assert ((o.double().cpu() - y).abs() <= err + 1e-30).all()


@gpu
@pytest.mark.parametrize("weight", [True, False])
def test_tiles_of_one_run_with_all_none_and_hundreds_of_adapters(weight):
    """More tiles than run at once; neighbouring runs of 256 tokens have 1, 0, about 200 and 3 adapters, so the loops over a tile's
    adapters are of very different lengths one after the other."""
    T, K, N, rank, n = 8192 - 5, 64, 1024, 16, 300
    d = inputs(T, K, N, rank, n, 11, weight=weight, base=not weight, out=torch.float32)
    rng = np.random.default_rng(5)
    adapter = np.full(T, -1, dtype=np.int32)
    for i in range(0, T, 256):
        m, kind = min(256, T - i), (i // 256) % 4
        adapter[i:i + m] = {0: rng.integers(0, n), 1: -1, 2: rng.integers(0, n, m), 3: rng.integers(0, 3, m)}[kind]
    tenant = torch.from_numpy(np.where(adapter < 0, n, adapter).astype(np.int32))           # (tenant n has no adapter)
    y, err = reference(d["x"], d["w"], d["base"], d["a"], d["b"], d["scale"], torch.from_numpy(adapter).long())
    g = {k: None if v is None else v.to(DEV) for k, v in d.items()}
    outs = [torch.empty(T, N, device=DEV) for _ in range(3)]
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for o in outs:
        B.moe_project(g["x"], g["w"], o, base=g["base"], a=g["a"], b=g["b"], scale=g["scale"], tenant_id=tenant.to(DEV), n_tenants=n + 1, status_out=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    assert ((outs[0].double().cpu() - y).abs() <= err + 1e-30).all()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@gpu
@pytest.mark.parametrize("T", [20, 130, 300, 900])
def test_one_tenants_numbers_do_not_reach_another(T):
    """Infinities and NaN in one adapter, in one token, in one row of w: they stay in their tokens and columns."""
    def bad_adapter(d):
        d["a"][1, 3, 5] = float("nan")
        d["b"][2, 7, :] = float("inf")
        d["b"][3, :, 0] = float("nan")

    def bad_tokens(d):
        d["x"][T // 2, 0] = float("nan")
        d["x"][3, 4] = float("inf")

    def bad_w(d):
        d["w"][9, 1] = float("nan")
    for layout in ("uniform", "contiguous"):
        check(T, 128, 200, rank=16, n=5, layout=layout, mutate=bad_adapter)
        check(T, 128, 200, rank=72, n=5, layout=layout, mutate=bad_adapter, weight=False)
        check(T, 128, 200, rank=16, n=5, layout=layout, mutate=bad_tokens)
        check(T, 128, 200, rank=16, n=5, layout=layout, mutate=bad_w)


@gpu
@pytest.mark.parametrize("T", [4, 40, 260])
def test_bad_ids_are_reported_and_have_no_adapter(T):
    d = inputs(T, 64, 96, 8, 3, seed=1)
    tenant = torch.arange(T, dtype=torch.int32) % 5
    table = torch.tensor([0, 3, -1, 2, -7], dtype=torch.int32)          # tenant 1 names an adapter that is not there
    bad = tenant.clone()
    bad[2] = 5
    bad[0] = -1
    adapter = table.long()[tenant.long()]
    adapter[tenant == 1] = -1
    adapter[adapter < 0] = -1
    for ids, want in ((tenant, B.MOE_DEV_BAD_ADAPTER), (bad, B.MOE_DEV_BAD_ADAPTER | B.MOE_DEV_BAD_TENANT)):
        ad = adapter.clone()
        ad[(ids < 0) | (ids > 4)] = -1
        y, err = reference(d["x"], d["w"], None, d["a"], d["b"], d["scale"], ad)
        o = torch.empty(T, 96, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.moe_project(d["x"].to(DEV), d["w"].to(DEV), o, a=d["a"].to(DEV), b=d["b"].to(DEV), scale=d["scale"].to(DEV), tenant_id=ids.to(DEV),
                      adapter_of_tenant=table.to(DEV), status_out=status)
        torch.cuda.synchronize()
        assert int(status) == want
        assert ((o.double().cpu() - y).abs() <= err).all()


@gpu
def test_no_tokens():
    e = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    B.moe_project(e, torch.zeros(32, 64, dtype=torch.bfloat16, device=DEV), torch.empty(0, 32, device=DEV))


@gpu
@pytest.mark.parametrize("T", [9, 200, 800])
def test_base_in_place_streams_graphs_and_repeats(T):
    d = inputs(T, 256, 320, 16, 6, seed=5, base=True, out=torch.float32)
    tenant = tenants(T, 6, "uniform", 3).to(DEV)
    g = {k: (v.to(DEV) if v is not None else None) for k, v in d.items()}
    kw = dict(a=g["a"], b=g["b"], scale=g["scale"], tenant_id=tenant)
    ref = torch.empty(T, 320, device=DEV)
    B.moe_project(g["x"], g["w"], ref, base=g["base"], **kw)
    torch.cuda.synchronize()
    # in place, on another stream, back to back, in a graph: the same bits
    o = g["base"].clone()
    B.moe_project(g["x"], g["w"], o, base=o, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o2 = torch.empty_like(ref)
    B.moe_project(g["x"], g["w"], o2, base=g["base"], stream=side, **kw)
    torch.cuda.synchronize()
    assert torch.equal(o, ref) and torch.equal(o2, ref)
    many = [torch.empty_like(ref) for _ in range(10)]
    ws = torch.empty(max(1, B.moe_project_workspace(T, 256, 320, 16, 6)), dtype=torch.uint8, device=DEV)
    for m in many:                                                  # one workspace, one stream
        B.moe_project(g["x"], g["w"], m, base=g["base"], workspace=ws, **kw)
    torch.cuda.synchronize()
    for m in many:
        assert torch.equal(m, ref)
    # two graphs, each with a workspace of its own, replayed side by side on two streams
    outs, graphs = [torch.empty_like(ref), torch.empty_like(ref)], []
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            B.moe_project(g["x"], g["w"], outs[i], base=g["base"], **kw)
        graphs.append(gr)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for i, s in enumerate((s1, s2)):
            with torch.cuda.stream(s):
                graphs[i].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], ref) and torch.equal(outs[1], ref)


@gpu
def test_weights_written_just_before_the_call_are_the_ones_used():
    """The call starts early (programmatic dependent launch): what the stream's earlier work wrote must still be seen, x and w
    of a plain copy as well as x from another call of the library."""
    T, K, N = 24, 1024, 1024
    d = inputs(T, K, N, 16, 4, seed=9)
    g = {k: (v.to(DEV) if v is not None else None) for k, v in d.items()}
    tenant = tenants(T, 4, "uniform", 3).to(DEV)
    mid, out = torch.empty(T, K, dtype=torch.bfloat16, device=DEV), torch.empty(T, N, device=DEV)
    w2 = (torch.randn(N, K, device=DEV) * 0.05).to(torch.bfloat16)
    w, x = torch.zeros_like(g["w"]), torch.zeros_like(g["x"])
    gamma = torch.ones(K, dtype=torch.bfloat16, device=DEV)
    for with_adapters in (False, True):
        kw = dict(a=g["a"], b=g["b"], scale=g["scale"], tenant_id=tenant) if with_adapters else {}
        first = None
        xn = torch.empty_like(x)
        for rep in range(20):
            w.zero_(); x.zero_(); xn.zero_()
            x.copy_(g["x"])
            w.copy_(g["w"])
            B.moe_add_rmsnorm(x, gamma, 1e-6, out=xn)
            B.moe_project(xn, w, mid, **kw)
            B.moe_project(mid, w2, out, **kw)
            torch.cuda.synchronize()
            if first is None:
                first = out.clone()
                ad = tenant.cpu().long() if with_adapters else torch.full((T,), -1)
                a = (d["a"], d["b"], d["scale"]) if with_adapters else (None, None, None)
                y, err = reference(xn.cpu(), d["w"], None, *a, ad)
                assert ((mid.double().cpu() - y).abs() <= err + 2.0 ** -8 * (y.abs() + err)).all()
                y, err = reference(mid.cpu(), w2.cpu(), None, *a, ad)
                assert ((out.double().cpu() - y).abs() <= err).all()
            assert torch.equal(out, first)


def _raw(**kw):
    a = dict(x=256, ldx=64, w=256, ldw=64, T=4, K=64, N=32, a=256, b=256, scale=None, n=2, rank=8, tenant=256, table=None, n_tenants=2, base=None, ldb=0,
             out=256, ldo=32, out_type=0, ws=256, ws_bytes=1 << 20, status=None)
    a.update(kw)
    return B.load_library().moe_project(*a.values(), None)


def test_refusals_need_no_gpu():
    for bad in (dict(x=None), dict(out=None), dict(T=300, ws=None), dict(a=None), dict(b=None), dict(tenant=None), dict(w=None, n=0), dict(x=None, n=0)):
        assert _raw(**bad) == B.MOE_ERR_NULL, bad
    for bad in (dict(T=-1), dict(T=(1 << 22) + 1), dict(K=0), dict(N=0), dict(n=-1), dict(ldx=56), dict(ldw=56), dict(ldo=31), dict(base=256, ldb=31), dict(rank=0),
                dict(rank=136), dict(n_tenants=0), dict(x=264), dict(w=264), dict(a=264), dict(b=260), dict(scale=258), dict(tenant=258), dict(table=258),
                dict(out=258), dict(out=257, out_type=1), dict(K=(1 << 30) + 8, ldx=1 << 31, ldw=1 << 31), dict(N=(1 << 30) + 1, ldo=1 << 31),
                dict(n=1 << 28), dict(base=258, ldb=32), dict(ws=128), dict(status=258)):
        assert _raw(**bad) == B.MOE_ERR_SHAPE, bad
    for bad in (dict(), dict(x=512, w=256), dict(x=512, w=512, b=512), dict(x=512, w=512, a=512), dict(x=512, w=512, n=0, base=256, ldb=40)):      # overlapping
        assert _raw(**bad) == B.MOE_ERR_SHAPE, bad
    for bad in (dict(K=60), dict(ldx=68), dict(ldw=68), dict(rank=12), dict(out_type=2)):
        assert _raw(**bad) == B.MOE_ERR_UNSUPPORTED, bad
    assert _raw(T=300, ws_bytes=255) == B.MOE_ERR_ALLOC
    assert _raw(T=0) == B.MOE_OK
    lib = B.load_library()
    assert lib.moe_project_workspace(-1, 64, 32, 8, 1) == B.MOE_ERR_SHAPE
    assert lib.moe_project_workspace(4, 64, 32, 129, 1) == B.MOE_ERR_SHAPE
    assert lib.moe_project_workspace(4, 64, 0, 8, 1) == B.MOE_ERR_SHAPE
    assert lib.moe_project_workspace(4, 64, 32, 8, 1 << 28) == B.MOE_ERR_SHAPE
    assert lib.moe_project_workspace(1 << 22, 64, 1 << 30, 8, 1) == 8 * 6 << 22          # (no overflow on the way)
    assert lib.moe_project_workspace(4, 64, 32, 0, 0) == 0
    assert lib.moe_project_workspace(1, 2048, 2048, 16, 3) == 0               # one pass, no workspace
    assert lib.moe_project_workspace(1000, 2048, 2048, 16, 3) == 1000 * 16 * 6


def test_binding_checks_tensors():
    bf = torch.bfloat16
    x, w, out = torch.zeros(4, 64, dtype=bf), torch.zeros(32, 64, dtype=bf), torch.zeros(4, 32)
    a, b, t = torch.zeros(2, 8, 64, dtype=bf), torch.zeros(2, 32, 8, dtype=bf), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.moe_project(x, w, out, a=a, b=b, tenant_id=t)
    for kw in (dict(a=a), dict(b=b), dict(a=a, b=b[:1], tenant_id=t), dict(a=a, b=b.transpose(1, 2), tenant_id=t), dict(a=a, b=b, tenant_id=t.long()),
               dict(a=a, b=b, tenant_id=t[:3]), dict(base=out.to(bf)), dict(a=a, b=b, tenant_id=t, scale=torch.ones(3)), dict(workspace=torch.zeros(300))):
        with pytest.raises(ValueError):
            B.moe_project(x, w, out, **kw)
    for bad in ((x.float(), w, out), (x, w[:, :32], out), (x, w, out.double()), (x[0], w, out), (x, w.t(), out)):
        with pytest.raises(ValueError):
            B.moe_project(*bad)


@gpu
@pytest.mark.parametrize("T", [3, 20, 130, 300, 900, 4000])
@pytest.mark.parametrize("out", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("weight", [True, False])
def test_an_inner_product_has_32_bits_in_batches_of_any_length(T, out, weight):
    """A base that takes the adapter's share back but for its rounding: what is left shows u to its last bits.  One product per output:
    u = scale * a is one fp32 rounding, its product with b is cut to 24 bits at most once per term it is handed over in (three) and
    once more where the base is added: 2^-24 + 4 * 2^-23 of |u b|, below 2^-20; then the output's own half step."""
    K, N, rank, n = 64, 200, 16, 5
    g = torch.Generator().manual_seed(T)
    a, b = torch.zeros(n, rank, K), torch.zeros(n, N, rank)
    a[:, 0, 0] = torch.rand(n, generator=g) + 0.5
    b[:, :, 0] = torch.rand(n, N, generator=g) + 0.5
    a, b, scale = a.to(torch.bfloat16), b.to(torch.bfloat16), torch.rand(n, generator=g) + 0.5
    x = torch.zeros(T, K)
    x[:, 0] = torch.rand(T, generator=g) + 0.5
    x = x.to(torch.bfloat16)
    adapter = torch.arange(T) % n
    share = (x[:, :1].double() * a[adapter, 0, :1].double() * scale[adapter].double()[:, None]) * b[adapter, :, 0].double()
    base = (-share).to(torch.bfloat16).to(out)
    y = share + base.double()
    o, dev = torch.empty(T, N, dtype=out, device=DEV), lambda t: t.to(DEV)
    w = torch.zeros(N, K, dtype=torch.bfloat16, device=DEV) if weight else None             # (adds nothing, but takes other shapes)
    B.moe_project(dev(x), w, o, base=dev(base), a=dev(a), b=dev(b), scale=dev(scale), tenant_id=dev(adapter.to(torch.int32)))
    torch.cuda.synchronize()
    lim = 2.0 ** -20 * share.abs() + (2.0 ** -8 if out == torch.bfloat16 else 2.0 ** -24) * y.abs()
    off = (o.double().cpu() - y).abs()
    assert (off <= lim).all(), f"{int((off > lim).sum())} of {off.numel()}, worst {float((off / lim).max()):.1f} of the bound"


@gpu
@pytest.mark.parametrize("rank", [8, 16, 72])
@pytest.mark.parametrize("T", [3, 20, 130, 300, 900])
@pytest.mark.parametrize("what", ["b", "u"])
def test_single_infinities_stay_infinities(T, rank, what):
    """One infinite element of B, or an infinite inner product: +-inf where the formula in 64 bits has it and NaN nowhere else, whatever
    shape the batch takes and however the inner product is handed over."""
    K, N, n = 128, 200, 4
    for weight, out in ((True, torch.float32), (True, torch.bfloat16), (False, torch.float32), (False, torch.bfloat16)):
        d = inputs(T, K, N, rank, n, T + rank, weight=weight, base=not weight, out=out, scale=False)
        adapter = torch.arange(T) % n
        if what == "b":
            d["b"][0, 7, 3], d["b"][1, 50, 1], d["b"][2, 9, 2] = float("inf"), -float("inf"), float("inf")
            # inner products of one bit, of which nothing is left to hand over behind the first term: 1, -2 and 2^-60
            d["x"][:3] = 0
            d["x"][0, 0], d["x"][1, 0], d["x"][2, 0] = 1, -2, 2.0 ** -60
            d["a"][:3, :, 0] = 1
        else:
            d["a"][1, 3, 5], d["a"][2, 0, 6] = float("inf"), -float("inf")
            d["x"][:, 5:7] = 1.0
        y, _ = reference(d["x"], d["w"], d["base"], d["a"], d["b"], None, adapter)
        g = {k: None if v is None else v.to(DEV) for k, v in d.items()}
        o, status = torch.empty(T, N, dtype=out, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        B.moe_project(g["x"], g["w"], o, base=g["base"], a=g["a"], b=g["b"], tenant_id=adapter.to(torch.int32).to(DEV), status_out=status)
        torch.cuda.synchronize()
        got = o.double().cpu()
        assert int(status) == 0 and bool(y.isinf().any()) and not y.isnan().any()
        assert not got.isnan().any(), f"{int(got.isnan().sum())} NaN, first at {got.isnan().nonzero()[0].tolist()}"
        assert torch.equal(got.isinf(), y.isinf()) and torch.equal(got[got.isinf()], y[y.isinf()])


@gpu
def test_status_without_a_status_word():
    """A call that passes no status_out leaves its bits in the device's own word, which is read and cleared."""
    d = inputs(20, 64, 96, 8, 3, seed=1)
    g = {k: None if v is None else v.to(DEV) for k, v in d.items()}
    o = torch.empty(20, 96, device=DEV)
    run = lambda ids, table=None: B.moe_project(g["x"], g["w"], o, a=g["a"], b=g["b"], scale=g["scale"], tenant_id=ids, adapter_of_tenant=table)
    ids = torch.zeros(20, dtype=torch.int32, device=DEV)
    B.moe_project_status()
    run(ids)
    assert B.moe_project_status() == 0
    ids[3] = 7
    run(ids)
    run(ids * 0, torch.full((1,), 5, dtype=torch.int32, device=DEV))
    assert B.moe_project_status() == B.MOE_DEV_BAD_TENANT | B.MOE_DEV_BAD_ADAPTER
    assert B.moe_project_status() == 0
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.moe_project(g["x"], g["w"], o, a=g["a"], b=g["b"], tenant_id=ids, status_out=status)
    assert B.moe_project_status() == 0 and int(status) == B.MOE_DEV_BAD_TENANT
    # from another stream, and out of a graph
    side = torch.cuda.Stream()
    B.moe_project(g["x"], g["w"], o, a=g["a"], b=g["b"], tenant_id=ids, stream=side)
    assert B.moe_project_status() == B.MOE_DEV_BAD_TENANT
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(ids)
    assert B.moe_project_status() == 0
    graph.replay()
    assert B.moe_project_status() == B.MOE_DEV_BAD_TENANT


def test_the_status_call_needs_somewhere_to_write():
    assert B.load_library().moe_project_status(None) == B.MOE_ERR_NULL
