"""Draws from the rows of a coupling: indices, log probabilities, masks, settings and refusals.

The reference is the header's definition in float64 (numpy, distances by differences, one row at a time).  Indices have to be equal.
logp: its error is that of the weights, of their sum and one rounding to fp32; the fp32 path of the kernel forms weights with
a relative error below 1e-3 in every case here (rows it cannot decide go to float64), so |logp - reference| <= 1e-3 + 2^-23 |reference|."""
import math

import numpy as np
import pytest


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def row_reference(z, k, p, r, us):
    """Indices and log probabilities of one row of exponents (natural units, -inf: masked)."""
    m = len(z)
    if np.isnan(z).any() or (z == np.inf).any() or (z == -np.inf).all():
        return [-1] * len(us), [math.nan] * len(us)
    w = np.exp(z - z.max())
    order = np.lexsort((np.arange(m), -z))
    keep = np.zeros(m, bool)
    head = order[:k] if k > 0 else order
    if p < 1.0:
        cum = np.cumsum(w[head])
        head = head[:1 + int((cum < p * cum[-1]).sum())]
    keep[head] = True
    keep &= (w >= r) & (w > 0)
    cum = np.cumsum(np.where(keep, w, 0.0))
    idx, lp = [], []
    for u in us:
        if not 0.0 <= u < 1.0:
            idx.append(-1); lp.append(math.nan)
            continue
        j = int(np.searchsorted(cum, u * cum[-1], side="right"))
        j = min(j, int(np.nonzero(keep)[0][-1]))
        idx.append(j); lp.append(math.log(w[j] / cum[-1]))
    return idx, lp


def reference(x, y, g, eps, u, T=None, k=None, p=None, r=None):
    W, n, S = u.shape
    idx, lp = np.empty((W, n, S), np.int64), np.empty((W, n, S))
    for t in range(W):
        Tt, kt, pt, rt = 1.0 if T is None else float(T[t]), 0 if k is None else int(k[t]), 1.0 if p is None else float(p[t]), 0.0 if r is None else float(r[t])
        if not (0 <= Tt < math.inf and kt >= 0 and pt > 0 and 0 <= rt <= 1 and 0 < float(eps[t]) < math.inf):
            idx[t], lp[t] = -1, math.nan
            continue
        if Tt == 0:
            Tt, kt = 1.0, 1
        for i in range(n):
            with np.errstate(all="ignore"):
                c = ((x[t, i][None, :] - y[t]) ** 2).sum(1)
                z = np.where(g[t] == -np.inf, -np.inf, (g[t] - c) / (float(eps[t]) * Tt))
                idx[t, i], lp[t, i] = row_reference(z, kt, pt, rt, u[t, i])
    return idx, lp


def check(B, x, y, g, eps, u, T=None, k=None, p=None, r=None, fmt=None):
    """x, y: CPU tensors of the storage type; the others numpy or None."""
    import torch
    dev = lambda v, dt: None if v is None else torch.as_tensor(np.asarray(v)).to(dt).cuda()
    f32, i32 = torch.float32, torch.int32
    xd, yd = x.cuda(), y.cuda()
    xh, yh = x.double().numpy(), y.double().numpy()
    if fmt is not None:
        xd, yd = B.cloud4_pack(xd, fmt), B.cloud4_pack(yd, fmt)
        xh, yh = xd.values().cpu().double().numpy(), yd.values().cpu().double().numpy()
    if u.ndim == 2:
        u = u[:, :, None]
    u = np.asarray(u, np.float32)
    eps = np.asarray(eps, np.float32)
    T, p, r = (None if v is None else np.asarray(v, np.float32) for v in (T, p, r))
    idx, lp = B.plan_draw(xd, yd, dev(g, torch.float64), dev(eps, f32), dev(u, f32), temperature=dev(T, f32), top_k=dev(k, i32),
                          top_p=dev(p, f32), min_p=dev(r, f32), logp=True)
    want, wlp = reference(xh, yh, np.asarray(g), eps, u.astype(np.float64), T, k, p, r)
    idx, lp = idx.cpu().numpy(), lp.cpu().numpy()
    np.testing.assert_array_equal(idx, want)
    np.testing.assert_array_equal(np.isnan(lp), np.isnan(wlp))
    fine = ~np.isnan(wlp)
    assert (np.abs(lp - wlp)[fine] <= 1e-3 + 2.0 ** -23 * np.abs(wlp[fine])).all()
    return idx


def clouds(seed, W, n, m, d, dtype="f32", spread=1.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    x, y = spread * torch.randn(W, n, d, generator=gen), spread * torch.randn(W, m, d, generator=gen)
    if dtype == "bf16":
        x, y = x.bfloat16(), y.bfloat16()
    rng = np.random.default_rng(seed)
    g = 0.1 * rng.standard_normal((W, m))
    return x, y, g, rng


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (3, 5, 1, 2), (2, 9, 2, 3), (8, 64, 64, 2), (4, 33, 100, 3), (3, 40, 129, 5), (2, 50, 512, 15), (5, 17, 1000, 8),
                                   (1, 12, 5000, 3), (1, 5, 20000, 2), (1, 4, 30000, 3), (2, 30, 77, 33), (1, 20, 130, 200), (1, 9, 60, 1024)])
@pytest.mark.parametrize("cut", ["none", "k", "p", "r", "all"])
def test_draws_of_every_shape_and_cut(B, shape, cut):
    W, n, m, d = shape
    x, y, g, rng = clouds(sum(shape), *shape, spread=1.0 / math.sqrt(d))
    eps = rng.uniform(0.02, 0.3, W)
    kw = {}
    if cut in ("k", "all"): kw["k"] = rng.integers(0, m + 3, W)
    if cut in ("p", "all"): kw["p"] = rng.uniform(0.2, 1.1, W)
    if cut in ("r", "all"): kw["r"] = rng.uniform(0.0, 0.3, W)
    if cut == "all": kw["T"] = rng.uniform(0.3, 2.0, W) * (rng.random(W) > 0.2)
    check(B, x, y, g, eps, rng.random((W, n, 3), np.float32), **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "mx4", "nv4"])
@pytest.mark.parametrize("shape", [(2, 20, 90, 8), (3, 30, 130, 40), (2, 70, 200, 64), (1, 140, 300, 128), (2, 33, 257, 200), (1, 50, 1100, 512), (1, 20, 64, 1024)])
def test_draws_from_other_storage_types(B, dtype, shape):
    W, n, m, d = shape
    x, y, g, rng = clouds(7 + sum(shape), *shape, dtype=dtype, spread=1.0 / math.sqrt(d))
    eps = rng.uniform(0.03, 0.2, W)
    u = rng.random((W, n, 2), np.float32)
    fmt = None if dtype == "bf16" else dtype
    check(B, x, y, g, eps, u, fmt=fmt)
    check(B, x, y, g, eps, u, k=np.full(W, 20), p=np.full(W, 0.9), r=np.full(W, 0.01), T=np.full(W, 0.8), fmt=fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [3, 64, 200])
def test_masked_targets_and_their_coordinates(B, d):
    # padding: -inf potentials with NaN and infinite coordinates behind them; a lane without any target
    import torch
    W, n, m = 6, 25, 150
    for dtype in ("f32", "bf16"):
        x, y, g, rng = clouds(3, W, n, m, d, dtype=dtype, spread=1.0 / math.sqrt(d))
        real = [0, 1, 75, 128, 149, 150]
        for t, c in enumerate(real):
            g[t, c:] = -np.inf
            y[t, c:] = float("nan") if t % 2 else float("inf")
        g[3, 5:40] = -np.inf
        u = rng.random((W, n, 2), np.float32)
        for kw in ({}, dict(k=np.full(W, 7)), dict(p=np.full(W, 0.5)), dict(r=np.full(W, 0.05), T=np.full(W, 0.0))):
            idx = check(B, x, y, g, np.full(W, 0.1), u, **kw)
            assert (idx[0] == -1).all() and (idx[1] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [2, 64])
def test_values_that_are_not_finite_give_no_draw(B, d):
    W, n, m = 8, 6, 40
    for dtype in ("f32", "bf16"):
        x, y, g, rng = clouds(4, W, n, m, d, dtype=dtype, spread=1.0 / math.sqrt(d))
        x[0, 2, 0] = float("nan")
        x[1, 3, 1] = float("inf")
        y[2, 5, 0] = float("nan")
        y[3, 5, 0] = float("-inf")                               # infinitely far away: a weight of zero
        g[4, 7] = np.nan
        g[5, 7] = np.inf
        g[6, 8] = -1e308                                         # finite, but no weight
        idx = check(B, x, y, g, np.full(W, 0.1), rng.random((W, n), np.float32))
        assert (idx[2] == -1).all() and (idx[4] == -1).all() and (idx[5] == -1).all() and (idx[3] >= 0).all() and (idx[6:] >= 0).all()
        assert (idx[0, 2] == -1).all() and (idx[1, 3] == -1).all() and (idx[0, :2] >= 0).all()


@pytest.mark.gpu
def test_settings_that_are_not_valid_close_their_lane_only(B):
    W, n, m, d = 16, 4, 30, 3
    x, y, g, rng = clouds(5, W, n, m, d)
    T, k, p, r, eps = np.ones(W), np.zeros(W, int), np.ones(W), np.zeros(W), np.full(W, 0.1)
    T[1], T[2], T[3] = -0.5, np.nan, np.inf
    k[4], p[5], p[6], p[7] = -1, 0.0, np.nan, -1.0
    r[8], r[9], r[10] = -0.1, 1.5, np.nan
    eps[11], eps[12], eps[13] = 0.0, -1.0, np.nan
    p[14], r[15] = 7.0, 1.0
    u = rng.random((W, n, 2), np.float32)
    u[0, 0, 0], u[0, 1, 1], u[0, 2, 0], u[0, 3, 0] = 1.0, -0.25, np.nan, 0.0
    idx = check(B, x, y, g, eps, u, T=T, k=k, p=p, r=r)
    assert (idx[1:14] == -1).all() and (idx[14:] >= 0).all() and idx[0, 0, 0] == idx[0, 1, 1] == idx[0, 2, 0] == -1 and idx[0, 3, 0] >= 0


@pytest.mark.gpu
@pytest.mark.parametrize("m", [7, 64, 200, 1500])
def test_equal_weights_are_taken_in_the_order_of_their_indices(B, m):
    # all targets in one place, and in a few places
    import torch
    W, n, d = 5, 8, 3
    rng = np.random.default_rng(m)
    x = torch.zeros(W, n, d)
    y = torch.ones(W, m, d)
    place = torch.from_numpy(rng.integers(0, 4, (W, m)))
    y[2:] = 0.25 * place[2:, :, None].float().expand(W - 2, m, d)
    g = np.zeros((W, m))
    u = rng.random((W, n, 4), np.float32)
    u[:, 0] = [0.0, 0.25, 0.5, 0.75]
    eps = np.full(W, 0.5)
    for kw in ({}, dict(k=np.array([1, 3, 2, m // 2, m - 1])), dict(p=np.array([0.5, 0.25, 0.5, 0.9, 0.05])), dict(T=np.zeros(W)),
               dict(k=np.full(W, m // 2 + 1), p=np.full(W, 0.75), r=np.full(W, 0.2))):
        check(B, x, y, g, eps, u, **kw)


@pytest.mark.gpu
def test_near_ties_and_borders_are_those_of_float64(B):
    # weights that differ in the tenth digit, shares and numbers that sit within 1e-7 of a border: fp32 cannot tell these
    import torch
    W, n, m, d = 4, 16, 300, 2
    rng = np.random.default_rng(9)
    x, y = torch.zeros(W, n, d), torch.from_numpy(rng.standard_normal((W, m, d)).astype(np.float32)) * 0.05
    g = (y.double().numpy() ** 2).sum(2) + 1e-11 * rng.permutation(m)[None, :]       # exponents 1e-10 apart
    eps = np.full(W, 0.1)
    u = np.minimum((np.arange(n * 4).reshape(1, n, 4) * 37 % m + rng.choice([-1e-7, 0.0, 1e-7], (W, n, 4))) / m, 1 - 1e-7).clip(0).astype(np.float32)
    check(B, x, y, g, eps, u)
    check(B, x, y, g, eps, u, k=np.array([1, 10, 150, 299]))
    check(B, x, y, g, eps, u, T=np.zeros(W))
    check(B, x, y, g, eps, u, p=np.array([0.1, 0.5, 2 / 3, 0.99]))
    check(B, x, y, g, eps, u, r=np.array([1.0, 1 - 1e-7, 0.999, 1.0]))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [100, 700, 3500, 9000])
def test_cuts_far_below_the_heavy_entries(B, m):
    # few entries carry the mass; ranks, shares and sizes that cut among those that weigh 2^-20 to 2^-200 of them
    import torch
    W, n, d = 4, 10, 3
    rng = np.random.default_rng(m)
    x, y = torch.from_numpy(0.05 * rng.standard_normal((W, n, d)).astype(np.float32)), torch.from_numpy(rng.standard_normal((W, m, d)).astype(np.float32))
    y[:, ::50] *= 0.05
    g, eps = np.zeros((W, m)), np.array([0.2, 0.05, 0.02, 0.01])
    u = rng.random((W, n, 3), np.float32)
    u[:, :, 0] = 1 - 2.0 ** -24                                  # the far end of the row
    u[:, :, 1] = 0.0
    check(B, x, y, g, eps, u, k=np.array([m // 2, m // 10 + 3, m - 1, m // 3]))
    check(B, x, y, g, eps, u, p=np.array([0.9999999, 0.999999, 0.99999994, 0.9999]))
    check(B, x, y, g, eps, u, r=np.array([1e-9, 1e-7, 1e-12, 1e-30]))
    check(B, x, y, g, eps, u, k=np.full(W, m // 4), p=np.full(W, 0.999999), r=np.full(W, 1e-8))


@pytest.mark.gpu
def test_far_and_large_exponents(B):
    # potentials of a million eps, sources far from every target, weights that underflow
    W, n, m, d = 4, 12, 260, 3
    x, y, g, rng = clouds(12, W, n, m, d)
    x = x + 50.0
    g[1] += 1e4
    g[2] *= 1e3
    u = rng.random((W, n, 3), np.float32)
    eps = np.array([0.01, 0.01, 0.05, 1e-3])
    check(B, x, y, g, eps, u)
    check(B, x, y, g, eps, u, k=np.array([5, 100, 200, 250]), p=np.full(W, 0.999))


@pytest.mark.gpu
def test_rows_and_outputs_of_a_call_stand_alone(B):
    # two calls at once on two streams, a captured and replayed one, strided inputs, outputs without logp
    import torch
    W, n, m, d = 20, 60, 300, 4
    x, y, g, rng = clouds(21, W, n, m, d)
    dev = lambda v: torch.as_tensor(v).cuda()
    xd, yd, gd, eps, u = x.cuda(), y.cuda(), dev(g), torch.full((W,), 0.1).cuda(), dev(rng.random((W, n, 2), np.float32))
    first = B.plan_draw(xd, yd, gd, eps, u)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = B.plan_draw(xd, yd, gd, eps, u)
    again, _ = B.plan_draw(xd, yd, gd, eps, u, logp=True)
    torch.cuda.synchronize()
    assert torch.equal(first, other) and torch.equal(first, again)
    assert torch.equal(first[:, :, 0], B.plan_draw(xd, yd, gd, eps, u[:, :, 0]))
    assert torch.equal(first, B.plan_draw(xd.transpose(1, 2).contiguous().transpose(1, 2), yd, gd, eps, u))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = B.plan_draw(xd, yd, gd, eps, u)
    u.copy_(torch.rand(W, n, 2))
    graph.replay()
    assert torch.equal(held, B.plan_draw(xd, yd, gd, eps, u)) and not torch.equal(held, first)


def test_refusals_of_draws(B):
    import ctypes
    import torch
    L, one = B.lib, ctypes.c_void_p(4096)

    def cfg(W=1, n=4, m=4, d=2, dt=0, draws=1, ws=4096, size=1 << 40):
        return B.SkbDrawConfig(W, n, m, d, dt, draws, workspace=ws, workspace_bytes=size)

    call = lambda c, x=one, y=one, g=one, e=one, u=one, i=one: L.sinkhorn_plan_draw(x, y, g, e, u, ctypes.byref(c), i, None)
    assert L.sinkhorn_plan_draw_workspace_bytes(ctypes.byref(cfg())) > 0
    for bad in (dict(W=0), dict(n=0), dict(m=0), dict(d=0), dict(d=1025), dict(draws=0), dict(dt=4), dict(dt=-1), dict(m=1 << 18), dict(n=1 << 18), dict(W=65536)):
        assert L.sinkhorn_plan_draw_workspace_bytes(ctypes.byref(cfg(**bad))) == 0
        assert call(cfg(**bad)) == 2 and L.sinkhorn_operator_last_error()
    for name in ("x", "y", "g", "e", "u", "i"):
        assert call(cfg(), **{name: None}) == 1
    assert call(cfg(ws=None)) == 4 and call(cfg(ws=4096 + 8)) == 4 and call(cfg(size=100)) == 4
    assert call(cfg(), x=ctypes.c_void_p(4096 + 4)) == 3 and call(cfg(dt=2), y=ctypes.c_void_p(4096 + 64)) == 3
    with pytest.raises(ValueError):
        B.plan_draw(torch.zeros(1, 4, 2), torch.zeros(1, 4, 2), None, None, None)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 20, 150, 65), (2, 30, 300, 100), (1, 25, 700, 333), (1, 10, 40, 1023)])
def test_draws_of_deep_bf16_clouds_of_any_depth(B, shape):
    # rows that are no multiple of 16 bytes
    W, n, m, d = shape
    x, y, g, rng = clouds(5 + sum(shape), *shape, dtype="bf16", spread=1.0 / math.sqrt(d))
    eps, u = rng.uniform(0.03, 0.2, W), rng.random((W, n, 2), np.float32)
    check(B, x, y, g, eps, u)
    check(B, x, y, g, eps, u, k=np.full(W, 12), p=np.full(W, 0.9), r=np.full(W, 0.01))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [None, "nv4"])
@pytest.mark.parametrize("shape", [(5, 5000, 6000, 64), (2, 14000, 12000, 64)])      # several lanes at a time, several rows of a lane
def test_lanes_and_rows_of_large_problems_are_those_of_small_ones(B, fmt, shape):
    import torch
    W, n, m, d = shape
    x, y, g, rng = clouds(9, W, n, m, d, dtype="bf16", spread=1.0 / math.sqrt(d))
    x, y, g = x.cuda(), y.cuda(), torch.as_tensor(g).cuda()
    g[:, m - 5:] = -math.inf
    eps, p = torch.full((W,), 0.1).cuda(), torch.full((W,), 0.9).cuda()
    u = torch.rand(W, n, generator=torch.Generator().manual_seed(4)).cuda()
    cloud = (lambda v: v) if fmt is None else (lambda v: B.cloud4_pack(v, fmt))
    whole = B.plan_draw(cloud(x), cloud(y), g, eps, u, top_p=p)
    assert bool((whole >= 0).all()) and bool((whole < m - 5).all())
    for t in range(W):
        for rows in (slice(0, 40), slice(n // 2, n // 2 + 300), slice(n - 70, n)):
            part = B.plan_draw(cloud(x[t:t + 1, rows]), cloud(y[t:t + 1]), g[t:t + 1], eps[:1], u[t:t + 1, rows], top_p=p[:1])
            assert torch.equal(part[0], whole[t, rows])


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(6, 40, 77, 8), (3, 30, 900, 3), (2, 20, 6000, 4)])      # rows to a warp, to a block; flat rows and lists
def test_log_probabilities_of_large_exponents(B, shape):
    # Exponents of hundreds and thousands.  Weights are formed to 2^-24 of at most 22 (times ln 2) and 2^-22 each, what weighs less than
    # 2^-22 may be 1 % off (m 2^-22 / 100 of the sum) or, up to 2^-20 of the sum, missing; the drawn one's difference rounds to
    # 2^-24 of itself.  Where the row's largest exponent is below 16 those within 22 of it are off by (d + 6) 2^-24 of 38, the
    # drawn one's and those of the sum.
    import torch
    W, n, m, d = shape
    x, y, g, rng = clouds(31, W, n, m, d)
    eps = np.exp(rng.uniform(np.log(0.003), np.log(0.5), W))
    u = rng.random((W, n, 3), np.float32)
    bound = 22 * 2.0 ** -24 * 0.6932 + 2.0 ** -22 + m * 2.0 ** -22 / 100 + 2.0 ** -20 + 2 * 0.6932 * (d + 6) * 2.0 ** -24 * 38 + 2.0 ** -23
    for kw in ({}, dict(k=np.full(W, 9), p=np.full(W, 0.9)), dict(r=np.full(W, 0.05)), dict(T=np.full(W, 0.3), p=np.full(W, 0.8))):
        f = lambda v, dt: torch.as_tensor(v).to(dt).cuda()
        args = dict(top_k=f(kw["k"], torch.int32) if "k" in kw else None, top_p=f(kw["p"], torch.float32) if "p" in kw else None,
                    min_p=f(kw["r"], torch.float32) if "r" in kw else None, temperature=f(kw["T"], torch.float32) if "T" in kw else None)
        idx, lp = B.plan_draw(x.cuda(), y.cuda(), f(g, torch.float64), f(eps, torch.float32), f(u, torch.float32), logp=True, **args)
        cut = {key: np.asarray(v, np.float32) if key != "k" else v for key, v in kw.items()}
        want, wlp = reference(x.double().numpy(), y.double().numpy(), g, eps.astype(np.float32), u.astype(np.float64),
                              cut.get("T"), cut.get("k"), cut.get("p"), cut.get("r"))
        np.testing.assert_array_equal(idx.cpu().numpy(), want)
        off = np.abs(lp.cpu().numpy() - wlp)
        assert (off <= bound + 2.0 ** -23 * np.abs(wlp)).all(), off.max()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 256, 512, 1024])
@pytest.mark.parametrize("fmt", [None, "mx4", "nv4"])
def test_products_that_the_matrix_unit_cuts_off_one_by_one(B, d, fmt):
    # One dimension carries a product of 1, each of the others one of just below 2^-25 (or a little more): beside the large sum
    # they are cut off one by one, which is far more than a unit in the last place of the sum for 16 dimensions.  Half of
    # the targets have only the first dimension.  Numbers around the border between the two halves' shares.
    import torch
    W, n, m = 8, 800, 4
    x, y = torch.zeros(W, n, d), torch.zeros(W, m, d)
    for t in range(W):
        size = (1.9921875 if fmt is None else 1.5) * 2.0 ** -(11 + t / 2 if fmt is None else 11 + t // 2)
        x[t], y[t, ::2] = size, size
        if fmt is not None:
            x[t, :, :32], y[t, :, :32] = 0.0, 0.0
    x[:, :, 0], y[:, :, 0] = 1.0, 1.0
    eps = np.full(W, 0.05)
    u = np.linspace(0.25 - 4e-4, 0.25 + 4e-4, n // 2)
    u = np.broadcast_to(np.concatenate((u, u + 0.25))[None, :], (W, n))
    g = (y.bfloat16().double() ** 2).sum(2).numpy()
    check(B, x.bfloat16(), y.bfloat16(), g, eps, u, fmt=fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [312, 600, 3000])                  # a whole row, lists
def test_shares_behind_a_rank_that_cuts_among_negligible_weights(B, m):
    # ten entries carry the mass, the others 2^-26 of the largest each, less than 2^-20 of the mass together; the rank cuts among
    # those.  The share is of what the rank left: shares between a border of that mass and the same border of all mass.
    import torch
    heavy = np.array([1.0, 0.9, 0.8, 0.7, 0.6, 0.5, 0.4, 0.3, 0.2, 0.1])
    tail = heavy.sum() * 0.9 * 2.0 ** -20 / (m - 10)
    W, n = 14 * 7, 4
    rng = np.random.default_rng(m)
    w = np.full((W, m), tail)
    p = np.empty(W, np.float32)
    for t in range(W):
        w[t, rng.choice(m, 10, replace=False)] = heavy
        left = np.sort(w[t])[::-1][:12]
        p[t] = left[:2 + t % 7].sum() / left.sum()
        for _ in range(t // 7):                                  # 0 to 13 steps below the border
            p[t] = np.nextafter(p[t], np.float32(0))
    u = (0.9 * rng.random((W, n, 2))).astype(np.float32)
    check(B, torch.zeros(W, n, 1), torch.zeros(W, m, 1), np.log(w), np.ones(W), u, k=np.full(W, 12), p=p)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", [None, "mx4", "nv4"])
@pytest.mark.parametrize("far", [2e19, 1e25, 1e36])
def test_deep_points_whose_squares_pass_the_range_of_fp32(B, fmt, far):
    # sources and targets at the same far place; some targets elsewhere (a weight of zero), some masked
    import torch
    W, n, m, d = 3, 12, 90, 64
    x, y, g, rng = clouds(int(math.log(far)), W, n, m, d, dtype="bf16", spread=0.1)
    x[0, :, 3] = far                                             # all targets there, but for three
    y[0, :, 3] = far
    y[0, 7:10, 3] = 0.0
    x[1, 4, 3] = far                                             # one source and one target
    y[1, 11, 3] = far
    y[2, :, 3] = far                                             # targets that no source is near
    x[2, 5, 3] = far
    g[:, 20:24] = -np.inf
    check(B, x, y, g, np.full(W, 0.1), rng.random((W, n, 4), np.float32), fmt=fmt)
    check(B, x, y, g, np.full(W, 0.1), rng.random((W, n, 4), np.float32), k=np.full(W, 5), p=np.full(W, 0.8), fmt=fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 8, 50, 1), (2, 5, 700, 3), (1, 3, 9000, 2)])
def test_distances_past_the_range_of_fp32_beside_an_eps_as_large(B, shape):
    W, n, m, d = shape
    x, y, g, rng = clouds(2, W, n, m, d)
    x, y = x * 1.5e19, y * 1.5e19
    check(B, x, y, g, np.full(W, 3e38), rng.random((W, n, 8), np.float32))
    check(B, x, y, g, np.full(W, 3e38), rng.random((W, n, 8), np.float32), p=np.full(W, 0.9), T=np.full(W, 3.0))


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-38, 2e-37, 1e-35, 1e-33, 1e-30])
@pytest.mark.parametrize("shape,dtype,fmt", [((2, 800, 50, 64), "bf16", None), ((2, 800, 50, 64), "bf16", "mx4"), ((2, 800, 50, 128), "bf16", "nv4"), ((2, 800, 50, 3), "f32", None)])
def test_distances_at_the_low_end_of_fp32_beside_an_eps_as_small(B, shape, dtype, fmt, eps):
    W, n, m, d = shape
    x, y, g, rng = clouds(2, W, n, m, d, dtype=dtype)
    x, y = x * (eps / d) ** 0.5, y * (eps / d) ** 0.5
    check(B, x, y, g * eps, np.full(W, eps), rng.random((W, n), np.float32), fmt=fmt)


@pytest.mark.gpu
def test_more_rows_than_32_bits_count(B):
    # 4.3e9 rows, a row to a warp.  Most lanes are without targets, which takes no time; those that have some, at both ends and across
    # the 2^32nd row, are drawn from like each for itself.  (The numbers, all within [0, 1), are the sources as well: 75 GB as a whole.)
    import torch
    W, n, m = 65535, 65540, 1000
    u = torch.full((W, n), 0.25, device="cuda")
    some = [0, 1, 32767, 65532, 65533, 65534]                    # 65532 has row 2^32
    assert W * n > 1 << 32 and (1 << 32) // n == 65532
    gen = torch.Generator("cuda").manual_seed(3)
    for t in some:
        u[t] = torch.rand(n, generator=gen, device="cuda")
    y = torch.rand(W, m, 1, generator=gen, device="cuda")
    g = torch.full((W, m), -math.inf, dtype=torch.float64, device="cuda")
    g[some] = 0.0
    eps = torch.full((W,), 0.01, device="cuda")
    index = B.plan_draw(u[:, :, None], y, g, eps, u)
    for lo in range(0, W, 8192):
        part = index[lo:lo + 8192]
        drawn = (part != -1).any(1).nonzero().reshape(-1).tolist()
        assert [lo + t for t in drawn] == [t for t in some if lo <= t < lo + 8192]
    for t in some:
        one = slice(t, t + 1)
        assert torch.equal(index[one], B.plan_draw(u[one, :, None], y[one], g[one], eps[one], u[one])) and bool((index[t] >= 0).all())
    del u, y, g, index, part
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("m,heavy", [(512, 512), (1024, 1024), (2000, 2000), (8192, 8192), (22000, 22000), (8000, 1900), (22900, 5700)])
def test_shares_of_rows_whose_sums_all_round_one_way(B, m, heavy):
    # Each thread's sum begins above 1 and every further weight is a whole number and 0.48 of its unit in the last place, which an
    # addition in fp32 loses: up to 180 times.  Shares just below and at borders among the small weights, of rows and (where most
    # entries are masked) of lists.
    import torch
    W, n = 12, 3
    rng = np.random.default_rng(m)
    w = np.zeros((W, m))
    w[:, :heavy] = (np.floor(6.6e-4 * rng.uniform(1.04, 1.6, (W, heavy)) * 2 ** 23) + 0.48) * 2.0 ** -23
    w[:, 0:128:4] = 1.0
    order = np.sort(w, axis=1)[:, ::-1]
    cum = np.cumsum(order, 1)
    p = np.empty(W, np.float32)
    for t in range(W):
        j = 32 + int((heavy - 33) * (t + 1) / (W + 1))
        p[t] = cum[t, j] / cum[t, -1]
        for _ in range(t % 4):
            p[t] = np.nextafter(p[t], np.float32(0))
    with np.errstate(divide="ignore"):
        g = np.log(w)
    u = rng.random((W, n), np.float32)
    u[:, 0] = 1 - 2.0 ** -24                                     # the last entry that is kept
    check(B, torch.zeros(W, n, 1), torch.zeros(W, m, 1), g, np.ones(W), u, p=p)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(6, 40, 77, 8), (3, 30, 900, 3), (2, 20, 6000, 4)])
def test_log_probabilities_on_both_sides_of_the_border_of_large_exponents(B, shape):
    # Rows whose largest exponent is A: from DRAW_FAR = 48 on weights above 2^-22 are formed from their points in double, and off by
    # 2^-24 of at most 22 (times ln 2) and 2^-22 each; below that exponents are off by (d + 6) 2^-24 (A + 22), the drawn one's
    # and those of the sum.  In both, what weighs less than 2^-22 may be 1 % off (m 2^-22 / 100 of the sum) or, up to 2^-20 of
    # the sum, missing, and the result rounds to 2^-24 of itself (twice: it is formed as a difference).
    import torch
    W, n, m, d = shape
    x, y, g, rng = clouds(31, W, n, m, d)
    eps = np.exp(rng.uniform(np.log(0.003), np.log(0.5), W)).astype(np.float32)
    u = rng.random((W, n, 3), np.float32)
    f = lambda v, dt: torch.as_tensor(v).to(dt).cuda()
    idx, lp = B.plan_draw(x.cuda(), y.cuda(), f(g, torch.float64), f(eps, torch.float32), f(u, torch.float32), logp=True)
    xh, yh = x.double().numpy(), y.double().numpy()
    want, wlp = reference(xh, yh, g, eps, u.astype(np.float64))
    np.testing.assert_array_equal(idx.cpu().numpy(), want)
    z = np.stack([(g[t] - g[t].max() - ((xh[t][:, None, :] - yh[t][None]) ** 2).sum(2)) / float(eps[t]) for t in range(W)]) / math.log(2)
    A = -z.max(2)[:, :, None]
    double = 22 * 2.0 ** -24 * 0.6932 + 2.0 ** -22 + m * 2.0 ** -22 / 100 + 2.0 ** -20 + 2.0 ** -23 * np.abs(wlp)
    single = double + 2 * 0.6932 * (d + 6) * 2.0 ** -24 * (A + 22) + 2.0 ** -23
    bound = np.where(A > 48.01, double, single)
    off = np.abs(lp.cpu().numpy() - wlp)
    assert (off <= bound).all(), (off / bound).max()
    assert (A > 48.01).any() and (A < 48).any()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [96, 128, 333, 1000])
def test_log_probabilities_of_deep_fp32_clouds(B, d):
    # Largest exponents between 4096 / (d + 6) and 48, a few targets of about the same weight: entries above a sixteenth and those drawn are
    # formed from their points in double.  The drawn one's difference and the sum's logarithm are of a few units (below 8) and round to
    # 2^-24 of that each, weights of the sum are good to 2^-22 and it to 2^-24; log2 and the product to three roundings of 8.
    import torch
    W, n, m = 6, 30, 8
    rng = np.random.default_rng(d)
    x = rng.standard_normal((W, n, d)) / math.sqrt(d)
    y = (rng.standard_normal((W, 1, d)) + 0.01 * rng.standard_normal((W, m, d))) / math.sqrt(d)
    x, y = x.astype(np.float32), y.astype(np.float32)
    g, eps = np.zeros((W, m)), np.full(W, 0.072, np.float32)
    u = rng.random((W, n, 2), np.float32)
    f = lambda v: torch.as_tensor(v).cuda()
    idx, lp = B.plan_draw(f(x), f(y), f(g), f(eps), f(u), logp=True)
    want, wlp = reference(x.astype(np.float64), y.astype(np.float64), g, eps, u.astype(np.float64))
    np.testing.assert_array_equal(idx.cpu().numpy(), want)
    z = -((x[:, :, None, :].astype(np.float64) - y[:, None]) ** 2).sum(3) / 0.072 / math.log(2)
    A = -z.max(2)
    w = np.exp2(z - z.max(2, keepdims=True))
    rows = (A > 4100 / (d + 6)) & (A < 48) & ((w / w.sum(2, keepdims=True)).min(2) > 0.07)
    assert rows.sum() > 20
    off = np.abs(lp.cpu().numpy() - wlp)[rows]
    assert off.max() <= 2.0 ** -22 + 2.0 ** -24 + 5 * 8 * 2.0 ** -24, off.max()
