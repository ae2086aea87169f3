"""Batches of clouds held in 4 bits, and draws from the plan of a finished batch: the operators as they are used together."""
import ctypes
import math

import numpy as np
import pytest

from test_draw import reference


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def problem(seed, W, n, m, d, fmt=None):
    """Embeddings in a few clusters, uneven weights; on the GPU."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    mu = torch.randn(W, 4, d, generator=gen)
    unit = lambda v: v / v.norm(dim=2, keepdim=True)
    pick = lambda k: torch.gather(mu, 1, torch.randint(4, (W, k, 1), generator=gen).expand(W, k, d))
    x, y = unit(torch.randn(W, n, d, generator=gen) + pick(n)), unit(torch.randn(W, m, d, generator=gen) + pick(m))
    a, b = 0.5 + torch.rand(W, n, generator=gen).double(), 0.5 + torch.rand(W, m, generator=gen).double()
    a, b = (a / a.sum(1, keepdim=True)).float(), (b / b.sum(1, keepdim=True)).float()
    eps = torch.full((W,), 0.1)
    return tuple(t.cuda() for t in (x, y, a, b, eps))


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
@pytest.mark.parametrize("shape,compute", [((5, 40, 50, 20), "auto"), ((3, 70, 66, 40), "f32"), ((4, 130, 100, 64), "auto"), ((3, 333, 257, 192), "tensor"),
                                           ((2, 1030, 300, 128), "auto"), ((6, 200, 210, 512), "auto"), ((2, 60, 90, 640), "auto")])
def test_a_packed_batch_is_the_batch_of_its_values(B, fmt, shape, compute):
    # The values are bf16 numbers.  Where no products are kept, the same kernels see the same inputs: equal bits.  Where they
    # are, they differ by the matrix unit's roundings: two runs of the parity suite's acceptance, potentials to 1e-4.
    import torch
    W, n, m, d = shape
    x, y, a, b, eps = problem(sum(shape), W, n, m, d)
    x4, y4 = B.cloud4_pack(x, fmt), B.cloud4_pack(y, fmt)
    kw = dict(compute=compute, max_iter=400)
    p = B.SinkhornBatch(x4, y4, a, b, eps, 1e-3, **kw)
    v = B.SinkhornBatch(x4.values(torch.bfloat16), y4.values(torch.bfloat16), a, b, eps, 1e-3, **kw)
    assert p.arithmetic() == v.arithmetic()
    p.drain(), v.drain()
    products = p.arithmetic() == "tensor"
    dp, dv = p.depths()[0], v.depths()[0]
    (fp, gp), (fv, gv) = p.potentials(f64=True), v.potentials(f64=True)
    img_p, img_v = p.apply_plan(y[:, :, :8]), v.apply_plan(y[:, :, :8])
    if not products:
        assert torch.equal(dp, dv) and torch.equal(fp, fv) and torch.equal(gp, gv) and torch.equal(img_p, img_v)
    else:
        assert bool(((dp - dv).abs() <= 1).all())
        same = dp == dv
        scale = max(float(fv.abs().max()), float(gv.abs().max()))
        assert bool(same.any()) and float((fp - fv)[same].abs().max()) <= 1e-4 * scale and float((gp - gv)[same].abs().max()) <= 1e-4 * scale
    assert bool((p.depths()[1] == B.LANE_DONE).all()) and float(torch.stack(p.residuals()).max()) <= 1e-3
    assert p.check_guards() == -1
    p.close(), v.close()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,shape", [(None, (3, 60, 45, 5)), ("nv4", (2, 130, 120, 128)), ("mx4", (3, 90, 100, 48))])
def test_pack_solve_and_draw_both_ways(B, fmt, shape):
    # the whole path, each draw the definition's with the potentials that the batch gives
    import torch
    W, n, m, d = shape
    x, y, a, b, eps = problem(7, W, n, m, d)
    if fmt:
        x, y = B.cloud4_pack(x, fmt), B.cloud4_pack(y, fmt)
    sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3)
    u, w = torch.rand(W, n, 2, generator=torch.Generator().manual_seed(1)).cuda(), torch.rand(W, m, generator=torch.Generator().manual_seed(2)).cuda()
    with pytest.raises(B.SkbError) as e:
        sb.draw_plan(u)
    assert e.value.code == 5                                     # not finished
    sb.drain()
    f, g = sb.potentials(f64=True)
    T, p = torch.full((W,), 0.8).cuda(), torch.full((W,), 0.9).cuda()
    idx, lp = sb.draw_plan(u, temperature=T, top_p=p, logp=True)
    assert torch.equal(idx, B.plan_draw(x, y, g, eps, u, temperature=T, top_p=p))
    back = sb.draw_plan(w, side="targets")
    assert back.shape == (W, m) and torch.equal(back, B.plan_draw(y, x, f, eps, w))
    h = lambda t: (t.values() if fmt and isinstance(t, B.Cloud4) else t).cpu().double().numpy()
    want, wlp = reference(h(x), h(y), g.cpu().numpy(), eps.cpu().numpy(), u.cpu().double().numpy(), T=T.cpu().numpy(), p=p.cpu().numpy())
    np.testing.assert_array_equal(idx.cpu().numpy(), want)
    assert np.abs(lp.cpu().numpy() - wlp).max() <= 1e-3
    want, _ = reference(h(y), h(x), f.cpu().numpy(), eps.cpu().numpy(), w.cpu().double().numpy()[:, :, None])
    np.testing.assert_array_equal(back.cpu().numpy(), want[:, :, 0])
    # the plan's own marginal: with many numbers, partners come up as often as the plan says (five standard deviations)
    many = torch.rand(W, n, 400, generator=torch.Generator().manual_seed(3)).cuda()
    got = sb.draw_plan(many).cpu().numpy()
    rows = sb.apply_plan(torch.eye(m, device="cuda")[None, :, :16].expand(W, m, 16).contiguous()).cpu().numpy()
    share = rows / a.cpu().numpy()[:, :, None]
    for j in range(16):
        hits, q = (got == j).sum(2), np.clip(share[:, :, j], 0, 1)
        total, expect, var = hits.sum(), 400 * q.sum(), 400 * (q * (1 - q)).sum()
        assert abs(total - expect) <= 5 * math.sqrt(var) + 400 * 1e-3 * W * n * q.mean() + 5
    sb.close()


@pytest.mark.gpu
def test_lanes_of_a_packed_batch_are_replaced(B):
    import torch
    W, n, m, d = 4, 150, 130, 128
    x, y, a, b, eps = problem(3, 2 * W, n, m, d)
    part = lambda t, s: t[s].contiguous()
    first, second = slice(0, W), slice(W, 2 * W)
    pk = lambda t, s: B.cloud4_pack(part(t, s), "nv4")
    sb = B.SinkhornBatch(pk(x, first), pk(y, first), a[first], b[first], eps[first], 1e-3, lane_capacity=2 * W)
    sb.drain()
    assert sb.refill(pk(x, second), pk(y, second), a[second], b[second], eps[second]) == W
    sb.drain()
    f, g = sb.potentials(f64=True)
    one = B.SinkhornBatch(pk(x, second), pk(y, second), a[second], b[second], eps[second], 1e-3)
    one.drain()
    f1, g1 = one.potentials(f64=True)
    assert torch.equal(sb.depths()[0][W:], one.depths()[0]) and torch.equal(f[W:], f1) and torch.equal(g[W:], g1)
    with pytest.raises(B.SkbError) as e:
        sb.draw_plan(torch.rand(W, n).cuda())
    assert e.value.code == 5                                     # the inputs of all lanes are not in one array
    with pytest.raises(ValueError):
        sb.refill(x[:1], y[:1], a[:1], b[:1], eps[:1])
    assert sb.check_guards() == -1
    sb.close(), one.close()


@pytest.mark.gpu
def test_packed_clouds_from_host_buffers(B):
    import torch
    W, n, m, d = 3, 100, 90, 200
    x, y, a, b, eps = problem(5, W, n, m, d)
    x4, y4 = B.cloud4_pack(x, "mx4"), B.cloud4_pack(y, "mx4")
    sb = B.SinkhornBatch(x4, y4, a, b, eps, 1e-3)
    sb.drain()
    want = sb.potentials()
    depth = sb.depths()[0].cpu()
    sb.close()
    cfg = B.make_config(W, n, m, d, format="mx4")
    ws = torch.empty(B.sinkhorn_batch_host_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.workspace, cfg.workspace_bytes = ws.data_ptr(), ws.numel()
    host = [t.cpu().contiguous() for t in (x4.buffer, y4.buffer, a, b, eps)]
    f, g, dep = torch.zeros(W, n), torch.zeros(W, m), torch.zeros(W, dtype=torch.int32)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    rc = B.lib.sinkhorn_batch_solve_host(*(ptr(t) for t in host), 1e-3, ctypes.byref(cfg), ptr(f), ptr(g), ptr(dep), None, None, None, None, None)
    assert rc == 0
    assert torch.equal(dep, depth) and torch.equal(f, want[0].cpu()) and torch.equal(g, want[1].cpu())


@pytest.mark.gpu
def test_a_nan_point_of_a_packed_cloud_is_reported(B):
    x, y, a, b, eps = problem(6, 2, 80, 70, 64)
    x[1, 3, 5] = float("inf")
    sb = B.SinkhornBatch(B.cloud4_pack(x, "nv4"), B.cloud4_pack(y, "nv4"), a, b, eps, 1e-3)
    with pytest.raises(B.SkbError) as e:
        sb.drain()
    assert e.value.code == 3
    sb.close()


def test_refusals_of_packed_batches_and_their_draws(B):
    ok = B.make_config(4, 64, 48, 128, format="nv4")
    plain = B.make_config(4, 64, 48, 128, bf16=True)
    staged = 4 * (64 + 48) * 128 * 2
    assert B.sinkhorn_batch_workspace_bytes(ok) == B.sinkhorn_batch_workspace_bytes(plain) + staged
    assert B.sinkhorn_batch_workspace_bytes(B.make_config(4, 64, 48, 1025, format="mx4")) == 0
    bad = B.make_config(4, 64, 48, 128)
    bad.xy_dtype = 4
    assert B.sinkhorn_batch_workspace_bytes(bad) == 0
    h, one, off = ctypes.c_void_p(), ctypes.c_void_p(4096), ctypes.c_void_p(4096 + 64)
    ok.workspace, ok.workspace_bytes = 4096, 1 << 40
    assert B.lib.sinkhorn_batch_create(off, one, one, one, one, 1e-3, ctypes.byref(ok), ctypes.byref(h)) == 3 and h.value is None
    assert b"aligned" in B.lib.sinkhorn_batch_last_error(None)
    ok.workspace_bytes = staged + 1000
    assert B.lib.sinkhorn_batch_create(one, one, one, one, one, 1e-3, ctypes.byref(ok), ctypes.byref(h)) == 4
    cfg = B.SkbDrawConfig(1, 4, 4, 2, 0, 1)
    assert B.lib.sinkhorn_batch_draw_plan(None, one, one, one, one, 0, ctypes.byref(cfg), one, None) == 1


@pytest.mark.gpu
def test_draws_from_a_batch_on_a_stream_of_its_own(B):
    # strided numbers and unaligned points are copied on the batch's stream, not behind what the current one is busy with
    import torch
    W, n, m, d = 2, 40, 50, 3
    x, y, a, b, eps = problem(12, W, n, m, d)
    room = torch.empty(W * n * d + 1, device="cuda")
    x = room[1:].copy_(x.reshape(-1)).view(W, n, d)
    u = torch.rand(4, n, W, generator=torch.Generator().manual_seed(5)).cuda().permute(2, 1, 0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3, stream=side)
    sb.drain()
    f, g = sb.potentials(f64=True)
    side.synchronize()
    want = B.plan_draw(x, y, g, eps, u)
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)                               # some 50 ms
    got = sb.draw_plan(u)
    side.synchronize()
    with torch.cuda.stream(side):
        assert torch.equal(got, want)
    torch.cuda.synchronize()
    sb.close()


@pytest.mark.gpu
@pytest.mark.parametrize("fmt,d", [(None, 3), ("bf16", 3), ("bf16", 64)])
def test_a_lane_that_went_non_finite_is_not_drawn_from(B, fmt, d):
    import torch
    W, n, m = 3, 40, 50
    x, y, a, b, eps = problem(8, W, n, m, d)
    if fmt:
        x, y = x.bfloat16(), y.bfloat16()
    u, w = torch.rand(W, n, 2, generator=torch.Generator().manual_seed(1)).cuda(), torch.rand(W, m, generator=torch.Generator().manual_seed(2)).cuda()
    out = []
    for broken in (False, True):
        if broken:
            y = y.clone()
            y[1, 5], y[1, 6] = 1e20, -1e20
        sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3, compute="f32")
        sb.drain()
        assert sb.depths()[1].tolist() == [B.LANE_DONE, B.LANE_NONFINITE if broken else B.LANE_DONE, B.LANE_DONE]
        out.append(sb.draw_plan(u, logp=True) + sb.draw_plan(w, side="targets", logp=True))
        sb.close()
    for fine, part in zip(*out):
        assert torch.equal(fine[::2], part[::2])
        assert bool((part[1] == -1).all()) if part.dtype == torch.int32 else bool(torch.isnan(part[1]).all())
        assert bool((fine != -1).all())


@pytest.mark.gpu
@pytest.mark.parametrize("mine", [False, True])
def test_draws_from_a_batch_on_another_stream_wait_for_their_numbers(B, mine):
    # the numbers and settings come from the caller's stream, which is busy, the draws are made on the batch's, the outputs are read on
    # the caller's; what it allocates next is not what the draws still read
    import torch
    W, n, m, d = 2, 40, 50, 3
    x, y, a, b, eps = problem(12, W, n, m, d)
    side, own = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3, stream=side)
    sb.drain()
    g = sb.potentials(f64=True)[1]
    torch.cuda.synchronize()
    u0, T0 = torch.rand(W, n, generator=torch.Generator().manual_seed(5)).cuda(), torch.full((W,), 0.7, device="cuda")
    want, wlp = B.plan_draw(x, y, g, eps, u0, temperature=T0, logp=True)
    torch.cuda.synchronize()
    with torch.cuda.stream(own if mine else torch.cuda.current_stream()):
        u, T = torch.zeros(W, n, device="cuda"), torch.zeros(W, device="cuda")
        torch.cuda._sleep(100_000_000)                           # some 50 ms
        u.copy_(u0), T.copy_(T0)
        got, lp = sb.draw_plan(u, temperature=T, logp=True)
        same = got.eq(want).all() & lp.eq(wlp).all()
        del u, T
        torch.full((W, n), 0.5, device="cuda")
        torch.full((W,), 3.0, device="cuda")
        assert bool(same)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(lp, wlp)
    sb.close()


@pytest.mark.gpu
@pytest.mark.parametrize("call", ["create", "potentials", "potentials64", "depths", "residuals", "apply_plan", "warm_start", "refill"])
def test_what_a_batch_on_another_stream_reads_and_writes_is_the_callers(B, call):
    # the caller's stream is busy with what the call reads, or has yet to clear what it writes
    import torch
    W, n, m, d = 3, 40, 50, 3
    parts = problem(12, W, n, m, d)
    side = torch.cuda.Stream()
    busy = lambda: torch.cuda._sleep(100_000_000)                # some 50 ms
    late = lambda t: torch.zeros_like(t).copy_(t)
    f0 = torch.linspace(-0.01, 0.01, W * n, dtype=torch.float64, device="cuda").view(W, n)
    v = torch.randn(W, m, 4, device="cuda")
    out = []
    for stream in (None, side):
        torch.cuda.synchronize()
        if call == "create":
            busy()
        sb = B.SinkhornBatch(*(late(t) if call == "create" else t for t in parts), 1e-3, stream=stream, lane_capacity=2 * W if call == "refill" else 0)
        if call == "warm_start":
            torch.cuda.synchronize()
            busy()
            sb.warm_start(late(f0))
        sb.drain()
        torch.cuda.synchronize()
        if call == "refill":
            busy()
            sb.refill(*(late(t) for t in parts))
            sb.drain()
            torch.cuda.synchronize()
        if call in ("potentials", "potentials64", "depths", "residuals"):
            busy()
            got = sb.potentials(f64=True) if call == "potentials64" else getattr(sb, call)()
        elif call == "apply_plan":
            busy()
            got = (sb.apply_plan(late(v)),)
        else:
            got = sb.potentials(f64=True) + sb.depths()
        got = [t.clone() for t in got]
        torch.cuda.synchronize()
        out.append(got)
        sb.close()
    assert bool((out[0][0] != 0).any())
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_a_refill_of_packed_clouds_that_is_refused_changes_nothing(B):
    # a misaligned cloud is seen before the values of the other one take the place of those that the plan is applied with
    import torch
    W, n, m, d = 2, 60, 50, 40
    x, y, a, b, eps = problem(9, 2 * W, n, m, d)
    x4, y4 = B.cloud4_pack(x[:W], "mx4"), B.cloud4_pack(y[:W], "mx4")
    sb = B.SinkhornBatch(x4, y4, a[:W], b[:W], eps[:W], 1e-3, lane_capacity=2 * W)
    sb.drain()
    v = torch.randn(W, m, 3, device="cuda")
    want = sb.apply_plan(v)
    other = B.cloud4_pack(x[W:], "mx4")
    room = torch.zeros(y4.buffer.numel() + 256, dtype=torch.uint8, device="cuda")
    first = ctypes.c_int(-1)
    ptr = lambda t, off=0: ctypes.c_void_p(t.data_ptr() + off)
    for bad in ((0, 64), (64, 0)):
        clouds = (ptr(other.buffer if bad[0] == 0 else room, bad[0]), ptr(room, bad[1]))
        assert B.lib.sinkhorn_batch_refill(sb.h, *clouds, ptr(a), ptr(b), ptr(eps), W, ctypes.byref(first)) == 3 and first.value == -1
        assert torch.equal(sb.apply_plan(v), want)
    sb.close()
