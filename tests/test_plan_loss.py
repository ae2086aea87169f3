"""The loss of scores against named entries of a coupling's rows, and its gradient, against the formulas in float64."""
import ctypes

import numpy as np
import pytest

U = 2.0 ** -24                                       # half a step of fp32, relative


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def formula(scores, index, logits, T, weight):
    """Loss, gradient and their error bounds, [r], [r, m], in float64 from float64 arrays.

    In fp32: an exponent (s - max) / T is off by 4 U of itself, an exponential by that and 2^-21.5, a sum of up to 128 terms in a chain by 128 U
    and what its terms are: 2^-16.5 covers a sum's relative error; logarithms add 2 U of themselves."""
    r, m = scores.shape
    named = (index >= 0) & (index < m)
    with np.errstate(all="ignore"):
        t = np.where(named, (np.zeros(index.shape) if logits is None else logits) / T, -np.inf)
        top = t.max(1, keepdims=True)
        live = (top > -np.inf).any(1) | np.isnan(t).any(1)
        t = t - np.where(top == -np.inf, 0.0, top)
        q = np.exp(t)
        q = q / np.where(live[:, None], q.sum(1, keepdims=True), 1.0)
        lq = np.log(q)
        z = (scores - scores.max(1, keepdims=True)) / T
        total = np.exp(z).sum(1, keepdims=True)
        zk = np.take_along_axis(z, np.where(named, index, 0), 1)
        lp = zk - np.log(total)
        terms = np.where(q > 0, q * (lq - lp), 0.0)
        loss = np.where(live, terms.sum(1), 0.0)
        p = np.exp(z) / total
        qs = np.zeros((r, m))
        for i in range(r):
            np.add.at(qs[i], index[i][named[i]], q[i][named[i]])
        w = (np.ones(r) if weight is None else weight)[:, None] / T
        grad = np.where(live[:, None], (p - qs) * w, 0.0)
        part = lambda v: np.where(q > 0, q * np.abs(v), 0.0).sum(1)
        err = 4 * U * (part(zk) + part(lq)) + 2.0 ** -16.5 + 2 * U * np.log(total[:, 0]) + part(lq - lp) * 2.0 ** -16 + part((lq - lp) * lq) * 4 * U
        gerr = np.abs(w) * (p * (4 * U * np.abs(np.where(p > 0, z, 0.0)) + 2.0 ** -16) + qs * 2.0 ** -15.5)
    return loss, grad, err, gerr, live


def run(B, scores, index, logits=None, T=1.0, weight=None, **kw):
    import torch
    cu = lambda v: None if v is None else v.cuda()
    loss, grad = B.plan_loss(scores.cuda(), index.cuda(), cu(logits), temperature=T, weight=cu(weight), grad=True)
    again = B.plan_loss(scores.cuda(), index.cuda(), cu(logits), temperature=T, weight=cu(weight))
    assert torch.equal(again.view(torch.int32), loss.view(torch.int32))         # (NaN is itself)
    assert grad.dtype == scores.dtype and grad.shape == scores.shape and loss.shape == scores.shape[:-1]
    return loss.cpu(), grad.cpu()


def check(B, scores, index, logits=None, T=1.0, weight=None):
    compare(*run(B, scores, index, logits, T, weight), scores, index, logits, T, weight)


def compare(loss, grad, scores, index, logits=None, T=1.0, weight=None):
    import torch
    loss, grad, scores, index, logits, weight = (None if v is None else v.cpu() for v in (loss, grad, scores, index, logits, weight))
    d = lambda v: None if v is None else v.double().numpy()
    want, wgrad, err, gerr, _ = formula(d(scores), index.numpy(), d(logits), T, d(weight))
    step = 2.0 ** -8 if scores.dtype == torch.bfloat16 else U
    assert (np.abs(loss.double().numpy() - want) <= err + U * np.abs(want)).all()
    assert (np.abs(grad.double().numpy() - wgrad) <= gerr + step * np.abs(wgrad) + 1e-37).all()


def inputs(rows, m, k, dtype, seed, logits=True, spread=3.0):
    import torch
    gen = torch.Generator().manual_seed(seed)
    scores = (spread * torch.randn(rows, m, generator=gen)).to(dtype)
    index = torch.randint(0, m, (rows, k), generator=gen, dtype=torch.int32)
    t = 2.0 * torch.randn(rows, k, generator=gen) if logits else None
    weight = torch.rand(rows, generator=gen)
    return scores, index, t, weight


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m", [1, 2, 7, 31, 64, 77, 500, 505, 512, 1021, 1024, 2043, 4090, 8185, 9000, 16390, 32761, 40001, 70001, 131068, 131069, 140000, 262143])
def test_rows_of_every_length(B, m, dtype):
    # the borders of a warp's, four warps', a block's and a cluster's registers, and rows that are read twice; odd lengths put rows at every
    # offset from a 16-byte boundary
    import torch
    rows = 9 if m < 9000 else 3
    scores, index, t, weight = inputs(rows, m, min(m, 5), getattr(torch, dtype), m)
    check(B, scores, index, t, 1.0, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m,k", [(1, 1), (5, 3), (8, 9), (31, 8), (64, 4), (121, 32), (128, 7), (200, 33), (250, 5), (256, 17), (257, 2), (300, 31), (505, 8), (512, 6)])
def test_many_short_rows(B, m, k, dtype):
    # several rows to a warp; entries named again, entries that name nothing, rows that name nothing, rows that start anywhere, gradients in place
    import torch
    rows, dt = 5003, getattr(torch, dtype)
    scores, index, t, weight = inputs(rows, m, k, dt, 7 * m + k)
    index[::3, -1] = index[::3, 0]
    index[1::7, 0] = -1
    index[2::11] = m
    check(B, scores, index, t, 1.3, weight)
    loss, grad = run(B, scores, index)
    compare(loss, grad, scores, index)
    wide = torch.zeros(rows, m + 3, dtype=dt, device="cuda")
    place = wide[:, 1:m + 1]
    place.copy_(scores)
    got, inplace = B.plan_loss(place, index.cuda(), t.cuda(), temperature=1.3, weight=weight.cuda(), grad=place)
    assert inplace.data_ptr() == place.data_ptr() and not wide[:, 0].any() and not wide[:, m + 1:].any()
    compare(got, inplace, scores, index, t, 1.3, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("m", [200, 255, 256, 257, 400, 505, 512, 513, 1000, 1017, 1024, 1025])
def test_very_many_short_rows(B, m, dtype):
    # 20481 rows that repeat 211 of them
    import torch
    dt = getattr(torch, dtype)
    scores, index, t, weight = inputs(211, m, 9, dt, m)
    index[::3, -1] = index[::3, 0]
    index[1::7, 0] = -1
    many = torch.arange(20481) % 211
    loss, grad = B.plan_loss(scores[many].cuda(), index[many].cuda(), t[many].cuda(), temperature=1.3, weight=weight[many].cuda(), grad=True)
    for first in (0, 211 * 97):
        n = min(211, 20481 - first)
        compare(loss[first:first + n], grad[first:first + n], *(v[:n] for v in (scores, index, t)), 1.3, weight[:n])
    bits = lambda v: v.contiguous().view(torch.int16 if v.dtype == torch.bfloat16 else torch.int32)
    if m % 8 == 0:                                                # (rows that start alike are summed alike)
        for r in (0, 1, 210):
            assert (bits(grad[r::211]) == bits(grad[r])).all() and (bits(loss[r::211]) == bits(loss[r:r + 1])).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_many_rows_of_middle_length(B, dtype):
    import torch
    for m in (3000, 5000, 8001):
        scores, index, t, weight = inputs(200, m, 8, getattr(torch, dtype), m, logits=False)
        check(B, scores, index, t, 0.7, weight)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,m", [("bfloat16", 32776), ("bfloat16", 40000), ("bfloat16", 98304), ("float32", 16388), ("float32", 20480), ("float32", 49152)])
def test_many_long_rows_of_whole_vectors(B, dtype, m):
    # more rows than blocks take at once, pieces that the last of them does not fill; every kind of entry among them
    import torch
    rows, k = 700, 40
    scores, index, t, weight = inputs(rows, m, k, getattr(torch, dtype), m)
    index[1] = 3
    index[2] = -1
    index[3, 5:] = -1
    t[4] = -float("inf")
    scores[5, 10:] = -float("inf")
    index[5] %= 10
    scores[6] = torch.finfo(scores.dtype).min
    want, wgrad = B.plan_loss(scores.cuda(), index.cuda(), t.cuda(), weight=weight.cuda(), grad=True)
    pick = torch.cat((torch.arange(16), torch.arange(rows - 160, rows)))
    compare(want[pick], wgrad[pick], scores[pick], index[pick], t[pick], 1.0, weight[pick])
    assert not torch.isnan(want).any() and not torch.isnan(wgrad).any()
    assert torch.equal(B.plan_loss(scores.cuda(), index.cuda(), t.cuda()), want)
    s = scores.cuda()
    loss, g = B.plan_loss(s, index.cuda(), t.cuda(), weight=weight.cuda(), grad=s)
    assert torch.equal(loss, want) and torch.equal(g, wgrad)
    # a NaN, plus infinity, nothing but minus infinity: their rows alone
    scores[8, m - 1], scores[9, 0], scores[11] = float("nan"), float("inf"), -float("inf")
    loss, g = B.plan_loss(scores.cuda(), index.cuda(), t.cuda(), weight=weight.cuda(), grad=True)
    bad = torch.tensor([8, 9, 11])
    assert torch.isnan(loss[bad]).all() and torch.isnan(g[bad]).all()
    rest = torch.ones(rows, dtype=torch.bool)
    rest[bad] = False
    assert torch.equal(loss[rest], want[rest]) and torch.equal(g[rest], wgrad[rest])


@pytest.mark.gpu
@pytest.mark.parametrize("k", [1, 2, 31, 32, 33, 64, 100, 255, 256])
@pytest.mark.parametrize("m", [300, 1500, 40000])
def test_numbers_of_named_entries(B, k, m):
    import torch
    scores, index, t, weight = inputs(6, m, k, torch.float32, k)
    check(B, scores, index, t, 2.0, weight)
    check(B, scores, index, None, 0.5, None)


@pytest.mark.gpu
@pytest.mark.parametrize("m", [20, 3000, 20000])
def test_entries_named_again_and_entries_that_name_nothing(B, m):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        scores, index, t, weight = inputs(12, m, 40, dtype, 5)
        index[0] = 3                                              # one entry, forty times
        index[1, ::2] = m - 1
        index[2] = -1                                             # nothing
        index[3, 5:] = -1
        index[4, :30], index[4, 30:] = m, 2 ** 31 - 1             # past the end: nothing
        index[5, 1:] = -2 ** 31
        t[6] = -float("inf")                                      # no weight at all
        t[7, 3:] = -float("inf")
        check(B, scores, index, t, 1.5, weight)
        check(B, scores, index, None, 1.0, None)
        loss, grad = run(B, scores, index, t)
        assert float(loss[2]) == 0.0 == float(loss[4]) == float(loss[6])
        assert not grad[2].any() and not grad[4].any() and not grad[6].any()


@pytest.mark.gpu
@pytest.mark.parametrize("m", [40, 2500, 20000])
def test_scores_of_minus_infinity_the_lowest_value_and_what_is_not_finite(B, m):
    import torch
    inf = float("inf")
    for dtype in (torch.float32, torch.bfloat16):
        scores, index, t, _ = inputs(9, m, 3, dtype, 8)
        index[:] = torch.tensor([1, 5, 9], dtype=torch.int32)
        scores[0, 10:] = -inf                                     # masked
        scores[1, 10:] = torch.finfo(dtype).min
        scores[2, 5] = -inf                                       # a named entry that the scores rule out
        scores[3] = -inf
        scores[4, 20] = float("nan")
        scores[5, 20] = inf
        scores[6, :] = torch.finfo(dtype).min
        t[7, 1] = float("nan")
        scores[8, :], index[8, :] = float("nan"), -1
        check(B, scores[:2], index[:2], t[:2])
        check(B, scores[6:7], index[6:7], t[6:7])
        loss, grad = run(B, scores, index, t)
        assert float(loss[2]) == inf and torch.isfinite(grad[2]).all() and float(grad[2, 5]) < 0
        for row in (3, 4, 5, 7):
            assert torch.isnan(loss[row])
        assert torch.isnan(grad[3]).all() and torch.isnan(grad[4]).all() and torch.isnan(grad[5]).all()
        assert float(loss[8]) == 0.0 and not grad[8].any()


@pytest.mark.gpu
def test_differences_of_the_loss(B):
    # central differences of the formula in float64, step h: off by h^2 / 6 of the third derivative, which is at most 2 / T^3 times the weight, and by
    # rounding, 2^-50 / h of a loss below 16
    import torch
    for m, T in ((11, 1.0), (300, 1.7)):
        scores, index, t, weight = inputs(4, m, 6, torch.float32, m)
        index[1, 1] = index[1, 0]
        _, grad = run(B, scores, index, t, T, weight)
        s = scores.double().numpy()
        _, _, _, gerr, _ = formula(s, index.numpy(), t.double().numpy(), T, weight.double().numpy())
        h = 1e-4
        for j in (0, 1, int(index[0, 0]), int(index[1, 0]), m - 1):
            up, down = s.copy(), s.copy()
            up[:, j] += h
            down[:, j] -= h
            a = formula(up, index.numpy(), t.double().numpy(), T, None)[0]
            b = formula(down, index.numpy(), t.double().numpy(), T, None)[0]
            want = weight.double().numpy() * (a - b) / (2 * h)
            assert (np.abs(grad[:, j].double().numpy() - want) <= gerr[:, j] + U * np.abs(want) + h * h / (3 * T ** 3) + 2.0 ** -46 / h).all()


@pytest.mark.gpu
@pytest.mark.parametrize("m", [45, 3001, 20000])
def test_spaced_rows_gradients_in_place_leading_shapes_and_one_entry(B, m):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        scores, index, t, weight = (v.cuda() for v in inputs(6, m, 4, dtype, 3))
        want, wgrad = B.plan_loss(scores, index, t, weight=weight, grad=True)
        wide = torch.full((6, m + 13), 5.0, dtype=dtype, device="cuda")
        wide[:, 2:m + 2] = scores
        view = wide[:, 2:m + 2]
        # (which scores a thread adds up goes by a row's distance from a 16-byte boundary: sums of a view differ from a copy's in rounding)
        loss, grad = B.plan_loss(view, index, t, weight=weight, grad=True)
        compare(loss, grad, scores, index, t, 1.0, weight)
        room = torch.full((6, m + 9), 5.0, dtype=dtype, device="cuda")
        B.plan_loss(view, index, t, weight=weight, grad=room[:, 1:m + 1])
        assert torch.equal(room[:, 1:m + 1], grad) and (room[:, 0] == 5).all() and (room[:, m + 1:] == 5).all()
        again, out = B.plan_loss(view, index, t, weight=weight, grad=view)
        assert out.data_ptr() == view.data_ptr() and torch.equal(loss, again) and torch.equal(view, grad)
        assert (wide[:, :2] == 5).all() and (wide[:, m + 2:] == 5).all()
        l3, g3 = B.plan_loss(scores.view(2, 3, m), index.view(2, 3, 4), t.view(2, 3, 4), weight=weight.view(2, 3), grad=True)
        assert torch.equal(l3.view(-1), want) and torch.equal(g3.view(6, m), wgrad)
        one = B.plan_loss(scores, index[:, 0].contiguous(), grad=True)
        two = B.plan_loss(scores, index[:, :1].contiguous(), grad=True)
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1])
        # columns that do not lie next to each other, rows that are one row
        assert torch.equal(B.plan_loss(scores.t().contiguous().t(), index, t), want)
        assert torch.equal(B.plan_loss(scores[:1].expand(6, m), index, t)[0], want[0])
        # one row
        assert torch.equal(B.plan_loss(scores[0], index[0], t[0]), want[0])


@pytest.mark.gpu
def test_a_step_that_learns_a_plan_continues_from_the_gradient(B):
    # scores of a bilinear matcher; its weights' gradient from the scores' against autograd's of the formula
    import torch
    gen = torch.Generator().manual_seed(1)
    W, n, m, d = 2, 60, 50, 8
    x, y = torch.randn(W, n, d, generator=gen).cuda(), torch.randn(W, m, d, generator=gen).cuda()
    a, b, eps = torch.full((W, n), 1 / n).cuda(), torch.full((W, m), 1 / m).cuda(), torch.full((W,), 0.5).cuda()
    sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3)
    sb.drain()
    index = sb.draw_plan(torch.rand(W, n, 4, generator=gen).cuda())
    sb.close()
    lin = torch.randn(d, d, generator=gen).cuda().requires_grad_()
    weight = torch.full((W, n), 1.0 / (W * n), device="cuda")
    scores = x @ lin @ y.transpose(1, 2)
    loss, grad = B.plan_loss(scores, index, weight=weight, grad=True)
    scores.backward(grad)
    ref = lin.detach().double().requires_grad_()
    s = x.double() @ ref @ y.double().transpose(1, 2)
    lp = torch.log_softmax(s, 2).gather(2, index.long())
    want = (-lp.mean(2) - np.log(4.0))
    (want.sum() / (W * n)).backward()
    # scores are sums of 64 products in fp32, so off by some 66 U of what they add up; the weights' gradient adds 120 rows of such p
    size = (x.abs().double() @ ref.detach().abs() @ y.abs().double().transpose(1, 2))
    ds = 80 * U * size
    assert ((loss.double() - want.detach()).abs() <= 2 * ds.amax(2) + 2.0 ** -15).all()
    bound = x.abs().double().transpose(1, 2) @ ((grad.abs().double() + weight.double()[:, :, None] / m) * (2 * ds.amax(2, keepdim=True) + 2.0 ** -14)) @ y.abs().double()
    assert ((lin.grad.double() - ref.grad).abs() <= bound.sum(0) * 4 + 1e-6 * ref.grad.abs().max()).all()


@pytest.mark.gpu
def test_another_stream_a_graph_and_its_replay_on_new_scores(B):
    import torch
    scores, index, t, weight = (v.cuda() for v in inputs(40, 700, 6, torch.bfloat16, 2))
    other = inputs(40, 700, 6, torch.bfloat16, 9)[0].cuda()
    want, want2 = B.plan_loss(scores, index, t, grad=True), B.plan_loss(other, index, t, grad=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = B.plan_loss(scores, index, t, grad=True)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    g = torch.cuda.CUDAGraph()
    static = scores.clone()
    with torch.cuda.graph(g):
        out = B.plan_loss(static, index, t, grad=True)
    g.replay()
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    static.copy_(other)
    g.replay()
    assert torch.equal(out[0], want2[0]) and torch.equal(out[1], want2[1])


def test_refusals_without_a_gpu(B):
    import torch
    one = ctypes.c_void_p(256)

    def call(scores=one, dtype=0, rows=4, m=8, ld=8, index=one, logits=None, k=2, T=1.0, weight=None, loss=one, grad=None, ldg=8):
        return B.lib.sinkhorn_plan_loss(scores, dtype, rows, m, ld, index, logits, k, T, weight, loss, grad, ldg, None)
    assert call(scores=None) == 1 and call(index=None) == 1 and call(loss=None) == 1
    for bad in (dict(rows=0), dict(m=0), dict(m=262144, ld=262144), dict(k=0), dict(k=257), dict(ld=7), dict(grad=ctypes.c_void_p(512), ldg=7),
                dict(grad=one, ld=9, ldg=8), dict(rows=2 ** 40)):
        assert call(**bad) == 2, bad
    for bad in (dict(dtype=2), dict(dtype=-1), dict(T=0.0), dict(T=-1.0), dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-31)):
        assert call(**bad) == 3, bad
    for bad in (dict(scores=ctypes.c_void_p(258)), dict(index=ctypes.c_void_p(258)), dict(logits=ctypes.c_void_p(257)), dict(weight=ctypes.c_void_p(6)),
                dict(loss=ctypes.c_void_p(2)), dict(grad=ctypes.c_void_p(514)), dict(dtype=1, scores=ctypes.c_void_p(257))):
        assert call(**bad) == 4, bad
    with pytest.raises(ValueError):
        B.plan_loss(torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32))


@pytest.mark.gpu
def test_refusals_on_the_device(B):
    import torch
    s, i = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    t, w = torch.zeros(4, 2, device="cuda"), torch.zeros(4, device="cuda")
    for args, kw in (((s.half(), i), {}), ((s, i.long()), {}), ((s, i.cpu()), {}), ((s, i[:3]), {}), ((s, i, t.double()), {}), ((s, i, t[:, :1]), {}),
                     ((s, i, t), dict(weight=w[:3])), ((s, i, t), dict(weight=w.double())), ((s, i, t), dict(grad=s.half())),
                     ((s, i, t), dict(grad=torch.zeros(8, 4, device="cuda").t())), ((s[:0], i[:0]), {}), ((s, i[:, :0]), {}),
                     ((torch.zeros(1, 262144, device="cuda"), i[:1]), {}), ((s, torch.zeros(4, 257, dtype=torch.int32, device="cuda")), {}),
                     ((s, i), dict(grad=torch.zeros(4, 8, device="cuda").t().contiguous().t()))):
        with pytest.raises(ValueError):
            B.plan_loss(*args, **kw)
    for T in (0.0, -1.0, float("nan")):
        with pytest.raises(B.SkbError):
            B.plan_loss(s, i, t, temperature=T)
