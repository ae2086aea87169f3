"""Images under the entropic map where least is to spare: rows without targets beside what is not finite, potentials of the lowest finite values, long banks of
values of one sign, products that one dimension carries, values far larger than those that have the weights."""
import pytest

from test_cloud8_map import B, U, formula, inputs, run  # noqa: F401  (B is the fixture)


def staged(B, W, n, m, d, dv=0):
    """Whether a call takes the kernel for many queries: its workspace holds the bank as bf16."""
    blocks = -(-d // 128) + (-(-dv // 128) if dv else 0)
    return B.lib.sinkhorn_cloud8_map_workspace_bytes(W, n, m, d, dv) > W * -(-m // 128) * 32768 * blocks


@pytest.mark.gpu
@pytest.mark.parametrize("W,n,m,many", [(7, 3, 300, False), (40, 20, 700, False), (7, 100, 3000, True), (7, 300, 6000, True), (40, 300, 400, True)])
def test_queries_without_targets_have_no_images_whatever_they_hold(B, W, n, m, many):
    import torch
    for own in (0, 24):
        assert staged(B, W, n, m, 96, own) == many
        x, y, g, eps, v = inputs(W, n, m, 96, own)
        for t in (0, 1):
            x[t, 1, 5], x[t, 2, 7] = float("nan"), -float("inf")
        g[0], g[2], g[3] = -float("inf"), -float("inf"), -float("inf")
        eps[2], eps[3] = -1.0, float("nan")
        g[1, 5:] = -float("inf")                                  # few targets, in the first tile of all
        g[4, :m - 5] = -float("inf")                              # ... and in the last
        x[4, 0, 0] = float("nan")
        y[0, 7], y[3, 9] = float("nan"), float("inf")
        lengths = torch.full((W,), m, dtype=torch.int32)
        lengths[5], eps[5], x[5, 0, 0] = 0, 0.0, float("nan")
        out, lse, _, _ = run(B, x, y, g, eps, v, lengths)
        for t in (0, 2, 3, 5):
            assert not out[t].any() and not torch.isnan(out[t]).any() and (lse[t] == -float("inf")).all(), t
        # with one target they are what they hold
        for t, i in ((1, 1), (1, 2), (4, 0)):
            assert torch.isnan(out[t, i]).all() and torch.isnan(lse[t, i])
        assert not torch.isnan(out[6]).any() and not torch.isnan(out[1, 0]).any() and not torch.isnan(out[4, 1:]).any()
        # an eps that is no number, with targets
        eps[6] = -1.0
        y[6, :] = 2.0 ** 70                                       # (squared lengths past fp32's range)
        out, lse, _, _ = run(B, x, y, g, eps, v, lengths)
        assert torch.isnan(out[6]).all() and torch.isnan(lse[6]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,m,many", [(3, 300, False), (20, 700, False), (300, 1500, True), (100, 3000, True)])
def test_potentials_of_the_lowest_finite_values_are_no_masks(B, n, m, many):
    # as a mask they leave nothing but the others; where there are no others all targets are alike
    import torch
    W, lowest = 7, (torch.finfo(torch.float32).min, torch.finfo(torch.float64).min)
    assert staged(B, W, n, m, 64, 16) == many
    x, y, g, eps, v = inputs(W, n, m, 64, 16)
    for t in (0, 1):
        g[t] = lowest[t]
        g[2 + t, ::2] = lowest[t]
        g[4 + t, 1:] = lowest[t]
    g[0, 5], g[1, 6] = -float("inf"), -float("inf")
    out, lse, _, vv = run(B, x, y, g, eps, v)
    for t, masked in ((0, 5), (1, 6)):
        keep = torch.arange(m) != masked
        want = vv[t, keep].double().mean(0)
        # weights are 1 exactly, and so are two e4m3 numbers for a power of two; 24 tiles of eight instructions that lose 2^-20.6 each: 2^-13; images are
        # rounded to bf16
        assert ((out[t] - want).abs() <= 2.0 ** -13 * vv[t].double().abs().mean(0) + 2.0 ** -8 * want.abs() + 1e-30).all()
        assert (lse[t] < -1e38).all()
    pick = slice(2, 7)
    g = torch.where(g < -1e30, -float("inf"), g)
    want, wl, err, lerr = formula(x[pick], B.cloud8_pack(y.cuda()).values().cpu()[pick], g[pick], eps[pick], vv[pick], None)
    assert ((out[pick] - want).abs() <= err).all() and ((lse[pick] - wl).abs() <= lerr).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,m,dv", [(9600, 262143, 16), (5, 262143, 16), (4864, 100001, 300), (300, 262143, 130)])
def test_long_banks_whose_values_have_one_sign(B, n, m, dv):
    # All points are zero, so weights are 2^(g / eps log2 e), between 1/2 and 1, and rounded to bf16 (rounding of them cancels over the bank; the second
    # e4m3 number of the kernel for few queries leaves less).  The values are positive, but for the last targets, which take back what the others came
    # to: what is left shows a sum's error without bf16's rounding of the image.
    #
    # The matrix unit cuts each of 16 products and the sum so far at 2^-25 of the largest, the result at 24 bits: 17 2^-25 + 2^-23 < 2^-20.6 of the sum
    # for each 16 targets, and sums of at most 64 tiles of 128 are added in fp32: 512 2^-20.6 = 2^-11.6 of the sum of magnitudes, 2^-16 for the
    # rest.
    import torch
    gen = torch.Generator().manual_seed(m)
    d, last = 16, 100
    g = -torch.rand(1, m, generator=gen, dtype=torch.float64) * 0.69
    g[0, -last:] = 0.0
    g[0, 0] = 0.0
    v = 1.0 + torch.rand(1, m, dv, generator=gen)
    v8 = B.cloud8_pack(v.cuda()).values().cpu().double()
    w = torch.exp(g[0])
    rounded = w.float().bfloat16().double() if staged(B, 1, n, m, d, dv) else w
    v[0, -last:] = -(rounded[:-last] @ v8[0, :-last] / last).float()
    v8 = B.cloud8_pack(v.cuda()).values().cpu().double()
    x, y, eps = torch.zeros(1, n, d, dtype=torch.bfloat16), torch.zeros(1, m, d), torch.ones(1)
    out, lse, _, _ = run(B, x, y, g, eps, v)
    want, size = rounded @ v8[0] / w.sum(), w @ v8[0].abs() / w.sum()
    assert ((out[0] - want).abs() <= (2.0 ** -11.6 + 2.0 ** -16) * size + 2.0 ** -8 * want.abs()).all(), float(((out[0] - want).abs() / size).max())
    assert ((lse[0] - torch.log(w.sum())).abs() <= 2.0 ** -16 + 2 * U * 13).all()


@pytest.mark.gpu
@pytest.mark.parametrize("W,n,m,dv", [(38, 140, 20000, 0), (20, 140, 30000, 150), (80, 100, 17000, 40)])
def test_long_banks_whose_exponents_rise_fall_begin_late_and_end_early(B, W, n, m, dv):
    # sums in parts of 64 tiles meet references that have been raised since, or that were not there yet
    import torch
    assert staged(B, W, n, m, 32, dv)
    x, y, g, eps, v = inputs(8, n, m, 32, dv, eps=0.3)
    ramp = torch.linspace(0, 12, m, dtype=torch.float64)
    g[0], g[1] = ramp, ramp.flip(0)
    g[2, :9000] = -float("inf")
    g[3, 8191:] = -float("inf")
    g[4, 5:m - 5] = -float("inf")
    g[5, 8190:8200] += 30
    x[6, 1, 3] = float("nan")
    lengths = torch.tensor([m, m, m, m, m, m, 8193, 8192], dtype=torch.int32)
    more = lambda t: None if t is None else t[torch.arange(W) % 8]
    out, lse, yv, vv = run(B, *(more(t) for t in (x, y, g, eps, v)), more(lengths))
    for t in list(range(8)) + [W - 1]:
        one = slice(t % 8, t % 8 + 1)
        want, wl, err, lerr = formula(x[one], yv[one], g[one], eps[one], vv[one], lengths[one])
        good = torch.arange(n) != (1 if t % 8 == 6 else -1)
        assert ((out[t] - want[0]).abs() <= err[0])[good].all() and ((lse[t] - wl[0]).abs() <= lerr[0])[good].all(), t
    assert torch.isnan(out[6, 1]).all() and torch.isnan(lse[6, 1])


@pytest.mark.gpu
@pytest.mark.parametrize("n,many", [(5, False), (300, True)])
@pytest.mark.parametrize("d", [64, 512, 1024])
def test_exponents_whose_products_one_dimension_carries(B, n, many, d):
    # A large first product and small ones of one sign beside it, each cut off where the sum begins: (0.67 d + 8) U of what an exponent is made of
    # (d to a whole 32): 17 2^-25 + 2^-23 < 2^-20.6 for each 16 dimensions in bf16, 33 2^-25 + 2^-23 < 2^-19.8 for each 32 in 8 bits, a fifteenth
    # more for the query's three parts; 8 for the terms in fp32
    import torch
    W, m = 7, 1500
    if staged(B, W, n, m, d) != many:
        assert d > 512
        return
    x = torch.full((W, n, d), 255 / 128 * 2.0 ** -9).bfloat16()
    x[:, :, 0] = 1.0
    y = torch.full((W, m, d), 1.875 * 2.0 ** -8)
    y[:, :, ::128] = 1.0
    y[:, :, 128::128] = 2.0 ** -1
    g = torch.full((W, m), -float("inf"), dtype=torch.float64)
    g[:, 1234] = 0.0
    eps = torch.full((W,), 1e-3)
    out, lse, yv, _ = run(B, x, y, g, eps)
    yv = yv[:, 1234].double()
    z = -(x.double() - yv[:, None]).square().sum(2) / eps.double()[:, None]
    made_of = (x.double().square().sum(2) + yv.square().sum(1)[:, None]) / eps.double()[:, None]
    assert ((lse - z).abs() <= (0.67 * (-(-d // 32) * 32) + 8) * U * made_of).all(), float(((lse - z).abs() / made_of / U).max())
    assert ((out - yv[:, None]).abs() <= 2.0 ** -8 * yv[:, None].abs()).all()


def weighted(x, y, g, eps, v):
    """Images, logarithms of the sums, and bounds, in float64: those of the formula beside the other tests, but for exponents, (0.67 d + 8) U, and for what two
    e4m3 numbers leave of a weight.  Weights w times their values' powers of two 2^e are taken against the largest such product of the tile, 2^M: the second number
    is off by up to 2^-14 of w 2^(e + 8 - M), the part of the image so by 448 2^-22 2^M, at most 2^-21 of the largest product of a weight and a value (which is above
    224 2^e).  Powers of a tile that differ by at most 2^3 are taken against the largest of them instead: 2^-18.  Never more than the product itself."""
    import torch
    masked = g == -float("inf")
    x, y, v, g = x.double(), torch.where(masked[:, :, None], 0.0, y.double()), torch.where(masked[:, :, None], 0.0, v.double()), torch.where(masked, 0.0, g)
    d = x.shape[2]
    e = eps.double()[:, None, None]
    made_of = (x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :] + g.abs()[:, None, :]) / e
    z = (g[:, None, :] - (x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :] - 2 * x @ y.transpose(1, 2))) / e
    z = torch.where(masked[:, None, :], -float("inf"), z)
    lse = torch.logsumexp(z, 2)
    p = torch.exp(z - lse[:, :, None])
    out = p @ v
    size = (0.67 * (-(-d // 32) * 32) + 8) * U * made_of
    mean = (p * size).sum(2)
    err = (p * (size + mean[:, :, None] + 2.0 ** -8 + 2.0 ** -16)) @ v.abs() + 2.0 ** -8 * out.abs()
    for j in range(0, v.shape[1], 128):
        for k in range(0, v.shape[2], 128):
            most = p[:, :, j:j + 128] * v[:, j:j + 128, k:k + 128].abs().amax(2)[:, None, :]
            err[:, :, k:k + 128] += torch.minimum(2.0 ** -18 * most.amax(2, keepdim=True), most).sum(2, keepdim=True)
    return out, lse, err, mean + 2.0 ** -16 + 2 * U * lse.abs()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 5, 12, 16, 31, 300])
@pytest.mark.parametrize("d,dv", [(64, 0), (64, 40), (256, 256), (512, 0), (128, 512), (1024, 0), (1024, 1024), (100, 700)])
def test_values_far_larger_than_those_that_have_the_weights(B, n, d, dv):
    import torch
    W, m = 4, 400
    x, y, g, eps, v = inputs(W, n, m, d, dv, seed=3)
    own = v is not None
    v = v if own else y
    # targets without weight whose values (their own, or far away points) are 2^20 times the others'; one of a tile, all but one, every other; blocks apart
    far = torch.zeros(W, m, dtype=torch.bool)
    far[0, ::128], far[1, :], far[2, ::2] = True, True, True
    far[1, 5::128] = False
    far[3, 200:] = True
    v = torch.where(far[:, :, None], v * 2.0 ** 20, v)
    if not own:
        y = v
    else:
        v[3, :, 128:] *= 2.0 ** 9
    g = torch.where(far, -1e3 * eps.double()[:, None], g)
    if not own:                                                       # (points that far away need no potential to have no weight)
        g[far] = 0.0
    y8, v8 = B.cloud8_pack(y.cuda()), B.cloud8_pack(v.cuda()) if own else None
    out, lse = B.cloud8_map(x.cuda(), y8, g.cuda(), eps.cuda(), v8, lse=True)
    yv = y8.values().cpu()
    want, wl, err, lerr = weighted(x, yv, g, eps, v8.values().cpu() if own else yv)
    out, lse = out.cpu().double(), lse.cpu().double()
    assert ((out - want).abs() <= err).all(), float(((out - want).abs() / err).max())
    assert ((lse - wl).abs() <= lerr).all()
    # weights of every size beside values of every size
    gen = torch.Generator().manual_seed(9)
    if own:
        power = torch.randint(-30, 31, (W, m, 1), generator=gen).double()
        v = (torch.randn(W, m, dv, generator=gen) * torch.exp2(power)).float()
        g = 0.1 * torch.randn(W, m, generator=gen, dtype=torch.float64) - eps.double()[:, None] * power[:, :, 0] * 0.7
        v8 = B.cloud8_pack(v.cuda())
        out, lse = B.cloud8_map(x.cuda(), y8, g.cuda(), eps.cuda(), v8, lse=True)
        want, wl, err, lerr = weighted(x, yv, g, eps, v8.values().cpu())
        assert ((out.cpu().double() - want).abs() <= err).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,m", [(3, 300), (20, 300), (300, 300), (300, 3000)])
def test_values_that_are_zeros_masked_or_not_finite_beside_large_ones(B, n, m):
    import torch
    W, dv = 5, 200
    x, y, g, eps, v = inputs(W, n, m, 64, dv, seed=4)
    v[:, ::3] *= 2.0 ** 25
    v[0, 1::3] = 0.0                                                  # (a target's values may be nothing)
    v[1] = 0.0
    v[2, :128] = 0.0
    g[3, ::3] = -float("inf")
    g[3, 128:256] = -float("inf")                                     # a tile without targets between others
    v[4, 131] = float("nan")
    v8, y8 = B.cloud8_pack(v.cuda()), B.cloud8_pack(y.cuda())
    out, lse = (t.cpu().double() for t in B.cloud8_map(x.cuda(), y8, g.cuda(), eps.cuda(), v8, lse=True))
    assert torch.isnan(out[4]).all() and not torch.isnan(lse).any()
    want, wl, err, lerr = weighted(x[:4], y8.values().cpu()[:4], g[:4], eps[:4], v8.values().cpu()[:4])
    assert ((out[:4] - want).abs() <= err).all() and ((lse[:4] - wl).abs() <= lerr).all()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 1, 6000, 512, 512), (32, 12, 4000, 128, 64), (5, 3, 9000, 1024, 1024), (6, 9, 3000, 600, 700), (40, 16, 900, 200, 256), (30, 8, 2500, 64, 1)])
def test_calls_over_values_far_apart_one_after_the_other(B, shape):
    # tiles of values alike between tiles of others: roles of a block that get out of step would show as images that differ
    import torch
    W, n, m, d, dv = shape
    x, y, g, eps, v = inputs(*shape)
    apart = (torch.arange(m) // 128 % 3 != 1) & (torch.arange(m) % 5 == 0)
    v[:, apart] *= 2.0 ** 12
    y8, v8 = B.cloud8_pack(y.cuda()), B.cloud8_pack(v.cuda())
    x, g, eps = x.cuda(), g.cuda(), eps.cuda()
    want, wl = B.cloud8_map(x, y8, g, eps, v8, lse=True)
    outs = [B.cloud8_map(x, y8, g, eps, v8, lse=True) for _ in range(40)]
    assert not torch.isnan(want).any()
    for out, lse in outs:
        assert torch.equal(out, want) and torch.equal(lse, wl)
    one = slice(1, 3)
    exact, wl2, err, lerr = weighted(x[one].cpu(), y8.values()[one].cpu(), g[one].cpu(), eps[one].cpu(), v8.values()[one].cpu())
    assert ((want[one].cpu().double() - exact).abs() <= err).all() and ((wl[one].cpu().double() - wl2).abs() <= lerr).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [30, 160])
def test_images_are_the_solved_plan_applied_to_the_values(B, n):
    # sum_j pi_ij v_j over sum_j pi_ij, which apply_plan forms in float64 and rounds to fp32
    import torch
    W, m, d, dv = 3, 200, 64, 15
    x, y, _, _, v = inputs(W, n, m, d, dv, seed=6)
    x8, y8, v8 = (B.cloud8_pack(t.float().cuda()) for t in (x, y, v))
    a, b, eps = torch.full((W, n), 1 / n).cuda(), torch.full((W, m), 1 / m).cuda(), torch.full((W,), 0.1).cuda()
    sb = B.SinkhornBatch(x8, y8, a, b, eps, 1e-4)
    sb.drain()
    g = sb.potentials(f64=True)[1]
    applied = sb.apply_plan(torch.cat((v8.values(), torch.ones(W, m, 1, device="cuda")), 2)).cpu().double()
    sb.close()
    out = B.cloud8_map(x8.values(torch.bfloat16), y8, g, eps, v8).cpu().double()
    want = applied[:, :, :dv] / applied[:, :, dv:]
    exact, _, err, _ = weighted(x8.values().cpu(), y8.values().cpu(), g.cpu(), eps.cpu(), v8.values().cpu())
    assert ((exact - want).abs() <= 2.0 ** -20 * v8.values().cpu().double().abs().amax(1, keepdim=True)).all()
    assert ((out - want).abs() <= err + 2.0 ** -20 * v8.values().cpu().double().abs().amax(1, keepdim=True)).all()
