"""Images under the entropic map of clouds held in 8 bits, against the formula in float64 on the values that the clouds stand for."""
import ctypes

import pytest

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def formula(x, y, g, eps, v, lengths):
    """Images, logarithms of the sums, and bounds of their errors, in float64.

    An exponent is off by (d/32 + 8) U of what it is made of; a weight by that (twice: itself and the sum), by what its rounding to eight
    bits loses, 2^-9 (half a step of bf16's is 2^-9 of the upper end of a binade, 2^-8 of the lower: 2^-8), and by 2^-16 for sums and
    exponentials in fp32; the result is rounded to bf16, 2^-8 of itself.

    Where weights are two e4m3 numbers, a weight w <= 1 (of the tile's largest) times its value's power of two 2^e is 256 w 2^(e - E), E the largest e of
    the 128 targets of the tile.  The second number has steps of 2^-9, a sixteenth each, so what is left of it is off by up to 2^-14 whatever its size,
    and by no more than itself.  Times the code (448 at most) and 2^E / 256 that is 448 2^-22 2^E; the tile's largest value of these 128 dimensions is above
    224 2^E: 2^-21 of it, and no more than the weight times the value; both times the tile's largest weight of all.  (Blocks' powers of two end at
    2^-100; the values here are far above.)"""
    import torch
    x, y, v = x.double(), y.double(), v.double()
    W, n, d = x.shape
    m = y.shape[1]
    g = torch.zeros(W, m, dtype=torch.float64) if g is None else g
    masked = g == -float("inf")
    if lengths is not None:
        masked = masked | (torch.arange(m)[None, :] >= lengths.long().clamp(0, m)[:, None])
    y, v = (torch.where(masked[:, :, None], 0.0, t) for t in (y, v))
    gz = torch.where(masked, 0.0, g)
    e = eps.double()[:, None, None]
    z = (gz[:, None, :] - (x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :] - 2 * x @ y.transpose(1, 2))) / e
    z = torch.where(masked[:, None, :], -float("inf"), z)
    lse = torch.logsumexp(z, 2)
    p = torch.where(lse[:, :, None] == -float("inf"), 0.0, torch.exp(z - lse[:, :, None]))
    out = p @ v
    size = (d / 32 + 8) * U * (x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :] + gz.abs()[:, None, :]) / e
    size = torch.where(masked[:, None, :], 0.0, size)
    mean = (p * size).sum(2)
    err = (p * (size + mean[:, :, None] + 2.0 ** -8 + 2.0 ** -16)) @ v.abs() + 2.0 ** -8 * out.abs()
    for j in range(0, m, 128):
        pt = p[:, :, j:j + 128]
        for k in range(0, v.shape[2], 128):
            most = v[:, j:j + 128, k:k + 128].abs().amax(2)                                    # of each target
            cut = 2.0 ** -21 * most.amax(1)[:, None, None] * pt.amax(2, keepdim=True)
            err[:, :, k:k + 128] += torch.minimum(cut, pt * most[:, None, :]).sum(2, keepdim=True)
    lerr = mean + 2.0 ** -16 + 2 * U * lse.abs() + size.amax(2) * 2.0 ** -3
    return out, lse, err, lerr


def run(B, x, y, g, eps, v=None, lengths=None):
    import torch
    cu = lambda t: None if t is None else t.cuda()
    y8, v8 = B.cloud8_pack(y.cuda()), None if v is None else B.cloud8_pack(v.cuda())
    out, lse = B.cloud8_map(x.cuda(), y8, cu(g), cu(eps), v8, lengths=cu(lengths), lse=True)
    assert out.dtype == torch.bfloat16 and lse.dtype == torch.float32
    yv = y8.values().cpu()
    return out.cpu().double(), lse.cpu().double(), yv, yv if v is None else v8.values().cpu()


def check(B, x, y, g, eps, v=None, lengths=None):
    import torch
    out, lse, yv, vv = run(B, x, y, g, eps, v, lengths)
    want, wl, err, lerr = formula(x, yv, g, eps, vv, lengths)
    assert not torch.isnan(out).any()
    assert ((out - want).abs() <= err).all(), float(((out - want).abs() / err.clamp(min=1e-300)).max())
    empty = wl == -float("inf")
    assert torch.equal(lse == -float("inf"), empty) and not out[empty].any()
    assert ((lse - wl).abs()[~empty] <= lerr[~empty]).all()


def inputs(W, n, m, d, dv=0, seed=0, eps=0.1, spread=1.0):
    import torch
    gen = torch.Generator().manual_seed(seed + 1000 * n + m + d)
    unit = lambda *s: (lambda t: t / t.norm(dim=2, keepdim=True))(torch.randn(*s, generator=gen))
    x, y = unit(W, n, d).bfloat16(), unit(W, m, d)
    g = 0.1 * torch.randn(W, m, generator=gen, dtype=torch.float64)
    v = spread * torch.randn(W, m, dv, generator=gen) if dv else None
    return x, y, g, torch.full((W,), eps) * (1 + 0.3 * torch.rand(W, generator=gen)), v


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 16, 17, 40, 63, 64, 65, 127, 128, 129, 200])
def test_numbers_of_queries(B, n):
    check(B, *inputs(2, n, 300, 128))
    check(B, *inputs(3, n, 130, 96, dv=40))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 100, 300])
@pytest.mark.parametrize("m", [1, 2, 15, 63, 64, 65, 127, 128, 129, 191, 257, 1000, 5000])
def test_numbers_of_targets(B, n, m):
    check(B, *inputs(2, n, m, 64))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 12, 150])
@pytest.mark.parametrize("d,dv", [(1, 0), (3, 0), (16, 5), (31, 0), (33, 129), (64, 256), (100, 1), (128, 300), (129, 0), (200, 96), (256, 0), (257, 512),
                                  (384, 384), (400, 0), (500, 640), (512, 0), (512, 64), (513, 0), (700, 1024), (1024, 0), (1024, 1024)])
def test_depths_of_bank_and_values(B, n, d, dv):
    check(B, *inputs(2, n, 150, d, dv))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 10, 140])
def test_lengths_and_masks(B, n):
    import torch
    for m in (70, 300):
        for own in (0, 24):
            x, y, g, eps, v = inputs(7, n, m, 96, own)
            lengths = torch.tensor([0, 1, 63, 64, 65, m, m + 50], dtype=torch.int32)
            check(B, x, y, g, eps, v, lengths)
            check(B, x, y, None, eps, v, torch.tensor([-5, 2, m - 1, 10, 20, 30, 2 ** 31 - 1], dtype=torch.int32))
            g[0] = -float("inf")                                  # nothing left
            g[1, 1:] = -float("inf")                              # one target
            g[2, ::2] = -float("inf")
            g[3, :m - 1] = -float("inf")
            g[4, 64:] = -float("inf")                             # a tile, and more, without any
            check(B, x, y, g, eps, v)
            # what masked targets hold does not matter
            for j, bad in ((0, float("nan")), (2, float("inf")), (6, -3e38)):
                y[2, j] = bad
                if v is not None:
                    v[2, j + 2] = bad
            check(B, x, y, g, eps, v)
            y[5, m - 3:] = float("nan")
            if v is not None:
                v[5, m - 3:] = float("inf")
            check(B, x, y, g, eps, v, torch.tensor([m, m, m, m, m, m - 3, m], dtype=torch.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2, 12, 140])
def test_what_is_not_finite_stays_in_its_row_or_lane(B, n):
    import torch
    x, y, g, eps, v = inputs(7, n, 100, 64, 32)
    x[0, 1, 5] = float("nan")
    x[1, 0, 63] = float("inf")
    y[2, 50, 3] = float("nan")
    v[3, 99, 0] = float("inf")
    g[4, 7] = float("nan")
    g[5, 9] = float("inf")
    eps[6] = -1.0
    out, lse, yv, vv = run(B, x, y, g, eps, v)
    assert torch.isnan(out[0, 1]).all() and torch.isnan(lse[0, 1]) and torch.isnan(out[1, 0]).all() and torch.isnan(lse[1, 0])
    for t in (2, 3, 4, 5, 6):
        assert torch.isnan(out[t]).all(), t
        assert torch.isnan(lse[t]).all() == (t != 3)
    want, wl, err, lerr = formula(x, yv, g, eps, vv, None)
    for t, keep in ((0, [0] + list(range(2, n))), (1, list(range(1, n)))):
        assert ((out[t] - want[t]).abs() <= err[t])[keep].all() and ((lse[t] - wl[t]).abs() <= lerr[t])[keep].all()
    assert ((lse[3] - wl[3]).abs() <= lerr[3]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [3, 130])
def test_scales_far_apart_sharp_rows_and_far_reference_points(B, n):
    import torch
    # values and points whose powers of two differ, up to the tile's documented reach; large clouds; rows that one target takes
    x, y, g, eps, v = inputs(3, n, 400, 300, 200, seed=1)
    gen = torch.Generator().manual_seed(5)
    v = v * 2.0 ** torch.randint(-9, 10, (3, 400, 1), generator=gen)
    v[:, :, 128:] *= 2.0 ** 20
    check(B, x, y, g, eps, v)
    check(B, (x.float() * 64).bfloat16(), y * 64, g * 4096, eps * 4096, v)
    check(B, (x.float() * 2.0 ** -30).bfloat16(), y * 2.0 ** -30, g * 2.0 ** -60, eps * 2.0 ** -60, v * 2.0 ** -40)
    check(B, x, y, g, eps * 0.02, v)
    # exponents that grow all along the bank, and that fall
    ramp = torch.linspace(0, 40, 400, dtype=torch.float64).expand(3, 400).clone()
    check(B, x, y, ramp, eps * 10, v)
    check(B, x, y, ramp.flip(1), eps * 10, v)


@pytest.mark.gpu
def test_the_most_queries_of_the_deepest_points(B):
    # more blocks of queries and values than a grid's second dimension takes
    import torch
    x, y, g, eps, v = inputs(1, 5, 3, 1024, 1024)
    y8, v8 = B.cloud8_pack(y.cuda()), B.cloud8_pack(v.cuda())
    want, wl = B.cloud8_map(x.cuda(), y8, g.cuda(), eps.cuda(), v8, lse=True)
    n = 262143
    many = x.cuda()[:, torch.arange(n, device="cuda") % 5]
    out, lse = B.cloud8_map(many, y8, g.cuda(), eps.cuda(), v8, lse=True)
    for i in range(5):
        assert torch.equal(out[0, i::5], want[0, i].expand(out[0, i::5].shape)) and (lse[0, i::5] == wl[0, i]).all()


@pytest.mark.gpu
def test_long_banks_are_split_and_every_part_counts(B):
    import torch
    for n, m, d, dv in ((1, 40000, 64, 0), (5, 20011, 128, 32), (20, 9000, 40, 0), (130, 12001, 64, 16)):
        x, y, g, eps, v = inputs(1, n, m, d, dv, eps=0.3)
        check(B, x, y, g, eps, v)
        check(B, x, y, None, eps, v, torch.tensor([m - 70], dtype=torch.int32))
        check(B, x, y, None, eps, v, torch.tensor([3], dtype=torch.int32))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [4, 200])
def test_results_do_not_change_from_call_to_call_stream_graph_and_offset(B, n):
    import torch
    x, y, g, eps, v = (t.cuda() for t in inputs(3, n, 700, 130, 60))
    y8, v8 = B.cloud8_pack(y), B.cloud8_pack(v)
    want, wl = B.cloud8_map(x, y8, g, eps, v8, lse=True)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a = B.cloud8_map(x, y8, g, eps, v8, lse=True)
        b = B.cloud8_map(x, y8, g, eps, v8)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(a[0], want) and torch.equal(a[1], wl) and torch.equal(b, want)
    # queries and images that start off a 16-byte boundary
    room = torch.zeros(x.numel() + 3, dtype=torch.bfloat16, device="cuda")
    xo = room[3:].view_as(x)
    xo.copy_(x)
    space = torch.full((want.numel() + 2,), 5.0, dtype=torch.bfloat16, device="cuda")
    out = space[1:-1].view_as(want)
    assert B.cloud8_map(xo, y8, g, eps, v8, out=out).data_ptr() == out.data_ptr()
    assert torch.equal(out, want) and float(space[0]) == 5.0 == float(space[-1])
    # strides
    assert torch.equal(B.cloud8_map(x.transpose(1, 2).contiguous().transpose(1, 2), y8, g, eps, v8), want)
    graph = torch.cuda.CUDAGraph()
    static = torch.zeros_like(x)
    with torch.cuda.graph(graph):
        got = B.cloud8_map(static, y8, g, eps, v8)
    static.copy_(x)
    graph.replay()
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(8, 1, 6000, 512, 0), (32, 12, 4000, 128, 64), (40, 16, 900, 300, 0), (5, 3, 9000, 1024, 0), (6, 9, 3000, 600, 700), (3, 700, 1500, 512, 0), (9, 100, 2000, 96, 40)])
def test_calls_one_after_the_other_without_a_wait(B, shape):
    # roles of a block that get out of step would show as images that differ, or as NaN where a wait ran out
    import torch
    W, n, m, d, dv = shape
    x, y, g, eps, v = inputs(*shape)
    y8, v8 = B.cloud8_pack(y.cuda()), None if v is None else B.cloud8_pack(v.cuda())
    x, g, eps = x.cuda(), g.cuda(), eps.cuda()
    want, wl = B.cloud8_map(x, y8, g, eps, v8, lse=True)
    outs = [B.cloud8_map(x, y8, g, eps, v8, lse=True) for _ in range(40)]
    assert not torch.isnan(want).any()
    for out, lse in outs:
        assert torch.equal(out, want) and torch.equal(lse, wl)


@pytest.mark.gpu
def test_images_of_a_solved_plan(B):
    # 8-bit clouds, solved, then the images of the source points against the plan applied to the targets
    import torch
    gen = torch.Generator().manual_seed(6)
    W, n, m, d = 3, 160, 200, 64
    unit = lambda t: (t / t.norm(dim=2, keepdim=True)).cuda()
    x8, y8 = B.cloud8_pack(unit(torch.randn(W, n, d, generator=gen))), B.cloud8_pack(unit(torch.randn(W, m, d, generator=gen)))
    a, b, eps = torch.full((W, n), 1 / n).cuda(), torch.full((W, m), 1 / m).cuda(), torch.full((W,), 0.1).cuda()
    sb = B.SinkhornBatch(x8, y8, a, b, eps, 1e-4)
    sb.drain()
    f, g = sb.potentials(f64=True)
    sb.close()
    x = x8.values(torch.bfloat16)
    out, lse = B.cloud8_map(x, y8, g, eps, lse=True)
    want, wl, err, lerr = formula(x.cpu(), y8.values().cpu(), g.cpu(), eps.cpu(), y8.values().cpu(), None)
    assert ((out.cpu().double() - want).abs() <= err).all()
    # the source's potential: f_i = -eps lse_i - eps log n once the rows' residual is zero; here it is at most 1e-4 in all, relative to a row's 1/n
    assert ((f.cpu() / eps.cpu().double()[:, None] + lse.cpu().double() + torch.log(torch.tensor(float(n)))).abs() <= 2 * n * 1e-4 + lerr).all()


def test_sizes_and_refusals_without_a_gpu(B):
    import torch
    one, ws = ctypes.c_void_p(256), B.lib.sinkhorn_cloud8_map_workspace_bytes
    assert ws(1, 1, 100, 64, 0) >= 256 and ws(1, 1, 100000, 64, 0) > ws(1, 1, 100, 64, 0) and ws(2, 4, 300, 64, 32) % 256 == 0
    for bad in ((0, 1, 1, 1, 0), (1, 0, 1, 1, 0), (1, 1, 0, 1, 0), (1, 1, 1, 0, 0), (1, 1, 1, 1025, 0), (1, 1, 1, 4, 1025), (65536, 1, 1, 1, 0),
                (1, 262144, 1, 1, 0), (1, 1, 262144, 1, 0), (1, 1, 1, 1, -1)):
        assert ws(*bad) == 0, bad

    def call(x=one, y=one, g=None, eps=one, v=None, lengths=None, W=1, n=1, m=8, d=16, dv=0, out=one, lse=None, work=one, size=1 << 20):
        return B.lib.sinkhorn_cloud8_map(x, y, g, eps, v, lengths, W, n, m, d, dv, out, lse, work, size, None)
    p = ctypes.c_void_p
    for bad in (dict(x=None), dict(y=None), dict(eps=None), dict(out=None), dict(work=None)):
        assert call(**bad) == 1, bad
    for bad in (dict(W=0), dict(n=0), dict(m=0), dict(d=0), dict(d=1025), dict(v=one, dv=0), dict(v=one, dv=1025), dict(W=65535, m=262143)):
        assert call(**bad) == 2, bad
    for bad in (dict(y=p(128)), dict(v=p(128), dv=4), dict(work=p(16)), dict(x=p(257)), dict(out=p(257)), dict(g=p(260)), dict(eps=p(258)), dict(lse=p(258)),
                dict(lengths=p(258)), dict(size=0)):
        assert call(**bad) == 4, bad
    # images over the queries, or over some of them
    for bad in (dict(), dict(x=p(1024), out=p(1024 + 2 * 16 - 2)), dict(x=p(1024), out=p(1024 - 2 * 16 + 2)), dict(n=4, x=p(1024), v=one, dv=8, out=p(1024 - 2 * 4 * 8 + 2))):
        assert call(**bad) == 3, bad
    with pytest.raises(ValueError):
        B.cloud8_map(torch.zeros(1, 1, 16, dtype=torch.bfloat16), torch.zeros(1, 8, 16), None, torch.ones(1))


@pytest.mark.gpu
def test_refusals_on_the_device(B):
    import torch
    x, y, g, eps, v = (t.cuda() for t in inputs(2, 3, 20, 32, 8))
    y8, v8 = B.cloud8_pack(y), B.cloud8_pack(v)
    for args in ((x.float(), y8, g, eps), (x[0], y8, g, eps), (x.cpu(), y8, g, eps), (x, y, g, eps), (x, y8, g.float(), eps), (x, y8, g[:, :5], eps),
                 (x, y8, g, eps.double()), (x, y8, g, None), (x[:1], y8, g[:1], eps[:1]), (x[:, :, :16], y8, g, eps), (x, y8, g, eps, v),
                 (x, y8, g, eps, B.cloud8_pack(v[:, :5])), (x, y8, g.cpu(), eps)):
        with pytest.raises(ValueError):
            B.cloud8_map(*args)
    for kw in (dict(lengths=torch.ones(2, device="cuda")), dict(lengths=torch.ones(3, dtype=torch.int32, device="cuda")),
               dict(out=torch.zeros(2, 3, 8, device="cuda")), dict(out=torch.zeros(2, 3, 9, dtype=torch.bfloat16, device="cuda"))):
        with pytest.raises(ValueError):
            B.cloud8_map(x, y8, g, eps, v8, **kw)
    with pytest.raises(B.SkbError):
        B.cloud8_map(x, y8, g, eps, out=x)
    with pytest.raises(B.SkbError):
        B.cloud8_map(torch.zeros(1, 0, 32, dtype=torch.bfloat16, device="cuda"), B.cloud8_pack(y[:1]), g[:1], eps[:1])
