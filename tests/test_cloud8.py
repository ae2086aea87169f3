"""Clouds held in 8-bit floating point: rounding, layout, values, norms, products and refusals.

The reference is the definition of the header in float64, by comparison with every value of e4m3.  Codes, scales and values are exact
numbers; norms and products have the bounds derived beside them."""
import ctypes

import numpy as np
import pytest

# the non-negative values of e4m3, by code
GRID = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def nearest_code(a):
    hi = np.clip(np.searchsorted(GRID, a, side="left"), 1, 126)
    lo = hi - 1
    dl, dh = a - GRID[lo], GRID[hi] - a
    return np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))


def reference(x):
    """codes [r, 32 ceil(d/32)], scale bytes [r, 4 ceil(d/512)], values [r, d] and norms [r] of x [r, d] (float64 holding the input's values)."""
    r, d = x.shape
    nb = -(-d // 128)
    v = np.zeros((r, nb, 128))
    v.reshape(r, -1)[:, :d] = x
    bad = ~np.isfinite(v).all((1, 2))
    v[bad] = 0.0
    top = np.abs(v).max(2)
    e = np.full(top.shape, -100)
    for step in range(-100, 121):
        e = np.where(top > 448.0 * 2.0 ** (step - 1), step, e)
    e = np.maximum(e, -100)
    scale = 2.0 ** e.astype(np.float64)
    q = np.abs(v) / scale[:, :, None]
    q = np.where((e == 120)[:, :, None], np.minimum(q, 240.0), q)
    code = nearest_code(q)
    values = (GRID[code] * scale[:, :, None] * np.where(np.signbit(v), -1.0, 1.0)).reshape(r, -1)
    code = (code + 128 * np.signbit(v)).reshape(r, -1)[:, :-(-d // 32) * 32].astype(np.uint8)
    byte = np.zeros((r, -(-d // 512) * 4), np.uint8)
    byte[:, :nb] = e + 127
    norms = (values ** 2).sum(1)
    if bad.any():
        code[bad], values[bad], norms[bad] = 0, np.nan, np.nan
        byte[bad, :nb] = 255
    return code, byte, values[:, :d], norms


def split(buf, rows, d):
    pad = lambda b: -(-b // 256) * 256
    cb, sb = -(-d // 32) * 32, -(-d // 512) * 4
    at = pad(rows * cb)
    end = at + pad(rows * sb)
    return (buf[:rows * cb].reshape(rows, cb), buf[at:at + rows * sb].reshape(rows, sb), buf[end:end + 4 * rows].copy().view(np.float32),
            end + pad(4 * rows))


def check(B, x, values=None):
    """x: a CPU tensor [W, npts, d]."""
    W, npts, d = x.shape
    got = B.cloud8_pack(x.cuda(), values=values)
    cloud, vals = got if values is not None else (got, None)
    code, byte, want, norms = reference(x.double().numpy().reshape(W * npts, d))
    gcode, gbyte, gnorm, total = split(cloud.buffer.cpu().numpy(), W * npts, d)
    assert total == cloud.buffer.numel()
    np.testing.assert_array_equal(gbyte, byte)
    np.testing.assert_array_equal(gcode, code)
    # sixteen squares are added in fp32, all else in float64, and the result is rounded: 17 half steps
    assert np.array_equal(np.isnan(gnorm), np.isnan(norms))
    big = norms > 3.4e38
    assert np.isinf(gnorm[big]).all()
    ok = np.isfinite(norms) & ~big
    assert (np.abs(gnorm[ok] - norms[ok]) <= 17 * 2.0 ** -24 * norms[ok] + 2.0 ** -149).all()
    want = want.reshape(W, npts, d)
    np.testing.assert_array_equal(cloud.values().cpu().double().numpy(), want)
    if vals is not None:
        assert vals.dtype == values
        np.testing.assert_array_equal(vals.cpu().double().numpy(), want)
        np.testing.assert_array_equal(cloud.values(values).cpu().double().numpy(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [1, 15, 16, 17, 33, 64, 100, 127, 128, 129, 200, 256, 333, 512, 513, 1000, 1024])
def test_codes_scales_and_values_of_every_depth(B, d):
    import torch
    gen = torch.Generator().manual_seed(d)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(3, 37, d, generator=gen) * torch.exp(3.0 * torch.randn(3, 37, 1, generator=gen))
        check(B, x.to(dtype), values=torch.bfloat16 if d % 2 else torch.float32)
        check(B, (x * torch.exp(2.0 * torch.randn(3, 37, d, generator=gen))).to(dtype))


@pytest.mark.gpu
def test_halves_borders_of_scales_zeros_and_the_ends_of_the_range(B):
    import torch
    rows = []
    for e in (-100, -3, 0, 119):
        s = np.float32(2.0) ** e
        ties = ((GRID[:-1] + GRID[1:]) / 2).astype(np.float32) * s          # halfway between neighbours, and one step off it
        for part in (ties, np.nextafter(ties, np.float32(0)), -np.nextafter(ties, np.float32(np.inf))):
            row = np.zeros(128, np.float32)
            row[:126] = part
            row[127] = 448 * s                                          # the block's largest: the scale is s
            rows.append(row)
        for top in (448.0, np.nextafter(np.float32(448.0), np.float32(900.0)), 224.0, np.nextafter(np.float32(224.0), np.float32(900.0))):
            row = np.zeros(128, np.float32)
            row[3], row[5] = np.float32(top) * s, -1.0 * s
            rows.append(row)
    for v in (0.0, -0.0, 1e-45, 3.4028234e38, 1.1754944e-38, 2.0 ** -100, 2.0 ** -110, 3e38):
        row = np.zeros(128, np.float32)
        row[64], row[65] = v, -v
        rows.append(row)
    x = torch.from_numpy(np.stack(rows))
    check(B, x[None], values=torch.float32)
    check(B, x[None].repeat(1, 1, 2), values=torch.bfloat16)


@pytest.mark.gpu
def test_points_that_are_not_finite_and_tensors_that_are_not_aligned(B):
    import torch
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(2, 9, 300, generator=gen)
    x[0, 3, 299], x[1, 0, 0], x[1, 8, 130] = float("nan"), float("inf"), -float("inf")
    check(B, x, values=torch.bfloat16)
    # a view that starts 4 bytes past a 16-byte boundary
    flat = torch.randn(1 + 5 * 128, generator=gen).cuda()
    v = flat[1:].view(1, 5, 128)
    assert v.data_ptr() % 16
    for one, two in zip(*(split(B.cloud8_pack(w).buffer.cpu().numpy(), 5, 128)[:3] for w in (v, v.clone()))):     # (padding is not written)
        np.testing.assert_array_equal(one, two)
    # strides: a transposed view is packed as its values
    t = torch.randn(2, 64, 7, generator=gen).cuda().transpose(1, 2)
    assert torch.equal(B.cloud8_pack(t).values(), B.cloud8_pack(t.contiguous()).values())


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (2, 3, 5, 7), (1, 128, 128, 32), (3, 129, 130, 96), (2, 100, 257, 128), (1, 300, 64, 200),
                                   (2, 127, 4, 333), (1, 256, 131, 512), (2, 65, 140, 520), (1, 40, 33, 1024)])
def test_products(B, shape):
    import torch
    W, n, m, d = shape
    gen = torch.Generator().manual_seed(n * m + d)
    spread = lambda k: torch.exp(2.0 * torch.randn(W, k, 1, generator=gen)) * torch.exp(1.5 * torch.randn(W, k, d, generator=gen))
    x8, y8 = (B.cloud8_pack((torch.randn(W, k, d, generator=gen) * spread(k)).cuda()) for k in (n, m))
    got = B.cloud8_dots(x8, y8).cpu().double()
    x, y = x8.values().cpu().double(), y8.values().cpu().double()
    want, weight = x @ y.transpose(1, 2), x.abs() @ y.abs().transpose(1, 2)
    # an instruction adds 32 products to the sum so far and cuts each of the 33 at 2^-25 of the largest, the result at 24 bits: at most
    # 33 2^-25 + 2^-23 < 2^-19.8 of the sum of magnitudes for each of ceil(d/32) instructions
    assert ((got - want).abs() <= -(-d // 32) * 2.0 ** -19.8 * weight + 1e-44).all()


@pytest.mark.gpu
def test_products_with_scales_far_from_one_and_points_that_are_nan(B):
    import torch
    gen = torch.Generator().manual_seed(11)
    x = torch.randn(1, 140, 256, generator=gen) * 2.0 ** torch.randint(-90, 60, (1, 140, 1), generator=gen)
    y = torch.randn(1, 70, 256, generator=gen) * 2.0 ** torch.randint(-50, 55, (1, 70, 1), generator=gen)
    x[:, :, 128:] *= 2.0 ** -12                                           # blocks of a point with scales of their own
    y[:, :, :128] *= 2.0 ** -9
    x[0, 5, 7] = float("nan")
    y[0, 69, 0] = float("inf")
    x8, y8 = B.cloud8_pack(x.cuda()), B.cloud8_pack(y.cuda())
    got = B.cloud8_dots(x8, y8).cpu().double()
    xv, yv = x8.values().cpu().double(), y8.values().cpu().double()
    want, weight = xv @ yv.transpose(1, 2), xv.abs() @ yv.abs().transpose(1, 2)
    assert torch.isnan(got[0, 5]).all() and torch.isnan(got[0, :, 69]).all()
    fine = ~torch.isnan(want) & (want.abs() < 3e38)
    assert not torch.isnan(got[fine]).any()
    assert ((got - want).abs()[fine] <= 8 * 2.0 ** -19.8 * weight[fine] + 2.0 ** -126).all()


@pytest.mark.gpu
def test_products_into_a_given_tensor_that_is_not_aligned_on_another_stream_and_in_a_graph(B):
    import torch
    gen = torch.Generator().manual_seed(2)
    x8, y8 = B.cloud8_pack(torch.randn(2, 70, 160, generator=gen).cuda()), B.cloud8_pack(torch.randn(2, 44, 160, generator=gen).cuda())
    want = B.cloud8_dots(x8, y8)
    room = torch.full((2 * 70 * 44 + 2,), 7.0, device="cuda")
    out = room[1:-1].view(2, 70, 44)
    B.cloud8_dots(x8, y8, out=out)
    assert torch.equal(out, want) and float(room[0]) == 7.0 and float(room[-1]) == 7.0
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = B.cloud8_dots(x8, y8)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(other, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.cloud8_dots(x8, y8, out=out)
    out.zero_()
    g.replay()
    assert torch.equal(out, want)


@pytest.mark.gpu
def test_a_batch_of_8_bit_clouds_is_the_batch_of_their_values(B):
    import torch
    gen = torch.Generator().manual_seed(3)
    W, n, m, d = 4, 96, 80, 128
    unit = lambda v: (v / v.norm(dim=2, keepdim=True)).cuda()
    x8, y8 = B.cloud8_pack(unit(torch.randn(W, n, d, generator=gen))), B.cloud8_pack(unit(torch.randn(W, m, d, generator=gen)))
    a, b, eps = torch.full((W, n), 1.0 / n).cuda(), torch.full((W, m), 1.0 / m).cuda(), torch.full((W,), 0.1).cuda()
    outs = []
    u = torch.rand(W, n, 3, generator=gen).cuda()
    for x, y in ((x8, y8), (x8.values(torch.bfloat16), y8.values(torch.bfloat16))):
        sb = B.SinkhornBatch(x, y, a, b, eps, 1e-3)
        sb.drain()
        outs.append((*sb.potentials(f64=True), sb.draw_plan(u)))
        sb.close()
    for one, two in zip(*outs):
        assert torch.equal(one, two)
    g = outs[0][1]
    assert torch.equal(B.plan_draw(x8, y8, g, eps, u), B.plan_draw(x8.values(torch.bfloat16), y8.values(torch.bfloat16), g, eps, u))
    with pytest.raises(ValueError):
        B.SinkhornBatch(x8, y8.values(), a, b, eps, 1e-3)


def test_sizes_and_refusals_without_a_gpu(B):
    import torch
    lib = B.lib
    for shape in ((1, 1, 1), (3, 37, 200), (64, 1024, 512), (2, 9, 513), (5, 100, 1024)):
        W, n, d = shape
        pad = lambda b: -(-b // 256) * 256
        want = pad(W * n * (-(-d // 32) * 32)) + pad(W * n * (-(-d // 512) * 4)) + pad(4 * W * n)
        assert lib.sinkhorn_cloud8_bytes(*shape) == B._cloud8_bytes(*shape) == want
    for shape in ((0, 4, 4), (1, 0, 4), (1, 4, 0), (1, 4, 1025), (65536, 65536, 4)):
        assert lib.sinkhorn_cloud8_bytes(*shape) == 0 == B._cloud8_bytes(*shape)
    one = ctypes.c_void_p(256)
    assert lib.sinkhorn_cloud8_pack(None, 0, 1, 4, 4, one, None, 0, None) == 1
    assert lib.sinkhorn_cloud8_pack(one, 0, 1, 4, 1025, one, None, 0, None) == 2
    assert lib.sinkhorn_cloud8_pack(one, 2, 1, 4, 4, one, None, 0, None) == 3
    assert lib.sinkhorn_cloud8_pack(one, 0, 1, 4, 4, one, one, 5, None) == 3
    assert lib.sinkhorn_cloud8_pack(one, 0, 1, 4, 4, ctypes.c_void_p(128), None, 0, None) == 4
    assert lib.sinkhorn_cloud8_pack(ctypes.c_void_p(258), 0, 1, 4, 4, one, None, 0, None) == 4
    assert lib.sinkhorn_cloud8_unpack(one, 1, 4, 4, None, 0, None) == 1
    assert lib.sinkhorn_cloud8_unpack(one, 1, 4, 0, one, 0, None) == 2
    assert lib.sinkhorn_cloud8_unpack(one, 1, 4, 4, one, 3, None) == 3
    assert lib.sinkhorn_cloud8_unpack(one, 1, 4, 4, ctypes.c_void_p(257), 0, None) == 4
    assert lib.sinkhorn_cloud8_dots(one, None, 1, 4, 4, 4, one, None) == 1
    assert lib.sinkhorn_cloud8_dots(one, one, 1, 4, 0, 4, one, None) == 2
    assert lib.sinkhorn_cloud8_dots(one, ctypes.c_void_p(264), 1, 4, 4, 4, one, None) == 4
    assert lib.sinkhorn_cloud8_dots(one, one, 1, 4, 4, 4, ctypes.c_void_p(258), None) == 4
    assert b"4-byte" in lib.sinkhorn_operator_last_error()
    with pytest.raises(ValueError):
        B.cloud8_pack(torch.zeros(1, 4, 4))
    with pytest.raises(ValueError):
        B.Cloud8(torch.zeros(4096, dtype=torch.uint8), 1, 4, 4)
    with pytest.raises(ValueError):
        B.cloud8_dots(torch.zeros(1, 4, 4), torch.zeros(1, 4, 4))


@pytest.mark.gpu
def test_refusals_on_the_device(B):
    import torch
    v = torch.zeros(2, 4, 40, device="cuda")
    for bad in (v[0], v.half(), torch.zeros(2, 4, 1025, device="cuda"), torch.zeros(2, 0, 40, device="cuda")):
        with pytest.raises(ValueError):
            B.cloud8_pack(bad)
    with pytest.raises(ValueError):
        B.cloud8_pack(v, values=torch.float16)
    c = B.cloud8_pack(v)
    for other in (B.cloud8_pack(v[:1]), B.cloud8_pack(v[:, :, :8]), B.cloud4_pack(v)):
        with pytest.raises(ValueError):
            B.cloud8_dots(c, other)
    with pytest.raises(ValueError):
        B.cloud8_dots(c, c, out=torch.zeros(2, 4, 5, device="cuda"))
    with pytest.raises(ValueError):
        B.Cloud8(c.buffer[:-1], 2, 4, 40)
    with pytest.raises(ValueError):
        c.values(torch.float16)
