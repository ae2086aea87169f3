"""Clouds in microscaled 4-bit floating point: rounding, layout, values and refusals.

The reference is the definition of the header in float64, by comparison with every value of the grid.  Codes, scales and
values are exact numbers, so nothing here has a tolerance."""
import numpy as np
import pytest

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def floor_log2(v):
    return np.frexp(v)[1] - 1


def nearest_code(a):
    """Index of the nearest grid value, halves to the even index."""
    a = np.minimum(a, 6.0)
    hi = np.clip(np.searchsorted(GRID, a, side="left"), 1, 7)
    lo = hi - 1
    dl, dh = a - GRID[lo], GRID[hi] - a
    return np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))


def e4m3_round(q):
    """Nearest e4m3 value of q in [0, 448], halves to even."""
    step = 2.0 ** (np.maximum(np.where(q > 0, floor_log2(np.where(q > 0, q, 1.0)), -6), -6) - 3)
    return np.rint(q / step) * step


def e4m3_byte(v):
    e = np.maximum(np.where(v > 0, floor_log2(np.where(v > 0, v, 1.0)), -6), -6)
    frac = v / 2.0 ** (e - 3)                                    # 0 .. 15 eighths
    return np.where(frac >= 8, (e + 7) * 8 + frac - 8, frac).astype(np.uint8)


def reference(x, fmt):
    """codes [r, 32 ceil(d/32)], scale bytes [r, words], points [r], values [r, d] of x [r, d] (float64 holding the input's values)."""
    r, d = x.shape
    size = 32 if fmt == "mx4" else 16
    nb = -(-d // 32) * (32 // size)
    v = np.zeros((r, nb * size))
    v[:, :d] = x
    bad = ~np.isfinite(v).all(1)
    v[bad] = 0.0
    block = np.abs(v.reshape(r, nb, size))
    top = block.max(2)
    point = np.ones(r)
    if fmt == "mx4":
        e = np.where(top > 0, floor_log2(np.where(top > 0, top, 1.0)) - 2, -127)
        e = np.maximum(e, -127)
        scale, byte = 2.0 ** e.astype(np.float64), (e + 127).astype(np.uint8)
    else:
        whole = top.max(1)
        pe = np.where(whole > 0, np.maximum(floor_log2(np.where(whole > 0, whole, 1.0)) - 10, -126), 0)
        point = 2.0 ** pe.astype(np.float64)
        s = e4m3_round(top / 6.0 / point[:, None])
        s = np.where((point == 2.0 ** 117)[:, None], np.minimum(s, 320.0), s)
        scale, byte = s * point[:, None], e4m3_byte(s)
    q = np.divide(block, scale[:, :, None], out=np.zeros_like(block), where=scale[:, :, None] > 0)
    code = nearest_code(q)
    values = (GRID[code] * scale[:, :, None]).reshape(r, -1) * np.where(v < 0, -1.0, 1.0)
    code = (code.reshape(r, -1) + 8 * np.signbit(v)).astype(np.uint8)
    if bad.any():
        code[bad], values[bad] = 0, np.nan
        byte[bad] = 255 if fmt == "mx4" else 127
    words = np.zeros((r, -(-nb // 4) * 4), np.uint8)
    words[:, :nb] = byte
    return code, words, point, values[:, :d]


def split(buf, rows, d, fmt):
    pad = lambda b: -(-b // 256) * 256
    cb, nb = -(-d // 32) * 16, -(-d // 32) * (1 if fmt == "mx4" else 2)
    sb = -(-nb // 4) * 4
    codes = buf[:rows * cb].reshape(rows, cb)
    code = np.stack((codes & 15, codes >> 4), 2).reshape(rows, -1)
    at = pad(rows * cb)
    scales = buf[at:at + rows * sb].reshape(rows, sb)
    at += pad(rows * sb)
    points = buf[at:at + 4 * rows].copy().view(np.float32) if fmt == "nv4" else np.ones(rows, np.float32)
    at += pad(4 * rows) if fmt == "nv4" else 0
    return code, scales, points, at


def check(B, x, fmt, values=None):
    """x: a CPU tensor [W, npts, d]."""
    import torch
    W, npts, d = x.shape
    v = x.cuda()
    got = B.cloud4_pack(v, fmt, values=values)
    cloud, vals = got if values is not None else (got, None)
    code, words, point, want = reference(x.double().numpy().reshape(W * npts, d), fmt)
    gcode, gwords, gpoint, total = split(cloud.buffer.cpu().numpy(), W * npts, d, fmt)
    assert total == cloud.buffer.numel()
    np.testing.assert_array_equal(gwords, words)
    np.testing.assert_array_equal(gpoint, point.astype(np.float32))
    np.testing.assert_array_equal(gcode, code)
    want = want.reshape(W, npts, d)
    np.testing.assert_array_equal(cloud.values().cpu().double().numpy(), want)
    if vals is not None:
        assert vals.dtype == values
        np.testing.assert_array_equal(vals.cpu().double().numpy(), want)
        np.testing.assert_array_equal(cloud.values(values).cpu().double().numpy(), want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
@pytest.mark.parametrize("d", [1, 2, 15, 16, 17, 32, 33, 48, 64, 100, 128, 129, 200, 256, 333, 512, 520, 640, 1000, 1024])
def test_codes_scales_and_values_of_every_depth(B, fmt, d):
    import torch
    gen = torch.Generator().manual_seed(d)
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(3, 37, d, generator=gen) * torch.exp(3.0 * torch.randn(3, 37, 1, generator=gen))
        check(B, x.to(dtype), fmt, values=torch.bfloat16 if d % 2 else torch.float32)
        check(B, (x * torch.exp(2.0 * torch.randn(3, 37, d, generator=gen))).to(dtype), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_halves_go_to_the_even_code_and_their_neighbours_do_not(B, fmt):
    # values at scale * (halfway between two grid values), one step of fp32 below and above, for every e4m3 mantissa
    import torch
    rows = []
    for eighths in range(8, 16):
        s = np.float32(eighths / 8.0) if fmt == "nv4" else np.float32(1.0)
        ties = np.float32([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]) * s
        block = np.concatenate([np.nextafter(ties, np.float32(0)), ties, np.nextafter(ties, np.float32(9)), [6 * s]])
        for part in (block[:15], block[7:]):
            row = np.zeros(32, np.float32)
            row[:len(part)] = part
            row[15] = 6 * s                                      # the block's largest: the scale is s
            row[16:] = -row[:16]
            rows.append(row)
    check(B, torch.from_numpy(np.stack(rows))[None], fmt, values=torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_scales_at_their_borders(B, fmt):
    # e4m3 scales exactly between two values, blocks far below their point's largest value, zeros, the ends of fp32
    import torch
    rng = np.random.default_rng(5)
    x = np.zeros((96, 64), np.float32)
    for i in range(64):
        q = np.float32((17 + 2 * (i % 8)) / 16.0) * np.float32(2.0 ** -(i // 8))      # halfway between two e4m3 values of its binade
        x[i, :16] = 6 * 8.0 / 8 * 32                             # fixes the point's power of two
        x[i, 16:32] = 6 * q
        x[i, 40] = 2.0 ** -(i // 2) * rng.uniform(1, 2)
    x[64:72] = rng.standard_normal((8, 64)) * 2.0 ** -120
    x[72:76] = rng.standard_normal((4, 64)) * 2.0 ** -140
    x[76, 3] = 2.0 ** -149
    x[77] = 3.4028235e38
    x[78, ::2] = -3.4028235e38
    x[79] = -0.0
    x[80:] = rng.standard_normal((16, 64)) * 10.0 ** rng.integers(-30, 30, (16, 1))
    check(B, torch.from_numpy(x)[None], fmt, values=torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_point_with_a_value_that_is_not_finite_is_nan_as_a_whole(B, fmt, bad):
    import torch
    for d in (24, 200, 600):
        x = torch.randn(2, 9, d, generator=torch.Generator().manual_seed(1))
        x[0, 3, d - 1] = bad
        x[1, 8, 0] = bad
        check(B, x, fmt, values=torch.float32)
        check(B, x.bfloat16(), fmt)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_unaligned_and_strided_inputs_and_another_stream(B, fmt):
    import torch
    base = torch.randn(4 * 50 * 64 + 1, generator=torch.Generator().manual_seed(2)).cuda()
    x = base[1:].view(4, 50, 64)                                 # contiguous, 4-byte aligned only
    want = B.cloud4_pack(x.clone(), fmt)
    np.testing.assert_array_equal(split(B.cloud4_pack(x, fmt).buffer.cpu().numpy(), 200, 64, fmt)[0],
                                  split(want.buffer.cpu().numpy(), 200, 64, fmt)[0])
    t = torch.randn(4, 64, 50, generator=torch.Generator().manual_seed(3)).cuda().transpose(1, 2)   # strided view
    a, b = B.cloud4_pack(t, fmt), B.cloud4_pack(t.contiguous(), fmt)
    assert torch.equal(a.values(), b.values())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = B.cloud4_pack(x, fmt, values=torch.float32)[1]
    side.synchronize()
    assert torch.equal(c, want.values())


@pytest.mark.gpu
def test_packing_is_captured_and_replayed_on_new_values(B):
    import torch
    x = torch.randn(2, 100, 96).cuda()
    B.cloud4_pack(x, "nv4", values=torch.float32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cloud, vals = B.cloud4_pack(x, "nv4", values=torch.float32)
    for _ in range(2):
        x.copy_(torch.randn(2, 100, 96))
        graph.replay()
        assert torch.equal(vals, B.cloud4_pack(x.clone(), "nv4").values())
        assert torch.equal(vals, cloud.values())


def test_refusals_of_pack_and_unpack(B):
    import ctypes
    import torch
    L, one = B.lib, ctypes.c_void_p(4096)
    assert L.sinkhorn_cloud4_bytes(1, 1, 1, 2) == 512 and L.sinkhorn_cloud4_bytes(1, 1, 1, 3) == 768
    assert L.sinkhorn_cloud4_bytes(64, 1024, 512, 2) == 64 * 1024 * (256 + 16)
    for shape in ((1, 1, 1), (3, 37, 100), (2, 5, 64), (7, 333, 1000), (1, 1, 1024)):
        for name, fmt in B.FORMATS.items():
            assert B._cloud4_bytes(*shape, name) == L.sinkhorn_cloud4_bytes(*shape, fmt) > 0
    for bad in ((0, 1, 1, 2), (1, 0, 1, 2), (1, 1, 0, 2), (1, 1, 1025, 2), (1, 1, 8, 1), (1, 1, 8, 4), (-1, 1, 8, 2), (1 << 16, 1 << 16, 8, 2)):
        assert L.sinkhorn_cloud4_bytes(*bad) == 0
        assert L.sinkhorn_cloud4_pack(one, 0, *bad, one, None, 0, None) == 2 and L.sinkhorn_operator_last_error()
        assert L.sinkhorn_cloud4_unpack(one, *bad, one, 0, None) == 2
    assert L.sinkhorn_cloud4_pack(None, 0, 1, 4, 8, 2, one, None, 0, None) == 1
    assert L.sinkhorn_cloud4_pack(one, 0, 1, 4, 8, 2, None, None, 0, None) == 1
    assert L.sinkhorn_cloud4_unpack(one, 1, 4, 8, 2, None, 0, None) == 1
    assert L.sinkhorn_cloud4_pack(one, 2, 1, 4, 8, 2, one, None, 0, None) == 3
    assert L.sinkhorn_cloud4_pack(one, 0, 1, 4, 8, 2, one, one, 5, None) == 3
    assert L.sinkhorn_cloud4_pack(one, 0, 1, 4, 8, 2, ctypes.c_void_p(4096 + 16), None, 0, None) == 4
    assert b"aligned" in L.sinkhorn_operator_last_error()
    with pytest.raises(ValueError):
        B.cloud4_pack(torch.zeros(2, 3, 4))                      # not on a GPU
    with pytest.raises(ValueError):
        B.Cloud4(torch.zeros(1024, dtype=torch.uint8), 1, 1, 8, "mx4")
    with pytest.raises(ValueError):
        B.Cloud4(torch.zeros(1024, dtype=torch.uint8), 1, 1, 2000, "mx4")


# ---- products

def exact_dots(x, y):
    """Float64 products of two Cloud4, and the sum of their terms' magnitudes."""
    import torch
    a, b = x.values().double(), y.values().double().transpose(1, 2)
    return torch.bmm(a, b), torch.bmm(a.abs(), b.abs())


def check_dots(B, x4, y4, out):
    # A matrix instruction adds 64 exact products to an fp32 accumulator.  Each is allowed two units in the last place of the
    # largest sum that can occur, the sum of the magnitudes; the powers of two of nv4 change nothing.
    import torch
    want, size = exact_dots(x4, y4)
    steps = -(-x4.d // 64)
    err = (out.double() - want).abs()
    assert bool((err <= steps * 2.0 ** -22 * size + 1e-300).all()), float((err / (size + 1e-300)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (1, 128, 128, 64), (1, 128, 128, 256), (2, 128, 256, 512), (3, 37, 45, 20), (1, 129, 257, 96), (2, 300, 130, 200),
                                   (5, 64, 33, 333), (2, 200, 100, 640), (1, 260, 516, 1024), (7, 1, 300, 48), (7, 300, 1, 48), (40, 130, 129, 160)])
def test_products_of_every_shape(B, fmt, shape):
    import torch
    W, n, m, d = shape
    gen = torch.Generator().manual_seed(sum(shape))
    x = (torch.randn(W, n, d, generator=gen) * torch.exp(torch.randn(W, n, 1, generator=gen))).cuda()
    y = (torch.randn(W, m, d, generator=gen) * torch.exp(torch.randn(W, m, d, generator=gen))).cuda()
    x4, y4 = B.cloud4_pack(x, fmt), B.cloud4_pack(y, fmt)
    # a result behind guards: rows past the last are left alone
    room = torch.full((W * n * m + 256,), -7.0, device="cuda")
    for at in (64, 65):                                          # 16-byte aligned, and not
        room.fill_(-7.0)
        out = room[at:at + W * n * m].view(W, n, m)
        B.cloud4_dots(x4, y4, out=out)
        check_dots(B, x4, y4, out)
        assert bool((room[:at] == -7.0).all()) and bool((room[at + W * n * m:] == -7.0).all())


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_products_are_exact_where_sums_are_small_integers(B, fmt):
    # every value a grid value with scale one or two: all sums are exact in fp32, so a scale or a code in the wrong place shows
    import torch
    gen = torch.Generator().manual_seed(11)
    grid = torch.tensor(list(GRID) + list(-GRID), dtype=torch.float32)
    for d in (64, 128, 192, 256, 500, 1024):
        x, y = grid[torch.randint(16, (2, 150, d), generator=gen)], grid[torch.randint(16, (2, 140, d), generator=gen)]
        x[:, :, ::16] = 6.0
        y[:, :, ::16] = 6.0
        x[:, :, : d // 2] *= 2.0
        y[:, 70:, :] *= 0.25
        x4, y4 = B.cloud4_pack(x.cuda(), fmt), B.cloud4_pack(y.cuda(), fmt)
        want, _ = exact_dots(x4, y4)
        assert torch.equal(B.cloud4_dots(x4, y4).double(), want), d


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_a_nan_point_gives_nan_in_its_row_and_column_only(B, fmt):
    import torch
    x, y = torch.randn(2, 140, 200).cuda(), torch.randn(2, 133, 200).cuda()
    x[1, 130, 199] = float("inf")
    y[0, 132, 0] = float("nan")
    x[0, 7] = 0.0
    out = B.cloud4_dots(B.cloud4_pack(x, fmt), B.cloud4_pack(y, fmt))
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[1, 130] = True
    bad[0, :, 132] = True
    assert torch.equal(torch.isnan(out), bad)
    assert bool((out[0, 7, :132] == 0).all())


@pytest.mark.gpu
def test_products_repeat_bit_for_bit_and_replay_from_a_graph(B):
    import torch
    x4, y4 = B.cloud4_pack(torch.randn(30, 200, 320).cuda(), "nv4"), B.cloud4_pack(torch.randn(30, 260, 320).cuda(), "nv4")
    first = B.cloud4_dots(x4, y4)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = B.cloud4_dots(x4, y4)                            # at the same time as the next
    again = B.cloud4_dots(x4, y4)
    torch.cuda.synchronize()
    assert torch.equal(first, again) and torch.equal(first, other)
    out = torch.empty_like(first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.cloud4_dots(x4, y4, out=out)
    y4.buffer.copy_(B.cloud4_pack(torch.randn(30, 260, 320).cuda(), "nv4").buffer)
    graph.replay()
    assert torch.equal(out, B.cloud4_dots(x4, y4)) and not torch.equal(out, first)


def test_refusals_of_products(B):
    import ctypes
    L, one = B.lib, ctypes.c_void_p(4096)
    assert L.sinkhorn_cloud4_dots(None, one, 1, 4, 4, 8, 2, one, None) == 1
    assert L.sinkhorn_cloud4_dots(one, None, 1, 4, 4, 8, 2, one, None) == 1
    assert L.sinkhorn_cloud4_dots(one, one, 1, 4, 4, 8, 2, None, None) == 1
    for bad in ((0, 4, 4, 8, 2), (1, 0, 4, 8, 2), (1, 4, 0, 8, 2), (1, 4, 4, 0, 3), (1, 4, 4, 1025, 3), (1, 4, 4, 8, 0), (1, 4, 4, 8, 1)):
        assert L.sinkhorn_cloud4_dots(one, one, *bad, one, None) == 2
    assert L.sinkhorn_cloud4_dots(ctypes.c_void_p(4096 + 16), one, 1, 4, 4, 8, 2, one, None) == 4
    assert L.sinkhorn_cloud4_dots(one, one, 1, 4, 4, 8, 2, ctypes.c_void_p(4098), None) == 4
    with pytest.raises(ValueError):
        B.cloud4_dots(None, None)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
@pytest.mark.parametrize("n", [33, 129, 150, 200, 230, 1000])
def test_last_rows_of_few_and_many_tiles(B, fmt, n):
    # tiles of which some warps have no rows, next to whole ones, many to a block: results are stored before their room is
    # written again.  Values are multiples of 1/4 and sums small: products are exact, and compared as a whole
    import torch
    gen = torch.Generator().manual_seed(n)
    W, m, d = 3, 20000, 64
    grid = torch.tensor(list(GRID) + list(-GRID), dtype=torch.float32)
    x, y = grid[torch.randint(16, (W, n, d), generator=gen)], grid[torch.randint(16, (W, m, d), generator=gen)]
    x[:, :, ::16] = 6.0
    y[:, :, ::16] = 6.0
    x4, y4 = B.cloud4_pack(x.cuda(), fmt), B.cloud4_pack(y.cuda(), fmt)
    want = (x4.values().double() @ y4.values().double().transpose(1, 2)).float()
    for _ in range(6):
        out = torch.full((W, n, m), float("nan"), device="cuda")
        B.cloud4_dots(x4, y4, out=out)
        assert torch.equal(out, want)


@pytest.mark.gpu
@pytest.mark.parametrize("fmt", ["mx4", "nv4"])
def test_offsets_past_32_bits(B, fmt):
    # 2.3e9 values, and 2.2e9 products; the last points alone give the same
    import torch
    x = torch.zeros(9, 250000, 1024, dtype=torch.bfloat16, device="cuda")
    x[8, -300:] = torch.randn(300, 1024, generator=torch.Generator().manual_seed(1)).cuda().bfloat16()
    big, values = B.cloud4_pack(x, fmt, values=torch.bfloat16)
    want = B.cloud4_pack(x[8:, -300:], fmt)
    assert torch.equal(values[8:, -300:], want.values(torch.bfloat16)) and not bool(values[:8].any())
    del values
    assert torch.equal(big.values(torch.bfloat16)[8:, -300:], want.values(torch.bfloat16))
    del big, x
    gen = torch.Generator().manual_seed(2)
    a, b = torch.randn(2, 33000, 64, generator=gen).cuda(), torch.randn(2, 33000, 64, generator=gen).cuda()
    out = B.cloud4_dots(B.cloud4_pack(a, fmt), B.cloud4_pack(b, fmt))
    part = B.cloud4_dots(B.cloud4_pack(a[1:, -200:], fmt), B.cloud4_pack(b[1:], fmt))
    assert torch.equal(out[1:, -200:], part)
    assert torch.equal(out[:1, 31000:31100], B.cloud4_dots(B.cloud4_pack(a[:1, 31000:31100], fmt), B.cloud4_pack(b[:1], fmt)))


@pytest.mark.gpu
@pytest.mark.parametrize("m", [64, 100, 131])
def test_nv4_products_of_large_and_small_points(B, m):
    # points of 1e-38 to 1e38: the sum, times one point's power of two, may be past fp32's range where the product is not
    import torch
    W, n, d = 4, 150, 64
    gen = torch.Generator().manual_seed(m)
    e = torch.linspace(-37, 37, n)[None, :, None].expand(W, n, 1)
    f = torch.linspace(-37, 37, m)[None, :, None].expand(W, m, 1)
    x, y = torch.randn(W, n, d, generator=gen).double() * 10.0 ** e.double(), torch.randn(W, m, d, generator=gen).double() * 10.0 ** f.double()
    x4, y4 = B.cloud4_pack(x.float().cuda(), "nv4"), B.cloud4_pack(y.float().cuda(), "nv4")
    want = torch.bmm(x4.values().double(), y4.values().double().transpose(1, 2))
    size = torch.bmm(x4.values().double().abs(), y4.values().double().abs().transpose(1, 2))
    out = B.cloud4_dots(x4, y4)
    # one step of 64: two units in the last place of the magnitudes' sum, and fp32's smallest number
    bound = 2.0 ** -22 * size + 2.0 ** -149
    inside = want.abs() + bound < 3.4e38
    assert bool(torch.isfinite(out[inside]).all()) and bool(((out.double() - want).abs() <= bound)[inside].all())
    big = want.abs() - bound > 3.5e38
    assert bool(torch.isinf(out[big]).all()) and bool((torch.sign(out) == torch.sign(want))[big].all())
    assert bool(inside.any()) and bool(big.any())
