"""Images under the entropic map where least is to spare: rows without targets beside what is not finite, potentials of the lowest finite values, long banks of
values of one sign, products that one dimension carries, values far larger than those that have the weights."""
import pytest

from test_cloud8_map import B, formula, inputs, run  # noqa: F401  (B is the fixture)


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
