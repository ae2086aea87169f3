"""The loss of scores against named entries where its arithmetic has least to spare: stretches of masked scores far below zero, logits far from zero,
sums next to one; gradients in the place of tensors that a graph or another row still needs."""
import ctypes

import numpy as np
import pytest

from test_plan_loss import B, U, check, compare, inputs, run  # noqa: F401  (B is the fixture)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,m", [(9, 20), (9, 400), (9, 1000), (9, 3000), (9, 8000), (5, 9000), (5, 16000), (5, 30000), (5, 60000), (5, 131000), (5, 262143),
                                    (5003, 60), (5003, 100), (5003, 250), (20480, 120), (20480, 500), (300, 40000)])
def test_stretches_of_masked_scores_beside_scores_far_below_zero(B, rows, m, dtype):
    # a thread that sees nothing but minus infinity has weights of 0, whatever the row's maximum: rows of every way through the kernels
    import torch
    scores, index, t, weight = inputs(min(rows, 211), m, min(m // 3, 4), getattr(torch, dtype), m)
    live = m // 3
    index %= live
    many = torch.arange(rows) % scores.shape[0]
    for shift, T in ((-300.0, 1.0), (-6.0, 0.05), (250.0, 1.0)):
        s = ((scores.float() * 3 * T).clamp(-10 * T, 10 * T) + shift).to(scores.dtype)
        s[:, live:] = -float("inf")
        s[1], s[1, m - live:] = -float("inf"), s[0, :live]                            # the live ones at the end
        at = index.clone()
        at[1] += m - live
        loss, grad = B.plan_loss(s[many].cuda(), at[many].cuda(), t[many].cuda(), temperature=T, weight=weight[many].cuda(), grad=True)
        assert not torch.isnan(loss).any() and not torch.isnan(grad).any()
        assert not grad[many != 1][:, live:].any() and not grad[many == 1][:, :m - live].any()
        for first in {0, (rows - 1) // 211 * 211}:
            n = min(211, rows - first)
            compare(loss[first:first + n], grad[first:first + n], s[:n], at[:n], t[:n], T, weight[:n])
        # a NaN beside them is its row's alone, and a row of nothing but masked scores is NaN
        s[2, m - 1], s[3] = float("nan"), -float("inf")
        loss, grad = (v[:5].cpu() for v in B.plan_loss(s[many].cuda(), at[many].cuda(), t[many].cuda(), temperature=T, grad=True))
        bad = torch.tensor([False, False, True, True, False][:loss.shape[0]])
        assert torch.equal(torch.isnan(loss), bad) and torch.equal(torch.isnan(grad).all(1), bad) and torch.equal(torch.isnan(grad).any(1), bad)


@pytest.mark.gpu
@pytest.mark.parametrize("m,k", [(30, 5), (300, 40), (3000, 200), (20000, 33), (40000, 64)])
def test_a_teachers_logits_may_all_be_shifted_and_be_of_any_finite_size(B, m, k):
    import torch
    for rows in (12, 300):
        scores, index, t, weight = inputs(rows, m, k, torch.float32, k)
        lowest, most = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
        # the softmax of differences: a shift that all logits share is nothing to it, however small the temperature
        check(B, scores * 0.01, index, (t * 0.01 + 1000.0), 0.01, weight)
        check(B, scores * 0.01, index, (t * 0.01 - 5e4), 0.01, weight)
        check(B, scores, index, t * 1e30, 3.0, weight)
        t[0] = lowest                                                 # (a mask, where it leaves nothing else: all alike)
        t[1], t[1, 3] = lowest, 1.0
        t[2] = most
        t[3, ::2] = lowest
        t[4, 1:] = -float("inf")
        t[5] = -float("inf")                                          # nothing
        check(B, scores, index, t, 0.25, weight)
        check(B, scores, index, t, 1.0, weight)


@pytest.mark.gpu
def test_losses_of_confident_rows(B):
    # log(1 + e), e = exp(-x): the exponential is off by 2 x U (its argument, twice) and 4 U, the sum by U of itself, the logarithm by 2 U of itself
    import torch
    x = torch.cat((torch.linspace(0.01, 16, 4001), torch.linspace(1e-4, 0.5, 777)))
    want = np.log1p(np.exp(-x.double().numpy()))
    e = np.exp(-x.double().numpy())
    for m in (2, 77, 700, 70000):
        n = len(x) if m < 1000 else 40
        scores = torch.full((n, m), -float("inf"))
        at = torch.arange(n) % (m - 1)
        scores[torch.arange(n), at] = 3.0
        scores[torch.arange(n), at + 1] = 3.0 - x[:n]
        gap = (3.0 - scores[torch.arange(n), at + 1]).double().numpy()                # (exact in fp32)
        want, e = np.log1p(np.exp(-gap)), np.exp(-gap)
        loss = B.plan_loss(scores.cuda(), at.int()[:, None].cuda()).cpu().double().numpy()
        assert (np.abs(loss - want) <= U * (1 + 2 * want + e / (1 + e) * (2 * gap + 4))).all()


@pytest.mark.gpu
def test_a_gradient_in_the_place_of_what_a_graph_saved_is_seen_by_it(B):
    import torch
    gen = torch.Generator().manual_seed(3)
    index = torch.randint(0, 50, (20, 3), generator=gen, dtype=torch.int32).cuda()
    start = torch.randn(20, 50, generator=gen).cuda()
    for act in (torch.tanh, torch.exp, torch.sigmoid, lambda h: torch.log_softmax(h, 1)):
        h = start.clone().requires_grad_()
        scores = act(h)
        _, grad = B.plan_loss(scores, index, grad=scores)
        with pytest.raises(RuntimeError):
            scores.backward(grad)                                     # (the operation saved its result, which is gone)
    h = start.clone().requires_grad_()
    kept = torch.tanh(h)
    B.plan_loss(start, index, grad=kept.detach())                     # (by way of another view of it)
    with pytest.raises(RuntimeError):
        kept.sum().backward()
    # a product does not need its result: the step goes on
    for place in (False, True):
        lin = start[:, :50].clone()[:8].requires_grad_()
        scores = start[:, :8] @ lin
        _, grad = B.plan_loss(scores, index, grad=scores if place else True)
        scores.backward(grad)
        if place:
            assert torch.equal(lin.grad, want)
        want = lin.grad
    # other tensors that are written where they are given
    x8, y8 = B.cloud8_pack(torch.randn(1, 4, 32, generator=gen).cuda()), B.cloud8_pack(torch.randn(1, 5, 32, generator=gen).cuda())
    dots, images, grad = torch.zeros(1, 4, 5).cuda(), torch.zeros(1, 4, 32, dtype=torch.bfloat16).cuda(), torch.zeros(20, 50).cuda()
    x4, y4 = B.cloud4_pack(torch.randn(1, 4, 32, generator=gen).cuda(), "mx4"), B.cloud4_pack(torch.randn(1, 5, 32, generator=gen).cuda(), "mx4")
    for t, call in ((dots, lambda: B.cloud8_dots(x8, y8, out=dots)), (images, lambda: B.cloud8_map(x8.values(torch.bfloat16), y8, None, torch.ones(1).cuda(), out=images)),
                    (grad, lambda: B.plan_loss(start, index, grad=grad)), (dots, lambda: B.cloud4_dots(x4, y4, out=dots))):
        before = t._version
        call()
        assert t._version > before
    with torch.inference_mode():
        s = start.clone()
        B.plan_loss(s, index, grad=s)


def overlapping(call):
    """Calls whose gradient overlaps the scores without being in their place: (scores, grad, rows, m, ld, ldg) in elements."""
    for grad, rows, m, ld, ldg in ((1, 4, 8, 8, 8), (-1, 4, 8, 8, 8), (8, 4, 8, 8, 8), (-8, 4, 8, 8, 8), (31, 4, 8, 8, 8), (-31, 4, 8, 8, 8), (8, 4, 8, 15, 15),
                                   (-7, 4, 8, 16, 16), (12, 4, 8, 19, 19), (8, 4, 8, 16, 24), (24, 4, 8, 16, 8), (17, 4, 8, 16, 16), (7, 1, 8, 8, 8), (4, 2, 1, 4, 4)):
        call(grad, rows, m, ld, ldg)


def test_gradients_that_overlap_the_scores_are_refused(B):
    p, base = ctypes.c_void_p, 1 << 16

    def call(grad, rows, m, ld, ldg):
        for dtype, size in ((0, 4), (1, 2)):
            assert B.lib.sinkhorn_plan_loss(p(base), dtype, rows, m, ld, p(256), None, 1, 1.0, None, p(256), p(base + size * grad), ldg, None) == 3, (grad, ld, ldg)
    overlapping(call)


@pytest.mark.gpu
def test_gradients_between_the_scores_rows_and_beside_them(B):
    import torch
    for dtype in (torch.float32, torch.bfloat16):
        scores, index, t, weight = (v.cuda() for v in inputs(6, 40, 3, dtype, 1))
        for ld, at, grad in ((80, 0, 40), (80, 40, 0), (91, 3, 47), (40, 0, 240), (40, 240, 0), (41, 0, 250)):
            room = torch.full((2 * 6 * ld + 16,), 7.0, dtype=dtype, device="cuda")
            s, g = (room.as_strided((6, 40), (ld, 1), first) for first in (at, grad))
            s.copy_(scores)
            loss, out = B.plan_loss(s, index, t, weight=weight, grad=g)
            assert out.data_ptr() == g.data_ptr() and torch.equal(s, scores)
            compare(loss, g, scores, index, t, 1.0, weight)
            rest = torch.ones_like(room, dtype=torch.bool)
            for first in (at, grad):
                rest.as_strided((6, 40), (ld, 1), first).fill_(False)
            assert (room[rest] == 7).all()
        room = torch.zeros(400, dtype=dtype, device="cuda")

        def call(grad, rows, m, ld, ldg):
            s, g = room.as_strided((rows, m), (ld, 1), 100), room.as_strided((rows, m), (ldg, 1), 100 + grad)
            with pytest.raises(B.SkbError):
                B.plan_loss(s, torch.zeros(rows, 1, dtype=torch.int32, device="cuda"), grad=g)
        overlapping(call)


@pytest.mark.gpu
def test_a_gradient_that_is_asked_for_by_any_true_value_is_given(B):
    import torch
    scores, index, t, weight = (v.cuda() for v in inputs(6, 40, 3, torch.float32, 1))
    want = B.plan_loss(scores, index, t, weight=weight, grad=True)
    for yes in (1, np.True_):
        loss, grad = B.plan_loss(scores, index, t, weight=weight, grad=yes)
        assert torch.equal(loss, want[0]) and torch.equal(grad, want[1])
    for no in (0, None, np.False_):
        assert torch.equal(B.plan_loss(scores, index, t, weight=weight, grad=no), want[0])
