"""Operators over 8-bit clouds as a program uses them together: embeddings are packed, coupled, partners are drawn, scores are taught the draws, points are
mapped; on two streams at once, and captured into a graph that is replayed on other embeddings."""
import pytest

from test_cloud8_map import formula as map_formula
from test_plan_loss import compare as compare_loss


@pytest.fixture(scope="module")
def B():
    from paper_2607_24741_b200 import build
    build.build()
    from paper_2607_24741_b200 import binding
    return binding


def embeddings(W, n, m, d, seed):
    import torch
    gen = torch.Generator().manual_seed(seed)
    unit = lambda k: (lambda t: t / t.norm(dim=2, keepdim=True))(torch.randn(W, k, d, generator=gen)).cuda()
    return unit(n), unit(m), torch.rand(W, n, 3, generator=gen).cuda()


def step(B, x, y, index, g, eps):
    """From embeddings and drawn partners to losses, gradients (in the scores' place) and images."""
    import torch
    x8, y8 = B.cloud8_pack(x), B.cloud8_pack(y)
    scores = B.cloud8_dots(x8, y8)
    kept = scores.clone()
    loss, grad = B.plan_loss(scores, index, temperature=0.25, grad=scores)
    images, lse = B.cloud8_map(x8.values(torch.bfloat16), y8, g, eps, lse=True)
    return kept, loss, grad, images, lse


@pytest.mark.gpu
@pytest.mark.parametrize("n", [20, 300])
def test_from_embeddings_to_images(B, n):
    import torch
    W, m, d = 4, 130, 96
    x, y, u = embeddings(W, n, m, d, 3)
    eps = torch.full((W,), 0.1).cuda()
    x8, y8 = B.cloud8_pack(x), B.cloud8_pack(y)
    sb = B.SinkhornBatch(x8, y8, torch.full((W, n), 1 / n).cuda(), torch.full((W, m), 1 / m).cuda(), eps, 1e-4)
    sb.drain()
    f, g = sb.potentials(f64=True)
    index = sb.draw_plan(u)
    assert torch.equal(index, B.plan_draw(x8, y8, g, eps, u))
    sb.close()
    scores, loss, grad, images, lse = step(B, x, y, index, g, eps)
    assert grad.dtype == torch.float32 and grad.shape == scores.shape
    xv, yv = x8.values().cpu().double(), y8.values().cpu().double()
    exact = xv @ yv.transpose(1, 2)
    assert ((scores.cpu().double() - exact).abs() <= 3 * 2.0 ** -19.8 * (xv.abs() @ yv.abs().transpose(1, 2))).all()
    compare_loss(loss.flatten(), grad.flatten(0, 1), scores.flatten(0, 1), index.flatten(0, 1), None, 0.25)
    want, wl, err, lerr = map_formula(x8.values().cpu(), yv, g.cpu(), eps.cpu(), yv, None)
    assert ((images.cpu().double() - want).abs() <= err).all() and ((lse.cpu().double() - wl).abs() <= lerr).all()

    # two streams at once, several times each
    other = embeddings(W, n, m, d, 4)[:2]
    first, second = step(B, x, y, index, g, eps), step(B, *other, index, g, eps)
    torch.cuda.synchronize()
    streams, results = [torch.cuda.Stream(), torch.cuda.Stream()], ([], [])
    for _ in range(5):
        for s, inputs, out in zip(streams, ((x, y), other), results):
            with torch.cuda.stream(s):
                out.append(step(B, *inputs, index, g, eps))
    torch.cuda.synchronize()
    for one, out in zip((first, second), results):
        for again in out:
            assert all(torch.equal(a, b) for a, b in zip(one, again))

    # captured, and replayed on other embeddings
    xs, ys = x.clone(), y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(B, xs, ys, index, g, eps)
    for inputs, one in ((other, second), ((x, y), first)):
        xs.copy_(inputs[0])
        ys.copy_(inputs[1])
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(one, got))
