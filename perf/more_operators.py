"""Operators beside the solver: clouds held in 8 bits, their products, maps over them, and the loss that teaches scores a coupling.

  pack   a cloud of embeddings rounded to 8-bit floating point (e4m3), a power of two for each block of 128 dimensions of a point
  dots   x_i . y_j of two such clouds
  map    images of query points under the entropic map of a stored target cloud: attention over a bank held in 8 bits,
             out_i = sum_j w_ij v_j,  w_i = softmax over j of (g_j - |x_i - y_j|^2) / eps
  loss   distillation of a coupling's rows into scores: sum_k q_k (log q_k - log p_k) of the entries k that the teacher
         names (its top logits, or draws from its rows), p the softmax of a row of scores, with the gradient

`run` computes them in plain torch operations where `own` is false, and calls the library where it is true.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"


def listed():
    pack = lambda name, W, n, d, dtype: dict(name=name, job="pack", W=W, n=n, d=d, dtype=dtype)
    dots = lambda name, W, n, m, d: dict(name=name, job="dots", W=W, n=n, m=m, d=d)
    map_ = lambda name, W, n, m, d, dv=0, ragged=False: dict(name=name, job="map", W=W, n=n, m=m, d=d, dv=dv, ragged=ragged)
    loss = lambda name, rows, m, k, dtype, teacher, temperature=1.0: dict(name=name, job="loss", rows=rows, m=m, k=k, dtype=dtype, teacher=teacher,
                                                                          temperature=temperature)
    return [
        # a minibatch of deep bf16 embeddings, with the values that training goes on with
        pack("pack8_feature", 64, 1024, 512, "bf16"),
        # the fp32 embeddings of a small ragged minibatch, the last block of 128 not full
        pack("pack8_ragged", 24, 333, 200, "f32"),
        # products of one small pair of clouds: latency
        dots("dots8_small", 1, 128, 100, 64),
        # ragged minibatches
        dots("dots8_ragged", 24, 500, 333, 200),
        # minibatch couplings of deep embeddings
        dots("dots8_feature", 64, 1024, 1024, 512),
        # serving: one query to each of a few banks, its image under the map
        map_("map8_single", 8, 1, 16384, 512),
        # serving a queue: a handful of queries to each bank of shallower embeddings, values of their own
        map_("map8_few", 32, 12, 8192, 128, dv=64),
        # ragged lanes, one of them empty, values of their own
        map_("map8_ragged", 24, 77, 333, 200, dv=96, ragged=True),
        # barycentric images of a whole minibatch of deep embeddings
        map_("map8_feature", 64, 1024, 1024, 512),
        # a small matcher taught four draws from every row
        loss("loss_tiny", 512, 64, 4, "f32", "draws"),
        # the scores of a minibatch of embeddings, taught draws from the coupling's rows
        loss("loss_feature", 65536, 1024, 8, "bf16", "draws"),
        # scores over a whole bank, taught the teacher's top logits, softened
        loss("loss_bank", 4096, 65536, 64, "bf16", "top", temperature=2.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    job = rng.choice(["pack", "dots", "map", "map", "loss", "loss"])
    if job == "pack":
        return dict(job=job, W=_log(rng, 1, 64), n=_log(rng, 32, 1024), d=_log(rng, 33, 512), dtype=rng.choice(["f32", "bf16"]))
    if job == "dots":
        return dict(job=job, W=_log(rng, 1, 64), n=_log(rng, 32, 1024), m=_log(rng, 32, 1024), d=rng.choice([64, 128, 256, 512, rng.randint(33, 512)]))
    if job == "map":
        n, m, d = _log(rng, 1, 1024), _log(rng, 64, 16384), rng.choice([64, 128, 256, 512, rng.randint(33, 512)])
        most = max(1, min(64, int(64 * 1024 * 1024 * 512 / (n * m * d)), (1 << 27) // (m * d)))
        return dict(job=job, W=_log(rng, 1, most), n=n, m=m, d=d, dv=rng.choice([0, 0, 64, 128, rng.randint(1, 256)]), ragged=rng.random() < 0.4)
    m = _log(rng, 32, 65536)
    return dict(job="loss", rows=_log(rng, 32, min(65536, 4096 * 65536 // m)), m=m, k=min(m, _log(rng, 1, 64)), dtype=rng.choice(["f32", "bf16"]),
                teacher=rng.choice(["draws", "top"]), temperature=rng.choice([1.0, 1.0, 2.0, round(rng.uniform(0.5, 4.0), 2)]))


def work(case):
    blocks = lambda d: -(-d // 128)
    if case["job"] == "pack":
        W, n, d = case["W"], case["n"], case["d"]
        # the cloud in; its codes, scales and norms, and the values that they stand for, out
        return {"bytes": W * n * (d * (2 if case["dtype"] == "bf16" else 4) + d + blocks(d) + 4 + 2 * d), "flops": 4 * W * n * d}
    if case["job"] == "dots":
        W, n, m, d = case["W"], case["n"], case["m"], case["d"]
        return {"bytes": W * ((n + m) * (d + blocks(d)) + 4 * n * m), "flops": 2 * W * n * m * d}
    if case["job"] == "map":
        W, n, m, d = case["W"], case["n"], case["m"], case["d"]
        if case["ragged"]:
            m = 0.75 * m
        dv = case["dv"] or d
        # queries, codes, scales, norms and potentials in (values of their own too), images and logarithms of the sums out
        bank = d + blocks(d) + 4 + 8 + (dv + blocks(dv) if case["dv"] else 0)
        return {"bytes": W * (n * (2 * d + 2 * dv + 4) + m * bank), "flops": W * n * m * (2 * d + 2 * dv + 4)}
    rows, m, width = case["rows"], case["m"], 2 if case["dtype"] == "bf16" else 4
    return {"bytes": rows * (2 * m * width + case["k"] * (8 if case["teacher"] == "top" else 4) + 8), "flops": 6 * rows * m}


# ------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000033 * int(seed) + 71)
    return gen


def _embeddings(W, counts, d, gen):
    """Clouds of unit vectors around ten class means, one cloud for each of the counts."""
    normal = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.float32)
    mu = normal(W, 10, d)
    out = []
    for k in counts:
        v = normal(W, k, d) + torch.gather(mu, 1, torch.randint(10, (W, k, 1), generator=gen, device=DEV).expand(W, k, d))
        out.append(v / v.norm(dim=2, keepdim=True))
    return out


def _potential(x, y, eps):
    """The target's potential after two cycles of the solver's updates, in float64 as the solver gives it."""
    (W, n, _), m = x.shape, y.shape[1]
    out = torch.empty(W, m, device=DEV, dtype=torch.float64)
    for t in range(W):
        c = torch.cdist(x[t], y[t]).square_() / eps
        g = torch.zeros(m, device=DEV)
        for _ in range(2):
            f = -math.log(n) - torch.logsumexp(g[None, :] - c, 1)
            g = -math.log(m) - torch.logsumexp(f[:, None] - c, 0)
        out[t] = eps * g.double()
    return out


def _map_inputs(case, gen):
    """Queries, the bank in fp32, its potential, its values in fp32 (or None) and the lanes' lengths (or None)."""
    W, n, m, d = case["W"], case["n"], case["m"], case["d"]
    x, y, sample = _embeddings(W, (n, m, min(m, 256)), d, gen)
    eps = 0.05
    g = _potential(sample, y, eps)
    v = torch.randn(W, m, case["dv"], generator=gen, device=DEV) if case["dv"] else None
    lengths = None
    if case["ragged"]:
        lengths = torch.randint((m + 1) // 2, m + 1, (W,), generator=gen, device=DEV, dtype=torch.int32)
        if W > 1:
            lengths[0] = 0
    return x.bfloat16(), y, g, torch.full((W,), eps, device=DEV), v, lengths


def prepare(case, seed):
    gen = _generator(seed)
    if case["job"] == "pack":
        x, = _embeddings(case["W"], (case["n"],), case["d"], gen)
        return {"case": case, "x": x.bfloat16() if case["dtype"] == "bf16" else x}
    if case["job"] == "dots":
        x, y = _embeddings(case["W"], (case["n"], case["m"]), case["d"], gen)
        return {"case": case, "x8": _lay_out(*_rounded(x)), "y8": _lay_out(*_rounded(y))}
    if case["job"] == "map":
        x, y, g, eps, v, lengths = _map_inputs(case, gen)
        return {"case": case, "x": x, "y8": _lay_out(*_rounded(y)), "g": g, "eps": eps,
                "v8": None if v is None else _lay_out(*_rounded(v)), "lengths": lengths}
    rows, m, k = case["rows"], case["m"], case["k"]
    # the student's scores are the teacher's, blurred; the teacher names draws from its rows, or its largest entries
    teacher = 3.0 * torch.randn(rows, m, generator=gen, device=DEV)
    scores = (teacher + torch.randn(rows, m, generator=gen, device=DEV)).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    if case["teacher"] == "draws":
        index = torch.multinomial(torch.softmax(teacher, 1), k, replacement=True, generator=gen).int()
        logits = None
    else:
        logits, index = torch.topk(teacher, k, 1)
        index, logits = index.int(), logits.contiguous()
    # rows without a partner, as draws from a masked row are
    index[torch.rand(rows, generator=gen, device=DEV) < 0.01] = -1
    weight = torch.rand(rows, generator=gen, device=DEV) / rows
    return {"case": case, "scores": scores, "index": index.contiguous(), "logits": logits, "weight": weight}


# ------------------------------------------------------------------- plain forms: 8-bit clouds

def _exponent(v):
    """floor(log2 v) of positive numbers."""
    return torch.frexp(v)[1] - 1


def _rounded(x):
    """Codes [W, n, 32 ceil(d/32)] and scale bytes [W, n, ceil(d/128)] (uint8), the values' squared norms [W, n] and d."""
    W, n, d = x.shape
    nb = -(-d // 128)
    v = torch.zeros(W, n, nb * 128, device=x.device)
    v[:, :, :d] = x
    block = v.view(W, n, nb, 128)
    top = block.abs().amax(3)
    # the smallest power of two that the block's largest value is at most 448 times of
    e = torch.where(top > 0, _exponent(top) - 8, -100)
    e = torch.where(top > torch.ldexp(torch.full_like(top, 448.0), e), e + 1, e).clamp(min=-100)
    q = torch.ldexp(block, -e[..., None])
    code = q.to(torch.float8_e4m3fn)
    value = torch.ldexp(code.float(), e[..., None]).double()
    code = code.view(torch.uint8).reshape(W, n, -1)[:, :, :-(-d // 32) * 32]
    return code.contiguous(), (e + 127).to(torch.uint8), value.square().sum((2, 3)).float(), d


def _pad(nbytes):
    return -(-nbytes // 256) * 256


def _room(d):
    """Bytes that a buffer keeps for a point's scales: a whole number of words."""
    return -(-d // 512) * 4


def _lay_out(code, byte, norm, d):
    """One buffer: codes, scales, squared norms."""
    byte = torch.cat((byte, byte.new_zeros(*byte.shape[:2], _room(d) - byte.shape[2])), 2)
    parts = [code, byte, norm.view(torch.uint8)]
    buf = torch.zeros(sum(_pad(p.numel()) for p in parts), device=code.device, dtype=torch.uint8)
    at = 0
    for p in parts:
        buf[at:at + p.numel()] = p.reshape(-1)
        at += _pad(p.numel())
    return buf


def _values(code, byte, d):
    """What codes and scales stand for, in 32 bits (exact)."""
    W, n, wide = code.shape
    scale = torch.exp2(byte.float() - 127.0).repeat_interleave(128, 2)[:, :, :wide]
    return (code.view(torch.float8_e4m3fn).float() * scale)[:, :, :d]


def _unpacked(buf, W, n, d):
    """The values of a buffer."""
    wide = -(-d // 32) * 32
    code = buf[:W * n * wide].view(W, n, wide)
    at = _pad(code.numel())
    byte = buf[at:at + W * n * _room(d)].view(W, n, -1)[:, :, :-(-d // 128)]
    return _values(code, byte, d)


# ---------------------------------------------------------------- plain forms: maps and the loss

def _mapped(state):
    case, x = state["case"], state["x"].float()
    W, m = case["W"], case["m"]
    y = _unpacked(state["y8"], W, m, case["d"])
    v = y if state["v8"] is None else _unpacked(state["v8"], W, m, case["dv"])
    dist = x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :] - 2.0 * torch.bmm(x, y.transpose(1, 2))
    z = (state["g"][:, None, :].float() - dist) / state["eps"][:, None, None]
    if state["lengths"] is not None:
        z = z.masked_fill(torch.arange(m, device=DEV)[None, None, :] >= state["lengths"][:, None, None], -math.inf)
    top = z.amax(2, keepdim=True)
    none = top == -math.inf
    w = torch.exp(z - torch.where(none, 0.0, top))
    total = w.sum(2, keepdim=True)
    out = torch.bmm(w, v) / torch.where(none, 1.0, total)
    return out.bfloat16(), (torch.log(total) + top).squeeze(2)


def _taught(state):
    case, s = state["case"], state["scores"]
    T = case["temperature"]
    index = state["index"].long()
    named = index >= 0
    t = torch.zeros(index.shape, device=DEV) if state["logits"] is None else state["logits"] / T
    t = torch.where(named, t, -math.inf)
    any_ = named.any(1, keepdim=True)
    q = torch.exp(t - torch.where(any_, t.amax(1, keepdim=True), 0.0))
    q = q / torch.where(any_, q.sum(1, keepdim=True), 1.0)
    z = s.float() / T
    z = z - z.amax(1, keepdim=True)
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    logp = torch.gather(z, 1, index.clamp(min=0)) - torch.log(total)
    loss = torch.where(q > 0, q * (torch.log(q) - logp), 0.0).sum(1)
    p = p / total * any_
    p.scatter_add_(1, index.clamp(min=0), -q)
    return loss, (p * (state["weight"][:, None] / T)).to(s.dtype)


def run(state):
    case = state["case"]
    if own:
        from paper_2607_24741_b200 import binding as B
        if case["job"] == "pack":
            return B.cloud8_pack(state["x"], values=torch.bfloat16)[1]
        if case["job"] == "dots":
            return B.cloud8_dots(B.Cloud8(state["x8"], case["W"], case["n"], case["d"]), B.Cloud8(state["y8"], case["W"], case["m"], case["d"]))
        if case["job"] == "map":
            y8 = B.Cloud8(state["y8"], case["W"], case["m"], case["d"])
            v8 = None if state["v8"] is None else B.Cloud8(state["v8"], case["W"], case["m"], case["dv"])
            return B.cloud8_map(state["x"], y8, state["g"], state["eps"], v8, lengths=state["lengths"], lse=True)
        return B.plan_loss(state["scores"], state["index"], state["logits"], temperature=case["temperature"], weight=state["weight"], grad=True)
    if case["job"] == "pack":
        code, byte, _, d = _rounded(state["x"])
        return _values(code, byte, d).bfloat16()
    if case["job"] == "dots":
        x, y = _unpacked(state["x8"], case["W"], case["n"], case["d"]), _unpacked(state["y8"], case["W"], case["m"], case["d"])
        return torch.bmm(x, y.transpose(1, 2))
    return _mapped(state) if case["job"] == "map" else _taught(state)


# ------------------------------------------------------------ the definitions, in 64 bits

def _exact_values(x):
    """The nearest values that blocks of e4m3 numbers can hold, from the spacings, halves to even."""
    out = torch.empty(x.shape, device=x.device, dtype=torch.float64)
    for lo in range(0, x.shape[2], 128):
        v = x[:, :, lo:lo + 128].double()
        top = v.abs().amax(2, keepdim=True)
        power = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448.0))
        # (a logarithm next to a whole number is decided by the definition)
        power = torch.where(torch.exp2(power - 1.0) * 448.0 >= top, power - 1.0, torch.where(torch.exp2(power) * 448.0 < top, power + 1.0, power))
        scale = torch.exp2(torch.where(top > 0, power, -100.0).clamp(min=-100.0))
        a = v.abs() / scale
        gap = torch.exp2(torch.frexp(a)[1].clamp(min=-5).double() - 4.0)
        out[:, :, lo:lo + 128] = torch.sign(v) * torch.round(a / gap) * gap * scale
    return out


def _exact_map(case, gen):
    x, y, g, eps, v, lengths = _map_inputs(case, gen)
    y = _exact_values(y)
    v = y if v is None else _exact_values(v)
    out = torch.zeros(case["W"], case["n"], v.shape[2], device=DEV, dtype=torch.float64)
    lse = torch.full((case["W"], case["n"]), -math.inf, device=DEV, dtype=torch.float64)
    for t in range(case["W"]):
        m = case["m"] if lengths is None else int(lengths[t])
        if m == 0:
            continue
        z = -torch.cdist(x[t].double(), y[t, :m], compute_mode="donot_use_mm_for_euclid_dist").square() + g[t, None, :m]
        z /= eps[t].double()
        lse[t] = torch.logsumexp(z, 1)
        out[t] = torch.exp(z - lse[t][:, None]) @ v[t, :m]
    return out, lse


def _exact_loss(state):
    s, T = state["scores"], state["case"]["temperature"]
    loss = torch.zeros(s.shape[0], device=DEV, dtype=torch.float64)
    grad = torch.zeros(s.shape, device=DEV, dtype=torch.float64)
    step = max(1, (1 << 27) // s.shape[1])
    for lo in range(0, s.shape[0], step):
        at = slice(lo, min(lo + step, s.shape[0]))
        index = state["index"][at].long()
        live = (index >= 0).any(1)
        t = index.double() * 0.0 if state["logits"] is None else state["logits"][at].double() / T
        logq = torch.log_softmax(t.masked_fill(index < 0, -math.inf), 1)
        logp = torch.log_softmax(s[at].double() / T, 1)
        terms = torch.exp(logq) * (logq - torch.gather(logp, 1, index.clamp(min=0)))
        loss[at] = torch.where(live, torch.where(index >= 0, terms, 0.0).sum(1), 0.0)
        part = torch.exp(logp)
        part.scatter_add_(1, index.clamp(min=0), torch.where(index >= 0, -torch.exp(logq), 0.0))
        grad[at] = torch.where(live[:, None], part * (state["weight"][at].double() / T)[:, None], 0.0)
    return loss, grad


def exact(case, seed):
    gen = _generator(seed)
    if case["job"] == "pack":
        return _exact_values(prepare(case, seed)["x"])
    if case["job"] == "dots":
        x, y = _embeddings(case["W"], (case["n"], case["m"]), case["d"], gen)
        return torch.bmm(_exact_values(x), _exact_values(y).transpose(1, 2))
    return _exact_map(case, gen) if case["job"] == "map" else _exact_loss(prepare(case, seed))
