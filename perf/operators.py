"""Operators beside the solver: clouds held in 4 bits, their products, and draws from a coupling.

  pack   a cloud of embeddings rounded to microscaled 4-bit values (blocks that share a scale)
  dots   x_i . y_j of two such clouds, the contraction that deep lanes' costs are made of
  draw   partners drawn from the rows of a coupling: softmax over j of (g_j - |x_i - y_j|^2) / (eps T),
         cut down by top-k, top-p and min-p, one draw for each uniform number that the caller gives

`run` computes them in plain torch operations where `own` is false, and calls the library where it is true.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda:0"

# A 4-bit code's low three bits; the fourth is the sign.
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    draw_case = lambda name, law, W, n, m, d, dtype="f32", draws=1, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, vary=False: dict(
        name=name, job="draw", law=law, W=W, n=n, m=m, d=d, dtype=dtype, draws=draws, temperature=temperature, top_k=top_k,
        top_p=top_p, min_p=min_p, vary=vary)
    pack = lambda name, W, n, d, dtype, fmt, law="feature": dict(name=name, job="pack", law=law, W=W, n=n, d=d, dtype=dtype, fmt=fmt)
    dots = lambda name, W, n, m, d, fmt: dict(name=name, job="dots", law="feature", W=W, n=n, m=m, d=d, fmt=fmt)
    return [
        # one partner for each point of a few small two-dimensional problems: nothing but latency
        draw_case("draw_tiny", "tiny", 8, 64, 64, 2),
        # training pairs from a day of sensor windows, sharpened, the tails of the rows cut off
        draw_case("draw_sensor", "sensor", 256, 512, 512, 15, temperature=0.7, top_p=0.9),
        # training pairs from a minibatch coupling of deep bf16 embeddings
        draw_case("draw_feature", "feature", 64, 1024, 1024, 512, dtype="bf16", top_p=0.95),
        # correspondences between two pairs of scans, four hypotheses a point from its 16 likeliest partners
        draw_case("draw_registration", "registration", 2, 8192, 8192, 3, draws=4, top_k=16),
        # ragged lanes with padding behind their targets, one lane without any, each with settings of its own
        draw_case("draw_ragged", "sweep", 96, 100, 77, 8, draws=3, vary=True),
        # a minibatch of bf16 embeddings into blocks of 32
        pack("pack_feature", 64, 1024, 512, "bf16", "mx4"),
        # the fp32 embeddings of a small ragged minibatch, blocks of 16, the last of them not full
        pack("pack_ragged", 24, 333, 200, "f32", "nv4"),
        # an embedding bank
        pack("pack_bank", 8, 16384, 512, "f32", "nv4"),
        # products of one small pair of clouds: latency
        dots("dots_small", 1, 128, 100, 64, "mx4"),
        # ragged minibatches
        dots("dots_ragged", 24, 500, 333, 200, "nv4"),
        # minibatch couplings of deep embeddings
        dots("dots_feature", 64, 1024, 1024, 512, "mx4"),
        # one large coupling
        dots("dots_large", 4, 4096, 4096, 512, "nv4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    job = rng.choice(["draw", "draw", "pack", "dots"])
    if job == "pack":
        W, n, d = _log(rng, 1, 64), _log(rng, 32, 1024), _log(rng, 33, 640)
        return dict(job=job, law="feature", W=W, n=n, d=d, dtype=rng.choice(["f32", "bf16"]), fmt=rng.choice(["mx4", "nv4"]))
    if job == "dots":
        W, n, m, d = _log(rng, 1, 64), _log(rng, 32, 1024), _log(rng, 32, 1024), rng.choice([64, 128, 256, 512, rng.randint(33, 512)])
        return dict(job=job, law="feature", W=W, n=n, m=m, d=d, fmt=rng.choice(["mx4", "nv4"]))
    law, dtype = rng.choice(["tiny", "sensor", "feature", "registration", "sweep"]), "f32"
    if law == "tiny":
        W, n, m, d = _log(rng, 2, 64), _log(rng, 16, 128), _log(rng, 16, 128), 2
    elif law == "sensor":
        W, n, m, d = _log(rng, 4, 256), _log(rng, 100, 512), _log(rng, 100, 512), rng.randint(9, 16)
    elif law == "feature":
        W, n, m = _log(rng, 2, 64), _log(rng, 128, 1024), _log(rng, 128, 1024)
        d, dtype = rng.choice([64, 128, 256, 320, 512]), rng.choice(["bf16", "bf16", "f32"])
        if dtype == "f32":
            W, d = min(W, 8), min(d, 128)
    elif law == "registration":
        n, d = _log(rng, 500, 8192), 3
        W, m = max(1, min(_log(rng, 1, 16), (2 * 8192 * 8192) // (n * n))), n
    else:
        W, n, m, d = _log(rng, 16, 512), _log(rng, 32, 256), _log(rng, 1, 256), rng.randint(4, 8)
    vary = law == "sweep"
    cut = rng.choice(["none", "k", "p", "m", "all"])
    return dict(job="draw", law=law, W=W, n=n, m=m, d=d, dtype=dtype, draws=rng.choice([1, 1, 2, 4]),
                temperature=round(rng.uniform(0.3, 2.0), 3), top_k=rng.randint(1, max(1, m // 2)) if cut in ("k", "all") else 0,
                top_p=round(rng.uniform(0.5, 0.99), 3) if cut in ("p", "all") else 1.0,
                min_p=round(rng.uniform(0.001, 0.1), 4) if cut in ("m", "all") else 0.0, vary=vary)


def work(case):
    W, n, d = case["W"], case["n"], case["d"]
    if case["job"] == "pack":
        width = 2 if case["dtype"] == "bf16" else 4
        # the cloud in; its codes and scales, and the values that they stand for, out
        return {"bytes": W * n * (d * width + d / 2 + d / (32 if case["fmt"] == "mx4" else 16) + 2 * d), "flops": 4 * W * n * d}
    m = case["m"]
    if case["job"] == "dots":
        block = 32 if case["fmt"] == "mx4" else 16
        return {"bytes": W * ((n + m) * (d / 2 + d / block) + 4 * n * m), "flops": 2 * W * n * m * d}
    width = 2 if case["dtype"] == "bf16" else 4
    # a product, a subtraction and an exponential for every pair; clouds, potentials and numbers in, indices and logarithms out
    return {"bytes": W * ((n + m) * d * width + 8 * m + 12 * n * case["draws"]), "flops": W * n * m * (2 * d + 4)}


# ------------------------------------------------------------------------------- inputs

def _generator(seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1000003 * int(seed) + 29)
    return gen


def _clouds(case, gen):
    """x [W,n,d], y [W,m,d], eps [W] of the laws that the solver's workloads follow."""
    W, n, m, d, law = case["W"], case["n"], case.get("m", 1), case["d"], case["law"]
    normal = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=torch.float32)
    uniform = lambda *s: torch.rand(*s, generator=gen, device=DEV, dtype=torch.float32)
    if law == "tiny":
        x, y = normal(W, n, d), 2.0 * uniform(W, 1, d) + (0.5 + 1.5 * uniform(W, 1, 1)).sqrt() * normal(W, m, d)
        eps = torch.full((W,), 0.05, device=DEV)
    elif law == "sensor":
        x = normal(W, n, d)
        y = 0.3 * normal(W, 1, d) + (1.0 + 0.5 * uniform(W, 1, d)).sqrt() * normal(W, m, d)
        eps = torch.full((W,), 0.2 * d, device=DEV) * (1.0 + 0.1 * uniform(W))
    elif law == "feature":
        mu = normal(W, 10, d)
        pick = lambda k: torch.gather(mu, 1, torch.randint(10, (W, k, 1), generator=gen, device=DEV).expand(W, k, d))
        unit = lambda v: v / v.norm(dim=2, keepdim=True)
        x, y = unit(normal(W, n, d) + pick(n)), unit(normal(W, m, d) + pick(m))
        eps = torch.full((W,), 0.05, device=DEV)
    elif law == "registration":
        v = normal(W, n, d)
        x = v / v.norm(dim=2, keepdim=True) * (1.0 + 0.02 * normal(W, n, 1))
        q, _ = torch.linalg.qr(normal(W, d, d).double())
        y = x @ q.transpose(1, 2).float() + 0.01 * normal(W, n, d)
        y = torch.where(uniform(W, n, 1) < 0.10, 2.0 * uniform(W, n, d) - 1.0, y)
        eps = torch.full((W,), 0.01, device=DEV)
    else:
        x, y = normal(W, n, d), normal(W, m, d)
        eps = torch.exp(math.log(0.01) + (math.log(0.5) - math.log(0.01)) * uniform(W))
    if case.get("dtype") == "bf16":
        x, y = x.bfloat16(), y.bfloat16()
    return x.contiguous(), y.contiguous(), eps.contiguous()


def _potential(x, y, eps):
    """The target's potential after two cycles of the solver's updates, in float64 as the solver gives it."""
    (W, n, _), m = x.shape, y.shape[1]
    out = torch.empty(W, m, device=DEV, dtype=torch.float64)
    for t in range(W):
        e = float(eps[t])
        c = torch.cdist(x[t].float(), y[t].float()).square_() / e
        g = torch.zeros(m, device=DEV)
        for _ in range(2):
            f = -math.log(n) - torch.logsumexp(g[None, :] - c, 1)
            g = -math.log(m) - torch.logsumexp(f[:, None] - c, 0)
        out[t] = e * g.double()
    return out


def prepare(case, seed):
    gen = _generator(seed)
    if case["job"] == "pack":
        x, _, _ = _clouds(case, gen)
        return {"case": case, "x": x}
    x, y, eps = _clouds(case, gen)
    if case["job"] == "dots":
        return {"case": case, "x4": _lay_out(*_rounded(x, case["fmt"])), "y4": _lay_out(*_rounded(y, case["fmt"]))}
    W, n, m, S = case["W"], case["n"], case["m"], case["draws"]
    g = _potential(x, y, eps)
    rand = lambda *s: torch.rand(*s, generator=gen, device=DEV, dtype=torch.float32)
    lane = lambda v, dt: torch.full((W,), v, device=DEV, dtype=dt)
    state = {"case": case, "x": x, "y": y, "g": g, "eps": eps, "u": rand(W, n, S), "temperature": lane(case["temperature"], torch.float32),
             "top_k": lane(case["top_k"], torch.int32), "top_p": lane(case["top_p"], torch.float32), "min_p": lane(case["min_p"], torch.float32)}
    if case["vary"]:
        state["temperature"] = 0.3 + 1.2 * rand(W)
        state["temperature"][1::7] = 0.0          # the likeliest partner alone
        state["top_k"] = torch.randint(0, m + 2, (W,), generator=gen, device=DEV, dtype=torch.int32)
        state["top_p"] = 0.5 + 0.6 * rand(W)
        state["min_p"] = 0.1 * rand(W)
        # padding: no mass, and whatever was in memory for coordinates
        real = torch.randint((m + 1) // 2, m + 1, (W, 1), generator=gen, device=DEV)
        real[0] = 0
        pad = torch.arange(m, device=DEV) >= real
        g.masked_fill_(pad, -math.inf)
        y.masked_fill_(pad[:, :, None], math.nan)
    return state


# ------------------------------------------------------------------- plain forms: 4-bit clouds

def _blocks(d, fmt):
    """Scales a point has: blocks of 32 (mx4) or of 16 (nv4), a whole number of 32 values."""
    return -(-d // 32) * (1 if fmt == "mx4" else 2)


def _room(d, fmt):
    """Bytes that a buffer keeps for them: a whole number of words."""
    return -(-_blocks(d, fmt) // 4) * 4


def _exponent(v):
    """floor(log2 v) of positive doubles."""
    return torch.frexp(v)[1].to(torch.float64) - 1.0


def _rounded(x, fmt):
    """Codes [W, n, 32 ceil(d/32)] (uint8), scale bytes [W, n, blocks] and the power of two of each point [W, n]."""
    W, n, d = x.shape
    nb = _blocks(d, fmt)
    v = torch.zeros(W, n, -(-d // 32) * 32, device=x.device, dtype=torch.float64)
    v[:, :, :d] = x
    block = v.view(W, n, nb, -1)
    top = block.abs().amax(3)
    if fmt == "mx4":
        # the exponent of the block's largest value, less that of the largest 4-bit value
        power = torch.where(top > 0, _exponent(top) - 2.0, -127.0).clamp(-127.0, 127.0)
        scale, byte, point = torch.exp2(power), (power + 127.0).to(torch.uint8), torch.ones(W, n, device=x.device, dtype=torch.float64)
    else:
        # a power of two for the point; then a sixth of the block's largest value, with three bits of mantissa
        whole = top.amax(2)
        point = torch.exp2(torch.where(whole > 0, _exponent(whole) - 10.0, 0.0).clamp(-126.0, 127.0))
        q = top / 6.0 / point[:, :, None]
        step = torch.exp2(torch.where(q > 0, _exponent(q), -6.0).clamp(min=-6.0) - 3.0)
        scale = torch.round(q / step) * step
        byte = scale.float().to(torch.float8_e4m3fn).view(torch.uint8)
        scale = scale * point[:, :, None]
    q = torch.where(scale[..., None] > 0, block.abs() / scale[..., None], 0.0)
    # halfway between two values of the grid: to the one with the even code
    code = (q > 0.25).to(torch.uint8) + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5.0)
    return (code + 8 * (block < 0)).view(W, n, -1), byte, point.float(), d, fmt


def _pad(nbytes):
    return -(-nbytes // 256) * 256


def _lay_out(code, byte, point, d, fmt):
    """One buffer: two codes to a byte, the even value low; the scales; for nv4 the points' powers of two."""
    W, n, _ = code.shape
    pair = code.view(W, n, -1, 2)
    byte = torch.cat((byte, byte.new_zeros(W, n, _room(d, fmt) - byte.shape[2])), 2)
    parts = [pair[..., 0] + 16 * pair[..., 1], byte] + ([point.view(torch.uint8)] if fmt == "nv4" else [])
    buf = torch.zeros(sum(_pad(p.numel()) for p in parts), device=code.device, dtype=torch.uint8)
    at = 0
    for p in parts:
        buf[at:at + p.numel()] = p.reshape(-1)
        at += _pad(p.numel())
    return buf


def _values(code, byte, point, d, fmt):
    """What codes and scales stand for, in 32 bits (exact: at most six bits of mantissa)."""
    W, n, wide = code.shape
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=code.device)
    scale = torch.exp2(byte.float() - 127.0) if fmt == "mx4" else byte.view(torch.float8_e4m3fn).float() * point[:, :, None]
    return (grid[code.long()].view(W, n, byte.shape[2], -1) * scale[..., None]).view(W, n, wide)[:, :, :d]


def _unpacked(buf, W, n, d, fmt):
    """The codes, scales and powers of two of a buffer."""
    wide, nb = -(-d // 32) * 32, _blocks(d, fmt)
    pair = buf[:W * n * wide // 2]
    code = torch.stack((pair & 15, pair >> 4), 1).view(W, n, wide)
    at = _pad(pair.numel())
    byte = buf[at:at + W * n * _room(d, fmt)].view(W, n, -1)
    at += _pad(byte.numel())
    byte = byte[:, :, :nb].contiguous()
    point = buf[at:at + 4 * W * n].view(torch.float32).view(W, n) if fmt == "nv4" else torch.ones(W, n, device=buf.device)
    return code, byte, point, d, fmt


# ------------------------------------------------------------------------ plain form: draws

def _setting(state):
    """Per lane, as [W, 1, 1]: temperature, k, p and the smallest share; a temperature of zero keeps the likeliest alone."""
    T, k, p, r = (state[key].double()[:, None, None] for key in ("temperature", "top_k", "top_p", "min_p"))
    greedy = T == 0
    k = torch.where(k == 0, math.inf, k)
    return torch.where(greedy, 1.0, T), torch.where(greedy, 1.0, k), torch.where(p >= 1.0, math.inf, p), r


def _drawn(state):
    x, y, g, u = state["x"].double(), state["y"].double(), state["g"], state["u"].double()
    T, k, p, r = _setting(state)
    z = torch.baddbmm(x.square().sum(2)[:, :, None] + y.square().sum(2)[:, None, :], x, y.transpose(1, 2), alpha=-2.0)
    z = (g[:, None, :] - z) / (state["eps"].double()[:, None, None] * T)
    z = torch.where(g[:, None, :] == -math.inf, -math.inf, z)
    top = z.amax(2, keepdim=True)
    none = top == -math.inf
    z = z - torch.where(none, 0.0, top)
    # largest first, ties in the order of their indices; each cut looks at what the one before it left
    w, order = torch.sort(z, dim=2, descending=True, stable=True)
    w = w.exp_()
    rank = torch.arange(w.shape[2], device=w.device)
    w = torch.where(rank < k, w, 0.0)
    share = p * w.sum(2, keepdim=True)
    before = torch.cumsum(w, 2) - w
    w = torch.where((before < share) & (w >= r) & (w > 0.0), w, 0.0)
    del before
    w = torch.zeros_like(z).scatter_(2, order, w)
    del order
    total = w.sum(2, keepdim=True)
    run_ = torch.cumsum(w, 2)
    index = torch.searchsorted(run_, u * run_[:, :, -1:], right=True).clamp_(max=w.shape[2] - 1)
    logp = torch.gather(z, 2, index) - torch.log(total)
    return torch.where(none, -1, index).int(), torch.where(none, math.nan, logp).float()


def run(state):
    case = state["case"]
    if own:
        from paper_2607_24741_b200 import binding as B
        if case["job"] == "pack":
            return B.cloud4_pack(state["x"], case["fmt"], values=torch.bfloat16)[1]
        if case["job"] == "dots":
            x4 = B.Cloud4(state["x4"], case["W"], case["n"], case["d"], case["fmt"])
            return B.cloud4_dots(x4, B.Cloud4(state["y4"], case["W"], case["m"], case["d"], case["fmt"]))
        return B.plan_draw(state["x"], state["y"], state["g"], state["eps"], state["u"], temperature=state["temperature"],
                           top_k=state["top_k"], top_p=state["top_p"], min_p=state["min_p"], logp=True)
    if case["job"] == "pack":
        return _values(*_rounded(state["x"], case["fmt"])).bfloat16()
    if case["job"] == "dots":
        x = _values(*_unpacked(state["x4"], case["W"], case["n"], case["d"], case["fmt"]))
        y = _values(*_unpacked(state["y4"], case["W"], case["m"], case["d"], case["fmt"]))
        return torch.bmm(x, y.transpose(1, 2))
    return _drawn(state)


# ------------------------------------------------------------ the definitions, in 64 bits

def _exact_values(x, fmt):
    """The nearest values that blocks of 4-bit numbers can hold, from spacings and halves to even."""
    W, n, d = x.shape
    size = 32 if fmt == "mx4" else 16
    out = torch.empty(W, n, d, device=x.device, dtype=torch.float64)
    whole = x.double().abs().amax(2)
    point = torch.where(whole > 0, torch.ldexp(torch.ones_like(whole), torch.frexp(whole)[1] - 11), 1.0)
    for lo in range(0, d, size):
        v = x[:, :, lo:lo + size].double()
        top = v.abs().amax(2)
        if fmt == "mx4":
            scale = torch.ldexp(torch.ones_like(top), torch.where(top > 0, torch.frexp(top)[1] - 3, -127))
        else:
            q = top / (6.0 * point)
            gap = torch.ldexp(torch.ones_like(q), torch.frexp(q)[1].clamp(min=-5) - 4)
            scale = torch.round(q / gap) * gap * point
        a = torch.where(scale[:, :, None] > 0, v.abs() / scale[:, :, None], 0.0)
        gap = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
        out[:, :, lo:lo + size] = torch.sign(v) * (torch.round(a / gap) * gap).clamp(max=6.0) * scale[:, :, None]
    return out


def _exact_drawn(state):
    """Row blocks of one lane at a time: distances by differences, cuts by comparing with the border values."""
    W, n, S = state["u"].shape
    m, d = state["y"].shape[1:]
    index = torch.empty(W, n, S, device=DEV, dtype=torch.int32)
    logp = torch.empty(W, n, S, device=DEV, dtype=torch.float64)
    temperature, top_k, top_p, min_p, eps = (state[key].tolist() for key in ("temperature", "top_k", "top_p", "min_p", "eps"))
    step = max(1, (1 << 24) // m)
    for t in range(W):
        T, k = (1.0, 1) if temperature[t] == 0 else (temperature[t], top_k[t] or m)
        for lo in range(0, n, step):
            x, y = state["x"][t, lo:lo + step].double(), state["y"][t].double()
            c = torch.zeros(x.shape[0], m, device=DEV, dtype=torch.float64)
            for a in range(d):
                c += (x[:, a, None] - y[None, :, a]).square()
            g = state["g"][t][None, :]
            z = torch.where(g > -math.inf, (g - c) / (eps[t] * T), -math.inf)
            if bool((z == -math.inf).all()):
                index[t, lo:lo + step], logp[t, lo:lo + step] = -1, math.nan
                continue
            z -= z.amax(1, keepdim=True)
            # place of every entry in the order of size
            place = torch.empty_like(z, dtype=torch.int64)
            order = torch.argsort(z, dim=1, descending=True, stable=True)
            place.scatter_(1, order, torch.arange(m, device=DEV).expand_as(order))
            w = torch.exp(z) * (place < k)
            if top_p[t] < 1.0:
                s = torch.gather(w, 1, order)
                mass = torch.cumsum(s, 1)
                # entries in front of the first place at which the mass reaches the share, and that one
                need = (mass < top_p[t] * mass[:, -1:]).sum(1, keepdim=True)
                w = w * (place <= need)
            w = w * (w >= min_p[t])
            mass = torch.cumsum(w, 1)
            target = state["u"][t, lo:lo + step].double() * mass[:, -1:]
            at = torch.searchsorted(mass, target.contiguous(), right=True).clamp(max=m - 1)
            index[t, lo:lo + step] = at.int()
            logp[t, lo:lo + step] = torch.log(torch.gather(w, 1, at) / mass[:, -1:])
    return index, logp


def exact(case, seed):
    state = prepare(case, seed)
    if case["job"] == "pack":
        return _exact_values(state["x"], case["fmt"])
    if case["job"] == "dots":
        gen = _generator(seed)
        x, y, _ = _clouds(case, gen)
        return torch.bmm(_exact_values(x, case["fmt"]), _exact_values(y, case["fmt"]).transpose(1, 2))
    return _exact_drawn(state)
