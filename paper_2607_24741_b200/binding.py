"""ctypes binding of libsinkhorn_batch.so — argument marshalling only.

Every step of the solve runs in the library's CUDA kernels; PyTorch supplies
device memory and the stream.  There is no fallback: if the shared library is
missing or fails to load, importing this module raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsinkhorn_batch.so")

SKB_OK = 0
STATUS_NAMES = {0: "SKB_OK", 1: "SKB_ERR_NULL", 2: "SKB_ERR_SHAPE", 3: "SKB_ERR_VALUE",
                4: "SKB_ERR_WORKSPACE", 5: "SKB_ERR_STATE", 6: "SKB_ERR_CUDA"}
MODES = {"active": 0, "masked": 1, "static": 2, "masked_exit": 3}
COMPUTE = {"auto": 0, "f32": 1, "mixed": 2, "f64": 3, "tensor": 4}
LANE_RUNNING, LANE_DONE, LANE_ITER_LIMIT, LANE_NONFINITE = 0, 1, 2, 3

EXPORTS = (
    "sinkhorn_batch_workspace_bytes", "sinkhorn_batch_create", "sinkhorn_batch_step",
    "sinkhorn_batch_drain", "sinkhorn_batch_active", "sinkhorn_batch_potentials",
    "sinkhorn_batch_potentials_f64", "sinkhorn_batch_depths", "sinkhorn_batch_residuals",
    "sinkhorn_batch_stats", "sinkhorn_batch_destroy", "sinkhorn_batch_last_error",
    "sinkhorn_batch_host_workspace_bytes", "sinkhorn_batch_solve_host",
    "sinkhorn_batch_launch_count", "sinkhorn_batch_profile_update", "sinkhorn_batch_arithmetic",
    "sinkhorn_batch_selftest_bounded_wait", "sinkhorn_batch_warm_start", "sinkhorn_batch_set_profiling",
    "sinkhorn_batch_cycle_trace", "sinkhorn_batch_selftest_unit_rates", "sinkhorn_batch_last_audit",
    "sinkhorn_batch_refill", "sinkhorn_batch_apply_plan", "sinkhorn_batch_check_guards", "sinkhorn_batch_draw_plan",
)
PHASES = ("create", "f_leg", "column_check", "plan", "emit_move", "g_leg")
# entry points outside the sinkhorn_batch_* family
EXTRA_EXPORTS = ("sinkhorn_row_residual_static", "sinkhorn_row_residual_static_last_error",
                 "sinkhorn_cloud4_bytes", "sinkhorn_cloud4_pack", "sinkhorn_cloud4_unpack", "sinkhorn_cloud4_dots", "sinkhorn_plan_draw_workspace_bytes", "sinkhorn_plan_draw",
                 "sinkhorn_operator_last_error")
DTYPES = {torch.float32: 0, torch.bfloat16: 1}
FORMATS = {"mx4": 2, "nv4": 3}


class SkbConfig(ctypes.Structure):
    _fields_ = [("W", ctypes.c_int), ("n", ctypes.c_int), ("m", ctypes.c_int), ("d", ctypes.c_int),
                ("xy_dtype", ctypes.c_int), ("mode", ctypes.c_int), ("compute", ctypes.c_int),
                ("max_iter", ctypes.c_int), ("audit_every", ctypes.c_int),
                ("tol_screen", ctypes.c_float), ("column_split", ctypes.c_int),
                ("cost_form", ctypes.c_int),
                ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t), ("guard_band", ctypes.c_float),
                ("lane_capacity", ctypes.c_int)]


class SkbDrawConfig(ctypes.Structure):
    _fields_ = [("W", ctypes.c_int), ("n", ctypes.c_int), ("m", ctypes.c_int), ("d", ctypes.c_int),
                ("xy_dtype", ctypes.c_int), ("draws", ctypes.c_int),
                ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p), ("stream", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class SkbError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2607_24741_b200.build` "
                          "(there is no CPU or PyTorch fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, cfgp = ctypes.c_void_p, ctypes.POINTER(SkbConfig)
    lib.sinkhorn_batch_workspace_bytes.restype = ctypes.c_size_t
    lib.sinkhorn_batch_workspace_bytes.argtypes = [cfgp]
    lib.sinkhorn_batch_host_workspace_bytes.restype = ctypes.c_size_t
    lib.sinkhorn_batch_host_workspace_bytes.argtypes = [cfgp]
    lib.sinkhorn_batch_create.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, cfgp, ctypes.POINTER(vp)]
    lib.sinkhorn_batch_step.argtypes = [vp, ctypes.c_int]
    lib.sinkhorn_batch_drain.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_active.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_potentials.argtypes = [vp, vp, vp]
    lib.sinkhorn_batch_potentials_f64.argtypes = [vp, vp, vp]
    lib.sinkhorn_batch_depths.argtypes = [vp, vp, vp]
    lib.sinkhorn_batch_residuals.argtypes = [vp, vp, vp]
    lib.sinkhorn_batch_stats.argtypes = [vp, ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_int),
                                         vp, ctypes.c_int, ctypes.POINTER(ctypes.c_longlong),
                                         ctypes.POINTER(ctypes.c_float)]
    lib.sinkhorn_batch_last_audit.argtypes = [vp, vp, vp, vp]
    lib.sinkhorn_batch_apply_plan.argtypes = [vp, vp, vp, vp, vp, ctypes.c_int, vp]
    lib.sinkhorn_batch_refill.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_warm_start.argtypes = [vp, vp, vp, ctypes.c_int]
    lib.sinkhorn_batch_set_profiling.argtypes = [vp, ctypes.c_int]
    lib.sinkhorn_batch_cycle_trace.argtypes = [vp, vp, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_selftest_bounded_wait.argtypes = [vp, ctypes.c_float, vp]
    lib.sinkhorn_batch_check_guards.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_selftest_unit_rates.argtypes = [ctypes.POINTER(ctypes.c_double), vp, vp]
    lib.sinkhorn_batch_arithmetic.argtypes = [vp, ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_batch_launch_count.argtypes = [vp, ctypes.POINTER(ctypes.c_longlong)]
    lib.sinkhorn_batch_profile_update.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_float)]
    lib.sinkhorn_batch_destroy.argtypes = [vp]
    lib.sinkhorn_batch_destroy.restype = None
    lib.sinkhorn_batch_last_error.argtypes = [vp]
    lib.sinkhorn_batch_last_error.restype = ctypes.c_char_p
    lib.sinkhorn_batch_solve_host.argtypes = [vp, vp, vp, vp, vp, ctypes.c_float, cfgp, vp, vp, vp, vp, vp, vp,
                                              ctypes.POINTER(ctypes.c_longlong), ctypes.POINTER(ctypes.c_int)]
    lib.sinkhorn_row_residual_static.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_int, ctypes.c_int,
                                                 ctypes.c_int, ctypes.c_int, vp, vp]
    lib.sinkhorn_row_residual_static.restype = ctypes.c_int
    lib.sinkhorn_row_residual_static_last_error.restype = ctypes.c_char_p
    ci = ctypes.c_int
    lib.sinkhorn_cloud4_bytes.restype = ctypes.c_size_t
    lib.sinkhorn_cloud4_bytes.argtypes = [ci, ci, ci, ci]
    lib.sinkhorn_cloud4_pack.argtypes = [vp, ci, ci, ci, ci, ci, vp, vp, ci, vp]
    lib.sinkhorn_cloud4_unpack.argtypes = [vp, ci, ci, ci, ci, vp, ci, vp]
    lib.sinkhorn_cloud4_dots.argtypes = [vp, vp, ci, ci, ci, ci, ci, vp, vp]
    drawp = ctypes.POINTER(SkbDrawConfig)
    lib.sinkhorn_plan_draw_workspace_bytes.restype = ctypes.c_size_t
    lib.sinkhorn_plan_draw_workspace_bytes.argtypes = [drawp]
    lib.sinkhorn_plan_draw.argtypes = [vp, vp, vp, vp, vp, drawp, vp, vp]
    lib.sinkhorn_batch_draw_plan.argtypes = [vp, vp, vp, vp, vp, ci, drawp, vp, vp]
    lib.sinkhorn_operator_last_error.restype = ctypes.c_char_p
    for name in EXPORTS:
        if name not in ("sinkhorn_batch_workspace_bytes", "sinkhorn_batch_host_workspace_bytes",
                        "sinkhorn_batch_destroy", "sinkhorn_batch_last_error"):
            getattr(lib, name).restype = ctypes.c_int
    return lib


lib = _load()


def _check(code, handle=None):
    if code != SKB_OK:
        msg = lib.sinkhorn_batch_last_error(handle)
        raise SkbError(code, msg.decode() if msg else "")


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def make_config(W, n, m, d, *, bf16=False, format=None, mode="active", compute="auto", max_iter=5000,
                audit_every=1, tol_screen=0.0, column_split=0, cost_form=0, stream=0, guard_band=0.0,
                lane_capacity=0) -> SkbConfig:
    return SkbConfig(W, n, m, d, FORMATS[format] if format else 1 if bf16 else 0, MODES[mode] if isinstance(mode, str) else mode,
                     COMPUTE[compute] if isinstance(compute, str) else compute, max_iter, audit_every,
                     tol_screen, column_split, cost_form, stream, None, 0, guard_band, lane_capacity)


# ---- functions with the C names ------------------------------------------------------

def sinkhorn_batch_workspace_bytes(cfg: SkbConfig) -> int:
    return lib.sinkhorn_batch_workspace_bytes(ctypes.byref(cfg))


def sinkhorn_batch_host_workspace_bytes(cfg: SkbConfig) -> int:
    return lib.sinkhorn_batch_host_workspace_bytes(ctypes.byref(cfg))


def sinkhorn_batch_create(x, y, a, b, eps, tol, cfg: SkbConfig):
    h = ctypes.c_void_p()
    _check(lib.sinkhorn_batch_create(_ptr(x), _ptr(y), _ptr(a), _ptr(b), _ptr(eps), tol, ctypes.byref(cfg),
                                     ctypes.byref(h)))
    return h


def sinkhorn_batch_step(h, cycles):
    _check(lib.sinkhorn_batch_step(h, cycles), h)


def sinkhorn_batch_drain(h) -> int:
    c = ctypes.c_int(0)
    _check(lib.sinkhorn_batch_drain(h, ctypes.byref(c)), h)
    return c.value


def sinkhorn_batch_active(h) -> int:
    c = ctypes.c_int(0)
    _check(lib.sinkhorn_batch_active(h, ctypes.byref(c)), h)
    return c.value


def sinkhorn_batch_destroy(h):
    lib.sinkhorn_batch_destroy(h)


def sinkhorn_row_residual_static(x, y, a, f, g, eps, stream=None):
    """Row residual of potentials (f, g) per lane, with no workspace and no allocation inside the
    library (see the header for limits and the sharing rule).  x, y, a, eps: float32 CUDA tensors;
    f, g: float64.  Returns the library's status code and writes into the tensor it returns."""
    W, n, d = x.shape
    m = y.shape[1]
    out = torch.empty(W, dtype=torch.float32, device=x.device)
    st = (stream or torch.cuda.current_stream(x.device)).cuda_stream
    rc = lib.sinkhorn_row_residual_static(_ptr(x), _ptr(y), _ptr(a), _ptr(f), _ptr(g), _ptr(eps), W, n, m, d,
                                          _ptr(out), st)
    if rc != SKB_OK:
        raise SkbError(rc, lib.sinkhorn_row_residual_static_last_error().decode())
    return out


def unit_rates(device=None):
    """Measured operations per second of the fp32 FMA, packed fp32x2 FMA, float64 FMA and fp32 ex2
    units (the library's self-test loops)."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    sink = torch.zeros(1, dtype=torch.float32, device=dev)
    out = (ctypes.c_double * 4)()
    with torch.cuda.device(dev):
        _check(lib.sinkhorn_batch_selftest_unit_rates(out, _ptr(sink), torch.cuda.current_stream(dev).cuda_stream))
    return dict(zip(("ffma", "ffma2", "dfma", "ex2"), list(out)))


# ---- operators beside the solver --------------------------------------------------------

def _check_op(code):
    if code != SKB_OK:
        raise SkbError(code, lib.sinkhorn_operator_last_error().decode())


# They run on the current stream of the tensors' device, and their outputs and workspaces belong to it.
_HERE_ALREADY = contextlib.nullcontext()


def _on(device):
    """The device's context; none where it is the current one (a call of a few microseconds is worth that)."""
    return _HERE_ALREADY if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _stream(device):
    return torch.cuda.current_stream(device).cuda_stream


def _cloud4_bytes(W, npts, d, format):
    """sinkhorn_cloud4_bytes for a valid shape, 0 otherwise."""
    if min(W, npts, d) < 1 or d > 1024 or W * npts > 0x7fffffff:
        return 0
    pad = lambda b: (b + 255) // 256 * 256
    rows, blocks = W * npts, (d + 31) // 32 * (2 if format == "nv4" else 1)
    return pad(rows * ((d + 31) // 32 * 16)) + pad(rows * ((blocks + 3) // 4 * 4)) + (pad(rows * 4) if format == "nv4" else 0)


class Cloud4:
    """A cloud [W, npts, d] held in 4 bits: `buffer` as sinkhorn_cloud4_pack lays it out (a uint8 CUDA tensor)."""

    def __init__(self, buffer, W, npts, d, format):
        if format not in FORMATS:
            raise ValueError(f"format must be one of {tuple(FORMATS)}")
        need = _cloud4_bytes(W, npts, d, format)
        if need == 0:
            raise ValueError("W, npts and d must be >= 1, d at most 1024")
        if buffer.dtype != torch.uint8 or not buffer.is_cuda or not buffer.is_contiguous() or buffer.numel() < need:
            raise ValueError(f"buffer must be a contiguous uint8 CUDA tensor of at least {need} bytes")
        if buffer.data_ptr() % 256:
            raise ValueError("buffer must be 256-byte aligned")
        self.buffer, self.W, self.npts, self.d, self.format = buffer, W, npts, d, format

    @property
    def shape(self):
        return (self.W, self.npts, self.d)

    @property
    def device(self):
        return self.buffer.device

    def values(self, dtype=torch.float32):
        """What the cloud stands for, [W, npts, d] float32 or bfloat16."""
        if dtype not in DTYPES:
            raise ValueError("dtype must be float32 or bfloat16")
        with _on(self.device):
            out = torch.empty(self.shape, dtype=dtype, device=self.device)
            _check_op(lib.sinkhorn_cloud4_unpack(_ptr(self.buffer), self.W, self.npts, self.d, FORMATS[self.format], _ptr(out),
                                                 DTYPES[dtype], _stream(self.device)))
        return out


def cloud4_pack(v, format="mx4", values=None):
    """Rounds v [W, npts, d] (float32 or bfloat16, CUDA) to 4 bits, format "mx4" or "nv4"; returns a Cloud4, or with
    `values` (torch.float32 or torch.bfloat16) the pair of it and the values that it stands for.  No gradient is recorded: a training
    step that wants one passes it through the rounding itself, v + (values - v).detach()."""
    if v.dim() != 3 or not v.is_cuda or v.dtype not in DTYPES:
        raise ValueError("v must be a float32 or bfloat16 CUDA tensor [W, npts, d]")
    if format not in FORMATS:
        raise ValueError(f"format must be one of {tuple(FORMATS)}")
    if values is not None and values not in DTYPES:
        raise ValueError("values must be torch.float32 or torch.bfloat16")
    v = v.contiguous()
    W, npts, d = v.shape
    need = _cloud4_bytes(W, npts, d, format)
    if need == 0:
        raise ValueError("W, npts and d must be >= 1, d at most 1024")
    with _on(v.device):
        buffer = torch.empty(need, dtype=torch.uint8, device=v.device)
        out = None if values is None else torch.empty(v.shape, dtype=values, device=v.device)
        _check_op(lib.sinkhorn_cloud4_pack(_ptr(v), DTYPES[v.dtype], W, npts, d, FORMATS[format], _ptr(buffer), _ptr(out),
                                           DTYPES.get(values, 0), _stream(v.device)))
    cloud = Cloud4(buffer, W, npts, d, format)
    return cloud if values is None else (cloud, out)


def cloud4_dots(x, y, out=None):
    """x_ti . y_tj of two Cloud4 of one format, [W, n, d] and [W, m, d]: float32 [W, n, m]."""
    if not isinstance(x, Cloud4) or not isinstance(y, Cloud4):
        raise ValueError("x and y must be Cloud4")
    if x.format != y.format or x.W != y.W or x.d != y.d or x.device != y.device:
        raise ValueError("x and y must have one format, W, d and device")
    shape = (x.W, x.npts, y.npts)
    if out is not None and (out.dtype != torch.float32 or out.device != x.device or tuple(out.shape) != shape or not out.is_contiguous()):
        raise ValueError("out must be a contiguous float32 tensor [W, n, m] on the clouds' device")
    with _on(x.device):
        if out is None:
            out = torch.empty(shape, dtype=torch.float32, device=x.device)
        _check_op(lib.sinkhorn_cloud4_dots(_ptr(x.buffer), _ptr(y.buffer), x.W, x.npts, y.npts, x.d, FORMATS[x.format], _ptr(out),
                                           _stream(x.device)))
    return out


def _raw(v):
    return v.buffer if isinstance(v, Cloud4) else v


def _cloud(v, name):
    """dtype, shape, pointer and the tensor to keep of a cloud: a tensor or a Cloud4."""
    if isinstance(v, Cloud4):
        return FORMATS[v.format], v.shape, v.buffer
    if not torch.is_tensor(v) or not v.is_cuda or v.dim() != 3 or v.dtype not in DTYPES:
        raise ValueError(f"{name} must be a float32 or bfloat16 CUDA tensor [W, points, d], or a Cloud4")
    v = v.contiguous()
    if v.data_ptr() % 16:
        v = v.clone()
    return DTYPES[v.dtype], tuple(v.shape), v


def _draw_config(W, n, m, d, dtype, u, settings, stream):
    """Configuration of a draw, with its settings checked; u [W, n] or [W, n, draws] is checked too."""
    device = u.device
    if not u.is_cuda or u.dtype != torch.float32 or u.dim() not in (2, 3) or tuple(u.shape[:2]) != (W, n):
        raise ValueError("u must be a float32 CUDA tensor [W, n] or [W, n, draws]")
    cfg = SkbDrawConfig(W, n, m, d, dtype, u.shape[2] if u.dim() == 3 else 1, stream=stream)
    for name, t in settings.items():
        if t is None:
            continue
        want = torch.int32 if name == "top_k" else torch.float32
        if not torch.is_tensor(t) or t.dtype != want or t.device != device or tuple(t.shape) != (W,) or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {want} tensor [W] on the device of the clouds")
        setattr(cfg, name, t.data_ptr())
    return cfg


def _draw_out(cfg, u, logp):
    index = torch.empty(u.shape, dtype=torch.int32, device=u.device)
    lp = torch.empty(u.shape, dtype=torch.float32, device=u.device) if logp else None
    need = lib.sinkhorn_plan_draw_workspace_bytes(ctypes.byref(cfg))
    if need == 0:
        raise SkbError(2, "shape not supported: W, n, m, d, draws >= 1, d <= 1024, n and m <= 262143, W <= 65535")
    ws = torch.empty(need, dtype=torch.uint8, device=u.device)
    cfg.workspace, cfg.workspace_bytes = ws.data_ptr(), need
    return index, lp, ws


def plan_draw(x, y, g, eps, u, *, temperature=None, top_k=None, top_p=None, min_p=None, logp=False):
    """Partners of x [W, n, d] among y [W, m, d] (tensors or Cloud4), drawn from the coupling's rows, softmax over j of
    (g_j - |x_i - y_j|^2) / (eps T), one for each number of u [W, n] or [W, n, draws]; see sinkhorn_plan_draw in
    the header.  Settings are tensors [W].  Returns the indices (int32, u's shape), with `logp` also their log
    probabilities."""
    dt, (W, n, d), xk = _cloud(x, "x")
    dty, ys, yk = _cloud(y, "y")
    m = ys[1]
    if dty != dt or ys != (W, m, d):
        raise ValueError("x and y must have one type, W and d")
    device = xk.device
    if yk.device != device or u.device != device:
        raise ValueError("all tensors must be on one device")
    if g.dtype != torch.float64 or g.device != device or tuple(g.shape) != (W, m):
        raise ValueError("g must be a float64 tensor [W, m] on the device of the clouds")
    if eps.dtype != torch.float32 or eps.device != device or tuple(eps.shape) != (W,):
        raise ValueError("eps must be a float32 tensor [W] on the device of the clouds")
    g, eps, u = g.contiguous(), eps.contiguous(), u.contiguous()
    with _on(device):
        cfg = _draw_config(W, n, m, d, dt, u, dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p),
                           _stream(device))
        index, lp, ws = _draw_out(cfg, u, logp)
        _check_op(lib.sinkhorn_plan_draw(_ptr(xk), _ptr(yk), _ptr(g), _ptr(eps), _ptr(u), ctypes.byref(cfg), _ptr(index), _ptr(lp)))
    return (index, lp) if logp else index


class _Apart:
    """A stream's work after what `here` has been given, and `here`'s after that: tensors that are made, cleared or freed on `here`
    are read and written there in between."""

    def __init__(self, here, there):
        self.here, self.there = here, there

    def __enter__(self):
        self.there.wait_stream(self.here)

    def __exit__(self, *_):
        self.here.wait_stream(self.there)


class SinkhornBatch:
    """One batch of W lanes on the current CUDA device (thin wrapper over the C calls)."""

    def __init__(self, x, y, a, b, eps, tol, *, mode="active", compute="auto", max_iter=5000,
                 audit_every=1, tol_screen=0.0, column_split=0, cost_form=0, stream=None, guard_band=0.0,
                 lane_capacity=0):
        self.format = x.format if isinstance(x, Cloud4) else None          # x and y may be clouds held in 4 bits
        if self.format is None:
            if isinstance(y, Cloud4):
                raise ValueError("x and y must both be tensors or both be Cloud4")
            if not (x.is_cuda and y.is_cuda and a.is_cuda and b.is_cuda and eps.is_cuda):
                raise ValueError("x, y, a, b, eps must be CUDA tensors")
            if x.dtype not in (torch.float32, torch.bfloat16) or y.dtype != x.dtype:
                raise ValueError("x and y must both be float32 or both be bfloat16")
        elif not isinstance(y, Cloud4) or y.format != x.format or not (a.is_cuda and b.is_cuda and eps.is_cuda):
            raise ValueError("x and y must be Cloud4 of one format, a, b, eps CUDA tensors")
        for t in (a, b, eps):
            if t.dtype != torch.float32:
                raise ValueError("a, b, eps must be float32")
        a, b, eps = (t.contiguous() for t in (a, b, eps))
        if self.format is None:
            x, y = x.contiguous(), y.contiguous()
        W, n, d = x.shape
        m = y.shape[1]
        if y.shape != (W, m, d) or a.shape != (W, n) or b.shape != (W, m) or eps.shape != (W,):
            raise ValueError("shapes must be x[W,n,d] y[W,m,d] a[W,n] b[W,m] eps[W]")
        self.W, self.n, self.m, self.d = W, n, m, d
        self.device = x.device
        self.stream = stream if stream is not None else torch.cuda.current_stream(x.device)
        self.cfg = make_config(W, n, m, d, bf16=self.format is None and x.dtype == torch.bfloat16, format=self.format, mode=mode, compute=compute,
                               max_iter=max_iter, audit_every=audit_every, tol_screen=tol_screen,
                               column_split=column_split, cost_form=cost_form, stream=self.stream.cuda_stream,
                               guard_band=guard_band, lane_capacity=lane_capacity)
        self.L = max(W, lane_capacity)
        need = sinkhorn_batch_workspace_bytes(self.cfg)
        if need == 0:
            raise SkbError(2, "configuration rejected (unsupported shape or bad option)")
        self.workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
        self.cfg.workspace = self.workspace.data_ptr()
        self.cfg.workspace_bytes = need
        self._keep = (x, y, a, b, eps)
        self.h = None
        with torch.cuda.device(x.device), self._after_here():
            self.h = sinkhorn_batch_create(_raw(x), _raw(y), a, b, eps, float(tol), self.cfg)

    def _after_here(self):
        """For calls that read or write tensors of the current stream on the batch's."""
        here = torch.cuda.current_stream(self.device)
        return _HERE_ALREADY if here == self.stream else _Apart(here, self.stream)

    def step(self, cycles=1):
        sinkhorn_batch_step(self.h, cycles)

    def drain(self) -> int:
        return sinkhorn_batch_drain(self.h)

    def active(self) -> int:
        return sinkhorn_batch_active(self.h)

    def potentials(self, f64=False):
        dt = torch.float64 if f64 else torch.float32
        f = torch.zeros(self.L, self.n, dtype=dt, device=self.device)
        g = torch.zeros(self.L, self.m, dtype=dt, device=self.device)
        fn = lib.sinkhorn_batch_potentials_f64 if f64 else lib.sinkhorn_batch_potentials
        with self._after_here():
            _check(fn(self.h, _ptr(f), _ptr(g)), self.h)
        return f, g

    def depths(self):
        depth = torch.zeros(self.L, dtype=torch.int32, device=self.device)
        status = torch.zeros(self.L, dtype=torch.int32, device=self.device)
        with self._after_here():
            _check(lib.sinkhorn_batch_depths(self.h, _ptr(depth), _ptr(status)), self.h)
        return depth, status

    def residuals(self):
        rr = torch.zeros(self.L, dtype=torch.float32, device=self.device)
        rc = torch.zeros(self.L, dtype=torch.float32, device=self.device)
        with self._after_here():
            _check(lib.sinkhorn_batch_residuals(self.h, _ptr(rr), _ptr(rc)), self.h)
        return rr, rc

    def warm_start(self, f0=None, g0=None, audit_initial=False):
        for t, shape in ((f0, (self.W, self.n)), (g0, (self.W, self.m))):
            if t is not None and (t.dtype != torch.float64 or not t.is_cuda or tuple(t.shape) != shape
                                  or not t.is_contiguous()):
                raise ValueError("f0 [W,n] and g0 [W,m] must be contiguous float64 CUDA tensors")
        with self._after_here():
            _check(lib.sinkhorn_batch_warm_start(self.h, _ptr(f0), _ptr(g0), 1 if audit_initial else 0), self.h)
        self._warm = (f0, g0)

    def check_guards(self) -> int:
        """Index of the first damaged guard strip of the workspace, -1 if all are intact (synchronises)."""
        bad = ctypes.c_int(-2)
        _check(lib.sinkhorn_batch_check_guards(self.h, ctypes.byref(bad)), self.h)
        return bad.value

    def last_audit(self):
        """Row screen value, column residual (NaN where not checked) and screen flag of the most recent audit."""
        rr = torch.full((self.L,), float("nan"), dtype=torch.float32, device=self.device)
        rc = torch.full((self.L,), float("nan"), dtype=torch.float32, device=self.device)
        fl = torch.full((self.L,), -1, dtype=torch.int32, device=self.device)
        with self._after_here():
            _check(lib.sinkhorn_batch_last_audit(self.h, _ptr(rr), _ptr(rc), _ptr(fl)), self.h)
        return rr, rc, fl

    def refill(self, x, y, a, b, eps) -> int:
        """New problems into the slots finished lanes have freed; returns their first lane number."""
        if (x.format if isinstance(x, Cloud4) else None) != self.format or (y.format if isinstance(y, Cloud4) else None) != self.format:
            raise ValueError("x and y must be of the batch's storage type")
        a, b, eps = (t.contiguous() for t in (a, b, eps))
        if self.format is None:
            x, y = x.contiguous(), y.contiguous()
        count = x.shape[0]
        if tuple(x.shape) != (count, self.n, self.d) or tuple(y.shape) != (count, self.m, self.d) or \
                tuple(a.shape) != (count, self.n) or tuple(b.shape) != (count, self.m) or tuple(eps.shape) != (count,):
            raise ValueError("shapes must be x[c,n,d] y[c,m,d] a[c,n] b[c,m] eps[c]")
        first = ctypes.c_int(-1)
        with self._after_here():
            _check(lib.sinkhorn_batch_refill(self.h, _ptr(_raw(x)), _ptr(_raw(y)), _ptr(a), _ptr(b), _ptr(eps), count, ctypes.byref(first)), self.h)
        self._keep = self._keep + (x, y, a, b, eps)
        return first.value

    def apply_plan(self, v):
        """out[t, i, :] = sum_j pi_ij v[t, j, :] with the plan of the finished lanes; v [W, m, dv] float32."""
        x, y, _a, _b, eps = self._keep[:5]
        v = v.contiguous()
        if v.dtype != torch.float32 or v.dim() != 3 or tuple(v.shape[:2]) != (self.W, self.m):
            raise ValueError("v must be float32 [W, m, dv]")
        out = torch.empty(self.W, self.n, v.shape[2], dtype=torch.float32, device=self.device)
        with self._after_here():
            _check(lib.sinkhorn_batch_apply_plan(self.h, _ptr(_raw(x)), _ptr(_raw(y)), _ptr(eps), _ptr(v), v.shape[2], _ptr(out)), self.h)
        return out

    def draw_plan(self, u, *, side="sources", temperature=None, top_k=None, top_p=None, min_p=None, logp=False):
        """Partners of the sources (u [W, n] or [W, n, draws]) or of the targets (side "targets", u [W, m] or [W, m, draws])
        drawn from the plan of the finished lanes; settings and outputs as those of plan_draw.  Runs on the batch's stream, after what
        the current one has been given and before what it is given next."""
        if side not in ("sources", "targets"):
            raise ValueError('side must be "sources" or "targets"')
        x, y, _a, _b, eps = self._keep[:5]
        other = side == "targets"
        n, m = (self.m, self.n) if other else (self.n, self.m)
        if u.device != self.device:
            raise ValueError("u must be on the batch's device")
        with torch.cuda.device(self.device):
            u = u.contiguous()
            if self.format is None:
                x, y = (v if v.data_ptr() % 16 == 0 else v.clone() for v in (x, y))
            cfg = _draw_config(self.W, n, m, self.d, self.cfg.xy_dtype, u,
                               dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p), self.stream.cuda_stream)
            index, lp, ws = _draw_out(cfg, u, logp)
            cfg.n, cfg.m = self.n, self.m
            with self._after_here():
                _check(lib.sinkhorn_batch_draw_plan(self.h, _ptr(_raw(x)), _ptr(_raw(y)), _ptr(eps), _ptr(u), 1 if other else 0,
                                                    ctypes.byref(cfg), _ptr(index), _ptr(lp)), self.h)
        return (index, lp) if logp else index

    def set_profiling(self, on=True):
        _check(lib.sinkhorn_batch_set_profiling(self.h, 1 if on else 0), self.h)

    def stats(self, widths_cap=0):
        slots, terms, cycles = ctypes.c_longlong(0), ctypes.c_longlong(0), ctypes.c_int(0)
        buf = (ctypes.c_int * max(widths_cap, 1))()
        ph = (ctypes.c_float * len(PHASES))()
        _check(lib.sinkhorn_batch_stats(self.h, ctypes.byref(slots), ctypes.byref(cycles),
                                        ctypes.cast(buf, ctypes.c_void_p), widths_cap, ctypes.byref(terms), ph), self.h)
        k = min(cycles.value, widths_cap)
        return {"slots": slots.value, "cycles": cycles.value, "pair_terms": terms.value,
                "widths": list(buf[:k]), "phase_ms": dict(zip(PHASES, list(ph)))}

    def cycle_trace(self):
        n = ctypes.c_int(0)
        _check(lib.sinkhorn_batch_cycle_trace(self.h, None, 0, ctypes.byref(n)), self.h)
        buf = (ctypes.c_float * max(n.value, 1))()
        _check(lib.sinkhorn_batch_cycle_trace(self.h, ctypes.cast(buf, ctypes.c_void_p), n.value, ctypes.byref(n)), self.h)
        return list(buf[:n.value])

    def arithmetic(self) -> str:
        c = ctypes.c_int(0)
        _check(lib.sinkhorn_batch_arithmetic(self.h, ctypes.byref(c)), self.h)
        return {v: k for k, v in COMPUTE.items()}[c.value]

    def launch_count(self) -> int:
        c = ctypes.c_longlong(0)
        _check(lib.sinkhorn_batch_launch_count(self.h, ctypes.byref(c)), self.h)
        return c.value

    def profile_update(self, leg=0, reps=10) -> float:
        ms = ctypes.c_float(0)
        _check(lib.sinkhorn_batch_profile_update(self.h, leg, reps, ctypes.byref(ms)), self.h)
        return ms.value

    def close(self):
        if self.h is not None:
            sinkhorn_batch_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
