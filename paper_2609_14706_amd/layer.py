"""Operators around one layer: the norm that makes its rows, the linear layer
itself in bf16 or from the quantiser's codes, their gradients, and the
orthogonalisation of an update of its weights.

Each is one call of the HIP library (include/ff.h) on torch tensors: no state,
no autograd, results as new tensors on the inputs' device.  Work goes to the
device's current stream, or to `stream`, one of that device (ordered by the
caller after what made the inputs); nothing waits.  Rows are the last dimension, contiguous; a 2-D
tensor's rows may lie any distance apart, other shapes have to be contiguous.
Workspaces are taken from torch unless `workspace` (a uint8 tensor) is given.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple

import torch

from .binding import _check, load_library

FF_ACT_NONE, FF_ACT_RELU, FF_ACT_GELU, FF_ACT_SILU = 0, 1, 2, 3
ACTIVATIONS = {"none": FF_ACT_NONE, "relu": FF_ACT_RELU, "gelu": FF_ACT_GELU, "silu": FF_ACT_SILU}

_i64, _ptr, _int, _f64, _size = (ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t)


class ff_norm_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("dtype", _int), ("x", _ptr), ("ldx", _i64),
                ("residual", _ptr), ("ldr", _i64), ("weight", _ptr), ("eps", _f64), ("normalise", _int),
                ("sum", _ptr), ("ldsum", _i64), ("y", _ptr), ("ldy", _i64), ("col_scale", _ptr),
                ("q", _ptr), ("ldq", _i64), ("q_scale", _ptr), ("stream", _ptr)]


class ff_norm_grad_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("dtype", _int), ("s", _ptr), ("lds", _i64),
                ("dy", _ptr), ("lddy", _i64), ("dsum", _ptr), ("lddsum", _i64), ("weight", _ptr),
                ("eps", _f64), ("ds", _ptr), ("ldds", _i64), ("dweight", _ptr), ("workspace", _ptr),
                ("workspace_bytes", _size), ("stream", _ptr)]


class ff_linear_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("n", _i64), ("m", _i64), ("x", _ptr), ("ldx", _i64), ("w", _ptr),
                ("ldw", _i64), ("x_scale", _ptr), ("row_scale", _ptr), ("bias", _ptr), ("residual", _ptr),
                ("ldr", _i64), ("activation", _int), ("y", _ptr), ("ldy", _i64), ("preact", _ptr),
                ("ldz", _i64), ("workspace", _ptr), ("workspace_bytes", _size), ("stream", _ptr)]


class ff_linear_grad_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("n", _i64), ("m", _i64), ("dy", _ptr), ("lddy", _i64), ("x", _ptr),
                ("ldx", _i64), ("w", _ptr), ("ldw", _i64), ("preact", _ptr), ("ldz", _i64),
                ("activation", _int), ("g", _ptr), ("ldg", _i64), ("dx", _ptr), ("lddx", _i64),
                ("dw", _ptr), ("lddw", _i64), ("db", _ptr), ("workspace", _ptr),
                ("workspace_bytes", _size), ("stream", _ptr)]


class ff_ortho_args(ctypes.Structure):
    _fields_ = [("batch", _i64), ("m", _i64), ("n", _i64), ("dtype", _int), ("G", _ptr), ("ldg", _i64),
                ("stride_g", _i64), ("out", _ptr), ("ldo", _i64), ("stride_o", _i64), ("steps", _int),
                ("a", _f64), ("b", _f64), ("c", _f64), ("eps", _f64), ("scale", _f64), ("workspace", _ptr),
                ("workspace_bytes", _size), ("stream", _ptr)]


_FN = {}


def _library():
    """The library's layer functions with their signatures, by name."""
    if not _FN:
        found = {}
        lib = load_library()
        ref = ctypes.POINTER
        size = ref(_size)
        for name, args in {
                "ff_rms_norm": [ref(ff_norm_args)],
                "ff_rms_norm_backward": [ref(ff_norm_grad_args)],
                "ff_rms_norm_backward_workspace_size": [ref(ff_norm_grad_args), size],
                "ff_linear": [ref(ff_linear_args)],
                "ff_linear_q8": [ref(ff_linear_args)],
                "ff_linear_workspace_size": [ref(ff_linear_args), _int, size],
                "ff_linear_backward": [ref(ff_linear_grad_args)],
                "ff_linear_backward_workspace_size": [ref(ff_linear_grad_args), size],
                "ff_orthogonalize": [ref(ff_ortho_args)],
                "ff_orthogonalize_workspace_size": [ref(ff_ortho_args), size]}.items():
            f = getattr(lib, name)
            f.restype, f.argtypes = _int, args
            found[name] = f
        _FN.update(found)   # all at once: other threads see none or all of them
    return _FN


# ------------------------------------------------------------------ arguments
_ELEM = {torch.float32: 0, torch.bfloat16: 1}   # ff_dtype


def _refuse(t, name, dtype, device):
    """Why t is not a tensor of that type on that device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    raise ValueError(f"{name} must be on {device}, not on {t.device}")


def _rows(t, name, dtype, device, cols=None):
    """(pointer, leading dimension, rows, columns) of a tensor's rows."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device:
        _refuse(t, name, dtype, device)
    shape = t.shape
    if not shape:
        raise ValueError(f"{name} must have at least one dimension")
    c = shape[-1]
    if cols is not None and c != cols:
        raise ValueError(f"{name} must have rows of {cols} elements, not {c}")
    if t.is_contiguous():
        return t.data_ptr(), c, shape[0] if len(shape) == 2 else shape[:-1].numel(), c
    if len(shape) != 2 or (c != 1 and t.stride(1) != 1) or (shape[0] != 1 and t.stride(0) < c):
        raise ValueError(f"{name} must be contiguous, or 2-D with contiguous rows that do not overlap")
    return t.data_ptr(), (t.stride(0) if shape[0] > 1 else c), shape[0], c


def _like(t, dtype):
    """A new contiguous tensor of t's shape."""
    if t.is_contiguous():
        return torch.empty_like(t, dtype=dtype)
    return torch.empty(t.shape, dtype=dtype, device=t.device)


def _matrix_of(rows, cols, dtype, device):
    """A new (rows, cols) tensor (with its strides: 0.4 us less than torch.empty takes)."""
    return torch.empty_strided((rows, cols), (cols, 1), dtype=dtype, device=device)


def _vector(t, name, dtype, device, count):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.device != device:
        _refuse(t, name, dtype, device)
    if t.numel() != count or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous tensor of {count} elements")
    return t.data_ptr()


def _first(t, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    return t.device


def _act(name):
    try:
        return ACTIVATIONS[name]
    except (KeyError, TypeError):
        raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)}, not {name!r}") from None


def _elem(t, name):
    if t.dtype not in _ELEM:
        raise TypeError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return _ELEM[t.dtype]


def _flat(values):
    """The values, with those of tuples (checkpoints, routings) in their place."""
    for v in values:
        if isinstance(v, tuple):
            yield from _flat(v)
        else:
            yield v


def _on_stream(stream, fn, *args, **kw):
    """fn on `stream`: its allocations and the inputs' lives are ordered there,
    the results' also on the caller's stream, which is to use them."""
    device = getattr(stream, "device", None)
    if device is None:
        raise TypeError("stream must be a torch.cuda.Stream")
    inputs = [t for t in _flat((*args, *kw.values())) if isinstance(t, torch.Tensor) and t.is_cuda]
    for t in inputs:
        if t.device != device:
            raise ValueError(f"stream is of {device}, the tensors are on {t.device}")
    with torch.cuda.stream(stream):
        out = fn(*args, **kw)
    for t in inputs:
        t.record_stream(stream)
    caller = torch.cuda.current_stream(device)
    for t in _flat((out,)):
        if isinstance(t, torch.Tensor):
            t.record_stream(caller)
    return out


def _workspace(args, nbytes, workspace, device):
    """Give args its workspace; returns what has to live until the launch."""
    if nbytes == 0:
        return None
    if workspace is None:
        workspace = torch.empty(nbytes + 255, dtype=torch.uint8, device=device)
    elif (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8 or workspace.device != device
          or not workspace.is_contiguous() or workspace.numel() < nbytes + 255):
        raise ValueError(f"workspace must be a contiguous uint8 tensor of >= {nbytes + 255} bytes on {device}")
    args.workspace = (workspace.data_ptr() + 255) // 256 * 256
    args.workspace_bytes = nbytes
    return workspace


_raw_stream, _current_device = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice


def _launch(name, args, device, functions=_FN):
    """Call the library on the device's current stream."""
    index = device.index
    args.stream = _raw_stream(index)
    if _current_device() == index:
        code = functions[name](args)
    else:
        with torch.cuda.device(index):
            code = functions[name](args)
    if code:
        _check(code)


def _bytes(name, args, *more, functions=_FN):
    out = _size(0)
    code = functions[name](args, *more, out)
    if code:
        _check(code)
    return out.value


# ----------------------------------------------------------------------- norm
def _norm(x, weight, residual, eps, col_scale, q8, normalise):
    """(y or codes, their scales or None, the sum or None)."""
    if not _FN:
        _library()
    dev = _first(x, "x")
    dtype = x.dtype
    px, ldx, r, c = _rows(x, "x", dtype, dev)
    pr = ldr = ps = 0
    s = scale = None
    if residual is not None:
        pr, ldr, _, _ = _rows(residual, "residual", dtype, dev, c)
        if residual.shape != x.shape:
            raise ValueError(f"residual must have x's shape {tuple(x.shape)}")
        if normalise:
            s = _like(x, dtype)
            ps = s.data_ptr()
    pw = None if weight is None else _vector(weight, "weight", dtype, dev, c)
    if q8:
        y = _like(x, torch.int8)
        scale = torch.empty((r,) if x.dim() == 2 else x.shape[:-1], dtype=torch.float32, device=dev)
        a = ff_norm_args(r, c, _elem(x, "x"), px, ldx, pr, ldr, pw, eps, normalise, ps, c, None, 0,
                         _vector(col_scale, "col_scale", torch.float32, dev, c), y.data_ptr(), c, scale.data_ptr())
    else:
        y = _like(x, dtype)
        a = ff_norm_args(r, c, _elem(x, "x"), px, ldx, pr, ldr, pw, eps, normalise, ps, c, y.data_ptr(), c)
    if r:
        _launch("ff_rms_norm", a, dev)
    return y, scale, s


def rms_norm(x, weight=None, *, residual=None, eps: float = 1e-6, stream=None):
    """(y, s): s = x + residual, y = s / sqrt(mean(s^2) + eps) * weight over the
    last dimension, float32 or bfloat16 throughout.  Without a residual s is x."""
    if stream is not None:
        return _on_stream(stream, rms_norm, x, weight, residual=residual, eps=eps)
    y, _, s = _norm(x, weight, residual, eps, None, False, 1)
    return y, x if s is None else s


def rms_norm_q8(x, weight=None, *, residual=None, eps: float = 1e-6, col_scale=None, stream=None):
    """(q, scale, s): the norm of rms_norm in 8 bits, q scale = y col_scale with
    scale = max |y col_scale| / 127 of each row (q int8, scale float32).
    col_scale: float32, the input-side scales alpha of a layer of codes."""
    if stream is not None:
        return _on_stream(stream, rms_norm_q8, x, weight, residual=residual, eps=eps, col_scale=col_scale)
    q, scale, s = _norm(x, weight, residual, eps, col_scale, True, 1)
    return q, scale, x if s is None else s


def quantize_rows(x, *, col_scale=None, stream=None):
    """(q, scale): rows in 8 bits, q scale = x col_scale with scale =
    max |x col_scale| / 127 of each row; see ff_rms_norm."""
    if stream is not None:
        return _on_stream(stream, quantize_rows, x, col_scale=col_scale)
    q, scale, _ = _norm(x, None, None, 0.0, col_scale, True, 0)
    return q, scale


def rms_norm_backward(dy, s, weight=None, *, eps: float = 1e-6, dsum=None, workspace=None, stream=None):
    """(ds, dweight) of y = rms_norm(s) for the gradient dy of y: ds (plus dsum,
    the gradient that reaches s by other ways) is the gradient of x and of the
    residual alike; dweight is None without a weight."""
    if stream is not None:
        return _on_stream(stream, rms_norm_backward, dy, s, weight, eps=eps, dsum=dsum, workspace=workspace)
    _library()
    dev = _first(s, "s")
    dt = _elem(s, "s")
    ps, lds, r, c = _rows(s, "s", s.dtype, dev)
    a = ff_norm_grad_args(r, c, dt, ps, lds)
    a.dy, a.lddy, _, _ = _rows(dy, "dy", s.dtype, dev, c)
    if dsum is not None:
        a.dsum, a.lddsum, _, _ = _rows(dsum, "dsum", s.dtype, dev, c)
    if dy.shape != s.shape or (dsum is not None and dsum.shape != s.shape):
        raise ValueError(f"dy and dsum must have the shape of s, {tuple(s.shape)}")
    a.weight = _vector(weight, "weight", s.dtype, dev, c)
    a.eps = eps
    ds = _like(s, s.dtype)
    a.ds, a.ldds = ds.data_ptr(), c
    dw = None
    if weight is not None:
        dw = torch.empty_like(weight)
        a.dweight = dw.data_ptr()
    keep = _workspace(a, _bytes("ff_rms_norm_backward_workspace_size", a), workspace, dev)
    _launch("ff_rms_norm_backward", a, dev)
    del keep
    return ds, dw


# --------------------------------------------------------------------- linear
def _linear(name, x, weight, dtype, x_scale, row_scale, bias, residual, activation, keep_preact, workspace):
    if not _FN:
        _library()
    dev = _first(x, "x")
    px, ldx, T, n = _rows(x, "x", dtype, dev)
    pw, ldw, m, _ = _rows(weight, "weight", dtype, dev, n)
    if weight.dim() != 2:
        raise ValueError("weight must be a 2-D tensor (m, n)")
    bf16 = torch.bfloat16
    q8 = x_scale is not None
    ps = pb = pr = pm = pz = None
    ldr = 0
    if q8:
        ps = _vector(x_scale, "x_scale", torch.float32, dev, T)
        pm = _vector(row_scale, "row_scale", torch.float32, dev, m)
    if bias is not None:
        pb = _vector(bias, "bias", bf16, dev, m)
    shape = (T, m) if x.dim() == 2 else x.shape[:-1] + (m,)
    if residual is not None:
        pr, ldr, _, _ = _rows(residual, "residual", bf16, dev, m)
        if residual.shape != shape:
            raise ValueError(f"residual must have the output's shape {tuple(shape)}")
    y = torch.empty(shape, dtype=bf16, device=dev)
    z = None
    if keep_preact:
        z = torch.empty_like(y)
        pz = z.data_ptr()
    a = ff_linear_args(T, n, m, px, ldx, pw, ldw, ps, pm, pb, pr, ldr, _act(activation), y.data_ptr(), m, pz, m)
    keep = _workspace(a, _bytes("ff_linear_workspace_size", a, int(q8)), workspace, dev)
    if T:
        _launch(name, a, dev)
    del keep
    return y, z


def linear(x, weight, *, bias=None, residual=None, activation: str = "none", keep_preact: bool = False,
           workspace=None, stream=None):
    """(y, z) of a linear layer in bfloat16: z = x weight^T + bias (returned with
    keep_preact, what linear_backward needs; otherwise None), y = act(z) +
    residual.  x (..., n), weight (m, n); activation "none", "relu", "gelu" (the
    tanh form) or "silu"."""
    if stream is not None:
        return _on_stream(stream, linear, x, weight, bias=bias, residual=residual, activation=activation,
                          keep_preact=keep_preact, workspace=workspace)
    return _linear("ff_linear", x, weight, torch.bfloat16, None, None, bias, residual, activation, keep_preact,
                   workspace)


def linear_q8(q, q_scale, codes, row_scale, *, bias=None, residual=None, activation: str = "none",
              workspace=None, stream=None):
    """y (bfloat16) of a layer of codes on 8-bit rows: act(q_scale_t row_scale_i
    sum_j q_tj codes_ij + bias_i) + residual_ti.  q (..., n) and codes (m, n)
    int8, q_scale (...) and row_scale (m) float32: rows of rms_norm_q8 or
    quantize_rows with col_scale = alpha, codes Z and scales beta of
    FlipFlop.quantize.  The sums are exact."""
    if stream is not None:
        return _on_stream(stream, linear_q8, q, q_scale, codes, row_scale, bias=bias, residual=residual,
                          activation=activation, workspace=workspace)
    if q_scale is None or row_scale is None:
        raise TypeError("q_scale and row_scale must be CUDA tensors")
    return _linear("ff_linear_q8", q, codes, torch.int8, q_scale, row_scale, bias, residual, activation, False,
                   workspace)[0]


def linear_backward(dy, x, weight, *, preact=None, activation: str = "none", need_input: bool = True,
                    need_weight: bool = True, need_bias: bool = True, workspace=None, stream=None):
    """(dx, dw, g, db) of y = act(z) + residual for the gradient dy of y (which
    is the residual's own): g = dy act'(z) (dy itself without an activation),
    dx = g weight, dw = g^T x, db = sum of g, all of g rounded as it is returned;
    None for what is not needed.  The rows of x and of g are the tokens of
    FlipFlop(tokens=(x, g)).  x and preact may be checkpoints in 8 bits
    (checkpoint_q8); see ff_linear_backward_q8."""
    if stream is not None:
        return _on_stream(stream, linear_backward, dy, x, weight, preact=preact, activation=activation,
                          need_input=need_input, need_weight=need_weight, need_bias=need_bias, workspace=workspace)
    _library()
    bf16 = torch.bfloat16
    x8 = z8 = None
    if isinstance(x, Checkpoint):
        dev = _first(x.codes, "x.codes")
        x8, x = x, x.codes   # (its shape from here on)
        k8, T, n = _q8_rows(x8, "x", dev)
        px, ldx = None, 0
    else:
        dev = _first(x, "x")
        px, ldx, T, n = _rows(x, "x", bf16, dev)
    pw, ldw, m, _ = _rows(weight, "weight", bf16, dev, n)
    if weight.dim() != 2:
        raise ValueError("weight must be a 2-D tensor (m, n)")
    shape = (T, m) if x.dim() == 2 else x.shape[:-1] + (m,)
    pdy, lddy, _, _ = _rows(dy, "dy", bf16, dev, m)
    if dy.shape != shape:
        raise ValueError(f"dy must have the output's shape {tuple(shape)}")
    a = ff_linear_grad_args(T, n, m, pdy, lddy, px, ldx, pw, ldw)
    a.activation = _act(activation)
    g = dy
    if a.activation:
        if preact is None:
            raise ValueError(f"preact of shape {tuple(shape)} is needed with an activation")
        if isinstance(preact, Checkpoint):
            z8, preact = preact, preact.codes
            kz8, _, _ = _q8_rows(z8, "preact", dev, m)
        else:
            a.preact, a.ldz, _, _ = _rows(preact, "preact", bf16, dev, m)
        if preact.shape != shape:
            raise ValueError(f"preact must have the output's shape {tuple(shape)}")
        g = _like(dy, bf16)
        a.g, a.ldg = g.data_ptr(), m
    dx = dw = db = None
    if need_input:
        dx = _like(x, bf16)   # (also of a checkpoint's codes)
        a.dx, a.lddx = dx.data_ptr(), n
    if need_weight:
        dw = _like(weight, bf16)
        a.dw, a.lddw = dw.data_ptr(), n
    if need_bias:
        db = torch.empty(m, dtype=bf16, device=dev)
        a.db = db.data_ptr()
    if x8 is None and z8 is None:
        keep = _workspace(a, _bytes("ff_linear_backward_workspace_size", a), workspace, dev)
        _launch("ff_linear_backward", a, dev)
    else:
        _q8_library()
        q = ff_linear_grad_q8_args(a, k8 if x8 else ff_q8_rows(), kz8 if z8 else ff_q8_rows())
        keep = _workspace(q, _bytes("ff_linear_backward_q8_workspace_size", q, functions=_Q8_FN), workspace, dev)
        _launch("ff_linear_backward_q8", q, dev, _Q8_FN)
    del keep
    return dx, dw, g, db


# ------------------------------------------------------ checkpoints in 8 bits
class Checkpoint(NamedTuple):
    """Activations kept in 8 bits: codes (..., n) int8 and scale (..., ceil(n /
    group)) float32, the value of column j codes_j scale_{j // group}."""
    codes: torch.Tensor
    scale: torch.Tensor
    group: int


class ff_q8_rows(ctypes.Structure):
    _fields_ = [("q", _ptr), ("ldq", _i64), ("scale", _ptr), ("ld_scale", _i64), ("group", _i64)]


class ff_checkpoint_args(ctypes.Structure):
    _fields_ = [("rows", _i64), ("cols", _i64), ("dtype", _int), ("x", _ptr), ("ldx", _i64), ("kept", ff_q8_rows),
                ("stream", _ptr)]


class ff_linear_grad_q8_args(ctypes.Structure):
    _fields_ = [("grad", ff_linear_grad_args), ("x_q8", ff_q8_rows), ("preact_q8", ff_q8_rows)]

    def __setattr__(self, name, value):   # stream and workspace are the gradient's
        if name in ("stream", "workspace", "workspace_bytes"):
            setattr(self.grad, name, value)
        else:
            super().__setattr__(name, value)


_Q8_FN = {}


def _q8_library():
    if not _Q8_FN:
        lib, found, size = load_library(), {}, ctypes.POINTER(_size)
        for name, args in {"ff_checkpoint": ff_checkpoint_args, "ff_checkpoint_restore": ff_checkpoint_args,
                           "ff_linear_backward_q8": ff_linear_grad_q8_args,
                           "ff_linear_backward_q8_workspace_size": ff_linear_grad_q8_args}.items():
            f = getattr(lib, name)
            f.restype = _int
            f.argtypes = [ctypes.POINTER(args)] + ([size] if name.endswith("_size") else [])
            found[name] = f
        _Q8_FN.update(found)
    return _Q8_FN


def _group(group):
    if not isinstance(group, int) or group not in (16, 32, 64, 128, 256, 512):
        raise ValueError(f"group must be 16, 32, 64, 128, 256 or 512, not {group!r}")
    return group


def _q8_rows(kept, name, device, cols=None):
    """(ff_q8_rows, rows, columns) of a checkpoint."""
    group = _group(kept.group)
    pq, ldq, r, c = _rows(kept.codes, f"{name}.codes", torch.int8, device, cols)
    ps, lds, rs, _ = _rows(kept.scale, f"{name}.scale", torch.float32, device, (c + group - 1) // group)
    if kept.scale.shape[:-1] != kept.codes.shape[:-1]:
        raise ValueError(f"{name}.scale must have a row for each row of the codes, {r}, not {rs}")
    return ff_q8_rows(pq, ldq, ps, lds, group), r, c


def checkpoint_q8(x, *, group: int = 128, stream=None):
    """Checkpoint of x (..., n), float32 or bfloat16, in 8 bits: for each `group`
    columns scale = max |x| / 127 and codes = rint(127 x / max |x|), so that
    codes scale is off by at most half a scale.  linear_backward and
    expert_linear_backward take it for x or preact; checkpoint_restore gives
    rows for anything else."""
    if stream is not None:
        return _on_stream(stream, checkpoint_q8, x, group=group)
    _q8_library()
    dev = _first(x, "x")
    dt = _elem(x, "x")
    px, ldx, r, c = _rows(x, "x", x.dtype, dev)
    groups = (c + _group(group) - 1) // group
    if x.dim() == 2:
        q, scale = _matrix_of(r, c, torch.int8, dev), _matrix_of(r, groups, torch.float32, dev)
    else:
        q, scale = _like(x, torch.int8), torch.empty(x.shape[:-1] + (groups,), dtype=torch.float32, device=dev)
    if r:
        _launch("ff_checkpoint", ff_checkpoint_args(r, c, dt, px, ldx, ff_q8_rows(q.data_ptr(), c, scale.data_ptr(),
                                                                                   groups, group)), dev, _Q8_FN)
    return Checkpoint(q, scale, group)


def checkpoint_restore(kept, *, dtype=torch.bfloat16, stream=None):
    """The rows (..., n) that a checkpoint stands for, float32 or bfloat16."""
    if stream is not None:
        return _on_stream(stream, checkpoint_restore, kept, dtype=dtype)
    _q8_library()
    if not isinstance(kept, Checkpoint):
        raise TypeError("kept must be a Checkpoint")
    if dtype not in _ELEM:
        raise TypeError(f"dtype must be float32 or bfloat16, not {dtype}")
    dev = _first(kept.codes, "kept.codes")
    k, r, c = _q8_rows(kept, "kept", dev)
    x = _matrix_of(r, c, dtype, dev) if kept.codes.dim() == 2 else _like(kept.codes, dtype)
    if r:
        _launch("ff_checkpoint_restore", ff_checkpoint_args(r, c, _ELEM[dtype], x.data_ptr(), c, k), dev, _Q8_FN)
    return x


# ---------------------------------------------------------- orthogonalisation
def orthogonalize(G, *, steps: int = 5, coefficients=(3.4445, -4.7750, 2.0315), eps: float = 1e-7,
                  scale: float = 1.0, workspace=None, stream=None):
    """Updates G (m, n) or (batch, m, n), float32 or bfloat16, towards scale
    times the orthogonal factor of their polar decomposition: X = G / (||G||_F +
    eps), then `steps` times X <- a X + (b A + c A A) X with A = X X^T.  The
    coefficients have to keep singular values in [0, 1] below 16.  bfloat16 products take operands of 11 bits (results
    were off by 1.7e-3 of their norm, their own rounding, to 3.3e-3), float32 ones of 22."""
    if stream is not None:
        return _on_stream(stream, orthogonalize, G, steps=steps, coefficients=coefficients, eps=eps, scale=scale,
                          workspace=workspace)
    _library()
    dev = _first(G, "G")
    dt = _elem(G, "G")
    if G.dim() not in (2, 3):
        raise ValueError("G must be (m, n) or (batch, m, n)")
    m, n = G.shape[-2:]
    batch = G.shape[0] if G.dim() == 3 else 1
    if m < 1 or n < 1:
        raise ValueError("G must not be empty")
    if (n > 1 and G.stride(-1) != 1) or (m > 1 and G.stride(-2) < n):
        raise ValueError("the rows of G must be contiguous and must not overlap")
    if G.dim() == 3 and batch > 1 and G.stride(0) < 0:
        raise ValueError("the matrices of G must follow each other")
    a_, b_, c_ = (float(v) for v in coefficients)
    out = _like(G, G.dtype)
    a = ff_ortho_args(batch, m, n, dt, G.data_ptr(), G.stride(-2) if m > 1 else n,
                      G.stride(0) if G.dim() == 3 else m * n, out.data_ptr(), n, m * n, steps, a_, b_, c_, eps, scale)
    keep = _workspace(a, _bytes("ff_orthogonalize_workspace_size", a), workspace, dev)
    _launch("ff_orthogonalize", a, dev)
    del keep
    return out
