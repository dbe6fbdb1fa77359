"""Operators around a layer of experts: the router's choice and its gradient,
the experts' linear layers on the rows that are routed to each, and the sums of a
token's rows.

As in layer.py: one call of the HIP library (include/ff.h) on torch tensors, no
state, no autograd, results as new tensors, work on the device's current stream
or on `stream`, nothing waits; how many rows an expert has stays on the device.
A slot is a token's j-th choice, t top + j; rows are the slots sorted by expert.
The rows of expert e, r.offsets[e] to r.offsets[e + 1] of x and of g, are the
tokens of FlipFlop(tokens=(x, g)) of its layer.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

from .binding import load_library
from .layer import (Checkpoint, _act, _bytes, _elem, _first, _i64, _int, _f64, _launch, _like, _matrix_of, _on_stream, _ptr,
                    _q8_rows, _refuse, _rows, _size, _vector, _workspace, ff_q8_rows)

FF_SCORE_SOFTMAX, FF_SCORE_SIGMOID = 0, 1
SCORES = {"softmax": FF_SCORE_SOFTMAX, "sigmoid": FF_SCORE_SIGMOID}


class Routing(NamedTuple):
    """Which experts T tokens take and where their slots lie: weights (T, top)
    float32 (None: no weights), experts (T, top), order (T top), offsets (E + 1)
    and place (T, top) int32; see route.  With offsets[a : b + 1] for offsets (and
    their weights) the products take experts a .. b - 1 alone: rows of the others are
    in no expert."""
    weights: Optional[torch.Tensor]
    experts: torch.Tensor
    order: torch.Tensor
    offsets: torch.Tensor
    place: torch.Tensor


class ff_routing(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("experts", _i64), ("top", _i64), ("weights", _ptr), ("order", _ptr),
                ("offsets", _ptr), ("place", _ptr)]


class ff_route_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("experts", _i64), ("top", _i64), ("dtype", _int), ("logits", _ptr), ("ldl", _i64),
                ("bias", _ptr), ("mask", _ptr), ("score", _int), ("groups", _i64), ("top_groups", _i64),
                ("renormalise", _int), ("scale", _f64), ("weights", _ptr), ("chosen", _ptr), ("order", _ptr),
                ("offsets", _ptr), ("place", _ptr), ("workspace", _ptr), ("workspace_bytes", _size), ("stream", _ptr)]


class ff_route_grad_args(ctypes.Structure):
    _fields_ = [("tokens", _i64), ("experts", _i64), ("top", _i64), ("dtype", _int), ("logits", _ptr), ("ldl", _i64),
                ("dweights", _ptr), ("chosen", _ptr), ("score", _int), ("renormalise", _int), ("scale", _f64),
                ("dlogits", _ptr), ("ldd", _i64), ("stream", _ptr)]


class ff_expert_linear_args(ctypes.Structure):
    _fields_ = [("routing", ff_routing), ("n", _i64), ("m", _i64), ("x", _ptr), ("ldx", _i64), ("by_slot", _int),
                ("w", _ptr), ("ldw", _i64), ("bias", _ptr), ("activation", _int), ("y", _ptr), ("ldy", _i64),
                ("preact", _ptr), ("ldz", _i64), ("workspace", _ptr), ("workspace_bytes", _size), ("stream", _ptr)]


class ff_expert_combine_args(ctypes.Structure):
    _fields_ = [("routing", ff_routing), ("cols", _i64), ("y", _ptr), ("ldy", _i64), ("residual", _ptr), ("ldr", _i64),
                ("out", _ptr), ("ldo", _i64), ("stream", _ptr)]


class ff_expert_combine_grad_args(ctypes.Structure):
    _fields_ = [("routing", ff_routing), ("cols", _i64), ("dout", _ptr), ("ldd", _i64), ("y", _ptr), ("ldy", _i64),
                ("dy", _ptr), ("lddy", _i64), ("dweights", _ptr), ("stream", _ptr)]


class ff_expert_grad_args(ctypes.Structure):
    _fields_ = [("routing", ff_routing), ("n", _i64), ("m", _i64), ("dy_dtype", _int), ("dy", _ptr), ("lddy", _i64),
                ("x", _ptr), ("ldx", _i64), ("x_q8", ff_q8_rows), ("by_slot", _int), ("w", _ptr), ("ldw", _i64),
                ("preact", _ptr), ("ldz", _i64), ("preact_q8", ff_q8_rows), ("activation", _int), ("g", _ptr),
                ("ldg", _i64), ("dx", _ptr), ("lddx", _i64), ("dw", _ptr), ("lddw", _i64), ("db", _ptr),
                ("workspace", _ptr), ("workspace_bytes", _size), ("stream", _ptr)]


_FN = {}


def _library():
    if not _FN:
        lib, found, size = load_library(), {}, ctypes.POINTER(_size)
        for name, args in {"ff_route": ff_route_args, "ff_route_workspace_size": ff_route_args,
                           "ff_expert_order": ff_route_args, "ff_route_backward": ff_route_grad_args,
                           "ff_expert_linear": ff_expert_linear_args,
                           "ff_expert_linear_workspace_size": ff_expert_linear_args,
                           "ff_expert_combine": ff_expert_combine_args,
                           "ff_expert_combine_backward": ff_expert_combine_grad_args,
                           "ff_expert_linear_backward": ff_expert_grad_args,
                           "ff_expert_linear_backward_workspace_size": ff_expert_grad_args}.items():
            f = getattr(lib, name)
            f.restype = _int
            f.argtypes = [ctypes.POINTER(args)] + ([size] if name.endswith("_size") else [])
            found[name] = f
        _FN.update(found)   # all at once: other threads see none or all of them
    return _FN


# -------------------------------------------------------------------- routing
def _score(name):
    try:
        return SCORES[name]
    except (KeyError, TypeError):
        raise ValueError(f"score must be one of {sorted(SCORES)}, not {name!r}") from None


def _count(value, name):
    if not isinstance(value, int) or isinstance(value, bool) or value < 1:
        raise ValueError(f"{name} must be a whole number >= 1, not {value!r}")
    return value


def _matrix(t, name, dtype, device, cols=None):
    """_rows of a 2-D tensor."""
    p, ld, r, c = _rows(t, name, dtype, device, cols)
    if t.dim() != 2:
        raise ValueError(f"{name} must be a 2-D tensor")
    return p, ld, r, c


def _slots(t, name, dtype, device, shape):
    """Pointer of a contiguous tensor of that shape."""
    p = _vector(t, name, dtype, device, shape.numel())
    if p is None or t.shape != shape:
        raise ValueError(f"{name} must be a tensor of shape {tuple(shape)}")
    return p


def _new_routing(a, tokens, experts, top, dev, choose):
    """experts (with choose), place, order and offsets of one allocation, for args a."""
    slots = tokens * top
    sizes = [slots, slots, slots, experts + 1] if choose else [slots, slots, experts + 1]
    all_ = torch.empty_strided((sum(sizes),), (1,), dtype=torch.int32, device=dev)
    parts, at = all_.split_with_sizes(sizes), all_.data_ptr()
    chosen = None
    if choose:
        chosen, parts, a.chosen = parts[0].view(tokens, top), parts[1:], at
        at += 4 * slots
    a.place, a.order, a.offsets = at, at + 4 * slots, at + 8 * slots
    return chosen, parts[1], parts[2], parts[0].view(tokens, top)


def route(logits, top: int, *, score: str = "softmax", bias=None, groups: int = 1, top_groups: int = 1,
          renormalise: bool = True, scale: float = 1.0, mask=None, workspace=None, stream=None):
    """Routing of T tokens by their logits (T, E), float32 or bfloat16, to `top` of
    E experts: s = softmax or sigmoid of the logits, chosen are the largest s +
    bias (bias (E) float32) in their order, the lowest index among equals, of the
    top_groups of `groups` groups whose two largest sum to most; weights are
    scale s, or with renormalise scale s over the sum of the chosen s.  Tokens
    whose mask (T) bool is False take no expert (experts -1, weights 0, no row).
    Choices are made in 64 bits.  See ff_route for rows that are not finite."""
    if stream is not None:
        return _on_stream(stream, route, logits, top, score=score, bias=bias, groups=groups, top_groups=top_groups,
                          renormalise=renormalise, scale=scale, mask=mask, workspace=workspace)
    _library()
    dev = _first(logits, "logits")
    dt = _elem(logits, "logits")
    p, ld, T, E = _matrix(logits, "logits", logits.dtype, dev)
    top = _count(top, "top")
    weights = _matrix_of(T, top, torch.float32, dev)
    a = ff_route_args(T, E, top, dt, p, ld, _vector(bias, "bias", torch.float32, dev, E),
                      _vector(mask, "mask", torch.bool, dev, T), _score(score), _count(groups, "groups"),
                      _count(top_groups, "top_groups"), 1 if renormalise else 0, scale, weights.data_ptr())
    experts, order, offsets, place = _new_routing(a, T, E, top, dev, True)
    keep = _workspace(a, _bytes("ff_route_workspace_size", a, functions=_FN), workspace, dev)
    _launch("ff_route", a, dev, _FN)
    del keep
    return Routing(weights, experts, order, offsets, place)


def expert_order(experts, num_experts: int, *, weights=None, workspace=None, stream=None):
    """The Routing of choices that are there already: experts (T, top) int32, where
    anything outside 0 .. num_experts - 1 is not routed, and weights (T, top)
    float32 (None: none)."""
    if stream is not None:
        return _on_stream(stream, expert_order, experts, num_experts, weights=weights, workspace=workspace)
    _library()
    dev = _first(experts, "experts")
    if experts.dim() != 2:
        raise ValueError("experts must be a 2-D tensor (T, top)")
    p = _slots(experts, "experts", torch.int32, dev, experts.shape)
    if weights is not None:
        _slots(weights, "weights", torch.float32, dev, experts.shape)
    T, top = experts.shape
    a = ff_route_args(T, _count(num_experts, "num_experts"), top)
    a.chosen = p
    _, order, offsets, place = _new_routing(a, T, num_experts, top, dev, False)
    keep = _workspace(a, _bytes("ff_route_workspace_size", a, functions=_FN), workspace, dev)
    _launch("ff_expert_order", a, dev, _FN)
    del keep
    return Routing(weights, experts, order, offsets, place)


def route_backward(dweights, logits, experts, *, score: str = "softmax", renormalise: bool = True, scale: float = 1.0,
                   stream=None):
    """The logits' gradient (T, E), in their type, for the gradient dweights (T, top)
    float32 of the weights of route, whose choice `experts` (and the bias behind
    it) counts as a constant."""
    if stream is not None:
        return _on_stream(stream, route_backward, dweights, logits, experts, score=score, renormalise=renormalise,
                          scale=scale)
    _library()
    dev = _first(logits, "logits")
    dt = _elem(logits, "logits")
    p, ld, T, E = _matrix(logits, "logits", logits.dtype, dev)
    if not isinstance(experts, torch.Tensor) or experts.dim() != 2 or experts.shape[0] != T:
        raise ValueError(f"experts must be a tensor of shape ({T}, top)")
    out = _matrix_of(T, E, logits.dtype, dev)
    a = ff_route_grad_args(T, E, experts.shape[1], dt, p, ld,
                           _slots(dweights, "dweights", torch.float32, dev, experts.shape),
                           _slots(experts, "experts", torch.int32, dev, experts.shape), _score(score),
                           1 if renormalise else 0, scale, out.data_ptr(), E)
    _launch("ff_route_backward", a, dev, _FN)
    return out


# ------------------------------------------------------------------- products
def _routing(r, device):
    """ff_routing of r."""
    if not isinstance(r, Routing):
        raise TypeError("routing must be a Routing")
    w, e, o, f, p = r
    i32 = torch.int32
    try:   # (what is right is taken at once: 1 us less than argument by argument)
        T, top = shape = e.shape
        if (o.dtype is i32 and f.dtype is i32 and p.dtype is i32 and e.device == device and o.device == device
                and f.device == device and p.device == device and p.shape == shape and o.shape == (T * top,)
                and f.dim() == 1 and f.shape[0] > 1 and o.is_contiguous() and f.is_contiguous() and p.is_contiguous()
                and (w is None or (w.dtype is torch.float32 and w.device == device and w.shape == shape
                                   and w.is_contiguous()))):
            return ff_routing(T, f.shape[0] - 1, top, None if w is None else w.data_ptr(), o.data_ptr(), f.data_ptr(),
                              p.data_ptr())
    except (AttributeError, TypeError, ValueError):
        pass
    if not isinstance(e, torch.Tensor) or e.dim() != 2:
        raise ValueError("routing.experts must be a 2-D tensor (T, top)")
    if e.device != device:
        _refuse(e, "routing.experts", e.dtype, device)
    shape = e.shape
    if w is not None:
        _slots(w, "routing.weights", torch.float32, device, shape)
    _slots(o, "routing.order", i32, device, torch.Size((shape.numel(),)))
    _slots(p, "routing.place", i32, device, shape)
    if not isinstance(f, torch.Tensor) or f.dim() != 1 or f.numel() < 2:
        raise ValueError("routing.offsets must be a 1-D tensor of E + 1 elements")
    _vector(f, "routing.offsets", i32, device, f.numel())
    raise ValueError("routing is not one of this device")


def _weights(w, device, experts, n=None):
    """(pointer, ld, m, n) of the experts' weights (E, m, n)."""
    if not isinstance(w, torch.Tensor) or w.dtype is not torch.bfloat16 or w.device != device:
        _refuse(w, "weight", torch.bfloat16, device)
    if w.dim() != 3 or w.shape[0] != experts or (n is not None and w.shape[2] != n) or w.shape[1] < 1 or w.shape[2] < 1:
        raise ValueError(f"weight must be a tensor ({experts}, m, {'n' if n is None else n}), not {tuple(w.shape)}")
    if not w.is_contiguous():
        raise ValueError("weight must be contiguous")
    return w.data_ptr(), w.shape[2], w.shape[1], w.shape[2]


def _bias(b, device, experts, m):
    if b is None:
        return None
    p = _vector(b, "bias", torch.bfloat16, device, experts * m)
    if b.shape != (experts, m):
        raise ValueError(f"bias must be a tensor of shape ({experts}, {m})")
    return p


def _slot_rows(t, name, dtype, device, r, by_slot, cols=None):
    p, ld, rows, c = _matrix(t, name, dtype, device, cols)
    want = r.tokens * r.top if by_slot else r.tokens
    if rows != want:
        raise ValueError(f"{name} must have a row for each {'slot' if by_slot else 'token'}, {want}, not {rows}")
    return p, ld, c


def expert_linear(x, weight, routing, *, bias=None, activation: str = "none", keep_preact: bool = False,
                  by_slot: bool = False, workspace=None, stream=None):
    """(y, z) of the experts' layers in bfloat16 on the rows of a routed batch: z =
    x weight_e^T + bias_e (returned with keep_preact, otherwise None), y = act(z),
    both (T top, m), zeros in rows of no expert.  x: the tokens' rows (T, n), or
    with by_slot a row for each slot (T top, n); weight (E, m, n), bias (E, m)."""
    if stream is not None:
        return _on_stream(stream, expert_linear, x, weight, routing, bias=bias, activation=activation,
                          keep_preact=keep_preact, by_slot=by_slot, workspace=workspace)
    if not _FN:
        _library()
    dev = _first(x, "x")
    bf16 = torch.bfloat16
    r = _routing(routing, dev)
    px, ldx, n = _slot_rows(x, "x", bf16, dev, r, by_slot)
    pw, ldw, m, _ = _weights(weight, dev, r.experts, n)
    rows = r.tokens * r.top
    y = _matrix_of(rows, m, bf16, dev)
    z = _matrix_of(rows, m, bf16, dev) if keep_preact else None
    a = ff_expert_linear_args(r, n, m, px, ldx, 1 if by_slot else 0, pw, ldw, _bias(bias, dev, r.experts, m),
                              _act(activation), y.data_ptr(), m, z.data_ptr() if keep_preact else None, m)
    if r.tokens:
        keep = _workspace(a, _bytes("ff_expert_linear_workspace_size", a, functions=_FN), workspace, dev)
        _launch("ff_expert_linear", a, dev, _FN)
        del keep
    return y, z


def expert_combine(y, routing, *, residual=None, stream=None):
    """(T, m) bfloat16: residual_t plus the sum of a token's rows of y (T top, m),
    each times its weight (one without weights)."""
    if stream is not None:
        return _on_stream(stream, expert_combine, y, routing, residual=residual)
    if not _FN:
        _library()
    dev = _first(y, "y")
    r = _routing(routing, dev)
    py, ldy, m = _slot_rows(y, "y", torch.bfloat16, dev, r, True)
    pr = ldr = 0
    if residual is not None:
        pr, ldr, _ = _slot_rows(residual, "residual", torch.bfloat16, dev, r, False, m)
    out = _matrix_of(r.tokens, m, torch.bfloat16, dev)
    if r.tokens:
        _launch("ff_expert_combine", ff_expert_combine_args(r, m, py, ldy, pr, ldr, out.data_ptr(), m), dev, _FN)
    return out


def expert_combine_backward(dout, y, routing, *, need_rows: bool = True, need_weights: bool = True, stream=None):
    """(dy, dweights) of expert_combine for the gradient dout (T, m) of its result
    (which is the residual's own): dy (T top, m) float32, each row its weight
    times its token's dout (expert_linear_backward rounds it once, as part of g),
    dweights (T, top) float32, the products <dout_t, y> of its rows; None for what
    is not needed."""
    if stream is not None:
        return _on_stream(stream, expert_combine_backward, dout, y, routing, need_rows=need_rows,
                          need_weights=need_weights)
    _library()
    dev = _first(dout, "dout")
    r = _routing(routing, dev)
    if routing.weights is None:
        raise ValueError("routing has no weights")
    pd, ldd, m = _slot_rows(dout, "dout", torch.bfloat16, dev, r, False)
    a = ff_expert_combine_grad_args(r, m, pd, ldd)
    dy = dweights = None
    if need_weights:
        a.y, a.ldy, _ = _slot_rows(y, "y", torch.bfloat16, dev, r, True, m)
        dweights = _matrix_of(r.tokens, r.top, torch.float32, dev)
        a.dweights = dweights.data_ptr()
    if need_rows:
        dy = _matrix_of(r.tokens * r.top, m, torch.float32, dev)
        a.dy, a.lddy = dy.data_ptr(), m
    if r.tokens:
        _launch("ff_expert_combine_backward", a, dev, _FN)
    return dy, dweights


def expert_linear_backward(dy, x, weight, routing, *, preact=None, activation: str = "none", by_slot: bool = False,
                           need_input: bool = True, need_weight: bool = True, need_bias: bool = True, workspace=None,
                           stream=None):
    """(dx, dw, g, db) of expert_linear for the gradient dy (T top, m), bfloat16 or
    float32, of y: g = dy act'(z) by rows, dx = g weight_e (T top, n), or without
    by_slot summed over each token's rows (T, n), dw (E, m, n) = g^T x and db (E, m)
    = sum of g of each expert's rows, all bfloat16; None for what is not needed.  x
    and preact may be checkpoints in 8 bits (checkpoint_q8)."""
    if stream is not None:
        return _on_stream(stream, expert_linear_backward, dy, x, weight, routing, preact=preact, activation=activation,
                          by_slot=by_slot, need_input=need_input, need_weight=need_weight, need_bias=need_bias,
                          workspace=workspace)
    _library()
    bf16 = torch.bfloat16
    dev = _first(dy, "dy")
    r = _routing(routing, dev)
    pdy, lddy, m = _slot_rows(dy, "dy", dy.dtype, dev, r, True)
    a = ff_expert_grad_args()
    a.routing, a.m, a.dy_dtype, a.dy, a.lddy = r, m, _elem(dy, "dy"), pdy, lddy
    a.by_slot = 1 if by_slot else 0
    X = r.tokens * r.top if by_slot else r.tokens

    def kept(v, name, rows, cols):
        k, have, c = _q8_rows(v, name, dev, cols)
        if v.codes.dim() != 2 or have != rows:
            raise ValueError(f"{name} must have {rows} rows")
        return k, c
    if isinstance(x, Checkpoint):
        a.x_q8, n = kept(x, "x", X, None)
    else:
        a.x, a.ldx, n = _slot_rows(x, "x", bf16, dev, r, by_slot)
    a.n = n
    a.w, a.ldw, wm, _ = _weights(weight, dev, r.experts, n)
    if wm != m:
        raise ValueError(f"dy must have rows of {wm} elements, not {m}")
    a.activation = _act(activation)
    if a.activation:
        if preact is None:
            raise ValueError(f"preact of shape {(r.tokens * r.top, m)} is needed with an activation")
        if isinstance(preact, Checkpoint):
            a.preact_q8, _ = kept(preact, "preact", r.tokens * r.top, m)
        else:
            a.preact, a.ldz, _ = _slot_rows(preact, "preact", bf16, dev, r, True, m)
    g = _matrix_of(r.tokens * r.top, m, bf16, dev)
    a.g, a.ldg = g.data_ptr(), m
    dx = dw = db = None
    if need_input:
        dx = _matrix_of(X, n, bf16, dev)
        a.dx, a.lddx = dx.data_ptr(), n
    if need_weight:
        dw = torch.empty_like(weight)
        a.dw, a.lddw = dw.data_ptr(), n
    if need_bias:
        db = _matrix_of(r.experts, m, bf16, dev)
        a.db = db.data_ptr()
    keep = _workspace(a, _bytes("ff_expert_linear_backward_workspace_size", a, functions=_FN), workspace, dev)
    _launch("ff_expert_linear_backward", a, dev, _FN)
    del keep
    return dx, dw, g, db
