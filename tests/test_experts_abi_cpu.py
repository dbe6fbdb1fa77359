"""Host-side checks of the C ABI around a layer of experts and of checkpoints (no GPU
needed): bad arguments are refused before a device is touched."""
import ctypes
import os
import types

import pytest

import paper_2609_14706_amd as ff
from paper_2609_14706_amd import experts

P = 1 << 40    # an aligned address that is never read; blocks are P apart


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(ff.LIB_PATH):
        from paper_2609_14706_amd.build import build
        build()
    return ff.load_library()


def _code(lib, name, args):
    code = getattr(lib, name)(ctypes.byref(args))
    assert code == 0 or ff.ff_last_error()
    return code


def _set(a, kw):
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def route(**kw):
    return _set(ff.ff_route_args(8, 12, 2, 0, P, 12, 2 * P, 3 * P, 0, 4, 2, 1, 1.0, 4 * P, 5 * P, 6 * P, 7 * P, 8 * P), kw)


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(tokens=(1 << 24) + 1), dict(tokens=1 << 24), dict(experts=0), dict(experts=1025), dict(top=0),
    dict(top=65), dict(top=7), dict(dtype=2), dict(logits=None), dict(logits=P + 2), dict(ldl=11), dict(bias=2 * P + 2),
    dict(score=2), dict(score=-1), dict(groups=5), dict(groups=-1), dict(groups=128), dict(top_groups=0), dict(top_groups=5),
    dict(renormalise=2), dict(scale=float("nan")), dict(scale=1e300), dict(weights=None), dict(weights=4 * P + 1),
    dict(chosen=None), dict(chosen=5 * P + 2), dict(order=None), dict(offsets=None), dict(place=None), dict(place=8 * P + 2),
    dict(weights=P), dict(chosen=4 * P), dict(order=5 * P), dict(place=6 * P), dict(offsets=3 * P)])
def test_route_refusals(lib, kw):
    assert _code(lib, "ff_route", route(**kw)) == ff.FF_ERR_INVALID_ARG


def test_order_refusals(lib):
    for kw in (dict(order=None), dict(offsets=None), dict(place=None), dict(chosen=None), dict(chosen=6 * P), dict(experts=0)):
        assert _code(lib, "ff_expert_order", route(**kw)) == ff.FF_ERR_INVALID_ARG
    for kw in (dict(workspace=None), dict(workspace=9 * P + 8, workspace_bytes=1 << 30), dict(workspace=9 * P, workspace_bytes=64)):
        assert _code(lib, "ff_route", route(tokens=1000, **kw)) == ff.FF_ERR_WORKSPACE
        assert _code(lib, "ff_expert_order", route(tokens=1000, **kw)) == ff.FF_ERR_WORKSPACE


def test_route_workspace(lib):
    size = ctypes.c_size_t(7)
    for T, some in ((0, False), (1, False), (64, False), (65, True), (1 << 20, True)):
        assert lib.ff_route_workspace_size(ctypes.byref(route(tokens=T)), ctypes.byref(size)) == 0
        assert (size.value > 0) == some
    assert lib.ff_route_workspace_size(None, ctypes.byref(size)) == 1
    assert lib.ff_route_workspace_size(ctypes.byref(route()), None) == 1
    for name in ("ff_route", "ff_expert_order", "ff_route_backward", "ff_expert_linear", "ff_expert_combine",
                 "ff_expert_combine_backward", "ff_expert_linear_backward", "ff_checkpoint", "ff_checkpoint_restore",
                 "ff_linear_backward_q8"):
        assert getattr(lib, name)(None) == ff.FF_ERR_INVALID_ARG


@pytest.mark.parametrize("kw", [
    dict(tokens=-1), dict(experts=0), dict(top=65), dict(dtype=3), dict(logits=None), dict(ldl=2), dict(dweights=None),
    dict(dweights=2 * P + 1), dict(chosen=None), dict(score=9), dict(renormalise=-1), dict(scale=float("inf")),
    dict(dlogits=None), dict(ldd=11), dict(dlogits=P, ldd=13), dict(dlogits=P + 4), dict(dlogits=2 * P)])
def test_route_gradient_refusals(lib, kw):
    a = ff.ff_route_grad_args(8, 12, 2, 0, P, 12, 2 * P, 3 * P, 0, 1, 1.0, 4 * P, 12)
    assert _code(lib, "ff_route_backward", _set(a, kw)) == ff.FF_ERR_INVALID_ARG
    assert _code(lib, "ff_route_backward", _set(a, dict(kw, tokens=0, experts=12, top=2, dtype=0, score=0, renormalise=1, scale=1.0))) == 0


def routing(**kw):
    return _set(ff.ff_routing(10, 4, 3, 20 * P, 21 * P, 22 * P, 23 * P), kw)


def linear(r=None, **kw):
    return _set(ff.ff_expert_linear_args(routing(**(r or {})), 64, 32, P, 64, 0, 2 * P, 64, None, 0, 3 * P, 32), kw)


@pytest.mark.parametrize("r,kw", [
    (dict(tokens=-1), {}), (dict(tokens=1 << 23), {}), (dict(experts=0), {}), (dict(experts=2000), {}), (dict(top=0), {}),
    (dict(order=None), {}), (dict(offsets=None), {}), (dict(order=21 * P + 1), {}), ({}, dict(n=0)), ({}, dict(m=(1 << 20) + 1)),
    ({}, dict(x=None)), ({}, dict(x=P + 1)), ({}, dict(ldx=63)), ({}, dict(w=None)), ({}, dict(ldw=8)), ({}, dict(bias=5 * P + 1)),
    ({}, dict(activation=4)), ({}, dict(activation=-1)), ({}, dict(by_slot=2)), ({}, dict(y=None)), ({}, dict(ldy=31)),
    ({}, dict(preact=4 * P, ldz=4)), ({}, dict(preact=3 * P + 64, ldz=32)), ({}, dict(y=P)), ({}, dict(y=2 * P)),
    ({}, dict(y=22 * P)), ({}, dict(y=21 * P))])
def test_linear_refusals(lib, r, kw):
    assert _code(lib, "ff_expert_linear", linear(r, **kw)) == ff.FF_ERR_INVALID_ARG


def test_linear_workspaces(lib):
    size = ctypes.c_size_t(7)

    def need(r=None, **kw):
        a = linear(r, **kw)
        assert lib.ff_expert_linear_workspace_size(ctypes.byref(a), ctypes.byref(size)) == 0
        return size.value
    many = dict(tokens=4000)
    assert need() == 0 and need(dict(tokens=0)) == 0      # few rows are taken as they lie
    assert need(many) == 0
    assert need(many, x=P + 2) > 0 and need(many, ldx=65) > 0 and need(many, w=2 * P + 2) > 0
    both = need(many, n=63)
    assert both >= 2 * 64 * (4000 + 4 * 32)
    # rows of tokens that lie beyond 2^31 bytes are laid out for each slot
    assert need(many, ldx=1 << 20) >= 4000 * 3 * 64 * 2 and need(many, ldx=1 << 20, by_slot=1) == 0
    a = linear(many, n=63)
    assert _code(lib, "ff_expert_linear", a) == ff.FF_ERR_WORKSPACE
    assert lib.ff_expert_linear_workspace_size(ctypes.byref(linear(dict(top=0))), ctypes.byref(size)) == 1
    assert lib.ff_expert_linear_workspace_size(ctypes.byref(linear()), None) == 1


@pytest.mark.parametrize("r,kw", [
    (dict(place=None), {}), (dict(offsets=None), {}), (dict(weights=20 * P + 2), {}), ({}, dict(cols=0)), ({}, dict(y=None)),
    ({}, dict(ldy=3)), ({}, dict(out=None)), ({}, dict(out=2 * P)), ({}, dict(residual=4 * P, ldr=1)), ({}, dict(ldo=0)),
    ({}, dict(residual=3 * P + 2, ldr=64)), ({}, dict(out=23 * P)), ({}, dict(out=20 * P))])
def test_combine_refusals(lib, r, kw):
    a = ff.ff_expert_combine_args(routing(**r), 64, 2 * P, 64, None, 0, 3 * P, 64)
    assert _code(lib, "ff_expert_combine", _set(a, kw)) == ff.FF_ERR_INVALID_ARG


@pytest.mark.parametrize("r,kw", [
    (dict(place=None), {}), (dict(order=None), {}), (dict(weights=None), {}), ({}, dict(cols=-1)), ({}, dict(dout=None)),
    ({}, dict(y=None)), ({}, dict(lddy=8)), ({}, dict(dy=4 * P + 2)), ({}, dict(dweights=5 * P + 1)), ({}, dict(dy=2 * P)),
    ({}, dict(dweights=4 * P)), ({}, dict(dweights=20 * P)), ({}, dict(ldd=8))])
def test_combine_gradient_refusals(lib, r, kw):
    a = ff.ff_expert_combine_grad_args(routing(**r), 64, 2 * P, 64, 3 * P, 64, 4 * P, 64, 5 * P)
    assert _code(lib, "ff_expert_combine_backward", _set(a, kw)) == ff.FF_ERR_INVALID_ARG


def grad(r=None, **kw):
    a = ff.ff_expert_grad_args()
    a.routing = routing(**(r or {}))
    base = dict(n=64, m=32, dy_dtype=1, dy=P, lddy=32, x=2 * P, ldx=64, w=3 * P, ldw=64, preact=4 * P, ldz=32, activation=1,
                g=5 * P, ldg=32, dx=6 * P, lddx=64, dw=7 * P, lddw=64, db=8 * P, workspace=9 * P, workspace_bytes=1 << 30)
    return _set(a, {**base, **kw})


def q8(q=10 * P, ldq=64, scale=11 * P, ld_scale=1, group=64):
    return ff.ff_q8_rows(q, ldq, scale, ld_scale, group)


@pytest.mark.parametrize("r,kw", [
    (dict(order=None), {}), (dict(place=None), {}), (dict(offsets=None), {}), ({}, dict(n=0)), ({}, dict(dy_dtype=2)),
    ({}, dict(dy=None)), ({}, dict(dy=P + 2, dy_dtype=0)), ({}, dict(lddy=31)), ({}, dict(x=None)), ({}, dict(ldx=8)),
    ({}, dict(w=None)), ({}, dict(preact=None)), ({}, dict(activation=9)), ({}, dict(by_slot=3)), ({}, dict(g=P)),
    ({}, dict(dx=2 * P)), ({}, dict(dw=3 * P)), ({}, dict(dw=None, dx=None, db=8 * P + 1)), ({}, dict(lddx=1)), ({}, dict(lddw=1)),
    ({}, dict(dx=7 * P)), ({}, dict(db=22 * P)), ({}, dict(x_q8=q8())), ({}, dict(x=None, x_q8=q8(group=24))),
    ({}, dict(x=None, x_q8=q8(group=8))), ({}, dict(x=None, x_q8=q8(group=1024))), ({}, dict(x=None, x_q8=q8(scale=None))),
    ({}, dict(x=None, x_q8=q8(ldq=63))), ({}, dict(x=None, x_q8=q8(group=32))), ({}, dict(x=None, x_q8=q8(scale=11 * P + 2))),
    ({}, dict(preact_q8=q8())), ({}, dict(preact=None, preact_q8=q8(ldq=31))), ({}, dict(x=None, x_q8=q8(q=7 * P))),
    ({}, dict(x=None, x_q8=q8(scale=5 * P)))])
def test_gradient_refusals(lib, r, kw):
    assert _code(lib, "ff_expert_linear_backward", grad(r, **kw)) == ff.FF_ERR_INVALID_ARG


def test_gradient_workspace(lib):
    size = ctypes.c_size_t(0)

    def need(**kw):
        assert lib.ff_expert_linear_backward_workspace_size(ctypes.byref(grad(**kw)), ctypes.byref(size)) == 0
        return size.value
    assert need(by_slot=1, db=None) == 0 < need(by_slot=1)    # everything is read as it lies, db has sums of its own
    assert need() > 0 and need(by_slot=1, ldw=65) > 0 and need(by_slot=1, x=None, x_q8=q8()) > 0
    assert need(by_slot=1, g=None, db=None) > 0 and need(by_slot=1, g=None, dx=None, dw=None, db=None) == 0
    for kw in (dict(workspace=None), dict(workspace=9 * P + 1), dict(workspace_bytes=16)):
        assert _code(lib, "ff_expert_linear_backward", grad(**kw)) == ff.FF_ERR_WORKSPACE


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=(1 << 32) + 1), dict(cols=0), dict(cols=(1 << 24) + 1), dict(dtype=2), dict(x=None), dict(x=P + 1),
    dict(ldx=99), dict(kept=q8(ldq=100, group=60)), dict(kept=q8(ldq=100, group=0)), dict(kept=q8(ldq=99, ld_scale=2)),
    dict(kept=q8(ldq=100, ld_scale=1)), dict(kept=q8(q=None, ldq=100, ld_scale=2)), dict(kept=q8(q=P, ldq=100, ld_scale=2)),
    dict(kept=q8(ldq=100, ld_scale=2, scale=P)), dict(kept=q8(ldq=100, ld_scale=2, scale=10 * P))])
def test_checkpoint_refusals(lib, kw):
    a = _set(ff.ff_checkpoint_args(8, 100, 0, P, 100, q8(ldq=100, ld_scale=2)), kw)
    for name in ("ff_checkpoint", "ff_checkpoint_restore"):
        assert _code(lib, name, a) == ff.FF_ERR_INVALID_ARG


def test_linear_gradient_from_checkpoints(lib):
    def args(x_q8=None, preact_q8=None, **kw):
        g = ff.ff_linear_grad_args(8, 64, 32, P, 32, None, 0, 3 * P, 64, None, 0, 1, 5 * P, 32, 6 * P, 64, 7 * P, 64, 8 * P,
                                   9 * P, 1 << 30)
        return ff.ff_linear_grad_q8_args(_set(g, kw), x_q8 or q8(), preact_q8 or q8(q=12 * P, ldq=32, scale=13 * P))
    for a in (args(x=2 * P, ldx=64), args(preact=4 * P, ldz=32), args(x_q8=q8(group=48)), args(x_q8=q8(scale=None)),
              args(preact_q8=q8(ldq=8)), args(x_q8=q8(q=7 * P)), args(x_q8=q8(scale=6 * P)), args(preact_q8=q8(q=5 * P, ldq=32)),
              args(x_q8=ff.ff_q8_rows()), args(preact_q8=ff.ff_q8_rows())):
        assert _code(lib, "ff_linear_backward_q8", a) == ff.FF_ERR_INVALID_ARG
    assert _code(lib, "ff_linear_backward_q8", args(workspace=None)) == ff.FF_ERR_WORKSPACE
    size = ctypes.c_size_t(0)
    assert lib.ff_linear_backward_q8_workspace_size(ctypes.byref(args()), ctypes.byref(size)) == 0 and size.value > 0
    assert lib.ff_linear_backward_q8_workspace_size(ctypes.byref(args(tokens=0)), ctypes.byref(size)) == 0 and size.value == 0
    assert lib.ff_linear_backward_q8_workspace_size(ctypes.byref(args(tokens=-1)), ctypes.byref(size)) == 1
    assert lib.ff_linear_backward_q8_workspace_size(None, ctypes.byref(size)) == 1


def test_another_thread_during_the_first_call(monkeypatch):
    """The table of functions is empty or whole at every moment."""
    seen = []

    class Library:
        def __getattr__(self, name):
            seen.append(len(experts._FN))
            return types.SimpleNamespace(name=name)
    monkeypatch.setattr(experts, "_FN", {})
    monkeypatch.setattr(experts, "load_library", Library)
    made = experts._library()
    assert len(seen) == len(made) and not any(seen) and experts._library() is experts._FN
