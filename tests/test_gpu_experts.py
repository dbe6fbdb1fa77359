"""expert_linear, expert_combine and their gradients against the formulas in 64 bits.

Tolerances as for the linear layer: an fp32 sum of n terms is off by at most n 2^-24
of the sum of magnitudes, slopes are below 1.13 and activations good to 2^-18,
outputs are rounded once (bf16 2^-8, fp32 2^-24); g is rounded to bf16 before dx, dw
and db read it, which the comparison with the returned g leaves out.  From a
checkpoint dw reads g and x in fp16: 2^-11 of each (g unrounded: 2^-8 of the returned one), or
2^-38 of the largest dy or x where they are far below it."""
import math

import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

HALF, BF16, F32 = 2.0 ** -8, torch.bfloat16, torch.float32


def _rand(gpu, *shape, seed=0, scale=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(gpu)


def _routing(gpu, T, E, top, how="some", seed=0):
    """how: "some" tokens not routed, "all" to one expert, "even", "none", "twice" the same expert."""
    g = torch.Generator().manual_seed(1000 * T + E + seed)
    e = torch.argsort(torch.rand((T, E), generator=g) * torch.linspace(0.3, 1, E), dim=1)[:, :top].int()
    if top > E:
        e = torch.randint(0, E, (T, top), generator=g, dtype=torch.int32)
    if how == "some":
        e[torch.rand((T, top), generator=g) < 0.2] = -1
        e[T - T // 8:] = -1
    elif how == "all":
        e[:] = E - 1
    elif how == "none":
        e[:] = -1
    elif how == "twice":
        e[:, :] = e[:, :1]
    w = torch.rand((T, top), generator=g) + 0.1
    return ffe.expert_order(e.to(gpu), E, weights=w.to(gpu))


def _parts(r):
    """(expert, its rows, their tokens) of the experts that have rows."""
    ends, order, top = r.offsets.tolist(), r.order.long(), r.experts.shape[1]
    return [(e, slice(a, b), order[a:b] // top) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]


def _act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def _slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    z = z.clone().requires_grad_()
    return torch.autograd.grad(_act64(z, act).sum(), z)[0]


def _close(got, want, tol):
    assert got.shape == want.shape, (got.shape, want.shape)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


# tokens, experts, top, n, m: single tokens, each form of the products and their edges, more
# experts than slots, k that ends inside a step, rows that are packed
SIZES = [(1, 1, 1, 64, 16), (1, 64, 8, 512, 130), (2, 5, 2, 1, 1), (7, 3, 3, 100, 33), (40, 12, 3, 250, 77), (100, 8, 2, 136, 72),
         (60, 2, 1, 1001, 250), (130, 1, 1, 64, 200), (200, 4, 2, 72, 136), (300, 3, 2, 513, 129), (700, 2, 3, 200, 333),
         (1500, 16, 2, 128, 264), (33, 1024, 4, 64, 64), (2600, 2, 1, 96, 520), (6000, 1, 2, 48, 40), (5, 2, 1, 40, 2000), (3000, 3, 4, 520, 1032)]


@pytest.mark.parametrize("how", ["some", "all", "even"])
@pytest.mark.parametrize("T,E,top,n,m", SIZES)
def test_expert_linear(gpu, T, E, top, n, m, how):
    r = _routing(gpu, T, E, top, how)
    W, b = _rand(gpu, E, m, n, seed=1, scale=2 / math.sqrt(n)), _rand(gpu, E, m, seed=2)
    W64, b64 = W.double(), b.double()
    for by_slot in (False, True):
        x = _rand(gpu, T * top if by_slot else T, n, seed=3)
        x64 = x.double()
        z64 = torch.zeros((T * top, m), dtype=torch.float64, device=gpu)
        mag, live = torch.zeros_like(z64), torch.zeros_like(z64)
        for e, rows, t in _parts(r):
            xe = x64[rows if by_slot else t]
            z64[rows], mag[rows], live[rows] = xe @ W64[e].T, xe.abs() @ W64[e].abs().T, 1.0
        bias = torch.zeros_like(z64)
        for e, rows, t in _parts(r):
            bias[rows] = b64[e]
        for act, with_bias in (("none", False), ("silu", True), ("gelu", False), ("relu", True)):
            y, z = ffe.expert_linear(x, W, r, bias=b if with_bias else None, activation=act, keep_preact=act != "none",
                                     by_slot=by_slot)
            want = z64 + (bias if with_bias else 0)
            tz = n * 2.0 ** -24 * mag + 2.0 ** -23 * want.abs()
            if z is not None:
                _close(z, want, tz + HALF * want.abs() + 1e-30)
            y64 = _act64(want, act) * live
            _close(y, y64, (1.13 * tz + (2.0 ** -18 + HALF * 1.01) * y64.abs() + 1e-30) * live)


@pytest.mark.parametrize("how", ["some", "none", "twice", "even"])
@pytest.mark.parametrize("T,E,top,m", [(1, 1, 1, 1), (1, 64, 8, 520), (3, 4, 2, 7), (40, 12, 3, 777), (700, 5, 2, 1000), (129, 9, 64, 65)])
def test_combine(gpu, T, E, top, m, how):
    r = _routing(gpu, T, E, top, how)
    y, res, dout = _rand(gpu, T * top, m, seed=1), _rand(gpu, T, m, seed=2), _rand(gpu, T, m, seed=3)
    y64, d64, w64, place = y.double(), dout.double(), r.weights.double(), r.place.long()
    live = place >= 0
    rows = torch.where(live[:, :, None], y64[place.clamp(min=0)], 0)
    for weights in (True, False):
        q = r if weights else r._replace(weights=None)
        w = w64 if weights else torch.ones_like(w64)
        want, mag = (w[:, :, None] * rows).sum(dim=1), (w[:, :, None] * rows).abs().sum(dim=1)
        _close(ffe.expert_combine(y, q), want, HALF * want.abs() + (top + 1) * 2.0 ** -24 * mag + 1e-30)
        want, mag = want + res.double(), mag + res.double().abs()
        _close(ffe.expert_combine(y, q, residual=res), want, HALF * want.abs() + (top + 2) * 2.0 ** -24 * mag + 1e-30)
    dy, dw = ffe.expert_combine_backward(dout, y, r)
    assert dy.dtype is F32 and dw.dtype is F32
    want = (d64[:, None] * rows).sum(dim=2)
    _close(dw, want, 2.0 ** -24 * ((m + 1) * (d64[:, None] * rows).abs().sum(dim=2)) + 1e-30)
    want = torch.zeros((T * top, m), dtype=torch.float64, device=gpu)
    slots = live.reshape(-1).nonzero().flatten()
    want[place.reshape(-1)[slots]] = w64.reshape(-1)[slots, None] * d64[slots // top]
    _close(dy, want, 2.0 ** -24 * want.abs())
    a, none = ffe.expert_combine_backward(dout, None, r, need_weights=False)
    assert none is None and torch.equal(a, dy)
    none, b = ffe.expert_combine_backward(dout, y, r, need_rows=False)
    assert none is None and torch.equal(b, dw)


def _value(k):
    n = k.codes.shape[1]
    return k.codes.double() * torch.repeat_interleave(k.scale.double(), k.group, dim=1)[:, :n]


@pytest.mark.parametrize("how", ["some", "all", "even"])
@pytest.mark.parametrize("T,E,top,n,m", SIZES)
def test_expert_linear_backward(gpu, T, E, top, n, m, how):
    r = _routing(gpu, T, E, top, how)
    S = T * top
    W = _rand(gpu, E, m, n, seed=1, scale=2 / math.sqrt(n))
    W64 = W.double()
    z = _rand(gpu, S, m, seed=2)
    live = torch.zeros((S, 1), dtype=torch.float64, device=gpu)
    for _, rows, _ in _parts(r):
        live[rows] = 1.0
    for by_slot, act, dtype, x8, z8 in ((False, "none", BF16, False, False), (True, "silu", F32, False, True),
                                        (False, "gelu", BF16, True, True), (True, "relu", F32, True, False)):
        x, dy = _rand(gpu, S if by_slot else T, n, seed=3), _rand(gpu, S, m, seed=4, dtype=dtype)
        kx, kz = ffe.checkpoint_q8(x, group=64), ffe.checkpoint_q8(z, group=32)
        x64, z64, d64 = _value(kx) if x8 else x.double(), _value(kz) if z8 else z.double(), dy.double()
        dx, dw, g, db = ffe.expert_linear_backward(dy, kx if x8 else x, W, r, preact=(kz if z8 else z) if act != "none" else None,
                                                   activation=act, by_slot=by_slot)
        want = d64 * _slope64(z64, act) * live
        _close(g, want, (HALF * 1.01 * want.abs() + 2.0 ** -18 * d64.abs() * 1.2 * (1 + z64.abs()) + 1e-30) * live)
        g64 = g.double()
        wx = torch.zeros_like(x64)
        mx, ww, mw = torch.zeros_like(wx), torch.zeros_like(W64), torch.zeros_like(W64)
        wb, mb = torch.zeros((E, m), dtype=torch.float64, device=gpu), torch.zeros((E, m), dtype=torch.float64, device=gpu)
        for e, rows, t in _parts(r):
            ge, xe = g64[rows], x64[rows if by_slot else t]
            if by_slot:
                wx[rows], mx[rows] = ge @ W64[e], ge.abs() @ W64[e].abs()
            else:
                wx.index_add_(0, t, ge @ W64[e])
                mx.index_add_(0, t, ge.abs() @ W64[e].abs())
            ww[e], mw[e], wb[e], mb[e] = ge.T @ xe, ge.abs().T @ xe.abs(), ge.sum(0), ge.abs().sum(0)
        _close(dx, wx, HALF * wx.abs() * 1.01 + (m + top) * 2.0 ** -24 * mx + 1e-30)
        _close(db, wb, HALF * wb.abs() * 1.01 + S * 2.0 ** -24 * mb + 1e-30)
        tol = HALF * ww.abs() * 1.01 + S * 2.0 ** -24 * mw + 1e-30
        if x8:
            far = S * 2.0 ** -38 * 1.2 * float(d64.abs().max() * x64.abs().max())
            tol = tol + (HALF + 2.0 ** -10) * 1.01 * mw + far
        _close(dw, ww, tol)


@pytest.mark.parametrize("T,E,top,n,m,how", [(3000, 2, 1, 1032, 2056, "even"), (900, 37, 2, 776, 1288, "some"), (2500, 3, 2, 2049, 515, "all"),
                                             (5000, 1, 1, 600, 4100, "even")])
def test_large_weight_gradients(gpu, T, E, top, n, m, how):
    """The products' largest tiles, in a stream: experts of very different and of no rows, ragged edges."""
    r = _routing(gpu, T, E, top, how)
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T * top, m, seed=1), _rand(gpu, E, m, n, seed=2, scale=0.05)
    kx = ffe.checkpoint_q8(x)
    for kept in (x, kx):
        _, dw, g, db = ffe.expert_linear_backward(dy, kept, W, r, need_input=False)
        x64 = _value(kx) if kept is kx else x.double()
        parts = {e: (rows, t) for e, rows, t in _parts(r)}
        for e in range(E):
            if e not in parts:
                assert not bool(dw[e].any()) and not bool(db[e].any())
                continue
            rows, t = parts[e]
            ge, xe = g[rows].double(), x64[t]
            want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
            far = T * top * 2.0 ** -38 * float(dy.double().abs().max() * x64.abs().max())
            tol = HALF * 1.01 * want.abs() + T * top * 2.0 ** -24 * mag + 1e-30
            _close(dw[e], want, tol + (2.0 ** -9 * mag + far if kept is kx else 0))
            want, mag = ge.sum(0), ge.abs().sum(0)
            _close(db[e], want, HALF * 1.01 * want.abs() + T * top * 2.0 ** -24 * mag + 1e-30)


def test_checkpoints_cost_little(gpu):
    """dw of checkpoints against the formula on the values that they stand for, unrounded g: two
    roundings of 2^-12 rms each beside the output's own, where bf16 operands would make it 1.7 times that."""
    T, E, top, n, m = 3000, 3, 2, 256, 200
    r = _routing(gpu, T, E, top, "even")
    x, z, dy = _rand(gpu, T, n), _rand(gpu, T * top, m, seed=1), _rand(gpu, T * top, m, seed=2)
    W = _rand(gpu, E, m, n, seed=3)
    kx, kz = ffe.checkpoint_q8(x), ffe.checkpoint_q8(z)
    _, dw, _, _ = ffe.expert_linear_backward(dy, kx, W, r, preact=kz, activation="silu")
    g64, x64 = dy.double() * _slope64(_value(kz), "silu"), _value(kx)
    want = torch.zeros((E, m, n), dtype=torch.float64, device=gpu)
    for e, rows, t in _parts(r):
        want[e] = g64[rows].T @ x64[t]
    # a rounding to nearest is off by at most 2^-9 of a value's binade, rms 2^-9 / sqrt(3) of it: 1.66e-3 of
    # the norm at most for bf16, an eighth of that each for the two in fp16
    assert float((dw.double() - want).norm() / want.norm()) < 1.1 * 2.0 ** -8 / math.sqrt(3)


@pytest.mark.parametrize("scales", [(1e-30, 1e-25), (1e30, 1e-30), (1e18, 1e17), (1.0, 0.0), (0.0, 1.0)])
def test_checkpoints_of_any_magnitude(gpu, scales):
    """The powers of two around fp16 undo themselves."""
    T, E, top, n, m = 200, 3, 2, 72, 40
    r = _routing(gpu, T, E, top)
    x, dy = _rand(gpu, T, n, scale=scales[0]), _rand(gpu, T * top, m, seed=1, scale=scales[1])
    W = _rand(gpu, E, m, n, seed=2)
    kx = ffe.checkpoint_q8(x, group=16)
    _, dw, g, _ = ffe.expert_linear_backward(dy, kx, W, r, need_input=False)
    x64 = _value(kx)
    for e, rows, t in _parts(r):
        want, mag = g[rows].double().T @ x64[t], g[rows].double().abs().T @ x64[t].abs()
        far = T * top * 2.0 ** -38 * float(dy.double().abs().max() * x64.abs().max())
        _close(dw[e], want, HALF * 1.01 * want.abs() + 2.0 ** -9 * mag + far + 2.0 ** -133)


def test_special_values(gpu):
    """NaN and infinities stay with the tokens and experts that they belong to."""
    T, E, top, n, m = 300, 4, 2, 136, 72
    r = _routing(gpu, T, E, top, "some")
    x, W, dy = _rand(gpu, T, n), _rand(gpu, E, m, n, seed=1), _rand(gpu, T * top, m, seed=2)
    y0, (dx0, dw0, _, db0) = ffe.expert_linear(x, W, r)[0], ffe.expert_linear_backward(dy, x, W, r)
    t = int(r.order[5]) // top
    x2 = x.clone()
    x2[t, 7] = math.nan
    y, _ = ffe.expert_linear(x2, W, r)
    mine = torch.zeros(T * top, dtype=torch.bool, device=gpu)
    mine[r.place[t][r.place[t] >= 0].long()] = True
    assert bool(y[mine].isnan().all()) and torch.equal(y[~mine], y0[~mine])
    dw = ffe.expert_linear_backward(dy, x2, W, r)[1]
    hit = torch.zeros(E, dtype=torch.bool, device=gpu)
    hit[r.experts[t][r.experts[t] >= 0].long()] = True
    assert bool(dw[hit][:, :, 7].isnan().all()) and torch.equal(dw[~hit], dw0[~hit])
    keep = torch.ones(n, dtype=torch.bool, device=gpu)
    keep[7] = False
    assert torch.equal(dw[:, :, keep], dw0[:, :, keep])
    # behind the last row nothing is read: its gradients may hold anything
    used = int(r.offsets[-1])
    assert used < T * top
    dy2 = dy.clone()
    dy2[used:] = math.nan
    dx, dw, g, db = ffe.expert_linear_backward(dy2, x, W, r)
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0) and torch.equal(db, db0) and not bool(g[used:].any())
    kx = ffe.checkpoint_q8(x)
    a, b = ffe.expert_linear_backward(dy2, kx, W, r), ffe.expert_linear_backward(dy, kx, W, r)
    assert not bool(a[1].isnan().any())
    # an expert of NaN weights that no token takes
    e = torch.where(r.experts == 2, torch.full_like(r.experts, -1), r.experts)
    q = ffe.expert_order(e, E)
    W2 = W.clone()
    W2[2] = math.nan
    assert not bool(ffe.expert_linear(x, W2, q)[0].isnan().any())
    dx, dw, _, db = ffe.expert_linear_backward(dy, x, W2, q)
    assert not bool(dx.isnan().any()) and not bool(dw[2].any()) and not bool(db[2].any())


@pytest.mark.parametrize("T,E,top,n,m", [(1, 3, 2, 40, 24), (70, 4, 2, 250, 77), (400, 2, 3, 136, 72), (1500, 2, 2, 1032, 2056)])
def test_nothing_routed(gpu, T, E, top, n, m):
    """No token takes any expert: zeros everywhere, whatever the inputs hold."""
    r = _routing(gpu, T, E, top, "none")
    x, W = torch.full((T, n), math.nan, dtype=BF16, device=gpu), _rand(gpu, E, m, n)
    dy = torch.full((T * top, m), math.inf, dtype=BF16, device=gpu)
    y, z = ffe.expert_linear(x, W, r, activation="gelu", keep_preact=True)
    assert not bool(y.any()) and not bool(z.any()) and not bool(ffe.expert_combine(y, r).any())
    for kept in (x, ffe.checkpoint_q8(x)):
        assert not any(bool(v.any()) for v in ffe.expert_linear_backward(dy, kept, W, r, preact=z, activation="gelu"))


@pytest.mark.parametrize("by_slot", [False, True])
def test_rows_in_no_expert_do_not_count(gpu, by_slot):
    """Tokens that are not routed and rows behind the last one may hold any numbers: they do not set
    the powers of two that the operands of a checkpoint's gradient are scaled by either."""
    T, E, top, n, m = 200, 3, 2, 72, 40
    r = _routing(gpu, T, E, top, "some")
    used, X = int(r.offsets[-1]), T * top if by_slot else T
    x, dy = _rand(gpu, X, n), _rand(gpu, T * top, m, seed=1)
    W = _rand(gpu, E, m, n, seed=2)
    idle = torch.arange(X, device=gpu) >= used if by_slot else (r.place < 0).all(dim=1)
    assert bool(idle.any()) and used < T * top
    want = ffe.expert_linear_backward(dy, ffe.checkpoint_q8(x), W, r, by_slot=by_slot)
    x2, dy2 = x.clone(), dy.clone()
    x2[idle], dy2[used:] = 1e30, -1e35
    got = ffe.expert_linear_backward(dy2, ffe.checkpoint_q8(x2), W, r, by_slot=by_slot)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_wrong_routings_stay_inside(gpu):
    """Arrays that are no routing: whatever comes out, nothing beyond the rows is touched."""
    T, E, top, n, m = 150, 5, 2, 64, 72
    r = _routing(gpu, T, E, top, "even")
    big = 2 ** 31 - 1
    x, W, dy = _rand(gpu, T, n), _rand(gpu, E, m, n, seed=1), _rand(gpu, T * top, m, seed=2)
    order, place, offsets = r.order.clone(), r.place.clone(), r.offsets.clone()
    order[::3], order[1::7] = big, -big
    place[::3], place[1::5] = big, -5
    bad = [r._replace(order=order), r._replace(place=place)]
    for o in ([0, big, 3, -4, big, 7], [big] * 6, [-1] * 6, [0, 300, 0, 300, 0, 300], [300, 0, 300, 0, 300, 0]):
        offsets = torch.tensor(o, dtype=torch.int32, device=gpu)
        bad.append(r._replace(offsets=offsets))
    for q in bad:
        y, _ = ffe.expert_linear(x, W, q)
        ffe.expert_linear(y, W.transpose(1, 2).contiguous(), q, by_slot=True)
        out = ffe.expert_combine(y, q)
        ffe.expert_combine_backward(out, y, q)
        ffe.expert_linear_backward(dy, x, W, q)
        ffe.expert_linear_backward(dy, ffe.checkpoint_q8(x), W, q)
    torch.cuda.synchronize()


def test_strides_streams_and_parts(gpu):
    T, E, top, n, m = 400, 3, 2, 130, 66
    r = _routing(gpu, T, E, top)
    xb, W = _rand(gpu, T, 301), _rand(gpu, E, m, n, seed=1)
    x = xb[:, 5:135]
    dyb = _rand(gpu, T * top, 99, seed=2)
    dy = dyb[:, 3:69]
    y, z = ffe.expert_linear(x, W, r, activation="silu", keep_preact=True)
    yc, zc = ffe.expert_linear(x.contiguous(), W, r, activation="silu", keep_preact=True)
    assert torch.equal(y, yc) and torch.equal(z, zc)
    full = ffe.expert_linear_backward(dy, x, W, r, preact=z, activation="silu")
    plain = ffe.expert_linear_backward(dy.contiguous(), x.contiguous(), W, r, preact=z, activation="silu")
    assert all(torch.equal(a, b) for a, b in zip(full, plain))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ys, _ = ffe.expert_linear(x, W, r, activation="silu", stream=side)
    outs = ffe.expert_combine(ys, r, stream=side)
    gs = ffe.expert_linear_backward(dy, x, W, r, preact=z, activation="silu", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(ys, y) and torch.equal(outs, ffe.expert_combine(y, r)) and all(torch.equal(a, b) for a, b in zip(gs, full))
    for which in range(3):
        need = [k == which for k in range(3)]
        part = ffe.expert_linear_backward(dy, x, W, r, preact=z, activation="silu", need_input=need[0], need_weight=need[1],
                                          need_bias=need[2])
        for got, want, k in zip((part[0], part[1], part[3]), (full[0], full[1], full[3]), need):
            assert (got is None) != k and (got is None or torch.equal(got, want))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=gpu)
    again = ffe.expert_linear_backward(dy, x, W, r, preact=z, activation="silu", workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(again, full))
    # no tokens
    q = ffe.expert_order(r.experts[:0], E, weights=r.weights[:0])
    y, z = ffe.expert_linear(x[:0], W, q, keep_preact=True)
    assert y.shape == z.shape == (0, m) and ffe.expert_combine(y, q).shape == (0, m)
    dx, dw, g, db = ffe.expert_linear_backward(y, x[:0], W, q)
    assert dx.shape == (0, n) and not bool(dw.any()) and not bool(db.any())
    dr, dwt = ffe.expert_combine_backward(y, y, q)
    assert dr.shape == (0, m) and dwt.shape == (0, top)


def test_rows_far_apart(gpu):
    """Tokens' rows that lie more than 2^31 bytes from the first to the last."""
    T, E, top, n, m = 600, 2, 2, 72, 40
    r = _routing(gpu, T, E, top, "even")
    wide = torch.empty((T, 2 << 20), dtype=BF16, device=gpu)
    x = wide[:, 64:64 + n]
    x.copy_(_rand(gpu, T, n))
    W, dy = _rand(gpu, E, m, n, seed=1), _rand(gpu, T * top, m, seed=2)
    assert torch.equal(ffe.expert_linear(x, W, r)[0], ffe.expert_linear(x.contiguous(), W, r)[0])
    a, b = ffe.expert_linear_backward(dy, x, W, r), ffe.expert_linear_backward(dy, x.contiguous(), W, r)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_captured(gpu):
    """A layer of experts forward and back in one graph, routed anew at every replay."""
    T, E, top, n, m = 200, 6, 2, 72, 48
    x, logits, dout = _rand(gpu, T, n), _rand(gpu, T, E, seed=1, dtype=F32), _rand(gpu, T, n, seed=2)
    up, down = _rand(gpu, E, m, n, seed=3, scale=0.2), _rand(gpu, E, n, m, seed=4, scale=0.2)

    def step():
        r = ffe.route(logits, top)
        h, z = ffe.expert_linear(x, up, r, activation="silu", keep_preact=True)
        kx, kz = ffe.checkpoint_q8(x), ffe.checkpoint_q8(z)
        y, _ = ffe.expert_linear(h, down, r, by_slot=True)
        out = ffe.expert_combine(y, r, residual=x)
        dy, dw = ffe.expert_combine_backward(dout, y, r)
        dh, ddown, _, _ = ffe.expert_linear_backward(dy, h, down, r, by_slot=True, need_bias=False)
        dx, dup, _, _ = ffe.expert_linear_backward(dh, kx, up, r, preact=kz, activation="silu", need_bias=False)
        return out, dx, dup, ddown, ffe.route_backward(dw, logits, r.experts)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(4):
        logits.copy_(_rand(gpu, T, E, seed=10 + k, dtype=F32, scale=1 + k))
        x.copy_(_rand(gpu, T, n, seed=20 + k))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))


def test_refusals(gpu):
    T, E, top, n, m = 10, 3, 2, 16, 8
    r = _routing(gpu, T, E, top)
    x, W, b, dy = _rand(gpu, T, n), _rand(gpu, E, m, n), _rand(gpu, E, m), _rand(gpu, T * top, m)
    both = (ValueError, TypeError, ffe.FlipFlopError)
    for args, kw in (((x, W[:2], r), {}), ((x, W[0], r), {}), ((x, W.transpose(1, 2), r), {}), ((x[:9], W, r), {}), ((x, W, tuple(r)), {}),
                     ((x, W, None), {}), ((x, W, r), dict(by_slot=True)), ((x.float(), W, r), {}), ((x.cpu(), W, r), {}),
                     ((x, W.cpu(), r), {}), ((x, W.float(), r), {}), ((x, W, r), dict(bias=b[:2])), ((x, W, r), dict(bias=b.view(m, E))),
                     ((x, W, r), dict(activation="tanh")), ((x[0], W, r), {}), ((x, W, r._replace(order=r.order[:-1])), {}),
                     ((x, W, r._replace(order=r.order.long())), {}), ((x, W, r._replace(offsets=r.offsets[:-1])), {}),
                     ((x, W, r._replace(place=r.place.t())), {}), ((x, W, r._replace(order=r.order.cpu())), {}),
                     ((x, W, r._replace(experts=None)), {}), ((x, W, r._replace(weights=r.weights.double())), {})):
        with pytest.raises(both):
            ffe.expert_linear(*args, **kw)
    y = dy
    dout = _rand(gpu, T, m)
    for args, kw in (((y[:-1], r), {}), ((y.float(), r), {}), ((y, r), dict(residual=y)), ((y, r), dict(residual=dout.float()))):
        with pytest.raises(both):
            ffe.expert_combine(*args, **kw)
    for args in ((dout[:-1], y, r), (dout, y[:-1], r), (dout, None, r), (dout, y, r._replace(weights=None)), (dout.float(), y, r)):
        with pytest.raises(both):
            ffe.expert_combine_backward(*args)
    k = ffe.checkpoint_q8(x)
    for args, kw in (((dy[:-1], x, W, r), {}), ((dy, x, W[:, :4].contiguous(), r), {}), ((dy, x, W, r), dict(activation="relu")),
                     ((dy, x, W, r), dict(activation="relu", preact=x)), ((dy, x, W, r), dict(by_slot=True)),
                     ((dy, k, W, r), dict(by_slot=True)), ((dy.half(), x, W, r), {}), ((dy, k._replace(group=8), W, r), {}),
                     ((dy, x, W, r), dict(activation="relu", preact=k)), ((dy, None, W, r), {}), ((dy, x, None, r), {})):
        with pytest.raises(both):
            ffe.expert_linear_backward(*args, **kw)


@pytest.mark.parametrize("scales", [(1e-30, 1e-8), (1e30, 1e-30), (1e18, 1e17), (1e-3, 1e3)])
@pytest.mark.parametrize("T,E,top,n,m", [(2000, 2, 1, 1032, 2056), (6144, 24, 1, 2056, 2056)])
def test_large_gradients_of_any_magnitude(gpu, T, E, top, n, m, scales):
    """As test_checkpoints_of_any_magnitude, in larger tiles and in a stream of the largest, whole ones and others."""
    r = _routing(gpu, T, E, top, "even")
    x, dy = _rand(gpu, T, n, scale=scales[0]), _rand(gpu, T * top, m, seed=1, scale=scales[1])
    W = torch.zeros((E, m, n), dtype=BF16, device=gpu)
    kx = ffe.checkpoint_q8(x)
    _, dw, g, _ = ffe.expert_linear_backward(dy, kx, W, r, need_input=False)
    x64 = _value(kx)
    for e, rows, t in _parts(r):
        want, mag = g[rows].double().T @ x64[t], g[rows].double().abs().T @ x64[t].abs()
        far = T * top * 2.0 ** -38 * float(dy.double().abs().max() * x64.abs().max())
        # (a result below fp32's normal range is rounded to its step and to bf16's, 2^-133, there)
        _close(dw[e], want, HALF * 1.01 * want.abs() + (2.0 ** -9 + T * 2.0 ** -24) * mag + far + 2.0 ** -133)


def test_more_weight_rows_than_slots(gpu):
    """Weights of more than 2^24 rows, whose rows are laid out for dx."""
    T, E, top, n, m = 3, 1024, 2, 9, 16400
    r = _routing(gpu, T, E, top, "all")
    W = torch.zeros((E, m, n), dtype=BF16, device=gpu)
    W[E - 1] = _rand(gpu, m, n, seed=1)
    dy = _rand(gpu, T * top, m, seed=2)
    dx, dw, g, db = ffe.expert_linear_backward(dy, torch.zeros((T, n), dtype=BF16, device=gpu), W, r, need_weight=False, need_bias=False)
    rows = torch.zeros((T * top, n), dtype=torch.float64, device=gpu)
    mag = torch.zeros_like(rows)
    for e, s, _ in _parts(r):
        rows[s], mag[s] = g[s].double() @ W[e].double(), g[s].double().abs() @ W[e].double().abs()
    at = r.place.long()
    want, mag = rows[at].sum(1), mag[at].sum(1)
    _close(dx, want, HALF * 1.01 * want.abs() + (m + top) * 2.0 ** -24 * mag)


@pytest.mark.parametrize("T,E,n,m", [(1200, 2, 776, 1288), (900, 18, 776, 1288), (6144, 24, 2056, 2056)])
@pytest.mark.parametrize("gap", [0, 3, 24])
def test_weight_gradient_rows_apart(gpu, gap, T, E, n, m):
    """dw with rows further apart than n, by the C ABI: the same bits as without gaps, which stay as they were."""
    import paper_2609_14706_amd.experts as X
    top = 1
    r = _routing(gpu, T, E, top, "even")
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T * top, m, seed=1), torch.zeros((E, m, n), dtype=BF16, device=gpu)
    want, g = ffe.expert_linear_backward(dy, x, W, r, need_input=False, need_bias=False)[1:3]
    dw = torch.full((E * m, n + gap), 7.0, dtype=BF16, device=gpu)
    a = X.ff_expert_grad_args()
    a.routing, a.n, a.m, a.dy_dtype, a.dy, a.lddy = X._routing(r, x.device), n, m, X._elem(dy, "dy"), dy.data_ptr(), m
    a.x, a.ldx, a.w, a.ldw, a.g, a.ldg = x.data_ptr(), n, W.data_ptr(), n, g.data_ptr(), m
    a.dw, a.lddw = dw.data_ptr(), n + gap
    keep = X._workspace(a, X._bytes("ff_expert_linear_backward_workspace_size", a, functions=X._FN), None, x.device)
    X._launch("ff_expert_linear_backward", a, x.device, X._FN)
    del keep
    assert torch.equal(dw[:, :n].reshape(E, m, n), want)
    assert bool((dw[:, n:] == 7.0).all())


@pytest.mark.parametrize("T,E,n,m", [(6144, 24, 2056, 2056), (1024, 1, 4104, 8200)])
def test_largest_weight_gradients(gpu, T, E, n, m):
    """A stream of 256 x 256 tiles, in bf16 and, from a checkpoint, in fp16."""
    r = _routing(gpu, T, E, 1, "some")
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T, m, seed=1), torch.zeros((E, m, n), dtype=BF16, device=gpu)
    kx = ffe.checkpoint_q8(x)
    for kept in (x, kx):
        _, dw, g, db = ffe.expert_linear_backward(dy, kept, W, r, need_input=False)
        x64 = _value(kx) if kept is kx else x.double()
        far = T * 2.0 ** -38 * float(dy.double().abs().max() * x64.abs().max())
        for e, rows, t in _parts(r):
            ge, xe = g[rows].double(), x64[t]
            want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
            tol = HALF * 1.01 * want.abs() + T * 2.0 ** -24 * mag + 1e-30
            _close(dw[e], want, tol + (2.0 ** -9 * mag + far if kept is kx else 0))
            want, mag = ge.sum(0), ge.abs().sum(0)
            _close(db[e], want, HALF * 1.01 * want.abs() + T * 2.0 ** -24 * mag + 1e-30)


# A size for each form of the products (tiles of 32 i x 32 j, pairs of k in flight, k in parts) that the
# sizes above leave out, by the rules that choose them.
FORMS = {"y skinny 2": (13, 1, 1, 40, 35), "y 4 8 3": (2744, 1, 1, 1233, 1427), "y 6 8 2": (13219, 1, 1, 45, 543),
         "y 8 8 2": (3474, 1, 1, 166, 3528), "dx 2 4 3 in 16": (2, 1, 1, 32, 4889), "dx 2 4 3 in 2": (605, 1, 1, 883, 3972),
         "dx 2 4 3 in 4": (1, 1, 1, 35, 1695), "dx 4 4 2": (19165, 1, 1, 134, 35), "dx 4 4 2 in 2": (17085, 1, 1, 37, 11007),
         "dx 4 4 2 in 4": (2453, 8, 8, 51, 8865), "dx 4 8 3": (1926, 1, 1, 2098, 1277), "dx 4 8 3 in 2": (1594, 1, 1, 2112, 11008),
         "dx 4 8 3 in 4": (4172, 2, 1, 458, 9945), "dx 6 8 2": (16541, 1, 1, 454, 33), "dx 6 8 2 in 2": (2788, 1, 1, 1832, 8712),
         "dx 6 8 2 in 4": (2185, 1, 1, 994, 9517), "dx 8 8 2": (12853, 1, 1, 939, 155), "dw 2 4 3 in 8": (2084, 1, 1, 47, 40),
         "dw 4 4 2": (162, 1, 1, 2539, 1603), "dw 4 4 2 in 2": (21217, 1, 1, 3081, 1068), "dw 4 4 2 in 4": (12755, 2, 2, 2007, 527),
         "dw 4 4 2 in 8": (19264, 1, 1, 135, 2238), "dw 8 8 2 in 16": (22749, 2, 2, 1057, 903), "dw 8 8 2 in 2": (9301, 1, 1, 1965, 2591),
         "dw 8 8 2 in 4": (11710, 1, 1, 943, 2477), "dw 8 8 2 in 8": (19693, 1, 1, 1561, 585)}


@pytest.mark.parametrize("form", FORMS)
def test_every_form(gpu, form):
    T, E, top, n, m = FORMS[form]
    r = _routing(gpu, T, E, top, "some")
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T * top, m, seed=1), _rand(gpu, E, m, n, seed=2, scale=0.05)
    y, _ = ffe.expert_linear(x, W, r)
    kx = ffe.checkpoint_q8(x)
    dx, dw, g, _ = ffe.expert_linear_backward(dy, x, W, r)
    dw8 = ffe.expert_linear_backward(dy, kx, W, r, need_input=False)[1]
    sums = torch.zeros((T * top + 1, n), dtype=torch.float64, device=gpu)
    mags = torch.zeros_like(sums)
    far = T * top * 2.0 ** -38 * float(dy.double().abs().max() * x.double().abs().max())
    for e, rows, t in _parts(r):
        ge, xe, we = g[rows].double(), x[t].double(), W[e].double()
        want = xe @ we.T
        _close(y[rows], want, HALF * 1.01 * want.abs() + n * 2.0 ** -24 * (xe.abs() @ we.abs().T))
        sums[rows], mags[rows] = ge @ we, ge.abs() @ we.abs()
        want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
        _close(dw[e], want, HALF * 1.01 * want.abs() + T * top * 2.0 ** -24 * mag)
        x8 = _value(kx)[t]
        want, mag = ge.T @ x8, ge.abs().T @ x8.abs()
        _close(dw8[e], want, HALF * 1.01 * want.abs() + (2.0 ** -9 + T * top * 2.0 ** -24) * mag + far)
    at = r.place.long()   # (-1, no row: the zeros at the end)
    want, mag = sums[at].sum(1), mags[at].sum(1)
    _close(dx, want, HALF * 1.01 * want.abs() + (m + top) * 2.0 ** -24 * mag)


@pytest.mark.parametrize("by_slot", [False, True])
@pytest.mark.parametrize("n", [2100, 4200])   # eight and sixteen waves share a row's k
@pytest.mark.parametrize("T,E,top", [(1, 1, 1), (5, 3, 2), (20, 1, 1), (40, 1, 1), (60, 2, 1)])
def test_few_rows_of_long_k(gpu, T, E, top, n, by_slot):
    m = 130
    r = _routing(gpu, T, E, top, "even")
    x, W, b = _rand(gpu, T * top if by_slot else T, n), _rand(gpu, E, m, n, seed=1, scale=0.05), _rand(gpu, E, m, seed=2)
    y, _ = ffe.expert_linear(x, W, r, bias=b, by_slot=by_slot)
    for e, rows, t in _parts(r):
        xe, we = (x[rows] if by_slot else x[t]).double(), W[e].double()
        want = xe @ we.T + b[e].double()
        _close(y[rows], want, HALF * 1.01 * want.abs() + (n + 1) * 2.0 ** -24 * (xe.abs() @ we.abs().T + b[e].double().abs()))
