"""The ends of what the operators around a layer of experts and of 8-bit checkpoints take:
magnitudes, tokens that are not routed, rows in no expert, arrays that are no routing.

References are the formulas in 64 bits (the routing's gradient: in 60 digits).  Tolerances as
for the operators' other tests: an fp32 sum of n terms is off by at most n 2^-24 of the sum of
magnitudes, a rounding by half a step (bf16 2^-8, fp32 2^-24), the fp16 operands of a
checkpoint's dW by 2^-11 of each value or 2^-38 of the largest."""
import decimal
import math

import pytest
import torch

import paper_2609_14706_amd as ffe
import paper_2609_14706_amd.experts as X

pytestmark = pytest.mark.gpu

HALF, BF16, F32 = 2.0 ** -8, torch.bfloat16, torch.float32


def _rand(gpu, *shape, seed=0, scale=1.0, dtype=BF16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(gpu)


def _routing(gpu, T, E, top, idle=0.0, seed=0):
    """Random choices, `idle` of them none."""
    g = torch.Generator().manual_seed(1000 * T + E + seed)
    e = torch.argsort(torch.rand((T, E), generator=g) * torch.linspace(0.3, 1, E), dim=1)[:, :top].int()
    e[torch.rand((T, top), generator=g) < idle] = -1
    w = torch.rand((T, top), generator=g) + 0.1
    return ffe.expert_order(e.to(gpu).contiguous(), E, weights=w.to(gpu))


def _parts(r):
    """(expert, its rows, their tokens) of the experts that have rows."""
    ends, order, top = r.offsets.tolist(), r.order.long(), r.experts.shape[1]
    return [(e, slice(a, b), order[a:b] // top) for e, (a, b) in enumerate(zip(ends, ends[1:])) if b > a]


def _value(k):
    return k.codes.double() * torch.repeat_interleave(k.scale.double(), k.group, dim=1)[:, :k.codes.shape[1]]


def _close(got, want, tol):
    assert got.shape == want.shape, (got.shape, want.shape)
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


# tokens, experts, n, m: both gradients in one launch, smaller tiles, sums cut along the rows, the largest
# tiles in a stream, whole ones and edges
@pytest.mark.parametrize("scales", [(1e-30, 1e35), (1e-35, 1e36), (1e35, 1e-30)])
@pytest.mark.parametrize("T,E,n,m", [(200, 3, 72, 40), (1000, 1, 136, 72), (162, 1, 2539, 1603), (2000, 2, 1032, 2056),
                                     (9301, 1, 1965, 2591), (6144, 24, 2056, 2056)])
def test_weight_gradient_of_opposite_magnitudes(gpu, T, E, n, m, scales):
    """One operand near the end of fp32's range, the other far below one: neither power of two alone
    takes the sums back, both together do."""
    r = _routing(gpu, T, E, 1)
    x, dy = _rand(gpu, T, n, scale=scales[0]), _rand(gpu, T, m, seed=1, scale=scales[1])
    W = torch.zeros((E, m, n), dtype=BF16, device=gpu)
    kx = ffe.checkpoint_q8(x)
    x64, g64 = _value(kx), dy.double()
    got = [ffe.expert_linear_backward(dy, kx, W, r, need_input=need)[1] for need in (False, True)]
    far = T * 2.0 ** -38 * float(g64.abs().max() * x64.abs().max())

    def check(dw, ge, xe):
        want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
        assert bool(torch.isfinite(dw).all())
        _close(dw, want, HALF * 1.01 * want.abs() + (2.0 ** -9 + T * 2.0 ** -24) * mag + far + 2.0 ** -133)
    for e, rows, t in _parts(r):
        for dw in got:
            check(dw[e], g64[rows], x64[t])
    if E == 1:   # the plain layer, whose rows lie in their order
        for need in (False, True):
            check(ffe.linear_backward(dy, kx, W[0], need_input=need)[1], g64, x64)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("E,top", [(7, 2), (60, 4), (130, 8), (1000, 20)])
def test_route_gradient_of_tokens_that_are_not_routed(gpu, E, top, dtype):
    """Their logits may hold anything: their rows of the gradient are zeros, the others as they were."""
    T = 75
    g = torch.Generator().manual_seed(E)
    logits = (2 * torch.randn((T, E), generator=g)).to(dtype)
    dw = torch.randn((T, top), generator=g)
    mask = torch.arange(T) % 3 > 0
    bad = logits.clone()
    for k, v in enumerate((math.nan, math.inf, -math.inf)):
        bad[9 * k] = v                  # (token 27 of no kind: finite)
        bad[9 * k + 3, E // 2] = v
        bad[9 * k + 6, E - 1] = v
    assert not bool(mask[:27:3].any())
    for score in ("softmax", "sigmoid"):
        r = ffe.route(bad.to(gpu), top, score=score, mask=mask.to(gpu))
        for renorm in (True, False):
            want = ffe.route_backward(dw.to(gpu), logits.to(gpu), r.experts, score=score, renormalise=renorm)
            got = ffe.route_backward(dw.to(gpu), bad.to(gpu), r.experts, score=score, renormalise=renorm)
            assert not bool(got[~mask].any()) and torch.equal(got, want) and bool(got[mask].any())
            # choices that are none, in place of the logits, of which nothing is left
            out = bad.to(gpu)
            none = torch.full((T, top), E, dtype=torch.int32, device=gpu)
            assert not bool(ffe.route_backward(dw.to(gpu), out, none, score=score, renormalise=renorm).any())


def _digits(values):
    return [decimal.Decimal(float(v)) for v in values]


def _route_gradient(logits, dw, chosen, score, renorm):
    """A token's gradient of the weights by its logits in 60 digits, and the magnitudes of the terms that a
    sum of differences has: dl_i = s_i sum_k s_k (d_i - d_k), d_j = sum_k w_k (dw_j - dw_k) / sum."""
    with decimal.localcontext() as c:
        c.prec = 60
        l, zero = _digits(logits), decimal.Decimal(0)
        if score == "sigmoid":
            s = [1 / (1 + (-v).exp()) for v in l]
            slope = [1 / (1 + v.exp()) for v in l]   # 1 - s
        else:
            e = [(v - max(l)).exp() for v in l]
            s = [v / sum(e) for v in e]
        dw = _digits(dw)
        d, m = [zero] * len(l), [zero] * len(l)
        total = sum(s[e] for e in chosen)
        for j, e in enumerate(chosen):
            if renorm:
                terms = [s[f] / total * (dw[j] - dw[k]) / total for k, f in enumerate(chosen)]
                d[e], m[e] = d[e] + sum(terms), m[e] + sum(abs(v) for v in terms)
            else:
                d[e], m[e] = d[e] + dw[j], m[e] + abs(dw[j])
        if score == "sigmoid":
            return ([float(a * b * q) for a, b, q in zip(d, s, slope)], [float(a * b * q) for a, b, q in zip(m, s, slope)])
        out, mag = [], []
        for i in range(len(l)):
            others = [k for k in range(len(l)) if k != i]
            out.append(float(s[i] * sum(s[k] * (d[i] - d[k]) for k in others)))
            mag.append(float(s[i] * sum(s[k] * (abs(d[i] - d[k]) + m[i] + m[k]) for k in others)))
        return out, mag


def _check_route_gradient(gpu, score, renorm, top, dtype):
    E = 9
    g = torch.Generator().manual_seed(top)
    logits = torch.randn((40, E), generator=g)
    for t in range(40):   # one expert, or all of them, further and further ahead of the others
        logits[t, t % E] += t
    if score == "sigmoid":
        logits[20:] += torch.arange(20.0)[:, None]
    logits = logits.to(dtype)
    dw = torch.randn((40, top), generator=g)
    r = ffe.route(logits.to(gpu), top, score=score)
    chosen = r.experts.cpu()
    chosen[5:40:7] = chosen[5:40:7].flip(1)
    chosen[3] = torch.arange(1, top + 1)      # not the largest scores: as a bias or the caller has it
    got = ffe.route_backward(dw.to(gpu), logits.to(gpu), chosen.to(gpu), score=score, renormalise=renorm).double().cpu()
    half = 2.0 ** -24 if dtype is F32 else 2.0 ** -8
    for t in range(40):
        want, mag = (torch.tensor(v, dtype=torch.float64)
                     for v in _route_gradient(logits[t].tolist(), dw[t].tolist(), chosen[t].tolist(), score, renorm))
        # (2^-149, 2^-133: the types' smallest steps)
        tol = half * 1.0001 * want.abs() + 1e-12 * mag + (2.0 ** -149 if dtype is F32 else 2.0 ** -133)
        assert bool(((got[t] - want).abs() <= tol).all()), (t, got[t].tolist(), want.tolist())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("top", [1, 3])
def test_route_gradient_of_sigmoids_near_one(gpu, top, dtype):
    """1 - sigmoid(l) is sigmoid(-l), not a difference of rounded numbers: nothing is left of that from l = 37 on."""
    _check_route_gradient(gpu, "sigmoid", False, top, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renorm", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("top", [1, 3])
def test_route_gradient_of_one_expert_far_ahead(gpu, top, score, renorm, dtype):
    """A score, or a weight, next to one: its gradient is a sum over the others, not one less a rounded number."""
    _check_route_gradient(gpu, score, renorm, top, dtype)


@pytest.mark.parametrize("z8", [False, True])
@pytest.mark.parametrize("act,off", [("relu", -1.0), ("silu", -60.0), ("gelu", -9.0)])
@pytest.mark.parametrize("T,E,top,n,m", [(150, 3, 2, 72, 40), (700, 2, 2, 513, 129), (1500, 1, 1, 1032, 2056)])
def test_weight_gradient_beside_units_that_are_off(gpu, T, E, top, n, m, act, off, z8):
    """The largest dy where the activation has no slope: dW's other sums are as good as without it."""
    r = _routing(gpu, T, E, top, 0.1)
    S = T * top
    x, W, z, dy = _rand(gpu, T, n), _rand(gpu, E, m, n, seed=1, scale=0.05), _rand(gpu, S, m, seed=2), _rand(gpu, S, m, seed=3)
    z[:, 16:32] = off                   # a group of its own
    dy[1::5, 16:32] *= 2.0 ** 60
    kx = ffe.checkpoint_q8(x)
    kz = ffe.checkpoint_q8(z, group=16) if z8 else z
    _, dw, g, _ = ffe.expert_linear_backward(dy, kx, W, r, preact=kz, activation=act)
    g64, x64 = g.double(), _value(kx)
    far = S * 2.0 ** -38 * float(g64.abs().max() * x64.abs().max()) * 1.01

    def check(dw, ge, xe):   # (g unrounded: 2^-8 of the returned one)
        want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
        _close(dw, want, HALF * 1.01 * want.abs() + (HALF * 1.01 + 2.0 ** -10 + S * 2.0 ** -24) * mag + far)
    assert float(g64.abs().max()) < 2.0 ** 10     # (what the slopes leave)
    for e, rows, t in _parts(r):
        check(dw[e], g64[rows], x64[t])
    if E == 1:
        _, dw, g, _ = ffe.linear_backward(dy, kx, W[0], preact=kz, activation=act)
        check(dw, g.double(), x64)


def _combine_gradient(r, dout, y):
    """(dy, dweights) by the C ABI, among rows and numbers that stay as they were."""
    S, m, dev = y.shape[0], y.shape[1], y.device
    dy, dw = torch.full((S + 4, m), 7.0, device=dev), torch.full((S + 64,), 7.0, device=dev)
    X._library()
    a = X.ff_expert_combine_grad_args(X._routing(r, dev), m, dout.data_ptr(), m, y.data_ptr(), m, dy[2:].data_ptr(), m,
                                      dw[32:].data_ptr())
    X._launch("ff_expert_combine_backward", a, dev, X._FN)
    assert bool((dy[:2] == 7.0).all()) and bool((dy[-2:] == 7.0).all())
    assert bool((dw[:32] == 7.0).all()) and bool((dw[-32:] == 7.0).all())
    return dy[2:-2], dw[32:-32].view(-1, r.experts.shape[1])


def test_weights_gradient_of_wrong_routings(gpu):
    """Arrays that are no routing: every weight's gradient is written, zero where order and place do not
    name each other, and dy's rows by order."""
    T, E, top, m = 150, 5, 2, 72
    r = _routing(gpu, T, E, top, 0.1)
    S, big = T * top, 2 ** 31 - 1
    dout, y = _rand(gpu, T, m), _rand(gpu, S, m, seed=1)
    order, place, turned = r.order.clone(), r.place.clone(), r.order.clone()
    order[::3], order[1::7], order[2::11] = big, -big, S
    place[::3], place[1::5], place[2::9] = big, -5, S
    turned[40:60] = turned[40:60].flip(0)
    twice = r.place.clone()
    twice[:, 1] = twice[:, 0]
    bad = [r, r._replace(order=order), r._replace(place=place), r._replace(order=order, place=place), r._replace(order=turned),
           r._replace(place=twice)]
    for o in ([0, 3, 9, 20, 40, 50], [0, 10, 20, 30, 40, 0], [0, big, 3, -4, big, 7], [-1] * 6, [0, 300, 0, 300, 0, 290]):
        bad.append(r._replace(offsets=torch.tensor(o, dtype=torch.int32, device=gpu)))
    for q in bad:
        used = min(max(int(q.offsets[-1]), 0), S)
        dy, dw = _combine_gradient(q, dout, y)
        o, p = q.order.cpu().long(), q.place.cpu().long().reshape(-1)
        d64, y64, w = dout.double().cpu(), y.double().cpu(), q.weights.double().cpu().reshape(-1)
        rows, mag, want = torch.zeros(S, m).double(), torch.zeros(S).double(), torch.zeros(S).double()
        for k in range(S):
            if k < used and 0 <= int(o[k]) < S:
                rows[k] = w[o[k]] * d64[o[k] // top]
            if 0 <= int(p[k]) < used and int(o[p[k]]) == k:
                terms = d64[k // top] * y64[p[k]]
                want[k], mag[k] = terms.sum(), terms.abs().sum()
        _close(dw.cpu().reshape(-1), want, (m + 1) * 2.0 ** -24 * mag)
        _close(dy.cpu(), rows, 2.0 ** -24 * rows.abs())


def _dirty(gpu, *tensors):
    """Leaves NaN in the memory that tensors like these are made of next."""
    gone = [torch.full_like(t, math.nan) for t in tensors for _ in range(2)]
    del gone


@pytest.mark.parametrize("lo,hi", [(2, 5), (0, 4), (3, 7), (4, 5)])
@pytest.mark.parametrize("T,top,n,m", [(9, 2, 64, 40), (40, 3, 250, 77), (700, 2, 200, 333), (1500, 2, 520, 1032), (2500, 3, 1032, 1288)])
def test_some_of_the_experts(gpu, T, top, n, m, lo, hi):
    """offsets and weights of neighbouring experts alone, as a program has them that spreads its experts: the
    others' rows are in no expert, before the first one's as well as behind the last."""
    S = T * top
    r = _routing(gpu, T, 7, top, 0.1)
    q = r._replace(offsets=r.offsets[lo:hi + 1])
    a, b = int(q.offsets[0]), int(q.offsets[-1])
    out = torch.ones(S, dtype=torch.bool, device=gpu)
    out[a:b] = False
    W, bias = _rand(gpu, hi - lo, m, n, seed=1, scale=1 / math.sqrt(n)), _rand(gpu, hi - lo, m, seed=2)
    W64, b64 = W.double(), bias.double()
    z, dy = _rand(gpu, S, m, seed=3), _rand(gpu, S, m, seed=4)
    dy[out] = math.nan
    ws = torch.empty(1 << 28, dtype=torch.uint8, device=gpu)

    def zeros(*shape):
        return torch.zeros(shape, dtype=torch.float64, device=gpu)
    for by_slot in (False, True):
        x = _rand(gpu, S if by_slot else T, n, seed=5)
        _dirty(gpu, dy)
        ws.fill_(255)
        y, pre = ffe.expert_linear(x, W, q, bias=bias, activation="relu", keep_preact=True, by_slot=by_slot, workspace=ws)
        assert not bool(y[out].any()) and not bool(pre[out].any())
        assert torch.equal(y, torch.where(pre > 0, pre, torch.zeros_like(pre)))
        for e, rows, t in _parts(q):
            xe = x[rows if by_slot else t].double()
            want, mag = xe @ W64[e].T + b64[e], xe.abs() @ W64[e].abs().T + b64[e].abs()
            _close(pre[rows], want, HALF * 1.01 * want.abs() + (n + 1) * 2.0 ** -24 * mag)
        if by_slot:
            x[out] = 1e30
        for kept in (x, ffe.checkpoint_q8(x)):
            x64 = x.double() if kept is x else _value(kept)
            _dirty(gpu, dy, x, W, bias)
            ws.fill_(255)
            dx, dw, g, db = ffe.expert_linear_backward(dy, kept, W, q, preact=z, activation="relu", by_slot=by_slot, workspace=ws)
            assert torch.equal(g, torch.where(out[:, None] | (z <= 0), torch.zeros_like(dy), dy))
            g64 = g.double()
            far = S * 2.0 ** -38 * float(g64.abs().max() * (x64[a:b] if by_slot else x64).abs().max()) if b > a else 0.0
            rows_x, mags_x = zeros(S + 1, n), zeros(S + 1, n)
            ww, mw, wb, mb = zeros(*W.shape), zeros(*W.shape), zeros(hi - lo, m), zeros(hi - lo, m)
            for e, rows, t in _parts(q):
                ge, xe = g64[rows], x64[rows if by_slot else t]
                rows_x[rows], mags_x[rows] = ge @ W64[e], ge.abs() @ W64[e].abs()
                ww[e], mw[e], wb[e], mb[e] = ge.T @ xe, ge.abs().T @ xe.abs(), ge.sum(0), ge.abs().sum(0)
            if by_slot:
                assert not bool(dx[out].any())
                want, mag = rows_x[:S], mags_x[:S]
            else:   # (-1, no row: the zeros at the end)
                want, mag = rows_x[r.place.long()].sum(1), mags_x[r.place.long()].sum(1)
            _close(dx, want, HALF * 1.01 * want.abs() + (m + top) * 2.0 ** -24 * mag)
            _close(db, wb, HALF * 1.01 * wb.abs() + S * 2.0 ** -24 * mb)
            extra = 0 if kept is x else 2.0 ** -9 * mw + far
            _close(dw, ww, HALF * 1.01 * ww.abs() + S * 2.0 ** -24 * mw + extra)
    # the sums' gradient: of all rows and of these
    dout, y = _rand(gpu, T, m, seed=6), _rand(gpu, S, m, seed=7)
    (dyp, dwp), (dyf, dwf) = _combine_gradient(q, dout, y), _combine_gradient(r, dout, y)
    assert torch.equal(dyp, torch.where(out[:, None], torch.zeros_like(dyf), dyf))
    here = (r.place >= a) & (r.place < b)
    assert torch.equal(dwp, torch.where(here, dwf, torch.zeros_like(dwf)))


def test_rows_before_the_first_expert_do_not_count(gpu):
    """Numbers in rows before the first expert's do not set the powers of two around fp16."""
    T, E, n, m = 400, 4, 72, 40
    r = _routing(gpu, T, E, 1)
    q = r._replace(offsets=r.offsets[2:])
    a = int(q.offsets[0])
    assert a > 0
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T, m, seed=1), _rand(gpu, 2, m, n, seed=2)
    z = _rand(gpu, T, m, seed=3)
    x2, dy2 = x.clone(), dy.clone()
    x2[:a], dy2[:a] = 1e30, -1e35
    for kw in ({}, dict(preact=z, activation="silu"), dict(preact=ffe.checkpoint_q8(z), activation="gelu")):
        want = ffe.expert_linear_backward(dy, ffe.checkpoint_q8(x), W, q, by_slot=True, **kw)
        got = ffe.expert_linear_backward(dy2, ffe.checkpoint_q8(x2), W, q, by_slot=True, **kw)
        assert all(torch.equal(u, v) for u, v in zip(got, want))


def test_checkpoint_of_the_largest_number(gpu):
    """The one group whose scale times 127 leaves fp32: that of its largest number, which a mask may have put
    there.  Restored it is within half a scale, as any other, and dW of it is finite."""
    most = torch.finfo(F32).max
    x = _rand(gpu, 40, 96, dtype=F32)
    x[0, 3], x[1, 20], x[2] = most, -most, most
    x[3, 40] = float(torch.nextafter(torch.tensor(most), torch.tensor(0.0)))
    kept = ffe.checkpoint_q8(x, group=16)
    back = ffe.checkpoint_restore(kept, dtype=F32)
    assert bool(torch.isfinite(back).all())
    scale = torch.repeat_interleave(kept.scale.double(), 16, dim=1)
    # half a scale, and the scale's and the product's roundings and the step down: 127 times 2^-24, 2^-24 and 2^-23
    assert bool(((back.double() - x.double()).abs() <= scale * (0.5 + 127 * 2.0 ** -22)).all())
    assert float(back[0, 3]) == -float(back[1, 20]) and abs(float(back[0, 3]) / most - 1) <= 2.0 ** -22
    dy = torch.zeros((40, 24), dtype=BF16, device=gpu)
    dy[0], dy[1] = 2.0 ** -20, 2.0 ** -21
    dw = ffe.linear_backward(dy, kept, torch.zeros((24, 96), dtype=BF16, device=gpu), need_input=False)[1]
    want = dy.double().T @ x.double()
    assert bool(torch.isfinite(dw).all())
    _close(dw[:, 3], want[:, 3], 2 * HALF * want[:, 3].abs())
    _close(dw[:, 20], want[:, 20], 2 * HALF * want[:, 20].abs())
    # NaN and infinite scales stay what they are
    odd = ffe.Checkpoint(kept.codes, kept.scale.clone(), 16)
    odd.scale[5, 0], odd.scale[6, 0] = math.nan, math.inf
    back = ffe.checkpoint_restore(odd, dtype=F32)
    assert bool(back[5, :16].isnan().all()) and not bool(torch.isfinite(back[6, :16]).any())


class _Guarded:
    """Tensors among numbers that have to stay as they were."""

    def __init__(self, gpu):
        self.gpu, self.all = gpu, []

    def new(self, *shape, dtype=BF16):
        n, pad = math.prod(shape), 4096
        whole = torch.full((n + 2 * pad,), 7 if dtype is torch.uint8 else 7.0, dtype=dtype, device=self.gpu)
        self.all.append(whole)
        return whole[pad:pad + n].view(shape)

    def check(self):
        for whole in self.all:
            assert bool((whole[:4096] == 7).all()) and bool((whole[-4096:] == 7).all())


# tiles and streams of them, forms for few rows, ragged and whole
@pytest.mark.parametrize("T,E,top,n,m", [(150, 5, 2, 64, 72), (20, 40, 2, 130, 77), (900, 3, 2, 264, 520), (1500, 2, 1, 1032, 2056)])
def test_wrong_routings_write_nothing_else(gpu, T, E, top, n, m):
    """Arrays that are no routing: outputs and workspaces are written, nothing around them."""
    r, S, big = _routing(gpu, T, E, top, 0.1), T * top, 2 ** 31 - 1
    order, place = r.order.clone(), r.place.clone()
    order[::3], order[1::7], order[2::11] = big, -big, S
    place[::3], place[1::5], place[2::9] = big, -5, S
    g = torch.Generator().manual_seed(1)
    bad = [r._replace(order=order), r._replace(place=place), r._replace(order=order, place=place)]
    for o in ([big] * (E + 1), [-1] * (E + 1), [k % 2 * S for k in range(E + 1)], [(k + 1) % 2 * S for k in range(E + 1)],
              torch.randint(-S, 2 * S, (E + 1,), generator=g).tolist()):
        bad.append(r._replace(offsets=torch.tensor(o, dtype=torch.int32, device=gpu), order=order))
    W, b, z = _rand(gpu, E, m, n, seed=1), _rand(gpu, E, m, seed=2), _rand(gpu, S, m, seed=3)
    for by_slot in (False, True):
        x, dy = _rand(gpu, S if by_slot else T, n, seed=4), _rand(gpu, S, m, seed=5)
        kx = ffe.checkpoint_q8(x)
        X._library()
        for q in bad:
            at, mem = X._routing(q, x.device), _Guarded(gpu)

            def run(name, a):
                need = X._bytes(name + "_workspace_size", a, functions=X._FN)
                X._workspace(a, need, mem.new(need + 255, dtype=torch.uint8) if need else None, x.device)
                X._launch(name, a, x.device, X._FN)
            y, pre = mem.new(S, m), mem.new(S, m)
            run("ff_expert_linear", X.ff_expert_linear_args(at, n, m, x.data_ptr(), n, by_slot, W.data_ptr(), n, b.data_ptr(), 2,
                                                            y.data_ptr(), m, pre.data_ptr(), m))
            for kept in (x, kx):
                a = X.ff_expert_grad_args()
                a.routing, a.n, a.m, a.dy_dtype, a.dy, a.lddy, a.by_slot = at, n, m, X._elem(dy, "dy"), dy.data_ptr(), m, by_slot
                if kept is x:
                    a.x, a.ldx = x.data_ptr(), n
                else:
                    a.x_q8 = X._q8_rows(kx, "x", x.device)[0]
                gr, dx, dw, db = mem.new(S, m), mem.new(*x.shape), mem.new(E, m, n), mem.new(E, m)
                a.w, a.ldw, a.preact, a.ldz, a.activation, a.g, a.ldg = W.data_ptr(), n, z.data_ptr(), m, 3, gr.data_ptr(), m
                a.dx, a.lddx, a.dw, a.lddw, a.db = dx.data_ptr(), n, dw.data_ptr(), n, db.data_ptr()
                run("ff_expert_linear_backward", a)
            out = mem.new(T, m)
            X._launch("ff_expert_combine", X.ff_expert_combine_args(at, m, y.data_ptr(), m, None, 0, out.data_ptr(), m), x.device, X._FN)
            mem.check()


@pytest.mark.parametrize("T,E,n,m", [(200, 3, 72, 40), (2000, 2, 1032, 2056)])
def test_weight_gradient_of_wide_ranges(gpu, T, E, n, m):
    """Columns of g, and of x, far below the largest: among fp16's last bits they count still."""
    r = _routing(gpu, T, E, 1)
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T, m, seed=1), torch.zeros((E, m, n), dtype=BF16, device=gpu)
    dy[:, :8] *= 2.0 ** -20
    dy[:, 8:16] *= 2.0 ** -32
    x[:, :16] *= 2.0 ** -16
    x[:, 16:32] *= 2.0 ** -31
    kx = ffe.checkpoint_q8(x, group=16)
    _, dw, g, _ = ffe.expert_linear_backward(dy, kx, W, r, need_input=False)
    x64 = _value(kx)
    for e, rows, t in _parts(r):
        ge, xe = g[rows].double(), x64[t]
        want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
        # 2^-38 of the largest g beside each x, and of the largest x (127 times the largest scale) beside each g
        far = 2.0 ** -38 * (float(ge.abs().max()) * xe.abs().sum(0)[None] + ge.abs().sum(0)[:, None] * float(x64.abs().max()))
        far = far + len(t) * 2.0 ** -76 * float(ge.abs().max() * x64.abs().max())
        _close(dw[e], want, HALF * 1.01 * want.abs() + (2.0 ** -9 + T * 2.0 ** -24) * mag + far)


# tokens, experts, top, n, m: the form for few rows with one, two and four 16-row tiles a workgroup (k short and among
# many waves), beside it tiles with few rows an expert; weights as they lie and packed
@pytest.mark.parametrize("by_slot", [False, True])
@pytest.mark.parametrize("T,E,top,n,m", [(1, 64, 8, 1000, 777), (13, 1, 1, 520, 35), (20, 3, 2, 4096, 130), (40, 1, 1, 600, 333),
                                         (70, 4, 2, 1024, 1000), (30, 3, 2, 1001, 250), (100, 3, 1, 4097, 130), (8, 70, 5, 75, 2050),
                                         (60, 64, 1, 1024, 4104), (37, 130, 7, 264, 520), (400, 24, 2, 520, 2056),
                                         (9, 24, 8, 512, 777), (200, 16, 3, 1001, 900)])
def test_few_rows_an_expert(gpu, T, E, top, n, m, by_slot):
    for idle in (0.0, 0.5):
        r = _routing(gpu, T, E, top, idle)
        x, W, b = _rand(gpu, T * top if by_slot else T, n), _rand(gpu, E, m, n, seed=1, scale=0.05), _rand(gpu, E, m, seed=2)
        y, z = ffe.expert_linear(x, W, r, bias=b, activation="relu", keep_preact=True, by_slot=by_slot)
        used = int(r.offsets[-1])
        assert not bool(y[used:].any()) and not bool(z[used:].any())
        assert torch.equal(y, torch.where(z > 0, z, torch.zeros_like(z)))
        for e, rows, t in _parts(r):
            xe, we = x[rows if by_slot else t].double(), W[e].double()
            want, mag = xe @ we.T + b[e].double(), xe.abs() @ we.abs().T + b[e].double().abs()
            _close(z[rows], want, HALF * 1.01 * want.abs() + (n + 1) * 2.0 ** -24 * mag)


@pytest.mark.parametrize("T,E,n,m", [(140, 1, 1290, 2949), (859, 3, 2315, 1675), (1091, 2, 2572, 2315), (623, 1, 1774, 2308)])
def test_weight_gradients_of_128_wide_tiles(gpu, T, E, n, m):
    """In a stream up to 512 rows an expert, without one beyond."""
    r = _routing(gpu, T, E, 1, 0.05)
    x, dy, W = _rand(gpu, T, n), _rand(gpu, T, m, seed=1), torch.zeros((E, m, n), dtype=BF16, device=gpu)
    kx = ffe.checkpoint_q8(x)
    for kept in (x, kx):
        _, dw, g, db = ffe.expert_linear_backward(dy, kept, W, r, need_input=False)
        x64 = x.double() if kept is x else _value(kx)
        far = 0.0 if kept is x else T * 2.0 ** -38 * float(dy.double().abs().max() * x64.abs().max())
        for e, rows, t in _parts(r):
            ge, xe = g[rows].double(), x64[t]
            want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
            _close(dw[e], want, HALF * 1.01 * want.abs() + (T * 2.0 ** -24 + (0 if kept is x else 2.0 ** -9)) * mag + far)
            want, mag = ge.sum(0), ge.abs().sum(0)
            _close(db[e], want, HALF * 1.01 * want.abs() + T * 2.0 ** -24 * mag)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,dtype", [(7, F32), (61, BF16), (300, F32), (1000, BF16)])
def test_route_gradient_in_place(gpu, E, dtype, score):
    """dlogits as the logits' own rows, which lie apart."""
    T, top = 333, 4
    wide = _rand(gpu, T, E + 5, scale=2.0, dtype=dtype)
    logits, before = wide[:, 2:2 + E], wide.clone()
    r = ffe.route(logits, top, score=score)
    dw = _rand(gpu, T, top, seed=1, dtype=F32)
    want = ffe.route_backward(dw, logits, r.experts, score=score)
    X._library()
    a = X.ff_route_grad_args(T, E, top, X._elem(logits, "logits"), logits.data_ptr(), E + 5, dw.data_ptr(), r.experts.data_ptr(),
                             X.SCORES[score], 1, 1.0, logits.data_ptr(), E + 5)
    X._launch("ff_route_backward", a, wide.device, X._FN)
    assert torch.equal(logits, want)
    assert torch.equal(wide[:, :2], before[:, :2]) and torch.equal(wide[:, 2 + E:], before[:, 2 + E:])


def test_sums_onto_the_residual(gpu):
    """out as the residual's own rows."""
    T, E, top, m = 200, 5, 3, 133
    r = _routing(gpu, T, E, top, 0.2)
    y, wide = _rand(gpu, T * top, m), _rand(gpu, T, m + 7, seed=1)
    out, before = wide[:, 3:3 + m], wide.clone()
    want = ffe.expert_combine(y, r, residual=out)
    X._library()
    a = X.ff_expert_combine_args(X._routing(r, y.device), m, y.data_ptr(), m, out.data_ptr(), m + 7, out.data_ptr(), m + 7)
    X._launch("ff_expert_combine", a, y.device, X._FN)
    assert torch.equal(out, want)
    assert torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 3 + m:], before[:, 3 + m:])


def test_most_slots(gpu):
    """2^24 slots, the most that are taken: their order is the stable sort by expert."""
    T, E, top = 1 << 22, 9, 4
    logits = torch.randn((T, E), device=gpu, generator=torch.Generator(device=gpu).manual_seed(1))
    r = ffe.route(logits, top)
    assert torch.equal(r.experts.long(), torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :top])
    key = r.experts.reshape(-1)
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(T * top, device=gpu)
    assert torch.equal(r.order.long(), order) and torch.equal(r.place.long().reshape(-1), place)
    assert r.offsets.tolist() == [int((key < e).sum()) for e in range(E + 1)]
    with pytest.raises(ffe.FlipFlopError):
        ffe.expert_order(torch.zeros((T + 1, top), dtype=torch.int32, device=gpu), E)


@pytest.mark.parametrize("top", [1, 2])
def test_results_of_more_than_2_31_numbers(gpu, top):
    """Rows, codes and gradients whose offsets do not fit 32 bits: the last rows, and sums over all."""
    T, E, n, m = (1 << 18) // top, 2, 64, 8264
    S = T * top
    assert S * m > 1 << 31
    r = _routing(gpu, T, E, top)
    g = torch.Generator(device=gpu).manual_seed(2)
    x, W = _rand(gpu, T, n), _rand(gpu, E, m, n, seed=1, scale=0.1)
    y, _ = ffe.expert_linear(x, W, r)
    tokens = r.order.long() // top
    starts = r.offsets.tolist()
    rows = torch.tensor([0, 1, starts[1] - 1, starts[1], S // 2, S - 2, S - 1], device=gpu)
    experts = (rows >= starts[1]).long()
    want = torch.einsum("rn,rmn->rm", x[tokens[rows]].double(), W[experts].double())
    mag = torch.einsum("rn,rmn->rm", x[tokens[rows]].double().abs(), W[experts].double().abs())
    _close(y[rows], want, HALF * 1.01 * want.abs() + n * 2.0 ** -24 * mag)
    # the checkpoint of them, back, and as pre-activations
    kept = ffe.checkpoint_q8(y, group=256)
    some = ffe.checkpoint_q8(y[rows].contiguous(), group=256)
    assert torch.equal(kept.codes[rows], some.codes) and torch.equal(kept.scale[rows], some.scale)
    back = ffe.checkpoint_restore(kept)
    assert torch.equal(back[rows], ffe.checkpoint_restore(some))
    del back
    dy = torch.empty((S, m), dtype=BF16, device=gpu).normal_(generator=g)
    dx, dw, gr, db = ffe.expert_linear_backward(dy, x, W, r, preact=kept, activation="relu")
    assert torch.equal(gr[rows], torch.where(some.codes > 0, dy[rows], torch.zeros_like(dy[rows])))
    out = ffe.expert_combine(y, r)
    last = torch.tensor([0, T - 1], device=gpu)
    at = r.place[last].long()
    terms = r.weights[last].double()[:, :, None] * y[at].double()
    want = terms.sum(1)
    _close(out[last], want, HALF * 1.01 * want.abs() + (top + 1) * 2.0 ** -24 * terms.abs().sum(1))
    del y, out, dy, kept
    W64 = W.double()
    of = (at >= starts[1]).long()
    want = sum(torch.einsum("tm,tmn->tn", gr[at[:, j]].double(), W64[of[:, j]]) for j in range(top))
    mag = sum(torch.einsum("tm,tmn->tn", gr[at[:, j]].double().abs(), W64[of[:, j]].abs()) for j in range(top))
    _close(dx[last], want, HALF * 1.01 * want.abs() + (m + top) * 2.0 ** -24 * mag)
    for e, part, t in _parts(r):
        cols = torch.tensor([0, m // 2, m - 1], device=gpu)
        ge, xe = gr[part][:, cols].double(), x[t].double()
        want, mag = ge.T @ xe, ge.abs().T @ xe.abs()
        _close(dw[e][cols], want, HALF * 1.01 * want.abs() + S * 2.0 ** -24 * mag)
        _close(db[e][cols], ge.sum(0), HALF * 1.01 * ge.sum(0).abs() + S * 2.0 ** -24 * ge.abs().sum(0))
