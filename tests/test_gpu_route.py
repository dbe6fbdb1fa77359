"""route, route_backward and expert_order against the definition in 64 bits.

Choices and orders are whole numbers and equal.  Scores are held in 64 bits
(exp and a division good to a few 2^-53 each), weights and gradients rounded once:
half a step of their type, and 1e-12 of the terms' magnitudes around it."""
import math

import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# tokens, experts, top, groups, top_groups: one workgroup and many, each number of
# experts a lane, groups of one, of all, and across lanes
SIZES = [(1, 1, 1, 1, 1), (1, 128, 8, 1, 1), (3, 5, 5, 1, 1), (64, 8, 8, 1, 1), (64, 256, 8, 8, 4), (65, 60, 4, 4, 2),
         (2, 1024, 64, 16, 8), (17, 12, 3, 12, 5), (200, 64, 1, 1, 1), (200, 65, 2, 5, 5), (333, 300, 7, 3, 1),
         (1000, 512, 10, 64, 8), (4100, 16, 2, 2, 1), (700, 1024, 6, 8, 3), (9000, 100, 3, 1, 1)]


def _logits(T, E, dtype, seed, step=None):
    g = torch.Generator().manual_seed(seed)
    v = 2 * torch.randn((T, E), generator=g)
    return (torch.round(v / step) * step if step else v).to(dtype)


def _scores(logits, score):
    v = logits.double()
    if score == "sigmoid":
        return 1 / (1 + torch.exp(-v))
    big = v.amax(dim=1, keepdim=True)
    e = torch.where(big == -math.inf, torch.zeros_like(v), torch.exp(v - big))
    total = e.sum(dim=1, keepdim=True)
    return torch.where(big == -math.inf, e, e / total)


def _rank(c):
    """Indices of each row by falling value, the lowest index first among equals; NaN last."""
    c = torch.where(c.isnan(), torch.full_like(c, -math.inf), c)
    return torch.sort(c, dim=1, descending=True, stable=True).indices


def _want(logits, top, score, bias, groups, top_groups, renorm, scale, mask):
    s = _scores(logits, score)
    T, E = s.shape
    c = s if bias is None else s + bias.double()
    order = _rank(c)
    if groups > 1:
        size = E // groups
        low = torch.where(c.isnan(), torch.full_like(c, -math.inf), c).view(T, groups, size)
        rank = torch.sort(low, dim=2, descending=True).values[:, :, :2].sum(dim=2)
        kept = torch.zeros((T, groups), dtype=torch.bool)
        kept.scatter_(1, _rank(rank)[:, :top_groups], True)
        inside = torch.gather(kept.repeat_interleave(size, dim=1), 1, order)
        order = torch.stack([torch.cat([o[i], o[~i]]) for o, i in zip(order, inside)])
    e = order[:, :top]
    w = torch.gather(s, 1, e)
    if renorm:
        total = w.sum(dim=1, keepdim=True)
        w = torch.where(total == 0, torch.zeros_like(w), w / torch.where(total == 0, torch.ones_like(total), total))
    w = scale * w
    if mask is not None:
        w = torch.where(mask[:, None], w, torch.zeros_like(w))
        e = torch.where(mask[:, None], e, -torch.ones_like(e))
    return w, e


def _check_order(r, experts, E):
    """order, offsets and place are the stable sort of the slots by expert."""
    flat = experts.reshape(-1).cpu().long()
    live = (flat >= 0) & (flat < E)
    key = torch.where(live, flat, torch.full_like(flat, E))
    order = torch.sort(key, stable=True).indices
    count = int(live.sum())
    offsets = torch.cat([torch.zeros(1, dtype=torch.long), torch.cumsum(torch.bincount(key, minlength=E + 1)[:E], 0)])
    place = torch.full((flat.numel(),), -1)
    place[order[:count]] = torch.arange(count)
    order = torch.where(torch.arange(flat.numel()) < count, order, torch.full_like(order, -1))
    assert torch.equal(r.order.cpu().long(), order)
    assert torch.equal(r.offsets.cpu().long(), offsets)
    assert torch.equal(r.place.cpu().long().reshape(-1), place)
    assert r.place.shape == experts.shape


def _check(gpu, logits, top, score="softmax", bias=None, groups=1, top_groups=1, renorm=True, scale=1.0, mask=None):
    r = ffe.route(logits.to(gpu), top, score=score, bias=None if bias is None else bias.to(gpu), groups=groups,
                  top_groups=top_groups, renormalise=renorm, scale=scale, mask=None if mask is None else mask.to(gpu))
    w, e = _want(logits, top, score, bias, groups, top_groups, renorm, scale, mask)
    assert torch.equal(r.experts.cpu().long(), e)
    got = r.weights.double().cpu()
    assert torch.equal(got.isnan(), w.isnan())
    ok = ~w.isnan()
    assert bool(((got - w).abs()[ok] <= (2.0 ** -24 + 1e-12) * w.abs()[ok] + 2.0 ** -149).all())
    _check_order(r, r.experts, logits.shape[1])
    return r


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,top,groups,top_groups", SIZES)
def test_route(gpu, T, E, top, groups, top_groups, dtype):
    g = torch.Generator().manual_seed(E)
    logits, bias = _logits(T, E, dtype, T + E), 0.2 * torch.randn(E, generator=g)
    mask = torch.rand(T, generator=g) < 0.8
    _check(gpu, logits, top, groups=groups, top_groups=top_groups)
    _check(gpu, logits, top, "sigmoid", bias, groups, top_groups, True, 2.5, mask)
    _check(gpu, logits, top, "softmax", bias, groups, top_groups, False, 1.0, None)
    _check(gpu, logits, top, "sigmoid", None, groups, top_groups, False, 0.3, mask)


@pytest.mark.parametrize("E,top,groups,top_groups", [(64, 6, 1, 1), (200, 9, 1, 1), (256, 8, 8, 3), (96, 4, 32, 2)])
def test_ties(gpu, E, top, groups, top_groups):
    """Equal logits: the lowest index first, of groups too."""
    logits = _logits(150, E, F32, 3, step=2.0)
    logits[:4] = 0
    for score in ("softmax", "sigmoid"):
        _check(gpu, logits, top, score, None, groups, top_groups)
        _check(gpu, logits, top, score, torch.zeros(E), groups, top_groups)


def test_neighbours_in_the_last_bits(gpu):
    """Scores that 32 bits do not tell apart are still in order."""
    E = 64
    logits = torch.zeros(100, E)
    logits[:, 40] = 2.0 ** -30          # e^(2^-30) is one in fp32
    logits[:, 7] = -(2.0 ** -30)
    r = _check(gpu, logits, 64)
    assert bool((r.experts[:, 0] == 40).all()) and bool((r.experts[:, 63] == 7).all())
    bias = torch.zeros(E)
    bias[50] = 2.0 ** -40               # 1 / 64 + 2^-40
    r = _check(gpu, torch.zeros(70, E), 2, bias=bias)
    assert bool((r.experts[:, 0] == 50).all()) and bool((r.experts[:, 1] == 0).all())


@pytest.mark.parametrize("groups,top_groups", [(1, 1), (4, 2)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_special_rows(gpu, score, groups, top_groups):
    E, inf, nan = 32, math.inf, math.nan
    logits = _logits(80, E, F32, 1)
    logits[0] = -inf                                  # nothing left
    logits[1, 3:] = -inf                              # fewer than top left
    logits[2] = 1e30                                  # far out
    logits[3] = -1e30
    logits[4, 0], logits[4, 1] = 3e38, -3e38
    logits[5, 9] = -inf
    logits[6] = -inf
    logits[6, 31] = 0
    logits[7] = -800.0                                # sigmoids below fp32, above zero in 64 bits
    logits[7, 5] = -745.0 if score == "softmax" else -700.0
    for renorm in (True, False):
        _check(gpu, logits, 6, score, None, groups, top_groups, renorm)
    bias = torch.zeros(E)
    bias[4], bias[8], bias[9] = inf, -inf, nan        # always, never, as if never
    _check(gpu, logits, 6, score, bias, groups, top_groups)
    # NaN (and under softmax +inf) rows: NaN weights where the scores are, and they harm no other row
    logits[10, 2], logits[11] = nan, nan
    if score == "softmax":
        logits[12, 3] = inf
    r = _check(gpu, logits, 4, score, None, groups, top_groups, False)
    rows = r.weights.isnan().any(dim=1).nonzero().flatten().tolist()
    assert rows == ([10, 11, 12] if score == "softmax" else [11])


def test_nothing_routed_and_no_tokens(gpu):
    logits = _logits(300, 20, F32, 1)
    r = _check(gpu, logits, 3, mask=torch.zeros(300, dtype=torch.bool))
    assert not bool(r.offsets.any()) and not bool(r.weights.any())
    r = ffe.route(logits[:0].to(gpu), 3)
    assert r.weights.shape == (0, 3) and r.order.shape == (0,) and torch.equal(r.offsets, torch.zeros_like(r.offsets))
    assert ffe.route_backward(r.weights, logits[:0].to(gpu), r.experts).shape == (0, 20)


@pytest.mark.parametrize("T,top,E", [(1, 1, 1), (5, 3, 2), (64, 8, 1024), (65, 7, 3), (513, 1, 100), (3000, 4, 1), (8000, 8, 777),
                                     (70000, 2, 1024)])
def test_expert_order(gpu, T, top, E):
    g = torch.Generator().manual_seed(T)
    # the same expert twice, many at one, and numbers that are none
    e = torch.randint(-2, E + 2, (T, top), generator=g, dtype=torch.int32)
    e = torch.where(torch.rand((T, top), generator=g) < 0.3, torch.full_like(e, E // 2), e)
    if T > 4:
        e[1, 0], e[2, 0] = 2 ** 31 - 1, -2 ** 31
    _check_order(ffe.expert_order(e.to(gpu), E), e, E)
    _check_order(ffe.expert_order(torch.full_like(e, E - 1).to(gpu), E), torch.full_like(e, E - 1), E)
    _check_order(ffe.expert_order(torch.full_like(e, -1).to(gpu), E), torch.full_like(e, -1), E)


def _grad_want(dw, logits, experts, score, renorm, scale):
    s = _scores(logits, score)
    live = (experts >= 0) & (experts < s.shape[1])
    e = torch.where(live, experts, torch.zeros_like(experts)).long()
    zero = torch.zeros_like(dw, dtype=torch.float64)
    w, d = torch.where(live, torch.gather(s, 1, e), zero), torch.where(live, scale * dw.double(), zero)
    mag = d.abs()
    if renorm:
        total = w.sum(dim=1, keepdim=True)
        total = torch.where(total == 0, torch.full_like(total, math.inf), total)
        mag = (mag + (mag * w).sum(dim=1, keepdim=True) / total) / total
        d = (d - (d * w).sum(dim=1, keepdim=True) / total) / total
    ds = torch.zeros_like(s).scatter_add_(1, e, torch.where(live, d, zero))
    ms = torch.zeros_like(s).scatter_add_(1, e, torch.where(live, mag, zero))
    if score == "sigmoid":
        return ds * s * (1 - s), ms * s
    return s * (ds - (s * ds).sum(dim=1, keepdim=True)), s * (ms + (s * ms).sum(dim=1, keepdim=True))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,top", [(1, 1, 1), (1, 128, 8), (7, 5, 5), (64, 60, 4), (333, 300, 7), (200, 1024, 64), (5000, 61, 2),
                                     (90, 512, 1)])
def test_route_backward(gpu, T, E, top, dtype):
    logits = _logits(T, E, dtype, T)
    g = torch.Generator().manual_seed(E)
    dw = torch.randn((T, top), generator=g)
    mask = torch.rand(T, generator=g) < 0.9
    for score in ("softmax", "sigmoid"):
        r = ffe.route(logits.to(gpu), top, score=score, mask=mask.to(gpu))
        for renorm, scale in ((True, 1.0), (False, 2.5)):
            got = ffe.route_backward(dw.to(gpu), logits.to(gpu), r.experts, score=score, renormalise=renorm, scale=scale)
            want, mag = _grad_want(dw, logits, r.experts.cpu(), score, renorm, scale)
            assert got.dtype is dtype and got.shape == (T, E)
            half = 2.0 ** -24 if dtype is F32 else 2.0 ** -8 + 2.0 ** -24
            assert bool(((got.double().cpu() - want).abs() <= half * want.abs() + 1e-12 * mag + 2.0 ** -133).all())
    # a choice twice counts twice, numbers that are none not at all
    e = torch.randint(-2, E + 2, (T, top), generator=g, dtype=torch.int32)
    got = ffe.route_backward(dw.to(gpu), logits.to(gpu), e.to(gpu), renormalise=False)
    want, mag = _grad_want(dw, logits, e, "softmax", False, 1.0)
    half = 2.0 ** -24 if dtype is F32 else 2.0 ** -8 + 2.0 ** -24
    assert bool(((got.double().cpu() - want).abs() <= half * want.abs() + 1e-12 * mag + 2.0 ** -133).all())


@pytest.mark.parametrize("score,renorm", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_route_backward_against_differences(gpu, score, renorm):
    """Steps of h on each logit that leave the choice as it is: (f(l + h) - f(l - h)) / 2h, off by
    h^2 / 6 of a third derivative (below 1 for both scores) times |dw|, and by the weights' fp32
    roundings 2^-24 / h."""
    T, E, top, h = 6, 9, 3, 2.0 ** -7
    logits = torch.stack([torch.randperm(E, generator=torch.Generator().manual_seed(k)).float() * 0.5 for k in range(T)])
    dw = torch.randn((T, top), generator=torch.Generator().manual_seed(1))
    r = ffe.route(logits.to(gpu), top, score=score, renormalise=renorm)
    got = ffe.route_backward(dw.to(gpu), logits.to(gpu), r.experts, score=score, renormalise=renorm).double().cpu()
    for e in range(E):
        f = []
        for sign in (1, -1):
            moved = logits.clone()
            moved[:, e] += sign * h
            q = ffe.route(moved.to(gpu), top, score=score, renormalise=renorm)
            assert torch.equal(q.experts, r.experts)
            f.append((q.weights.double().cpu() * dw.double()).sum(dim=1))
        diff = (f[0] - f[1]) / (2 * h)
        # renormalised weights' third derivatives: at most 6 over the chosen scores' smallest sum cubed, and scores >= 0.5 there
        tol = (h * h / 6 * (6 if renorm else 1) * 8 + 2.0 ** -23 / h) * dw.double().abs().sum(dim=1)
        assert bool(((got[:, e] - diff).abs() <= tol).all())


def test_strides_streams_and_workspace(gpu):
    wide = _logits(500, 90, BF16, 5).to(gpu)
    logits = wide[:, 3:80]
    plain = ffe.route(logits.contiguous(), 5, score="sigmoid")

    def same(a, b):
        return all(torch.equal(u, v) for u, v in zip(a, b))
    assert same(ffe.route(logits, 5, score="sigmoid"), plain)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = ffe.route(logits, 5, score="sigmoid", stream=side)
    again = ffe.expert_order(other.experts, 77, weights=other.weights, stream=side)
    dl = ffe.route_backward(other.weights, logits, other.experts, score="sigmoid", stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert same(other, plain) and same(again, plain)
    assert torch.equal(dl, ffe.route_backward(plain.weights, logits.contiguous(), plain.experts, score="sigmoid"))
    ws = torch.empty(1 << 20, dtype=torch.uint8, device=gpu)
    assert same(ffe.route(logits, 5, score="sigmoid", workspace=ws), plain)
    with pytest.raises(ValueError):
        ffe.route(logits, 5, workspace=ws[:64])


@pytest.mark.parametrize("T", [7, 900])
def test_captured(gpu, T):
    logits = _logits(T, 70, F32, 1).to(gpu)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = ffe.route(logits, 4)
        ffe.route_backward(r.weights, logits, r.experts)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = ffe.route(logits, 4)
        d = ffe.route_backward(r.weights, logits, r.experts)
    for k in range(4):
        logits.copy_(_logits(T, 70, F32, 10 + k))
        graph.replay()
        torch.cuda.synchronize()
        want = ffe.route(logits, 4)
        assert all(torch.equal(u, v) for u, v in zip(r, want))
        assert torch.equal(d, ffe.route_backward(want.weights, logits, want.experts))


def test_refusals(gpu):
    logits = _logits(8, 12, F32, 1).to(gpu)
    for kw in (dict(top=0), dict(top=13), dict(top=65), dict(top=2.0), dict(score="max"), dict(groups=5), dict(groups=0),
               dict(groups=4, top_groups=5), dict(groups=4, top_groups=0), dict(groups=4, top_groups=1, top=4),
               dict(bias=torch.zeros(11, device=gpu)), dict(mask=torch.ones(7, dtype=torch.bool, device=gpu)),
               dict(scale=math.inf), dict(scale=1e39)):
        with pytest.raises((ValueError, ffe.FlipFlopError)):
            ffe.route(logits, **{"top": 2, **kw})
    for bad, kw in ((logits.half(), {}), (logits.cpu(), {}), (logits, dict(bias=torch.zeros(12, device=gpu).double())),
                    (logits, dict(mask=torch.ones(8, device=gpu))), (logits, dict(bias=torch.zeros(12)))):
        with pytest.raises(TypeError):
            ffe.route(bad, 2, **kw)
    for bad in (logits[0], logits.view(2, 4, 12), logits.t()):
        with pytest.raises(ValueError):
            ffe.route(bad, 1)
    with pytest.raises(ffe.FlipFlopError):
        ffe.route(torch.zeros(2, 1025, device=gpu), 1)
    e = torch.zeros(8, 2, dtype=torch.int32, device=gpu)
    for args in ((e, 0), (e, 1025), (e.view(-1), 4), (e.long(), 4), (e.cpu(), 4)):
        with pytest.raises((ValueError, TypeError, ffe.FlipFlopError)):
            ffe.expert_order(*args)
    dw = torch.zeros(8, 2, device=gpu)
    for args in ((dw[:7], logits, e), (dw.double(), logits, e), (dw, logits, e[:7]), (dw, logits, e.long()), (dw, logits, None)):
        with pytest.raises((ValueError, TypeError)):
            ffe.route_backward(*args)


# a wave a token for few experts and many choices, groups within, across and beside lanes' experts, two
# experts a lane, one workgroup and many
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,top,groups,top_groups", [(30, 20, 17, 1, 1), (300, 50, 20, 5, 3), (70, 64, 64, 1, 1), (300, 64, 17, 64, 40), (9, 128, 24, 8, 2),
                                                       (500, 128, 40, 1, 1), (333, 256, 32, 64, 16), (7, 250, 60, 10, 4), (600, 500, 33, 50, 20), (90, 30, 4, 3, 2), (2000, 32, 16, 2, 1),
                                                       (400, 17, 2, 1, 1), (1000, 240, 16, 48, 9), (600, 252, 5, 63, 7)])
def test_route_other_forms(gpu, T, E, top, groups, top_groups, dtype):
    test_route(gpu, T, E, top, groups, top_groups, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,top", [(40, 200, 12), (600, 130, 64), (3, 256, 8), (2000, 30, 30)])
def test_route_backward_other_forms(gpu, T, E, top, dtype):
    test_route_backward(gpu, T, E, top, dtype)
