"""linear, linear_q8 and linear_backward against the formulas in 64 bits.

Tolerances: a product's fp32 sum of n terms is off by at most n 2^-24 of the
sum of magnitudes (8-bit sums are exact, their conversion and scaling three
roundings); the activations' slopes are below 1.13; exp is good to 2^-18 of an
activation at these arguments; outputs are rounded once to bf16 (2^-8)."""
import math

import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
BF16 = torch.bfloat16
ACTS = ["none", "relu", "gelu", "silu"]

# tokens, n, m: single tokens, each width of the few-token form and its ends, both
# tiles and their edges, k split and not, k that ends inside a step
SIZES = [(1, 64, 16), (1, 4096, 1000), (2, 100, 33), (7, 1001, 250), (16, 777, 130), (17, 512, 512), (33, 640, 8200),
         (48, 250, 300), (64, 2049, 65), (65, 1, 1), (65, 8, 129), (100, 2000, 300), (128, 128, 128), (129, 1000, 257),
         (300, 72, 1000), (513, 520, 777), (1000, 136, 640), (3000, 320, 4000), (4100, 1032, 3208)]


def _rand(gpu, *shape, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(BF16).to(gpu)


def _act64(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def _close(got, want, tol):
    assert got.shape == want.shape
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("T,n,m", SIZES)
def test_linear(gpu, T, n, m):
    x, W = _rand(gpu, T, n, seed=1), _rand(gpu, m, n, seed=2, scale=2 / math.sqrt(n))
    b, r = _rand(gpu, m, seed=3), _rand(gpu, T, m, seed=4)
    x64, W64 = x.double(), W.double()
    prod, mag = x64 @ W64.T, x64.abs() @ W64.abs().T
    for act, bias, res in (("none", None, None), ("relu", b, None), ("gelu", b, r), ("silu", None, r)):
        y, z = ffe.linear(x, W, bias=bias, residual=res, activation=act, keep_preact=act != "relu")
        z64 = prod + (bias.double() if bias is not None else 0)
        tz = n * 2.0 ** -24 * mag + 2.0 ** -23 * z64.abs() + 1e-30
        if z is not None:
            _close(z, z64, tz + HALF * z64.abs())
        a64 = _act64(z64, act)
        y64 = a64 + (res.double() if res is not None else 0)
        _close(y, y64, 1.13 * tz + 2.0 ** -18 * a64.abs() + HALF * 1.01 * y64.abs())


@pytest.mark.parametrize("T,n,m", SIZES)
def test_linear_q8(gpu, T, n, m):
    g = torch.Generator().manual_seed(n + m)
    q = torch.randint(-127, 128, (T, n), generator=g, dtype=torch.int8).to(gpu)
    Z = torch.randint(-128, 128, (m, n), generator=g, dtype=torch.int8).to(gpu)
    scale = (torch.rand(T, generator=g) + 0.5).to(gpu) / (70 * 70 * math.sqrt(n))
    beta = (torch.rand(m, generator=g) + 0.5).to(gpu)
    b, r = _rand(gpu, m, seed=3), _rand(gpu, T, m, seed=4)
    prod = (q.double() @ Z.double().T) * scale.double()[:, None] * beta.double()
    for act, bias, res in (("none", None, None), ("silu", b, r), ("gelu", None, None), ("relu", None, r)):
        y = ffe.linear_q8(q, scale, Z, beta, bias=bias, residual=res, activation=act)
        z64 = prod + (bias.double() if bias is not None else 0)
        tz = 2.0 ** -21 * (prod.abs() + z64.abs()) + 1e-30
        a64 = _act64(z64, act)
        y64 = a64 + (res.double() if res is not None else 0)
        _close(y, y64, 1.13 * tz + 2.0 ** -18 * a64.abs() + HALF * 1.01 * y64.abs())


def test_q8_longest_sums(gpu):
    """The largest n: sums of 127^2 131072 just stay inside 32 bits."""
    n = 131072
    q = torch.full((3, n), 127, dtype=torch.int8, device=gpu)
    Z = torch.full((5, n), -127, dtype=torch.int8, device=gpu)
    one = torch.ones(5, device=gpu)
    want = torch.full((3, 5), -127.0 * 127.0 * n).to(BF16).to(gpu)
    assert torch.equal(ffe.linear_q8(q, one[:3].clone(), Z, one), want)
    q = q[:1].expand(70, n).contiguous()
    y = ffe.linear_q8(q, torch.ones(70, device=gpu), Z, one)
    assert torch.equal(y, want[:1].expand(70, 5))
    with pytest.raises(ffe.FlipFlopError):
        ffe.linear_q8(torch.zeros(1, n + 16, dtype=torch.int8, device=gpu), one[:1].clone(),
                      torch.zeros(5, n + 16, dtype=torch.int8, device=gpu), one)


@pytest.mark.parametrize("pairs", range(1, 10))
@pytest.mark.parametrize("T,m", [(70, 100), (200, 130), (300, 500)])
def test_lengths_of_k(gpu, T, m, pairs):
    # every number of 128-byte pieces up to more than are ever in flight, whole
    # and with a last one that is cut
    for n in (64 * pairs, 64 * pairs - 8, 64 * pairs - 56):
        x, W = _rand(gpu, T, n, seed=n), _rand(gpu, m, n, seed=n + 1, scale=2 / math.sqrt(n))
        x64, W64 = x.double(), W.double()
        want = x64 @ W64.T
        _close(ffe.linear(x, W)[0], want, n * 2.0 ** -24 * (x64.abs() @ W64.abs().T) + HALF * 1.01 * want.abs() + 1e-30)


@pytest.mark.parametrize("T", [3, 40, 200])
def test_strides_alignment_and_higher_rank(gpu, T):
    n, m = 250, 130
    xb, wb, rb = _rand(gpu, T, 301, seed=1), _rand(gpu, m, 333, seed=2), _rand(gpu, T, 141, seed=3)
    x, W, r = xb[:, 5:255], wb[:, 7:257], rb[:, 1:131]
    y, z = ffe.linear(x, W, residual=r, activation="silu", keep_preact=True)
    yc, zc = ffe.linear(x.contiguous(), W.contiguous(), residual=r.contiguous(), activation="silu", keep_preact=True)
    assert torch.equal(y, yc) and torch.equal(z, zc)
    x3 = x.contiguous().view(1, T, n)
    y3, _ = ffe.linear(x3, W.contiguous(), activation="relu")
    assert y3.shape == (1, T, m)
    one, _ = ffe.linear(x[0].contiguous(), W.contiguous())
    assert one.shape == (m,)
    # the product does not depend on which rows lie beside a row
    if T > 1:
        q, s = ffe.quantize_rows(x)
        Z = (W.float() * 100).round().clamp(-128, 127).to(torch.int8)
        beta = torch.ones(m, device=gpu)
        yq = ffe.linear_q8(q, s, Z, beta)
        qb = torch.zeros(T, 333, dtype=torch.int8, device=gpu)
        qb[:, 3:253] = q
        assert torch.equal(yq, ffe.linear_q8(qb[:, 3:253], s, Z, beta))
        assert torch.equal(yq[1:2], ffe.linear_q8(q[1:2], s[1:2], Z, beta))


def test_special_values(gpu):
    """NaN and infinities stay in the rows and columns that they belong to."""
    for T in (5, 200):
        x, W = _rand(gpu, T, 264, seed=1), _rand(gpu, 140, 264, seed=2)
        want, _ = ffe.linear(x, W)
        x2, W2 = x.clone(), W.clone()
        x2[1, 263] = float("nan")
        W2[3, 0] = float("inf")
        y, _ = ffe.linear(x2, W2)
        assert bool(y[1].isnan().all()) and not bool(y[0].isnan().any())
        keep = torch.ones_like(y, dtype=torch.bool)
        keep[1], keep[:, 3] = False, False
        assert torch.equal(y[keep], want[keep])
        assert bool(y[:, 3][x2[:, 0] > 0].isinf().any())


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("T,n,m", [(1, 64, 48), (5, 33, 100), (64, 520, 130), (65, 100, 77), (200, 264, 1000),
                                   (517, 640, 391), (1030, 1000, 2050), (2048, 2100, 2304)])
def test_backward(gpu, T, n, m, act):
    x, W, dy = _rand(gpu, T, n, seed=1), _rand(gpu, m, n, seed=2, scale=2 / math.sqrt(n)), _rand(gpu, T, m, seed=3)
    z = _rand(gpu, T, m, seed=4, scale=2.0) if act != "none" else None
    dx, dw, g, db = ffe.linear_backward(dy, x, W, preact=z, activation=act)
    if act == "none":
        assert torch.equal(g, dy)
    else:
        z64 = z.double().requires_grad_()
        _act64(z64, act).sum().backward()
        slope = z64.grad if act != "relu" else (z > 0).double()
        want = dy.double() * slope
        _close(g, want, HALF * want.abs() + 2.0 ** -16 * dy.double().abs())
    g64, x64, W64 = g.double(), x.double(), W.double()
    want, mag = g64 @ W64, g64.abs() @ W64.abs()
    _close(dx, want, m * 2.0 ** -24 * mag + HALF * 1.01 * want.abs() + 1e-30)
    want, mag = g64.T @ x64, g64.abs().T @ x64.abs()
    _close(dw, want, T * 2.0 ** -24 * mag + HALF * 1.01 * want.abs() + 1e-30)
    want, mag = g64.sum(0), g64.abs().sum(0)
    _close(db, want, T * 2.0 ** -24 * mag + HALF * 1.01 * want.abs() + 1e-30)
    # what is not needed changes nothing of the rest
    only = ffe.linear_backward(dy, x, W, preact=z, activation=act, need_input=False, need_bias=False)
    assert only[0] is None and only[3] is None and torch.equal(only[1], dw) and torch.equal(only[2], g)
    only = ffe.linear_backward(dy, x, W, preact=z, activation=act, need_weight=False)
    assert only[1] is None and torch.equal(only[0], dx) and torch.equal(only[3], db)


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_slopes_against_differences(gpu, act):
    z = torch.linspace(-12, 12, 4096).to(BF16).to(gpu).view(1, -1)
    one = torch.ones_like(z)
    g = ffe.linear_backward(one, torch.ones(1, 8, dtype=BF16, device=gpu), torch.ones(4096, 8, dtype=BF16, device=gpu),
                            preact=z, activation=act, need_input=False, need_weight=False, need_bias=False)[2]
    h = 1e-4
    want = (_act64(z.double() + h, act) - _act64(z.double() - h, act)) / (2 * h)
    _close(g, want, HALF * want.abs() + 2.0 ** -16)
    # far out, where squares overflow: 0 and 1, no NaN
    far = torch.tensor([[-3e38, -1e20, 1e20, 3e38]], device=gpu).to(BF16)
    g = ffe.linear_backward(torch.ones_like(far), torch.ones(1, 8, dtype=BF16, device=gpu),
                            torch.ones(4, 8, dtype=BF16, device=gpu), preact=far, activation=act, need_input=False,
                            need_weight=False, need_bias=False)[2]
    assert g.tolist() == [[0.0, 0.0, 1.0, 1.0]]


def test_forward_and_backward_are_adjoint(gpu):
    """<dy, W v> = <W^T dy, v> and <dy, U x> = <dW, U> across the two calls."""
    T, n, m = 300, 500, 400
    x, W, dy, v = (_rand(gpu, *s, seed=k) for k, s in enumerate([(T, n), (m, n), (T, m), (T, n)]))
    U = _rand(gpu, m, n, seed=9)
    dx, dw, _, _ = ffe.linear_backward(dy, x, W)
    for left, right in (((dy, ffe.linear(v, W)[0]), (dx, v)), ((dy, ffe.linear(x, U)[0]), (dw, U))):
        a, b = (p[0].double() * p[1].double() for p in (left, right))
        # independent roundings of 2^-8 on each side's terms: ten standard deviations
        tol = 10 * HALF * float(a.norm() + b.norm())
        assert abs(float(a.sum() - b.sum())) <= tol


def test_backward_of_strided_inputs(gpu):
    T, n, m = 150, 250, 130
    xb, wb, db_, zb = _rand(gpu, T, 300, seed=1), _rand(gpu, m, 301, seed=2), _rand(gpu, T, 133, seed=3), _rand(gpu, T, 151, seed=4)
    x, W, dy, z = xb[:, 1:251], wb[:, 2:252], db_[:, 3:133], zb[:, 5:135]
    got = ffe.linear_backward(dy, x, W, preact=z, activation="gelu")
    want = ffe.linear_backward(dy.contiguous(), x.contiguous(), W.contiguous(), preact=z.contiguous(), activation="gelu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_tokens(gpu):
    x = torch.empty(0, 64, dtype=BF16, device=gpu)
    W = _rand(gpu, 48, 64)
    y, z = ffe.linear(x, W, keep_preact=True)
    assert y.shape == (0, 48) and z.shape == (0, 48)
    dx, dw, g, db = ffe.linear_backward(y, x, W)
    assert dx.shape == (0, 64) and not bool(dw.any()) and not bool(db.any())
    q = torch.empty(0, 64, dtype=torch.int8, device=gpu)
    assert ffe.linear_q8(q, torch.empty(0, device=gpu), torch.zeros(48, 64, dtype=torch.int8, device=gpu),
                         torch.ones(48, device=gpu)).shape == (0, 48)


def test_on_another_stream_and_in_a_workspace(gpu):
    x, W, dy = _rand(gpu, 333, 515, seed=1), _rand(gpu, 140, 515, seed=2), _rand(gpu, 333, 140, seed=3)
    want = (ffe.linear(x, W)[0], *ffe.linear_backward(dy, x, W))
    s = torch.cuda.Stream(gpu)
    s.wait_stream(torch.cuda.current_stream(gpu))
    got = (ffe.linear(x, W, stream=s)[0], *ffe.linear_backward(dy, x, W, stream=s))
    torch.cuda.current_stream(gpu).wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.full((64 << 20,), 255, dtype=torch.uint8, device=gpu)    # NaNs wherever it is read unwritten
    got = (ffe.linear(x, W, workspace=ws[3:])[0], *ffe.linear_backward(dy, x, W, workspace=ws))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError):
        ffe.linear(x, W, workspace=ws[:1024])
    with pytest.raises(ValueError):
        ffe.linear_backward(dy, x, W, workspace=ws[:1024])


def test_in_a_graph(gpu):
    """Captured once, replayed on new inputs: each replay against the eager result."""
    x, W, dy = _rand(gpu, 333, 512, seed=1), _rand(gpu, 140, 512, seed=2), _rand(gpu, 333, 140, seed=3)
    n = torch.ones(512, dtype=BF16, device=gpu)

    def step():
        h, _ = ffe.rms_norm(x, n)
        y, z = ffe.linear(h, W, activation="silu", keep_preact=True)
        return (y, *ffe.linear_backward(dy, h, W, preact=z, activation="silu"), ffe.orthogonalize(W))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(_rand(gpu, 333, 512, seed=10 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals(gpu):
    x, W = _rand(gpu, 4, 64), _rand(gpu, 48, 64)
    b, r = _rand(gpu, 48), _rand(gpu, 4, 48)
    with pytest.raises(TypeError):
        ffe.linear(x.float(), W)
    with pytest.raises(TypeError):
        ffe.linear(x, W.float())
    with pytest.raises(TypeError):
        ffe.linear(x, W, bias=b.float())
    with pytest.raises(ValueError):
        ffe.linear(x, W[:, :63])
    with pytest.raises(ValueError):
        ffe.linear(x, W, bias=b[:47])
    with pytest.raises(ValueError):
        ffe.linear(x, W, residual=r[:3])
    with pytest.raises(ValueError):
        ffe.linear(x, W, activation="tanh")
    with pytest.raises(ValueError):
        ffe.linear(x, W.t().contiguous().t())
    q, Z = torch.zeros(4, 64, dtype=torch.int8, device=gpu), torch.zeros(48, 64, dtype=torch.int8, device=gpu)
    s, beta = torch.ones(4, device=gpu), torch.ones(48, device=gpu)
    with pytest.raises(TypeError):
        ffe.linear_q8(x, s, Z, beta)
    with pytest.raises(TypeError):
        ffe.linear_q8(q, s, Z.int(), beta)
    with pytest.raises(TypeError):
        ffe.linear_q8(q, None, Z, beta)
    with pytest.raises(ValueError):
        ffe.linear_q8(q, s[:3], Z, beta)
    with pytest.raises(ValueError):
        ffe.linear_backward(r, x, W, activation="gelu")
    with pytest.raises(ValueError):
        ffe.linear_backward(r[:3], x, W)
