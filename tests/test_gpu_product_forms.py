"""linear, linear_q8 and orthogonalize in every form of their products (the
sizes of product_forms.py) against the formulas in 64 bits.

Tolerances: linear layers as in test_gpu_linear.py.  Updates as in
test_gpu_orthogonalize.py for the whole matrix, and for each element, whose errors are
of one size and independent, ten times their root mean square."""
import math

import pytest
import torch

import paper_2609_14706_amd as ffe
from product_forms import FEW, LENGTHS, LINEAR, ORTHO
from test_gpu_orthogonalize import DT, TOL, _formula

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
BF16 = torch.bfloat16


def _check(got, want, tol):
    bad = (got.double() - want).abs() > tol
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


def _bf16(gpu, T, n, m):
    g = torch.Generator(gpu).manual_seed(T + n + m)
    x, W = torch.randn(T, n, device=gpu, generator=g).to(BF16), (torch.randn(m, n, device=gpu, generator=g) / math.sqrt(n)).to(BF16)
    b, r = torch.randn(m, device=gpu, generator=g).to(BF16), torch.randn(T, m, device=gpu, generator=g).to(BF16)
    y, z = ffe.linear(x, W, bias=b, residual=r, activation="relu", keep_preact=True)
    x64, W64 = x.double(), W.double()
    z64 = x64 @ W64.T + b.double()
    tz = n * 2.0 ** -24 * (x64.abs() @ W64.abs().T) + 2.0 ** -23 * z64.abs() + 1e-30
    _check(z, z64, tz + HALF * z64.abs())
    y64 = z64.clamp(min=0) + r.double()
    _check(y, y64, tz + HALF * 1.01 * y64.abs())


def _int8(gpu, T, n, m):
    g = torch.Generator(gpu).manual_seed(T + n + m)
    q = torch.randint(-128, 128, (T, n), device=gpu, generator=g, dtype=torch.int8)
    Z = torch.randint(-128, 128, (m, n), device=gpu, generator=g, dtype=torch.int8)
    scale, beta = (torch.rand(k, device=gpu, generator=g) + 0.5 for k in (T, m))
    scale /= 70 * 70 * math.sqrt(n)
    b, r = torch.randn(m, device=gpu, generator=g).to(BF16), torch.randn(T, m, device=gpu, generator=g).to(BF16)
    y = ffe.linear_q8(q, scale, Z, beta, bias=b, residual=r, activation="relu")
    z64 = (q.double() @ Z.double().T) * scale.double()[:, None] * beta.double()
    tz = 2.0 ** -21 * (z64.abs() + (z64 + b.double()).abs()) + 1e-30
    y64 = (z64 + b.double()).clamp(min=0) + r.double()
    _check(y, y64, tz + HALF * 1.01 * y64.abs())


RUN = {"bf16": _bf16, "int8": _int8}


@pytest.mark.parametrize("kind,size", [(k, s) for k in RUN for s in LINEAR[k]])
def test_tiles(gpu, kind, size):
    RUN[kind](gpu, *size)


@pytest.mark.parametrize("kind,size", [(k, s) for k in RUN for s in FEW[k]])
def test_few_tokens(gpu, kind, size):
    RUN[kind](gpu, *size)


@pytest.mark.parametrize("kind", list(RUN))
@pytest.mark.parametrize("T,m", LENGTHS)
def test_lengths_of_k(gpu, T, m, kind):
    # whole 128-byte pieces of k, more than are ever in flight, and a last one that is cut
    unit = 64 if kind == "bf16" else 128
    for n in [unit * p - unit * cut // 64 for p in range(1, 10) for cut in (0, 8, 56)]:
        RUN[kind](gpu, T, n, m)


@pytest.mark.parametrize("kind,size", [(k, s) for k in DT for s in ORTHO[k]])
def test_updates(gpu, kind, size):
    batch, m, n = size
    g = torch.Generator(gpu).manual_seed(m + n)

    def randn(*s):
        return torch.randn(s, device=gpu, generator=g)
    G = torch.stack([1e-3 * (randn(m, 4) @ randn(4, n) + randn(m, n)) for _ in range(batch)]).to(DT[kind])
    got = ffe.orthogonalize(G)
    for k in {0, batch // 2, batch - 1}:
        want = _formula(G[k])     # its products in 64 bits on the GPU
        off = got[k].double() - want
        size = float(want.norm())
        assert float(off.norm()) <= TOL[kind] * size
        half = HALF if kind == "bf16" else 2.0 ** -24
        _check(got[k], want, half * want.abs() + 10 * TOL[kind] * size / math.sqrt(m * n))
