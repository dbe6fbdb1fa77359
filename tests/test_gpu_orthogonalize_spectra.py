"""orthogonalize of bf16 updates whose spectrum decays or ends, against the
formula in 64 bits: the steps take up to 3.4445^5 = 485 of what a rounding puts
into directions that the update hardly has.

Tolerance (2-norm).  The result's rounding to bf16: 1.7e-3 of its norm.  Each
step rounds X, A and b A + c A A to fp16 for its products, 1.4e-4 (2^-12 / sqrt(3))
of each; within the update's own directions a step passes at most 5 of it on
(|3 b u + 5 c u^2| for u = s^2 up to 1.3) and later steps about as much as they
get, their signs changing: sqrt(5 steps) 5 1.4e-4 = 1.6e-3 for X, and as much for A and b A +
c A A together where their diagonals round alike (rows nearly orthogonal).  Into
the other directions X's rounding at the last step alone is passed on, by 3.4445
of 2.1e-4 or less.  Together below 4e-3."""
import pytest
import torch

import paper_2609_14706_amd as ffe
from test_gpu_orthogonalize import _formula

pytestmark = pytest.mark.gpu

TOL = 4e-3


def _update(kind, m, n, seed):
    g = torch.Generator().manual_seed(seed)

    def randn(*s):
        return torch.randn(s, generator=g, dtype=torch.float64)
    if kind.startswith("rank"):
        k = int(kind[4:])
        G = randn(m, k) @ randn(k, n)
    elif kind.startswith("floor"):      # four directions over noise
        G = randn(m, 4) @ randn(4, n) + float(kind[5:]) * randn(m, n)
    elif kind.startswith("power"):      # singular values i^-p
        r = min(m, n)
        u, v = torch.linalg.qr(randn(m, r))[0], torch.linalg.qr(randn(n, r))[0]
        G = (u * torch.arange(1, r + 1, dtype=torch.float64) ** -float(kind[5:])) @ v.T
    elif kind == "rows":                # an eighth of the rows, the others zero
        G = randn(m, n)
        G[m // 8:] = 0
    else:                               # one entry in a hundred
        G = randn(m, n) * (torch.rand(m, n, generator=g) < 0.01)
    return (1e-3 * G).to(torch.bfloat16)


KINDS = ["rank1", "rank8", "rank16", "floor0.001", "floor0.03", "floor0.1", "power0.5", "power1.5", "power3", "rows", "sparse"]


# matrices that one workgroup takes (96 x 80 in two parts, 128 x 128 in one), and larger ones
@pytest.mark.parametrize("m,n", [(96, 80), (128, 128), (100, 192), (150, 150), (300, 1000), (1000, 300), (512, 512)])
@pytest.mark.parametrize("kind", KINDS)
def test_spectra(gpu, kind, m, n):
    G = _update(kind, m, n, seed=m + n)
    want = _formula(G)
    got = ffe.orthogonalize(G.to(gpu)).double().cpu()
    assert float((got - want).norm()) <= TOL * float(want.norm())


@pytest.mark.parametrize("steps,abc", [(1, (3.4445, -4.7750, 2.0315)), (2, (3.4445, -4.7750, 2.0315)), (8, (1.875, -1.25, 0.375)),
                                       (12, (1.5, -0.5, 0.0))])
@pytest.mark.parametrize("m,n", [(128, 128), (300, 500)])
def test_other_steps(gpu, m, n, steps, abc):
    """Any number of steps, the last of them alone or at either buffer of X."""
    for kind in ("rank8", "floor0.03", "power1.5"):
        G = _update(kind, m, n, seed=steps)
        want = _formula(G, steps, abc)
        got = ffe.orthogonalize(G.to(gpu), steps=steps, coefficients=abc).double().cpu()
        assert float((got - want).norm()) <= TOL * float(want.norm()), kind


def test_batches_in_one_part(gpu):
    G = torch.stack([_update(k, 130, 200, seed=5) for k in ("rank16", "floor0.03", "rows")])
    got = ffe.orthogonalize(G.to(gpu)).double().cpu()
    for k in range(3):
        want = _formula(G[k])
        assert float((got[k] - want).norm()) <= TOL * float(want.norm())
