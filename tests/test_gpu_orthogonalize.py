"""orthogonalize against its formula in 64 bits (on the CPU) and by what it is for.

Tolerances (2-norm): a bf16 result is rounded once (about 1.7e-3 of its norm);
three operands a step are rounded to fp16 before (2^-11 / sqrt(3) of each at
most, random), which the steps pass on at most about doubled: sqrt(15) 2
2.8e-4 = 2.2e-3, together below 4e-3.  With fp32 operands in two fp16 parts
every product is good to about 4e-7: 15 of them, doubled, below 1e-5.  Doubled
holds for updates with a noise floor; directions that G lacks altogether grow
from roundings alone, by a = 3.4445 a step: 22-bit operands (2^-23 of the norm, which is 1)
give a matrix of rank one up to 485 2^-23 = 5.8e-5 there."""
import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
TOL = {"bf16": 4e-3, "f32": 1e-5}
ABC = (3.4445, -4.7750, 2.0315)


def _formula(G, steps=5, abc=ABC, eps=1e-7, scale=1.0):
    a, b, c = abc
    X = G.double()
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.mT
    X = X / (X.square().sum((-2, -1), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return scale * (X.mT if tall else X)


def _update(*shape, dtype="bf16", seed=0, size=1e-3):
    g = torch.Generator().manual_seed(seed)
    u, v = torch.randn(*shape[:-1], 4, generator=g), torch.randn(*shape[:-2], 4, shape[-1], generator=g)
    return (size * (u @ v + torch.randn(shape, generator=g))).to(DT[dtype])


def _close(got, want, dtype):
    got, want = got.double().cpu(), want
    assert got.shape == want.shape
    assert float((got - want).norm()) <= TOL[dtype] * float(want.norm())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 100), (100, 1), (7, 5), (64, 128), (128, 64), (65, 63), (96, 80),
                                 (130, 257), (333, 100), (256, 256), (500, 515), (1000, 777), (600, 1500)])
def test_formula(gpu, m, n, dtype):
    G = _update(m, n, dtype=dtype, seed=m + n)
    _close(ffe.orthogonalize(G.to(gpu)), _formula(G), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large(gpu, dtype):
    m, n = (2048, 2300) if dtype == "bf16" else (1100, 2048)
    G = _update(m, n, dtype=dtype, seed=1)
    # the oracle's products in 64 bits on the GPU
    _close(ffe.orthogonalize(G.to(gpu)), _formula(G.to(gpu)).cpu(), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,m,n", [(3, 64, 40), (5, 33, 130), (2, 300, 200), (40, 16, 16)])
def test_batches(gpu, batch, m, n, dtype):
    G = _update(batch, m, n, dtype=dtype, seed=batch)
    got = ffe.orthogonalize(G.to(gpu))
    for k in range(batch):
        _close(got[k], _formula(G[k]), dtype)


@pytest.mark.parametrize("size", [1e-20, 1e-3, 1.0, 1e18])
def test_magnitudes(gpu, size):
    G = _update(100, 140, dtype="f32", seed=3, size=size)
    _close(ffe.orthogonalize(G.to(gpu), eps=0.0), _formula(G, eps=0.0), "f32")


def test_steps_coefficients_and_scale(gpu):
    G = _update(90, 200, dtype="f32", seed=4)
    for steps, abc in ((1, ABC), (2, ABC), (8, (1.875, -1.25, 0.375)), (20, (1.5, -0.5, 0.0))):
        _close(ffe.orthogonalize(G.to(gpu), steps=steps, coefficients=abc, scale=0.25),
               _formula(G, steps, abc, scale=0.25), "f32")


def test_it_orthogonalises(gpu):
    """Coefficients that converge: orthonormal rows, the factor of the polar decomposition."""
    G = _update(60, 150, dtype="f32", seed=5)
    X = ffe.orthogonalize(G.to(gpu), steps=24, coefficients=(1.875, -1.25, 0.375)).double().cpu()
    assert float((X @ X.T - torch.eye(60, dtype=torch.float64)).norm()) <= 1e-4
    U, _, Vh = torch.linalg.svd(G.double(), full_matrices=False)
    assert float((X - U @ Vh).norm()) <= 1e-4 * 60 ** 0.5


def test_few_directions_and_none(gpu):
    G = torch.outer(torch.arange(1.0, 71.0), torch.arange(1.0, 91.0))
    assert float((ffe.orthogonalize(G.to(gpu)).double().cpu() - _formula(G)).norm()) <= ABC[0] ** 5 * 2.0 ** -23
    assert not bool(ffe.orthogonalize(torch.zeros(50, 60, device=gpu)).any())
    G = _update(2, 50, 60, dtype="f32", seed=6)
    G[0, 3, 4] = float("nan")
    got = ffe.orthogonalize(G.to(gpu))
    assert bool(got[0].isnan().all())
    _close(got[1], _formula(G[1]), "f32")


def test_strides(gpu):
    B = _update(3, 70, 133, dtype="bf16", seed=7).to(gpu)
    G = B[:, 1:66, 3:128]
    assert torch.equal(ffe.orthogonalize(G), ffe.orthogonalize(G.contiguous()))
    assert torch.equal(ffe.orthogonalize(G[1]), ffe.orthogonalize(G)[1])
    E = G[:1].expand(3, 65, 125)   # one matrix three times
    assert torch.equal(ffe.orthogonalize(E)[2], ffe.orthogonalize(G[0].contiguous()))


def test_same_bits_streams_and_workspace(gpu):
    G = _update(400, 520, dtype="bf16", seed=8).to(gpu)
    want = ffe.orthogonalize(G)
    assert torch.equal(want, ffe.orthogonalize(G))
    s = torch.cuda.Stream(gpu)
    s.wait_stream(torch.cuda.current_stream(gpu))
    got = ffe.orthogonalize(G, stream=s)
    torch.cuda.current_stream(gpu).wait_stream(s)
    assert torch.equal(got, want)
    ws = torch.full((16 << 20,), 255, dtype=torch.uint8, device=gpu)   # NaNs wherever it is read unwritten
    assert torch.equal(ffe.orthogonalize(G, workspace=ws[1:]), want)
    with pytest.raises(ValueError):
        ffe.orthogonalize(G, workspace=ws[:1000])


def test_refusals(gpu):
    G = torch.zeros(8, 8, device=gpu)
    with pytest.raises(TypeError):
        ffe.orthogonalize(G.cpu())
    with pytest.raises(TypeError):
        ffe.orthogonalize(G.half())
    with pytest.raises(ValueError):
        ffe.orthogonalize(G[0])
    with pytest.raises(ValueError):
        ffe.orthogonalize(G[:0])
    with pytest.raises(ValueError):
        ffe.orthogonalize(G.t()[:, :4])
    for kw in (dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(scale=float("inf")),
               dict(coefficients=(9.0, -4.0, 2.0)), dict(coefficients=(float("nan"), 0.0, 0.0))):
        with pytest.raises(ffe.FlipFlopError):
            ffe.orthogonalize(G, **kw)
    assert ffe.orthogonalize(torch.zeros(0, 8, 8, device=gpu)).shape == (0, 8, 8)
