"""The operators around a layer of experts together, as examples/expert_block.py
uses them: the example runs, and its gradients are those of the block.

The gradients are compared with the block's in 64 bits, on the same choice of
experts, by the norm of the difference.  A bf16 rounding is off by at most 2^-8 of a
value, in norm 2^-8 / sqrt(3) = 2.3e-3 of it, an 8-bit checkpoint by at most half a
254th of its group's largest, in norm 1 / (254 sqrt(3)) times the 3 to 4 that the largest
of 128 normal values is of their rms: 8e-3.  On the way of each gradient lie at most
ten bf16 tensors (h, logits, z, u, v, dl, dy, g, their products' results) and two
checkpoints, each a factor of its terms: sqrt(10) 2.3e-3 + 2 8e-3 = 2.3e-2, and cancellation in the
router's gradient (a difference of products of the experts' outputs) up to three times that."""
import importlib.util
import math
import os

import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("expert_block", os.path.join(ROOT, "examples", "expert_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("hidden,inner,experts,top,tokens", [(256, 384, 8, 2, 2048), (120, 200, 5, 3, 1001)])
def test_example_runs(gpu, hidden, inner, experts, top, tokens):
    out = _example().run(hidden, inner, experts, top, tokens, steps=4)
    assert len(out["losses"]) == 4 and all(math.isfinite(v) for v in out["losses"])
    assert sum(out["rows"]) == tokens * top
    for name, n, m in (("W1", hidden, inner), ("W2", inner, hidden)):
        A, B = out["factors"][name]
        assert A.shape == (n, n) and B.shape == (m, m)
        assert abs(float(A.trace()) / n - 1) < 1e-3 and bool(torch.isfinite(B).all()) and bool((B.diagonal() > 0).all())


def _block64(x, p, experts, live):
    """The block in 64 bits on given choices (T, top)."""
    h = x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + 1e-6) * p["norm"]
    s = torch.softmax(h @ p["Wr"].T, dim=1).gather(1, experts)
    w = s / s.sum(dim=1, keepdim=True)
    y = x
    for j in range(experts.shape[1]):
        e = experts[:, j]
        z = torch.einsum("tn,tmn->tm", h, p["W1"][e]) + p["b1"][e]
        v = torch.einsum("tm,tnm->tn", z * torch.sigmoid(z), p["W2"][e])
        y = y + torch.where(live[:, None], w[:, j, None] * v, 0)
    return y


@pytest.mark.parametrize("padded", [False, True])
@pytest.mark.parametrize("hidden,inner,experts,top,tokens", [(128, 192, 6, 2, 200), (72, 40, 3, 3, 77), (64, 64, 16, 1, 150)])
def test_gradients_of_the_block(gpu, hidden, inner, experts, top, tokens, padded):
    ex = _example()
    gen = torch.Generator(device=gpu)
    gen.manual_seed(hidden)
    p = ex.new_block(hidden, inner, experts, gen, gpu)
    p["b1"] = (0.3 * torch.randn(p["b1"].shape, generator=gen, device=gpu)).to(torch.bfloat16)
    x = torch.randn((tokens, hidden), generator=gen, device=gpu).to(torch.bfloat16)
    dy = torch.randn((tokens, hidden), generator=gen, device=gpu).to(torch.bfloat16)
    live = torch.arange(tokens, device=gpu) < (tokens - tokens // 6 if padded else tokens)
    y, kept = ex.forward(x, p, top, mask=live if padded else None)
    grads, _ = ex.backward(dy, p, kept)
    r = kept[3]
    assert torch.equal(r.experts[:, 0] >= 0, live)
    q = {k: v.double().cpu().requires_grad_() for k, v in p.items()}
    x64 = x.double().cpu().requires_grad_()
    want = _block64(x64, q, r.experts.long().clamp(min=0).cpu(), live.cpu())
    want.backward(dy.double().cpu())

    def off(a, b):
        return float((a.double().cpu() - b).norm() / b.norm())
    assert off(y, want.detach()) < 0.023
    assert off(grads["x"], x64.grad) < 0.023
    for name, v in q.items():
        if name == "Wr" and top == 1:   # one weight of one: no gradient but roundings
            assert float(grads[name].double().norm()) < 1e-6 * float(v.detach().norm()) * tokens
            continue
        assert off(grads[name], v.grad) < (0.07 if name == "Wr" else 0.023), name


def test_two_streams_at_once(gpu):
    """The same block on two streams, each with its own workspaces from torch."""
    ex = _example()
    gen = torch.Generator(device=gpu)
    gen.manual_seed(3)
    p = ex.new_block(96, 160, 4, gen, gpu)
    xs = [torch.randn((300, 96), generator=gen, device=gpu).to(torch.bfloat16) for _ in range(2)]
    dy = torch.randn((300, 96), generator=gen, device=gpu).to(torch.bfloat16)

    def step(x):
        y, kept = ex.forward(x, p, 2)
        return [y] + list(ex.backward(dy, p, kept)[0].values())
    want = [step(x) for x in xs]
    streams = [torch.cuda.Stream() for _ in xs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(3):
        for s, x in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(step(x))
    torch.cuda.synchronize()
    for k, out in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(out, want[k % 2]))
