"""One feed-forward block from its training to its codes, on one MI355X.

    y = x + W2 act(W1 norm(x))

1. Training: the block learns another block's outputs; every weight's update is
   orthogonalised (rms_norm, linear, their gradients, orthogonalize).
2. Calibration: the tokens of each layer, its input rows and the gradients of
   its pre-activations, give its Kronecker curvature A (x) B (FlipFlop).
3. Quantisation: WaterKron turns each layer into integer codes under that
   curvature (FlipFlop.quantize).
4. Serving: the block runs from 8-bit rows and codes (rms_norm_q8,
   quantize_rows, linear_q8).

    python examples/layer_block.py [hidden] [inner] [tokens] [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2609_14706_amd as ffe  # noqa: E402

ACT = "silu"


def forward(x, p):
    """The block's output and what its gradient needs."""
    h, s = ffe.rms_norm(x, p["norm"])
    u, z = ffe.linear(h, p["W1"], bias=p["b1"], activation=ACT, keep_preact=True)
    y, _ = ffe.linear(u, p["W2"], residual=s)
    return y, (s, h, z, u)


def backward(dy, p, kept):
    """(gradients by name, tokens (x, g) of each layer)."""
    s, h, z, u = kept
    du, dW2, g2, _ = ffe.linear_backward(dy, u, p["W2"], need_bias=False)
    dh, dW1, g1, db1 = ffe.linear_backward(du, h, p["W1"], preact=z, activation=ACT)
    _, dnorm = ffe.rms_norm_backward(dh, s, p["norm"], dsum=dy)
    return {"W1": dW1, "W2": dW2, "b1": db1, "norm": dnorm}, {"W1": (h, g1), "W2": (u, g2)}


def new_block(n, m, gen, device, scale=1.0):
    def r(*shape):
        return torch.randn(shape, generator=gen, device=device)
    p = {"norm": torch.ones(n, device=device), "W1": scale * r(m, n) / n ** 0.5, "b1": torch.zeros(m, device=device),
         "W2": scale * r(n, m) / m ** 0.5}
    return {k: v.to(torch.bfloat16) for k, v in p.items()}


def train(p, teacher, tokens, steps, gen, rate=0.02):
    """The loss of each step; p is updated in place from fp32 copies."""
    n = p["norm"].numel()
    master = {k: v.float() for k, v in p.items()}
    momentum = {k: torch.zeros_like(v) for k, v in master.items()}
    losses = []
    for k in range(steps):
        x = torch.randn((tokens, n), generator=gen, device=p["norm"].device).to(torch.bfloat16)
        want, _ = forward(x, teacher)
        y, kept = forward(x, p)
        diff = y.float() - want.float()
        losses.append(float(diff.square().mean()))
        grads, _ = backward((diff / diff.numel() ** 0.5).to(torch.bfloat16), p, kept)
        step = rate * (1 - k / steps)
        for name, g in grads.items():
            mom = momentum[name].mul_(0.9).add_(g.float())
            if g.dim() == 2:   # an update of norm one in every direction, scaled to the weights' entries
                rows, cols = g.shape
                mom = ffe.orthogonalize(mom, scale=max(rows, cols) ** 0.5 * 0.2)
                master[name].sub_(step * mom)
            else:
                master[name].sub_(step * mom / (mom.norm() / mom.numel() ** 0.5 + 1e-12))
            p[name].copy_(master[name])
    return losses


def quantise(p, tokens, gamma, iters=3):
    """{layer: (codes int8, alpha, beta, V)} under the layers' Kronecker curvature."""
    out = {}
    for name, (x, g) in tokens.items():
        f = ffe.FlipFlop(tokens=(x.contiguous(), g.contiguous()), damping=0.1)
        f.iterate(iters)
        Z, V, alpha, beta, _ = f.quantize(p[name].float(), gamma=gamma)
        f.close()
        if int(Z.abs().max()) > 127:
            raise ValueError(f"the codes of {name} do not fit 8 bits: take a larger gamma")
        out[name] = (Z.to(torch.int8), alpha, beta, V)
    return out


def serve(x, p, q):
    """The block from 8-bit rows and codes."""
    Z1, alpha1, beta1, _ = q["W1"]
    Z2, alpha2, beta2, _ = q["W2"]
    h, hs, s = ffe.rms_norm_q8(x, p["norm"], col_scale=alpha1)
    u = ffe.linear_q8(h, hs, Z1, beta1, bias=p["b1"], activation=ACT)
    u8, us = ffe.quantize_rows(u, col_scale=alpha2)
    return ffe.linear_q8(u8, us, Z2, beta2, residual=s)


def run(hidden=256, inner=512, tokens=4096, steps=30, gamma=0.01, seed=0, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    teacher, p = new_block(hidden, inner, gen, device), new_block(hidden, inner, gen, device, scale=0.5)
    losses = train(p, teacher, tokens, steps, gen)
    x = torch.randn((tokens, hidden), generator=gen, device=device).to(torch.bfloat16)
    want, _ = forward(x, teacher)
    y, kept = forward(x, p)
    diff = y.float() - want.float()
    # calibration: the loss's gradient at labels the block itself is unsure of
    noise = torch.randn(diff.shape, generator=gen, device=device)
    _, layers = backward((diff + noise).to(torch.bfloat16), p, kept)
    q = quantise(p, layers, gamma)
    served = serve(x, p, q)
    coded = dict(p, W1=q["W1"][3].to(torch.bfloat16), W2=q["W2"][3].to(torch.bfloat16))
    y_coded, _ = forward(x, coded)

    def off(a, b):   # of what the block adds to x
        return float((a.float() - b.float()).norm() / (b.float() - x[:len(b)].float()).norm())
    bits = {k: float(torch.log2((2 * v[0].float().abs().amax() + 1))) for k, v in q.items()}
    return {"losses": losses, "codes against weights": off(y_coded, y), "8-bit rows against bf16 rows": off(served, y_coded),
            "one token against the batch": off(serve(x[:1], p, q), served[:1]), "bits": bits}


if __name__ == "__main__":
    r = run(*(int(v) for v in sys.argv[1:5]))
    print(f"loss {r['losses'][0]:.4f} -> {r['losses'][-1]:.4f} in {len(r['losses'])} steps")
    for k in ("codes against weights", "8-bit rows against bf16 rows"):
        print(f"{k}: {100 * r[k]:.2f}%")
    print("bits of the widest code:", ", ".join(f"{k} {v:.1f}" for k, v in r["bits"].items()))
