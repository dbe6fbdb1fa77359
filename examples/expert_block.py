"""One feed-forward block of experts, its training step and its calibration, on one MI355X.

    h = norm(x),  l = h Wr^T,  y = x + sum over the chosen experts of w_e W2_e act(W1_e h)

1. Training: the block learns another block's outputs.  Between forward and
   backward a step keeps the experts' activations in 8 bits (route,
   expert_linear, expert_combine, checkpoint_q8 and their gradients).
2. Balance: experts that many tokens took lose some bias, the others gain some;
   it changes who is chosen, not with what weight.
3. Calibration: the rows of x and g of an expert are its layers' tokens, from
   which FlipFlop makes their Kronecker curvature A (x) B.

    python examples/expert_block.py [hidden] [inner] [experts] [top] [tokens] [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2609_14706_amd as ffe  # noqa: E402

ACT = "silu"


def forward(x, p, top, bias=None, mask=None):
    """The block's output and what its gradient needs, the experts' activations in 8 bits."""
    h, _ = ffe.rms_norm(x, p["norm"])
    logits, _ = ffe.linear(h, p["Wr"])
    r = ffe.route(logits, top, bias=bias, mask=mask)
    u, z = ffe.expert_linear(h, p["W1"], r, bias=p["b1"], activation=ACT, keep_preact=True)
    v, _ = ffe.expert_linear(u, p["W2"], r, by_slot=True)
    y = ffe.expert_combine(v, r, residual=x)
    return y, (x, h, logits, r, ffe.checkpoint_q8(h), ffe.checkpoint_q8(z), ffe.checkpoint_q8(u), v)


def backward(dy, p, kept):
    """(gradients by name with that of x, rows (x, g) of each of the experts' layers)."""
    x, h, logits, r, h8, z8, u8, v = kept
    dv, dw = ffe.expert_combine_backward(dy, v, r)
    du, dW2, g2, _ = ffe.expert_linear_backward(dv, u8, p["W2"], r, by_slot=True, need_bias=False)
    dh, dW1, g1, db1 = ffe.expert_linear_backward(du, h8, p["W1"], r, preact=z8, activation=ACT)
    dl = ffe.route_backward(dw, logits, r.experts)
    dh2, dWr, _, _ = ffe.linear_backward(dl, h, p["Wr"], need_bias=False)
    dx, dnorm = ffe.rms_norm_backward(dh.add_(dh2), x, p["norm"], dsum=dy)
    return {"W1": dW1, "b1": db1, "W2": dW2, "Wr": dWr, "norm": dnorm, "x": dx}, {"W1": (h8, g1), "W2": (u8, g2)}


def new_block(hidden, inner, experts, gen, device, scale=1.0):
    def r(*shape):
        return torch.randn(shape, generator=gen, device=device)
    p = {"norm": torch.ones(hidden, device=device), "Wr": r(experts, hidden) / hidden ** 0.5,
         "W1": scale * r(experts, inner, hidden) / hidden ** 0.5, "b1": torch.zeros((experts, inner), device=device),
         "W2": scale * r(experts, hidden, inner) / inner ** 0.5}
    return {k: v.to(torch.bfloat16) for k, v in p.items()}


def train(p, teacher, top, tokens, steps, gen, rate=0.02):
    """(loss of each step, the bias that balances the experts); p is updated in place from fp32 copies."""
    device, experts = p["norm"].device, p["W1"].shape[0]
    master = {k: v.float() for k, v in p.items()}
    bias, losses = torch.zeros(experts, device=device), []
    for k in range(steps):
        x = torch.randn((tokens, p["norm"].numel()), generator=gen, device=device).to(torch.bfloat16)
        want, _ = forward(x, teacher, top)
        y, kept = forward(x, p, top, bias=bias)
        diff = y.float() - want.float()
        losses.append(float(diff.square().mean()))
        grads, _ = backward((diff / diff.numel() ** 0.5).to(torch.bfloat16), p, kept)
        for name in master:
            g = grads[name].float()
            master[name].sub_(rate * (1 - k / steps) * master[name].abs().mean() * g / (g.square().mean().sqrt() + 1e-12))
            p[name].copy_(master[name])
        counts = kept[3].offsets.diff().float()
        bias += 0.01 * torch.sign(counts.mean() - counts)
    return losses, bias


def curvature(rows, r, by_slot, expert, iters=3):
    """(A, B) of one expert's layer from its rows (x in 8 bits, g): its input rows and token gradients."""
    x8, g = rows
    a, b = r.offsets[expert:expert + 2].tolist()
    x = ffe.checkpoint_restore(x8)
    x = x[a:b] if by_slot else x[r.order[a:b].long() // r.experts.shape[1]]
    f = ffe.FlipFlop(tokens=(x.contiguous(), g[a:b].contiguous()), damping=0.1)
    f.iterate(iters)
    A, B = f.factors()
    f.close()
    return A, B


def run(hidden=256, inner=384, experts=8, top=2, tokens=4096, steps=20, seed=0, device="cuda:0"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    teacher = new_block(hidden, inner, experts, gen, device)
    p = new_block(hidden, inner, experts, gen, device, scale=0.5)
    losses, bias = train(p, teacher, top, tokens, steps, gen)
    x = torch.randn((tokens, hidden), generator=gen, device=device).to(torch.bfloat16)
    y, kept = forward(x, p, top, bias=bias)
    want, _ = forward(x, teacher, top)
    _, layers = backward((y.float() - want.float() + torch.randn(y.shape, generator=gen, device=device)).to(torch.bfloat16), p, kept)
    r = kept[3]
    full = int(r.offsets.diff().argmax())
    factors = {name: curvature(rows, r, name == "W2", full) for name, rows in layers.items()}
    return {"losses": losses, "rows": r.offsets.diff().tolist(), "expert": full, "factors": factors}


if __name__ == "__main__":
    out = run(*(int(v) for v in sys.argv[1:7]))
    print(f"loss {out['losses'][0]:.4f} -> {out['losses'][-1]:.4f} in {len(out['losses'])} steps")
    print(f"rows of the experts: {out['rows']}")
    for name, (A, B) in out["factors"].items():
        print(f"{name} of expert {out['expert']}: A {tuple(A.shape)}, B {tuple(B.shape)}, tr(B) {float(B.trace()):.4e}")
