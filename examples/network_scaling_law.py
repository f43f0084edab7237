"""From a network to its scaling law, on one GPU: train a residual network, form the Gram matrix of its Jacobian (its NTK),
take the log-determinant and fit the curve of Alg. 2 to those of the leading blocks.

    python examples/network_scaling_law.py [samples] [width] [outputs] [steps]

The network is f = W3 h2 + b3 with h1 = gelu(W1 x + b1) and h2 = h1 + gelu(W2 h1 + b2).  Training runs in bfloat16 on
copies of fp32 parameters, with optimiser states in 8 bits; the Jacobian is taken in fp32 at those parameters and its
Gram matrix formed in fp64 (an NTK's condition number needs it).
"""
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2503_04424_amd as M  # noqa: E402


def network(x, p):
    """The network's outputs, with gradients (three launches forward)."""
    h1 = M.linear(x, p[0], p[1], activation="gelu")
    h2 = M.linear(h1, p[2], p[3], residual=h1, activation="gelu")
    return M.linear(h2, p[4], p[5])


def train(x, y, width, steps, generator):
    """Parameters after `steps` steps of a least-squares fit, and the losses on the way."""
    sizes = [x.shape[1], width, width, y.shape[1]]
    params = []
    for a, b in zip(sizes[:-1], sizes[1:]):
        params += [torch.randn(b, a, generator=generator, device="cuda") * math.sqrt(1.0 / a), torch.zeros(b, device="cuda")]
    opt = M.AdamW(params, lr=3e-3, weight_decay=1e-4, state_bits=8, copy_dtype=torch.bfloat16)
    losses = []
    xb, yb = x.to(torch.bfloat16), y.to(torch.bfloat16)
    for _ in range(steps):
        for c in opt.copies:
            c.requires_grad_().grad = None
        loss = (network(xb, opt.copies) - yb).float().square().mean()
        loss.backward()
        opt.step([c.grad for c in opt.copies])
        losses.append(loss.detach())
    return params, torch.stack(losses)


def ntk(x, p, dtype=torch.float64):
    """Lower triangle of J J^T, rows in the order sample by sample, output by output."""
    n, d = x.shape[0], p[4].shape[0]
    z1, z2 = x.new_empty(n, p[0].shape[0]), x.new_empty(n, p[2].shape[0])
    h1 = M.mdet_linear_forward(x, p[0], p[1], activation="gelu", preact=z1)
    h2 = M.mdet_linear_forward(h1, p[2], p[3], h1, "gelu", preact=z2)
    # derivatives of output r at sample i in row i d + r, from the last layer back; W's gradients are never formed
    each = lambda t: t.repeat_interleave(d, 0)          # noqa: E731
    g3 = torch.eye(d, device="cuda", dtype=x.dtype).repeat(n, 1)
    dh2 = M.mdet_linear_backward(g3, each(h2), p[4], dw=False, db=False)[0]
    g2, g1 = torch.empty_like(dh2), torch.empty_like(dh2)
    dh1 = M.mdet_linear_backward(dh2, each(h1), p[2], each(z2), "gelu", dw=False, db=False, dz=g2)[0].add_(dh2)
    M.mdet_linear_backward(dh1, each(x), p[0], each(z1), "gelu", dx=False, dw=False, db=False, dz=g1)
    return M.mdet_ntk_gram([x, h1, h2], [g1, g2, g3], torch.zeros(n * d, n * d, dtype=dtype, device="cuda"), outputs=d)


def run(samples=1000, width=256, outputs=2, steps=100, inputs=32, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(samples, inputs, generator=g, device="cuda")
    y = torch.sin(x @ torch.randn(inputs, outputs, generator=g, device="cuda") * (2.0 / math.sqrt(inputs)))
    params, losses = train(x, y, width, steps, g)
    K = ntk(x, params)
    kept = K.clone()
    order = samples * outputs
    diag = torch.empty(order, dtype=torch.float64, device="cuda")
    r = M.mdet_logdet_device(K, overwrite=True, diag=diag)
    ell = M.mdet_principal_logdets(diag)
    # the curve from the first half of the samples, every `outputs`-th block, against the whole
    coef = M.mdet_flodance_fit(ell, outputs, max(8, samples // 20), samples // 2, 1)
    predicted = samples * float(M.mdet_flodance_eval(coef, 1, torch.tensor([float(samples)], dtype=torch.float64, device="cuda")))
    return {"losses": losses.cpu(), "params": params, "x": x, "ntk": kept, "logabsdet": r.logabsdet, "sign": r.sign, "predicted": predicted}


if __name__ == "__main__":
    names = ("samples", "width", "outputs", "steps")
    out = run(**{k: int(v) for k, v in zip(names, sys.argv[1:])})
    print(f"loss {float(out['losses'][0]):.4f} -> {float(out['losses'][-1]):.4f}; order {out['ntk'].shape[0]}: "
          f"log|det| = {out['logabsdet']:.4f} (sign {out['sign']}), extrapolated from half the samples {out['predicted']:.4f}")
