"""The example that trains a network, forms its NTK and fits its scaling law, at a small size."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

from conftest import ROOT

pytestmark = pytest.mark.gpu


def load():
    spec = importlib.util.spec_from_file_location("network_scaling_law", os.path.join(ROOT, "examples", "network_scaling_law.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def jacobian(x, params):
    """J in 64 bits by autograd, one row for each sample and output."""
    p = [v.double().requires_grad_() for v in params]
    gelu = torch.nn.functional.gelu
    rows = []
    for i in range(x.shape[0]):
        h1 = gelu(x[i].double() @ p[0].t() + p[1])
        f = (h1 + gelu(h1 @ p[2].t() + p[3])) @ p[4].t() + p[5]
        for r in range(f.shape[0]):
            rows.append(torch.cat([v.reshape(-1) for v in torch.autograd.grad(f[r], p, retain_graph=True)]))
    return torch.stack(rows)


def test_example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    E = load()
    out = E.run(samples=96, width=64, outputs=2, steps=60, inputs=16)
    assert float(out["losses"][-1]) < 0.5 * float(out["losses"][0])
    J = jacobian(out["x"], out["params"])
    want = J @ J.t()
    # the Jacobian is taken in fp32: a few hundred terms a derivative
    assert float((out["ntk"] - torch.tril(want)).abs().max()) <= 1e-4 * float(want.abs().max())
    whole = out["ntk"] + torch.tril(out["ntk"], -1).t()
    sign, logabsdet = torch.linalg.slogdet(whole)
    assert out["sign"] == int(sign) and abs(out["logabsdet"] - float(logabsdet)) <= 1e-8 * max(1.0, abs(float(logabsdet)))
    assert out["predicted"] == out["predicted"]
