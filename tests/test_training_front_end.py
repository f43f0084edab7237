"""CPU-only checks of the front ends of the training operators: what they hand to the library's entry points, for which plain
stand-ins take their place here that insist on the library's terms (rows of consecutive elements, further apart than they are long)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M


def is_matrix(t):
    return t.dim() == 2 and (t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1])


def value(z, act):
    return z.tanh() if act == "silu" else z         # any function will do: both stand-ins use it


@pytest.fixture
def calls(monkeypatch):
    """The stand-ins, and what they were called with."""
    seen = {"forward": [], "backward": []}

    def forward(x, w, bias=None, residual=None, activation="none", out=None, preact=None, workspace=None, stream=None):
        assert all(t is None or is_matrix(t) for t in (x, w, residual, preact))
        assert bias is None or bias.is_contiguous()
        seen["forward"].append({"preact": preact})
        z = x @ w.t() + (0 if bias is None else bias)
        if preact is not None:
            preact.copy_(z)
        return value(z, activation) + (0 if residual is None else residual)

    def backward(dy, x, w, preact=None, activation="none", dx=True, dw=True, db=True, **_):
        assert all(t is None or is_matrix(t) for t in (dy, x, w, preact))
        seen["backward"].append({})
        dz = dy * (1 - preact.tanh() ** 2) if activation == "silu" else dy
        return dz @ w if dx else None, dz.t() @ x if dw else None, dz.sum(0) if db else None
    monkeypatch.setattr(M.binding, "mdet_linear_forward", forward)
    monkeypatch.setattr(M.binding, "mdet_linear_backward", backward)
    return seen


def normal(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


LOSSES = {"sum": lambda y: y.sum(), "sum over rows": lambda y: y.sum(0).square().sum(), "mean over rows": lambda y: (y.mean(0) * 2).sum(),
          "one column": lambda y: y[..., -1].sum(), "transposed": lambda y: (y.transpose(0, 1).contiguous() ** 2).sum()}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("shape", [(5, 7), (3, 4, 7)])
@pytest.mark.parametrize("n", [1, 6])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_gradients_that_autograd_hands_over_repeated(calls, loss, shape, n, act):
    x, w, b = (normal(*s, seed=i).requires_grad_() for i, s in enumerate((shape, (n, 7), (n,))))
    got = torch.autograd.grad(LOSSES[loss](M.linear(x, w, b, activation=act)), (x, w, b))
    want = torch.autograd.grad(LOSSES[loss](value(x @ w.t() + b, act)), (x, w, b))
    assert len(calls["backward"]) == 1
    for a, v in zip(got, want):
        assert a.shape == v.shape and torch.allclose(a, v, rtol=1e-12, atol=1e-12)


def test_operands_that_are_repeated(calls):
    """One row for all samples, one residual and one bias for all: views of distance zero."""
    one, w, r, b = normal(1, 7), normal(6, 7, seed=1), normal(1, 6, seed=2), normal(1, seed=3)
    x, residual, bias = one.expand(4, 7), r.expand(4, 6), b.expand(6)
    assert torch.allclose(M.linear(x, w, bias, residual), x @ w.t() + bias + residual)
    assert torch.allclose(M.linear(normal(4, 7), w[:1].expand(6, 7)), normal(4, 7) @ w[:1].expand(6, 7).t())
    wide = normal(2, 3, 7).expand(2, 3, 7)[:, :1].expand(2, 3, 7)
    leaf = r.clone().requires_grad_()
    y = M.linear(wide, w, None, leaf.expand(2, 3, 6))
    assert torch.allclose(y, wide @ w.t() + leaf)
    assert torch.allclose(torch.autograd.grad(y.sum(), leaf)[0], torch.full((1, 6), 6.0, dtype=torch.float64))


def test_axes_that_are_empty(calls):
    for shape, n in (((4, 0), 6), ((0, 7), 6), ((2, 0, 7), 6), ((2, 3, 0), 6), ((4, 7), 0), ((0, 0), 0)):
        x, w, b = normal(*shape).requires_grad_(), normal(n, shape[-1]).requires_grad_(), normal(n).requires_grad_()
        y = M.linear(x, w, b, normal(*shape[:-1], n), "silu")
        assert y.shape == (*shape[:-1], n)
        for got, of in zip(torch.autograd.grad(y.sum(), (x, w, b)), (x, w, b)):
            assert got.shape == of.shape


def test_shapes_are_refused(calls):
    for x, w in ((normal(4, 7), normal(7)), (torch.tensor(1.0), normal(6, 7))):
        with pytest.raises(ValueError):
            M.linear(x, w)
    with pytest.raises(ValueError):
        M.linear(normal(4, 7), normal(6, 7), residual=normal(6))


def test_nothing_is_kept_where_no_gradient_can_be_asked_for(calls):
    x, w, b = normal(4, 7), normal(6, 7, seed=1).requires_grad_(), normal(6, seed=2).requires_grad_()
    y = M.linear(x, w, b, activation="silu")
    assert calls["forward"][-1]["preact"] is not None and y.requires_grad
    for off in (torch.no_grad, torch.inference_mode):
        with off():
            z = M.linear(x, w, b, activation="silu")
        assert calls["forward"][-1]["preact"] is None and not z.requires_grad and torch.equal(y.detach(), z)
    M.linear(x, w.detach(), b.detach(), normal(4, 6).requires_grad_(), activation="silu")       # the residual's gradient is dy
    assert calls["forward"][-1]["preact"] is None
