"""The autograd front end of the linear layer on operands and gradients that are one row, or one element, repeated, and on empty
axes, against the same in 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, act64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def normal(*shape, seed=0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


LOSSES = {"sum": lambda y: y.sum(), "sum over rows": lambda y: y.sum(0).sum(), "mean over rows": lambda y: (y.mean(0) * 2).sum(),
          "one column": lambda y: y[..., -1].sum()}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("shape", [(5, 40), (70, 40), (3, 17, 40)], ids=str)
@pytest.mark.parametrize("n", [1, 8, 33])
def test_gradients_that_autograd_hands_over_repeated(M, loss, shape, n):
    for act in ("none", "gelu"):
        ops = [normal(*s, seed=i).requires_grad_() for i, s in enumerate((shape, (n, 40), (n,)))]
        got = torch.autograd.grad(LOSSES[loss](M.linear(*ops, activation=act)), ops)
        wide = [v.detach().double().requires_grad_() for v in ops]
        want = torch.autograd.grad(LOSSES[loss](act64(act, wide[0] @ wide[1].t() + wide[2])[0]), wide)
        for a, v in zip(got, want):
            # sums of at most 70 terms: dy (up to 2) times a slope (up to 1.13) times an operand (up to 5)
            assert a.shape == v.shape and float((a.double() - v).abs().max()) <= 70 * EPS32 * 70 * 2 * 1.13 * 5


def test_operands_that_are_repeated(M):
    x, w, r, b = normal(1, 40).expand(9, 40), normal(24, 40, seed=1), normal(1, 24, seed=2).expand(9, 24), normal(1, seed=3).expand(24)
    y = M.linear(x, w, b, r)
    want = x.double() @ w.double().t() + b.double() + r.double()
    # 42 terms, each at most 25
    assert float((y.double() - want).abs().max()) <= 42 * EPS32 * 42 * 25
    same = M.linear(x.contiguous(), w, b.contiguous(), r.contiguous())
    assert torch.equal(y, same)
    assert torch.equal(M.linear(x, w[:1].expand(24, 40)), M.linear(x, w[:1].repeat(24, 1)))


def test_axes_that_are_empty(M):
    for shape, n in (((4, 0), 6), ((0, 7), 6), ((2, 0, 7), 6), ((2, 3, 0), 6), ((4, 7), 0)):
        x, w, b = normal(*shape).requires_grad_(), normal(n, shape[-1]).requires_grad_(), normal(n).requires_grad_()
        y = M.linear(x, w, b, None, "relu")
        assert y.shape == (*shape[:-1], n)
        if shape[-1] == 0:                       # an empty sum: the bias alone
            assert torch.equal(y, torch.relu(b).detach().expand_as(y))
        grads = torch.autograd.grad(y.sum(), (x, w, b))
        assert all(g.shape == t.shape for g, t in zip(grads, (x, w, b)))
        assert not grads[1].any()                # no rows, or no columns
        if shape[-1] == 0:
            assert torch.equal(grads[2], y.shape[:-1].numel() * (b > 0).float())


def test_a_gradient_through_weights_from_before_a_step_is_refused(M):
    """The step writes parameters and copies in place: autograd notices that a graph from before it has lost its values."""
    w = normal(24, 40).requires_grad_()
    opt = M.AdamW([w], copy_dtype=torch.bfloat16)
    for p in (w, opt.copies[0].requires_grad_()):
        x = normal(8, 40, seed=1).to(p.dtype).requires_grad_()
        old = M.linear(x, p, activation="gelu")
        opt.step([torch.ones_like(w)])
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            old.sum().backward()
        M.linear(x, p, activation="gelu").sum().backward()
        assert x.grad is not None and p.grad is not None


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
def test_empty_axes_beside_long_ones(M, dtype):
    """An empty batch through a wide layer and back, a layer without inputs, one without outputs."""
    for m, n, k in ((0, 640, 1024), (0, 9000, 520), (1000, 64, 0), (1000, 0, 64)):
        x, w, b = (normal(*s).to(dtype).requires_grad_() for s in ((m, k), (n, k), (n,)))
        y = M.linear(x, w, b, activation="gelu")
        dx, dw, db = torch.autograd.grad(y.sum(), (x, w, b))
        assert y.shape == (m, n) and dx.shape == x.shape and dw.shape == w.shape and not dx.any() and not dw.any()
        assert bool(db.any()) == (m * n > 0)
