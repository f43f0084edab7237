"""CPU-only checks of the token operators' front ends: what they hand to the library's entry points, for which plain stand-ins take their
place here that insist on the library's terms (rows of consecutive elements, vectors in one piece)."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M
from test_training_front_end import is_matrix, normal


@pytest.fixture
def calls(monkeypatch):
    """The stand-ins, and what they were called with."""
    seen = []

    def fits(*matrices, vectors=()):
        assert all(t is None or is_matrix(t) for t in matrices) and all(t is None or (t.dim() == 1 and t.is_contiguous()) for t in vectors)

    def embed(ids, table, scale=1.0, out=None, stream=None):
        fits(table, vectors=(ids,))
        inside = (ids >= 0) & (ids < table.shape[0])
        return table[torch.where(inside, ids, 0).long()] * scale * inside[:, None]

    def embed_grad(dy, ids, vocab, scale=1.0, **_):
        fits(dy, vectors=(ids,))
        inside = (ids >= 0) & (ids < vocab)
        return torch.zeros(vocab, dy.shape[1], dtype=dy.dtype).index_add(0, ids[inside].long(), dy[inside] * scale)

    def norm(x, weight=None, bias=None, eps=1e-5, out=None, mean=True, rstd=True, stream=None):
        fits(x, vectors=(weight, bias))
        seen.append(mean is not False)
        m, r = x.mean(1), (x.var(1, unbiased=False) + eps).rsqrt()
        y = (x - m[:, None]) * r[:, None] * (1 if weight is None else weight) + (0 if bias is None else bias)
        return y, m if mean else None, r if rstd else None

    def norm_grad(dy, x, mean, rstd, weight=None, dx=True, dw=True, db=True, **_):
        fits(dy, x, vectors=(mean, rstd, weight))
        h, u = (x - mean[:, None]) * rstd[:, None], dy * (1 if weight is None else weight)
        d = rstd[:, None] * (u - u.mean(1, keepdim=True) - h * (u * h).mean(1, keepdim=True))
        return d if dx else None, (dy * h).sum(0) if dw else None, dy.sum(0) if db else None

    def counted(target, n, ignore):
        return (target >= 0) & (target < n) & (target != ignore)

    def xent(x, w, target, bias=None, ignore=-100, loss=True, lse=True, keep=False, **_):
        fits(x, w, vectors=(target, bias))
        seen.append((lse, keep))
        z = x @ w.t() + (0 if bias is None else bias)
        c = counted(target, w.shape[0], ignore)
        l = torch.logsumexp(z, 1)
        return torch.where(c, l - z.gather(1, torch.where(c, target, 0).long()[:, None])[:, 0], 0.0), l if lse else None, z if keep else None

    def xent_grad(dloss, x, w, target, lse, bias=None, ignore=-100, kept=None, dx=True, dw=True, db=None, **_):
        fits(x, w, vectors=(dloss, target, lse, bias))
        seen.append(kept is not None)
        c = counted(target, w.shape[0], ignore)
        e = torch.exp(x @ w.t() + (0 if bias is None else bias) - lse[:, None])
        e[torch.nonzero(c)[:, 0], target[c].long()] -= 1
        e = e * torch.where(c, dloss, 0.0)[:, None]
        return e @ w if dx else None, e.t() @ x if dw else None, e.sum(0) if db else None

    def reduce(loss, target, vocab, ignore=-100, mean=True, out=True, weights=True, stream=None):
        fits(vectors=(loss, target))
        c = counted(target, vocab, ignore)
        weight = 1 / c.sum().double() if mean else torch.ones(())
        total = loss[c].sum()
        return total / c.sum() if mean else total, c * weight.to(loss.dtype) if weights else None
    for name, f in dict(mdet_embedding_forward=embed, mdet_embedding_backward=embed_grad, mdet_layernorm_forward=norm, mdet_layernorm_backward=norm_grad,
                        mdet_xent_forward=xent, mdet_xent_reduce=reduce, mdet_xent_backward=xent_grad).items():
        monkeypatch.setattr(M.binding, name, f)
    return seen


LOSSES = {"sum": lambda y: y.sum(), "mean over rows": lambda y: (y.mean(0) * 2).sum(), "one column": lambda y: y[..., -1].sum(),
          "transposed": lambda y: (y.transpose(0, 1).contiguous() ** 2).sum()}


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("width", [1, 6])
def test_embedding(calls, loss, width):
    table = normal(9, width).requires_grad_()
    ids = torch.tensor([[3, 3, -1, 8], [0, 9, 3, 100], [7, 0, 1, 2]])
    inside = (ids >= 0) & (ids < 9)
    for i in (ids, ids.int(), ids.t().contiguous().t()):
        got = torch.autograd.grad(LOSSES[loss](M.embedding(i, table, 2.5)), table)[0]
        want = torch.autograd.grad(LOSSES[loss](table[torch.where(inside, ids, 0)] * 2.5 * inside[..., None]), table)[0]
        assert torch.allclose(got, want, rtol=1e-12, atol=1e-12)
    assert M.embedding(ids[0, 0], table).shape == (width,) and M.embedding(ids[:0], table).shape == (0, 4, width)
    with torch.no_grad():
        assert torch.equal(M.embedding(ids, table, 2.5), M.embedding(ids, table, 2.5).detach())
        assert torch.equal(M.embedding(ids, table[:1].expand(9, width)), table[:1].expand(9, width)[torch.where(inside, ids, 0)] * inside[..., None])
    with pytest.raises(ValueError):
        M.embedding(ids, table[0])


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("shape", [(5, 7), (3, 4, 7)])
@pytest.mark.parametrize("affine", [(True, True), (True, False), (False, True), (False, False)])
def test_layer_norm(calls, loss, shape, affine):
    x = normal(*shape).requires_grad_()
    w, b = (normal(7, seed=i + 1).requires_grad_() if on else None for i, on in enumerate(affine))
    leaves = [v for v in (x, w, b) if v is not None]
    got = torch.autograd.grad(LOSSES[loss](M.layer_norm(x, w, b)), leaves)
    want = torch.autograd.grad(LOSSES[loss](torch.nn.functional.layer_norm(x, (7,), w, b)), leaves)
    for a, v in zip(got, want):
        assert a.shape == v.shape and torch.allclose(a, v, rtol=1e-9, atol=1e-9)
    calls.clear()
    with torch.no_grad():
        y = M.layer_norm(x, w, b)
    assert calls == [False] and not y.requires_grad                     # nothing is kept where no gradient can be asked for
    z = M.layer_norm(x.transpose(0, -2), w, normal(1).expand(7))        # operands that are views, or one element repeated
    assert torch.allclose(z, torch.nn.functional.layer_norm(x.transpose(0, -2), (7,), w, normal(1).expand(7)))
    assert M.layer_norm(x[:0], w, b).shape == (0, *shape[1:])
    with pytest.raises(ValueError):
        M.layer_norm(torch.tensor(1.0))


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("biased", [False, True])
def test_linear_cross_entropy(calls, reduction, keep, biased):
    x, w = normal(3, 4, 7).requires_grad_(), normal(9, 7, seed=1).requires_grad_()
    b = normal(9, seed=2).requires_grad_() if biased else None
    t = torch.tensor([[0, 8, -100, 3], [5, 5, 2, 9], [-1, 1, 0, 5]])
    leaves = [v for v in (x, w, b) if v is not None]
    for ignore in (-100, 5):
        counts = (t >= 0) & (t < 9) & (t != ignore)
        plain = torch.nn.functional.cross_entropy((x @ w.t() + (0 if b is None else b)).flatten(0, 1), torch.where(counts, t, -100).flatten(), reduction=reduction)
        got = M.linear_cross_entropy(x, w, t, b, ignore, reduction, keep)
        assert torch.allclose(got.flatten(), plain.flatten()) and got.shape == (t.shape if reduction == "none" else ())
        scale = normal(*got.shape, seed=3) if reduction == "none" else 3.0
        for a, v in zip(torch.autograd.grad((got * scale).sum(), leaves), torch.autograd.grad((plain.view(got.shape) * scale).sum(), leaves)):
            assert a.shape == v.shape and torch.allclose(a, v, rtol=1e-9, atol=1e-9)
        assert calls[-1] is keep
    only, = torch.autograd.grad(M.linear_cross_entropy(x.detach(), w, t, None if b is None else b.detach()).sum(), w)
    assert only.shape == w.shape
    y = M.linear_cross_entropy(x.transpose(0, 1), w[:1].expand(9, 7), t.t(), b, reduction="sum")
    z = (x.transpose(0, 1) @ w[:1].expand(9, 7).t() + (0 if b is None else b)).flatten(0, 1)
    assert torch.allclose(y, torch.nn.functional.cross_entropy(z, torch.where((t >= 0) & (t < 9), t, -100).t().flatten(), reduction="sum"))
    calls.clear()
    with torch.no_grad():
        M.linear_cross_entropy(x, w, t, b, keep=True)
    assert calls == [(False, False)]
    none = torch.full_like(t, -100)
    assert torch.isnan(M.linear_cross_entropy(x, w, none, b)) and not M.linear_cross_entropy(x, w, none, b, reduction="sum").any()


def test_cross_entropy_refuses(calls):
    x, w, t = normal(3, 4, 7), normal(9, 7), torch.zeros(3, 4, dtype=torch.int64)
    for bad in (dict(w=w[0]), dict(target=t[:, :3]), dict(target=t.flatten()), dict(reduction="max"), dict(x=torch.tensor(1.0))):
        with pytest.raises(ValueError):
            M.linear_cross_entropy(**{"x": x, "w": w, "target": t, **bad})
