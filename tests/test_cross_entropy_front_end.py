"""CPU-only checks of what the cross entropy's front end asks the library for, with plain stand-ins in the place of its entry points."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M
from test_tokens_front_end import calls          # noqa: F401 (a fixture)
from test_training_front_end import normal

TARGET = torch.tensor([0, 5, -100, 8, 2])


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("which", [None, 0, 1, 2])
def test_nothing_is_kept_for_a_gradient_that_nobody_can_ask_for(calls, which, reduction):    # noqa: F811
    """Gradients are on, as they are by default, but no operand wants one: an evaluation that does not say no_grad."""
    ops = [normal(5, 7), normal(9, 7, seed=1), normal(9, seed=2)]
    if which is not None:
        ops[which].requires_grad_()
    loss = M.linear_cross_entropy(ops[0], ops[1], TARGET, ops[2], reduction=reduction, keep=True)
    assert loss.requires_grad == (which is not None) and calls[0][1] is (which is not None)


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_the_gradient_gets_the_rows_losses(calls, monkeypatch, reduction, keep):    # noqa: F811
    """Those of the forward pass, whatever becomes of the result in the meantime; from what was kept it has them already."""
    given, stand_in = [], M.binding.mdet_xent_backward

    def gradient(*args, loss=None, **kw):
        given.append(loss)
        return stand_in(*args, **kw)
    monkeypatch.setattr(M.binding, "mdet_xent_backward", gradient)
    x, w = normal(5, 7).requires_grad_(), normal(9, 7, seed=1).requires_grad_()
    rows = M.binding.mdet_xent_forward(x.detach(), w.detach(), TARGET)[0]
    loss = M.linear_cross_entropy(x, w, TARGET, reduction=reduction, keep=keep)
    plain = torch.nn.functional.cross_entropy(x @ w.t(), TARGET, reduction=reduction)
    loss *= 2.0
    for a, b in zip(torch.autograd.grad(loss.sum(), (x, w)), torch.autograd.grad(2.0 * plain.sum(), (x, w))):
        assert torch.allclose(a, b, rtol=1e-9, atol=1e-9)
    assert len(given) == 1 and (given[0] is None if keep else torch.equal(given[0], rows))
