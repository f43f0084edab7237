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
