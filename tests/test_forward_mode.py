"""CPU-only checks that no front end loses a tangent of forward mode: plain stand-ins take the place of the library's entry points, which see
addresses and no tangents.  The autograd nodes have no forward mode, so a call with a tangent raises, also where gradients are switched off:
``no_grad`` is about reverse mode, torch's own functions carry tangents through it."""
import pytest

torch = pytest.importorskip("torch")
import torch.autograd.forward_ad as forward

import paper_2503_04424_amd as M
from test_tokens_front_end import calls as tokens             # noqa: F401 (a fixture)
from test_training_front_end import calls as training, normal  # noqa: F401

IDS, TARGET = torch.tensor([3, 0, 8, 3, 1]), torch.tensor([0, 5, -100, 8, 2])
# name: (shapes of the operands, the call)
CALLS = {"linear": (((5, 7), (6, 7), (6,), (5, 6)), lambda x, w, b, r: M.linear(x, w, b, r, "silu")),
         "embedding": (((9, 7),), lambda table: M.embedding(IDS, table, 2.0)),
         "layer_norm": (((5, 7), (7,), (7,)), M.layer_norm),
         "linear_cross_entropy": (((5, 7), (9, 7), (9,)), lambda x, w, b: M.linear_cross_entropy(x, w, TARGET, b))}
CASES = [(name, i) for name, (shapes, _) in CALLS.items() for i in range(len(shapes))]


@pytest.fixture(autouse=True)
def stand_ins(tokens, training):                              # noqa: F811
    pass


def operands(name):
    return [normal(*s, seed=i) for i, s in enumerate(CALLS[name][0])]


@pytest.mark.parametrize("name,which", CASES)
@pytest.mark.parametrize("gradients", [False, True])
def test_a_tangent_is_not_lost(name, which, gradients):
    ops = operands(name)
    with torch.set_grad_enabled(gradients), forward.dual_level():
        ops[which] = forward.make_dual(ops[which], torch.ones_like(ops[which]))
        with pytest.raises(NotImplementedError, match="jvp"):
            CALLS[name][1](*ops)


@pytest.mark.parametrize("name", CALLS)
def test_without_tangents_the_call_is_as_outside_of_forward_mode(name):
    ops = operands(name)
    with torch.no_grad():
        want = CALLS[name][1](*ops)
        with forward.dual_level():
            assert torch.equal(CALLS[name][1](*ops), want)
            only = [forward.make_dual(v, torch.ones_like(v)) for v in ops]
        assert torch.equal(CALLS[name][1](*only), want)       # the level is over, and their tangents with it
