"""CPU-only checks of the optimiser object: what it counts, keeps, takes over and hands to the library's step, for which a stand-in
takes its place."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M


@pytest.fixture
def steps(monkeypatch):
    """The number and seed of each step that was taken."""
    taken = []

    def step(params, grads, exp_avg, exp_avg_sq, *, step, seed, **_):
        if any(g.shape != p.shape for p, g in zip(params, grads)):
            raise ValueError("refused")
        taken.append((step, seed))
    monkeypatch.setattr(M.binding, "mdet_adamw_step", step)
    return taken


def tensors(*shapes):
    return [torch.randn(*s, generator=torch.Generator().manual_seed(i)) for i, s in enumerate(shapes)]


def test_a_step_that_is_refused_does_not_count(steps):
    p = tensors((4, 3), (5,))
    opt = M.AdamW(p, seed=100)
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step([p[0], p[0]])
        with pytest.raises(ValueError):
            opt.step()                          # no gradients
    assert opt.steps == 0
    opt.step([t.clone() for t in p])
    with pytest.raises(ValueError):
        opt.step([p[1], p[1]])
    opt.step([t.clone() for t in p])
    assert steps == [(1, 101), (2, 102)] and opt.steps == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_a_state_of_other_shapes_is_refused_whole(steps, bits):
    opt = M.AdamW(tensors((4, 3), (300,)), state_bits=bits, seed=5)
    opt.step(tensors((4, 3), (300,)))
    for t in opt.exp_avg + opt.exp_avg_sq + (opt.scales or []):
        t.fill_(7)
    same = M.AdamW(tensors((4, 3), (300,)), state_bits=bits)
    same.load_state_dict(opt.state_dict())
    assert same.steps == 1 and same.seed == 5
    assert all(bool((t == 7).all()) for t in same.exp_avg + same.exp_avg_sq + (same.scales or []))
    for shapes in (((4, 3), (1,)), ((4, 3), (300, 1)), ((3, 4), (300,)), ((4, 3),), ((4, 3), (300,), (2,)), ()):
        other = M.AdamW(tensors(*shapes), state_bits=bits)
        source = M.AdamW(tensors((4, 3), (300,)), state_bits=bits)
        for into, state in ((other, opt.state_dict()), (source, other.state_dict())):
            with pytest.raises(ValueError):
                into.load_state_dict(state)
            assert into.steps == 0 and not any(bool(t.any()) for t in into.exp_avg + into.exp_avg_sq + (into.scales or []))
    with pytest.raises(ValueError):
        M.AdamW(tensors((4, 3), (300,)), state_bits=40 - bits).load_state_dict(opt.state_dict())
    state = {**opt.state_dict(), "exp_avg_sq": opt.exp_avg_sq[:1]}
    with pytest.raises(ValueError):
        same.load_state_dict(state)


def test_a_tensor_twice_is_refused():
    """Its update would run in several workgroups at once."""
    a, b = tensors((40, 30), (5,))
    flat = torch.zeros(100)
    for bad in ([a, b, a], [a, b, a.view(30, 40)], [flat[:60], flat[59:]], [flat, flat[99:]], [a, a.detach()]):
        with pytest.raises(ValueError, match="twice"):
            M.AdamW(bad)
    M.AdamW([a, b, flat[:60], flat[60:], torch.zeros(0), torch.zeros(0), flat[:0]])


def test_copies_follow_parameters_that_were_brought_back_with_a_state(steps):
    p = tensors((4, 3), (5,))
    opt = M.AdamW(p, copy_dtype=torch.bfloat16)
    for c in opt.copies:
        c.requires_grad_()
    saved = M.AdamW(p).state_dict()
    for t in p:
        t.mul_(2).add_(1)                       # a checkpoint's values
    opt.load_state_dict(saved)
    for t, c in zip(p, opt.copies):
        assert torch.equal(c.detach(), t.to(torch.bfloat16)) and c.requires_grad
