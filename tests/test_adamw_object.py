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
