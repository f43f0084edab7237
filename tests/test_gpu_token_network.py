"""The token operators together with the linear layer and the optimiser, as a network over tokens uses them: gradients against torch's own
in 64 bits, a step captured in a graph, batches that are padded."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
VOCAB, WIDTH, HIDDEN = 301, 48, 104


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def parameters(dtype=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(5)
    shapes = [(VOCAB, WIDTH), (WIDTH,), (WIDTH,), (HIDDEN, WIDTH), (HIDDEN,), (WIDTH, HIDDEN), (WIDTH,), (WIDTH,), (WIDTH,)]
    p = [torch.randn(s, generator=g, device="cuda") / math.sqrt(s[-1]) for s in shapes]
    for i in (1, 7):
        p[i] = 1 + 0.2 * p[i]
    return [v.to(dtype) for v in p]


def batch(seed, rows=6, length=11):
    """Tokens and, for each, the next one; the ends of the rows are padding."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    text = torch.randint(0, VOCAB, (rows, length + 1), generator=g, device="cuda")
    ids, target = text[:, :-1].clone(), text[:, 1:].clone()
    for r in range(rows):
        ids[r, length - r:] = -1
        target[r, max(0, length - 1 - r):] = -100
    return ids, target


def loss_of(M, p, ids, target, **kw):
    """Embedding, one block behind a norm with its sum, a norm, and the loss with the embedding's table as the last matrix."""
    h = M.embedding(ids, p[0], scale=math.sqrt(WIDTH))
    n = M.layer_norm(h, p[1], p[2])
    h = M.linear(M.linear(n, p[3], p[4], activation="gelu"), p[5], p[6], residual=h)
    return M.linear_cross_entropy(M.layer_norm(h, p[7], p[8]), p[0], target, **kw)


def loss64(p, ids, target):
    F = torch.nn.functional
    inside = (ids >= 0)[..., None]
    h = p[0][ids.clamp(min=0)] * math.sqrt(WIDTH) * inside
    n = F.layer_norm(h, (WIDTH,), p[1], p[2])
    h = F.gelu(n @ p[3].t() + p[4]) @ p[5].t() + p[6] + h
    z = F.layer_norm(h, (WIDTH,), p[7], p[8]) @ p[0].t()
    return F.cross_entropy(z.flatten(0, 1), target.flatten(), ignore_index=-100)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("keep", [False, True])
def test_gradients(M, dtype, keep):
    """Against autograd in 64 bits at the same parameters.  Every value on the way is rounded to `dtype` (fp32: its sums), ten of them one
    behind the other and as many on the way back, each by half a step at most: 20 half steps of a gradient's size, twice that for
    what the derivatives of the norms and the softmax make of them."""
    p = [v.requires_grad_() for v in parameters(dtype)]
    ids, target = batch(1)
    scale = 256.0 if dtype == torch.float16 else 1.0
    loss = loss_of(M, p, ids, target, keep=keep)
    got = torch.autograd.grad(loss * scale, p)
    q = [v.detach().double().requires_grad_() for v in p]
    want64 = loss64(q, ids, target)
    want = torch.autograd.grad(want64 * scale, q)
    want64 = want64.detach()
    unit = {torch.float32: 2.0 ** -18, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}[dtype]
    assert abs(float(loss.detach()) - float(want64)) <= 40 * unit * abs(float(want64))
    for a, b in zip(got, want):
        assert float((a.double() - b).norm()) <= 40 * unit * float(b.norm())


def test_tied_table_in_place(M):
    """The table's gradient by both of its uses, the embedding's added to the last layer's in place: the same as the sum of the two."""
    p = parameters(torch.bfloat16)
    ids, target = (v.flatten() for v in batch(2))
    x = M.mdet_embedding_forward(ids, p[0])
    loss, lse, _ = M.mdet_xent_forward(x, p[0], target)
    g = torch.full_like(loss, 1 / 40)
    dx, dw, _ = M.mdet_xent_backward(g, x, p[0], target, lse, grad_dtype=torch.float32)
    alone = M.mdet_embedding_backward(dx, ids, VOCAB, grad_dtype=torch.float32)
    both = dw.clone()
    M.mdet_embedding_backward(dx, ids, VOCAB, dtable=both, accumulate=True)
    assert torch.equal(both, dw + alone)


def test_a_step_in_a_graph(M):
    """Forward, backward and the optimiser's step, captured and replayed on new batches, against the same steps one call after the other."""
    def make():
        p = [v.requires_grad_() for v in parameters(torch.bfloat16)]
        return p, M.AdamW(p, lr=1e-3)

    def step(p, opt, ids, target):
        loss = loss_of(M, p, ids, target)
        opt.step(torch.autograd.grad(loss, p))
        return loss.detach()
    eager, opt = make()
    batches = [batch(10 + i) for i in range(5)]
    want = [step(eager, opt, *batches[0]).clone() for _ in range(1)]
    held, opt_held = make()
    ids, target = (v.clone() for v in batches[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = step(held, opt_held, ids, target)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):           # a step's number is part of what is captured: each replay is the second step's arithmetic
        out = step(held, opt_held, ids, target)
    for b in batches[1:]:
        ids.copy_(b[0])
        target.copy_(b[1])
        graph.replay()
        torch.cuda.synchronize()
        opt.steps = 1
        loss = step(eager, opt, *b)
        torch.cuda.synchronize()
        assert torch.equal(out, loss)
        assert all(torch.equal(a, c) for a, c in zip(held, eager))


def test_it_runs(M):
    """Some steps on one batch, from the tensors' own .grad."""
    p = [v.requires_grad_() for v in parameters(torch.float32)]
    opt = M.AdamW(p, lr=3e-3)
    ids, target = batch(3)
    before = [v.detach().clone() for v in p]
    for _ in range(5):
        for v in p:
            v.grad = None
        loss_of(M, p, ids, target).backward()
        opt.step()
    assert all(torch.isfinite(v).all() for v in p) and not any(torch.equal(a, b.detach()) for a, b in zip(before, p))


def test_two_calls_at_once(M):
    """Two streams, each with its own operands and workspaces, at the same time."""
    p = parameters(torch.bfloat16)
    work = [batch(20 + i, rows=40, length=50) for i in range(2)]
    want = []
    for ids, target in work:
        x = M.mdet_embedding_forward(ids.flatten(), p[0])
        loss, lse, kept = M.mdet_xent_forward(x, p[0], target.flatten(), keep=True)
        dx, dw, _ = M.mdet_xent_backward(torch.ones_like(loss), x, p[0], target.flatten(), lse, kept=kept)
        want.append((loss, dx, dw, M.mdet_embedding_backward(dx, ids.flatten(), VOCAB)))
    streams = [torch.cuda.Stream() for _ in work]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for turn in range(6):
        for i, ((ids, target), s) in enumerate(zip(work, streams)):
            with torch.cuda.stream(s):
                x = M.mdet_embedding_forward(ids.flatten(), p[0])
                loss, lse, kept = M.mdet_xent_forward(x, p[0], target.flatten(), keep=True)
                dx, dw, _ = M.mdet_xent_backward(torch.ones_like(loss), x, p[0], target.flatten(), lse, kept=kept)
                got[i].append((loss, dx, dw, M.mdet_embedding_backward(dx, ids.flatten(), VOCAB)))
    torch.cuda.synchronize()
    for i in range(2):
        for results in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(results, want[i]))
