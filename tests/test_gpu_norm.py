"""The layer norm and its gradient against 64-bit references.  Sums over a row run over n / 64 terms a lane at most and a tree over the
lanes behind that: DEPTH roundings in fp32."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, check, strided

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# each way of sharing a row out, up to its last column and beyond, for both sizes of elements
COLS = [1, 7, 8, 33, 64, 65, 128, 129, 256, 257, 512, 513, 1000, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384, 16385, 32768, 32769, 70001]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def depth(n):
    return n / 64 + 24


def operands(m, n, dtype, seed, pad=0, shift=0, mean=0.7):
    g = gen(seed)
    x = strided(m, n, dtype, g, 2.0, pad, shift)
    x += mean
    w = strided(1, n, dtype, g, 0.5, 0, shift)[0]
    w += 1
    return x, w, strided(1, n, dtype, g, 0.5, 0, shift)[0]


def forward64(x, w, b, eps):
    """y, mean, rstd, each with a bound."""
    x, n = x.double(), x.shape[1]
    mean = x.mean(1, keepdim=True)
    c = x - mean
    var = (c * c).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    em = (depth(n) + 2) * EPS32 * x.abs().mean(1, keepdim=True)
    # the mean's error enters the variance squared: the deviations add up to zero
    ev = (depth(n) + 6) * EPS32 * var + em * em
    er = rstd * (0.5 * ev / (var + eps) + 4 * EPS32)
    y = c * rstd
    ey = (em + EPS32 * c.abs()) * rstd + c.abs() * er + em * er + 2 * EPS32 * y.abs()
    if w is not None:
        y, ey = y * w.double(), ey * w.double().abs() + EPS32 * (y * w.double()).abs()
    if b is not None:
        y = y + b.double()
        ey = ey + EPS32 * (y.abs() + b.double().abs())
    return (y, ey), (mean[:, 0], em[:, 0]), (rstd[:, 0], er[:, 0])


def backward64(dy, x, mean, rstd, w):
    """dx, dw, db, each with a bound."""
    m, n = x.shape
    dy, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    u = dy if w is None else dy * w.double()
    c0, c1 = u.mean(1, keepdim=True), (u * h).mean(1, keepdim=True)
    e0, e1 = ((depth(n) + k) * EPS32 * v.abs().mean(1, keepdim=True) for k, v in ((4, u), (8, u * h)))
    dx = r * (u - c0 - h * c1)
    ex = r * (e0 + h.abs() * e1 + 6 * EPS32 * (u.abs() + c0.abs() + (h * c1).abs()))
    return (dx, ex), ((dy * h).sum(0), (m + 8) * EPS32 * (dy * h).abs().sum(0)), (dy.sum(0), (m + 4) * EPS32 * dy.abs().sum(0))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", COLS)
def test_sizes(M, n, dtype):
    for i, (m, pad, shift) in enumerate([(1, 0, 0), (5, 3, 1), (37, 8, 0)]):
        x, w, b = operands(m, n, dtype, m + n, pad, shift)
        w, b = (w, b) if i else (None, None)
        out = torch.full((m, n + pad), float("nan"), dtype=dtype, device="cuda")
        y, mean, rstd = M.mdet_layernorm_forward(x, w, b, 1e-5, out=out[:, :n])
        (wy, ey), (wm, em), (wr, er) = forward64(x, w, b, 1e-5)
        check(y, wy, ey, dtype, f"y {m} pad {pad}")
        check(mean, wm, em, torch.float32, "mean")
        check(rstd, wr, er, torch.float32, "rstd")
        assert torch.isnan(out[:, n:]).all()
        bare = M.mdet_layernorm_forward(x, w, b, 1e-5, mean=False, rstd=None)
        assert torch.equal(bare[0], y) and bare[1] is None and bare[2] is None
        dy = strided(m, n, dtype, gen(n), 1.0, pad, shift)
        for gt in {dtype, torch.float32}:
            dx = torch.full((m, n + pad), float("nan"), dtype=dtype, device="cuda")
            got = M.mdet_layernorm_backward(dy, x, mean, rstd, w, dx=dx[:, :n], grad_dtype=gt)
            for v, (want, err), t, name in zip(got, backward64(dy, x, mean, rstd, w), (dtype, gt, gt), ("dx", "dw", "db")):
                assert v.dtype == t
                check(v, want, err, t, f"{name} {m} pad {pad}")
            assert torch.isnan(dx[:, n:]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("n", [100, 1000, 4096, 40000])
def test_parts_and_many_rows(M, n, dtype):
    """More rows than workgroups; each gradient by itself."""
    m = 20000 if n < 4096 else 2100 if n < 40000 else 70
    x, w, b = operands(m, n, dtype, n)
    dy = strided(m, n, dtype, gen(n))
    _, mean, rstd = M.mdet_layernorm_forward(x, w, b)
    whole = M.mdet_layernorm_backward(dy, x, mean, rstd, w, grad_dtype=torch.float32)
    for v, (want, err), t, name in zip(whole, backward64(dy, x, mean, rstd, w), (dtype, torch.float32, torch.float32), ("dx", "dw", "db")):
        check(v, want, err, t, name)
    for k in range(3):
        want = [i == k for i in range(3)]
        got = M.mdet_layernorm_backward(dy, x, mean, rstd, w, dx=want[0], dw=want[1], db=want[2], grad_dtype=torch.float32)
        for i in range(3):
            assert (got[i] is None) == (i != k)
        assert torch.equal(got[k], whole[k])


@pytest.mark.parametrize("n", [50, 700, 3000, 12000])
def test_rows_with_a_large_mean(M, n):
    """A mean of 1000 deviations: the variance keeps its digits, and the bound says how many."""
    x, w, b = operands(9, n, torch.float32, n, mean=2000.0)
    y, mean, rstd = M.mdet_layernorm_forward(x, w, b)
    (wy, ey), (wm, em), (wr, er) = forward64(x, w, b, 1e-5)
    check(y, wy, ey, torch.float32)
    check(rstd, wr, er, torch.float32)
    assert float((er / wr).max()) < 2e-3


def test_rows_that_are_constant_or_not_finite(M):
    x = torch.randn(6, 200, device="cuda")
    x[1] = 3.0
    x[2, 7] = float("nan")
    x[3, 5] = float("inf")
    x[4] = 0.0
    y, mean, rstd = M.mdet_layernorm_forward(x, eps=1e-5)
    assert not y[1].any() and not y[4].any() and abs(float(rstd[1]) - 1e-5 ** -0.5) < 1e-3
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()          # as an average over such a row is
    for i in (0, 5):
        assert torch.equal(y[i:i + 1], M.mdet_layernorm_forward(x[i:i + 1], eps=1e-5)[0])


@pytest.mark.parametrize("dtype,value", [(torch.float32, 1.5 * 2.0 ** 120), (torch.bfloat16, 1.5 * 2.0 ** 120), (torch.float32, -1.25 * 2.0 ** 120)], ids=str)
@pytest.mark.parametrize("n", [1, 50, 100, 129])
def test_gradient_of_a_large_constant_row(M, n, dtype, value):
    """mean rstd is more than fp32 holds, and nothing of it is needed: the row is its mean."""
    x = torch.full((3, n), value, dtype=dtype, device="cuda")
    dy = strided(3, n, dtype, gen(n))
    y, mean, rstd = M.mdet_layernorm_forward(x, eps=1e-6)
    assert not y.any() and bool((mean == value).all()) and bool(torch.isinf(mean * rstd).all())
    got = M.mdet_layernorm_backward(dy, x, mean, rstd)
    for v, (want, err), name in zip(got, backward64(dy, x, mean, rstd, None), ("dx", "dw", "db")):
        check(v, want, err, dtype, name)


def test_sizes_of_zero(M):
    x = torch.randn(4, 8, device="cuda")
    y, mean, rstd = M.mdet_layernorm_forward(x[:, :0], eps=0.25)
    assert y.shape == (4, 0) and not mean.any() and bool((rstd == 2.0).all())
    y, mean, rstd = M.mdet_layernorm_forward(x[:0])
    assert y.shape == (0, 8) and mean.shape == (0,)
    dx, dw, db = M.mdet_layernorm_backward(x[:0], x[:0], mean, rstd, torch.ones(8, device="cuda"))
    assert dx.shape == (0, 8) and not dw.any() and not db.any() and dw.shape == (8,)
    dx, dw, db = M.mdet_layernorm_backward(x[:, :0], x[:, :0], torch.zeros(4, device="cuda"), torch.ones(4, device="cuda"))
    assert dx.shape == (4, 0) and dw.shape == (0,)


def test_gradient_against_differences(M):
    """Central differences of the 64-bit loss sum(y t).  With h = 1e-4 they are off by h^2 / 6 of a third derivative, of the order of
    the loss's own terms, and the kernels by fp32 sums: 2e-4 of the sum of sizes holds both."""
    m, n = 7, 150
    x, w, b = operands(m, n, torch.float32, 5)
    t = torch.randn(m, n, generator=gen(6), device="cuda")
    _, mean, rstd = M.mdet_layernorm_forward(x, w, b)
    grads = M.mdet_layernorm_backward(t, x, mean, rstd, w)
    ops = [x.double(), w.double(), b.double()]

    def loss(o):
        return float((forward64(o[0], o[1], o[2], 1e-5)[0][0] * t.double()).sum())
    for i, grad in enumerate(grads):
        d = torch.randn(ops[i].shape, generator=gen(40 + i), device="cuda").double()
        plus, minus = [o.clone() for o in ops], [o.clone() for o in ops]
        plus[i] += 1e-4 * d
        minus[i] -= 1e-4 * d
        want, got = (loss(plus) - loss(minus)) / 2e-4, float((grad.double() * d).sum())
        assert abs(got - want) <= 2e-4 * float((grad.double() * d).abs().sum())


def test_the_workspace_asked_for_is_enough(M):
    for m, n in ((1, 3), (40, 70), (3000, 900), (20, 17000), (5, 70001)):
        x, w, b = operands(m, n, torch.bfloat16, n)
        _, mean, rstd = M.mdet_layernorm_forward(x, w, b)
        need = M.mdet_layernorm_workspace_query(torch.bfloat16, m, n)
        room = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        got = M.mdet_layernorm_backward(x, x, mean, rstd, w, workspace=room[:need])
        for a, c in zip(got, M.mdet_layernorm_backward(x, x, mean, rstd, w)):
            assert torch.equal(a, c)
        assert bool((room[need:] == 0xFF).all())


def test_streams_and_graphs(M):
    m, n = 300, 777
    x, w, b = operands(m, n, torch.bfloat16, 1)
    dy = strided(m, n, torch.bfloat16, gen(2))

    def both(**kw):
        y, mean, rstd = M.mdet_layernorm_forward(x, w, b, **kw)
        return (y, mean, rstd, *M.mdet_layernorm_backward(dy, x, mean, rstd, w, **kw))
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for turn in range(4):
        x.copy_(operands(m, n, torch.bfloat16, 10 + turn)[0])
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_front_end(M, dtype):
    x, w, b = (v.clone().requires_grad_() for v in operands(30, 64, dtype, 3))
    t = torch.randn(5, 6, 64, generator=gen(4), device="cuda").to(dtype)
    y = M.layer_norm(x.view(5, 6, 64), w, b)
    got = torch.autograd.grad((y * t).sum(), (x, w, b))
    _, mean, rstd = M.mdet_layernorm_forward(x.detach(), w.detach(), b.detach())
    for v, (want, err), name in zip(got, backward64(t.view(30, 64), x.detach(), mean, rstd, w.detach()), ("dx", "dw", "db")):
        check(v, want, err, dtype, name)
    with torch.no_grad():
        assert torch.equal(M.layer_norm(x.view(5, 6, 64), w, b), y)
    z = M.layer_norm(x.view(5, 6, 64).transpose(0, 1))                 # no weights; a view; a gradient that is one element, repeated
    assert torch.equal(z, M.layer_norm(x.view(5, 6, 64)).transpose(0, 1))
    got, = torch.autograd.grad(z.sum(), x)
    (want, err), _, _ = backward64(torch.ones(30, 64, device="cuda", dtype=dtype), x.detach(), mean, rstd, None)
    check(got, want, err, dtype)
