"""The linear layer and its gradient against 64-bit references, with bounds derived from the arithmetic (fp32 sums, one
rounding to the stored type; dz is rounded to the operands' type in front of the gradient's products)."""
import pytest

torch = pytest.importorskip("torch")

from training import ACTS, EPS32, LEAST, UNIT, act64, check, forward64, strided

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
SIZES = [(1, 1, 1), (1, 5, 3), (2, 16, 64), (7, 65, 33), (16, 64, 64), (17, 130, 72), (64, 64, 128), (65, 129, 130), (33, 300, 1000),
         (130, 257, 191), (1, 2048, 1536), (5, 1000, 4104), (256, 256, 256), (300, 520, 264), (1025, 96, 40), (600, 1031, 520)]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def operands(m, n, k, dtype, seed, pad=0, shift=0):
    g = gen(seed)
    x = strided(m, k, dtype, g, 1.0, pad, shift)
    w = strided(n, k, dtype, g, max(k, 1) ** -0.5, pad, shift)
    bias = strided(1, n, dtype, g, 0.3, 0, shift)[0]
    residual = strided(m, n, dtype, g, 1.0, pad, shift)
    return x, w, bias, residual


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_forward_sizes(M, m, n, k, dtype):
    for i, (pad, shift) in enumerate([(0, 0), (3, 1), (8, 0)]):
        act = ACTS[(m + n + i) % 5]
        x, w, bias, residual = operands(m, n, k, dtype, 10 * m + n + k, pad, shift)
        z = torch.empty(m, n, dtype=dtype, device="cuda")
        y = M.mdet_linear_forward(x, w, bias, residual, act, preact=z)
        want, wz, err, errz = forward64(x, w, bias, residual, act)
        check(y, want, err, dtype, f"{act} pad {pad} shift {shift}")
        check(z, wz, errz, dtype, "z")
        bare = M.mdet_linear_forward(x, w)
        want, _, err, _ = forward64(x, w, None, None, "none")
        check(bare, want, err, dtype, "bare")


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_forward_activations(M, act, dtype):
    for bias_on, res_on in ((True, True), (False, True), (True, False)):
        x, w, bias, residual = operands(70, 200, 96, dtype, 3)
        x.mul_(3)
        bias, residual = bias if bias_on else None, residual if res_on else None
        y = M.mdet_linear_forward(x, w, bias, residual, act)
        want, _, err, _ = forward64(x, w, bias, residual, act)
        check(y, want, err, dtype, act)


def grad64(dy, x, w, z, act, dtype, out_dtype):
    """dx, dw, db, each with a bound: dz has a relative error of one rounding plus the slope's, sums are fp32."""
    u = UNIT[dtype] if act != "none" else 0.0
    dz = dy.double()
    if act != "none":
        dz = dz * act64(act, z.double())[1]
    slope_err = 0 if act in ("none", "relu") else 2.0 ** -18 * dy.double().abs() * (1 + (z.double().abs() if z is not None else 0))
    m, n = dz.shape
    dzerr = u * dz.abs() + slope_err + (LEAST[dtype] if act != "none" else 0)
    wa, xa = w.double().abs(), x.double().abs()
    dx, dw, db = dz @ w.double(), dz.t().contiguous() @ x.double(), dz.sum(0)
    ex = dzerr @ wa + (n + 4) * EPS32 * (dz.abs() @ wa)
    ew = dzerr.t().contiguous() @ xa + (m + 4) * EPS32 * (dz.abs().t().contiguous() @ xa)
    eb = (slope_err if torch.is_tensor(slope_err) else torch.zeros_like(dz)).sum(0) + (m + 4) * EPS32 * dz.abs().sum(0)
    return (dx, ex), (dw, ew), (db, eb)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gradient_sizes(M, m, n, k, dtype):
    for i, (pad, shift) in enumerate([(0, 0), (3, 1), (8, 0)]):
        act = ACTS[(m + k + i) % 5]
        g = gen(m + n + k)
        x, w, _, _ = operands(m, n, k, dtype, m + 3 * n + k, pad, shift)
        dy, z = strided(m, n, dtype, g, 1.0, pad, shift), strided(m, n, dtype, g, 1.5, pad, shift)
        for gt in ([dtype] if i else {dtype, torch.float32}):
            dz = torch.empty(m, n, dtype=dtype, device="cuda")
            got = M.mdet_linear_backward(dy, x, w, z if act != "none" else None, act, grad_dtype=gt, dz=dz if i == 2 else None)
            for v, (want, err), t, name in zip(got, grad64(dy, x, w, z, act, dtype, gt), (dtype, gt, gt), ("dx", "dw", "db")):
                assert v.dtype == t
                check(v, want, err, t, f"{name} {act} pad {pad} shift {shift}")
            if i == 2:
                wz = dy.double() * act64(act, z.double())[1]
                check(dz, wz, 2.0 ** -18 * dy.double().abs() * (1 + z.double().abs()), dtype, "dz")


def test_gradient_of_parts(M):
    g = gen(5)
    x, w, _, _ = operands(90, 70, 50, torch.bfloat16, 5)
    dy, z = strided(90, 70, torch.bfloat16, g), strided(90, 70, torch.bfloat16, g)
    whole = M.mdet_linear_backward(dy, x, w, z, "silu")
    for k in range(3):
        want = [i == k for i in range(3)]
        got = M.mdet_linear_backward(dy, x, w, z, "silu", dx=want[0], dw=want[1], db=want[2])
        for i in range(3):
            assert (got[i] is None) == (i != k)
        assert torch.equal(got[k], whole[k])


@pytest.mark.parametrize("act", ACTS)
def test_gradient_against_differences(M, act):
    """Central differences of the 64-bit loss sum(y t) in directions of every operand, against the kernels' gradients in
    fp32.  With h = 1e-4 the differences are off by h^2 / 6 times a third derivative (of the order of the loss's own terms)
    and by rounding of 64 bits over h; the kernels by fp32 sums: 2e-4 of the sum of magnitudes holds both."""
    m, n, k = 19, 23, 31
    x, w, bias, residual = operands(m, n, k, torch.float32, 11)
    t = torch.randn(m, n, generator=gen(2), device="cuda")
    z = torch.empty(m, n, device="cuda")
    M.mdet_linear_forward(x, w, bias, residual, act, preact=z)
    dx, dw, db = M.mdet_linear_backward(t, x, w, z, act)
    ops = [x.double(), w.double(), bias.double(), residual.double()]

    def loss(o):
        return float(((act64(act, o[0] @ o[1].t() + o[2])[0] + o[3]) * t.double()).sum())
    for i, grad in enumerate((dx, dw, db, t)):
        d = torch.randn(ops[i].shape, generator=gen(40 + i), device="cuda").double()
        if act == "relu":       # no kink within the step
            zz = ops[0] @ ops[1].t() + ops[2]
            assert float(zz.abs().min()) > 0
            h = min(1e-4, 0.01 * float(zz.abs().min()))
        else:
            h = 1e-4
        plus, minus = [o.clone() for o in ops], [o.clone() for o in ops]
        plus[i] += h * d
        minus[i] -= h * d
        want = (loss(plus) - loss(minus)) / (2 * h)
        got = float((grad.double() * d).sum())
        assert abs(got - want) <= 2e-4 * float((grad.double() * d).abs().sum()), (i, got, want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_sizes_of_zero(M, dtype):
    x, w, bias, residual = operands(4, 6, 0, dtype, 1)
    y = M.mdet_linear_forward(x, w, bias, residual, "gelu")          # an empty sum
    want, _, err, _ = forward64(x, w, bias, residual, "gelu")
    check(y, want, err, dtype)
    assert M.mdet_linear_forward(x.new_empty(0, 5), x.new_empty(6, 5), bias).shape == (0, 6)
    assert M.mdet_linear_forward(x.new_empty(3, 5), x.new_empty(0, 5)).shape == (3, 0)
    dx, dw, db = M.mdet_linear_backward(x.new_empty(0, 6), x.new_empty(0, 5), x.new_ones(6, 5))
    assert dx.shape == (0, 5) and not dw.any() and not db.any() and dw.shape == (6, 5)
    dx, dw, db = M.mdet_linear_backward(x.new_empty(3, 0), x.new_ones(3, 5), x.new_empty(0, 5))
    assert not dx.any() and dx.shape == (3, 5) and dw.shape == (0, 5) and db.shape == (0,)


def test_values_that_are_not_finite(M):
    """Infinities and NaN stay in the rows (columns) that they enter."""
    for dtype in TYPES:
        for m in (9, 150):
            x, w, bias, _ = operands(m, 80, 70, dtype, 9)
            x[3, 5], x[7, 60] = float("nan"), float("inf")
            y = M.mdet_linear_forward(x, w, bias, None, "silu")
            rows = torch.isfinite(y).all(1)
            assert not rows[3] and not rows[7] and int(rows.sum()) == m - 2
            assert torch.isnan(y[3]).all()
    # a pre-activation that overflowed its 16 bits has the slope of its side
    z = torch.tensor([[float("inf"), -float("inf"), 60000.0, -60000.0]], dtype=torch.float16, device="cuda")
    one, x, w = torch.ones_like(z), torch.ones(1, 8, dtype=torch.float16, device="cuda"), torch.ones(4, 8, dtype=torch.float16, device="cuda")
    for act in ACTS[1:]:
        db = M.mdet_linear_backward(one, x, w, z, act, dx=False, dw=False)[2]
        assert db.tolist() == [1.0, 0.0, 1.0, 0.0], act
        w2 = torch.tensor([[1.0], [-1.0]], dtype=torch.float16, device="cuda")
        y = M.mdet_linear_forward(torch.full((1, 1), 65504.0, dtype=torch.float16, device="cuda"), w2, activation=act)
        assert y[0, 0] == 65504 and y[0, 1] == 0, act


@pytest.mark.parametrize("m,n,k", [(1, 777, 2048), (40, 300, 3000), (512, 640, 768)])
def test_same_bits_each_time_and_on_another_stream(M, m, n, k):
    for dtype in TYPES:
        x, w, bias, residual = operands(m, n, k, dtype, 21)
        dy, z = strided(m, n, dtype, gen(1)), strided(m, n, dtype, gen(2))
        y = M.mdet_linear_forward(x, w, bias, residual, "gelu")
        grads = M.mdet_linear_backward(dy, x, w, z, "gelu")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for s in (None, side):
            y2 = M.mdet_linear_forward(x, w, bias, residual, "gelu", stream=s)
            g2 = M.mdet_linear_backward(dy, x, w, z, "gelu", stream=s)
            torch.cuda.synchronize()
            assert torch.equal(y, y2)
            assert all(torch.equal(a, b) for a, b in zip(grads, g2))


def test_output_over_the_residual(M):
    for m in (1, 70):
        x, w, bias, residual = operands(m, 520, 1040, torch.bfloat16, 4)
        y = M.mdet_linear_forward(x, w, bias, residual, "relu")
        assert M.mdet_linear_forward(x, w, bias, residual, "relu", out=residual) is residual
        assert torch.equal(y, residual)


def test_captured_in_a_graph(M):
    """A decoding step and a gradient, replayed between the program's own work with new inputs."""
    m, n, k = 1, 512, 2048
    x, w, bias, residual = operands(m, n, k, torch.bfloat16, 8)
    xb, wb, _, _ = operands(300, 256, 520, torch.bfloat16, 9)
    dy, z = strided(300, 256, torch.bfloat16, gen(3)), strided(300, 256, torch.bfloat16, gen(4))
    ws = torch.empty(max(256, M.mdet_linear_workspace_query(x.dtype, m, n, k),
                         M.mdet_linear_workspace_query(x.dtype, 300, 256, 520, backward=True)), dtype=torch.uint8, device="cuda")
    y, outs = torch.empty(m, n, dtype=x.dtype, device="cuda"), M.mdet_linear_backward(dy, xb, wb, z, "gelu")

    def step():
        M.mdet_linear_forward(x, w, bias, residual, "gelu", out=y, workspace=ws)
        M.mdet_linear_backward(dy, xb, wb, z, "gelu", *outs, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(torch.randn(m, k, generator=gen(50 + i), device="cuda"))
        dy.copy_(torch.randn(300, 256, generator=gen(60 + i), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, M.mdet_linear_forward(x, w, bias, residual, "gelu"))
        for a, b in zip(outs, M.mdet_linear_backward(dy, xb, wb, z, "gelu")):
            assert torch.equal(a, b)


def test_autograd_front_end(M):
    """`linear` on three-dimensional inputs, with a transposed weight and every gradient, against the same in 64 bits."""
    g = gen(31)
    x = torch.randn(3, 17, 40, generator=g, device="cuda").requires_grad_()
    w = torch.randn(40, 24, generator=g, device="cuda").t().requires_grad_()
    b = torch.randn(24, generator=g, device="cuda").requires_grad_()
    r = torch.randn(3, 17, 24, generator=g, device="cuda").requires_grad_()
    t = torch.randn(3, 17, 24, generator=g, device="cuda")
    for act in ACTS:
        y = M.linear(x, w, b, r, act)
        got = torch.autograd.grad((y * t).sum(), (x, w, b, r))
        ops = [v.detach().double().requires_grad_() for v in (x, w, b, r)]
        y64 = act64(act, ops[0] @ ops[1].t() + ops[2])[0] + ops[3]
        want = torch.autograd.grad((y64 * t.double()).sum(), ops)
        assert torch.allclose(y.double(), y64, rtol=1e-4, atol=1e-4)
        for a, v in zip(got, want):       # fp32 sums of at most 51 terms of size about 10
            assert float((a.double() - v).abs().max()) <= 51 * EPS32 * 60 * 2, act


def test_refusals(M):
    x, w, bias, residual = operands(8, 12, 16, torch.float32, 1)
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x, w.half())
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x, w[:, :15])
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x, w, bias[:11])
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x, w, bias, residual[:7])
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x, w, activation="swish")
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x.t(), w[:, :8])
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x.cpu(), w)
    with pytest.raises(ValueError):
        M.mdet_linear_forward(x.double(), w.double())
    with pytest.raises(ValueError):
        M.mdet_linear_backward(residual, x, w, None, "gelu")
    with pytest.raises(M.MemdetError) as e:
        M.mdet_linear_backward(residual, x, w, grad_dtype=torch.bfloat16)
    assert e.value.status == M.Status.EINVAL
    with pytest.raises(M.MemdetError) as e:
        M.mdet_linear_backward(residual, x, w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda")[:8])
    assert e.value.status == M.Status.ENOMEM_DEVICE
