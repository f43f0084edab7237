"""The Gram matrix of a network's Jacobian against J J^T in 64 bits, with bounds derived from the arithmetic."""
import pytest

torch = pytest.importorskip("torch")

from training import strided

pytestmark = pytest.mark.gpu
PAIRS = [(torch.float32, torch.float32), (torch.float64, torch.float64), (torch.float32, torch.float64), (torch.bfloat16, torch.float32),
         (torch.float16, torch.float32), (torch.bfloat16, torch.float64)]
# n, outputs, layers of (p, q)
SIZES = [(1, 1, [(1, 1)]), (2, 1, [(3, 5)]), (63, 1, [(17, 64), (64, 1)]), (130, 1, [(100, 96), (96, 33), (33, 1)]), (257, 1, [(64, 128)]),
         (5, 3, [(7, 9), (9, 3)]), (43, 3, [(50, 40), (40, 3)]), (30, 10, [(65, 32), (32, 10)]), (300, 1, [(8, 520), (520, 16)]), (1, 70, [(5, 70)])]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def layers(n, d, widths, dtype, seed, pad=0, shift=0):
    g = gen(seed)
    return ([strided(n, p, dtype, g, 1.0, pad, shift) for p, _ in widths],
            [strided(n * d, q, dtype, g, max(q, 1) ** -0.5, pad, shift) for _, q in widths])


def gram64(inputs, signals, d, bias=1.0):
    """J J^T and a bound of its rounding errors in units of the arithmetic's eps."""
    total = size = 0
    for a, g in zip(inputs, signals):
        a, g = a.double().repeat_interleave(d, 0), g.double()
        first, second = a @ a.t() + bias, g @ g.t()
        f_abs, s_abs = a.abs() @ a.abs().t() + abs(bias), g.abs() @ g.abs().t()
        total = total + first * second
        # each product's sum of p (q) terms, the multiplication and the sum over layers
        size = size + (a.shape[1] + g.shape[1] + len(inputs) + 6) * f_abs * s_abs
    return total, size


@pytest.mark.parametrize("dtype,out", PAIRS, ids=str)
@pytest.mark.parametrize("n,d,widths", SIZES)
def test_sizes(M, n, d, widths, dtype, out):
    eps = 2.0 ** -23 if out == torch.float32 else 2.0 ** -52
    for pad, shift in ((0, 0), (3, 1), (8, 0)):
        inputs, signals = layers(n, d, widths, dtype, n + d, pad, shift)
        k = torch.full((n * d, n * d + pad), 7.0, dtype=out, device="cuda")[:, :n * d]
        got = M.mdet_ntk_gram(inputs, signals, k, outputs=d, scale=0.25)
        assert got is k
        want, size = gram64(inputs, signals, d)
        low = torch.tril(torch.ones_like(want, dtype=torch.bool))
        off = (k.double() - 0.25 * want).abs()
        assert bool((off <= eps * 0.25 * size)[low].all()), float((off / (eps * 0.25 * size))[low].max())
        assert bool((k == 7.0)[~low].all())                       # nothing above the diagonal
        # added to what is there, without a bias, and layer by layer
        M.mdet_ntk_gram(inputs, signals, k, outputs=d, bias=0.0, scale=-0.5, accumulate=True)
        w0, s0 = gram64(inputs, signals, d, 0.0)
        off = (k.double() - (0.25 * want - 0.5 * w0)).abs()
        assert bool((off <= eps * (size + s0))[low].all())


def test_it_is_the_jacobians_gram_matrix(M):
    """A network of two layers: J from autograd in 64 bits."""
    n, d, widths = 11, 3, (6, 8, 3)
    g = gen(1)
    x = torch.randn(n, widths[0], generator=g, device="cuda").double()
    ws = [torch.randn(b, a, generator=g, device="cuda").double().requires_grad_() for a, b in zip(widths[:-1], widths[1:])]
    bs = [torch.randn(b, generator=g, device="cuda").double().requires_grad_() for b in widths[1:]]
    z1 = x @ ws[0].t() + bs[0]
    h = torch.tanh(z1)
    f = h @ ws[1].t() + bs[1]
    rows, g1 = [], []
    for i in range(n):
        for r in range(d):
            grads = torch.autograd.grad(f[i, r], [*ws, *bs, z1], retain_graph=True)
            rows.append(torch.cat([v.reshape(-1) for v in grads[:4]]))
            g1.append(grads[4][i])
    J = torch.stack(rows)
    signals = [torch.stack(g1), torch.eye(d, dtype=torch.float64, device="cuda").repeat(n, 1)]
    K = M.mdet_ntk_gram([x, h.detach()], signals, outputs=d)
    want = torch.tril(J @ J.t())
    assert K.dtype == torch.float64 and float((K - want).abs().max()) <= 1e-13 * float(want.abs().max())


def test_more_layers_than_a_launch_takes(M):
    for dtype, out in ((torch.float32, torch.float32), (torch.float32, torch.float64)):
        inputs, signals = layers(70, 1, [(5 + i % 7, 3 + i % 5) for i in range(71)], dtype, 3)
        K = M.mdet_ntk_gram(inputs, signals, torch.zeros(70, 70, dtype=out, device="cuda"))
        want, size = gram64(inputs, signals, 1)
        eps = 2.0 ** -23 if out == torch.float32 else 2.0 ** -52
        assert bool(((K.double() - torch.tril(want)).abs() <= 2 * eps * torch.tril(size) + 1e-300).all())


def test_sizes_of_zero_and_widths_of_zero(M):
    e = torch.empty(0, 4, device="cuda")
    assert M.mdet_ntk_gram([e], [e]).shape == (0, 0)
    a, g = torch.empty(5, 0, device="cuda"), torch.randn(5, 3, generator=gen(1), device="cuda")
    K = M.mdet_ntk_gram([a], [g], bias=2.0)                        # a . a' = 0: the bias alone
    assert torch.allclose(K, torch.tril(2 * (g @ g.t())), rtol=1e-5)
    K = M.mdet_ntk_gram([g], [a])
    assert K.shape == (5, 5) and not K.any()


def test_values_that_are_not_finite_stay_in_their_rows(M):
    for dtype in (torch.float32, torch.float64, torch.bfloat16):
        inputs, signals = layers(150, 1, [(70, 50), (50, 20)], dtype, 8)
        inputs[0][40, 3], signals[1][90, 19] = float("nan"), float("inf")
        K = M.mdet_ntk_gram(inputs, signals)
        bad = ~torch.isfinite(K)
        want = torch.zeros_like(bad)
        want[40, :41] = want[90, :91] = True
        want[40:, 40] = want[90:, 90] = True
        assert torch.equal(bad, want)


def test_same_bits_on_another_stream_and_in_a_graph(M):
    for dtype, out in ((torch.float32, torch.float64), (torch.bfloat16, torch.float32)):
        inputs, signals = layers(40, 3, [(33, 40), (40, 3)], dtype, 5)
        want = M.mdet_ntk_gram(inputs, signals, torch.zeros(120, 120, dtype=out, device="cuda"), outputs=3)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        K = torch.zeros(120, 120, dtype=out, device="cuda")
        side.wait_stream(torch.cuda.current_stream())
        M.mdet_ntk_gram(inputs, signals, K, outputs=3, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(K, want)
        ws = torch.empty(max(256, M.mdet_ntk_workspace_query(inputs, signals, out, outputs=3)), dtype=torch.uint8, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            M.mdet_ntk_gram(inputs, signals, K, outputs=3, workspace=ws)
        for i in range(4):
            inputs[0].copy_(torch.randn(40, 33, generator=gen(70 + i), device="cuda"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(K, M.mdet_ntk_gram(inputs, signals, torch.zeros_like(K), outputs=3))


def test_log_determinant_of_what_it_forms(M):
    """The lower triangle goes straight into the log-determinant: K + I against the eigenvalues in 64 bits."""
    inputs, signals = layers(90, 2, [(30, 50), (50, 2)], torch.float64, 12)
    K = M.mdet_ntk_gram(inputs, signals, outputs=2)
    K.diagonal().add_(1.0)
    r = M.mdet_logdet_device(K)
    whole = gram64(inputs, signals, 2)[0] + torch.eye(180, dtype=torch.float64, device="cuda")
    assert r.sign == 1 and abs(r.logabsdet - float(torch.linalg.eigvalsh(whole).log().sum())) <= 1e-9


def test_refusals(M):
    a, g = torch.zeros(6, 4, device="cuda"), torch.zeros(6, 3, device="cuda")
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([], [])
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g, g])
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g[:5]])
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g], outputs=2)
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g], outputs=0)
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a, a.half()], [g, g])
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g], accumulate=True)
    with pytest.raises(ValueError):
        M.mdet_ntk_gram([a], [g], torch.zeros(6, 6, dtype=torch.bfloat16, device="cuda"))
    for bad, status in ((lambda: M.mdet_ntk_gram([a.double()], [g.double()], torch.zeros(6, 6, device="cuda")), M.Status.EINVAL),
                        (lambda: M.mdet_ntk_gram([a], [g], bias=float("inf")), M.Status.EINVAL),
                        (lambda: M.mdet_ntk_gram([a], [g], torch.zeros(6, 6, dtype=torch.float64, device="cuda"),
                                                 workspace=torch.zeros(256, dtype=torch.uint8, device="cuda")[:64]), M.Status.ENOMEM_DEVICE)):
        with pytest.raises(M.MemdetError) as e:
            bad()
        assert e.value.status == status


@pytest.mark.parametrize("dtype,out,n,d", [(torch.float64, torch.float64, 8010, 1), (torch.float64, torch.float64, 8190, 1),
                                           (torch.bfloat16, torch.float32, 811, 10)], ids=str)
def test_large_orders(M, dtype, out, n, d):
    """Orders that are cut into large blocks, what is left over behind whole rounds of them into quarters."""
    inputs, signals = layers(n, d, [(40, 48)], dtype, n)
    k = M.mdet_ntk_gram(inputs, signals, torch.full((n * d, n * d), 7.0, dtype=out, device="cuda"), outputs=d)
    want, size = gram64(inputs, signals, d)
    eps = 2.0 ** -23 if out == torch.float32 else 2.0 ** -52
    off = torch.tril((k.double() - want).abs() - eps * size)
    assert float(off.max()) <= 0
    assert bool((torch.triu(k, 1) == torch.triu(torch.full_like(k, 7.0), 1)).all())
