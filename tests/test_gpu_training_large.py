"""The training operators where elements or workgroups pass 32 bits."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    yield m
    torch.cuda.empty_cache()


def test_column_sums_of_more_rows_than_a_launch_takes(M):
    """2^30 rows of one element: strips of 64 rows for 2^24 workgroups and one more.  Sums of small whole numbers are exact."""
    m = 2 ** 30 + 70
    dy = torch.zeros(m, 1, dtype=torch.bfloat16, device="cuda")
    dy[:3], dy[-7:] = 1, 2
    x, w = dy.new_empty(m, 0), dy.new_empty(1, 0)
    db = M.mdet_linear_backward(dy, x, w, dx=False, dw=False)[2]
    assert db.tolist() == [17.0]
    z, dz = torch.ones_like(dy), torch.full_like(dy, 5.0)
    z[-3:] = -1
    db = M.mdet_linear_backward(dy, x, w, z, "relu", dx=False, dw=False, dz=dz)[2]
    assert db.tolist() == [11.0]
    dy[-3:] = 0
    assert torch.equal(dz, dy)


def test_column_sums_of_more_columns_than_a_launch_takes(M):
    """One row: its column sums are itself.  Sixteen columns a workgroup: 2^24 of them and three more."""
    n = 2 ** 28 + 40
    dy = (torch.arange(n, device="cuda") % 251).to(torch.bfloat16).view(1, n)
    db = M.mdet_linear_backward(dy, dy.new_empty(1, 0), dy.new_empty(n, 0), dx=False, dw=False)[2]
    assert torch.equal(db, dy[0])


def test_operands_of_more_elements_than_a_launch_takes_are_widened(M):
    """A layer of 2^32 and some elements in 16 bits, the Gram matrix in 64: all columns but the outermost are zero, so that a
    few columns are its reference."""
    n, q = 16384, 262208
    assert n * q > 2 ** 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    g = torch.zeros(n, q, dtype=torch.bfloat16, device="cuda")
    ends = torch.randn(n, 8, generator=gen, device="cuda").to(torch.bfloat16)
    g[:, :3], g[:, -5:] = ends[:, :3], ends[:, 3:]
    a = torch.randn(n, 4, generator=gen, device="cuda").to(torch.bfloat16)
    k = M.mdet_ntk_gram([a], [g], torch.zeros(n, n, dtype=torch.float64, device="cuda"))
    del g
    a, e = a.double(), ends.double()
    want, size = (a @ a.t() + 1) * (e @ e.t()), (a.abs() @ a.abs().t() + 1) * (e.abs() @ e.abs().t())
    # products of 4 and 8 terms, one multiplication; sums with zeros are exact
    assert float((torch.tril(k - want).abs() - 20 * 2.0 ** -52 * size).max()) <= 0


def normal(*shape, seed=0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed))


def far(rows, cols, apart, dtype, seed, scale=1.0):
    """A matrix whose rows stand `apart` elements from each other; what lies between is not set."""
    m = torch.empty((rows - 1) * apart + cols, dtype=dtype, device="cuda").as_strided((rows, cols), (apart, 1))
    return m.copy_(normal(rows, cols, seed=seed) * scale)


@pytest.mark.parametrize("m,n,k", [(3, 40, 200), (70, 90, 330)])
def test_rows_so_far_apart_that_offsets_within_a_slab_pass_32_bits(M, m, n, k):
    """Each operand by itself and all together, in all three layouts; the rest is that of the same values side by side."""
    dtype, apart = torch.bfloat16, 40_000_000
    x, w, dy = (normal(*s, seed=i).to(dtype) for i, s in enumerate(((m, k), (n, k), (m, n))))
    fx, fw, fdy = far(m, k, apart, dtype, 0), far(n, k, apart, dtype, 1), far(m, n, apart + 1, dtype, 2)
    assert torch.equal(fx, x) and torch.equal(fw, w) and torch.equal(fdy, dy)
    y, (dx, dw, db) = M.mdet_linear_forward(x, w), M.mdet_linear_backward(dy, x, w)
    want = (x.double() @ w.double().t(), dy.double() @ w.double(), dy.double().t() @ x.double())
    for a, b, c in ((fx, w, dy), (x, fw, dy), (x, w, fdy), (fx, fw, fdy)):
        got = M.mdet_linear_forward(a, b)
        gx, gw, gb = M.mdet_linear_backward(c, a, b)
        out = far(m, n, apart, dtype, 3)
        assert torch.equal(M.mdet_linear_forward(a, b, out=out), got)
        for v, t in zip((got, gx, gw), want):
            # sums of up to 330 products of at most 20, one rounding to 16 bits
            assert float(((v.double() - t).abs() - 2.0 ** -8 * t.abs()).max()) <= 330 * 2.0 ** -23 * 330 * 20 * 2
        assert torch.equal(gb, db)


def test_results_of_more_than_32_bits_of_elements(M):
    m, n, k = 70_000, 65_600, 72
    x, w = normal(m, k).to(torch.bfloat16), normal(n, k, seed=1).to(torch.bfloat16)
    y = M.mdet_linear_forward(x, w, activation="relu")
    assert y.numel() > 2 ** 32
    for rows in (slice(0, 40), slice(35_000, 35_040), slice(m - 40, m)):
        want = torch.relu(x[rows].double() @ w.double().t())
        assert float(((y[rows].double() - want).abs() - 2.0 ** -8 * want).max()) <= 76 * 2.0 ** -23 * 72 * 20
    del y
    a, g = normal(m, 6), normal(m, 9, seed=2)
    kk = M.mdet_ntk_gram([a], [g], torch.zeros(m, m, device="cuda"))
    assert kk.numel() > 2 ** 32
    for r0 in (0, 35_000, m - 40):
        rows = slice(r0, r0 + 40)
        f, s = a[rows].double() @ a.double().t() + 1, g[rows].double() @ g.double().t()
        size = (a[rows].double().abs() @ a.double().abs().t() + 1) * (g[rows].double().abs() @ g.double().abs().t())
        low = torch.arange(m, device="cuda")[None, :] <= torch.arange(r0, r0 + 40, device="cuda")[:, None]
        off = (kk[rows].double() - f * s).abs() - 22 * 2.0 ** -23 * size
        assert float(off[low].max()) <= 0 and not kk[rows][~low].any()


def test_a_tensor_of_more_than_32_bits_of_elements(M):
    """Element by element: its ends are as those of short tensors of the same values."""
    n, h = 2 ** 32 + 1000, dict(lr=1e-2, step=3)
    p, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    m, v = (torch.zeros(n, dtype=torch.float32, device="cuda") for _ in range(2))
    ends = [slice(0, 3000), slice(2 ** 32 - 3000, n)]
    short = []
    for i, e in enumerate(ends):
        for t, scale in ((p, 1.0), (g, 0.1), (m, 0.1), (v, 0.1)):
            t[e] = (normal(t[e].numel(), seed=i) * scale).abs().to(t.dtype)
        short.append([t[e].clone() for t in (p, g, m, v)])
    M.mdet_adamw_step([p], [g], [m], [v], **h)
    for e, (sp, sg, sm, sv) in zip(ends, short):
        M.mdet_adamw_step([sp], [sg], [sm], [sv], **h)
        assert torch.equal(sp, p[e]) and torch.equal(sm, m[e]) and torch.equal(sv, v[e])
