"""The token operators where places, elements and workgroups no longer fit 32 bits: against the same calls on parts that do, or against
64-bit references of a few rows."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, UNIT, check

pytestmark = pytest.mark.gpu
GIB = 1 << 30


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 100 * GIB:
        pytest.skip("100 GiB of device memory wanted")
    import paper_2503_04424_amd as m
    m.load()
    yield m
    torch.cuda.empty_cache()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_embedding_of_a_table_beyond_32_bits(M):
    vocab, width, n = 1_200_000, 4096, 700                 # 4.9e9 elements
    table = torch.empty(vocab, width, dtype=torch.bfloat16, device="cuda")
    table.copy_((torch.arange(vocab, device="cuda") % 251)[:, None].expand(vocab, width))
    ids = torch.randint(0, vocab, (n,), generator=gen(1), device="cuda")
    ids[:4] = torch.tensor([0, vocab - 1, vocab, -1], device="cuda")
    y = M.mdet_embedding_forward(ids, table, 2.0)
    want = torch.where((ids >= 0) & (ids < vocab), ids % 251 * 2, 0).to(torch.bfloat16)
    assert torch.equal(y, want[:, None].expand(n, width))
    dy = torch.randn(n, width, generator=gen(2), device="cuda").bfloat16()
    table.fill_(float("nan"))
    M.mdet_embedding_backward(dy, ids, vocab, dtable=table)
    assert int(torch.count_nonzero(table.view(-1, 4096 * 100).float().abs().amax(1))) <= n and torch.isfinite(table[::997]).all()
    for i in (0, 1, 4, 5, 699):
        v = int(ids[i])
        total = dy[ids == v].double().sum(0)
        check(table[v], total, 4 * EPS32 * dy[ids == v].double().abs().sum(0), torch.bfloat16)


def test_norm_of_more_elements_than_32_bits_count(M):
    m, n = 1_060_000, 4100                                  # 4.3e9 elements, rows off 16 bytes
    x = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
    part = torch.randn(10_000, n, generator=gen(3), device="cuda").bfloat16()
    for i in range(0, m, 10_000):
        x[i:i + 10_000] = part
    y, mean, rstd = M.mdet_layernorm_forward(x)
    one = M.mdet_layernorm_forward(part)
    for i in (0, 10_000, m - 10_000):
        assert torch.equal(y[i:i + 10_000], one[0]) and torch.equal(mean[i:i + 10_000], one[1])
    dx, dw, db = M.mdet_layernorm_backward(x, x, mean, rstd, None, dx=y, grad_dtype=torch.float32)
    small = M.mdet_layernorm_backward(part, part, one[1], one[2], None, grad_dtype=torch.float32)
    for i in (0, m - 10_000):
        assert torch.equal(dx[i:i + 10_000], small[0])
    # sums of 106 times the same rows, in blocks of a few hundred and then 1024 of those
    size = part.double().abs().sum(0) * 106
    assert bool(((db.double() - 106 * part.double().sum(0)).abs() <= 1200 * EPS32 * size).all())


def test_cross_entropy_of_more_logits_than_32_bits_count(M):
    m, n, k = 36_000, 125_000, 16                           # 4.5e9 logits, several pieces of the vocabulary
    x = torch.randn(m, k, generator=gen(4), device="cuda").bfloat16()
    w = torch.randn(n, k, generator=gen(5), device="cuda").bfloat16()
    t = torch.randint(0, n, (m,), generator=gen(6), device="cuda")
    g = torch.rand(m, generator=gen(7), device="cuda")
    loss, lse, kept = M.mdet_xent_forward(x, w, t, keep=True)
    rows = torch.tensor([0, 1, 17_000, m - 1], device="cuda")
    z = x[rows].double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    assert float((lse[rows].double() - want).abs().max()) <= 1e-5 and \
        float((loss[rows].double() - (want - z.gather(1, t[rows][:, None])[:, 0])).abs().max()) <= 1e-5
    e = torch.softmax(z, 1) * g[rows].double()[:, None]
    e[torch.arange(4, device="cuda"), t[rows]] -= g[rows].double()
    want = e @ w.double()
    bound = 3 * UNIT[torch.bfloat16] * (e.abs() @ w.double().abs()) + 1e-6
    for what in (None, kept):
        dx, dw, _ = M.mdet_xent_backward(g, x, w, t, lse, kept=what)
        assert bool(((dx[rows].double() - want).abs() <= bound).all())
        for j in (0, 70_000, n - 1):
            zj = x.double() @ w[j].double()
            ej = g.double() * (torch.exp(zj - lse.double()) - (t == j).double())
            size = ej.abs() @ x.double().abs()
            assert bool(((dw[j].double() - ej @ x.double()).abs() <= 4 * UNIT[torch.bfloat16] * size + 1e-6).all())
