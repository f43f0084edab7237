"""The embedding and the gradient of its table against 64-bit references.  A value is scaled in fp32 and rounded once; a sum of c
terms in fp32, in any order, is off by c + 2 roundings of the sum of their sizes."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, check, strided

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# tokens, vocabulary, width: one run and several, widths that are no whole pieces, chunks of columns, buckets of several tokens
SIZES = [(1, 1, 1), (1, 300, 8), (15, 3, 33), (16, 5, 64), (17, 5, 65), (33, 1, 130), (100, 1000, 7), (1000, 257, 520), (1025, 5003, 100), (4100, 40, 24),
         (2500, 9001, 1029)]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def tokens(n, vocab, seed, dtype=torch.int64, outside=True):
    """Some numbers far more often than others; with some that are none of the table."""
    g = gen(seed)
    ids = (torch.rand(n, generator=g, device="cuda").pow(4) * vocab).long().clamp(0, vocab - 1)
    if outside and n > 2:
        pick = torch.randint(0, n, (max(1, n // 9),), generator=g, device="cuda")
        bad = torch.tensor([-1, vocab, -(2 ** 31), 2 ** 31 - 1, -100], device="cuda")
        ids[pick] = bad[torch.randint(0, 5, pick.shape, generator=g, device="cuda")]
    return ids.to(dtype)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_forward(M, n, vocab, width, dtype):
    for i, (pad, shift) in enumerate([(0, 0), (3, 1), (8, 0)]):
        table = strided(vocab, width, dtype, gen(n + vocab), 1.0, pad, shift)
        ids = tokens(n, vocab, n + i, (torch.int64, torch.int32)[i % 2])
        scale = (1.0, 45.25, -0.3)[i]
        out = strided(n, width, dtype, gen(1), 0.0, pad, shift)
        out.fill_(float("nan"))
        whole = out.as_strided((n * (width + pad),), (1,))
        assert M.mdet_embedding_forward(ids, table, scale, out=out) is out
        inside = (ids >= 0) & (ids < vocab)
        want = table.double()[torch.where(inside, ids.long(), 0)] * scale * inside[:, None]
        check(out, want, 2 * EPS32 * want.abs(), dtype)
        assert not out[~inside].any()
        if pad:
            assert torch.isnan(whole.view(n, width + pad)[:, width:]).all()          # what lies between the rows is left alone
        if scale == 1.0:
            assert torch.equal(out, want.to(dtype))


def grad64(dy, ids, vocab, scale, before=None):
    """The gradient and a bound of its error."""
    inside = torch.nonzero((ids >= 0) & (ids < vocab))[:, 0]
    at = ids[inside].long()
    total = torch.zeros(vocab, dy.shape[1], dtype=torch.float64, device="cuda")
    size = total.index_add(0, at, dy.double()[inside].abs()) * abs(scale)
    count = torch.bincount(at, minlength=vocab)[:, None]
    total = total.index_add(0, at, dy.double()[inside]) * scale
    err = (count + 2) * EPS32 * size
    if before is not None:
        total = total + before.double()
        err = err + EPS32 * total.abs()
    return total, err, count[:, 0]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n,vocab,width", SIZES)
def test_gradient(M, n, vocab, width, dtype):
    for i, (pad, shift) in enumerate([(0, 0), (3, 1), (8, 0)]):
        for gt in {dtype, torch.float32}:
            dy = strided(n, width, dtype, gen(n + width), 1.0, pad, shift)
            ids = tokens(n, vocab, n + i, (torch.int32, torch.int64)[i % 2])
            dy[(ids < 0) | (ids >= vocab)] = float("nan")                            # padding has no part in it
            scale = (1.0, 0.125, -3.3)[i]
            got = strided(vocab, width, gt, gen(2), 0.0, pad, shift)
            got.fill_(float("nan"))
            whole = got.as_strided((vocab * (width + pad),), (1,))
            M.mdet_embedding_backward(dy, ids, vocab, scale, got, grad_dtype=gt)
            want, err, count = grad64(dy, ids, vocab, scale)
            check(got, want, err, gt, f"pad {pad} shift {shift}")
            assert not got[count == 0].any()
            if pad:
                assert torch.isnan(whole.view(vocab, width + pad)[:, width:]).all()
            # added to what is there; rows that do not occur keep every bit, NaN among them
            before = strided(vocab, width, gt, gen(3), 1.0, pad, shift)
            before[count == 0] = float("nan")
            after = before.clone()
            M.mdet_embedding_backward(dy, ids, vocab, scale, after, accumulate=True)
            want, err, _ = grad64(dy, ids, vocab, scale, before)
            check(after[count > 0], want[count > 0], err[count > 0], gt, "added")
            assert torch.isnan(after[count == 0]).all()


@pytest.mark.parametrize("n", [7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 1000, 20000])
@pytest.mark.parametrize("kind", ["one token", "in order", "backwards", "two in turn", "none"])
def test_orders(M, n, kind):
    """Runs of one token over many parts of the sum, each token once, tokens that end where a part ends."""
    i = torch.arange(n, device="cuda")
    ids = {"one token": torch.full_like(i, 7), "in order": i, "backwards": n - 1 - i, "two in turn": i % 2 * 300, "none": torch.full_like(i, -1)}[kind]
    vocab, width = max(n, 400), 40
    dy = strided(n, width, torch.bfloat16, gen(n))
    got = M.mdet_embedding_backward(dy, ids, vocab, grad_dtype=torch.float32)
    want, err, _ = grad64(dy, ids, vocab, 1.0)
    check(got, want, err, torch.float32)
    # the same bits from 32-bit ids, and each time
    for _ in range(3):
        assert torch.equal(M.mdet_embedding_backward(dy, ids.int(), vocab, grad_dtype=torch.float32), got)


@pytest.mark.parametrize("n,width", [(6143, 72), (6144, 72), (8400, 1001), (1000, 8400), (20000, 420)])
@pytest.mark.parametrize("kind", ["some often", "one token", "in order"])
def test_orders_of_wide_rows(M, n, width, kind):
    """Each length of a run: of four sorted tokens, of eight, and of sixteen where there are 2^23 elements or more."""
    i = torch.arange(n, device="cuda")
    ids = {"some often": tokens(n, n, n), "one token": torch.full_like(i, 7), "in order": i}[kind]
    dy = strided(n, width, torch.bfloat16, gen(n), 1.0, 3, 1)
    got = M.mdet_embedding_backward(dy, ids, n, 0.5, grad_dtype=torch.float32)
    want, err, _ = grad64(dy, ids, n, 0.5)
    check(got, want, err, torch.float32)
    before = strided(n, width, torch.float32, gen(3))
    want, err, _ = grad64(dy, ids, n, 0.5, before)
    check(M.mdet_embedding_backward(dy, ids, n, 0.5, before, accumulate=True), want, err, torch.float32, "added")
    assert torch.equal(M.mdet_embedding_backward(dy, ids.int(), n, 0.5, grad_dtype=torch.float32), got)


def test_many_tokens_of_a_bucket(M):
    """A vocabulary whose buckets are as large as they get, and one that has more of them."""
    for vocab in (524287, 524288, 1048575, 1100000):
        g = gen(vocab)
        ids = torch.randint(0, vocab, (5000,), generator=g, device="cuda")
        ids[:300] = vocab - 1 - 512 * torch.arange(300, device="cuda")          # those of one bucket
        ids[300:400] = vocab - 1
        dy = strided(5000, 3, torch.float32, g)
        got = M.mdet_embedding_backward(dy, ids, vocab)
        want, err, _ = grad64(dy, ids, vocab, 1.0)
        check(got, want, err, torch.float32)


def test_sizes_of_zero(M):
    t = torch.ones(5, 8, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    assert M.mdet_embedding_forward(none, t).shape == (0, 8)
    assert M.mdet_embedding_forward(torch.zeros(3, dtype=torch.int32, device="cuda"), t[:, :0]).shape == (3, 0)
    assert not M.mdet_embedding_forward(torch.zeros(3, dtype=torch.int32, device="cuda"), t[:0]).any()
    assert not M.mdet_embedding_backward(torch.empty(0, 8, device="cuda"), none, 5).any()
    before = torch.randn(5, 8, device="cuda")
    after = before.clone()
    M.mdet_embedding_backward(torch.empty(0, 8, device="cuda"), none, 5, dtable=after, accumulate=True)
    assert torch.equal(before, after)
    assert M.mdet_embedding_backward(torch.ones(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"), 0).shape == (0, 8)


def test_the_workspace_asked_for_is_enough(M):
    """A workspace of just the size that the query names, NaN and ones in it and behind it."""
    for n, vocab, width in ((1, 5, 3), (40, 300, 70), (3000, 900, 33)):
        need = M.mdet_embedding_workspace_query(n, vocab, width)
        room = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
        dy, ids = strided(n, width, torch.float32, gen(n)), tokens(n, vocab, n)
        got = M.mdet_embedding_backward(dy, ids, vocab, workspace=room[:need])
        assert torch.equal(got, M.mdet_embedding_backward(dy, ids, vocab))
        assert bool((room[need:] == 0xFF).all())


def test_streams_and_graphs(M):
    n, vocab, width = 700, 900, 96
    table, dy, ids = strided(vocab, width, torch.bfloat16, gen(1)), strided(n, width, torch.bfloat16, gen(2)), tokens(n, vocab, 3)
    y, g = M.mdet_embedding_forward(ids, table, 2.0), M.mdet_embedding_backward(dy, ids, vocab, 2.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = M.mdet_embedding_forward(ids, table, 2.0, stream=side), M.mdet_embedding_backward(dy, ids, vocab, 2.0, stream=side)
    side.synchronize()
    assert torch.equal(a, y) and torch.equal(b, g)
    out, grad = torch.zeros_like(y), torch.zeros_like(g)
    ws = torch.empty(M.mdet_embedding_workspace_query(n, vocab, width), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.mdet_embedding_forward(ids, table, 2.0, out=out)
        M.mdet_embedding_backward(dy, ids, vocab, 2.0, grad, workspace=ws)
    for turn in range(4):
        ids.copy_(tokens(n, vocab, 10 + turn))
        y, g = M.mdet_embedding_forward(ids, table, 2.0), M.mdet_embedding_backward(dy, ids, vocab, 2.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, y) and torch.equal(grad, g)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_front_end(M, dtype):
    vocab, width = 50, 24
    table = strided(vocab, width, dtype, gen(1)).clone().requires_grad_()
    ids = tokens(60, vocab, 2).view(3, 20)
    y = M.embedding(ids, table, 3.0)
    assert y.shape == (3, 20, width) and y.dtype == dtype
    t = torch.randn(y.shape, generator=gen(3), device="cuda").to(dtype)
    got, = torch.autograd.grad((y * t).sum(), table)
    want, err, _ = grad64(t.view(-1, width), ids.view(-1), vocab, 3.0)
    check(got, want, err, dtype)
    got, = torch.autograd.grad(M.embedding(ids[:, ::2], table, 3.0).sum(), table)      # a gradient of ones that is one element, repeated
    want, err, _ = grad64(torch.ones(30, width, device="cuda", dtype=dtype), ids[:, ::2].reshape(-1), vocab, 3.0)
    check(got, want, err, dtype)
    with torch.no_grad():
        assert torch.equal(M.embedding(ids, table, 3.0), y)
    # against differences: the map is linear in the table
    d = torch.randn(vocab, width, generator=gen(4), device="cuda").to(dtype)
    if dtype == torch.float32:
        slope = float((M.embedding(ids, d, 3.0).double() * t.double()).sum())
        got, = torch.autograd.grad((M.embedding(ids, table, 3.0) * t).sum(), table)
        assert abs(float((got.double() * d.double()).sum()) - slope) <= 70 * EPS32 * 3 * float((d.double().abs().sum()) * t.double().abs().max())
