"""The softmax cross entropy of a linear layer and its gradient against 64-bit references, with bounds derived from the arithmetic: a
logit is a sum of k + 1 terms in fp32; an exponential is good to a few roundings and those of its argument; e is rounded to the operands'
type in front of its two products (what the forward pass kept was rounded once before, to fp16's or fp32's bits)."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, LEAST, UNIT, check, strided

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# rows, vocabulary, k: few rows (by themselves), every tile shape, several slabs, strips that end inside a tile
SIZES = [(1, 1, 1), (1, 50, 5), (3, 100, 64), (4, 9000, 520), (16, 64, 64), (16, 1003, 2100), (17, 130, 72), (40, 1000, 33), (65, 129, 130), (130, 300, 257),
         (300, 5003, 96), (300, 12001, 200), (520, 25003, 72), (260, 50000, 136), (1030, 257, 64), (600, 3001, 1030), (530, 12001, 77),
         (300, 2000, 1501)]


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
    """x, w, bias, target, g: some rows sure of their target, some targets that do not count."""
    g = gen(seed)
    w = strided(n, k, dtype, g, k ** -0.5, pad, shift)
    t = torch.randint(0, n, (m,), generator=g, device="cuda")
    x = strided(m, k, dtype, g, 1.0, pad, shift)
    x += (torch.rand(m, 1, generator=g, device="cuda") * 12 * w[t].float()).to(dtype)
    out = torch.rand(m, generator=g, device="cuda") < 0.15
    if m > 2:
        t[out] = torch.tensor([-100, n, -1], device="cuda")[torch.randint(0, 3, (m,), generator=g, device="cuda")][out]
    weight = torch.randn(m, generator=g, device="cuda") / m
    return x, w, strided(1, n, dtype, g, 0.5, 0, shift)[0], t, weight


def logits64(x, w, bias):
    """z and a bound of its error."""
    x, w = x.double(), w.double()
    z, size = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    return z, (x.shape[1] + 4) * EPS32 * size


def forward64(z, ez, t, n):
    """loss and lse with bounds; which rows count."""
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    # the sum of the exponentials: relative errors of one (EPS32 (4 + |argument|), and |argument| p stays below 1), of a sum over strips
    el = (p * ez).sum(1) + (n / 512 + 64) * EPS32 + 2 * EPS32 * lse.abs()
    counts = (t >= 0) & (t < n)
    at = torch.where(counts, t, 0)[:, None]
    loss = torch.where(counts, lse - z.gather(1, at)[:, 0], 0.0)
    return (loss, (el + ez.gather(1, at)[:, 0] + 2 * EPS32 * (lse.abs() + z.gather(1, at)[:, 0].abs())) * counts), (lse, el), counts


def backward64(z, ez, x, w, t, g, lse, counts, dtype, kept, wide=False):
    """dx, dw, db with bounds, for the kernel's own lse.  wide: dw and db in 32 bits, of an e that is not rounded to fewer (two fp16 numbers
    are off by two of their roundings one behind the other, 2^-22, three of bf16 hold all 24 bits), nor taken from what was kept."""
    kept = kept and not (wide and dtype != torch.float32)
    m, n = z.shape
    arg = z - lse.double()[:, None]
    p = torch.exp(arg)
    rel = ez + EPS32 * (z.abs() + lse.double().abs()[:, None] + 4 * arg.abs() + 4)
    weight = torch.where(counts, g.double(), 0.0)[:, None]
    e = p.clone()
    rows = torch.nonzero(counts)[:, 0]
    e[rows, t[rows]] -= 1
    e *= weight
    exact = (p * rel + EPS32 * e.abs()) * weight.abs()                 # in front of the rounding
    if kept:                                                           # rounded once before (bf16: to fp16's bits, of a part of 1), but the target's own
        first = (2.0 ** -11 * p + 2.0 ** -24 if dtype == torch.bfloat16 else 2.0 ** -23 * p) * weight.abs()
        first[rows, t[rows]] = 0
        exact = exact + first
    least = LEAST[dtype] * (1.0 if dtype != torch.float16 else 2.0 ** -13 * float(weight.abs().max()))
    err = exact + UNIT[dtype] * (e.abs() + exact) + least
    errw = exact + 2.0 ** -22 * e.abs() + least if wide and dtype != torch.float32 else err
    x = torch.where(counts[:, None], x.double(), 0.0)
    xa, wa, ea = x.abs(), w.double().abs(), e.abs()
    et = e.t().contiguous()
    return ((e @ w.double(), err @ wa + (n + 8) * EPS32 * (ea @ wa)), (et @ x, errw.t().contiguous() @ xa + (3 * m + 8) * EPS32 * (et.abs() @ xa)),
            (e.sum(0), exact.sum(0) + (m + 8) * EPS32 * ea.sum(0)))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(M, m, n, k, dtype):
    for i, (pad, shift) in enumerate([(0, 0), (3, 1), (8, 0)]):
        x, w, bias, t, g = operands(m, n, k, dtype, m + n + k, pad, shift)
        bias = (None, bias, bias)[i]
        t = t.int() if i == 1 else t
        z, ez = logits64(x, w, bias)
        (wl, el), (ws, es), counts = forward64(z, ez, t.long(), n)
        loss, lse, none = M.mdet_xent_forward(x, w, t, bias)
        assert none is None
        check(lse, ws, es, torch.float32, f"lse pad {pad}")
        check(loss, wl, el, torch.float32, f"loss pad {pad}")
        kloss, klse, kept = M.mdet_xent_forward(x, w, t, bias, keep=True)
        assert torch.equal(kloss, loss) and torch.equal(klse, lse)
        for gt in ([dtype] if i else {dtype, torch.float32}):
            for what in (None, kept):
                dx = torch.full((m, k + pad), float("nan"), dtype=dtype, device="cuda")
                dw = torch.full((n, k + pad), float("nan"), dtype=gt, device="cuda")
                got = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=what, dx=dx[:, :k], dw=dw[:, :k], db=True, grad_dtype=gt)
                want = backward64(z, ez, x, w, t.long(), g, lse, counts, dtype, what is not None, gt == torch.float32)
                for v, (a, err), ty, name in zip(got, want, (dtype, gt, gt), ("dx", "dw", "db")):
                    assert v.dtype == ty
                    check(v, a, err, ty, f"{name} pad {pad} kept {what is not None} {gt}")
                assert torch.isnan(dx[:, k:]).all() and torch.isnan(dw[:, k:]).all()


@pytest.mark.parametrize("m,n,k,dtype", [(4200, 140000, 24, torch.bfloat16), (140000, 4500, 20, torch.float16), (4200, 140000, 12, torch.float32)], ids=str)
def test_several_pieces_of_the_vocabulary(M, m, n, k, dtype):
    """More elements of e than are held at once: dx adds up over the pieces.  Against the same call on the rows' halves, which fit one piece
    each and are checked above: dx to one rounding, dw and db as sums of two."""
    x, w, bias, t, g = operands(m, n, k, dtype, 3)
    loss, lse, _ = M.mdet_xent_forward(x, w, t, bias)
    h = (m + 1) // 2 if m < 100000 else m // 4
    for keep in (False, True):
        kept = M.mdet_xent_forward(x, w, t, bias, keep=True)[2] if keep else None
        got = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True, grad_dtype=torch.float32)
        sums, sizes = None, None
        for i in range(0, m, h):
            part = slice(i, min(m, i + h))
            ploss, plse, pkept = M.mdet_xent_forward(x[part], w, t[part], bias, keep=keep)
            dx, dw, db = M.mdet_xent_backward(g[part], x[part], w, t[part], plse, bias, kept=pkept, db=True, grad_dtype=torch.float32)
            # probabilities differ by what two sums of fp32 differ by, which can move a rounding of e by one step; and values of dx itself that
            # differ by however little can be rounded to neighbours: 2 UNIT of them apart, or, below fp16's normal numbers (dx is
            # 1e-5 and less here, they begin at 6e-5), the distance of its multiples of 2^-24, whose half is the error of each of the two roundings
            size = float(dx.double().abs().max())
            assert float((got[0][part].double() - dx.double()).abs().max()) <= 4 * UNIT[dtype] * size + 1e-4 * size + LEAST[dtype]
            sums = [dw.double(), db.double()] if sums is None else [sums[0] + dw, sums[1] + db]
        for v, s in zip(got[1:], sums):
            size = float(s.abs().max())
            assert float((v.double() - s).abs().max()) <= 4 * UNIT[dtype] * size + 1e-4 * size
            assert torch.isfinite(v).all()


def test_rows_that_do_not_count(M):
    """Nothing of them comes through, whatever they hold; a number of the vocabulary can be the one that is ignored."""
    for dtype in TYPES:
        for m, n, k in ((40, 300, 64), (9, 300, 64)):
            x, w, bias, t, g = operands(m, n, k, dtype, 8)
            t = t.clamp(0, n - 1)
            t[::3] = 5
            x[::3] = float("nan")
            x[3] = float("inf")
            g[::3] = float("nan")
            rest = torch.tensor([i for i in range(m) if i % 3], device="cuda")
            t[rest] = torch.where(t[rest] == 5, 6, t[rest])
            for keep in (False, True):
                loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, ignore=5, keep=keep)
                assert not loss[::3].any()
                dx, dw, db = M.mdet_xent_backward(g, x, w, t, lse, bias, ignore=5, kept=kept, db=True)
                assert not dx[::3].any() and all(torch.isfinite(v).all() for v in (dx, dw, db))
                z, ez = logits64(x[rest], w, bias)
                (wl, el), (ws, es), counts = forward64(z, ez, t[rest], n)
                check(loss[rest], wl, el, torch.float32)
                want = backward64(z, ez, x[rest], w, t[rest], g[rest], lse[rest], counts, dtype, keep)
                for v, (a, err), name in zip((dx[rest], dw, db), want, ("dx", "dw", "db")):
                    # the sums run over the m rows, zeros among them
                    check(v, a, err, dtype, name)
            t[:] = -100                                                  # none at all
            loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=True)
            for kept in (None, kept):
                grads = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True)
                assert not loss.any() and not any(v.any() for v in grads)


def test_masked_vocabulary(M):
    """A bias of -inf takes words out: they get no gradient; a target among them costs infinitely much; a row of which nothing is left has
    no loss that is a number."""
    m, n, k = 33, 700, 48
    x, w, bias, t, g = operands(m, n, k, torch.float32, 4)
    bias[100:400] = float("-inf")                                        # whole strips, and parts of them
    t = torch.arange(m, device="cuda") % 90
    t[7] = 200
    for rows in (33, 8):
        for keep in (False, True):
            loss, lse, kept = M.mdet_xent_forward(x[:rows], w, t[:rows], bias, keep=keep)
            z, _ = logits64(x[:rows], w, bias)
            want = torch.logsumexp(z, 1)
            assert float((lse.double() - want).abs().max()) < 1e-4 and float(loss[7]) == float("inf")
            fine = torch.arange(rows, device="cuda") != 7
            assert torch.isfinite(loss[fine]).all()
            dx, dw, db = M.mdet_xent_backward(g[:rows], x[:rows], w, t[:rows], lse, bias, kept=kept, db=True)
            alone = torch.zeros(300, dtype=torch.float32, device="cuda")
            alone[100] = -g[7]                                           # the derivative by its logit is -g all the same
            assert torch.allclose(db[100:400], alone, atol=1e-6) and torch.isfinite(dx).all() and torch.isfinite(dw).all()
    loss, lse, _ = M.mdet_xent_forward(x, w, t, torch.full_like(bias, float("-inf")))
    assert bool((lse == float("-inf")).all()) and torch.isnan(loss).all()


@pytest.mark.parametrize("dtype,up", [(torch.float32, 60), (torch.float16, 15), (torch.bfloat16, 60)], ids=str)
def test_logits_far_beyond_the_exponential(M, dtype, up):
    """One word's logit is 2^(2 up), all the others' half of that or less: every number of the result is exact, in both directions."""
    n, k, best = 700, 8, 333
    for m in (3, 7, 14, 40, 300):
        x, w = torch.zeros(m, k, dtype=dtype, device="cuda"), torch.zeros(n, k, dtype=dtype, device="cuda")
        x[:, 2] = 2.0 ** up
        w[:, 2] = 2.0 ** (up - 1) * (torch.arange(n, device="cuda") % 3 - 1)
        w[best, 2] = 2.0 ** up
        t = torch.arange(m, device="cuda") % n
        t[0] = best
        g = torch.full((m,), 2.0 ** -9, device="cuda")
        z = x.double() @ w.double().t()
        e = -torch.eye(n, dtype=torch.float64, device="cuda")[t]
        e[:, best] += 1
        e *= 2.0 ** -9
        for keep in (False, True):
            loss, lse, kept = M.mdet_xent_forward(x, w, t, keep=keep)
            assert torch.equal(lse.double(), z[:, best]) and torch.equal(loss.double(), (z[:, best:best + 1] - z.gather(1, t[:, None]))[:, 0])
            dx, dw, db = M.mdet_xent_backward(g, x, w, t, lse, kept=kept, db=True)
            for got, want in zip((dx, dw, db), (e @ w.double(), e.t() @ x.double(), e.sum(0))):
                assert torch.equal(got, want.to(dtype))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m", [3, 8, 16, 40, 300])
def test_loss_of_rows_that_are_sure(M, m, dtype):
    """Logits of a thousand, exact, the target's 8 above all others: the loss keeps the digits that lse, a number of a thousand, has not."""
    n, k = 700, 24
    x, w = torch.zeros(m, k, dtype=dtype, device="cuda"), torch.zeros(n, k, dtype=dtype, device="cuda")
    x[:, 1], w[:, 1], w[77, 1] = 32.0, 31.75, 32.0
    t = torch.full((m,), 77, device="cuda")
    loss, lse, _ = M.mdet_xent_forward(x, w, t)
    want = torch.log1p((n - 1) * torch.exp(torch.tensor(-8.0, dtype=torch.float64)))
    part = float((n - 1) * torch.exp(torch.tensor(-8.0)))
    # sums of 700 numbers over strips and lanes, each below 64 roundings of a sum up to 1.3; an exponential of -8 to 12 EPS32; the logarithm's own
    assert float((loss.double() - float(want)).abs().max()) <= 64 * 2.0 ** -24 * 1.3 + 12 * EPS32 * part + 2 * EPS32
    assert float((lse.double() - 1024 - float(want)).abs().max()) <= 2.0 ** -13 + 1e-5


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m", [8, 40, 300])
def test_masked_words_beside_small_logits(M, m, dtype):
    """Whole strips of -inf where all of the other logits lie so low that the exponential of -lse is infinite."""
    n, k = 700, 48
    x, w, bias, t, g = operands(m, n, k, dtype, 6)
    bias -= 300
    bias[128:512] = float("-inf")
    t = torch.where((t >= 128) & (t < 512), 5, t)
    live = torch.cat((torch.arange(128), torch.arange(512, n))).cuda()
    place = torch.full((n,), -1, device="cuda")
    place[live] = torch.arange(len(live), device="cuda")
    u = torch.where((t >= 0) & (t < n), place[t.clamp(0, n - 1)], -1)    # the same rows over the words that are left
    z, ez = logits64(x, w[live], bias[live])
    (wl, el), (ws, es), counts = forward64(z, ez, u, len(live))
    for keep in (False, True):
        loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=keep)
        check(lse, ws, es, torch.float32)
        check(loss, wl, el, torch.float32)
        dx, dw, db = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True)
        assert not dw[128:512].any() and not db[128:512].any()
        want = backward64(z, ez, x, w[live], u, g, lse, counts, dtype, keep)
        for v, (a, err), name in zip((dx, dw[live], db[live]), want, ("dx", "dw", "db")):
            check(v, a, err, dtype, f"{name} kept {keep}")


@pytest.mark.parametrize("m", [0, 1, 63, 1024, 4097, 20000])
@pytest.mark.parametrize("index", [torch.int32, torch.int64])
def test_reduction(M, m, index):
    loss = torch.rand(m, generator=gen(m + 1), device="cuda") * 10
    t = torch.randint(-2, 12, (m,), generator=gen(m), device="cuda", dtype=index)
    counts = (t >= 0) & (t < 10) & (t != 7)
    loss[~counts] = float("nan")                                         # is not looked at
    number, total = int(counts.sum()), float(loss[counts].double().sum())
    for mean in (True, False):
        out, weights = M.mdet_xent_reduce(loss, t, 10, 7, mean=mean)
        assert out.shape == () and weights.shape == (m,) and not weights[~counts].any()
        if number == 0:
            assert torch.isnan(out) if mean else not out.any()
            continue
        want, weight = (total / number, torch.tensor(1 / number, dtype=torch.float32)) if mean else (total, torch.tensor(1.0))
        # a thread's m / 1024 terms and a tree of ten, all of one sign, and the quotient
        assert abs(float(out) - want) <= (m / 1024 + 12) * EPS32 * want
        assert bool((weights[counts] == weight.cuda()).all())
        held = torch.empty(1, device="cuda")
        again, none = M.mdet_xent_reduce(loss, t, 10, 7, mean=mean, out=held, weights=False)
        assert again is held and none is None and torch.equal(held[0], out)


def test_small_probabilities_in_fp16(M):
    """A probability of 1e-8 and a weight of 1 / 4096 are far below fp16's least number: the gradients of the many words nobody expects
    add up to as much as that of the one that came."""
    m, n, k = 64, 20000, 64
    x, w, bias, t, _ = operands(m, n, k, torch.float16, 9)
    t = t.clamp(0, n - 1)
    g = torch.full((m,), 1 / 4096, device="cuda")
    loss, lse, _ = M.mdet_xent_forward(x, w, t)
    _, _, db = M.mdet_xent_backward(g, x, w, t, lse, dx=False, dw=False, db=True, grad_dtype=torch.float32)
    dx, dw, _ = M.mdet_xent_backward(g, x, w, t, lse, grad_dtype=torch.float32)
    z, ez = logits64(x, w, None)
    e = torch.softmax(z, 1) / 4096
    e[torch.arange(m, device="cuda"), t] -= 1 / 4096
    unseen = torch.ones(n, dtype=torch.bool, device="cuda")
    unseen[t] = False
    want = (e.t().contiguous() @ x.double())[unseen]
    assert float((dw[unseen].double() - want).norm() / want.norm()) < 2e-3
    narrow = M.mdet_xent_backward(g * 4096, x, w, t, lse)[1].double()[unseen] / 4096         # 16-bit results, of a loss that is scaled
    assert float((narrow - want).norm() / want.norm()) < 2e-3


def test_parts(M):
    m, n, k = 90, 700, 50
    for dtype in (torch.bfloat16, torch.float16):
        x, w, bias, t, g = operands(m, n, k, dtype, 5)
        loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=True)
        assert torch.equal(M.mdet_xent_forward(x, w, t, bias, lse=False)[0], loss)
        assert torch.equal(M.mdet_xent_forward(x, w, t, bias, loss=None)[1], lse)
        for what in (None, kept):
            whole = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=what, db=True)
            for j in range(3):
                want = [i == j for i in range(3)]
                got = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=what, dx=want[0], dw=want[1], db=want[2])
                assert all((got[i] is None) == (i != j) for i in range(3)) and torch.equal(got[j], whole[j])
            for _ in range(3):                                           # the same bits each time
                assert all(torch.equal(a, b) for a, b in zip(whole, M.mdet_xent_backward(g, x, w, t, lse, bias, kept=what, db=True)))


def test_sizes_of_zero(M):
    x, w, t = torch.randn(4, 8, device="cuda"), torch.randn(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    loss, lse, kept = M.mdet_xent_forward(x[:0], w, t[:0], keep=True)
    assert loss.shape == (0,)
    dx, dw, db = M.mdet_xent_backward(loss, x[:0], w, t[:0], lse, kept=kept, db=True)
    assert dx.shape == (0, 8) and not dw.any() and not db.any()
    loss, lse, _ = M.mdet_xent_forward(x, w[:0], t)
    assert not loss.any() and bool((lse == float("-inf")).all())
    dx, dw, db = M.mdet_xent_backward(torch.ones(4, device="cuda"), x, w[:0], t, lse, db=True)
    assert not dx.any() and dw.shape == (0, 8) and db.shape == (0,)
    for keep in (False, True):
        loss, lse, kept = M.mdet_xent_forward(x[:, :0], w[:, :0], t, keep=keep)
        assert float((lse - torch.log(torch.tensor(10.0))).abs().max()) < 1e-6
        dx, dw, db = M.mdet_xent_backward(torch.ones(4, device="cuda"), x[:, :0], w[:, :0], t, lse, kept=kept, db=True)
        assert dx.shape == (4, 0) and dw.shape == (10, 0)
        assert torch.allclose(db, torch.tensor([0.4 - 4] + [0.4] * 9, device="cuda"), atol=1e-5)


@pytest.mark.parametrize("keep", [False, True])
def test_gradient_against_differences(M, keep):
    """Central differences of the 64-bit loss sum(g loss).  With h = 1e-4 they are off by h^2 / 6 of a third derivative and by 64-bit
    rounding over h, the kernels by fp32 sums: 2e-4 of the sum of sizes holds both."""
    m, n, k = 19, 53, 31
    x, w, bias, t, g = operands(m, n, k, torch.float32, 11)
    _, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=keep)
    grads = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True)
    ops = [x.double(), w.double(), bias.double()]
    counts = (t >= 0) & (t < n)

    def loss(o):
        z = o[0] @ o[1].t() + o[2]
        return float(((torch.logsumexp(z, 1) - z.gather(1, torch.where(counts, t, 0)[:, None])[:, 0]) * g.double() * counts).sum())
    for i, grad in enumerate(grads):
        d = torch.randn(ops[i].shape, generator=gen(40 + i), device="cuda").double()
        plus, minus = [o.clone() for o in ops], [o.clone() for o in ops]
        plus[i] += 1e-4 * d
        minus[i] -= 1e-4 * d
        want, got = (loss(plus) - loss(minus)) / 2e-4, float((grad.double() * d).sum())
        assert abs(got - want) <= 2e-4 * float((grad.double() * d).abs().sum())


def test_the_workspaces_asked_for_are_enough(M):
    for dtype, gt in ((torch.float16, torch.float16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.float16, torch.float32)):
        for m, n, k in ((1, 5, 3), (40, 1000, 33), (7, 300, 64), (64, 64, 8192), (600, 2000, 130), (800, 700, 1001)):
            x, w, bias, t, g = operands(m, n, k, dtype, 1)
            sizes = (M.mdet_xent_workspace_query(dtype, m, n, k), M.mdet_xent_kept_query(dtype, m, n, k),
                     M.mdet_xent_workspace_query(dtype, m, n, k, True, gt))
            a, b, c = (torch.full((s + 4096,), 0xFF, dtype=torch.uint8, device="cuda") for s in sizes)
            loss, lse, _ = M.mdet_xent_forward(x, w, t, bias, workspace=a[:sizes[0]])
            again = M.mdet_xent_forward(x, w, t, bias, keep=b[:sizes[1]])
            assert torch.equal(again[0], loss) and torch.equal(again[1], lse)
            for kept in (None, b[:sizes[1]]):
                got = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True, grad_dtype=gt, workspace=c[:sizes[2]])
                want = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True, grad_dtype=gt)
                assert all(torch.equal(p, q) for p, q in zip(got, want))
            assert all(bool((room[s:] == 0xFF).all()) for room, s in zip((a, b, c), sizes))


@pytest.mark.parametrize("keep", [False, True])
def test_streams_and_graphs(M, keep):
    m, n, k = 150, 1500, 96
    x, w, bias, t, g = operands(m, n, k, torch.float16, 1)

    def both(**kw):
        loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=keep, **kw)
        return (loss, lse, *M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True, **kw))
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
        new = operands(m, n, k, torch.float16, 10 + turn)
        x.copy_(new[0])
        t.copy_(new[3])
        g.copy_(new[4])
        want = both()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_front_end(M, dtype):
    x, w, bias, t, _ = operands(30, 200, 40, dtype, 3)
    x, w, bias, t = x.clone().requires_grad_(), w.clone().requires_grad_(), bias.clone().requires_grad_(), t.view(5, 6)
    z, ez = logits64(x.detach(), w.detach(), bias.detach())
    (wl, el), _, counts = forward64(z, ez, t.view(-1), 200)
    lse = M.mdet_xent_forward(x.detach(), w.detach(), t.view(-1), bias.detach())[1]
    weight = torch.rand(5, 6, generator=gen(4), device="cuda")
    for keep in (False, True):
        for reduction, g in (("mean", counts / counts.sum()), ("sum", counts * 1.0), ("none", weight.view(-1))):
            loss = M.linear_cross_entropy(x.view(5, 6, 40), w, t, bias, reduction=reduction, keep=keep)
            if reduction == "none":
                check(loss.view(-1), wl, el, torch.float32)
                total = (loss * weight).sum()
            else:
                total = loss
                assert abs(float(loss.detach()) - float((wl * g).sum())) <= float(((el + 64 * EPS32 * wl.abs()) * g).sum())
            got = torch.autograd.grad(total, (x, w, bias))
            want = backward64(z, ez, x.detach(), w.detach(), t.view(-1), g.float(), lse, counts, dtype, keep)
            for v, (a, err), name in zip(got, want, ("dx", "dw", "db")):
                check(v, a, err, dtype, f"{name} {reduction} {keep}")
    with torch.no_grad():
        assert torch.equal(M.linear_cross_entropy(x.view(5, 6, 40), w, t, bias), M.linear_cross_entropy(x.view(5, 6, 40), w, t, bias).detach())


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_front_end_in_a_graph(M, reduction):
    """Both passes in a graph, replayed between eager ones: so many rows that a reduction over all of them takes more than one workgroup."""
    m, n, k = 20000, 130, 16
    x, w, bias, t, _ = operands(m, n, k, torch.bfloat16, 1)
    held = [v.contiguous() for v in (x, w, bias)] + [t]

    def step():
        leaves = [v.detach().requires_grad_() for v in held[:3]]
        loss = M.linear_cross_entropy(leaves[0], leaves[1], held[3], leaves[2], reduction=reduction)
        return (loss.detach(), *torch.autograd.grad(loss, leaves, torch.ones_like(loss)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for turn in range(4):
        new = operands(m, n, k, torch.bfloat16, 10 + turn)
        for v, u in zip(held, new):
            v.copy_(u)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, step()))
        torch.cuda.synchronize()
