"""The gradient of the cross entropy for rows that are sure of their target: what is left of its probability, 1 - p, is a small number, and the target's
e = -g (1 - p) has to keep it where lse, a number of the logits' size, is rounded to more than 1 - p."""
import pytest

torch = pytest.importorskip("torch")

from training import EPS32, LEAST, UNIT, check

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]
# rows and vocabulary: few rows, every tile shape, more strips of a row than a wavefront joins
SIZES = [(3, 700), (8, 700), (16, 700), (40, 700), (300, 701), (530, 12001), (17, 70001)]
K = 24


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def operands(m, n, dtype):
    """Logits that are exact in every type: of row i 32 s for word 77 and 31.75 s for all others, s = 64, 32, 16 in turn (word 77 is 16, 8 and 4 above
    the others, at 2048, 1024 and 512).  Column 2 of W is there for word 77 alone and zero in x: dx of it is the target's e.  Every seventh row has
    another target."""
    x, w = torch.zeros(m, K, dtype=dtype, device="cuda"), torch.zeros(n, K, dtype=dtype, device="cuda")
    x[:, 1] = torch.tensor([64.0, 32.0, 16.0], device="cuda")[torch.arange(m, device="cuda") % 3].to(dtype)
    w[:, 1], w[77, 1], w[77, 2] = 31.75, 32.0, 1.0
    t = torch.full((m,), 77, device="cuda")
    t[6::7] = 3
    g = torch.rand(m, generator=torch.Generator(device="cuda").manual_seed(m), device="cuda") * 2 - 1
    return x, w, t, g


def want64(x, w, t, g, dtype, kept, wide):
    """dx, dw, db in 64 bits, with bounds.  The target's e is g expm1(-loss): of the loss, 48 additions to a sum of exponentials next to 1 on any path
    (16 in a lane, 2 across lanes, 3 strips, 6 across lanes, 15 across wavefronts), half a step of numbers below 1.5 each (s = 16: 1 + 700 exp(-4) = 14
    for 700 words, to whose logarithm the same relative errors go), 12 EPS32 of the exponentials, that of the logarithm, of a loss up to 30 and of
    expm1; times its derivative, p.  The others' e is g exp(z - lse), from the rounding of lse, a difference and an exponential; bf16 keeps 11 bits of
    them."""
    m, n = x.shape[0], w.shape[0]
    z = x.double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    rows = torch.arange(m, device="cuda")
    arg = z - lse[:, None]
    p = torch.exp(arg)
    weight = g.double()[:, None]
    loss = -arg[rows, t]
    others = 1 - torch.exp(z.amax(1) - lse)
    e = p.clone()
    own = torch.expm1(-loss)
    e[rows, t] = own
    rel = EPS32 * (lse.abs()[:, None] + 4 * arg.abs() + 4)
    err = p * rel + EPS32 * p
    if kept:
        err = err + (2.0 ** -11 * p + 2.0 ** -24 if dtype == torch.bfloat16 else 2.0 ** -23 * p)
    err[rows, t] = torch.exp(-loss) * (48 * 2.0 ** -24 * 1.5 + 12 * EPS32 * others + 2 * EPS32 * (1 + loss)) + 4 * EPS32 * own.abs()
    e, exact = e * weight, (err + EPS32 * e.abs()) * weight.abs()
    least = LEAST[dtype] * (1.0 if dtype != torch.float16 else 2.0 ** -13 * float(weight.abs().max()))
    err = exact + UNIT[dtype] * (e.abs() + exact) + least
    errw = exact + 2.0 ** -22 * e.abs() + least if wide else err
    xa, wa, ea, et = x.double().abs(), w.double().abs(), e.abs(), e.t().contiguous()
    return ((e @ w.double(), err @ wa + (n + 8) * EPS32 * (ea @ wa)), (et @ x.double(), errw.t().contiguous() @ xa + (3 * m + 8) * EPS32 * (et.abs() @ xa)),
            (e.sum(0), exact.sum(0) + (m + 8) * EPS32 * ea.sum(0)))


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("m,n", SIZES)
def test_gradient(M, m, n, dtype, keep):
    x, w, t, g = operands(m, n, dtype)
    loss, lse, kept = M.mdet_xent_forward(x, w, t, keep=keep)
    for gt in {dtype, torch.float32}:
        wide = gt != dtype
        want = want64(x, w, t, g, dtype, keep and not wide, wide)
        calls = [dict(loss=loss)] if not keep else [dict(kept=kept), dict(kept=kept, loss=loss)]
        for kw in calls:
            got = M.mdet_xent_backward(g, x, w, t, lse, db=True, grad_dtype=gt, **kw)
            for v, (a, err), ty, name in zip(got, want, (dtype, gt, gt), ("dx", "dw", "db")):
                assert v.dtype == ty
                check(v, a, err, ty, f"{name} {gt} {sorted(kw)}")
            # the target's e by itself: its rounding and the loss's, and nothing that is added up
            sure = t == 77
            a, err = want[0][0][sure, 2], want[0][1][sure, 2] - (n + 8) * EPS32 * want[0][0][sure, 2].abs()
            check(got[0][sure, 2], a, err + EPS32 * a.abs(), dtype, f"e {gt} {sorted(kw)}")


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("reduction", ["none", "sum"])
def test_front_end(M, dtype, keep, reduction):
    x, w, t, g = operands(40, 700, dtype)
    if reduction == "sum":
        g = torch.ones_like(g)
    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    loss = M.linear_cross_entropy(a, b, t, reduction=reduction, keep=keep)
    loss *= 2.0                                  # in place, as any result may be
    got = torch.autograd.grad(loss, (a, b), 0.5 * g if reduction == "none" else torch.tensor(0.5, device="cuda"))
    for v, (want, err), name in zip(got, want64(x, w, t, g, dtype, keep, False), ("dx", "dw")):
        check(v, want, err, dtype, name)


def test_more_than_one_piece_of_the_vocabulary(M):
    """Word 77's part is taken by a word of the last of two pieces, whose e is formed behind the first one's."""
    m, n, f32 = 4200, 140000, torch.float32
    x, w, t, g = operands(m, n, f32)
    best = n - 5
    w[77, 1], w[77, 2], w[best, 1], w[best, 2] = 31.75, 0.0, 32.0, 1.0
    t[t == 77] = best
    left = (n - 1) * torch.exp(-0.25 * x[:, 1].double())                 # all others' exponentials, beside 1 of this word
    p = 1 / (1 + left)
    own = torch.where(t == best, -left * p, p)
    # bounds as above, of rows with this target and with another
    off = torch.where(t == best, p * (48 * 2.0 ** -24 * 1.5 + 12 * EPS32 * left * p + 2 * EPS32 * (1 - torch.log(p))) + 4 * EPS32 * own.abs(),
                      p * EPS32 * (2 * 2048 + 4 * 16 + 8))
    own, off = own * g.double(), (off + EPS32 * own.abs()) * g.double().abs()
    for keep in (False, True):
        loss, lse, kept = M.mdet_xent_forward(x, w, t, keep=keep)
        dx, dw, db = M.mdet_xent_backward(g, x, w, t, lse, kept=kept, db=True, loss=None if keep else loss)
        check(dx[:, 2], own, off + EPS32 * own.abs(), f32, f"dx {keep}")
        check(db[best], own.sum(), off.sum() + (m + 8) * EPS32 * own.abs().sum(), f32, f"db {keep}")
        size = own.abs() * x[:, 1].double()
        check(dw[best, 1], (own * x[:, 1].double()).sum(), (off * x[:, 1].double()).sum() + (m + 8) * EPS32 * size.sum(), f32, f"dw {keep}")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_what_is_kept_does_not_depend_on_the_results_asked_for(M, dtype):
    """The losses are among what is kept, also where the caller wants none; where both are there the result is the same, bit by bit."""
    x, w, t, g = operands(40, 701, dtype)
    t[::5] = -100
    loss, lse, kept = M.mdet_xent_forward(x, w, t, keep=True)
    want = M.mdet_xent_backward(g, x, w, t, lse, kept=kept, db=True)
    for without in (dict(loss=None), dict(lse=None), dict(loss=None, lse=None)):
        other = M.mdet_xent_forward(x, w, t, keep=True, **without)[2]
        for given in (None, loss):
            assert all(torch.equal(a, b) for a, b in zip(want, M.mdet_xent_backward(g, x, w, t, lse, kept=other, db=True, loss=given)))
