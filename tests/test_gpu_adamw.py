"""The AdamW step against 64 bits and against its own formula in single roundings."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UNIT = {torch.float32: U, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SIZES = [1, 3, 255, 256, 257, 4095, 4096, 4097, 0, 10000, 64, 12289]
H = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1)


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def flat(n, dtype, g, scale, shift):
    """n normal elements, `shift` of them behind an aligned address, NaN around them."""
    whole = torch.full((n + shift + 16,), float("nan"), dtype=torch.float32, device="cuda").to(dtype)
    v = whole[shift:shift + n]
    v.copy_(torch.randn(n, generator=g, device="cuda") * scale)
    return v


def step64(p, g, m, v, t):
    m = H["beta1"] * m + (1 - H["beta1"]) * g
    v = H["beta2"] * v + (1 - H["beta2"]) * g * g
    up = (m / (1 - H["beta1"] ** t)) / ((v / (1 - H["beta2"] ** t)).sqrt() + H["eps"])
    return p - H["lr"] * (H["weight_decay"] * p + up), m, v, up


@pytest.mark.parametrize("ptype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16, torch.float16], ids=str)
def test_states_in_32_bits(M, ptype, gtype):
    for shift in (0, 1):
        g = gen(shift)
        p = [flat(n, ptype, g, 0.5, shift) for n in SIZES]
        gr = [flat(n, gtype, g, 10.0 ** -(i % 3), shift) for i, n in enumerate(SIZES)]
        m = [flat(n, torch.float32, g, 0.1, shift) for n in SIZES]
        v = [flat(n, torch.float32, g, 0.1, shift).abs_() for n in SIZES]
        copies = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in SIZES] if ptype == torch.float32 else None
        scale = torch.tensor([0.5], device="cuda")
        want = [step64(a.double(), b.double() * 0.5, c.double(), d.double(), 3) for a, b, c, d in zip(p, gr, m, v)]
        M.mdet_adamw_step(p, gr, m, v, step=3, copies=copies, grad_scale=scale, **H)
        for i, (wp, wm, wv, up) in enumerate(want):
            # m: two products and a sum, factors rounded; cancellation between the two terms
            assert bool(((m[i].double() - wm).abs() <= 4 * U * (wm.abs() + 0.2 * gr[i].double().abs() + 1)).all())
            assert bool(((v[i].double() - wv).abs() <= 8 * U * wv + 1e-44).all())
            # p: the two terms to a few units, m's error times the rate over the root, one rounding to its type
            err = 8 * U * wp.abs() + H["lr"] * 40 * U * (up.abs() + (0.2 * gr[i].double().abs() + 1) / (wv.sqrt() + H["eps"]))
            assert bool(((p[i].double() - wp).abs() <= err + UNIT[ptype] * wp.abs() + 2.0 ** -25).all())
            if copies is not None:
                assert torch.equal(copies[i], p[i].to(torch.bfloat16))


def test_a_tensor_gives_the_same_bits_alone_and_among_others(M):
    g = gen(4)
    sizes = [700 + 13 * i for i in range(101)]                 # three launches
    p = [flat(n, torch.float32, g, 1.0, i % 4) for i, n in enumerate(sizes)]
    gr = [torch.randn(n, generator=g, device="cuda") for n in sizes]
    m, v = [torch.zeros(n, device="cuda") for n in sizes], [torch.zeros(n, device="cuda") for n in sizes]
    alone = [(a.clone(), torch.zeros_like(b), torch.zeros_like(b)) for a, b in zip(p, gr)]
    M.mdet_adamw_step(p, gr, m, v, step=1, **H)
    for i in range(0, 101, 9):
        a = alone[i]
        M.mdet_adamw_step([a[0]], [gr[i]], [a[1]], [a[2]], step=1, **H)
        assert torch.equal(a[0], p[i]) and torch.equal(a[1], m[i]) and torch.equal(a[2], v[i])


def eight(n):
    return (torch.zeros(n, dtype=torch.int8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"),
            torch.zeros((n + 255) // 256, 2, device="cuda"))


def decode(code, scales, column):
    return code.double() * scales[:, column].double().repeat_interleave(256)[:code.numel()]


@pytest.mark.parametrize("shift", [0, 1, 2])
def test_states_in_8_bits(M, shift):
    """Ten steps: the stored state stays within one code of what was rounded, and each update is that of the state the
    step began with."""
    g = gen(7)
    p = [flat(n, torch.float32, g, 0.5, shift) for n in SIZES]
    states = [eight(n + 4) for n in SIZES]
    m = [s[0][shift:shift + n] for s, n in zip(states, SIZES)]
    u = [s[1][shift:shift + n] for s, n in zip(states, SIZES)]
    sc = [torch.zeros((n + 255) // 256, 2, device="cuda") for n in SIZES]
    for t in range(1, 11):
        gr = [flat(n, torch.bfloat16, g, 0.1, shift) for n in SIZES]
        before = [(decode(a, s, 0), decode(b, s, 1)) for a, b, s in zip(m, u, sc)]
        want = [step64(a.double(), b.double(), c[0], c[1] ** 2, t) for a, b, c in zip(p, gr, before)]
        M.mdet_adamw_step(p, gr, m, u, scales=sc, step=t, seed=t, **H)
        for i, (wp, wm, wv, up) in enumerate(want):
            err = 8 * U * wp.abs() + H["lr"] * 40 * U * (up.abs() + (gr[i].double().abs() + wm.abs()) / (wv.sqrt() + H["eps"]))
            assert bool(((p[i].double() - wp).abs() <= err).all())
            if not SIZES[i]:
                continue
            for k, (code, x, most) in enumerate(((m[i], wm, 127), (u[i], wv.sqrt(), 255))):
                blocks = torch.nn.functional.pad(x.abs(), (0, -len(x) % 256)).view(-1, 256).amax(1)
                assert torch.allclose(sc[i][:, k].double(), blocks / most, rtol=1e-5, atol=1e-30)
                off = (decode(code, sc[i], k) - x).abs()
                assert bool((off <= 1.001 * sc[i][:, k].double().repeat_interleave(256)[:len(x)] + 1e-30).all())
            assert bool((u[i][wv > 0] >= 1).all())


def test_8_bit_rounding_has_the_right_mean(M):
    """Many seeds on one state: the mean of the decoded values is the value.  Each decoded value is within a code of it,
    so the mean over s seeds has a deviation of at most half a code over sqrt(s); six of them over 512 elements."""
    n, seeds = 512, 400
    g = torch.randn(n, generator=gen(1), device="cuda") * 0.01
    g[0], g[256] = 0.05, 0.05
    sums = [torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2)]
    for s in range(seeds):
        m, u, sc = eight(n)
        M.mdet_adamw_step([torch.zeros(n, device="cuda")], [g], [m], [u], scales=[sc], step=1, seed=s * 7919 + 3, **H)
        sums[0] += decode(m, sc, 0)
        sums[1] += decode(u, sc, 1)
    step = sc.double().repeat_interleave(256, 0)
    wm, wu = (1 - H["beta1"]) * g.double(), math.sqrt(1 - H["beta2"]) * g.double().abs()
    assert bool(((sums[0] / seeds - wm).abs() <= 6 * 0.5 / math.sqrt(seeds) * step[:, 0]).all())
    big = wu > step[:, 1]                                      # below a code the root is kept away from zero
    assert bool(((sums[1] / seeds - wu).abs() <= 6 * 0.5 / math.sqrt(seeds) * step[:, 1])[big].all())


def test_a_second_moment_in_8_bits_decays(M):
    """One large gradient, then none: after s steps v is beta2^s of what it was, give or take the rounding."""
    n = 256 * 64
    p, m = torch.zeros(n, device="cuda"), None
    m, u, sc = eight(n)
    g = torch.rand(n, generator=gen(2), device="cuda") + 0.5
    M.mdet_adamw_step([p], [g], [m], [u], scales=[sc], step=1, seed=0, lr=0.0, beta2=0.999)
    first = decode(u, sc, 1).square().sum()
    for t in range(2, 702):
        M.mdet_adamw_step([p], [torch.zeros_like(g)], [m], [u], scales=[sc], step=t, seed=t, lr=0.0, beta2=0.999)
    left = float(decode(u, sc, 1).square().sum() / first)
    # noise of a code a step adds at most (scale / 2)^2, about (2 / 255 / 2)^2 of v a step
    assert 0.9 * 0.999 ** 700 <= left <= 0.999 ** 700 + 700 * (1.0 / 255) ** 2


def test_blocks_of_zeros_and_of_values_that_are_not_finite(M):
    n = 1024
    p, g = torch.ones(n, device="cuda"), torch.randn(n, generator=gen(3), device="cuda")
    g[:256] = 0
    g[300], g[600] = float("nan"), float("inf")
    m, u, sc = eight(n)
    M.mdet_adamw_step([p], [g], [m], [u], scales=[sc], step=1, lr=1e-3, weight_decay=0.0)
    assert not m[:256].any() and not u[:256].any() and not sc[0].any() and bool((p[:256] == 1).all())
    bad = ~torch.isfinite(p)
    assert bad.nonzero().flatten().tolist() == [300, 600]
    assert not torch.isfinite(sc[1]).any() and not torch.isfinite(sc[2]).any() and torch.isfinite(sc[3]).all()
    M.mdet_adamw_step([p], [torch.zeros_like(g)], [m], [u], scales=[sc], step=2, lr=1e-3, weight_decay=0.0)
    assert torch.isnan(p[256:768]).all() and torch.isfinite(p[:256]).all() and torch.isfinite(p[768:]).all()


def test_optimiser_class(M):
    """A least-squares problem solved to a tenth of its loss by both widths of states; the state can be taken away and
    brought back; the 16-bit copy follows."""
    for bits in (32, 8):
        a = torch.randn(200, 50, generator=gen(5), device="cuda")
        y = a @ torch.randn(50, 3, generator=gen(6), device="cuda")
        w = torch.zeros(50, 3, device="cuda").requires_grad_()
        opt = M.AdamW([w], lr=0.05, weight_decay=0.0, state_bits=bits, copy_dtype=torch.bfloat16)
        first = float((a @ w.detach() - y).square().mean())
        for _ in range(120):
            w.grad = None
            (a @ w - y).square().mean().backward()
            opt.step()
        assert float((a @ w.detach() - y).square().mean()) < 0.1 * first
        assert torch.equal(opt.copies[0], w.detach().to(torch.bfloat16))
        other = M.AdamW([w.detach().clone()], lr=0.05, weight_decay=0.0, state_bits=bits)
        other.load_state_dict(opt.state_dict())
        grad = torch.randn(50, 3, generator=gen(8), device="cuda")
        opt.step([grad])
        other.step([grad])
        assert torch.equal(other.params[0], w.detach())


def test_refusals(M):
    p, g = [torch.zeros(8, device="cuda")], [torch.zeros(8, device="cuda")]
    s = [torch.zeros(8, device="cuda")]
    with pytest.raises(ValueError):
        M.mdet_adamw_step(p, [], s, s, lr=1e-3, step=1)
    with pytest.raises(ValueError):
        M.mdet_adamw_step(p, [g[0][:7]], s, s, lr=1e-3, step=1)
    with pytest.raises(ValueError):
        M.mdet_adamw_step([torch.zeros(4, 4, device="cuda").t()[:2]], [torch.zeros(2, 4, device="cuda")], s, s, lr=1e-3, step=1)
    with pytest.raises(ValueError):
        M.mdet_adamw_step(p, g, [s[0].half()], s, lr=1e-3, step=1)
    for bad in (dict(step=0), dict(step=1, beta1=1.0), dict(step=1, beta2=-0.1), dict(step=1, eps=-1.0), dict(step=1, lr=float("nan"))):
        with pytest.raises(M.MemdetError) as e:
            M.mdet_adamw_step(p, g, s, s, **{"lr": 1e-3, **bad})
        assert e.value.status == M.Status.EINVAL
    with pytest.raises(ValueError):
        M.AdamW(p, state_bits=4)
