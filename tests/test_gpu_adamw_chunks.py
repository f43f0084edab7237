"""Steps over so many elements that a workgroup takes several rounds of them, against the same tensors one at a time."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu
SIZES = [3_000_001, 5, 1_500_003, 4095, 4097, 0, 12_289, 1023]
H = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-6, weight_decay=0.1, step=3)


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    return m


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gtype", [torch.float32, torch.bfloat16], ids=str)
def test_many_elements(M, bits, gtype):
    assert sum(SIZES) > 4 << 20 > max(SIZES)        # four rounds a workgroup for all of them, one for any by itself
    g = torch.Generator(device="cuda").manual_seed(bits)

    def normal(n, scale=1.0):
        return torch.randn(n, generator=g, device="cuda") * scale
    p, gr = [normal(n) for n in SIZES], [normal(n, 0.1).to(gtype) for n in SIZES]
    if bits == 32:
        m, v, sc = [normal(n, 0.1) for n in SIZES], [normal(n, 0.1).square() for n in SIZES], None
    else:
        m = [torch.randint(-127, 128, (n,), generator=g, device="cuda").to(torch.int8) for n in SIZES]
        v = [torch.randint(1, 256, (n,), generator=g, device="cuda").to(torch.uint8) for n in SIZES]
        sc = [torch.rand((n + 255) // 256, 2, generator=g, device="cuda") * 1e-3 for n in SIZES]
    copies = [torch.empty(n, dtype=torch.bfloat16, device="cuda") for n in SIZES]
    state = [p, m, v, copies] + ([sc] if sc else [])
    before = [[t.clone() for t in part] for part in state]
    M.mdet_adamw_step(p, gr, m, v, scales=sc, copies=copies, seed=9, **H)
    for i, n in enumerate(SIZES):
        # alone in the call, with its number (the rounding goes by it): the others are empty
        only = [[t if j == i else t[:0] for j, t in enumerate(part)] for part in before]
        M.mdet_adamw_step(only[0], [t if j == i else t[:0] for j, t in enumerate(gr)], only[1], only[2], scales=only[4] if sc else None,
                          copies=only[3], seed=9, **H)
        for part, mine in zip(only, state):
            assert torch.equal(part[i], mine[i]), (i, n)
    assert torch.equal(copies[0], p[0].to(torch.bfloat16)) and bool(torch.isfinite(p[0]).all())
