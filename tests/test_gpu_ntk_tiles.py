"""Every tile shape of the Gram matrix, over layers of several slabs with something left over, with rows that start on 16 bytes and rows
that do not, one output and several, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_ntk import gram64, layers

pytestmark = pytest.mark.gpu
F16, BF16, F32, F64 = torch.float16, torch.bfloat16, torch.float32, torch.float64
WIDTHS = [(100, 161), (161, 96), (320, 7)]
# operands, K, samples, outputs
CASES = [
    (F32, F32, 1600, 1), (F32, F32, 530, 3), (F32, F32, 160, 10),                    # 64 x 64
    (F32, F32, 400, 3),                                                            # 32 x 32, several outputs
    (F64, F64, 1601, 1), (F64, F64, 530, 3), (F64, F64, 4010, 2),                    # 64 x 64
    (F64, F64, 700, 1), (F64, F64, 120, 10),                                       # 32 x 32
    (F64, F64, 8010, 1), (F64, F64, 8200, 1), (F64, F64, 2690, 3),                   # 128 x 128, with quarters and without
    (F64, F64, 4499, 1), (F64, F64, 4500, 1), (F64, F64, 1501, 3), (F64, F64, 470, 10),   # on both sides of the choice
    (F32, F64, 1601, 1), (F32, F64, 2690, 3), (BF16, F64, 530, 3),                   # widened
    (BF16, F32, 1601, 1), (F16, F32, 530, 3), (F16, F32, 4010, 2),                   # 64 x 64
    (BF16, F32, 811, 10), (F16, F32, 2690, 3), (BF16, F32, 1200, 7),                 # 128 x 128
]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    yield m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,out,n,d", CASES, ids=str)
def test_tiles(M, dtype, out, n, d):
    eps = 2.0 ** -23 if out == F32 else 2.0 ** -52
    for pad, shift in ((0, 0), (1, 1), (16, 0)):
        # rows of whole pieces where none stand between them: straight to LDS; the narrow last layer's are not
        widths = WIDTHS if pad else [(96, 160), (160, 96), (320, 8)]
        inputs, signals = layers(n, d, widths, dtype, n + d, pad, shift)
        k = torch.full((n * d, n * d), 7.0, dtype=out, device="cuda")
        M.mdet_ntk_gram(inputs, signals, k, outputs=d, scale=0.25)
        want, size = gram64(inputs, signals, d)
        off = torch.tril((k.double() - 0.25 * want).abs() - eps * 0.25 * size)
        assert float(off.max()) <= 0, (pad, shift)
        assert bool((torch.triu(k, 1) == torch.triu(torch.full_like(k, 7.0), 1)).all())
        again = M.mdet_ntk_gram(inputs, signals, torch.full_like(k, 7.0), outputs=d, scale=0.25)
        assert torch.equal(again, k)
        del want, size, off, again
