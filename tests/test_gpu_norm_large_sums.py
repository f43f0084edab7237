"""The layer norm's weight gradient over more elements than 32 bits count, against 64-bit sums."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_tokens_large import M, gen         # noqa: F401 (M: a fixture)
from training import EPS32

pytestmark = pytest.mark.gpu


def test_column_sums(M):                         # noqa: F811
    m, n, times = 1_060_000, 4100, 106           # 4.3e9 elements, rows off 16 bytes; the same 10000 rows again and again
    part = torch.randn(m // times, n, generator=gen(3), device="cuda").bfloat16()
    x = part.repeat(times, 1)
    mean, rstd = (v.repeat(times) for v in M.mdet_layernorm_forward(part)[1:])
    _, dw, db = M.mdet_layernorm_backward(x, x, mean, rstd, None, dx=False, grad_dtype=torch.float32)
    dy = part.double()
    h = (dy - mean[:m // times].double()[:, None]) * rstd[:m // times].double()[:, None]
    for got, terms in ((dw, dy * h), (db, dy)):
        # a term is off by a difference, a product and a fused product's rounding; sums in blocks of a few hundred and then 1024 of those
        assert bool(((got.double() - times * terms.sum(0)).abs() <= (1200 + 3) * EPS32 * times * terms.abs().sum(0)).all())
