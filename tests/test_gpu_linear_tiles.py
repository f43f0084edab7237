"""Every tile shape of the linear layer's products in its three layouts, over sums of several slabs with something left over, with
rows that start on 16 bytes and rows that do not, against 64 bits."""
import pytest

torch = pytest.importorskip("torch")

import linear_tiles
from test_gpu_linear import gen, grad64, operands
from training import check, forward64, strided

pytestmark = pytest.mark.gpu
PLACES = [(0, 0), (8, 0), (3, 1)]          # elements between rows, and in front of the first
CASES = [(t, *s) for t in (torch.bfloat16, torch.float16, torch.float32) for s in linear_tiles.sizes(t.itemsize)]


@pytest.fixture(scope="module")
def M():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2503_04424_amd as m
    m.load()
    yield m
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype,rows,cols,k,tile,split", CASES, ids=str)
def test_forward(M, dtype, rows, cols, k, tile, split):
    for pad, shift in PLACES:
        x, w, bias, residual = operands(rows, cols, k, dtype, rows + k, pad, shift)
        z = torch.empty(rows, cols, dtype=dtype, device="cuda")
        y = M.mdet_linear_forward(x, w, bias, residual, "gelu", preact=z)
        want, wz, err, errz = forward64(x, w, bias, residual, "gelu")
        check(y, want, err, dtype, f"pad {pad} shift {shift}")
        check(z, wz, errz, dtype, f"z, pad {pad} shift {shift}")
        bare = M.mdet_linear_forward(x, w)
        want, _, err, _ = forward64(x, w, None, None, "none")
        check(bare, want, err, dtype, f"bare, pad {pad} shift {shift}")


@pytest.mark.parametrize("dtype,rows,cols,k,tile,split", CASES, ids=str)
def test_gradient_by_x(M, dtype, rows, cols, k, tile, split):
    """dx = dz w: its second operand's rows run across the sum."""
    for i, (pad, shift) in enumerate(PLACES):
        act, g = ("none", "silu")[i % 2], gen(i)
        w = strided(k, cols, dtype, g, k ** -0.5, pad, shift)
        dy, z = strided(rows, k, dtype, g, 1.0, pad, shift), strided(rows, k, dtype, g, 1.5, pad, shift)
        x = torch.zeros(rows, cols, dtype=dtype, device="cuda")
        dx = M.mdet_linear_backward(dy, x, w, z, act, dw=False, db=False)[0]
        check(dx, *grad64(dy, x, w, z, act, dtype, dtype)[0], dtype, f"{act} pad {pad} shift {shift}")


@pytest.mark.parametrize("dtype,rows,cols,k,tile,split", CASES, ids=str)
def test_gradient_by_w(M, dtype, rows, cols, k, tile, split):
    """dw = dz^T x: the rows of both operands run across the sum; in the operands' type and in fp32."""
    for i, (pad, shift) in enumerate(PLACES):
        act, g = ("none", "silu")[i % 2], gen(i)
        x = strided(k, cols, dtype, g, 1.0, pad, shift)
        dy, z = strided(k, rows, dtype, g, 1.0, pad, shift), strided(k, rows, dtype, g, 1.5, pad, shift)
        w = torch.zeros(rows, cols, dtype=dtype, device="cuda")
        for gt in {dtype, torch.float32}:
            _, dw, db = M.mdet_linear_backward(dy, x, w, z, act, dx=False, grad_dtype=gt)
            _, want, wdb = grad64(dy, x, w, z, act, dtype, gt)
            check(dw, *want, gt, f"{act} pad {pad} shift {shift} {gt}")
            check(db, *wdb, gt, f"db {act} pad {pad} shift {shift} {gt}")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("size,tile", linear_tiles.PAIRS, ids=str)
def test_both_products_in_one_launch(M, size, tile, dtype):
    m, n, k = size
    for i, (pad, shift) in enumerate(PLACES):
        act, g = ("none", "silu")[i % 2], gen(i)
        x, w = strided(m, k, dtype, g, 1.0, pad, shift), strided(n, k, dtype, g, k ** -0.5, pad, shift)
        dy, z = strided(m, n, dtype, g, 1.0, pad, shift), strided(m, n, dtype, g, 1.5, pad, shift)
        for gt in (dtype, torch.float32):
            got = M.mdet_linear_backward(dy, x, w, z, act, grad_dtype=gt)
            for v, (want, err), t, name in zip(got, grad64(dy, x, w, z, act, dtype, gt), (dtype, gt, gt), ("dx", "dw", "db")):
                check(v, want, err, t, f"{name} {act} pad {pad} shift {shift} {gt}")


@pytest.mark.parametrize("dtype,m,n,k", [(torch.bfloat16, 4096, 4104, 520), (torch.float16, 2100, 2200, 1000), (torch.bfloat16, 1100, 1000, 2048),
                                         (torch.float32, 3700, 3701, 150), (torch.float32, 1100, 1000, 777)], ids=str)
def test_same_bits_each_time(M, dtype, m, n, k):
    x, w, bias, residual = operands(m, n, k, dtype, 2)
    dy, z = strided(m, n, dtype, gen(3)), strided(m, n, dtype, gen(4))
    first = None
    for _ in range(12):
        got = (M.mdet_linear_forward(x, w, bias, residual, "gelu"), *M.mdet_linear_backward(dy, x, w, z, "gelu"))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("m,n,k", [(1, 9001, 1001), (4, 16384, 2048), (5, 9001, 520), (16, 10000, 2049), (2, 33000, 64), (17, 9001, 520)])
def test_few_rows_of_a_long_layer(M, m, n, k, dtype):
    """Up to four rows (16 in fp32) by the kernel that reads W once, the others by tiles."""
    for pad, shift in PLACES:
        x, w, bias, residual = operands(m, n, k, dtype, m + n, pad, shift)
        y = M.mdet_linear_forward(x, w, bias, residual, "silu")
        want, _, err, _ = forward64(x, w, bias, residual, "silu")
        check(y, want, err, dtype, f"pad {pad} shift {shift}")
