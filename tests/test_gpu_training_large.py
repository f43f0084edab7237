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
