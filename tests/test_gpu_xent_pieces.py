"""The cross entropy's gradient over several pieces of the vocabulary, every element against a 64-bit reference: results of the operands' own type, so that
what the forward pass kept is used on both sides of a piece's end, words next to the ends among the targets."""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_xent import M, backward64, forward64, logits64, operands      # noqa: F401 (M: a fixture)
from training import check

pytestmark = pytest.mark.gpu
GIB = 1 << 30
# rows, vocabulary, k, type, and where the second piece begins: half of the words, in multiples of 256 (more than 2^29 elements of e; of 140000 rows 4096
# words are taken at once)
CASES = [(4200, 140000, 24, torch.bfloat16, 70144), (140000, 4500, 20, torch.float16, 2304), (4200, 140000, 12, torch.float32, 70144),
         (140000, 4500, 8, torch.bfloat16, 2304)]


@pytest.mark.parametrize("keep", [False, True])
@pytest.mark.parametrize("m,n,k,dtype,end", CASES, ids=str)
def test_every_element(M, m, n, k, dtype, end, keep):                        # noqa: F811
    if torch.cuda.mem_get_info()[0] < 100 * GIB:
        pytest.skip("100 GiB of device memory wanted")
    x, w, bias, t, g = operands(m, n, k, dtype, 12)
    for i, word in enumerate((0, end - 2, end - 1, end, end + 1, n - 1)):
        t[i::1000] = word
    z, ez = logits64(x, w, bias)
    (wl, el), (ws, es), counts = forward64(z, ez, t, n)
    loss, lse, kept = M.mdet_xent_forward(x, w, t, bias, keep=keep)
    check(lse, ws, es, torch.float32, "lse")
    check(loss, wl, el, torch.float32, "loss")
    # the target's e goes by the loss, whose error is its own (times the derivative of expm1, the probability)
    own = el * torch.exp(-wl) * g.double().abs() * counts
    at = torch.where(counts, t, 0)
    more = (own[:, None] * w.double().abs()[at], torch.zeros(n, k, dtype=torch.float64, device="cuda").index_add_(0, at, own[:, None] * x.double().abs()),
            torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, at, own))
    want = backward64(z, ez, x, w, t, g, lse, counts, dtype, keep)
    del z, ez
    for given in (loss, None):
        got = M.mdet_xent_backward(g, x, w, t, lse, bias, kept=kept, db=True, loss=given)
        for v, (a, err), extra, name in zip(got, want, more, ("dx", "dw", "db")):
            assert v.dtype == dtype
            check(v, a, err + extra, dtype, f"{name} kept {keep} loss {given is not None}")
    torch.cuda.empty_cache()
