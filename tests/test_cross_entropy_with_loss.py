"""CPU-only checks of the cross entropy's gradient from the forward call's losses: operands and refusals, of the binding and of the C ABI."""
import pytest

torch = pytest.importorskip("torch")

from test_tokens_host_logic import A, BF16, EINVAL, ENOMEM, F16, F32, F64, M      # noqa: F401 (M: a fixture)
from test_tokens_operands import F, I, library                                   # noqa: F401 (a fixture)
from test_training_operands import on

import paper_2503_04424_amd as package


def test_operands(library):                                                       # noqa: F811
    g, x, w, t, lse, loss, dx, dw = (on(0, *s, dtype=d) for s, d in (((4,), F), ((4, 8), F), ((10, 8), F), ((4,), I), ((4,), F), ((4,), F), ((4, 8), F), ((10, 8), F)))

    def gradient(loss):
        package.mdet_xent_backward(g, x, w, t, lse, dx=dx, dw=dw, workspace=on(0, 64), stream=0, loss=loss)
    gradient(None)
    before = loss._version
    gradient(loss)
    (plain, a), (name, b) = library
    assert (plain, name) == ("mdet_xent_backward", "mdet_xent_backward_with_loss")
    # the same operands in the same order, and the losses behind lse (but for the workspaces, each call's own)
    assert a[14] == lse.data_ptr() and b[15] == loss.data_ptr() and a[:15] == b[:15] and a[15:-3] == b[16:-3] and loss._version == before
    for bad in (on(1, 4), on(-1, 4), on(0, 5), on(0, 4, 1), on(0, 8)[::2], on(0, 4, dtype=torch.bfloat16), on(0, 4, dtype=torch.float64)):
        with pytest.raises(ValueError, match="loss"):
            gradient(bad)
    assert len(library) == 2


def entry(M, dtype=F32, gt=F32, bits=64, m=4, n=10, k=8, g=A, x=A, ldx=8, w=A, ldw=8, b=None, t=A, ignore=-100, lse=A, loss=A, kept=None, kb=0, dx=A, lddx=8,    # noqa: F811
          dw=A, lddw=8, db=None, ws=A, wsb=1 << 40):
    return M.lib().mdet_xent_backward_with_loss(dtype, gt, bits, m, n, k, g, x, ldx, w, ldw, b, t, ignore, lse, loss, kept, kb, dx, lddx, dw, lddw, db, ws, wsb,
                                                None)


@pytest.mark.parametrize("bad", [dict(loss=A + 2), dict(loss=A + 1), dict(lse=None), dict(g=None), dict(dtype=F64), dict(dtype=F16, gt=BF16), dict(bits=1), dict(m=-1),
                                 dict(x=None), dict(w=None), dict(t=None), dict(ldx=7), dict(lddw=7), dict(dx=A + 2), dict(db=A + 2), dict(ws=None),
                                 dict(kept=A + 64, kb=1 << 30)])
def test_refusals(M, bad):                                                        # noqa: F811
    assert entry(M, **bad) == EINVAL


def test_workspaces_and_nothing_to_do(M):                                         # noqa: F811
    need = M.mdet_xent_workspace_query(F32, 4, 10, 8, True)
    assert entry(M, wsb=need - 1) == ENOMEM and entry(M, kept=A, kb=8) == ENOMEM
    assert entry(M, dx=None, dw=None) == 0 and entry(M, dx=None, dw=None, loss=None) == 0
