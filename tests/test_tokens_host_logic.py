"""CPU-only checks of the token operators' C ABI (embedding, layer norm, cross entropy): refusals, workspace figures, how products are
cut.  No GPU call is made: every call here is refused or has nothing to do."""
import ctypes as C
import os

import pytest

OK, EINVAL, ENOMEM = 0, 1, 3
F32, F64, F16, BF16 = 0, 1, 2, 3
A = 4096                      # an address that nothing is read from


@pytest.fixture(scope="module")
def M():
    import paper_2503_04424_amd as m
    if not os.path.exists(m.lib_path()):
        from paper_2503_04424_amd import build
        build.build()
    m.load()
    return m


def embed(M, dtype=F32, bits=64, n=4, vocab=10, width=8, ids=A, table=A, ldt=8, scale=1.0, y=A, ldy=8):
    return M.lib().mdet_embedding_forward(dtype, bits, n, vocab, width, ids, table, ldt, scale, y, ldy, None)


def embed_grad(M, dtype=F32, gt=F32, bits=64, n=4, vocab=10, width=8, ids=A, dy=A, lddy=8, scale=1.0, add=0, g=A, ldt=8, ws=A, wsb=1 << 30):
    return M.lib().mdet_embedding_backward(dtype, gt, bits, n, vocab, width, ids, dy, lddy, scale, add, g, ldt, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(dtype=F64), dict(dtype=7), dict(bits=16), dict(bits=0), dict(n=-1), dict(n=1 << 31), dict(vocab=-1), dict(vocab=1 << 31),
                                 dict(width=-1), dict(ids=None), dict(ids=A + 4), dict(table=None), dict(table=A + 2), dict(ldt=7), dict(ldy=7), dict(y=None),
                                 dict(y=A + 1), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e39), dict(n=1 << 30, width=1 << 30)])
def test_embedding_refuses(M, bad):
    assert embed(M, **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(dtype=F64), dict(gt=BF16), dict(dtype=F16, gt=BF16), dict(bits=8), dict(n=(1 << 31) - 1), dict(vocab=1 << 31), dict(ids=None),
                                 dict(ids=A + 4), dict(dy=None), dict(lddy=7), dict(dy=A + 2), dict(g=None), dict(ldt=7), dict(g=A + 2), dict(scale=-1e39),
                                 dict(ws=None), dict(ws=A + 128)])
def test_embedding_gradient_refuses(M, bad):
    assert embed_grad(M, **bad) == EINVAL


def test_embedding_workspace(M):
    need = M.mdet_embedding_workspace_query(100, 1000, 64)
  # sorted places and ids, starts and counts, parts of thirteen runs
    assert need % 256 == 0 and need >= 2 * 100 * 4 + 2 * 1000 * 4 + 13 * 2 * 64 * 4
    assert embed_grad(M, n=100, vocab=1000, width=64, lddy=64, ldt=64, wsb=need - 1) == ENOMEM
    assert embed(M, n=0, ids=None, y=None) == OK and embed(M, width=0, table=None, y=None) == OK
    assert embed_grad(M, n=0, ids=None, dy=None, add=1) == OK and embed_grad(M, vocab=0, g=None) == OK and embed_grad(M, width=0, dy=None, g=None) == OK
    for bad in ((-1, 5, 5), (5, -1, 5), (5, 5, -1), (1 << 31, 5, 5), (5, 1 << 31, 5)):
        with pytest.raises(M.MemdetError):
            M.mdet_embedding_workspace_query(*bad)


def norm(M, dtype=F32, m=4, n=8, x=A, ldx=8, w=None, b=None, eps=1e-5, y=A, ldy=8, mean=None, rstd=None):
    return M.lib().mdet_layernorm_forward(dtype, m, n, x, ldx, w, b, eps, y, ldy, mean, rstd, None)


def norm_grad(M, dtype=F32, gt=F32, m=4, n=8, dy=A, lddy=8, x=A, ldx=8, mean=A, rstd=A, w=None, dx=A, lddx=8, dw=A, db=A, ws=A, wsb=1 << 30):
    return M.lib().mdet_layernorm_backward(dtype, gt, m, n, dy, lddy, x, ldx, mean, rstd, w, dx, lddx, dw, db, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(dtype=F64), dict(m=-1), dict(n=-1), dict(m=1 << 41), dict(n=(1 << 32) + 1, m=1, ldx=1 << 33, ldy=1 << 33), dict(x=None),
                                 dict(y=None), dict(ldx=7), dict(ldy=7), dict(x=A + 2), dict(y=A + 1), dict(w=A + 2), dict(b=A + 1), dict(eps=-1e-9),
                                 dict(eps=float("nan")), dict(eps=float("inf")), dict(eps=1e39), dict(mean=A + 2), dict(rstd=A + 1)])
def test_layernorm_refuses(M, bad):
    assert norm(M, **bad) == EINVAL


@pytest.mark.parametrize("bad", [dict(dtype=F64), dict(gt=BF16), dict(dtype=BF16, gt=F16), dict(m=-1), dict(dy=None), dict(x=None), dict(lddy=7), dict(ldx=7),
                                 dict(lddx=7), dict(mean=None), dict(rstd=None), dict(mean=A + 2), dict(w=A + 2), dict(dw=A + 2), dict(db=A + 1), dict(dx=A + 2),
                                 dict(ws=None), dict(ws=A + 64)])
def test_layernorm_gradient_refuses(M, bad):
    assert norm_grad(M, **bad) == EINVAL


def test_layernorm_workspace(M):
    for dtype in (F32, F16, BF16):
        for m, n in ((1, 1), (4, 8), (777, 1301), (16384, 4096), (5, 100000), (1 << 20, 8), (3, 1 << 32)):
            need = M.mdet_layernorm_workspace_query(dtype, m, n)
            assert need % 256 == 0 and 8 * n <= need <= 8 * n * min(m, 1024) + 256
    need = M.mdet_layernorm_workspace_query(F32, 4, 8)
    assert norm_grad(M, wsb=need - 1) == ENOMEM
    assert norm(M, m=0, x=None, y=None) == OK and norm(M, n=0, x=None, y=None) == OK
    assert norm_grad(M, dx=None, dw=None, db=None, ws=None, wsb=0) == OK and norm_grad(M, n=0, dy=None, x=None, ws=None, wsb=0) == OK
    for bad in ((F64, 1, 1), (F32, -1, 1), (F32, 1, (1 << 32) + 1)):
        with pytest.raises(M.MemdetError):
            M.mdet_layernorm_workspace_query(*bad)


def xent(M, dtype=F32, bits=64, m=4, n=10, k=8, x=A, ldx=8, w=A, ldw=8, b=None, t=A, ignore=-100, loss=A, lse=A, kept=None, kb=0, ws=A, wsb=1 << 30):
    return M.lib().mdet_xent_forward(dtype, bits, m, n, k, x, ldx, w, ldw, b, t, ignore, loss, lse, kept, kb, ws, wsb, None)


def xent_grad(M, dtype=F32, gt=F32, bits=64, m=4, n=10, k=8, g=A, x=A, ldx=8, w=A, ldw=8, b=None, t=A, ignore=-100, lse=A, kept=None, kb=0, dx=A, lddx=8,
              dw=A, lddw=8, db=None, ws=A, wsb=1 << 40):
    return M.lib().mdet_xent_backward(dtype, gt, bits, m, n, k, g, x, ldx, w, ldw, b, t, ignore, lse, kept, kb, dx, lddx, dw, lddw, db, ws, wsb, None)


def reduce(M, bits=64, m=4, n=10, loss=A, t=A, mean=1, out=A, weights=A):
    return M.lib().mdet_xent_reduce(bits, m, n, loss, t, -100, mean, out, weights, None)


@pytest.mark.parametrize("bad", [dict(bits=8), dict(m=-1), dict(n=-1), dict(m=1 << 41), dict(loss=None), dict(loss=A + 2), dict(t=None), dict(t=A + 4),
                                 dict(out=None), dict(out=A + 1), dict(weights=A + 2)])
def test_reduction_refuses(M, bad):
    assert reduce(M, **bad) == EINVAL


SIZES = [dict(m=-1), dict(n=-1), dict(k=-1), dict(m=1 << 41), dict(m=(1 << 31) - 32, n=64), dict(n=(1 << 31) - 32, k=64, ldx=64, ldw=64)]


@pytest.mark.parametrize("bad", SIZES + [dict(dtype=F64), dict(bits=16), dict(x=None), dict(w=None), dict(t=None), dict(t=A + 4), dict(ldx=7), dict(ldw=7), dict(x=A + 2),
                                         dict(w=A + 1), dict(b=A + 2), dict(loss=A + 2), dict(lse=A + 1), dict(ws=None), dict(ws=A + 8), dict(kept=A + 8, kb=1 << 30)])
def test_cross_entropy_refuses(M, bad):
    assert xent(M, **bad) == EINVAL


@pytest.mark.parametrize("bad", SIZES + [dict(dtype=F64), dict(gt=BF16), dict(dtype=F16, gt=BF16), dict(bits=1), dict(g=None), dict(g=A + 2), dict(lse=None), dict(x=None),
                                         dict(w=None), dict(t=None), dict(t=A + 4), dict(ldx=7), dict(ldw=7), dict(lddx=7), dict(lddw=7), dict(dx=A + 2),
                                         dict(dw=A + 2), dict(db=A + 2), dict(b=A + 2), dict(ws=None), dict(ws=A + 8), dict(kept=A + 64, kb=1 << 30)])
def test_cross_entropy_gradient_refuses(M, bad):
    assert xent_grad(M, **bad) == EINVAL


def test_cross_entropy_workspace(M):
    for dtype, size in ((F32, 4), (F16, 2), (BF16, 2)):
        for m, n, k in ((1, 1, 1), (4, 10, 8), (40, 1000, 33), (300, 50003, 64), (8192, 131072, 4096), (1 << 18, 1 << 17, 64), (1, 1 << 30, 1)):
            forward, kept, back = (M.mdet_xent_workspace_query(dtype, m, n, k), M.mdet_xent_kept_query(dtype, m, n, k),
                                   M.mdet_xent_workspace_query(dtype, m, n, k, True))
            assert all(v % 256 == 0 for v in (forward, kept, back))
            # of 16 words or more a strip: a float pair; each row: a float
            assert forward <= m * ((n + 15) // 16) * 8 + m * 4 + 512
            each = 2 if dtype == BF16 else 4
            assert m * n * each + forward <= kept <= m * (n + (7 if n < 1024 else 63)) * each + forward + 256
            # never the whole of e: 2^29 elements, or a few thousand words, with their column sums; x; dx and parts in fp32
            piece = min(n, max((1 << 29) // m, 4096))
            assert back <= m * (piece + 264) * size * 1.2 + (m // 16 + 32) * (piece + 256) * 4 + m * (k + 8) * (size + 4) + 4 * 256 * 65536 * 2 + 4096
    need = M.mdet_xent_workspace_query(F32, 4, 10, 8)
    assert xent(M, wsb=need - 1) == ENOMEM and xent(M, kept=A, kb=M.mdet_xent_kept_query(F32, 4, 10, 8) - 1) == ENOMEM
    need = M.mdet_xent_workspace_query(F32, 4, 10, 8, True)
    assert xent_grad(M, wsb=need - 1) == ENOMEM and xent_grad(M, kept=A, kb=8) == ENOMEM
    assert xent(M, m=0, x=None, t=None) == OK and xent(M, loss=None, lse=None) == OK
    assert xent_grad(M, dx=None, dw=None) == OK
    # of 16-bit operands, 32 bits of dw take e in two or three parts
    for dtype, parts in ((F16, 2), (BF16, 3)):
        one, more = (M.mdet_xent_workspace_query(dtype, 1000, 5000, 64, True, g) for g in (dtype, F32))
        assert more - one >= (parts - 1) * 1000 * 5000 * 2
    assert M.mdet_xent_workspace_query(F32, 1000, 5000, 64, True, F32) == M.mdet_xent_workspace_query(F32, 1000, 5000, 64, True)
    with pytest.raises(M.MemdetError):
        M.mdet_xent_workspace_query(F16, 1, 1, 1, True, BF16)
    for bad in ((F64, 1, 1, 1), (F32, -1, 1, 1), (F32, 1 << 31, 64, 1)):
        for query in (M.mdet_xent_workspace_query, M.mdet_xent_kept_query):
            with pytest.raises(M.MemdetError):
                query(*bad)


def test_empty_axes_come_back(M):
    """Sizes of zero beside large ones, in a process of their own: a division by zero would end it."""
    import subprocess
    import sys
    code = f"""
import ctypes as C
import paper_2503_04424_amd as M
L, A = M.load(), {A}
for dtype in ({F32}, {F16}, {BF16}):
    for m, n, k in ((0, 0, 0), (0, 50000, 512), (1000, 0, 64), (1000, 50000, 0), (0, 0, 100000), (17, 0, 0), (0, 1000, 0)):
        assert all(f(dtype, m, n, k) >= 0 for f in (M.mdet_xent_workspace_query, M.mdet_xent_kept_query, lambda *a: M.mdet_xent_workspace_query(*a, True)))
        assert M.mdet_embedding_workspace_query(m, n, k) >= 0 and M.mdet_layernorm_workspace_query(dtype, m, n) >= 0
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])


def test_how_products_are_cut(M, tmp_path):
    """The header by itself: every tile is covered once, parts of a sum cover it without gaps, workspaces hold what the launches write."""
    import shutil
    import subprocess
    compiler = shutil.which("g++") or shutil.which("c++")
    if not compiler:
        pytest.skip("no compiler")
    here = os.path.dirname(os.path.abspath(__file__))
    out = tmp_path / "check"
    subprocess.run([compiler, "-std=c++17", "-O2", "-o", str(out), os.path.join(here, "host", "xent_cut_check.cpp")], check=True, capture_output=True, timeout=300)
    done = subprocess.run([str(out)], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout[-500:]
