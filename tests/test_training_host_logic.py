"""CPU-only checks of the training operators' C ABI: refusals, workspace figures, structs.  No GPU call is made: every call
here is refused or has nothing to do."""
import ctypes as C
import os

import pytest

EINVAL, ENOMEM = 1, 3
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


def forward(M, dtype=F32, act=0, m=4, n=8, k=16, x=A, ldx=16, w=A, ldw=16, bias=None, r=None, ldr=0, y=A, ldy=8, z=None, ldz=0, ws=None, wsb=0):
    return M.lib().mdet_linear_forward(dtype, act, m, n, k, x, ldx, w, ldw, bias, r, ldr, y, ldy, z, ldz, ws, wsb, None)


def backward(M, dtype=F32, gt=F32, act=0, m=4, n=8, k=16, dy=A, lddy=8, z=None, ldz=0, x=A, ldx=16, w=A, ldw=16, dx=A, lddx=16, dw=A, lddw=16,
             db=None, dz=None, lddz=0, ws=None, wsb=0):
    return M.lib().mdet_linear_backward(dtype, gt, act, m, n, k, dy, lddy, z, ldz, x, ldx, w, ldw, dx, lddx, dw, lddw, db, dz, lddz, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(dtype=F64), dict(dtype=7), dict(act=5), dict(act=-1), dict(m=-1), dict(k=-1), dict(m=1 << 41), dict(x=None),
                                 dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=15), dict(ldy=7), dict(x=A + 2), dict(y=A + 1), dict(bias=A + 2),
                                 dict(r=A, ldr=7), dict(z=A, ldz=7), dict(z=A + 3, ldz=8), dict(m=1 << 30, n=1 << 30, ldy=1 << 30)])
def test_forward_refuses(M, bad):
    assert forward(M, **bad) == EINVAL


def test_forward_workspace(M):
    # a sum over a long axis for few tiles is split: its parts need a place, on 256 bytes
    need = M.mdet_linear_workspace_query(F32, 64, 64, 8192)
    assert need > 0 and need % 256 == 0
    call = dict(m=64, n=64, k=8192, ldx=8192, ldw=8192, ldy=64)
    assert forward(M, **call) == EINVAL
    assert forward(M, ws=A + 8, wsb=need, **call) == EINVAL
    assert forward(M, ws=A, wsb=need - 1, **call) == ENOMEM
    assert forward(M, m=0) == 0 and forward(M, n=0, ldy=0) == 0


@pytest.mark.parametrize("bad", [dict(gt=BF16), dict(dtype=F16, gt=BF16), dict(act=1), dict(act=1, z=A, ldz=7), dict(lddx=15), dict(lddw=15),
                                 dict(dw=A + 2), dict(db=A + 2), dict(dz=A, lddz=7), dict(dy=None), dict(ldx=3), dict(w=None), dict(ws=None),
                                 dict(ws=A + 128, wsb=1 << 30)])
def test_backward_refuses(M, bad):
    assert backward(M, **{"ws": A, "wsb": 1 << 30, **bad}) == EINVAL


def test_backward_workspace(M):
    need = M.mdet_linear_workspace_query(F32, 4, 8, 16, backward=True)
    assert need > 0 and backward(M, ws=A, wsb=need - 1) == ENOMEM
    assert backward(M, m=0, n=0, k=0, ws=A, wsb=1 << 20) == 0
    with pytest.raises(M.MemdetError):
        M.mdet_linear_workspace_query(F64, 1, 1, 1)
    with pytest.raises(M.MemdetError):
        M.mdet_linear_workspace_query(F32, -1, 1, 1)
    # dz (bf16 rows of whole pieces), column sums of strips of 16 rows
    assert M.mdet_linear_workspace_query(BF16, 100, 100, 50, backward=True) >= 100 * 104 * 2 + 7 * 100 * 4


def adamw(M, tensors=None, count=1, **fields):
    p = M.binding._AdamwParams()
    p.struct_size = C.sizeof(p)
    values = dict(dtype=F32, grad_dtype=F32, state_bits=32, copy_dtype=-1, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0)
    for k, v in {**values, **fields}.items():
        setattr(p, k, v)
    table = (C.c_uint64 * 7)(*(tensors or [A, A, A, A, 0, 0, 8]))
    return M.lib().mdet_adamw_step(C.byref(p), C.cast(table, C.c_void_p), count, None)


@pytest.mark.parametrize("bad", [dict(struct_size=8), dict(dtype=F64), dict(grad_dtype=F64), dict(state_bits=16), dict(copy_dtype=F32), dict(step=0),
                                 dict(beta1=1.0), dict(beta2=-0.5), dict(beta1=float("nan")), dict(eps=-1.0), dict(lr=float("inf")),
                                 dict(weight_decay=float("nan")), dict(count=-1), dict(state_bits=8), dict(copy_dtype=BF16),
                                 dict(tensors=[A, A, A, A, 0, 0, (1 << 64) - 1]), dict(tensors=[0, A, A, A, 0, 0, 8]), dict(tensors=[A, A, 0, A, 0, 0, 8]),
                                 dict(tensors=[A + 2, A, A, A, 0, 0, 8]), dict(tensors=[A, A + 1, A, A, 0, 0, 8]), dict(tensors=[A, A, A + 2, A, 0, 0, 8])])
def test_adamw_refuses(M, bad):
    assert adamw(M, **bad) == EINVAL


def test_adamw_without_work(M):
    assert adamw(M, count=0) == 0
    assert adamw(M, tensors=[0, 0, 0, 0, 0, 0, 0]) == 0
    assert C.sizeof(M.binding._AdamwParams) == 80 and C.sizeof(M.binding._NtkLayer) == 48


def ntk(M, dtype=F32, out=F32, n=4, d=1, layers=((A, 8, 8, A, 8, 8),), count=None, bias=1.0, scale=1.0, K=A, ldk=4, ws=None, wsb=0):
    table = (M.binding._NtkLayer * max(1, len(layers)))(*[M.binding._NtkLayer(*v) for v in layers])
    return M.lib().mdet_ntk_gram(dtype, out, n, d, C.cast(table, C.c_void_p), len(layers) if count is None else count, bias, scale, 0, K, ldk, ws, wsb, None)


@pytest.mark.parametrize("bad", [dict(dtype=9), dict(out=F16), dict(dtype=F64, out=F32), dict(n=-1), dict(d=0), dict(count=-1), dict(K=None), dict(ldk=3),
                                 dict(K=A + 2), dict(bias=float("inf")), dict(scale=float("nan")), dict(layers=((None, 8, 8, A, 8, 8),)),
                                 dict(layers=((A, 7, 8, A, 8, 8),)), dict(layers=((A, 8, 8, A, 7, 8),)), dict(layers=((A + 2, 8, 8, A, 8, 8),)),
                                 dict(layers=((A, 8, -1, A, 8, 8),)), dict(n=1 << 20, d=1 << 20, ldk=1 << 40), dict(out=F64), dict(d=2, ldk=8)])
def test_ntk_refuses(M, bad):
    assert ntk(M, **bad) == EINVAL


def test_ntk_workspace(M):
    def query(dtype, out, n, d, p, q):
        b = C.c_uint64(0)
        table = (M.binding._NtkLayer * 1)(M.binding._NtkLayer(None, 0, p, None, 0, q))
        assert M.lib().mdet_ntk_workspace_query(dtype, out, n, d, C.cast(table, C.c_void_p), 1, C.byref(b)) == 0
        return b.value
    assert query(F32, F32, 100, 1, 8, 8) == 0
    assert query(F32, F32, 100, 3, 8, 8) >= 100 * 100 * 4                     # first factors
    assert query(BF16, F64, 100, 1, 7, 9) >= 100 * 8 * 8 + 100 * 10 * 8       # operands widened, rows of whole pieces
    assert ntk(M, d=3, ldk=12, ws=A, wsb=16) == ENOMEM
    assert ntk(M, d=3, ldk=12, ws=A + 64, wsb=1 << 20) == EINVAL
    assert ntk(M, n=0) == 0


def test_the_hash_is_even():
    """The rounding's random bits, in numpy: each of the 32 is set half the time, consecutive elements, seeds and the two halves
    are uncorrelated.  2^20 samples: a mean off by 6 standard deviations (0.003) or a correlation of 0.006 fails."""
    import numpy as np

    def bits(key, i):
        h = (i * np.uint32(0x6A09E667) + key).astype(np.uint32)
        h = (h ^ (h >> np.uint32(16))) * np.uint32(0xBB67AE85)
        h = (h ^ (h >> np.uint32(15))) * np.uint32(0x3C6EF373)
        return h ^ (h >> np.uint32(16))
    with np.errstate(over="ignore"):
        i = np.arange(1 << 20, dtype=np.uint32)
        for seed in (0, 1, 12345):
            h = bits(np.uint32(seed), i)
            for b in range(32):
                assert abs(float(((h >> np.uint32(b)) & np.uint32(1)).mean()) - 0.5) < 0.003
            low, high = (h & np.uint32(0xFFFF)) / 65536.0, (h >> np.uint32(16)) / 65536.0
            other = bits(np.uint32(seed + 1), i) & np.uint32(0xFFFF)
            for u, v in ((low, high), (low[:-1], low[1:]), (high[:-1], high[1:]), (low, other / 65536.0)):
                assert abs(float(np.corrcoef(u, v)[0, 1])) < 0.006
            assert abs(float(low.mean()) - 0.5) < 0.002 and abs(float(low.var()) - 1 / 12) < 0.002


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_empty_axes_beside_long_ones(M, dtype):
    """A result without elements is cut into no tiles, however long the sum is that it would have been: figures and calls come
    back (in a process of their own: a division by zero would end it)."""
    import subprocess
    import sys
    code = f"""
import ctypes as C
import paper_2503_04424_amd as M
L, A = M.load(), {A}
for m, n, k in ((0, 512, 512), (0, 9000, 4096), (1000, 64, 0), (1000, 0, 64), (0, 0, 100000), (100000, 0, 0), (0, 1000, 0), (17, 0, 100000)):
    for back in (0, 1):
        b = C.c_uint64(1)
        assert L.mdet_linear_workspace_query({dtype}, back, m, n, k, C.byref(b)) == 0
        assert b.value < (1 << 30)
    if m == 0 or n == 0:
        assert L.mdet_linear_forward({dtype}, 2, m, n, k, A, k, A, k, None, None, 0, A, n, None, 0, A, 1 << 30, None) == 0
assert L.mdet_linear_backward({dtype}, {dtype}, 0, 0, 0, 100000, A, 0, None, 0, A, 100000, A, 100000, A, 100000, A, 100000, A, None, 0, A, 1 << 30, None) == 0
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, (done.returncode, done.stderr[-500:])


def test_products_beyond_a_launch_are_refused(M):
    """A launch holds fewer than 2^32 threads; such a product is refused before anything is queued.  (These rows are single
    elements: 2147483616 of them would be 2^32 threads.)"""
    tall = (1 << 31) - 32
    for m, n in ((tall, 1), (1, tall), (tall, 32), (1 << 18, (1 << 18) + 1)):
        assert forward(M, m=m, n=n, k=1, ldx=1, ldw=1, ldy=n) == EINVAL
    call = dict(n=1, k=1, lddy=1, ldx=1, ldw=1, lddx=1, lddw=1, ws=A, wsb=1 << 62)
    assert backward(M, m=tall, dw=None, **call) == EINVAL
    assert backward(M, **{**call, "m": 1, "n": tall, "lddy": tall, "dx": None}) == EINVAL


def test_factors_beyond_the_arithmetics_type_are_refused(M):
    """Finite in 64 bits, infinite in the 32 that they are used in: every result would be infinite or NaN."""
    for bad in (dict(bias=1e39), dict(scale=-1e200), dict(scale=3.5e38)):
        assert ntk(M, **bad) == EINVAL
    for bad in (dict(lr=1e39), dict(lr=1e38, beta1=0.999), dict(lr=1e30, weight_decay=1e30), dict(eps=1e39)):
        assert adamw(M, **bad) == EINVAL
