"""CPU-only checks of what the token operators' calls accept as operands: tensors that say they are on a GPU, and a library that only notes
what it is asked to do."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M
from test_training_operands import OnGpu, on

B = M.binding
QUERIES = ["mdet_embedding_workspace_query", "mdet_layernorm_workspace_query", "mdet_xent_workspace_query", "mdet_xent_kept_query"]


@pytest.fixture
def library(monkeypatch):
    """Names of the entry points that were called to queue work, with their arguments."""
    called = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                called.append((name, args))
                return M.Status.OK
            return entry
    monkeypatch.setattr(B, "load", lambda: Library())
    for query in QUERIES:
        monkeypatch.setattr(B, query, lambda *a, **k: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_one_gpu", False)
    monkeypatch.setattr(B, "_new", lambda stream, make: make())
    return called


F, I = torch.float32, torch.int64


def embed(gpus=(0,) * 3):
    ids, table, y = on(gpus[0], 4, dtype=I), on(gpus[1], 10, 8), on(gpus[2], 4, 8)
    return M.mdet_embedding_forward(ids, table, out=y, stream=0)


def embed_grad(gpus=(0,) * 3, ws=None):
    dy, ids, g = on(gpus[0], 4, 8), on(gpus[1], 4, dtype=I), on(gpus[2], 10, 8)
    return M.mdet_embedding_backward(dy, ids, 10, dtable=g, workspace=ws, stream=0)


def norm(gpus=(0,) * 6):
    x, w, b, y, mean, rstd = (on(g, *s) for g, s in zip(gpus, ((4, 8), (8,), (8,), (4, 8), (4,), (4,))))
    return M.mdet_layernorm_forward(x, w, b, out=y, mean=mean, rstd=rstd, stream=0)


def norm_grad(gpus=(0,) * 8, ws=None):
    dy, x, mean, rstd, w, dx, dw, db = (on(g, *s) for g, s in zip(gpus, ((4, 8), (4, 8), (4,), (4,), (8,), (4, 8), (8,), (8,))))
    return M.mdet_layernorm_backward(dy, x, mean, rstd, w, dx, dw, db, workspace=ws, stream=0)


def xent(gpus=(0,) * 7, ws=None):
    x, w, t, b, loss, lse, kept = (on(g, *s, dtype=d) for g, s, d in zip(gpus, ((4, 8), (10, 8), (4,), (10,), (4,), (4,), (4096,)), (F, F, I, F, F, F, torch.uint8)))
    return M.mdet_xent_forward(x, w, t, b, loss=loss, lse=lse, keep=kept, workspace=ws, stream=0)


def reduce(gpus=(0,) * 4):
    loss, t, out, weights = (on(g, *s, dtype=d) for g, s, d in zip(gpus, ((4,), (4,), (1,), (4,)), (F, I, F, F)))
    return M.mdet_xent_reduce(loss, t, 10, out=out, weights=weights, stream=0)


def xent_grad(gpus=(0,) * 10, ws=None):
    shapes = ((4,), (4, 8), (10, 8), (4,), (4,), (10,), (4096,), (4, 8), (10, 8), (10,))
    types = (F, F, F, I, F, F, torch.uint8, F, F, F)
    g, x, w, t, lse, b, kept, dx, dw, db = (on(v, *s, dtype=d) for v, s, d in zip(gpus, shapes, types))
    return M.mdet_xent_backward(g, x, w, t, lse, b, kept=kept, dx=dx, dw=dw, db=db, workspace=ws, stream=0)


CALLS = {"mdet_embedding_forward": (embed, 3), "mdet_embedding_backward": (embed_grad, 3), "mdet_layernorm_forward": (norm, 6),
         "mdet_layernorm_backward": (norm_grad, 8), "mdet_xent_forward": (xent, 7), "mdet_xent_reduce": (reduce, 4), "mdet_xent_backward": (xent_grad, 10)}
WITH_ROOM = [n for n in CALLS if n.endswith("_backward") or n == "mdet_xent_forward"]


@pytest.mark.parametrize("name", CALLS)
def test_operands_are_on_one_gpu(library, name):
    """Each operand by itself on another GPU, or in host memory, is refused before anything is queued."""
    call, count = CALLS[name]
    call()
    assert [n for n, _ in library] == [name]
    for i in range(count):
        for other in (1, -1):
            with pytest.raises(ValueError):
                call(tuple(other if j == i else 0 for j in range(count)))
    assert len(library) == 1


@pytest.mark.parametrize("name", WITH_ROOM)
def test_a_workspace_is_device_memory_of_its_own_size(library, name):
    call, _ = CALLS[name]
    call(ws=on(0, 4096, dtype=torch.uint8))
    assert [n for n, _ in library] == [name] and library[0][1][-2] == 4096          # its bytes, in front of the stream
    one = torch.zeros(1, dtype=torch.uint8).expand(1 << 20).as_subclass(OnGpu)      # a byte that says it is a million
    every_other = torch.zeros(8192, dtype=torch.uint8)[::2].as_subclass(OnGpu)
    for bad in (torch.zeros(4096, dtype=torch.uint8), one, every_other, on(1, 4096, dtype=torch.uint8)):
        with pytest.raises(ValueError, match="workspace"):
            call(ws=bad)
    assert len(library) == 1


@pytest.mark.parametrize("name", CALLS)
def test_the_operands_gpu_is_the_current_one_of_the_call(library, monkeypatch, name):
    current, at = [0], []

    class Guard:
        def __init__(self, gpu):
            self.gpu = gpu

        def __enter__(self):
            self.before, current[0] = current[0], self.gpu

        def __exit__(self, *_):
            current[0] = self.before
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch.cuda, "device", Guard)
    noted = B.load()

    class Library:
        def __getattr__(self, entry):
            def run(*args):
                at.append((entry, current[0]))
                return getattr(noted, entry)(*args)
            return run
    monkeypatch.setattr(B, "load", lambda: Library())
    call, count = CALLS[name]
    for gpu in (0, 3):
        call((gpu,) * count)
    assert [g for entry, g in at if entry == name] == [0, 3] and current == [0]


def test_what_a_call_writes_counts_as_changed(library):
    """Tensors of the caller's that are written through their addresses: their autograd version goes up; those read, not."""
    x, w, b, t, y = on(0, 4, 8), on(0, 8), on(0, 8), on(0, 4, dtype=I), on(0, 4, 8)
    table, bias, dw, db, kept = on(0, 10, 8), on(0, 10), on(0, 10, 8), on(0, 10), on(0, 4096, dtype=torch.uint8)
    m, r, nw, nb = on(0, 4), on(0, 4), on(0, 8), on(0, 8)
    every = dict(x=x, w=w, b=b, t=t, y=y, table=table, bias=bias, dw=dw, db=db, kept=kept, m=m, r=r, nw=nw, nb=nb)

    def changed(call):
        before = {name: v._version for name, v in every.items()}
        call()
        return {name for name, v in every.items() if v._version != before[name]}
    assert changed(lambda: M.mdet_embedding_forward(t, table, out=y, stream=0)) == {"y"}
    assert changed(lambda: M.mdet_embedding_backward(x, t, 10, dtable=dw, stream=0)) == {"dw"}
    assert changed(lambda: M.mdet_embedding_backward(x, t, 10, dtable=dw, accumulate=True, stream=0)) == {"dw"}
    assert changed(lambda: M.mdet_layernorm_forward(x, w, b, out=y, mean=m, rstd=r, stream=0)) == {"y", "m", "r"}
    assert changed(lambda: M.mdet_layernorm_forward(x, w, b, out=y, mean=False, rstd=None, stream=0)) == {"y"}
    assert changed(lambda: M.mdet_layernorm_backward(x, x, m, r, w, y, nw, nb, stream=0)) == {"y", "nw", "nb"}
    assert changed(lambda: M.mdet_xent_forward(x, table, t, bias, loss=m, lse=r, keep=kept, stream=0)) == {"m", "r", "kept"}
    assert changed(lambda: M.mdet_xent_reduce(m, t, 10, out=r[:1], weights=r, stream=0)) == {"r"}
    assert changed(lambda: M.mdet_xent_reduce(m, t, 10, weights=r, stream=0)) == {"r"}
    assert changed(lambda: M.mdet_xent_backward(m, x, table, t, r, bias, kept=kept, dx=y, dw=dw, db=db, stream=0)) == {"y", "dw", "db"}
    assert changed(lambda: M.mdet_xent_backward(m, x, table, t, r, bias, dx=False, dw=dw, stream=0)) == {"dw"}


def test_what_is_refused(library):
    """Shapes, types and places that do not fit: an error before anything is queued."""
    x, w, b, t = on(0, 4, 8), on(0, 8), on(0, 8), on(0, 4, dtype=I)
    table, m, half = on(0, 10, 8), on(0, 4), on(0, 4, 8, dtype=torch.bfloat16)
    calls = [lambda: M.mdet_embedding_forward(t.view(2, 2), table, stream=0), lambda: M.mdet_embedding_forward(t.float(), table, stream=0),
             lambda: M.mdet_embedding_forward(on(0, 4, dtype=torch.int16), table, stream=0), lambda: M.mdet_embedding_forward(on(0, 8, dtype=I)[::2], table, stream=0),
             lambda: M.mdet_embedding_forward(t, on(0, 10, 8, dtype=torch.float64), stream=0), lambda: M.mdet_embedding_forward(t, table.t(), stream=0),
             lambda: M.mdet_embedding_forward(t, table, out=on(0, 4, 7), stream=0), lambda: M.mdet_embedding_forward(t, table, out=half, stream=0),
             lambda: M.mdet_embedding_backward(x, on(0, 5, dtype=I), 10, stream=0), lambda: M.mdet_embedding_backward(x, t, 10, accumulate=True, stream=0),
             lambda: M.mdet_embedding_backward(x, t, -1, stream=0), lambda: M.mdet_embedding_backward(x, t, 9, dtable=table, stream=0),
             lambda: M.mdet_embedding_backward(x, t, 10, dtable=table, grad_dtype=torch.bfloat16, stream=0),
             lambda: M.mdet_layernorm_forward(w, stream=0), lambda: M.mdet_layernorm_forward(x, on(0, 7), stream=0), lambda: M.mdet_layernorm_forward(x, w, on(0, 9), stream=0),
             lambda: M.mdet_layernorm_forward(half, w, stream=0), lambda: M.mdet_layernorm_forward(x.t(), stream=0), lambda: M.mdet_layernorm_forward(x, mean=on(0, 5), stream=0),
             lambda: M.mdet_layernorm_forward(x, rstd=on(0, 4, dtype=torch.bfloat16), stream=0), lambda: M.mdet_layernorm_backward(half, x, m, m, w, stream=0),
             lambda: M.mdet_layernorm_backward(x, x, on(0, 3), m, w, stream=0), lambda: M.mdet_layernorm_backward(x, x, m, m, w, dw=on(0, 8, dtype=torch.bfloat16), stream=0),
             lambda: M.mdet_layernorm_backward(x, x, m, on(0, 8)[::2], w, stream=0),
             lambda: M.mdet_xent_forward(x, table, on(0, 5, dtype=I), stream=0), lambda: M.mdet_xent_forward(x, on(0, 10, 7), t, stream=0),
             lambda: M.mdet_xent_forward(half, table, t, stream=0), lambda: M.mdet_xent_forward(x, table, t, on(0, 9), stream=0), lambda: M.mdet_xent_forward(x, table, x, stream=0),
             lambda: M.mdet_xent_forward(x, table, t, loss=on(0, 5), stream=0), lambda: M.mdet_xent_forward(x, table, t, keep=torch.zeros(8), stream=0),
             lambda: M.mdet_xent_forward(x.double(), table.double(), t, stream=0), lambda: M.mdet_xent_backward(t, x, table, t, m, stream=0),
             lambda: M.mdet_xent_backward(m, x, table, t, on(0, 4, dtype=torch.bfloat16), stream=0), lambda: M.mdet_xent_backward(m, x, table, t, m, dx=on(0, 8, 4).t(), stream=0),
             lambda: M.mdet_xent_backward(m, x, table, t, m, db=on(0, 10, dtype=torch.bfloat16), stream=0), lambda: M.mdet_xent_reduce(x, t, 10, stream=0),
             lambda: M.mdet_xent_reduce(m, m, 10, stream=0), lambda: M.mdet_xent_reduce(m, t[:3], 10, stream=0), lambda: M.mdet_xent_reduce(m, t, 10, out=None, stream=0),
             lambda: M.mdet_xent_reduce(m, t, 10, out=on(0, 4), stream=0), lambda: M.mdet_xent_reduce(m, t, 10, weights=on(0, 5), stream=0)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    assert not library
