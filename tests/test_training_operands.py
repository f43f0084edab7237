"""CPU-only checks of what the training operators' calls accept as operands: tensors that say they are on a GPU, and a library that
only notes what it is asked to do."""
import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M

B = M.binding


class OnGpu(torch.Tensor):
    """A tensor in host memory that says it is on GPU number `gpu`."""
    gpu = 0
    is_cuda = property(lambda self: self.gpu >= 0)
    device = property(lambda self: torch.device("cuda", self.gpu) if self.gpu >= 0 else torch.device("cpu"))

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        if func is torch.Tensor.get_device:
            return args[0].gpu
        return super().__torch_function__(func, types, args, kwargs or {})


def on(gpu, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)
    t.gpu = gpu
    return t


@pytest.fixture
def library(monkeypatch):
    """Names of the entry points that were called to queue work."""
    called = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                if not name.endswith("_query"):
                    called.append(name)
                return M.Status.OK
            return entry
    monkeypatch.setattr(B, "load", lambda: Library())
    monkeypatch.setattr(B, "mdet_linear_workspace_query", lambda *a, **k: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(B, "_one_gpu", False)           # several, wherever this runs
    return called


def layer(gpus=(0,) * 6, ws=None):
    x, w, b, r, y, z = (on(g, *s) for g, s in zip(gpus, ((4, 16), (8, 16), (8,), (4, 8), (4, 8), (4, 8))))
    return M.mdet_linear_forward(x, w, b, r, "gelu", out=y, preact=z, workspace=ws, stream=0)


def gradient(gpus=(0,) * 8, ws=None):
    dy, x, w, z, dx, dw, db, dz = (on(g, *s) for g, s in zip(gpus, ((4, 8), (4, 16), (8, 16), (4, 8), (4, 16), (8, 16), (8,), (4, 8))))
    return M.mdet_linear_backward(dy, x, w, z, "gelu", dx, dw, db, dz=dz, workspace=ws, stream=0)


def gram(gpus=(0,) * 5, ws=None):
    a, g, a2, g2, k = (on(v, *s) for v, s in zip(gpus, ((4, 8), (4, 5), (4, 5), (4, 1), (4, 4))))
    return M.mdet_ntk_gram([a, a2], [g, g2], k, workspace=ws, stream=0)


CALLS = {"mdet_linear_forward": layer, "mdet_linear_backward": gradient, "mdet_ntk_gram": gram}


@pytest.mark.parametrize("name", CALLS)
def test_a_workspace_is_device_memory_of_its_own_size(library, name):
    CALLS[name](ws=on(0, 4096, dtype=torch.uint8))
    assert library == [name]
    one = torch.zeros(1, dtype=torch.uint8).expand(1 << 20).as_subclass(OnGpu)      # a byte that says it is a million
    every_other = torch.zeros(8192, dtype=torch.uint8)[::2].as_subclass(OnGpu)
    for bad in (torch.zeros(4096, dtype=torch.uint8), one, every_other):
        with pytest.raises(ValueError, match="workspace"):
            CALLS[name](ws=bad)
    assert library == [name]


def step(gpus=(0,) * 7, count=2):
    kinds = [torch.float32, torch.float32, torch.int8, torch.uint8, None, torch.bfloat16]
    lists = [[on(g, 300, dtype=t) for _ in range(count)] if t else [on(g, 2, 2) for _ in range(count)] for g, t in zip(gpus, kinds)]
    p, g, m, v, sc, co = lists
    M.mdet_adamw_step(p, g, m, v, lr=1e-3, step=1, scales=sc, copies=co, grad_scale=on(gpus[6], 1), stream=0)


@pytest.mark.parametrize("name,count", [("mdet_linear_forward", 6), ("mdet_linear_backward", 8), ("mdet_ntk_gram", 5), ("mdet_adamw_step", 7)])
def test_operands_are_on_one_gpu(library, name, count):
    """A kernel runs on one: each operand by itself on another, or in host memory, is refused before anything is queued."""
    call = {**CALLS, "mdet_adamw_step": step}[name]
    call((0,) * count)
    assert library == [name]
    for i in range(count):
        for other in (1, -1):
            with pytest.raises(ValueError):
                call(tuple(other if j == i else 0 for j in range(count)))
    if name in CALLS:
        with pytest.raises(ValueError):
            call(ws=on(1, 4096, dtype=torch.uint8))
    assert library == [name]


def test_one_tensor_of_a_list_on_another_gpu_is_refused(library):
    lists = [[on(0, 8), on(0, 8)] for _ in range(4)]
    for tensors in lists:
        tensors[1].gpu = 1
        with pytest.raises(ValueError):
            M.mdet_adamw_step(*lists, lr=1e-3, step=1, stream=0)
        tensors[1].gpu = 0
    assert not library


@pytest.mark.parametrize("name,count", [("mdet_linear_forward", 6), ("mdet_linear_backward", 8), ("mdet_ntk_gram", 5), ("mdet_adamw_step", 7)])
def test_the_operands_gpu_is_the_current_one_of_the_call(library, monkeypatch, name, count):
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
    call = {**CALLS, "mdet_adamw_step": step}[name]
    for gpu in (0, 3):
        call((gpu,) * count)
    assert [g for entry, g in at if entry == name] == [0, 3] and current == [0]


def test_what_a_call_writes_counts_as_changed(library):
    """Tensors of the caller's that are written through their addresses: their autograd version goes up; those read, not."""
    x, w, b, r, y, z = on(0, 4, 16), on(0, 8, 16), on(0, 8), on(0, 4, 8), on(0, 4, 8), on(0, 4, 8)
    dx, dw, db, dz = on(0, 4, 16), on(0, 8, 16), on(0, 8), on(0, 4, 8)
    p, g, m, v, c = (on(0, 8, dtype=t) for t in (torch.float32, torch.float32, torch.float32, torch.float32, torch.bfloat16))
    k = on(0, 4, 4)
    every = dict(x=x, w=w, b=b, r=r, y=y, z=z, dx=dx, dw=dw, db=db, dz=dz, p=p, g=g, c=c, k=k)

    def changed(call):
        before = {name: t._version for name, t in every.items()}
        call()
        return {name for name, t in every.items() if t._version != before[name]}
    assert changed(lambda: M.mdet_linear_forward(x, w, b, r, "gelu", out=y, preact=z, stream=0)) == {"y", "z"}
    assert changed(lambda: M.mdet_linear_forward(x, w, b, r, out=r, stream=0)) == {"r"}
    assert changed(lambda: M.mdet_linear_backward(y, x, w, z, "gelu", dx, dw, db, dz=dz, stream=0)) == {"dx", "dw", "db", "dz"}
    assert changed(lambda: M.mdet_linear_backward(y, x, w, z, "gelu", False, dw, None, stream=0)) == {"dw"}
    assert changed(lambda: M.mdet_adamw_step([p], [g], [m], [v], lr=1e-3, step=1, copies=[c], stream=0)) == {"p", "c"}
    assert changed(lambda: M.mdet_adamw_step([p.detach()], [g], [m], [v], lr=1e-3, step=2, stream=0)) == {"p"}
    assert changed(lambda: M.mdet_ntk_gram([x], [y], k, stream=0)) == {"k"}

    def refused():
        with pytest.raises(ValueError):
            M.mdet_adamw_step([p], [g[:7]], [m], [v], lr=1e-3, step=3, stream=0)
    assert changed(refused) == set()
