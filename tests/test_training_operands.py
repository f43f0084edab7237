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

    def get_device(self):
        return self.gpu


def on(gpu, *shape, dtype=torch.float32):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)
    t.gpu = gpu
    return t


@pytest.fixture
def library(monkeypatch):
    """Names of the library's entry points that were called."""
    called = []

    class Library:
        def __getattr__(self, name):
            def entry(*args):
                called.append(name)
                return M.Status.OK
            return entry
    monkeypatch.setattr(B, "load", lambda: Library())
    monkeypatch.setattr(B, "mdet_linear_workspace_query", lambda *a, **k: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
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
