"""CPU-only check of the token operators' first calls in a process: at every line of one thread's first call another thread makes its own, which
finds what the binding remembers from the first call on either complete or not begun.  Tensors that say they are on a GPU, and a library that only
notes what it is asked to do."""
import sys
import threading
import types

import pytest

torch = pytest.importorskip("torch")

import paper_2503_04424_amd as M
from test_training_operands import on

F, I = torch.float32, torch.int64
PATH = M.binding.__file__
CODE = compile(open(PATH).read(), PATH, "exec")

CALLS = {
    "embedding_forward": lambda B: B.mdet_embedding_forward(on(0, 4, dtype=I), on(0, 10, 8), stream=0),
    "embedding_backward": lambda B: B.mdet_embedding_backward(on(0, 4, 8), on(0, 4, dtype=I), 10, stream=0),
    "layernorm_forward": lambda B: B.mdet_layernorm_forward(on(0, 4, 8), on(0, 8), stream=0),
    "layernorm_backward": lambda B: B.mdet_layernorm_backward(on(0, 4, 8), on(0, 4, 8), on(0, 4), on(0, 4), stream=0),
    "xent_forward": lambda B: B.mdet_xent_forward(on(0, 4, 8), on(0, 10, 8), on(0, 4, dtype=I), keep=True, stream=0),
    "xent_reduce": lambda B: B.mdet_xent_reduce(on(0, 4), on(0, 4, dtype=I), 10, stream=0),
    "xent_backward": lambda B: B.mdet_xent_backward(on(0, 4), on(0, 4, 8), on(0, 10, 8), on(0, 4, dtype=I), on(0, 4), stream=0),
}


class Library:
    def __getattr__(self, name):
        return lambda *args: M.Status.OK


def process():
    """The binding as a process has it before the first call."""
    B = types.ModuleType("paper_2503_04424_amd.binding")
    B.__file__, B.__package__ = PATH, "paper_2503_04424_amd"
    exec(CODE, B.__dict__)
    B.load = Library
    for name in ("embedding", "layernorm", "xent"):
        setattr(B, f"mdet_{name}_workspace_query", lambda *a, **k: 256)
    B.mdet_xent_kept_query = lambda *a, **k: 256
    B._one_gpu, B._new = True, lambda stream, make: make()
    B._fresh = lambda like, shape, dtype, stream: on(0, shape, dtype=dtype)
    return B


def call_in_a_thread(call, B):
    """What the call raises in a thread of its own."""
    raised = []

    def run():
        try:
            call(B)
        except BaseException as e:
            raised.append(e)
    thread = threading.Thread(target=run)
    thread.start()
    thread.join()
    return raised


def interrupted(first, second, stop):
    """The first call up to its line number `stop` (counted as they are run, in the binding), the second one in another thread, the rest of the first:
    whether there are so many lines, and what the second raised."""
    B, seen, raised = process(), [0], []

    def trace(frame, event, _):
        if frame.f_code.co_filename != PATH:
            return None
        if event == "line":
            seen[0] += 1
            if seen[0] == stop:
                raised.extend(call_in_a_thread(second, B))
        return trace
    before = sys.gettrace()
    sys.settrace(trace)
    try:
        first(B)
    finally:
        sys.settrace(before)
    return seen[0] >= stop, raised


@pytest.mark.parametrize("second", CALLS)
@pytest.mark.parametrize("first", CALLS)
def test_a_second_thread_in_the_middle_of_the_first_call(first, second):
    stop = 1
    while True:
        there, raised = interrupted(CALLS[first], CALLS[second], stop)
        assert not raised, (stop, raised)
        if not there:
            break
        stop += 1
    assert stop > 10
