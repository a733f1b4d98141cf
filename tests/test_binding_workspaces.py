"""CPU: the scratch memory that the binding takes for a call without one of the caller's.  A stand-in library notes what each call is given; tensors are the CPU's, said to be CUDA's."""
import threading

import pytest
import torch

from paper_2509_25149_amd import binding as nv


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def on_gpu(*size, dtype=torch.bfloat16):
    return torch.zeros(*size, dtype=dtype).as_subclass(OnGpu)


class Library:
    """In place of the real one: the sizes are the real library's, the calls with a workspace run `between` (while the call is under way) and note (address, bytes)."""
    WORKSPACE_AT = dict(nvfp4_quantize=11, nvfp4_amax=7, nvfp4_rmsnorm_backward=17, nvfp4_activation_backward=11)

    def __init__(self, between=lambda: None):
        self.real, self.between, self.given = nv.load_library(), between, []

    def __getattr__(self, name):
        if name not in self.WORKSPACE_AT:
            return getattr(self.real, name)
        at = self.WORKSPACE_AT[name]

        def call(*args):
            self.between()
            self.given.append((args[at], args[at + 1]))
            return 0
        return call


# Both calls of a pair need the same bytes, so that nothing but the sharing decides where they lie.
CALLS = {
    "quantize": lambda rows: nv.nvfp4_quantize(on_gpu(rows, 256), nv.LAYOUT_ROW),
    "amax": lambda rows: nv.nvfp4_amax(on_gpu(rows, 256), out=on_gpu(2, dtype=torch.float32)),
    "rmsnorm_backward": lambda rows: nv.nvfp4_rmsnorm_backward(on_gpu(rows, 2064), on_gpu(rows, 2064), on_gpu(rows, dtype=torch.float32), dgamma=on_gpu(2064, dtype=torch.float32)),
    "activation_backward": lambda rows: nv.nvfp4_activation_backward(on_gpu(rows, 2064), dbias=on_gpu(2064, dtype=torch.float32)),
}


@pytest.fixture
def stand_in(monkeypatch):
    def use(between=lambda: None):
        lib = Library(between)
        monkeypatch.setattr(nv, "load_library", lambda: lib)
        return lib
    monkeypatch.setattr(nv, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return use


def disjoint(a, b):
    return a[0] + a[1] <= b[0] or b[0] + b[1] <= a[0]


@pytest.mark.parametrize("second", list(CALLS))
@pytest.mark.parametrize("first", list(CALLS))
def test_two_threads_on_one_stream_do_not_share_a_workspace(stand_in, first, second):
    """The second thread's call goes through whole while the first one's launches are half enqueued: what the first has in its workspace then has to stay."""
    at_work = threading.local()

    def between():
        if getattr(at_work, "is_first", False):
            at_work.is_first = False
            other = threading.Thread(target=CALLS[second], args=(512,))
            other.start()
            other.join()
    lib = stand_in(between)
    at_work.is_first = True
    CALLS[first](512)
    assert len(lib.given) == 2 and all(p and n for p, n in lib.given)
    assert disjoint(*lib.given)


@pytest.mark.parametrize("name", list(CALLS))
def test_a_captured_call_has_a_workspace_of_its_own(stand_in, monkeypatch, name):
    """A graph keeps the address.  So it must not be one that a later call is given, nor one that is freed when a later call needs more."""
    alive, empty = [], torch.empty                      # (kept alive here: addresses that are freed could be given out again)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: alive.append(empty(*a, **k)) or alive[-1])
    lib, capturing = stand_in(), [False]
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    CALLS[name](512)
    capturing[0] = True
    CALLS[name](512)
    CALLS[name](512)
    capturing[0] = False
    CALLS[name](512)
    CALLS[name](2048)
    before, captured, captured_too, after, larger = lib.given
    assert before == after                              # (one buffer as long as it is large enough)
    for graph in (captured, captured_too):
        for other in (before, after, larger):
            assert disjoint(graph, other)
    assert disjoint(captured, captured_too)
