"""Which GPU the training operators' calls are made on, with torch's device state replaced (CPU only)."""
import contextlib

import pytest
import torch

from paper_2204_08211_amd import binding as B


class OnGpu1(torch.Tensor):
    def get_device(self):
        return 1


class State:
    """GPU 0 is current; the library's calls are recorded with the GPU that is current then and their stream."""

    def __init__(self):
        self.current, self.calls = 0, []

    def _cuda_getDevice(self):
        return self.current

    def _cuda_getCurrentRawStream(self, gpu):
        return 100 + gpu

    @contextlib.contextmanager
    def device(self, gpu):
        before, self.current = self.current, gpu
        yield
        self.current = before

    def _made(self, args, stream):
        self.calls.append((self.current, stream))
        return B.OK

    co3_layernorm = co3_layernorm_backward = _made


class Stream:
    def __init__(self, gpu, handle):
        self.device, self.cuda_stream = torch.device("cuda", gpu), handle


@pytest.fixture
def state(monkeypatch):
    s = State()
    monkeypatch.setattr(B, "_torch_c", s)
    monkeypatch.setattr(B, "lib", lambda: s)
    monkeypatch.setattr(torch.cuda, "device", s.device)
    return s


def calls(stream):
    x = torch.zeros(4, 8).as_subclass(OnGpu1)
    row = torch.zeros(4).as_subclass(OnGpu1)
    grad = torch.zeros(8).as_subclass(OnGpu1)
    ws = torch.zeros(64, dtype=torch.uint8).as_subclass(OnGpu1)
    B.co3_layernorm(x, y=x, mean=row, rstd=row, stream=stream)
    B.co3_layernorm_backward(x, x, None, row, row, dx=x, dweight=grad, workspace=ws, stream=stream)


@pytest.mark.parametrize("handle", [0, 77])   # a GPU's default stream has the handle 0, which by itself means the current GPU's
def test_layernorm_runs_on_the_streams_gpu(state, handle):
    calls(Stream(1, handle))
    assert state.calls == [(1, handle)] * 2 and state.current == 0


def test_layernorm_on_the_current_gpu(state):
    with pytest.raises(ValueError):
        calls(None)
    with pytest.raises(ValueError):
        calls(Stream(0, 0))
    state.current = 1
    calls(None)
    calls(Stream(1, 0))
    assert state.calls == [(1, 101)] * 2 + [(1, 0)] * 2


class Library(State):
    """Takes what it is given, and keeps the argument structures."""

    def __init__(self):
        super().__init__()
        self.current, self.kept = 1, []

    def co3_layernorm_backward(self, args, stream):
        self.kept.append(B.LayernormBackwardArgs.from_buffer_copy(args))
        return B.OK

    def co3_orthogonalize(self, plan, args, stream):
        self.kept.append(B.OrthogonalizeArgs.from_buffer_copy(args))
        return B.OK

    def co3_matrix_plan_destroy(self, plan):
        pass


@pytest.fixture
def library(monkeypatch):
    s = Library()
    monkeypatch.setattr(B, "_torch_c", s)
    monkeypatch.setattr(B, "lib", lambda: s)
    return s


def with_workspace(workspace, status=None):
    x, row, grad = (torch.zeros(*shape).as_subclass(OnGpu1) for shape in ((4, 8), (4,), (8,)))
    B.co3_layernorm_backward(x, x, None, row, row, dx=x, dweight=grad, workspace=workspace)
    plan = B.MatrixPlan.__new__(B.MatrixPlan)
    plan.handle, plan.gpu, plan.dtype, plan.elements, plan.workspace_bytes = 1, 1, torch.float32, 32, 4096
    g = torch.zeros(32).as_subclass(OnGpu1)
    B.co3_orthogonalize(plan, g, g, workspace=workspace, status=status)


def test_a_workspace_counts_its_bytes(library):
    for dtype, size in ((torch.uint8, 1), (torch.float32, 4), (torch.int64, 8)):
        with_workspace(torch.zeros(100, dtype=dtype).as_subclass(OnGpu1))
        assert [a.workspace_bytes for a in library.kept[-2:]] == [100 * size] * 2


def test_memory_that_is_not_there_is_refused(library):
    """A tensor that is expanded, or has gaps, does not have the memory that its elements stand for."""
    ok = torch.zeros(4096, dtype=torch.uint8)
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(4096), ok[::2]):
        with pytest.raises(ValueError):
            with_workspace(bad.as_subclass(OnGpu1))
        plan = B.MatrixPlan.__new__(B.MatrixPlan)
        plan.handle, plan.gpu, plan.dtype, plan.elements, plan.workspace_bytes = 1, 1, torch.float32, 32, 4096
        with pytest.raises(ValueError):
            B.co3_orthogonalize(plan, torch.zeros(32).as_subclass(OnGpu1), workspace=bad.as_subclass(OnGpu1))
    for bad in (torch.zeros(1, dtype=torch.int64).expand(B.STATUS_WORDS), torch.zeros(2 * B.STATUS_WORDS, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            with_workspace(ok.as_subclass(OnGpu1), bad.as_subclass(OnGpu1))
