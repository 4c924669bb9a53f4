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
