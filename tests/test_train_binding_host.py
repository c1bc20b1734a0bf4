"""The training operators' binding without a GPU: what it asks of streams and the allocator, with stand-ins for both."""
import contextlib
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2104_05588_amd import _lib as L
from paper_2104_05588_amd import _train as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class FakeStream:
    def __init__(self, handle, device_index=0):
        self.cuda_stream, self.device_index, self.device = handle, device_index, torch.device("cuda", device_index)
        self.capturing, self.waits = False, []

    def wait_stream(self, other):
        self.waits.append(other.cuda_stream)


class FakeWorkspace:
    def __init__(self):
        self.recorded = []

    def record_stream(self, stream):
        self.recorded.append(stream.cuda_stream)


@pytest.fixture
def cuda(monkeypatch):
    """torch.cuda with a current stream and device 0, and no GPU."""
    state = {"stream": FakeStream(0)}

    @contextlib.contextmanager
    def on(stream):
        before, state["stream"] = state["stream"], stream
        yield
        state["stream"] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: state["stream"])
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: FakeStream(0))
    monkeypatch.setattr(torch.cuda, "ExternalStream", FakeStream)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: state["stream"].capturing)
    monkeypatch.setattr(L, "_current_raw_stream", lambda device: state["stream"].cuda_stream)
    return state


def prepared(made_on):
    """A MuonStep made on a stream of that handle, whose C call notes the stream that it gets."""
    step, calls = T.MuonStep.__new__(T.MuonStep), []
    step._workspace, step._device, step._byref = FakeWorkspace(), 0, None
    step._made_on = ctypes.c_void_p(made_on).value
    step._streams = {step._made_on}

    def fn(args, handle):
        calls.append(handle.value or 0)
        return L.DASO_OK

    step._fn = fn
    return step, calls


@pytest.mark.parametrize("made_on", [0, 0x1000])
def test_muon_step_on_another_stream_waits_and_is_recorded(cuda, made_on):
    step, calls = prepared(made_on)
    own, other = FakeStream(made_on), FakeStream(0x2000)
    step(own)
    assert calls == [made_on] and step._workspace.recorded == []
    step(other), step(other)
    assert calls == [made_on, 0x2000, 0x2000]
    assert other.waits == [made_on] and step._workspace.recorded == [0x2000]  # before the first call, and for good
    third = FakeStream(0x3000)
    with torch.cuda.stream(third):
        step()
    assert calls[-1] == 0x3000 and third.waits == [made_on] and step._workspace.recorded == [0x2000, 0x3000]
    step(own)
    assert len(step._workspace.recorded) == 2


def test_muon_step_captured_on_another_stream_waits_for_nothing_outside(cuda):
    step, calls = prepared(0)
    side = FakeStream(0x2000)
    side.capturing = True
    step(side)
    assert calls == [0x2000] and side.waits == [] and step._workspace.recorded == [0x2000]
    side.capturing = False
    step(side)
    assert side.waits == [0]


def test_muon_step_that_is_made_on_the_default_stream_may_be_called_there_by_name(cuda):
    step, _ = prepared(0x1000)
    named = FakeStream(0)
    step(named), step(named)
    assert named.waits == [0x1000] and step._workspace.recorded == [0]


class FakeTensor:
    """A tensor that passes the checks of a call on device 0."""

    def __init__(self, *shape, dtype=torch.float32):
        self.shape, self.dtype, self.is_cuda, self.device = torch.Size(shape), dtype, True, torch.device("cuda", 0)

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def is_contiguous(self):
        return True

    def stride(self):
        return (self.shape[-1], 1)[-self.dim():]

    def data_ptr(self):
        return 0x10000000

    def new_empty(self, *args, **kwargs):
        raise AssertionError("allocates before the stream is refused")


def test_a_stream_of_another_device_is_refused(cuda, monkeypatch):
    """Before anything is allocated, and before the device of the stream would become the current one."""
    def no_allocation(*args, **kwargs):
        raise AssertionError("allocates before the stream is refused")

    monkeypatch.setattr(torch, "empty", no_allocation)
    other = FakeStream(0x2000, device_index=1)
    x, v, t = FakeTensor(4, 8), FakeTensor(4), FakeTensor(4, dtype=torch.int64)
    w, flat = FakeTensor(5, 8), FakeTensor(64)
    for call in (lambda: T.layer_norm(x, stream=other), lambda: T.layer_norm_backward(x, x, None, v, v, stream=other),
                 lambda: T.linear_cross_entropy(x, w, t, stream=other),
                 lambda: T.linear_cross_entropy_backward(v, x, w, t, v, stream=other), lambda: T.orthogonalize(x, stream=other),
                 lambda: T.muon_step([flat], flat, flat, [(0, 4, 4)], 0.1, stream=other)):
        with pytest.raises(ValueError, match="the stream is of cuda:1"):
            call()
    step, calls = prepared(0)
    with pytest.raises(ValueError, match="the stream is of cuda:1"):
        step(other)
    assert calls == [] and step._workspace.recorded == []


def test_the_plan_of_a_large_batch_takes_no_memory_by_its_size():
    """daso_orthogonalize_workspace of 2^31 - 1 matrices within 2 GiB of address space more than the library itself."""
    program = """
import ctypes, resource, sys
from paper_2104_05588_amd import _train as T
lib = T._load()
pages = int(open("/proc/self/statm").read().split()[0])
limit = pages * resource.getpagesize() + (2 << 30)
resource.setrlimit(resource.RLIMIT_AS, (limit, limit))
a = T.daso_orthogonalize_args(batch=2 ** 31 - 1, rows=1, cols=1, type=0, out_type=0)
n = ctypes.c_size_t(0)
rc = lib.daso_orthogonalize_workspace(ctypes.byref(a), ctypes.byref(n))
print("status", rc, n.value)
"""
    res = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=120, cwd=ROOT)
    status = [line.split() for line in res.stdout.splitlines() if line.startswith("status")]
    assert res.returncode == 0 and status, res.stderr[-2000:]
    assert int(status[0][1]) == L.DASO_OK and 0 < int(status[0][2]) < 1 << 20
