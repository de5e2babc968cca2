"""What layers.py does around the library's calls, on the CPU: tensors stand in as
fake ones of GPUs that are not there, the library as a recorder of calls."""
import contextlib
import warnings

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2510_23621_amd import layers as L

warnings.filterwarnings("ignore", message=".*data pointer of FakeTensor.*")


class Machine:
    """The current device as torch keeps it, and the library's calls with the device
    that was current for each and the stream they got."""

    def __init__(self, monkeypatch):
        self.current, self.calls = 0, []
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.current, raising=False)
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.current)
        monkeypatch.setattr(torch.cuda, "device", self.device)
        monkeypatch.setattr(torch.cuda, "stream", lambda s: self.device(s.device.index))
        monkeypatch.setattr(L, "_current_stream", lambda t: 1000 + t.get_device())
        monkeypatch.setattr(L.B, "lib", lambda: self)

    @contextlib.contextmanager
    def device(self, index):
        before, self.current = self.current, torch.device("cuda", index).index if isinstance(index, int) else index.index
        try:
            yield
        finally:
            self.current = before

    def __getattr__(self, name):
        if not name.startswith("mace_"):
            raise AttributeError(name)

        def call(*args):
            if name.endswith("_workspace_bytes"):
                return 256
            self.calls.append((name, self.current, args))
            return 0
        return call


class Stream:
    def __init__(self, index):
        self.device = torch.device("cuda", index)


@pytest.fixture
def machine(monkeypatch):
    with FakeTensorMode(allow_non_fake_inputs=True):
        yield Machine(monkeypatch)


def tensors(device):
    f, i = torch.float32, torch.int32
    x, w, rows = (torch.empty(*s, dtype=f, device=device) for s in [(6, 8), (8, 8), (12, 8)])
    plan = L.Route(*(torch.empty(*s, dtype=i, device=device) for s in [(6, 2), (12,), (4,)]))
    return x, w, rows, plan, torch.empty(6, 2, dtype=i, device=device), torch.empty(6, 2, dtype=f, device=device)


def calls(device, **kw):
    x, w, rows, plan, expert, weights = tensors(device)
    return {"linear": lambda: L.linear(x, w, act="silu", save=True, **kw),
            "linear by name": lambda: L.linear(w=w, x=x, **kw),
            "linear_backward": lambda: L.linear_backward(x, x, w, x, act="silu", **kw),
            "route": lambda: L.route(expert, 3, **kw),
            "route_rows": lambda: L.route_rows(x, plan, **kw),
            "combine_rows": lambda: L.combine_rows(rows, plan, weights, **kw),
            "combine_rows_backward": lambda: L.combine_rows_backward(x, rows, plan, weights, **kw),
            "route_rows_backward": lambda: L.route_rows_backward(rows, plan, **kw),
            "orthogonalise": lambda: L.orthogonalise(x, **kw)}


NAMES = ["linear", "linear by name", "linear_backward", "route", "route_rows", "combine_rows", "combine_rows_backward",
         "route_rows_backward", "orthogonalise"]


@pytest.mark.parametrize("name", NAMES)
def test_the_tensors_device_is_current_for_the_call(machine, name):
    for index in (0, 1, 3):
        machine.calls.clear()
        calls(f"cuda:{index}")[name]()
        assert [c[1] for c in machine.calls] == [index] and machine.current == 0
        assert machine.calls[0][2][-1] == 1000 + index


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_of_another_device_is_refused(machine, name):
    calls("cuda:1", stream=Stream(1))[name]()
    assert [c[1] for c in machine.calls] == [1] and machine.current == 0
    machine.calls.clear()
    with pytest.raises(ValueError, match="stream"):
        calls("cuda:1", stream=Stream(0))[name]()
    assert not machine.calls and machine.current == 0


@pytest.mark.parametrize("name", ["route_rows", "combine_rows", "combine_rows_backward", "route_rows_backward"])
def test_a_plan_of_another_device_is_refused(machine, name, monkeypatch):
    other = tensors("cuda:1")[3]
    for field in L.Route._fields:
        with pytest.raises(ValueError, match="plan"):
            x, _, rows, plan, _, weights = tensors("cuda:0")
            plan = plan._replace(**{field: getattr(other, field)})
            {"route_rows": lambda: L.route_rows(x, plan), "combine_rows": lambda: L.combine_rows(rows, plan, weights),
             "combine_rows_backward": lambda: L.combine_rows_backward(x, rows, plan, weights),
             "route_rows_backward": lambda: L.route_rows_backward(rows, plan)}[name]()
    assert not machine.calls
