"""Every call of the library runs with its tensors' device current, whatever
device the caller's is (no GPU needed: the query, the switch and the library
are stand-ins)."""
import contextlib
import types

import pytest
import torch

import paper_2607_13500_gb300 as altr
from paper_2607_13500_gb300 import _device, _lib, api, attention

HOST = -1  # the index that host tensors report


class _Devices:
    """The caller's current device, and the switches made."""

    def __init__(self, monkeypatch, current):
        self.current, self.switches = current, []
        monkeypatch.setattr(_device, "_current", lambda: self.current)
        monkeypatch.setattr(_device, "_made_current", self.switch)

    @contextlib.contextmanager
    def switch(self, index):
        before, self.current = self.current, index
        self.switches.append(index)
        try:
            yield
        finally:
            self.current = before


class _Library:
    """Answers every attention call with success, noting the device it ran on."""

    def __init__(self, devices):
        self.devices, self.ran = devices, []

    def __getattr__(self, name):
        def call(*args):
            self.ran.append((name, self.devices.current))
            return 256 if name.endswith("workspace_bytes") else 0
        return call


def _rotary_on_host(calls):
    r = altr.Rotary.__new__(altr.Rotary)
    r.calls, r.device, r.index, r.head_dim, r.rot_dim, r.axes, r._struct = calls, torch.device("cpu"), HOST, 64, 64, 1, b""
    return r


def _cache_on_host(calls):
    c = altr.PagedCache.__new__(altr.PagedCache)
    c.k = c.v = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    c.calls, c.device, c.index, c.dtype = calls, torch.device("cpu"), HOST, torch.bfloat16
    c.pages, c.heads, c.page, c.head_dim = c.k.shape
    c.error, c._fixed, c._sizes = torch.zeros(1, dtype=torch.int32), (1, 2, 1, 4, 2, 16, 64), {}
    return c


@pytest.mark.parametrize("current", [0, 3, HOST])
def test_attention_calls(monkeypatch, current):
    devices = _Devices(monkeypatch, current)
    calls = _Library(devices)
    streams = []
    monkeypatch.setattr(attention, "_stream", lambda i: streams.append(i) or 0)
    r, c = _rotary_on_host(calls), _cache_on_host(calls)
    rows = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    q, k, v = rows[:, :4], rows[:, 4:6], rows[:, 6:]
    i32 = lambda *t: torch.tensor(t, dtype=torch.int32)
    pos, table, w = i32(0, 1, 2), i32(0, 1)[None], torch.ones(64)
    r.apply(q, k, pos)
    r.backward(q, k, pos, q=q, q_weight=w)
    c.append(k, v, table, i32(3), i32(0, 3), rotary=r, pos=pos, q=q)
    c.attend(q, table, i32(3), i32(0, 3))
    names = ["rotary_apply", "rotary_backward_workspace_bytes", "rotary_backward", "cache_append",
             "cache_attend_workspace_bytes", "cache_attend"]
    assert calls.ran == [(n, HOST) for n in names]
    assert streams and set(streams) == {HOST}
    assert devices.current == current
    assert devices.switches == ([] if current == HOST else [HOST] * len(names))


class _Seen(Exception):
    pass


def _far(devices):
    """A tensor on CUDA device 1 for a binding that only looks at its device first."""
    class Far:
        device = torch.device("cuda", 1)

        def __getattr__(self, name):
            assert devices.current == 1, name
            raise _Seen

        def __iter__(self):
            return self.items
    return Far()


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("name", ["workspace_bytes", "score", "select", "reduce", "mlp", "project_kept", "project"])
def test_functions(monkeypatch, name, current):
    devices = _Devices(monkeypatch, current)
    monkeypatch.setattr(api, "load", lambda: None)
    args = {"workspace_bytes": 3, "score": 3, "select": 4, "reduce": 3, "mlp": 3, "project_kept": 4, "project": 2}[name]
    far = _far(devices)
    with pytest.raises(_Seen):
        getattr(api, name)(*[far] * args)
    first = {"mlp": "x_pre", "project": "y"}.get(name, "x")
    rest = {"mlp": ("w1", "w2"), "project": ("w",), "project_kept": ("idx", "cu_k", "w"),
            "select": ("x_pre", "x_post", "stats")}.get(name, ("x_pre", "x_post"))
    with pytest.raises(_Seen):
        getattr(api, name)(**{n: far for n in (first, *rest)})
    assert devices.current == current and set(devices.switches) == (set() if current == 1 else {1})


@pytest.mark.parametrize("current", [0, 1])
@pytest.mark.parametrize("cls,method,args", [
    (api.Reducer, "run", 3), (api.Reducer, "graph", 3), (api.Reducer, "run_split", 3),
    (api.Reducer, "run_select_gather", 4), (api.Reducer, "run_separate", 3), (api.Reducer, "run_host", 6),
    (api.Pipeline, "submit", 3), (api.Pipeline, "submit_host", 5), (api.Pipeline, "graph", 3),
    (api.Pipeline, "graph_host", 5), (api.Pipeline, "wait", 1), (api.Mlp, "run", 1)])
def test_methods(monkeypatch, cls, method, args, current):
    devices = _Devices(monkeypatch, current)
    far = _far(devices)  # stands in for the object too: its first attribute is looked up on device 1
    with pytest.raises(_Seen):
        getattr(cls, method)(far, *[far] * args)
    assert devices.current == current and devices.switches == ([] if current == 1 else [1])


def test_a_device_without_an_index_is_the_current_one(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 2)
    assert _device.resolved("cuda") == torch.device("cuda", 2)
    assert _device.resolved("cuda:1") == torch.device("cuda", 1)
    assert _device.resolved("cpu") == torch.device("cpu")


@pytest.mark.parametrize("cls", [api.Reducer, api.Pipeline])
def test_tokens_of_another_device_are_refused(monkeypatch, cls):
    x = types.SimpleNamespace(device=torch.device("cuda", 0))
    monkeypatch.setattr(api, "_flatten", lambda *a: (x, x, x, [1]))
    r = cls.__new__(cls)
    r.seqlens, r.device, r._handle = [1], torch.device("cuda", 1), None
    with pytest.raises(ValueError, match="cuda:1"):
        r._bind(x, x, x)
