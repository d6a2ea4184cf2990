"""The device a library call runs on.

libtr launches on the current device and its streams' raw handles do not say
whose they are (every device's default stream is 0), so the binding makes the
tensors' device current around each call."""
from __future__ import annotations

import functools

import torch

try:  # without torch.cuda.current_device's look at whether CUDA is up: whoever has a tensor there knows
    from torch._C import _cuda_getDevice as _current
except ImportError:
    _current = torch.cuda.current_device
_made_current = torch.cuda.device


def at(index, fn):
    """``fn``, made to run with CUDA device ``index`` current if another one is."""
    if _current() == index:
        return fn

    def call(*args):
        with _made_current(index):
            return fn(*args)
    return call


def resolved(device) -> torch.device:
    """``device`` with its index: a CUDA device named without one is the current one."""
    dev = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if dev.type == "cuda" and dev.index is None else dev


def on_device_of(name):
    """Runs a function with the CUDA device of its first argument current: a
    tensor (``name`` when passed by keyword) or an object with a ``device``.
    What is not on a CUDA device is for the function itself to refuse."""
    def wrap(fn):
        @functools.wraps(fn)
        def call(*args, **kwargs):
            dev = getattr(args[0] if args else kwargs.get(name), "device", None)
            if getattr(dev, "type", None) != "cuda" or dev.index is None or _current() == dev.index:
                return fn(*args, **kwargs)
            with _made_current(dev.index):
                return fn(*args, **kwargs)
        return call
    return wrap
