"""Torch's memory for calls on a stream that is not torch's current one, and the device of a
call's tensors."""
from __future__ import annotations

import torch

from . import sbp

_TENSOR = torch.Tensor


def torch_stream(handle: int):
    return torch.cuda.ExternalStream(handle) if handle else torch.cuda.default_stream()


def on_stream(stream: int, call, *args):
    """call(*args) with `stream` (a handle) as torch's current stream.

    What the call allocates then comes from that stream's blocks of memory. A block of
    the caller's stream may still be read or written by work queued there when `stream`
    starts on it, and one that the call drops may be given to the caller's next work while
    `stream` uses it; in its own blocks a stream only meets its own work. The tensors that
    the call returns are the caller's to use once its stream waits for `stream`: they are
    recorded there, so that dropping them keeps their memory until that use is over."""
    caller = torch.cuda.current_stream()
    with torch.cuda.stream(torch_stream(stream)):
        out = call(*args)
    for t in out:
        if isinstance(t, torch.Tensor):
            t.record_stream(caller)
    return out


def same_device(*tensors):
    """The library's calls run on the current device, whose tensors these must be (None and
    workspaces that are no tensors aside)."""
    device = sbp.current_device()
    for t in tensors:
        if t is not None and isinstance(t, _TENSOR) and t.device.index != device:
            raise ValueError("tensors are on %s, the current device is cuda:%d"
                             % (t.device, device))
