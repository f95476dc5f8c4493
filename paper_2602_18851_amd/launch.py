"""Calls on the current torch stream of a tensor's device, and what they refuse."""

from __future__ import annotations

import torch
from torch._C import _cuda_getCurrentRawStream as _raw_stream  # the handle without a Stream object around it


def on_stream_of(device: torch.device, call, *args) -> None:
    """call(*args, stream) with the device as the current one."""
    index = device.index
    if torch.cuda.current_device() == index:
        call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            call(*args, _raw_stream(index))


def refuse_autograd(name: str) -> None:
    """Raises where autograd would expect the gradient, of a call that it does not see, of a tensor that requires it."""
    if torch.is_grad_enabled():
        raise ValueError(f"{name} requires gradients, which this call does not record: pass {name}.detach() or call it "
                         "under torch.no_grad(), and call the gradient yourself")
