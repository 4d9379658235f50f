"""Tensors as the C ABI takes them: checks of shape, type, device and layout, and the leading dimension."""
from __future__ import annotations

import torch

from . import binding as B

TORCH_TYPES = {B.MMM_F32: torch.float32, B.MMM_BF16: torch.bfloat16, B.MMM_F16: torch.float16, B.MMM_F64: torch.float64}
CODES = {t: code for code, t in TORCH_TYPES.items()}


def places(device, needed: int, names, *tensors):
    """Tensor, shape and torch type of each in turn; the first `needed` have to be there.  Address and leading dimension (of a vector: 0) of each, one after
    the other; None and 0 of those that are None."""
    at = B.native.places(device, needed, *tensors)
    if type(at) is tuple:
        return at
    # what is wrong with it
    name, (t, shape, dtype) = names[at], tensors[3 * at:3 * at + 3]
    if t is None:
        raise ValueError(f"{name} is needed")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} is not a tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape if shape is None else tuple(shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    raise ValueError(f"the elements of {name} are not neighbours in memory")


def own_device(device) -> torch.device:
    d = torch.device(device)
    return torch.device(d.type, torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


def check_device(device: torch.device) -> None:
    """Kernels are launched on the current device, and on its current stream where none is given."""
    if device.index is not None and device.index != B.current_device() and device.type == "cuda":
        raise ValueError(f"the current device is cuda:{B.current_device()}, the tensors are on {device}")


def capturing(stream) -> bool:
    """Whether work on this stream (a stream, its handle, or None: the current one) goes into a graph."""
    if isinstance(stream, int):
        if stream == 0:
            return False
        stream = torch.cuda.ExternalStream(stream)
    with torch.cuda.stream(stream):   # (None: the current one)
        return torch.cuda.is_current_stream_capturing()
