"""Tensors as the C ABI takes them: checks of shape, type, device and layout, and the leading dimension."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B

TORCH_TYPES = {B.MMM_F32: torch.float32, B.MMM_BF16: torch.bfloat16, B.MMM_F16: torch.float16, B.MMM_F64: torch.float64}
CODES = {t: code for code, t in TORCH_TYPES.items()}


def rows(name: str, t: Optional[torch.Tensor], shape, dtype: int, device, optional: bool = True):
    """(address, leading dimension) of a matrix, or of a vector (leading dimension 0); (None, 0) of none."""
    if t is None:
        if not optional:
            raise ValueError(f"{name} is needed")
        return None, 0
    at = B.native.place(t, shape, TORCH_TYPES.get(dtype), device)
    if at is not None:
        return at
    # what is wrong with it
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} is not a tensor")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")
    if CODES.get(t.dtype) != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {TORCH_TYPES.get(dtype)}")
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
