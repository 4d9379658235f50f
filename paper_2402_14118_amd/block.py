"""Convenience holders for what stands around a masked product in a residual block, on the current CUDA/HIP device.

They own workspaces, check that the tensors they are given have the shapes and types of the block, and forward to the C ABI; they do no
arithmetic of their own.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .tensors import check_device, own_device, rows


class BlockNorm:
    """The norms behind a block and in front of the next one, with the gate and the residual between them (mmm_block_norm):

        v  = norm(Y) * post_weight + post_bias        (post)
        h' = alpha * H + gate * v                     (H_out; without a block, Y=None: h' = H)
        n  = norm(h') * pre_weight + pre_bias         (normed)

    dtype: of normed, gate, weights and biases; dtype_h, dtype_y: of H, H_out and of Y (that type or MMM_F32).  training: owns
    the workspace that backward() needs for sums over rows; two of its calls that may run at the same time need a holder each."""

    def __init__(self, M: int, N: int, dtype: int = B.MMM_F32, post: int = B.MMM_NORM_NONE, pre: int = B.MMM_NORM_RMS, gate: int = B.MMM_GATE_NONE,
                 alpha: float = 1.0, eps: float = 1e-5, dtype_h: Optional[int] = None, dtype_y: Optional[int] = None, training: bool = False,
                 device="cuda:0"):
        self.desc = B.BlockNormDesc(M, N, dtype, dtype if dtype_h is None else dtype_h, dtype if dtype_y is None else dtype_y, post, pre, gate, eps, alpha)
        self.device = own_device(device)
        nbytes = B.mmm_block_norm_backward_workspace_bytes(M, N)   # (checks M and N)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if training else None

    def _gate(self, name, t, sums=False):
        d = self.desc
        shape = {B.MMM_GATE_ROW: (d.M,), B.MMM_GATE_COL: (d.N,), B.MMM_GATE_FULL: (d.M, d.N)}.get(d.gate)
        if shape is None and t is not None:
            raise ValueError(f"{name} is given, but there is no gate")
        return rows(name, t, shape, B.MMM_F32 if sums and d.gate != B.MMM_GATE_FULL else d.dt, self.device)

    def _vector(self, name, t, dtype):
        return rows(name, t, (self.desc.N,), dtype, self.device)[0]

    def forward(self, H: torch.Tensor, normed: Optional[torch.Tensor] = None, H_out: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                gate: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                pre_weight: Optional[torch.Tensor] = None, pre_bias: Optional[torch.Tensor] = None, stream=None) -> None:
        """H_out may be H."""
        d, shape = self.desc, (self.desc.M, self.desc.N)
        check_device(self.device)
        B.mmm_block_norm(d, *rows("H", H, shape, d.dt_h, self.device, False), *rows("Y", Y, shape, d.dt_y, self.device), *self._gate("gate", gate),
                         self._vector("post_weight", post_weight, d.dt), self._vector("post_bias", post_bias, d.dt),
                         self._vector("pre_weight", pre_weight, d.dt), self._vector("pre_bias", pre_bias, d.dt),
                         *rows("H_out", H_out, shape, d.dt_h, self.device), *rows("normed", normed, shape, d.dt, self.device), stream)

    def backward(self, H_out: Optional[torch.Tensor] = None, grad_normed: Optional[torch.Tensor] = None, grad_H_out: Optional[torch.Tensor] = None,
                 grad_H: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                 grad_Y: Optional[torch.Tensor] = None, grad_gate: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                 post_bias: Optional[torch.Tensor] = None, pre_weight: Optional[torch.Tensor] = None, grad_post_weight: Optional[torch.Tensor] = None,
                 grad_post_bias: Optional[torch.Tensor] = None, grad_pre_weight: Optional[torch.Tensor] = None,
                 grad_pre_bias: Optional[torch.Tensor] = None, stream=None) -> None:
        """H_out: as the forward call left it (H where there was no block).  grad_H may be grad_H_out.  Gradients that are not given are
        not worked out; those of weights, biases and of a gate per row or column are float."""
        d, shape, f = self.desc, (self.desc.M, self.desc.N), B.MMM_F32
        p = B._ptr
        check_device(self.device)
        ho, ldho = rows("H_out", H_out, shape, d.dt_h, self.device)
        y, ldy = rows("Y", Y, shape, d.dt_y, self.device)
        ga, ldga = self._gate("gate", gate)
        dn, lddn = rows("grad_normed", grad_normed, shape, d.dt, self.device)
        dho, lddho = rows("grad_H_out", grad_H_out, shape, d.dt_h, self.device)
        dh, lddh = rows("grad_H", grad_H, shape, d.dt_h, self.device)
        dy, lddy = rows("grad_Y", grad_Y, shape, d.dt_y, self.device)
        dg, lddg = self._gate("grad_gate", grad_gate, sums=True)
        g = B.BlockNormGrads(p(ho), ldho, p(y), ldy, p(ga), ldga, p(self._vector("post_weight", post_weight, d.dt)),
                             p(self._vector("post_bias", post_bias, d.dt)), p(self._vector("pre_weight", pre_weight, d.dt)), p(dn), lddn, p(dho), lddho,
                             p(dh), lddh, p(dy), lddy, p(dg), lddg, p(self._vector("grad_post_weight", grad_post_weight, f)),
                             p(self._vector("grad_post_bias", grad_post_bias, f)), p(self._vector("grad_pre_weight", grad_pre_weight, f)),
                             p(self._vector("grad_pre_bias", grad_pre_bias, f)))
        B.mmm_block_norm_backward(d, g, self.workspace, 0 if self.workspace is None else self.workspace.numel(), stream)
