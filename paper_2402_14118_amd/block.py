"""Convenience holders for what stands around a masked product in a residual block, on the current CUDA/HIP device.

They own workspaces, check that the tensors they are given have the shapes and types of the block, and forward to the C ABI; they do no
arithmetic of their own.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .engine import MaskedMatmul
from .tensors import TORCH_TYPES, capturing, check_device, own_device, places


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
        # shapes and types of the operands
        self.shape, self.columns = (M, N), (N,)
        self.gate_shape = {B.MMM_GATE_ROW: (M,), B.MMM_GATE_COL: (N,), B.MMM_GATE_FULL: (M, N)}.get(gate)
        self.type, self.type_h, self.type_y = (TORCH_TYPES.get(t) for t in (dtype, self.desc.dt_h, self.desc.dt_y))
        self.type_grad_gate = self.type if gate == B.MMM_GATE_FULL else torch.float32
        self.device = own_device(device)
        nbytes = B.mmm_block_norm_backward_workspace_bytes(M, N)   # (checks M and N)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device) if training else None
        self.room = (self.workspace.data_ptr(), nbytes) if training else (None, 0)
        self.fields = self.desc.fields()

    def forward(self, H: torch.Tensor, normed: Optional[torch.Tensor] = None, H_out: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None,
                gate: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None,
                pre_weight: Optional[torch.Tensor] = None, pre_bias: Optional[torch.Tensor] = None, stream=None, later: bool = False):
        """H_out may be H.  later: tensors are checked now, and launch() takes what is returned."""
        t, th, shape, columns = self.type, self.type_h, self.shape, self.columns
        check_device(self.device)
        if gate is not None and self.gate_shape is None:
            raise ValueError("gate is given, but there is no gate")
        h, ldh, y, ldy, g, ldg, pw, _, pb, _, w, _, b, _, ho, ldho, n, ldn = places(
            self.device, 1, ("H", "Y", "gate", "post_weight", "post_bias", "pre_weight", "pre_bias", "H_out", "normed"), H, shape, th, Y, shape, self.type_y,
            gate, self.gate_shape, t, post_weight, columns, t, post_bias, columns, t, pre_weight, columns, t, pre_bias, columns, t, H_out, shape, th, normed, shape, t)
        if later:
            return h, ldh, y, ldy, g, ldg, pw, pb, w, b, ho, ldho, n, ldn
        B._check(B.native.block_norm(self.fields, h, ldh, y, ldy, g, ldg, pw, pb, w, b, ho, ldho, n, ldn, B._stream(stream)), "mmm_block_norm")

    def launch(self, operands, stream=None) -> None:
        B._check(B.native.block_norm(self.fields, *operands, B._stream(stream)), "mmm_block_norm")

    def backward(self, H_out: Optional[torch.Tensor] = None, grad_normed: Optional[torch.Tensor] = None, grad_H_out: Optional[torch.Tensor] = None,
                 grad_H: Optional[torch.Tensor] = None, Y: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                 grad_Y: Optional[torch.Tensor] = None, grad_gate: Optional[torch.Tensor] = None, post_weight: Optional[torch.Tensor] = None,
                 post_bias: Optional[torch.Tensor] = None, pre_weight: Optional[torch.Tensor] = None, grad_post_weight: Optional[torch.Tensor] = None,
                 grad_post_bias: Optional[torch.Tensor] = None, grad_pre_weight: Optional[torch.Tensor] = None,
                 grad_pre_bias: Optional[torch.Tensor] = None, stream=None) -> None:
        """H_out: as the forward call left it (H where there was no block).  Y: that of the forward call, also where no value of it is needed; without it
        there was no block, and grad_H is not scaled by alpha.  grad_H may be grad_H_out.  Gradients that are not given are not worked out; those of
        weights, biases and of a gate per row or column are float."""
        t, th, ty, shape, columns, f = self.type, self.type_h, self.type_y, self.shape, self.columns, torch.float32
        check_device(self.device)
        if self.gate_shape is None and (gate is not None or grad_gate is not None):
            raise ValueError("gate is given, but there is no gate")
        (ho, ldho, y, ldy, ga, ldga, pw, _, pb, _, w, _, dn, lddn, dho, lddho, dh, lddh, dy, lddy, dg, lddg, dpw, _, dpb, _, dw, _, db, _) = places(
            self.device, 0, ("H_out", "Y", "gate", "post_weight", "post_bias", "pre_weight", "grad_normed", "grad_H_out", "grad_H", "grad_Y", "grad_gate",
                             "grad_post_weight", "grad_post_bias", "grad_pre_weight", "grad_pre_bias"),
            H_out, shape, th, Y, shape, ty, gate, self.gate_shape, t, post_weight, columns, t, post_bias, columns, t, pre_weight, columns, t,
            grad_normed, shape, t, grad_H_out, shape, th, grad_H, shape, th, grad_Y, shape, ty, grad_gate, self.gate_shape, self.type_grad_gate,
            grad_post_weight, columns, f, grad_post_bias, columns, f, grad_pre_weight, columns, f, grad_pre_bias, columns, f)
        B._check(B.native.block_norm_backward(self.fields, ho, ldho, y, ldy, ga, ldga, pw, pb, w, dn, lddn, dho, lddho, dh, lddh, dy, lddy, dg, lddg, dpw, dpb, dw, db,
                                              *self.room, B._stream(stream)), "mmm_block_norm_backward")


class MaskedMlp:
    """A residual MLP block on masked products, from the norm in front of it to the norm in front of the next one:

        a  = act(N x W1 + b1)                        N: the normed stream, M x width
        y  = M(a) x W2 + b2                          what the activation leaves at zero is skipped
        h' = alpha H + gate norm(y),  n' = norm(h')

    W1 (width x hidden) and W2 (hidden x width) are masked in blocks of their rows (a block that holds only zeros is off, and learns nothing); rows of W2 (hidden units) may be selected by context.  The
    holder owns the maps of both products, the activations between them and, with training=True, the gradients on the way and the
    workspaces of backward(): two calls that may run at the same time need a holder each.  y and the gradients on the way have the type of the weights.  fused (few rows of ReLU activations, not for
    training): the second product evaluates their mask itself, in one launch.

    A dense operand is multiplied by the matrix kernel (4 x 4096 x 16384 bf16, all blocks on: 29 us with its build, 109 by the pair kernel); for
    ReLU's zeros the choice of kernel goes by count(), once there has been one."""

    def __init__(self, M: int, width: int, hidden: int, block_width: int = 32, dtype: int = B.MMM_BF16, activation: int = B.MMM_ACT_RELU,
                 post: int = B.MMM_NORM_RMS, pre: int = B.MMM_NORM_RMS, gate: int = B.MMM_GATE_NONE, alpha: float = 1.0, eps: float = 1e-5,
                 dtype_h: Optional[int] = None, fused: bool = False, training: bool = False, device="cuda:0"):
        if dtype not in (B.MMM_F32, B.MMM_BF16, B.MMM_F16):
            raise ValueError("the norms of the block take floats and 16-bit types")
        if fused and training:
            raise ValueError("the gradients need the maps of the activations, which a fused product does not make")
        if fused and activation != B.MMM_ACT_RELU:
            raise ValueError("a fused product is for activations with many zeros, those of ReLU")
        self.M, self.width, self.hidden, self.dtype, self.activation, self.fused, self.training = M, width, hidden, dtype, activation, fused, training
        self.device = own_device(device)
        self.up = MaskedMatmul(M, width, hidden, block_width, dtype, self.device)
        self.down = MaskedMatmul(M, hidden, width, block_width, dtype, self.device)
        self.norm = BlockNorm(M, width, dtype, post, pre, gate, alpha, eps, dtype_h, training=training, device=self.device)
        self.up.set_path(B.MMM_PATH_MATRIX)
        if activation != B.MMM_ACT_RELU:
            self.down.set_path(B.MMM_PATH_MATRIX)

        def room(*shape, t=None):
            return torch.empty(shape, dtype=TORCH_TYPES[dtype if t is None else t], device=self.device)
        self.a, self.y = room(M, hidden), room(M, width)
        # what the slope is taken at: ReLU's is told by its value
        self.preact = self.a if activation in (B.MMM_ACT_RELU, B.MMM_ACT_NONE) else room(M, hidden) if training else None
        self.W1 = self.b1 = self.W2 = self.b2 = self.built = None   # built: where the N of the last forward call is
        self.counted = False   # and the form of floats has not been chosen since
        if training:
            self.grad_a, self.grad_y = room(M, hidden), room(M, width)
            nbytes = max(B.mmm_epilogue_backward_workspace_bytes(M, n) for n in (hidden, width))
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def close(self) -> None:
        self.up.close()
        self.down.close()

    def set_weights(self, W1: torch.Tensor, W2: torch.Tensor, b1: Optional[torch.Tensor] = None, b2: Optional[torch.Tensor] = None,
                    keep_blocks1: Optional[torch.Tensor] = None, keep_blocks2: Optional[torch.Tensor] = None,
                    keep_rows2: Optional[torch.Tensor] = None, stream=None) -> None:
        """Build the maps of both weights; again after a weight or a selection has changed.  All of them are kept (see count()).
        Where calls have been captured into a graph, keep_rows2 is given from then on exactly if it was then."""
        check_device(self.device)
        t = TORCH_TYPES[self.dtype]
        places(self.device, 2, ("W1", "W2", "b1", "b2"), W1, (self.width, self.hidden), t, W2, (self.hidden, self.width), t, b1, (self.hidden,), t, b2, (self.width,), t)
        self.W1, self.W2, self.b1, self.b2 = W1, W2, b1, b2
        self.masks = dict(keep_blocks=keep_blocks1), dict(keep_rows=keep_rows2, keep_blocks=keep_blocks2)
        self.up.build_maps(None, W1, stream=stream, **self.masks[0])
        self.down.build_maps(None, W2, stream=stream, **self.masks[1])

    def count(self, stream=None):
        """Count the densities of the last forward call (waits for the stream): what the choice of kernel, of tiles and of the form of floats goes by
        from then on.  A side of a product that is built alone keeps the form of the other: the next forward call on floats that is not captured into a
        graph builds the maps of the weights again, in one with those of its activations.  Returns ((non-zeros, blocks, products) of the first product, the
        same of the second; None where its mask is fused)."""
        check_device(self.device)
        counts = self.up.stats(stream), None if self.fused else self.down.stats(stream)
        self.counted = self.dtype == B.MMM_F32
        return counts

    def forward(self, N: torch.Tensor, H: torch.Tensor, H_out: torch.Tensor, normed: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                post_weight: Optional[torch.Tensor] = None, post_bias: Optional[torch.Tensor] = None, pre_weight: Optional[torch.Tensor] = None,
                pre_bias: Optional[torch.Tensor] = None, stream=None) -> None:
        """H_out may be H (backward() does not need H); normed receives n'."""
        if self.W1 is None:
            raise ValueError("set_weights() comes first")
        # (everything is checked before the first launch)
        norm = self.norm.forward(H, normed, H_out, self.y, gate, post_weight, post_bias, pre_weight, pre_bias, later=True)
        self.built = places(self.device, 1, ("N",), N, (self.M, self.width), TORCH_TYPES[self.dtype])
        kept = self.preact if self.training and self.preact is not self.a else None
        both = self.counted and not capturing(stream)
        W1, W2, masks = (self.W1, self.W2, self.masks) if both else (None, None, ({}, {}))
        self.up.build_maps(N, W1, stream=stream, **masks[0])
        self.up.matmul_epilogue(N, self.W1, self.a, bias=self.b1, activation=self.activation, preact=kept, stream=stream)
        if not self.fused:
            self.down.build_maps(self.a, W2, stream=stream, **masks[1])   # (by the value, not by the sign: NaN has to reach the stream)
        self.down.matmul_epilogue(self.a, self.W2, self.y, bias=self.b2, pred=B.MMM_PRED_NONZERO if self.fused else None, stream=stream)
        self.norm.launch(norm, stream)
        if both:
            self.counted = False

    def backward(self, N: torch.Tensor, H_out: torch.Tensor, grad_N: torch.Tensor, grad_H: torch.Tensor, grad_normed: Optional[torch.Tensor] = None,
                 grad_H_out: Optional[torch.Tensor] = None, grad_W1: Optional[torch.Tensor] = None, grad_W2: Optional[torch.Tensor] = None,
                 grad_b1: Optional[torch.Tensor] = None, grad_b2: Optional[torch.Tensor] = None, accumulate: bool = False, stream=None, **norm) -> None:
        """The gradients of the forward call before it (N as it was then, H_out as it left it).  grad_W1, grad_W2, grad_b1, grad_b2 are float;
        accumulate: those of the weights are added to.  norm: the values (gate, post_weight, post_bias, pre_weight) and gradients (grad_gate,
        grad_post_weight, grad_post_bias, grad_pre_weight, grad_pre_bias) of BlockNorm.backward."""
        if not self.training:
            raise ValueError("made without training=True")
        M, ws, od = self.M, self.workspace, self.dtype
        # (checked before anything is launched, or added to)
        mk, t, f = (M, self.width), TORCH_TYPES[od], torch.float32
        at = places(self.device, 1, ("N", "grad_N", "grad_W1", "grad_W2", "grad_b1", "grad_b2"), N, mk, t, grad_N, mk, t, grad_W1, (self.width, self.hidden), f,
                    grad_W2, (self.hidden, self.width), f, grad_b1, (self.hidden,), f, grad_b2, (self.width,), f)
        if at[:2] != self.built:
            raise ValueError("N is not that of a forward call")
        if grad_N is None and grad_W1 is None:
            raise ValueError("grad_N or grad_W1 is needed")
        for name, grad, ld in (("grad_N", grad_N, at[3]), ("grad_W1", grad_W1, at[5]), ("grad_W2", grad_W2, at[7])):
            if grad is not None and ld < grad.shape[1]:
                raise ValueError(f"rows of {name} overlap")
        self.norm.backward(H_out=H_out, grad_normed=grad_normed, grad_H_out=grad_H_out, grad_H=grad_H, Y=self.y, grad_Y=self.grad_y, stream=stream, **norm)
        if grad_b2 is not None:
            B.mmm_epilogue_backward(M, self.width, od, od, B.MMM_ACT_NONE, self.grad_y, self.width, None, 0, None, 0, grad_b2, ws, ws.numel(), stream)
        # (a unit that ReLU has turned off has no slope; elsewhere a zero is a value like others)
        self.down.matmul_backward(self.a, self.W2, self.grad_y, dX=self.grad_a, dY=grad_W2, accumulate=accumulate,
                                  all_x=self.activation != B.MMM_ACT_RELU, stream=stream)
        B.mmm_epilogue_backward(M, self.hidden, od, od, self.activation, self.grad_a, self.hidden, self.preact, self.hidden, self.grad_a, self.hidden,
                                grad_b1, ws, ws.numel(), stream)
        self.up.matmul_backward(N, self.W1, self.grad_a, dX=grad_N, dY=grad_W1, accumulate=accumulate, all_x=True, stream=stream)
