"""A layer of experts: trained in groups of rows, its gradients clipped with those of other layers, answered from in 4 bits.

Rows offsets[e] .. offsets[e+1]-1 of x are expert e's, which has weights and a bias of its own:

    y = act(x W_e^T + bias_e)

Training keeps fp32 weights and multiplies a 16-bit copy of them; the update is momentum, orthogonalised by Newton-Schulz steps, of all experts in one
call.  ``quantized`` brings the weights to 4 bits with a scale for each group of a row: the layer that answers a few rows (tokens) at a time.

Buffers and call order only: the arithmetic is in the library's entry points (the momentum and the additions to the weights are element-wise torch operations).
Everything runs on the weights' device and its current stream, in buffers made once, so that a training step or an answer can be captured into a CUDA graph and
replayed; the offsets are read on the device.  A second stream or thread needs an object of its own.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as ebs
from .search import COEFF

_CODE = {torch.float16: ebs.EBS_F16, torch.bfloat16: ebs.EBS_BF16}


def _check(name, t, shape, dtype, device):
    if t is not None and (t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() or t.device != device):
        raise ValueError(f"{name} must be dense {dtype} {list(shape)} on {device}")


class ExpertLinear:
    """weight: fp32 [experts, n, k] and bias fp32 [experts, n], both updated in place; rows: rows of every x (those that are no expert's included); dtype: fp16 or bf16,
    of x, y and the products."""

    def __init__(self, weight: torch.Tensor, rows: int, dtype: torch.dtype, bias: Optional[torch.Tensor] = None, act: int = ebs.EBS_ACT_NONE, steps: int = 5):
        if weight.dim() != 3 or not weight.is_cuda or rows < 1 or dtype not in _CODE:
            raise ValueError("weight must be [experts, n, k] on a GPU, rows at least 1, dtype fp16 or bf16")
        self.experts, n, k = weight.shape
        self.device, self.dtype, self.rows, self.act, self.steps = weight.device, dtype, rows, act, steps
        _check("weight", weight, weight.shape, torch.float32, self.device)
        _check("bias", bias, (self.experts, n), torch.float32, self.device)
        self.weight, self.bias = weight, bias
        self.desc = ebs.linear_desc(rows, n, k, _CODE[dtype], act)
        need = [ebs.ebs_grouped_workspace_bytes(self.desc, self.experts, True), ebs.ebs_orthogonalize_workspace_bytes(self.experts, n, k, ebs.EBS_F32, steps)]
        if min(need) == 0:                                    # (what the entry points answer to arguments that they refuse)
            raise ValueError("act, steps or sizes are out of range")
        new = lambda t, *shape: torch.zeros(shape, dtype=t, device=self.device)  # noqa: E731
        self.w, self.dw, self.momentum, self.update = (new(t, self.experts, n, k) for t in (dtype, dtype, torch.float32, torch.float32))
        self.b, self.dbias = (None, None) if bias is None else (new(dtype, self.experts, n), new(dtype, self.experts, n))
        self.dx, self.y, self.z = new(dtype, rows, k), new(dtype, rows, n), new(dtype, rows, n)
        self.x = self.offsets = None
        need.append(ebs.ebs_grouped_workspace_bytes(self.desc, self.experts, False))
        self._workspace = torch.empty(max(need), dtype=torch.uint8, device=self.device)
        self._copy()

    def _copy(self):
        self.w.copy_(self.weight.detach())
        if self.bias is not None:
            self.b.copy_(self.bias.detach())

    @torch.no_grad()
    def forward(self, x: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """x: [rows, k], offsets: int32 [experts + 1], both left as they are until backward().  The result stays valid until the next call; its rows that are no
        expert's hold whatever was there."""
        n, k = self.weight.shape[1:]
        _check("x", x, (self.rows, k), self.dtype, self.device)
        _check("offsets", offsets, (self.experts + 1,), torch.int32, self.device)
        self.x, self.offsets = x, offsets
        with torch.cuda.device(self.device):
            ebs.ebs_grouped_forward(x, self.w, self.b, None, offsets, self.experts, self.desc, self.y, self.z if self.act else None, self._workspace)
        return self.y

    @torch.no_grad()
    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """Gradient with respect to the x of the last forward pass, zero in rows that are no expert's; those of the weights (dw) and biases (dbias) are kept for step()."""
        if self.x is None:
            raise RuntimeError("backward() before forward()")
        _check("dy", dy, (self.rows, self.weight.shape[1]), self.dtype, self.device)
        self.dx.zero_()                                       # (the library leaves rows that are no expert's: they may have been one's in the step before)
        with torch.cuda.device(self.device):
            ebs.ebs_grouped_backward(dy, self.x, self.w, self.z if self.act else None, self.offsets, self.experts, self.desc, self.dx, self.dw, self.dbias, self._workspace)
        return self.dx

    @torch.no_grad()
    def step(self, rate: float, decay: float = 0.95) -> None:
        """weight <- weight - rate * orthogonalised(decay * momentum + dw), each expert's on its own; the biases take a plain gradient step."""
        self.momentum.mul_(decay).add_(self.dw)
        n, k = self.weight.shape[1:]
        with torch.cuda.device(self.device):
            ebs.ebs_orthogonalize(self.momentum, self.experts, n, k, ebs.EBS_F32, self.steps, COEFF, 1e-7, 1.0, self.update, self._workspace)
        self.weight.sub_(self.update, alpha=rate)
        if self.bias is not None:
            self.bias.sub_(self.dbias, alpha=rate)
        self._copy()

    def quantized(self, rows: int, group: int = 128) -> "QuantizedExperts":
        """The layer as it answers `rows` rows (the largest number of a call), from the weights as they are now."""
        return QuantizedExperts(self.weight.detach(), rows, self.dtype, None if self.bias is None else self.bias.detach(), self.act, group)


class QuantizedExperts:
    """weight: fp32 [experts, n, k], brought to 4 bits and not kept; bias: fp32 [experts, n], kept in the layer's type; rows: the most of a call."""

    def __init__(self, weight: torch.Tensor, rows: int, dtype: torch.dtype, bias: Optional[torch.Tensor] = None, act: int = ebs.EBS_ACT_NONE, group: int = 128):
        if weight.dim() != 3 or not weight.is_cuda or rows < 1 or dtype not in _CODE:
            raise ValueError("weight must be [experts, n, k] on a GPU, rows at least 1, dtype fp16 or bf16")
        self.experts, self.n, self.k = weight.shape
        self.device, self.dtype, self.rows, self.act = weight.device, dtype, rows, act
        _check("weight", weight, weight.shape, torch.float32, self.device)
        _check("bias", bias, (self.experts, self.n), torch.float32, self.device)
        self.q4 = ebs.q4_desc(self.n, self.k, group, _CODE[dtype], self.experts)
        size = ebs.ebs_q4_packed_bytes(self.q4)
        if size == 0 or not ebs.EBS_ACT_NONE <= act <= ebs.EBS_ACT_SILU:
            raise ValueError("group, act or sizes are out of range")
        self.packed = torch.empty(size, dtype=torch.uint8, device=self.device)
        self.bias = None if bias is None else bias.to(dtype)
        self.y = torch.zeros((rows, self.n), dtype=dtype, device=self.device)
        # (a call of fewer rows may be run in another form, which wants more)
        most = max(ebs.ebs_linear_q4_workspace_bytes(self._desc(m), self.q4) for m in range(1, rows + 1))
        self._workspace = torch.empty(max(16, most), dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            ebs.ebs_pack_weights_q4(weight, ebs.EBS_F32, self.q4, self.packed)

    def _desc(self, m):
        return ebs.linear_desc(m, self.n, self.k, _CODE[self.dtype], self.act)

    @torch.no_grad()
    def answer(self, x: torch.Tensor, offsets: torch.Tensor) -> torch.Tensor:
        """x: [m, k] with m <= rows, offsets: int32 [experts + 1] within 0 .. m.  The result stays valid until the next call; its rows that are no
        expert's hold whatever was there."""
        if x.dim() != 2 or x.shape[0] > self.rows:
            raise ValueError(f"x has up to {self.rows} rows")
        m = x.shape[0]
        _check("x", x, (m, self.k), self.dtype, self.device)
        _check("offsets", offsets, (self.experts + 1,), torch.int32, self.device)
        y = self.y[:m]
        if m:
            with torch.cuda.device(self.device):
                ebs.ebs_linear_q4_forward(x, self.packed, self.bias, None, offsets, self._desc(m), self.q4, y, self._workspace)
        return y
