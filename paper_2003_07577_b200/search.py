"""One layer of the bitwidth search, trained: blended weights and activations, their product, its gradients and an update.

During the search (Sec. 4.1) a layer keeps full-precision meta weights; every pass quantizes them and the activations at all
candidate bitwidths and blends the results (Eq. 6-7).  What is multiplied are the blended, real-valued tensors:

    x_hat = blend(x),  w_hat = blend(w),  y = act(x_hat w_hat^T + bias) + residual

The quantizers are passed straight through in the backward pass: the gradient of x_hat is that of x inside the clip range and
zero outside, the gradient of w_hat is that of w.  The update is momentum, orthogonalised by Newton-Schulz steps.  A k x k
convolution takes this form on the matrix of its windows, a 1x1 convolution on its pixels.

Buffers and call order only: the arithmetic is in the library's entry points (the clip mask and the momentum are element-wise
torch operations).  Everything runs on the weights' device and its current stream, in buffers made once, so that a training step can be captured into a
CUDA graph and replayed; a second stream or thread needs an object of its own.  Autograd sees none of it: the weights may be leaves that require
gradients, backward() is the gradient.
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import binding as ebs

COEFF = (3.4445, -4.7750, 2.0315)      # steep at zero; singular values end in about 0.7 .. 1.2


class SearchLinear:
    """Meta weights fp32 [n, k] and bias fp32 [n], both updated in place; `rows`: rows of every x.  bits: the candidate bitwidths;
    coeff_w / coeff_x: their blend coefficients (softmax of the strengths); alpha: the activations' clip value."""

    def __init__(self, weight: torch.Tensor, rows: int, bits: Sequence[int], coeff_w: Sequence[float], coeff_x: Sequence[float],
                 alpha: float, bias: Optional[torch.Tensor] = None, act: int = ebs.EBS_ACT_NONE, steps: int = 5):
        if weight.dim() != 2 or not weight.is_cuda or rows < 1:
            raise ValueError("weight must be a matrix on a GPU, rows at least 1")
        n, k = weight.shape
        self._check("weight", weight, (n, k), weight.device)
        self._check("bias", bias, (n,), weight.device)
        self.weight, self.bias, self.rows = weight, bias, rows
        self.bits, self.coeff_w, self.coeff_x = list(bits), list(coeff_w), list(coeff_x)
        self.alpha, self.act, self.steps = float(alpha), act, steps
        self.desc = ebs.linear_desc(rows, n, k, ebs.EBS_F32, act)
        new = lambda *shape: torch.zeros(shape, dtype=torch.float32, device=weight.device)  # noqa: E731
        self.w_hat, self.dw, self.momentum, self.update = new(n, k), new(n, k), new(n, k), new(n, k)
        self.dbias = None if bias is None else new(n)
        self.x_hat, self.dx, self.y, self.z = new(rows, k), new(rows, k), new(rows, n), new(rows, n)
        self.x = None
        self._scratch = torch.zeros(4, dtype=torch.int32, device=weight.device)
        need = [ebs.ebs_linear_workspace_bytes(self.desc, True), ebs.ebs_orthogonalize_workspace_bytes(1, n, k, ebs.EBS_F32, steps)]
        if min(need) == 0:                                    # (what the entry points answer to arguments that they refuse)
            raise ValueError("act, steps or sizes are out of range")
        need = max(need + [ebs.ebs_linear_workspace_bytes(self.desc, False)])
        self._workspace = torch.empty(need, dtype=torch.uint8, device=weight.device)

    @staticmethod
    def _check(name, t, shape, device):
        if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous() or t.device != device):
            raise ValueError(f"{name} must be dense fp32 {list(shape)} on {device}")

    @torch.no_grad()
    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: fp32 [rows, k], left as it is until backward().  The result stays valid until the next call."""
        n, k = self.weight.shape
        self._check("x", x, (self.rows, k), self.weight.device)
        self._check("residual", residual, (self.rows, n), self.weight.device)
        self.x = x
        with torch.cuda.device(self.weight.device):
            ebs.ebs_search_weight_forward(self.weight, self.bits, self.coeff_w, self.w_hat, self._scratch)
            ebs.ebs_search_act_forward(x, self.alpha, self.bits, self.coeff_x, self.x_hat)
            ebs.ebs_linear_forward(self.x_hat, self.w_hat, self.bias, residual, self.desc, self.y, self.z, self._workspace)
        return self.y

    @torch.no_grad()
    def backward(self, dy: torch.Tensor) -> torch.Tensor:
        """Gradient with respect to the x of the last forward pass (that of its residual is dy); those of the weights (dw) and the
        bias (dbias) are kept for step()."""
        if self.x is None:
            raise RuntimeError("backward() before forward()")
        self._check("dy", dy, (self.rows, self.weight.shape[0]), self.weight.device)
        with torch.cuda.device(self.weight.device):
            ebs.ebs_linear_backward(dy, self.x_hat, self.w_hat, self.z, self.desc, self.dx, self.dw, self.dbias, self._workspace)
        return self.dx.masked_fill(~((self.x > 0) & (self.x < self.alpha)), 0.0)

    @torch.no_grad()
    def step(self, rate: float, decay: float = 0.95) -> None:
        """w <- w - rate * orthogonalised(decay * momentum + dw); the bias takes a plain gradient step."""
        self.momentum.mul_(decay).add_(self.dw)
        n, k = self.weight.shape
        with torch.cuda.device(self.weight.device):
            ebs.ebs_orthogonalize(self.momentum, 1, n, k, ebs.EBS_F32, self.steps, COEFF, 1e-7, 1.0, self.update, self._workspace)
        self.weight.sub_(self.update, alpha=rate)
        if self.bias is not None:
            self.bias.sub_(self.dbias, alpha=rate)
