"""Performance cases of the operators that train and answer with real-valued layers next to the bit-plane convolutions.

Three operators, each through the public entry points:

  forward        y = act(x W^T + bias) + residual: the classifier behind the last block, the layers that stay unquantized, and
                 the product of the bitwidth search, whose blended weights and activations are real values
  backward       the gradients of that layer with respect to x, W and bias, from dy and the kept pre-activations
  orthogonalize  an update matrix G -> the Newton-Schulz iterate of G / |G|: X <- a X + b (X X^T) X + c (X X^T)^2 X, `steps` times

Inputs are synthetic, from the seed alone: normal activations (rectified ones behind a rectified layer), weights of standard
deviation 1/sqrt(k), gradients of a batch mean, and update matrices of a decaying spectrum with noise on it.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
COEFF = (3.4445, -4.7750, 2.0315)          # the quintic's usual coefficients: steep at zero, singular values end in about 0.7 .. 1.2
EPS = 1e-7


# ---------------------------------------------------------------------------------------------------- the cases
def _linear(kind, m, k, n, dtype, act, bias=True, residual=False, keep_z=False, pad=0):
    """m rows of x, k input and n output features; pad: elements between the end of a row of x and the next row."""
    return {"kind": kind, "m": m, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias, "residual": residual,
            "keep_z": keep_z, "pad": pad}


def _ortho(batch, rows, cols, dtype, steps=5):
    return {"kind": "orthogonalize", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype, "steps": steps}


def listed():
    return [
        # the classifier of ResNet-18 for one image: latency
        dict(_linear("forward", 1, 512, 1000, "f32", "none"), name="classifier_one_image"),
        # a feed-forward layer for the three tokens of a decoding step: bound by the weights' bytes
        dict(_linear("forward", 3, 4096, 4096, "bf16", "silu", residual=True), name="tokens_few"),
        # odd sizes throughout, rows that start on odd elements
        dict(_linear("forward", 250, 1027, 333, "f16", "gelu", residual=True, pad=6), name="forward_ragged"),
        # the product of one search step: a 3x3 layer of 128 channels at 14x14, 64 images, as a matrix of its windows
        dict(_linear("forward", 12544, 1152, 256, "f32", "relu", keep_z=True), name="search_product"),
        # a training step of a wide layer on 8192 rows, pre-activations kept for the backward pass
        dict(_linear("forward", 8192, 4096, 4096, "bf16", "gelu_tanh", residual=True, keep_z=True), name="forward_wide"),
        # training the classifier of ResNet-18 on a small batch
        dict(_linear("backward", 128, 512, 1000, "f32", "none"), name="classifier_gradients"),
        # odd sizes throughout
        dict(_linear("backward", 1531, 517, 259, "f16", "silu", pad=3), name="backward_ragged"),
        # the gradients of the search step's product
        dict(_linear("backward", 12544, 1152, 256, "f32", "relu"), name="search_gradients"),
        # the gradients of the wide layer
        dict(_linear("backward", 8192, 4096, 4096, "bf16", "gelu"), name="backward_wide"),
        # the updates of the six 3x3 layers of 64 channels of a network, in one call
        dict(_ortho(6, 64, 576, "f32"), name="updates_64_channels"),
        # the update of a 3x3 layer of 512 channels
        dict(_ortho(1, 512, 4608, "bf16"), name="update_512_channels"),
        # the update of a wide layer
        dict(_ortho(1, 4096, 4096, "bf16"), name="update_wide"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of all sizes are multiples of 64, as most layers have them, the others any number."""
    v = _log(rng, lo, hi)
    return max(64, 64 * round(v / 64)) if hi >= 64 and rng.random() < 0.5 else v


def draw(rng: random.Random):
    kind = rng.choice(["forward", "forward", "backward", "backward", "orthogonalize", "orthogonalize"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind == "orthogonalize":
        c = _ortho(_log(rng, 1, 32), _size(rng, 2, 8192), _size(rng, 2, 8192), dtype, rng.choice([3, 5, 5, 6]))
        while _ortho_flops(c) > 0.8 * _ortho_flops(_ortho(1, 4096, 4096, "f32")):
            if c["batch"] > 1:
                c["batch"] = (c["batch"] + 1) // 2
            else:
                side = "rows" if c["rows"] > c["cols"] else "cols"
                c[side] = (c[side] + 1) // 2
        return c
    c = _linear(kind, _log(rng, 1, 16384), _size(rng, 8, 8192), _size(rng, 8, 8192), dtype, rng.choice(ACTS),
                bias=rng.random() < 0.7, residual=kind == "forward" and rng.random() < 0.5,
                keep_z=kind == "forward" and rng.random() < 0.4, pad=rng.choice([0, 0, 0, 1, 8]))
    while c["m"] > 1 and (c["m"] * c["n"] * c["k"] > 8192 * 4096 * 4096 or c["m"] * (c["n"] + c["k"]) > 8192 * 8192):
        c["m"] = (c["m"] + 1) // 2
    return c


# ---------------------------------------------------------------------------------------------------- sizes
def _ortho_flops(case):
    """Per step: the two symmetric products (one half of each determines it) and the product with X; m the shorter side."""
    m, n = sorted((case["rows"], case["cols"]))
    return case["batch"] * case["steps"] * (m * m * n + m * m * m + 2 * m * m * n)


def work(case):
    b = SIZE[case["dtype"]]
    if case["kind"] == "orthogonalize":
        return {"bytes": 2 * b * case["batch"] * case["rows"] * case["cols"], "flops": _ortho_flops(case)}
    m, k, n = case["m"], case["k"], case["n"]
    bias = n if case["bias"] else 0
    if case["kind"] == "forward":
        outs = 1 + case["residual"] + case["keep_z"]
        return {"bytes": b * (m * k + n * k + bias + outs * m * n), "flops": 2 * m * n * k}
    z = 0 if case["act"] == "none" else m * n
    return {"bytes": b * (2 * m * k + 2 * n * k + bias + m * n + z), "flops": 4 * m * n * k}


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t = TYPES[case["dtype"]]
    S = SimpleNamespace(case=case)
    if case["kind"] == "orthogonalize":
        b, rows, cols = case["batch"], case["rows"], case["cols"]
        rank = max(1, min(rows, cols) // 4)
        s = torch.arange(1, rank + 1, device="cuda", dtype=torch.float32).rsqrt()
        G = torch.bmm(_normal(g, b, rows, rank) * s, _normal(g, b, rank, cols)).add_(_normal(g, b, rows, cols), alpha=0.5)
        S.g = G.mul_(0.01).to(t)
        return S
    m, k, n = case["m"], case["k"], case["n"]
    x = _normal(g, m, k + case["pad"])
    if case["act"] == "relu":
        x = x.clamp_(min=0.0)                       # behind a layer of the same kind
    S.x = x.to(t)[:, :k]
    S.w = (_normal(g, n, k) / math.sqrt(k)).to(t)
    S.bias = (0.2 * _normal(g, n)).to(t) if case["bias"] else None
    if case["kind"] == "forward":
        S.residual = _normal(g, m, n).to(t) if case["residual"] else None
        return S
    S.dy = (_normal(g, m, n) * (2.0 / math.sqrt(m))).to(t)
    S.z = None
    if case["act"] != "none":                       # what the forward pass kept
        S.z = torch.matmul(S.x, S.w.t())
        if S.bias is not None:
            S.z = S.z + S.bias
    return S


def prepare(case, seed):
    S = _inputs(case, seed)
    if not own:
        return S
    from paper_2003_07577_b200 import binding as ebs
    dtype = {"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}[case["dtype"]]
    t = TYPES[case["dtype"]]
    empty = lambda *shape: torch.empty(shape, dtype=t, device="cuda")  # noqa: E731
    S.ebs, S.dtype = ebs, dtype
    if case["kind"] == "orthogonalize":
        S.out = torch.empty_like(S.g)
        bytes_ = ebs.ebs_orthogonalize_workspace_bytes(case["batch"], case["rows"], case["cols"], dtype, case["steps"])
    else:
        act = {"none": ebs.EBS_ACT_NONE, "relu": ebs.EBS_ACT_RELU, "gelu": ebs.EBS_ACT_GELU,
               "gelu_tanh": ebs.EBS_ACT_GELU_TANH, "silu": ebs.EBS_ACT_SILU}[case["act"]]
        m, k, n = case["m"], case["k"], case["n"]
        if case["kind"] == "forward":
            S.desc = ebs.linear_desc(m, n, k, dtype, act, ldx=k + case["pad"])
            S.y, S.keep = empty(m, n), empty(m, n) if case["keep_z"] else None
        else:
            S.desc = ebs.linear_desc(m, n, k, dtype, act, ldx=k + case["pad"])
            S.dx_rows, S.dw = empty(m, k + case["pad"]), empty(n, k)      # a gradient has the row stride of its tensor
            S.dx, S.dbias = S.dx_rows[:, :k], empty(n) if case["bias"] else None
        bytes_ = ebs.ebs_linear_workspace_bytes(S.desc, case["kind"] == "backward")
    S.workspace = torch.empty(max(16, bytes_), dtype=torch.uint8, device="cuda")
    return S


# ---------------------------------------------------------------------------------------------------- one pass
def _run_own(S):
    ebs, case = S.ebs, S.case
    if case["kind"] == "orthogonalize":
        ebs.ebs_orthogonalize(S.g, case["batch"], case["rows"], case["cols"], S.dtype, case["steps"], COEFF, EPS, 1.0, S.out,
                              S.workspace)
        return S.out
    if case["kind"] == "forward":
        ebs.ebs_linear_forward(S.x, S.w, S.bias, S.residual, S.desc, S.y, S.keep, S.workspace)
        return [S.y] if S.keep is None else [S.y, S.keep]
    ebs.ebs_linear_backward(S.dy, S.x, S.w, S.z, S.desc, S.dx, S.dw, S.dbias, S.workspace)
    return [S.dx, S.dw] if S.dbias is None else [S.dx, S.dw, S.dbias]


def _activation(z, act):
    if act == "none":
        return z
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z)


def _slope(z, act):
    """The activation's derivative."""
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        c = math.sqrt(2.0 / math.pi)
        th = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + th) + 0.5 * z * (1.0 - th * th) * c * (1.0 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(z)
    return s * (1.0 + z * (1.0 - s))


def run(S):
    if own:
        return _run_own(S)
    case = S.case
    t = TYPES[case["dtype"]]
    if case["kind"] == "orthogonalize":
        a, b, c = COEFF
        X = S.g.float()
        norm = X.double().pow(2).sum(dim=(1, 2), keepdim=True).sqrt()
        X = (X / (norm + EPS)).float()
        tall = case["rows"] > case["cols"]
        if tall:
            X = X.transpose(1, 2)
        for _ in range(case["steps"]):
            A = torch.bmm(X, X.transpose(1, 2))
            X = a * X + torch.bmm(b * A + c * torch.bmm(A, A), X)
        return (X.transpose(1, 2) if tall else X).contiguous().to(t)
    x, w = S.x.float(), S.w.float()
    if case["kind"] == "forward":
        z = torch.matmul(x, w.t())
        if S.bias is not None:
            z = z + S.bias.float()
        y = _activation(z, case["act"])
        if S.residual is not None:
            y = y + S.residual.float()
        return [y.to(t), z.to(t)] if case["keep_z"] else [y.to(t)]
    dz = S.dy.float()
    if S.z is not None:
        dz = dz * _slope(S.z.float(), case["act"])
    out = [torch.matmul(dz, w).to(t), torch.matmul(dz.t(), x).to(t)]
    return out + [dz.sum(dim=0).to(t)] if S.bias is not None else out


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    S = _inputs(case, seed)
    if case["kind"] == "orthogonalize":
        X = S.g.double()
        X = X / (torch.linalg.vector_norm(X, dim=(1, 2), keepdim=True) + EPS)
        a, b, c = COEFF
        for _ in range(case["steps"]):              # X X^T X = X (X^T X): the product over the shorter side
            if case["rows"] <= case["cols"]:
                A = X @ X.mT
                X = a * X + (b * A + c * (A @ A)) @ X
            else:
                A = X.mT @ X
                X = a * X + X @ (b * A + c * (A @ A))
        return X
    x, w, f = S.x.double(), S.w.double(), torch.nn.functional
    act = {"none": lambda v: v, "relu": torch.relu, "gelu": f.gelu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"),
           "silu": f.silu}[case["act"]]
    if case["kind"] == "forward":
        z = torch.einsum("mk,nk->mn", x, w)
        z = z if S.bias is None else z + S.bias.double()
        y = act(z) if S.residual is None else act(z) + S.residual.double()
        return [y, z] if case["keep_z"] else [y]
    dz = S.dy.double()
    if S.z is not None:
        z = S.z.double().requires_grad_(True)
        (dz,) = torch.autograd.grad(act(z), z, dz)
    out = [torch.einsum("mn,nk->mk", dz, w), torch.einsum("mn,mk->nk", dz, x)]
    return out if S.bias is None else out + [dz.sum(dim=0)]
