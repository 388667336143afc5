"""Performance cases of the operators around layers of experts: trained in groups of rows, their gradients clipped, answered from in 4 bits.

Five operators, each through the public entry points:

  grouped_forward    rows sorted by expert, expert e has rows offsets[e] .. offsets[e+1]-1:  y = act(x W_e^T + bias_e) + residual
  grouped_backward   the gradients of that with respect to x, every W_e and every bias_e, from dy and the kept pre-activations
  clip               norm = sqrt(sum of g^2) over all gradients of a network;  out = min(1, max_norm / norm) g
  pack_q4            weights -> codes of 4 bits and a scale for each `group` weights of a row, and back into the values they stand for:
                     scale = max|w| / 7 in the layer's type, code = floor(w / scale + 1/2) within -8 .. 7
  linear_q4          y = act(x W_e^T + bias_e) + residual for a few rows, W_e = scale * code

Inputs are synthetic, from the seed alone: normal activations and gradients, weights of standard deviation 1/sqrt(k), rows dealt to
the experts with some experts sought more than others (and some not at all).
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


# ---------------------------------------------------------------------------------------------------- the cases
def _grouped(kind, rows, experts, k, n, dtype, act, bias=True, residual=False, keep_z=False, spare=0, pad=0):
    """rows of x, the last `spare` of which belong to no expert (a padded batch); pad: elements between the end of a row of x and the next row."""
    return {"kind": kind, "rows": rows, "experts": experts, "k": k, "n": n, "dtype": dtype, "act": act, "bias": bias,
            "residual": residual, "keep_z": keep_z, "spare": spare, "pad": pad}


def _clip(layers, n, k, dtype, vectors, ratio, pad=0):
    """The gradients of `layers` layers: two matrices [n, k] and [k, n] (pad: elements between their rows) of one type, two vectors of
    another.  ratio: max_norm over the expected norm."""
    return {"kind": "clip", "layers": layers, "n": n, "k": k, "dtype": dtype, "vectors": vectors, "ratio": ratio, "pad": pad}


def _pack(experts, n, k, group, source, dtype):
    """source: the weights' type; dtype: that of the layer, its scales and the values read back."""
    return {"kind": "pack_q4", "experts": experts, "n": n, "k": k, "group": group, "source": source, "dtype": dtype}


def _q4(rows, experts, k, n, group, dtype, act, bias=False, residual=False, pad=0):
    return {"kind": "linear_q4", "rows": rows, "experts": experts, "k": k, "n": n, "group": group, "dtype": dtype, "act": act,
            "bias": bias, "residual": residual, "pad": pad}


def listed():
    return [
        # a decoding step of 24 tokens over 8 experts: bound by the weights of the experts that are sought
        dict(_grouped("grouped_forward", 24, 8, 1024, 2048, "bf16", "silu", bias=False), name="experts_few_rows"),
        # a training step: 16384 rows over 16 experts, pre-activations kept for the backward pass
        dict(_grouped("grouped_forward", 16384, 16, 2048, 4096, "bf16", "gelu_tanh", keep_z=True), name="experts_forward"),
        # the gradients of a small ragged layer: odd sizes throughout, a padded batch
        dict(_grouped("grouped_backward", 777, 5, 517, 259, "f16", "silu", spare=33, pad=3), name="experts_gradients_ragged"),
        # the gradients of the training step
        dict(_grouped("grouped_backward", 16384, 16, 2048, 4096, "bf16", "gelu_tanh"), name="experts_gradients"),
        # the gradients of a small network's layers of 64 channels as matrices of their windows: latency
        dict(_clip(10, 64, 576, "f32", "f32", 0.3), name="clip_small_network"),
        # a network of 16-bit matrices with fp32 vectors, rows padded, whose norm is within the bound: nothing to scale
        dict(_clip(12, 1000, 1531, "f16", "f32", 2.0, pad=5), name="clip_within_bound"),
        # a wide network of 537 million parameters
        dict(_clip(4, 4096, 16384, "bf16", "bf16", 0.3), name="clip_wide_network"),
        # the classifier of ResNet-18 brought to 4 bits from its fp32 weights
        dict(_pack(1, 1000, 512, 32, "f32", "f32"), name="pack_classifier"),
        # the weights of a layer of 16 experts after training
        dict(_pack(16, 4096, 2048, 128, "f32", "bf16"), name="pack_experts"),
        # the classifier for one image: latency
        dict(_q4(1, 1, 512, 1000, 32, "f32", "none", bias=True), name="classifier_q4"),
        # one token through a wide layer: bound by the weights' bytes
        dict(_q4(1, 1, 8192, 28672, 128, "bf16", "silu"), name="token_q4"),
        # 24 tokens over 32 experts
        dict(_q4(24, 32, 2048, 1536, 64, "f16", "none", residual=True), name="experts_q4"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Half of all sizes are multiples of 64, as most layers have them, the others any number."""
    v = _log(rng, lo, hi)
    return max(64, 64 * round(v / 64)) if hi >= 64 and rng.random() < 0.5 else v


def draw(rng: random.Random):
    kind = rng.choice(["grouped_forward", "grouped_backward", "clip", "pack_q4", "linear_q4", "linear_q4"])
    dtype = rng.choice(["f32", "f16", "bf16"])
    if kind == "clip":
        c = _clip(_log(rng, 1, 32), _size(rng, 8, 4096), _size(rng, 8, 16384), dtype, rng.choice([dtype, "f32"]),
                  rng.choice([0.03, 0.3, 0.3, 0.9, 2.0]), pad=rng.choice([0, 0, 0, 8, 1, 5]))
        while c["layers"] > 1 and c["layers"] * c["n"] * c["k"] > 4 * 4096 * 16384:
            c["layers"] = (c["layers"] + 1) // 2
        return c
    if kind == "pack_q4":
        c = _pack(_log(rng, 1, 32), _size(rng, 8, 8192), _size(rng, 8, 8192), rng.choice([32, 64, 128]), rng.choice(["f32", dtype]), dtype)
        while c["experts"] * c["n"] * c["k"] > 16 * 4096 * 2048:
            if c["experts"] > 1:
                c["experts"] = (c["experts"] + 1) // 2
            else:
                c["n"] = (c["n"] + 1) // 2
        return c
    if kind == "linear_q4":
        c = _q4(_log(rng, 1, 64), rng.choice([1, 1, _log(rng, 2, 64)]), _size(rng, 32, 16384), _size(rng, 8, 28672), rng.choice([32, 64, 128]),
                dtype, rng.choice(ACTS), bias=rng.random() < 0.5, residual=rng.random() < 0.5, pad=rng.choice([0, 0, 0, 1, 8]))
        while c["experts"] * c["n"] * c["k"] > 8192 * 28672:
            if c["experts"] > 1:
                c["experts"] = (c["experts"] + 1) // 2
            else:
                c["n"] = (c["n"] + 1) // 2
        return c
    c = _grouped(kind, _log(rng, 1, 16384), _log(rng, 1, 64), _size(rng, 8, 4096), _size(rng, 8, 4096), rng.choice(["f16", "bf16"]), rng.choice(ACTS),
                 bias=rng.random() < 0.7, residual=kind == "grouped_forward" and rng.random() < 0.5,
                 keep_z=kind == "grouped_forward" and rng.random() < 0.4, spare=0, pad=rng.choice([0, 0, 0, 1, 8]))
    while c["rows"] > 1 and c["rows"] * c["n"] * c["k"] > 16384 * 4096 * 2048:
        c["rows"] = (c["rows"] + 1) // 2
    while c["experts"] > 1 and c["experts"] * c["n"] * c["k"] > 16 * 4096 * 4096:
        c["experts"] = (c["experts"] + 1) // 2
    c["spare"] = rng.randint(0, c["rows"] // 4)
    return c


# ---------------------------------------------------------------------------------------------------- sizes
def _clip_count(case):
    return case["layers"] * 2 * case["n"] * case["k"], case["layers"] * (case["n"] + case["k"])


def _sought(experts, rows):
    """Experts that get a row, expected where every row takes any of them."""
    return experts * (1.0 - (1.0 - 1.0 / experts) ** rows)


def work(case):
    kind = case["kind"]
    if kind == "clip":
        m, v = _clip_count(case)
        return {"bytes": 2 * (m * SIZE[case["dtype"]] + v * SIZE[case["vectors"]]), "flops": 3 * (m + v)}
    n, k, b = case["n"], case["k"], SIZE[case["dtype"]]
    if kind == "pack_q4":
        count = case["experts"] * n * k
        return {"bytes": count * (SIZE[case["source"]] + b), "flops": 4 * count}
    m = case["rows"] - case.get("spare", 0)
    live = _sought(case["experts"], m) if m else 0.0
    bias = live * n if case["bias"] else 0
    if kind == "linear_q4":
        weights = live * n * (0.5 * k + b * -(-k // case["group"]))
        return {"bytes": int(weights + b * (m * k + bias + (1 + case["residual"]) * m * n)), "flops": 2 * m * n * k}
    if kind == "grouped_forward":
        outs = 1 + case["residual"] + case["keep_z"]
        return {"bytes": int(b * (m * k + live * n * k + bias + outs * m * n)), "flops": 2 * m * n * k}
    z = 0 if case["act"] == "none" else m * n
    bias = case["experts"] * n if case["bias"] else 0
    return {"bytes": int(b * (2 * m * k + (live + case["experts"]) * n * k + bias + m * n + z)), "flops": 4 * m * n * k}


# ---------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _deal(case, seed):
    """Rows of each expert: some are sought twice as often as others."""
    rng = random.Random(int(seed))
    share = [math.exp(rng.gauss(0.0, 0.4)) for _ in range(case["experts"])]
    counts = [0] * case["experts"]
    for e in rng.choices(range(case["experts"]), weights=share, k=case["rows"] - case.get("spare", 0)):
        counts[e] += 1
    return counts


def _clip_layout(case):
    """Places of the gradients in two buffers, one for the matrices and one for the vectors: (start, rows, columns, stride), each start on
    16 bytes."""
    matrices, vectors, ends = [], [], [0, 0]

    def place(to, which, rows, cols, ld, size):
        to.append((ends[which], rows, cols, ld))
        ends[which] += -(-rows * ld * size // 16) * 16 // size
    for _ in range(case["layers"]):
        for rows, cols in ((case["n"], case["k"]), (case["k"], case["n"])):
            place(matrices, 0, rows, cols, cols + case["pad"], SIZE[case["dtype"]])
        for cols in (case["n"], case["k"]):
            place(vectors, 1, 1, cols, cols, SIZE[case["vectors"]])
    return matrices, vectors, ends


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    t = TYPES[case["dtype"]]
    S = SimpleNamespace(case=case)
    if case["kind"] == "clip":
        S.matrices, S.vectors, ends = _clip_layout(case)
        S.flat = []
        for places, end, kind in ((S.matrices, ends[0], case["dtype"]), (S.vectors, ends[1], case["vectors"])):
            flat = torch.zeros(end, dtype=TYPES[kind], device="cuda")
            for at, rows, cols, ld in places:       # (what lies between the gradients stays zero)
                flat.as_strided((rows, cols), (ld, 1), at).copy_(_normal(g, rows, cols).mul_(0.01))
            S.flat.append(flat)
        S.max_norm = case["ratio"] * 0.01 * math.sqrt(sum(_clip_count(case)))
        return S
    k, n, experts = case["k"], case["n"], case["experts"]
    if case["kind"] == "pack_q4":
        S.w = (_normal(g, experts, n, k) / math.sqrt(k)).to(TYPES[case["source"]])
        return S
    m = case["rows"]
    counts = _deal(case, seed)
    S.most = max(1, max(counts))                    # (the capacity that a program plans for an expert)
    S.offsets = torch.tensor([0] + counts, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()
    S.x = _normal(g, m, k + case["pad"]).to(t)[:, :k]
    w = torch.empty(experts, n, k, dtype=t, device="cuda")
    for e in range(experts):
        w[e] = (_normal(g, n, k) / math.sqrt(k)).to(t)
    S.w = w
    S.bias = (0.2 * _normal(g, experts, n)).to(t) if case["bias"] else None
    if case["kind"] == "grouped_backward":
        S.dy = (_normal(g, m, n) * (2.0 / math.sqrt(m))).to(t)
        # what the forward pass kept: of the size of x W^T
        S.z = _normal(g, m, n).to(t) if case["act"] != "none" else None
    else:
        S.residual = _normal(g, m, n).to(t) if case["residual"] else None
    return S


def _pack_codes(w, group, t):
    """Codes of 4 bits, two in a byte, [experts, n, groups, group / 2], and the scales [experts, n, groups]."""
    experts, n, k = w.shape
    groups = -(-k // group)
    v = torch.zeros(experts, n, groups * group, dtype=w.dtype, device=w.device)
    v[:, :, :k] = w
    v = v.view(experts, n, groups, group)
    scales = (v.abs().amax(dim=3).float() / 7.0).to(t)
    s = scales.double()[..., None]
    codes = torch.where(s > 0, torch.floor(v.double() / s + 0.5).clamp(-8, 7), torch.zeros_like(s)).to(torch.int8) & 15
    return (codes[..., 0::2] | (codes[..., 1::2] << 4)).to(torch.uint8), scales


def _values(bytes_, scales, k):
    """The values that codes and scales stand for, in 32 bits."""
    low, high = (bytes_ & 15).to(torch.int8), (bytes_ >> 4).to(torch.int8)
    codes = torch.stack((low, high), dim=4).flatten(3)
    codes = codes - 16 * (codes >= 8).to(torch.int8)
    return (codes.float() * scales.float()[..., None]).flatten(2)[:, :, :k]


def prepare(case, seed):
    S = _inputs(case, seed)
    t = TYPES[case["dtype"]]
    if not own:
        if case["kind"] == "linear_q4":
            S.codes, S.scales = _pack_codes(S.w, case["group"], t)
            del S.w
        return S
    from paper_2003_07577_b200 import binding as ebs
    dtypes = {"f32": ebs.EBS_F32, "f16": ebs.EBS_F16, "bf16": ebs.EBS_BF16}
    act = {"none": ebs.EBS_ACT_NONE, "relu": ebs.EBS_ACT_RELU, "gelu": ebs.EBS_ACT_GELU,
           "gelu_tanh": ebs.EBS_ACT_GELU_TANH, "silu": ebs.EBS_ACT_SILU}
    new = lambda *shape: torch.zeros(shape, dtype=t, device="cuda")  # noqa: E731
    bytes_ = lambda count: torch.empty(max(16, count), dtype=torch.uint8, device="cuda")  # noqa: E731
    S.ebs = ebs
    if case["kind"] == "clip":
        S.out = [torch.zeros_like(f) for f in S.flat]
        views = lambda flats: [flats[i].as_strided((r, c), (ld, 1), at)  # noqa: E731
                               for i, places in enumerate((S.matrices, S.vectors)) for at, r, c, ld in places]
        S.plan = ebs.clip_plan(views(S.flat), views(S.out))
        S.norm = torch.zeros(1, dtype=torch.float32, device="cuda")
        S.workspace = bytes_(ebs.ebs_clip_workspace_bytes(S.plan))
        return S
    n, k, experts = case["n"], case["k"], case["experts"]
    if case["kind"] in ("pack_q4", "linear_q4"):
        S.q4 = ebs.q4_desc(n, k, case["group"], dtypes[case["dtype"]], experts)
        S.packed = bytes_(ebs.ebs_q4_packed_bytes(S.q4))
        if case["kind"] == "pack_q4":
            S.source, S.values = dtypes[case["source"]], new(experts, n, k)
            return S
        ebs.ebs_pack_weights_q4(S.w, dtypes[case["dtype"]], S.q4, S.packed)
        del S.w
        S.desc = ebs.linear_desc(case["rows"], n, k, dtypes[case["dtype"]], act[case["act"]], ldx=k + case["pad"])
        S.y = new(case["rows"], n)
        S.workspace = bytes_(ebs.ebs_linear_q4_workspace_bytes(S.desc, S.q4))
        return S
    m, ld = case["rows"], k + case["pad"]
    S.desc = ebs.linear_desc(m, n, k, dtypes[case["dtype"]], act[case["act"]], ldx=ld)
    if case["kind"] == "grouped_forward":
        S.y, S.keep = new(m, n), new(m, n) if case["keep_z"] else None
    else:
        S.dx_rows, S.dw = new(m, ld), new(experts, n, k)              # a gradient has the row stride of its tensor
        S.dx, S.dbias = S.dx_rows[:, :k], new(experts, n) if case["bias"] else None
    S.workspace = bytes_(ebs.ebs_grouped_workspace_bytes(S.desc, experts, case["kind"] == "grouped_backward"))
    return S


# ---------------------------------------------------------------------------------------------------- one pass
def _run_own(S):
    ebs, case = S.ebs, S.case
    if case["kind"] == "clip":
        ebs.ebs_clip_gradients(S.plan, S.max_norm, S.norm, S.workspace)
        return [S.norm, *S.out]
    if case["kind"] == "pack_q4":
        ebs.ebs_pack_weights_q4(S.w, S.source, S.q4, S.packed)
        ebs.ebs_unpack_weights_q4(S.packed, S.q4, S.values, S.q4.dtype)
        return [S.values]
    if case["kind"] == "linear_q4":
        offsets = S.offsets if case["experts"] > 1 else None
        ebs.ebs_linear_q4_forward(S.x, S.packed, S.bias, S.residual, offsets, S.desc, S.q4, S.y, S.workspace)
        return [S.y]
    if case["kind"] == "grouped_forward":
        ebs.ebs_grouped_forward(S.x, S.w, S.bias, S.residual, S.offsets, case["experts"], S.desc, S.y, S.keep, S.workspace)
        return [S.y] if S.keep is None else [S.y, S.keep]
    ebs.ebs_grouped_backward(S.dy, S.x, S.w, S.z, S.offsets, case["experts"], S.desc, S.dx, S.dw, S.dbias, S.workspace)
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


def _spread(S, rows):
    """Where each expert's rows are, [experts, most], and which of these places are rows."""
    first, last = S.offsets[:-1, None].long(), S.offsets[1:, None].long()
    at = first + torch.arange(S.most, device="cuda")
    return at.clamp(max=rows - 1), at < last


def _by_expert(v, at, there):
    """[rows, cols] -> fp32 [experts, most, cols], zero where there is no row."""
    return v[at].float() * there[..., None]


def _to_rows(v, at, there, rows, t):
    out = torch.zeros(rows, v.shape[2], dtype=t, device="cuda")
    out[at[there]] = v[there].to(t)
    return out


def run(S):
    if own:
        return _run_own(S)
    case = S.case
    t = TYPES[case["dtype"]]
    if case["kind"] == "clip":
        norm = torch.stack([f.double().square().sum() for f in S.flat]).sum().sqrt()
        factor = torch.where(norm <= S.max_norm, torch.ones_like(norm), S.max_norm / norm).float()
        return [norm.float().reshape(1), *[(f.float() * factor).to(f.dtype) for f in S.flat]]
    if case["kind"] == "pack_q4":
        codes, scales = _pack_codes(S.w, case["group"], t)
        return [_values(codes, scales, case["k"]).to(t)]
    m = case["rows"]
    at, there = _spread(S, m)
    x = _by_expert(S.x, at, there)
    if case["kind"] in ("linear_q4", "grouped_forward"):
        w = _values(S.codes, S.scales, case["k"]) if case["kind"] == "linear_q4" else S.w.float()
        z = torch.bmm(x, w.transpose(1, 2))
        if S.bias is not None:
            z = z + S.bias.float()[:, None, :]
        y = _activation(z, case["act"])
        if S.residual is not None:
            y = y + _by_expert(S.residual, at, there)
        out = [_to_rows(y, at, there, m, t)]
        return out + [_to_rows(z, at, there, m, t)] if case.get("keep_z") else out
    dz = _by_expert(S.dy, at, there)
    if S.z is not None:
        dz = dz * _slope(_by_expert(S.z, at, there), case["act"])
    dx = torch.zeros(m, case["k"] + case["pad"], dtype=t, device="cuda")[:, :case["k"]]
    dx[at[there]] = torch.bmm(dz, S.w.float())[there].to(t)
    out = [dx, torch.bmm(dz.transpose(1, 2), x).to(t)]
    return out + [dz.sum(dim=1).to(t)] if S.bias is not None else out


# ---------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_weights(w, group, t):
    out = torch.empty(w.shape, dtype=torch.float64, device="cuda")
    for first in range(0, w.shape[2], group):
        part = w[:, :, first:first + group].double()
        scale = (part.abs().max(dim=2, keepdim=True).values.float() / 7.0).to(t).double()      # (part of the definition: kept in the layer's type)
        code = torch.floor(part / scale + 0.5).clamp(-8, 7)
        out[:, :, first:first + group] = torch.where(scale > 0, scale * code, torch.zeros_like(code))
    return out


def exact(case, seed):
    S = _inputs(case, seed)
    t = TYPES[case["dtype"]]
    if case["kind"] == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(f, dtype=torch.float64)) ** 2 for f in S.flat))
        factor = min(1.0, S.max_norm / norm)
        return [torch.tensor([norm], dtype=torch.float64), *[f.double() * factor for f in S.flat]]
    if case["kind"] == "pack_q4":
        return [_exact_weights(S.w, case["group"], t)]
    f = torch.nn.functional
    act = {"none": lambda v: v, "relu": torch.relu, "gelu": f.gelu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"),
           "silu": f.silu}[case["act"]]
    n, m, experts = case["n"], case["rows"], case["experts"]
    offsets = S.offsets.tolist()
    new = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    y, z, dx, dw, db = new(m, n), new(m, n), new(m, case["k"]), None, new(experts, n)
    if case["kind"] == "grouped_backward":
        dw = new(experts, n, case["k"])
    for e in range(experts):
        rows = slice(offsets[e], offsets[e + 1])
        if offsets[e] == offsets[e + 1]:
            continue
        x = S.x[rows].double()
        w = _exact_weights(S.w[e:e + 1], case["group"], t)[0] if case["kind"] == "linear_q4" else S.w[e].double()
        if case["kind"] != "grouped_backward":
            z[rows] = torch.einsum("mk,nk->mn", x, w)
            if S.bias is not None:
                z[rows] += S.bias[e].double()
            y[rows] = act(z[rows]) if S.residual is None else act(z[rows]) + S.residual[rows].double()
            continue
        dz = S.dy[rows].double()
        if S.z is not None:
            v = S.z[rows].double().requires_grad_(True)
            (dz,) = torch.autograd.grad(act(v), v, dz)
        dx[rows], dw[e], db[e] = torch.einsum("mn,nk->mk", dz, w), torch.einsum("mn,mk->nk", dz, x), dz.sum(dim=0)
    if case["kind"] == "grouped_backward":
        return [dx, dw] if S.bias is None else [dx, dw, db]
    return [y, z] if case.get("keep_z") else [y]
