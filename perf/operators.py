"""Timed calls of the fully-connected layer's operators: 4-bit weights with group scales, and
8-bit activation checkpoints.

A case is a dict of plain values; ``op`` names the operator:

  quantize    kq_quantize_groups, then kq_reconstruct_groups: 4-bit codes and group scales of a
              weight matrix, and the weights they stand for
  linear      kq_group_linear: Y = X W^T + b from the codes, one token to a prompt
  grad_input  kq_group_linear_grad_input: dX = dY W
  checkpoint  kq_checkpoint_pack, then kq_checkpoint_restore: an activation in 8 bits, and back
  grad        from the 8-bit checkpoint of X: kq_checkpoint_grad_scales (``of`` = "scales": the
              gradient of the group scales and of the bias) or kq_checkpoint_grad_weight
              (``of`` = "weight": the gradient of the whole matrix)

``m`` tokens, ``n`` output features, ``k`` input features, ``group`` weights to a scale, ``levels``
whether the 16 levels come from a table (else they are -8 .. 7).  Sizes are those of VGG-16's
fully-connected layers (25088 -> 4096 -> 4096 -> 1000) and ResNet-18's classifier (512 -> 1000).

The packed weights are tiles of 16 rows by 128 columns, [ceil(n/16), ceil(k/128), 16, 64] bytes; _pack
says where a column stands in its row's 64 bytes.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_MOST = 2 * 2048 * 4096 * 25088   # operations of the largest listed product


def listed():
    return [
        # compressing a small classifier held in bf16, odd width, with a learned level table
        {"name": "quantize_1000x1023_levels", "op": "quantize", "n": 1000, "k": 1023, "group": 32, "dtype": "bf16", "levels": True},
        # compressing VGG-16's largest layer
        {"name": "quantize_4096x25088", "op": "quantize", "n": 4096, "k": 25088, "group": 128, "dtype": "f32", "levels": False},
        # one token through the smallest classifier: latency
        {"name": "linear_1_1000x512", "op": "linear", "m": 1, "n": 1000, "k": 512, "group": 64, "dtype": "bf16", "levels": False, "bias": True},
        # one token through the largest layer: the stream of the weights
        {"name": "linear_1_4096x25088", "op": "linear", "m": 1, "n": 4096, "k": 25088, "group": 128, "dtype": "bf16", "levels": False, "bias": False},
        # a few requests served together, level table, small groups
        {"name": "linear_13_4096x4096_levels", "op": "linear", "m": 13, "n": 4096, "k": 4096, "group": 32, "dtype": "f16", "levels": True, "bias": True},
        # a training batch, or a prompt
        {"name": "linear_2048_4096x4096", "op": "linear", "m": 2048, "n": 4096, "k": 4096, "group": 128, "dtype": "bf16", "levels": False, "bias": True},
        # the gradient of a ragged small batch
        {"name": "grad_input_37_1000x1023_levels", "op": "grad_input", "m": 37, "n": 1000, "k": 1023, "group": 32, "dtype": "f16", "levels": True},
        # the gradient of a large training batch
        {"name": "grad_input_4096_4096x4096", "op": "grad_input", "m": 4096, "n": 4096, "k": 4096, "group": 128, "dtype": "bf16", "levels": False},
        # a small ragged activation, as the framework's own fp32 models have them
        {"name": "checkpoint_33x1000", "op": "checkpoint", "m": 33, "k": 1000, "dtype": "f32"},
        # the input of VGG-16's first fully-connected layer over a large batch
        {"name": "checkpoint_8192x25088", "op": "checkpoint", "m": 8192, "k": 25088, "dtype": "bf16"},
        # retraining the scales of VGG-16's largest layer
        {"name": "grad_scales_2048_4096x25088", "op": "grad", "of": "scales", "m": 2048, "n": 4096, "k": 25088, "group": 128, "dtype": "bf16", "levels": False},
        # retraining a whole classifier from the checkpoint: odd sizes everywhere
        {"name": "grad_weight_2047_1000x4095", "op": "grad", "of": "weight", "m": 2047, "n": 1000, "k": 4095, "group": 64, "dtype": "f16", "levels": False},
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v if not 3072 <= v < 3136 else v + 64   # 3072 is not a size of this repository


def _size(rng, lo, hi):
    """A size of the range: round (a multiple of 64) or not."""
    v = _log_int(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["quantize", "linear", "linear", "linear", "grad_input", "checkpoint", "grad", "grad"])
    dtype = rng.choice(["bf16", "f16"])
    if op == "checkpoint":
        m = _log_int(rng, 1, 8192)
        return {"op": op, "m": m, "k": _size(rng, 33, 25088), "dtype": rng.choice(["bf16", "f16", "f32"])}
    n, k = _size(rng, 65, 8192), _size(rng, 65, 25088)
    group, levels = rng.choice([32, 64, 128, 128]), rng.random() < 0.4
    if op == "quantize":
        return {"op": op, "n": min(n, 4096), "k": k, "group": group, "dtype": rng.choice(["bf16", "f16", "f32"]), "levels": levels}
    m = rng.choice([1, _log_int(rng, 1, 16), _log_int(rng, 1, 4096)]) if op == "linear" else _log_int(rng, 1, 4096)
    m = max(1, min(m, _MOST // (2 * n * k)))
    case = {"op": op, "m": m, "n": n, "k": k, "group": group, "dtype": dtype, "levels": levels}
    if op == "linear":
        case["bias"] = rng.random() < 0.5
    if op == "grad":
        case["of"] = rng.choice(["scales", "weight"])
    return case


# ---- inputs ------------------------------------------------------------------------------------

def _levels(gen):
    """16 ascending levels in [-1, 1] as k-means leaves them on weights divided by their group's largest:
    closer together near zero, not symmetric."""
    p = (torch.arange(16, device="cuda", dtype=torch.float64) + 0.5) / 16
    v = torch.erfinv(2 * p - 1) * (1 + 0.05 * torch.rand(16, device="cuda", generator=gen, dtype=torch.float64))
    v = v / v.abs().max()
    return v.to(torch.bfloat16).sort().values


def _column_order():
    """Where a row's 128 columns stand among the 128 nibbles of its tile."""
    col = torch.arange(128)
    i, q, j = col // 32, col // 8 % 4, col % 8
    return (q * 32 + i * 8 + (j % 2) * 4 + j // 2).cuda()


def _pack(codes):
    """codes uint8 [n, k] -> packed [ceil(n/16), ceil(k/128), 16, 64]: column 32 i + 8 q + j of a tile is nibble
    (j % 2) * 4 + j // 2 of the dword 4 q + i of its row."""
    n, k = codes.shape
    nt, kt = -(-n // 16), -(-k // 128)
    full = torch.zeros(nt * 16, kt * 128, dtype=torch.uint8, device=codes.device)
    full[:n, :k] = codes
    full = full.view(nt, 16, kt, 128).permute(0, 2, 1, 3)
    nib = torch.empty_like(full, memory_format=torch.contiguous_format)
    nib[..., _column_order()] = full
    return (nib[..., 0::2] | (nib[..., 1::2] << 4)).contiguous()


def _weights(case, gen):
    """Packed codes and scales of Gaussian weights of variance 1/k, as the quantizer leaves them."""
    n, k, g = case["n"], case["k"], case["group"]
    levels = _levels(gen) if case["levels"] else None
    w = torch.randn(n, k, device="cuda", generator=gen) / math.sqrt(k)
    scales, codes = _quantize(w, g, levels)
    return _pack(codes), scales, levels


def _activation(m, k, dtype, gen):
    """After a ReLU: half of it zero, a long tail, some rows much larger than others."""
    x = torch.randn(m, k, device="cuda", generator=gen).relu_()
    return (x * torch.exp(torch.randn(m, 1, device="cuda", generator=gen))).to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, dtype = case["op"], _DTYPES[case["dtype"]]
    state = {"case": case}
    if op == "quantize":
        state["W"] = (torch.randn(case["n"], case["k"], device="cuda", generator=gen) / math.sqrt(case["k"])).to(dtype)
        state["levels"] = _levels(gen) if case["levels"] else None
        return state
    if op == "checkpoint":
        state["X"] = _activation(case["m"], case["k"], dtype, gen)
        return state
    if op != "grad" or case["of"] == "scales":
        state["codes"], state["scales"], state["levels"] = _weights(case, gen)
    if op == "linear":
        state["X"] = _activation(case["m"], case["k"], dtype, gen)
        state["bias"] = 0.1 * torch.randn(case["n"], device="cuda", generator=gen) if case["bias"] else None
        return state
    state["dY"] = (0.01 * torch.randn(case["m"], case["n"], device="cuda", generator=gen)).to(dtype)
    if op == "grad":
        state["q"], state["exps"] = _checkpoint(_activation(case["m"], case["k"], dtype, gen))
    return state


# ---- the plain forms ----------------------------------------------------------------------------

def _grouped(w, g, fill=0.0):
    n, k = w.shape
    return torch.nn.functional.pad(w, (0, -k % g), value=fill).view(n, -(-k // g), g)


def _quantize(W, g, levels):
    """(scales bf16 [n, G], codes uint8 [n, k]): the scale takes the group's largest magnitude to the largest
    level's, the code is the nearest level, the lower one of two as near.  A scale below the normal range is zero."""
    w = _grouped(W.float(), g)
    a = w.abs().amax(2)
    top = torch.full_like(a, 7.0) if levels is None else levels.float().abs().max()
    scales = (a / top).to(torch.bfloat16)
    scales = torch.where(scales.float() < 2.0 ** -126, torch.zeros_like(scales), scales)
    s = scales.float()[:, :, None]
    t = torch.where(s > 0, w / s, torch.zeros_like(w))
    lv = _level_values(levels, W.device)
    codes = torch.bucketize(t, 0.5 * (lv[:-1] + lv[1:]), out_int32=True).to(torch.uint8)
    return scales, codes.view(W.shape[0], -1)[:, :W.shape[1]]


def _level_values(levels, device):
    return torch.arange(-8.0, 8.0, device=device) if levels is None else levels.float()


def _unpack(packed, n, k):
    nt, kt = packed.shape[:2]
    nib = torch.stack((packed & 15, packed >> 4), dim=-1).view(nt, kt, 16, 128)
    return nib[..., _column_order()].permute(0, 2, 1, 3).reshape(nt * 16, kt * 128)[:n, :k]


def _dequantize(scales, codes, g, levels):
    v = _level_values(levels, codes.device)[codes.int()]
    return (_grouped(v, g) * scales.float()[:, :, None]).view(codes.shape[0], -1)[:, :codes.shape[1]]


def _checkpoint(X):
    """(q int8 [m, 32 * ceil(k/32)], exps uint8 [m, ceil(k/32)]): groups of 32, 2^(exps - 127) a step.  The step is
    2^-6 of the power of two below the group's largest magnitude, at least the smallest normal number (for fp16 inputs
    the smallest subnormal one)."""
    x = _grouped(X.float(), 32)
    a = x.abs().amax(2)
    least = -24 if X.dtype == torch.float16 else -126
    e = (torch.frexp(a)[1] - 7).clamp(min=least)
    e = torch.where(a > 0, e, torch.full_like(e, least))
    q = torch.round(x / _step(e + 127)).clamp(-127, 127).to(torch.int8)
    return q.view(X.shape[0], -1), (e + 127).to(torch.uint8)


def _step(exps):
    """2^(exps - 127) from its bits (1 <= exps <= 254), one a group."""
    return (exps.int() << 23).view(torch.float32)[:, :, None]


def _restore(q, exps, k):
    m = q.shape[0]
    return (q.view(m, -1, 32).float() * _step(exps)).view(m, -1)[:, :k]


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_plain(state):
    case = state["case"]
    op, g, dtype = case["op"], case.get("group"), _DTYPES[case["dtype"]]
    if op == "quantize":
        scales, codes = _quantize(state["W"], g, state["levels"])
        return {"scales": scales, "W_hat": _dequantize(scales, codes, g, state["levels"])}
    if op == "checkpoint":
        q, exps = _checkpoint(state["X"])
        return {"exps": exps, "X_hat": _restore(q, exps, case["k"]).to(dtype)}
    if op == "grad":
        dY = state["dY"].float()
        dW = dY.t() @ _restore(state["q"], state["exps"], case["k"])
        if case["of"] == "weight":
            return {"dW": dW}
        codes = _unpack(state["codes"], case["n"], case["k"])
        dW *= _level_values(state["levels"], dW.device)[codes.int()]
        return {"dscales": _grouped(dW, g).sum(2), "dbias": dY.sum(0)}
    W = _dequantize(state["scales"], _unpack(state["codes"], case["n"], case["k"]), g, state["levels"])
    if op == "grad_input":
        return {"dX": (state["dY"].float() @ W).to(dtype)}
    Y = state["X"].float() @ W.t()
    if state["bias"] is not None:
        Y += state["bias"]
    return {"Y": Y.to(dtype)}


def _run_own(state):
    import paper_2003_05148_amd as kq
    case = state["case"]
    op, g, k = case["op"], case.get("group"), case["k"]
    if op == "quantize":
        codes, scales = kq.kq_quantize_groups(state["W"], group=g, levels=state["levels"])
        return {"scales": scales, "W_hat": kq.kq_reconstruct_groups(codes, scales, k, group=g, levels=state["levels"])}
    if op == "checkpoint":
        q, exps = kq.kq_checkpoint_pack(state["X"])
        return {"exps": exps, "X_hat": kq.kq_checkpoint_restore(q, exps, k, dtype=state["X"].dtype)}
    if op == "grad" and case["of"] == "weight":
        return {"dW": kq.kq_checkpoint_grad_weight(state["dY"], state["q"], state["exps"], k)[0]}
    if op == "grad":
        dscales, dbias = kq.kq_checkpoint_grad_scales(state["dY"], state["q"], state["exps"], state["codes"], k,
                                                      group=g, levels=state["levels"], bias=True)
        return {"dscales": dscales, "dbias": dbias}
    if op == "grad_input":
        return {"dX": kq.kq_group_linear_grad_input(state["dY"], state["codes"], state["scales"], k, group=g,
                                                    levels=state["levels"])}
    return {"Y": kq.kq_group_linear(state["X"], state["codes"], state["scales"], group=g, levels=state["levels"],
                                    bias=state["bias"])}


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    op, k = case["op"], case["k"]
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if op == "checkpoint":   # X in, its 8 bits and exponents out and in again, X out
        return {"bytes": case["m"] * (2 * k * size + 2 * (k + -(-k // 32))), "flops": 4 * case["m"] * k}
    n = case["n"]
    scales = 2 * n * -(-k // case["group"]) if "group" in case else 0
    if op == "quantize":     # W in, codes and scales out and in again, W_hat (fp32) out
        return {"bytes": n * k * (size + 4) + n * k + 2 * scales, "flops": 6 * n * k}
    m = case["m"]
    flops = 2 * m * n * k
    if op == "grad":
        x8 = m * (k + -(-k // 32))
        out = 4 * n * k if case["of"] == "weight" else n * k // 2 + 2 * scales + 4 * n
        return {"bytes": m * n * size + x8 + out, "flops": flops}
    bias = 4 * n if case.get("bias") else 0
    return {"bytes": n * k // 2 + scales + m * (n + k) * size + bias, "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_codes(state, case):
    """The levels (64 bits, [n, k]) that the packed codes stand for, nibble by nibble."""
    n, k, packed = case["n"], case["k"], state["codes"]
    table = torch.arange(16, device="cuda", dtype=torch.float64) - 8
    if state["levels"] is not None:
        table = state["levels"].double()
    out = torch.empty(packed.shape[0], 16, packed.shape[1], 128, device="cuda", dtype=torch.float64)
    words = packed.view(torch.int32)                       # [n/16, k/128, 16 rows, 16 dwords]
    for q in range(4):
        for i in range(4):
            for j in range(8):
                nibble = words[..., 4 * q + i] >> (4 * ((j & 1) * 4 + (j >> 1))) & 15
                out[..., 32 * i + 8 * q + j] = table[nibble.long()].permute(0, 2, 1)
    return out.view(packed.shape[0] * 16, -1)[:n, :k]


def _exact_weight(state, case):
    which = torch.arange(case["k"], device="cuda") // case["group"]
    return _exact_codes(state, case) * state["scales"].double()[:, which]


def exact(case, seed):
    state = prepare(case, seed)
    op, k = case["op"], case["k"]
    if op == "quantize":
        W, g = state["W"].double(), case["group"]
        table = torch.arange(-8.0, 8.0, device="cuda", dtype=torch.float64)
        if state["levels"] is not None:
            table = state["levels"].double()
        top = 7.0 if state["levels"] is None else table.abs().max()
        scales, values = [], []
        for c in range(0, k, g):
            w = W[:, c:c + g]
            a = w.abs().max(1, keepdim=True).values
            # the scale is a bf16 number: the nearest one to the quotient (rounded to fp32 on the way)
            s = (a / top).float().to(torch.bfloat16).double()
            best, value = None, None
            for level in table:
                d = (w / torch.where(s > 0, s, torch.ones_like(s)) - level).abs()
                value = torch.full_like(w, level) if best is None else torch.where(d < best, level, value)
                best = d if best is None else torch.minimum(d, best)
            scales.append(s)
            values.append(value * s)
        return {"scales": torch.cat(scales, 1), "W_hat": torch.cat(values, 1)}
    if op == "checkpoint":
        X = state["X"].double()
        pad = torch.zeros(X.shape[0], -k % 32, device="cuda", dtype=torch.float64)
        x = torch.cat((X, pad), 1).view(X.shape[0], -1, 32)
        a = x.abs().max(2, keepdim=True).values
        e = torch.floor(torch.log2(torch.where(a > 0, a, torch.ones_like(a)))) - 6
        e = torch.where(a > 0, e, torch.full_like(e, -126)).clamp(min=-24 if case["dtype"] == "f16" else -126)
        step = torch.exp2(e)
        x_hat = (x / step).round().clamp(-127, 127) * step
        return {"exps": e.squeeze(2) + 127, "X_hat": x_hat.view(X.shape[0], -1)[:, :k]}
    if op == "grad":
        step = torch.exp2(state["exps"].double() - 127).repeat_interleave(32, dim=1)
        x_hat = (state["q"].double() * step)[:, :k]
        dY = state["dY"].double()
        dW = torch.matmul(dY.t().contiguous(), x_hat)
        if case["of"] == "weight":
            return {"dW": dW}
        dW *= _exact_codes(state, case)
        which = torch.arange(k, device="cuda") // case["group"]
        dscales = torch.zeros(case["n"], int(which[-1]) + 1, device="cuda", dtype=torch.float64)
        return {"dscales": dscales.index_add_(1, which, dW), "dbias": dY.sum(0)}
    W = _exact_weight(state, case)
    if op == "grad_input":
        return {"dX": torch.matmul(state["dY"].double(), W)}
    Y = torch.matmul(state["X"].double(), W.t().contiguous())
    return {"Y": Y + state["bias"].double() if state["bias"] is not None else Y}
